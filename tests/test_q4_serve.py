"""Serving from the 4-bit cache: attention over a window with sinks and of drafted trees, kept rows, planned steps.  Refusals on the CPU;
everything else against definitions in 64 bits on the GPU."""
import math
import random

import pytest
import torch

from paper_2608_23843_b200 import pkv
from q4_reference import attention, offsets_of, quantised
from q4_select_reference import Plan, attention_seen, pack, tree_bits, tree_seen, window_seen
from test_q4_cache import BF16, FP16, INTS, SHAPES, Filled, check, config, room, rows_of  # noqa: F401

LONGS = dict(dtype=torch.int64)


# ---- CPU: refusals -----------------------------------------------------------------------------------------------------
def _dry():
    cache = pkv.Q4Cache(config(), dry_run=True)
    return cache, torch.zeros(3, 4, **INTS), torch.zeros(3, **INTS), torch.zeros(3, 2, 8, 128, dtype=BF16)


def test_calls_that_are_accepted_in_a_dry_run():
    c, t, n, q = _dry()
    off = offsets_of([0, 5, 1])
    assert c.attention(t, n, q, window=5).shape == q.shape
    assert c.attention(t, n, q, window=2 ** 31 - 1, sinks=2 ** 31 - 1).shape == q.shape
    assert c.attention(t, n, q, tree=torch.zeros(3, 2, 1, **LONGS)).shape == q.shape
    assert c.attention(t, n, q, tree=torch.zeros(3, 2, 7, **LONGS), window=9, sinks=4).shape == q.shape
    assert c.attention(t, n, q.flatten(0, 1), offsets=off, max_q_len=5, tree=torch.zeros(6, 1, **LONGS)).shape == (6, 8, 128)
    assert c.attention_partial(t, n, q, window=3).shape == (3, 2, 8, 130)
    assert c.attention(t, n, q[:, :0], tree=torch.zeros(3, 0, 1, **LONGS)).shape == (3, 0, 8, 128)
    masks, depths = c.tree_masks(torch.zeros(3, 65, **INTS))
    assert masks.shape == (3, 65, 2) and depths.shape == (3, 65)
    masks, depths = c.tree_masks(torch.zeros(6, **INTS), n, off, max_q_len=5, window=3, sinks=2)
    assert masks.shape == (6, 1) and depths.shape == (6,)
    assert c.keep_rows(t, n, torch.zeros(3, 2, **INTS), n, 2).shape == (3,)
    assert c.keep_rows(t, n, torch.zeros(3, 0, **INTS), n, 6, offsets=off).shape == (3,)
    ring, counters = c.new_ring()
    assert ring.tolist() == list(range(16)) and counters.tolist() == [0, 16, 0, 0]
    p = c.plan(t, n, n, torch.zeros(3, 2, **INTS), ring, counters, 7, window=5, sinks=1)
    assert p.slots.shape == p.positions.shape == (7,) and p.offsets.shape == (4,) and p.spans.shape == (3, 2)
    assert [x.data_ptr() % x.element_size() for x in p] == [0] * 6
    c.plan(t, n, n, torch.zeros(3, 2, **INTS), ring, counters, 0, out=p._replace(positions=None, slots=None))


def _spans():
    return torch.zeros(3, 2, **INTS)


def _ring():
    return torch.zeros(16, **INTS), torch.zeros(4, **LONGS)


@pytest.mark.parametrize("call", [
    lambda c, t, n, q: c.attention(t, n, q, window=-1),
    lambda c, t, n, q: c.attention(t, n, q, sinks=4),                          # sinks without a window
    lambda c, t, n, q: c.attention(t, n, q, window=4, sinks=-1),
    lambda c, t, n, q: c.attention(t, n, q, window=2 ** 31),
    lambda c, t, n, q: c.attention(t, n, q, window=2 ** 32 + 4),                # would arrive as 4
    lambda c, t, n, q: c.tree_masks(torch.zeros(3, 2, **INTS), n, window=2 ** 32 + 4),
    lambda c, t, n, q: c.plan(t, n, n, _spans(), *_ring(), 4, window=4, sinks=2 ** 32),
    lambda c, t, n, q: c.attention(t, n, q, tree=torch.zeros(3, 2, 1, **INTS)),
    lambda c, t, n, q: c.attention(t, n, q, tree=torch.zeros(3, 2, **LONGS)),
    lambda c, t, n, q: c.attention(t, n, q, tree=torch.zeros(3, 3, 1, **LONGS)),
    lambda c, t, n, q: c.attention(t, n, q, tree=torch.zeros(3, 2, 0, **LONGS)),
    lambda c, t, n, q: c.attention(t, n, q, tree=torch.zeros(3, 2, 2, **LONGS)[..., ::2]),
    lambda c, t, n, q: c.attention(t, n, q.flatten(0, 1), offsets=offsets_of([2, 2, 2]), tree=torch.zeros(3, 2, 1, **LONGS)),
    lambda c, t, n, q: c.attention(t, n, torch.zeros(3, 65, 8, 128, dtype=BF16), tree=torch.zeros(3, 65, 1, **LONGS)),
    lambda c, t, n, q: c.attention_partial(t, n, q, sinks=4),
    lambda c, t, n, q: c.tree_masks(torch.zeros(3, 2, **LONGS)),
    lambda c, t, n, q: c.tree_masks(torch.zeros(6, **INTS)),
    lambda c, t, n, q: c.tree_masks(torch.zeros(3, 2, **INTS), offsets=offsets_of([2, 2, 2])),
    lambda c, t, n, q: c.tree_masks(torch.zeros(3, 2, **INTS), window=4, sinks=2),             # lengths are needed
    lambda c, t, n, q: c.tree_masks(torch.zeros(3, 2, **INTS), n[:2], window=4),
    lambda c, t, n, q: c.tree_masks(torch.zeros(3, 2, **INTS), n, sinks=2),
    lambda c, t, n, q: c.tree_masks(torch.zeros(6, **INTS), n, offsets_of([2, 2, 2]), max_q_len=7),
    lambda c, t, n, q: c.keep_rows(t, n, torch.zeros(3, 2, **LONGS), n, 2),
    lambda c, t, n, q: c.keep_rows(t, n, torch.zeros(2, 2, **INTS), n, 2),
    lambda c, t, n, q: c.keep_rows(t, n, torch.zeros(3, 2, **INTS), n[:2], 2),
    lambda c, t, n, q: c.keep_rows(t, n, torch.zeros(3, 2, **INTS), n, -1),
    lambda c, t, n, q: c.keep_rows(t, n, torch.zeros(3, 2, **INTS), n, 2, out=n),              # in place
    lambda c, t, n, q: c.keep_rows(t, n, torch.zeros(3, 2, **INTS), n, 2, out=n.long()),
    lambda c, t, n, q: c.plan(t, n, n.long(), _spans(), *_ring(), 4),
    lambda c, t, n, q: c.plan(t, n, n, _spans()[:2], *_ring(), 4),
    lambda c, t, n, q: c.plan(t, n, n, _spans(), _ring()[0][:15], _ring()[1], 4),
    lambda c, t, n, q: c.plan(t, n, n, _spans(), _ring()[0], _ring()[1].int(), 4),
    lambda c, t, n, q: c.plan(t, n, n, _spans(), *_ring(), 4, window=-1),
    lambda c, t, n, q: c.plan(t, n, n, _spans(), *_ring(), 4, sinks=1),
    lambda c, t, n, q: c.plan(t, n, n, _spans(), *_ring(), 4, out=c.plan(t, n, n, _spans(), *_ring(), 5)),
    lambda c, t, n, q: c.plan(t.long(), n, n, _spans(), *_ring(), 4),
    lambda c, t, n, q: c.keep_rows(t, n, torch.zeros(3, 2, **INTS), n, 2 ** 62),               # more than 64 bits in all
    lambda c, t, n, q: c.keep_rows(t, n, torch.zeros(3, 2, **INTS), n, 2.0),
    lambda c, t, n, q: c.new_ring([0, 1, 1]),
    lambda c, t, n, q: c.new_ring([16]),
    lambda c, t, n, q: c.new_ring(torch.arange(17)),
])
def test_calls_that_are_refused(call):
    with pytest.raises(pkv.PkvError) as e:
        call(*_dry())
    assert e.value.status == pkv.PKV_ERR_INVALID_ARG and str(e.value)


def test_refusals_of_the_c_entry_points():
    import ctypes
    c, t, n, q = _dry()
    h, L, bad = c.handle, pkv.lib(), pkv.PKV_ERR_INVALID_ARG
    size = ctypes.c_int64()
    for sel, words in [(pkv.PkvQ4Select(-1, 0, None, 0), 0), (pkv.PkvQ4Select(0, 1, None, 0), 0), (pkv.PkvQ4Select(4, -2, None, 0), 0),
                       (pkv.PkvQ4Select(0, 0, 12, 1), 1), (pkv.PkvQ4Select(0, 0, 16, 0), 0), (pkv.PkvQ4Select(0, 0, 16, -1), 0)]:
        assert L.pkv_q4_attention_select_workspace(h, 3, 2, 64, ctypes.byref(sel), ctypes.byref(size)) == bad
        assert L.pkv_q4_attention_select(h, 3, 0, 4, 0, 6, 0, 2, 0, ctypes.byref(sel), 0, 1024, 128, 0, 1024, 128, 0, 0, 0, 0) == bad
    sel = pkv.PkvQ4Select(0, 0, 16, 1)
    assert L.pkv_q4_attention_select_workspace(h, 3, 65, 64, ctypes.byref(sel), ctypes.byref(size)) == bad
    assert L.pkv_q4_attention_select_workspace(h, 3, 64, 64, ctypes.byref(sel), None) == bad
    assert L.pkv_q4_attention_select_workspace(h, 3, 64, 64, None, ctypes.byref(size)) == bad
    assert L.pkv_q4_attention_select(h, 3, 0, 4, 0, 6, 0, 2, 0, None, 0, 1024, 128, 0, 1024, 128, 0, 0, 0, 0) == bad
    assert L.pkv_q4_attention_select(None, 3, 0, 4, 0, 6, 0, 2, 0, ctypes.byref(sel), 0, 1024, 128, 0, 1024, 128, 0, 0, 0, 0) == bad
    masks = lambda **k: L.pkv_q4_tree_masks(*{**dict(h=h, S=3, n=0, rows=6, off=0, most=2, par=0, W=0, sinks=0, tree=0, words=1, dep=0, st=0), **k}.values())  # noqa: E731
    assert masks() == pkv.PKV_OK
    for k in [dict(h=None), dict(S=0), dict(rows=7), dict(off=4, most=7), dict(par=2), dict(dep=1), dict(tree=4), dict(words=0), dict(rows=195), dict(W=-1), dict(sinks=3)]:
        assert masks(**k) == bad, k
    keep = lambda **k: L.pkv_q4_keep_rows(*{**dict(h=h, S=3, t=0, mp=4, n=0, rows=6, off=0, path=0, m=2, cnt=0, out=0, st=0), **k}.values())  # noqa: E731
    assert keep() == pkv.PKV_OK
    for k in [dict(h=None), dict(S=0), dict(mp=0), dict(rows=-1), dict(m=-1), dict(path=2), dict(cnt=1), dict(out=2), dict(n=64, out=64), dict(n=64, out=72), dict(n=64, out=56)]:
        assert keep(**k) == bad, k
    plan = lambda **k: L.pkv_q4_plan(*{**dict(h=h, S=3, t=0, mp=4, n=0, r=0, sp=0, ring=0, cnt=0, W=0, sinks=0, no=0, so=0, co=0, off=0, rows=6, pos=0, slot=0, work=0, wb=0, st=0), **k}.values())  # noqa: E731
    assert plan() == pkv.PKV_OK
    for k in [dict(h=None), dict(S=0), dict(S=65536), dict(mp=0), dict(mp=1 << 28), dict(rows=-1), dict(rows=1 << 31), dict(W=-1), dict(sinks=1),
              dict(t=2), dict(n=1), dict(ring=2), dict(cnt=4), dict(co=4), dict(slot=4), dict(pos=2), dict(off=1)]:
        assert plan(**k) == bad, k
    assert L.pkv_q4_plan_workspace(h, 3, 6, None) == bad and L.pkv_q4_plan_workspace(h, 0, 6, ctypes.byref(size)) == bad
    assert pkv.pkv_q4_plan_workspace(h, 3, 6) == 0 and pkv.pkv_q4_plan_workspace(h, 3, 1 << 20) > 0 and pkv.pkv_q4_plan_workspace(h, 5000, 6) > 0


# What serves which call: kernel (0: even shares, 1: row blocks, 2: small CTAs), CTAs of a cluster.  (n_ctas leaves the row blocks alone: few of the
# others make them the choice for short sequences too.)
ROUTES = [
    ("small, one CTA to a segment", dict(H=2, G=4, n_ctas=20), 20, 1, 300, dict(window=200, sinks=5), 2, 1),
    ("small, segments in turn", dict(H=2, G=4), 320, 1, 300, dict(window=200, sinks=5), 2, 1),
    ("small, clusters of 2", dict(H=2, G=4, n_ctas=20), 8, 1, 700, dict(window=300, sinks=5), 2, 2),
    ("small, clusters of 4", dict(H=2, G=4, n_ctas=50), 8, 2, 1000, dict(window=700, sinks=5), 2, 4),
    ("small, clusters of 8", dict(H=2, G=4), 3, 5, 1500, dict(window=1400), 2, 8),
    ("small, a tree", dict(H=1, G=7), 2, 7, 1500, dict(tree=True), 2, 8),
    ("small, a tree and a window", dict(H=2, G=3), 2, 12, 2000, dict(tree=True, window=900, sinks=70), 2, 8),
    ("even shares, 8 rows", dict(H=1, G=4), 1, 1, 20000, dict(window=18000, sinks=100), 0, 1),
    ("even shares, 8 rows, a tree", dict(H=2, G=2), 1, 4, 30000, dict(tree=True), 0, 1),
    ("even shares, 16 rows", dict(H=2, G=4), 4, 4, 20000, dict(tree=True, window=19000, sinks=3), 0, 1),
    ("even shares, two tiles", dict(H=2, G=4), 4, 6, 20000, dict(window=19500), 0, 1),
    ("row blocks, halves in turn", dict(H=2, G=4, n_ctas=10), 4, 30, 2000, dict(tree=True), 1, 1),
    ("row blocks, halves in turn, a window", dict(H=3, G=3, n_ctas=10), 5, 40, 2500, dict(window=1100, sinks=20), 1, 1),
    ("row blocks, both halves", dict(H=2, G=4, n_ctas=10), 5, 50, 1500, dict(tree=True, window=700, sinks=9), 1, 1),
    ("row blocks, several", dict(H=2, G=8, n_ctas=10), 5, 100, 1200, dict(window=333, sinks=65), 1, 1),
    ("row blocks, more than eight", dict(H=1, G=16, n_ctas=10), 2, 150, 700, dict(window=64, sinks=1), 1, 1),
    ("row blocks, a tree over several", dict(H=1, G=8, n_ctas=10), 6, 90, 900, dict(tree=True), 1, 1),
]


def _route(cache, S, n, most, kw):
    return pkv.pkv_q4_attention_route(cache.handle, S, n, most, kw.get("window", 0), kw.get("sinks", 0), kw.get("tree"), -(-n // 64))


@pytest.mark.parametrize("name, shape, S, n, T, kw, kernel, cluster", ROUTES, ids=[r[0] for r in ROUTES])
def test_which_kernel_serves_a_call(name, shape, S, n, T, kw, kernel, cluster):
    H, G = shape["H"], shape["G"]
    cache = pkv.Q4Cache(config(n_kv_heads=H, n_q_heads=H * G, n_ctas=shape.get("n_ctas", 0)), dry_run=True)
    got = _route(cache, S, n, -(-T // 64) * 64, kw)
    assert (got[0], got[2]) == (kernel, cluster), got
    if name == "small, segments in turn":
        assert got[1] < S * H
    assert pkv.pkv_q4_attention_route(cache.handle, 1, 1, 64)[0] == 0
    for bad in ((0, 1, 64), (1, 0, 64), (1, 1, 0)):
        with pytest.raises(pkv.PkvError):
            pkv.pkv_q4_attention_route(cache.handle, *bad)


def test_calls_without_ctypes_check_their_numbers():
    from paper_2608_23843_b200 import _pkvcall
    c, t, n, q = _dry()
    h = c.handle.value
    good = dict(append_kv=(h, 3, 0, 4, 0, 6, 0, 0, 256, 128, 0, 256, 128, 0), attention=(h, 3, 0, 4, 0, 6, 0, 2, 0, 0, 1024, 128, 0, 1024, 128, 0, 0, 0, 0),
                attention_select=(h, 3, 0, 4, 0, 6, 0, 2, 0, 0, 1024, 128, 0, 1024, 128, 0, 0, 0, 0, 9, 4, None, 0),
                tree_masks=(h, 3, None, 6, None, 2, 0, 0, 0, 0, 1, 0, 0), keep_rows=(h, 3, 0, 4, 0, 6, 0, 0, 2, 0, 0, 0),
                plan=(h, 3, 0, 4, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 6, 0, 0, 0, 0, 0))
    good["read_kv"] = good["append_kv"]
    for name, args in good.items():
        fn = getattr(_pkvcall, name)
        assert fn(*args) == pkv.PKV_OK, name
        assert fn(None, *args[1:]) == pkv.PKV_ERR_INVALID_ARG
        with pytest.raises(TypeError):
            fn(*args[:-1])
        with pytest.raises(TypeError):
            fn(h, 3.0, *args[2:])
        for wrong in (1 << 31, -(1 << 31) - 1, 1 << 64):                             # n_seqs
            with pytest.raises(OverflowError):
                fn(h, wrong, *args[2:])


def test_the_references_agree_with_one_another():
    """A tree without branches is causal; a window wider than everything is none; packed masks hold the bits."""
    T, n = 40, 9
    line, depths = tree_bits([j - 1 for j in range(n)])
    assert depths == list(range(n))
    for W, S in ((0, 0), (5, 0), (5, 3), (100, 7), (1, 0)):
        bits, _ = tree_bits([j - 1 for j in range(n)], T - n, W, S)
        assert torch.equal(tree_seen(T, bits, W, S), window_seen(T, n, W, S)), (W, S)
    q, K, V = torch.randn(n, 2, 64).to(BF16), torch.randn(T, 1, 64, **dict(dtype=torch.float64)), torch.randn(T, 1, 64, dtype=torch.float64)
    for a, b in zip(attention_seen(q, K, V, window_seen(T, n, 0, 0), 0.1, BF16), attention(q, K, V, T - n, 0.1, BF16)):
        assert torch.allclose(a, b, rtol=1e-12, atol=0)
    wide = torch.rand(70, 70) < 0.5
    words = pack(wide)
    assert all(bool(wide[j, i]) == bool(int(words[j, i // 64]) >> (i % 64) & 1) for j in range(70) for i in range(70))


# ---- GPU helpers ------------------------------------------------------------------------------------------------------
def seen_by(f, q, s, see, scale=None):
    return attention_seen(q, f.K[s], f.V[s], see, scale or 1 / math.sqrt(f.d), f.dtype)


def random_parents(rng, n, reach=9):
    return [rng.randint(max(-1, j - reach), j - 1) for j in range(n)]


def without_hidden_pages(f, P, ns, window, sinks):
    """The table as it is when pages that no query sees have gone back."""
    table = f.rows.table.clone()
    for s, (T, n) in enumerate(zip(f.lens, ns)):
        low = max(0, T - n + 1 - window)
        for e in range(table.shape[1]):
            if e * P >= sinks and (e + 1) * P <= low:
                table[s, e] = -1
    return table.cuda()


# ---- GPU: windows ------------------------------------------------------------------------------------------------------
WINDOWS = [(1, 0), (16, 0), (17, 1), (64, 4), (100, 70), (256, 16), (5000, 3)]


@pytest.mark.usefixtures("room")
@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("G", [1, 4, 12])
def test_window_decode(shape, G):
    f = Filled([1, 16, 17, 64, 65, 129, 300, 1000], G=G, **shape)
    q = torch.stack(f.queries([1] * 8))
    for W, S in WINDOWS:
        table = without_hidden_pages(f, shape["P"], [1] * 8, W, S)
        out = f.cache.attention(table, f.lengths, q.cuda(), window=W, sinks=S)
        for s in range(8):
            check(out[s], *seen_by(f, q[s], s, window_seen(f.lens[s], 1, W, S))[::2])
    f.clean()


@pytest.mark.usefixtures("room")
@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("n, G", [(2, 4), (5, 7), (17, 8), (40, 4), (130, 3)])
def test_window_of_several_positions(shape, n, G):
    f = Filled([n, n + 1, 64 + n, 701], G=G, seed=n, **shape)
    q = torch.stack(f.queries([n] * 4))
    for W, S in WINDOWS:
        table = without_hidden_pages(f, shape["P"], [n] * 4, W, S)
        out = f.cache.attention(table, f.lengths, q.cuda(), window=W, sinks=S)
        for s in range(4):
            check(out[s], *seen_by(f, q[s], s, window_seen(f.lens[s], n, W, S))[::2])
    f.clean()


@pytest.mark.usefixtures("room")
@pytest.mark.gpu
@pytest.mark.parametrize("dtype, d, g, G, lens", [(BF16, 128, 32, 4, [1200]), (FP16, 64, 64, 7, [700, 10, 390]), (BF16, 128, 128, 1, [2600, 300])])
@pytest.mark.parametrize("W, S", [(1, 0), (100, 5), (256, 64), (513, 130)])
def test_window_of_whole_prompts(dtype, d, g, G, lens, W, S):
    """Blocks of query rows whose windows begin in very different places."""
    f = Filled(lens, dtype=dtype, d=d, g=g, G=G, H=1, P=32, seed=27)
    qs = f.queries(lens)
    out = f.cache.attention(f.table, f.lengths, torch.cat(qs).cuda(), offsets=f.off, max_q_len=max(lens), window=W, sinks=S).cpu()
    at = 0
    for s, q in enumerate(qs):
        check(out[at:at + lens[s]], *seen_by(f, q, s, window_seen(lens[s], lens[s], W, S))[::2])
        at += lens[s]
    f.clean()


@pytest.mark.gpu
@pytest.mark.parametrize("W, S", [(1000, 4), (70000, 300)])
def test_window_in_a_very_long_sequence(W, S):
    f = Filled([300_003], G=2, H=1, P=256, d=64, seed=33)
    for n in (1, 7, 40):
        q = f.queries([n])[0]
        see = window_seen(f.lens[0], n, W, S)
        out = f.cache.attention(without_hidden_pages(f, 256, [n], W, S), f.lengths, q[None].cuda(), window=W, sinks=S)
        check(out[0], *seen_by(f, q, 0, see)[::2])
    f.clean()


@pytest.mark.gpu
def test_window_of_a_long_prompt_in_more_blocks_than_a_warp_looks_up_at_once():
    n, G, W, S = 2200, 8, 300, 20
    f = Filled([n], G=G, H=1, P=64, seed=28)
    q = f.queries([n])[0]
    out = f.cache.attention(f.table, f.lengths, q[None].cuda(), window=W, sinks=S)[0].cpu()
    see = window_seen(n, n, W, S)
    for j in [0, 1, 31, 32, 33, 63, 64, 299, 300, 301, 320, 1000, 1023, 1024, 1025, 2111, 2112, 2198, 2199]:
        ref, _, tol = seen_by(f, q[j:j + 1], 0, see[j:j + 1])
        check(out[j:j + 1], ref, tol)
    f.clean()


@pytest.mark.gpu
@pytest.mark.parametrize("n_ctas", [1, 3, 40])
@pytest.mark.parametrize("n, G", [(1, 4), (3, 8), (64, 4)])
def test_windows_spread_over_few_and_many_ctas(n_ctas, n, G):
    f = Filled([64, 2500, 65, 1700, 129], H=2, G=G, P=32, seed=5, n_ctas=n_ctas, room=3000)
    q = torch.stack(f.queries([n] * 5))
    for W, S in ((70, 5), (1500, 100), (2000, 0)):
        for hint in (0, 64):
            out = f.cache.attention(f.table, f.lengths, q.cuda(), window=W, sinks=S, max_len=hint)
            for s in range(5):
                check(out[s], *seen_by(f, q[s], s, window_seen(f.lens[s], n, W, S))[::2])
    f.clean()


@pytest.mark.usefixtures("room")
@pytest.mark.gpu
@pytest.mark.parametrize("n, G", [(1, 4), (4, 8), (70, 4)])
@pytest.mark.parametrize("what", ["k", "v"])
def test_what_lies_outside_the_window_does_not_matter(n, G, what):
    """Infinite and NaN rows, and rows 2^40 times larger, before the window and behind the sinks."""
    W, S = 100, 20
    f = Filled([400 + n, 700], G=G, H=1, P=16, seed=6)
    q = torch.stack(f.queries([n] * 2))
    want = f.cache.attention(f.table, f.lengths, q.cuda(), window=W, sinks=S)
    bad = [x.clone() for x in getattr(f, what)]
    for s, T in enumerate(f.lens):
        low = T - n + 1 - W
        bad[s][S:low] *= 2.0 ** 40
        bad[s][S:low:3] = math.nan
        bad[s][S + 1:low:3, 0, 5] = math.inf
    k, v = (torch.cat(bad if what == x else getattr(f, x)).cuda() for x in "kv")
    f.cache.append_kv(f.table, f.lengths, k, v, f.off)
    out = f.cache.attention(f.table, f.lengths, q.cuda(), window=W, sinks=S)
    for s in range(2):
        ref, _, tol = seen_by(f, q[s], s, window_seen(f.lens[s], n, W, S))
        check(want[s], ref, tol)
        check(out[s], ref, tol)


@pytest.mark.usefixtures("room")
@pytest.mark.gpu
@pytest.mark.parametrize("n, G", [(1, 4), (4, 4), (70, 4)])
@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_windows_over_values_of_very_different_sizes(n, G, dtype):
    W, S = 60, 10
    f = Filled([200, 90], G=G, H=1, seed=4, dtype=dtype)
    for s in range(2):
        f.v[s][:, :, :64] *= 2.0 ** -12
        f.v[s][::3] *= 2.0 ** 9
        f.k[s] *= 2.0 ** 8
    f.cache.append_kv(f.table, f.lengths, torch.cat(f.k).cuda(), torch.cat(f.v).cuda(), f.off)
    f.K, f.V = [quantised(x, 32) for x in f.k], [quantised(x, 32) for x in f.v]
    qs = [q * 2.0 ** -9 for q in f.queries([n, n])]
    out = f.cache.attention(f.table, f.lengths, torch.stack(qs).cuda(), window=W, sinks=S)
    for s, q in enumerate(qs):
        check(out[s], *seen_by(f, q, s, window_seen(f.lens[s], n, W, S))[::2])


FORMATS = [dict(dtype=BF16, d=128, g=32, P=64), dict(dtype=FP16, d=64, g=64, P=16), dict(dtype=FP16, d=128, g=128, P=32), dict(dtype=BF16, d=64, g=32, P=64),
           dict(dtype=BF16, d=128, g=64, P=128)]


@pytest.mark.gpu
@pytest.mark.parametrize("form", range(len(FORMATS)))
@pytest.mark.parametrize("name, shape, S, n, T, kw, kernel, cluster", ROUTES, ids=[r[0] for r in ROUTES])
def test_every_kernel(name, shape, S, n, T, kw, kernel, cluster, form):
    """Ragged lengths and rows on each kernel, what is not seen being anything: pages gone back, keys and values infinite and NaN.
    (d = 64 and other formats may be served by another kernel than the one named, as the rule sees fit.)"""
    rng = random.Random(S * n + form)
    lens = [T] + [rng.choice([n, n + 1, rng.randint(n, T), rng.randint(n, T)]) for _ in range(S - 1)]
    ns = [n] + [rng.choice([0, 1, n, rng.randint(0, n)]) for _ in range(S - 1)]
    f = Filled(lens, seed=form, room=T, **shape, **FORMATS[form])
    W, sinks, tree = kw.get("window", 0), kw.get("sinks", 0), kw.get("tree", False)
    if form == 0:
        assert _route(f.cache, S, n, f.table.shape[1] * FORMATS[form]["P"], kw)[::2] == (kernel, cluster)
    table = without_hidden_pages(f, FORMATS[form]["P"], ns, W, sinks) if W else f.table
    if W:
        k, v = [x.clone() for x in f.k], [x.clone() for x in f.v]
        for s, (T_s, n_s) in enumerate(zip(lens, ns)):
            low = max(0, T_s - n_s + 1 - W)
            k[s][sinks:low:3] *= 2.0 ** 5
            k[s][sinks + 1:low:7] = math.nan
            v[s][sinks:low:5] = math.inf
        f.cache.append_kv(f.table, f.lengths, torch.cat(k).cuda(), torch.cat(v).cuda(), f.off)
    qs = f.queries(ns)
    off = offsets_of(ns, start=1).cuda()
    pad = torch.zeros(1, f.H * f.G, f.d, dtype=f.dtype)
    q = torch.cat([pad, *qs, pad]).cuda()
    parents = [random_parents(rng, x, 6) for x in ns]
    masks = f.cache.tree_masks(torch.tensor([0] + sum(parents, []) + [0], **INTS).cuda(), f.lengths, off, n, W, sinks)[0] if tree else None
    out = torch.full_like(q, 5.0)
    f.cache.attention(table, f.lengths, q, out=out, offsets=off, max_q_len=n, window=W, sinks=sinks, tree=masks)
    state = f.cache.attention_partial(table, f.lengths, q, offsets=off, max_q_len=n, window=W, sinks=sinks, tree=masks)
    assert (out[0] == 5).all() and (out[-1] == 5).all()
    out, state, at = out.cpu(), state.to("cpu", torch.float64), 1
    for s, (n_s, T_s) in enumerate(zip(ns, lens)):
        if n_s:
            see = tree_seen(T_s, tree_bits(parents[s], T_s - n_s, W, sinks)[0], W, sinks) if tree else window_seen(T_s, n_s, W, sinks)
            ref, lse, tol = seen_by(f, qs[s], s, see)
            check(out[at:at + n_s], ref, tol)
            st = state[at:at + n_s]
            check(st[..., :f.d] / st[..., f.d + 1:], ref, tol)
            assert (st[..., f.d] + torch.log2(st[..., f.d + 1]) - lse).abs().max() < 2.0 ** -12      # (as for the causal states)
        at += n_s
    f.clean()


@pytest.mark.gpu
def test_a_window_as_wide_as_the_sequence_and_none_agree_with_the_causal_call():
    f = Filled([700, 1100, 33], G=4, H=2, seed=15, P=16)
    for n in (1, 2, 30):
        q = torch.stack(f.queries([n] * 3)).cuda()
        want = f.cache.attention(f.table, f.lengths, q)
        assert torch.equal(want, f.cache.attention(f.table, f.lengths, q, window=0, sinks=0))
        for W, S in ((1100, 0), (2 ** 31 - 1, 2 ** 31 - 1), (5, 1100)):
            out = f.cache.attention(f.table, f.lengths, q, window=W, sinks=S)
            for s in range(3):
                check(out[s], *seen_by(f, q[s].cpu(), s, window_seen(f.lens[s], n, 0, 0))[::2])
    f.clean()


# ---- GPU: trees --------------------------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 200])
@pytest.mark.parametrize("W, S", [(0, 0), (1, 0), (7, 0), (7, 12), (300, 12)])
def test_masks_from_parents(n, W, S):
    rng = random.Random(n)
    cache = pkv.Q4Cache(config())
    parents = [random_parents(rng, n), [j - 1 for j in range(n)], [-1] * n, random_parents(rng, n, n)]
    lengths = [n, n + 3, n + 200, n + 9]
    masks, depths = cache.tree_masks(torch.tensor(parents, **INTS).cuda(), torch.tensor(lengths, **INTS).cuda(), window=W, sinks=S)
    for s in range(4):
        bits, deep = tree_bits(parents[s], lengths[s] - n, W, S)
        assert torch.equal(masks[s].cpu(), pack(bits)) and depths[s].tolist() == deep
    assert cache.stats() == {"device_timeouts": 0, "bad_pages": 0, "bad_lengths": 0}


@pytest.mark.gpu
def test_masks_of_ragged_rows_and_of_long_branches():
    rng = random.Random(1)
    cache = pkv.Q4Cache(config())
    ns = [0, 3000, 1, 130]
    trees = [random_parents(rng, n, 1 if n == 3000 else 5) for n in ns]
    parents = torch.tensor([-9] + sum(trees, []) + [77], **INTS).cuda()
    masks, depths = cache.tree_masks(parents, offsets=offsets_of(ns, start=1).cuda(), max_q_len=3000)
    at = 1
    for tree in trees:
        if tree:
            bits, deep = tree_bits(tree)
            assert torch.equal(masks[at:at + len(tree)].cpu(), pack(bits, 47)) and depths[at:at + len(tree)].tolist() == deep
        at += len(tree)
    assert cache.stats()["bad_lengths"] == 0


@pytest.mark.gpu
def test_parents_that_make_no_sense_and_more_rows_than_the_bound():
    cache = pkv.Q4Cache(config())
    parents = torch.tensor([[0, 5, 1, -2, 3, 2 ** 31 - 1]], **INTS)                # rows 0, 1, 3 and 5 continue nothing that is there
    masks, depths = cache.tree_masks(parents.cuda())
    bits, deep = tree_bits([-1, -1, 1, -1, 3, -1])
    assert torch.equal(masks[0].cpu(), pack(bits)) and depths[0].tolist() == deep
    assert cache.stats()["bad_lengths"] == 4
    L = pkv.lib()
    masks, depths = torch.full((6, 1), 5, **LONGS).cuda(), torch.full((6,), 5, **INTS).cuda()
    off = torch.tensor([0, 4, 6], **INTS).cuda()
    assert L.pkv_q4_tree_masks(cache.handle, 2, None, 6, off.data_ptr(), 3, torch.full((6,), -1, **INTS).cuda().data_ptr(), 0, 0, masks.data_ptr(), 1,
                               depths.data_ptr(), torch.cuda.current_stream().cuda_stream) == pkv.PKV_OK
    assert masks[:, 0].tolist() == [1, 2, 4, 5, 1, 2] and depths.tolist() == [0, 0, 0, 5, 0, 0]
    assert cache.stats()["bad_lengths"] == 5


@pytest.mark.usefixtures("room")
@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("n, G", [(2, 4), (7, 1), (7, 4), (16, 2), (17, 8), (64, 4), (70, 4), (130, 3)])
def test_trees(shape, n, G):
    rng = random.Random(n)
    f = Filled([n, n + 1, 64 + n, 401, 1300], G=G, seed=n, **shape)
    parents = [random_parents(rng, n) for _ in f.lens]
    q = torch.stack(f.queries([n] * 5))
    for W, S in ((0, 0), (5, 3), (200, 40)):
        masks, _ = f.cache.tree_masks(torch.tensor(parents, **INTS).cuda(), f.lengths, window=W, sinks=S)
        out = f.cache.attention(f.table, f.lengths, q.cuda(), tree=masks, window=W, sinks=S)
        for s, T in enumerate(f.lens):
            bits, _ = tree_bits(parents[s], T - n, W, S)
            check(out[s], *seen_by(f, q[s], s, tree_seen(T, bits, W, S))[::2])
    f.clean()


@pytest.mark.usefixtures("room")
@pytest.mark.gpu
@pytest.mark.parametrize("n, G", [(3, 4), (16, 2), (70, 4)])
def test_any_masks(n, G):
    """Masks that are no tree's: rows that see nothing new, rows that see later rows, bits of rows that the sequence does not have."""
    f = Filled([n, n + 30, 500], G=G, H=2, seed=40)
    gen = torch.Generator().manual_seed(n)
    bits = torch.rand(3, n, n, generator=gen) < 0.3
    bits[:, 0] = False
    bits[:, n - 1] = True
    words = -(-n // 64) + 2
    q = torch.stack(f.queries([n] * 3))
    masks = torch.stack([pack(b, words) for b in bits])
    masks[:, :, n // 64] |= -(1 << (n % 64))                                       # bits of rows n, n + 1, ...
    masks[:, :, n // 64 + 1:] = -1
    for W, S in ((0, 0), (90, 7)):
        out = f.cache.attention(f.table, f.lengths, q.cuda(), tree=masks.cuda(), window=W, sinks=S)
        for s, T in enumerate(f.lens):
            check(out[s], *seen_by(f, q[s], s, tree_seen(T, bits[s], W, S))[::2])
        assert (out[0, 0] == 0).all()                                              # no context, no bits
    f.clean()


@pytest.mark.gpu
@pytest.mark.parametrize("P", [16, 64])
@pytest.mark.parametrize("n, G, n_ctas, kernel", [(3, 4, 0, 2), (20, 4, 1, 1), (40, 4, 1, 1), (4, 2, 0, 0)])
def test_the_page_that_ends_before_a_window_may_be_gone(n, G, n_ctas, kernel, P):
    """The last position of a page is the first that no row sees: the page has gone back."""
    long = 30000 if kernel == 0 else 0
    C = 20 * P + 5 + long // P * P
    W = C - (4 * P - 1)                                    # C + 1 - W: the first position of page 4
    f = Filled([C + n], G=G, H=2, P=P, seed=60, n_ctas=n_ctas)
    assert _route(f.cache, 1, n, f.table.shape[1] * P, dict(window=W, sinks=3, tree=True))[0] == kernel
    parents = random_parents(random.Random(n), n)
    q = f.queries([n])[0]
    for tree in (True, False):
        masks = f.cache.tree_masks(torch.tensor([parents], **INTS).cuda(), f.lengths, window=W, sinks=3)[0] if tree else None
        table = f.table.clone()
        table[0, 1:4] = -1
        out = f.cache.attention(table, f.lengths, q[None].cuda(), tree=masks, window=W, sinks=3)
        see = tree_seen(C + n, tree_bits(parents, C, W, 3)[0], W, 3) if tree else window_seen(C + n, n, W, 3)
        assert see[:, 4 * P].any() and not see[:, P:4 * P].any()
        check(out[0], *seen_by(f, q, 0, see)[::2])
    f.clean()


@pytest.mark.usefixtures("room")
@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES[:4], ids=str)
@pytest.mark.parametrize("ns", [[0, 1, 5, 0, 33], [3, 0, 0, 0, 0], [1, 1, 1, 1, 1], [0, 1, 2, 150, 300]])
@pytest.mark.parametrize("W, S", [(0, 0), (50, 5)])
def test_ragged_trees_and_windows(shape, ns, W, S):
    rng = random.Random(3)
    f = Filled([0, 1, 200, 150, 310], G=4, seed=11, **shape)
    ns = [min(a, b) for a, b in zip(ns, f.lens)]
    qs = f.queries(ns)
    pad = torch.zeros(1, f.H * f.G, f.d, dtype=f.dtype)
    q = torch.cat([pad, *qs, pad]).cuda()
    off = offsets_of(ns, start=1).cuda()
    parents = [random_parents(rng, n) for n in ns]
    for most in (max(ns), None):
        masks, _ = f.cache.tree_masks(torch.tensor([0] + sum(parents, []) + [0], **INTS).cuda(), f.lengths, off, most, W, S)
        for tree in ([masks, None] if W else [masks]):
            out = torch.full_like(q, 5.0)
            f.cache.attention(f.table, f.lengths, q, out=out, offsets=off, max_q_len=most, window=W, sinks=S, tree=tree)
            assert (out[0] == 5).all() and (out[-1] == 5).all()
            at = 1
            for s, (n, T) in enumerate(zip(ns, f.lens)):
                if n:
                    see = window_seen(T, n, W, S) if tree is None else tree_seen(T, tree_bits(parents[s], T - n, W, S)[0], W, S)
                    check(out[at:at + n], *seen_by(f, qs[s], s, see)[::2])
                at += n
    f.clean()


@pytest.mark.usefixtures("room")
@pytest.mark.gpu
@pytest.mark.parametrize("n, G", [(4, 4), (70, 4)])
@pytest.mark.parametrize("what", ["k", "v"])
def test_drafted_rows_that_are_not_finite_reach_only_their_branch(n, G, what):
    f = Filled([60 + n, 300], G=G, H=1, seed=6)
    parents = [[-1] + [random.Random(s).randint(0, j - 1) if j > 2 else -1 for j in range(1, n)] for s in range(2)]
    q = torch.stack(f.queries([n] * 2))
    rows = [x.clone() for x in getattr(f, what)]
    hit = 1                                                                         # row 1: a branch of its own
    for s in range(2):
        rows[s][f.lens[s] - n + hit, 0, 40] = math.nan if s else math.inf
    k, v = (torch.cat(rows if what == x else getattr(f, x)).cuda() for x in "kv")
    f.cache.append_kv(f.table, f.lengths, k, v, f.off)
    masks, _ = f.cache.tree_masks(torch.tensor(parents, **INTS).cuda())
    out = f.cache.attention(f.table, f.lengths, q.cuda(), tree=masks)
    for s, T in enumerate(f.lens):
        bits, _ = tree_bits(parents[s])
        ref, _, tol = seen_by(f, q[s], s, tree_seen(T, bits))
        blind = ~bits[:, hit]
        check(out[s].cpu()[blind], ref[blind], tol[blind])
        assert torch.isnan(out[s].cpu()[~blind][:, :, 32:64]).all()


@pytest.mark.usefixtures("room")
@pytest.mark.gpu
@pytest.mark.parametrize("n, G", [(2, 4), (8, 4), (70, 2)])
def test_selected_pages_and_lengths_that_make_no_sense(n, G):
    """Bad page numbers in the window are skipped and counted, others are not looked at; lengths are held inside the table."""
    W, S, P = 60, 3, 32
    f = Filled([150, 290], G=G, H=2, P=P, seed=8)
    table = f.table.clone()
    low = [max(0, T - n + 1 - W) for T in f.lens]
    gone = []
    for s, T in enumerate(f.lens):
        e = (T - n) // P
        table[s, e] = (f.rows.n_pages, -1)[s]
        gone.append(range(e * P, min(T, e * P + P)))
        for hidden in range(-(-S // P), low[s] // P):
            table[s, hidden] = 1 << 30
    q = torch.stack(f.queries([n, n]))
    out = f.cache.attention(table, f.lengths, q.cuda(), window=W, sinks=S)
    assert f.cache.stats()["bad_pages"] > 0
    for s, T in enumerate(f.lens):
        see = window_seen(T, n, W, S)
        see[:, list(gone[s])] = False
        check(out[s], *seen_by(f, q[s], s, see)[::2])
    bad = f.cache.stats()["bad_lengths"]
    out = f.cache.attention(f.table, torch.tensor([-5, 290], **INTS).cuda(), q.cuda(), window=W, sinks=S)
    assert (out[0] == 0).all() and f.cache.stats()["bad_lengths"] > bad
    check(out[1], *seen_by(f, q[1], 1, window_seen(290, n, W, S))[::2])
    masks = f.cache.tree_masks(torch.full((2, n), -1, **INTS).cuda())[0]
    out = f.cache.attention(f.table, torch.tensor([-5, 290], **INTS).cuda(), q.cuda(), tree=masks)
    assert (out[0] == 0).all()                                                      # (no position is there)
    check(out[1], *seen_by(f, q[1], 1, tree_seen(290, torch.eye(n, dtype=torch.bool)))[::2])


@pytest.mark.usefixtures("room")
@pytest.mark.gpu
@pytest.mark.parametrize("n, G, H", [(1, 4, 2), (6, 8, 1), (80, 4, 2)])
@pytest.mark.parametrize("dtype, d", [(BF16, 128), (FP16, 64)])
def test_selected_states(n, G, H, dtype, d):
    f = Filled([n, 130 + n, 700], G=G, H=H, d=d, dtype=dtype, seed=12)
    q = torch.stack(f.queries([n] * 3))
    rng = random.Random(n)
    parents = [random_parents(rng, n) for _ in range(3)]
    for tree in (False, True):
        W, S = 77, 9
        masks = f.cache.tree_masks(torch.tensor(parents, **INTS).cuda(), f.lengths, window=W, sinks=S)[0] if tree else None
        st = f.cache.attention_partial(f.table, f.lengths, q.cuda(), window=W, sinks=S, tree=masks).to("cpu", torch.float64)
        for s, T in enumerate(f.lens):
            see = tree_seen(T, tree_bits(parents[s], T - n, W, S)[0], W, S) if tree else window_seen(T, n, W, S)
            ref, lse, tol = seen_by(f, q[s], s, see)
            check(st[s, ..., :d] / st[s, ..., d + 1:], ref, tol)
            assert (st[s, ..., d] + torch.log2(st[s, ..., d + 1]) - lse).abs().max() < 2.0 ** -12      # (as for the causal states)


@pytest.mark.usefixtures("room")
@pytest.mark.gpu
@pytest.mark.parametrize("n, G", [(1, 4), (3, 8), (90, 4)])
def test_selected_attention_of_strided_queries(n, G):
    f = Filled([150, 91], G=G, H=2, seed=14)
    q = torch.stack(f.queries([n, n]))
    hq, W, S = 2 * G, 40, 2
    fused = torch.randn(2, n, hq + 4, 128).to(BF16).cuda()
    fused[:, :, :hq] = q.cuda()
    wide = torch.full((2, n, hq + 1, 136), 7.0, dtype=BF16, device="cuda")
    f.cache.attention(f.table, f.lengths, fused[:, :, :hq], out=wide[:, :, 1:, :128], window=W, sinks=S)
    for s in range(2):
        check(wide[s, :, 1:, :128], *seen_by(f, q[s], s, window_seen(f.lens[s], n, W, S))[::2])
    assert (wide[:, :, 0] == 7).all() and (wide[..., 128:] == 7).all()


@pytest.mark.gpu
@pytest.mark.parametrize("n, G", [(1, 4), (3, 8), (64, 4)])
@pytest.mark.parametrize("fill", [0xff, 0x00, 0x7b])
def test_what_the_workspace_of_a_selection_held_does_not_matter(n, G, fill):
    lens, W, S = [4000, max(n, 64), max(n, 100)], 3000, 5
    f = Filled(lens, G=G, H=2, P=16, seed=17, room=4800)
    q = torch.stack(f.queries([n] * 3))
    out = torch.empty_like(q, device="cuda")
    size = pkv.pkv_q4_attention_select_workspace(f.cache.handle, 3, n, 4800, W, S)
    work = torch.full((max(16, size),), fill, dtype=torch.uint8, device="cuda")
    strides = (2 * G * 128, 128)
    pkv.pkv_q4_attention_select(f.cache.handle, 3, f.table, f.table.shape[1], f.lengths, 3 * n, None, n, 4800, W, S, None, 0, q.cuda(), strides, out, strides,
                                None, work, size, torch.cuda.current_stream())
    for s in range(3):
        check(out[s], *seen_by(f, q[s], s, window_seen(lens[s], n, W, S))[::2])


@pytest.mark.usefixtures("room")
@pytest.mark.gpu
@pytest.mark.parametrize("G", [33, 64])
def test_windows_with_many_query_heads_per_kv_head(G):
    for n, H in ((1, 2), (9, 1)):
        f = Filled([9, 70, 333], G=G, H=H, seed=24)
        q = torch.stack(f.queries([n] * 3))
        out = f.cache.attention(f.table, f.lengths, q.cuda(), window=50, sinks=3)
        for s in range(3):
            check(out[s], *seen_by(f, q[s], s, window_seen(f.lens[s], n, 50, 3))[::2])


@pytest.mark.gpu
@pytest.mark.parametrize("n, most", [(1, 40), (1, 3000), (9, 40)])
def test_windows_of_more_sequences_than_a_cta_has_threads(n, most):
    gen = torch.Generator().manual_seed(n)
    lens = [0 if i % 7 == 0 else max(n, int(t)) for i, t in enumerate(torch.randint(1, 41, (900,), generator=gen))]
    f = Filled(lens, G=2, H=1, P=16, seed=26)
    q = torch.stack(f.queries([n] * 900))
    out = f.cache.attention(f.table, f.lengths, q.cuda(), max_len=most, window=11, sinks=2).cpu()
    for s in range(900):
        if lens[s]:
            check(out[s], *seen_by(f, q[s], s, window_seen(lens[s], n, 11, 2))[::2])
        else:
            assert (out[s] == 0).all()
    f.clean()


@pytest.mark.usefixtures("room")
@pytest.mark.gpu
@pytest.mark.parametrize("n, G", [(1, 4), (2, 4), (64, 4)])
def test_selected_attention_has_the_same_bits_every_run_on_any_stream_and_in_a_graph(n, G):
    f = Filled([700, 1100, 90], G=G, H=2, seed=15, P=16)
    qs = torch.stack(f.queries([n] * 3)).cuda()
    parents = torch.tensor([random_parents(random.Random(s), n) for s in range(3)], **INTS).cuda()

    def calls():
        masks, depths = f.cache.tree_masks(parents, f.lengths, window=300, sinks=4)
        return (f.cache.attention(f.table, f.lengths, qs, window=300, sinks=4), f.cache.attention(f.table, f.lengths, qs, tree=masks),
                f.cache.attention(f.table, f.lengths, qs, tree=masks, window=300, sinks=4), masks, depths)

    first = calls()
    torch.cuda.synchronize()
    same = lambda xs: all(torch.equal(a, b) for a, b in zip(first, xs))             # noqa: E731
    for _ in range(3):
        assert same(calls())
    streams = [torch.cuda.Stream() for _ in range(4)]
    outs = []
    for s in streams * 3:
        with torch.cuda.stream(s):
            outs.append(calls())
    torch.cuda.synchronize()
    assert all(same(o) for o in outs)
    graphs, kept = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            kept.append(calls())
        graphs.append(g)
    for _ in range(3):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    assert all(same(o) for o in kept)
    f.clean()


# ---- GPU: kept rows ----------------------------------------------------------------------------------------------------
def values_of(f, table, lengths, lens):
    k, v = (torch.empty(sum(lens), f.H, f.d, dtype=f.dtype, device="cuda") for _ in "kv")
    f.cache.read_kv(table, lengths, k, v, offsets_of(lens).cuda())
    return [x.cpu().split(lens) for x in (k, v)]


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("n", [1, 2, 17, 64, 300])
def test_kept_rows(shape, n):
    rng = random.Random(n)
    lens = [n, n + 1, n + 33, 500 + n]
    f = Filled(lens, seed=n, **shape)
    counts = [0, n, n // 2, max(1, n - 1)]
    paths = [sorted(rng.sample(range(n), c)) for c in counts]
    table = torch.tensor([p + [99] * (n - len(p)) for p in paths], **INTS)          # (entries behind the counts do not matter)
    kept = f.cache.keep_rows(f.table, f.lengths, table.cuda(), torch.tensor(counts, **INTS).cuda(), n)
    want = [T - n + c for T, c in zip(lens, counts)]
    assert kept.tolist() == want and f.lengths.tolist() == lens
    K, V = values_of(f, f.table, f.lengths, lens)
    for s, T in enumerate(lens):
        C = T - n
        rows = list(range(C)) + [C + p for p in paths[s]] + list(range(C + counts[s], T))      # (what is behind stays)
        assert torch.equal(K[s], f.K[s][rows].to(f.dtype)) and torch.equal(V[s], f.V[s][rows].to(f.dtype))
    f.clean()


@pytest.mark.gpu
def test_kept_rows_ragged_with_paths_that_make_no_sense():
    f = Filled([40, 0, 25, 9], P=16, H=3, seed=7)
    ns = [9, 0, 20, 9]
    off = offsets_of(ns, start=3).cuda()
    paths = torch.tensor([[1, 0, 9, 8, -1], [5, 5, 5, 5, 5], [4, 4, 19, 7, 12], [0, 1, 2, 3, 4]], **INTS)
    counts = torch.tensor([5, 3, 4, 900], **INTS)
    out = torch.full((4,), -1, **INTS).cuda()
    kept = f.cache.keep_rows(f.table, f.lengths, paths.cuda(), counts.cuda(), sum(ns) + 5, offsets=off, out=out)
    assert kept is out and out.tolist() == [31 + 5, 0, 5 + 4, 0 + 5]
    # sequence 0: rows 1 (0 < 1), 2 (9 is no row) and 4 (-1) are left, row 3 becomes row 8;  2: the same row twice is fine
    assert f.cache.stats() == {"device_timeouts": 0, "bad_pages": 0, "bad_lengths": 3 + 1 + 1}
    K, _ = values_of(f, f.table, f.lengths, f.lens)
    assert torch.equal(K[0], f.K[0][list(range(31)) + [32, 32, 33, 39, 35, 36, 37, 38, 39]].to(BF16))
    assert torch.equal(K[2], f.K[2][list(range(5)) + [9, 9, 24, 12] + list(range(9, 25))].to(BF16))
    assert torch.equal(K[3], f.K[3].to(BF16))


@pytest.mark.gpu
def test_kept_rows_with_bad_pages_and_more_rows_than_tokens():
    f = Filled([40, 5], P=16, H=1, seed=7)
    table = f.table.clone()
    table[0, 2] = f.rows.n_pages                                                    # positions 32 .. 39
    before = f.cache.pool.clone()
    paths = torch.tensor([[8, 9], [0, 1]], **INTS).cuda()
    kept = f.cache.keep_rows(table, f.lengths, paths, torch.tensor([2, 2], **INTS).cuda(), 10)
    assert kept.tolist() == [32, 0] and torch.equal(before, f.cache.pool)
    stats = f.cache.stats()
    assert stats["bad_pages"] > 0 and stats["bad_lengths"] > 0


# ---- GPU: planned steps ------------------------------------------------------------------------------------------------
def device_plan(cache, ref, spare=0):
    t = lambda x, **kw: torch.tensor(x, **kw).cuda()                                # noqa: E731
    return dict(page_table=t(ref.table, **INTS), lengths=t(ref.lengths, **INTS), spans=t(ref.spans, **INTS), ring=t(ref.ring, **INTS),
                counters=t([ref.head, ref.tail, 9, 9], **LONGS))


def same_plan(ref, dev, p, result, capacity):
    missing, refused, offsets, positions, slots = result
    assert p.counters.tolist() == [ref.head, ref.tail, missing, refused]
    assert p.offsets.tolist() == offsets and p.lengths.tolist() == ref.lengths and [tuple(x) for x in p.spans.tolist()] == ref.spans
    if p.positions is not None:
        assert p.positions.tolist() == positions + [-5] * (capacity - len(positions))
    if p.slots is not None:
        assert p.slots.tolist() == slots + [-5] * (capacity - len(slots))
    assert dev["ring"].tolist() == ref.ring and dev["page_table"].tolist() == ref.table


def outputs(n_seqs, capacity):
    full = lambda n, kw: torch.full((n,) if isinstance(n, int) else n, -5, **kw).cuda()      # noqa: E731
    return pkv.Q4Plan(full(n_seqs, INTS), full(n_seqs + 1, INTS), full(capacity, INTS), full(capacity, LONGS), full((n_seqs, 2), INTS), full(4, LONGS))


@pytest.mark.gpu
@pytest.mark.parametrize("P", [16, 64, 256])
@pytest.mark.parametrize("S, most", [(1, 40), (5, 500), (33, 100), (1500, 30), (300, 90)])
@pytest.mark.parametrize("W, sinks", [(0, 0), (100, 0), (37, 70)])
def test_planned_steps(P, S, most, W, sinks):
    """Steps in a row: growing, finished and starting requests, a ring that goes round, steps that cannot be served."""
    rng = random.Random(S * P + W)
    max_pages = -(-6 * most // P) + 1
    n_pages = max(3, S * max_pages // 2)
    cache = pkv.Q4Cache(config(n_kv_heads=1, n_q_heads=1, n_pages=n_pages, page_size=P, head_dim=64))
    order = rng.sample(range(n_pages), n_pages)
    ref = Plan(P, n_pages, max_pages, [[-7] * max_pages for _ in range(S)], [0] * S, [(0, 0)] * S, order, 0, n_pages)
    dev = device_plan(cache, ref)
    served = 0
    for step in range(12):
        rows = [rng.choice([0, 1, 1, rng.randint(1, most)]) if rng.random() < 0.85 else -1 for _ in range(S)]
        rows = [n if T + n <= max_pages * P or step == 5 else -1 for n, T in zip(rows, ref.lengths)]
        capacity = sum(max(0, n) for n in rows) + rng.choice([0, 3, -1 if step == 7 else 1])
        capacity = max(0, capacity)
        lengths = list(ref.lengths)
        result = ref.step(rows, capacity, W, sinks)
        out = outputs(S, capacity)
        p = cache.plan(**dev, rows=torch.tensor(rows, **INTS).cuda(), n_rows=capacity, window=W, sinks=sinks, out=out)
        assert p is out
        same_plan(ref, dev, p, result, capacity)
        assert dev["lengths"].tolist() == lengths                                   # (inputs stay)
        dev.update(lengths=p.lengths, spans=p.spans, counters=p.counters)
        served += result[:2] == (0, 0)
    assert served >= 4
    assert cache.stats() == {"device_timeouts": 0, "bad_pages": 0, "bad_lengths": 0}


@pytest.mark.gpu
@pytest.mark.parametrize("S, n", [(4, 5000), (2100, 9), (3, 1)])
def test_a_plan_in_place_and_without_positions(S, n):
    P = 32
    cache = pkv.Q4Cache(config(n_kv_heads=1, n_q_heads=1, n_pages=S * (2 * n // P + 2), page_size=P, head_dim=64))
    max_pages = 2 * n // P + 2
    ring, counters = cache.new_ring()
    ref = Plan(P, ring.numel(), max_pages, [[-1] * max_pages for _ in range(S)], [0] * S, [(0, 0)] * S, ring.tolist(), 0, ring.numel())
    dev = device_plan(cache, ref)
    rows = torch.full((S,), n, **INTS).cuda()
    whole = outputs(S, S * n)
    out = whole._replace(lengths=dev["lengths"], spans=dev["spans"], counters=dev["counters"])
    for _ in range(2):
        result = ref.step([n] * S, S * n)
        cache.plan(**dev, rows=rows, n_rows=S * n, out=out)
        same_plan(ref, dev, out, result, S * n)
    result = ref.step([-1] * S, 0)
    cache.plan(**dev, rows=torch.full((S,), -1, **INTS).cuda(), n_rows=0, out=out._replace(positions=None, slots=None))
    same_plan(ref, dev, out._replace(positions=None, slots=None), result, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("S", [3, 1300])
@pytest.mark.parametrize("bad", ["rows", "length", "too long", "first", "end", "span", "head", "tail", "full ring", "capacity", "missing"])
def test_steps_that_make_no_sense_change_nothing(S, bad):
    P, max_pages, n_pages = 16, 8, 4 * S
    cache = pkv.Q4Cache(config(n_kv_heads=1, n_q_heads=1, n_pages=n_pages, page_size=P, head_dim=64))
    held = 2
    table = [[s * held, s * held + 1] + [-1] * 6 for s in range(S)]
    ring = list(range(held * S, n_pages)) + [-1] * (held * S)
    ref = Plan(P, n_pages, max_pages, table, [20] * S, [(0, held)] * S, ring, 0, 2 * S)
    rows, capacity = [1] * S, S
    if bad == "rows":
        rows[1] = -2
    elif bad == "length":
        ref.lengths[1] = -1
    elif bad == "too long":
        rows[1], capacity = 109, S + 200
    elif bad == "first":
        ref.spans[1] = (-1, 2)
    elif bad == "end":
        ref.spans[1] = (0, 9)
    elif bad == "span":
        ref.spans[1] = (2, 1)
    elif bad == "head":
        ref.head = -1
    elif bad == "tail":
        ref.head = 3 * S
    elif bad == "full ring":
        rows, ref.tail = [-1] * S, 4 * S
    elif bad == "capacity":
        capacity = S - 1
    else:
        rows, capacity = [29] * S, 29 * S
        ref.head = 2 * S - 1
    dev = device_plan(cache, ref)
    result = ref.step(rows, capacity)
    assert result[0] + result[1] > 0
    out = outputs(S, capacity)
    cache.plan(**dev, rows=torch.tensor(rows, **INTS).cuda(), n_rows=capacity, out=out)
    same_plan(ref, dev, out, result, capacity)


@pytest.mark.gpu
def test_windows_trees_and_kept_rows_in_pages_beyond_four_gigabytes():
    H, P, n, T = 8, 64, 5, 180
    cache = pkv.Q4Cache(config(n_kv_heads=H, n_q_heads=H, n_pages=70000, page_size=P))
    assert 60000 * cache.sizes.page_bytes > 1 << 32
    gen = torch.Generator().manual_seed(1)
    k, v, q = (rows_of(gen, T, H, 128, BF16) for _ in "kvq")
    table, lengths = torch.tensor([[69999, 65000, 60000]], **INTS).cuda(), torch.tensor([T], **INTS).cuda()
    cache.append_kv(table, lengths, k[None].cuda(), v[None].cuda())
    K, V, q = quantised(k, 32), quantised(v, 32), q[-n:]
    parents = [-1, 0, 0, 1, -1]
    masks, _ = cache.tree_masks(torch.tensor([parents], **INTS).cuda(), lengths, window=100, sinks=3)
    out = cache.attention(table, lengths, q[None].cuda(), tree=masks, window=100, sinks=3)
    ref, _, tol = attention_seen(q, K, V, tree_seen(T, tree_bits(parents, T - n, 100, 3)[0], 100, 3), 1 / math.sqrt(128), BF16)
    check(out[0], ref, tol)
    kept = cache.keep_rows(table, lengths, torch.tensor([[0, 1, 3]], **INTS).cuda(), torch.tensor([3], **INTS).cuda(), n)
    ko, vo = (torch.empty(1, T - 2, H, 128, dtype=BF16, device="cuda") for _ in "kv")
    cache.read_kv(table, kept, ko, vo)
    rows = list(range(T - n)) + [T - n + i for i in (0, 1, 3)]
    assert kept.tolist() == [T - 2] and torch.equal(ko[0].cpu(), K[rows].to(BF16)) and torch.equal(vo[0].cpu(), V[rows].to(BF16))


@pytest.mark.gpu
def test_windows_plans_and_kept_rows_of_as_many_sequences_as_a_call_takes():
    """65535 requests of one token, every ninth empty: each sees its own token, the value as it was quantised."""
    S, H, d, P = 65535, 2, 64, 16
    cache = pkv.Q4Cache(config(n_kv_heads=H, n_q_heads=2 * H, head_dim=d, page_size=P, n_pages=S))
    rows = torch.ones(S, dtype=torch.int32)
    rows[::9] = 0
    n = int(rows.sum())
    ring, counters = cache.new_ring(torch.randperm(S, generator=torch.Generator().manual_seed(1)))
    table = torch.full((S, 2), -1, **INTS).cuda()
    p = cache.plan(table, torch.zeros(S, **INTS).cuda(), rows.cuda(), torch.zeros(S, 2, **INTS).cuda(), ring, counters, n, window=40, sinks=3)
    assert p.counters.tolist() == [n, S, 0, 0] and torch.equal(p.lengths.cpu(), rows) and torch.equal(p.offsets[1:].cpu(), rows.cumsum(0).int())
    there = rows.bool()
    assert torch.equal(p.slots.cpu(), table.cpu()[there, 0].long() * P) and (p.positions == 0).all()
    assert torch.equal(table.cpu()[there, 0], ring.cpu()[:n])
    k, v = (torch.randn(n, H, d, generator=torch.Generator().manual_seed(i)).to(BF16) for i in (2, 3))
    cache.append_kv(table, p.lengths, k.cuda(), v.cuda(), p.offsets)
    q = torch.randn(n, 2 * H, d, generator=torch.Generator().manual_seed(4)).to(BF16).cuda()
    # (one token: the result is code * scale, off by half a bf16 step where it lies between two numbers, and by 2^-20 from exp2; see the
    # causal call's test of the same)
    exact = quantised(v, 32).repeat_interleave(2, 1)
    near = lambda out: ((out.cpu().double() - exact).abs() <= exact.abs() * (2.0 ** -8 + 2.0 ** -20)).all()      # noqa: E731
    assert near(cache.attention(table, p.lengths, q, offsets=p.offsets, max_q_len=1, window=40, sinks=3))
    masks, depths = cache.tree_masks(torch.full((n,), -1, **INTS).cuda(), p.lengths, p.offsets, 1)
    assert (masks == 1).all() and (depths == 0).all()
    assert near(cache.attention(table, p.lengths, q, offsets=p.offsets, max_q_len=1, tree=masks))
    counts = (torch.arange(S) % 2).int()
    kept = cache.keep_rows(table, p.lengths, torch.zeros(S, 1, **INTS).cuda(), torch.minimum(counts, rows).cuda(), n, p.offsets)
    assert torch.equal(kept.cpu(), torch.minimum(counts, rows))
    done = cache.plan(table, p.lengths, torch.full((S,), -1, **INTS).cuda(), p.spans, ring, p.counters, 0)
    assert done.counters.tolist() == [n, S + n, 0, 0] and torch.equal(ring[:n].cpu(), table.cpu()[there, 0])
    assert cache.stats() == {"device_timeouts": 0, "bad_pages": 0, "bad_lengths": 0}


# ---- GPU: a run of them together --------------------------------------------------------------------------------------
class Served:
    """Requests served with planned steps, drafted trees and kept rows; what they hold, in 64 bits."""

    def __init__(self, S, H, G, P, W, sinks, n_pages, max_pages, dtype=BF16, d=128, g=32, seed=0):
        self.S, self.H, self.G, self.W, self.sinks, self.d, self.g, self.dtype = S, H, G, W, sinks, d, g, dtype
        self.gen, self.rng = torch.Generator().manual_seed(seed), random.Random(seed)
        self.cache = pkv.Q4Cache(config(n_kv_heads=H, n_q_heads=H * G, head_dim=d, group_size=g, page_size=P, dtype=dtype, n_pages=n_pages))
        self.cache.pool.fill_(0xff)
        self.table = torch.full((S, max_pages), -1, **INTS).cuda()
        self.lengths, self.spans = torch.zeros(S, **INTS).cuda(), torch.zeros(S, 2, **INTS).cuda()
        self.ring, self.counters = self.cache.new_ring(torch.randperm(n_pages, generator=self.gen))
        self.K = [torch.empty(0, H, d, dtype=torch.float64) for _ in range(S)]
        self.V = list(self.K)

    def step(self, rows, tree=False, keep=True):
        cache, n = self.cache, sum(max(0, x) for x in rows)
        p = cache.plan(self.table, self.lengths, torch.tensor(rows, **INTS).cuda(), self.spans, self.ring, self.counters, n, window=self.W, sinks=self.sinks)
        self.spans, self.counters = p.spans, p.counters
        assert p.counters[2:].tolist() == [0, 0]
        new = [max(0, x) for x in rows]
        k, v, q = (rows_of(self.gen, n, h, self.d, self.dtype, False) for h in (self.H, self.H, self.H * self.G))
        cache.append_kv(self.table, p.lengths, k.cuda(), v.cuda(), p.offsets)
        parents, masks = [random_parents(self.rng, x, 4) for x in new], None
        if tree:
            masks, depths = cache.tree_masks(torch.tensor(sum(parents, []), **INTS).cuda(), p.lengths, p.offsets, max(new), self.W, self.sinks)
        out = cache.attention(self.table, p.lengths, q.cuda(), offsets=p.offsets, max_q_len=max(new), window=self.W, sinks=self.sinks, tree=masks).cpu()
        at, kept = 0, [[] for _ in rows]
        for s, x in enumerate(rows):
            if x < 0:
                self.K[s], self.V[s] = self.K[s][:0], self.V[s][:0]
                continue
            here = slice(at, at + x)
            at += x
            K, V = torch.cat([self.K[s], quantised(k[here], self.g)]), torch.cat([self.V[s], quantised(v[here], self.g)])
            T, C = K.shape[0], K.shape[0] - x
            if x:
                if tree:
                    bits, deep = tree_bits(parents[s], C, self.W, self.sinks)
                    assert depths[here].tolist() == deep
                see = tree_seen(T, bits, self.W, self.sinks) if tree else window_seen(T, x, self.W, self.sinks)
                ref, _, tol = attention_seen(q[here], K, V, see, 1 / math.sqrt(self.d), self.dtype)
                check(out[here], ref, tol)
            if tree:                                                                # a branch is accepted
                j = self.rng.randint(-1, x - 1)
                while j >= 0:
                    kept[s].insert(0, j)
                    j = parents[s][j]
                K, V = K[list(range(C)) + [C + i for i in kept[s]]], V[list(range(C)) + [C + i for i in kept[s]]]
            self.K[s], self.V[s] = K, V
        self.lengths = p.lengths
        if tree:
            m = max(new)
            paths = torch.tensor([x + [0] * (m - len(x)) for x in kept], **INTS)
            self.lengths = cache.keep_rows(self.table, p.lengths, paths.cuda(), torch.tensor([len(x) for x in kept], **INTS).cuda(), n, p.offsets)
        assert self.lengths.tolist() == [x.shape[0] for x in self.K]


@pytest.mark.gpu
@pytest.mark.parametrize("W, sinks, P, pages", [(0, 0, 16, 260), (90, 5, 16, 100), (64, 16, 32, 60)])
@pytest.mark.parametrize("dtype, d, g, G", [(BF16, 128, 32, 4), (FP16, 64, 64, 7)])
def test_serving_with_plans_trees_and_windows(W, sinks, P, pages, dtype, d, g, G):
    """Prompts in chunks, decode steps, drafted trees of which a branch is kept, requests that finish and start; with a window the
    pool is smaller than what the requests hold in all."""
    f = Served(4, 2, G, P, W, sinks, pages, 60, dtype, d, g, seed=W + P)
    f.step([100, 40, 0, 7])
    f.step([60, 1, 33, 1])
    for i in range(6):
        f.step([7, 7, 7, 7] if i % 2 else [12, 1, 5, 9], tree=True)
        f.step([1, 1, 1, 1])
    f.step([-1, 1, 1, 90])
    f.step([55, 1, -1, 1])
    for _ in range(3):
        f.step([24, 3, 0, 24], tree=True)
    assert f.cache.stats() == {"device_timeouts": 0, "bad_pages": 0, "bad_lengths": 0}


@pytest.mark.gpu
def test_a_drafting_step_in_one_captured_graph():
    """plan -> append -> masks -> attention -> keep, captured once, lengths, entries and ring in place, replayed while windows slide over pages."""
    S, n, H, G, P, W, sinks = 3, 6, 2, 4, 16, 70, 3
    gen, rng = torch.Generator().manual_seed(5), random.Random(5)
    cache = pkv.Q4Cache(config(n_kv_heads=H, n_q_heads=H * G, page_size=P, n_pages=30))
    table = torch.full((S, 40), -1, **INTS).cuda()
    lengths, drafted, spans = torch.zeros(S, **INTS).cuda(), torch.zeros(S, **INTS).cuda(), torch.zeros(S, 2, **INTS).cuda()
    ring, counters = cache.new_ring()
    rows, parents = torch.full((S,), n, **INTS).cuda(), torch.full((S, n), -1, **INTS).cuda()
    paths, counts = torch.zeros(S, n, **INTS).cuda(), torch.zeros(S, **INTS).cuda()
    k, v, q = (torch.zeros(S, n, h, 128, dtype=BF16, device="cuda") for h in (H, H, H * G))
    out = torch.zeros_like(q)
    plan_out = outputs(S, S * n)._replace(lengths=drafted, spans=spans, counters=counters)

    def step():
        cache.plan(table, lengths, rows, spans, ring, counters, S * n, window=W, sinks=sinks, out=plan_out)
        cache.append_kv(table, drafted, k, v)
        masks, _ = cache.tree_masks(parents, drafted, window=W, sinks=sinks)
        cache.attention(table, drafted, q, out=out, tree=masks, window=W, sinks=sinks)
        cache.keep_rows(table, drafted, paths, counts, n, out=lengths)

    start = [x.clone() for x in (table, lengths, spans, ring, counters)]
    step()                                                                          # (warm-up; undone below)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for x, y in zip((table, lengths, spans, ring, counters), start):
        x.copy_(y)
    K = [torch.empty(0, H, 128, dtype=torch.float64) for _ in range(S)]
    V = list(K)
    for i in range(120):
        trees = [random_parents(rng, n, 3) for _ in range(S)]
        new = [rows_of(gen, S * n, h, 128, BF16, False).view(S, n, h, 128) for h in (H, H, H * G)]
        kept = []
        for s in range(S):
            j, path = rng.randint(0, n - 1), []
            while j >= 0:
                path.insert(0, j)
                j = trees[s][j]
            kept.append(path)
        for dst, src in zip((k, v, q, parents, paths, counts), (*new, torch.tensor(trees, **INTS), torch.tensor([p + [0] * (n - len(p)) for p in kept], **INTS),
                                                                torch.tensor([len(p) for p in kept], **INTS))):
            dst.copy_(src)
        g.replay()
        for s in range(S):
            C = K[s].shape[0]
            Ks, Vs = torch.cat([K[s], quantised(new[0][s], 32)]), torch.cat([V[s], quantised(new[1][s], 32)])
            bits, _ = tree_bits(trees[s], C, W, sinks)
            ref, _, tol = attention_seen(new[2][s], Ks, Vs, tree_seen(C + n, bits, W, sinks), 1 / math.sqrt(128), BF16)
            check(out[s], ref, tol)
            rows_kept = list(range(C)) + [C + j for j in kept[s]]
            K[s], V[s] = Ks[rows_kept], Vs[rows_kept]
        assert lengths.tolist() == [x.shape[0] for x in K] and counters[2:].tolist() == [0, 0]
    assert counters[1].item() > 30                                                  # the ring has gone round
    assert cache.stats() == {"device_timeouts": 0, "bad_pages": 0, "bad_lengths": 0}


@pytest.mark.gpu
def test_windowed_and_full_layers_of_one_model():
    """Layers are sequences of one call: a windowed layer's tables beside a full layer's, kept rows of both in one call."""
    H, G, P, T, n = 2, 4, 16, 200, 8
    f = Filled([T, T], H=H, G=G, P=P, seed=50)
    q = torch.stack(f.queries([n, n]))
    parents = random_parents(random.Random(2), n, 3)
    masks, _ = f.cache.tree_masks(torch.tensor([parents], **INTS).cuda())
    bits, _ = tree_bits(parents)
    full = f.cache.attention(f.table[:1].contiguous(), f.lengths[:1], q[:1].cuda(), tree=masks)
    part = f.cache.attention(f.table[1:].contiguous(), f.lengths[1:], q[1:].cuda(), tree=masks, window=100)
    check(full[0], *seen_by(f, q[0], 0, tree_seen(T, bits))[::2])
    check(part[0], *seen_by(f, q[1], 1, tree_seen(T, bits, 100))[::2])
    path = torch.tensor([[1, 4, 7]] * 2, **INTS).cuda()
    kept = f.cache.keep_rows(f.table, f.lengths, path, torch.tensor([3, 3], **INTS).cuda(), n)
    assert kept.tolist() == [T - n + 3] * 2
    K, V = values_of(f, f.table, kept, [T - n + 3] * 2)
    for s in range(2):
        rows = list(range(T - n)) + [T - n + i for i in (1, 4, 7)]
        assert torch.equal(K[s], f.K[s][rows].to(BF16)) and torch.equal(V[s], f.V[s][rows].to(BF16))


@pytest.mark.usefixtures("room")
@pytest.mark.gpu
@pytest.mark.parametrize("seed", range(8))
def test_random_selections(seed):
    rng = random.Random(seed)
    for _ in range(6):
        d = rng.choice([64, 128])
        shape = dict(dtype=rng.choice([BF16, FP16]), d=d, g=rng.choice([x for x in (32, 64, 128) if x <= d]),
                     P=rng.choice([16, 32, 64, 128, 256]), H=rng.randint(1, 3), G=rng.choice([1, 2, 3, 5, 8, 9, 16]))
        lens = [rng.choice([0, 1, rng.randint(1, 64), rng.randint(1, 700), rng.randint(1, 2500)]) for _ in range(rng.randint(1, 6))]
        most = rng.choice([1, 2, 5, 30, 100])
        ns = [min(t, rng.randint(0, most)) for t in lens]
        W = rng.choice([0, rng.randint(1, 40), rng.randint(1, 1500)])
        S = rng.choice([0, 3, rng.randint(1, 200)]) if W else 0
        tree = rng.random() < 0.5 or not W
        f = Filled(lens, seed=seed, **shape)
        qs = f.queries(ns)
        off = offsets_of(ns).cuda()
        bound = max(1, min(most, sum(ns)))
        parents = [random_parents(rng, n) for n in ns]
        masks = f.cache.tree_masks(torch.tensor(sum(parents, []), **INTS).cuda(), f.lengths, off, bound, W, S)[0] if tree and sum(ns) else None
        table = without_hidden_pages(f, shape["P"], ns, W, S) if W else f.table
        out = f.cache.attention(table, f.lengths, torch.cat(qs).cuda(), offsets=off, max_q_len=bound, window=W, sinks=S, tree=masks)
        at = 0
        for s, (n, T) in enumerate(zip(ns, lens)):
            if n:
                see = tree_seen(T, tree_bits(parents[s], T - n, W, S)[0], W, S) if masks is not None else window_seen(T, n, W, S)
                check(out[at:at + n], *seen_by(f, qs[s], s, see)[::2])
            at += n
        f.clean()


def captured_first():
    """Every call of a step is captured before it has ever run; the replay does what the calls do."""
    S, n, H, G, P = 2, 3, 2, 4, 16
    cache = pkv.Q4Cache(config(n_kv_heads=H, n_q_heads=H * G, page_size=P, n_pages=40))
    table, lengths = torch.full((S, 12), -1, **INTS).cuda(), torch.zeros(S, **INTS).cuda()
    ring, counters = cache.new_ring()
    rows, spans = torch.full((S,), n, **INTS).cuda(), torch.zeros(S, 2, **INTS).cuda()
    parents, paths, counts = torch.full((S, n), -1, **INTS).cuda(), torch.zeros(S, 1, **INTS).cuda(), torch.ones(S, **INTS).cuda()
    gen = torch.Generator().manual_seed(3)
    k, v, q = (rows_of(gen, S * n, h, 128, BF16, False).view(S, n, h, 128).cuda() for h in (H, H, H * G))

    def step():
        p = cache.plan(table, lengths, rows, spans, ring, counters, S * n, window=20, sinks=2)
        cache.append_kv(table, p.lengths, k, v)
        masks, _ = cache.tree_masks(parents, p.lengths, window=20, sinks=2)
        return (cache.attention(table, p.lengths, q, tree=masks, window=20, sinks=2), cache.attention(table, p.lengths, q, window=2),
                cache.keep_rows(table, p.lengths, paths, counts, n))

    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        outs = step()
    g.replay()
    torch.cuda.synchronize()
    assert outs[2].tolist() == [1, 1]
    for s in range(S):
        K, V = quantised(k[s].cpu(), 32), quantised(v[s].cpu(), 32)
        for out, see in ((outs[0], torch.eye(n, dtype=torch.bool)), (outs[1], window_seen(n, n, 2, 0))):
            ref, _, tol = attention_seen(q[s].cpu(), K, V, see, 1 / math.sqrt(128), BF16)
            check(out[s], ref, tol)
    assert cache.stats() == {"device_timeouts": 0, "bad_pages": 0, "bad_lengths": 0}


@pytest.mark.gpu
def test_in_a_process_whose_first_calls_are_captured():
    import os
    import subprocess
    import sys
    here = os.path.dirname(os.path.abspath(__file__))
    r = subprocess.run([sys.executable, "-c", "import test_q4_serve as t; t.captured_first()"], capture_output=True, text=True, timeout=600, cwd=here,
                       env={**os.environ, "PYTHONPATH": os.pathsep.join([os.path.dirname(here), here])})
    assert r.returncode == 0, (r.stdout + r.stderr)[-3000:]


@pytest.mark.gpu
def test_in_a_process_without_caches_that_overlap():
    """Kernels are launched differently there (other test files make a page cache whose decodes do not wait): the tests of calls that follow one
    another, by themselves."""
    import subprocess
    import sys
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-m", "gpu", "-k", "every_kernel or serving or captured or same_bits or random or planned or kept", "-p", "no:cacheprovider", __file__],
                       capture_output=True, text=True, timeout=900)
    assert r.returncode == 0, r.stdout[-3000:]
