"""Serving from the 4-bit cache at its limits: rows that leave a warp in part, arrays that lie on top of one another, more CTAs than 16 bits count,
numbers that are none, bindings that were not built."""
import ctypes

import pytest
import torch

from paper_2608_23843_b200 import pkv
from q4_select_reference import attention_seen, window_seen
from test_q4_cache import BF16, FP16, INTS, Filled, check, config
from test_q4_serve import _dry, offsets_of, seen_by

LONGS = dict(dtype=torch.int64)


def refused(call):
    with pytest.raises(pkv.PkvError) as e:
        call()
    assert e.value.status == pkv.PKV_ERR_INVALID_ARG and str(e.value)
    return str(e.value)


# ---- arrays on top of one another ----------------------------------------------------------------------------------------
def test_kept_lengths_must_not_lie_on_what_is_read():
    """The CTAs of all KV heads read counts, paths, offsets and tables; one of them writes the lengths."""
    c, t, n, _ = _dry()
    counts, paths, off = torch.ones_like(n), torch.zeros(3, 2, **INTS), offsets_of([2, 2, 2])
    for name, out in (("counts", counts), ("paths", paths.flatten()[:3]), ("paths", paths.flatten()[3:]), ("page_table", t[1, 1:]), ("lengths", n)):
        assert name in refused(lambda: c.keep_rows(t, n, paths, counts, 2, out=out))
    for at in (0, 1):
        assert "offsets" in refused(lambda: c.keep_rows(t, n, paths, counts, 6, offsets=off, out=off[at:at + 3]))
    around = torch.zeros(9, **INTS)                        # side by side is fine
    assert c.keep_rows(t, around[3:6], paths, around[6:], 2, out=around[:3]).data_ptr() == around.data_ptr()
    keep = lambda **k: pkv.lib().pkv_q4_keep_rows(*{**dict(h=c.handle, S=3, t=0, mp=4, n=0, rows=6, off=0, path=0, m=2, cnt=0, out=256, st=0), **k}.values())  # noqa: E731
    assert keep(cnt=244) == keep(cnt=268) == keep(path=232) == keep(off=240) == keep(t=208) == pkv.PKV_OK
    for k in (dict(cnt=248), dict(cnt=264), dict(path=236), dict(path=264), dict(off=244), dict(off=264), dict(t=212), dict(t=264), dict(n=256), dict(n=248)):
        assert keep(**k) == pkv.PKV_ERR_INVALID_ARG, k


def test_what_a_plan_writes_must_not_lie_on_other_arrays():
    """Only lengths, spans and counters may be written in place, as whole arrays."""
    c, t, n, _ = _dry()
    spans, (ring, counters) = torch.zeros(3, 2, **INTS), c.new_ring()
    rows = torch.ones_like(n)
    plan = lambda out, n_rows=4: c.plan(t, n, rows, spans, ring, counters, n_rows, out=out)      # noqa: E731
    out = plan(None)
    plan(out._replace(lengths=n, spans=spans, counters=counters))
    both = torch.zeros(6, **INTS)
    longs = torch.zeros(8, **LONGS)
    for bad in (dict(lengths=rows), dict(lengths=spans.flatten()[1:4]), dict(spans=t.flatten()[:6].view(3, 2)),
                dict(offsets=t[1]), dict(offsets=ring[:4]), dict(offsets=ring[12:]), dict(positions=ring[3:7]), dict(positions=t[2]),
                dict(lengths=both[:3], spans=both.view(3, 2)), dict(positions=out.offsets), dict(slots=counters), dict(counters=longs[1:5], slots=longs[4:])):
        refused(lambda: plan(out._replace(**bad)))
    lengths = torch.zeros(4, **INTS)                       # neither in place nor apart
    refused(lambda: c.plan(t, lengths[:3], rows, spans, ring, counters, 4, out=out._replace(lengths=lengths[1:])))
    plan = lambda **k: pkv.lib().pkv_q4_plan(*{**dict(h=c.handle, S=3, t=0, mp=4, n=0, r=0, sp=0, ring=0, cnt=0, W=0, sinks=0, no=0, so=0, co=0, off=0, rows=6, pos=0,      # noqa: E731
                                                      slot=0, work=0, wb=0, st=0), **k}.values())
    assert plan(n=256, no=256, sp=512, so=512, cnt=768, co=768) == pkv.PKV_OK
    assert plan(S=2000, work=4096, wb=1 << 20) == pkv.PKV_OK
    assert plan(S=2000, work=4096, wb=1 << 20, slot=4096 + 64) == pkv.PKV_ERR_INVALID_ARG


def test_masks_must_not_lie_on_what_is_read_or_written_with_them():
    """CTAs read the parents of rows that others write masks and depths of; an attention call's heads read the masks one after another."""
    c, t, n, q = _dry()
    L, bad = pkv.lib(), pkv.PKV_ERR_INVALID_ARG
    masks = lambda **k: L.pkv_q4_tree_masks(*{**dict(h=c.handle, S=3, n=0, rows=6, off=0, most=2, par=0, W=4, sinks=2, tree=0, words=2, dep=0, st=0), **k}.values())  # noqa: E731
    assert masks(tree=1024, dep=1120, par=1000) == masks(dep=256, par=280) == masks(tree=1024, n=1012, off=1120) == pkv.PKV_OK
    assert masks(tree=1024, n=1024, W=0, sinks=0) == pkv.PKV_OK                         # (not looked at)
    for k in (dict(tree=1024, dep=1116), dict(tree=1024, par=1004), dict(dep=256, par=256), dict(dep=256, par=276), dict(tree=1024, n=1016), dict(dep=256, off=244), dict(dep=256, n=276)):
        assert masks(**k) == bad, k
    words = torch.zeros(3, 2, 1, **LONGS)
    c.attention(t, n, q, tree=words)
    state = torch.zeros(3 * 2 * 8 * 130 + 12)
    tail = state[-12:].view(torch.int64).view(3, 2, 1)
    assert c.attention_partial(t, n, q, state=state[:-12].view(3, 2, 8, 130), tree=tail).shape == (3, 2, 8, 130)
    assert "state" in refused(lambda: c.attention_partial(t, n, q, state=state[:-12].view(3, 2, 8, 130), tree=state[-14:-2].view(torch.int64).view(3, 2, 1)))
    out = torch.zeros(6 * 1024 + 32, dtype=q.dtype)
    assert out.data_ptr() % 16 == 0
    there = out[:6144].view(3, 2, 8, 128)
    assert c.attention(t, n, q, out=there, tree=out[6144:6168].view(torch.int64).view(3, 2, 1)) is there
    assert "out" in refused(lambda: c.attention(t, n, q, out=there, tree=out[6140:6164].view(torch.int64).view(3, 2, 1)))
    room = ctypes.c_int64()                                # a call that joins states needs a workspace
    sel = pkv.PkvQ4Select(0, 0, 1 << 30, 1)
    assert L.pkv_q4_attention_select_workspace(c.handle, 1, 64, 60000, ctypes.byref(sel), ctypes.byref(room)) == pkv.PKV_OK and room.value > 0
    call = lambda work: L.pkv_q4_attention_select(c.handle, 1, 0, 1000, 0, 64, 0, 64, 60000, ctypes.byref(sel), 0, 1024, 128, 0, 1024, 128, 0, work, room.value, 0)      # noqa: E731
    assert call((1 << 30) + 64 * 8) == call(0) == pkv.PKV_OK
    assert call((1 << 30) + 63 * 8) == call((1 << 30) - room.value + 8) == bad


# ---- how many CTAs a call may take -----------------------------------------------------------------------------------------
@pytest.mark.parametrize("n_ctas", [1, 2, 3, 7, 20, 148, 296, 1000, 65535])
def test_a_call_takes_no_more_ctas_than_configured(n_ctas):
    """Half as many of twice the size for sixteen rows, twice as many of half the size for short segments; a CTA per SM for row blocks."""
    cache = pkv.Q4Cache(config(n_kv_heads=4, n_q_heads=16, n_ctas=n_ctas), dry_run=True)
    kernels = set()
    for S in (1, 3, 64, 700):
        for n in (1, 2, 3, 4, 9, 70):
            for T in (64, 1000, 30000):
                for kw in (dict(), dict(window=40), dict(window=900, sinks=100), dict(tree=True, tree_words=2), dict(window=20000)):
                    kernel, n_cta, cluster = pkv.pkv_q4_attention_route(cache.handle, S, n, T, **kw)
                    most = {0: n_ctas if n * 4 <= 8 else max(1, n_ctas // 2), 1: 148, 2: 2 * n_ctas}[kernel]
                    assert 1 <= n_cta <= most and n_cta % cluster == 0, (S, n, T, kw)
                    kernels.add(kernel)
    assert kernels >= {0, 1, 2} or n_ctas < 20


# ---- numbers that are none -----------------------------------------------------------------------------------------------
def test_none_is_no_number():
    """None may stand for a pointer; as a number it would arrive as 0, and rows would be kept of none."""
    c, t, n, _ = _dry()
    off = offsets_of([2, 2, 2])
    refused(lambda: c.keep_rows(t, n, torch.zeros(3, 2, **INTS), n, None, offsets=off))
    h = c.handle.value
    kinds = dict(append_kv="pipiplppllpllp", attention="pipiplpiipllpllpplp", attention_select="pipiplpiipllpllpplpiipi", tree_masks="piplpipiipipp",
                 keep_rows="pipiplppippp", plan="pipipppppiipppplppplp")
    good = dict(append_kv=(h, 3, 0, 4, 0, 6, 0, 0, 256, 128, 0, 256, 128, 0), attention=(h, 3, 0, 4, 0, 6, 0, 2, 0, 0, 1024, 128, 0, 1024, 128, 0, 0, 0, 0),
                attention_select=(h, 3, 0, 4, 0, 6, 0, 2, 0, 0, 1024, 128, 0, 1024, 128, 0, 0, 0, 0, 9, 4, 0, 0),
                tree_masks=(h, 3, 0, 6, 0, 2, 0, 0, 0, 0, 1, 0, 0), keep_rows=(h, 3, 0, 4, 0, 6, 0, 0, 2, 0, 0, 0), plan=(h, 3, 0, 4) + (0,) * 11 + (6,) + (0,) * 5)
    kinds["read_kv"], good["read_kv"] = kinds["append_kv"], good["append_kv"]
    for name, args in good.items():
        fn = getattr(pkv._calls(), name)
        assert len(args) == len(kinds[name]) and fn(*args) == pkv.PKV_OK, name
        for i, kind in enumerate(kinds[name]):
            with_none = args[:i] + (None,) + args[i + 1:]
            if kind == "p":
                assert fn(*with_none) == (pkv.PKV_OK if i else pkv.PKV_ERR_INVALID_ARG), (name, i)
            else:
                with pytest.raises(TypeError):
                    fn(*with_none)


def test_pages_of_a_ring_are_whole_numbers_below_the_pools():
    c = _dry()[0]
    for pages in ([0.5, 1.7], [1.0, 2.0], [True, False], torch.tensor([2 ** 32 + 4]), [2 ** 32 + 4], torch.tensor([-2 ** 32 + 4]), [-1], [16], [3, 3]):
        assert "page numbers" in refused(lambda: c.new_ring(pages))
    for pages in ([7, 3], torch.tensor([7, 3]), torch.tensor([[7], [3]], dtype=torch.int16), torch.tensor([7, 3], dtype=torch.uint8), torch.tensor([7, 3], dtype=torch.uint32)):
        ring, counters = c.new_ring(pages)
        assert ring.tolist() == [7, 3] + [-1] * 14 and counters.tolist() == [0, 2, 0, 0] and ring.dtype == torch.int32
    for pages in ([], torch.empty(0)):
        assert c.new_ring(pages)[1].tolist() == [0, 0, 0, 0]


def test_sizes_are_refused_before_anything_is_allocated_by_them():
    """... and as other arguments are, not by the allocator or by a comparison."""
    c, t, n, q = _dry()
    off, parents, spans = offsets_of([2, 2, 2]), torch.full((6,), -1, **INTS), torch.zeros(3, 2, **INTS)
    for most in (7, 2 ** 50, -1, 2.0, "2"):
        assert "max_q_len" in refused(lambda: c.tree_masks(parents, n, off, max_q_len=most))
    for n_rows in (-1, 2 ** 30, 2 ** 50, 2.0, None):
        assert "n_rows" in refused(lambda: c.plan(t, n, n, spans, *c.new_ring(), n_rows))
    for _ in range(2):
        for bad in (dict(window=4.0), dict(window="4"), dict(window=4, sinks=2.5), dict(window=4, sinks=None), dict(window=None, sinks=3)):
            for call in (lambda: c.attention(t, n, q, **bad), lambda: c.tree_masks(parents, n, off, **bad), lambda: c.plan(t, n, n, spans, *c.new_ring(), 4, **bad)):
                assert "whole number" in refused(call)
        c.attention(t, n, q, window=4, sinks=2)
    import numpy
    assert c.tree_masks(parents, n, off, max_q_len=numpy.int64(2), window=numpy.int32(4))[0].shape == (6, 1)
    assert c.attention(t, n, q, window=numpy.int64(4), sinks=numpy.int16(1)).shape == q.shape
    assert c.plan(t, n, n, spans, *c.new_ring(), numpy.int64(5)).slots.shape == (5,)


# ---- bindings that were not built ----------------------------------------------------------------------------------------
def test_the_binding_is_named_for_its_interpreter(tmp_path, monkeypatch):
    """... so that another one does not load it; without a C compiler or Python's headers the library is built all the same."""
    import os
    import sysconfig
    from paper_2608_23843_b200 import build
    assert build.CALL.endswith("_pkvcall" + sysconfig.get_config_var("EXT_SUFFIX")) and os.path.basename(build.CALL) != "_pkvcall.so"
    call = str(tmp_path / os.path.basename(build.CALL))
    monkeypatch.setattr(build, "CALL", call)
    assert build.build_call() == call and os.path.exists(call)
    for name, value in (("CC", "false"), ("CC", str(tmp_path / "no compiler"))):
        monkeypatch.setenv(name, value)
        with pytest.warns(UserWarning, match="ctypes"):
            assert build.build_call(force=True) is None
        assert not os.path.exists(call) and os.listdir(tmp_path) == []
    monkeypatch.setattr(pkv, "_calls_module", None)
    assert isinstance(pkv._calls(), pkv._CtypesCalls)
    c, t, n, q = _dry()
    assert c.attention(t, n, q, window=5, sinks=1).shape == q.shape and c.keep_rows(t, n, torch.zeros(3, 2, **INTS), n, 2).shape == (3,)
    refused(lambda: c.keep_rows(t, n, torch.zeros(3, 2, **INTS), n, 2, out=n))
    refused(lambda: c.keep_rows(t, n, torch.zeros(3, 2, **INTS), n, 2.0))


def test_the_binding_is_passed_over_for_another_library(tmp_path, monkeypatch):
    """(it would bring the one that it was linked with beside it)"""
    import os
    from paper_2608_23843_b200 import build
    other = tmp_path / "libpkv.so"
    os.symlink(build.LIB, other)
    monkeypatch.setattr(pkv, "_calls_module", None)
    monkeypatch.setattr(pkv, "LIB_PATH", str(other))
    assert not isinstance(pkv._calls(), pkv._CtypesCalls)                  # the same file
    other.unlink()
    other.write_bytes(b"")
    monkeypatch.setattr(pkv, "_calls_module", None)
    assert isinstance(pkv._calls(), pkv._CtypesCalls)
    monkeypatch.setattr(build, "LIB", str(tmp_path / "none"))              # no library in the tree
    monkeypatch.setattr(pkv, "_calls_module", None)
    assert isinstance(pkv._calls(), pkv._CtypesCalls)


def test_calls_through_ctypes_check_their_numbers():
    c, t, n, q = _dry()
    h = c.handle.value
    good = dict(append_kv=(h, 3, 0, 4, 0, 6, 0, 0, 256, 128, 0, 256, 128, 0), attention=(h, 3, 0, 4, 0, 6, 0, 2, 0, 0, 1024, 128, 0, 1024, 128, 0, 0, 0, 0),
                attention_select=(h, 3, 0, 4, 0, 6, 0, 2, 0, 0, 1024, 128, 0, 1024, 128, 0, 0, 0, 0, 9, 4, None, 0),
                tree_masks=(h, 3, None, 6, None, 2, 0, 0, 0, 0, 1, 0, 0), keep_rows=(h, 3, 0, 4, 0, 6, 0, 0, 2, 0, 0, 0), plan=(h, 3, 0, 4) + (0,) * 11 + (6,) + (0,) * 5)
    good["read_kv"] = good["append_kv"]
    assert sorted(good) == sorted(pkv._CALLS)
    for name, args in good.items():
        fn = getattr(pkv._CtypesCalls(), name)
        assert fn(*args) == pkv.PKV_OK and fn(None, *args[1:]) == pkv.PKV_ERR_INVALID_ARG, name
        for bad in (args[:-1], (h, 3.0, *args[2:]), (h, None, *args[2:])):
            with pytest.raises(TypeError):
                fn(*bad)
        for wrong in (1 << 31, -(1 << 31) - 1, 1 << 64):
            with pytest.raises(OverflowError):
                fn(h, wrong, *args[2:])


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 5])
def test_calls_through_ctypes_do_the_same(n, monkeypatch):
    results = []
    for through in (pkv._calls(), pkv._CtypesCalls()):
        monkeypatch.setattr(pkv, "_calls_module", through)
        f = Filled([300, 90, 700], seed=3)
        ns = [n] * 3
        q = torch.stack(f.queries(ns)).cuda()
        parents = torch.tensor([[j - 1 - j % 2 for j in range(n)]] * 3, **INTS).cuda()
        masks, depths = f.cache.tree_masks(parents, f.lengths, window=200, sinks=5)
        got = [masks, depths, f.cache.attention(f.table, f.lengths, q), f.cache.attention(f.table, f.lengths, q, window=100, sinks=4),
               f.cache.attention_partial(f.table, f.lengths, q, window=200, sinks=5, tree=masks)]
        kept = f.cache.keep_rows(f.table, f.lengths, torch.tensor([[n - 1]] * 3, **INTS).cuda(), torch.ones(3, **INTS).cuda(), n)
        got += [kept, *f.cache.read_kv(f.table, kept, *(torch.empty(3, 9, f.H, f.d, dtype=f.dtype, device="cuda") for _ in "kv"))]
        spans = torch.stack([torch.zeros_like(kept), (kept + 63) // 64], 1).to(torch.int32)
        ring, counters = f.cache.new_ring([0, 1, 2, 3])
        got += [*f.cache.plan(f.table, kept, torch.ones_like(kept), spans, ring, counters, 3), f.table, ring]
        results.append(got)
        f.clean()
    assert all(torch.equal(a, b) for a, b in zip(*results))


@pytest.mark.gpu
def test_the_functions_of_the_binding_do_what_the_cache_does():
    f = Filled([300, 90, 700], seed=4)
    c, n, S, W, sinks = f.cache, 5, 3, 100, 4
    h, (_, max_pages) = c.handle, f.table.shape
    q = torch.stack(f.queries([n] * S)).cuda()
    parents = torch.tensor([[-1, 0, 0, 1, 3]] * S, **INTS).cuda()
    masks, depths = c.tree_masks(parents, f.lengths, window=W, sinks=sinks)
    masks2, depths2 = torch.empty_like(masks), torch.empty_like(depths)
    pkv.pkv_q4_tree_masks(h, S, f.lengths, S * n, None, n, parents, W, sinks, masks2, 1, depths2)
    assert torch.equal(masks, masks2) and torch.equal(depths, depths2)
    size = pkv.pkv_q4_attention_select_workspace(h, S, n, max_pages * 64, W, sinks, masks, 1)
    work = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")
    strides, out = (q.stride(1), q.stride(2)), torch.empty_like(q)
    pkv.pkv_q4_attention_select(h, S, f.table, max_pages, f.lengths, S * n, None, n, max_pages * 64, W, sinks, masks, 1, q, strides, out, strides, None, work, size)
    assert torch.equal(out, c.attention(f.table, f.lengths, q, window=W, sinks=sinks, tree=masks))
    paths, counts = torch.tensor([[0, 1, 3]] * S, **INTS).cuda(), torch.tensor([3, 1, 0], **INTS).cuda()
    pool, kept = c.pool.clone(), torch.empty_like(f.lengths)
    pkv.pkv_q4_keep_rows(h, S, f.table, max_pages, f.lengths, S * n, None, paths, 3, counts, kept)
    moved = c.pool.clone()
    c.pool.copy_(pool)
    kept2 = c.keep_rows(f.table, f.lengths, paths, counts, n)
    assert torch.equal(kept, kept2) and torch.equal(moved, c.pool) and kept.tolist() == [298, 86, 695]
    for last in (30, 5):                                   # 695 + 30 rows are more than the table takes: nothing is done
        results = []
        for by_hand in (True, False):
            table, (ring, counters) = f.table.clone(), c.new_ring([1, 0, 2, 3])
            spans = torch.stack([torch.zeros_like(kept), (kept + 63) // 64], 1).to(torch.int32)
            rows = torch.tensor([1, -1, last], **INTS).cuda()
            p = pkv.Q4Plan(*(torch.full_like(x, 7) for x in (kept, torch.empty(S + 1, **INTS).cuda(), torch.empty(31, **INTS).cuda(), torch.empty(31, **LONGS).cuda(), spans, counters)))
            if by_hand:
                assert pkv.pkv_q4_plan_workspace(h, S, 31) == 0
                pkv.pkv_q4_plan(h, S, table, max_pages, kept, rows, spans, ring, counters, W, sinks, p.lengths, p.spans, p.counters, p.offsets, 31, p.positions, p.slots, None, 0)
            else:
                assert c.plan(table, kept, rows, spans, ring, counters, 31, window=W, sinks=sinks, out=p) is p
            results.append([*p, table, ring])
        assert all(torch.equal(a, b) for a, b in zip(*results))
        assert p.counters[3] == (last == 30) and p.lengths.tolist() == ([299, 0, 700] if last == 5 else kept.tolist())
    f.clean()


# ---- refusals that must not depend on what was called before -------------------------------------------------------------
@pytest.mark.parametrize("before", [False, True])
@pytest.mark.parametrize("kw", [dict(), dict(window=5), dict(window=5, sinks=2)])
def test_masks_without_words_are_refused_whatever_was_called_before(before, kw):
    """(their data pointer is NULL, which would make the call a causal one)"""
    c, t, n, q = _dry()
    if before:
        c.attention(t, n, q, **kw)
    for call in (c.attention, c.attention_partial):
        assert "tree" in refused(lambda: call(t, n, q, tree=torch.zeros(3, 2, 0, **LONGS), **kw))
        assert "tree" in refused(lambda: call(t, n, q[:, :0], tree=torch.zeros(3, 0, 0, **LONGS), **kw))


def test_empty_arrays_and_gaps_overlap_nothing():
    c, t, n, q = _dry()
    L, h = pkv.lib(), c.handle
    assert L.pkv_q4_keep_rows(h, 3, 0, 4, 0, 6, 0, 260, 0, 0, 256, 0) == pkv.PKV_OK                            # no paths
    assert L.pkv_q4_tree_masks(h, 3, 0, 0, 260, 0, 264, 0, 0, 256, 1, 264, 0) == pkv.PKV_OK                    # no rows
    plan = [h, 3, 256, 4, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 260, 264, 0, 0, 0]
    assert L.pkv_q4_plan(*plan) == pkv.PKV_OK
    plan[15] = 1
    assert L.pkv_q4_plan(*plan) == pkv.PKV_ERR_INVALID_ARG
    row = torch.zeros(1, 1, 8, 136, dtype=BF16)             # masks beside a head's channels
    masks = row.flatten()[128:132].view(torch.int64).view(1, 1, 1)
    assert c.attention(t[:1], n[:1], q[:1, :1], out=row[..., :128], tree=masks).shape == (1, 1, 8, 128)


# ---- clusters whose joins leave a warp in part ---------------------------------------------------------------------------
# A segment's states are rows * d / 4 pieces for 96 threads, and rows * d / 4 / cluster for each CTA of a cluster: these end inside a warp.
@pytest.mark.gpu
@pytest.mark.parametrize("dtype, d, g", [(BF16, 128, 32), (FP16, 64, 32), (BF16, 64, 64)])
@pytest.mark.parametrize("G", [1, 3, 5, 7])
@pytest.mark.parametrize("S, T, W, n_ctas, cluster", [(20, 300, 200, 20, 1), (8, 700, 300, 20, 2), (2, 1500, 1400, 8, 4), (2, 1500, 1400, 0, 8)])
def test_clusters_join_any_number_of_rows(dtype, d, g, G, S, T, W, n_ctas, cluster):
    f = Filled([T - 50 * s % T for s in range(S)], seed=G, dtype=dtype, d=d, g=g, H=2, G=G, n_ctas=n_ctas)
    assert pkv.pkv_q4_attention_route(f.cache.handle, S, 1, f.table.shape[1] * 64, W, 3)[::2] == (2, cluster)
    qs = f.queries([1] * S)
    q = torch.stack(qs).cuda()
    out = f.cache.attention(f.table, f.lengths, q, window=W, sinks=3).cpu()
    state = f.cache.attention_partial(f.table, f.lengths, q, window=W, sinks=3).to("cpu", torch.float64)
    for s in range(S):
        ref, _, tol = seen_by(f, qs[s], s, window_seen(f.lens[s], 1, W, 3))
        check(out[s], ref, tol)
        check(state[s][..., :d] / state[s][..., d + 1:], ref, tol)
    f.clean()


# ---- more CTAs than 16 bits count ----------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("S, H, n_ctas", [(50000, 3, 40000), (65535, 3, 65535), (65535, 2, 65535)])
def test_windows_on_more_ctas_than_16_bits_count(S, H, n_ctas):
    """Segments that do not divide among the CTAs, on grids beyond 65536: each is worked on once, none is left out.  All sequences
    read the same page, and every 320 the same positions with the same queries."""
    f = Filled([64], H=H, G=1, n_ctas=n_ctas)
    kernel, grid, cluster = pkv.pkv_q4_attention_route(f.cache.handle, S, 1, 64, 40, 2)
    assert kernel == 2 and cluster == 1 and grid == min(2 * n_ctas, S * H) and grid > 65536
    qs = f.queries([1] * 5)
    lens = [1 + s % 64 for s in range(320)]
    repeat = lambda x: x.repeat(-(-S // 320), *[1] * (x.dim() - 1))[:S].contiguous().cuda()      # noqa: E731
    q = repeat(torch.stack([qs[s % 5] for s in range(320)]))
    out = torch.full_like(q, 5.0)
    f.cache.attention(f.table[:1].expand(S, -1).contiguous(), repeat(torch.tensor(lens, **INTS)), q, out=out, window=40, sinks=2)
    out = out.cpu()
    for s in range(320):
        T = lens[s]
        ref, _, tol = attention_seen(qs[s % 5], f.K[0][:T], f.V[0][:T], window_seen(T, 1, 40, 2), 128 ** -0.5, BF16)
        check(out[s], ref, tol)
    assert torch.equal(out, out[:320].repeat(-(-S // 320), 1, 1, 1)[:S])
    f.clean()
