"""The paged cache held in 4 bits: sizes and refusals on the CPU; writer, reader and attention against the definition in
64 bits on the GPU."""
import itertools
import math

import pytest
import torch

from paper_2608_23843_b200 import pkv
from q4_reference import SCALE_MOST, Rows, attention, offsets_of, quantised

BF16, FP16 = torch.bfloat16, torch.float16
INTS = dict(dtype=torch.int32)


def config(**kw):
    base = dict(n_kv_heads=2, n_q_heads=8, n_pages=16)
    base.update(kw)
    return pkv.make_q4_config(**base)


# ---- CPU: sizes, refusals --------------------------------------------------------------------------------------------
@pytest.mark.parametrize("d, g, P, H, token_bytes", [(128, 32, 64, 8, 144), (128, 64, 16, 2, 136), (128, 128, 256, 1, 132),
                                                     (64, 32, 32, 4, 72), (64, 64, 128, 3, 68)])
def test_sizes(d, g, P, H, token_bytes):
    s = pkv.pkv_q4_query_sizes(config(n_kv_heads=H, n_q_heads=2 * H, head_dim=d, group_size=g, page_size=P, n_pages=11))
    assert s.page_bytes == H * P * token_bytes and s.pool_bytes == 11 * s.page_bytes and s.meta_bytes >= 32


@pytest.mark.parametrize("change, status", [
    (dict(head_dim=96), pkv.PKV_ERR_UNSUPPORTED), (dict(head_dim=256), pkv.PKV_ERR_UNSUPPORTED),
    (dict(group_size=16), pkv.PKV_ERR_UNSUPPORTED), (dict(head_dim=64, group_size=128), pkv.PKV_ERR_UNSUPPORTED),
    (dict(page_size=8), pkv.PKV_ERR_UNSUPPORTED), (dict(page_size=48), pkv.PKV_ERR_UNSUPPORTED),
    (dict(page_size=512), pkv.PKV_ERR_UNSUPPORTED), (dict(n_q_heads=130), pkv.PKV_ERR_UNSUPPORTED),
    (dict(n_q_heads=7), pkv.PKV_ERR_INVALID_ARG), (dict(n_kv_heads=0), pkv.PKV_ERR_INVALID_ARG),
    (dict(n_pages=0), pkv.PKV_ERR_INVALID_ARG), (dict(n_pages=1 << 31), pkv.PKV_ERR_UNSUPPORTED),
    (dict(softmax_scale=math.inf), pkv.PKV_ERR_INVALID_ARG), (dict(softmax_scale=math.nan), pkv.PKV_ERR_INVALID_ARG),
    (dict(softmax_scale=-1.0), pkv.PKV_ERR_INVALID_ARG), (dict(softmax_scale=3e38), pkv.PKV_ERR_INVALID_ARG), (dict(n_ctas=-1), pkv.PKV_ERR_INVALID_ARG)])
def test_configurations_that_are_refused(change, status):
    with pytest.raises(pkv.PkvError) as e:
        pkv.Q4Cache(config(**change), dry_run=True)
    assert e.value.status == status


def test_a_type_that_is_refused():
    with pytest.raises(pkv.PkvError):
        config(dtype=torch.float32)


def _dry():
    cache = pkv.Q4Cache(config(), dry_run=True)
    table, lengths = torch.zeros(3, 4, **INTS), torch.zeros(3, **INTS)
    return cache, table, lengths, torch.zeros(3, 2, 2, 128, dtype=BF16), torch.zeros(3, 2, 8, 128, dtype=BF16)


def test_calls_that_are_accepted_in_a_dry_run():
    cache, table, lengths, k, q = _dry()
    fused = torch.zeros(6, 12, 128, dtype=BF16)
    off = offsets_of([0, 5, 1])
    cache.append_kv(table, lengths, k, k)
    cache.append_kv(table, lengths, fused[:, 8:10], fused[:, 10:], off)
    cache.read_kv(table, lengths, k, k)
    assert cache.attention(table, lengths, q).shape == q.shape
    assert cache.attention(table, lengths, fused[:, :8], offsets=off, max_q_len=5).shape == (6, 8, 128)
    assert cache.attention_partial(table, lengths, q).shape == (3, 2, 8, 130)
    cache.append_kv(table, lengths, k[:, :0], k[:, :0])                       # no rows
    cache.attention(table, lengths, q[:, :0])
    cache.append_kv(table, lengths, torch.zeros(2, 3, 2, 128, dtype=BF16).permute(1, 2, 0, 3), k)      # heads first
    cache.append_kv(table, lengths, k[..., :1, :].expand(3, 2, 2, 128).contiguous(), k)
    assert cache.stats() == {"device_timeouts": 0, "bad_pages": 0, "bad_lengths": 0}


@pytest.mark.parametrize("call", [
    lambda c, t, n, k, q: c.append_kv(t.long(), n, k, k),                               # types
    lambda c, t, n, k, q: c.append_kv(t, n.long(), k, k),
    lambda c, t, n, k, q: c.append_kv(t, n, k.half(), k),
    lambda c, t, n, k, q: c.append_kv(t, n, k, k.float()),
    lambda c, t, n, k, q: c.append_kv(t[0], n, k, k),                                   # shapes
    lambda c, t, n, k, q: c.append_kv(t, n[:2], k, k),
    lambda c, t, n, k, q: c.append_kv(t, n, k[:2], k[:2]),
    lambda c, t, n, k, q: c.append_kv(t, n, k[:, :, :1], k[:, :, :1]),
    lambda c, t, n, k, q: c.append_kv(t, n, k[..., :64], k[..., :64]),
    lambda c, t, n, k, q: c.append_kv(t, n, k, k[:, :1]),
    lambda c, t, n, k, q: c.append_kv(t, n, k, k, offsets_of([2, 2, 2])),               # [n_seqs, n, ...] with offsets
    lambda c, t, n, k, q: c.append_kv(t, n, k.flatten(0, 1), k.flatten(0, 1)),          # [rows, ...] without
    lambda c, t, n, k, q: c.append_kv(t, n, k.flatten(0, 1), k.flatten(0, 1), offsets_of([3, 3])),
    lambda c, t, n, k, q: c.append_kv(t.T.contiguous().T, n, k, k),                     # strides
    lambda c, t, n, k, q: c.append_kv(t, n, k.transpose(2, 3).contiguous().transpose(2, 3), k),
    lambda c, t, n, k, q: c.append_kv(t, n, torch.zeros(3, 3, 2, 128, dtype=BF16)[:, :2], k),      # unequal steps between rows
    lambda c, t, n, k, q: c.append_kv(t, n, torch.zeros(3, 2, 2, 132, dtype=BF16)[..., :128], k),  # heads off 16-byte steps
    lambda c, t, n, k, q: c.append_kv(t, n, torch.zeros(3 * 2 * 2 * 128 + 8, dtype=BF16)[1:-7].view(3, 2, 2, 128), k),
    lambda c, t, n, k, q: c.append_kv(t, n, k[:, :, :1].expand(3, 2, 2, 128), k),       # heads on top of one another
    lambda c, t, n, k, q: c.append_kv(t, n, k[:1, :1].expand(3, 2, 2, 128), k),         # rows on top of one another
    lambda c, t, n, k, q: c.append_kv(t, n, torch.zeros(2000, dtype=BF16).as_strided((3, 2, 2, 128), (256, 128, 128, 1)), k),      # head 1 on row 1
    lambda c, t, n, k, q: c.read_kv(t, n, k, k.half()),
    lambda c, t, n, k, q: c.attention(t, n, k),
    lambda c, t, n, k, q: c.attention(t, n, q.half()),
    lambda c, t, n, k, q: c.attention(t, n, q, out=torch.zeros(3, 2, 8, 64, dtype=BF16)),
    lambda c, t, n, k, q: c.attention(t, n, q, out=torch.zeros(3, 2, 8, 128)),
    lambda c, t, n, k, q: c.attention(t, n, q.flatten(0, 1), offsets=offsets_of([2, 2, 2]), max_q_len=-1),
    lambda c, t, n, k, q: c.attention(t, n, q.flatten(0, 1), offsets=offsets_of([2, 2, 2]), max_q_len=7),
    lambda c, t, n, k, q: c.attention_partial(t, n, q, state=torch.zeros(3, 2, 8, 128)),
    lambda c, t, n, k, q: c.attention_partial(t, n, q, state=torch.zeros(3, 2, 8, 130, dtype=BF16)),
    lambda c, t, n, k, q: c.append_kv(t[:0], n[:0], k[:0], k[:0]),                      # no sequences
    lambda c, t, n, k, q: c.append_kv(t[:, :0], n, k, k),                               # no pages
])
def test_calls_that_are_refused(call):
    with pytest.raises(pkv.PkvError) as e:
        call(*_dry())
    assert e.value.status == pkv.PKV_ERR_INVALID_ARG and str(e.value)


def test_refusals_of_the_c_entry_points():
    cache, table, lengths, k, q = _dry()
    h, L = cache.handle, pkv.lib()
    s = (256, 128)
    kp = k.data_ptr()
    for args in [(h, 0, 0, 4, 0, 6, 0, kp, *s, kp, *s, 0),                    # no sequences
                 (h, 70000, 0, 4, 0, 70000, 0, kp, *s, kp, *s, 0),
                 (h, 3, 0, 0, 0, 6, 0, kp, *s, kp, *s, 0),                    # no pages
                 (h, 3, 0, 1 << 28, 0, 6, 0, kp, *s, kp, *s, 0),              # more positions than 31 bits
                 (h, 3, 0, 4, 0, -1, 0, kp, *s, kp, *s, 0),
                 (h, 3, 0, 4, 0, 7, 0, kp, *s, kp, *s, 0),                    # 7 rows, 3 sequences
                 (h, 3, 0, 4, 0, 1 << 40, 4, kp, *s, kp, *s, 0),
                 (h, 3, 2, 4, 0, 6, 0, kp, *s, kp, *s, 0),                    # misaligned table
                 (h, 3, 0, 4, 0, 6, 0, kp + 2, *s, kp, *s, 0),
                 (h, 3, 0, 4, 0, 6, 0, kp, -256, 128, kp, *s, 0),
                 (h, 3, 0, 4, 0, 6, 0, kp, 256, 64, kp, *s, 0),
                 (None, 3, 0, 4, 0, 6, 0, kp, *s, kp, *s, 0)]:
        assert L.pkv_q4_append_kv(*args) == pkv.PKV_ERR_INVALID_ARG
        assert L.pkv_q4_read_kv(*args) == pkv.PKV_ERR_INVALID_ARG
    assert L.pkv_q4_init_cache(None, None, None, None) == pkv.PKV_ERR_INVALID_ARG
    assert L.pkv_q4_attention_workspace(h, 0, 1, 1, None) == pkv.PKV_ERR_INVALID_ARG
    assert L.pkv_q4_destroy_cache(None) == pkv.PKV_ERR_INVALID_ARG
    with pytest.raises(pkv.PkvError):
        pkv.pkv_q4_attention_workspace(h, 1, 0, 16)


# ---- GPU helpers ------------------------------------------------------------------------------------------------------
def rows_of(gen, n, heads, d, dtype, spread=True):
    x = torch.randn(n, heads, d, generator=gen)
    if spread:
        x = x * torch.exp(torch.rand(heads, d, generator=gen) * math.log(16) + math.log(0.5))
    return x.to(dtype)


class Filled:
    """A cache on the GPU holding sequences of random rows, and what it stands for in 64 bits."""
    room = 0                                               # tokens that the tables have place for, at least

    def __init__(self, lengths, dtype=BF16, d=128, g=32, P=64, H=2, G=4, seed=0, room=None, **kw):
        gen = torch.Generator().manual_seed(seed)
        self.gen, self.dtype, self.d, self.g, self.H, self.G, self.lens = gen, dtype, d, g, H, G, list(lengths)
        self.rows = Rows(lengths, P, seed, max_pages=max(-(-t // P) for t in [1, room or self.room, *lengths]))
        self.cache = pkv.Q4Cache(config(n_kv_heads=H, n_q_heads=H * G, head_dim=d, group_size=g, page_size=P, dtype=dtype,
                                        n_pages=self.rows.n_pages, **kw))
        self.cache.pool.fill_(0xff)                        # what no row was written to reads as NaN
        self.table, self.lengths = self.rows.device()
        self.k = [rows_of(gen, t, H, d, dtype) for t in lengths]
        self.v = [rows_of(gen, t, H, d, dtype, False) for t in lengths]
        self.off = offsets_of(lengths).cuda()
        if sum(lengths):
            self.cache.append_kv(self.table, self.lengths, torch.cat(self.k).cuda(), torch.cat(self.v).cuda(), self.off)
        self.K, self.V = [quantised(x, g) for x in self.k], [quantised(x, g) for x in self.v]

    def queries(self, ns):
        return [rows_of(self.gen, n, self.H * self.G, self.d, self.dtype, False) for n in ns]

    def expected(self, q, s, scale=None):
        n = q.shape[0]
        return attention(q, self.K[s], self.V[s], self.lens[s] - n, scale or 1 / math.sqrt(self.d), self.dtype)

    def clean(self):
        assert self.cache.stats() == {"device_timeouts": 0, "bad_pages": 0, "bad_lengths": 0}


def check(out, ref, tol):
    out = out.to("cpu", torch.float64)
    assert torch.isfinite(out).all()
    worst = ((out - ref).abs() / tol.clamp(min=1e-300)).max().item() if out.numel() else 0.0
    assert worst <= 1, worst
    return worst


SHAPES = [dict(dtype=BF16, d=128, g=32, P=64, H=2), dict(dtype=FP16, d=128, g=64, P=16, H=1), dict(dtype=BF16, d=128, g=128, P=32, H=3),
          dict(dtype=FP16, d=64, g=32, P=32, H=2), dict(dtype=BF16, d=64, g=64, P=128, H=1), dict(dtype=FP16, d=128, g=32, P=256, H=2)]


# ---- GPU: writing and reading ---------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_rows_read_back_as_the_values_they_were_quantised_to(shape):
    f = Filled([1, 0, 257, 15, 16, 130], **shape)
    k, v = (torch.full((sum(f.lens) + 2, f.H, f.d), 3.0, dtype=f.dtype, device="cuda") for _ in "kv")
    off = offsets_of(f.lens, start=1).cuda()
    f.cache.read_kv(f.table, f.lengths, k, v, off)
    assert torch.equal(k[1:-1].cpu(), torch.cat(f.K).to(f.dtype)) and torch.equal(v[1:-1].cpu(), torch.cat(f.V).to(f.dtype))
    for x in (k, v):                                       # rows that belong to no sequence
        assert (x[0] == 3).all() and (x[-1] == 3).all()
    f.clean()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("g", [32, 128])
def test_every_border_between_codes_is_decided_as_the_division_decides(dtype, g):
    """Groups whose largest value is drawn from all magnitudes of the type, filled with values on and next to the borders
    (k + 1/2) * scale."""
    info = torch.finfo(dtype)
    gen = torch.Generator().manual_seed(7)
    n = 4096
    top = torch.exp2(torch.empty(n).uniform_(math.log2(info.smallest_normal) - 6, math.log2(info.max), generator=gen).double())
    x = torch.empty(n, 128, dtype=torch.float64)
    top = top.clamp(max=info.max).to(dtype).double()
    scale = (top / 7).to(BF16).double().clamp(max=SCALE_MOST)
    border = (torch.randint(-7, 7, (n, 128), generator=gen).double() + 0.5) * scale[:, None]
    x = border.clamp(-top[:, None], top[:, None]).to(dtype)
    bits = x.view(torch.int16) + torch.randint(-1, 2, x.shape, generator=gen).to(torch.int16)
    near = bits.view(dtype)
    x = torch.where(torch.isfinite(near) & (near.double().abs() <= top[:, None]), near, x)
    x[:, ::g] = top[:, None].to(dtype)
    x = x.view(n, 1, 128)
    cache = pkv.Q4Cache(config(n_kv_heads=1, n_q_heads=1, group_size=g, n_pages=n // 64, dtype=dtype))
    table, lengths = torch.arange(n // 64, **INTS).view(1, -1).cuda(), torch.tensor([n], **INTS).cuda()
    y = x.flip(0).contiguous()
    cache.append_kv(table, lengths, x.view(1, n, 1, 128).cuda(), y.view(1, n, 1, 128).cuda())
    k, v = (torch.empty(1, n, 1, 128, dtype=dtype, device="cuda") for _ in "kv")
    cache.read_kv(table, lengths, k, v)
    for got, src in ((k, x), (v, y)):
        want = quantised(src, g).to(dtype).flatten()
        bad = got.cpu().flatten() != want
        assert not bad.any(), (src.flatten()[bad][:4], got.cpu().flatten()[bad][:4], want[bad][:4])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_largest_zero_and_non_finite_groups(dtype):
    big = torch.finfo(dtype).max
    x = torch.zeros(6, 1, 128, dtype=dtype)
    x[0, 0, 0] = big
    x[0, 0, 1] = -big
    x[1, 0, 32] = math.inf
    x[1, 0, 33] = 1.0
    x[2, 0, 64] = math.nan
    x[3, 0, 96] = -math.inf
    x[4, 0, :32] = -0.0
    x[5] = 1.0
    cache = pkv.Q4Cache(config(n_kv_heads=1, n_q_heads=1, dtype=dtype))
    table, lengths = torch.tensor([[5]], **INTS).cuda(), torch.tensor([6], **INTS).cuda()
    cache.append_kv(table, lengths, x.view(1, 6, 1, 128).cuda(), x.view(1, 6, 1, 128).cuda())
    k, v = (torch.empty(1, 6, 1, 128, dtype=dtype, device="cuda") for _ in "kv")
    cache.read_kv(table, lengths, k, v)
    want = quantised(x, 32).to(dtype)
    for got in (k, v):
        got = got.cpu().view(6, 1, 128)
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(), want.nan_to_num())
    assert torch.isnan(want).sum() == 3 * 32 and torch.isfinite(want[0]).all()


@pytest.mark.gpu
def test_strided_rows_and_rows_written_in_several_calls():
    """Slices of a fused projection, one token at a time and in pieces, uniform and ragged, leave the same cache as one
    call; rows of other positions and the buffers' other rows stay as they were."""
    f = Filled([70, 5, 64], P=16, H=2, G=3, seed=3)
    other = pkv.Q4Cache(f.cache.cfg)
    other.pool.fill_(0x11)
    have = [0, 0, 0]
    for ns in ([64, 0, 3], [1, 1, 1], [0, 1, 57], [5, 3, 3]):
        fused = torch.randn(sum(ns) + 2, 6 + 4, 128).to(BF16).cuda()
        rows = [(f.k[s][have[s]:have[s] + n], f.v[s][have[s]:have[s] + n]) for s, n in enumerate(ns)]
        fused[1:-1, 6:8] = torch.cat([r[0] for r in rows]).cuda()
        fused[1:-1, 8:] = torch.cat([r[1] for r in rows]).cuda()
        have = [h + n for h, n in zip(have, ns)]
        lengths = torch.tensor(have, **INTS).cuda()
        if ns == [1, 1, 1]:
            x = fused[1:-1].unflatten(0, (3, 1))
            other.append_kv(f.table, lengths, x[:, :, 6:8], x[:, :, 8:])
        else:
            other.append_kv(f.table, lengths, fused[:, 6:8], fused[:, 8:], offsets_of(ns, start=1).cuda())
    n = sum(f.lens)
    wide = torch.full((n, 7, 136), 2.0, dtype=BF16, device="cuda")
    k, v = wide[:, 1:3, 8:], wide[:, 4:6, :128]
    other.read_kv(f.table, f.lengths, k, v, f.off)
    assert torch.equal(k.cpu(), torch.cat(f.K).to(BF16)) and torch.equal(v.cpu(), torch.cat(f.V).to(BF16))
    wide[:, 1:3, 8:] = 2.0
    wide[:, 4:6, :128] = 2.0
    assert (wide == 2.0).all()
    assert other.stats() == {"device_timeouts": 0, "bad_pages": 0, "bad_lengths": 0}


@pytest.mark.gpu
def test_pages_beyond_four_gigabytes():
    """Offsets into the pool pass 32 bits."""
    H, P = 8, 64
    cfg = config(n_kv_heads=H, n_q_heads=H, n_pages=70000, page_size=P)
    cache = pkv.Q4Cache(cfg)
    assert 60000 * cache.sizes.page_bytes > 1 << 32
    gen = torch.Generator().manual_seed(1)
    k, v, q = (rows_of(gen, 100, H, 128, BF16) for _ in "kvq")
    table, lengths = torch.tensor([[69999, 60000]], **INTS).cuda(), torch.tensor([100], **INTS).cuda()
    cache.append_kv(table, lengths, k[None].cuda(), v[None].cuda())
    ko, vo = (torch.empty(1, 100, H, 128, dtype=BF16, device="cuda") for _ in "kv")
    cache.read_kv(table, lengths, ko, vo)
    assert torch.equal(ko[0].cpu(), quantised(k, 32).to(BF16)) and torch.equal(vo[0].cpu(), quantised(v, 32).to(BF16))
    out = cache.attention(table, lengths, q[None, -2:].cuda())
    ref, _, tol = attention(q[-2:], quantised(k, 32), quantised(v, 32), 98, 1 / math.sqrt(128), BF16)
    check(out[0], ref, tol)


# ---- GPU: attention ---------------------------------------------------------------------------------------------------
@pytest.fixture(params=["no more pages than used", "room for more"])
def room(request, monkeypatch):
    """How long the sequences could be steers which kernel runs, how it is spread and whether states are joined."""
    monkeypatch.setattr(Filled, "room", 3000 * (request.param == "room for more"))


def run_uniform(f, n, **kw):
    qs = f.queries([n] * len(f.lens))
    out = f.cache.attention(f.table, f.lengths, torch.stack(qs).cuda(), **kw)
    return [check(out[s], *f.expected(q, s)[::2]) for s, q in enumerate(qs)]


@pytest.mark.usefixtures("room")
@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("G", [1, 4, 8, 7, 12])
def test_decode(shape, G):
    f = Filled([1, 16, 17, 63, 64, 65, 300, 1000], G=G, **shape)
    run_uniform(f, 1)
    f.clean()


@pytest.mark.usefixtures("room")
@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("n, G", [(2, 4), (3, 1), (4, 4), (5, 7), (16, 2), (17, 8), (40, 4), (130, 3)])
def test_several_positions(shape, n, G):
    f = Filled([n, n + 1, 64 + n, 401], G=G, seed=n, **shape)
    run_uniform(f, n)
    f.clean()


@pytest.mark.usefixtures("room")
@pytest.mark.gpu
@pytest.mark.parametrize("n_ctas", [1, 3, 40])
@pytest.mark.parametrize("n, G", [(1, 4), (3, 8), (64, 4)])
def test_spread_over_few_and_many_ctas(n_ctas, n, G):
    """Every way a sequence can be cut: CTAs that hold many sequences, sequences that span many CTAs, cuts anywhere."""
    f = Filled([64, 1500, 65, 700, 129], H=2, G=G, P=32, seed=5, n_ctas=n_ctas)
    run_uniform(f, n)
    run_uniform(f, n, max_len=64)                          # the hint is wrong: the result is not
    f.clean()


@pytest.mark.gpu
@pytest.mark.parametrize("n, G", [(1, 4), (3, 8), (64, 4)])
@pytest.mark.parametrize("fill", [0xff, 0x00, 0x7b])
@pytest.mark.parametrize("lens", [[90, 0, 200], [1, 1, 1], [700, 64, 100]])
def test_what_the_workspace_held_does_not_matter(n, G, fill, lens):
    """Sequences far shorter than the table allows, so that CTAs of the launch stay without work; the scratch is full of
    NaN, zeros, large numbers."""
    lens = [max(n, t) if t else 0 for t in lens]
    f = Filled(lens, G=G, H=2, P=16, seed=17)
    table = torch.nn.functional.pad(f.table, (0, 300 - f.table.shape[1])).contiguous()
    qs = f.queries([n] * 3)
    q = torch.stack(qs).cuda()
    out = torch.empty_like(q)
    size = pkv.pkv_q4_attention_workspace(f.cache.handle, 3, n, 4800)
    work = torch.full((max(16, size),), fill, dtype=torch.uint8, device="cuda")
    strides = (2 * G * 128, 128)
    pkv.pkv_q4_attention(f.cache.handle, 3, table, 300, f.lengths, 3 * n, None, n, 4800, q, strides, out, strides, None, work, size,
                         torch.cuda.current_stream())
    for s in range(3):
        check(out[s], *f.expected(qs[s], s)[::2])


@pytest.mark.usefixtures("room")
@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES[:4], ids=str)
@pytest.mark.parametrize("ns", [[0, 1, 5, 0, 33], [3, 0, 0, 0, 0], [1, 1, 1, 1, 1], [100, 1, 2, 150, 300]])
def test_ragged_rows(shape, ns):
    """Sequences with different numbers of new rows, none among them; rows before the first and behind the last sequence
    stay as they were."""
    f = Filled([0, 1, 200, 150, 310], G=4, seed=11, **shape)
    ns = [min(a, b) for a, b in zip(ns, f.lens)]
    qs = f.queries(ns)
    pad = torch.zeros(2, f.H * f.G, f.d, dtype=f.dtype)
    q = torch.cat([pad[:1], *qs, pad[:1]]).cuda()
    off = offsets_of(ns, start=1).cuda()
    for most in (max(ns), None):
        out = torch.full_like(q, 5.0)
        f.cache.attention(f.table, f.lengths, q, out=out, offsets=off, max_q_len=most)
        assert (out[0] == 5).all() and (out[-1] == 5).all()
        at = 1
        for s, n in enumerate(ns):
            check(out[at:at + n], *f.expected(qs[s], s)[::2])
            at += n
    f.clean()


@pytest.mark.usefixtures("room")
@pytest.mark.gpu
@pytest.mark.parametrize("n, G", [(1, 4), (4, 8), (70, 4)])
def test_empty_sequences_and_queries_before_the_start_give_zeros(n, G):
    f = Filled([0, 1, max(1, n - 1), n + 3], G=G, seed=2)
    qs = f.queries([n] * 4)
    out = f.cache.attention(f.table, f.lengths, torch.stack(qs).cuda())
    for s, q in enumerate(qs):
        ref, _, tol = f.expected(q, s)
        first = max(0, n - f.lens[s])
        assert (out[s, :first] == 0).all()
        check(out[s], ref, tol)
    state = f.cache.attention_partial(f.table, f.lengths, torch.stack(qs).cuda())
    assert (state[0, :, :, 128 + 1] == 0).all() and (state[0, :, :, :128] == 0).all()


@pytest.mark.usefixtures("room")
@pytest.mark.gpu
@pytest.mark.parametrize("n, G", [(1, 4), (2, 4), (1, 16), (70, 4)])
@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_values_of_very_different_sizes(n, G, dtype):
    """Queries, keys and values up to the type's range: what matters is held relative to the largest."""
    f = Filled([200, 90], G=G, H=1, seed=4, dtype=dtype)
    for s in range(2):
        f.v[s][:, :, :64] *= 2.0 ** -12
        f.v[s][::3] *= 2.0 ** 9
        f.k[s] *= 2.0 ** 8
    f.cache.append_kv(f.table, f.lengths, torch.cat(f.k).cuda(), torch.cat(f.v).cuda(), f.off)
    f.K, f.V = [quantised(x, 32) for x in f.k], [quantised(x, 32) for x in f.v]
    qs = [q * 2.0 ** -9 for q in f.queries([n, n])]
    qs[1][..., 0] *= 2.0 ** 6
    out = f.cache.attention(f.table, f.lengths, torch.stack(qs).cuda())
    for s, q in enumerate(qs):
        check(out[s], *f.expected(q, s)[::2])


@pytest.mark.usefixtures("room")
@pytest.mark.gpu
@pytest.mark.parametrize("n, G", [(1, 4), (4, 4), (70, 4)])
@pytest.mark.parametrize("k, v", [(50, 0), (-50, 0), (0, 55), (0, -55), (50, -55)])
def test_magnitudes_near_the_ends_of_the_documented_range(n, G, k, v):
    f = Filled([150, 90], G=G, H=1, seed=30)
    ks, vs = [x * 2.0 ** k for x in f.k], [x * 2.0 ** v for x in f.v]
    f.cache.append_kv(f.table, f.lengths, torch.cat(ks).cuda(), torch.cat(vs).cuda(), f.off)
    f.K, f.V = [quantised(x, 32) for x in ks], [quantised(x, 32) for x in vs]
    qs = [q * 2.0 ** -k for q in f.queries([n, n])]
    out = f.cache.attention(f.table, f.lengths, torch.stack(qs).cuda())
    for s, q in enumerate(qs):
        check(out[s], *f.expected(q, s)[::2])


@pytest.mark.usefixtures("room")
@pytest.mark.gpu
@pytest.mark.parametrize("n, G", [(1, 4), (4, 4), (70, 4)])
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_queries_that_are_not_finite_leave_the_others_alone(n, G, value):
    f = Filled([200, 90], G=G, H=2, seed=31)
    qs = torch.stack(f.queries([n, n]))
    bad = qs.clone()
    bad[0, n // 2, 1, 5] = value
    out = f.cache.attention(f.table, f.lengths, bad.cuda()).cpu()
    if value != value:
        assert torch.isnan(out[0, n // 2, 1]).all()
    for s in range(2):
        ref, _, tol = f.expected(qs[s], s)
        if s == 0:
            out[0, n // 2, 1] = 0.0
            ref[n // 2, 1] = 0.0
        check(out[s], ref, tol)


@pytest.mark.usefixtures("room")
@pytest.mark.gpu
@pytest.mark.parametrize("n, G", [(1, 4), (4, 4), (70, 4)])
def test_infinite_and_nan_rows_reach_only_the_queries_that_see_them(n, G):
    """A key or value that is not finite makes the queries that see it NaN (a value: at least its group's channels) and
    leaves the others alone, whether they come before it or belong to other sequences."""
    f = Filled([80 + n, 100, 64], G=G, H=1, seed=6)
    T = f.lens[0]
    hit = T - 1 if n > 1 else 10                           # several positions: only the last query sees it
    qs = f.queries([n] * 3)
    for what, value in (("k", math.nan), ("v", math.inf), ("v", math.nan)):
        rows = getattr(f, what)[0].clone()
        rows[hit, 0, 40] = value
        k, v = (torch.cat([rows if what == x else getattr(f, x)[0], *getattr(f, x)[1:]]).cuda() for x in "kv")
        f.cache.append_kv(f.table, f.lengths, k, v, f.off)
        out = f.cache.attention(f.table, f.lengths, torch.stack(qs).cuda())
        for s, q in enumerate(qs):
            ref, _, tol = f.expected(q, s)
            blind = n if s else (n - 1 if n > 1 else 0)
            check(out[s, :blind], ref[:blind], tol[:blind])
        assert torch.isnan(out[0, -1, :, 32:64]).all()


@pytest.mark.usefixtures("room")
@pytest.mark.gpu
@pytest.mark.parametrize("n, G", [(1, 4), (8, 4), (70, 2)])
def test_pages_and_lengths_that_make_no_sense(n, G):
    """Bad page numbers are skipped and counted; lengths are held inside the table."""
    f = Filled([150, 90], G=G, H=2, P=32, seed=8)
    table = f.table.clone()
    table[0, 1], table[1, 0] = f.rows.n_pages, -1          # tokens 32..63 and 0..31 are not there
    qs = f.queries([n, n])
    out = f.cache.attention(table, f.lengths, torch.stack(qs).cuda())
    assert f.cache.stats()["bad_pages"] > 0
    for s, (q, gone) in enumerate(zip(qs, (32, 0))):
        keep = [t for t in range(f.lens[s]) if not gone <= t < gone + 32]
        for j in range(n):
            see = [t for t in keep if t <= f.lens[s] - n + j]
            ref, _, tol = attention(q[j:j + 1], f.K[s][see], f.V[s][see], len(see) - 1, 1 / math.sqrt(128), BF16)
            check(out[s, j:j + 1], ref, tol)
    before = f.cache.pool.clone()
    one = torch.zeros(2, 1, 2, 128, dtype=BF16, device="cuda")
    f.cache.append_kv(table, torch.tensor([60, 5], **INTS).cuda(), one, one)
    assert torch.equal(before, f.cache.pool)
    k = torch.full_like(one, 4.0)
    f.cache.read_kv(table, torch.tensor([60, 5], **INTS).cuda(), k, k.clone())
    assert (k == 4).all()
    bad = f.cache.stats()["bad_lengths"]
    f.cache.append_kv(f.table, torch.tensor([-3, 0], **INTS).cuda(), one, one)
    assert torch.equal(before, f.cache.pool) and f.cache.stats()["bad_lengths"] > bad
    q = torch.stack(qs).cuda()
    out = f.cache.attention(f.table, torch.tensor([-5, 90], **INTS).cuda(), q)
    assert (out[0] == 0).all()
    check(out[1], *f.expected(qs[1], 1)[::2])
    bad = f.cache.stats()["bad_lengths"]
    f.cache.attention(f.table, torch.tensor([1 << 30, 90], **INTS).cuda(), q)      # as if it filled its table
    assert f.cache.stats()["bad_lengths"] > bad


@pytest.mark.usefixtures("room")
@pytest.mark.gpu
@pytest.mark.parametrize("G", [33, 64])
def test_many_query_heads_per_kv_head(G):
    f = Filled([1, 70, 333], G=G, H=2, seed=24)
    run_uniform(f, 1)
    run_uniform(Filled([9, 200], G=G, H=1, seed=25), 9)


@pytest.mark.gpu
@pytest.mark.parametrize("n, most", [(1, 40), (1, 3000), (9, 40)])
def test_more_sequences_than_a_cta_has_threads(n, most):
    """900 sequences, empty ones among them; `most` is the length the call is told to expect."""
    gen = torch.Generator().manual_seed(n)
    lens = [0 if i % 7 == 0 else max(n, int(t)) for i, t in enumerate(torch.randint(1, 41, (900,), generator=gen))]
    f = Filled(lens, G=2, H=1, P=16, seed=26)
    qs = f.queries([n] * 900)
    out = f.cache.attention(f.table, f.lengths, torch.stack(qs).cuda(), max_len=most).cpu()
    for s, q in enumerate(qs):
        check(out[s], *f.expected(q, s)[::2])
    f.clean()


@pytest.mark.usefixtures("room")
@pytest.mark.gpu
@pytest.mark.parametrize("dtype, d, g, G, lens", [(BF16, 128, 32, 4, [1200]), (FP16, 64, 64, 7, [700, 10, 390]), (BF16, 128, 128, 1, [2600, 300])])
def test_whole_prompts(dtype, d, g, G, lens):
    """Every position of the prompts is a query: blocks of very different lengths, more than a warp looks up at once."""
    f = Filled(lens, dtype=dtype, d=d, g=g, G=G, H=1, P=32, seed=27)
    qs = f.queries(lens)
    out = f.cache.attention(f.table, f.lengths, torch.cat(qs).cuda(), offsets=f.off, max_q_len=max(lens)).cpu()
    at = 0
    for s, q in enumerate(qs):
        check(out[at:at + lens[s]], *f.expected(q, s)[::2])
        at += lens[s]
    f.clean()


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 9, 40])
def test_many_kv_heads(n):
    f = Filled([21, 70], G=1, H=200, P=16, d=64, seed=32)
    k, v = (torch.empty(91, 200, 64, dtype=BF16, device="cuda") for _ in "kv")
    f.cache.read_kv(f.table, f.lengths, k, v, f.off)
    assert torch.equal(k.cpu(), torch.cat(f.K).to(BF16)) and torch.equal(v.cpu(), torch.cat(f.V).to(BF16))
    qs = f.queries([min(n, 21), n])
    out = f.cache.attention(f.table, f.lengths, torch.cat(qs).cuda(), offsets=offsets_of([min(n, 21), n]).cuda(), max_q_len=n).cpu()
    check(out[:min(n, 21)], *f.expected(qs[0], 0)[::2])
    check(out[min(n, 21):], *f.expected(qs[1], 1)[::2])
    f.clean()


@pytest.mark.gpu
@pytest.mark.parametrize("max_len", [16, 0])
def test_as_many_sequences_as_a_call_takes(max_len):
    """65535 sequences of one token, every ninth empty: attention gives the token's value, as it was quantised."""
    S, H, d, P = 65535, 2, 64, 16
    cache = pkv.Q4Cache(config(n_kv_heads=H, n_q_heads=2 * H, head_dim=d, page_size=P, n_pages=S))
    table = torch.full((S, 1 if max_len else 200), -1, dtype=torch.int32)
    table[:, 0] = torch.randperm(S, generator=torch.Generator().manual_seed(1)).int()
    lengths = torch.ones(S, dtype=torch.int32)
    lengths[::9] = 0
    off = offsets_of(lengths.tolist()).cuda()
    table, there = table.cuda(), lengths.bool()
    n = int(there.sum())
    k, v = (torch.randn(n, H, d, generator=torch.Generator().manual_seed(i)).to(BF16) for i in (2, 3))
    cache.append_kv(table, lengths.cuda(), k.cuda(), v.cuda(), off)
    q = torch.randn(n, 2 * H, d, generator=torch.Generator().manual_seed(4)).to(BF16).cuda()
    out = cache.attention(table, lengths.cuda(), q, offsets=off, max_q_len=1, max_len=max_len)
    # One token: o = w * code * scale and l = w for one weight w = 2^-E (1 + e), |e| <= 2^-20 (the exponent is score - (score +
    # E), of numbers below 2^4 here: half an fp32 step is 2^-20, times ln 2; exp2 is good to 2^-22).  w * scale is rounded to fp16:
    # scale has 8 bits and fp16 holds 11, so that is 2^-E scale itself.  o / l is then code * scale (1 - e), and a code * scale
    # that lies halfway between two bf16 numbers may go to either: half a step, 2^-8 of the value, and e.
    exact = quantised(v, 32).repeat_interleave(2, 1)
    assert ((out.cpu().double() - exact).abs() <= exact.abs() * (2.0 ** -8 + 2.0 ** -20)).all()
    uniform = cache.attention(table, lengths.cuda(), torch.ones(S, 1, 2 * H, d, dtype=BF16, device="cuda"), max_len=max_len)[:, 0]
    assert ((uniform[there.cuda()].cpu().double() - exact).abs() <= exact.abs() * (2.0 ** -8 + 2.0 ** -20)).all()
    assert (uniform[~there.cuda()] == 0).all()
    assert cache.stats() == {"device_timeouts": 0, "bad_pages": 0, "bad_lengths": 0}


@pytest.mark.gpu
def test_one_very_long_sequence():
    f = Filled([300_003], G=2, H=1, P=256, d=64, seed=33)
    for n in (1, 7, 40):
        q = f.queries([n])[0]
        check(f.cache.attention(f.table, f.lengths, q[None].cuda())[0], *f.expected(q, 0)[::2])
    f.clean()


@pytest.mark.gpu
def test_a_long_prompt_in_more_blocks_than_a_warp_looks_up_at_once():
    n, G = 2200, 8                                         # 69 blocks of 256 rows
    f = Filled([n], G=G, H=1, P=64, seed=28)
    q = f.queries([n])[0]
    out = f.cache.attention(f.table, f.lengths, q[None].cuda())[0].cpu()
    rows = torch.tensor([0, 1, 31, 32, 33, 63, 64, 1000, 1023, 1024, 1025, 2111, 2112, 2198, 2199])
    for j in rows.tolist():
        ref, _, tol = attention(q[j:j + 1], f.K[0][:j + 1], f.V[0][:j + 1], j, 1 / math.sqrt(128), BF16)
        check(out[j:j + 1], ref, tol)
    f.clean()


@pytest.mark.usefixtures("room")
@pytest.mark.gpu
def test_more_rows_than_the_bound_says():
    f = Filled([100, 50], G=4, seed=9)
    qs = f.queries([5, 2])
    q = torch.cat(qs).cuda()
    out = torch.full_like(q, 5.0)
    f.cache.attention(f.table, f.lengths, q, out=out, offsets=offsets_of([5, 2]).cuda(), max_q_len=3)
    check(out[:3], *[x[:3] for x in f.expected(qs[0], 0)[::2]])
    assert (out[3:5] == 5).all() and f.cache.stats()["bad_lengths"] > 0
    check(out[5:], *f.expected(qs[1], 1)[::2])


@pytest.mark.usefixtures("room")
@pytest.mark.gpu
@pytest.mark.parametrize("n, G, H", [(1, 4, 2), (6, 8, 1), (80, 4, 2)])
@pytest.mark.parametrize("dtype, d", [(BF16, 128), (FP16, 64)])
def test_states(n, G, H, dtype, d):
    """o / l is the attention and m + log2 l the logarithm of the sum of weights."""
    f = Filled([n, 130 + n, 700], G=G, H=H, d=d, dtype=dtype, seed=12)
    qs = f.queries([n] * 3)
    st = f.cache.attention_partial(f.table, f.lengths, torch.stack(qs).cuda()).to("cpu", torch.float64)
    for s, q in enumerate(qs):
        ref, lse, tol = f.expected(q, s)
        check(st[s, ..., :d] / st[s, ..., d + 1:], ref, tol)
        # l: fp32 sums and exp2, scores off by ds as in the tolerance of the values; 2^-12 in base-2 units is far above both
        assert (st[s, ..., d] + torch.log2(st[s, ..., d + 1]) - lse).abs().max() < 2.0 ** -12


@pytest.mark.usefixtures("room")
@pytest.mark.gpu
@pytest.mark.parametrize("scale", [0.02, 1.0])
def test_softmax_scale(scale):
    f = Filled([90, 33], G=4, seed=13, softmax_scale=scale)
    qs = f.queries([2, 2])
    out = f.cache.attention(f.table, f.lengths, torch.stack(qs).cuda())
    for s, q in enumerate(qs):
        check(out[s], *f.expected(q, s, scale)[::2])


@pytest.mark.usefixtures("room")
@pytest.mark.gpu
@pytest.mark.parametrize("n, G", [(1, 4), (3, 8), (90, 4)])
def test_strided_queries_and_results(n, G):
    f = Filled([150, 91], G=G, H=2, seed=14)
    qs = f.queries([n, n])
    hq = 2 * G
    fused = torch.randn(2, n, hq + 4, 128).to(BF16).cuda()
    fused[:, :, :hq] = torch.stack(qs).cuda()
    wide = torch.full((2, n, hq + 1, 136), 7.0, dtype=BF16, device="cuda")
    out = wide[:, :, 1:, :128]
    f.cache.attention(f.table, f.lengths, fused[:, :, :hq], out=out)
    for s, q in enumerate(qs):
        check(out[s], *f.expected(q, s)[::2])
    assert (wide[:, :, 0] == 7).all() and (wide[..., 128:] == 7).all()


# ---- GPU: how a user's program runs them ------------------------------------------------------------------------------
@pytest.mark.usefixtures("room")
@pytest.mark.gpu
@pytest.mark.parametrize("n, G", [(1, 4), (2, 4), (64, 4)])
def test_same_bits_every_run_on_any_stream_and_in_a_graph(n, G):
    f = Filled([700, 1100, 33], G=G, H=2, seed=15, P=16)
    qs = torch.stack(f.queries([n] * 3)).cuda()
    first = f.cache.attention(f.table, f.lengths, qs)
    torch.cuda.synchronize()
    for _ in range(3):
        assert torch.equal(first, f.cache.attention(f.table, f.lengths, qs))
    streams = [torch.cuda.Stream() for _ in range(4)]      # calls in flight at the same time
    outs = []
    for s in streams * 3:
        with torch.cuda.stream(s):
            outs.append(f.cache.attention(f.table, f.lengths, qs))
    torch.cuda.synchronize()
    assert all(torch.equal(first, o) for o in outs)
    graphs, kept = [], []
    for _ in range(2):                                     # two graphs, replayed side by side
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            kept.append(f.cache.attention(f.table, f.lengths, qs))
        graphs.append(g)
    for _ in range(3):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(first, o) for o in kept)
    f.clean()


@pytest.mark.gpu
def test_a_decode_loop_in_one_captured_graph():
    """append -> attend, captured once with lengths and page table on the device and replayed while sequences grow across
    pages, one of them idle (no new row, as in a padded batch)."""
    P, G, H, steps = 16, 4, 2, 40
    f = Filled([30, 0, 17], P=P, G=G, H=H, seed=16)
    gen = torch.Generator().manual_seed(3)
    table = torch.arange(3 * 8, **INTS).view(3, 8).cuda()
    cache = pkv.Q4Cache(config(n_kv_heads=H, n_q_heads=H * G, page_size=P, n_pages=24))
    lengths, off = f.lengths.clone(), offsets_of([1, 0, 1]).cuda()
    cache.append_kv(table, lengths, torch.cat(f.k).cuda(), torch.cat(f.v).cuda(), f.off)
    k, v, q = (torch.zeros(2, h, 128, dtype=BF16, device="cuda") for h in (H, H, H * G))
    out = torch.zeros_like(q)
    one = torch.tensor([1, 0, 1], **INTS).cuda()

    def step():
        lengths.add_(one)
        cache.append_kv(table, lengths, k, v, off)
        cache.attention(table, lengths, q, out=out, offsets=off, max_q_len=1)

    step()                                                 # (warm-up; undone below)
    torch.cuda.synchronize()
    lengths.copy_(f.lengths)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    lengths.copy_(f.lengths)
    K, V = [f.K[0], f.K[2]], [f.V[0], f.V[2]]
    for i in range(steps):
        new = [rows_of(gen, 2, h, 128, BF16, False) for h in (H, H, H * G)]
        for dst, src in zip((k, v, q), new):
            dst.copy_(src)
        g.replay()
        for r in range(2):
            K[r], V[r] = torch.cat([K[r], quantised(new[0][r:r + 1], 32)]), torch.cat([V[r], quantised(new[1][r:r + 1], 32)])
            ref, _, tol = attention(new[2][r:r + 1], K[r], V[r], K[r].shape[0] - 1, 1 / math.sqrt(128), BF16)
            check(out[r:r + 1], ref, tol)
    assert cache.stats() == {"device_timeouts": 0, "bad_pages": 0, "bad_lengths": 0}


@pytest.mark.gpu
def test_prefill_in_chunks_then_speculative_steps():
    """The calls in a row as a user makes them: chunks of a prompt are written and attended to, then steps of a few
    positions of which some are taken back (shorter lengths; the rows are overwritten by the next step)."""
    H, G, P = 2, 4, 32
    gen = torch.Generator().manual_seed(21)
    cache = pkv.Q4Cache(config(n_kv_heads=H, n_q_heads=H * G, page_size=P, n_pages=20))
    table = torch.randperm(20, generator=gen).to(torch.int32).view(1, 20).cuda()
    K, V = torch.empty(0, H, 128, dtype=torch.float64), torch.empty(0, H, 128, dtype=torch.float64)
    for n, taken in ((100, 100), (77, 77), (150, 150), (4, 1), (4, 4), (4, 2), (1, 1)):
        k, v, q = (rows_of(gen, n, h, 128, BF16, False) for h in (H, H, H * G))
        lengths = torch.tensor([K.shape[0] + n], **INTS).cuda()
        cache.append_kv(table, lengths, k[None].cuda(), v[None].cuda())
        out = cache.attention(table, lengths, q[None].cuda())
        kq, vq = torch.cat([K, quantised(k, 32)]), torch.cat([V, quantised(v, 32)])
        ref, _, tol = attention(q, kq, vq, K.shape[0], 1 / math.sqrt(128), BF16)
        check(out[0], ref, tol)
        K, V = kq[:K.shape[0] + taken], vq[:K.shape[0] + taken]
    assert cache.stats() == {"device_timeouts": 0, "bad_pages": 0, "bad_lengths": 0}


@pytest.mark.gpu
def test_old_tokens_in_4_bits_recent_ones_in_a_dense_and_factor_cache():
    """The states of this cache and of the framework's page cache merge to attention over both."""
    H, G, old, recent = 2, 4, 500, 130
    f = Filled([old], H=H, G=G, seed=22)
    c = pkv.Cache(pkv.make_config(n_layers=1, n_kv_heads=H, n_q_heads=H * G, rank=16, sink_tokens=64, recent_tokens=64, max_seqs=1,
                                  max_pages_per_seq=8, n_dense_slots=8, n_factor_slots=1))
    k, v = rows_of(f.gen, recent, H, 128, BF16), rows_of(f.gen, recent, H, 128, BF16, False)
    c.append_kv(0, [0], [recent], k.cuda(), v.cuda())
    q = f.queries([1])[0]
    states = torch.empty(2, 1, H * G, 130, device="cuda")
    f.cache.attention_partial(f.table, f.lengths, q[None].cuda(), state=states[:1])
    c.decode_attention_partial(0, [0], q.cuda(), state=states[1])
    out = torch.empty(1, H * G, 128, dtype=BF16, device="cuda")
    pkv.pkv_merge_attention_states(states, 2, H * G, out=out, stream=torch.cuda.current_stream())
    K, V = torch.cat([f.K[0], k.double()]), torch.cat([f.V[0], v.double()])
    ref, _, tol = attention(q, K, V, old + recent - 1, 1 / math.sqrt(128), BF16)
    # the dense rows' weights are rounded to bf16 there: one unit of 2^-9 of the largest value, instead of fp16's 2^-11
    check(out, ref, tol + 2.0 ** -9 * V.abs().max())
    c.close()


@pytest.mark.gpu
@pytest.mark.parametrize("n, G", [(1, 4), (5, 8)])
def test_states_of_an_empty_cache_merge_as_nothing(n, G):
    f = Filled([0, 100], H=2, G=G, seed=34)
    q = f.queries([n])[0]
    both = torch.stack([q, q]).cuda()
    states = f.cache.attention_partial(f.table, f.lengths, both)      # shard 0 has no tokens
    out = torch.empty(n, 2 * G, 128, dtype=BF16, device="cuda")
    pkv.pkv_merge_attention_states(states, 2, n * 2 * G, out=out, stream=torch.cuda.current_stream())
    check(out, *f.expected(q, 1)[::2])


@pytest.mark.gpu
def test_shared_pages():
    """Two sequences read one prefix."""
    f = Filled([128, 10], H=1, G=4, P=64, seed=23)
    table = torch.cat([f.table[:1, :2], f.table[:1, :2]]).contiguous()
    q = torch.stack(f.queries([1, 1])).cuda()
    out = f.cache.attention(table, torch.tensor([128, 65], **INTS).cuda(), q)
    check(out[0], *f.expected(q[0].cpu(), 0)[::2])
    ref, _, tol = attention(q[1].cpu(), f.K[0][:65], f.V[0][:65], 64, 1 / math.sqrt(128), BF16)
    check(out[1], ref, tol)


@pytest.mark.usefixtures("room")
@pytest.mark.gpu
@pytest.mark.parametrize("seed", range(6))
def test_random_configurations(seed):
    import random
    rng = random.Random(seed)
    for _ in range(6):
        d = rng.choice([64, 128])
        shape = dict(dtype=rng.choice([BF16, FP16]), d=d, g=rng.choice([x for x in (32, 64, 128) if x <= d]),
                     P=rng.choice([16, 32, 64, 128, 256]), H=rng.randint(1, 3), G=rng.choice([1, 2, 3, 5, 8, 9, 16]))
        lens = [rng.choice([0, 1, rng.randint(1, 64), rng.randint(1, 700)]) for _ in range(rng.randint(1, 6))]
        most = rng.choice([1, 2, 5, 30, 100])
        ns = [min(t, rng.randint(0, most)) for t in lens]
        f = Filled(lens, seed=seed, **shape)
        qs = f.queries(ns)
        q = torch.cat(qs).cuda()
        out = f.cache.attention(f.table, f.lengths, q, offsets=offsets_of(ns).cuda(), max_q_len=max(1, min(most, sum(ns))))
        at = 0
        for s, n in enumerate(ns):
            check(out[at:at + n], *f.expected(qs[s], s)[::2])
            at += n
        f.clean()


@pytest.mark.gpu
def test_between_decodes_of_the_page_cache_that_do_not_wait_for_one_another():
    """A page cache whose decode launches overlap freely (decode_overlap = 2) shares the stream: rows appended before one of
    its launches are there for the attention behind it, whatever memory the buffers in between get."""
    H, G, T = 2, 4, 2000
    f = Filled([T, 300], H=H, G=G, seed=35, room=3000)
    c = pkv.Cache(pkv.make_config(n_layers=1, n_kv_heads=H, n_q_heads=H * G, rank=16, sink_tokens=64, recent_tokens=64, max_seqs=1,
                                  max_pages_per_seq=8, n_dense_slots=8, n_factor_slots=1, decode_overlap=2))
    k, v = rows_of(f.gen, 130, H, 128, BF16), rows_of(f.gen, 130, H, 128, BF16, False)
    c.append_kv(0, [0], [130], k.cuda(), v.cuda())
    q = f.queries([1])[0]
    qs = [torch.stack(f.queries([n, n])).cuda() for n in (1, 4, 40)]
    qd = q.cuda()
    want = [f.cache.attention(f.table, f.lengths, x) for x in qs]
    dense, _, tol = attention(q, k.double(), v.double(), 129, 1 / math.sqrt(128), BF16)
    torch.cuda.synchronize()
    rows = [torch.cat(x).cuda() for x in (f.k, f.v)]
    kept = []
    for i in range(12):
        f.cache.append_kv(f.table, f.lengths, *rows, f.off)
        a = torch.empty(1, H * G, 128, dtype=BF16, device="cuda")
        c.decode_attention(0, [0], qd, out=a)
        b = f.cache.attention(f.table, f.lengths, qs[i % 3])
        back = [torch.empty_like(x) for x in rows]
        c.decode_attention(0, [0], qd, out=torch.empty_like(a))
        f.cache.read_kv(f.table, f.lengths, *back, f.off)
        kept.append((a, b, back))
    torch.cuda.synchronize()
    for i, (a, b, back) in enumerate(kept):
        assert torch.equal(b, want[i % 3])
        check(a, dense, tol + 2.0 ** -9 * v.abs().max())      # (bf16 weights there, see above)
        assert torch.equal(back[0].cpu(), torch.cat(f.K).to(BF16)) and torch.equal(back[1].cpu(), torch.cat(f.V).to(BF16))
    f.clean()
    c.close()


@pytest.mark.gpu
def test_in_a_process_without_such_a_cache():
    """Kernels are launched differently there: the tests of calls that follow one another, by themselves."""
    import subprocess
    import sys
    names = "same_bits or decode_loop or prefill_in_chunks or written_in_several_calls or random_configurations or whole_prompts"
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-m", "gpu", "-k", names, "-p", "no:cacheprovider", __file__],
                       capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-3000:]
