"""The 4-bit cache's attention where numbers of very different sizes meet: every channel is judged by its own group's values, and rows
that a query does not see must not matter to it."""
import math

import pytest
import torch

from paper_2608_23843_b200 import pkv
from q4_precision_reference import attention
from q4_reference import Rows, offsets_of, quantised

BF16, FP16 = torch.bfloat16, torch.float16
# new positions and query heads per KV head: eight query rows at a time, sixteen; row blocks of both halves, of one
ROWS = [(1, 4), (2, 4), (4, 4)]
BLOCKS = [(70, 4), (20, 4)]


class Held:
    """A cache on the GPU and the rows that were written to it."""

    def __init__(self, k, v, G=4, g=32, P=64, room=3000, **kw):
        """k, v: a list of [T, H, d] per sequence."""
        _, H, d = k[0].shape
        self.k, self.v, self.g, self.G, self.d, self.H, self.dtype = k, v, g, G, d, H, k[0].dtype
        lens = [x.shape[0] for x in k]
        self.rows = Rows(lens, P, 1, max_pages=max(-(-t // P) for t in [room, *lens]))
        self.cache = pkv.Q4Cache(pkv.make_q4_config(n_kv_heads=H, n_q_heads=H * G, head_dim=d, page_size=P, group_size=g,
                                                    dtype=self.dtype, n_pages=self.rows.n_pages, **kw))
        self.cache.pool.fill_(0xff)
        self.table, self.lengths = self.rows.device()
        self.cache.append_kv(self.table, self.lengths, torch.cat(k).cuda(), torch.cat(v).cuda(), offsets_of(lens).cuda())

    def attend(self, qs, **kw):
        return self.cache.attention(self.table, self.lengths, torch.stack(qs).cuda(), **kw).cpu()

    def expected(self, q, s, steps=None):
        return attention(q, self.k[s], self.v[s], self.g, self.k[s].shape[0] - q.shape[0], 1 / math.sqrt(self.d), self.dtype, steps)


def randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed))


def check(out, ref, tol):
    out = out.to(torch.float64)
    assert torch.isfinite(out).all()
    worst = ((out - ref).abs() / tol).max().item()
    assert worst <= 1, worst


@pytest.mark.gpu
@pytest.mark.parametrize("n, G", ROWS + BLOCKS)
@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_scores_beside_a_large_query_channel(n, G, dtype):
    """A query's large channel meets keys whose codes are zero there: it must not cost the other channels' products."""
    T = 500
    k, q = randn(1, T, 1, 128), randn(2, n, G, 128)
    k[..., 3] *= 0.0
    q[..., 3] = 30000.0
    h = Held([k.to(dtype)], [randn(3, T, 1, 128).to(dtype)], G=G)
    q = q.to(dtype)
    check(h.attend([q])[0], *h.expected(q, 0))


@pytest.mark.gpu
@pytest.mark.parametrize("n, G", ROWS[1:] + BLOCKS)
@pytest.mark.parametrize("what", ["k", "v"])
@pytest.mark.parametrize("power", [20, 40])
def test_a_row_that_is_not_seen_does_not_matter_whatever_its_size(n, G, what, power):
    """The last key or value row is far larger than the others: the queries before it do not see it."""
    T = 300
    k, v, q = randn(1, T, 1, 128), randn(2, T, 1, 128), randn(3, n, G, 128).to(BF16)
    (k if what == "k" else v)[-1] *= 2.0 ** power
    h = Held([k.to(BF16)], [v.to(BF16)], G=G)
    ref, tol = h.expected(q, 0)
    check(h.attend([q])[0, :-1], ref[:-1], tol[:-1])


@pytest.mark.gpu
@pytest.mark.parametrize("n, G", ROWS + BLOCKS)
@pytest.mark.parametrize("dtype, g, power", [(BF16, 32, 12), (BF16, 32, 20), (BF16, 64, 26), (FP16, 32, 12), (FP16, 64, 20)])
def test_channel_groups_of_different_sizes(n, G, dtype, g, power):
    """The first group's values are 2^power times the others'."""
    T = 400
    v = randn(1, T, 1, 128) * 2.0 ** (-power // 2)
    v[..., :g] *= 2.0 ** power
    h = Held([randn(2, T, 1, 128).to(dtype)], [v.to(dtype)], G=G, g=g)
    q = randn(3, n, G, 128).to(dtype)
    check(h.attend([q])[0], *h.expected(q, 0))


@pytest.mark.gpu
@pytest.mark.parametrize("n, G", ROWS + BLOCKS)
@pytest.mark.parametrize("power", [8, 16, 25])
def test_large_values_of_no_weight(n, G, power):
    """Every seventh token has values 2^power times the others' and a weight of nothing."""
    T = 300
    k, v, q = randn(1, T, 1, 128), randn(2, T, 1, 128), randn(3, n, G, 128)
    q[..., 0], k[..., 0] = 10.0, 0.0
    k[3::7, :, 0] = -80.0                                  # 71 nepers below
    v[3::7] *= 2.0 ** power
    k[::7, :, 0] = -20.0                                   # and some between
    h = Held([k.to(BF16)], [v.to(BF16)], G=G)
    q = q.to(BF16)
    check(h.attend([q])[0], *h.expected(q, 0))


@pytest.mark.gpu
@pytest.mark.parametrize("n, G", ROWS + BLOCKS)
@pytest.mark.parametrize("dtype, power", [(BF16, 16), (BF16, 20), (BF16, 26), (FP16, 14)])
def test_keys_and_queries_of_opposite_sizes(n, G, dtype, power):
    """The first group's keys are 2^power times the others', and the queries' channels there as much smaller."""
    T = 400
    k, q = randn(1, T, 1, 128) * 2.0 ** (-power // 2), randn(2, n, G, 128) * 2.0 ** (power // 2)
    k[..., :32] *= 2.0 ** power
    q[..., :32] *= 2.0 ** -power
    h = Held([k.to(dtype)], [randn(3, T, 1, 128).to(dtype)], G=G)
    q = q.to(dtype)
    check(h.attend([q])[0], *h.expected(q, 0))


@pytest.mark.gpu
@pytest.mark.parametrize("n, G", [(1, 4), (4, 4), (9, 4)])
@pytest.mark.parametrize("weight", [0.97, 0.999])
@pytest.mark.parametrize("ratio", [1, 16, 64])
def test_one_token_with_nearly_all_the_weight(n, G, weight, ratio):
    """A first token of small values that holds nearly all the weight, the rest spread thin over 33000; the first channel group
    is `ratio` times the others."""
    T = 33000
    k, v, q = randn(1, T, 1, 128) * 0.05, 1 + 0.3 * randn(2, T, 1, 128), randn(3, n, G, 128)
    q[..., 0], k[..., 0] = 16.0, 0.0
    k[0, :, 0] = math.log(weight / (1 - weight) * T) / 16 * math.sqrt(128)
    v[0] *= 2.0 ** -6
    v[..., :32] *= ratio
    h = Held([k.to(FP16)], [v.to(FP16)], G=G, room=0)
    q = q.to(FP16)
    # (the units of 64 tokens are spread over 14 CTAs at least, 7 warps or two halves each: 18 units of four runs at most)
    check(h.attend([q])[0], *h.expected(q, 0, 80))


@pytest.mark.gpu
@pytest.mark.parametrize("n, G", ROWS + BLOCKS)
@pytest.mark.parametrize("room", [0, 3000])
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_a_value_that_is_not_finite_reaches_its_channel_group_only(n, G, room, value):
    T, hit = 700, 650
    k, v, q = (randn(i, *s).to(BF16) for i, s in enumerate(((T, 1, 128), (T, 1, 128), (n, G, 128))))
    h = Held([k], [v], G=G, room=room)
    bad = v.clone()
    bad[hit, 0, 40] = value
    h.cache.append_kv(h.table, h.lengths, k[None].cuda(), bad[None].cuda())
    ref, tol = h.expected(q, 0)
    sees = max(0, hit - (T - n))                           # the first query that sees it
    outs = [h.attend([q])[0]]
    st = h.cache.attention_partial(h.table, h.lengths, q[None].cuda())[0].cpu()
    outs.append(st[..., :128] / st[..., 129:])
    for out in outs:
        check(out[:sees], ref[:sees], tol[:sees]) if sees else None
        assert torch.isnan(out[sees:, :, 32:64]).all()
        rest = [c for c in range(128) if not 32 <= c < 64]
        check(out[..., rest], ref[..., rest], tol[..., rest])


@pytest.mark.gpu
@pytest.mark.parametrize("n, G", ROWS + BLOCKS)
@pytest.mark.parametrize("d, g, P", [(128, 32, 64), (128, 64, 16), (128, 128, 32), (64, 32, 32), (64, 64, 128)])
@pytest.mark.parametrize("seed", range(2))
def test_sizes_drawn_at_random(n, G, d, g, P, seed):
    """Every token and channel group has a size of its own; some tokens are zero; sequences of several lengths, in several shares."""
    gen = torch.Generator().manual_seed(100 * seed + n)
    power = lambda lo, hi, *s: torch.exp2(torch.randint(lo, hi + 1, s, generator=gen).float())      # noqa: E731
    H = 2
    k, v, qs = [], [], []
    groups = power(-8, 8, H, d // g, 1)                    # of the keys; the queries the other way round
    for T in (n, 37 + n, 300, 901):
        some = (torch.rand(T, 1, 1, 1, generator=gen) < 0.3).float()
        kt, vt = (torch.randn(T, H, d // g, g, generator=gen) for _ in "kv")
        kt = kt * groups * torch.where(some > 0, power(-16, 1, T, 1, 1, 1), torch.ones(1))
        vt = vt * power(-10, 10, T, H, d // g, 1) * torch.where(some > 0, power(-20, 20, T, 1, 1, 1), torch.ones(1))
        zero = torch.rand(T, 1, 1, 1, generator=gen) < 0.05
        k.append(kt.masked_fill(zero, 0.0).flatten(2).to(BF16))
        v.append(vt.masked_fill(zero.roll(1, 0) & (torch.arange(T) > 0).view(T, 1, 1, 1), 0.0).flatten(2).to(BF16))
        q = torch.randn(n, H, G, d // g, g, generator=gen) / groups[:, None]
        qs.append(q.view(n, H * G, d).to(BF16))
    h = Held(k, v, G=G, g=g, P=P, room=3000 * seed)
    out = h.attend(qs)
    for s, q in enumerate(qs):
        check(out[s], *h.expected(q, s))
    assert h.cache.stats() == {"device_timeouts": 0, "bad_pages": 0, "bad_lengths": 0}


@pytest.mark.parametrize("dtype, g, power", [(BF16, 32, 12), (BF16, 64, 26), (FP16, 32, 12)])
def test_the_tolerance_judges_every_group_by_its_own_values(dtype, g, power):
    """Results of zero, or off by a tenth, would not pass in the small groups either."""
    T, n, G = 200, 2, 4
    k, v, q = randn(1, T, 1, 128).to(dtype), randn(2, T, 1, 128) * 2.0 ** (-power // 2), randn(3, n, G, 128).to(dtype)
    v[..., :g] *= 2.0 ** power
    ref, tol = attention(q, k, v.to(dtype), g, T - n, 1 / math.sqrt(128), dtype)
    for group in (tol / ref.abs()).split(g, -1):
        assert group.median() < 0.06 and (group < 1).float().mean() > 0.95
