"""Attention of windows and trees over the 4-bit cache where numbers of very different sizes meet, on each kernel: every channel is judged by its own group's
values; what a query does not see, of any size or not finite, must not matter to it."""
import math
import random

import pytest
import torch

from q4_reference import offsets_of  # noqa: F401
from q4_select_reference import attention_precise, tree_bits, tree_seen, window_seen
from test_q4_precision import Held, check
from test_q4_serve import INTS, ROUTES, _route, random_parents

BF16, FP16 = torch.bfloat16, torch.float16
NAMES = ["small, clusters of 8", "small, a tree and a window", "even shares, 8 rows", "even shares, 16 rows", "row blocks, halves in turn",
         "row blocks, halves in turn, a window", "row blocks, both halves", "row blocks, a tree over several"]
CASES = [r for r in ROUTES if r[0] in NAMES]
assert len(CASES) == len(NAMES)


def sizes(gen, shape, lo, hi):
    return torch.exp2(torch.randint(lo, hi + 1, shape, generator=gen).float())


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["each token and group", "a group", "every other token", "zeros", "hidden ones large", "hidden ones not finite"])
@pytest.mark.parametrize("dtype, d, g", [(BF16, 128, 32), (FP16, 64, 32), (FP16, 128, 64)])
@pytest.mark.parametrize("name, shape, S, n, T, kw, kernel, cluster", CASES, ids=[r[0] for r in CASES])
def test_numbers_of_different_sizes(name, shape, S, n, T, kw, kernel, cluster, dtype, d, g, kind):
    H, G = shape["H"], shape["G"]
    gen, rng = torch.Generator().manual_seed(len(name) + d), random.Random(n)
    W, sinks, tree = kw.get("window", 0), kw.get("sinks", 0), kw.get("tree", False)
    parents = [random_parents(rng, n, 6) for _ in range(S)]
    see = [tree_seen(T, tree_bits(parents[s], T - n, W, sinks)[0], W, sinks) if tree else window_seen(T, n, W, sinks) for s in range(S)]
    ks, vs = [], []
    for s in range(S):
        k, v = torch.randn(T, H, d, generator=gen), torch.randn(T, H, d, generator=gen)
        some = see[s].any(0)
        if kind == "each token and group":
            k *= sizes(gen, (T, H, d // g, 1), -9, 1).expand(T, H, d // g, g).reshape(T, H, d)
            v *= sizes(gen, (T, H, d // g, 1), -10, 10).expand(T, H, d // g, g).reshape(T, H, d)
        elif kind == "a group":
            k[..., :g] *= 2.0 ** -7
            v[..., :g] *= 2.0 ** 9
        elif kind == "every other token":
            k[::2] *= 2.0 ** -12
            v[1::2] *= 2.0 ** 7
        elif kind == "zeros":
            v[rng.randint(0, 3)::3] = 0.0
            k[::5] = 0.0
        elif kind == "hidden ones large":
            k[~some] *= 2.0 ** 6
            v[~some] *= 2.0 ** 9
        else:
            k[~some], v[~some] = math.nan, math.inf
        ks.append(k.to(dtype))
        vs.append(v.to(dtype))
    h = Held(ks, vs, G=G, g=g, P=64, room=T, n_ctas=shape.get("n_ctas", 0))
    if d == 128:
        assert _route(h.cache, S, n, h.table.shape[1] * 64, kw)[0] == kernel
    qs = [torch.randn(n, H * G, d, generator=gen).to(dtype) for _ in range(S)]
    masks = h.cache.tree_masks(torch.tensor(parents, **INTS).cuda(), h.lengths, window=W, sinks=sinks)[0] if tree else None
    out = h.attend(qs, window=W, sinks=sinks, tree=masks)
    for s in range(S):
        check(out[s], *attention_precise(qs[s], ks[s], vs[s], g, see[s], 1 / math.sqrt(d), dtype))
    assert h.cache.stats() == {"device_timeouts": 0, "bad_pages": 0, "bad_lengths": 0}


@pytest.mark.gpu
@pytest.mark.parametrize("name, shape, S, n, T, kw, kernel, cluster", CASES, ids=[r[0] for r in CASES])
def test_a_value_that_is_not_finite_makes_its_group_not_a_number_where_it_is_seen(name, shape, S, n, T, kw, kernel, cluster):
    H, G, d, g = shape["H"], shape["G"], 128, 32
    gen, rng = torch.Generator().manual_seed(len(name)), random.Random(n)
    W, sinks, tree = kw.get("window", 0), kw.get("sinks", 0), kw.get("tree", False)
    parents = random_parents(rng, n, 6)
    see = tree_seen(T, tree_bits(parents, T - n, W, sinks)[0], W, sinks) if tree else window_seen(T, n, W, sinks)
    k, v = (torch.randn(T, H, d, generator=gen).to(BF16) for _ in "kv")
    bad = v.clone()
    hit = T - n + (1 if n > 1 else 0)                      # a new row that some of the others may not see
    bad[hit, 0, 2 * g + 5] = math.inf
    h = Held([bad], [bad], G=G, g=g, P=64, room=T, n_ctas=shape.get("n_ctas", 0))
    h.cache.append_kv(h.table, h.lengths, k[None].cuda(), bad[None].cuda())
    q = torch.randn(n, H * G, d, generator=gen).to(BF16)
    masks = h.cache.tree_masks(torch.tensor([parents], **INTS).cuda(), h.lengths, window=W, sinks=sinks)[0] if tree else None
    out = h.attend([q], window=W, sinks=sinks, tree=masks)[0]
    hits = see[:, hit]
    assert hits.any()
    assert torch.isnan(out[hits][:, :G, 2 * g:3 * g]).all()
    out[hits, :G, 2 * g:3 * g] = 0.0
    ref, tol = attention_precise(q, k, v, g, see, 1 / math.sqrt(d), BF16)
    keep = torch.ones_like(ref, dtype=torch.bool)
    keep[hits, :G, 2 * g:3 * g] = False
    check(out[keep], ref[keep], tol[keep])
