"""The 4-bit cache in 64 bits, for the tests: written from the format's definition, on the CPU."""
import math

import numpy as np
import torch

SCALE_MOST = 36.25 * 2.0 ** 120


def quantised(x, group):
    """x: [..., d] of a 16-bit type -> the values the cache stands for, fp64 (NaN for groups that are not finite)."""
    y = x.to(torch.float64).unflatten(-1, (-1, group))
    bad = ~torch.isfinite(y).all(-1, keepdim=True)
    y = torch.where(torch.isfinite(y), y, 0.0)
    scale = (y.abs().amax(-1, keepdim=True) / 7).to(torch.bfloat16).to(torch.float64).clamp(max=SCALE_MOST)
    codes = torch.where(scale > 0, y / torch.where(scale > 0, scale, 1.0), 0.0).round().clamp(-7, 7)
    return torch.where(bad, math.nan, codes * scale).flatten(-2)


class Rows:
    """Sequences, their pages and the rows of a call, on the CPU."""

    def __init__(self, lengths, page_size, seed=0, spare=3, max_pages=None):
        gen = torch.Generator().manual_seed(seed)
        self.lengths = list(lengths)
        pages = [-(-t // page_size) for t in lengths]
        self.n_pages = sum(pages) + spare
        order = torch.randperm(self.n_pages, generator=gen).to(torch.int32)
        self.table = torch.full((len(lengths), max_pages or max(1, max(pages))), -7, dtype=torch.int32)
        at = 0
        for s, n in enumerate(pages):
            self.table[s, :n] = order[at:at + n]
            at += n

    def device(self):
        return self.table.cuda(), torch.tensor(self.lengths, dtype=torch.int32).cuda()


def offsets_of(ns, start=0):
    return torch.tensor(np.concatenate([[start], start + np.cumsum(ns)]).astype(np.int32))


def attention(q, K, V, first_position, scale, out_type):
    """One sequence: q [n, H_q, d] (any type), K and V [T, H, d] fp64 as the cache stands for them (finite where a query that is
    compared sees them).  Query j sees positions up to first_position + j.  -> (out fp64 [n, H_q, d], lse in base 2 [n, H_q], tolerance per element).

    The tolerance bounds what a kernel does that is exact but for these roundings (A = sum of weight * |v| per channel):
      the result to its type                                  eps / 2 * |out|, at least half its smallest step
      each product weight * scale to fp16                     2^-11 * A   (relative half step of fp16)
                                                              + 2^-25 * tokens * vmax / l: half its smallest step, for
                                                              weights relative to the largest (l: their sum)
                                                              + 17 * 2^-23 * tokens / 16 * vmax: fp32 sums over 16 tokens each of
                                                              weight * scale * (c0 + 16 c1), |c0 + 16 c1| <= 119 = 17 * 7, two codes
                                                              to a product, and c0 as their difference
      scores: fp32 sums of d products of |q| with codes up to 15 and their offset 8 (the codes are stored + 8), every
      partial sum off by 2^-23 of the largest one: ds = 2^-23 * (d + 8) * 4 * sum|q| |k|max in base-2 units; it moves a
      weight by a factor 1 +- ds, numerator and denominator alike
      exp2 and the fp32 sums of weights and products          2^-19 * A   (2^-22 for exp2, and sums that are joined pairwise
                                                              and by tile: fewer than 8 roundings of 2^-24 in a row matter)
    """
    info = torch.finfo(out_type)
    n, hq, d = q.shape
    T, hk = K.shape[0], K.shape[1]
    q = q.to(torch.float64)
    out = torch.zeros(n, hq, d, dtype=torch.float64)
    tol = torch.zeros_like(out)
    lse = torch.full((n, hq), -math.inf, dtype=torch.float64)
    see = first_position + torch.arange(1, n + 1)                  # tokens that query j sees
    any_seen = see > 0
    hidden = torch.arange(T)[None] >= see[:, None]
    seen = torch.where(hidden, 0.0, 1.0)
    for h in range(hq):
        k, v = K[:, h // (hq // hk)], V[:, h // (hq // hk)]
        s = ((q[:, h] @ k.T) * scale * math.log2(math.e)).masked_fill(hidden, -math.inf)
        m = torch.where(any_seen, s.amax(-1) if T else torch.zeros(n, dtype=torch.float64), 0.0)
        w = torch.exp2(s - m[:, None])
        l = w.sum(-1)
        some = l > 0
        l1 = torch.where(some, l, 1.0)
        lse[:, h] = torch.where(some, m + torch.log2(l1), -math.inf)
        out[:, h] = (w @ v.nan_to_num()) / l1[:, None]
        A = (w @ v.nan_to_num().abs()) / l1[:, None]
        # the largest key and value that each query sees
        kmax = (seen * k.nan_to_num().abs().amax(-1)).amax(-1) if T else torch.zeros(n, dtype=torch.float64)
        vmax = (seen * v.nan_to_num().abs().amax(-1)).amax(-1) if T else torch.zeros(n, dtype=torch.float64)
        ds = 2.0 ** -23 * (d + 8) * 4 * q[:, h].abs().sum(-1) * kmax * scale * math.log2(math.e)
        steps = (see.clamp(min=0) + 15) // 16
        tol[:, h] = (info.eps / 2 * out[:, h].abs().clamp(min=info.smallest_normal) + (2.0 ** -11 + 2.0 ** -19 + 2 * ds[:, None]) * A
                     + ((2.0 ** -25 * see / l1 + 17 * 2.0 ** -23 * steps) * vmax)[:, None])
        tol[~any_seen, h] = 0.0
    return out, lse, tol
