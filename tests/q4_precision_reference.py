"""Attention over the 4-bit cache in 64 bits, with a tolerance that judges every channel by the values of its own group."""
import math

import torch

from q4_reference import SCALE_MOST, quantised


def group_scales(x, group):
    """[T, H, d] -> the scales of the channel groups, fp64 [T, H, d / group] (finite rows)."""
    y = x.to(torch.float64).unflatten(-1, (-1, group)).abs().amax(-1) / 7
    return y.to(torch.bfloat16).to(torch.float64).clamp(max=SCALE_MOST)


def attention(q, k, v, group, first_position, scale, out_type, steps=None):
    """One sequence: q [n, H_q, d], k and v [T, H, d] as they were written (finite where a query sees them); query j sees positions up to
    first_position + j, at least one.  -> (out fp64 [n, H_q, d], tolerance).  `steps`: runs of 16 tokens that one set of
    accumulators takes at most (default: all of them).

    With w a query's weights relative to its largest, l their sum, S the scale of a value's group, S* the largest scale of the
    value's row, and A = sum of w |value| / l per channel, a kernel's result may be off by
      the result's rounding to its type            eps / 2 of it
      weights (times S) rounded to fp16            2^-11 A
      ... those that are too small for that        fp16's smallest step is 2^-24, half of it 2^-25.  A kernel that places the largest w S of
                                                   a query and channel group at 2 or above: 2^-26 max(w S) on each of w S, 7 times that in
                                                   a sum with codes.  One that has weights for all groups alike and brings values to fp16
                                                   with a power of two 2^E for a run of tokens, 2^(E - 4) <= S* < 2^(E + 1), its largest
                                                   weight times 2^E at 2^5 or above: the largest w S* is 2^(5 - 4) of those units or more, a weight
                                                   is off by 2^-25 2^-E of them, so w S* by 2^-25 max(w S*) and the product with a
                                                   value by 2^-25 max(w S*) |value| / S*
      fp32 sums                                    a run of 16 products and the sum so far are aligned to the largest of the 17 and lose
                                                   less than 2^-25 of it each: 17 * 2^-25 < 2^-20 of sum(w S |c0 + 16 c1|) / l per run, with
                                                   |c0 + 16 c1| <= 119: two neighbouring codes share a product; c0 is a difference of sums.
                                                   exp2 and the joins of states: 2^-19 A
      the scores, by ds in base 2: weights change by a factor 1 +- ds, so does l: 2 ds A.  Products of queries and codes are exact
                                                   (each of the d / 16 runs of 16 loses up to 2^-20 of sum(|q| |k|), the sum over groups
                                                   2^-23 of it per group); the factors and exponents that follow round 2^-23 of a number up
                                                   to |score| + 64 twice
    """
    info = torch.finfo(out_type)
    n, hq, d = q.shape
    T, hk, _ = k.shape
    K, V, S = quantised(k, group), quantised(v, group), group_scales(v, group)
    q = q.to(torch.float64)
    to2 = scale * math.log2(math.e)
    out, tol = torch.empty(n, hq, d, dtype=torch.float64), torch.empty(n, hq, d, dtype=torch.float64)
    see = first_position + torch.arange(1, n + 1)
    assert (see > 0).all()
    hidden = torch.arange(T)[None] >= see[:, None]
    runs = ((see + 15) // 16).clamp(max=steps or T).to(torch.float64)[:, None]
    for h in range(hq):
        kk, vv, ss = (x[:, h // (hq // hk)] for x in (K.nan_to_num(), V.nan_to_num(), S))
        s = ((q[:, h] @ kk.T) * to2).masked_fill(hidden, -math.inf)
        w = torch.exp2(s - s.amax(-1, keepdim=True))
        l = w.sum(-1, keepdim=True)
        out[:, h] = w @ vv / l
        A = w @ vv.abs() / l
        star = ss.amax(-1)
        per_group = torch.stack([(w * ss[:, i]).amax(-1) for i in range(ss.shape[1])], -1) / l               # max(w S) / l
        own = (7 * 2.0 ** -26 * see[:, None] * per_group).repeat_interleave(group, -1)
        ratio = vv.abs() / star.clamp(min=1e-300)[:, None]
        alike = 2.0 ** -25 * ((w * star).amax(-1, keepdim=True) / l) * ((~hidden).to(torch.float64) @ ratio)
        sums = (119 * 2.0 ** -20 * runs * (w @ ss) / l).repeat_interleave(group, -1)
        size = ((q[:, h].abs() @ kk.abs().T) * to2).masked_fill(hidden, 0.0).amax(-1, keepdim=True)
        ds = (2.0 ** -20 * d / 16 + 2.0 ** -23 * d / group) * size + 2.0 ** -22 * (size + 64)
        tol[:, h] = (info.eps / 2 * out[:, h].abs().clamp(min=info.smallest_normal) + (2.0 ** -11 + 2.0 ** -19 + 2 * ds) * A +
                     torch.maximum(own, alike) + sums)
    return out, tol
