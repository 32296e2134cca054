"""Attention over a part of the positions, trees of drafted tokens, kept rows and planned steps of the 4-bit cache: the definitions in 64 bits (or
whole numbers), on the CPU, one sequence and one row at a time."""
import math

import torch


def window_seen(T, n, window, sinks):
    """[n, T]: which positions the last n positions of T see."""
    p = torch.arange(T - n, T)[:, None]
    t = torch.arange(T)[None]
    see = t <= p
    if window:
        see = see & ((t > p - window) | (t < sinks))
    return see


def tree_bits(parents, C=0, window=0, sinks=0):
    """Which rows each row of one sequence sees [n, n], and depths, from the definition."""
    n = len(parents)
    see = torch.zeros(n, n, dtype=torch.bool)
    depths = []
    for j in range(n):
        branch, i = [], j
        while i >= 0:
            branch.append(i)
            i = parents[i]
        depth = len(branch) - 1
        depths.append(depth)
        for back, i in enumerate(branch):
            see[j, i] = not window or back < window or C + depth - back < sinks
    return see, depths


def tree_seen(T, bits, window=0, sinks=0):
    """[n, T]: what rows with such masks (bool [n, n]) see."""
    n = bits.shape[0]
    C, t = T - n, torch.arange(T)
    see = torch.zeros(n, T, dtype=torch.bool)
    for j in range(n):
        low = max(0, C + max(1, int(bits[j].sum())) - window) if window else 0
        see[j] = (t >= low) | (t < sinks)
        see[j, max(C, 0):] = bits[j, max(0, -C):]
    return see


def pack(bits, words=None):
    """bool [n, n] -> int64 [n, words]."""
    n = bits.shape[0]
    words = words or max(1, -(-n // 64))
    out = torch.zeros(n, words, dtype=torch.int64)
    for i in range(bits.shape[1]):
        bit = -(1 << 63) if i % 64 == 63 else 1 << (i % 64)
        out[:, i // 64] |= torch.where(bits[:, i], bit, 0)
    return out


def attention_seen(q, K, V, see, scale, out_type):
    """One sequence: q [n, H_q, d], K and V [T, H, d] fp64 as the cache stands for them, see [n, T] bool.
    -> (out fp64, log2 of the sum of weights, tolerance per element).  The tolerance is that of q4_reference.attention():
      the result to its type             eps / 2 * |out|, at least half its smallest step
      weight * scale to fp16             2^-11 * A + 2^-25 * tokens * vmax / l       (A: sum of weight * |v|; l: sum of weights)
      fp32 sums over a tile of 16        17 * 2^-23 * tiles * vmax, for the tiles that hold a token that is seen
      scores                             2 ds A, ds = 2^-23 (d + 8) 4 sum|q| |k|max in base 2
      exp2, fp32 sums                    2^-19 * A
    """
    info = torch.finfo(out_type)
    n, hq, d = q.shape
    T, hk = K.shape[0], K.shape[1]
    q = q.to(torch.float64)
    out = torch.zeros(n, hq, d, dtype=torch.float64)
    tol = torch.zeros_like(out)
    lse = torch.full((n, hq), -math.inf, dtype=torch.float64)
    if T == 0:
        return out, lse, tol
    some = see.any(-1)
    seen = see.to(torch.float64)
    count = seen.sum(-1)
    tiles = torch.nn.functional.pad(see, (0, -T % 16)).view(n, -1, 16).any(-1).sum(-1).to(torch.float64)
    for h in range(hq):
        k, v = K[:, h // (hq // hk)].nan_to_num(), V[:, h // (hq // hk)].nan_to_num()
        s = ((q[:, h] @ k.T) * scale * math.log2(math.e)).masked_fill(~see, -math.inf)
        m = torch.where(some, s.amax(-1), 0.0)
        w = torch.exp2(s - m[:, None])
        l = w.sum(-1)
        l1 = torch.where(some, l, 1.0)
        lse[:, h] = torch.where(some, m + torch.log2(l1), -math.inf)
        out[:, h] = (w @ v) / l1[:, None]
        A = (w @ v.abs()) / l1[:, None]
        kmax, vmax = (seen * k.abs().amax(-1)).amax(-1), (seen * v.abs().amax(-1)).amax(-1)
        ds = 2.0 ** -23 * (d + 8) * 4 * q[:, h].abs().sum(-1) * kmax * scale * math.log2(math.e)
        tol[:, h] = (info.eps / 2 * out[:, h].abs().clamp(min=info.smallest_normal) + (2.0 ** -11 + 2.0 ** -19 + 2 * ds[:, None]) * A
                     + ((2.0 ** -25 * count / l1 + 17 * 2.0 ** -23 * tiles) * vmax)[:, None])
        tol[~some, h] = 0.0
    return out, lse, tol


class Plan:
    """A step's plan in whole numbers.  Pages and requests as lists; `step` changes them, or nothing."""

    def __init__(self, page, n_pages, max_pages, table, lengths, spans, ring, head, tail):
        self.page, self.n_pages, self.max_pages = page, n_pages, max_pages
        self.table, self.lengths, self.spans, self.ring = [list(r) for r in table], list(lengths), [tuple(x) for x in spans], list(ring)
        self.head, self.tail = head, tail

    def step(self, rows, capacity, window=0, sinks=0):
        """-> (missing, refused, offsets, positions, slots)"""
        P = self.page
        su = -(-sinks // P) if window else 0
        refused = sum(n < -1 or T < 0 or T + max(n, 0) > self.max_pages * P or not 0 <= a <= b <= self.max_pages
                      for n, T, (a, b) in zip(rows, self.lengths, self.spans))
        good = [n >= -1 and T >= 0 and T + max(n, 0) <= self.max_pages * P and 0 <= a <= b <= self.max_pages
                for n, T, (a, b) in zip(rows, self.lengths, self.spans)]
        new = [max(n, 0) if ok else 0 for n, ok in zip(rows, good)]
        refused += sum(new) > capacity
        taken, back = [], []
        for s, (n, T, (first, end)) in enumerate(zip(rows, self.lengths, self.spans)):
            if not good[s]:
                continue
            if n < 0:
                back += [(s, e) for e in range(end) if e < su or e >= first]
            else:
                if window:
                    back += [(s, e) for e in range(max(first, su), end) if (e + 1) * P <= T + 1 - window]
                taken += [(s, e) for e in range(end, -(-(T + n) // P))]
        free = self.tail - self.head
        ring_ok = self.head >= 0 and 0 <= free <= self.n_pages and free + len(back) <= self.n_pages
        refused += not ring_ok
        missing = max(0, len(taken) - free) if ring_ok else 0
        nothing = [0] * (len(rows) + 1)
        if refused or missing:
            return missing, refused, nothing, [], []
        for k, (s, e) in enumerate(back):
            self.ring[(self.tail + k) % self.n_pages] = self.table[s][e]
            if rows[s] >= 0:
                self.spans[s] = (e + 1, self.spans[s][1])
        for k, (s, e) in enumerate(taken):
            self.table[s][e] = self.ring[(self.head + k) % self.n_pages]
            self.spans[s] = (self.spans[s][0], e + 1)
        self.head += len(taken)
        self.tail += len(back)
        offsets, positions, slots = [0], [], []
        for s, n in enumerate(new):
            for t in range(self.lengths[s], self.lengths[s] + n):
                page = self.table[s][t // P]
                positions.append(t)
                slots.append(page * P + t % P if 0 <= page < self.n_pages else -1)
            offsets.append(offsets[-1] + n)
            self.lengths[s] += n
            if rows[s] < 0:
                self.lengths[s], self.spans[s] = 0, (0, 0)
        return 0, 0, offsets, positions, slots


def attention_precise(q, k, v, group, see, scale, out_type):
    """q4_precision_reference.attention() - every channel judged by its own group's values, the same roundings counted - for queries that
    see what `see` says ([n, T] bool, something each).  k, v: as they were written, finite where a query sees them."""
    from q4_precision_reference import group_scales
    from q4_reference import quantised
    info = torch.finfo(out_type)
    n, hq, d = q.shape
    T, hk, _ = k.shape
    some = see.any(0)
    k, v = (torch.where(some[:, None, None], x, torch.zeros((), dtype=x.dtype)) for x in (k, v))
    K, V, S = quantised(k, group), quantised(v, group), group_scales(v, group)
    q = q.to(torch.float64)
    to2 = scale * math.log2(math.e)
    out, tol = torch.empty(n, hq, d, dtype=torch.float64), torch.empty(n, hq, d, dtype=torch.float64)
    assert see.any(-1).all()
    seen = see.to(torch.float64)
    count = seen.sum(-1, keepdim=True)
    runs = torch.nn.functional.pad(see, (0, -T % 16)).view(n, -1, 16).any(-1).sum(-1, keepdim=True).to(torch.float64)
    for h in range(hq):
        kk, vv, ss = (x[:, h // (hq // hk)] for x in (K, V, S))
        s = ((q[:, h] @ kk.T) * to2).masked_fill(~see, -math.inf)
        w = torch.exp2(s - s.amax(-1, keepdim=True))
        l = w.sum(-1, keepdim=True)
        out[:, h] = w @ vv / l
        A = w @ vv.abs() / l
        star = ss.amax(-1)
        per_group = torch.stack([(w * ss[:, i]).amax(-1) for i in range(ss.shape[1])], -1) / l
        own = (7 * 2.0 ** -26 * count * per_group).repeat_interleave(group, -1)
        ratio = vv.abs() / star.clamp(min=1e-300)[:, None]
        alike = 2.0 ** -25 * ((w * star).amax(-1, keepdim=True) / l) * (seen @ ratio)
        sums = (119 * 2.0 ** -20 * runs * (w @ ss) / l).repeat_interleave(group, -1)
        size = (((q[:, h].abs() @ kk.abs().T) * to2) * seen).amax(-1, keepdim=True)
        ds = (2.0 ** -20 * d / 16 + 2.0 ** -23 * d / group) * size + 2.0 ** -22 * (size + 64)
        tol[:, h] = (info.eps / 2 * out[:, h].abs().clamp(min=info.smallest_normal) + (2.0 ** -11 + 2.0 ** -19 + 2 * ds) * A +
                     torch.maximum(own, alike) + sums)
    return out, tol
