"""Cases of the operators on a paged cache that holds keys and values in 4 bits.

Four things are measured: `append` (new rows are quantised into the cache and read back), `read` (whole sequences
are read back as 16-bit rows), `decode` (one query per sequence attends over the cache) and `positions` (several new
positions per sequence attend over it, causally).

The form of the cache: a row of `dim` channels of one token and KV head is cut into groups of `group` channels; a
group has scale = bf16(max|x| / 7) and codes round(x / scale), ties to even, in [-7, 7] (all 0 where the scale is 0),
and stands for code * scale.  Position t of a sequence lies in row t % page of physical page table[sequence, t // page].
New rows of a sequence of length T (the rows included) are its last positions: row j of n has position T - n + j, and
a query there sees the positions up to its own.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _case(name, op, seqs, shortest, longest, new=1, type="bf16", kv_heads=8, q_heads=32, dim=128, group=32, page=64, fused=False):
    return {"name": name, "op": op, "seqs": seqs, "shortest": shortest, "longest": longest, "new": new, "type": type,
            "kv_heads": kv_heads, "q_heads": q_heads, "dim": dim, "group": group, "page": page, "fused": fused}


def listed():
    return [
        # a decode step of 64 requests writes one row each: k and v are slices of the fused projection's output
        _case("append, 64 x 1", "append", 64, 2048, 65536, new=1, fused=True),
        # prompts of uneven lengths are written after their prefill
        _case("append, 8 prompts", "append", 8, 1021, 8191, new=0, type="fp16", page=16, fused=True),
        # a long prompt of one request
        _case("append, prompt of 65536", "append", 1, 65536, 65536, new=0),
        # short prefixes are read back for an attention that wants 16-bit rows (64 channels per head)
        _case("read, 16 short", "read", 16, 33, 1000, type="fp16", kv_heads=4, q_heads=28, dim=64, group=64, page=32),
        # a context of 128K tokens is read back whole (Qwen3-32B shapes)
        _case("read, 128K", "read", 1, 131072, 131072, q_heads=64),
        # the smallest decode step: one request, one KV head, four query heads
        _case("decode, 1 x 1024", "decode", 1, 1024, 1024, kv_heads=1, q_heads=4),
        # Llama-3-8B shapes, eight requests of 32K
        _case("decode, 8 x 32K", "decode", 8, 32768, 32768),
        # Qwen3-32B shapes, one request of 128K
        _case("decode, 1 x 128K", "decode", 1, 131072, 131072, q_heads=64),
        # a ragged serving batch on small pages
        _case("decode, 32 ragged", "decode", 32, 512, 16384, type="fp16", group=64, page=16),
        # a speculative step: four new positions of each of eight requests
        _case("positions, 8 x 4", "positions", 8, 32768, 32768, new=4),
        # a chunk of a prefill against the context before it
        _case("positions, chunk of 2048", "positions", 1, 32768, 32768, new=2048),
        # a few dozen positions of ragged requests, 64 channels per head, seven query heads per KV head
        _case("positions, 5 x 37", "positions", 5, 37, 4001, new=37, type="fp16", kv_heads=4, q_heads=28, dim=64, group=32, page=32),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "read", "decode", "positions"])
    dim = rng.choice([64, 128])
    case = {"op": op, "type": rng.choice(["bf16", "fp16"]), "dim": dim, "group": rng.choice([32, 64, dim]),
            "page": rng.choice([16, 32, 64]), "kv_heads": rng.choice([1, 2, 4, 5, 8]), "fused": rng.random() < 0.5}
    case["q_heads"] = case["kv_heads"] * rng.randint(1, 8)
    new = {"append": rng.choice([0, 1, _log_int(rng, 1, 4096)]), "read": 0, "decode": 1,
           "positions": _log_int(rng, 2, 2048)}[op]
    case["longest"] = max(new, _log_int(rng, 64, 65536))
    case["shortest"] = max(1, new, _log_int(rng, 1, case["longest"]))
    # rows of all sequences up to 262144, query rows x tokens up to those of the listed chunk
    most = max(1, 262144 // case["longest"])
    if op == "positions":
        most = max(1, min(most, 2048 * 32768 * 32 // (case["longest"] * new * case["q_heads"])))
    case["seqs"] = _log_int(rng, 1, min(64, most))
    case["new"] = new
    return case


def _shape(case):
    """(length of each sequence, new rows of each sequence): the same for every seed."""
    rng = random.Random("%d %d %d" % (case["seqs"], case["shortest"], case["longest"]))
    lens = [_log_int(rng, case["shortest"], case["longest"]) for _ in range(case["seqs"])]
    return lens, [case["new"] if case["new"] else n for n in lens]


def work(case):
    lens, new = _shape(case)
    d, hk, hq, g = case["dim"], case["kv_heads"], case["q_heads"], case["group"]
    held = hk * 2 * (d / 2 + 2 * d / g)                  # bytes of a token in the cache, keys and values
    if case["op"] == "append":                           # rows in, cache written, rows back out
        return {"bytes": sum(new) * (2 * hk * d * 2 * 2 + held), "flops": 0}
    if case["op"] == "read":
        return {"bytes": sum(lens) * (held + 2 * hk * d * 2), "flops": 0}
    seen = sum(n * t - n * (n - 1) // 2 for t, n in zip(lens, new))
    return {"bytes": sum(lens) * held + 2 * sum(new) * hq * d * 2, "flops": 4 * seen * hq * d}


def _draws(case, seed):
    """The inputs of a seed, on the GPU: rows of the whole sequences (or the new rows alone for `append`) and queries."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype, d, hk, hq = DTYPES[case["type"]], case["dim"], case["kv_heads"], case["q_heads"]
    lens, new = _shape(case)
    rows = sum(new) if case["op"] == "append" else sum(lens)
    # keys have channels of very different sizes, values have not
    channel = torch.exp(torch.rand(hk, d, generator=gen, device="cuda") * math.log(16.0) + math.log(0.5))
    if case["fused"] and case["op"] == "append":         # slices of [rows, q | k | v]
        x = torch.randn(rows, hq + 2 * hk, d, generator=gen, device="cuda", dtype=dtype)
        k, v = x[:, hq:hq + hk], x[:, hq + hk:]
        k.mul_(channel)
    else:
        k = torch.randn(rows, hk, d, generator=gen, device="cuda", dtype=dtype).mul_(channel)
        v = torch.randn(rows, hk, d, generator=gen, device="cuda", dtype=dtype)
    q = torch.randn(sum(new), hq, d, generator=gen, device="cuda", dtype=dtype)
    P = case["page"]
    pages = [-(-t // P) for t in lens]
    order = torch.randperm(sum(pages) + 3, generator=gen, device="cuda")
    at = [0] + [int(x) for x in np.cumsum(pages)]
    table = torch.zeros(len(lens), max(pages), dtype=torch.int32, device="cuda")
    for i, n in enumerate(pages):
        table[i, :n] = order[at[i]:at[i] + n]
    return k, v, q, table, sum(pages) + 3


def prepare(case, seed):
    lens, new = _shape(case)
    k, v, q, table, n_pages = _draws(case, seed)
    d, hk, g, P = case["dim"], case["kv_heads"], case["group"], case["page"]
    ints = lambda xs: torch.tensor(xs, dtype=torch.int32, device="cuda")  # noqa: E731
    first = lambda ns: ints([0] + [int(x) for x in np.cumsum(ns)])        # noqa: E731
    state = {"op": case["op"], "page": P, "group": g, "table": table, "lengths": ints(lens), "offsets": first(new),
             "scale": 1 / math.sqrt(d), "heads": hk}
    whole = first(lens)
    if own:
        from paper_2608_23843_b200 import pkv
        cfg = pkv.make_q4_config(n_kv_heads=hk, n_q_heads=case["q_heads"], head_dim=d, page_size=P, group_size=g,
                                 dtype=DTYPES[case["type"]], n_pages=n_pages)
        state["cache"] = cache = pkv.Q4Cache(cfg)
        if case["op"] != "append":
            cache.append_kv(table, state["lengths"], k, v, whole)
    else:
        state["store"] = tuple(torch.zeros(n_pages, P, hk, *s, dtype=t, device="cuda")
                               for _ in "kv" for s, t in (((d,), torch.int8), ((d // g,), torch.bfloat16)))
        if case["op"] != "append":
            _write(state["store"], _rows(state, whole, k.shape[0]), k, v, g)
    if case["op"] == "append":
        state["k"], state["v"] = k, v
    if case["op"] in ("append", "read"):
        state["k_out"], state["v_out"] = torch.empty_like(k, memory_format=torch.contiguous_format), torch.empty_like(v, memory_format=torch.contiguous_format)
        if case["op"] == "read":
            state["offsets"] = whole
    else:
        state["q"] = q.view(len(lens), new[0], case["q_heads"], d)
    return state


def run(state):
    if own:
        cache, table, lengths = state["cache"], state["table"], state["lengths"]
        if state["op"] in ("append", "read"):
            if state["op"] == "append":
                cache.append_kv(table, lengths, state["k"], state["v"], state["offsets"])
            cache.read_kv(table, lengths, state["k_out"], state["v_out"], state["offsets"])
            return state["k_out"], state["v_out"]
        return cache.attention(table, lengths, state["q"])
    if state["op"] in ("append", "read"):
        rows = _rows(state, state["offsets"], state["k_out"].shape[0])
        if state["op"] == "append":
            _write(state["store"], rows, state["k"], state["v"], state["group"])
        kc, ks, vc, vs = (x[rows] for x in state["store"])
        return _values(kc, ks).to(state["k_out"].dtype), _values(vc, vs).to(state["v_out"].dtype)
    return _attend(state)


# ---- plain form ---------------------------------------------------------------------------------------------------
def _rows(state, offsets, n):
    """(physical page, row in it) of each of the n new rows."""
    row = torch.arange(n, device="cuda")
    seq = torch.searchsorted(offsets.long(), row, right=True) - 1
    pos = state["lengths"].long()[seq] - (offsets.long()[seq + 1] - row)
    return state["table"].long()[seq, pos // state["page"]], pos % state["page"]


def _quantised(x, group):
    x = x.float().unflatten(-1, (-1, group))
    scale = (x.abs().amax(-1) / 7).to(torch.bfloat16)
    s = scale.float().unsqueeze(-1)
    codes = torch.where(s > 0, x / torch.where(s > 0, s, 1.0), 0.0).round().clamp(-7, 7)
    return codes.flatten(-2).to(torch.int8), scale


def _write(store, rows, k, v, group):
    kc, ks, vc, vs = store
    kc[rows], ks[rows] = _quantised(k, group)
    vc[rows], vs[rows] = _quantised(v, group)


def _values(codes, scale):
    return (codes.float().unflatten(-1, (scale.shape[-1], -1)) * scale.float().unsqueeze(-1)).flatten(-2)


def _attend(state):
    q, table, T = state["q"], state["table"].long(), state["lengths"].long()
    hk, (S, n, hq, d) = state["heads"], q.shape
    G = hq // hk
    x = q.float().view(S, n, hk, G, d).permute(0, 2, 1, 3, 4).reshape(S, hk, n * G, d)
    kc, ks, vc, vs = (c[table].flatten(1, 2).transpose(1, 2) for c in state["store"])      # [S, H, tokens, ...]
    s = torch.matmul(x, _values(kc, ks).transpose(-1, -2)).mul_(state["scale"])
    t = torch.arange(s.shape[-1], device="cuda")
    last = T[:, None] - n + torch.arange(n, device="cuda")                                 # the last position a query sees
    hidden = (t > last[..., None]).repeat_interleave(G, 1)[:, None]
    s = s.masked_fill_(hidden, -math.inf)
    p = s.sub_(s.amax(-1, keepdim=True)).exp_()
    o = torch.matmul(p, _values(vc, vs)) / p.sum(-1, keepdim=True)
    return o.view(S, hk, n, G, d).permute(0, 2, 1, 3, 4).reshape(q.shape).to(q.dtype)


# ---- the definition in 64 bits ---------------------------------------------------------------------------------------
def exact(case, seed):
    lens, new = _shape(case)
    k, v, q, _, _ = _draws(case, seed)
    d, g, hk = case["dim"], case["group"], case["kv_heads"]

    def held(x):                                         # what the cache stands for, one group per row
        y = x.double().reshape(-1, g)
        step = (y.abs().max(dim=1, keepdim=True).values / 7).to(torch.bfloat16).double()
        n = torch.round(y / step.clamp_min(1e-300)).clamp(-7, 7)
        return (n * step).reshape(x.shape)

    if case["op"] in ("append", "read"):
        return held(k), held(v)
    out = torch.empty(q.shape, dtype=torch.float64, device="cuda")
    t0 = r0 = 0
    for T, n in zip(lens, new):
        K, V = held(k[t0:t0 + T]), held(v[t0:t0 + T])
        see = torch.arange(T, device="cuda")[None] <= torch.arange(T - n, T, device="cuda")[:, None]
        for h in range(case["q_heads"]):
            kv = h // (case["q_heads"] // hk)
            z = (q[r0:r0 + n, h].double() @ K[:, kv].T / math.sqrt(d)).masked_fill_(~see, -math.inf)
            out[r0:r0 + n, h] = torch.softmax(z, dim=1) @ V[:, kv]
        t0, r0 = t0 + T, r0 + n
    return out.view(len(lens), new[0], case["q_heads"], d)
