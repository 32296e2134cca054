"""Cases of the operators around serving from the paged 4-bit cache: attention over a sliding window with sinks, attention of a
tree of drafted tokens, keeping the accepted rows of a tree, and the planning of a step's pages on the GPU.

The form of the cache: a row of `dim` channels of one token and KV head is cut into groups of `group` channels; a
group has scale = bf16(max|x| / 7) and codes round(x / scale), ties to even, in [-7, 7] (all 0 where the scale is 0),
and stands for code * scale.  Position t of a sequence lies in row t % page of physical page table[sequence, t // page].
A sequence of length T has n new rows, its last positions; the C = T - n tokens before them are its context.

`window`: the query of row j is at position p = C + j and sees the positions t <= p with t > p - window, and those with
t < sinks.  Pages that hold no such position have gone back to the pool: their table entries are -1.

`tree`: the new rows are drafted tokens; parents[j] < j is the row that row j continues, -1 stands for the last token of the
context.  A row sees itself, its ancestors and the context.  With a window, its position is C + depth, and it sees what lies in
the window (an ancestor's position being C + its depth) or below `sinks`.  Results: the attention and the rows' depths.

`keep`: of each sequence's n drafted rows those of an accepted path (row numbers that ascend) become the sequence's first
new rows, in order, and its length becomes C + the path's length.  A pass writes the drafted rows, keeps, and reads the kept
rows back; results: the rows kept, as the values the cache stands for, and the lengths.

`plan`: request s has length T and table entries [first, end) of the pages it holds (and the pages of its sinks).  rows[s] >= 0
new rows are asked for: length T + rows, pages for them from a ring of free pages (from its head, requests in order, then their
pages in order), end = max(end, ceil(length / page)).  rows[s] = -1: the request is done, its pages go back, length and
entries become 0.  With a window, pages that lie wholly below T + 1 - window and behind the sinks' pages go back too, and
`first` moves up.  What goes back is written behind the ring's tail (requests in order, their pages in order) and is not given out in
the same step.  Results: lengths, offsets of the rows (prefix sums), position and slot (page * page size + row in it) of every row,
entries held, the ring's (head, tail, pages missing, requests refused), ring and table.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _case(name, op, seqs, shortest, longest, new=1, type="bf16", kv_heads=8, q_heads=32, dim=128, group=32, page=64, window=0, sinks=0,
          done=0.0):
    return {"name": name, "op": op, "seqs": seqs, "shortest": shortest, "longest": longest, "new": new, "type": type,
            "kv_heads": kv_heads, "q_heads": q_heads, "dim": dim, "group": group, "page": page, "window": window, "sinks": sinks,
            "done": done}


def listed():
    return [
        # the smallest decode step of a windowed layer: one request, one KV head, four query heads
        _case("window, decode 1 x 2048", "window", 1, 2048, 2048, kv_heads=1, q_heads=4, window=512, sinks=4),
        # Llama-3-8B shapes with a window of 4096: eight requests of 32K
        _case("window, decode 8 x 32K", "window", 8, 32768, 32768, window=4096, sinks=4),
        # a ragged serving batch on small pages, some requests shorter than the window
        _case("window, decode 64 ragged", "window", 64, 256, 65536, type="fp16", group=64, page=16, window=1024, sinks=16),
        # a chunk of a prefill in a windowed layer
        _case("window, chunk of 2048", "window", 1, 32768, 32768, new=2048, window=4096, sinks=64),
        # a small draft of one request
        _case("tree, 1 x 7", "tree", 1, 1500, 1500, new=7, kv_heads=2, q_heads=8),
        # Llama-3-8B shapes, eight requests of 32K with 64 drafted tokens each
        _case("tree, 8 x 64", "tree", 8, 32768, 32768, new=64),
        # a ragged batch of a model with 64 channels per head and windowed layers
        _case("tree, 16 x 25 windowed", "tree", 16, 300, 20000, new=25, type="fp16", kv_heads=4, q_heads=28, dim=64, page=32,
              window=2048, sinks=4),
        # after the verification of eight requests' trees
        _case("keep, 8 x 64", "keep", 8, 32768, 32768, new=64),
        # a large batch of small drafts
        _case("keep, 128 x 13", "keep", 128, 100, 4000, new=13, type="fp16", kv_heads=4, q_heads=28, dim=64, group=64, page=16),
        # a decode step of 64 requests
        _case("plan, 64 x 1", "plan", 64, 100, 32768, new=1),
        # a step that mixes decodes, chunks of prompts and finished requests, windowed, on small pages
        _case("plan, 700 mixed", "plan", 700, 1, 32768, new=1500, page=16, window=4096, sinks=4, done=0.1),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["window", "tree", "keep", "plan"])
    dim = rng.choice([64, 128])
    case = {"op": op, "type": rng.choice(["bf16", "fp16"]), "dim": dim, "group": rng.choice([32, 64, dim]),
            "page": rng.choice([16, 32, 64]), "kv_heads": rng.choice([1, 2, 4, 5, 8]), "done": 0.0}
    case["q_heads"] = case["kv_heads"] * rng.randint(1, 8)
    windowed = op == "window" or rng.random() < 0.4
    case["window"] = _log_int(rng, 16, 8192) if windowed else 0
    case["sinks"] = rng.choice([0, 1, 4, 16, 64, _log_int(rng, 1, 300)]) if windowed else 0
    if op == "plan":
        case["seqs"] = _log_int(rng, 1, 1024)
        case["new"] = rng.choice([1, _log_int(rng, 1, 2048)])
        case["done"] = rng.choice([0.0, 0.0, 0.1, 0.5])
        case["longest"] = _log_int(rng, 64, 32768)
        case["shortest"] = _log_int(rng, 1, case["longest"])
        return case
    case["new"] = {"window": rng.choice([1, 1, _log_int(rng, 2, 2048)]), "tree": _log_int(rng, 2, 256), "keep": _log_int(rng, 2, 256)}[op]
    case["longest"] = max(case["new"], _log_int(rng, 64, 65536))
    case["shortest"] = max(case["new"], _log_int(rng, 1, case["longest"]))
    # query rows x tokens seen up to those of the largest listed case, rows up to 262144
    seen = min(case["longest"], case["window"] + case["sinks"] + case["new"]) if windowed else case["longest"]
    largest = 8 * 64 * 32768 * 32
    case["new"] = min(case["new"], max(1, largest // (seen * case["q_heads"])))
    most = max(1, min(262144 // seen, largest // (seen * case["new"] * case["q_heads"])))
    case["seqs"] = _log_int(rng, 1, min(64, most))
    return case


def _shape(case):
    """Lengths and new rows of each sequence: the same for every seed.  (plan: lengths before the step, rows asked for)"""
    rng = random.Random("%d %d %d" % (case["seqs"], case["shortest"], case["longest"]))
    lens = [_log_int(rng, case["shortest"], case["longest"]) for _ in range(case["seqs"])]
    if case["op"] != "plan":
        return lens, [case["new"]] * len(lens)
    new = []
    for i in range(len(lens)):
        if rng.random() < case["done"]:
            new.append(-1)
        elif case["new"] > 1 and rng.random() < 0.1:     # a chunk of a prompt
            new.append(_log_int(rng, 1, case["new"]))
        else:
            new.append(0 if rng.random() < 0.05 else 1)
    return lens, new


def _lowest(case, T, n):
    """The first position in the window of any of the last n positions."""
    return max(0, T - n + 1 - case["window"]) if case["window"] else 0


def work(case):
    lens, new = _shape(case)
    d, hk, hq, g = case["dim"], case["kv_heads"], case["q_heads"], case["group"]
    held = hk * 2 * (d / 2 + 2 * d / g)                  # bytes of a token in the cache, keys and values
    if case["op"] == "plan":                             # lengths, rows, entries in and out; positions, slots, a page per page size
        rows = sum(max(0, n) for n in new)
        return {"bytes": len(lens) * 32 + rows * 12 + rows / case["page"] * 8, "flops": 0}
    if case["op"] == "keep":                             # drafted rows in, half of them kept, moved and read back
        return {"bytes": sum(new) * (2 * hk * d * 2 + held + 0.5 * (2 * held + 2 * hk * d * 2)), "flops": 0}
    tokens = rows = 0
    for T, n in zip(lens, new):
        lo = _lowest(case, T, n)
        tokens += T - lo + min(case["sinks"], lo)
        for j in range(n):
            p = T - n + (j if case["op"] == "window" else 0)             # (a drafted row's depth is not known here: 0)
            a = max(0, p + 1 - case["window"]) if case["window"] else 0
            rows += p + 1 - a + min(case["sinks"], a)
    return {"bytes": tokens * held + 2 * sum(new) * hq * d * 2, "flops": 4 * rows * hq * d}


def _held(case, T, n):
    """Positions that a sequence still holds: the sinks' pages, and the pages from the window's lowest on."""
    P, lo = case["page"], _lowest(case, T, n)
    sinks = min(-(-case["sinks"] // P) * P, lo // P * P)
    return list(range(sinks)) + list(range(lo // P * P, T))


def _draws(case, seed):
    """The inputs of a seed, on the GPU: keys and values of the tokens held (sequence after sequence), queries, pages, trees."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    cpu = np.random.default_rng(seed)
    dtype, d, hk, hq, P = DTYPES[case["type"]], case["dim"], case["kv_heads"], case["q_heads"], case["page"]
    lens, new = _shape(case)
    held = [_held(case, T, n) for T, n in zip(lens, new)]
    rows = sum(len(x) for x in held)
    # keys have channels of very different sizes, values have not
    channel = torch.exp(torch.rand(hk, d, generator=gen, device="cuda") * math.log(16.0) + math.log(0.5))
    k = torch.randn(rows, hk, d, generator=gen, device="cuda", dtype=dtype).mul_(channel)
    v = torch.randn(rows, hk, d, generator=gen, device="cuda", dtype=dtype)
    q = torch.randn(len(lens), new[0], hq, d, generator=gen, device="cuda", dtype=dtype) if case["op"] != "keep" else None
    pages = [sorted({t // P for t in x}) for x in held]
    n_pages = sum(len(x) for x in pages) + 3
    order = cpu.permutation(n_pages)
    table = np.full((len(lens), -(-max(lens) // P)), -1, dtype=np.int32)
    at = 0
    for s, x in enumerate(pages):
        table[s, x] = order[at:at + len(x)]
        at += len(x)
    n = new[0]
    # drafted rows continue one of the last few rows before them, or the context
    parents = np.array([[int(cpu.integers(max(-1, j - 9), j)) for j in range(n)] for _ in lens], dtype=np.int32)
    # (as many rows are kept with every seed: results have one shape)
    counts = np.random.default_rng(len(lens) * 1000 + n).integers(0, n + 1, len(lens)).astype(np.int32)
    paths = np.zeros((len(lens), n), dtype=np.int32)
    for s, c in enumerate(counts):
        paths[s, :c] = np.sort(cpu.permutation(n)[:c])
    return {"held": held, "k": k, "v": v, "q": q, "table": table, "n_pages": n_pages, "parents": parents, "counts": counts, "paths": paths}


def _plan_draws(case, seed):
    """The state of a plan before the step: pages held at random places of the pool, the others in the ring."""
    cpu = np.random.default_rng(seed)
    P = case["page"]
    lens, new = _shape(case)
    sinks = -(-case["sinks"] // P)
    spans, held = [], []
    for T in lens:                                       # pages below the window of an earlier step have gone back
        end = -(-T // P)
        first = 0
        if case["window"]:
            first = max(0, T + 1 - case["window"] - int(cpu.integers(0, 3 * P))) // P
            first = first if first > sinks else 0
        spans.append((first, end))
        held.append([p for p in range(end) if p < sinks or p >= first])
    need = sum(max(0, -(-(T + n) // P) - -(-T // P)) for T, n in zip(lens, new) if n > 0)
    n_held = sum(len(x) for x in held)
    n_pages = sum(-(-T // P) for T in lens) + need + 100 # (the same with every seed)
    free = need + int(cpu.integers(0, n_pages - n_held - need + 1))
    order = cpu.permutation(n_pages)
    table = np.full((len(lens), max(1, -(-max(T + max(0, n) for T, n in zip(lens, new)) // P))), -1, dtype=np.int32)
    at = 0
    for s, x in enumerate(held):
        table[s, x] = order[at:at + len(x)]
        at += len(x)
    ring = np.full(n_pages, -1, dtype=np.int32)
    head = int(cpu.integers(0, 5 * n_pages))
    ring[(head + np.arange(free)) % n_pages] = order[at:at + free]
    return {"lens": lens, "new": new, "spans": np.array(spans, dtype=np.int32), "table": table, "ring": ring,
            "counters": np.array([head, head + free, 0, 0], dtype=np.int64)}


def _cache(case, n_pages):
    from paper_2608_23843_b200 import pkv
    return pkv.Q4Cache(pkv.make_q4_config(n_kv_heads=case["kv_heads"], n_q_heads=case["q_heads"], head_dim=case["dim"],
                                          page_size=case["page"], group_size=case["group"], dtype=DTYPES[case["type"]], n_pages=n_pages))


def prepare(case, seed):
    on_gpu = lambda x: torch.as_tensor(x, device="cuda")                  # noqa: E731
    ints = lambda xs: torch.tensor(xs, dtype=torch.int32, device="cuda")  # noqa: E731
    state = {"op": case["op"], "page": case["page"], "group": case["group"], "window": case["window"], "sinks": case["sinks"],
             "heads": case["kv_heads"], "scale": 1 / math.sqrt(case["dim"])}
    if case["op"] == "plan":
        x = _plan_draws(case, seed)
        rows = sum(max(0, n) for n in x["new"])
        state.update(lengths=ints(x["lens"]), rows=ints(x["new"]), n_rows=rows)
        state.update({name: on_gpu(x[name]) for name in ("spans", "table", "ring", "counters")})
        if own:
            state["cache"] = _cache(case, len(x["ring"]))
        return state
    x = _draws(case, seed)
    lens, new = _shape(case)
    n, table = new[0], on_gpu(x["table"])
    state.update(table=table, lengths=ints(lens), new=n, q=x["q"], parents=on_gpu(x["parents"]), n_pages=x["n_pages"])
    if own:
        state["cache"] = _cache(case, x["n_pages"])
    else:
        d, g, shape = case["dim"], case["group"], (x["n_pages"], case["page"], case["kv_heads"])
        state["store"] = tuple(torch.zeros(*shape, *s, dtype=t, device="cuda")
                               for _ in "kv" for s, t in (((d,), torch.int8), ((d // g,), torch.bfloat16)))
    # what the cache holds, written as the pieces of each sequence that it still has
    first = np.cumsum([0] + [len(y) for y in x["held"]])
    last = []
    for s, held in enumerate(x["held"]):
        held = np.array(held)
        cut = np.flatnonzero(np.diff(held) > 1)          # behind the sinks' pages
        a = int(cut[0]) + 1 if len(cut) else 0
        for lo, hi in ((0, a), (a, len(held))):
            if hi == lo:
                continue
            piece, T = slice(first[s] + lo, first[s] + hi), int(held[hi - 1]) + 1
            k, v = x["k"][piece], x["v"][piece]
            if own:
                state["cache"].append_kv(table[s:s + 1], ints([T]), k[None], v[None])
            else:
                t = on_gpu(held[lo:hi])
                _write(state["store"], (table[s].long()[t // case["page"]], t % case["page"]), k, v, case["group"])
        last.append(np.arange(first[s + 1] - n, first[s + 1]))
    if case["op"] == "keep":
        last = on_gpu(np.stack(last))
        state["k"], state["v"] = x["k"][last], x["v"][last]                # the drafted rows [seqs, n, heads, d]
        state["paths"], state["counts"] = on_gpu(x["paths"]), on_gpu(x["counts"])
        kept = int(x["counts"].sum())
        state["offsets"] = ints([0] + [int(c) for c in np.cumsum(x["counts"])])
        state["k_out"], state["v_out"] = (torch.empty(kept, *state["k"].shape[2:], dtype=state["k"].dtype, device="cuda") for _ in "kv")
    return state


def run(state):
    if own:
        return _run_own(state)
    return {"plan": _plan, "keep": _keep, "window": _attend, "tree": _attend}[state["op"]](state)


def _run_own(state):
    cache, table, lengths, W, S = state["cache"], state["table"], state["lengths"], state["window"], state["sinks"]
    if state["op"] == "plan":
        p = cache.plan(table, lengths, state["rows"], state["spans"], state["ring"], state["counters"], state["n_rows"], window=W, sinks=S)
        return p.lengths, p.offsets, p.positions, p.slots, p.spans, p.counters, state["ring"], table
    if state["op"] == "keep":
        cache.append_kv(table, lengths, state["k"], state["v"])
        kept = cache.keep_rows(table, lengths, state["paths"], state["counts"], new_rows=state["new"])
        cache.read_kv(table, kept, state["k_out"], state["v_out"], state["offsets"])
        return state["k_out"], state["v_out"], kept
    if state["op"] == "window":
        return cache.attention(table, lengths, state["q"], window=W, sinks=S)
    masks, depths = cache.tree_masks(state["parents"], lengths, window=W, sinks=S)
    return cache.attention(table, lengths, state["q"], tree=masks, window=W, sinks=S), depths


# ---- plain form ---------------------------------------------------------------------------------------------------
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


def _places(state, t):
    """(physical page, row in it) of positions t [seqs, m]."""
    return torch.gather(state["table"].long(), 1, t // state["page"]), t % state["page"]


def _depths(parents):
    """Depths [seqs, n], and which rows are a row or its ancestors [seqs, n, n]."""
    n = parents.shape[1]
    line = (parents[:, :, None] == torch.arange(n, device=parents.device)).float() + torch.eye(n, device=parents.device)
    for _ in range(max(1, (n - 1).bit_length())):        # ancestors up to twice as far each time
        line = (torch.matmul(line, line) > 0).float()
    return line.sum(-1).long() - 1, line > 0


def _attend(state):
    q, T, W, sinks = state["q"], state["lengths"].long(), state["window"], state["sinks"]
    hk, (S, n, hq, d) = state["heads"], q.shape
    G, C = hq // hk, T - n
    row = torch.arange(n, device="cuda")
    if state["op"] == "tree":
        depth, line = _depths(state["parents"])
    else:
        depth, line = row.expand(S, n), (row[:, None] >= row).expand(S, n, n)
    at = C[:, None] + depth                                                # position of each row
    # the tokens that some row may see: the first ones, and from the window's lowest on, as positions [seqs, m]
    lo = (C + 1 - W).clamp(min=0) if W else torch.zeros_like(C)
    # (host: as long as the longest sequence needs)
    m = int((T - lo).max()) if not W else W + n - 1
    t = torch.cat([torch.arange(sinks, device="cuda").expand(S, sinks), lo[:, None] + torch.arange(m, device="cuda")], 1)
    there = torch.cat([torch.arange(sinks, device="cuda") < lo[:, None], t[:, sinks:] < T[:, None]], 1)
    i = t - C[:, None]                                                     # new row that a position is, if it is one
    new = i >= 0
    where = C[:, None] + torch.gather(depth, 1, i.clamp(0, n - 1))         # ... and the place it stands for
    pos = torch.where(new, where, t)
    see = torch.where(new[:, None], torch.gather(line, 2, i.clamp(0, n - 1)[:, None].expand(S, n, -1)), True)
    if W:
        see = see & ((pos[:, None] > at[:, :, None] - W) | (pos < sinks)[:, None])
    see = see & there[:, None]
    x = q.float().view(S, n, hk, G, d).permute(0, 2, 1, 3, 4).reshape(S, hk, n * G, d)
    page, r = _places(state, torch.where(there, t, T[:, None] - 1))
    kc, ks, vc, vs = (c[page, r].transpose(1, 2) for c in state["store"])  # [S, H, tokens, ...]
    s = torch.matmul(x, _values(kc, ks).transpose(-1, -2)).mul_(state["scale"])
    s = s.masked_fill_(~see.repeat_interleave(G, 1)[:, None], -math.inf)
    p = s.sub_(s.amax(-1, keepdim=True)).exp_()
    o = torch.matmul(p, _values(vc, vs)) / p.sum(-1, keepdim=True)
    o = o.view(S, hk, n, G, d).permute(0, 2, 1, 3, 4).reshape(q.shape).to(q.dtype)
    return (o, depth.int()) if state["op"] == "tree" else o


def _keep(state):
    n, T, counts = state["new"], state["lengths"].long(), state["counts"].long()
    C = T - n
    i = torch.arange(n, device="cuda")
    _write(state["store"], _places(state, C[:, None] + i), state["k"], state["v"], state["group"])
    some = i < counts[:, None]
    page, r = _places(state, C[:, None] + torch.where(some, state["paths"].long(), i))
    to = _places(state, C[:, None] + i)
    for x in state["store"]:
        x[to] = x[page, r]
    kc, ks, vc, vs = (x[to][some] for x in state["store"])
    dtype = state["k_out"].dtype
    return _values(kc, ks).to(dtype), _values(vc, vs).to(dtype), (C + counts).int()


def _plan(state):
    """(every request can be served: what the listed and drawn steps are like)"""
    T, n, table, ring, P, W = state["lengths"].long(), state["rows"].long(), state["table"], state["ring"], state["page"], state["window"]
    first, end = state["spans"].long().unbind(1)
    sinks = -(-state["sinks"] // P) if W else 0
    done, new = n < 0, n.clamp(min=0)
    after = torch.where(done, 0, T + new)
    need = torch.where(done, 0, (-(-after // P) - end).clamp(min=0))
    entry = torch.arange(table.shape[1], device="cuda")
    lowest = torch.div((T + 1 - W).clamp(min=0), P, rounding_mode="floor") if W else torch.zeros_like(T)
    holds = (entry < end[:, None]) & ((entry < sinks) | (entry >= first[:, None]))
    back = holds & (done[:, None] | ((entry >= sinks) & (entry < lowest[:, None])))
    taken = (entry >= end[:, None]) & (entry < (end + need)[:, None])
    size, head, tail = ring.shape[0], state["counters"][0], state["counters"][1]
    returned = table[back]                                                 # (in the order of requests, then entries)
    ring[(tail + torch.arange(returned.shape[0], device="cuda")) % size] = returned
    got = torch.cumsum(taken.flatten(), 0).view_as(taken) - 1
    table.copy_(torch.where(taken, ring[(head + got) % size], table))
    moved = torch.maximum(first, torch.minimum(lowest, end))
    first = torch.where(done, 0, torch.where((moved > first) & (moved > sinks), moved, first))
    offsets = torch.cumsum(torch.cat([torch.zeros_like(n[:1]), new]), 0)
    row = torch.arange(state["n_rows"], device="cuda")
    seq = torch.searchsorted(offsets, row, right=True) - 1
    pos = T[seq] + row - offsets[seq]
    slots = table[seq, pos // P].long() * P + pos % P
    counters = torch.stack([head + need.sum(), tail + returned.shape[0], torch.zeros_like(head), torch.zeros_like(head)])
    spans = torch.stack([first, torch.where(done, 0, end + need)], 1)
    return after.int(), offsets.int(), pos.int(), slots, spans.int(), counters, ring, table


# ---- the definition, in 64 bits and one sequence at a time ----------------------------------------------------------
def exact(case, seed):
    if case["op"] == "plan":
        return _exact_plan(case, seed)
    x = _draws(case, seed)
    lens, new = _shape(case)
    d, g, hk, hq, W, n = case["dim"], case["group"], case["kv_heads"], case["q_heads"], case["window"], new[0]

    def stands_for(y):                                   # what the cache stands for, one group per row
        y = y.double().reshape(-1, g)
        step = (y.abs().max(dim=1, keepdim=True).values / 7).to(torch.bfloat16).double()
        return torch.round(y / step.clamp_min(1e-300)).clamp(-7, 7) * step

    first = np.cumsum([0] + [len(h) for h in x["held"]])
    outs, depths, lengths = [], [], []
    for s, T in enumerate(lens):
        rows = slice(int(first[s]), int(first[s + 1]))
        C = T - n
        if case["op"] == "keep":
            pick = torch.as_tensor(first[s + 1] - n + x["paths"][s, :x["counts"][s]].astype(np.int64), device="cuda")
            outs.append([stands_for(y[pick]).view(-1, hk, d) for y in (x["k"], x["v"])])
            lengths.append(C + int(x["counts"][s]))
            continue
        K, V = (stands_for(y[rows]).view(-1, hk, d) for y in (x["k"], x["v"]))
        up = x["parents"][s] if case["op"] == "tree" else np.arange(n) - 1
        depth = np.zeros(n, dtype=np.int64)
        lines = []
        for j in range(n):
            lines.append({j} | (lines[up[j]] if up[j] >= 0 else set()) if case["op"] == "tree" else range(j + 1))
            depth[j] = depth[up[j]] + 1 if up[j] >= 0 else 0
        held = np.array(x["held"][s])
        see = np.zeros((n, len(held)), dtype=bool)
        for j in range(n):
            p = C + depth[j]
            old = held < C
            see[j] = old if not W else old & ((held > p - W) | (held < case["sinks"]))
            mine = np.array(sorted(lines[j]))
            where = C + depth[mine]
            if W:
                mine = mine[(where > p - W) | (where < case["sinks"])]
            see[j, len(held) - n + mine] = True          # (all new rows are held)
        see = torch.as_tensor(see, device="cuda")
        out = torch.empty(n, hq, d, dtype=torch.float64, device="cuda")
        for h in range(hq):
            kv = h // (hq // hk)
            z = (x["q"][s, :, h].double() @ K[:, kv].T / math.sqrt(d)).masked_fill_(~see, -math.inf)
            out[:, h] = torch.softmax(z, dim=1) @ V[:, kv]
        outs.append(out)
        depths.append(depth)
    if case["op"] == "keep":
        return torch.cat([o[0] for o in outs]), torch.cat([o[1] for o in outs]), np.array(lengths, dtype=np.int32)
    out = torch.stack(outs)
    return (out, np.array(depths, dtype=np.int32)) if case["op"] == "tree" else out


def _exact_plan(case, seed):
    x = _plan_draws(case, seed)
    P, W, size = case["page"], case["window"], len(x["ring"])
    sinks = -(-case["sinks"] // P) if W else 0
    table, ring, (head, tail) = x["table"], x["ring"].copy(), (int(c) for c in x["counters"][:2])
    lengths, offsets, positions, slots, spans = [], [0], [], [], []
    for s, (T, n) in enumerate(zip(x["lens"], x["new"])):
        first, end = (int(v) for v in x["spans"][s])
        if n < 0:
            for p in range(end):
                if p < sinks or p >= first:
                    ring[tail % size] = table[s, p]
                    tail += 1
            lengths.append(0)
            offsets.append(offsets[-1])
            spans.append((0, 0))
            continue
        for p in range(max(first, sinks), end):
            if W and (p + 1) * P <= T + 1 - W:
                ring[tail % size] = table[s, p]
                tail += 1
                first = p + 1
        while end * P < T + n:
            table[s, end] = x["ring"][head % size]
            head += 1
            end += 1
        for t in range(T, T + n):
            positions.append(t)
            slots.append(int(table[s, t // P]) * P + t % P)
        lengths.append(T + n)
        offsets.append(offsets[-1] + n)
        spans.append((first, end))
    i32 = lambda v: np.array(v, dtype=np.int32)          # noqa: E731
    return (i32(lengths), i32(offsets), i32(positions), np.array(slots, dtype=np.int64), i32(spans),
            np.array([head, tail, 0, 0], dtype=np.int64), ring, table)
