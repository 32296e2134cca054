"""Binding of libpkv.so (see include/pkv.h) by ctypes, and for the calls of a decode step by a small C module where it has been built: argument
marshalling only.

Module-level functions carry the C names (`pkv_init_cache`, `pkv_append_kv`,
`pkv_compress_eligible_pages`, `pkv_decode_attention`, ...).  `Cache` is a
convenience wrapper that allocates the caller-owned device buffers with torch
and forwards to those functions; every computation runs in the CUDA library.
There is no CPU fallback: if the library has not been built, loading fails.
"""
import ctypes
import os
from operator import index
from typing import NamedTuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpkv.so")

PKV_OK = 0
PKV_ERR_INVALID_ARG = -1
PKV_ERR_POOL_EXHAUSTED = -2
PKV_ERR_BAD_SEQ = -3
PKV_ERR_CUDA = -4
PKV_ERR_NOT_CONVERGED = -5
PKV_ERR_UNSUPPORTED = -6
PKV_ERR_DEVICE_TIMEOUT = -7
PKV_KIND_DENSE, PKV_KIND_FACTOR = 0, 1

EXPORTS = [
    "pkv_query_sizes", "pkv_init_cache", "pkv_append_kv", "pkv_compress_eligible_pages",
    "pkv_decode_attention", "pkv_decode_attention_host", "pkv_get_page_table", "pkv_get_stats",
    "pkv_free_seq", "pkv_destroy_cache", "pkv_last_error", "pkv_read_factors", "pkv_write_factors",
    "pkv_read_dense", "pkv_get_decode_plan", "pkv_decode_attention_static_scratch", "pkv_get_decode_trace",
    "pkv_decode_attention_multi", "pkv_compress_begin", "pkv_compress_commit",
    "pkv_decode_attention_partial", "pkv_merge_attention_states",
    "pkv_get_rotation_schedule", "pkv_read_basis", "pkv_get_row_block_ranges",
    "pkv_q4_query_sizes", "pkv_q4_init_cache", "pkv_q4_destroy_cache", "pkv_q4_last_error", "pkv_q4_get_stats",
    "pkv_q4_append_kv", "pkv_q4_read_kv", "pkv_q4_attention_workspace", "pkv_q4_attention",
    "pkv_q4_attention_select_workspace", "pkv_q4_attention_select", "pkv_q4_tree_masks", "pkv_q4_keep_rows",
    "pkv_q4_plan_workspace", "pkv_q4_plan", "pkv_q4_attention_route",
]


class PkvConfig(ctypes.Structure):
    _fields_ = [
        ("n_layers", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32), ("page_size", ctypes.c_int32), ("rank_k", ctypes.c_int32),
        ("rank_v", ctypes.c_int32), ("sink_tokens", ctypes.c_int32), ("recent_tokens", ctypes.c_int32),
        ("max_seqs", ctypes.c_int32), ("max_pages_per_seq", ctypes.c_int32),
        ("n_dense_slots", ctypes.c_int64), ("n_factor_slots", ctypes.c_int64),
        ("softmax_scale", ctypes.c_float), ("jacobi_max_sweeps", ctypes.c_int32),
        ("jacobi_tol", ctypes.c_float), ("n_ctas", ctypes.c_int32), ("decode_variant", ctypes.c_int32),
        ("jacobi_energy_tol", ctypes.c_float), ("factor_bits", ctypes.c_int32), ("decode_overlap", ctypes.c_int32),
        ("global_rank", ctypes.c_int32),
    ]


class PkvSizes(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("dense_slot_bytes", "factor_slot_bytes", "dense_pool_bytes",
                                              "factor_pool_bytes", "meta_bytes", "workspace_bytes")]


class PkvStats(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("dense_slots_in_use", "factor_slots_in_use", "pages_compressed",
                                              "page_svds_not_converged", "device_timeouts", "bad_slot_indices",
                                              "last_decode_bytes", "last_decode_units", "page_svds", "jacobi_rounds")]


PKV_DTYPE_BF16, PKV_DTYPE_FP16 = 0, 1


class PkvQ4Config(ctypes.Structure):
    _fields_ = [
        ("n_kv_heads", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
        ("page_size", ctypes.c_int32), ("group_size", ctypes.c_int32), ("dtype", ctypes.c_int32),
        ("n_pages", ctypes.c_int64), ("softmax_scale", ctypes.c_float), ("n_ctas", ctypes.c_int32),
    ]


class PkvQ4Sizes(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("page_bytes", "pool_bytes", "meta_bytes")]


class PkvQ4Stats(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("device_timeouts", "bad_pages", "bad_lengths")]


class PkvQ4Select(ctypes.Structure):
    _fields_ = [("window", ctypes.c_int32), ("sinks", ctypes.c_int32), ("tree", ctypes.c_void_p), ("tree_words", ctypes.c_int32)]


class PkvError(RuntimeError):
    def __init__(self, status, message=""):
        super().__init__("pkv status %d: %s" % (status, message))
        self.status = status


_lib = None


def lib():
    """The loaded CUDA library.  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libpkv.so is missing: build it with `python -m paper_2608_23843_b200.build` "
                               "(there is no CPU fallback)")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
        ip = ctypes.POINTER(ctypes.c_int32)
        L.pkv_query_sizes.argtypes = [ctypes.POINTER(PkvConfig), ctypes.POINTER(PkvSizes)]
        L.pkv_init_cache.argtypes = [ctypes.POINTER(PkvConfig), vp, vp, vp, vp, ip, ip, ctypes.POINTER(vp)]
        L.pkv_append_kv.argtypes = [vp, i32, i32, ip, ip, vp, vp, vp]
        L.pkv_compress_eligible_pages.argtypes = [vp, i32, ctypes.POINTER(i64), vp]
        L.pkv_decode_attention.argtypes = [vp, i32, i32, ip, vp, vp, vp, vp]
        L.pkv_decode_attention_static_scratch.argtypes = [vp, i32, i32, ip, vp, vp, vp, vp]
        L.pkv_decode_attention_multi.argtypes = [vp, i32, i32, ip, i32, vp, vp, vp, vp]
        L.pkv_compress_begin.argtypes = [vp, i32, vp, vp, ctypes.POINTER(i64)]
        L.pkv_decode_attention_partial.argtypes = [vp, i32, i32, ip, vp, vp, vp]
        L.pkv_merge_attention_states.argtypes = [vp, i32, i64, vp, vp, vp]
        L.pkv_compress_commit.argtypes = [vp, i32, vp, ctypes.POINTER(i64)]
        L.pkv_decode_attention_host.argtypes = [vp, i32, i32, ip, vp, vp, vp, vp, vp]
        L.pkv_get_page_table.argtypes = [vp, i32, i32, ip, ip, ip, ip]
        L.pkv_get_stats.argtypes = [vp, ctypes.POINTER(PkvStats), vp]
        L.pkv_free_seq.argtypes = [vp, i32]
        L.pkv_destroy_cache.argtypes = [vp]
        L.pkv_last_error.argtypes = [vp]
        L.pkv_last_error.restype = ctypes.c_char_p
        L.pkv_read_factors.argtypes = [vp, i64, i32, vp, vp, vp, vp, vp]
        L.pkv_write_factors.argtypes = [vp, i64, i32, vp, vp, vp, vp, vp]
        L.pkv_read_dense.argtypes = [vp, i64, i32, vp, vp, vp]
        L.pkv_read_basis.argtypes = [vp, i32, i32, i32, vp, vp, vp]
        L.pkv_get_decode_plan.argtypes = [vp, i32, ip, ip, ip, ip]
        L.pkv_get_decode_trace.argtypes = [vp, ctypes.POINTER(ctypes.c_int64), i32, vp]
        L.pkv_get_rotation_schedule.argtypes = [i32, ctypes.POINTER(ctypes.c_uint8), i64, ip, ip, ip]
        L.pkv_get_row_block_ranges.argtypes = [i64, i32, i32, i32, ip]
        L.pkv_q4_query_sizes.argtypes = [ctypes.POINTER(PkvQ4Config), ctypes.POINTER(PkvQ4Sizes)]
        L.pkv_q4_init_cache.argtypes = [ctypes.POINTER(PkvQ4Config), vp, vp, ctypes.POINTER(vp)]
        L.pkv_q4_destroy_cache.argtypes = [vp]
        L.pkv_q4_last_error.argtypes = [vp]
        L.pkv_q4_last_error.restype = ctypes.c_char_p
        L.pkv_q4_get_stats.argtypes = [vp, ctypes.POINTER(PkvQ4Stats), vp]
        L.pkv_q4_append_kv.argtypes = [vp, i32, vp, i32, vp, i64, vp, vp, i64, i64, vp, i64, i64, vp]
        L.pkv_q4_read_kv.argtypes = L.pkv_q4_append_kv.argtypes
        L.pkv_q4_attention_workspace.argtypes = [vp, i32, i32, i32, ctypes.POINTER(i64)]
        L.pkv_q4_attention.argtypes = [vp, i32, vp, i32, vp, i64, vp, i32, i32, vp, i64, i64, vp, i64, i64, vp, vp, i64, vp]
        sel = ctypes.POINTER(PkvQ4Select)
        L.pkv_q4_attention_select_workspace.argtypes = [vp, i32, i32, i32, sel, ctypes.POINTER(i64)]
        L.pkv_q4_attention_select.argtypes = [vp, i32, vp, i32, vp, i64, vp, i32, i32, sel, vp, i64, i64, vp, i64, i64, vp, vp, i64, vp]
        L.pkv_q4_attention_route.argtypes = [vp, i32, i32, i32, sel, ip, ip, ip]
        L.pkv_q4_tree_masks.argtypes = [vp, i32, vp, i64, vp, i32, vp, i32, i32, vp, i32, vp, vp]
        L.pkv_q4_keep_rows.argtypes = [vp, i32, vp, i32, vp, i64, vp, vp, i32, vp, vp, vp]
        L.pkv_q4_plan_workspace.argtypes = [vp, i32, i64, ctypes.POINTER(i64)]
        L.pkv_q4_plan.argtypes = [vp, i32, vp, i32, vp, vp, vp, vp, vp, i32, i32, vp, vp, vp, vp, i64, vp, vp, vp, i64, vp]
        for name in EXPORTS:
            if name not in ("pkv_last_error", "pkv_q4_last_error"):
                getattr(L, name).restype = ctypes.c_int32
        _lib = L
    return _lib


# The calls of a decode step and their arguments, a letter each: p a pointer (None is NULL), i a number of 32 bits, l one of 64.
_CALLS = {"append_kv": "pipiplppllpllp", "read_kv": "pipiplppllpllp", "attention": "pipiplpiipllpllpplp", "attention_select": "pipiplpiipllpllpplpiipi",
          "tree_masks": "piplpipiipipp", "keep_rows": "pipiplppippp", "plan": "pipipppppiipppplppplp"}
_calls_module = None


class _CtypesCalls:
    """The calls of _pkvcall through ctypes, with the same checks, where that module has not been built for this interpreter."""

    def __init__(self):
        for name, kinds in _CALLS.items():
            setattr(self, name, self._checked(kinds, self._select if name == "attention_select" else getattr(lib(), "pkv_q4_" + name)))

    @staticmethod
    def _checked(kinds, fn):
        def call(*args):
            if len(args) != len(kinds):
                raise TypeError("%d arguments expected, not %d" % (len(kinds), len(args)))
            for i, (x, kind) in enumerate(zip(args, kinds)):
                if x is None and kind == "p":
                    continue
                bits = 31 if kind == "i" else 63
                if not -1 << bits <= index(x) < 1 << bits:
                    raise OverflowError("argument %d does not fit %d bits" % (i, bits + 1))
            return fn(*args)
        return call

    @staticmethod
    def _select(*args):
        sel = PkvQ4Select(*args[19:])
        return lib().pkv_q4_attention_select(*args[:9], ctypes.byref(sel), *args[9:19])


def _calls():
    """The calls of a decode step: numbers in, a status out.  By a C module (ctypes takes 3 us more each) if it has been built for this interpreter, and
    links this library."""
    global _calls_module
    if _calls_module is None:
        from . import build
        lib()                                            # (says what to do where nothing has been built)
        built = os.path.exists(build.CALL) and os.path.exists(build.LIB) and os.path.samefile(LIB_PATH, build.LIB)
        if built:
            from . import _pkvcall
        _calls_module = _pkvcall if built else _CtypesCalls()
    return _calls_module


_INT_ARRAYS = {}


def _ints(xs):
    """A ctypes int32 array for a sequence of ints (decode calls pass the same id list every step: remembered)."""
    if len(xs) > 4096:                                   # e.g. slot orders: built once, not worth remembering
        vals = [int(x) for x in xs]
        return (ctypes.c_int32 * len(vals))(*vals), len(vals)
    key = tuple(xs)
    hit = _INT_ARRAYS.get(key)
    if hit is None:
        vals = [int(x) for x in key]
        hit = ((ctypes.c_int32 * len(vals))(*vals), len(vals))
        if len(_INT_ARRAYS) >= 256:
            _INT_ARRAYS.clear()
        _INT_ARRAYS[key] = hit
    return hit


def _ptr(t):
    """Device (or host) address of a tensor as a plain int: ctypes converts it for a void* parameter, and building
    a c_void_p object per argument is a measurable part of a 5 us call."""
    return None if t is None else t.data_ptr()


def _stream(stream):
    if stream is None or isinstance(stream, int):
        return stream
    return stream.cuda_stream


try:                                                     # raw handle of the current stream without a Stream object (2 us less per call)
    _raw_current_stream = torch._C._cuda_getCurrentRawStream
except AttributeError:                                   # pragma: no cover
    _raw_current_stream = None


# ---- functions with the C names -------------------------------------------------
def pkv_query_sizes(cfg: PkvConfig) -> PkvSizes:
    out = PkvSizes()
    st = lib().pkv_query_sizes(ctypes.byref(cfg), ctypes.byref(out))
    if st != PKV_OK:
        raise PkvError(st, "pkv_query_sizes")
    return out


def pkv_init_cache(cfg, dense_pool, factor_pool, meta, workspace, dense_slot_order=None, factor_slot_order=None):
    """Tensors (or None for all four = dry run) -> opaque handle."""
    h = ctypes.c_void_p()
    d_ord = f_ord = None
    if dense_slot_order is not None:
        d_ord, _ = _ints(dense_slot_order)
    if factor_slot_order is not None:
        f_ord, _ = _ints(factor_slot_order)
    st = lib().pkv_init_cache(ctypes.byref(cfg), _ptr(dense_pool), _ptr(factor_pool), _ptr(meta), _ptr(workspace),
                              d_ord, f_ord, ctypes.byref(h))
    if st != PKV_OK:
        raise PkvError(st, "pkv_init_cache")
    return h


def _check(handle, st):
    if st != PKV_OK:
        raise PkvError(st, lib().pkv_last_error(handle).decode())


def pkv_append_kv(handle, layer, seq_ids, n_new, k, v, stream=None):
    ids, n = _ints(seq_ids)
    cnt, _ = _ints(n_new)
    _check(handle, lib().pkv_append_kv(handle, layer, n, ids, cnt, _ptr(k), _ptr(v), _stream(stream)))


def pkv_compress_eligible_pages(handle, layer=-1, stream=None) -> int:
    n = ctypes.c_int64(0)
    st = lib().pkv_compress_eligible_pages(handle, layer, ctypes.byref(n), _stream(stream))
    _check(handle, st)
    return int(n.value)


def pkv_compress_begin(handle, layer, main_stream=None, side_stream=None) -> int:
    """Starts factorizing the layer's eligible pages on side_stream; returns how many.  The pages stay dense until
    pkv_compress_commit.  If the factor pool runs out, PkvError carries the status and `begun` the pages begun."""
    n = ctypes.c_int64(0)
    st = lib().pkv_compress_begin(handle, layer, _stream(main_stream), _stream(side_stream), ctypes.byref(n))
    if st != PKV_OK:
        msg = lib().pkv_last_error(handle)
        e = PkvError(st, msg.decode() if msg else "")
        e.begun = int(n.value)
        raise e
    return int(n.value)


def pkv_compress_commit(handle, layer=-1, main_stream=None) -> int:
    n = ctypes.c_int64(0)
    _check(handle, lib().pkv_compress_commit(handle, layer, _stream(main_stream), ctypes.byref(n)))
    return int(n.value)


def pkv_decode_attention(handle, layer, seq_ids, q, out, out_f32=None, stream=None):
    ids, n = _ints(seq_ids)
    _check(handle, lib().pkv_decode_attention(handle, layer, n, ids, _ptr(q), _ptr(out), _ptr(out_f32), _stream(stream)))


def pkv_decode_attention_multi(handle, layer, seq_ids, q_len, q, out, out_f32=None, stream=None):
    """q, out: [n_seqs, q_len, H_q, d]; query j of a sequence belongs to its position T - q_len + j (causal)."""
    ids, n = _ints(seq_ids)
    _check(handle, lib().pkv_decode_attention_multi(handle, layer, n, ids, q_len, _ptr(q), _ptr(out), _ptr(out_f32),
                                                    _stream(stream)))


def pkv_decode_attention_partial(handle, layer, seq_ids, q, state, stream=None):
    """state: fp32 [n_seqs, H_q, d + 2] = (o unnormalised, m in base-2 units, l) over this cache's tokens."""
    ids, n = _ints(seq_ids)
    _check(handle, lib().pkv_decode_attention_partial(handle, layer, n, ids, _ptr(q), _ptr(state), _stream(stream)))


def pkv_merge_attention_states(states, n_shards, n_rows, out=None, out_f32=None, stream=None):
    """Eq. 5 over n_shards state arrays stored back to back ([n_shards, n_rows, d + 2] fp32)."""
    st = lib().pkv_merge_attention_states(_ptr(states), n_shards, n_rows, _ptr(out), _ptr(out_f32), _stream(stream))
    if st != PKV_OK:
        raise PkvError(st, "pkv_merge_attention_states")


def pkv_decode_attention_static_scratch(handle, layer, seq_ids, q, out, out_f32=None, stream=None):
    """Same result as pkv_decode_attention; the split-K scratch is a fixed array inside the library, for
    callers that cannot supply a workspace.  Shared by all calls on the device: do not overlap calls."""
    ids, n = _ints(seq_ids)
    _check(handle, lib().pkv_decode_attention_static_scratch(handle, layer, n, ids, _ptr(q), _ptr(out), _ptr(out_f32),
                                                             _stream(stream)))


def pkv_decode_attention_host(handle, layer, seq_ids, q_host, out_host, q_stage, out_stage, stream=None):
    ids, n = _ints(seq_ids)
    _check(handle, lib().pkv_decode_attention_host(handle, layer, n, ids, _ptr(q_host), _ptr(out_host),
                                                   _ptr(q_stage), _ptr(out_stage), _stream(stream)))


def pkv_get_page_table(handle, seq, layer, max_pages):
    kinds = (ctypes.c_int32 * max_pages)()
    slots = (ctypes.c_int32 * max_pages)()
    n_pages, n_tokens = ctypes.c_int32(0), ctypes.c_int32(0)
    st = lib().pkv_get_page_table(handle, seq, layer, kinds, slots, ctypes.byref(n_pages), ctypes.byref(n_tokens))
    if st != PKV_OK:
        raise PkvError(st, "pkv_get_page_table")
    n = n_pages.value
    return list(kinds[:n]), list(slots[:n]), int(n_tokens.value)


def pkv_get_stats(handle, stream=None) -> dict:
    s = PkvStats()
    _check(handle, lib().pkv_get_stats(handle, ctypes.byref(s), _stream(stream)))
    return {n: int(getattr(s, n)) for n, _ in PkvStats._fields_}


def pkv_get_decode_plan(handle, layer, n_ctas, n_seqs, n_kv_heads):
    """-> (cta_starts [(position, head, unit)] incl. end sentinel, seg_parts [(cta_first, n_parts)])."""
    starts = (ctypes.c_int32 * (3 * (n_ctas + 1)))()
    segs = (ctypes.c_int32 * (2 * n_seqs * n_kv_heads))()
    n_used, n_segs = ctypes.c_int32(0), ctypes.c_int32(0)
    st = lib().pkv_get_decode_plan(handle, layer, ctypes.byref(n_used), starts, ctypes.byref(n_segs), segs)
    if st != PKV_OK:
        raise PkvError(st, "pkv_get_decode_plan")
    return ([tuple(starts[3 * j:3 * j + 3]) for j in range(n_used.value + 1)],
            [tuple(segs[2 * s:2 * s + 2]) for s in range(n_segs.value)])


def pkv_get_decode_trace(handle, n_ctas, stream=None):
    """Per-CTA time stamps of the last decode launch (needs PKV_DECODE_TRACE=1 at init): list of 16-tuples."""
    buf = (ctypes.c_int64 * (16 * n_ctas))()
    _check(handle, lib().pkv_get_decode_trace(handle, buf, n_ctas, _stream(stream)))
    return [tuple(buf[16 * i:16 * i + 16]) for i in range(n_ctas)]


def pkv_free_seq(handle, seq):
    _check(handle, lib().pkv_free_seq(handle, seq))


def pkv_destroy_cache(handle):
    lib().pkv_destroy_cache(handle)


def pkv_read_factors(handle, slot, kv_head, A_k, B_k, A_v, B_v, stream=None):
    _check(handle, lib().pkv_read_factors(handle, slot, kv_head, _ptr(A_k), _ptr(B_k), _ptr(A_v), _ptr(B_v), _stream(stream)))


def pkv_write_factors(handle, slot, kv_head, A_k, B_k, A_v, B_v, stream=None):
    _check(handle, lib().pkv_write_factors(handle, slot, kv_head, _ptr(A_k), _ptr(B_k), _ptr(A_v), _ptr(B_v), _stream(stream)))


def pkv_get_rotation_schedule(page_size):
    """-> list of rounds, each a list of groups (tuples of member indices)."""
    buf = (ctypes.c_uint8 * 4096)()
    nr, ng, gs = ctypes.c_int32(), ctypes.c_int32(), ctypes.c_int32()
    rc = lib().pkv_get_rotation_schedule(int(page_size), buf, 4096, ctypes.byref(nr), ctypes.byref(ng), ctypes.byref(gs))
    if rc != PKV_OK:
        raise PkvError(rc, "pkv_get_rotation_schedule(%r)" % (page_size,))
    flat = list(buf[:nr.value * ng.value * gs.value])
    it = iter(flat)
    return [[tuple(next(it) for _ in range(gs.value)) for _ in range(ng.value)] for _ in range(nr.value)]


def pkv_get_row_block_ranges(n_row_blocks, longest_tokens, page_size, n_sms):
    """-> token ranges per row block of a tcgen05 row-block launch (1 = the blocks are not cut)."""
    n = ctypes.c_int32()
    rc = lib().pkv_get_row_block_ranges(int(n_row_blocks), int(longest_tokens), int(page_size), int(n_sms), ctypes.byref(n))
    if rc != PKV_OK:
        raise PkvError(rc, "pkv_get_row_block_ranges(%r, %r, %r, %r)" % (n_row_blocks, longest_tokens, page_size, n_sms))
    return n.value


def pkv_read_dense(handle, slot, kv_head, K, V, stream=None):
    _check(handle, lib().pkv_read_dense(handle, slot, kv_head, _ptr(K), _ptr(V), _stream(stream)))


def pkv_read_basis(handle, seq, layer, kv_head, B_k, B_v, stream=None):
    _check(handle, lib().pkv_read_basis(handle, seq, layer, kv_head, _ptr(B_k), _ptr(B_v), _stream(stream)))


# ---- the paged cache held in 4 bits ------------------------------------------------
def pkv_q4_query_sizes(cfg: PkvQ4Config) -> PkvQ4Sizes:
    out = PkvQ4Sizes()
    st = lib().pkv_q4_query_sizes(ctypes.byref(cfg), ctypes.byref(out))
    if st != PKV_OK:
        raise PkvError(st, "pkv_q4_query_sizes")
    return out


def pkv_q4_init_cache(cfg, pool, meta):
    """Tensors (or None for both = dry run) -> opaque handle."""
    h = ctypes.c_void_p()
    st = lib().pkv_q4_init_cache(ctypes.byref(cfg), _ptr(pool), _ptr(meta), ctypes.byref(h))
    if st != PKV_OK:
        raise PkvError(st, "pkv_q4_init_cache")
    return h


def _q4_check(handle, st):
    if st != PKV_OK:
        raise PkvError(st, lib().pkv_q4_last_error(handle).decode())


def pkv_q4_destroy_cache(handle):
    lib().pkv_q4_destroy_cache(handle)


def pkv_q4_get_stats(handle, stream=None) -> dict:
    s = PkvQ4Stats()
    _q4_check(handle, lib().pkv_q4_get_stats(handle, ctypes.byref(s), _stream(stream)))
    return {n: int(getattr(s, n)) for n, _ in PkvQ4Stats._fields_}


def pkv_q4_append_kv(handle, n_seqs, page_table, max_pages, lengths, n_rows, offsets, k, k_strides, v, v_strides, stream=None):
    """k, v: [n_rows, H_kv, d]; k_strides, v_strides: (row, head) in elements."""
    _q4_check(handle, lib().pkv_q4_append_kv(handle, n_seqs, _ptr(page_table), max_pages, _ptr(lengths), n_rows, _ptr(offsets),
                                             _ptr(k), *k_strides, _ptr(v), *v_strides, _stream(stream)))


def pkv_q4_read_kv(handle, n_seqs, page_table, max_pages, lengths, n_rows, offsets, k, k_strides, v, v_strides, stream=None):
    _q4_check(handle, lib().pkv_q4_read_kv(handle, n_seqs, _ptr(page_table), max_pages, _ptr(lengths), n_rows, _ptr(offsets),
                                           _ptr(k), *k_strides, _ptr(v), *v_strides, _stream(stream)))


def pkv_q4_attention_workspace(handle, n_seqs, max_q_len, max_len) -> int:
    n = ctypes.c_int64(0)
    st = lib().pkv_q4_attention_workspace(handle, n_seqs, max_q_len, max_len, ctypes.byref(n))
    if st != PKV_OK:
        raise PkvError(st, "pkv_q4_attention_workspace(%r, %r, %r)" % (n_seqs, max_q_len, max_len))
    return n.value


def pkv_q4_attention(handle, n_seqs, page_table, max_pages, lengths, n_rows, offsets, max_q_len, max_len, q, q_strides, out,
                     out_strides, state, workspace, workspace_bytes, stream=None):
    """q, out: [n_rows, H_q, d]; state: fp32 [n_rows, H_q, d + 2] instead of out."""
    _q4_check(handle, lib().pkv_q4_attention(handle, n_seqs, _ptr(page_table), max_pages, _ptr(lengths), n_rows, _ptr(offsets),
                                             max_q_len, max_len, _ptr(q), *q_strides, _ptr(out), *out_strides, _ptr(state),
                                             _ptr(workspace), workspace_bytes, _stream(stream)))


def pkv_q4_attention_select_workspace(handle, n_seqs, max_q_len, max_len, window=0, sinks=0, tree=None, tree_words=0) -> int:
    """tree: the masks, or anything that is not None (its contents do not matter for the size)."""
    n = ctypes.c_int64(0)
    sel = PkvQ4Select(window, sinks, None if tree is None else 8, tree_words)
    st = lib().pkv_q4_attention_select_workspace(handle, n_seqs, max_q_len, max_len, ctypes.byref(sel), ctypes.byref(n))
    if st != PKV_OK:
        raise PkvError(st, "pkv_q4_attention_select_workspace(%r, %r, %r, window %r, sinks %r)" % (n_seqs, max_q_len, max_len, window, sinks))
    return n.value


def pkv_q4_attention_select(handle, n_seqs, page_table, max_pages, lengths, n_rows, offsets, max_q_len, max_len, window, sinks, tree,
                            tree_words, q, q_strides, out, out_strides, state, workspace, workspace_bytes, stream=None):
    """q, out, state as pkv_q4_attention(); tree: int64 [n_rows, tree_words] or None."""
    sel = PkvQ4Select(window, sinks, _ptr(tree), tree_words)
    _q4_check(handle, lib().pkv_q4_attention_select(handle, n_seqs, _ptr(page_table), max_pages, _ptr(lengths), n_rows, _ptr(offsets), max_q_len,
                                                    max_len, ctypes.byref(sel), _ptr(q), *q_strides, _ptr(out), *out_strides, _ptr(state),
                                                    _ptr(workspace), workspace_bytes, _stream(stream)))


def pkv_q4_attention_route(handle, n_seqs, max_q_len, max_len, window=0, sinks=0, tree=None, tree_words=0):
    """-> (kernel, n_ctas, cluster), see include/pkv.h; tree as for pkv_q4_attention_select_workspace()."""
    out = [ctypes.c_int32(0) for _ in range(3)]
    sel = PkvQ4Select(window, sinks, None if tree is None else 8, tree_words)
    st = lib().pkv_q4_attention_route(handle, n_seqs, max_q_len, max_len, ctypes.byref(sel), *(ctypes.byref(x) for x in out))
    if st != PKV_OK:
        raise PkvError(st, "pkv_q4_attention_route(%r, %r, %r, window %r, sinks %r)" % (n_seqs, max_q_len, max_len, window, sinks))
    return tuple(x.value for x in out)


def pkv_q4_tree_masks(handle, n_seqs, lengths, n_rows, offsets, max_q_len, parents, window, sinks, tree, tree_words, depths, stream=None):
    _q4_check(handle, lib().pkv_q4_tree_masks(handle, n_seqs, _ptr(lengths), n_rows, _ptr(offsets), max_q_len, _ptr(parents), window, sinks,
                                              _ptr(tree), tree_words, _ptr(depths), _stream(stream)))


def pkv_q4_keep_rows(handle, n_seqs, page_table, max_pages, lengths, n_rows, offsets, paths, max_path, counts, lengths_out, stream=None):
    _q4_check(handle, lib().pkv_q4_keep_rows(handle, n_seqs, _ptr(page_table), max_pages, _ptr(lengths), n_rows, _ptr(offsets), _ptr(paths),
                                             max_path, _ptr(counts), _ptr(lengths_out), _stream(stream)))


def pkv_q4_plan_workspace(handle, n_seqs, n_rows) -> int:
    n = ctypes.c_int64(0)
    st = lib().pkv_q4_plan_workspace(handle, n_seqs, n_rows, ctypes.byref(n))
    if st != PKV_OK:
        raise PkvError(st, "pkv_q4_plan_workspace(%r, %r)" % (n_seqs, n_rows))
    return n.value


def pkv_q4_plan(handle, n_seqs, page_table, max_pages, lengths, rows, spans, ring, counters, window, sinks, lengths_out, spans_out,
                counters_out, offsets, n_rows, positions, slots, workspace, workspace_bytes, stream=None):
    _q4_check(handle, lib().pkv_q4_plan(handle, n_seqs, _ptr(page_table), max_pages, _ptr(lengths), _ptr(rows), _ptr(spans), _ptr(ring),
                                        _ptr(counters), window, sinks, _ptr(lengths_out), _ptr(spans_out), _ptr(counters_out), _ptr(offsets),
                                        n_rows, _ptr(positions), _ptr(slots), _ptr(workspace), workspace_bytes, _stream(stream)))


# ---- convenience wrapper ----------------------------------------------------------
def make_config(n_layers, n_kv_heads, n_q_heads, rank, sink_tokens, recent_tokens, max_seqs, max_pages_per_seq,
                n_dense_slots, n_factor_slots, head_dim=128, page_size=64, rank_v=None, softmax_scale=0.0,
                jacobi_max_sweeps=0, jacobi_tol=0.0, n_ctas=0, decode_variant=0, decode_overlap=0,
                jacobi_energy_tol=0.0, factor_bits=0, global_rank=0) -> PkvConfig:
    return PkvConfig(n_layers, n_kv_heads, n_q_heads, head_dim, page_size, rank, rank if rank_v is None else rank_v,
                     sink_tokens, recent_tokens, max_seqs, max_pages_per_seq, n_dense_slots, n_factor_slots,
                     softmax_scale, jacobi_max_sweeps, jacobi_tol, n_ctas, decode_variant, jacobi_energy_tol, factor_bits, decode_overlap,
                     global_rank)


class Cache:
    """Owns the device buffers (torch uint8 tensors) and the library handle."""

    def __init__(self, cfg: PkvConfig, device="cuda", dense_slot_order=None, factor_slot_order=None, dry_run=False):
        self.cfg = cfg
        self.sizes = pkv_query_sizes(cfg)
        self.dry_run = dry_run
        if dry_run:
            self.dense_pool = self.factor_pool = self.meta = self.workspace = None
            self.stream = None
        else:
            self.device = torch.device(device)
            self._device_index = self.dense_pool_device_index(self.device)
            mk = lambda n: torch.empty(max(int(n), 256), dtype=torch.uint8, device=self.device)
            self.dense_pool, self.factor_pool = mk(self.sizes.dense_pool_bytes), mk(self.sizes.factor_pool_bytes)
            self.meta, self.workspace = mk(self.sizes.meta_bytes), mk(self.sizes.workspace_bytes)
        self.handle = pkv_init_cache(cfg, self.dense_pool, self.factor_pool, self.meta, self.workspace,
                                     dense_slot_order, factor_slot_order)

    @staticmethod
    def dense_pool_device_index(device):
        return device.index if device.index is not None else torch.cuda.current_device()

    def _st(self):
        if self.dry_run:
            return None
        if _raw_current_stream is not None:
            return _raw_current_stream(self._device_index)
        return torch.cuda.current_stream(self.device)

    def append_kv(self, layer, seq_ids, n_new, k=None, v=None):
        pkv_append_kv(self.handle, layer, seq_ids, n_new, k, v, self._st())

    def compress_eligible_pages(self, layer=-1):
        return pkv_compress_eligible_pages(self.handle, layer, self._st())

    def compress_begin(self, layer, side_stream=None):
        return pkv_compress_begin(self.handle, layer, self._st(), side_stream)

    def compress_commit(self, layer=-1):
        return pkv_compress_commit(self.handle, layer, self._st())

    def decode_attention(self, layer, seq_ids, q=None, out=None, out_f32=None):
        if out is None and q is not None:
            out = torch.empty_like(q)
        pkv_decode_attention(self.handle, layer, seq_ids, q, out, out_f32, self._st())
        return out

    def decode_attention_multi(self, layer, seq_ids, q_len, q=None, out=None, out_f32=None):
        if out is None and q is not None:
            out = torch.empty_like(q)
        pkv_decode_attention_multi(self.handle, layer, seq_ids, q_len, q, out, out_f32, self._st())
        return out

    def decode_attention_partial(self, layer, seq_ids, q, state=None):
        if state is None:
            state = torch.empty((q.shape[0], q.shape[1], q.shape[2] + 2), dtype=torch.float32, device=q.device)
        pkv_decode_attention_partial(self.handle, layer, seq_ids, q, state, self._st())
        return state

    def decode_attention_host(self, layer, seq_ids, q_host, out_host, q_stage, out_stage):
        pkv_decode_attention_host(self.handle, layer, seq_ids, q_host, out_host, q_stage, out_stage, self._st())

    def page_table(self, seq, layer):
        return pkv_get_page_table(self.handle, seq, layer, self.cfg.max_pages_per_seq)

    def stats(self):
        return pkv_get_stats(self.handle, self._st())

    def free_seq(self, seq):
        pkv_free_seq(self.handle, seq)

    def read_basis(self, seq, layer, kv_head):
        """Global SVD form: (B_k, B_v), each [global_rank, d] bf16."""
        c = self.cfg
        B_k = torch.empty((c.global_rank, c.head_dim), dtype=torch.bfloat16, device=self.device)
        B_v = torch.empty_like(B_k)
        pkv_read_basis(self.handle, seq, layer, kv_head, B_k, B_v, self._st())
        return B_k, B_v

    def read_factors(self, slot, kv_head):
        c = self.cfg
        mk = lambda *s: torch.empty(s, dtype=torch.bfloat16, device=self.device)
        if c.global_rank > 0:                               # only the token rows are stored per page
            A_k, A_v = mk(c.page_size, c.global_rank), mk(c.page_size, c.global_rank)
            pkv_read_factors(self.handle, slot, kv_head, A_k, None, A_v, None, self._st())
            return A_k, None, A_v, None
        A_k, B_k = mk(c.page_size, c.rank_k), mk(c.rank_k, c.head_dim)
        A_v, B_v = mk(c.page_size, c.rank_v), mk(c.rank_v, c.head_dim)
        pkv_read_factors(self.handle, slot, kv_head, A_k, B_k, A_v, B_v, self._st())
        return A_k, B_k, A_v, B_v

    def write_factors(self, slot, kv_head, A_k, B_k, A_v, B_v):
        ts = [t.to(device=self.device, dtype=torch.bfloat16).contiguous() for t in (A_k, B_k, A_v, B_v)]
        pkv_write_factors(self.handle, slot, kv_head, *ts, self._st())
        torch.cuda.current_stream(self.device).synchronize()     # keep `ts` alive until the copy kernel ran

    def read_dense(self, slot, kv_head):
        c = self.cfg
        K = torch.empty((c.page_size, c.head_dim), dtype=torch.bfloat16, device=self.device)
        V = torch.empty_like(K)
        pkv_read_dense(self.handle, slot, kv_head, K, V, self._st())
        return K, V

    def close(self):
        if self.handle is not None:
            if not self.dry_run:
                torch.cuda.synchronize(self.device)
            pkv_destroy_cache(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


_INT32, _INT64 = torch.int32, torch.int64
_Q4_DTYPES = {torch.bfloat16: PKV_DTYPE_BF16, torch.float16: PKV_DTYPE_FP16}


def make_q4_config(n_kv_heads, n_q_heads, n_pages, head_dim=128, page_size=64, group_size=32, dtype=torch.bfloat16,
                   softmax_scale=0.0, n_ctas=0) -> PkvQ4Config:
    if dtype not in _Q4_DTYPES:
        raise PkvError(PKV_ERR_UNSUPPORTED, "dtype must be torch.bfloat16 or torch.float16, not %r" % (dtype,))
    return PkvQ4Config(n_kv_heads, n_q_heads, head_dim, page_size, group_size, _Q4_DTYPES[dtype], n_pages, softmax_scale, n_ctas)


class Q4Plan(NamedTuple):
    """What Q4Cache.plan() writes: int32 lengths [n_seqs], offsets [n_seqs + 1], positions [n_rows], spans [n_seqs, 2], int64 slots
    [n_rows], counters [4] (head, tail, pages missing, requests refused)."""
    lengths: torch.Tensor
    offsets: torch.Tensor
    positions: torch.Tensor
    slots: torch.Tensor
    spans: torch.Tensor
    counters: torch.Tensor


class Q4Cache:
    """A paged KV cache held in 4 bits (see include/pkv.h): owns the pool and the library handle.

    page_table: int32 [n_seqs, max_pages], lengths: int32 [n_seqs] (tokens of each sequence, the rows of the call included),
    both on the cache's device.  Row buffers are either [n_seqs, n, heads, d] (n rows of every sequence) or, with
    offsets (int32 [n_seqs + 1]), [rows, heads, d] with rows offsets[s] .. offsets[s + 1] - 1 belonging to sequence s; the rows
    are the sequence's last positions.  Rows and heads may be strided (slices of a fused projection).  Calls run on the
    current stream of the cache's device.
    """

    def __init__(self, cfg: PkvQ4Config, device="cuda", dry_run=False):
        self.cfg = cfg
        self.handle = None
        self.sizes = pkv_q4_query_sizes(cfg)
        self.dry_run = dry_run
        self.dtype = torch.float16 if cfg.dtype == PKV_DTYPE_FP16 else torch.bfloat16
        self._d, self._hq, self._hk = cfg.head_dim, cfg.n_q_heads, cfg.n_kv_heads
        self._workspaces = {}
        if dry_run:
            self.device, self._device_index, self.pool, self.meta = torch.device("cpu"), -1, None, None
            self.handle = pkv_q4_init_cache(cfg, None, None)
        else:
            self._device_index = Cache.dense_pool_device_index(torch.device(device))
            self.device = torch.device("cuda", self._device_index)
            self.pool = torch.empty(self.sizes.pool_bytes, dtype=torch.uint8, device=self.device)
            self.meta = torch.empty(self.sizes.meta_bytes, dtype=torch.uint8, device=self.device)
            with torch.cuda.device(self._device_index):
                self.handle = pkv_q4_init_cache(cfg, self.pool, self.meta)

    def _fail(self, message):
        raise PkvError(PKV_ERR_INVALID_ARG, message)

    def _stream(self):
        if self.dry_run:
            return None
        if _raw_current_stream is not None:
            return _raw_current_stream(self._device_index)
        return torch.cuda.current_stream(self.device).cuda_stream

    def _call(self, fn, *args):
        """A C call with the cache's device current (the library refuses another one)."""
        handle = None if self.handle is None else self.handle.value
        try:
            st = fn(handle, *args)
        except (TypeError, OverflowError) as e:          # an argument that is no whole number, or too large for the C call
            self._fail(str(e))
        if st != PKV_OK:
            if not self.dry_run and torch.cuda.current_device() != self._device_index:
                with torch.cuda.device(self._device_index):
                    st = fn(handle, *args)
            _q4_check(self.handle, st)

    # A decode step makes a few of these calls per layer and each is some microseconds of host time: the checks below are
    # written for the calls that pass them.
    def _seqs(self, page_table, lengths, offsets):
        dev, shape = self._device_index, page_table.shape
        if not (len(shape) == 2 and page_table.dtype is _INT32 and page_table.get_device() == dev and page_table.is_contiguous()):
            self._fail("page_table must be a contiguous int32 tensor [n_seqs, max_pages] on %s" % self.device)
        if not (lengths.dim() == 1 and lengths.numel() == shape[0] and lengths.dtype is _INT32 and lengths.get_device() == dev and lengths.is_contiguous()):
            self._fail("lengths must be a contiguous int32 tensor [n_seqs] on %s" % self.device)
        if offsets is not None and not (offsets.dim() == 1 and offsets.numel() == shape[0] + 1 and offsets.dtype is _INT32 and
                                        offsets.get_device() == dev and offsets.is_contiguous()):
            self._fail("offsets must be a contiguous int32 tensor [n_seqs + 1] on %s" % self.device)
        return shape

    def _rows(self, name, t, heads, n_seqs, ragged):
        """-> rows, row stride, head stride of a row buffer."""
        shape, d = t.shape, self._d
        if t.dtype is not self.dtype or t.get_device() != self._device_index:
            self._fail("%s must be %s on %s" % (name, self.dtype, self.device))
        if ragged:
            if len(shape) != 3 or shape[1] != heads or shape[2] != d:
                self._fail("%s must be [rows, %d, %d] with offsets" % (name, heads, d))
            row, head, ch = t.stride()
            n = shape[0]
        else:
            if len(shape) != 4 or shape[0] != n_seqs or shape[2] != heads or shape[3] != d:
                self._fail("%s must be [%d, n, %d, %d] without offsets" % (name, n_seqs, heads, d))
            seq, row, head, ch = t.stride()
            n = n_seqs * shape[1]
            if shape[1] <= 1:
                row = seq
            elif n_seqs > 1 and seq != shape[1] * row:
                self._fail("%s: the rows of all sequences must be equally far apart (pass [rows, heads, d] and offsets)" % name)
        if ch != 1:
            self._fail("%s: the channels of a head must be adjacent" % name)
        if heads == 1:
            head = d                                     # a size-1 axis may carry any stride
        if n <= 1:
            row = heads * d
        return n, row, head

    def append_kv(self, page_table, lengths, k, v, offsets=None):
        """Quantises the new rows k, v into the cache."""
        self._copy(_calls().append_kv, page_table, lengths, k, v, offsets)

    def read_kv(self, page_table, lengths, k, v, offsets=None):
        """Reads the last positions of each sequence back into k, v."""
        self._copy(_calls().read_kv, page_table, lengths, k, v, offsets)
        return k, v

    def _copy(self, fn, page_table, lengths, k, v, offsets):
        n_seqs, max_pages = self._seqs(page_table, lengths, offsets)
        ragged = offsets is not None
        n, k_row, k_head = self._rows("k", k, self._hk, n_seqs, ragged)
        nv, v_row, v_head = self._rows("v", v, self._hk, n_seqs, ragged)
        if n != nv:
            self._fail("k and v must have the same number of rows")
        self._call(fn, n_seqs, page_table.data_ptr(), max_pages, lengths.data_ptr(), n, offsets.data_ptr() if ragged else None,
                   k.data_ptr(), k_row, k_head, v.data_ptr(), v_row, v_head, self._stream())

    def attention(self, page_table, lengths, q, out=None, offsets=None, max_q_len=None, max_len=0, window=0, sinks=0, tree=None):
        """Attention of the newest positions over the cache; out (default: a new tensor of q's shape) is returned.  With
        offsets, max_q_len bounds the rows of a sequence (default, and at most: all rows); it and max_len, the longest length
        expected, choose the kernel and how the work is spread, so tight ones are faster.  Rows that belong to no sequence are
        left as they were (undefined in a new tensor); without rows nothing is done.

        window > 0: a query sees its own position, the window - 1 before it and the first `sinks` ones; pages that hold none of these may
        have gone back to the pool.  tree (int64, q's rows by words, see tree_masks()): the rows are drafted tokens, which see the context (or its
        part in the window) and the rows whose bits are set."""
        if out is None:
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
        elif out.shape != q.shape:
            self._fail("out must have the shape of q")
        self._attention(page_table, lengths, q, out, None, offsets, max_q_len, max_len, window, sinks, tree)
        return out

    def attention_partial(self, page_table, lengths, q, state=None, offsets=None, max_q_len=None, max_len=0, window=0, sinks=0, tree=None):
        """The same as softmax states [..., d + 2] fp32 (o, m, l) for pkv_merge_attention_states()."""
        shape = (*q.shape[:-1], q.shape[-1] + 2)
        if state is None:
            state = torch.empty(shape, dtype=torch.float32, device=q.device)
        elif state.shape != shape or state.dtype != torch.float32 or state.device != self.device or not state.is_contiguous():
            self._fail("state must be a contiguous fp32 tensor of shape %r on %s" % (shape, self.device))
        self._attention(page_table, lengths, q, None, state, offsets, max_q_len, max_len, window, sinks, tree)
        return state

    def _attention(self, page_table, lengths, q, out, state, offsets, max_q_len, max_len, window, sinks, tree):
        n_seqs, max_pages = self._seqs(page_table, lengths, offsets)
        ragged = offsets is not None
        n, q_row, q_head = self._rows("q", q, self._hq, n_seqs, ragged)
        o_row, o_head = q_row, q_head
        if out is not None:
            _, o_row, o_head = self._rows("out", out, self._hq, n_seqs, ragged)
        words = 0
        if tree is not None:
            if not (tree.dim() == q.dim() - 1 and tree.shape[:-1] == q.shape[:-2] and tree.dtype is _INT64 and tree.get_device() == self._device_index and
                    tree.is_contiguous() and tree.shape[-1] > 0):
                self._fail("tree must be a contiguous int64 tensor %r on %s, of a word at least" % ([*q.shape[:-2], "words"], self.device))
            words = tree.shape[-1]
        part = window or sinks or tree is not None
        if part:
            self._positions(window, sinks)
        if n == 0:
            return
        if not ragged:
            max_q_len = q.shape[1]
        elif max_q_len is None:
            max_q_len = n
        if max_q_len == 0:
            return
        most = max_pages * self.cfg.page_size
        if not 0 < max_len < most:
            max_len = most
        key = (n_seqs, max_q_len, max_len, window, sinks, words) if part else (n_seqs, max_q_len, max_len)
        size = self._workspaces.get(key)
        if size is None:
            if len(self._workspaces) >= 256:
                self._workspaces.clear()
            if part:
                size = pkv_q4_attention_select_workspace(self.handle, n_seqs, max_q_len, max_len, window, sinks, tree, words)
            else:
                size = pkv_q4_attention_workspace(self.handle, n_seqs, max_q_len, max_len)
            self._workspaces[key] = size
        # (from the caching allocator at each call: ordered with this stream, and private to a graph that is being captured)
        work = torch.empty(size, dtype=torch.uint8, device=self.device) if size and not self.dry_run else None
        if part:
            self._call(_calls().attention_select, n_seqs, page_table.data_ptr(), max_pages, lengths.data_ptr(), n,
                       offsets.data_ptr() if ragged else None, max_q_len, max_len, q.data_ptr(), q_row, q_head,
                       None if out is None else out.data_ptr(), o_row, o_head, None if state is None else state.data_ptr(),
                       None if work is None else work.data_ptr(), size, self._stream(), window, sinks, None if tree is None else tree.data_ptr(), words)
            return
        self._call(_calls().attention, n_seqs, page_table.data_ptr(), max_pages, lengths.data_ptr(), n,
                   offsets.data_ptr() if ragged else None, max_q_len, max_len, q.data_ptr(), q_row, q_head,
                   None if out is None else out.data_ptr(), o_row, o_head, None if state is None else state.data_ptr(),
                   None if work is None else work.data_ptr(), size, self._stream())

    def _positions(self, window, sinks):
        self._whole("window", window, (1 << 31) - 1)      # (beyond 32 bits they would arrive as other numbers)
        self._whole("sinks", sinks, (1 << 31) - 1)

    def _whole(self, name, x, most):
        """A size, from 0 to `most`: looked at before anything is allocated by it."""
        if type(x) is int and 0 <= x <= most:
            return
        try:
            ok = 0 <= index(x) <= most
        except TypeError:
            ok = False
        if not ok:
            self._fail("%s must be a whole number from 0 to %d, not %r" % (name, most, x))

    def _ints(self, name, t, shape, dtype=_INT32):
        if not (t.shape == shape and t.dtype is dtype and t.get_device() == self._device_index and t.is_contiguous()):
            self._fail("%s must be a contiguous %s tensor %r on %s" % (name, str(dtype)[6:], list(shape), self.device))

    def tree_masks(self, parents, lengths=None, offsets=None, max_q_len=None, window=0, sinks=0):
        """Masks and depths of drafted tokens.  parents: int32 [n_seqs, n], or [rows] with offsets: the row of the same sequence, an
        earlier one, that a row continues, -1 for the last token of the context.  -> (int64 parents.shape + (words,), for attention(tree=...),
        int32 depths of parents' shape: a row's position is the context's length + its depth).  With a window and sinks, those of the attention call and the
        sequences' lengths (the rows included).  With offsets, max_q_len bounds the rows of a sequence (default: all rows)."""
        self._positions(window, sinks)
        shape, n, dev = parents.shape, parents.numel(), self._device_index
        if offsets is None:
            if len(shape) != 2:
                self._fail("parents must be [rows] with offsets and [n_seqs, n] without")
            n_seqs, max_q_len = shape
        else:
            if len(shape) != 1:
                self._fail("parents must be [rows] with offsets and [n_seqs, n] without")
            n_seqs = offsets.numel() - 1
            if max_q_len is None:
                max_q_len = n
            self._whole("max_q_len", max_q_len, n)
            self._ints("offsets", offsets, (n_seqs + 1,))
        if not (parents.dtype is _INT32 and parents.get_device() == dev and parents.is_contiguous()):
            self._ints("parents", parents, shape)
        if lengths is not None:
            if not (lengths.dtype is _INT32 and lengths.shape == (n_seqs,) and lengths.get_device() == dev and lengths.is_contiguous()):
                self._ints("lengths", lengths, (n_seqs,))
        elif window and sinks:
            self._fail("a window with sinks needs the sequences' lengths")
        words = max_q_len + 63 >> 6 if max_q_len > 0 else 1
        depths = torch.empty_like(parents)
        masks = torch.empty(*shape, words, dtype=_INT64, device=self.device)
        self._call(_calls().tree_masks, n_seqs, None if lengths is None else lengths.data_ptr(), n, None if offsets is None else offsets.data_ptr(),
                   max_q_len, parents.data_ptr(), window, sinks, masks.data_ptr(), words, depths.data_ptr(), self._stream())
        return masks, depths

    def keep_rows(self, page_table, lengths, paths, counts, new_rows, offsets=None, out=None):
        """Keeps the accepted ones of the newest rows: row paths[s, i] (int32 [n_seqs, m]) of sequence s becomes its new row i, for
        i < counts[s] (int32 [n_seqs]); rows of a path ascend.  new_rows: how many new rows each sequence has, or with offsets how many
        the call has.  -> the lengths (out, a tensor that overlaps none of the others, or a new one)."""
        n_seqs, max_pages = self._seqs(page_table, lengths, offsets)
        dev, most = self._device_index, paths.shape
        if not (len(most) == 2 and most[0] == n_seqs and paths.dtype is counts.dtype is _INT32 and counts.shape == (n_seqs,) and
                paths.get_device() == counts.get_device() == dev and paths.is_contiguous() and counts.is_contiguous()):
            self._ints("paths", paths, (n_seqs, most[-1] if len(most) == 2 else "m"))
            self._ints("counts", counts, (n_seqs,))
        if out is None:
            out = torch.empty_like(lengths)
        else:
            self._ints("out", out, (n_seqs,))
        n = new_rows if offsets is not None else new_rows * n_seqs
        self._call(_calls().keep_rows, n_seqs, page_table.data_ptr(), max_pages, lengths.data_ptr(), n, None if offsets is None else offsets.data_ptr(),
                   paths.data_ptr(), most[1], counts.data_ptr(), out.data_ptr(), self._stream())
        return out

    def new_ring(self, pages=None):
        """Free pages (default: all of the pool) as plan() takes them: (ring int32 [n_pages], counters int64 [4])."""
        n = self.cfg.n_pages
        pages = torch.arange(n) if pages is None else torch.as_tensor(pages).flatten().cpu()
        whole = pages.numel() == 0 or not (pages.is_floating_point() or pages.is_complex() or pages.dtype is torch.bool)
        pages = pages.to(_INT64)                         # (in 32 bits 2^32 + 4 would be 4)
        if not whole or pages.numel() > n or (pages.numel() and not (0 <= int(pages.min()) and int(pages.max()) < n)) or pages.unique().numel() != pages.numel():
            self._fail("pages must be different page numbers of the pool")
        ring = torch.full((n,), -1, dtype=_INT32)
        ring[:pages.numel()] = pages.to(_INT32)
        return ring.to(self.device), torch.tensor([0, pages.numel(), 0, 0], dtype=_INT64, device=self.device)

    def plan(self, page_table, lengths, rows, spans, ring, counters, n_rows, window=0, sinks=0, out=None):
        """Plans a step on the device (see pkv_q4_plan in include/pkv.h): rows int32 [n_seqs] new rows for each request, -1 where it is
        done; spans int32 [n_seqs, 2] the table entries it holds; ring, counters: free pages, see new_ring(); n_rows: a bound of the new rows
        in all.  Writes new entries into page_table and returned pages into ring.  -> Q4Plan of new tensors, or `out`, whose
        lengths, spans and counters may be the ones given (in place; no other tensors may overlap).  Where pages are missing or requests make no sense nothing is done: counters[2:]."""
        n_seqs, max_pages = self._seqs(page_table, lengths, None)
        self._positions(window, sinks)
        self._whole("n_rows", n_rows, 0x3fffffff)
        dev, one = self._device_index, (n_seqs,)
        if not (rows.dtype is spans.dtype is ring.dtype is _INT32 and counters.dtype is _INT64 and rows.shape == one and spans.shape == (n_seqs, 2) and
                ring.shape == (self.cfg.n_pages,) and counters.shape == (4,) and
                rows.get_device() == spans.get_device() == ring.get_device() == counters.get_device() == dev and
                rows.is_contiguous() and spans.is_contiguous() and ring.is_contiguous() and counters.is_contiguous()):
            self._ints("rows", rows, one)
            self._ints("spans", spans, (n_seqs, 2))
            self._ints("ring", ring, (self.cfg.n_pages,))
            self._ints("counters", counters, (4,), _INT64)
        if out is None:
            # (each from the allocator: slices of one tensor take longer)
            out = Q4Plan(torch.empty_like(lengths), lengths.new_empty(n_seqs + 1), lengths.new_empty(n_rows), counters.new_empty(n_rows), torch.empty_like(spans),
                         torch.empty_like(counters))
        else:
            self._ints("out.lengths", out.lengths, one)
            self._ints("out.spans", out.spans, (n_seqs, 2))
            self._ints("out.counters", out.counters, (4,), _INT64)
            self._ints("out.offsets", out.offsets, (n_seqs + 1,))
            if out.positions is not None:
                self._ints("out.positions", out.positions, (n_rows,))
            if out.slots is not None:
                self._ints("out.slots", out.slots, (n_rows,), _INT64)
        key = (n_seqs, n_rows)
        size = self._workspaces.get(key)
        if size is None:
            if len(self._workspaces) >= 256:
                self._workspaces.clear()
            size = self._workspaces[key] = pkv_q4_plan_workspace(self.handle, n_seqs, n_rows)
        work = torch.empty(size, dtype=torch.uint8, device=self.device) if size and not self.dry_run else None
        pos, slots = out.positions, out.slots
        self._call(_calls().plan, n_seqs, page_table.data_ptr(), max_pages, lengths.data_ptr(), rows.data_ptr(), spans.data_ptr(), ring.data_ptr(),
                   counters.data_ptr(), window, sinks, out.lengths.data_ptr(), out.spans.data_ptr(), out.counters.data_ptr(), out.offsets.data_ptr(), n_rows,
                   None if pos is None else pos.data_ptr(), None if slots is None else slots.data_ptr(), None if work is None else work.data_ptr(), size,
                   self._stream())
        return out

    def stats(self):
        if not self.dry_run:
            with torch.cuda.device(self._device_index):
                return pkv_q4_get_stats(self.handle, self._stream())
        return pkv_q4_get_stats(self.handle)

    def close(self):
        if self.handle is not None:
            if not self.dry_run:
                torch.cuda.synchronize(self.device)
            pkv_q4_destroy_cache(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
