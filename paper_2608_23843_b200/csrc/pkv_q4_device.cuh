// Device-side helpers shared by the kernels that attend over the 4-bit cache.  Internal linkage, as in pkv_device.cuh.
#pragma once

#include <cuda_fp16.h>

#include "pkv_device.cuh"
#include "pkv_q4.h"

namespace pkv {

namespace {

constexpr int kQ4Unit = 64;            // tokens per unit: four tiles
constexpr int kQ4UnitTiles = kQ4Unit / kQ4Tile;
// Weights in fp16: a reference places the largest near 2^kQ4Place and follows when one may have passed 2^kQ4Most (fp16
// holds 2^16 less an eighth).  fp16's smallest step is 2^-24, so weights down to 2^-(13 + kQ4Place) of the largest are rounded by 2^-11
// of themselves and smaller ones by 2^-(24 + kQ4Place) of the largest.  Placed higher, the reference moves more often (kQ4Place 6 / 8 / 10: one
// sequence of 128K 41.5 / 42 / 43 us, 8 x 4 positions 110 / 114 / 118, 2048 positions 1254 / 1281 / 1296); at 6 what 2^17 tokens lose together is 2^-13 of the
// largest at most.
constexpr float kQ4Place = 6.f, kQ4Most = 15.9f;

// A segment that begins in a CTA and ends in another (seq < 0: none); slot: where its first part is (see below)
struct Q4Part { int seq, tile, head, slot, last_cta; };

// Partial states: two per CTA (its first segment, its last), each [rows of a tile or block][D] o, then m and l of the rows.
__host__ __device__ inline long long q4_state_floats(int rows, int d) { return (long long)rows * (d + 2); }
__host__ __device__ inline long long q4_parts_bytes(int n_ctas) { return ((long long)n_ctas * (int)sizeof(Q4Part) + 255) / 256 * 256; }

// The rows of a sequence that the call works on; `all`: with those beyond the caller's bound, which the positions go by.
__device__ __forceinline__ int q4_new_rows(const Q4AttentionArgs &a, int s, int &first, int &all, int *status) {
    first = q4_first_row(a.rows, s);
    all = q4_first_row(a.rows, s + 1) - first;
    if (status && all > a.max_q_len) atomicAdd(status + 2, 1);
    return max(0, min(all, a.max_q_len));
}

// ---- Queries that see a part of the positions (Q4AttentionArgs: window, sinks, tree) -----------------------------------
// A run of units (64 tokens) that holds what any of some query rows sees: the first `su` of a sequence, then those behind a gap.
struct Q4Span { int units, su, gap, lo; };             // lo: the lowest position behind the sinks that one of the rows sees
// see: the positions below it are visited; low: the rows' lowest position in the window (0 or less: no gap)
__device__ __forceinline__ Q4Span q4_span(const Q4AttentionArgs &a, int see, int low) {
    const int all = (see + kQ4Unit - 1) / kQ4Unit;
    Q4Span r;
    r.lo = max(0, low);
    r.su = min((int)(((unsigned)a.sinks + kQ4Unit - 1) / kQ4Unit), all);
    r.gap = max(0, r.lo / kQ4Unit - r.su);
    r.units = max(1, all - r.gap);
    return r;
}
// The lowest position in the window of new row j of a sequence with a context of C tokens, or of any row of a tree (whose own position counts at
// least).  Pages below it may have gone back.
__device__ __forceinline__ int q4_lowest(const Q4AttentionArgs &a, int C, int j) {
    return a.window ? C + (a.tree ? 0 : j) + 1 - a.window : 0;
}
// Tiles of the unit at t0 that have to be there (of the first `tiles`): those of parts - a page's, or the whole unit - that hold a position
// below the sinks or from lo on.  Pages of other parts may be anyone's.
__device__ __forceinline__ uint32_t q4_needed(const Q4AttentionArgs &a, int t0, int lo, int tiles, int n_parts, int per_page, int per_tiles) {
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < n_parts && (t0 + i * per_page < a.sinks || t0 + (i + 1) * per_page > lo)) bits |= ((1u << per_tiles) - 1u) << (i * per_tiles);
    return bits & ((1u << tiles) - 1u);
}
// What a query row sees: positions from lo (or below the sinks) up to `end`, and new rows by the bits of its mask.
struct Q4Seen { int lo, end; };
__device__ __forceinline__ Q4Seen q4_seen(const Q4AttentionArgs &a, int T, int all, int first, int j) {
    const int C = T - all;
    if (!a.tree) return Q4Seen{a.window ? max(0, C + j + 1 - a.window) : 0, C + j + 1};
    int own = 0;
    if (a.window) {                                    // new rows that it sees, of those the sequence has
        const unsigned long long *w = a.tree + (long long)(first + j) * a.tree_words;
        for (int i = 0; i < min(a.tree_words, (all + 63) >> 6); ++i) own += __popcll(__ldg(w + i) & (all - 64 * i >= 64 ? ~0ull : (1ull << (all - 64 * i)) - 1ull));
    }
    return Q4Seen{a.window ? max(0, C + max(own, 1) - a.window) : 0, C};
}
__device__ __forceinline__ unsigned long long q4_below(int x) { return x <= 0 ? 0ull : x >= 64 ? ~0ull : (1ull << x) - 1ull; }
// ... as bits of the unit at t0
__device__ __forceinline__ unsigned long long q4_unit_mask(const Q4AttentionArgs &a, const Q4Seen &v, int t0, int T, int all, long long row) {
    unsigned long long m = q4_below(v.end - t0) & (~q4_below(v.lo - t0) | q4_below(a.sinks - t0));
    const int at = t0 - (T - all);                     // the unit's first token as a new row
    if (a.tree && at > -64) {
        const unsigned long long *w = a.tree + row * a.tree_words;
        const int i = at >> 6, sh = at & 63;
        unsigned long long x = 0;
        if (i >= 0 && i < a.tree_words) x = __ldg(w + i) >> sh;
        if (sh && i + 1 < a.tree_words) x |= __ldg(w + i + 1) << (64 - sh);      // (i + 1 >= 0)
        m |= x & q4_below(T - t0);
    }
    return m;
}
// the tiles that are there, 16 bits each
__device__ __forceinline__ unsigned long long q4_tile_mask(uint32_t tiles) {
    const uint32_t lo = (tiles & 1u ? 0xffffu : 0u) | (tiles & 2u ? 0xffff0000u : 0u), hi = (tiles & 4u ? 0xffffu : 0u) | (tiles & 8u ? 0xffff0000u : 0u);
    return (unsigned long long)hi << 32 | lo;
}

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t max_bf16(uint32_t x, uint32_t y) {      // (the other operand where one is NaN)
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(y));
    return r;
}
__device__ __forceinline__ uint32_t sub_h2(uint32_t x, uint32_t y) {
    uint32_t r;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(y));
    return r;
}
// (volatile: where it is written down, and not kept in registers for later)
__device__ __forceinline__ void lds128(uint32_t *r, uint32_t at) {
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at));
}
// Bounded wait that also ends when another warp has given up.  The thread sleeps until the phase completes (or for some
// microseconds at a time): a warp that polls instead takes issue slots from the ones that work.
__device__ __forceinline__ bool mbar_sleep(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(bar), "r"(parity), "r"(20000u) : "memory");
    return ok != 0;
}
__device__ __forceinline__ bool mbar_wait_or(uint32_t bar, uint32_t parity, volatile int *abort_flag) {
    if (mbar_sleep(bar, parity)) return true;
    const long long t0 = clock64();
    while (!mbar_sleep(bar, parity))
        if (clock64() - t0 > kWaitClocks || *abort_flag) return false;
    return true;
}
// the same for a whole warp: the outcome is the same for all lanes
__device__ __forceinline__ bool mbar_wait_warp(uint32_t bar, uint32_t parity, volatile int *abort_flag) {
    return __all_sync(0xffffffffu, mbar_wait_or(bar, parity, abort_flag));
}

}  // namespace

}  // namespace pkv
