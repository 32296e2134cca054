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
