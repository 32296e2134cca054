// Attention over the paged 4-bit cache, many query rows per KV head (a chunk of a prefill, a few dozen new positions), on
// the fifth-generation tensor cores.
//
// A CTA works on blocks of up to 256 query rows of one (sequence, KV head), as two halves of 128 (the M dimension of every
// product; one thread owns one row).  A block of at most 128 rows gives both halves the same rows and every other unit, and
// their states are joined at its end.  Tokens come in units of 64:
//     one warp       looks up pages and copies a unit's tiles of codes and scales into a ring,
//     four warps     widen, a tile each: codes times scales as fp16 into shared memory, in the layouts the products read
//                    (128-byte swizzle, panels of 64 channels).  A code (3 bits and a sign) times a bf16 scale (8 bits) has
//                    11 bits, so fp16 holds it exactly where the scale is in its range: a power of two per tile, or per token in tiles of
//                    uneven sizes, is handed on to the rows, and what is left lies at the upper end of the range, so that channel groups
//                    down to 2^-19 (values: 2^-20) of their row's largest are exact too,
//     one warp       issues the products, one lane: s = Q K^T with Q and, later, p as row operands in tensor memory,
//                    o += p V; while one half's rows are in their softmax the other half's products run,
//     eight warps    softmax (fp32): s from tensor memory, p as fp16 back over it, o rescaled only when a row's weights may have passed
//                    fp16's range (see kQ4Place).
// Measured: 2048 positions against 32K (32 / 8 heads, d = 128, g = 32; 1.07 TFLOP, one call) 1256 to 1293 us, 840 TFLOP/s; 5 x 37
// positions of sequences up to 4001 (28 / 4 heads, d = 64) 28 us, of which the launch, the partition, the first units, the last
// states and the join are most.
// What bounds it: products and exponentials each take 1024 cycles per unit of 256 rows, but a half's chain - s, softmax, o,
// the hand-overs between them - is some 1800 cycles long even with both for free, and the widening competes with the softmax
// for issue slots (tensor pipe 39 %, exponentials 40 %, issue slots 55 % busy).  Tried on the same call and not kept: Q of one half in shared memory
// so that s of the next unit can be computed behind the softmax (the products then wait for shared memory), s in two
// buffers of 32 tokens for the same end (1509 us: twice the hand-overs, 40 products to issue per unit instead of 24; 1364 with an
// issuing warp per half, which by itself costs more than it gives, 1501), five or six
// widening warps, a quarter of the exponentials by polynomial, the halves' exponentials in turn, weights with the old
// reference before the maximum is known.
// Where queries see a part of the positions (kSel) a block visits the units from its first row's window on and those of the sinks: 2048 positions with a
// window of 4096 211 us (140 GFLOP, 66 units a block), 8 drafted trees of 64 against 32K 354 us (274 GFLOP).
// CTAs share the batch's units evenly, one CTA per SM; blocks that span CTAs leave states that a second kernel joins.  Units
// after a block's last visible position are not visited.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <type_traits>

#include "pkv_q4_device.cuh"
#include "pkv_umma.cuh"

namespace pkv {

namespace {

constexpr int kBRows = kQ4BlockRows, kBHalf = 128;
constexpr int kBRowWarps = 8;
// kPairs: where a call's blocks have 128 rows at most, and queries see a part of the positions, keys and values of a tile are widened by a warp
// each: both halves then have the same rows and every other unit, and the widening is what takes longest (8 x 16 drafted tokens against 16000: 162 ->
// 140 us; with rows of their own for both halves the row threads need the issue slots: 8 x 64 against 32K 356 -> 370).  The 18 warps take
// registers in the shares below, in whole groups of four warps (two idle ones make up the last): they start with 96 a thread.  The shares do not
// hold everything: 500 to 580 bytes of a thread's values are spilled and 690 to 740 loaded again, against 200 to 230 and 360 to 370 without kPairs (128 registers a thread).
__host__ __device__ constexpr int block_widen_warps(bool pairs) { return pairs ? 2 * kQ4UnitTiles : kQ4UnitTiles; }
__host__ __device__ constexpr int block_threads(bool pairs) { return 32 * (kBRowWarps + block_widen_warps(pairs) + (pairs ? 4 : 2)); }
constexpr int kBRegs = 96, kBRowRegs = 144, kBWidenRegs = 64, kBOtherRegs = 64;
static_assert(block_threads(true) * kBRegs <= 65536 && 256 * kBRowRegs + 256 * kBWidenRegs + 128 * kBOtherRegs <= block_threads(true) * kBRegs,
              "more would be waited for in vain");
constexpr uint32_t kBTmemCols = 512;

template <int D, int NG>
struct BlockShape {
    static constexpr int kPanels = D / 64, kSide = kPanels * kQ4Unit * 128, kWide = 2 * kSide;      // K panels, then V panels of a unit
    static constexpr int kTile = kQ4Tile * (D + 4 * NG), kUnitBytes = kQ4UnitTiles * kTile, kCodes = (kUnitBytes + 127) / 128 * 128;
    static constexpr int kWideStages = 4, kFit = (222 * 1024 - kWideStages * kWide) / kCodes, kCodeStages = kFit < 8 ? kFit : 8;
    static constexpr int kSmem = kWideStages * kWide + kCodeStages * kCodes + 1024;                 // (+ alignment)
    static_assert(kCodeStages >= 4 && kSmem <= 220 * 1024, "fits one CTA per SM");
    // columns of tensor memory: o of both halves, Q of both (fp16 pairs), s of both
    static constexpr uint32_t kColO = 0, kColQ = 2 * D, kColS = kColQ + D;
    static_assert(kColS + 2 * kQ4Unit <= kBTmemCols, "fits tensor memory");
};

// sum over i < n of floor((a i + b) / m), for a, b >= 0 and m > 0 (by the Euclid-like recursion on (a, m))
__device__ long long floor_sum(long long n, long long m, long long a, long long b) {
    long long sum = 0;
    while (n > 0) {
        sum += n * (n - 1) / 2 * (a / m) + n * (b / m);
        a %= m;
        b %= m;
        const long long y = a * n + b;
        if (y < m) break;
        n = y / m;
        b = y % m;
        const long long t = m;
        m = a;
        a = t;
    }
    return sum;
}

// A sequence's blocks of query rows.  Block r's last row sees the first `see` tokens; it visits the units that hold them.
struct BlockSeq { int first, all, n, T, blocks, G; };

__device__ __forceinline__ BlockSeq block_seq(const Q4AttentionArgs &a, int s, int *status) {
    BlockSeq q;
    q.n = q4_new_rows(a, s, q.first, q.all, status);
    q.T = q4_length(a.rows, a.geo, s, status);
    q.G = a.geo.group;
    q.blocks = (int)(((long long)q.n * q.G + kBRows - 1) / kBRows);
    return q;
}
__device__ __forceinline__ int block_see(const BlockSeq &q, int r) {
    const int last = min(q.n - 1, ((r + 1) * kBRows - 1) / q.G);
    return q.all > q.T ? q.T : q.T - q.all + last + 1;                   // (more rows than tokens: not worth a rule of its own)
}
// kSel: what the block's rows see, from the window of its first row on (all rows of a tree visit the same)
__device__ __forceinline__ Q4Span block_span(const Q4AttentionArgs &a, const BlockSeq &q, int r) {
    return q4_span(a, a.tree ? q.T : block_see(q, r), q.all > q.T ? 0 : q4_lowest(a, q.T - q.all, (int)((long long)r * kBRows / q.G)));
}
template <bool kSel>
__device__ __forceinline__ int block_units(const Q4AttentionArgs &a, const BlockSeq &q, int r) {
    return kSel ? block_span(a, q, r).units : max(1, (block_see(q, r) + kQ4Unit - 1) / kQ4Unit);
}
// What a block costs a CTA beside its units - queries, results, the first unit's latency - in units.
constexpr int kBSegCost = 5;
// Units and fixed costs of all blocks of a sequence, for one head.  (The last block may end before its 256 rows do; the others
// have a closed form: block i's last row is 256 i + 255, its units floor((T - all + 1 + floor((256 i + 255) / G) + 63) / 64).)
// kSel: less the units before a block's window and behind the sinks, g(i) = max(0, floor((T - all + 1 - W + floor(256 i / G)) / 64) - su), whose
// terms are above zero from some block on.
template <bool kSel>
__device__ long long block_weight(const Q4AttentionArgs &a, const BlockSeq &q) {
    if (q.blocks == 0) return 0;
    const long long fixed = (long long)q.blocks * kBSegCost;
    if (q.all > q.T || (kSel && a.tree)) return fixed + (long long)q.blocks * block_units<kSel>(a, q, 0);
    long long sum = fixed + block_units<kSel>(a, q, q.blocks - 1);
    if (q.blocks <= 8) {                            // (few: adding them up beats the recursion's divisions)
        for (int i = 0; i < q.blocks - 1; ++i) sum += block_units<kSel>(a, q, i);
        return sum;
    }
    const long long A = (long long)q.T - q.all + 1 + kQ4Unit - 1;
    sum += floor_sum(q.blocks - 1, (long long)kQ4Unit * q.G, kBRows, kBRows - 1 + A * q.G);
    if (kSel && a.window) {
        const long long W = (long long)q.T - q.all + 1 - a.window, su = ((long long)a.sinks + kQ4Unit - 1) / kQ4Unit;
        const long long need = kQ4Unit * (su + 1) - W;                   // floor(256 i / G) from here on
        const long long i0 = need <= 0 ? 0 : (need * q.G + kBRows - 1) / kBRows;
        const long long n = q.blocks - 1 - i0;
        if (n > 0) sum -= floor_sum(n, (long long)kQ4Unit * q.G, kBRows, W * q.G + kBRows * i0) - n * su;
    }
    return sum;
}
// The block that holds position `at` of a sequence's weights (blocks in turn, all heads of one before the next), and the
// position where it begins; a whole warp, 32 blocks at a time.
template <bool kSel>
__device__ int block_locate(const Q4AttentionArgs &a, const BlockSeq &q, int H, long long at, long long &begins) {
    const int lane = threadIdx.x & 31;
    long long base = 0;
    for (int r0 = 0;; r0 += 32) {
        const int r = r0 + lane;
        const int v = r < q.blocks ? block_units<kSel>(a, q, r) + kBSegCost : 0;
        int x = v;                                  // (at most 32 * 2^25)
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, d);
            if (lane >= d) x += y;
        }
        const uint32_t before = __ballot_sync(0xffffffffu, base + (long long)x * H <= at);      // blocks that end before `at`
        const int k = __popc(before);
        const long long all = base + (long long)__shfl_sync(0xffffffffu, x, 31) * H;
        if (k < 32 || r0 + 32 >= q.blocks) {
            const int kk = min(k, min(31, q.blocks - 1 - r0));
            begins = base + (long long)(__shfl_sync(0xffffffffu, x, kk) - __shfl_sync(0xffffffffu, v, kk)) * H;
            return r0 + kk;
        }
        base = all;
    }
}

// A place in the batch's order of units: sequence, block, head, unit.
struct BlockCursor {
    int seq, block, head, unit, units;
    BlockSeq q;
    int su, gap, lo;                                // kSel: see Q4Span
};
template <bool kSel>
__device__ __forceinline__ void block_enter(const Q4AttentionArgs &a, BlockCursor &c) {
    if (kSel) {
        const Q4Span r = block_span(a, c.q, c.block);
        c.units = r.units; c.su = r.su; c.gap = r.gap; c.lo = r.lo;
    } else {
        c.units = block_units<false>(a, c.q, c.block);
    }
}
template <bool kSel>
__device__ __forceinline__ int block_unit_at(const BlockCursor &c, int unit) { return unit + (kSel && unit >= c.su ? c.gap : 0); }
template <bool kSel>
__device__ __forceinline__ void block_advance(const Q4AttentionArgs &a, BlockCursor &c, int by) {
    c.unit += by;
    while (c.unit >= c.units) {
        c.unit -= c.units;
        if (++c.head < a.geo.n_kv_heads) continue;
        c.head = 0;
        if (++c.block == c.q.blocks) {
            c.block = 0;
            do {
                if (++c.seq >= a.rows.n_seqs) return;
                c.q = block_seq(a, c.seq, nullptr);
            } while (c.q.blocks == 0);
        }
        block_enter<kSel>(a, c);
    }
}

// A tile's scales lose one power of two, that of the largest, which comes to 2^kBTop .. 2^(kBTop + 1): seven times that fits fp16, and
// a scale 2^-29 of it times a code is still exact.  Where a token's largest is further below than kBKeys (kBValues), the tile is uneven:
// each token has a power of two of its own.
constexpr uint32_t kBKeys = 10, kBValues = 9;
constexpr int kBTop = 12;
// Where values spread more than 2^kBSpread, a reference goes by each token's own.  Placed there, weights stay inside fp16: a token's may be
// 2^kBValues above what it adds.  (Measured, 2048 positions: 1256 us; with every other token's values 64 times larger 1494, with every
// other token's keys 1024 times smaller, all tiles uneven, 2145.)
constexpr uint32_t kBSpread = 4;
static_assert(kQ4Place + kBValues < kQ4Most, "see above");
// (values that are zero count as the least there are: their tokens' weights must not set the reference that all share)
constexpr int kBLeast = -80;                        // least exponent: below those of all values of the documented range, far above fp32's least

// What the widening warps tell the rows about a unit.
struct __align__(16) UnitInfo {
    float tk[kQ4Unit];                              // powers of two taken out of each token's keys, in uneven tiles
    float tv[kQ4Unit];                              // exponents of each token's values, in uneven tiles and where they spread
    float ek[kQ4UnitTiles];                         // ... of the other tiles' keys (uneven: 1)
    float ev[kQ4UnitTiles], ev_inv[kQ4UnitTiles];   // ... and values: exponents, and 2^-exponent (uneven: 0, 0)
    uint8_t odd_keys[kQ4UnitTiles];                 // kPairs: the first of these, by the warp that has the keys
    uint8_t odd[kQ4UnitTiles];                      // 1: uneven keys, 2: uneven values, 4: values that are not finite, 8: values that spread
    uint16_t v_nan[kQ4UnitTiles][4];                // per channel group: tokens whose values are not finite there (zeros here)
    uint32_t tiles, tokens;                         // which tiles are there; tokens of the sequence in the unit
};

__device__ __forceinline__ uint32_t h2_mul(uint32_t x, uint32_t y) {
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(y));
    return r;
}
// two codes as fp16 integers, from bits 0-3 (4-7) of either half: 1024 + 8 + code and 64 + 8 + code under a constant's exponent
__device__ __forceinline__ uint32_t codes_lo(uint32_t x) { return sub_h2((x & 0x000f000fu) | 0x64006400u, 0x64086408u); }
__device__ __forceinline__ uint32_t codes_hi(uint32_t x) { return sub_h2((x & 0x00f000f0u) | 0x54005400u, 0x54805480u); }

// shared-memory accesses in the order they are written down
__device__ __forceinline__ void lds32(uint32_t *r, uint32_t at) { asm volatile("ld.shared.u32 %0, [%1];" : "=r"(r[0]) : "r"(at)); }
__device__ __forceinline__ void lds64(uint32_t *r, uint32_t at) { asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "r"(at)); }
__device__ __forceinline__ void sts128(uint32_t at, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
template <int NG>
__device__ __forceinline__ void lds_scales(uint32_t *r, uint32_t at) {      // a token's scales, two to a word
    if (NG == 4) lds64(r, at);
    else if (NG == 2) lds32(r, at);
    else { uint16_t x; asm volatile("ld.shared.u16 %0, [%1];" : "=h"(x) : "r"(at)); r[0] = x; }
}

__device__ __forceinline__ uint64_t f2_fma3(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }      // -126 <= e <= 127

// kSel: the queries see a part of the positions
template <int D, int NG, bool H16, bool kSel, bool kPairs>
__global__ void __launch_bounds__(block_threads(kPairs), 1) q4_block_kernel(const __grid_constant__ Q4AttentionArgs a) {
    using S = BlockShape<D, NG>;
    constexpr int NW = D / 32, WPG = NW / NG, kWS = S::kWideStages, kCS = S::kCodeStages;
    constexpr int kBThreads = block_threads(kPairs), kWiden = block_widen_warps(kPairs), kBIssueWarp = kBRowWarps + kWiden, kBCopyWarp = kBIssueWarp + 1;
    const Q4Geometry &geo = a.geo;
    extern __shared__ unsigned char smem_raw[];
    unsigned char *wide = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u), *codes = wide + kWS * S::kWide;
    __shared__ unsigned long long code_full[kCS], code_empty[kCS], wide_full[kWS], wide_empty[kWS];
    __shared__ unsigned long long s_full[2], p_ready[2], q_ready[2], o_done[2], drain, state_ready, state_read;
    __shared__ uint32_t code_tiles[kCS], code_tokens[kCS];
    __shared__ UnitInfo info[kWS];
    __shared__ float2 ml_other[kBHalf];
    __shared__ uint32_t bad_other[kBHalf];
    __shared__ long long sums[kBThreads / 32], found_at;
    __shared__ int found_seq, gave_up;
    __shared__ uint32_t tmem_slot;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    volatile int *abort_flag = &gave_up;
    if (tid == 0) {
        for (int s = 0; s < kCS; ++s) { mbar_init(smem_u32(&code_full[s]), 1); mbar_init(smem_u32(&code_empty[s]), kWiden); }
        for (int s = 0; s < kWS; ++s) { mbar_init(smem_u32(&wide_full[s]), kWiden); mbar_init(smem_u32(&wide_empty[s]), 1); }
        for (int x = 0; x < 2; ++x) {
            mbar_init(smem_u32(&s_full[x]), 1); mbar_init(smem_u32(&p_ready[x]), kBHalf);
            mbar_init(smem_u32(&q_ready[x]), kBHalf); mbar_init(smem_u32(&o_done[x]), 1);
        }
        mbar_init(smem_u32(&drain), 1);
        mbar_init(smem_u32(&state_ready), kBHalf);
        mbar_init(smem_u32(&state_read), kBHalf);
        gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (a.chained || a.join) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    // ---- this CTA's share of the batch's units ----
    const int H = geo.n_kv_heads, n_seqs = a.rows.n_seqs;
    int *status = blockIdx.x == 0 ? a.status : nullptr;
    auto weight = [&](int s, int *st) -> long long {
        if (s >= n_seqs) return 0;
        return block_weight<kSel>(a, block_seq(a, s, st)) * H;
    };
    const bool once = kSel && n_seqs <= kBThreads;             // a sequence to a thread: one scan for the sum and the place
    long long total = 0, upto = 0, own_weight = 0;
    if (n_seqs == 1) {
        total = weight(0, tid == 0 ? status : nullptr);
    } else if (once) {
        own_weight = upto = weight(tid, status);
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += y;
        }
        if (lane == 31) sums[warp] = upto;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kBThreads / 32; ++w) {
            if (w < warp) upto += sums[w];
            total += sums[w];
        }
    } else {
        long long mine = 0;
        for (int s = tid; s < n_seqs; s += kBThreads) mine += weight(s, status);
#pragma unroll
        for (int d = 16; d; d >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, d);
        if (lane == 0) sums[warp] = mine;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kBThreads / 32; ++w) total += sums[w];
    }
    const int n_ctas = (int)min((long long)gridDim.x, max(1LL, total / (4 + kBSegCost)));
    // (b * total / n without a 64-bit division where the total has 31 bits)
    auto share = [&](long long b) -> long long {
        if (!kSel || total >> 31) return total * b / n_ctas;
        const unsigned q = (unsigned)total / (unsigned)n_ctas, r = (unsigned)total % (unsigned)n_ctas;
        return (long long)q * b + r * (unsigned)b / (unsigned)n_ctas;
    };
    const long long begin = share(blockIdx.x), end = share(blockIdx.x + 1LL);
    Q4Part *parts = reinterpret_cast<Q4Part *>(a.workspace);
    float *states = reinterpret_cast<float *>(a.workspace + q4_parts_bytes(gridDim.x));
    if (blockIdx.x >= n_ctas || begin >= end) {
        if (tid == 0 && gridDim.x > 1) parts[blockIdx.x].seq = -1;
        return;
    }
    BlockCursor seg;
    long long at0 = begin;                                     // `begin` within its sequence
    if (n_seqs == 1) {
        seg.seq = 0;
    } else if (once) {
        if (begin >= upto - own_weight && begin < upto) { found_seq = tid; found_at = begin - (upto - own_weight); }
        __syncthreads();
        seg.seq = found_seq;
        at0 = found_at;
    } else {
        long long base = 0;
        for (int s0 = 0; s0 < n_seqs; s0 += kBThreads) {
            const long long v = weight(s0 + tid, nullptr);
            long long x = v;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const long long y = __shfl_up_sync(0xffffffffu, x, d);
                if (lane >= d) x += y;
            }
            __syncthreads();
            if (lane == 31) sums[warp] = x;
            __syncthreads();
            long long before = base, all = 0;
#pragma unroll
            for (int w = 0; w < kBThreads / 32; ++w) {
                if (w < warp) before += sums[w];
                all += sums[w];
            }
            const long long lo = before + x - v;
            if (begin >= lo && begin < lo + v) { found_seq = s0 + tid; found_at = begin - lo; }
            base += all;
            if (base > begin) break;
        }
        __syncthreads();
        seg.seq = found_seq;
        at0 = found_at;
    }
    seg.q = block_seq(a, seg.seq, nullptr);
    long long seg_pos;                                         // where the current block begins, on the scale of the weights
    {
        long long b0;
        seg.block = block_locate<kSel>(a, seg.q, H, at0, b0);
        block_enter<kSel>(a, seg);
        const int len = seg.units + kBSegCost;
        seg.head = (int)((at0 - b0) / len);
        const int off = (int)(at0 - b0 - (long long)seg.head * len);
        seg.unit = min(off, seg.units);
        seg_pos = begin - off;
        if (seg.unit == seg.units) {                           // the share begins behind a block's units
            seg_pos += len;
            block_advance<kSel>(a, seg, 0);
        }
    }
    int left = 0;                                              // units of the CTA
    {
        BlockCursor w = seg;
        long long pos = seg_pos;
        while (w.seq < n_seqs && pos + w.unit < end) {
            const int here = (int)min((long long)(w.units - w.unit), end - pos - w.unit);
            left += here;
            if (here < w.units - w.unit) break;
            pos += w.units + kBSegCost;
            block_advance<kSel>(a, w, w.units - w.unit);
        }
    }
    if (left == 0) {
        if (tid == 0 && gridDim.x > 1) parts[blockIdx.x].seq = -1;
        return;
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(kBTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tm = tmem_slot;
    const long long limit = kWaitClocks;

    if (kPairs && warp >= kBIssueWarp) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kBOtherRegs));
    if (warp == kBCopyWarp) {
        // ---------------- copies: 32 units are looked up at a time, a lane each, and issued in turn ----------------
        const int per_page = min(kQ4Unit, geo.page), n_parts = kQ4Unit / per_page, per_tiles = per_page / kQ4Tile;
        BlockCursor nx = seg;
        if (lane < left) block_advance<kSel>(a, nx, lane);
        bool ok = true;
        int st = 0, use = 0, u = 0;
        for (int at = lane; u < left && ok; at += 32) {
            uint32_t bits = 0;
            int pg[4] = {-1, -1, -1, -1};
            const int t0 = block_unit_at<kSel>(nx, nx.unit) * kQ4Unit, head = nx.head, tokens = at < left ? max(0, min(kQ4Unit, nx.q.T - t0)) : 0;
            if (at < left) {
                const int tiles = (tokens + kQ4Tile - 1) / kQ4Tile;
                bits = kSel ? q4_needed(a, t0, nx.lo, tiles, n_parts, per_page, per_tiles) : (1u << tiles) - 1u;
                const uint32_t wanted = bits;
                auto want = [&](int i) { return kSel ? (wanted >> (i * per_tiles) & 1u) != 0u : i * per_tiles < tiles; };      // (a part from its first tile on)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (want(i))
                        pg[i] = __ldg(a.rows.table + (long long)nx.seq * a.rows.max_pages + ((t0 + i * per_page) >> geo.page_shift));
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (want(i) && (unsigned)pg[i] >= (unsigned)geo.n_pages) {
                        atomicAdd(a.status + 1, 1);
                        bits &= ~(((1u << per_tiles) - 1u) << (i * per_tiles));
                    }
                if (at + 32 < left) block_advance<kSel>(a, nx, 32);
            }
            for (int i = 0; i < 32 && u < left; ++i, ++u) {
                const uint32_t bar = smem_u32(&code_full[st]);
                if (use > 0 && !mbar_wait_warp(smem_u32(&code_empty[st]), (use - 1) & 1, abort_flag)) { ok = false; break; }
                if (lane == i) {
                    code_tiles[st] = bits;
                    code_tokens[st] = tokens;
                    if (bits) mbar_arrive_expect_tx(bar, __popc(bits) * S::kTile);
                    else mbar_arrive(bar);
                    const uint32_t dst = smem_u32(codes) + st * S::kCodes;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        if (k >= n_parts) break;
                        const int n = __popc(bits >> (k * per_tiles) & ((1u << per_tiles) - 1u));
                        if (n > 0)
                            bulk_g2s_keep(dst + k * per_tiles * S::kTile,
                                          a.pool + (long long)pg[k] * geo.page_bytes + (long long)head * geo.head_bytes +
                                              (((t0 + k * per_page) & (geo.page - 1)) / kQ4Tile) * S::kTile, n * S::kTile, bar);
                    }
                }
                __syncwarp();
                if (++st == kCS) { st = 0; ++use; }
            }
        }
        if (!ok && lane == 0 && !*abort_flag) { *abort_flag = 1; atomicAdd(a.status, 1); }
        // copies in flight must land before the CTA retires: wait (bounded) for the stages armed last
        for (int back = 1; back <= min(u, kCS); ++back) (void)mbar_wait(smem_u32(&code_full[(u - back) % kCS]), ((u - back) / kCS) & 1, limit);
    } else if (kPairs && warp >= kBRowWarps && warp < kBRowWarps + kWiden) {
        // ---------------- codes times scales as fp16, a side of a tile per warp (as below, where a warp sees to both) ----------------
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kBWidenRegs));
        const int c = lane & 3, i8 = lane >> 2, t_lane = (i8 >> 1) ^ (i8 & 1 ? 5 : 0), dw = (warp - kBRowWarps) % kQ4UnitTiles;
        constexpr uint32_t kNext = q4_k_chunk(D, 8, 0);
        const uint32_t d_row = smem_u32(wide) + (dw * kQ4Tile + t_lane) * 128, d_at[2] = {d_row + ((c ^ (t_lane & 7)) << 4), d_row + (((4 + c) ^ (t_lane & 7)) << 4)};
        auto widen = [&](auto side) {
            constexpr bool kV = decltype(side)::value;
            constexpr uint32_t kScales = kV ? q4_vs_base(D, NG) : q4_ks_base(D), kFar = kV ? kBValues : kBKeys;
            const uint32_t a_at = kV ? q4_v_base(D) + q4_v_chunk(D, t_lane, 2 * c) : q4_k_chunk(D, t_lane, c), b_at = q4_v_base(D) + q4_v_chunk(D, t_lane, 2 * c + 1);
            bool ok = true;
            int cs = 0, cu = 0;
            for (int u = 0; u < left; ++u) {
                const int ws = u % kWS, wu = u / kWS;
                if (!mbar_wait_warp(smem_u32(&code_full[cs]), cu & 1, abort_flag)) { ok = false; break; }
                const uint32_t bits = code_tiles[cs], tokens = code_tokens[cs];
                const int valid = (bits >> dw) & 1 ? min(max((int)tokens - dw * kQ4Tile, 0), kQ4Tile) : 0;
                const uint32_t tp = smem_u32(codes) + cs * S::kCodes + dw * S::kTile;
                uint32_t z2[(NG + 1) / 2], sc[2][(NG + 1) / 2], x0[2][kV ? (NW + 1) / 2 : NW], x1[2][(NW + 1) / 2];
                lds_scales<NG>(z2, tp + kScales + (lane & 15) * 2 * NG);
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    lds_scales<NG>(sc[half], tp + kScales + (t_lane + 8 * half) * 2 * NG);
                    if (!kV) {
                        if (NW == 4) lds128(x0[half], tp + a_at + half * kNext);
                        else lds64(x0[half], tp + a_at + half * kNext);
                    } else if (NW == 4) {
                        lds64(x0[half], tp + a_at + half * kNext);
                        lds64(x1[half], tp + b_at + half * kNext);
                    } else {
                        lds32(x0[half], tp + a_at + half * kNext);
                        lds32(x1[half], tp + b_at + half * kNext);
                    }
                }
                // (lanes l and l + 16 have the same token)
                uint32_t z = z2[0], nans[NG] = {};
                if (NG == 4) z = __vmaxu2(z, z2[(NG - 1) / 2]);
                z = max(z & 0xffffu, z >> 16);
                const bool there = (lane & 15) < valid;
                if (!there) z = 0u;
                bool plain = valid == kQ4Tile;
                if (__any_sync(0xffffffffu, z > 0x7f80u)) {
                    const bool some = z != 0u;
                    plain = false;
                    z = 0u;
#pragma unroll
                    for (int k = 0; k < NG; ++k) {
                        const uint32_t x = some ? (z2[k / 2] >> (16 * (k & 1))) & 0xffffu : 0u;
                        nans[k] = __ballot_sync(0xffffffffu, x > 0x7f80u) & 0xffffu;
                        if (x <= 0x7f80u) z = max(z, x);
                    }
                }
                const uint32_t own = z >> 7, most = __reduce_max_sync(0xffffffffu, own);
                const bool uneven = __any_sync(0xffffffffu, there && (kV ? own + kFar < most || most == 0u : z != 0u && own + kFar < most));
                const bool spread = kV && __any_sync(0xffffffffu, there && own + kBSpread < most);
                const int top = 127 + kBTop, e = min(max((int)own - top, kBLeast), 100), e1 = min(max((int)most - top, kBLeast), 100);
                float f[2];
                f[0] = f[1] = pow2(-e1);
                if (uneven)
#pragma unroll
                    for (int half = 0; half < 2; ++half) f[half] = pow2(-__shfl_sync(0xffffffffu, e, t_lane + 8 * half));
                if (wu > 0 && !mbar_wait_warp(smem_u32(&wide_empty[ws]), (wu - 1) & 1, abort_flag)) { ok = false; break; }
                UnitInfo &inf = info[ws];
                if (lane < 16 && (uneven || spread)) (kV ? inf.tv : inf.tk)[dw * kQ4Tile + lane] = kV ? (float)e : pow2(e);
                if (lane == 0) {
                    if (kV) {
                        uint32_t any = 0;
#pragma unroll
                        for (int k = 0; k < NG; ++k) {
                            any |= nans[k];
                            inf.v_nan[dw][k] = (uint16_t)nans[k];
                        }
                        inf.ev[dw] = uneven ? 0.f : (float)e1;
                        inf.ev_inv[dw] = uneven ? 0.f : pow2(-e1);
                        inf.odd[dw] = (uint8_t)((uneven ? 2 : 0) | (any ? 4 : 0) | (spread ? 8 : 0));
                    } else {
                        inf.ek[dw] = uneven ? 1.f : pow2(e1);
                        inf.odd_keys[dw] = uneven ? 1 : 0;
                        if (dw == 0) { inf.tiles = bits; inf.tokens = tokens; }
                    }
                }
                const uint32_t d0 = d_at[0] + ws * S::kWide + (kV ? S::kSide : 0), d1 = d_at[1] + ws * S::kWide + (kV ? S::kSide : 0);
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    uint32_t s2[NG];
#pragma unroll
                    for (int k = 0; k < NG; ++k) {
                        float y = (k & 1 ? bf16hi_f(sc[half][k / 2]) : bf16lo_f(sc[half][k / 2])) * f[half];
                        if (!plain) {
                            if (t_lane + 8 * half >= valid) y = 0.f;
                            if (kV && y != y) y = 0.f;
                        }
                        s2[k] = pack_f16(y, y);
                    }
#pragma unroll
                    for (int w = 0; w < NW; ++w) {
                        const uint32_t x = kV ? __byte_perm(x0[half][w / 2], x1[half][w / 2], w & 1 ? 0x7632u : 0x5410u) : x0[half][kV ? 0 : w], x8 = x >> 8, m = s2[w / WPG];
                        sts128((w & 1 ? d1 : d0) + (w >> 1) * (kQ4Unit * 128) + half * 1024, h2_mul(codes_lo(x), m), h2_mul(codes_hi(x), m),
                               h2_mul(codes_lo(x8), m), h2_mul(codes_hi(x8), m));
                    }
                }
                fence_async_smem();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(smem_u32(&wide_full[ws]));
                    mbar_arrive(smem_u32(&code_empty[cs]));
                }
                if (++cs == kCS) { cs = 0; ++cu; }
            }
            if (!ok && lane == 0 && !*abort_flag) { *abort_flag = 1; atomicAdd(a.status, 1); }
        };
        if (warp < kBRowWarps + kQ4UnitTiles) widen(std::false_type());
        else widen(std::true_type());
    } else if (!kPairs && warp >= kBRowWarps && warp < kBRowWarps + kWiden) {
        // ---------------- codes times scales as fp16: a tile of 16 tokens per warp, keys or values ----------------
        const int c = lane & 3, i8 = lane >> 2;
        const int t_lane = (i8 >> 1) ^ (i8 & 1 ? 5 : 0);       // tokens t and t ^ 5 side by side: different halves of a line of codes, different banks of a line of fp16
        bool ok = true;
        const int dw = warp - kBRowWarps;                      // tile of the unit
        const uint32_t k_at = q4_k_chunk(D, t_lane, c), va_at = q4_v_base(D) + q4_v_chunk(D, t_lane, 2 * c), vb_at = q4_v_base(D) + q4_v_chunk(D, t_lane, 2 * c + 1);
        const uint32_t s_at = (lane < 16 ? q4_ks_base(D) : q4_vs_base(D, NG)) + (lane & 15) * 2 * NG;
        constexpr uint32_t kNext = q4_k_chunk(D, 8, 0);        // tokens t + 8: the same place eight rows on, for V too
        static_assert(q4_v_chunk(D, 8, 0) == (int)kNext && q4_v_chunk(D, 13, 5) == q4_v_chunk(D, 5, 5) + (int)kNext, "the pattern repeats");
        // where this lane's 16-byte blocks of a row go: words 0, 2 and words 1, 3
        const uint32_t d_row = smem_u32(wide) + (dw * kQ4Tile + t_lane) * 128, d_at[2] = {d_row + ((c ^ (t_lane & 7)) << 4), d_row + (((4 + c) ^ (t_lane & 7)) << 4)};
        int cs = 0, cu = 0;                                    // stage of the codes and times it has been used before
        for (int u = 0; u < left; ++u) {
            const int ws = u % kWS, wu = u / kWS;
            if (!mbar_wait_warp(smem_u32(&code_full[cs]), cu & 1, abort_flag)) { ok = false; break; }
            const uint32_t bits = code_tiles[cs], tokens = code_tokens[cs];
            const int valid = (bits >> dw) & 1 ? min(max((int)tokens - dw * kQ4Tile, 0), kQ4Tile) : 0;      // tokens of this tile
            const uint32_t tp = smem_u32(codes) + cs * S::kCodes + dw * S::kTile;
            // everything is read before anything is written: nothing here waits for a store
            uint32_t z2[(NG + 1) / 2], ksc[2][(NG + 1) / 2], vsc[2][(NG + 1) / 2], kw[2][NW], va[2][(NW + 1) / 2], vb[2][(NW + 1) / 2];
            lds_scales<NG>(z2, tp + s_at);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                lds_scales<NG>(ksc[half], tp + q4_ks_base(D) + (t_lane + 8 * half) * 2 * NG);
                lds_scales<NG>(vsc[half], tp + q4_vs_base(D, NG) + (t_lane + 8 * half) * 2 * NG);
                if (NW == 4) {
                    lds128(kw[half], tp + k_at + half * kNext);
                    lds64(va[half], tp + va_at + half * kNext);
                    lds64(vb[half], tp + vb_at + half * kNext);
                } else {
                    lds64(kw[half], tp + k_at + half * kNext);
                    lds32(va[half], tp + va_at + half * kNext);
                    lds32(vb[half], tp + vb_at + half * kNext);
                }
            }
            // exponents of the largest scales (lanes 0-15: keys of token `lane`, 16-31: values): as bits, which order like the values
            uint32_t z = z2[0], nans[NG] = {};
            if (NG == 4) z = __vmaxu2(z, z2[(NG - 1) / 2]);
            z = max(z & 0xffffu, z >> 16);
            if ((lane & 15) >= valid) z = 0u;
            bool plain = valid == kQ4Tile;                     // all tokens there, all groups finite
            if (__any_sync(0xffffffffu, z > 0x7f80u)) {        // a group that is not finite: look at the others of its token
                const bool there = z != 0u;
                plain = false;
                z = 0u;
#pragma unroll
                for (int k = 0; k < NG; ++k) {
                    const uint32_t x = there ? (z2[k / 2] >> (16 * (k & 1))) & 0xffffu : 0u;
                    nans[k] = __ballot_sync(0xffffffffu, x > 0x7f80u) >> 16;
                    if (x <= 0x7f80u) z = max(z, x);
                }
            }
            // one for the tile's keys and one for its values, or for each token
            const uint32_t own = z >> 7, side = lane & 16, k_most = __reduce_max_sync(0xffffffffu, side ? 0u : own), v_most = __reduce_max_sync(0xffffffffu, side ? own : 0u);
            const bool there = (lane & 15) < valid;
            const uint32_t uneven = __ballot_sync(0xffffffffu, there && (side ? own + kBValues < v_most || v_most == 0u : z != 0u && own + kBKeys < k_most));
            const bool spread = __any_sync(0xffffffffu, there && side && own + kBSpread < v_most);
            const bool each = uneven >> side & 0xffffu;
            const int top = 127 + kBTop, e = min(max((int)own - top, kBLeast), 100);
            const int ek = min(max((int)k_most - top, kBLeast), 100), ev = min(max((int)v_most - top, kBLeast), 100);
            float fk[2], fv[2];                                // of tokens t_lane, t_lane + 8
            fk[0] = fk[1] = pow2(-ek);
            fv[0] = fv[1] = pow2(-ev);
            if (uneven)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int x = __shfl_sync(0xffffffffu, e, t_lane + 8 * half), y = __shfl_sync(0xffffffffu, e, 16 + t_lane + 8 * half);
                    if (uneven & 0xffffu) fk[half] = pow2(-x);
                    if (uneven >> 16) fv[half] = pow2(-y);
                }
            if (wu > 0 && !mbar_wait_warp(smem_u32(&wide_empty[ws]), (wu - 1) & 1, abort_flag)) { ok = false; break; }
            if (side ? spread || each : each) (side ? info[ws].tv : info[ws].tk)[dw * kQ4Tile + (lane & 15)] = side ? (float)e : pow2(e);
            if (lane == 0) {
                uint32_t any = 0;
#pragma unroll
                for (int k = 0; k < NG; ++k) {
                    any |= nans[k];
                    info[ws].v_nan[dw][k] = (uint16_t)nans[k];
                }
                info[ws].ek[dw] = uneven & 0xffffu ? 1.f : pow2(ek);
                info[ws].ev[dw] = uneven >> 16 ? 0.f : (float)ev;
                info[ws].ev_inv[dw] = uneven >> 16 ? 0.f : pow2(-ev);
                info[ws].odd[dw] = (uint8_t)((uneven & 0xffffu ? 1 : 0) | (uneven >> 16 ? 2 : 0) | (any ? 4 : 0) | (spread ? 8 : 0));
                if (dw == 0) { info[ws].tiles = bits; info[ws].tokens = tokens; }
            }
            const uint32_t d0 = d_at[0] + ws * S::kWide, d1 = d_at[1] + ws * S::kWide;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                uint32_t sk[NG], sv[NG];
#pragma unroll
                for (int k = 0; k < NG; ++k) {
                    float x = (k & 1 ? bf16hi_f(ksc[half][k / 2]) : bf16lo_f(ksc[half][k / 2])) * fk[half];
                    float y = (k & 1 ? bf16hi_f(vsc[half][k / 2]) : bf16lo_f(vsc[half][k / 2])) * fv[half];
                    if (!plain) {
                        if (t_lane + 8 * half >= valid) x = y = 0.f;
                        if (y != y) y = 0.f;                   // (a value that is not finite: told to the rows by v_nan)
                    }
                    sk[k] = pack_f16(x, x);
                    sv[k] = pack_f16(y, y);
                }
#pragma unroll
                for (int w = 0; w < NW; ++w) {                 // K: a 16-byte block of eight channels per word
                    const uint32_t x = kw[half][w], x8 = x >> 8, k = sk[w / WPG];
                    sts128((w & 1 ? d1 : d0) + (w >> 1) * (kQ4Unit * 128) + half * 1024, h2_mul(codes_lo(x), k), h2_mul(codes_hi(x), k),
                           h2_mul(codes_lo(x8), k), h2_mul(codes_hi(x8), k));
                }
#pragma unroll
                for (int w = 0; w < NW; ++w) {
                    // V: four channels of chunk 2c below four of chunk 2c + 1; a register then holds channels i and i + 4 of the
                    // eight, an order that the rows undo when they write o (kVOrder)
                    const uint32_t x = __byte_perm(va[half][w / 2], vb[half][w / 2], w & 1 ? 0x7632u : 0x5410u), x8 = x >> 8, v = sv[w / WPG];
                    sts128((w & 1 ? d1 : d0) + S::kSide + (w >> 1) * (kQ4Unit * 128) + half * 1024, h2_mul(codes_lo(x), v), h2_mul(codes_hi(x), v),
                           h2_mul(codes_lo(x8), v), h2_mul(codes_hi(x8), v));
                }
            }
            fence_async_smem();                                // the products read through the async proxy
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(smem_u32(&wide_full[ws]));
                mbar_arrive(smem_u32(&code_empty[cs]));
            }
            if (++cs == kCS) { cs = 0; ++cu; }
        }
        if (!ok && lane == 0 && !*abort_flag) { *abort_flag = 1; atomicAdd(a.status, 1); }
    } else if (warp == kBIssueWarp) {
        // ---------------- products (one lane) ----------------
        if (elect_one()) {
            const uint32_t wide_a = smem_u32(wide);
            bool ok = true;
            uint32_t ph_p[2] = {0, 0}, ph_q[2] = {0, 0};
            int u = 0;
            // s of half x [128 x 64] = Q . K^T: steps of 16 channels, four to a panel
            auto qk = [&](int x, int stage) {
                const uint64_t dk = umma_desc(wide_a + stage * S::kWide, 16, 1024, 2);
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks)
                    umma_ts(tm + S::kColS + x * kQ4Unit, tm + S::kColQ + x * (D / 2) + ks * 8, umma_desc_step(dk, (ks >> 2) * (kQ4Unit * 128) + (ks & 3) * 32),
                            umma_idesc<true>(128, kQ4Unit, 0), ks > 0);
                umma_commit(smem_u32(&s_full[x]));
            };
            // o of half x [128 x D] (+)= p . V: steps of 16 tokens
            auto pv = [&](int x, int stage, bool add) {
                const uint64_t dv = umma_desc(wide_a + stage * S::kWide + S::kSide, kQ4Unit * 128, 1024, 2);
#pragma unroll
                for (int ks = 0; ks < kQ4Unit / 16; ++ks)
                    umma_ts(tm + S::kColO + x * D, tm + S::kColS + x * kQ4Unit + ks * 8, umma_desc_step(dv, ks * 2048), umma_idesc<true>(128, D, 1), add || ks > 0);
            };
            BlockCursor c = seg;
            while (u < left && ok) {
                const int n_units = min(left - u, c.units - c.unit);
                const bool two = (long long)c.block * kBRows + kBHalf < (long long)c.q.n * c.q.G;      // the halves have rows of their own
                // the halves in turn: job k is a unit of half k & 1 (its own copy of unit k / 2, or unit k).  A half's s may
                // be overwritten once its p, which lies there, has been used.
                const int jobs = two ? 2 * n_units : n_units;
                for (int k = 0; k < jobs + 2; ++k) {
                    const int x = k & 1;
                    if (k >= 2) {
                        if (k - 2 >= jobs) break;
                        const int i = two ? (k - 2) >> 1 : k - 2, stage = (u + i) % kWS;
                        if (!mbar_wait_or(smem_u32(&p_ready[x]), ph_p[x], abort_flag)) { ok = false; break; }
                        ph_p[x] ^= 1;
                        tc_fence_after();
                        pv(x, stage, k >= 4);
                        if (!two || x == 1) umma_commit(smem_u32(&wide_empty[stage]));
                        if (k >= jobs) umma_commit(smem_u32(&o_done[x]));      // the half's last
                    }
                    if (k < jobs) {
                        const int i = two ? k >> 1 : k, stage = (u + i) % kWS;
                        if (k < 2) {
                            if (!mbar_wait_or(smem_u32(&q_ready[x]), ph_q[x], abort_flag)) { ok = false; break; }
                            ph_q[x] ^= 1;
                        }
                        if (!mbar_wait_or(smem_u32(&wide_full[stage]), ((u + i) / kWS) & 1, abort_flag)) { ok = false; break; }
                        tc_fence_after();
                        qk(x, stage);
                    }
                }
                u += n_units;
                if (u < left && ok) block_advance<kSel>(a, c, n_units);
            }
            if (!ok && !*abort_flag) { *abort_flag = 1; atomicAdd(a.status, 1); }
            // nothing of this CTA's may still be running on the tensor cores when tensor memory is given back
            umma_commit(smem_u32(&drain));
            (void)mbar_wait(smem_u32(&drain), 0, limit);
        }
    } else if (warp < kBRowWarps) {
        // ---------------- rows: one query row per thread ----------------
        if (kPairs) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kBRowRegs));
        const int x = warp >> 2, r_half = (warp & 3) * 32 + lane;
        const uint32_t t_lane = tm + ((uint32_t)((warp & 3) * 32) << 16);
        const uint32_t t_o = t_lane + S::kColO + x * D, t_s = t_lane + S::kColS + x * kQ4Unit;
        bool ok = true;
        uint32_t ph_s = 0, ph_o = 0, ph_st = 0;
        int u = 0;
        BlockCursor c = seg;
        while (u < left && ok) {
            const int n_units = min(left - u, c.units - c.unit), G = geo.group;
            const bool two = (long long)c.block * kBRows + kBHalf < (long long)c.q.n * G;
            const long long row = (long long)c.block * kBRows + (two ? x * kBHalf : 0) + r_half;
            const int j = (int)(row / G), h = c.head * G + (int)(row - (long long)j * G);
            const bool row_ok = j < c.q.n;
            const int i0 = two ? 0 : x, step = two ? 1 : 2;    // this half's units
            float F = kNegInf, l = 0.f;
            uint32_t bad = 0;                                  // channel groups in which the row sees a value that is not finite
            if (i0 < n_units) {
                // ---- Q: times a power of two that brings the row's largest magnitude to 2^14 .. 2^15; channels 2^-28 (bf16: 2^-31) of it
                // are exact in fp16 ----
                float f;
                {
                    const uint4 *qg = reinterpret_cast<const uint4 *>(reinterpret_cast<const unsigned short *>(a.q) + (long long)(c.q.first + j) * a.q_row + (long long)h * a.q_head);
                    uint4 raw[D / 8];
                    uint32_t mx = 0;
#pragma unroll
                    for (int i = 0; i < D / 8; ++i) {
                        raw[i] = row_ok ? __ldg(qg + i) : make_uint4(0u, 0u, 0u, 0u);
                        mx = __vmaxu2(mx, __vmaxu2(__vmaxu2(raw[i].x & 0x7fff7fffu, raw[i].y & 0x7fff7fffu), __vmaxu2(raw[i].z & 0x7fff7fffu, raw[i].w & 0x7fff7fffu)));
                    }
                    mx = max(mx & 0xffffu, mx >> 16);
                    const float big = H16 ? __half2float(__ushort_as_half((unsigned short)mx)) : __uint_as_float(mx << 16);
                    const int e = min(max((int)(__float_as_uint(big) >> 23) - 127, -60), 60) - 14;
                    const float up = pow2(-e);
                    f = pow2(e) * geo.scale_log2e;
#pragma unroll
                    for (int i = 0; i < D / 32; ++i) {
                        uint32_t pk[16];
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const uint32_t w[4] = {raw[4 * i + k].x, raw[4 * i + k].y, raw[4 * i + k].z, raw[4 * i + k].w};
#pragma unroll
                            for (int b = 0; b < 4; ++b) {
                                float lo, hi;
                                if (H16) {
                                    const float2 v = __half22float2(*reinterpret_cast<const __half2 *>(&w[b]));
                                    lo = v.x; hi = v.y;
                                } else {
                                    lo = bf16lo_f(w[b]); hi = bf16hi_f(w[b]);
                                }
                                pk[4 * k + b] = pack_f16(lo * up, hi * up);
                            }
                        }
                        tmem_st16(t_lane + S::kColQ + x * (D / 2) + 16 * i, pk);
                    }
                    tmem_st_wait();
                    tc_fence_before();
                    mbar_arrive(smem_u32(&q_ready[x]));
                }
                const int vis = row_ok ? c.q.T - c.q.all + j + 1 : c.q.T;
                Q4Seen part{0, c.q.T};                         // kSel: what the row sees; what all of the warp's see
                int vis_all = 0, lo_all = 0;
                if (kSel) {
                    if (row_ok) part = q4_seen(a, c.q.T, c.q.all, c.q.first, j);
                    vis_all = __reduce_min_sync(0xffffffffu, part.end);
                    lo_all = __reduce_max_sync(0xffffffffu, part.lo);
                }
                for (int i = i0; i < n_units; i += step) {
                    const int ws = (u + i) % kWS;
                    // what the unit is like, while its scores are being computed
                    if (!mbar_wait_warp(smem_u32(&wide_full[ws]), ((u + i) / kWS) & 1, abort_flag)) { ok = false; break; }
                    const UnitInfo &inf = info[ws];
                    const int t0 = block_unit_at<kSel>(c, c.unit + i) * kQ4Unit, lim = kSel ? 0 : min(vis - t0, (int)inf.tokens);
                    const uint32_t tiles = inf.tiles, odd = *reinterpret_cast<const uint32_t *>(inf.odd) | (kPairs ? *reinterpret_cast<const uint32_t *>(inf.odd_keys) : 0u);
                    const bool part_of = kSel && !(t0 + kQ4Unit <= vis_all && (t0 >= lo_all || t0 + kQ4Unit <= a.sinks));      // (the same for the warp)
                    const bool special = (kSel ? part_of || (odd & 0x07070707u) != 0u : __any_sync(0xffffffffu, lim < kQ4Unit || (odd & 0x07070707u) != 0u)) ||
                                         tiles != (1u << kQ4UnitTiles) - 1u;
                    unsigned long long mask = ~0ull;           // kSel: tokens of the unit that the row sees
                    if (kSel && special) {
                        if (part_of && row_ok) mask = q4_unit_mask(a, part, t0, c.q.T, c.q.all, c.q.first + j);
                        mask &= q4_tile_mask(tiles) & q4_below((int)inf.tokens);
                    }
                    float fk[kQ4UnitTiles], ev[kQ4UnitTiles];
#pragma unroll
                    for (int k = 0; k < kQ4UnitTiles; ++k) {
                        fk[k] = fmaxf(f * inf.ek[k], 1.2e-38f);      // (never 0: a hidden score is -inf)
                        ev[k] = inf.ev[k];
                    }
                    if (!mbar_wait_warp(smem_u32(&s_full[x]), ph_s, abort_flag)) { ok = false; break; }
                    ph_s ^= 1;
                    tc_fence_after();
                    float sv[kQ4Unit];
                    tmem_ld<kQ4Unit>(t_s, reinterpret_cast<uint32_t *>(sv));
                    float apart = 0.f, apart_m = kNegInf;      // sum of the weights of tiles with uneven values, relative to 2^apart_m
                    if (special) {
                        if (odd & 0x07070707u) {
                            // each token's powers of two, in tensor memory, a tile at a time: out of the way of the registers
#pragma unroll 1
                            for (int k = 0; k < kQ4UnitTiles; ++k) {
                                const uint32_t un = odd >> (8 * k);
                                const int see = tiles >> k & 1 ? lim : 0;
                                const uint32_t m16 = (uint32_t)(mask >> (k * kQ4Tile)) & 0xffffu;
                                auto sees = [&](int b) { return kSel ? (m16 >> b & 1u) != 0u : k * kQ4Tile + b < see; };
                                if (un & 4u) {
                                    const uint32_t seen = kSel ? m16 : (1u << min(max(see - k * kQ4Tile, 0), kQ4Tile)) - 1u;
#pragma unroll 1
                                    for (int b = 0; b < NG; ++b) bad |= (inf.v_nan[k][b] & seen) ? 1u << b : 0u;
                                }
                                if (!(un & 3u)) continue;
                                const float fx = fmaxf(f * inf.ek[k], 1.2e-38f);
                                float x[kQ4Tile];
                                tmem_ld16(t_s + k * kQ4Tile, reinterpret_cast<uint32_t *>(x));
                                tmem_ld_wait();
                                if (un & 1u) {
#pragma unroll
                                    for (int b = 0; b < kQ4Tile; b += 4) {
                                        const float4 t = *reinterpret_cast<const float4 *>(inf.tk + k * kQ4Tile + b);
                                        x[b] *= t.x; x[b + 1] *= t.y; x[b + 2] *= t.z; x[b + 3] *= t.w;
                                    }
                                }
                                if (un & 2u) {
                                    float m = apart_m, sum = 0.f;
#pragma unroll
                                    for (int b = 0; b < kQ4Tile; ++b) {
                                        x[b] *= fx;
                                        if (sees(b)) m = fmaxf(m, x[b]);
                                    }
#pragma unroll
                                    for (int b = 0; b < kQ4Tile; ++b) sum += sees(b) ? ex2(x[b] - m) : 0.f;
                                    apart = fmaf(apart, ex2(apart_m - m), sum);
                                    apart_m = m;
#pragma unroll
                                    for (int b = 0; b < kQ4Tile; b += 4) {
                                        const float4 t = *reinterpret_cast<const float4 *>(inf.tv + k * kQ4Tile + b);
                                        x[b] += t.x; x[b + 1] += t.y; x[b + 2] += t.z; x[b + 3] += t.w;
                                    }
                                }
                                tmem_st16(t_s + k * kQ4Tile, reinterpret_cast<const uint32_t *>(x));
                            }
                            tmem_st_wait();
                            tmem_ld<kQ4Unit>(t_s, reinterpret_cast<uint32_t *>(sv));
#pragma unroll
                            for (int k = 0; k < kQ4UnitTiles; ++k)
                                if (odd >> (8 * k) & 2u) fk[k] = 1.f;      // (its columns are x itself)
                        }
#pragma unroll
                        for (int k = 0; k < kQ4Unit; ++k)
                            if (!(kSel ? (mask >> k & 1ull) != 0ull : k < lim && (tiles >> (k / kQ4Tile) & 1))) sv[k] = -INFINITY;
                    }
                    // x = s * f 2^Ek + Ev, against a reference of the row's own
                    float top = -INFINITY;
#pragma unroll
                    for (int k = 0; k < kQ4UnitTiles; ++k) {
                        const float *p = sv + k * kQ4Tile;
                        float m0 = max3(p[0], p[1], p[2]), m1 = max3(p[3], p[4], p[5]);
                        m0 = max3(m0, p[6], p[7]); m1 = max3(m1, p[8], p[9]);
                        m0 = max3(m0, p[10], p[11]); m1 = max3(m1, p[12], p[13]);
                        m0 = max3(m0, p[14], p[15]);
                        top = fmaxf(top, fmaf(fmaxf(m0, m1), fk[k], ev[k]));
                    }
                    if (__any_sync(0xffffffffu, top > F + kQ4Most)) {
                        float own = top;
                        if (odd & 0x08080808u) {               // the largest x, each token with its own Ev
                            own = -INFINITY;
#pragma unroll 1
                            for (int k = 0; k < kQ4UnitTiles; ++k) {
                                const uint32_t un = odd >> (8 * k);
                                const int see = (tiles >> k & 1 ? lim : 0) - k * kQ4Tile;
                                const uint32_t m16 = (uint32_t)(mask >> (k * kQ4Tile));
                                auto sees = [&](int b) { return kSel ? (m16 >> b & 1u) != 0u : b < see; };
                                const float fx = un & 2u ? 1.f : fmaxf(f * inf.ek[k], 1.2e-38f);
                                float x[kQ4Tile];
                                tmem_ld16(t_s + k * kQ4Tile, reinterpret_cast<uint32_t *>(x));
                                tmem_ld_wait();
#pragma unroll
                                for (int b = 0; b < kQ4Tile; b += 4) {
                                    const float4 t = (un & 10u) == 8u ? *reinterpret_cast<const float4 *>(inf.tv + k * kQ4Tile + b) : make_float4(inf.ev[k], inf.ev[k], inf.ev[k], inf.ev[k]);
                                    if (sees(b)) own = fmaxf(own, fmaf(x[b], fx, t.x));
                                    if (sees(b + 1)) own = fmaxf(own, fmaf(x[b + 1], fx, t.y));
                                    if (sees(b + 2)) own = fmaxf(own, fmaf(x[b + 2], fx, t.z));
                                    if (sees(b + 3)) own = fmaxf(own, fmaf(x[b + 3], fx, t.w));
                                }
                            }
                        }
                        const float Fn = top > F + kQ4Most ? fmaxf(own - kQ4Place, top - kQ4Most) : F, corr = ex2(F - Fn);
                        F = Fn;
                        l *= corr;
                        if (i > i0) {                          // (every earlier product of this half is complete: s was committed behind it)
                            uint32_t r[32];
#pragma unroll 1
                            for (int b = 0; b < D / 32; ++b) {
                                tmem_ld32(t_o + 32 * b, r);
                                tmem_ld_wait();
#pragma unroll
                                for (int k = 0; k < 32; ++k) r[k] = __float_as_uint(__uint_as_float(r[k]) * corr);
                                tmem_st32(t_o + 32 * b, r);
                            }
                        }
                    }
                    l = fmaf(apart, ex2(apart_m - F), l);
                    uint32_t pk[kQ4Unit / 2];
#pragma unroll
                    for (int k = 0; k < kQ4UnitTiles; ++k) {
                        const uint64_t m2 = f2_pack(fk[k], fk[k]), b2 = f2_pack(ev[k] - F, ev[k] - F);
                        uint64_t sum[2] = {0ull, 0ull};
#pragma unroll
                        for (int b = 0; b < kQ4Tile / 2; ++b) {
                            const int q = k * kQ4Tile + 2 * b;
                            float y0, y1;
                            f2_unpack(f2_fma3(f2_pack(sv[q], sv[q + 1]), m2, b2), y0, y1);
                            y0 = exp2_fast(y0);
                            y1 = exp2_fast(y1);
                            sum[b & 1] = f2_add(sum[b & 1], f2_pack(y0, y1));
                            pk[q / 2] = pack_f16(y0, y1);
                        }
                        float s0, s1;
                        f2_unpack(f2_add(sum[0], sum[1]), s0, s1);
                        l = fmaf(s0 + s1, inf.ev_inv[k], l);
                    }
                    tmem_st32(t_s, pk);
                    tmem_st_wait();
                    tc_fence_before();
                    mbar_arrive(smem_u32(&p_ready[x]));
                }
                if (!ok) break;
                if (!mbar_wait_warp(smem_u32(&o_done[x]), ph_o, abort_flag)) { ok = false; break; }
                ph_o ^= 1;
                tc_fence_after();
            }
            // ---- the halves' states become one where they had the same rows: the first half writes it ----
            float f0 = 1.f, f1 = 0.f;
            if (!two) {
                if (x == 1) {
                    ml_other[r_half] = make_float2(F, l);
                    bad_other[r_half] = bad;
                    tc_fence_before();
                    mbar_arrive(smem_u32(&state_ready));
                    if (!mbar_wait_warp(smem_u32(&state_read), ph_st, abort_flag)) { ok = false; break; }
                } else {
                    if (!mbar_wait_warp(smem_u32(&state_ready), ph_st, abort_flag)) { ok = false; break; }
                    tc_fence_after();
                    if (n_units > 1) {
                        const float2 other = ml_other[r_half];
                        const float M = fmaxf(F, other.x);
                        f0 = ex2(F - M);
                        f1 = ex2(other.x - M);
                        F = M;
                        l = f0 * l + f1 * other.y;
                        bad |= bad_other[r_half];
                    }
                }
                ph_st ^= 1;
            }
            // ---- the block's result, or its state where the block goes on in another CTA ----
            if (two || x == 0) {
                const bool complete = c.unit == 0 && n_units == c.units;
                const int slot = u == 0 ? 0 : 1, r_block = (two ? x * kBHalf : 0) + r_half;
                // (a state with l from 1 to 2, so that m is near the largest score whatever the values' size)
                float inv = 1.f;
                if (complete && !a.state) {
                    inv = l != 0.f ? 1.f / l : 0.f;
                } else if (l > 0.f) {
                    const int e = min(max((int)(__float_as_uint(l) >> 23) - 127, -120), 120);
                    inv = pow2(-e);
                    l *= inv;
                    F += (float)e;
                }
                const bool merge = !two && n_units > 1;
                f0 *= inv;
                f1 *= inv;
                float *dst = nullptr;
                if (!complete) dst = states + (2LL * blockIdx.x + slot) * q4_state_floats(kBRows, D) + r_block * 4;      // (four channels of all rows, then the next four)
                else if (a.state && row_ok) dst = a.state + ((long long)(c.q.first + j) * geo.n_q_heads + h) * (D + 2);
                unsigned short *out = reinterpret_cast<unsigned short *>(a.out) + (long long)(c.q.first + j) * a.out_row + (long long)h * a.out_head;
#pragma unroll 1
                for (int b = 0; b < D / 32; ++b) {
                    uint32_t r[32];
                    tmem_ld32(t_o + 32 * b, r);
                    tmem_ld_wait();
#pragma unroll
                    for (int k = 0; k < 32; ++k) r[k] = __float_as_uint(__uint_as_float(r[k]) * f0);
                    // (channel i of eight is column kVOrder[i]: the order in which V was widened)
                    constexpr int kVOrder[8] = {0, 2, 4, 6, 1, 3, 5, 7};
                    if (merge) {
                        uint32_t r1[32];
                        tmem_ld32(t_o + D + 32 * b, r1);       // the second half's o, the same lanes
                        tmem_ld_wait();
#pragma unroll
                        for (int k = 0; k < 32; ++k) r[k] = __float_as_uint(fmaf(__uint_as_float(r1[k]), f1, __uint_as_float(r[k])));
                    }
                    if (bad >> (b / WPG) & 1)                  // (a group is 32 channels or more)
#pragma unroll
                        for (int k = 0; k < 32; ++k) r[k] = 0x7fc00000u;
                    if (!complete) {                           // (16-byte aligned, unlike a row of the caller's states; neighbours side by side)
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            *reinterpret_cast<uint4 *>(dst + (8 * b + k) * (4 * kBRows)) =
                                make_uint4(r[(4 * k & ~7) + kVOrder[4 * k & 7]], r[(4 * k & ~7) + kVOrder[(4 * k + 1) & 7]],
                                           r[(4 * k & ~7) + kVOrder[(4 * k + 2) & 7]], r[(4 * k & ~7) + kVOrder[(4 * k + 3) & 7]]);
                    } else if (dst) {
#pragma unroll
                        for (int k = 0; k < 16; ++k) *reinterpret_cast<uint2 *>(dst + 32 * b + 2 * k) = make_uint2(r[(2 * k & ~7) + kVOrder[2 * k & 7]], r[(2 * k & ~7) + kVOrder[(2 * k + 1) & 7]]);
                    } else if (row_ok) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            uint32_t w[4];
#pragma unroll
                            for (int m = 0; m < 4; ++m) {
                                const float y0 = __uint_as_float(r[8 * k + kVOrder[2 * m]]), y1 = __uint_as_float(r[8 * k + kVOrder[2 * m + 1]]);
                                w[m] = H16 ? pack_f16(y0, y1) : pack_bf16(y0, y1);
                            }
                            *reinterpret_cast<uint4 *>(out + 32 * b + 8 * k) = make_uint4(w[0], w[1], w[2], w[3]);
                        }
                    }
                }
                if (!complete) {
                    float *ml = states + (2LL * blockIdx.x + slot) * q4_state_floats(kBRows, D) + (long long)kBRows * D;
                    ml[r_block] = F;
                    ml[kBRows + r_block] = l;
                } else if (dst) {
                    *reinterpret_cast<float2 *>(dst + D) = make_float2(F, l);
                }
                tc_fence_before();                             // (o has been read when the next block's Q, which its products wait for, is handed over)
                if (!two) mbar_arrive(smem_u32(&state_read));
            }
            u += n_units;
            if (tid == 0 && gridDim.x > 1 && u == left) {
                Q4Part p{-1, 0, 0, 0, 0};
                if (c.unit == 0 && n_units < c.units) {
                    // the CTA whose share holds the block's last unit
                    p = Q4Part{c.seq, c.block, c.head, u == n_units ? 0 : 1, (int)(((seg_pos + c.units) * n_ctas - 1) / total)};
                }
                parts[blockIdx.x] = p;
            }
            seg_pos += c.units + kBSegCost;
            if (u < left) block_advance<kSel>(a, c, n_units);
        }
        if (!ok && lane == 0 && !*abort_flag) { *abort_flag = 1; atomicAdd(a.status, 1); }
        if (!ok && tid == 0 && gridDim.x > 1) parts[blockIdx.x].seq = -1;
    }
    // ---------------- every thread: give tensor memory back ----------------
    tc_fence_before();
    __syncthreads();
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tm), "r"(kBTmemCols) : "memory");
}

#define PKV_Q4_SHAPES(X) X(128, 4) X(128, 2) X(128, 1) X(64, 2) X(64, 1)

}  // namespace

cudaError_t q4_block_setup(const Q4Geometry &g) {
    cudaError_t e;
#define PKV_Q4_SETUP2(D, NG, H16, SEL, PAIRS) \
    if (g.head_dim == D && g.groups == NG && (g.fp16 != 0) == H16 && (e = cudaFuncSetAttribute(q4_block_kernel<D, NG, H16, SEL, PAIRS>, cudaFuncAttributeMaxDynamicSharedMemorySize, BlockShape<D, NG>::kSmem)) != cudaSuccess) return e;
#define PKV_Q4_SETUP1(D, NG, H16) PKV_Q4_SETUP2(D, NG, H16, false, false) PKV_Q4_SETUP2(D, NG, H16, true, false) PKV_Q4_SETUP2(D, NG, H16, true, true)
#define PKV_Q4_SETUP(D, NG) PKV_Q4_SETUP1(D, NG, false) PKV_Q4_SETUP1(D, NG, true)
    PKV_Q4_SHAPES(PKV_Q4_SETUP)
    return cudaSuccess;
}

// CTAs: one per SM, four units each at least, as far as the host can tell.
int q4_block_grid(const Q4Geometry &g, int n_seqs, int max_q_len, int max_len, const Q4Select &sel) {
    const double blocks = (double)(((long long)max_q_len * g.group + kBRows - 1) / kBRows);
    double units = (max_len + kQ4Unit - 1) / kQ4Unit;
    if (sel.window > 0 && !sel.tree) units = std::min(units, ((double)sel.window + sel.sinks + kBRows / g.group) / kQ4Unit + 2);      // (a block's window)
    const double all = (double)n_seqs * g.n_kv_heads * blocks * (units + kBSegCost) / (4 + kBSegCost);
    return all >= g.n_sms ? g.n_sms : all < 1 ? 1 : (int)all;
}

cudaError_t launch_q4_block(const Q4AttentionArgs &a, int n, cudaStream_t st) {
    const Q4Geometry &g = a.geo;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = a.chained;
    cfg.gridDim = dim3(n);
    const bool part = a.window > 0 || a.tree, pairs = part && (long long)a.max_q_len * g.group <= kBHalf;
    cfg.blockDim = dim3(block_threads(pairs));
#define PKV_Q4_LAUNCH1(D, NG, H16)                                                                       \
    if (g.head_dim == D && g.groups == NG && (g.fp16 != 0) == H16) {                                     \
        cfg.dynamicSmemBytes = BlockShape<D, NG>::kSmem;                                                 \
        return pairs  ? cudaLaunchKernelEx(&cfg, q4_block_kernel<D, NG, H16, true, true>, a)             \
               : part ? cudaLaunchKernelEx(&cfg, q4_block_kernel<D, NG, H16, true, false>, a)            \
                      : cudaLaunchKernelEx(&cfg, q4_block_kernel<D, NG, H16, false, false>, a);          \
    }
#define PKV_Q4_LAUNCH(D, NG) PKV_Q4_LAUNCH1(D, NG, false) PKV_Q4_LAUNCH1(D, NG, true)
    PKV_Q4_SHAPES(PKV_Q4_LAUNCH)
    return cudaErrorInvalidValue;
}

}  // namespace pkv
