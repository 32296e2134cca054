// Attention over the paged 4-bit cache, few query rows per KV head: decoding, speculative steps.
//
// Bound by HBM in principle - a token costs d + 4 d/g bytes per KV head and is read once, against 4 G d flop - and by the
// path from codes to operands in fact: in the time that HBM takes for a unit of 64 tokens (9216 bytes at d = 128, g = 32) the
// SMs can issue some 1600 warp instructions for it, and it takes 1200.  So the contractions go to the tensor cores, tokens as the row dimension of s = K q^T and the
// contraction dimension of o^T += V^T p, so that eight query rows (NT = 1) fill the column dimension of one m16n8k16 product:
//   K codes become fp16 operands by masking alone: code + 8 in the low bits of a 16-bit word is an fp16 subnormal,
//     (code + 8) 2^-24 exactly, and in bits 4-7 that times 16 (the queries of those channels are divided by 16).  The + 8
//     is taken away for all groups at once by one product of the scales with -8 * sum(q) (measured: a query channel 30000
//     times the others costs these nothing).  Each group's product is multiplied by its scale in fp32.
//   V codes become exact fp16 integers, two products' rows from each byte (see there; as subnormals they would lose the
//     contributions of small weights next to a large one's + 8).  The scales go to the weights: p * scale, rounded once to
//     fp16.  Where the largest of them lies in fp16's range is kept per query row and channel group, going by the tokens that the
//     row sees (see q4_follow), so values may be of any size and the sizes may differ from group to group and token to token.  It moves
//     only when something may have passed fp16's range; a unit that moves nothing costs one vote, and no product more
//     while the groups of a row share a reference.  (One reference for all rows and groups of a warp, with the largest at 1, was 5 % faster
//     at eight rows and 8 % at sixteen, and rounded small weights, and groups of smaller values, to few bits or to zero.)
//   Queries are brought to fp16 with a power of two per row, which is exact for bf16 and fp16 alike.
// Measured, 8 KV heads, d = 128, g = 32: 8 sequences of 32K (302 MB) 71 to 74 us with 4 or 8 rows per KV head (4.1 TB/s; issue slots
// 58 % busy, tensor pipe 26 %), 112 us with 16; one of 128K 41.5 us; the kernel's rate on further tokens is 5.5 to 5.8 TB/s,
// and some 15 us of a call that joins states are launches, the first copies, the last units and the join.
// Where queries see a part of the positions (kSel: a window with sinks, a drafted tree) units that nobody sees are not visited, units seen in part get
// 64 bits a row, and short segments go to small CTAs, clusters of them where there are few (kSmall).  8 sequences of 32K with a window of 4096: 17.5 us (37.9
// MB; three rounds of a unit's chain, 3.5 us each with twelve warps per SM, and 7 us of launch, share, first copies and join), 64 ragged ones
// with 1024: 27.6 us (71 MB, seven rounds, 41 % of the issue slots), 7 drafted tokens against 1500: 9.9 us.
// One warp of a CTA looks up pages and issues the bulk copies; the others take the units of 64 tokens in turn and keep (m, l, o)
// in registers; at the end of a (sequence, KV head, row tile) segment the warps' states are joined through shared memory.  The CTAs of
// a launch share the whole batch's units evenly, whatever the lengths; a segment that spans CTAs leaves its states in the
// workspace and a second kernel joins them in token order.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "pkv_q4_device.cuh"

namespace pkv {

namespace {

// What a segment costs a CTA beside its units - queries, joining the warps' states - in units: a CTA of many short segments
// takes no longer than one of few long ones (32 sequences of 512 to 16384 tokens: 47.7 -> 42.6 us; 16 rows against 8 x 32K:
// 103.5 -> 101.8 us).
__host__ __device__ constexpr int q4_seg_cost(int nt) { return nt == 1 ? 6 : 12; }
// Warps of a CTA, the last one for the copies: the kernel is bound by instruction issue and latency, so as many warps as their
// registers allow - of one column of query rows, in 128 registers a thread, two CTAs of eight per SM (one CTA of sixteen, which
// idles while it joins its warps' states: 87 us instead of 69 for 8 x 32K when this was measured); of two columns, in 168 registers, one CTA of
// twelve (two of six, with one consumer fewer and twice the segments: 115 us instead of 103).
// Where queries see a part of the positions a segment is often short: four CTAs of four warps (`small`), and clusters of them to a segment.
__host__ __device__ constexpr int q4_warps(int nt, bool small = false) { return small ? 4 : nt == 1 ? 8 : 12; }
__host__ __device__ constexpr int q4_ctas_per_sm(int nt, bool small = false) { return small ? 4 : nt == 1 ? 2 : 1; }

template <int D, int NG, int NT, bool kSmall = false>
struct Q4Shape {
    static constexpr int kWarps = q4_warps(NT, kSmall), kCons = kWarps - 1, kThreads = 32 * kWarps, kPerSM = q4_ctas_per_sm(NT, kSmall);
    // tiles per softmax step: with one column a whole unit, which leaves the scheduler most to choose from (8 x 32K: one tile 72 us,
    // two 69, four 66.7); with two columns more than one would spill (16 rows, two tiles: 105 us instead of 103)
    static constexpr int kStep = NT == 1 ? 4 : 1;
    static constexpr int kQueries = NT * (D / 32) * 512;                            // query operands, in shared memory: registers are what is short
    static constexpr int kTile = kQ4Tile * (D + 4 * NG), kUnitBytes = kQ4UnitTiles * kTile;
    static constexpr int kRowFloats = D + 4;                                        // a row of o in shared memory, padded against bank conflicts
    static constexpr int kFlush = 8 * kRowFloats * 4;                               // a warp's o (eight rows at a time) at a segment's end: over the stage it has just read
    static constexpr int kStage = ((kUnitBytes > kFlush ? kUnitBytes : kFlush) + 127) / 128 * 128;
    // the other arrays in shared memory: per warp the states' (m, l), references and gains, per stage two barriers and a word; 1 KB is the system's
    // (kSmall: and the cluster's share of the segment's state)
    static constexpr int kOther = 1024 + kCons * (64 + NT * (128 + 16 * NG)) + 32 / kPerSM * 20 + 256 + (kSmall ? 8 * D * 4 + 512 + kCons * 64 + 128 : 0);
    static constexpr int kFit = (227 * 1024 / kPerSM - kOther - kQueries) / kStage, kStages = kFit < 32 / kPerSM ? kFit : 32 / kPerSM;
    static constexpr int kSmem = kStages * kStage;
    static_assert(kStages > kCons && kPerSM * (kSmem + kQueries + kOther) <= 227 * 1024, "a stage per warp and some in flight");
};

__device__ __forceinline__ void mma_f16(float *d, const uint32_t *a, uint32_t b0, uint32_t b1, const float *c) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}
__device__ __forceinline__ void mma_bf16_k16(float *d, const uint32_t *a, uint32_t b0, uint32_t b1) {      // d = a b
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ void mma_bf16_k8(float *d, uint32_t a0, uint32_t a1, uint32_t b0) {
    asm("mma.sync.aligned.m16n8k8.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5}, {%6}, {%7, %7, %7, %7};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(b0), "f"(0.f));
}
__device__ __forceinline__ uint32_t movmatrix(uint32_t x) {
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
// two fp32 values at once
__device__ __forceinline__ uint64_t f2(float lo, float hi) {
    uint64_t v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(lo), "f"(hi));
    return v;
}
__device__ __forceinline__ void f2_split(uint64_t v, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t f2_fma(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint32_t fma_h2(uint32_t x, uint32_t y, uint32_t z) {
    uint32_t r;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(x), "r"(y), "r"(z));
    return r;
}
__device__ __forceinline__ uint64_t f2_sum(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}

// a lane's scales of rows g and g + 8: bf16, two to a word (one group: one in the low half)
template <int NG>
__device__ __forceinline__ void q4_scales(const unsigned char *p, int g, uint32_t *s0, uint32_t *s1) {
    if (NG == 4) {
        const uint2 x = *reinterpret_cast<const uint2 *>(p + g * 8), y = *reinterpret_cast<const uint2 *>(p + (g + 8) * 8);
        s0[0] = x.x; s0[(NG - 1) / 2] = x.y; s1[0] = y.x; s1[(NG - 1) / 2] = y.y;
    } else if (NG == 2) {
        s0[0] = *reinterpret_cast<const uint32_t *>(p + g * 4); s1[0] = *reinterpret_cast<const uint32_t *>(p + (g + 8) * 4);
    } else {
        s0[0] = *reinterpret_cast<const unsigned short *>(p + g * 2); s1[0] = *reinterpret_cast<const unsigned short *>(p + (g + 8) * 2);
    }
}

__device__ __forceinline__ float q4_pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
// The largest of a column of scores: the lanes of the same c.
__device__ __forceinline__ float q4_max_rows(float x) {
    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
    return fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
}

// The softmax's references of a query row (a column).  The weights are 2^(score - F) * value scale, and what brings the largest near
// 2^kQ4Place in a group of channels is
//     R = the group's largest score + log2(value scale), less kQ4Place,
// a whole number away from the largest score, so that this one's weight is a power of two times the scale and is not rounded.
// F is the largest R of the groups.  A group whose R is not far below shares it; the others get a reference A near R of their own,
// and their weights a gain of 2^(F - A), F - A whole.  Only tokens that the row sees enter, each with its own scores and scales.
// The lanes of a column share the work: a lane has group (g / 2) % NG of column 2c + g % 2.
// The largest of a column's eight lanes for each group, to the lane that has it:
template <int NG>
__device__ __forceinline__ float q4_own_max(const float (*best)[2], int lane) {
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float lo = best[(i >> 1) % NG][i & 1], hi = best[(2 + (i >> 1)) % NG][i & 1];
        v[i] = fmaxf(lane & 16 ? hi : lo, __shfl_xor_sync(0xffffffffu, lane & 16 ? lo : hi, 16));
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) v[i] = fmaxf(lane & 8 ? v[i + 2] : v[i], __shfl_xor_sync(0xffffffffu, lane & 8 ? v[i] : v[i + 2], 8));
    return fmaxf(lane & 4 ? v[1] : v[0], __shfl_xor_sync(0xffffffffu, lane & 4 ? v[0] : v[1], 4));
}
__device__ __forceinline__ float q4_max_groups(float x) {      // of a column, over the lanes of its groups
    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
    return fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
}
constexpr int kQ4Even = 2;
constexpr float kQ4Share = 2.f;        // how far below F a group's R may be for the group to share F
// Where values are tiny or zero the scores set F: p stays below 2^(kQ4Floor + 10), so that its sum is far from fp32's largest.
constexpr float kQ4Floor = 90.f;
// A of the lane, from the gains of its group (bf16, both columns)
__device__ __forceinline__ float q4_shared_ref(float F, uint32_t gains, int lane) {
    return F - (float)((int)((lane & 4 ? gains >> 23 : gains >> 7) & 0xffu) - 127);
}
// The lane's references when its column has reached `best` and `score`; corr: what o of the group is multiplied by.
struct Q4Refs { float R, A, F, gain, corr; };
__device__ __forceinline__ Q4Refs q4_follow(float best, float score, float F, float R, float A, int lane) {
    const uint32_t passed = __ballot_sync(0xffffffffu, best > A + kQ4Most || score > F + kQ4Floor + 10.f);
    Q4Refs r{R, A, F, 1.f, 1.f};
    const bool follow = (passed >> (lane & 7)) & 0x01010101u;  // some group of the column
    if (follow) r.R = fmaxf(r.R, score + (ceilf(best - score) - kQ4Place));      // (the other operand where nothing is seen: NaN)
    const float top = fmaxf(q4_max_groups(r.R), score - kQ4Floor);
    int apart = __float2int_rn(F - A);
    if (follow) {
        r.F = fmaxf(F, top);
        apart = r.R > kNegInf && r.F - r.R > kQ4Share ? min(__float2int_rn(r.F - r.R), 126) : 0;
        r.A = r.F - (float)apart;
        r.corr = ex2(A - r.A);
    }
    r.gain = q4_pow2(min(max(apart, 0), 126));
    return r;
}
// The scores up to which nothing of the lane's columns can have been passed, given the largest value scale of each group.
template <int NG>
__device__ __forceinline__ void q4_pass(float *pass, float F, float A, const uint32_t *big, int lane) {
    const int k = (lane >> 3) % NG;
    const uint32_t w = k & 2 ? big[(NG - 1) / 2] : big[0];
    float t = fminf(F + kQ4Floor + 10.f, A + kQ4Most - __log2f(k & 1 ? bf16hi_f(w) : bf16lo_f(w)));
    t = -q4_max_groups(-t);
    pass[0] = __shfl_sync(0xffffffffu, t, lane & 3);
    pass[1] = __shfl_sync(0xffffffffu, t, 4 | (lane & 3));
}

// Where a unit is: positions in the batch's order of units (sequence, row tile, head, unit of 64 tokens).
struct Q4Cursor {
    int seq, tile, head, unit;         // seq == n_seqs: past the end
    int T, tiles, units;               // of the sequence
    int su, gap, lo;                   // kSel: see Q4Span (every row tile visits what the sequence's rows see)
};
template <bool kSel>
__device__ __forceinline__ int q4_unit_at(const Q4Cursor &c, int unit) { return unit + (kSel && unit >= c.su ? c.gap : 0); }

// units of 64 tokens that a sequence's rows visit
template <bool kSel>
__device__ __forceinline__ int q4_seq_units(const Q4AttentionArgs &a, int T, int all) {
    return kSel ? q4_span(a, T, q4_lowest(a, T - all, 0)).units : max(1, (T + kQ4Unit - 1) / kQ4Unit);
}
template <bool kSel>
__device__ __forceinline__ void q4_load_seq(const Q4AttentionArgs &a, int rows_per_tile, Q4Cursor &c) {
    int first, all;
    const int n = q4_new_rows(a, c.seq, first, all, nullptr);
    c.T = q4_length(a.rows, a.geo, c.seq, nullptr);
    c.tiles = (n * a.geo.group + rows_per_tile - 1) / rows_per_tile;
    if (kSel) {
        const Q4Span r = q4_span(a, c.T, q4_lowest(a, c.T - all, 0));
        c.units = r.units; c.su = r.su; c.gap = r.gap; c.lo = r.lo;
    } else {
        c.units = max(1, (c.T + kQ4Unit - 1) / kQ4Unit);
    }
}
template <bool kSel>
__device__ __forceinline__ void q4_advance(const Q4AttentionArgs &a, int rows_per_tile, Q4Cursor &c, int by) {
    c.unit += by;
    while (c.unit >= c.units) {
        c.unit -= c.units;
        if (++c.head == a.geo.n_kv_heads) {
            c.head = 0;
            if (++c.tile == c.tiles) {
                c.tile = 0;
                do {
                    if (++c.seq >= a.rows.n_seqs) return;
                    q4_load_seq<kSel>(a, rows_per_tile, c);
                } while (c.tiles == 0);
            }
        }
    }
}

// (.aligned: the warp has to be converged, so a __syncwarp() comes before them wherever its lanes may have gone different ways)
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t cluster_at(uint32_t at, int rank) {      // the same place in another CTA's shared memory
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(at), "r"(rank));
    return r;
}
__device__ __forceinline__ void cluster_st4(uint32_t at, const float4 &v) {
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(at), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}
__device__ __forceinline__ void cluster_st2(uint32_t at, float x, float y) {
    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(at), "f"(x), "f"(y) : "memory");
}

// kSel: the queries see a part of the positions.  kSmall: whole segments only, each by one CTA or by a cluster whose CTAs take an equal run
// of its units each.  They join their states through shared memory: each CTA sees to some of the channels, the others push theirs there (read by
// those that need them instead, behind one barrier and ahead of another: 10.9 us for 7 drafted tokens against 1500).
template <int D, int NG, bool H16, int NT, bool kSel, bool kSmall = false>
__global__ void __launch_bounds__(Q4Shape<D, NG, NT, kSmall>::kThreads, q4_ctas_per_sm(NT, kSmall)) q4_decode_kernel(const __grid_constant__ Q4AttentionArgs a) {
    static_assert(!kSmall || (kSel && NT == 1), "see above");
    using S = Q4Shape<D, NG, NT, kSmall>;
    constexpr int NW = D / 32, WPG = NW / NG, R = 8 * NT;      // 32-channel words per row, words per scale, query rows
    constexpr int TS = S::kStep, kSt = S::kStages, kQ4Warps = S::kWarps, kCons = S::kCons, kQ4Threads = S::kThreads, kSegCost = q4_seg_cost(NT);
    const Q4Geometry &geo = a.geo;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ unsigned long long full[kSt], empty[kSt];
    __shared__ uint32_t tiles_here[kSt];                       // which tiles of a stage's unit are there
    __shared__ float2 ml[kCons][8];
    __shared__ float refs[kCons][NT][32];                      // R of the lane's group and column, see q4_own_max
    __shared__ uint32_t gains[kCons][NT][NG][4];               // bf16, two columns to a word
    __shared__ int vis[kSel ? 1 : 8 * NT];                     // tokens a column's query sees
    __shared__ Q4Seen part[kSel ? 8 * NT : 1];                 // kSel: which ones
    __shared__ __align__(8) uint16_t seen[kSel ? kCons : 1][8 * NT][kQ4UnitTiles];      // ... in a warp's unit, a bit each
    __shared__ __align__(16) float share_o[kSmall ? 8 * D : 1];      // kSmall: [CTA of the cluster][row][this CTA's channels], and (m, l)
    __shared__ float2 share_ml[kSmall ? 8 : 1][8];
    __shared__ uint4 queries[NT][NW][32];                      // of the segment, as the lanes of a warp take them
    __shared__ long long sums[kQ4Warps], found_at;
    __shared__ int found_seq, offs[kCons], gave_up;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;
    if (tid == 0) {
        for (int s = 0; s < kSt; ++s) { mbar_init(smem_u32(&full[s]), 1); mbar_init(smem_u32(&empty[s]), 1); }
        gave_up = 0;
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (a.chained || a.join) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    // kSmall: clusters take the place of CTAs in what follows
    const int cluster = kSmall ? a.cluster : 1, rank = kSmall ? (int)blockIdx.x % cluster : 0;
    const int block = kSmall ? (int)blockIdx.x / cluster : (int)blockIdx.x, grid = kSmall ? (int)gridDim.x / cluster : (int)gridDim.x;
    const bool a_whole = kSmall || a.whole;

    // ---- this CTA's share of the batch's units (a.whole: of its segments) ----
    const int H = geo.n_kv_heads, n_seqs = a.rows.n_seqs;
    int *status = blockIdx.x == 0 ? a.status : nullptr;
    auto weight = [&](int s, int *st) -> long long {           // units of a sequence, over its row tiles and heads
        if (s >= n_seqs) return 0;
        int first, all;
        const int n = q4_new_rows(a, s, first, all, st), T = q4_length(a.rows, geo, s, st);
        return (long long)((n * geo.group + R - 1) / R) * H * (a_whole ? 1 : q4_seq_units<kSel>(a, T, all) + kSegCost);
    };
    const bool once = kSel && n_seqs <= kQ4Threads;            // a sequence to a thread: one scan for the sum and the place
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
        for (int w = 0; w < kQ4Warps; ++w) {
            if (w < warp) upto += sums[w];
            total += sums[w];
        }
    } else {
        long long mine = 0;
        for (int s = tid; s < n_seqs; s += kQ4Threads) mine += weight(s, status);
#pragma unroll
        for (int d = 16; d; d >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, d);
        if (lane == 0) sums[warp] = mine;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kQ4Warps; ++w) total += sums[w];
    }
    // (no more CTAs than there are units for a warp of each; the launch could only estimate that)
    const int n_ctas = (int)min((long long)grid, max(1LL, a_whole ? total : total / (kCons + kSegCost)));
    // (b * total / n without a 64-bit division where the total has 31 bits and r * b below, less than n squared, 32: kSmall has up to 2 * 65535 CTAs)
    auto share = [&](long long b) -> long long {
        if (total >> 31 || n_ctas > 65536) return total * b / n_ctas;
        const unsigned q = (unsigned)total / (unsigned)n_ctas, r = (unsigned)total % (unsigned)n_ctas;
        return (long long)q * b + r * (unsigned)b / (unsigned)n_ctas;
    };
    const long long begin = share(block), end = share(block + 1LL);
    Q4Part *parts = reinterpret_cast<Q4Part *>(a.workspace);
    float *states = reinterpret_cast<float *>(a.workspace + q4_parts_bytes(gridDim.x));
    const bool joined = !a_whole && gridDim.x > 1;             // segments may span CTAs
    if (block >= n_ctas || begin >= end) {
        if (tid == 0 && joined) parts[blockIdx.x].seq = -1;
        return;
    }
    Q4Cursor seg;                                              // of the CTA: the segment being worked on, and its first unit here
    long long at0 = begin;                                     // `begin` within its sequence
    if (n_seqs == 1) {
        seg.seq = 0;
        __syncthreads();                                       // (the barriers are initialised)
    } else if (once) {
        if (begin >= upto - own_weight && begin < upto) { found_seq = tid; found_at = begin - (upto - own_weight); }
        __syncthreads();
        seg.seq = found_seq;
        at0 = found_at;
    } else {                                                   // the sequence that holds `begin`
        long long base = 0;
        for (int s0 = 0; s0 < n_seqs; s0 += kQ4Threads) {
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
            for (int w = 0; w < kQ4Warps; ++w) {
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
    q4_load_seq<kSel>(a, R, seg);
    int left_cta;                                              // units of the CTA
    long long seg_pos = 0;                                     // where the current segment begins, on the scale of the weights
    if (a_whole) {
        seg.unit = 0;
        seg.head = (int)(at0 % H);
        seg.tile = (int)(at0 / H);
        Q4Cursor w = seg;
        left_cta = w.units;
        for (int k = 1; k < (int)(end - begin); ++k) {
            q4_advance<kSel>(a, R, w, w.units);
            left_cta += w.units;
        }
        if (kSmall && cluster > 1) {                           // (its one segment: the launch gives every segment a cluster)
            seg.unit = (int)((long long)seg.units * rank / cluster);
            left_cta = (int)((long long)seg.units * (rank + 1) / cluster) - seg.unit;
            cluster_arrive();                                  // (waited for before anything is written to another CTA's shared memory: it has begun)
        }
    } else {
        const int len = seg.units + kSegCost;
        const int idx = (int)(at0 / len), off = (int)(at0 - (long long)idx * len);      // (a sequence's segments number fewer than 2^31)
        seg.head = idx % H;
        seg.tile = idx / H;
        seg.unit = min(off, seg.units);
        seg_pos = begin - off;
        if (seg.unit == seg.units) {                           // the share begins behind a segment's units
            seg_pos += len;
            q4_advance<kSel>(a, R, seg, 0);
        }
        left_cta = 0;
        Q4Cursor w = seg;
        long long pos = seg_pos;
        while (w.seq < n_seqs && pos + w.unit < end) {
            const int here = (int)min((long long)(w.units - w.unit), end - pos - w.unit);
            left_cta += here;
            if (here < w.units - w.unit) break;
            pos += w.units + kSegCost;
            q4_advance<kSel>(a, R, w, w.units - w.unit);
        }
        if (left_cta == 0) {
            if (tid == 0 && joined) parts[blockIdx.x].seq = -1;
            return;
        }
    }
    volatile int *abort_flag = &gave_up;

    if (warp == kCons) {
        // ---- copies: 32 units are looked up at a time, a lane each, and issued in turn ----
        const int per_page = min(kQ4Unit, geo.page), n_parts = kQ4Unit / per_page, per_tiles = per_page / kQ4Tile;      // copies per unit: 1, 2 or 4
        Q4Cursor nx = seg;
        if (lane < left_cta) q4_advance<kSel>(a, R, nx, lane);
        bool ok = true;
        int st = 0, use = 0, u = 0;                            // stage, times it has been used before; units issued
        for (int at = lane; u < left_cta && ok; at += 32) {
            uint32_t bits = 0;
            int pg[4] = {-1, -1, -1, -1};
            const int t0 = q4_unit_at<kSel>(nx, nx.unit) * kQ4Unit, head = nx.head;
            if (at < left_cta) {
                const int tiles = (max(0, min(kQ4Unit, nx.T - t0)) + kQ4Tile - 1) / kQ4Tile;
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
                if (at + 32 < left_cta) q4_advance<kSel>(a, R, nx, 32);
            }
            for (int i = 0; i < 32 && u < left_cta; ++i, ++u) {
                const uint32_t bar = smem_u32(&full[st]);
                if (use > 0 && !(mbar_wait_warp(smem_u32(&empty[st]), (use - 1) & 1, abort_flag))) { ok = false; break; }
                if (lane == i) {
                    tiles_here[st] = bits;
                    if (bits) mbar_arrive_expect_tx(bar, __popc(bits) * S::kTile);
                    else mbar_arrive(bar);
                    const uint32_t dst = smem_u32(smem) + st * S::kStage;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        if (k >= n_parts) break;
                        const int n = __popc(bits >> (k * per_tiles) & ((1u << per_tiles) - 1u));      // tiles of this part
                        if (n > 0)
                            bulk_g2s(dst + k * per_tiles * S::kTile,
                                     a.pool + (long long)pg[k] * geo.page_bytes + (long long)head * geo.head_bytes +
                                         (((t0 + k * per_page) & (geo.page - 1)) / kQ4Tile) * S::kTile, n * S::kTile, bar);
                    }
                }
                __syncwarp();
                if (++st == kSt) { st = 0; ++use; }
            }
        }
        if (!ok && lane == 0 && !*abort_flag) { *abort_flag = 1; atomicAdd(a.status, 1); }
        // copies in flight must land before the CTA retires: wait (bounded) for the stages armed last
        for (int back = 1; back <= min(u, kSt); ++back) (void)mbar_wait(smem_u32(&full[(u - back) % kSt]), ((u - back) / kSt) & 1);
        if (kSmall && cluster > 1) {
            __syncwarp();
            cluster_wait();
            cluster_arrive();
            cluster_wait();
        }
        return;
    }

    const int v_at[4] = {q4_v_chunk(D, 2 * c, g), q4_v_chunk(D, 2 * c + 1, g), q4_v_chunk(D, 2 * c + 8, g), q4_v_chunk(D, 2 * c + 9, g)};
    // (bar.sync asks for converged warps, and the loops before it may end with some lanes of a warp in their last round)
    auto consumers_sync = [] { __syncwarp(); asm volatile("bar.sync 1, %0;" ::"n"(32 * kCons) : "memory"); };
    int at = warp;                                             // this warp's next unit, within the CTA's units
    int seg_lo = 0;                                            // the segment's first unit, within the CTA's units
    int st = warp, phase = 0;                                  // its stage and the parity of that use
    const float scale = geo.scale_log2e;
    do {                                                       // (there is one, if without units: a cluster's CTA)
        const int seg_hi = min(left_cta, seg_lo + seg.units - seg.unit);
        // ---- the segment's queries ----
        int first, all;
        const int n = q4_new_rows(a, seg.seq, first, all, nullptr), G = geo.group;
        uint32_t bias[NT][2], big_run[(NG + 1) / 2];           // (big_run: a bound of each group's value scales so far, as they are stored)
        float F[NT][2], pass[NT][2], o[NT][2 * NW][4];         // the reference; the score up to which it cannot have been passed
        uint64_t fcol[NT], l[NT];                              // (columns 2c, 2c + 1)
        uint32_t gained = 0;                                   // bit nt: some group of a column has a reference of its own
#pragma unroll
        for (int i = 0; i < (NG + 1) / 2; ++i) big_run[i] = 0;
        int vis_all = seg.T, lo_all = 0;                       // tokens every row of the tile sees (kSel: from lo_all on)
        if (kSel) {
            const int col = lane % (8 * NT), j = (seg.tile * R + col) / G;
            const Q4Seen v = j < n ? q4_seen(a, seg.T, all, first, j) : Q4Seen{0, seg.T};
            if (warp == 0 && lane < 8 * NT) part[col] = v;
            vis_all = min(vis_all, v.end);
            lo_all = (int)__reduce_max_sync(0xffffffffu, (unsigned)v.lo);
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int row = seg.tile * R + nt * 8 + g, j = row / G, h = row - j * G;
            const bool in = j < n;
            float x[NW][8];
            float mx = 0.f;
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const uint4 raw = in ? __ldg(reinterpret_cast<const uint4 *>(
                                           reinterpret_cast<const unsigned short *>(a.q) + (long long)(first + j) * a.q_row +
                                           (long long)(seg.head * G + h) * a.q_head + 32 * w + 8 * c))
                                     : make_uint4(0u, 0u, 0u, 0u);
                const uint32_t u[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (H16) {
                        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&u[i]));
                        x[w][2 * i] = f.x; x[w][2 * i + 1] = f.y;
                    } else {
                        x[w][2 * i] = bf16lo_f(u[i]); x[w][2 * i + 1] = bf16hi_f(u[i]);
                    }
                    mx = fmaxf(mx, fmaxf(fabsf(x[w][2 * i]), fabsf(x[w][2 * i + 1])));
                }
            }
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
            // times 2^(14 - exponent of the largest): 2^14 .. 2^15, so that a sixteenth of a channel 2^-24 (bf16: 2^-27) of the
            // largest is exact too
            const int e = min(max((int)(__float_as_uint(mx) >> 23) - 127, -90), 126);
            const float up = q4_pow2(14 - e);
            uint32_t qf[NW][4];
            float sum[NG];
#pragma unroll
            for (int k = 0; k < NG; ++k) sum[k] = 0.f;
#pragma unroll
            for (int w = 0; w < NW; ++w)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float f = i & 1 ? up * 0.0625f : up;
                    qf[w][i] = pack_f16(x[w][2 * i] * f, x[w][2 * i + 1] * f);
                    const float2 r = __half22float2(*reinterpret_cast<const __half2 *>(&qf[w][i]));
                    sum[w / WPG] += (r.x + r.y) * (i & 1 ? 16.f : 1.f);
                }
            if (warp == 0)                                     // (every warp has the same: it needs its sums anyway)
#pragma unroll
                for (int w = 0; w < NW; ++w) queries[nt][w][lane] = make_uint4(qf[w][0], qf[w][1], qf[w][2], qf[w][3]);
            // -8 * sum(q) per group, to be multiplied by the tokens' scales in one product: as a column operand of three bf16
            // terms, k = group + NG * term
            const float fr = 1024.f * q4_pow2(e) * scale;      // 2^24 / up: the factor of the scores
            uint32_t term[3][NG];
#pragma unroll
            for (int k = 0; k < NG; ++k) {
                sum[k] += __shfl_xor_sync(0xffffffffu, sum[k], 1);
                sum[k] += __shfl_xor_sync(0xffffffffu, sum[k], 2);
                float left = sum[k] * (-8.f / 16777216.f);
#pragma unroll
                for (int t = 0; t < 3; ++t) {
                    term[t][k] = pack_bf16(left, 0.f);
                    left -= bf16lo_f(term[t][k]);
                }
            }
            if (NG == 4) {
                // b0: term c / 2, groups 2 (c & 1) and + 1; b1: term 2 for c < 2
                const uint32_t x0 = c & 1 ? term[0][NG / 2] | term[0][NG - 1] << 16 : term[0][0] | term[0][NG / 4] << 16;
                const uint32_t x1 = c & 1 ? term[1][NG / 2] | term[1][NG - 1] << 16 : term[1][0] | term[1][NG / 4] << 16;
                const uint32_t x2 = c & 1 ? term[2][NG / 2] | term[2][NG - 1] << 16 : term[2][0] | term[2][NG / 4] << 16;
                bias[nt][0] = c & 2 ? x1 : x0;
                bias[nt][1] = c & 2 ? 0u : x2;
            } else {
                // term c (none for c = 3), groups 0 and 1
                const uint32_t lo = c == 0 ? term[0][0] : c == 1 ? term[1][0] : c == 2 ? term[2][0] : 0u;
                const uint32_t hi = NG == 1 ? 0u : c == 0 ? term[0][NG - 1] : c == 1 ? term[1][NG - 1] : c == 2 ? term[2][NG - 1] : 0u;
                bias[nt][0] = lo | hi << 16;
                bias[nt][1] = 0u;
            }
            float fb[2];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const int col = 2 * c + b, r2 = seg.tile * R + nt * 8 + col, j2 = r2 / G;
                fb[b] = fmaxf(__shfl_sync(0xffffffffu, fr, 4 * col), 1.2e-38f);      // (never 0: a hidden score is -inf)
                if (!kSel) {
                    const int v = j2 < n ? seg.T - all + j2 + 1 : seg.T;
                    if (warp == 0 && g == 0) vis[nt * 8 + col] = v;
                    vis_all = min(vis_all, v);
                }
                F[nt][b] = pass[nt][b] = kNegInf;
            }
            refs[warp][nt][lane] = kNegInf;
#pragma unroll
            for (int k = 0; k < NG; ++k) gains[warp][nt][k][c] = 0x3f803f80u;
            fcol[nt] = f2(fb[0], fb[1]);
            l[nt] = f2(0.f, 0.f);
#pragma unroll
            for (int i = 0; i < 2 * NW; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) o[nt][i][k] = 0.f;
        }
        vis_all = __reduce_min_sync(0xffffffffu, vis_all);
        consumers_sync();                                      // (the queries are there; those before were done with at the segment's end)
        const uint32_t q_at = smem_u32(&queries[0][0][lane]);

        // ---- the segment's units ----
        const bool any = at < seg_hi;
        int st_last = 0;
        while (at < seg_hi) {
            const int t_unit = q4_unit_at<kSel>(seg, seg.unit + at - seg_lo) * kQ4Unit;
            uint32_t tiles = 0;
            if ((mbar_wait_warp(smem_u32(&full[st]), phase, abort_flag))) tiles = tiles_here[st];
            else if (lane == 0 && !*abort_flag) { *abort_flag = 1; atomicAdd(a.status, 1); }      // (the unit counts as not there)
            uint32_t need = (1u << kQ4UnitTiles) - 1u;         // kSel: tiles that some row sees a token of
            const bool whole = tiles == (1u << kQ4UnitTiles) - 1u && t_unit + kQ4Unit <= vis_all && (!kSel || t_unit >= lo_all || t_unit + kQ4Unit <= a.sinks);
            if (kSel && !whole) {                              // what each row sees of the unit, a lane each
                uint32_t lo = 0, hi = 0;                       // (rows that are not there see nothing)
                if (lane < 8 * NT) {
                    const int j = (seg.tile * R + lane) / G;
                    const unsigned long long m = j < n ? q4_unit_mask(a, part[lane], t_unit, seg.T, all, first + j) & q4_tile_mask(tiles) : 0ull;
                    lo = (uint32_t)m;
                    hi = (uint32_t)(m >> 32);
                    *reinterpret_cast<uint2 *>(&seen[warp][lane][0]) = make_uint2(lo, hi);
                }
                lo = __reduce_or_sync(0xffffffffu, lo);
                hi = __reduce_or_sync(0xffffffffu, hi);
                need = (lo & 0xffffu ? 1u : 0u) | (lo >> 16 ? 2u : 0u) | (hi & 0xffffu ? 4u : 0u) | (hi >> 16 ? 8u : 0u);
                __syncwarp();
            }
            // (not kept in registers)
            auto sees = [&](int col, int tile) -> uint32_t { return kSel ? (whole ? 0xffffu : *const_cast<const volatile uint16_t *>(&seen[warp][col][tile])) : 0u; };
            const unsigned char *sp = smem + st * S::kStage;
            // bounds of the value scales so far (lane: tokens 2 lane, 2 lane + 1)
            {
                const unsigned char *vs = sp + (lane >> 3) * S::kTile + q4_vs_base(D, NG) + (lane & 7) * 4 * NG;
                const bool tile_ok = (tiles >> (lane >> 3)) & 1;
                const bool ok0 = whole || (tile_ok && t_unit + 2 * lane < seg.T), ok1 = whole || (tile_ok && t_unit + 2 * lane + 1 < seg.T);
                uint32_t z[(NG + 1) / 2];
                if (NG == 4) {
                    const uint4 x = *reinterpret_cast<const uint4 *>(vs);
                    z[0] = max_bf16(ok0 ? x.x : 0u, ok1 ? x.z : 0u);
                    z[(NG - 1) / 2] = max_bf16(ok0 ? x.y : 0u, ok1 ? x.w : 0u);
                } else if (NG == 2) {
                    const uint2 x = *reinterpret_cast<const uint2 *>(vs);
                    z[0] = max_bf16(ok0 ? x.x : 0u, ok1 ? x.y : 0u);
                } else {
                    const uint32_t x = *reinterpret_cast<const uint32_t *>(vs);
                    z[0] = max_bf16(ok0 ? x & 0xffffu : 0u, ok1 ? x >> 16 : 0u);
                }
                bool more = false;
#pragma unroll
                for (int i = 0; i < (NG + 1) / 2; ++i) {
                    z[i] = max_bf16(z[i] | 0x001f001fu, big_run[i]);      // (two bits of the mantissa: seldom passed)
                    more |= z[i] != big_run[i];
                }
                if (__any_sync(0xffffffffu, more)) {
#pragma unroll
                    for (int i = 0; i < (NG + 1) / 2; ++i) {
#pragma unroll
                        for (int d = 1; d < 32; d <<= 1) z[i] = max_bf16(z[i], __shfl_xor_sync(0xffffffffu, z[i], d));
                        big_run[i] = z[i];
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        const float Fb = lane & 4 ? F[nt][1] : F[nt][0];
                        q4_pass<NG>(pass[nt], Fb, q4_shared_ref(Fb, gains[warp][nt][(lane >> 3) % NG][c], lane), big_run, lane);
                    }

                }
            }
            // Some tiles of the unit.  kCareful: some of the unit's tokens are hidden from some row, or not there, or groups have
            // references of their own (where that comes up on the way, the tiles are not added, and done again carefully).
            auto work = [&](int step, auto careful) -> bool {
                constexpr bool kCareful = decltype(careful)::value;
                const unsigned char *tp0 = sp + step * TS * S::kTile;
                const int t0 = t_unit + step * TS * kQ4Tile;
                const uint32_t here = tiles >> (step * TS);
                float sc[TS][NT][4];
                // ---- scores ----
#pragma unroll
                for (int tl = 0; tl < TS; ++tl) {
                    const unsigned char *tp = tp0 + tl * S::kTile;
                    if (kCareful && kSel && !(need >> (step * TS + tl) & 1u)) {
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int i = 0; i < 4; ++i) sc[tl][nt][i] = -INFINITY;
                        continue;
                    }
                    uint32_t k0[NW], k1[NW], s0[(NG + 1) / 2], s1[(NG + 1) / 2];
                    if (NW == 4) {
                        const uint4 x = *reinterpret_cast<const uint4 *>(tp + q4_k_chunk(D, g, c)), y = *reinterpret_cast<const uint4 *>(tp + q4_k_chunk(D, g + 8, c));
                        k0[0] = x.x; k0[1] = x.y; k0[NW - 2] = x.z; k0[NW - 1] = x.w;
                        k1[0] = y.x; k1[1] = y.y; k1[NW - 2] = y.z; k1[NW - 1] = y.w;
                    } else {
                        const uint2 x = *reinterpret_cast<const uint2 *>(tp + q4_k_chunk(D, g, c)), y = *reinterpret_cast<const uint2 *>(tp + q4_k_chunk(D, g + 8, c));
                        k0[0] = x.x; k0[1] = x.y; k1[0] = y.x; k1[1] = y.y;
                    }
                    q4_scales<NG>(tp + q4_ks_base(D), g, s0, s1);
                    // sum over the groups of scale * (-8 sum(q)): the scales, as stored, are the row operand
                    if (NG == 4) {
                        const unsigned char *ks = tp + q4_ks_base(D) + 4 * (c & 1);
                        const uint32_t x = *reinterpret_cast<const uint32_t *>(ks + g * 8), y = *reinterpret_cast<const uint32_t *>(ks + (g + 8) * 8);
                        const uint32_t sa[4] = {x, y, x, y};
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) mma_bf16_k16(sc[tl][nt], sa, bias[nt][0], bias[nt][1]);
                    } else {
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) mma_bf16_k8(sc[tl][nt], s0[0], s1[0], bias[nt][0]);
                    }
#pragma unroll
                    for (int k = 0; k < NG; ++k) {
                        float acc[NT][4];
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int i = 0; i < 4; ++i) acc[nt][i] = 0.f;
#pragma unroll
                        for (int w = k * WPG; w < (k + 1) * WPG; ++w) {
                            const uint32_t x0 = k0[w] >> 8, x1 = k1[w] >> 8;
                            const uint32_t fa[4] = {k0[w] & 0x000f000fu, k1[w] & 0x000f000fu, k0[w] & 0x00f000f0u, k1[w] & 0x00f000f0u};
                            const uint32_t fb[4] = {x0 & 0x000f000fu, x1 & 0x000f000fu, x0 & 0x00f000f0u, x1 & 0x00f000f0u};
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                uint32_t q[4];
                                lds128(q, q_at + (nt * NW + w) * 512);
                                mma_f16(acc[nt], fa, q[0], q[1], acc[nt]);
                                mma_f16(acc[nt], fb, q[2], q[3], acc[nt]);
                            }
                        }
                        const float f0 = k & 1 ? bf16hi_f(s0[k / 2]) : bf16lo_f(s0[k / 2]), f1 = k & 1 ? bf16hi_f(s1[k / 2]) : bf16lo_f(s1[k / 2]);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            sc[tl][nt][0] += f0 * acc[nt][0]; sc[tl][nt][1] += f0 * acc[nt][1];
                            sc[tl][nt][2] += f1 * acc[nt][2]; sc[tl][nt][3] += f1 * acc[nt][3];
                        }
                    }
                    if (kCareful)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                if (kSel) {
                                    if (!(sees(nt * 8 + 2 * c + (i & 1), step * TS + tl) >> (g + (i >> 1) * 8) & 1u)) sc[tl][nt][i] = -INFINITY;
                                } else {
                                    const int t = t0 + tl * kQ4Tile + g + (i >> 1) * 8;
                                    if (!(t < vis[nt * 8 + 2 * c + (i & 1)] && ((here >> tl) & 1))) sc[tl][nt][i] = -INFINITY;
                                }
                            }
                }
                // ---- softmax ----
                float mx[NT][2];
                bool passed = false;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    float fc[2];
                    f2_split(fcol[nt], fc[0], fc[1]);
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        float x = fmaxf(sc[0][nt][b], sc[0][nt][b + 2]);
#pragma unroll
                        for (int tl = 1; tl < TS; ++tl) x = fmaxf(x, fmaxf(sc[tl][nt][b], sc[tl][nt][b + 2]));
                        mx[nt][b] = x * fc[b];
                        passed |= mx[nt][b] > pass[nt][b];
                    }
                }
                if (__any_sync(0xffffffffu, passed)) {         // references follow where a row's own tokens have passed them
                    // value scales that differ by less than 2^kQ4Even in each group: a row's largest score and the largest scale will do
                    // for its largest sum of the two
                    bool even = true;
                    uint32_t most = 0;                         // of the lane's group
                    {
                        const unsigned char *vs = sp + (lane >> 3) * S::kTile + q4_vs_base(D, NG) + (lane & 7) * 4 * NG;
                        const bool tile_ok = (tiles >> (lane >> 3)) & 1;
                        const bool ok0 = whole || (tile_ok && t_unit + 2 * lane < seg.T), ok1 = whole || (tile_ok && t_unit + 2 * lane + 1 < seg.T);
#pragma unroll
                        for (int k = 0; k < NG; ++k) {
                            const uint32_t x = *reinterpret_cast<const unsigned short *>(vs + 2 * k), y = *reinterpret_cast<const unsigned short *>(vs + 2 * (NG + k));
                            const uint32_t hi = __reduce_max_sync(0xffffffffu, max(ok0 ? x : 0u, ok1 ? y : 0u));
                            const uint32_t lo = __reduce_min_sync(0xffffffffu, min(ok0 ? x : 0xffffu, ok1 ? y : 0xffffu));
                            even &= hi < 0x7f80u && lo >= 0x80u && hi - lo < (uint32_t)kQ4Even << 7;
                            if ((lane >> 3) % NG == k) most = hi;
                        }
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        if (NT > 1 && !__any_sync(0xffffffffu, mx[nt][0] > pass[nt][0] || mx[nt][1] > pass[nt][1])) continue;
                        const float s0 = q4_max_rows(mx[nt][0]), s1 = q4_max_rows(mx[nt][1]), sx = lane & 4 ? s1 : s0;
                        float x = sx + __log2f(__uint_as_float(most << 16));
                        if (!even) {
                            float fc[2], best[NG][2];          // the largest score + log2(value scale)
                            f2_split(fcol[nt], fc[0], fc[1]);
#pragma unroll
                            for (int k = 0; k < NG; ++k) best[k][0] = best[k][1] = -INFINITY;
#pragma unroll
                            for (int tl = 0; tl < TS; ++tl) {
                                uint32_t v0[(NG + 1) / 2], v1[(NG + 1) / 2];
                                q4_scales<NG>(tp0 + tl * S::kTile + q4_vs_base(D, NG), g, v0, v1);
#pragma unroll
                                for (int k = 0; k < NG; ++k) { // (a scale that is not a number counts as none)
                                    const float e0 = __log2f(k & 1 ? bf16hi_f(v0[k / 2]) : bf16lo_f(v0[k / 2])), e1 = __log2f(k & 1 ? bf16hi_f(v1[k / 2]) : bf16lo_f(v1[k / 2]));
#pragma unroll
                                    for (int b = 0; b < 2; ++b)
                                        best[k][b] = fmaxf(best[k][b], fmaxf(fmaf(sc[tl][nt][b], fc[b], e0), fmaf(sc[tl][nt][b + 2], fc[b], e1)));
                                }
                            }
                            x = q4_own_max<NG>(best, lane);
                        }
                        const float Fb = lane & 4 ? F[nt][1] : F[nt][0];
                        const Q4Refs r = q4_follow(x, sx, Fb, refs[warp][nt][lane], q4_shared_ref(Fb, gains[warp][nt][(lane >> 3) % NG][c], lane), lane);
                        refs[warp][nt][lane] = r.R;
                        const uint32_t both = pack_bf16(r.gain, __shfl_down_sync(0xffffffffu, r.gain, 4));
                        if (lane < 8 * NG && !(lane & 4)) gains[warp][nt][(lane >> 3) % NG][c] = both;
                        __syncwarp();
                        gained = (gained & ~(1u << nt)) | (uint32_t)__any_sync(0xffffffffu, r.gain != 1.f) << nt;
                        float lx, ly;
                        f2_split(l[nt], lx, ly);
                        const float F0 = __shfl_sync(0xffffffffu, r.F, c), F1 = __shfl_sync(0xffffffffu, r.F, 4 | c);
                        l[nt] = f2(lx * ex2(F[nt][0] - F0), ly * ex2(F[nt][1] - F1));
                        F[nt][0] = F0;
                        F[nt][1] = F1;
                        if (__any_sync(0xffffffffu, r.corr != 1.f))
#pragma unroll
                            for (int k = 0; k < NG; ++k) {
                                const float c0 = __shfl_sync(0xffffffffu, r.corr, 8 * k + c), c1 = __shfl_sync(0xffffffffu, r.corr, 8 * k + 4 + c);
#pragma unroll
                                for (int i = 2 * k * WPG; i < 2 * (k + 1) * WPG; ++i)
#pragma unroll
                                    for (int m = 0; m < 4; ++m) o[nt][i][m] *= m & 1 ? c1 : c0;
                            }
                        q4_pass<NG>(pass[nt], r.F, r.A, big_run, lane);
                    }
                    if (!kCareful && gained) return false;
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const uint64_t F2 = f2(-F[nt][0], -F[nt][1]);
#pragma unroll
                    for (int tl = 0; tl < TS; ++tl)
#pragma unroll
                        for (int i = 0; i < 4; i += 2) {
                            float x, y;
                            f2_split(f2_fma(f2(sc[tl][nt][i], sc[tl][nt][i + 1]), fcol[nt], F2), x, y);
                            sc[tl][nt][i] = ex2(x);
                            sc[tl][nt][i + 1] = ex2(y);
                            l[nt] = f2_sum(l[nt], f2(sc[tl][nt][i], sc[tl][nt][i + 1]));
                        }
                }
                // ---- o^T += V^T (p * scale) ----
#pragma unroll
                for (int tl = 0; tl < TS; ++tl) {
                    const unsigned char *tp = tp0 + tl * S::kTile, *vp = tp + q4_v_base(D);
                    if (kCareful && kSel && !(need >> (step * TS + tl) & 1u)) continue;
                    uint32_t s0[(NG + 1) / 2], s1[(NG + 1) / 2];
                    q4_scales<NG>(tp + q4_vs_base(D, NG), g, s0, s1);
                    // words of tokens 2c, 2c + 1, 2c + 8, 2c + 9: chunk g
                    uint32_t wd[4][(NW + 1) / 2];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const unsigned char *p = vp + v_at[i];
                        if (NW == 4) {
                            const uint2 x = *reinterpret_cast<const uint2 *>(p);
                            wd[i][0] = x.x; wd[i][(NW - 1) / 2] = x.y;
                        } else {
                            wd[i][0] = *reinterpret_cast<const uint32_t *>(p);
                        }
                    }
#pragma unroll
                    for (int k = 0; k < NG; ++k) {
                        const float f0 = k & 1 ? bf16hi_f(s0[k / 2]) : bf16lo_f(s0[k / 2]), f1 = k & 1 ? bf16hi_f(s1[k / 2]) : bf16lo_f(s1[k / 2]);
                        uint32_t b0[NT], b1[NT];
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            const float *p = sc[tl][nt];
                            float w0 = p[0] * f0, w1 = p[1] * f0, w2 = p[2] * f1, w3 = p[3] * f1;
                            if (kCareful) {                    // a hidden token's weight is zero whatever its scale holds
                                const uint32_t gain = *const_cast<const volatile uint32_t *>(&gains[warp][nt][k][c]);      // (not kept in registers)
                                w0 *= bf16lo_f(gain); w1 *= bf16hi_f(gain); w2 *= bf16lo_f(gain); w3 *= bf16hi_f(gain);
                                if (kSel) {
                                    const uint32_t m0 = sees(nt * 8 + 2 * c, step * TS + tl) >> g, m1 = sees(nt * 8 + 2 * c + 1, step * TS + tl) >> g;
                                    if (!(m0 & 1u)) w0 = 0.f;
                                    if (!(m1 & 1u)) w1 = 0.f;
                                    if (!(m0 & 256u)) w2 = 0.f;
                                    if (!(m1 & 256u)) w3 = 0.f;
                                } else {
                                    const int t = t0 + tl * kQ4Tile + g;
                                    const bool ok = (here >> tl) & 1;
                                    if (!(ok && t < vis[nt * 8 + 2 * c + 0])) w0 = 0.f;
                                    if (!(ok && t < vis[nt * 8 + 2 * c + 1])) w1 = 0.f;
                                    if (!(ok && t + 8 < vis[nt * 8 + 2 * c + 0])) w2 = 0.f;
                                    if (!(ok && t + 8 < vis[nt * 8 + 2 * c + 1])) w3 = 0.f;
                                }
                            }
                            b0[nt] = movmatrix(pack_f16(w0, w1));
                            b1[nt] = movmatrix(pack_f16(w2, w3));
                        }
#pragma unroll
                        for (int w = k * WPG; w < (k + 1) * WPG; ++w) {
                            const uint32_t sel = w & 1 ? 0x7632u : 0x5410u;
                            const uint32_t x = __byte_perm(wd[0][w / 2], wd[1][w / 2], sel), y = __byte_perm(wd[2][w / 2], wd[3][w / 2], sel);
                            // a byte is u0 + 16 u1 (u = code + 8, never 0); as fp16 under an exponent that makes its last bit 1:
                            // m = 1024 + u0 + 16 u1.  m - 1160 = c0 + 16 c1, and m / 16 + 1023.5 rounds to 1088 + u1 since u0 / 16 lies
                            // strictly inside (0, 1): c1 without a mask, on the pipe that has room.  Row g of the product gets
                            // c0 + 16 c1 and row g + 8 gets c1; the segment's end takes them apart.
                            uint32_t fa[4], fb[4];
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                const uint32_t v = i ? y : x, m0 = __byte_perm(v, 0x64646464u, 0x4240u), m1 = __byte_perm(v, 0x64646464u, 0x4341u);
                                fa[2 * i] = sub_h2(m0, 0x64886488u);
                                fb[2 * i] = sub_h2(m1, 0x64886488u);
                                fa[2 * i + 1] = sub_h2(fma_h2(m0, 0x2c002c00u, 0x63ff63ffu), 0x64486448u);
                                fb[2 * i + 1] = sub_h2(fma_h2(m1, 0x2c002c00u, 0x63ff63ffu), 0x64486448u);
                            }
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                mma_f16(o[nt][2 * w], fa, b0[nt], b1[nt], o[nt][2 * w]);
                                mma_f16(o[nt][2 * w + 1], fb, b0[nt], b1[nt], o[nt][2 * w + 1]);
                            }
                        }
                    }
                }
                return true;
            };
#pragma unroll 1
            for (int step = 0; step < kQ4UnitTiles / TS; ++step)
                if (!(whole && gained == 0 && work(step, std::false_type()))) work(step, std::true_type());
            at += kCons;
            st_last = st;
            st += kCons;
            if (st >= kSt) { st -= kSt; phase ^= 1; }
            __syncwarp();
            if (at < seg_hi && lane == 0) mbar_arrive(smem_u32(&empty[st_last]));      // (the segment's last stage is kept for the states)
        }

        // ---- join the warps' states ----
        float *mine = reinterpret_cast<float *>(smem + st_last * S::kStage);
        const bool starts = seg.unit == 0, ends = seg_hi - seg_lo == seg.units - seg.unit;
        const bool complete = starts && ends;
        const int slot = seg_lo == 0 ? 0 : 1;
        if (lane == 0) offs[warp] = any ? st_last * S::kStage : -1;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                float lx, ly;
                f2_split(l[nt], lx, ly);
                float v = b ? ly : lx;
                v += __shfl_xor_sync(0xffffffffu, v, 4);
                v += __shfl_xor_sync(0xffffffffu, v, 8);
                v += __shfl_xor_sync(0xffffffffu, v, 16);
                // as a state whose l is from 1 to 2, so that m is near the largest score whatever the values' size
                const int e = v > 0.f ? min(max((int)(__float_as_uint(v) >> 23) - 127, -120), 120) : 0;
                if (g == 0) ml[warp][2 * c + b] = any ? make_float2(F[nt][b] + (float)e, v * q4_pow2(-e)) : make_float2(kNegInf, 0.f);
                if (any)
#pragma unroll
                    for (int w = 0; w < NW; ++w) {
                        const float *x = o[nt][2 * w], *y = o[nt][2 * w + 1];
                        // (a gain is a power of two from 1 to 2^126: its inverse)
                        const uint32_t gain = gains[warp][nt][w / WPG][c];
                        const float f = __uint_as_float((254u << 23) - __float_as_uint(b ? bf16hi_f(gain) : bf16lo_f(gain)));
                        const float fe = q4_pow2(-e);
                        *reinterpret_cast<float4 *>(mine + (2 * c + b) * S::kRowFloats + 32 * w + 4 * g) =
                            make_float4(fmaf(-16.f, x[2 + b], x[b]) * f * fe, x[2 + b] * f * fe, fmaf(-16.f, y[2 + b], y[b]) * f * fe, y[2 + b] * f * fe);
                    }
            }
            consumers_sync();
            float *part = states + (2LL * blockIdx.x + slot) * q4_state_floats(R, D);
            // row r's state (M, L, acc at channels ch ..) to where it goes
            auto write = [&](int r, int ch, float M, float L, const float4 &acc) {
                const int row = seg.tile * R + r, j = row / G;
                if (j >= n) return;
                const int h = seg.head * G + row - j * G;
                if (a.state) {
                    float *dst = a.state + ((long long)(first + j) * geo.n_q_heads + h) * (D + 2);
                    *reinterpret_cast<float2 *>(dst + ch) = make_float2(acc.x, acc.y);
                    *reinterpret_cast<float2 *>(dst + ch + 2) = make_float2(acc.z, acc.w);
                    if (ch == 0) *reinterpret_cast<float2 *>(dst + D) = make_float2(M, L);
                } else {
                    const float inv = L != 0.f ? 1.f / L : 0.f;
                    const uint2 v = H16 ? make_uint2(pack_f16(acc.x * inv, acc.y * inv), pack_f16(acc.z * inv, acc.w * inv))
                                        : make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
                    *reinterpret_cast<uint2 *>(reinterpret_cast<unsigned short *>(a.out) + (long long)(first + j) * a.out_row +
                                               (long long)h * a.out_head + ch) = v;
                }
            };
            if (kSmall && cluster > 1) cluster_wait();
            const int rows_here = kSmall ? min(8, n * G - seg.tile * R) : 8;
            for (int i = tid; i < rows_here * (D / 4); i += 32 * kCons) {
                const int r8 = i / (D / 4), r = nt * 8 + r8, ch = i % (D / 4) * 4;
                float M = kNegInf;
#pragma unroll
                for (int w = 0; w < kCons; ++w) M = fmaxf(M, ml[w][r8].x);
                float L = 0.f;
                float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < kCons; ++w) {
                    const int off = offs[w];
                    if (off < 0) continue;
                    const float f = ex2(ml[w][r8].x - M);
                    const float4 x = *reinterpret_cast<const float4 *>(smem + off + (r8 * S::kRowFloats + ch) * 4);
                    L += f * ml[w][r8].y;
                    acc.x += f * x.x; acc.y += f * x.y; acc.z += f * x.z; acc.w += f * x.w;
                }
                if (kSmall && cluster > 1) {
                    const int own = D / cluster, to = ch / own, in = ch - to * own;
                    cluster_st4(cluster_at(smem_u32(share_o + (rank * 8 + r) * own + in), to), acc);
                    if (in == 0) cluster_st2(cluster_at(smem_u32(&share_ml[rank][r]), to), M, L);
                    continue;
                }
                if (!complete) {
                    *reinterpret_cast<float4 *>(part + r * D + ch) = acc;
                    if (ch == 0) { part[R * D + r] = M; part[R * D + R + r] = L; }
                    continue;
                }
                write(r, ch, M, L, acc);
            }
            if (kSmall && cluster > 1) {                       // this CTA's channels of all parts, in order
                __syncwarp();                                  // (rows_here * D / 4 states need not fill the last round's warps)
                cluster_arrive();
                cluster_wait();
                const int own = D / cluster;
                for (int i = tid; i < rows_here * (own / 4); i += 32 * kCons) {
                    const int r = i / (own / 4), in = i % (own / 4) * 4;
                    float M = kNegInf, L = 0.f;
                    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
                    for (int k = 0; k < cluster; ++k) M = fmaxf(M, share_ml[k][r].x);
                    for (int k = 0; k < cluster; ++k) {
                        const float f = ex2(share_ml[k][r].x - M);
                        const float4 x = *reinterpret_cast<const float4 *>(share_o + (k * 8 + r) * own + in);
                        L += f * share_ml[k][r].y;
                        acc.x += f * x.x; acc.y += f * x.y; acc.z += f * x.z; acc.w += f * x.w;
                    }
                    write(r, rank * own + in, M, L, acc);
                }
            }
            if (nt == NT - 1) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // the stages go back to the copies
            consumers_sync();
        }
        if (tid == 0 && joined && seg_hi == left_cta) {
            // the CTA's last segment: does it begin here and go on elsewhere?
            Q4Part p{-1, 0, 0, 0, 0};
            if (starts && !ends) {
                // the CTA whose share holds the last unit
                p = Q4Part{seg.seq, seg.tile, seg.head, slot, (int)(((seg_pos + seg.units) * n_ctas - 1) / total)};
            }
            parts[blockIdx.x] = p;
        }
        if (any && lane == 0) mbar_arrive(smem_u32(&empty[st_last]));
        seg_lo = seg_hi;
        if (seg_lo < left_cta) {
            seg_pos += seg.units + kSegCost;
            q4_advance<kSel>(a, R, seg, seg.units - seg.unit);
        }
    } while (seg_lo < left_cta);
}

// Joins the states of the segments (tiles of R rows) that span CTAs, in token order: blocks (b, y) take the rows of the
// segment that begins in CTA b.  A chain of loads over the parts would cost a trip to L2 each (37 parts of a 128K sequence:
// 41 us), so the parts of a row are shared by four warps (kRows = 1); of a row block's rows, many of few parts, a warp takes
// four at once, eight lanes each (a warp per row: 13 us instead of 7 for 148 parts of 256 rows).
constexpr int kQ4JoinWarps = 4;
template <int D, bool H16, int kRows>
__global__ void __launch_bounds__(32 * kQ4JoinWarps) q4_join_kernel(const __grid_constant__ Q4AttentionArgs a, int R) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (a.chained) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const Q4Geometry &geo = a.geo;
    const int b = blockIdx.x;
    const Q4Part p = reinterpret_cast<const Q4Part *>(a.workspace)[b];
    if (p.seq < 0) return;
    constexpr int W = kRows == 1 ? kQ4JoinWarps : 1;           // warps that share a row
    constexpr int LR = 32 / kRows, C = D / LR;                 // lanes and channels per lane of a row, the latter in groups of four (two)
    constexpr int V = C < 4 ? C : 4, NV = C / V;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, l = lane % LR;
    const int r = kRows == 1 ? (int)blockIdx.y : ((int)blockIdx.y * kQ4JoinWarps + warp) * kRows + lane / LR;
    int first, all;
    const int n = q4_new_rows(a, p.seq, first, all, nullptr), G = geo.group;
    const long long row = (long long)p.tile * R + r;
    const int j = (int)(row / G);
    if (W > 1 && j >= n) return;                               // (the same for the whole CTA)
    const bool in = j < n;
    const float *states = reinterpret_cast<const float *>(a.workspace + q4_parts_bytes(gridDim.x));
    const long long per = q4_state_floats(R, D);
    // the first part is in slot p.slot of CTA b, the others in slot 0 of the CTAs behind it
    auto state = [&](int k) { return states + (2LL * k + (k == b ? p.slot : 0)) * per; };
    // the parts in one pass, some at a time: the weights are not waited for before o is asked for
    constexpr int kAhead = kRows == 1 ? 4 : 2;
    float M = kNegInf, L = 0.f, acc[C];
#pragma unroll
    for (int i = 0; i < C; ++i) acc[i] = 0.f;
    for (int k0 = b + (W == 1 ? 0 : warp); k0 <= p.last_cta; k0 += W * kAhead) {
        float m[kAhead], s1[kAhead], x[kAhead][C], top = M;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int k = k0 + i * W;
            m[i] = kNegInf;
            s1[i] = 0.f;
#pragma unroll
            for (int c = 0; c < C; ++c) x[i][c] = 0.f;
            if (in && k <= p.last_cta) {
                const float *s = state(k);
                m[i] = s[R * D + r];
                s1[i] = s[R * D + R + r];
#pragma unroll
                for (int c = 0; c < NV; ++c) {
                    // (row after row; of a row block, four channels of all rows, then the next four: how the row threads store it side by side)
                    const float *src = kRows == 1 ? s + r * D + (c * LR + l) * V : s + ((c * LR + l) * V / 4 * R + r) * 4 + (c * LR + l) * V % 4;
                    if (V == 4) { const float4 v = *reinterpret_cast<const float4 *>(src); x[i][4 * c] = v.x; x[i][4 * c + 1] = v.y; x[i][4 * c + V - 2] = v.z; x[i][4 * c + V - 1] = v.w; }
                    else { const float2 v = *reinterpret_cast<const float2 *>(src); x[i][2 * c] = v.x; x[i][2 * c + 1] = v.y; }
                }
            }
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) top = fmaxf(top, m[i]);
        const float f = ex2(M - top);
        M = top;
        L *= f;
#pragma unroll
        for (int c = 0; c < C; ++c) acc[c] *= f;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const float w = ex2(m[i] - M);
            L += w * s1[i];
#pragma unroll
            for (int c = 0; c < C; ++c) acc[c] += w * x[i][c];
        }
    }
    if (W > 1) {
        __shared__ float part[kQ4JoinWarps][D + 2];
#pragma unroll
        for (int i = 0; i < C; ++i) part[warp][C * lane + i] = acc[i];
        if (lane == 0) { part[warp][D] = L; part[warp][D + 1] = M; }
        __syncthreads();
        if (warp > 0) return;
#pragma unroll
        for (int w = 0; w < W; ++w) M = fmaxf(M, part[w][D + 1]);
        L = 0.f;
#pragma unroll
        for (int i = 0; i < C; ++i) acc[i] = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float f = ex2(part[w][D + 1] - M);
#pragma unroll
            for (int i = 0; i < C; ++i) acc[i] += f * part[w][C * lane + i];
            L += f * part[w][D];
        }
    }
    if (!in) return;
    const int h = p.head * G + (int)(row - (long long)j * G);
    if (a.state) {
        float *dst = a.state + ((long long)(first + j) * geo.n_q_heads + h) * (D + 2);
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int i = 0; i < V; i += 2) *reinterpret_cast<float2 *>(dst + (c * LR + l) * V + i) = make_float2(acc[V * c + i], acc[V * c + i + 1]);
        if (l == 0) *reinterpret_cast<float2 *>(dst + D) = make_float2(M, L);
    } else {
        const float inv = L != 0.f ? 1.f / L : 0.f;
        unsigned short *dst = reinterpret_cast<unsigned short *>(a.out) + (long long)(first + j) * a.out_row + (long long)h * a.out_head;
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int i = 0; i < V; i += 2)
                *reinterpret_cast<uint32_t *>(dst + (c * LR + l) * V + i) =
                    H16 ? pack_f16(acc[V * c + i] * inv, acc[V * c + i + 1] * inv) : pack_bf16(acc[V * c + i] * inv, acc[V * c + i + 1] * inv);
    }
}

int q4_rows_per_tile(const Q4Geometry &g, int max_q_len) { return (long long)max_q_len * g.group <= 8 ? 8 : 16; }

// Sequences of up to 24 units (1536 tokens), as far as the host can tell: a segment stays in one CTA (at most four rounds of
// its warps, 1.7 us each), which saves the second kernel (4 us).
bool q4_whole(int max_len) { return (max_len + kQ4Unit - 1) / kQ4Unit <= 24; }

// Segments of the column kernel, as far as the host can tell.
double q4_segments(const Q4Geometry &g, int n_seqs, int max_q_len) {
    const int R = q4_rows_per_tile(g, max_q_len);
    return (double)n_seqs * g.n_kv_heads * (((long long)max_q_len * g.group + R - 1) / R);
}

// Many query rows per KV head go to the row-block kernel (pkv_q4_block.cu).  The column kernel reads a sequence once per sixteen
// rows, the row-block kernel once per 256 but with a long chain of steps per unit: 8 sequences of 32K, 8 KV heads, column
// against block, 16 rows 102 and 238 us, 24 and 32 rows 189 and 239, 48 rows 278 and 240; one of 128K, 32 rows 99 and 131.  Where
// short sequences leave an SM no more than one segment, a segment's length is all that counts (four of 1000, 64 rows: 18
// and 28 us; one of 1500, 256 rows: 20 and 35); with more, the blocks again (four of 1000, 148 rows: 45 and 36 us).
bool q4_by_blocks(const Q4Geometry &g, int n_seqs, int max_q_len, int max_len) {
    return (long long)max_q_len * g.group > 32 && !(q4_whole(max_len) && q4_segments(g, n_seqs, max_q_len) <= g.n_ctas / 2);
}

// CTAs of a launch: enough units for every warp of each, as far as the host can tell.
int q4_grid(const Q4Geometry &g, int n_seqs, int max_q_len, int max_len, bool whole) {
    const int nt = q4_rows_per_tile(g, max_q_len) / 8, most = max(1, g.n_ctas * q4_ctas_per_sm(nt) / 2);
    const double segs = q4_segments(g, n_seqs, max_q_len), units = (max_len + kQ4Unit - 1) / kQ4Unit;
    const double all = whole ? segs : segs * units / (q4_warps(nt) - 1);
    return all >= most ? most : all < 1 ? 1 : (int)all;
}

#define PKV_Q4_SHAPES(X) X(128, 4) X(128, 2) X(128, 1) X(64, 2) X(64, 1)

}  // namespace

cudaError_t q4_attention_setup(const Q4Geometry &g) {
    cudaError_t e = q4_block_setup(g);
    if (e != cudaSuccess) return e;
    cudaFuncAttributes known;              // (asking for them loads a kernel: not on its first call, which may be captured)
#define PKV_Q4_LOAD(D, H16) \
    if (g.head_dim == D && (g.fp16 != 0) == H16 && ((e = cudaFuncGetAttributes(&known, q4_join_kernel<D, H16, 1>)) != cudaSuccess || \
                                                    (e = cudaFuncGetAttributes(&known, q4_join_kernel<D, H16, 4>)) != cudaSuccess)) return e;
    PKV_Q4_LOAD(128, false) PKV_Q4_LOAD(128, true) PKV_Q4_LOAD(64, false) PKV_Q4_LOAD(64, true)
#define PKV_Q4_OWN(D, NG, H16) g.head_dim == D && g.groups == NG && (g.fp16 != 0) == H16
#define PKV_Q4_SETUP2(D, NG, H16, NT, SEL) \
    if (PKV_Q4_OWN(D, NG, H16) && (e = cudaFuncSetAttribute(q4_decode_kernel<D, NG, H16, NT, SEL>, cudaFuncAttributeMaxDynamicSharedMemorySize, Q4Shape<D, NG, NT>::kSmem)) != cudaSuccess) return e;
#define PKV_Q4_SETUP1(D, NG, H16, NT) PKV_Q4_SETUP2(D, NG, H16, NT, false) PKV_Q4_SETUP2(D, NG, H16, NT, true)
#define PKV_Q4_SETUP3(D, NG, H16) \
    if (PKV_Q4_OWN(D, NG, H16) && (e = cudaFuncSetAttribute(q4_decode_kernel<D, NG, H16, 1, true, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, Q4Shape<D, NG, 1, true>::kSmem)) != cudaSuccess) return e;
#define PKV_Q4_SETUP(D, NG) PKV_Q4_SETUP3(D, NG, false) PKV_Q4_SETUP3(D, NG, true) PKV_Q4_SETUP1(D, NG, false, 1) PKV_Q4_SETUP1(D, NG, false, 2) PKV_Q4_SETUP1(D, NG, true, 1) PKV_Q4_SETUP1(D, NG, true, 2)
    PKV_Q4_SHAPES(PKV_Q4_SETUP)
    return cudaSuccess;
}

// Tokens that a call's rows visit of a sequence at most, as far as the host can tell: what steers the launch where the queries see a part.
int q4_visited(int max_q_len, int max_len, const Q4Select &sel) {
    const long long most = (long long)sel.window + max_q_len + sel.sinks + 2 * kQ4Unit - 2;      // (units are cut at both ends)
    return sel.window > 0 && most < max_len ? (int)most : max_len;
}

// How a call is launched: which kernel, on how many CTAs, with how many rows to a tile.
struct Q4Route { int blocks, small, whole, cluster, n, R; };

Q4Route q4_route(const Q4Geometry &g, int n_seqs, int max_q_len, int max_len, const Q4Select &sel) {
    Q4Route r{};
    r.cluster = 1;
    const bool part = sel.window > 0 || sel.tree;
    if (part) max_len = q4_visited(max_q_len, max_len, sel);
    const double units = (max_len + kQ4Unit - 1) / kQ4Unit, rows = (double)max_q_len * g.group, heads = (double)n_seqs * g.n_kv_heads;
    r.blocks = q4_by_blocks(g, n_seqs, max_q_len, max_len);
    if (part) {
        // Estimates in us, fitted to 44 shapes (1 to 128 sequences, 1 to 64 new rows, windows of 256 to 16384 and whole contexts up to 64K, d = 128; the
        // choice is within 3 % of the best of the three in all but one, 13 %.  At d = 64 the small CTAs' rounds and the even shares take some 60 to 70 % of this, which only the
        // row blocks' term allows for: 32 of 39 shapes within 1 %, one 8, six 13 to 34 % too early away from the small CTAs):
        // small CTAs: rounds of a unit's chain, 1.5 us alone and 3.7 with all warps busy (one request, window of 4096: 13.5 against 17.0 us on the
        // column kernel's even shares; 64 requests, 1024: 31 against 62; 32 requests, 8192: 86.0 against 84.6; one, 16384: 25.6 against 19.2)
        const double segs = heads * std::ceil(rows / 8), slots = 2. * g.n_ctas;
        int c = 1;
        while (c < 8 && segs * 2 * c <= slots && 3 * c < units) c *= 2;
        const double waves = std::ceil(segs * c / slots), busy = std::min(1., segs * c / slots);
        const double small = 8 + waves * std::ceil(units / (3 * c)) * (1.5 + 2.2 * busy) + 4 * (waves - 1);
        // even shares: units, what a segment costs beside them, two launches (8 rows / 16 rows to a tile)
        const double tiles = heads * std::ceil(rows / 16), blocks = heads * std::ceil(rows / kQ4BlockRows), share = 296. / g.n_ctas;
        const double split = rows <= 8 ? std::max(17 + segs * units * 1.3e-3 * share, 10 + segs * (units + 31) * 2.05e-3 * share)
                                       : std::max(24.5, 17.6 + tiles * (units + 15) * 2.95e-3 * share);
        // row blocks (8 requests, 64 rows x 4 heads against 32K: 355 us and 1540 by even shares; 16 rows x 4 heads against 16K: 140 us and about 230)
        const double per = (g.head_dim == 128 ? 1. : 0.7) * (rows <= 128 ? 1.06 : 1.49);
        const double by_blocks = (rows <= 128 ? 20 : g.head_dim == 128 ? 33 : 25) + blocks * (units + 4) * per / g.n_sms;
        r.small = small <= split && small <= by_blocks;
        r.blocks = !r.small && by_blocks < split;
        if (r.small) {
            r.whole = 1;
            r.cluster = c;
            r.R = 8;
            r.n = c * (int)std::min(segs, std::floor(slots / c));
            return r;
        }
    }
    r.R = r.blocks ? kQ4BlockRows : q4_rows_per_tile(g, max_q_len);
    r.whole = !part && !r.blocks && q4_whole(max_len);
    r.n = r.blocks ? q4_block_grid(g, n_seqs, max_q_len, max_len, sel) : q4_grid(g, n_seqs, max_q_len, max_len, r.whole);
    return r;
}

long long q4_attention_workspace(const Q4Geometry &g, int n_seqs, int max_q_len, int max_len, const Q4Select &sel) {
    const Q4Route r = q4_route(g, n_seqs, max_q_len, max_len, sel);
    return r.n <= 1 || r.whole ? 0 : q4_parts_bytes(r.n) + 2LL * r.n * q4_state_floats(r.R, g.head_dim) * 4;
}

void q4_attention_route(const Q4Geometry &g, int n_seqs, int max_q_len, int max_len, const Q4Select &sel, int *kernel, int *n_ctas, int *cluster) {
    const Q4Route r = q4_route(g, n_seqs, max_q_len, max_len, sel);
    *kernel = r.small ? 2 : r.blocks ? 1 : 0;
    *n_ctas = r.n;
    *cluster = r.cluster;
}

cudaError_t launch_q4_attention(Q4AttentionArgs a, cudaStream_t st) {
    const Q4Geometry &g = a.geo;
    const bool part = a.window > 0 || a.tree;
    const Q4Route r = q4_route(g, a.rows.n_seqs, a.max_q_len, a.max_len, Q4Select{a.window, a.sinks, a.tree != nullptr});
    const int n = r.n, R = r.R;
    a.whole = r.whole;
    a.cluster = r.cluster;
    a.chained = q4_chained();
    a.join = n > 1 && !a.whole;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = r.cluster;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = a.chained;
    cudaError_t e = cudaErrorInvalidValue;
#define PKV_Q4_LAUNCH1(D, NG, H, NT)                                        \
    if ((g.fp16 != 0) == H && R == 8 * NT && !r.small) {                    \
        cfg.gridDim = dim3(n);                                              \
        cfg.blockDim = dim3(Q4Shape<D, NG, NT>::kThreads);                  \
        cfg.dynamicSmemBytes = Q4Shape<D, NG, NT>::kSmem;                   \
        e = part ? cudaLaunchKernelEx(&cfg, q4_decode_kernel<D, NG, H, NT, true>, a) : cudaLaunchKernelEx(&cfg, q4_decode_kernel<D, NG, H, NT, false>, a); \
    }
#define PKV_Q4_LAUNCH2(D, NG, H)                                            \
    if ((g.fp16 != 0) == H && r.small) {                                    \
        cfg.gridDim = dim3(n);                                              \
        cfg.blockDim = dim3(Q4Shape<D, NG, 1, true>::kThreads);             \
        cfg.dynamicSmemBytes = Q4Shape<D, NG, 1, true>::kSmem;              \
        cfg.attrs = a.chained ? at : at + 1;                                \
        cfg.numAttrs = a.chained + 1;                                       \
        e = cudaLaunchKernelEx(&cfg, q4_decode_kernel<D, NG, H, 1, true, true>, a); \
    }
#define PKV_Q4_LAUNCH(D, NG)                                                                     \
    if (g.head_dim == D && g.groups == NG) {                                                     \
        PKV_Q4_LAUNCH2(D, NG, false) PKV_Q4_LAUNCH2(D, NG, true)                                 \
        PKV_Q4_LAUNCH1(D, NG, false, 1) PKV_Q4_LAUNCH1(D, NG, false, 2)                          \
        PKV_Q4_LAUNCH1(D, NG, true, 1) PKV_Q4_LAUNCH1(D, NG, true, 2)                            \
    }
    if (r.blocks) {
        e = launch_q4_block(a, n, st);
    } else {
        PKV_Q4_SHAPES(PKV_Q4_LAUNCH)
    }
    if (e != cudaSuccess || !a.join) return e;
    cfg.numAttrs = 1;
    cfg.gridDim = dim3(n, r.blocks ? R / (4 * kQ4JoinWarps) : R);
    cfg.blockDim = dim3(32 * kQ4JoinWarps);
    cfg.dynamicSmemBytes = 0;
#define PKV_Q4_JOIN(D, H)                                                                                         \
    if (g.head_dim == D && (g.fp16 != 0) == H)                                                                    \
        return r.blocks ? cudaLaunchKernelEx(&cfg, q4_join_kernel<D, H, 4>, a, R) : cudaLaunchKernelEx(&cfg, q4_join_kernel<D, H, 1>, a, R);
    PKV_Q4_JOIN(128, false) PKV_Q4_JOIN(128, true) PKV_Q4_JOIN(64, false) PKV_Q4_JOIN(64, true)
    return cudaErrorInvalidValue;
}

}  // namespace pkv
