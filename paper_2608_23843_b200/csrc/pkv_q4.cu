// Paged cache that holds keys and values in 4 bits: C ABI, and the kernels that quantise rows into the cache and read
// them back.  The attention over it is in pkv_q4_attention.cu.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <new>

#include "pkv_q4.h"

using namespace pkv;

namespace {

// ---- kernels -------------------------------------------------------------------------------------------------------
// Both copy kernels are bound by HBM: 4 d bytes of 16-bit rows and d + 4 d/g bytes of cache per token and KV head.  A CTA
// takes a few rows of the call: it looks up where they lie once, a thread each, while the first 16-byte loads are in flight
// (K and V of a row and head together), so that nothing but the loads, the arithmetic and the stores is paid per
// head.  Measured, 8 heads, d = 128, g = 32, bf16: append of 65536 rows 65 us (5.3 TB/s), read of 131072 rows 120 us
// (5.7 TB/s); both have issue slots 65 % and the integer pipe 58 % busy, next to a copy's 6.45 TB/s.
constexpr int kCopyThreads = 256, kCopyUnroll = 4, kCopyRows = 128;

struct RowPlace { long long off; int t, ok; };      // byte offset of the head-0 tile in the pool; token within its tile

// Where row i of a call lies: its sequence, its position, the page that holds it.
__device__ __forceinline__ RowPlace place_of(const Q4Rows &r, const Q4Geometry &g, int i, int *status) {
    int s, end;
    if (!r.offsets) {
        s = i / r.per_seq;
        end = (s + 1) * r.per_seq;
        if (s >= r.n_seqs) return RowPlace{0, 0, 0};
    } else {
        int lo = 0, hi = r.n_seqs;                  // the last s with offsets[s] <= i
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (__ldg(r.offsets + mid) <= i) lo = mid;
            else hi = mid;
        }
        s = lo;
        end = min(__ldg(r.offsets + s + 1), (int)r.n_rows);
        if (i < __ldg(r.offsets + s) || i >= end) return RowPlace{0, 0, 0};          // rows before or behind the sequences
    }
    const int pos = q4_length(r, g, s, status) - (end - i);
    if (pos < 0) {                                  // more new rows than the sequence is long
        if (status) atomicAdd(status + 2, 1);
        return RowPlace{0, 0, 0};
    }
    const int page = __ldg(r.table + (long long)s * r.max_pages + (pos >> g.page_shift));
    if (page < 0 || page >= g.n_pages) {
        if (status) atomicAdd(status + 1, 1);
        return RowPlace{0, 0, 0};
    }
    const int in_page = pos & (g.page - 1);
    return RowPlace{page * g.page_bytes + (long long)(in_page / kQ4Tile) * g.tile_bytes, in_page & (kQ4Tile - 1), 1};
}

template <bool H16>
__device__ __forceinline__ void unpack8(const uint4 &w, float *x) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (H16) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&u[i]));
            x[2 * i] = f.x; x[2 * i + 1] = f.y;
        } else {
            x[2 * i] = __uint_as_float(u[i] << 16); x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
    }
}

// Codes of eight values x of a group with scale s (a bf16 value >= 0), packed: value n's code + 8 (1..15) in the nibble of word
// kV ? n : n / 2 + 4 (n % 2).
// The quotient decides between neighbouring codes, and x / s may lie exactly on a border (both have few bits): a plain
// x * (1/s) would land beside it.  x has 11 significant bits at most and s eight, so a quotient up to 7.5 that is not on a
// border is at least 2^-14 away from it; rounding x * (1/s) (off by less than 2^-18, with a reciprocal good to 2^-22) to a multiple of 2^-16 first -
// adding 192 - therefore gives the border itself where the true quotient is on it and keeps the side everywhere else, and
// the rounding to an integer that follows - adding 2^23 * 1.5 - takes ties to even like the division would.
template <bool kV>
__device__ __forceinline__ uint32_t codes8(const float *x, float s) {
    uint32_t w = 0;
    if (s < 5.4210109e-20f) {                       // below 2^-64 (some are subnormal bf16 numbers, whose reciprocal overflows): both sides times 2^64
        const float inv = s > 0.f ? 1.f / (s * 1.8446744e19f) : 0.f;
#pragma unroll
        for (int n = 0; n < 8; ++n) {
            const float q = fminf(fmaxf(__fmul_rn(__fmul_rn(x[n], 1.8446744e19f), inv), -7.f), 7.f);      // (a subnormal scale may be rounded far down)
            const float r = __fadd_rn(__fadd_rn(q, 192.f), 12582912.f + 8.f - 192.f);
            w += __float_as_uint(r) << (kV ? 4 * n : 4 * (n >> 1) + 16 * (n & 1));
        }
    } else {                                        // |q| < 7.04: no clamp
        float inv;
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));
#pragma unroll
        for (int n = 0; n < 8; n += 2) {
            float lo, hi;
            asm("{\n\t.reg .b64 a, b;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %4};\n\tmul.rn.f32x2 a, a, b;\n\tmov.b64 b, {%5, %5};\n\tadd.rn.f32x2 a, a, b;\n\t"
                "mov.b64 b, {%6, %6};\n\tadd.rn.f32x2 a, a, b;\n\tmov.b64 {%0, %1}, a;\n\t}"
                : "=f"(lo), "=f"(hi) : "f"(x[n]), "f"(x[n + 1]), "f"(inv), "f"(192.f), "f"(12582912.f + 8.f - 192.f));
            w += __float_as_uint(lo) << (kV ? 4 * n : 2 * n);
            w += __float_as_uint(hi) << (kV ? 4 * n + 4 : 2 * n + 16);
        }
    }
    return w - 0x4b400000u * 0x11111111u;           // (the eight exponents of the last sums: 0x4b400000 in every shift, modulo 2^32)
}

// The scale bf16(max / 7) from max * (1/7), off by less than 2^-22: a seventh of a number of at most 11 bits is at least 2^-13
// of itself away from the middle between two bf16 numbers.
// (its clamp: 7 * scale has to be finite in bf16; bf16(max / 7) of the type's two largest values is not)
constexpr float kScaleMost = 4.8183102e37f;          // 36.25 * 2^120

// A lane's sixteen channels of one row: the codes' two words and the group's scale (of which the lane holds a half, a quarter
// or an eighth: sixteen channels to a lane rather than eight, so that what is done once per lane - the group's maximum over the
// lanes, scale, reciprocal, addresses - is done half as often; the kernel was bound by instructions).
template <int GL, bool H16, bool kV>
__device__ __forceinline__ void quantise16(const uint4 *raw, uint32_t *w, unsigned short &scale) {
    // largest magnitude of the group, as bits: non-negative 16-bit floats order like integers, infinities and NaN last
    uint32_t mx = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i)
        mx = __vmaxu2(mx, __vmaxu2(__vmaxu2(raw[i].x & 0x7fff7fffu, raw[i].y & 0x7fff7fffu), __vmaxu2(raw[i].z & 0x7fff7fffu, raw[i].w & 0x7fff7fffu)));
    mx = max(mx & 0xffffu, mx >> 16);
#pragma unroll
    for (int d = 1; d < GL; d <<= 1) mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, d));
    const float amax = H16 ? __half2float(__ushort_as_half((unsigned short)mx)) : __uint_as_float(mx << 16);
    const __nv_bfloat16 sb = __float2bfloat16_rn(fminf(amax * (1.f / 7.f), kScaleMost));
    scale = __bfloat16_as_ushort(sb);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        float v[8];
        unpack8<H16>(raw[i], v);
        w[i] = codes8<kV>(v, __bfloat162float(sb));
    }
    if (mx >= (H16 ? 0x7c00u : 0x7f80u)) { w[0] = w[1] = 0x88888888u; scale = 0x7fc0u; }      // not finite: zero codes, and a NaN for a scale
}

// Rows of a CTA and where they lie.
struct CopyRows {
    int row0, n_jobs;                               // jobs: (row, KV head)
};
template <int D>
__device__ __forceinline__ CopyRows copy_rows(const Q4CopyArgs &a) {
    const int row0 = (int)blockIdx.x * a.rows_per_cta;
    return CopyRows{row0, min(a.rows_per_cta, (int)a.rows.n_rows - row0) * a.geo.n_kv_heads};
}

template <int D, int NG, bool H16>
__global__ void __launch_bounds__(kCopyThreads) q4_append_kernel(const __grid_constant__ Q4CopyArgs a) {
    constexpr int LR = D / 16, GL = LR / NG, kSlots = kCopyThreads / LR, kUnroll = 2;      // lanes per row and head, lanes per group
    __shared__ RowPlace places[kCopyRows];
    const Q4Geometry &geo = a.geo;
    const CopyRows cr = copy_rows<D>(a);
    const int l = threadIdx.x % LR, slot = threadIdx.x / LR, j = l >> 1, b = l & 1;      // 32-channel word j, its half b
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (a.chained) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    bool looked_up = false;
    for (int base = 0; base < cr.n_jobs; base += kSlots * kUnroll) {
        uint4 k[kUnroll][2], v[kUnroll][2];
        int row[kUnroll], head[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int job = base + u * kSlots + slot;
            row[u] = __float2int_rz((job + 0.5f) * a.inv_heads);
            head[u] = job - row[u] * geo.n_kv_heads;
            k[u][0] = k[u][1] = v[u][0] = v[u][1] = make_uint4(0u, 0u, 0u, 0u);
            if (job < cr.n_jobs) {
                const long long i = cr.row0 + row[u];
                const uint4 *kp = reinterpret_cast<const uint4 *>(reinterpret_cast<const unsigned short *>(a.k) + i * a.k_row + head[u] * a.k_head) + 2 * l;
                const uint4 *vp = reinterpret_cast<const uint4 *>(reinterpret_cast<const unsigned short *>(a.v) + i * a.v_row + head[u] * a.v_head) + 2 * l;
                k[u][0] = __ldg(kp); k[u][1] = __ldg(kp + 1);
                v[u][0] = __ldg(vp); v[u][1] = __ldg(vp + 1);
            }
        }
        if (!looked_up) {
            looked_up = true;
            if (threadIdx.x < a.rows_per_cta && cr.row0 + threadIdx.x < a.rows.n_rows) places[threadIdx.x] = place_of(a.rows, geo, cr.row0 + threadIdx.x, a.status);
            __syncthreads();
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            if (base + u * kSlots >= cr.n_jobs) break;          // (the same for all threads)
            uint32_t wk[2], wv[2];
            unsigned short sk, sv;
            quantise16<GL, H16, false>(k[u], wk, sk);
            quantise16<GL, H16, true>(v[u], wv, sv);
            // V: this lane has chunks 4b .. 4b + 3 of word j, lane l ^ 2 those of word j ^ 1; even words keep the first two
            // chunks of both lanes and odd words the other two
            const uint32_t other = __shfl_xor_sync(0xffffffffu, j & 1 ? wv[0] : wv[1], 2);
            if (base + u * kSlots + slot >= cr.n_jobs) continue;
            const RowPlace at = places[row[u]];
            if (!at.ok) continue;
            unsigned char *tile = a.pool + at.off + (long long)head[u] * geo.head_bytes;
            const uint32_t lo = j & 1 ? other : wv[0], hi = j & 1 ? wv[1] : other;      // words j & ~1 and j | 1 of two chunks
            *reinterpret_cast<uint32_t *>(tile + q4_k_chunk(D, at.t, 2 * b) + j * 4) = wk[0];
            *reinterpret_cast<uint32_t *>(tile + q4_k_chunk(D, at.t, 2 * b + 1) + j * 4) = wk[1];
            unsigned char *vt = tile + q4_v_base(D) + (j >> 1) * 4;
            const int g0 = 4 * b + 2 * (j & 1);
            *reinterpret_cast<uint32_t *>(vt + q4_v_chunk(D, at.t, g0)) = __byte_perm(lo, hi, 0x5410);
            *reinterpret_cast<uint32_t *>(vt + q4_v_chunk(D, at.t, g0 + 1)) = __byte_perm(lo, hi, 0x7632);
            if (l % GL == 0) {
                *reinterpret_cast<unsigned short *>(tile + q4_ks_base(D) + (at.t * NG + l / GL) * 2) = sk;
                *reinterpret_cast<unsigned short *>(tile + q4_vs_base(D, NG) + (at.t * NG + l / GL) * 2) = sv;
            }
        }
    }
}

// Eight values code * scale, rounded once: w holds value n's code + 8 in nibble n / 2 + 4 (n % 2).
template <bool H16>
__device__ __forceinline__ uint4 values8(uint32_t w, unsigned short scale) {
    uint32_t o[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const uint32_t u = (w >> (4 * p)) & 0x000f000fu;
        if (H16) {                                  // (the scale need not be an fp16 number: products in fp32)
            const uint32_t m = u | 0x64006400u;     // 1024 + code + 8
            const __half2 code = __hsub2(*reinterpret_cast<const __half2 *>(&m), __floats2half2_rn(1032.f, 1032.f));
            const float2 f = __half22float2(code);
            const float s = __uint_as_float((uint32_t)scale << 16);
            const __half2 t = __floats2half2_rn(f.x * s, f.y * s);
            o[p] = *reinterpret_cast<const uint32_t *>(&t);
        } else {
            const uint32_t m = u | 0x43004300u, s = scale | (uint32_t)scale << 16;      // 128 + code + 8
            const __nv_bfloat162 code = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&m), __floats2bfloat162_rn(136.f, 136.f));
            const __nv_bfloat162 t = __hmul2(code, *reinterpret_cast<const __nv_bfloat162 *>(&s));
            o[p] = *reinterpret_cast<const uint32_t *>(&t);
        }
    }
    return make_uint4(o[0], o[1], o[2], o[3]);
}

template <int D, int NG, bool H16>
__global__ void __launch_bounds__(kCopyThreads) q4_read_kernel(const __grid_constant__ Q4CopyArgs a) {
    constexpr int LR = D / 8, GL = LR / NG, kSlots = kCopyThreads / LR;
    __shared__ RowPlace places[kCopyRows];
    const Q4Geometry &geo = a.geo;
    const CopyRows cr = copy_rows<D>(a);
    const int l = threadIdx.x % LR, slot = threadIdx.x / LR, j = l >> 2, c = l & 3;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (a.chained) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (threadIdx.x < a.rows_per_cta && cr.row0 + threadIdx.x < a.rows.n_rows) places[threadIdx.x] = place_of(a.rows, geo, cr.row0 + threadIdx.x, a.status);
    __syncthreads();
    for (int base = 0; base < cr.n_jobs; base += kSlots * kCopyUnroll) {
        uint32_t wk[kCopyUnroll], wv[kCopyUnroll];
        unsigned short sk[kCopyUnroll], sv[kCopyUnroll];
        int row[kCopyUnroll], head[kCopyUnroll];
#pragma unroll
        for (int u = 0; u < kCopyUnroll; ++u) {
            const int job = base + u * kSlots + slot;
            row[u] = __float2int_rz((job + 0.5f) * a.inv_heads);
            head[u] = job - row[u] * geo.n_kv_heads;
            wk[u] = wv[u] = 0;
            sk[u] = sv[u] = 0;
            if (job >= cr.n_jobs) { row[u] = -1; continue; }
            const RowPlace at = places[row[u]];
            if (!at.ok) { row[u] = -1; continue; }
            const unsigned char *tile = a.pool + at.off + (long long)head[u] * geo.head_bytes;
            wk[u] = __ldg(reinterpret_cast<const uint32_t *>(tile + q4_k_chunk(D, at.t, c) + j * 4));
            wv[u] = __ldg(reinterpret_cast<const uint32_t *>(tile + q4_v_base(D) + q4_v_chunk(D, at.t, 2 * c + (j & 1)) + (j >> 1) * 4));
            sk[u] = __ldg(reinterpret_cast<const unsigned short *>(tile + q4_ks_base(D) + (at.t * NG + l / GL) * 2));
            sv[u] = __ldg(reinterpret_cast<const unsigned short *>(tile + q4_vs_base(D, NG) + (at.t * NG + l / GL) * 2));
        }
#pragma unroll
        for (int u = 0; u < kCopyUnroll; ++u) {
            if (base + u * kSlots >= cr.n_jobs) break;          // (the same for all threads)
            const uint32_t other = __shfl_xor_sync(0xffffffffu, wv[u], 4);
            if (row[u] < 0) continue;
            // V: nibble n is channel n; put it into the order of values8()
            uint32_t w = j & 1 ? __byte_perm(other, wv[u], 0x7632) : __byte_perm(wv[u], other, 0x5410);
            const uint32_t ev = w & 0x0f0f0f0fu, od = (w >> 4) & 0x0f0f0f0fu;      // channels 0 2 4 6 / 1 3 5 7, a byte each
            const uint32_t e2 = (ev | ev >> 4) & 0x00ff00ffu, o2 = (od | od >> 4) & 0x00ff00ffu;
            w = __byte_perm(e2, o2, 0x6420);
            const long long i = cr.row0 + row[u];
            reinterpret_cast<uint4 *>(reinterpret_cast<unsigned short *>(a.k) + i * a.k_row + head[u] * a.k_head)[l] = values8<H16>(wk[u], sk[u]);
            reinterpret_cast<uint4 *>(reinterpret_cast<unsigned short *>(a.v) + i * a.v_row + head[u] * a.v_head)[l] = values8<H16>(w, sv[u]);
        }
    }
}

template <bool kWrite>
cudaError_t launch_copy(Q4CopyArgs a, cudaStream_t st) {
    const Q4Geometry &g = a.geo;
    const long long n = a.rows.n_rows;
    if (n <= 0) return cudaSuccess;
    // rows per CTA: 64 (128 at d = 64) jobs (row, head), twice that where it leaves three CTAs per SM, so that a CTA's start, the
    // look-up, is paid half as often (8 heads: 4096 rows, append 13.3 and 14.4 us with the double, 8192 rows 18.4 and 17.4; read of
    // 131072 rows 123 and 117; 40 heads, 4096 rows: append 38.9 and 30.8); fewer where SMs would be idle
    const int slots = kCopyThreads / (g.head_dim / 8);
    long long rows = slots * kCopyUnroll / g.n_kv_heads;
    const long long more = 2LL * slots * kCopyUnroll / g.n_kv_heads;
    if (more > 0 && n / more > 3LL * g.n_sms) rows = more;
    if (rows > n / g.n_sms) rows = n / g.n_sms;
    if (rows < 1) rows = 1;
    if (rows > kCopyRows) rows = kCopyRows;
    a.rows_per_cta = (int)rows;
    a.inv_heads = 1.f / (float)g.n_kv_heads;
    a.chained = q4_chained();
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((n + rows - 1) / rows));
    cfg.blockDim = dim3(kCopyThreads);
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = a.chained;
#define PKV_Q4_COPY1(D, NG, H16) \
    return kWrite ? cudaLaunchKernelEx(&cfg, q4_append_kernel<D, NG, H16>, a) : cudaLaunchKernelEx(&cfg, q4_read_kernel<D, NG, H16>, a);
#define PKV_Q4_COPY(D, NG)                          \
    if (g.head_dim == D && g.groups == NG) {        \
        if (g.fp16) PKV_Q4_COPY1(D, NG, true)       \
        PKV_Q4_COPY1(D, NG, false)                  \
    }
    PKV_Q4_COPY(128, 4) PKV_Q4_COPY(128, 2) PKV_Q4_COPY(128, 1) PKV_Q4_COPY(64, 2) PKV_Q4_COPY(64, 1)
#undef PKV_Q4_COPY
#undef PKV_Q4_COPY1
    return cudaErrorInvalidValue;
}

}  // namespace

namespace pkv {
cudaError_t launch_q4_append(const Q4CopyArgs &a, cudaStream_t st) { return launch_copy<true>(a, st); }
cudaError_t launch_q4_read(const Q4CopyArgs &a, cudaStream_t st) { return launch_copy<false>(a, st); }
}  // namespace pkv

// ---- host side -----------------------------------------------------------------------------------------------------
struct pkv_q4_cache {
    pkv_q4_config cfg;
    Q4Geometry geo;
    bool dry;
    int device;
    unsigned char *pool;
    int *status;
    char err[256];
};

namespace {

pkv_status q4_fail(pkv_q4_cache *c, pkv_status code, const char *fmt, ...) {
    if (c) {
        va_list ap;
        va_start(ap, fmt);
        vsnprintf(c->err, sizeof c->err, fmt, ap);
        va_end(ap);
    }
    return code;
}

pkv_status q4_validate(const pkv_q4_config *cfg, Q4Geometry *g) {
    if (!cfg) return PKV_ERR_INVALID_ARG;
    if (cfg->n_kv_heads <= 0 || cfg->n_q_heads <= 0 || cfg->n_pages <= 0 || cfg->n_ctas < 0 || cfg->n_ctas > 65535 ||
        cfg->n_q_heads % cfg->n_kv_heads != 0 || !std::isfinite(cfg->softmax_scale) || cfg->softmax_scale < 0)
        return PKV_ERR_INVALID_ARG;
    if ((cfg->head_dim != 64 && cfg->head_dim != 128) ||
        (cfg->group_size != 32 && cfg->group_size != 64 && cfg->group_size != 128) || cfg->group_size > cfg->head_dim ||
        cfg->page_size < kQ4Tile || cfg->page_size > 256 || (cfg->page_size & (cfg->page_size - 1)) ||
        (cfg->dtype != PKV_DTYPE_BF16 && cfg->dtype != PKV_DTYPE_FP16) || cfg->n_kv_heads > 1024 ||
        cfg->n_q_heads / cfg->n_kv_heads > 64 || cfg->n_pages > 0x7fffffffLL)
        return PKV_ERR_UNSUPPORTED;
    *g = Q4Geometry{};
    g->n_kv_heads = cfg->n_kv_heads;
    g->n_q_heads = cfg->n_q_heads;
    g->group = cfg->n_q_heads / cfg->n_kv_heads;
    g->head_dim = cfg->head_dim;
    g->page = cfg->page_size;
    for (g->page_shift = 0; (1 << g->page_shift) < g->page;) ++g->page_shift;
    g->groups = cfg->head_dim / cfg->group_size;
    g->tile_bytes = kQ4Tile * (cfg->head_dim + 4 * g->groups);
    g->head_bytes = g->page / kQ4Tile * g->tile_bytes;
    g->fp16 = cfg->dtype == PKV_DTYPE_FP16;
    g->page_bytes = (long long)g->n_kv_heads * g->head_bytes;
    g->n_pages = cfg->n_pages;
    if (g->n_pages > (1LL << 60) / g->page_bytes) return PKV_ERR_INVALID_ARG;
    const float scale = cfg->softmax_scale > 0 ? cfg->softmax_scale : 1.f / std::sqrt((float)cfg->head_dim);
    g->scale_log2e = scale * 1.4426950408889634f;
    if (!std::isfinite(g->scale_log2e)) return PKV_ERR_INVALID_ARG;
    return PKV_OK;
}

// What append, read and attention have in common: the sequences, and the rows that belong to them.
pkv_status q4_rows(pkv_q4_cache *c, const char *what, int32_t n_seqs, const int32_t *table, int32_t max_pages,
                   const int32_t *lengths, int64_t n_rows, const int32_t *offsets, Q4Rows *r, bool with_table = true, bool with_lengths = true) {
    if (n_seqs < 1 || n_seqs > 65535) return q4_fail(c, PKV_ERR_INVALID_ARG, "%s: n_seqs %d out of range", what, n_seqs);
    if (max_pages < 1 || max_pages > ((1 << 30) >> c->geo.page_shift))
        return q4_fail(c, PKV_ERR_INVALID_ARG, "%s: max_pages %d out of range", what, max_pages);
    if (n_rows < 0 || n_rows > 0x7fffffff / (2 * c->geo.n_q_heads))
        return q4_fail(c, PKV_ERR_INVALID_ARG, "%s: n_rows %lld out of range", what, (long long)n_rows);
    if (!offsets && n_rows % n_seqs != 0)
        return q4_fail(c, PKV_ERR_INVALID_ARG, "%s: %lld rows do not divide among %d sequences (give offsets)", what, (long long)n_rows, n_seqs);
    if (!c->dry && ((with_table && !table) || (with_lengths && !lengths)))
        return q4_fail(c, PKV_ERR_INVALID_ARG, "%s: %s is NULL", what, with_table ? "page_table or lengths" : "lengths");
    if (((uintptr_t)table | (uintptr_t)lengths | (uintptr_t)offsets) & 3)
        return q4_fail(c, PKV_ERR_INVALID_ARG, "%s: page_table, lengths and offsets must be 4-byte aligned", what);
    *r = Q4Rows{table, lengths, offsets, n_seqs, max_pages, offsets ? 0 : (int)(n_rows / n_seqs), n_rows};
    return PKV_OK;
}

pkv_status q4_device(pkv_q4_cache *c, const char *what) {
    int dev = -1;
    const cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return q4_fail(c, PKV_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
    if (dev != c->device) return q4_fail(c, PKV_ERR_INVALID_ARG, "%s: the cache is on device %d, the current device is %d", what, c->device, dev);
    return PKV_OK;
}

// strides of a [rows, heads, d] buffer in elements: rows and heads on 16-byte boundaries, none on top of another
bool q4_strides(const void *p, int64_t row, int64_t head, int d, int heads, int64_t n_rows) {
    if (((uintptr_t)p & 15) || row % 8 || head % 8 || row < 0 || head < 0) return false;
    if (row > (1LL << 31) || head > (1LL << 31)) return false;
    if (heads == 1) return n_rows <= 1 || row >= d;
    if (n_rows <= 1) return head >= d;
    // rows of all heads one after the other, or the other way round
    return (head >= d && row >= (heads - 1) * head + d) || (row >= d && head >= (n_rows - 1) * row + d);
}

pkv_status q4_copy(pkv_q4_cache *c, bool write, int32_t n_seqs, const int32_t *table, int32_t max_pages, const int32_t *lengths,
                   int64_t n_rows, const int32_t *offsets, void *k, int64_t k_row, int64_t k_head, void *v, int64_t v_row,
                   int64_t v_head, void *stream) {
    if (!c) return PKV_ERR_INVALID_ARG;
    const char *what = write ? "pkv_q4_append_kv" : "pkv_q4_read_kv";
    Q4CopyArgs a{};
    if (pkv_status st = q4_rows(c, what, n_seqs, table, max_pages, lengths, n_rows, offsets, &a.rows)) return st;
    const Q4Geometry &g = c->geo;
    if (!c->dry && n_rows > 0 && (!k || !v)) return q4_fail(c, PKV_ERR_INVALID_ARG, "%s: k or v is NULL", what);
    if (!q4_strides(k, k_row, k_head, g.head_dim, g.n_kv_heads, n_rows) || !q4_strides(v, v_row, v_head, g.head_dim, g.n_kv_heads, n_rows))
        return q4_fail(c, PKV_ERR_INVALID_ARG, "%s: k and v need 16-byte aligned rows: strides that are multiples of 8 elements, no row or "
                                               "head on top of another", what);
    if (c->dry || n_rows == 0) return PKV_OK;
    if (pkv_status st = q4_device(c, what)) return st;
    a.geo = g;
    a.pool = c->pool;
    a.k = k; a.v = v;
    a.k_row = k_row; a.k_head = k_head; a.v_row = v_row; a.v_head = v_head;
    a.status = c->status;
    const cudaError_t e = write ? launch_q4_append(a, (cudaStream_t)stream) : launch_q4_read(a, (cudaStream_t)stream);
    if (e != cudaSuccess) return q4_fail(c, PKV_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
    return PKV_OK;
}

// An array of a call; the first ones of a list are written.  Kernels read and write in no particular order, so what is written must not lie on
// anything else.
struct Q4Array { const char *name; const void *at; long long bytes; };
pkv_status q4_apart(pkv_q4_cache *c, const char *what, const Q4Array *x, int n_written, int n) {
    for (int i = 0; i < n_written; ++i)
        for (int k = i + 1; k < n; ++k) {
            const uintptr_t a = (uintptr_t)x[i].at, b = (uintptr_t)x[k].at;
            if (a && b && x[i].bytes > 0 && x[k].bytes > 0 && a < b + x[k].bytes && b < a + x[i].bytes) return q4_fail(c, PKV_ERR_INVALID_ARG, "%s: %s overlaps %s", what, x[i].name, x[k].name);
        }
    return PKV_OK;
}

// ---- attention: what every form checks -----------------------------------------------------------------------------------
// What is wrong with a choice of positions, or NULL.
const char *q4_select_error(const pkv_q4_select &s, int max_q_len) {
    if (s.window < 0 || s.sinks < 0) return "window and sinks must not be negative";
    if (s.sinks > 0 && s.window == 0) return "sinks need a window";
    if ((uintptr_t)s.tree & 7) return "the tree's masks must be 8-byte aligned";
    if (s.tree && (s.tree_words < 1 || s.tree_words < (max_q_len + 63LL) / 64)) return "tree_words must be max_q_len / 64, rounded up, at least";
    return nullptr;
}
// (positions stay below 2^30: a wider window is none, and sums of a few stay in 32 bits)
Q4Select q4_selection(const pkv_q4_select &s) { return Q4Select{std::min(s.window, 1 << 30), std::min(s.sinks, 1 << 30), s.tree != nullptr}; }

pkv_status q4_attend(pkv_q4_cache *c, const char *what, int32_t n_seqs, const int32_t *page_table, int32_t max_pages, const int32_t *lengths,
                     int64_t n_rows, const int32_t *offsets, int32_t max_q_len, int32_t max_len, const pkv_q4_select *select, const void *q,
                     int64_t q_row_stride, int64_t q_head_stride, void *out, int64_t out_row_stride, int64_t out_head_stride, float *state,
                     void *workspace, int64_t workspace_bytes, void *stream) {
    if (!c) return PKV_ERR_INVALID_ARG;
    Q4AttentionArgs a{};
    if (pkv_status st = q4_rows(c, what, n_seqs, page_table, max_pages, lengths, n_rows, offsets, &a.rows)) return st;
    const Q4Geometry &g = c->geo;
    const int capacity = max_pages << g.page_shift;
    if (!offsets) max_q_len = a.rows.per_seq;
    if (n_rows > 0 && (max_q_len < 0 || max_q_len > n_rows)) return q4_fail(c, PKV_ERR_INVALID_ARG, "%s: max_q_len %d out of range", what, max_q_len);
    if (max_len < 0) return q4_fail(c, PKV_ERR_INVALID_ARG, "%s: max_len %d out of range", what, max_len);
    if (max_len == 0 || max_len > capacity) max_len = capacity;
    if (!c->dry && n_rows > 0 && (!q || (!out == !state)))
        return q4_fail(c, PKV_ERR_INVALID_ARG, "%s: q is NULL, or not exactly one of out and state is given", what);
    if (!q4_strides(q, q_row_stride, q_head_stride, g.head_dim, g.n_q_heads, n_rows) ||
        (out && !q4_strides(out, out_row_stride, out_head_stride, g.head_dim, g.n_q_heads, n_rows)))
        return q4_fail(c, PKV_ERR_INVALID_ARG, "%s: q and out need 16-byte aligned rows: strides that are multiples of 8 elements, no row or "
                                               "head on top of another", what);
    if (select)
        if (const char *error = q4_select_error(*select, n_rows > 0 ? max_q_len : 0)) return q4_fail(c, PKV_ERR_INVALID_ARG, "%s: %s", what, error);
    const Q4Select sel = select ? q4_selection(*select) : Q4Select{};
    if ((uintptr_t)state & 7) return q4_fail(c, PKV_ERR_INVALID_ARG, "%s: state must be 8-byte aligned", what);
    if (n_rows == 0 || max_q_len == 0) return PKV_OK;
    const long long need = q4_attention_workspace(g, n_seqs, max_q_len, max_len, sel);
    if (!c->dry && need > 0 && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 15)))
        return q4_fail(c, PKV_ERR_INVALID_ARG, "%s: the workspace needs %lld bytes, 16-byte aligned", what, need);
    if (select && select->tree) {                      // (read by all KV heads, while the first of them write)
        // (strided results may have anything between their rows)
        const long long heads = (long long)n_rows * g.n_q_heads, span = (n_rows - 1) * out_row_stride + (g.n_q_heads - 1) * out_head_stride + g.head_dim;
        const Q4Array arrays[] = {{"tree", select->tree, 8LL * n_rows * select->tree_words}, {"state", state, heads * (g.head_dim + 2) * 4}, {"workspace", need > 0 ? workspace : nullptr, need},
                                  {"out", out, span == heads * g.head_dim ? 2 * span : 0}};
        if (pkv_status st = q4_apart(c, what, arrays, 1, 4)) return st;
    }
    if (c->dry) return PKV_OK;
    if (pkv_status st = q4_device(c, what)) return st;
    a.geo = g;
    a.pool = c->pool;
    a.q = q; a.out = out; a.state = state;
    a.q_row = q_row_stride; a.q_head = q_head_stride; a.out_row = out_row_stride; a.out_head = out_head_stride;
    a.max_q_len = max_q_len;
    a.max_len = max_len;
    a.workspace = static_cast<unsigned char *>(workspace);
    a.status = c->status;
    a.window = sel.window;
    a.sinks = sel.sinks;
    if (select) {
        a.tree = reinterpret_cast<const unsigned long long *>(select->tree);
        a.tree_words = select->tree_words;
    }
    const cudaError_t e = launch_q4_attention(a, (cudaStream_t)stream);
    if (e != cudaSuccess) return q4_fail(c, PKV_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
    return PKV_OK;
}

}  // namespace

extern "C" {

pkv_status pkv_q4_query_sizes(const pkv_q4_config *cfg, pkv_q4_sizes *out) {
    if (!out) return PKV_ERR_INVALID_ARG;
    Q4Geometry g;
    if (pkv_status st = q4_validate(cfg, &g)) return st;
    out->page_bytes = g.page_bytes;
    out->pool_bytes = g.page_bytes * g.n_pages;
    out->meta_bytes = 256;
    return PKV_OK;
}

pkv_status pkv_q4_init_cache(const pkv_q4_config *cfg, void *pool, void *meta, pkv_q4_cache **out) {
    if (!out) return PKV_ERR_INVALID_ARG;
    *out = nullptr;
    Q4Geometry g;
    if (pkv_status st = q4_validate(cfg, &g)) return st;
    const bool dry = !pool && !meta;
    if (!dry && (!pool || !meta || (((uintptr_t)pool | (uintptr_t)meta) & 255))) return PKV_ERR_INVALID_ARG;
    pkv_q4_cache *c = new (std::nothrow) pkv_q4_cache();
    if (!c) return PKV_ERR_INVALID_ARG;
    c->cfg = *cfg;
    c->dry = dry;
    c->pool = static_cast<unsigned char *>(pool);
    c->status = static_cast<int *>(meta);
    c->err[0] = 0;
    g.n_sms = 148;
    if (!dry) {
        cudaError_t e = cudaGetDevice(&c->device);
        if (e == cudaSuccess) e = cudaDeviceGetAttribute(&g.n_sms, cudaDevAttrMultiProcessorCount, c->device);
        if (e == cudaSuccess) e = q4_attention_setup(g);
        if (e == cudaSuccess) e = q4_serve_setup(g);
        if (e == cudaSuccess) e = cudaMemset(meta, 0, 256);
        if (e != cudaSuccess) { delete c; return PKV_ERR_CUDA; }
    }
    g.n_ctas = cfg->n_ctas > 0 ? cfg->n_ctas : 2 * g.n_sms;
    c->geo = g;
    *out = c;
    return PKV_OK;
}

pkv_status pkv_q4_destroy_cache(pkv_q4_cache *c) {
    if (!c) return PKV_ERR_INVALID_ARG;
    delete c;
    return PKV_OK;
}

const char *pkv_q4_last_error(const pkv_q4_cache *c) { return c ? c->err : "cache is NULL"; }

pkv_status pkv_q4_append_kv(pkv_q4_cache *c, int32_t n_seqs, const int32_t *page_table, int32_t max_pages, const int32_t *lengths,
                            int64_t n_rows, const int32_t *offsets, const void *k, int64_t k_row_stride, int64_t k_head_stride,
                            const void *v, int64_t v_row_stride, int64_t v_head_stride, void *stream) {
    return q4_copy(c, true, n_seqs, page_table, max_pages, lengths, n_rows, offsets, const_cast<void *>(k), k_row_stride, k_head_stride,
                   const_cast<void *>(v), v_row_stride, v_head_stride, stream);
}

pkv_status pkv_q4_read_kv(pkv_q4_cache *c, int32_t n_seqs, const int32_t *page_table, int32_t max_pages, const int32_t *lengths,
                          int64_t n_rows, const int32_t *offsets, void *k, int64_t k_row_stride, int64_t k_head_stride, void *v,
                          int64_t v_row_stride, int64_t v_head_stride, void *stream) {
    return q4_copy(c, false, n_seqs, page_table, max_pages, lengths, n_rows, offsets, k, k_row_stride, k_head_stride, v, v_row_stride,
                   v_head_stride, stream);
}

pkv_status pkv_q4_attention_workspace(const pkv_q4_cache *c, int32_t n_seqs, int32_t max_q_len, int32_t max_len, int64_t *bytes) {
    if (!c || !bytes || n_seqs < 1 || n_seqs > 65535 || max_q_len < 1 || max_len < 1) return PKV_ERR_INVALID_ARG;
    *bytes = q4_attention_workspace(c->geo, n_seqs, max_q_len, max_len, Q4Select{});
    return PKV_OK;
}

pkv_status pkv_q4_attention(pkv_q4_cache *c, int32_t n_seqs, const int32_t *page_table, int32_t max_pages, const int32_t *lengths,
                            int64_t n_rows, const int32_t *offsets, int32_t max_q_len, int32_t max_len, const void *q,
                            int64_t q_row_stride, int64_t q_head_stride, void *out, int64_t out_row_stride, int64_t out_head_stride,
                            float *state, void *workspace, int64_t workspace_bytes, void *stream) {
    return q4_attend(c, "pkv_q4_attention", n_seqs, page_table, max_pages, lengths, n_rows, offsets, max_q_len, max_len, nullptr, q, q_row_stride,
                     q_head_stride, out, out_row_stride, out_head_stride, state, workspace, workspace_bytes, stream);
}

pkv_status pkv_q4_attention_select_workspace(const pkv_q4_cache *c, int32_t n_seqs, int32_t max_q_len, int32_t max_len,
                                             const pkv_q4_select *select, int64_t *bytes) {
    if (!c || !bytes || !select || n_seqs < 1 || n_seqs > 65535 || max_q_len < 1 || max_len < 1) return PKV_ERR_INVALID_ARG;
    if (q4_select_error(*select, max_q_len)) return PKV_ERR_INVALID_ARG;
    *bytes = q4_attention_workspace(c->geo, n_seqs, max_q_len, max_len, q4_selection(*select));
    return PKV_OK;
}

pkv_status pkv_q4_attention_route(const pkv_q4_cache *c, int32_t n_seqs, int32_t max_q_len, int32_t max_len, const pkv_q4_select *select,
                                  int32_t *kernel, int32_t *n_ctas, int32_t *cluster) {
    if (!c || !kernel || !n_ctas || !cluster || n_seqs < 1 || n_seqs > 65535 || max_q_len < 1 || max_len < 1) return PKV_ERR_INVALID_ARG;
    if (select && q4_select_error(*select, max_q_len)) return PKV_ERR_INVALID_ARG;
    q4_attention_route(c->geo, n_seqs, max_q_len, max_len, select ? q4_selection(*select) : Q4Select{}, kernel, n_ctas, cluster);
    return PKV_OK;
}

pkv_status pkv_q4_attention_select(pkv_q4_cache *c, int32_t n_seqs, const int32_t *page_table, int32_t max_pages, const int32_t *lengths,
                                   int64_t n_rows, const int32_t *offsets, int32_t max_q_len, int32_t max_len, const pkv_q4_select *select,
                                   const void *q, int64_t q_row_stride, int64_t q_head_stride, void *out, int64_t out_row_stride,
                                   int64_t out_head_stride, float *state, void *workspace, int64_t workspace_bytes, void *stream) {
    if (!c) return PKV_ERR_INVALID_ARG;
    const char *what = "pkv_q4_attention_select";
    if (!select) return q4_fail(c, PKV_ERR_INVALID_ARG, "%s: select is NULL", what);
    return q4_attend(c, what, n_seqs, page_table, max_pages, lengths, n_rows, offsets, max_q_len, max_len, select, q, q_row_stride, q_head_stride,
                     out, out_row_stride, out_head_stride, state, workspace, workspace_bytes, stream);
}

pkv_status pkv_q4_tree_masks(pkv_q4_cache *c, int32_t n_seqs, const int32_t *lengths, int64_t n_rows, const int32_t *offsets,
                             int32_t max_q_len, const int32_t *parents, int32_t window, int32_t sinks, uint64_t *tree,
                             int32_t tree_words, int32_t *depths, void *stream) {
    if (!c) return PKV_ERR_INVALID_ARG;
    const char *what = "pkv_q4_tree_masks";
    Q4TreeArgs a{};
    const bool far = window > 0 && sinks > 0;      // lengths are needed
    if (pkv_status st = q4_rows(c, what, n_seqs, nullptr, 1, lengths, n_rows, offsets, &a.rows, false, far)) return st;
    if (!offsets) max_q_len = a.rows.per_seq;
    if (n_rows > 0 && (max_q_len < 0 || max_q_len > n_rows)) return q4_fail(c, PKV_ERR_INVALID_ARG, "%s: max_q_len %d out of range", what, max_q_len);
    const pkv_q4_select sel{window, sinks, tree, tree_words};
    if (const char *error = q4_select_error(sel, max_q_len)) return q4_fail(c, PKV_ERR_INVALID_ARG, "%s: %s", what, error);
    if (tree_words < 1 || tree_words < (max_q_len + 63LL) / 64) return q4_fail(c, PKV_ERR_INVALID_ARG, "%s: tree_words %d out of range", what, tree_words);
    if (((uintptr_t)parents | (uintptr_t)depths) & 3) return q4_fail(c, PKV_ERR_INVALID_ARG, "%s: parents and depths must be 4-byte aligned", what);
    if (!c->dry && n_rows > 0 && (!parents || !tree)) return q4_fail(c, PKV_ERR_INVALID_ARG, "%s: parents or tree is NULL", what);
    const Q4Array arrays[] = {{"tree", tree, 8LL * n_rows * tree_words}, {"depths", depths, 4LL * n_rows}, {"parents", parents, 4LL * n_rows},
                              {"lengths", far ? lengths : nullptr, 4LL * n_seqs}, {"offsets", offsets, 4LL * (n_seqs + 1)}};
    if (pkv_status st = q4_apart(c, what, arrays, 2, 5)) return st;
    if (c->dry || n_rows == 0 || max_q_len == 0) return PKV_OK;
    if (pkv_status st = q4_device(c, what)) return st;
    if (!far) a.rows.lengths = nullptr;
    a.parents = parents;
    a.tree = reinterpret_cast<unsigned long long *>(tree);
    a.depths = depths;
    a.status = c->status;
    a.max_q_len = max_q_len;
    a.words = tree_words;
    a.window = q4_selection(sel).window;
    a.sinks = q4_selection(sel).sinks;
    const cudaError_t e = launch_q4_tree_masks(a, (cudaStream_t)stream);
    if (e != cudaSuccess) return q4_fail(c, PKV_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
    return PKV_OK;
}

pkv_status pkv_q4_keep_rows(pkv_q4_cache *c, int32_t n_seqs, const int32_t *page_table, int32_t max_pages, const int32_t *lengths,
                            int64_t n_rows, const int32_t *offsets, const int32_t *paths, int32_t max_path, const int32_t *counts,
                            int32_t *lengths_out, void *stream) {
    if (!c) return PKV_ERR_INVALID_ARG;
    const char *what = "pkv_q4_keep_rows";
    Q4KeepArgs a{};
    if (pkv_status st = q4_rows(c, what, n_seqs, page_table, max_pages, lengths, n_rows, offsets, &a.rows)) return st;
    if (max_path < 0) return q4_fail(c, PKV_ERR_INVALID_ARG, "%s: max_path %d out of range", what, max_path);
    if (((uintptr_t)paths | (uintptr_t)counts | (uintptr_t)lengths_out) & 3)
        return q4_fail(c, PKV_ERR_INVALID_ARG, "%s: paths, counts and lengths_out must be 4-byte aligned", what);
    if (!c->dry && ((!paths && max_path > 0) || !counts || !lengths_out)) return q4_fail(c, PKV_ERR_INVALID_ARG, "%s: paths, counts or lengths_out is NULL", what);
    const Q4Array arrays[] = {{"lengths_out", lengths_out, 4LL * n_seqs}, {"lengths", lengths, 4LL * n_seqs}, {"counts", counts, 4LL * n_seqs},
                              {"paths", paths, 4LL * n_seqs * max_path}, {"offsets", offsets, 4LL * (n_seqs + 1)},
                              {"page_table", page_table, 4LL * n_seqs * max_pages}};
    if (pkv_status st = q4_apart(c, what, arrays, 1, 6)) return st;
    if (c->dry) return PKV_OK;
    if (pkv_status st = q4_device(c, what)) return st;
    a.geo = c->geo;
    a.pool = c->pool;
    a.paths = paths;
    a.counts = counts;
    a.lengths_out = lengths_out;
    a.status = c->status;
    a.max_path = max_path;
    const cudaError_t e = launch_q4_keep(a, (cudaStream_t)stream);
    if (e != cudaSuccess) return q4_fail(c, PKV_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
    return PKV_OK;
}

pkv_status pkv_q4_plan_workspace(const pkv_q4_cache *c, int32_t n_seqs, int64_t n_rows, int64_t *bytes) {
    if (!c || !bytes || n_seqs < 1 || n_seqs > 65535 || n_rows < 0 || n_rows > 0x3fffffff) return PKV_ERR_INVALID_ARG;
    *bytes = q4_plan_workspace(n_seqs, n_rows);
    return PKV_OK;
}

pkv_status pkv_q4_plan(pkv_q4_cache *c, int32_t n_seqs, int32_t *page_table, int32_t max_pages, const int32_t *lengths, const int32_t *rows,
                       const int32_t *spans, int32_t *ring, const int64_t *counters, int32_t window, int32_t sinks, int32_t *lengths_out,
                       int32_t *spans_out, int64_t *counters_out, int32_t *offsets, int64_t n_rows, int32_t *positions, int64_t *slots,
                       void *workspace, int64_t workspace_bytes, void *stream) {
    if (!c) return PKV_ERR_INVALID_ARG;
    const char *what = "pkv_q4_plan";
    const Q4Geometry &g = c->geo;
    if (n_seqs < 1 || n_seqs > 65535) return q4_fail(c, PKV_ERR_INVALID_ARG, "%s: n_seqs %d out of range", what, n_seqs);
    if (max_pages < 1 || max_pages > ((1 << 30) >> g.page_shift)) return q4_fail(c, PKV_ERR_INVALID_ARG, "%s: max_pages %d out of range", what, max_pages);
    if (n_rows < 0 || n_rows > 0x3fffffff) return q4_fail(c, PKV_ERR_INVALID_ARG, "%s: n_rows %lld out of range", what, (long long)n_rows);
    const pkv_q4_select sel{window, sinks, nullptr, 0};
    if (const char *error = q4_select_error(sel, 0)) return q4_fail(c, PKV_ERR_INVALID_ARG, "%s: %s", what, error);
    if (((uintptr_t)page_table | (uintptr_t)lengths | (uintptr_t)rows | (uintptr_t)spans | (uintptr_t)ring | (uintptr_t)lengths_out |
         (uintptr_t)spans_out | (uintptr_t)offsets | (uintptr_t)positions) & 3 ||
        ((uintptr_t)counters | (uintptr_t)counters_out | (uintptr_t)slots) & 7)
        return q4_fail(c, PKV_ERR_INVALID_ARG, "%s: int32 arrays must be 4-byte and int64 arrays 8-byte aligned", what);
    if (!c->dry && (!page_table || !lengths || !rows || !spans || !ring || !counters || !lengths_out || !spans_out || !counters_out || !offsets))
        return q4_fail(c, PKV_ERR_INVALID_ARG, "%s: only positions and slots may be NULL", what);
    const long long need = q4_plan_workspace(n_seqs, n_rows);
    // (in place is the same array, not a part of it: a thread reads its own request before it writes it)
    const Q4Array arrays[] = {{"page_table", page_table, 4LL * n_seqs * max_pages}, {"ring", ring, 4LL * g.n_pages},
                              {"lengths_out", lengths_out, 4LL * n_seqs}, {"spans_out", spans_out, 8LL * n_seqs}, {"counters_out", counters_out, 32},
                              {"offsets", offsets, 4LL * (n_seqs + 1)}, {"positions", positions, 4LL * n_rows}, {"slots", slots, 8LL * n_rows},
                              {"workspace", need > 0 ? workspace : nullptr, need}, {"rows", rows, 4LL * n_seqs},
                              {"lengths", lengths == lengths_out ? nullptr : lengths, 4LL * n_seqs}, {"spans", spans == spans_out ? nullptr : spans, 8LL * n_seqs},
                              {"counters", counters == counters_out ? nullptr : counters, 32}};
    if (pkv_status st = q4_apart(c, what, arrays, 9, 13)) return st;
    if (!c->dry && need > 0 && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 15)))
        return q4_fail(c, PKV_ERR_INVALID_ARG, "%s: the workspace needs %lld bytes, 16-byte aligned", what, need);
    if (c->dry) return PKV_OK;
    if (pkv_status st = q4_device(c, what)) return st;
    Q4PlanArgs a{};
    a.n_seqs = n_seqs;
    a.max_pages = max_pages;
    a.page_shift = g.page_shift;
    a.window = q4_selection(sel).window;
    a.sink_pages = window > 0 ? (int)(((long long)q4_selection(sel).sinks + g.page - 1) >> g.page_shift) : 0;
    a.n_pages = g.n_pages;
    a.n_rows = n_rows;
    a.table = page_table;
    a.ring = ring;
    a.lengths = lengths;
    a.rows = rows;
    a.spans = spans;
    a.counters = reinterpret_cast<const long long *>(counters);
    a.lengths_out = lengths_out;
    a.spans_out = spans_out;
    a.counters_out = reinterpret_cast<long long *>(counters_out);
    a.offsets = offsets;
    a.positions = positions;
    a.slots = reinterpret_cast<long long *>(slots);
    a.workspace = static_cast<unsigned char *>(workspace);
    const cudaError_t e = launch_q4_plan(a, (cudaStream_t)stream);
    if (e != cudaSuccess) return q4_fail(c, PKV_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
    return PKV_OK;
}

pkv_status pkv_q4_get_stats(pkv_q4_cache *c, pkv_q4_stats *out, void *stream) {
    if (!c || !out) return PKV_ERR_INVALID_ARG;
    int words[kQ4StatusWords] = {};
    if (!c->dry) {
        if (pkv_status st = q4_device(c, "pkv_q4_get_stats")) return st;
        cudaError_t e = cudaMemcpyAsync(words, c->status, sizeof words, cudaMemcpyDeviceToHost, (cudaStream_t)stream);
        if (e == cudaSuccess) e = cudaStreamSynchronize((cudaStream_t)stream);
        if (e != cudaSuccess) return q4_fail(c, PKV_ERR_CUDA, "pkv_q4_get_stats: %s", cudaGetErrorString(e));
    }
    out->device_timeouts = words[0];
    out->bad_pages = words[1];
    out->bad_lengths = words[2];
    return PKV_OK;
}

}  // extern "C"
