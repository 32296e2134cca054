// Attention over the paged 4-bit cache for queries that see a part of the positions: a sliding window and the first
// positions, or the ancestors of a drafted token.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "pkv_q4_device.cuh"

namespace pkv {

namespace {

// code * scale of one element of a tile (exact in fp32)
__device__ __forceinline__ float q4_value(const Q4Geometry &g, const unsigned char *tile, bool v, int t, int ch) {
    const int d = g.head_dim, w = ch >> 5, in = ch & 31;
    const int off = v ? q4_v_base(d) + q4_v_chunk(d, t, in >> 2) + w * 2 + ((in & 3) >> 1) : q4_k_chunk(d, t, in >> 3) + w * 4;
    int nib;
    if (v) nib = tile[off] >> (4 * (in & 1)) & 15;
    else nib = *reinterpret_cast<const uint32_t *>(tile + off) >> (4 * ((in & 7) >> 1) + 16 * (in & 1)) & 15;
    const unsigned short s = *reinterpret_cast<const unsigned short *>(tile + (v ? q4_vs_base(d, g.groups) : q4_ks_base(d)) +
                                                                       (t * g.groups + ch / (d / g.groups)) * 2);
    return (float)(nib - 8) * __uint_as_float((uint32_t)s << 16);
}

// The simplest form: a warp per query row and head, a token at a time.
__global__ void __launch_bounds__(128) q4_simple_kernel(const __grid_constant__ Q4AttentionArgs a) {
    const Q4Geometry &g = a.geo;
    const int lane = threadIdx.x & 31, d = g.head_dim, per = d / 32, s = blockIdx.y;
    const long long job = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    const int j = (int)(job / g.n_q_heads), h = (int)(job - (long long)j * g.n_q_heads);
    int first, all;
    const int n = q4_new_rows(a, s, first, all, job == 0 && lane == 0 ? a.status : nullptr);
    const int T = q4_length(a.rows, g, s, job == 0 && lane == 0 ? a.status : nullptr);
    if (j >= n) return;
    const int kv = h / g.group, C = T - all;
    const unsigned long long *bits = a.tree ? a.tree + (long long)(first + j) * a.tree_words : nullptr;
    const int see = a.tree ? T : C + j + 1;
    int own = j + 1;                       // new rows that the query sees
    if (a.tree) {
        own = 0;
        for (int w = 0; w < min(a.tree_words, (all + 63) / 64); ++w) own += __popcll(bits[w] & (all - 64 * w >= 64 ? ~0ull : (1ull << (all - 64 * w)) - 1));
    }
    const int lo = a.window ? max(0, C + own - a.window) : 0;
    float q[4], o[4] = {0.f, 0.f, 0.f, 0.f}, m = -1e30f, l = 0.f;
    for (int i = 0; i < per; ++i) {
        const long long at = (first + j) * a.q_row + h * a.q_head + lane + 32 * i;
        q[i] = g.fp16 ? __half2float(reinterpret_cast<const __half *>(a.q)[at]) : __bfloat162float(reinterpret_cast<const __nv_bfloat16 *>(a.q)[at]);
    }
    for (int t = 0; t < see; ++t) {
        if (a.tree && t >= C) {
            const int i = t - C;
            if (i >= a.tree_words * 64LL || !(bits[i >> 6] >> (i & 63) & 1)) continue;
        } else if (t < lo && t >= a.sinks) {
            t = min(lo, a.tree ? max(C, 0) : see) - 1;
            continue;
        }
        const int page = a.rows.table[(long long)s * a.rows.max_pages + (t >> g.page_shift)];
        if (page < 0 || page >= g.n_pages) {
            if (lane == 0 && (t & (g.page - 1)) == 0) atomicAdd(a.status + 1, 1);
            continue;
        }
        const int in = t & (g.page - 1);
        const unsigned char *tile = a.pool + page * g.page_bytes + (long long)kv * g.head_bytes + in / kQ4Tile * g.tile_bytes;
        float x = 0.f;
        for (int i = 0; i < per; ++i) x += q[i] * q4_value(g, tile, false, in & 15, lane + 32 * i);
        for (int k = 16; k; k >>= 1) x += __shfl_xor_sync(0xffffffffu, x, k);
        x *= g.scale_log2e;
        const float mn = fmaxf(m, x), f = exp2f(m - mn), p = exp2f(x - mn);
        m = mn;
        l = l * f + p;
        for (int i = 0; i < per; ++i) o[i] = o[i] * f + p * q4_value(g, tile, true, in & 15, lane + 32 * i);
    }
    const float inv = l != 0.f ? 1.f / l : 0.f;
    const long long row = first + j;
    for (int i = 0; i < per; ++i) {
        const int ch = lane + 32 * i;
        if (a.state) {
            a.state[(row * g.n_q_heads + h) * (d + 2) + ch] = o[i];
        } else {
            const long long at = row * a.out_row + h * a.out_head + ch;
            if (g.fp16) reinterpret_cast<__half *>(a.out)[at] = __float2half_rn(o[i] * inv);
            else reinterpret_cast<__nv_bfloat16 *>(a.out)[at] = __float2bfloat16_rn(o[i] * inv);
        }
    }
    if (a.state && lane == 0) {
        a.state[(row * g.n_q_heads + h) * (d + 2) + d] = m;
        a.state[(row * g.n_q_heads + h) * (d + 2) + d + 1] = l;
    }
}

}  // namespace

long long q4_select_workspace(const Q4Geometry &, int, int, int, const Q4Select &) { return 0; }

cudaError_t launch_q4_select(Q4AttentionArgs a, cudaStream_t st) {
    const long long jobs = (long long)a.max_q_len * a.geo.n_q_heads;
    q4_simple_kernel<<<dim3((unsigned)((jobs + 3) / 4), a.rows.n_seqs), 128, 0, st>>>(a);
    return cudaGetLastError();
}

}  // namespace pkv
