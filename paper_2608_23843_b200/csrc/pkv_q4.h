// Internal declarations of the paged cache that holds keys and values in 4 bits: geometry, storage format, launchers.
//
// A page belongs to one layer and holds P tokens of every KV head, head after head.  A head's part is a run of tiles of
// 16 tokens, and a tile is
//     [K codes 16 x d/2 bytes][V codes 16 x d/2 bytes][K scales 16 x d/g bf16][V scales 16 x d/g bf16]
// so that the tiles a query needs of a page are one contiguous piece whatever the page size, and one bulk copy brings
// them.  A code is stored as code + 8 (1..15).  The order of the codes is the register order of the tensor-core operand
// each matrix is read as, with c = lane & 3 and g = lane >> 2 of the reading warp:
//   K: 32-bit word w of chunk c of a token's row holds channels 32 w + 8 c + 2 i (nibble i) and + 1 (nibble i + 4),
//      i < 4: (word >> 4 i) & 0x000F000F is a pair of neighbouring channels, the k index of a row operand.
//   V: 16-bit word w of chunk g of a token's row holds channels 32 w + 4 g + n (nibble n): the rows of a transposed row
//      operand whose k index is the token, so a register joins two tokens' words.  The chunks of neighbouring rows are
//      spread over the banks by q4_v_chunk().
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "pkv.h"

namespace pkv {

constexpr int kQ4Tile = 16;            // tokens per tile
constexpr int kQ4StatusWords = 8;      // [0] waits that ran out, [1] page numbers out of range, [2] lengths or offsets out of range

struct Q4Geometry {
    int n_kv_heads, n_q_heads, group;  // group = H_q / H_kv
    int head_dim, page, page_shift;    // P = 1 << page_shift
    int groups;                        // d / g: scales per row
    int tile_bytes, head_bytes;        // head_bytes = P / 16 * tile_bytes
    int fp16;                          // 0: bf16 rows and queries, 1: fp16
    long long page_bytes, n_pages;
    float scale_log2e;
    int n_ctas, n_sms;
};

// Rows of a call (append, read, queries): sequence s owns rows [offsets[s], offsets[s + 1]) (offsets NULL: n_rows /
// n_seqs each), which are its last positions.
struct Q4Rows {
    const int *table, *lengths, *offsets;
    int n_seqs, max_pages, per_seq;
    long long n_rows;
};

struct Q4CopyArgs {
    Q4Geometry geo;
    Q4Rows rows;
    unsigned char *pool;
    void *k, *v;                       // read by append, written by read
    long long k_row, k_head, v_row, v_head;      // strides in elements
    int *status;
    int chained;                       // set by the launcher: the next kernel may be set up early (see q4_chained)
    int rows_per_cta;                  // ... rows of a CTA, with 1 / n_kv_heads
    float inv_heads;
};

struct Q4AttentionArgs {
    Q4Geometry geo;
    Q4Rows rows;
    const unsigned char *pool;
    const void *q;
    void *out;
    float *state;                      // NULL, or rows of d + 2 floats (o, m, l) instead of out
    long long q_row, q_head, out_row, out_head;
    int max_q_len;                     // no sequence has more rows than this
    int max_len;                       // hint: lengths are expected up to this
    int whole;                         // set by the launcher: no segment is cut
    int chained;                       // ... the kernel that follows the call's last may be set up early (see q4_chained)
    int join;                          // ... the call's second kernel follows
    unsigned char *workspace;
    int *status;
};

// Calls of this cache are launched so that one may be set up while the kernel before it on the stream finishes
// (programmatic stream serialization): each waits for that kernel before it touches memory, and only then lets the next one
// start.  That orders a chain of kernels as long as all of them wait.  Decode launches with decode_overlap = 2 do not: one of
// them between two kernels of this cache would hide the first from the second.  Once a process has such a cache, kernels
// here are launched the ordinary way (1 to 2 us per call), but for the one that joins the states of its own call.
extern std::atomic<bool> unordered_decodes;
inline bool q4_chained() { return !unordered_decodes; }

cudaError_t launch_q4_append(const Q4CopyArgs &a, cudaStream_t st);
cudaError_t launch_q4_read(const Q4CopyArgs &a, cudaStream_t st);
cudaError_t launch_q4_attention(Q4AttentionArgs a, cudaStream_t st);
cudaError_t q4_attention_setup();      // raises dynamic shared-memory limits, once per cache
// the row-block kernel (pkv_q4_block.cu); n: CTAs, from q4_block_grid
constexpr int kQ4BlockRows = 256;
cudaError_t q4_block_setup();
int q4_block_grid(const Q4Geometry &g, int n_seqs, int max_q_len, int max_len);
long long q4_block_workspace(const Q4Geometry &g, int n_seqs, int max_q_len, int max_len);
cudaError_t launch_q4_block(const Q4AttentionArgs &a, int n, cudaStream_t st);
long long q4_attention_workspace(const Q4Geometry &g, int n_seqs, int max_q_len, int max_len);

// byte offsets inside a tile
__host__ __device__ constexpr int q4_v_base(int d) { return kQ4Tile * d / 2; }
__host__ __device__ constexpr int q4_ks_base(int d) { return kQ4Tile * d; }
__host__ __device__ constexpr int q4_vs_base(int d, int groups) { return kQ4Tile * d + kQ4Tile * groups * 2; }
// K: a row is d/2 bytes, chunk c = d/8 bytes of it
__host__ __device__ constexpr int q4_k_chunk(int d, int t, int c) { return t * (d / 2) + c * (d / 8); }
// V: chunk g = d/16 bytes (8 or 4).  A warp reads chunk g of tokens 2c (then 2c + 1, ...) in one load: within each 128-byte
// line the chunks are XORed so that the lanes that are served together hit different banks.
__host__ __device__ constexpr int q4_v_chunk(int d, int t, int g) {
    if (d == 128) {                    // a line is two tokens of eight 8-byte chunks
        const int line = t >> 1, slot = ((t & 1) << 3 | g) ^ ((line & 1) << 2 | ((line >> 1) & 1) << 3);
        return line * 128 + slot * 8;
    }
    const int line = t >> 2, slot = ((t & 3) << 3 | g) ^ ((line & 1) << 3);      // four tokens of eight 4-byte chunks
    return line * 128 + slot * 4;
}

#ifdef __CUDACC__
// The rows of a call as the kernels see them: offsets are held inside [0, n_rows], so no row outside the buffers is ever
// touched whatever the arrays say.
__device__ __forceinline__ int q4_first_row(const Q4Rows &r, int s) {
    if (!r.offsets) return s * r.per_seq;
    return min(max(__ldg(r.offsets + s), 0), (int)r.n_rows);
}
__device__ __forceinline__ int q4_length(const Q4Rows &r, const Q4Geometry &g, int s, int *status) {
    const int T = __ldg(r.lengths + s), most = r.max_pages << g.page_shift;
    if (T < 0 || T > most) {
        if (status) atomicAdd(status + 2, 1);
        return T < 0 ? 0 : most;
    }
    return T;
}
#endif

}  // namespace pkv
