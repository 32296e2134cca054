// Around the attention of the paged 4-bit cache, what a serving step needs on the device: masks of drafted trees, keeping the
// rows that were accepted, planning a step's pages.
#include <type_traits>

#include "pkv_q4_device.cuh"

namespace pkv {

namespace {

// A launch that may be set up while the kernel before it finishes; each kernel here waits before it touches memory.
template <typename Args>
cudaError_t launch_chained(void (*kernel)(Args), const Args &a, dim3 grid, int threads, cudaStream_t st, int cluster = 1) {
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = cluster;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.stream = st;
    cfg.attrs = cluster > 1 ? at : at + 1;
    cfg.numAttrs = (cluster > 1) + a.chained;
    return cudaLaunchKernelEx(&cfg, kernel, a);
}

// ---- masks of drafted trees ---------------------------------------------------------------------------------------------
// A thread per row walks up its branch: once for the depth, which says where the window ends, once for the bits.  Ancestors
// have smaller numbers, so a word is finished when the walk leaves it.  A CTA's rows belong to one sequence; its parents up to
// kTreeHeld lie in shared memory, since the walk is a chain of loads.  (A few KB in and out: latency and the launch; 7 rows 1.6 us, 16 x 25 with
// a window 3.1 us in a row of them.)
constexpr int kTreeThreads = 128, kTreeHeld = 2048;

__global__ void __launch_bounds__(kTreeThreads) q4_tree_kernel(const __grid_constant__ Q4TreeArgs a) {
    __shared__ int held[kTreeHeld];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (a.chained) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int s = blockIdx.x, first = q4_first_row(a.rows, s), all = q4_first_row(a.rows, s + 1) - first;
    const int n = max(0, min(all, a.max_q_len)), j0 = blockIdx.y * kTreeThreads;
    if (threadIdx.x == 0 && blockIdx.y == 0 && all > a.max_q_len) atomicAdd(a.status + 2, 1);
    if (j0 >= n) return;
    const int here = min(n, j0 + kTreeThreads);
    for (int i = threadIdx.x; i < min(here, kTreeHeld); i += kTreeThreads) {
        int p = __ldg(a.parents + first + i);
        if (p < -1 || p >= i) {                 // (counted once, by the CTA that has the row)
            if (i >= j0) atomicAdd(a.status + 2, 1);
            p = -1;
        }
        held[i] = p;
    }
    __syncthreads();
    const int j = j0 + threadIdx.x;
    if (j >= n) return;
    auto parent = [&](int i) -> int {
        if (i < kTreeHeld) return held[i];
        const int p = __ldg(a.parents + first + i);
        return p < -1 || p >= i ? -1 : p;
    };
    if (j >= kTreeHeld) {
        const int p = __ldg(a.parents + first + j);
        if (p < -1 || p >= j) atomicAdd(a.status + 2, 1);
    }
    int depth = 0;
    for (int i = parent(j); i >= 0; i = parent(i)) ++depth;
    // ancestors at depths below `low` (in the sinks) or above `high` (in the window) are seen
    const int C = a.rows.lengths ? max(0, __ldg(a.rows.lengths + s)) - all : 0;
    const int low = a.rows.lengths ? a.sinks - C : 0, high = a.window ? depth - a.window : -1;
    unsigned long long *out = a.tree + (long long)(first + j) * a.words, bits = 0;
    int word = a.words - 1, e = depth;
    for (int i = j; i >= 0; i = parent(i), --e) {
        for (; word > i >> 6; --word) { out[word] = bits; bits = 0; }
        if (e > high || e < low) bits |= 1ull << (i & 63);
    }
    for (; word >= 0; --word) { out[word] = bits; bits = 0; }
    if (a.depths) a.depths[first + j] = depth;
}

// ---- accepted rows --------------------------------------------------------------------------------------------------------
// A CTA moves the rows of one sequence and KV head, eight lanes a row: K codes and V's chunks (which lie differently in every
// row of a tile), then the scales.  Row i comes from row path[i] >= i, so 128 rows at a time are read, then written: what a
// later 128 reads was not written before.  (Bound by latency: a trip for the path, one for the pages, one for the rows; 8 x 64 drafted rows, about half
// of them kept, with their append and reading back 8.2 us, of which this is a third.)
constexpr int kKeepThreads = 256, kKeepUnroll = 4, kKeepSlots = kKeepThreads / 8;

template <int D, int NG>
__global__ void __launch_bounds__(kKeepThreads) q4_keep_kernel(const __grid_constant__ Q4KeepArgs a) {
    using Piece = typename std::conditional<D == 128, uint2, uint32_t>::type;      // an eighth of a row's codes
    using Scales = typename std::conditional<NG == 4, uint2, typename std::conditional<NG == 2, uint32_t, unsigned short>::type>::type;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (a.chained) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const Q4Geometry &geo = a.geo;
    const int s = blockIdx.x, head = blockIdx.y, l = threadIdx.x & 7, slot = threadIdx.x >> 3;
    int *status = head == 0 && l == 0 ? a.status : nullptr;
    const int first = q4_first_row(a.rows, s), n = max(0, q4_first_row(a.rows, s + 1) - first);
    const int T = q4_length(a.rows, geo, s, threadIdx.x == 0 ? status : nullptr), C = T - n;
    const int count = max(0, min(min(__ldg(a.counts + s), n), a.max_path));
    if (threadIdx.x == 0 && head == 0) {
        if (count != __ldg(a.counts + s) || C < 0) atomicAdd(a.status + 2, 1);
        a.lengths_out[s] = max(0, C + count);
    }
    // the tile of a position (head `head`) and the token in it; NULL: there is none
    auto tile_of = [&](int pos, int &t) -> unsigned char * {
        t = pos & (kQ4Tile - 1);
        if (pos < 0 || pos >= T) return nullptr;
        const int page = __ldg(a.rows.table + (long long)s * a.rows.max_pages + (pos >> geo.page_shift));
        if (page < 0 || page >= geo.n_pages) {
            if (status) atomicAdd(status + 1, 1);
            return nullptr;
        }
        return a.pool + page * geo.page_bytes + (long long)head * geo.head_bytes + (pos & (geo.page - 1)) / kQ4Tile * geo.tile_bytes;
    };
    for (int base = 0; base < count; base += kKeepSlots * kKeepUnroll) {
        Piece k[kKeepUnroll], v[kKeepUnroll];
        Scales sc[kKeepUnroll];
        unsigned char *to[kKeepUnroll];
        int to_t[kKeepUnroll];
#pragma unroll
        for (int u = 0; u < kKeepUnroll; ++u) {
            const int i = base + u * kKeepSlots + slot;
            to[u] = nullptr;
            if (i >= count) continue;
            const int p = __ldg(a.paths + (long long)s * a.max_path + i);
            if (p < i || p >= n) {
                if (status) atomicAdd(status + 2, 1);
                continue;
            }
            if (p == i) continue;
            int t;
            const unsigned char *from = tile_of(C + p, t);
            unsigned char *dst = tile_of(C + i, to_t[u]);
            if (!from || !dst) continue;
            to[u] = dst;
            k[u] = *reinterpret_cast<const Piece *>(from + t * (D / 2) + l * (D / 16));
            v[u] = *reinterpret_cast<const Piece *>(from + q4_v_base(D) + q4_v_chunk(D, t, l));
            if (l < 2) sc[u] = *reinterpret_cast<const Scales *>(from + (l ? q4_vs_base(D, NG) : q4_ks_base(D)) + t * NG * 2);
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kKeepUnroll; ++u) {
            if (!to[u]) continue;
            const int t = to_t[u];
            *reinterpret_cast<Piece *>(to[u] + t * (D / 2) + l * (D / 16)) = k[u];
            *reinterpret_cast<Piece *>(to[u] + q4_v_base(D) + q4_v_chunk(D, t, l)) = v[u];
            if (l < 2) *reinterpret_cast<Scales *>(to[u] + (l ? q4_vs_base(D, NG) : q4_ks_base(D)) + t * NG * 2) = sc[u];
        }
        __syncthreads();
    }
}

// ---- planning a step ------------------------------------------------------------------------------------------------------
// Prefix sums over the requests - new rows, pages taken, pages given back - from which every row, taken page and returned page follows
// by itself: a thread each, which finds its request by bisection in the sums.  Up to kPlanHeld requests the sums fit shared memory,
// and up to kPlanFew rows (of the caller's bound) a CTA, or a cluster of eight that all work them out, fills everything in (64 requests: 4.6 us, all latency: launch, counters and lengths, the scan,
// pages, results; 700 requests with chunks of prompts 7.5 us, and one kernel for the sums and one for the rest 10.6 and a launch more).  More requests
// or rows leave the sums in the workspace to a second kernel over the SMs.  The launch goes by requests and rows, which is what most steps are
// made of; pages that go back are the threads' work too, but the host does not know their number, so a step in which many long requests are done takes longer
// (64 of 32K on pages of 16, 131072 pages: 85.6 us by one CTA, 14.5 where the bound of the rows brings the cluster; 777 of 11000, 534576 pages: 445).  Entries that are read (below `end`) and written (from it on), and
// places of the ring that are read (from the head) and written (from the tail), are different ones, so the order does not matter.
constexpr int kPlanThreads = 1024, kPlanFillThreads = 256, kPlanCluster = 8;
constexpr int kPlanHeld = 1024;                  // a thread each
constexpr long long kPlanAlone = 2048, kPlanFew = 65536;      // rows that one CTA, a cluster see to

struct PlanRequest { int T, end, a, b; };        // length and end before the step; entries [0, a) and from b on go back
struct PlanHead { long long head, tail; int rows, taken, back, ok; };
// (sums: [n_seqs + 1] each of rows, pages taken, pages given back)
struct PlanSums { int *rows, *taken, *back; PlanRequest *req; PlanHead *head; };

struct PlanNeed { int rows, taken, back, bad, T, n, first, end, first_out, end_out, a, b; };

__device__ __forceinline__ PlanNeed plan_need(const Q4PlanArgs &p, int s) {
    PlanNeed q{};
    q.T = p.lengths[s];
    q.n = p.rows[s];
    q.first = p.spans[2 * s];
    q.end = p.spans[2 * s + 1];
    const int most = p.max_pages << p.page_shift, P = 1 << p.page_shift;
    if (q.n < -1 || q.T < 0 || q.T > most || q.n > most - q.T || q.first < 0 || q.first > q.end || q.end > p.max_pages) {
        q.bad = 1;
        return q;
    }
    const int held = min(max(q.first, p.sink_pages), q.end);      // behind the sinks' pages, the first entry that is held
    if (q.n < 0) {
        q.a = min(p.sink_pages, q.end);
        q.b = held;
        q.back = q.a + q.end - held;
        return q;
    }
    q.rows = q.n;
    const int pages = (int)(((long long)q.T + q.n + P - 1) >> p.page_shift);
    q.end_out = max(q.end, pages);
    q.taken = q.end_out - q.end;
    q.first_out = q.first;
    q.b = held;
    if (p.window > 0) {
        const int to = min(max(0, q.T + 1 - p.window) >> p.page_shift, q.end);
        if (to > held) {
            q.back = to - held;
            q.first_out = to;
        }
    }
    return q;
}

// the last of n + 1 ascending sums that is not above i, among the first n
__device__ __forceinline__ int plan_find(const int *sums, int n, int i) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (sums[mid] <= i) lo = mid;
        else hi = mid;
    }
    return lo;
}

// rows, taken and returned pages number me, me + many, ...
__device__ __forceinline__ void plan_fill(const Q4PlanArgs &p, const PlanSums &z, const PlanHead &h, int me, int many) {
    const long long n = p.n_pages;
    const long long head = h.head % n, tail = h.tail % n;
    auto free_page = [&](int k) -> int {
        const long long at = head + k;
        return p.ring[at >= n ? at - n : at];
    };
    const int rows = p.positions || p.slots ? h.rows : 0;
    for (long long i0 = me; i0 < (long long)rows + h.taken + h.back; i0 += many) {
        if (i0 < rows) {
            const int i = (int)i0, s = plan_find(z.rows, p.n_seqs, i);
            const PlanRequest r = z.req[s];
            const int pos = r.T + i - z.rows[s], e = pos >> p.page_shift;
            if (p.positions) p.positions[i] = pos;
            if (p.slots) {
                const int page = e < r.end ? p.table[(long long)s * p.max_pages + e] : free_page(z.taken[s] + e - r.end);
                p.slots[i] = page < 0 || page >= n ? -1LL : ((long long)page << p.page_shift) + (pos & ((1 << p.page_shift) - 1));
            }
        } else if (i0 < (long long)rows + h.taken) {
            const int k = (int)(i0 - rows), s = plan_find(z.taken, p.n_seqs, k);
            p.table[(long long)s * p.max_pages + z.req[s].end + k - z.taken[s]] = free_page(k);
        } else {
            const int k = (int)(i0 - rows - h.taken), s = plan_find(z.back, p.n_seqs, k), x = k - z.back[s];
            const PlanRequest r = z.req[s];
            const long long at = tail + k;
            p.ring[at >= n ? at - n : at] = p.table[(long long)s * p.max_pages + (x < r.a ? x : r.b + x - r.a)];
        }
    }
}

__host__ __device__ inline PlanSums plan_sums(unsigned char *w, int n_seqs) {
    PlanSums z;
    z.head = reinterpret_cast<PlanHead *>(w);
    z.req = reinterpret_cast<PlanRequest *>(w + 64);
    z.rows = reinterpret_cast<int *>(z.req + n_seqs);
    z.taken = z.rows + n_seqs + 1;
    z.back = z.taken + n_seqs + 1;
    return z;
}
constexpr int kPlanBytes = 64 + kPlanHeld * (int)sizeof(PlanRequest) + 3 * (kPlanHeld + 1) * 4;
static_assert(sizeof(PlanHead) <= 64 && kPlanBytes <= 48 * 1024, "fits shared memory");

// kAll: the sums stay in shared memory and the same CTA, or its cluster, fills in everything.  Outputs may be inputs: the cluster's first CTA
// writes them once all CTAs have read.
template <bool kAll>
__global__ void __launch_bounds__(kPlanThreads) q4_plan_kernel(const __grid_constant__ Q4PlanArgs p) {
    __shared__ __align__(16) unsigned char here[kAll ? kPlanBytes : 16];
    __shared__ long long warps[3][32];
    __shared__ int bad_warps[32];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (p.chained || !kAll) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const PlanSums z = plan_sums(kAll ? here : p.workspace, p.n_seqs);
    const bool shared = kAll && gridDim.x > 1, writes = !kAll || blockIdx.x == 0;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const long long head = p.counters[0], tail = p.counters[1];
    // this thread's requests: neighbours
    const int per = (p.n_seqs + kPlanThreads - 1) / kPlanThreads, s0 = min(tid * per, p.n_seqs), s1 = min(s0 + per, p.n_seqs);
    long long mine[3] = {0, 0, 0};
    int bad = 0;
    PlanNeed q{};
    for (int s = s0; s < s1; ++s) {
        q = plan_need(p, s);
        mine[0] += q.rows;
        mine[1] += q.taken;
        mine[2] += q.back;
        bad += q.bad;
    }
    long long x[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        x[i] = mine[i];
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, x[i], d);
            if (lane >= d) x[i] += y;
        }
        if (lane == 31) warps[i][warp] = x[i];
    }
    bad = __reduce_add_sync(0xffffffffu, bad);
    if (lane == 0) bad_warps[warp] = bad;
    __syncthreads();
    long long total[3], before[3];
    bad = 0;
    {
        // every warp adds the warps' sums up by itself, a lane each
        long long w[3];
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            w[i] = warps[i][lane];
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const long long y = __shfl_up_sync(0xffffffffu, w[i], d);
                if (lane >= d) w[i] += y;
            }
            total[i] = __shfl_sync(0xffffffffu, w[i], 31);
            const long long up = __shfl_sync(0xffffffffu, w[i], max(warp - 1, 0));
            before[i] = (warp ? up : 0) + x[i] - mine[i];
        }
        bad = __reduce_add_sync(0xffffffffu, bad_warps[lane]);
    }
    const bool ring_ok = head >= 0 && tail >= head && tail - head <= p.n_pages && total[2] <= p.n_pages - (tail - head);
    const int refused = bad + (total[0] > p.n_rows) + !ring_ok;
    const long long missing = ring_ok ? max(0LL, total[1] - (tail - head)) : 0;
    const bool ok = refused == 0 && missing == 0;
    if (shared) {
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
    for (int s = s0; s < s1; ++s) {
        if (per > 1) q = plan_need(p, s);        // (its inputs are this thread's own: it has not written them yet)
        const int rows = (int)before[0];
        if (writes) p.offsets[s] = ok ? rows : 0;
        if (ok) {
            z.rows[s] = rows;
            z.taken[s] = (int)before[1];
            z.back[s] = (int)before[2];
            z.req[s] = PlanRequest{q.T, q.end, q.a, q.b};
            before[0] += q.rows;
            before[1] += q.taken;
            before[2] += q.back;
        }
        if (!writes) continue;
        p.lengths_out[s] = !ok ? q.T : q.n < 0 ? 0 : q.T + q.n;
        p.spans_out[2 * s] = !ok ? q.first : q.first_out;
        p.spans_out[2 * s + 1] = !ok ? q.end : q.end_out;
    }
    const PlanHead h{head, tail, ok ? (int)total[0] : 0, ok ? (int)total[1] : 0, ok ? (int)total[2] : 0, ok};
    if (tid == 0) {
        if (writes) p.offsets[p.n_seqs] = h.rows;
        if (ok) {
            z.rows[p.n_seqs] = h.rows;
            z.taken[p.n_seqs] = h.taken;
            z.back[p.n_seqs] = h.back;
        }
        if (!kAll) *z.head = h;
        if (writes) {
            p.counters_out[0] = head + h.taken;
            p.counters_out[1] = tail + h.back;
            p.counters_out[2] = missing;
            p.counters_out[3] = refused;
        }
    }
    if (!kAll) return;
    __syncthreads();
    plan_fill(p, z, h, (int)blockIdx.x * kPlanThreads + tid, (int)gridDim.x * kPlanThreads);
}

__global__ void __launch_bounds__(kPlanFillThreads) q4_plan_fill_kernel(const __grid_constant__ Q4PlanArgs p) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (p.chained) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const PlanSums z = plan_sums(p.workspace, p.n_seqs);
    plan_fill(p, z, *z.head, (int)(blockIdx.x * kPlanFillThreads + threadIdx.x), (int)(gridDim.x * kPlanFillThreads));
}

bool plan_at_once(int n_seqs, long long n_rows) { return n_seqs <= kPlanHeld && n_rows <= kPlanFew; }

}  // namespace

// Loads the kernels of a cache's format: a first call may be captured.
cudaError_t q4_serve_setup(const Q4Geometry &g) {
    cudaFuncAttributes known;
    cudaError_t e;
    if ((e = cudaFuncGetAttributes(&known, q4_tree_kernel)) != cudaSuccess || (e = cudaFuncGetAttributes(&known, q4_plan_kernel<true>)) != cudaSuccess ||
        (e = cudaFuncGetAttributes(&known, q4_plan_kernel<false>)) != cudaSuccess || (e = cudaFuncGetAttributes(&known, q4_plan_fill_kernel)) != cudaSuccess)
        return e;
#define PKV_Q4_LOAD(D, NG) \
    if (g.head_dim == D && g.groups == NG) return cudaFuncGetAttributes(&known, q4_keep_kernel<D, NG>);
    PKV_Q4_LOAD(128, 4) PKV_Q4_LOAD(128, 2) PKV_Q4_LOAD(128, 1) PKV_Q4_LOAD(64, 2) PKV_Q4_LOAD(64, 1)
#undef PKV_Q4_LOAD
    return cudaErrorInvalidValue;
}

cudaError_t launch_q4_tree_masks(Q4TreeArgs a, cudaStream_t st) {
    a.chained = q4_chained();
    return launch_chained(q4_tree_kernel, a, dim3(a.rows.n_seqs, (a.max_q_len + kTreeThreads - 1) / kTreeThreads), kTreeThreads, st);
}

cudaError_t launch_q4_keep(Q4KeepArgs a, cudaStream_t st) {
    const Q4Geometry &g = a.geo;
    a.chained = q4_chained();
    const dim3 grid(a.rows.n_seqs, g.n_kv_heads);
#define PKV_Q4_KEEP(D, NG) \
    if (g.head_dim == D && g.groups == NG) return launch_chained(q4_keep_kernel<D, NG>, a, grid, kKeepThreads, st);
    PKV_Q4_KEEP(128, 4) PKV_Q4_KEEP(128, 2) PKV_Q4_KEEP(128, 1) PKV_Q4_KEEP(64, 2) PKV_Q4_KEEP(64, 1)
#undef PKV_Q4_KEEP
    return cudaErrorInvalidValue;
}

long long q4_plan_workspace(int n_seqs, long long n_rows) {
    return plan_at_once(n_seqs, n_rows) ? 0 : 64 + (long long)n_seqs * (int)sizeof(PlanRequest) + 3LL * (n_seqs + 1) * 4;
}

cudaError_t launch_q4_plan(Q4PlanArgs a, cudaStream_t st) {
    a.chained = q4_chained();
    if (plan_at_once(a.n_seqs, a.n_rows)) {
        const int n = a.n_rows <= kPlanAlone ? 1 : kPlanCluster;
        return launch_chained(q4_plan_kernel<true>, a, dim3(n), kPlanThreads, st, n);
    }
    cudaError_t e = launch_chained(q4_plan_kernel<false>, a, dim3(1), kPlanThreads, st);
    if (e != cudaSuccess) return e;
    const long long jobs = a.n_rows + a.n_seqs;
    const int grid = (int)(jobs / kPlanFillThreads + 1 < 592 ? jobs / kPlanFillThreads + 1 : 592);
    return launch_chained(q4_plan_fill_kernel, a, dim3(grid), kPlanFillThreads, st);
}

}  // namespace pkv
