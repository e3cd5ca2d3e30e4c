// Eviction from a paged cache by accumulated attention weight.
//
// Of the L rows of a (sequence, KV head), min(L, budget) are kept: the first
// `sinks`, the last `recent`, and of those between the budget - sinks - recent
// with the largest weight (ties: the lower slot; NaN below everything).  The kept
// rows go in order to the pages of a second table, so rows stay in the order of
// their positions.
//
// Bound by the kept rows' bytes, read once and written once: the selection reads 4
// bytes a row and KV head, the copy moves 8 D in bf16.  Two kernels, since the copy
// wants every SM whatever the number of (sequence, KV head) pairs.  Measured: 16
// sequences of 3900 to 4351 rows and 8 KV heads cut to 4096, 87 us (6.2 TB/s; 79.5 at
// the rate of a plain copy); one of 65537 rows cut to 4096, 23 us, of which 15 are the
// selection's chain of loads, four passes and cluster barriers.
#include "paged.cuh"

namespace prism {
namespace {

constexpr int kEvBatch = 4;              // rows a thread has in flight
constexpr uint32_t kNan = 0x7FFFFFFFu;
constexpr int kEvCached = 48 * 1024;     // rows whose keys shared memory holds

// Weight as an unsigned key with the same order: NaN 0, then -inf ... +inf; -0 as +0.
__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return 0u;
    const uint32_t u = __float_as_uint(w + 0.f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// One cluster of cs CTAs per (sequence, KV head), each with a contiguous share of
// the rows: radix selection of the smallest kept key, eight bits a pass over the
// keys in shared memory (read from the pool again where a share is more than it
// holds), the shares' histograms added into every CTA's through distributed shared
// memory; then the kept slots in order.  Shared-memory additions of one to the same
// counter by many lanes are cheap: counting lanes of equal digit first took longer
// (selection of 65537 rows 29 against 22 us).
template <int kEvThreads>
__global__ void __launch_bounds__(kEvThreads) evict_select_kernel(EvictArgs a, int cs, int cached) {
    constexpr int kEvWarps = kEvThreads / 32;
    extern __shared__ uint32_t keys[];
    __shared__ __align__(16) int hist[4][256], total[4][256];   // this share's counts of each pass; the cluster's
    __shared__ int warp_eq[kEvWarps], warp_gt[kEvWarps], share_eq[8], share_gt[8], pick[2];
    pdl_wait();
    pdl_trigger();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int row = blockIdx.x / cs, rank = blockIdx.x % cs;
    const int b = row / a.Hkv, h = row % a.Hkv;
    const int len = paged_len(a.src, b, 0, a.err);
    int32_t *kept = a.kept + (long long)row * a.budget;
    if (len <= a.budget) {               // the same for the whole cluster
        for (int j = rank * kEvThreads + tid; j < a.budget; j += cs * kEvThreads) kept[j] = j < len ? j : -1;
        return;
    }
    const int first = a.sinks, want = a.budget - a.recent - first;
    const int n = want > 0 ? len - a.recent - first : 0;   // rows to choose from, more than want (none to choose: 0)
    const int share = ((n + cs - 1) / cs + 31) & ~31, s0 = min(n, rank * share), m = min(n, s0 + share) - s0;
    const int32_t *table = a.src.table + (long long)b * a.src.table_pages;
    // Keys of kEvBatch rows of this share, kEvThreads apart: their table entries
    // together, then their weights together.
    auto load = [&](int i, uint32_t (&k)[kEvBatch]) {
        int page[kEvBatch], off[kEvBatch];
#pragma unroll
        for (int u = 0; u < kEvBatch; ++u) {
            const int slot = first + s0 + i + u * kEvThreads, idx = slot / a.src.page_size;
            off[u] = slot - idx * a.src.page_size;
            page[u] = i + u * kEvThreads < m ? table[idx] : -1;
        }
#pragma unroll
        for (int u = 0; u < kEvBatch; ++u)                 // a bad entry is reported by the copy if its row is kept
            k[u] = (unsigned)page[u] < (unsigned)a.src.n_pages
                       ? __float_as_uint(a.src.weights[((long long)page[u] * a.Hkv + h) * a.src.page_size + off[u]])
                       : kNan;
#pragma unroll
        for (int u = 0; u < kEvBatch; ++u) k[u] = weight_key(__uint_as_float(k[u]));
    };
    const bool held = share <= cached;
    // f(key) for every row of this share
    auto each = [&](auto f) {
        for (int i0 = 0; i0 < m; i0 += kEvBatch * kEvThreads) {
            uint32_t k[kEvBatch];
            if (!held) load(i0 + tid, k);
#pragma unroll
            for (int u = 0; u < kEvBatch; ++u) {
                const int i = i0 + u * kEvThreads + tid;
                if (i < m) f(held ? keys[i] : k[u]);
            }
        }
    };
    if (held)
        for (int i0 = tid; i0 < m; i0 += kEvBatch * kEvThreads) {
            uint32_t k[kEvBatch];
            load(i0, k);
#pragma unroll
            for (int u = 0; u < kEvBatch; ++u)
                if (i0 + u * kEvThreads < m) keys[i0 + u * kEvThreads] = k[u];
        }
    for (int i = tid; i < 4 * 256; i += kEvThreads) hist[i >> 8][i & 255] = total[i >> 8][i & 255] = 0;
    cluster_sync_all();                  // every CTA's counts are clear before another adds to them
    uint32_t prefix = 0, mask = 0;
    int need = want;                     // rows still to be taken of those that match the prefix
    if (n > 0) {
#pragma unroll 1
        for (int pass = 0; pass < 4; ++pass) {
            const int shift = 24 - 8 * pass;
            each([&](uint32_t k) {
                if ((k & mask) == prefix) atomicAdd(&hist[pass][(k >> shift) & 255u], 1);
            });
            __syncthreads();
            if (cs > 1) {
                const int c = tid < 256 ? hist[pass][tid] : 0;
                if (c)
                    for (int r = 0; r < cs; ++r) dsmem_add(&total[pass][tid], r, c);
                cluster_sync_all();
            }
            if (warp == 0) {             // the bin of the need-th largest; lane's bins are 255 - 8 lane and the seven below
                const int *t = (cs > 1 ? total : hist)[pass] + 248 - 8 * lane;
                const int4 hi = *(const int4 *)(t + 4), lo = *(const int4 *)t;
                const int c[8] = {hi.w, hi.z, hi.y, hi.x, lo.w, lo.z, lo.y, lo.x};
                const int s = hi.w + hi.z + hi.y + hi.x + lo.w + lo.z + lo.y + lo.x;
                int up = s;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int t = __shfl_up_sync(0xFFFFFFFFu, up, o);
                    if (lane >= o) up += t;
                }
                int above = up - s;
                if (above < need && need <= up) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        if (above < need && need <= above + c[e]) {
                            pick[0] = 255 - (8 * lane + e);
                            pick[1] = above;
                        }
                        above += c[e];
                    }
                }
            }
            __syncthreads();
            prefix |= (uint32_t)pick[0] << shift;
            need -= pick[1];
            mask |= 255u << shift;
        }
    }
    // the prefix is now that key: larger keys are kept, and the first `need` equal ones
    const int per = ((m + kEvWarps - 1) / kEvWarps + 31) & ~31, lo = min(m, warp * per), hi = min(m, lo + per);
    auto key = [&](int i) {
        if (held) return keys[i];
        const int slot = first + s0 + i, idx = slot / a.src.page_size, page = table[idx];
        if ((unsigned)page >= (unsigned)a.src.n_pages) return weight_key(__uint_as_float(kNan));
        return weight_key(a.src.weights[((long long)page * a.Hkv + h) * a.src.page_size + slot - idx * a.src.page_size]);
    };
    int gt = 0, eq = 0;
    for (int i = lo + lane; i < hi; i += 32) {
        const uint32_t k = key(i);
        gt += k > prefix;
        eq += k == prefix;
    }
    gt = __reduce_add_sync(0xFFFFFFFFu, gt);
    eq = __reduce_add_sync(0xFFFFFFFFu, eq);
    if (lane == 0) warp_gt[warp] = gt, warp_eq[warp] = eq;
    __syncthreads();
    if (warp == 0) {
        const int g = __reduce_add_sync(0xFFFFFFFFu, lane < kEvWarps ? warp_gt[lane] : 0);
        const int e = __reduce_add_sync(0xFFFFFFFFu, lane < kEvWarps ? warp_eq[lane] : 0);
        if (lane < cs) dsmem_st(&share_gt[rank], lane, g), dsmem_st(&share_eq[rank], lane, e);
    }
    static_assert(kEvWarps <= 32, "a lane per warp");
    cluster_sync_all();
    gt = eq = 0;
    for (int r = 0; r < rank; ++r) gt += share_gt[r], eq += share_eq[r];
    for (int w = 0; w < warp; ++w) gt += warp_gt[w], eq += warp_eq[w];
    for (int i0 = lo; i0 < hi; i0 += 32) {
        const int i = i0 + lane;
        const uint32_t k = i < hi ? key(i) : 0u;
        const bool is_gt = i < hi && k > prefix, is_eq = i < hi && k == prefix;
        const uint32_t bg = __ballot_sync(0xFFFFFFFFu, is_gt), be = __ballot_sync(0xFFFFFFFFu, is_eq), below = (1u << lane) - 1u;
        const int rank_eq = eq + __popc(be & below);
        if (is_gt || (is_eq && rank_eq < need)) kept[first + gt + __popc(bg & below) + min(rank_eq, need)] = first + s0 + i;
        gt += __popc(bg);
        eq += __popc(be);
    }
    for (int j = rank * kEvThreads + tid; j < first; j += cs * kEvThreads) kept[j] = j;
    for (int j = rank * kEvThreads + tid; j < a.recent; j += cs * kEvThreads) kept[first + want + j] = len - a.recent + j;
}

__device__ __forceinline__ int ticket_release(int *counter) {
    int n;
    asm volatile("atom.add.release.gpu.global.s32 %0, [%1], 1;" : "=r"(n) : "l"(counter) : "memory");
    return n;
}

// Copies the kept rows of K, V and the weights, kCpRows destination rows of one KV
// head per warp: a lane each looks the rows up, then the warp moves them 512 bytes
// at a time.  Rows that are kept whatever their weights (all of a sequence within
// its budget, the sinks, the recent ones) do not wait for the selection: the copy
// starts beside it, the last rows first.  Also sets the destination's lengths.
constexpr int kCpThreads = 128;
constexpr int kCpRows = 8;
constexpr int kCpUnroll = 4;
__global__ void __launch_bounds__(kCpThreads) evict_copy_kernel(EvictArgs a, int row_bytes) {
    // Before the wait: the selection lets this kernel start once its own wait is over,
    // so all but `kept` is final.
    pdl_trigger();
    const int lane = threadIdx.x & 31;
    const long long gid = (long long)blockIdx.x * kCpThreads + threadIdx.x;
    const int chunks = (a.budget + kCpRows - 1) / kCpRows, heads = a.B * a.Hkv;
    const long long w = gid >> 5;
    const int chunk = chunks - 1 - (int)(w / heads), bh = (int)(w % heads);
    const bool work = chunk >= 0;
    const int b = bh / a.Hkv, h = bh - b * a.Hkv, j0 = chunk * kCpRows, j = j0 + lane;
    const int len = paged_len(a.src, b, 0, nullptr);
    // The last CTA to come here sets the lengths at its end: dst's may be src's, which
    // every warp has read by then.  The release orders those reads, the CTA's by the
    // barrier, before its ticket; the fence at the end the tickets before the lengths.
    __syncthreads();
    bool last = false;
    if (threadIdx.x == 0) last = ticket_release(a.counter) == (int)gridDim.x - 1;
    const bool early = len <= a.budget || j0 + kCpRows <= a.sinks || j0 >= a.budget - a.recent;
    if (!(work && early)) pdl_wait();
    last = __any_sync(0xFFFFFFFFu, last);
    int slot = -1;
    if (work && lane < kCpRows && j < a.budget) {
        if (len <= a.budget) slot = j < len ? j : -1;
        else slot = !early ? a.kept[(long long)bh * a.budget + j] : j < a.sinks ? j : len - a.budget + j;
    }
    bool ok = slot >= 0;
    long long from = 0, to = 0;
    if (ok) {
        const int i = slot / a.src.page_size, o = slot - i * a.src.page_size, i2 = j / a.dst.page_size, o2 = j - i2 * a.dst.page_size;
        const int p = a.src.table[(long long)b * a.src.table_pages + i], p2 = a.dst.table[(long long)b * a.dst.table_pages + i2];
        ok = (unsigned)p < (unsigned)a.src.n_pages && (unsigned)p2 < (unsigned)a.dst.n_pages;
        if (!ok) set_err(a.err, kErrPage);
        from = p * a.src.page_stride + h * a.src.head_stride + o * a.src.row_stride;
        to = p2 * a.dst.page_stride + h * a.dst.head_stride + o2 * a.dst.row_stride;
        if (ok && a.dst.weights)
            a.dst.weights[((long long)p2 * a.Hkv + h) * a.dst.page_size + o2] =
                a.src.weights[((long long)p * a.Hkv + h) * a.src.page_size + o];
    }
    const int per = row_bytes / 16, both = 2 * per;      // 16-byte pieces of a K row, of a K and a V row
    const uint32_t rows = __ballot_sync(0xFFFFFFFFu, ok);
    for (int c0 = 0; rows && c0 < kCpRows * both; c0 += 32 * kCpUnroll) {
        uint4 x[kCpUnroll];
        char *dst[kCpUnroll];
#pragma unroll
        for (int u = 0; u < kCpUnroll; ++u) {
            const int c = c0 + 32 * u + lane, row = c / both, k = c - row * both;
            const long long f = __shfl_sync(0xFFFFFFFFu, from, row), t = __shfl_sync(0xFFFFFFFFu, to, row);
            const bool v = k >= per;
            dst[u] = rows >> row & 1 ? (v ? a.dst.v : a.dst.k) + t + (v ? k - per : k) * 16 : nullptr;
            if (dst[u]) x[u] = *(const uint4 *)((v ? a.src.v : a.src.k) + f + (v ? k - per : k) * 16);
        }
#pragma unroll
        for (int u = 0; u < kCpUnroll; ++u)
            if (dst[u]) *(uint4 *)dst[u] = x[u];
    }
    if (!last) return;
    pdl_wait();                          // the selection reads them too
    __threadfence();
    __syncwarp();                        // lane 0 has the ticket, every lane writes
    for (int i = lane; i < a.B; i += 32) a.dst.kv_len[i] = min(paged_len(a.src, i, 0, nullptr), a.budget);
    if (lane == 0) *a.counter = 0;
}

}  // namespace

cudaError_t prepare_evict_kernels() {
    return cudaFuncSetAttribute(evict_select_kernel<1024>, cudaFuncAttributeMaxDynamicSharedMemorySize, kEvCached * 4);
}

// CTAs per (sequence, KV head) of the selection: as many as give every SM two, up
// to the portable cluster size, each with 8192 rows or more of the table.
static int select_cluster(int rows, long long cap, int sms) {
    int cs = 8;
    while (cs > 1 && (rows * cs > 2 * sms || cap < 8192LL * cs)) cs >>= 1;
    return cs;
}

cudaError_t launch_paged_evict(const EvictArgs &a, int row_bytes, int sms, cudaStream_t s) {
    const long long cap = (long long)a.src.table_pages * a.src.page_size;
    const int cs = select_cluster(a.B * a.Hkv, cap, sms);
    const long long share = (cap + cs - 1) / cs + 32;
    const int cached = (int)(share < kEvCached ? share : kEvCached);
    // Short rows: CTAs of 256 threads, up to eight on an SM (728 rows of up to 170, a whole call:
    // 22 us, 33 with 1024 threads).
    const bool small = cap <= 2048;
    const cudaError_t e = launch_cluster(small ? evict_select_kernel<256> : evict_select_kernel<1024>, dim3(a.B * a.Hkv * cs),
                                         dim3(small ? 256 : 1024), (size_t)cached * 4, cs, s, a, cs, cached);
    if (e != cudaSuccess) return e;
    const long long warps = (long long)a.B * a.Hkv * ((a.budget + kCpRows - 1) / kCpRows);
    return launch_k(evict_copy_kernel, dim3((unsigned)((warps * 32 + kCpThreads - 1) / kCpThreads)), dim3(kCpThreads), 0, s, true, a, row_bytes);
}

}  // namespace prism
