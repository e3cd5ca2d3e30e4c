// Eviction from a paged cache by accumulated attention weight.
//
// Of the L rows of a (sequence, KV head), min(L, budget) are kept: the first
// `sinks`, the last `recent`, and of those between the budget - sinks - recent
// with the largest weight (ties: the lower slot; NaN below everything).  The kept
// rows go in order to the pages of a second table, so rows stay in the order of
// their positions.
//
// Bound by the kept rows' bytes, read once and written once: the selection reads 4
// bytes a row and KV head, the copy moves 8 D in bf16.
#include "paged.cuh"

namespace prism {
namespace {

constexpr int kEvThreads = 1024;
constexpr int kEvWarps = kEvThreads / 32;
constexpr int kEvCached = 48 * 1024;     // rows whose keys shared memory holds

// Weight as an unsigned key with the same order: NaN 0, then -inf ... +inf; -0 as +0.
__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return 0u;
    const uint32_t u = __float_as_uint(w + 0.f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// One CTA per (sequence, KV head): radix selection of the smallest kept key, eight
// bits a pass over the keys in shared memory (read from the pool again where there
// are more than it holds), then the kept slots in order.
__global__ void __launch_bounds__(kEvThreads) evict_select_kernel(EvictArgs a, int cached) {
    extern __shared__ uint32_t keys[];
    __shared__ int hist[256], pick[2], warp_eq[kEvWarps], warp_gt[kEvWarps];
    pdl_wait();
    pdl_trigger();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int b = blockIdx.x / a.Hkv, h = blockIdx.x % a.Hkv;
    const int len = paged_len(a.src, b, 0, a.err);
    int32_t *kept = a.kept + (long long)blockIdx.x * a.budget;
    if (len <= a.budget) {
        for (int j = tid; j < a.budget; j += kEvThreads) kept[j] = j < len ? j : -1;
        return;
    }
    const int first = a.sinks, want = a.budget - a.recent - first;
    const int n = want > 0 ? len - a.recent - first : 0;   // rows to choose from, more than want (none to choose: 0)
    const int32_t *table = a.src.table + (long long)b * a.src.table_pages;
    auto load = [&](int i) {
        const int slot = first + i, idx = slot / a.src.page_size, page = table[idx];
        if ((unsigned)page >= (unsigned)a.src.n_pages) return 0u;      // reported by the copy if it is kept
        return weight_key(a.src.weights[((long long)page * a.Hkv + h) * a.src.page_size + slot - idx * a.src.page_size]);
    };
    const bool held = n <= cached;
    auto key = [&](int i) { return held ? keys[i] : load(i); };
    if (held)
        for (int i = tid; i < n; i += kEvThreads) keys[i] = load(i);
    uint32_t prefix = 0, mask = 0;
    int need = want;                     // rows still to be taken of those that match the prefix
    for (int shift = 24; shift >= 0 && need > 0; shift -= 8) {
        if (tid < 256) hist[tid] = 0;
        __syncthreads();
        for (int i0 = 0; i0 < n; i0 += kEvThreads) {
            const int i = i0 + tid;
            const uint32_t k = i < n ? key(i) : 0u;
            const bool in = i < n && (k & mask) == prefix;
            const uint32_t bin = in ? (k >> shift) & 255u : 256u;
            const uint32_t same = __match_any_sync(0xFFFFFFFFu, bin);
            if (in && lane == __ffs(same) - 1) atomicAdd(hist + bin, __popc(same));
        }
        __syncthreads();
        if (warp == 0) {                 // the bin in which the need-th largest lies
            int c[8], s = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) s += c[e] = hist[255 - (8 * lane + e)];
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
        mask |= 255u << shift;
        need -= pick[1];
    }
    // the prefix is now that key: larger keys are kept, and the first `need` equal ones
    const int per = ((n + kEvWarps - 1) / kEvWarps + 31) & ~31, lo = min(n, warp * per), hi = min(n, lo + per);
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
    gt = eq = 0;
    for (int w = 0; w < warp; ++w) gt += warp_gt[w], eq += warp_eq[w];
    for (int i0 = lo; i0 < hi; i0 += 32) {
        const int i = i0 + lane;
        const uint32_t k = i < hi ? key(i) : 0u;
        const bool is_gt = i < hi && k > prefix, is_eq = i < hi && k == prefix;
        const uint32_t bg = __ballot_sync(0xFFFFFFFFu, is_gt), be = __ballot_sync(0xFFFFFFFFu, is_eq), below = (1u << lane) - 1u;
        const int rank = eq + __popc(be & below);
        if (is_gt || (is_eq && rank < need)) kept[first + gt + __popc(bg & below) + min(rank, need)] = first + i;
        gt += __popc(bg);
        eq += __popc(be);
    }
    for (int j = tid; j < first; j += kEvThreads) kept[j] = j;
    for (int j = tid; j < a.recent; j += kEvThreads) kept[first + want + j] = len - a.recent + j;
}

// Copies the kept rows of K, V and the weights, 32 destination rows of one KV head
// per warp: each lane looks one row up, then the warp moves them 512 bytes at a
// time.  Also sets the destination's lengths.
constexpr int kCpThreads = 256;
constexpr int kCpUnroll = 8;
__global__ void __launch_bounds__(kCpThreads) evict_copy_kernel(EvictArgs a, int row_bytes) {
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31;
    const long long gid = (long long)blockIdx.x * kCpThreads + threadIdx.x;
    for (long long b = gid; b < a.B; b += (long long)gridDim.x * kCpThreads)
        a.dst.kv_len[b] = min(paged_len(a.src, (int)b, 0, nullptr), a.budget);
    const int chunks = (a.budget + 31) / 32;
    const long long w = gid >> 5;
    const long long bh = w / chunks;
    if (bh >= (long long)a.B * a.Hkv) return;
    const int b = (int)(bh / a.Hkv), h = (int)(bh - (long long)b * a.Hkv), j = (int)(w - bh * chunks) * 32 + lane;
    const int slot = j < a.budget ? a.kept[bh * a.budget + j] : -1;
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
    if (!rows) return;
    for (int c0 = 0; c0 < 32 * both; c0 += 32 * kCpUnroll) {
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
}

}  // namespace

cudaError_t prepare_evict_kernels() {
    return cudaFuncSetAttribute(evict_select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kEvCached * 4);
}

cudaError_t launch_paged_evict(const EvictArgs &a, int row_bytes, cudaStream_t s) {
    const long long cap = (long long)a.src.table_pages * a.src.page_size;
    const int cached = (int)(cap < kEvCached ? cap : kEvCached);
    cudaError_t e = launch_k(evict_select_kernel, dim3(a.B * a.Hkv), dim3(kEvThreads), (size_t)cached * 4, s, true, a, cached);
    if (e != cudaSuccess) return e;
    const long long warps = (long long)a.B * a.Hkv * ((a.budget + 31) / 32);
    return launch_k(evict_copy_kernel, dim3((unsigned)((warps * 32 + kCpThreads - 1) / kCpThreads)), dim3(kCpThreads), 0, s, true, a, row_bytes);
}

}  // namespace prism
