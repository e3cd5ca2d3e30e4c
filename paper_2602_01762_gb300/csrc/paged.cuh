// Launch interfaces and device helpers of the paged-cache operators
// (paged_attend.cu, paged_rope.cu, paged_evict.cu; ABI in paged_api.cu).
#pragma once

#include "common.cuh"

namespace prism {

enum PagedErr : int {
    kErrPage = 16,      // a block-table entry outside the pool
    kErrPosition = 32,  // a rotary position outside the table
};

// A paged cache on the device.  Strides in bytes; row `slot` of sequence b and
// KV head h lies in page table[b, slot / page_size] at row slot % page_size.
struct PagedView {
    char *k, *v;
    long long page_stride, head_stride, row_stride;
    float *weights;              // [n_pages, Hkv, page_size] or null
    const int32_t *table;        // [B, table_pages]
    int32_t *kv_len;             // [B]
    int n_pages, table_pages, page_size;
};

// A [B, max_new, heads, D] tensor by base and byte strides (D contiguous).
struct HeadsView {
    char *p;
    long long sb, st, sh;
};

struct NormRopeArgs {
    HeadsView q, k, v, q_out, k_out;     // append: v read, k_out unused
    PagedView cache;                     // append only
    const void *g_q, *g_k;               // [D] wtype, or both null: no norm
    const float *rope;                   // [rope_len, 2, D/2]: cosines, then sines
    const int32_t *pos, *n_new;          // [B]; n_new null: max_new rows each
    int rope_len, B, max_new, Hq, Hkv, split, heads;   // heads: of a row that a warp takes at a time
    float eps;
    int *err;
};

struct NormRopeGradArgs {
    HeadsView dq_out, dk_out, q, k, dq, dk;
    const void *g_q, *g_k;
    const float *rope;
    const int32_t *pos, *n_new;
    float *dg_q, *dg_k;                  // [D] fp32 (null without gains)
    float *part;                         // [CTAs, 2, D]
    int *counter;                        // last-CTA ticket (left at zero)
    int rope_len, B, max_new, Hq, Hkv, split, heads;
    float eps;
    int *err;
};

struct AttendArgs {
    PagedView cache;
    const void *q;                       // [B, Hq, D]
    void *out;                           // [B, Hq, D]
    float *lse;                          // [B, Hq] or null
    float *scores;                       // base-2 scores (paged_scores.h), or null
    float2 *stat;                        // [B, Hq]: (maximum score, 1 / sum), with scores
    float *part;                         // two pieces per CTA
    int *counter;                        // [B * head tiles] tickets (left at zero)
    int *group_counter;                  // two per CTA (left at zero)
    int B, Hq, Hkv, added;
    int cluster;                         // CTAs of a cluster per segment; 1: a persistent grid (set by the launch)
    float scale_log2;                    // softmax scale * log2(e)
    int *err;
};

struct EvictArgs {
    PagedView src, dst;
    int32_t *kept;                       // [B, Hkv, budget]
    int *counter;                        // last-CTA ticket (left at zero)
    int B, Hkv, budget, sinks, recent;
    int *err;
};

constexpr int kAttendUnit = 64;          // keys per unit of the attention's work split
constexpr int kAttendCost = 1;           // units that a segment costs beside its keys
// The most passes over a KV head's rows that its G query heads take.
int attend_head_tiles(int G);
size_t attend_part_floats(int D, int G, int sms);
int attend_ctas(int sms);
// Kernel attributes, before any capture.
cudaError_t prepare_attend_kernels();
cudaError_t prepare_evict_kernels();
cudaError_t prepare_rope_kernels();
cudaError_t launch_paged_attend(const AttendArgs &a, bool bf16, int D, int sms, cudaStream_t s);
cudaError_t launch_norm_rope(const NormRopeArgs &a, bool bf16, int D, bool append, int sms, cudaStream_t s);
int norm_rope_grad_ctas(int sms);
cudaError_t launch_norm_rope_grad(const NormRopeGradArgs &a, bool bf16, int D, int sms, cudaStream_t s);
cudaError_t launch_paged_evict(const EvictArgs &a, int row_bytes, int sms, cudaStream_t s);

// Launch in clusters of cs CTAs, with programmatic stream serialization.
template <typename Kern, typename... Args>
cudaError_t launch_cluster(Kern k, dim3 grid, dim3 block, size_t smem, int cs, cudaStream_t s, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cs;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, k, args...);
}

#ifdef __CUDACC__
// Rows of sequence b, held to [0, table rows] (outside: the cache-range bit).
__device__ __forceinline__ int paged_len(const PagedView &c, int b, int added, int *err) {
    const long long n = (long long)c.kv_len[b] + added, cap = (long long)c.table_pages * c.page_size;
    if (n >= 0 && n <= cap) return (int)n;
    set_err(err, kErrCache);
    return n < 0 ? 0 : (int)cap;
}

// 16 bytes from global to shared memory, asynchronously; not ok: zeros, nothing is read.
__device__ __forceinline__ void cp16(uint32_t dst, const void *src, bool ok) {
    const int n = ok ? 16 : 0;
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
// The same for data read once: its lines leave L2 first.
__device__ __forceinline__ void cp16_once(uint32_t dst, const void *src, bool ok, uint64_t policy) {
    const int n = ok ? 16 : 0;
    asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2, %3;" ::"r"(dst), "l"(src), "r"(n), "l"(policy) : "memory");
}
__device__ __forceinline__ void cp_group() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait_group() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ uint4 lds16(uint32_t addr) {
    uint4 u;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "r"(addr) : "memory");
    return u;
}

// Two floats rounded to bf16 (nearest even, NaN kept), the first in the low half.
__device__ __forceinline__ uint32_t cvt_bf16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// Two fp32 values in one 64-bit register and their packed arithmetic: half the
// instructions where those, not bytes, hold a kernel up.
typedef unsigned long long F2;
__device__ __forceinline__ F2 f2(float x, float y) {
    F2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ float2 f2_values(F2 a) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a));
    return r;
}
__device__ __forceinline__ F2 f2_mul(F2 a, F2 b) {
    F2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ F2 f2_fma(F2 a, F2 b, F2 c) {
    F2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ F2 f2_add(F2 a, F2 b) {
    F2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ F2 f2_sub(F2 a, F2 b) {
    F2 r;
    asm("sub.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float f2_sum(F2 a) {
    const float2 v = f2_values(a);
    return v.x + v.y;
}

__device__ __forceinline__ F2 lds8(uint32_t addr) {
    F2 r;
    asm volatile("ld.shared.b64 %0, [%1];" : "=l"(r) : "r"(addr));
    return r;
}

__device__ __forceinline__ void lds16(uint32_t addr, F2 &a, F2 &b) {
    asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(a), "=l"(b) : "r"(addr) : "memory");
}

// E values of a 16-byte vector as floats and back (E = 8 bf16 or 4 fp32).
template <typename T> struct Vec16;
template <> struct Vec16<uint16_t> {
    static constexpr int E = 8;
    static __device__ __forceinline__ void unpack(const uint4 &u, float (&f)[8]) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = bf16lo(w[i]);
            f[2 * i + 1] = bf16hi(w[i]);
        }
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[8]) {
        return make_uint4(cvt_bf16x2(f[0], f[1]), cvt_bf16x2(f[2], f[3]), cvt_bf16x2(f[4], f[5]), cvt_bf16x2(f[6], f[7]));
    }
};
template <> struct Vec16<float> {
    static constexpr int E = 4;
    static __device__ __forceinline__ void unpack(const uint4 &u, float (&f)[4]) {
        f[0] = __uint_as_float(u.x);
        f[1] = __uint_as_float(u.y);
        f[2] = __uint_as_float(u.z);
        f[3] = __uint_as_float(u.w);
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[4]) {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
};

// The same shared variable in another CTA of the cluster: load, add, set.
__device__ __forceinline__ uint32_t dsmem_at(const void *local, uint32_t rank) {
    uint32_t remote;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"((uint32_t)__cvta_generic_to_shared(local)), "r"(rank));
    return remote;
}
__device__ __forceinline__ void dsmem_ld(const float *local, uint32_t rank, float4 &v) {
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(dsmem_at(local, rank)) : "memory");
}
__device__ __forceinline__ void dsmem_ld(const float *local, uint32_t rank, float2 &v) {
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(dsmem_at(local, rank)) : "memory");
}
__device__ __forceinline__ void dsmem_add(int *local, uint32_t rank, int v) {
    asm volatile("red.relaxed.cluster.shared::cluster.add.s32 [%0], %1;" ::"r"(dsmem_at(local, rank)), "r"(v) : "memory");
}
__device__ __forceinline__ void dsmem_st(int *local, uint32_t rank, int v) {
    asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(dsmem_at(local, rank)), "r"(v) : "memory");
}

// Ragged work split into equal contiguous shares.  Sequence b of rows(b) rows has
// blocks_of(rows) >= 1 blocks of keys, each for `heads` heads; units run over (b, head, block).
// Every CTA takes `per` units from u0 on, in sequence b; false: none are left for
// it.  All threads of the CTA call it.
struct UnitRange {
    int u0, u1, per;   // this CTA's units; units per CTA
    int b, first;      // sequence of u0 and that sequence's first unit
    int lens;          // lane i: rows of sequence i (B <= 32 alone)
};
template <int THREADS, typename Rows, typename Blocks>
__device__ __forceinline__ bool unit_range(UnitRange &r, int B, int heads, const Rows &rows, const Blocks &blocks_of) {
    const int tid = threadIdx.x, lane = tid & 31;
    const int cta = blockIdx.x, ctas = gridDim.x;
    auto blocks = [&](int b) { return blocks_of(rows(b)); };
    if (B <= 32) {                       // every warp for itself
        r.lens = lane < B ? rows(lane) : 0;
        const int n = lane < B ? blocks_of(r.lens) : 0;
        int s = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int t = __shfl_up_sync(0xFFFFFFFFu, s, o);
            if (lane >= o) s += t;
        }
        const int units = __shfl_sync(0xFFFFFFFFu, s, 31) * heads;
        r.per = (units + ctas - 1) / ctas;
        if ((long long)cta * r.per >= units) return false;
        r.u0 = cta * r.per;
        r.u1 = min(r.u0 + r.per, units);
        const int at = r.u0 / heads;
        r.b = __popc(__ballot_sync(0xFFFFFFFFu, lane < B && s <= at));
        r.first = __shfl_sync(0xFFFFFFFFu, s - n, r.b) * heads;
        return true;
    }
    __shared__ int warp_sum[THREADS / 32], found[2];
    int total = 0;
    for (int b = tid; b < B; b += THREADS) total += blocks(b);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xFFFFFFFFu, total, o);
    if (lane == 0) warp_sum[tid >> 5] = total;
    __syncthreads();
    total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) total += warp_sum[w];
    const int units = total * heads;
    r.per = (units + ctas - 1) / ctas;
    if ((long long)cta * r.per >= units) return false;
    r.u0 = cta * r.per;
    r.u1 = min(r.u0 + r.per, units);
    const int at = r.u0 / heads;
    int before = 0;
    for (int base = 0; base < B && before <= at; base += THREADS) {
        const int n = base + tid < B ? blocks(base + tid) : 0;
        int s = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int t = __shfl_up_sync(0xFFFFFFFFu, s, o);
            if (lane >= o) s += t;
        }
        __syncthreads();                 // the sums of the step before were read
        if (lane == 31) warp_sum[tid >> 5] = s;
        __syncthreads();
        int all = 0;
#pragma unroll
        for (int w = 0; w < THREADS / 32; ++w) {
            if (w < (tid >> 5)) s += warp_sum[w];
            all += warp_sum[w];
        }
        if (n > 0 && before + s - n <= at && at < before + s) {
            found[0] = base + tid;
            found[1] = before + s - n;
        }
        before += all;
    }
    __syncthreads();
    r.b = found[0];
    r.first = found[1] * heads;
    return true;
}
#endif

}  // namespace prism
