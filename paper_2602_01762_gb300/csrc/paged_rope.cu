// Per-head norm of queries and keys with the position rotation, dense or stored
// into a paged cache, and its gradient.
//
//   n = x / sqrt(mean(x^2) + eps),  z = g * n           (each head on its own)
//   y_j       = z_j cos - z_{j+D/2} sin
//   y_{j+D/2} = z_{j+D/2} cos + z_j sin                 (j < D/2, angle of the row's position)
//
// Bound by bytes: every row is read once and written once.  A lane holds the 16
// bytes at j and the 16 bytes at j + D/2 of one head, so a rotation pair never
// leaves its lane and the mean is one exchange over D/2 / E lanes (E values per
// 16 bytes); a warp takes 32 E / (D/2) heads of a row at a time and keeps the
// row's cosines and sines in registers over all its heads.
#include "paged.cuh"

namespace prism {
namespace {

constexpr int kNrThreads = 128;
constexpr int kNrUnroll = 2;             // head groups a warp has in flight

template <typename T, int D> struct Rope {
    static constexpr int E = Vec16<T>::E, kLanes = D / 2 / E, kHeads = 32 / kLanes;
    float cs[E], sn[E];
    __device__ __forceinline__ void load(const float *rope, int pos) {
        const int j = (threadIdx.x & 31) % kLanes * E;
        const float *p = rope + (long long)pos * D + j;
#pragma unroll
        for (int i = 0; i < E; i += 4) {
            *(float4 *)(cs + i) = __ldg((const float4 *)(p + i));
            *(float4 *)(sn + i) = __ldg((const float4 *)(p + D / 2 + i));
        }
    }
};

template <int LANES> __device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

// Rotary position of row i of sequence b, held to the table.
__device__ __forceinline__ int row_position(const int32_t *pos, int b, int i, int rope_len, int *err) {
    const long long p = (long long)pos[b] + i;
    if (p >= 0 && p < rope_len) return (int)p;
    set_err(err, kErrPosition);
    return p < 0 ? 0 : rope_len - 1;
}
__device__ __forceinline__ int row_count(const int32_t *n_new, int b, int max_new, int *err) {
    if (!n_new) return max_new;
    const int n = n_new[b];
    if (n >= 0 && n <= max_new) return n;
    set_err(err, kErrNNew);
    return n < 0 ? 0 : max_new;
}

// One warp per row and share of its head groups (`split` shares).  APPEND: keys
// and values go to the paged cache, and their accumulated weights start at 0.
template <typename T, int D, bool APPEND>
__global__ void __launch_bounds__(kNrThreads) norm_rope_kernel(NormRopeArgs a) {
    using R = Rope<T, D>;
    constexpr int E = R::E;
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31;
    const long long w = (long long)blockIdx.x * (kNrThreads / 32) + (threadIdx.x >> 5);
    const long long row = w / a.split;
    const int share = (int)(w - row * a.split);
    const int b = (int)(row / a.max_new), i = (int)(row - (long long)b * a.max_new);
    if (b >= a.B || i >= row_count(a.n_new, b, a.max_new, a.err)) return;
    R rope;
    rope.load(a.rope, row_position(a.pos, b, i, a.rope_len, a.err));

    const int sub = lane % R::kLanes, own = lane / R::kLanes;
    const int hk = a.Hq, hv = a.Hq + a.Hkv, all = APPEND ? hv + a.Hkv : hv;
    long long at = 0, wt = 0;            // the new row's place in the pool and in the weights (KV head 0)
    bool stored = true;
    if (APPEND) {
        const long long slot = (long long)a.cache.kv_len[b] + i;
        stored = slot >= 0 && slot < (long long)a.cache.table_pages * a.cache.page_size;
        if (!stored) {
            set_err(a.err, kErrCache);
        } else {
            const int idx = (int)(slot / a.cache.page_size), off = (int)(slot - (long long)idx * a.cache.page_size);
            const int page = a.cache.table[(long long)b * a.cache.table_pages + idx];
            stored = (unsigned)page < (unsigned)a.cache.n_pages;
            if (!stored) set_err(a.err, kErrPage);
            at = page * a.cache.page_stride + off * a.cache.row_stride;
            wt = (long long)page * a.Hkv * a.cache.page_size + off;
        }
    }
    for (int g0 = share; g0 * R::kHeads < all; g0 += kNrUnroll * a.split) {
        uint4 lo[kNrUnroll], hi[kNrUnroll];
#pragma unroll
        for (int u = 0; u < kNrUnroll; ++u) {
            const int h = (g0 + u * a.split) * R::kHeads + own;
            if (h >= all) continue;
            const HeadsView &x = h < hk ? a.q : h < hv ? a.k : a.v;
            const char *p = x.p + b * x.sb + i * x.st + (h < hk ? h : h < hv ? h - hk : h - hv) * x.sh;
            lo[u] = *((const uint4 *)p + sub);
            hi[u] = *((const uint4 *)(p + D / 2 * sizeof(T)) + sub);
        }
#pragma unroll
        for (int u = 0; u < kNrUnroll; ++u) {
            const int h = (g0 + u * a.split) * R::kHeads + own;
            const bool in = h < all;
            float x[E], y[E];
            if (in) {
                Vec16<T>::unpack(lo[u], x);
                Vec16<T>::unpack(hi[u], y);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) x[e] = y[e] = 0.f;
            }
            if (a.g_q) {
                float s = 0.f;
#pragma unroll
                for (int e = 0; e < E; ++e) s = fmaf(x[e], x[e], fmaf(y[e], y[e], s));
                const float r = rsqrtf(lanes_sum<R::kLanes>(s) * (1.f / D) + a.eps);
                const uint4 *g = (const uint4 *)(h < hk ? a.g_q : a.g_k) + sub;
                float gx[E], gy[E];
                Vec16<T>::unpack(__ldg(g), gx);
                Vec16<T>::unpack(__ldg(g + R::kLanes), gy);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    x[e] = x[e] * r * gx[e];
                    y[e] = y[e] * r * gy[e];
                }
            }
            if (!in) continue;
            float p[E], q[E];
#pragma unroll
            for (int e = 0; e < E; ++e) {
                p[e] = x[e] * rope.cs[e] - y[e] * rope.sn[e];
                q[e] = y[e] * rope.cs[e] + x[e] * rope.sn[e];
            }
            uint4 l = Vec16<T>::pack(p), r = Vec16<T>::pack(q);
            char *to;
            if (h < hk) {
                to = a.q_out.p + b * a.q_out.sb + i * a.q_out.st + h * a.q_out.sh;
            } else if (!APPEND) {
                to = a.k_out.p + b * a.k_out.sb + i * a.k_out.st + (h - hk) * a.k_out.sh;
            } else {
                if (!stored) continue;
                const int kh = h < hv ? h - hk : h - hv;
                to = (h < hv ? a.cache.k : a.cache.v) + at + kh * a.cache.head_stride;
                if (h >= hv) {
                    l = lo[u];
                    r = hi[u];
                } else if (sub == 0 && a.cache.weights) {
                    a.cache.weights[wt + (long long)kh * a.cache.page_size] = 0.f;
                }
            }
            *((uint4 *)to + sub) = l;
            *((uint4 *)(to + D / 2 * sizeof(T)) + sub) = r;
        }
    }
}

// Gradient.  With dz = the inverse rotation of dy, n and r = 1 / sqrt(mean(x^2) + eps):
//   dx = r (g dz - n mean(g dz n)),  dg = sum over rows and heads of dz n.
// x is read again instead of keeping n from the forward pass: the same bytes, and
// nothing to store between the passes.  Each lane adds its 2 E dims of dg over
// every row and head it meets; lanes, warps and CTAs are then added in a fixed
// order (the last CTA to finish adds the CTAs' rows in CTA order), so dg does not
// depend on the order in which they ran.
constexpr int kNgThreads = 512;

template <typename T, int D> struct GainGrad {
    float x[Vec16<T>::E], y[Vec16<T>::E];
};

template <typename T, int D>
__device__ __forceinline__ void grad_heads(const NormRopeGradArgs &a, const HeadsView &gy, const HeadsView &xv, const HeadsView &dx,
                                           const void *gain, const Rope<T, D> &rope, GainGrad<T, D> &dg, int b, int i, bool valid,
                                           int h, int heads) {
    using R = Rope<T, D>;
    constexpr int E = R::E;
    const int sub = (threadIdx.x & 31) % R::kLanes;
    const bool in = h < heads;
    float x[E], y[E], p[E], q[E];
    if (in && valid) {
        const char *sx = xv.p + b * xv.sb + i * xv.st + h * xv.sh, *sg = gy.p + b * gy.sb + i * gy.st + h * gy.sh;
        const uint4 l = *((const uint4 *)sx + sub), r = *((const uint4 *)(sx + D / 2 * sizeof(T)) + sub);
        const uint4 m = *((const uint4 *)sg + sub), n = *((const uint4 *)(sg + D / 2 * sizeof(T)) + sub);
        Vec16<T>::unpack(l, x);
        Vec16<T>::unpack(r, y);
        Vec16<T>::unpack(m, p);
        Vec16<T>::unpack(n, q);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = y[e] = p[e] = q[e] = 0.f;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const float u = p[e], v = q[e];
        p[e] = u * rope.cs[e] + v * rope.sn[e];
        q[e] = v * rope.cs[e] - u * rope.sn[e];
    }
    if (gain) {
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) s = fmaf(x[e], x[e], fmaf(y[e], y[e], s));
        const float r = rsqrtf(lanes_sum<R::kLanes>(s) * (1.f / D) + a.eps);
        const uint4 *g = (const uint4 *)gain + sub;
        float gx[E], gy2[E];
        Vec16<T>::unpack(__ldg(g), gx);
        Vec16<T>::unpack(__ldg(g + R::kLanes), gy2);
        float c = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            x[e] *= r;
            y[e] *= r;
            dg.x[e] = fmaf(p[e], x[e], dg.x[e]);
            dg.y[e] = fmaf(q[e], y[e], dg.y[e]);
            p[e] *= gx[e];
            q[e] *= gy2[e];
            c = fmaf(p[e], x[e], fmaf(q[e], y[e], c));
        }
        c = lanes_sum<R::kLanes>(c) * (1.f / D);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            p[e] = r * (p[e] - x[e] * c);
            q[e] = r * (q[e] - y[e] * c);
        }
    }
    if (!in) return;
    char *to = dx.p + b * dx.sb + i * dx.st + h * dx.sh;
    *((uint4 *)to + sub) = Vec16<T>::pack(p);
    *((uint4 *)(to + D / 2 * sizeof(T)) + sub) = Vec16<T>::pack(q);
}

template <typename T, int D>
__global__ void __launch_bounds__(kNgThreads) norm_rope_grad_kernel(NormRopeGradArgs a) {
    using R = Rope<T, D>;
    constexpr int E = R::E, kWarps = kNgThreads / 32;
    __shared__ float sum[kWarps][2 * D];
    __shared__ int last;
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane % R::kLanes, own = lane / R::kLanes;
    GainGrad<T, D> dq, dk;
#pragma unroll
    for (int e = 0; e < E; ++e) dq.x[e] = dq.y[e] = dk.x[e] = dk.y[e] = 0.f;
    const long long items = (long long)a.B * a.max_new * a.split;
    const int gq = (a.Hq + R::kHeads - 1) / R::kHeads, gk = (a.Hkv + R::kHeads - 1) / R::kHeads;
    for (long long w = (long long)blockIdx.x * kWarps + warp; w < items; w += (long long)gridDim.x * kWarps) {
        const long long row = w / a.split;
        const int share = (int)(w - row * a.split);
        const int b = (int)(row / a.max_new), i = (int)(row - (long long)b * a.max_new);
        const bool valid = i < row_count(a.n_new, b, a.max_new, a.err);
        R rope;
        rope.load(a.rope, valid ? row_position(a.pos, b, i, a.rope_len, a.err) : 0);
        for (int g = share; g < gq; g += a.split)
            grad_heads<T, D>(a, a.dq_out, a.q, a.dq, a.g_q, rope, dq, b, i, valid, g * R::kHeads + own, a.Hq);
        // the shares go on over the key groups where those of the queries ended
        for (int g = (share - gq % a.split + a.split) % a.split; g < gk; g += a.split)
            grad_heads<T, D>(a, a.dk_out, a.k, a.dk, a.g_k, rope, dk, b, i, valid, g * R::kHeads + own, a.Hkv);
    }
    if (!a.g_q) return;
    // lanes that hold the same dims, then warps, then CTAs
    auto fold = [&](float v) {
#pragma unroll
        for (int o = R::kLanes; o < 32; o <<= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
        return v;
    };
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const float v[4] = {fold(dq.x[e]), fold(dq.y[e]), fold(dk.x[e]), fold(dk.y[e])};
        if (own == 0) {
#pragma unroll
            for (int c = 0; c < 4; ++c) sum[warp][c * (D / 2) + sub * E + e] = v[c];
        }
    }
    __syncthreads();
    for (int d = threadIdx.x; d < 2 * D; d += kNgThreads) {
        float v = 0.f;
#pragma unroll
        for (int i = 0; i < kWarps; ++i) v += sum[i][d];
        __stcg(a.part + (long long)blockIdx.x * 2 * D + d, v);
    }
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) last = atomicAdd(a.counter, 1) == (int)gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    // threads take (a share of the CTAs, a float4 of the 2 D columns)
    constexpr int kCols = 2 * D / 4, kShares = kNgThreads / kCols;
    const int col = threadIdx.x % kCols, mine = threadIdx.x / kCols;
    float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int i = mine; i < (int)gridDim.x; i += kShares) {
        const float4 v = __ldcg((const float4 *)(a.part + (long long)i * 2 * D) + col);
        t.x += v.x;
        t.y += v.y;
        t.z += v.z;
        t.w += v.w;
    }
    static_assert(kShares <= kWarps, "one shared row per share");
    *((float4 *)sum[mine] + col) = t;
    __syncthreads();
    for (int d = threadIdx.x; d < 2 * D; d += kNgThreads) {
        float v = 0.f;
#pragma unroll
        for (int i = 0; i < kShares; ++i) v += sum[i][d];
        (d < D ? a.dg_q : a.dg_k)[d < D ? d : d - D] = v;
    }
    if (threadIdx.x == 0) *a.counter = 0;
}

// Warps per row: one where the rows alone give every SM 16 warps, else more, up
// to one per head group.
int row_split(long long rows, int groups, int sms) {
    long long s = ((long long)sms * 16 + rows - 1) / rows;
    return (int)(s < 1 ? 1 : s > groups ? groups : s);
}
int heads_per_warp(bool bf16, int D) { return 32 / (D / 2 / (bf16 ? 8 : 4)); }

}  // namespace

cudaError_t launch_norm_rope(const NormRopeArgs &args, bool bf16, int D, bool append, int sms, cudaStream_t s) {
    NormRopeArgs a = args;
    const int hpw = heads_per_warp(bf16, D), heads = a.Hq + a.Hkv * (append ? 2 : 1);
    const long long rows = (long long)a.B * a.max_new;
    a.split = row_split(rows, (heads + hpw - 1) / hpw, sms);
    const dim3 grid((unsigned)((rows * a.split + kNrThreads / 32 - 1) / (kNrThreads / 32)));
    auto go = [&](auto k) { return launch_k(k, grid, dim3(kNrThreads), 0, s, true, a); };
    if (append) {
        if (bf16) return D == 128 ? go(norm_rope_kernel<uint16_t, 128, true>) : go(norm_rope_kernel<uint16_t, 64, true>);
        return D == 128 ? go(norm_rope_kernel<float, 128, true>) : go(norm_rope_kernel<float, 64, true>);
    }
    if (bf16) return D == 128 ? go(norm_rope_kernel<uint16_t, 128, false>) : go(norm_rope_kernel<uint16_t, 64, false>);
    return D == 128 ? go(norm_rope_kernel<float, 128, false>) : go(norm_rope_kernel<float, 64, false>);
}

int norm_rope_grad_ctas(int sms) { return sms; }

cudaError_t launch_norm_rope_grad(const NormRopeGradArgs &args, bool bf16, int D, int sms, cudaStream_t s) {
    NormRopeGradArgs a = args;
    const int hpw = heads_per_warp(bf16, D);
    const long long rows = (long long)a.B * a.max_new;
    a.split = row_split(rows, (a.Hq + hpw - 1) / hpw + (a.Hkv + hpw - 1) / hpw, sms);
    const long long ctas = (rows * a.split + kNgThreads / 32 - 1) / (kNgThreads / 32);
    const int most = norm_rope_grad_ctas(sms);
    const dim3 grid((unsigned)(ctas < most ? ctas : most));
    auto go = [&](auto k) { return launch_k(k, grid, dim3(kNgThreads), 0, s, true, a); };
    if (bf16) return D == 128 ? go(norm_rope_grad_kernel<uint16_t, 128>) : go(norm_rope_grad_kernel<uint16_t, 64>);
    return D == 128 ? go(norm_rope_grad_kernel<float, 128>) : go(norm_rope_grad_kernel<float, 64>);
}

}  // namespace prism
