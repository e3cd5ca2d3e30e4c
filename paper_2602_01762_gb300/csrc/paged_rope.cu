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
constexpr int kNrRing = 8;               // head groups a warp has in flight
constexpr int kNrStage = 1024;           // bytes of one: the lanes' low pieces, then their high ones

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

// One warp per row and share of its head groups (`split` shares), kNrRing - 1 of
// them on their way at a time: they are requested before the row's position and
// place are known.  APPEND: keys and values go to the paged cache, and their
// accumulated weights start at 0.
template <typename T, int D, bool APPEND>
__global__ void __launch_bounds__(kNrThreads) norm_rope_kernel(NormRopeArgs a) {
    using R = Rope<T, D>;
    constexpr int E = R::E;
    __shared__ __align__(16) unsigned char smem[kNrThreads / 32 * kNrRing * kNrStage];
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31;
    const long long w = (long long)blockIdx.x * (kNrThreads / 32) + (threadIdx.x >> 5);
    const long long row = w / a.split;
    const int share = (int)(w - row * a.split);
    const int b = (int)(row / a.max_new), i = (int)(row - (long long)b * a.max_new);
    if (b >= a.B || i >= row_count(a.n_new, b, a.max_new, a.err)) return;
    const int sub = lane % R::kLanes, own = lane / R::kLanes;
    const int hk = a.Hq, hv = a.Hq + a.Hkv, all = APPEND ? hv + a.Hkv : hv;
    // each lane copies what it reads itself, so that its own waits are enough
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + (threadIdx.x >> 5) * (kNrRing * kNrStage) + lane * 16;
    auto copy = [&](int g, int stage) {
        const int h = g * R::kHeads + own;
        if (h < all) {
            const HeadsView &x = h < hk ? a.q : h < hv ? a.k : a.v;
            const char *p = x.p + b * x.sb + i * x.st + (h < hk ? h : h < hv ? h - hk : h - hv) * x.sh + sub * 16;
            cp16(ring + stage * kNrStage, p, true);
            cp16(ring + stage * kNrStage + 512, p + D / 2 * sizeof(T), true);
        }
        cp_group();
    };
#pragma unroll
    for (int u = 0; u < kNrRing - 1; ++u) copy(share + u * a.split, u);
    R rope;
    rope.load(a.rope, row_position(a.pos, b, i, a.rope_len, a.err));
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
    int stage = 0;
    for (int g = share; g * R::kHeads < all; g += a.split) {
        copy(g + (kNrRing - 1) * a.split, stage == 0 ? kNrRing - 1 : stage - 1);
        cp_wait_group<kNrRing - 1>();
        const int h = g * R::kHeads + own;
        const bool in = h < all;
        uint4 l = make_uint4(0u, 0u, 0u, 0u), r = l;
        if (in) {
            l = lds16(ring + stage * kNrStage);
            r = lds16(ring + stage * kNrStage + 512);
        }
        stage = stage + 1 == kNrRing ? 0 : stage + 1;
        if (g * R::kHeads < hv) {        // a group with query or key heads (the same for the warp)
            float x[E], y[E];
            Vec16<T>::unpack(l, x);
            Vec16<T>::unpack(r, y);
            if (a.g_q) {
                float s = 0.f;
#pragma unroll
                for (int e = 0; e < E; ++e) s = fmaf(x[e], x[e], fmaf(y[e], y[e], s));
                const float f = rsqrtf(lanes_sum<R::kLanes>(s) * (1.f / D) + a.eps);
                const uint4 *gain = (const uint4 *)(h < hk ? a.g_q : a.g_k) + sub;
                float gx[E], gy[E];
                Vec16<T>::unpack(__ldg(gain), gx);
                Vec16<T>::unpack(__ldg(gain + R::kLanes), gy);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    x[e] = x[e] * f * gx[e];
                    y[e] = y[e] * f * gy[e];
                }
            }
            float p[E], q[E];
#pragma unroll
            for (int e = 0; e < E; ++e) {
                p[e] = x[e] * rope.cs[e] - y[e] * rope.sn[e];
                q[e] = y[e] * rope.cs[e] + x[e] * rope.sn[e];
            }
            if (h < hv) {                // values stay as they are
                l = Vec16<T>::pack(p);
                r = Vec16<T>::pack(q);
            }
        }
        char *to = nullptr;
        if (h < hk) {
            to = a.q_out.p + b * a.q_out.sb + i * a.q_out.st + h * a.q_out.sh;
        } else if (!APPEND) {
            if (in) to = a.k_out.p + b * a.k_out.sb + i * a.k_out.st + (h - hk) * a.k_out.sh;
        } else if (in && stored) {
            const int kh = h < hv ? h - hk : h - hv;
            to = (h < hv ? a.cache.k : a.cache.v) + at + kh * a.cache.head_stride;
            if (h < hv && sub == 0 && a.cache.weights) a.cache.weights[wt + (long long)kh * a.cache.page_size] = 0.f;
        }
        if (to) {
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
// Persistent CTAs, one per SM; each warp walks over its rows' head groups with a
// ring of kNgRing groups requested ahead by cp.async, across rows.
constexpr int kNgThreads = 512;
constexpr int kNgRing = 5;
constexpr int kNgStage = 2048 + 512;     // x and dy, low and high pieces of each lane; the row's cosines and sines

template <typename T, int D> struct GainGrad {
    float x[Vec16<T>::E], y[Vec16<T>::E];
};

// The heads of one group: x and dy from the stage, dx to `to` (null: a lane without a head).
template <typename T, int D>
__device__ __forceinline__ void grad_group(uint32_t stage, char *to, const void *gain, float eps, const Rope<T, D> &rope, GainGrad<T, D> &dg) {
    using R = Rope<T, D>;
    constexpr int E = R::E;
    const int lane = threadIdx.x & 31, sub = lane % R::kLanes;
    float x[E], y[E], p[E], q[E];
    Vec16<T>::unpack(lds16(stage + lane * 16), x);
    Vec16<T>::unpack(lds16(stage + 512 + lane * 16), y);
    Vec16<T>::unpack(lds16(stage + 1024 + lane * 16), p);
    Vec16<T>::unpack(lds16(stage + 1536 + lane * 16), q);
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
        const float r = rsqrtf(lanes_sum<R::kLanes>(s) * (1.f / D) + eps);
        const uint4 *g = (const uint4 *)gain + sub;
        float gx[E], gy[E];
        Vec16<T>::unpack(__ldg(g), gx);
        Vec16<T>::unpack(__ldg(g + R::kLanes), gy);
        float c = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            x[e] *= r;
            y[e] *= r;
            dg.x[e] = fmaf(p[e], x[e], dg.x[e]);
            dg.y[e] = fmaf(q[e], y[e], dg.y[e]);
            p[e] *= gx[e];
            q[e] *= gy[e];
            c = fmaf(p[e], x[e], fmaf(q[e], y[e], c));
        }
        c = lanes_sum<R::kLanes>(c) * (1.f / D);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            p[e] = r * (p[e] - x[e] * c);
            q[e] = r * (q[e] - y[e] * c);
        }
    }
    if (!to) return;
    *((uint4 *)to + sub) = Vec16<T>::pack(p);
    *((uint4 *)(to + D / 2 * sizeof(T)) + sub) = Vec16<T>::pack(q);
}

// A warp's walk over (row, share) items and the head groups of each.
struct RowWalk {
    int w, b, i, g;
    bool live, valid;
    __device__ __forceinline__ void at(const NormRopeGradArgs &a, int item, int items) {
        w = item;
        live = item < items;
        valid = false;
        if (!live) return;
        const int row = item / a.split;
        g = item - row * a.split;
        b = row / a.max_new;
        i = row - b * a.max_new;
        valid = i < row_count(a.n_new, b, a.max_new, a.err);
    }
};

template <typename T, int D>
__global__ void __launch_bounds__(kNgThreads) norm_rope_grad_kernel(NormRopeGradArgs a) {
    using R = Rope<T, D>;
    constexpr int E = R::E, kWarps = kNgThreads / 32;
    extern __shared__ __align__(16) unsigned char dyn[];
    __shared__ int last;
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane % R::kLanes, own = lane / R::kLanes;
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(dyn) + warp * (kNgRing * kNgStage);
    GainGrad<T, D> dq, dk;
#pragma unroll
    for (int e = 0; e < E; ++e) dq.x[e] = dq.y[e] = dk.x[e] = dk.y[e] = 0.f;
    const int items = a.B * a.max_new * a.split, step = gridDim.x * kWarps;
    const int gq = (a.Hq + R::kHeads - 1) / R::kHeads, groups = gq + (a.Hkv + R::kHeads - 1) / R::kHeads;
    auto head_at = [&](const HeadsView &v, const RowWalk &r, int h) { return v.p + r.b * v.sb + r.i * v.st + h * v.sh; };

    RowWalk f;                           // loads ahead: the next group to request, in rows that count
    f.at(a, blockIdx.x * kWarps + warp, items);
    while (f.live && !f.valid) f.at(a, f.w + step, items);
    bool fresh = true;                   // its row's first group: the row's table line comes with it
    int stage_in = 0;
    auto request = [&]() {
        if (f.live) {
            const uint32_t to = ring + stage_in * kNgStage;
            const bool is_q = f.g < gq;
            const int h = (is_q ? f.g : f.g - gq) * R::kHeads + own;
            const bool ok = h < (is_q ? a.Hq : a.Hkv);
            const char *x = ok ? head_at(is_q ? a.q : a.k, f, h) : a.q.p, *y = ok ? head_at(is_q ? a.dq_out : a.dk_out, f, h) : a.q.p;
            cp16(to + lane * 16, x + sub * 16, ok);
            cp16(to + 512 + lane * 16, x + D / 2 * sizeof(T) + sub * 16, ok);
            cp16(to + 1024 + lane * 16, y + sub * 16, ok);
            cp16(to + 1536 + lane * 16, y + D / 2 * sizeof(T) + sub * 16, ok);
            if (fresh && lane < D / 4)
                cp16(to + 2048 + lane * 16, a.rope + (long long)row_position(a.pos, f.b, f.i, a.rope_len, a.err) * D + lane * 4, true);
            f.g += a.split;
            fresh = f.g >= groups;
            if (fresh) {
                f.at(a, f.w + step, items);
                while (f.live && !f.valid) f.at(a, f.w + step, items);
            }
        }
        cp_group();
        stage_in = stage_in + 1 == kNgRing ? 0 : stage_in + 1;
    };
#pragma unroll
    for (int u = 0; u < kNgRing - 1; ++u) request();

    int stage = 0;
    RowWalk r;
    for (r.at(a, blockIdx.x * kWarps + warp, items); r.live; r.at(a, r.w + step, items)) {
        if (!r.valid) {                  // rows past n_new have zero gradients
            for (; r.g < groups; r.g += a.split) {
                const bool is_q = r.g < gq;
                const int h = (is_q ? r.g : r.g - gq) * R::kHeads + own;
                if (h >= (is_q ? a.Hq : a.Hkv)) continue;
                char *to = head_at(is_q ? a.dq : a.dk, r, h);
                *((uint4 *)to + sub) = *((uint4 *)(to + D / 2 * sizeof(T)) + sub) = make_uint4(0u, 0u, 0u, 0u);
            }
            continue;
        }
        R rope;
        for (bool first = true; r.g < groups; r.g += a.split, first = false) {
            cp_wait_group<kNgRing - 2>();
            __syncwarp();
            request();                   // into the stage that was read last
            const uint32_t at = ring + stage * kNgStage;
            if (first) {
#pragma unroll
                for (int e = 0; e < E; e += 4) {
                    const uint4 c = lds16(at + 2048 + (sub * E + e) * 4), s = lds16(at + 2048 + (D / 2 + sub * E + e) * 4);
                    Vec16<float>::unpack(c, *(float(*)[4])(rope.cs + e));
                    Vec16<float>::unpack(s, *(float(*)[4])(rope.sn + e));
                }
            }
            if (r.g < gq) {
                const int h = r.g * R::kHeads + own;
                grad_group<T, D>(at, h < a.Hq ? head_at(a.dq, r, h) : nullptr, a.g_q, a.eps, rope, dq);
            } else {
                const int h = (r.g - gq) * R::kHeads + own;
                grad_group<T, D>(at, h < a.Hkv ? head_at(a.dk, r, h) : nullptr, a.g_k, a.eps, rope, dk);
            }
            stage = stage + 1 == kNgRing ? 0 : stage + 1;
        }
    }
    cp_wait_group<0>();
    if (!a.g_q) return;
    // lanes that hold the same dims, then warps, then CTAs
    __syncthreads();                     // the rings are free
    float(*sum)[2 * D] = (float(*)[2 * D])dyn;
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
constexpr int kNgSmem = kNgThreads / 32 * kNgRing * kNgStage;
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

cudaError_t prepare_rope_kernels() {
    auto set = [](auto k) { return cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kNgSmem); };
    cudaError_t e = set(norm_rope_grad_kernel<uint16_t, 64>);
    if (e == cudaSuccess) e = set(norm_rope_grad_kernel<uint16_t, 128>);
    if (e == cudaSuccess) e = set(norm_rope_grad_kernel<float, 64>);
    if (e == cudaSuccess) e = set(norm_rope_grad_kernel<float, 128>);
    return e;
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
    auto go = [&](auto k) { return launch_k(k, grid, dim3(kNgThreads), kNgSmem, s, true, a); };
    if (bf16) return D == 128 ? go(norm_rope_grad_kernel<uint16_t, 128>) : go(norm_rope_grad_kernel<uint16_t, 64>);
    return D == 128 ? go(norm_rope_grad_kernel<float, 128>) : go(norm_rope_grad_kernel<float, 64>);
}

}  // namespace prism
