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
// 16 bytes); a warp takes 32 E / (D/2) heads at a time, of one row or of several that
// have few, and keeps the rows' cosines and sines in registers over all their heads.  All arithmetic is fp32,
// each result is rounded once.  Measured: append of 8 prompts of 1021 to 2048 rows (32
// + 2 x 8 heads of 128, bf16) 50 us (6.2 TB/s; 45.5 at the rate of a plain copy);
// forward and gradient of 14196 of 16384 rows (32 + 8 heads) 137 us (5.6 TB/s; 113).
#include "paged_rope.cuh"

#include <type_traits>

namespace prism {
namespace {

template <typename T, int D, bool APPEND, bool ROWS>
__global__ void __launch_bounds__(kNrThreads, 5) norm_rope_kernel(NormRopeArgs a) {
    __shared__ __align__(16) unsigned char smem[kNrShared];
    pdl_wait();
    pdl_trigger();
    norm_rope_rows<T, D, APPEND, ROWS>(a, blockIdx.x, smem);
}

// Gradient.  With dz = the inverse rotation of dy, n and r = 1 / sqrt(mean(x^2) + eps):
//   dx = r (g dz - n mean(g dz n)),  dg = sum over rows and heads of dz n.
// x is read again instead of keeping n from the forward pass: the same bytes, and
// nothing to store between the passes.  Each lane adds its 2 E dims of dg over
// every row and head it meets; lanes, warps and CTAs are then added in a fixed
// order (the last CTA to finish adds the CTAs' rows in CTA order), so dg does not
// depend on the order in which they ran.
// Persistent CTAs, one per SM; each warp walks over its rows' head groups with a
// ring of kNgRing groups requested ahead by cp.async, across rows.  What holds it at
// 5 TB/s is the latency of some 300 instructions a group at 12 warps an SM: the sums of
// dg, the rotation and the data take up to 142 registers (16 warps of 128 spill: 145
// against 137 us with the forward; a ring of 7 instead of 5 leaves too little L1: 140).
constexpr int kNgThreads = 384;
constexpr int kNgRing = 5;
constexpr int kNgStage = 2048 + 512;     // x and dy, low and high pieces of each lane; the row's cosines and sines
// With several rows to a warp (ROWS): every lane has its own cosines and sines.
template <bool ROWS> constexpr int kNgDepth = ROWS ? 4 : kNgRing;
template <bool ROWS> constexpr int kNgBytes = ROWS ? 2048 + 2048 : kNgStage;
template <bool ROWS> constexpr int kNgShared = kNgThreads / 32 * kNgDepth<ROWS> * kNgBytes<ROWS> + 2 * 128 * 4;

template <typename T, int D> struct GainGrad {
    F2 x[Rope<T, D>::N], y[Rope<T, D>::N];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int e = 0; e < Rope<T, D>::N; ++e) x[e] = y[e] = 0ull;
    }
};

// The heads of one group: x and dy from the stage, dx to `to` (null: a lane without a head).
template <typename T, int D>
__device__ __forceinline__ void grad_group(uint32_t stage, char *to, bool norm, uint32_t gain, float eps, const Rope<T, D> &rope,
                                           GainGrad<T, D> &dg) {
    using R = Rope<T, D>;
    constexpr int N = R::N;
    const int lane = threadIdx.x & 31;
    F2 p[N], q[N];
    {
        F2 u[N], v[N];
        Pairs<T>::unpack(lds16(stage + 1024 + lane * 16), u);
        Pairs<T>::unpack(lds16(stage + 1536 + lane * 16), v);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            p[e] = f2_fma(u[e], rope.cs[e], f2_mul(v[e], rope.sn[e]));
            q[e] = f2_sub(f2_mul(v[e], rope.cs[e]), f2_mul(u[e], rope.sn[e]));
        }
    }
    if (norm) {
        F2 x[N], y[N];
        Pairs<T>::unpack(lds16(stage + lane * 16), x);
        Pairs<T>::unpack(lds16(stage + 512 + lane * 16), y);
        // with v = g dz:  dx = r v - (x r) r^2 mean(v x),  dg += dz (x r); both sums go together
        F2 s = 0ull, c = 0ull, v[N], w[N];
#pragma unroll
        for (int e = 0; e < N; e += 2) {
            lds16(gain + (e / 2 * R::kLanes + lane % R::kLanes) * 16, v[e], v[e + 1]);
            lds16(gain + ((N + e) / 2 * R::kLanes + lane % R::kLanes) * 16, w[e], w[e + 1]);
        }
#pragma unroll
        for (int e = 0; e < N; ++e) {
            v[e] = f2_mul(p[e], v[e]);
            w[e] = f2_mul(q[e], w[e]);
            s = f2_fma(x[e], x[e], f2_fma(y[e], y[e], s));
            c = f2_fma(v[e], x[e], f2_fma(w[e], y[e], c));
        }
        float ss = f2_sum(s), cc = f2_sum(c);
#pragma unroll
        for (int o = R::kLanes / 2; o > 0; o >>= 1) {
            ss += __shfl_xor_sync(0xFFFFFFFFu, ss, o);
            cc += __shfl_xor_sync(0xFFFFFFFFu, cc, o);
        }
        // each factor r beside a factor x: no power of r that overflows where the result does not
        // (a lane without a head adds nothing to dg, also where eps is 0)
        const float r = to ? rsqrtf(ss * (1.f / D) + eps) : 0.f, k = -(cc * (1.f / D) * r) * r;
        const F2 rr = f2(r, r), kk = f2(k, k);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            x[e] = f2_mul(x[e], rr);
            y[e] = f2_mul(y[e], rr);
            dg.x[e] = f2_fma(p[e], x[e], dg.x[e]);
            dg.y[e] = f2_fma(q[e], y[e], dg.y[e]);
            p[e] = f2_fma(x[e], kk, f2_mul(v[e], rr));
            q[e] = f2_fma(y[e], kk, f2_mul(w[e], rr));
        }
    }
    if (!to) return;
    *(uint4 *)to = Pairs<T>::pack(p);
    *(uint4 *)(to + D / 2 * sizeof(T)) = Pairs<T>::pack(q);
}

// A warp's walk over its rows (every `rows`-th, from its own on; with ROWS blocks of
// rows, a lane in one of them) and, in each, its share of the head groups; sequence
// and row are stepped without a division.
template <bool ROWS> struct RowWalk {
    int b, i, g, share, step_b, step_i;
    bool live, valid;                    // of this lane's row
    bool some_live, some_valid;          // of the warp's
    __device__ __forceinline__ void begin(const NormRopeGradArgs &a, int warp, int warps, int per, int mine) {
        const int rows = warps / a.split;                // warps past rows * split have none
        const int row = warp / a.split * per + mine;
        share = warp % a.split;
        b = row / a.max_new;
        i = row - b * a.max_new;
        step_b = rows * per / a.max_new;
        step_i = rows * per - step_b * a.max_new;
        live = warp < rows * a.split;
        look(a);
    }
    __device__ __forceinline__ void next(const NormRopeGradArgs &a) {
        b += step_b;
        i += step_i;
        if (i >= a.max_new) {
            i -= a.max_new;
            ++b;
        }
        look(a);
    }
    __device__ __forceinline__ void look(const NormRopeGradArgs &a) {
        g = share;
        live = live && b < a.B;
        valid = live && i < row_count(a.n_new, b, a.max_new, a.err);
        some_live = ROWS ? __any_sync(0xFFFFFFFFu, live) : live;
        some_valid = ROWS ? __any_sync(0xFFFFFFFFu, valid) : valid;
    }
};

template <typename T, int D, bool ROWS>
__global__ void __launch_bounds__(kNgThreads) norm_rope_grad_kernel(NormRopeGradArgs a) {
    using R = Rope<T, D>;
    constexpr int kWarps = kNgThreads / 32, kRing = kNgDepth<ROWS>, kStage = kNgBytes<ROWS>;
    extern __shared__ __align__(16) unsigned char dyn[];
    __shared__ int last;
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane % R::kLanes;
    // heads of a row that the warp takes at a time, this lane's head of them and row
    const int heads = ROWS ? a.heads : R::kHeads, log = ROWS ? 31 - __clz(a.heads) : 0;
    const int own = ROWS ? lane / R::kLanes & (heads - 1) : lane / R::kLanes, row_of = ROWS ? lane / R::kLanes >> log : 0;
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(dyn) + warp * (kRing * kStage);
    // both gains as fp32 behind the rings, four values of each lane side by side
    float *gain = (float *)(dyn + kWarps * kRing * kStage);
    const uint32_t gains = (uint32_t)__cvta_generic_to_shared(gain);
    if (a.g_q)
        for (int i = threadIdx.x; i < 2 * D; i += kNgThreads) {
            const int d = i % D, half = d / (D / 2), l = d % (D / 2) / R::E, e = d % R::E;
            gain[i - d + ((half * R::E + e) / 4 * R::kLanes + l) * 4 + e % 4] = Elem<T>::load((const T *)(i < D ? a.g_q : a.g_k), d);
        }
    __syncthreads();
    GainGrad<T, D> dq, dk;
    dq.clear();
    dk.clear();
    const int gq = (a.Hq + heads - 1) / heads, groups = gq + (a.Hkv + heads - 1) / heads;
    auto row_at = [&](const HeadsView &v, const RowWalk<ROWS> &r) { return v.p + r.b * v.sb + r.i * v.st + sub * 16; };

    RowWalk<ROWS> f;                     // loads ahead: the next group to request, in rows that count
    f.begin(a, blockIdx.x * kWarps + warp, gridDim.x * kWarps, ROWS ? R::kHeads >> log : 1, row_of);
    RowWalk<ROWS> r = f;
    while (f.some_live && !f.some_valid) f.next(a);
    bool fresh = true;                   // its row's first group: the row's table line comes with it
    const char *x = nullptr, *y = nullptr;   // its heads in q or k, and in dq_out or dk_out
    long long x_step = 0, y_step = 0;
    int fh = 0;
    int stage_in = 0;
    auto request = [&]() {
        if (f.some_live) {
            const uint32_t to = ring + stage_in * kStage + lane * 16;
            if (ROWS && fresh)
                R::copy_own(ring + stage_in * kStage + 2048, a.rope, f.valid ? row_position(a.pos, f.b, f.i, a.rope_len, a.err) : 0, f.valid);
            if (!ROWS && fresh && lane < D / 4)
                cp16(to + 2048, a.rope + (long long)row_position(a.pos, f.b, f.i, a.rope_len, a.err) * D + lane * 4, true);
            const bool is_q = f.g < gq;
            if (fresh || (!is_q && f.g - a.split < gq)) {
                const HeadsView &vx = is_q ? a.q : a.k, &vy = is_q ? a.dq_out : a.dk_out;
                fh = (is_q ? f.g : f.g - gq) * heads + own;
                x = row_at(vx, f) + fh * vx.sh;
                y = row_at(vy, f) + fh * vy.sh;
                x_step = a.split * heads * vx.sh;
                y_step = a.split * heads * vy.sh;
            }
            const bool ok = (!ROWS || f.valid) && fh < (is_q ? a.Hq : a.Hkv);
            const char *xs = ok ? x : a.q.p, *ys = ok ? y : a.q.p;
            cp16(to, xs, ok);
            cp16(to + 512, xs + D / 2 * sizeof(T), ok);
            cp16(to + 1024, ys, ok);
            cp16(to + 1536, ys + D / 2 * sizeof(T), ok);
            x += x_step;
            y += y_step;
            fh += a.split * heads;
            f.g += a.split;
            fresh = f.g >= groups;
            if (fresh) {
                do f.next(a);
                while (f.some_live && !f.some_valid);
            }
        }
        cp_group();
        stage_in = stage_in + 1 == kRing ? 0 : stage_in + 1;
    };
#pragma unroll
    for (int u = 0; u < kRing - 1; ++u) request();

    int stage = 0;
    for (; r.some_live; r.next(a)) {
        if (r.live && !r.valid) {        // rows past n_new have zero gradients
            for (int g = r.share; g < groups; g += a.split) {
                const bool is_q = g < gq;
                const int h = (is_q ? g : g - gq) * heads + own;
                if (h >= (is_q ? a.Hq : a.Hkv)) continue;
                char *to = is_q ? row_at(a.dq, r) + h * a.dq.sh : row_at(a.dk, r) + h * a.dk.sh;
                *(uint4 *)to = *(uint4 *)(to + D / 2 * sizeof(T)) = make_uint4(0u, 0u, 0u, 0u);
            }
        }
        if (!r.some_valid) continue;
        R rope;
        bool first = true;
        auto take = [&]() {
            cp_wait_group<kRing - 2>();
            __syncwarp();
            request();                   // into the stage that was read last
            const uint32_t at = ring + stage * kStage;
            stage = stage + 1 == kRing ? 0 : stage + 1;
            if (first && ROWS) rope.load_own(at + 2048);
            if (first && !ROWS) rope.load_shared(at + 2048);
            first = false;
            return at;
        };
        char *to = row_at(a.dq, r);
        for (; r.g < gq; r.g += a.split) {
            const uint32_t at = take();
            const int h = r.g * heads + own;
            grad_group<T, D>(at, (!ROWS || r.valid) && h < a.Hq ? to + h * a.dq.sh : nullptr, a.g_q, gains, a.eps, rope, dq);
        }
        to = row_at(a.dk, r);
        for (; r.g < groups; r.g += a.split) {
            const uint32_t at = take();
            const int h = (r.g - gq) * heads + own;
            grad_group<T, D>(at, (!ROWS || r.valid) && h < a.Hkv ? to + h * a.dk.sh : nullptr, a.g_k, gains + 4 * D, a.eps, rope, dk);
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
    for (int e = 0; e < R::N; ++e) {
        const float2 v[4] = {f2_values(dq.x[e]), f2_values(dq.y[e]), f2_values(dk.x[e]), f2_values(dk.y[e])};
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const float x = fold(v[c].x), y = fold(v[c].y);
            if (lane < R::kLanes) {
                sum[warp][c * (D / 2) + sub * R::E + 2 * e] = x;
                sum[warp][c * (D / 2) + sub * R::E + 2 * e + 1] = y;
            }
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
// Heads of a row that a warp takes at a time, of the hpw it has lanes for; it takes
// hpw / heads rows.  Fewer than hpw where that saves an eighth of the lanes' turns and
// the rows still give every SM 16 warps.  Measured, one row a warp against several: append
// of 160000 rows of 2 + 2 x 1 heads of 64 171 and 38 us, of 123000 of 4 + 2 x 4 132 and
// 81, of 40000 of 8 + 2 x 2 of 128 57 and 45; forward and gradient of the same 336 and
// 89, 254 and 168, 126 and 110; where a tenth is saved (fp32, 16 + 2 x 1 of 128) 58.4
// and 60.0: one row.
template <typename F> int heads_at_once(int hpw, long long rows, int sms, const F &groups) {
    int best = hpw;
    for (int h = hpw / 2; h > 0 && rows * h >= (long long)hpw * sms * 16; h /= 2)
        if (8 * groups(h) * h <= 7 * groups(best) * best) best = h;
    return best;
}
int heads_per_warp(bool bf16, int D) { return 32 / (D / 2 / (bf16 ? 8 : 4)); }

}  // namespace

unsigned plan_norm_rope(NormRopeArgs &a, bool bf16, int D, bool append, int sms) {
    const int hpw = heads_per_warp(bf16, D), sections = append ? 2 : 1;
    const long long rows = (long long)a.B * a.max_new;
    auto groups = [&](int heads) { return (a.Hq + heads - 1) / heads + sections * ((a.Hkv + heads - 1) / heads); };
    a.heads = heads_at_once(hpw, rows, sms, groups);
    const long long blocks = (rows * a.heads + hpw - 1) / hpw;
    a.split = row_split(blocks, groups(a.heads), sms);
    a.one_row = a.heads == hpw;
    return (unsigned)((blocks * a.split + kNrThreads / 32 - 1) / (kNrThreads / 32));
}

cudaError_t launch_norm_rope(const NormRopeArgs &args, bool bf16, int D, bool append, int sms, cudaStream_t s) {
    NormRopeArgs a = args;
    const dim3 grid(plan_norm_rope(a, bf16, D, append, sms));
    auto go = [&](auto one, auto many) { return launch_k(a.one_row ? one : many, grid, dim3(kNrThreads), 0, s, true, a); };
    auto form = [&](auto t, auto d) {
        using T = decltype(t);
        return append ? go(norm_rope_kernel<T, d, true, false>, norm_rope_kernel<T, d, true, true>)
                      : go(norm_rope_kernel<T, d, false, false>, norm_rope_kernel<T, d, false, true>);
    };
    const std::integral_constant<int, 64> small;
    const std::integral_constant<int, 128> large;
    if (bf16) return D == 128 ? form(uint16_t(), large) : form(uint16_t(), small);
    return D == 128 ? form(0.f, large) : form(0.f, small);
}

cudaError_t prepare_rope_kernels() {
    cudaError_t e = cudaSuccess;
    auto set = [&](auto one, auto rows) {
        if (e == cudaSuccess) e = cudaFuncSetAttribute(one, cudaFuncAttributeMaxDynamicSharedMemorySize, kNgShared<false>);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(rows, cudaFuncAttributeMaxDynamicSharedMemorySize, kNgShared<true>);
    };
    set(norm_rope_grad_kernel<uint16_t, 64, false>, norm_rope_grad_kernel<uint16_t, 64, true>);
    set(norm_rope_grad_kernel<uint16_t, 128, false>, norm_rope_grad_kernel<uint16_t, 128, true>);
    set(norm_rope_grad_kernel<float, 64, false>, norm_rope_grad_kernel<float, 64, true>);
    set(norm_rope_grad_kernel<float, 128, false>, norm_rope_grad_kernel<float, 128, true>);
    return e;
}

int norm_rope_grad_ctas(int sms) { return sms; }

cudaError_t launch_norm_rope_grad(const NormRopeGradArgs &args, bool bf16, int D, int sms, cudaStream_t s) {
    NormRopeGradArgs a = args;
    const int hpw = heads_per_warp(bf16, D);
    const long long rows = (long long)a.B * a.max_new;
    auto groups = [&](int heads) { return (a.Hq + heads - 1) / heads + (a.Hkv + heads - 1) / heads; };
    a.heads = heads_at_once(hpw, rows, sms, groups);
    const long long blocks = (rows * a.heads + hpw - 1) / hpw;
    a.split = row_split(blocks, groups(a.heads), sms);
    const int most = norm_rope_grad_ctas(sms);
    if (a.split > most * (kNgThreads / 32)) a.split = most * (kNgThreads / 32);   // a row's shares fit the grid
    const long long ctas = (blocks * a.split + kNgThreads / 32 - 1) / (kNgThreads / 32);
    const dim3 grid((unsigned)(ctas < most ? ctas : most));
    auto go = [&](auto one, auto many) {
        return a.heads == hpw ? launch_k(one, grid, dim3(kNgThreads), kNgShared<false>, s, true, a)
                              : launch_k(many, grid, dim3(kNgThreads), kNgShared<true>, s, true, a);
    };
    if (bf16)
        return D == 128 ? go(norm_rope_grad_kernel<uint16_t, 128, false>, norm_rope_grad_kernel<uint16_t, 128, true>)
                        : go(norm_rope_grad_kernel<uint16_t, 64, false>, norm_rope_grad_kernel<uint16_t, 64, true>);
    return D == 128 ? go(norm_rope_grad_kernel<float, 128, false>, norm_rope_grad_kernel<float, 128, true>)
                    : go(norm_rope_grad_kernel<float, 64, false>, norm_rope_grad_kernel<float, 64, true>);
}

}  // namespace prism
