// Device helpers of the per-head norm and rotation (paged_rope.cu, paged_codes.cu).
#pragma once

#include "paged.cuh"

namespace prism {
namespace {

// 16 bytes as pairs of values, and back.
template <typename T> struct Pairs {
    static constexpr int N = Vec16<T>::E / 2;
    static __device__ __forceinline__ void unpack(const uint4 &u, F2 (&f)[N]) {
        float x[2 * N];
        Vec16<T>::unpack(u, x);
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = f2(x[2 * i], x[2 * i + 1]);
    }
    static __device__ __forceinline__ uint4 pack(const F2 (&f)[N]) {
        float x[2 * N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float2 v = f2_values(f[i]);
            x[2 * i] = v.x;
            x[2 * i + 1] = v.y;
        }
        return Vec16<T>::pack(x);
    }
};

// A lane's part of one row's rotation: cosines and sines of its dims.
template <typename T, int D> struct Rope {
    static constexpr int E = Vec16<T>::E, N = E / 2, kLanes = D / 2 / E, kHeads = 32 / kLanes;
    F2 cs[N], sn[N];
    __device__ __forceinline__ void set(int i, const float4 &c, const float4 &s) {
        cs[i] = f2(c.x, c.y);
        cs[i + 1] = f2(c.z, c.w);
        sn[i] = f2(s.x, s.y);
        sn[i + 1] = f2(s.z, s.w);
    }
    __device__ __forceinline__ void load(const float *rope, int pos) {
        const float *p = rope + (long long)pos * D + (threadIdx.x & 31) % kLanes * E;
#pragma unroll
        for (int i = 0; i < N; i += 2) set(i, __ldg((const float4 *)(p + 2 * i)), __ldg((const float4 *)(p + D / 2 + 2 * i)));
    }
    // As copied by copy_own: piece k of lane l at 512 k + 16 l.
    __device__ __forceinline__ void load_own(uint32_t at) {
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            float c[4], s[4];
            Vec16<float>::unpack(lds16(at + i / 2 * 512 + (threadIdx.x & 31) * 16), c);
            Vec16<float>::unpack(lds16(at + (N + i) / 2 * 512 + (threadIdx.x & 31) * 16), s);
            set(i, make_float4(c[0], c[1], c[2], c[3]), make_float4(s[0], s[1], s[2], s[3]));
        }
    }
    static __device__ __forceinline__ void copy_own(uint32_t at, const float *rope, int pos, bool ok) {
        const float *p = rope + (long long)pos * D + (threadIdx.x & 31) % kLanes * E;
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            cp16(at + i / 2 * 512 + (threadIdx.x & 31) * 16, p + 2 * i, ok);
            cp16(at + (N + i) / 2 * 512 + (threadIdx.x & 31) * 16, p + D / 2 + 2 * i, ok);
        }
    }
    __device__ __forceinline__ void load_shared(uint32_t at) {
        const uint32_t p = at + (threadIdx.x & 31) % kLanes * (E * 4);
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            float c[4], s[4];
            Vec16<float>::unpack(lds16(p + 8 * i), c);
            Vec16<float>::unpack(lds16(p + D / 2 * 4 + 8 * i), s);
            set(i, make_float4(c[0], c[1], c[2], c[3]), make_float4(s[0], s[1], s[2], s[3]));
        }
    }
};

// A lane's part of a gain vector.
template <typename T, int D> struct Gain {
    static constexpr int N = Rope<T, D>::N;
    F2 x[N], y[N];
    __device__ __forceinline__ void load(const void *g) {
        if (!g) return;
        const uint4 *p = (const uint4 *)g + (threadIdx.x & 31) % Rope<T, D>::kLanes;
        Pairs<T>::unpack(__ldg(p), x);
        Pairs<T>::unpack(__ldg(p + Rope<T, D>::kLanes), y);
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

constexpr int kNrThreads = 128;
constexpr int kNrRing = 6;               // head groups a warp has in flight
constexpr int kNrStage = 1024;           // bytes of one: the lanes' low pieces, then their high ones
constexpr int kNrShared = kNrThreads / 32 * kNrRing * kNrStage;

// One warp per row, or per few rows with a.heads of each at a time, and share of
// their head groups (`split` shares), kNrRing - 1 groups on their way at a time: they
// are requested before the row's position and place are known.  APPEND: keys and
// values go to the paged cache, and their accumulated weights start at 0.
template <typename T, int D, bool APPEND, bool ROWS>
__device__ __forceinline__ void norm_rope_rows(const NormRopeArgs &a, unsigned cta, unsigned char *smem) {
    using R = Rope<T, D>;
    constexpr int N = R::N;
    const int lane = threadIdx.x & 31;
    const unsigned w = cta * (kNrThreads / 32) + (threadIdx.x >> 5), block = w / (unsigned)a.split;
    const int share = (int)(w - block * a.split), sub = lane % R::kLanes;
    const int heads = ROWS ? a.heads : R::kHeads, log = 31 - __clz(heads), own = lane / R::kLanes & (heads - 1);
    const int row = ROWS ? (int)block * (R::kHeads >> log) + (lane / R::kLanes >> log) : (int)block;
    bool live = row < a.B * a.max_new;
    const int b = live ? row / a.max_new : 0, i = live ? row - b * a.max_new : 0;
    live = live && i < row_count(a.n_new, b, a.max_new, a.err);
    if (ROWS ? !__any_sync(0xFFFFFFFFu, live) : !live) return;
    const int Hq = !ROWS || live ? a.Hq : 0, Hkv = !ROWS || live ? a.Hkv : 0;   // heads of this lane's row
    // head groups: the queries', the keys', with APPEND the values'
    const int gq = (a.Hq + heads - 1) / heads, gk = (a.Hkv + heads - 1) / heads, end_k = gq + gk;
    const int groups = APPEND ? end_k + gk : end_k;
    // each lane copies what it reads itself, so that its own waits are enough; `from`
    // walks over the heads of a section (queries, keys, values)
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + (threadIdx.x >> 5) * (kNrRing * kNrStage) + lane * 16;
    int lg = share, l_end = 0, l_heads = 0, lh = 0;
    const char *from = nullptr;
    long long l_step = 0;
    auto copy = [&](int stage) {
        if (lg < groups) {
            if (lg >= l_end) {           // the section of group lg
                const bool is_q = lg < gq, is_k = lg < end_k;
                const HeadsView &v = is_q ? a.q : is_k ? a.k : a.v;
                lh = (is_q ? lg : is_k ? lg - gq : lg - end_k) * heads + own;
                l_end = is_q ? gq : is_k ? end_k : groups;
                l_heads = is_q ? Hq : Hkv;
                l_step = (long long)a.split * heads * v.sh;
                from = v.p + b * v.sb + i * v.st + lh * v.sh + sub * 16;
            }
            if (lh < l_heads) {
                cp16(ring + stage * kNrStage, from, true);
                cp16(ring + stage * kNrStage + 512, from + D / 2 * sizeof(T), true);
            }
            lg += a.split;
            lh += a.split * heads;
            from += l_step;
        }
        cp_group();
    };
#pragma unroll
    for (int u = 0; u < kNrRing - 1; ++u) copy(u);
    Gain<T, D> gain;
    gain.load(a.g_q);
    R rope;
    rope.load(a.rope, live ? row_position(a.pos, b, i, a.rope_len, a.err) : 0);
    char *qo = a.q_out.p + b * a.q_out.sb + i * a.q_out.st + sub * 16;
    char *ko = APPEND ? nullptr : a.k_out.p + b * a.k_out.sb + i * a.k_out.st + sub * 16, *vo = nullptr;
    float *weight = nullptr;             // of the new row and KV head 0
    if (APPEND && live) {
        const int len = a.cache.kv_len[b];
        const long long slot = (long long)len + i;
        if (len < 0 || slot >= (long long)a.cache.table_pages * a.cache.page_size) {   // no slot of a negative length is the row's
            set_err(a.err, kErrCache);
        } else {
            const int idx = (int)(slot / a.cache.page_size), off = (int)(slot - (long long)idx * a.cache.page_size);
            const int page = a.cache.table[(long long)b * a.cache.table_pages + idx];
            if ((unsigned)page >= (unsigned)a.cache.n_pages) {
                set_err(a.err, kErrPage);
            } else {
                const long long at = page * a.cache.page_stride + off * a.cache.row_stride + sub * 16;
                ko = a.cache.k + at;
                vo = a.cache.v + at;
                if (a.cache.weights) weight = a.cache.weights + (long long)page * a.Hkv * a.cache.page_size + off;
            }
        }
    }
    const long long ko_sh = APPEND ? a.cache.head_stride : a.k_out.sh;
    int stage = 0;
    // the next group's stage, with a later group requested in its place
    auto take = [&]() {
        copy(stage == 0 ? kNrRing - 1 : stage - 1);
        cp_wait_group<kNrRing - 1>();
        const uint32_t at = ring + stage * kNrStage;
        stage = stage + 1 == kNrRing ? 0 : stage + 1;
        return at;
    };
    auto turn = [&](int h, int end, char *to) {
        const uint32_t at = take();
        uint4 l = make_uint4(0u, 0u, 0u, 0u), r = l;
        if (h < end) {
            l = lds16(at);
            r = lds16(at + 512);
        }
        F2 x[N], y[N];
        Pairs<T>::unpack(l, x);
        Pairs<T>::unpack(r, y);
        if (a.g_q) {
            F2 s = f2_mul(x[0], x[0]);
#pragma unroll
            for (int e = 1; e < N; ++e) s = f2_fma(x[e], x[e], s);
#pragma unroll
            for (int e = 0; e < N; ++e) s = f2_fma(y[e], y[e], s);
            const float f = rsqrtf(lanes_sum<R::kLanes>(f2_sum(s)) * (1.f / D) + a.eps);
            const F2 ff = f2(f, f);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                x[e] = f2_mul(f2_mul(x[e], ff), gain.x[e]);
                y[e] = f2_mul(f2_mul(y[e], ff), gain.y[e]);
            }
        }
        if (h >= end || !to) return;
        F2 p[N], q[N];
#pragma unroll
        for (int e = 0; e < N; ++e) {
            p[e] = f2_sub(f2_mul(x[e], rope.cs[e]), f2_mul(y[e], rope.sn[e]));
            q[e] = f2_fma(y[e], rope.cs[e], f2_mul(x[e], rope.sn[e]));
        }
        *(uint4 *)to = Pairs<T>::pack(p);
        *(uint4 *)(to + D / 2 * sizeof(T)) = Pairs<T>::pack(q);
    };
    int g = share;
    for (; g < gq; g += a.split) {
        const int h = g * heads + own;
        turn(h, Hq, qo + h * a.q_out.sh);
    }
    gain.load(a.g_k);
    for (; g < end_k; g += a.split) {
        const int h = (g - gq) * heads + own;
        turn(h, Hkv, ko ? ko + h * ko_sh : nullptr);
        if (APPEND && weight && sub == 0 && h < Hkv) weight[(long long)h * a.cache.page_size] = 0.f;
    }
    for (; g < groups; g += a.split) {   // values go as they are
        const int h = (g - end_k) * heads + own;
        const uint32_t at = take();
        if (!vo || h >= Hkv) continue;
        char *to = vo + h * ko_sh;
        *(uint4 *)to = lds16(at);
        *(uint4 *)(to + D / 2 * sizeof(T)) = lds16(at + 512);
    }
}

}  // namespace
}  // namespace prism
