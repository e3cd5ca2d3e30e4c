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

}  // namespace
}  // namespace prism
