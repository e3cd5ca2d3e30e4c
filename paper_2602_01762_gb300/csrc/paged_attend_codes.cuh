// The paged attention (paged_attend.cuh) over a cache held in 8 bits, with a scale for
// each block of rows.
//
//   z_j = scale * s^K_j (q . c^K_j),   out = sum_j (p_j s^V_j) c^V_j
//
// Bound by the bytes of the codes: 2 D a row and KV head, half of bf16's.  The codes go
// to the tensor cores as fp16, which holds every code of both formats exactly (e4m3 by
// the hardware's conversion, int8 as the low byte of 1024 + 128 + c), and the scales
// stay outside: K's multiplies a row's score, V's its probability.
//
// Measured, D = 128, bf16 queries: e4m3, 64 sequences of 6001 to 16384 rows, G = 8, 233 us
// (6.3 TB/s); one of 131071, G = 4, 50 us (5.4, of which 39 us are the bytes and the rest
// its start and joins); int8 with a scale a row, 16 sequences of 1 to 8192 rows, 34 us
// (4.1); 517 rows 6.2 us. A tile of 16 rows takes 362 instructions a warp with e4m3 (a
// pair of codes is one conversion) and 469 with int8; three CTAs an SM give the warps that
// hide them (two: 276 us for the first case; four, of 128 registers: 298).
#pragma once

#include "paged_attend.cuh"

namespace prism {
namespace {

__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, bool fresh) {
    if (fresh)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
            : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t cvt_f16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float2 f16x2_values(uint32_t h) {
    float2 v;
    asm("{.reg .b16 l, u;\n mov.b32 {l, u}, %2;\n cvt.f32.f16 %0, l;\n cvt.f32.f16 %1, u;}" : "=f"(v.x), "=f"(v.y) : "r"(h));
    return v;
}
// Two values as three fp16 parts each, rounded: their sum is the value, down to 2^-25.
__device__ __forceinline__ void three_parts16(float x, float y, uint32_t &p0, uint32_t &p1, uint32_t &p2) {
    p0 = cvt_f16x2(x, y);
    float2 v = f16x2_values(p0);
    x -= v.x, y -= v.y;
    p1 = cvt_f16x2(x, y);
    v = f16x2_values(p1);
    p2 = cvt_f16x2(x - v.x, y - v.y);
}

// 2^x; 0 below 2^-126.
__device__ __forceinline__ float power2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Four codes as fp16: `lo` the first two, `hi` the others.
template <int FORMAT> __device__ __forceinline__ void code_values(uint32_t codes, uint32_t &lo, uint32_t &hi) {
    if (FORMAT == kE4m3) {
        asm("{.reg .b16 l, u;\n mov.b32 {l, u}, %2;\n cvt.rn.f16x2.e4m3x2 %0, l;\n cvt.rn.f16x2.e4m3x2 %1, u;}" : "=r"(lo), "=r"(hi) : "r"(codes));
    } else {
        const uint32_t c = codes ^ 0x80808080u;          // code + 128
        asm("sub.f16x2 %0, %1, %2;" : "=r"(lo) : "r"(__byte_perm(c, 0x64646464u, 0x4140)), "r"(0x64806480u));
        asm("sub.f16x2 %0, %1, %2;" : "=r"(hi) : "r"(__byte_perm(c, 0x64646464u, 0x4342)), "r"(0x64806480u));
    }
}

// Keys in the 16-row dimension M and query heads in the 8-column dimension N of
// warp-level products, as for bf16 rows:
//   S^T[key][h] = K[key][:] . q[h][:]        A = 16 rows of K, B = q^T in registers
//   O^T[d][h]  += V^T[d][keys] W^T[keys][h]  A = V^T, B = W^T, W = p s^V
// Which dim is which k of S (and which row of O^T) is free: a lane's 16 bytes of a row
// of K are four steps over D, and its D / 8 bytes of four rows of V, two and two
// interleaved, the A of every tile of O^T, so no code is moved between lanes.
//
// q enters as fp16 times a power of two for its head that brings the largest value to
// 2^14: a bf16 value keeps its 8 bits down to 2^-31 of that (and below within 2^-39 of
// it); fp32 takes three parts, its 24 bits as far down.  W is fp16 parts of p s^V over a
// power of two for the head: two for bf16, 22 bits, at most 4 units of 2^-24 of a weight
// where the result's own rounding is 2^15 of them (a third: the cases above 252, 53, 35.5
// us); three for fp32, 24 bits; below 2^-15 of the head's largest fewer, within 2^-38 of
// it.  With up to four heads two parts share a product, in columns 0 to 3 and 4 to 7.
//
// Two running maxima, of the scores (for the sum of probabilities) and of the scores
// with log2 s^V (for W, so that it stays in fp16's range whatever the scales are; kept
// as its distance from the first, in which log2 s^V is not lost beside a score of 2^24
// or more); both are whole numbers, so that rescaling is exact.  The tensor cores
// drop bits below their accumulator: each tile's O is added by the CUDA cores.
enum HeadMode : int { kPacked = 0, kEight = 1, kSixteen = 2 };
template <typename T_, int D_, int MODE, int FORMAT, int KT_ = 32> struct CodeTile {
    using T = T_;
    static constexpr int D = D_, KT = KT_, NT = MODE == kSixteen ? 2 : 1;
    static constexpr int kRow = D, kStage = 2 * KT * kRow + 8 * KT;   // bytes
    static constexpr bool kScaled = true;
    using Args = CodeAttendArgs;
    static constexpr int kHeads = MODE == kPacked ? 4 : 8 * NT;
    static constexpr int kQ = sizeof(T) == 2 ? 1 : MODE == kPacked ? 2 : 3;  // products of K and q
    static constexpr int kParts = (sizeof(T) == 2 ? 2 : 3) - (MODE == kPacked ? 1 : 0);   // products of V and W
    static_assert(sizeof(T) == 2 || MODE != kSixteen, "fp32 queries go eight heads at a time: sixteen take 96 registers");
    static constexpr int kMergeStride = D + 4;
    // a segment's end costs what two blocks of 8-bit rows do, or three: with 1, 2 and 3 units 16
    // sequences of 1 to 8192 int8 rows 36.5, 34.3 and 33.2 us, 64 of 1 to 2048 43.9, 37.5 and 36.6,
    // 64 of 6001 to 16384 e4m3 rows 232.6, 231.5 and 231.0, 64 with a window of 4096 97.2, 95.7 and 96.1
    static constexpr int kCost = 2;
    static constexpr int kCtas = MODE == kSixteen || kQ == 3 ? 2 : 3, kStages = (D == 128 ? 2 : 4) * 32 / KT + (kCtas == 2 ? 1 : 0);
    // where a cluster's CTAs have few rows (see start_attend), tiles of 16 spread them over the
    // warps: 8 KV heads of 100, 512, 1000 and 2000 rows 5.5, 6.0, 6.4 and 7.9 us in tiles of
    // 32, 5.0, 5.6, 6.4 and 8.1 in tiles of 16 (sixteen heads' sums need a stage of 32)
    using Short = CodeTile<T, D, MODE, FORMAT, MODE == kSixteen ? 32 : 16>;
    static constexpr int kClusterRows = (MODE == kSixteen ? 1024 : 512) * 128 / D;   // see attend_cluster
    static constexpr int kWindowRows = kClusterRows * 5 / 4, kWindowCluster = 2;     // see window_cluster
    // p s^V over its base stays below 2^2, one for each of the slack and log2 s cut to a
    // whole number: W up to 2^15 leaves the most below.
    static constexpr float kSlackW = 1.f, kLift = 8192.f;
    // The maximum of no score: scores of -inf are still -inf over it, so that none needs another base.
    static constexpr float kLowest = -3.402823466e38f;
    uint32_t qf[D / 16][kQ][NT][2];
    float qs[NT][2];                                     // scale of the scores over q's power of two
    float m[NT][2], n[NT][2], l[NT][2], f[NT][2];        // n: of the scores with log2 s^V, over m; f: W over p s^V
    F2 o[D / 16][NT][2];                                 // two dims of a head pair

    // Shared address of 16-byte piece c of row r: the eight lanes of a load (two rows of
    // K, or two pieces of four rows of V of one parity) meet all banks.
    static __device__ __forceinline__ uint32_t piece(int r, int c) {
        const int turn = (r >> 1 & 3) << 1;
        if (D == 128) return (uint32_t)(r * 128 + ((c ^ turn ^ (r & 1) << 2) << 4));
        return (uint32_t)((r >> 1) * 128 + ((((r & 1) << 2 | c) ^ turn) << 4));
    }
    // Four dims from d on of a head.
    static __device__ __forceinline__ void four(const T *q, int d, float (&x)[4]) {
        if (sizeof(T) == 2) {
            const uint2 u = *(const uint2 *)(q + d);
            x[0] = bf16lo(u.x), x[1] = bf16hi(u.x), x[2] = bf16lo(u.y), x[3] = bf16hi(u.y);
        } else {
            const float4 u = *(const float4 *)(q + d);
            x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w;
        }
    }
    __device__ __forceinline__ void load_q(const T *q, int heads, float scale) {
        const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int u = 0; u < NT; ++u) {
            const int h = MODE == kPacked ? (g & 3) : g + 8 * u;
            const T *from = q + (h < heads ? h : 0) * D + 16 * t;
            float x[D / 16][4];
            uint32_t top = 0;                            // bits of the largest finite magnitude
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                four(from, k / 4 * 64 + k % 4 * 4, x[k]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (h >= heads) x[k][i] = 0.f;
                    const uint32_t b = __float_as_uint(x[k][i]) & 0x7FFFFFFFu;
                    top = max(top, b < 0x7F800000u ? b : 0u);
                }
            }
            top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
            top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
            const int e = min(14 + 127 - (int)(top >> 23), 126);   // largest value to 2^14
            const float up = __uint_as_float((uint32_t)(127 + e) << 23), down = __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    uint32_t p[3];
                    three_parts16(x[k][2 * i] * up, x[k][2 * i + 1] * up, p[0], p[1], p[2]);
                    if (sizeof(T) == 4 && MODE == kPacked) {   // columns 4 to 7: the second parts
                        qf[k][0][u][i] = g < 4 ? p[0] : p[1];
                        qf[k][kQ - 1][u][i] = g < 4 ? p[2] : 0u;
                    } else {
#pragma unroll
                        for (int j = 0; j < kQ; ++j) qf[k][j][u][i] = p[j];
                    }
                }
            }
            // of this lane's columns 2 t, 2 t + 1
            qs[u][0] = scale * __shfl_sync(0xFFFFFFFFu, down, 8 * t);
            qs[u][1] = scale * __shfl_sync(0xFFFFFFFFu, down, 8 * t + 4);
        }
    }
    __device__ __forceinline__ void reset() {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                m[t][i] = kLowest;
                n[t][i] = l[t][i] = 0.f;
                f[t][i] = kLift;
            }
#pragma unroll
            for (int d = 0; d < D / 16; ++d) o[d][t][0] = o[d][t][1] = 0ull;
        }
    }
    // log2 of a scale, its fraction cut (of 0 -127, of an infinite one or NaN 128).
    static __device__ __forceinline__ float whole_log2(float s) {
        return __uint_as_float((__float_as_uint(s) & 0x7FFFFFFFu) >> 23 | 0x4B000000u) - 8388735.f;   // 2^23 + exponent
    }
    static __device__ __forceinline__ float lds4(uint32_t addr) {
        float v;
        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
        return v;
    }
    // This lane's D / 8 bytes of a row of V.
    static __device__ __forceinline__ void value_row(uint32_t at, uint32_t (&w)[D / 32]) {
        if (D == 128) {
            const uint4 u = lds16(at);
            w[0] = u.x, w[1] = u.y, w[D / 32 - 2] = u.z, w[D / 32 - 1] = u.w;
        } else {
            const F2 u = lds8(at);
            w[0] = (uint32_t)u, w[1] = (uint32_t)(u >> 32);
        }
    }
    template <typename Rows>
    __device__ __forceinline__ void tile(uint32_t ks, uint32_t vs, float *, int key0, const Rows &seen, float, float *, int) {
        const int lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3;
        // piece() of row g's first part and of this lane's part of row 2 t; eight rows on it
        // is the same, a step over D or an odd row the other 64 bytes of a line
        uint32_t k_at = ks + piece(g, t4), v_at = vs + (D == 128 ? piece(2 * t4, g) : piece(2 * t4, g >> 1) + 8 * (g & 1));
        uint32_t scales = vs + KT * kRow + 4 * g;
        int base = key0;
#pragma unroll 1
        for (int sub = 0; sub < KT / 16; ++sub, base += 16, k_at += 16 * kRow, v_at += 16 * kRow, scales += 64) {
            if (sub > 0 && base >= seen.len) break;
            float s[NT][4], s2[NT][4];                   // even and odd steps over D: half the chain of products
#pragma unroll
            for (int c = 0; c < D / 64; ++c) {
                const uint4 x = lds16(k_at ^ 64 * c), y = lds16((k_at ^ 64 * c) + 8 * kRow);
                const uint32_t xw[4] = {x.x, x.y, x.z, x.w}, yw[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    uint32_t a[4];
                    code_values<FORMAT>(xw[w], a[0], a[2]);
                    code_values<FORMAT>(yw[w], a[1], a[3]);
                    const int k = 4 * c + w;
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int i = kQ - 1; i >= 0; --i)   // last parts first
                            mma_f16(k & 1 ? s2[t] : s[t], a, qf[k][i][t][0], qf[k][i][t][1], k < 2 && i == kQ - 1);
                }
            }
            const float k0 = lds4(scales), k1 = lds4(scales + 32), v0 = lds4(scales + 4 * KT), v1 = lds4(scales + 4 * KT + 32);
            const float e0 = whole_log2(v0), e1 = whole_log2(v1);
            const bool all = seen.sees_all(base, 16);
            const bool in0 = all || seen.sees(base + g), in1 = all || seen.sees(base + g + 8);
            float over[NT][4];                           // scores over the maximum
            bool grew = false;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[t][i] += s2[t][i];
                    if (sizeof(T) == 4 && MODE == kPacked) s[t][i] += __shfl_xor_sync(0xFFFFFFFFu, s[t][i], 2);
                    s[t][i] *= (i < 2 ? k0 : k1) * qs[t][i & 1];
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if (!in0) s[t][i] = -INFINITY;
                    if (!in1) s[t][2 + i] = -INFINITY;
                    over[t][i] = s[t][i] - m[t][i];
                    over[t][2 + i] = s[t][2 + i] - m[t][i];
                    grew |= fmaxf(s[t][i], s[t][2 + i]) > m[t][i] + kSlack || fmaxf(over[t][i] + e0, over[t][2 + i] + e1) > n[t][i] + kSlackW;
                }
            }
            if (__any_sync(0xFFFFFFFFu, grew)) {
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    float a[2];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        // the largest score, and the largest with log2 s^V over it
                        float top = fmaxf(fmaxf(s[t][i], s[t][2 + i]), kLowest), y = fmaxf(s[t][i] - top + e0, s[t][2 + i] - top + e1);
#pragma unroll
                        for (int x = 4; x < 32; x <<= 1) {
                            const float o_top = __shfl_xor_sync(0xFFFFFFFFu, top, x), o_y = __shfl_xor_sync(0xFFFFFFFFu, y, x);
                            const float most = fmaxf(top, o_top);
                            y = fmaxf(y + (top - most), o_y + (o_top - most));
                            top = most;
                        }
                        const float level = fmaxf(m[t][i], ceilf(top)), down = m[t][i] - level;
                        y = ceilf(y + (top - level));
                        m[t][i] = level;
                        over[t][i] = s[t][i] - level;
                        over[t][2 + i] = s[t][2 + i] - level;
                        // no further below than p f's range (scales below 2^-106 lose bits of W)
                        y = fmaxf(fmaxf(n[t][i] + down, y), -106.f);
                        l[t][i] *= exp2f(down);
                        a[i] = exp2f(n[t][i] + down - y);
                        n[t][i] = y;
                        f[t][i] = exp2f(-y) * kLift;
                    }
                    const F2 both = f2(a[0], a[1]);
#pragma unroll
                    for (int d = 0; d < D / 16; ++d) {
                        o[d][t][0] = f2_mul(o[d][t][0], both);
                        o[d][t][1] = f2_mul(o[d][t][1], both);
                    }
                }
            }
            uint32_t part[kParts][NT][2];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const float p0 = power2(over[t][2 * u]), p1 = power2(over[t][2 * u + 1]), v = u ? v1 : v0;
                    l[t][0] += p0;
                    l[t][1] += p1;
                    uint32_t x, y, z;
                    three_parts16(p0 * f[t][0] * v, p1 * f[t][1] * v, x, y, z);
                    if (MODE == kPacked) {               // columns 4 to 7: the second parts
                        part[0][t][u] = transpose8((lane & 2) ? y : x);
                        if (kParts == 2) part[kParts - 1][t][u] = transpose8((lane & 2) ? 0u : z);
                    } else {
                        part[0][t][u] = transpose8(x);
                        part[kParts > 1 ? 1 : 0][t][u] = transpose8(y);
                        if (kParts == 3) part[kParts - 1][t][u] = transpose8(z);
                    }
                }
            }
            uint32_t v[4][D / 32];                       // rows 2 t4, 2 t4 + 1, 2 t4 + 8, 2 t4 + 9
#pragma unroll
            for (int i = 0; i < 4; ++i) value_row((i & 1 ? (v_at ^ 64) + (D == 128 ? kRow : 0) : v_at) + (i >> 1) * 8 * kRow, v[i]);
#pragma unroll
            for (int d = 0; d < D / 16; ++d) {
                const uint32_t pick = d & 1 ? 0x7362 : 0x5140;
                uint32_t a[4];
                code_values<FORMAT>(__byte_perm(v[0][d / 2], v[1][d / 2], pick), a[0], a[1]);
                code_values<FORMAT>(__byte_perm(v[2][d / 2], v[3][d / 2], pick), a[2], a[3]);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    float x[4];
#pragma unroll
                    for (int i = kParts - 1; i >= 0; --i) mma_f16(x, a, part[i][t][0], part[i][t][1], i == kParts - 1);
                    o[d][t][0] = f2_add(o[d][t][0], f2(x[0], x[1]));
                    o[d][t][1] = f2_add(o[d][t][1], f2(x[2], x[3]));
                }
            }
        }
    }
    // This warp's state: sums as [head][D] (row stride kMergeStride), over the scores' maximum, and maximum and sum per head.
    __device__ __forceinline__ void store(float *so, float *sm, float *sl) {
        const int lane = threadIdx.x & 31, g = lane >> 2, c = 2 * (lane & 3);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            float back[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float v = l[t][i];
                v += __shfl_xor_sync(0xFFFFFFFFu, v, 4);
                v += __shfl_xor_sync(0xFFFFFFFFu, v, 8);
                v += __shfl_xor_sync(0xFFFFFFFFu, v, 16);
                if (g == 0 && 8 * t + c + i < kHeads) {
                    sm[8 * t + c + i] = v == 0.f ? -INFINITY : m[t][i];
                    sl[8 * t + c + i] = v;
                }
                back[i] = exp2f(n[t][i]) / kLift;
            }
#pragma unroll
            for (int d = 0; d < D / 16; ++d) {
                const float2 x[2] = {f2_values(o[d][t][0]), f2_values(o[d][t][1])};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float v = (i & 1 ? x[i >> 1].y : x[i >> 1].x) * back[i & 1];
                    if (MODE == kPacked) v += __shfl_xor_sync(0xFFFFFFFFu, v, 2);
                    if (8 * t + c < kHeads) so[(8 * t + c + (i & 1)) * kMergeStride + D / 8 * g + 2 * d + (i >> 1)] = v;
                }
            }
        }
    }
};

template <int FORMAT, typename F> cudaError_t with_code_tile(bool bf16, int D, int heads, const F &f) {
    if (bf16) {
        if (D == 128)
            return heads == 4 ? f(CodeTile<uint16_t, 128, kPacked, FORMAT>()) : heads == 8 ? f(CodeTile<uint16_t, 128, kEight, FORMAT>()) : f(CodeTile<uint16_t, 128, kSixteen, FORMAT>());
        return heads == 4 ? f(CodeTile<uint16_t, 64, kPacked, FORMAT>()) : heads == 8 ? f(CodeTile<uint16_t, 64, kEight, FORMAT>()) : f(CodeTile<uint16_t, 64, kSixteen, FORMAT>());
    }
    if (D == 128) return heads == 4 ? f(CodeTile<float, 128, kPacked, FORMAT>()) : f(CodeTile<float, 128, kEight, FORMAT>());
    return heads == 4 ? f(CodeTile<float, 64, kPacked, FORMAT>()) : f(CodeTile<float, 64, kEight, FORMAT>());
}
inline int code_head_tile(bool bf16, int G) {
    const int ht = attend_head_tile(G);
    return bf16 || ht < 16 ? ht : 8;
}
template <int FORMAT> cudaError_t prepare_codes(bool bf16, int D, int G) {
    return with_code_tile<FORMAT>(bf16, D, code_head_tile(bf16, G), [](auto tile) { return prepare_attend<decltype(tile), WindowRows>(); });
}
template <int FORMAT> cudaError_t start_codes(const CodeAttendArgs &a, bool bf16, int D, int sms, cudaStream_t s) {
    const int ht = code_head_tile(bf16, a.Hq / a.Hkv);
    return with_code_tile<FORMAT>(bf16, D, ht, [&](auto tile) { return start_attend<decltype(tile), WindowRows>(a, ht, sms, s); });
}

}  // namespace
}  // namespace prism
