// Tiles of bf16 and fp32 rows for the paged attention (paged_attend.cuh).
#pragma once

#include "paged_attend.cuh"

namespace prism {
namespace {

constexpr int kPaStage = 8192;           // bytes of one warp's stage: KT rows of K, then of V

// bf16 rows on warp-level tensor-core products, keys in the 16-row dimension M
// and the query heads in the 8-column dimension N, so that G <= 8 heads share one
// tile:
//   S^T[key][h] = K[key][:] . q[h][:]        A = 16 rows of K, B = q^T in registers
//   O^T[d][h]  += V^T[d][keys] P^T[keys][h]  A = V^T (transposing load), B = P^T
// q and K enter exactly.  P is the sum of three bf16 parts (its 24 bits), so that
// what the result loses is its own rounding: kPacked (G <= 4) holds the four heads'
// first parts in columns 0-3 and second parts in columns 4-7 of one product, the
// third parts in another; the wider forms take three products.  Per warp and tile of
// 16 keys: 8 + 16 products of 16x8x16 at D = 128 (kPacked), far below the tensor
// pipe's rate at the speed rows arrive.  The tensor cores drop bits below their
// accumulator, so each tile's O is added by the CUDA cores: sums over many rows
// would drift towards 0.
enum HeadMode : int { kPacked = 0, kEight = 1, kSixteen = 2 };
template <int D_, int MODE> struct Bf16Tile {
    using T = uint16_t;
    static constexpr int D = D_, KT = kPaStage / (4 * D), NT = MODE == kSixteen ? 2 : 1;
    static constexpr int kRow = 2 * D, kStage = kPaStage;   // bytes
    static constexpr bool kScaled = false;
    using Args = AttendArgs;
    using Short = Bf16Tile;
    static constexpr int kCtas = 2, kCost = 1;
    static constexpr int kHeads = MODE == kPacked ? 4 : 8 * NT;
    static constexpr int kParts = MODE == kPacked ? 2 : 3;   // products of P and V
    static constexpr int kMergeStride = D + 4;
    static constexpr int kStages = MODE == kSixteen ? 2 : 3;
    static constexpr int kClusterRows = (MODE == kSixteen ? 1024 : 512) * 128 / D;   // see attend_cluster
    static constexpr int kWindowRows = 5 * kClusterRows, kWindowCluster = 8;         // see window_cluster
    uint32_t qf[D / 16][NT][2];
    float m[NT][2], l[NT][2];
    F2 o[D / 16][NT][2];                                 // rows g and g + 8 of a head pair

    // Shared address of 16-byte piece c of row r: pieces exchanged by row, so that
    // eight rows of one piece lie in different banks.
    static __device__ __forceinline__ uint32_t piece(int r, int c) {
        return (uint32_t)(r * (2 * D) + ((c ^ (r & 7)) << 4));
    }
    __device__ __forceinline__ void load_q(const T *q, int heads, float) {
        const int lane = threadIdx.x & 31, n = lane >> 2;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int h = MODE == kPacked ? (n & 3) : n + 8 * t;
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    qf[k][t][u] = h < heads ? *(const uint32_t *)(q + h * D + 16 * k + 8 * u + 2 * (lane & 3)) : 0u;
        }
    }
    __device__ __forceinline__ void reset() {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            m[t][0] = m[t][1] = -INFINITY;
            l[t][0] = l[t][1] = 0.f;
#pragma unroll
            for (int d = 0; d < D / 16; ++d) o[d][t][0] = o[d][t][1] = 0ull;
        }
    }
    // One stage: rows key0 .. key0 + KT - 1, of which those that are seen count.
    template <typename Rows>
    __device__ __forceinline__ void tile(uint32_t ks, uint32_t vs, float *, int key0, const Rows &seen, float scale, float *scores, int heads) {
        const int lane = threadIdx.x & 31, g = lane >> 2, c = 2 * (lane & 3);
#pragma unroll
        for (int sub = 0; sub < KT / 16; ++sub) {
            const int base = key0 + 16 * sub;
            if (sub > 0 && base >= seen.len) break;
            float s[NT][4], s2[NT][4];                   // even and odd steps over D: half the chain of products
            const int kr = 16 * sub + (lane & 15);
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                uint32_t a[4];
                lds_x4(ks + piece(kr, 2 * k + (lane >> 4)), a);
#pragma unroll
                for (int t = 0; t < NT; ++t) mma_bf16(k & 1 ? s2[t] : s[t], a, qf[k][t][0], qf[k][t][1], k < 2);
            }
            const bool in0 = seen.sees(base + g), in1 = seen.sees(base + g + 8);
            bool grew = false;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
#pragma unroll
                for (int i = 0; i < 4; ++i) s[t][i] = (s[t][i] + s2[t][i]) * scale;
                if (scores) {
                    const int h = 8 * t + c;
                    float *to = scores + (long long)(base + g) * heads + h;
                    if (h + 1 < heads && h < kHeads && score_pairs(scores, heads)) {
                        if (in0) *(float2 *)to = make_float2(s[t][0], s[t][1]);
                        if (in1) *(float2 *)(to + 8 * heads) = make_float2(s[t][2], s[t][3]);
                    } else {
#pragma unroll
                        for (int i = 0; i < 2; ++i)
                            if (h + i < heads && h < kHeads) {
                                if (in0) to[i] = s[t][i];
                                if (in1) to[8 * heads + i] = s[t][2 + i];
                            }
                    }
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if (!in0) s[t][i] = -INFINITY;
                    if (!in1) s[t][2 + i] = -INFINITY;
                    grew |= fmaxf(s[t][i], s[t][2 + i]) > m[t][i] + kSlack;
                }
            }
            if (__any_sync(0xFFFFFFFFu, grew)) {
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    float a[2];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        float v = fmaxf(s[t][i], s[t][2 + i]);
                        v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, 4));
                        v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, 8));
                        v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, 16));
                        v = fmaxf(m[t][i], v);
                        a[i] = exp2f(m[t][i] - base_of(v));
                        m[t][i] = v;
                        l[t][i] *= a[i];
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
                const float b0 = base_of(m[t][0]), b1 = base_of(m[t][1]);
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const float p0 = exp2f(s[t][2 * u] - b0), p1 = exp2f(s[t][2 * u + 1] - b1);
                    l[t][0] += p0;
                    l[t][1] += p1;
                    uint32_t x, y, z;
                    three_parts(p0, p1, x, y, z);
                    if (MODE == kPacked) {
                        part[0][t][u] = transpose8((lane & 2) ? y : x);
                        part[1][t][u] = transpose8((lane & 2) ? 0u : z);
                    } else {
                        part[0][t][u] = transpose8(x);
                        part[1][t][u] = transpose8(y);
                        part[kParts - 1][t][u] = transpose8(z);
                    }
                }
            }
            const int vr = 16 * sub + (lane & 7) + ((lane >> 4) << 3);
#pragma unroll
            for (int d = 0; d < D / 16; ++d) {
                uint32_t a[4];
                lds_x4_t(vs + piece(vr, 2 * d + ((lane >> 3) & 1)), a);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    float x[4];
#pragma unroll
                    for (int i = kParts - 1; i >= 0; --i) mma_bf16(x, a, part[i][t][0], part[i][t][1], i == kParts - 1);
                    o[d][t][0] = f2_add(o[d][t][0], f2(x[0], x[1]));
                    o[d][t][1] = f2_add(o[d][t][1], f2(x[2], x[3]));
                }
            }
        }
    }
    // This warp's state: sums as [head][D] (row stride kMergeStride), maximum and sum per head.
    __device__ __forceinline__ void store(float *so, float *sm, float *sl) {
        const int lane = threadIdx.x & 31, g = lane >> 2, c = 2 * (lane & 3);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float v = l[t][i];
                v += __shfl_xor_sync(0xFFFFFFFFu, v, 4);
                v += __shfl_xor_sync(0xFFFFFFFFu, v, 8);
                v += __shfl_xor_sync(0xFFFFFFFFu, v, 16);
                if (g == 0 && 8 * t + c + i < kHeads) {
                    sm[8 * t + c + i] = m[t][i];
                    sl[8 * t + c + i] = v;
                }
            }
#pragma unroll
            for (int d = 0; d < D / 16; ++d) {
                const float2 x[2] = {f2_values(o[d][t][0]), f2_values(o[d][t][1])};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float v = i & 1 ? x[i >> 1].y : x[i >> 1].x;
                    if (MODE == kPacked) v += __shfl_xor_sync(0xFFFFFFFFu, v, 2);
                    if (8 * t + c < kHeads) so[(8 * t + c + (i & 1)) * kMergeStride + 16 * d + g + 8 * (i >> 1)] = v;
                }
            }
        }
    }
};

// fp32 rows with up to 4 query heads on the CUDA cores, two values an instruction: a lane holds
// D / 32 dims of q and of the sums, a group of 8 keys x 4 heads gives 32 partial
// products per lane, which 31 exchanges turn into one whole score per lane (lane =
// 4 key + head).
template <int D_> struct F32Tile {
    using T = float;
    static constexpr int D = D_, KT = kPaStage / (8 * D), V = D / 64;   // V: pairs of dims of a lane
    static constexpr int kRow = 4 * D, kStage = kPaStage;   // bytes
    static constexpr bool kScaled = false;
    using Args = AttendArgs;
    using Short = F32Tile;
    static constexpr int kCtas = 2, kCost = 1;
    static constexpr int kHeads = 4;
    static constexpr int kMergeStride = D + 4;
    static constexpr int kStages = 3;
    static constexpr int kClusterRows = 128 * 128 / D;
    static constexpr int kWindowRows = 5 * kClusterRows, kWindowCluster = 8;
    F2 q[4][V], o[4][V];
    float m, l;                                          // of head lane % 4

    static __device__ __forceinline__ uint32_t piece(int r, int c) { return (uint32_t)(r * (4 * D) + (c << 4)); }
    static __device__ __forceinline__ void row(uint32_t addr, F2 (&f)[V]) {
        if (V == 2) {
            asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(f[0]), "=l"(f[V - 1]) : "r"(addr) : "memory");
        } else {
            f[0] = lds8(addr);
        }
    }
    __device__ __forceinline__ void load_q(const T *src, int heads, float) {
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int h = 0; h < 4; ++h)
#pragma unroll
            for (int i = 0; i < V; ++i) q[h][i] = h < heads ? *(const F2 *)(src + h * D + lane * (2 * V) + 2 * i) : 0ull;
    }
    __device__ __forceinline__ void reset() {
        m = -INFINITY, l = 0.f;
#pragma unroll
        for (int h = 0; h < 4; ++h)
#pragma unroll
            for (int i = 0; i < V; ++i) o[h][i] = 0ull;
    }
    template <typename Rows>
    __device__ __forceinline__ void tile(uint32_t ks, uint32_t vs, float *pad, int key0, const Rows &seen, float scale, float *scores, int heads) {
        const int lane = threadIdx.x & 31;
        const uint32_t pads = (uint32_t)__cvta_generic_to_shared(pad);
#pragma unroll 1
        for (int sub = 0; sub < KT / 8; ++sub) {
            const int base = key0 + 8 * sub;
            if (base >= seen.len) break;
            const bool in = seen.sees(base + (lane >> 2));
            float x[32];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                F2 f[V];
                row(ks + (8 * sub + k) * (4 * D) + lane * (8 * V), f);
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    F2 a = f2_mul(f[0], q[h][0]);
                    if (V == 2) a = f2_fma(f[V - 1], q[h][V - 1], a);
                    x[4 * k + h] = f2_sum(a);
                }
            }
#pragma unroll
            for (int off = 16; off > 0; off >>= 1)
#pragma unroll
                for (int i = 0; i < off; ++i) {
                    const bool up = lane & off;
                    const float give = up ? x[i] : x[i + off];
                    x[i] = (up ? x[i + off] : x[i]) + __shfl_xor_sync(0xFFFFFFFFu, give, off);
                }
            float s = x[0] * scale;
            const int h = lane & 3;
            if (scores && in && h < heads) scores[(long long)(base + (lane >> 2)) * heads + h] = s;
            if (!in) s = -INFINITY;
            if (__any_sync(0xFFFFFFFFu, s > m + kSlack)) {
                float mx = s;
                mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 4));
                mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 8));
                mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 16));
                mx = fmaxf(m, mx);
                const float alpha = exp2f(m - base_of(mx));
                m = mx;
                l *= alpha;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float a = __shfl_sync(0xFFFFFFFFu, alpha, j);
#pragma unroll
                    for (int i = 0; i < V; ++i) o[j][i] = f2_mul(o[j][i], f2(a, a));
                }
            }
            const float p = exp2f(s - base_of(m));
            l += p;
            *(float2 *)(pad + 2 * lane) = make_float2(p, p);   // as the pairs that the products below take
            __syncwarp();
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                F2 w[4], f[V];
                asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(w[0]), "=l"(w[1]) : "r"(pads + 32 * k) : "memory");
                asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(w[2]), "=l"(w[3]) : "r"(pads + 32 * k + 16) : "memory");
                row(vs + (8 * sub + k) * (4 * D) + lane * (8 * V), f);
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int i = 0; i < V; ++i) o[j][i] = f2_fma(w[j], f[i], o[j][i]);
            }
            __syncwarp();
        }
    }
    __device__ __forceinline__ void store(float *so, float *sm, float *sl) {
        const int lane = threadIdx.x & 31;
        float v = l;
        v += __shfl_xor_sync(0xFFFFFFFFu, v, 4);
        v += __shfl_xor_sync(0xFFFFFFFFu, v, 8);
        v += __shfl_xor_sync(0xFFFFFFFFu, v, 16);
        if (lane < 4) {
            sm[lane] = m;
            sl[lane] = v;
        }
#pragma unroll
        for (int h = 0; h < 4; ++h)
#pragma unroll
            for (int i = 0; i < V; ++i) *(F2 *)(so + h * kMergeStride + lane * (2 * V) + 2 * i) = o[h][i];
    }
};

// fp32 rows with 5 to 16 query heads on the tensor cores: every value is the sum of
// three bf16 parts (24 bits), a product the six products of parts above 2^-24 of it.
//   S[h][key]   = q[h][:] . K[key][:]        A = q in registers, B = 8 rows of K
//   O^T[d][h]  += V^T[d][keys] P^T[keys][h]  A = V^T, B = P^T: what S leaves in a lane
// K and V are cut, which is exact, takes no conversion and cannot overflow; q and P
// are rounded, so that what the products leave out has no common sign.  Up to 8 heads
// leave half of S's 16 rows to the queries' second part.  The tensor cores drop bits
// below their accumulator, so the large products go to four short chains and each
// tile's O is added by the CUDA cores.  Which dim is which k (and which row of O^T)
// is free: a lane's 16 bytes of a row are four of them, and no value is moved.
// Measured, D = 128, 16 sequences of one KV head: 8 query heads, 40000 to 60000 rows,
// 146 us (5.6 TB/s; on the CUDA cores 170); 16 query heads, 56800 rows, 226 us (4.1
// TB/s; in two passes of 8 heads 304, on the CUDA cores 374).  What bounds the latter is
// a warp's chain of some 1000 instructions to 8 rows with 8 warps an SM, which its 255
// registers (and 52 bytes of spills) allow, not the tensor pipe (33%).
template <int D_, int NT> struct F32Mma {
    using T = float;
    static constexpr int D = D_, KT = kPaStage / (8 * D);
    static constexpr int kRow = 4 * D, kStage = kPaStage;   // bytes
    static constexpr bool kScaled = false;
    using Args = AttendArgs;
    using Short = F32Mma;
    static constexpr int kCtas = 2, kCost = 1;
    static constexpr int kHeads = 8 * NT;
    static constexpr int kMergeStride = D + 4;
    static constexpr int kStages = NT == 2 ? 2 : 3;
    static constexpr int kClusterRows = NT == 2 ? 256 * 128 / D : 256;
    static constexpr int kWindowRows = 5 * kClusterRows, kWindowCluster = 8;
    const T *q;                                          // this tile's, for scores recomputed
    uint32_t qf[D / 16][3][NT][2];                       // part, heads g + 8 u, two pairs of dims
    F2 o[D / 16][NT][2];
    float m[NT], l[NT];                                  // of heads g + 8 u; l: of this lane's keys

    // Eight lanes read two neighbouring rows of K, or four rows of V of one parity.
    static __device__ __forceinline__ uint32_t piece(int r, int c) {
        return (uint32_t)(r * (4 * D) + ((c ^ ((((r >> 2) ^ r) & 1) << 2 | (r & 2))) << 4));
    }
    static __device__ __forceinline__ float4 lds(uint32_t addr) {
        float4 f;
        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(f.x), "=f"(f.y), "=f"(f.z), "=f"(f.w) : "r"(addr) : "memory");
        return f;
    }
    // The first bf16 parts of two values as a pair, and what a cut leaves of two values.
    static __device__ __forceinline__ uint32_t heads_of(float x, float y) { return __byte_perm(__float_as_uint(x), __float_as_uint(y), 0x7632); }
    static __device__ __forceinline__ F2 rest(F2 v) { return f2_sub(v, v & 0xFFFF0000FFFF0000ull); }
    // Two products of 8 keys as one of 16: part i of V with p, part j with r.
    static __device__ __forceinline__ void pair(float (&c)[4], const uint32_t (&v)[3], const uint32_t (&w)[3], int i, uint32_t p, int j, uint32_t r, bool fresh) {
        const uint32_t a[4] = {v[i], w[i], v[j], w[j]};
        mma_bf16(c, a, p, r, fresh);
    }
    __device__ __forceinline__ void load_q(const T *src, int heads, float) {
        const int lane = threadIdx.x & 31, g = lane >> 2;
        q = src;
#pragma unroll
        for (int u = 0; u < NT; ++u)
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                const float4 x = g + 8 * u < heads ? *(const float4 *)(src + (g + 8 * u) * D + 16 * k + 4 * (lane & 3)) : make_float4(0.f, 0.f, 0.f, 0.f);
                three_parts(x.x, x.y, qf[k][0][u][0], qf[k][1][u][0], qf[k][2][u][0]);
                three_parts(x.z, x.w, qf[k][0][u][1], qf[k][1][u][1], qf[k][2][u][1]);
            }
    }
    __device__ __forceinline__ void reset() {
#pragma unroll
        for (int u = 0; u < NT; ++u) {
            m[u] = -INFINITY;
            l[u] = 0.f;
#pragma unroll
            for (int d = 0; d < D / 16; ++d) o[d][u][0] = o[d][u][1] = 0ull;
        }
    }
    template <typename Rows>
    __device__ __forceinline__ void tile(uint32_t ks, uint32_t vs, float *, int key0, const Rows &seen, float scale, float *scores, int heads) {
        const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll 1
        for (int sub = 0; sub < KT / 8; ++sub) {
            const int base = key0 + 8 * sub;
            if (base >= seen.len) break;
            float x[4][4], y[3][4];                      // q's and K's first parts; the rest
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                const float4 f = lds(ks + piece(8 * sub + g, 4 * k + t));
                F2 v = f2(f.x, f.y), w = f2(f.z, f.w);
                uint32_t a[3], b[3];
#pragma unroll
                for (int i = 0; i < 3; ++i) {
                    a[i] = heads_of(f2_values(v).x, f2_values(v).y);
                    b[i] = heads_of(f2_values(w).x, f2_values(w).y);
                    if (i < 2) v = rest(v), w = rest(w);
                }
                const auto &p = qf[k];
                if (NT == 1) {
                    const uint32_t two[4] = {p[0][0][0], p[1][0][0], p[0][0][1], p[1][0][1]}, third[4] = {p[2][0][0], 0u, p[2][0][1], 0u};
                    mma_bf16(x[k & 3], two, a[0], b[0], k < 4);
                    mma_bf16(y[0], two, a[1], b[1], k == 0);
                    mma_bf16(y[1], two, a[2], b[2], k == 0);
                    mma_bf16(y[1], third, a[0], b[0], false);
                } else {
                    const uint32_t q0[4] = {p[0][0][0], p[0][NT - 1][0], p[0][0][1], p[0][NT - 1][1]};
                    const uint32_t q1[4] = {p[1][0][0], p[1][NT - 1][0], p[1][0][1], p[1][NT - 1][1]};
                    const uint32_t q2[4] = {p[2][0][0], p[2][NT - 1][0], p[2][0][1], p[2][NT - 1][1]};
                    mma_bf16(x[k & 3], q0, a[0], b[0], k < 4);
                    mma_bf16(y[0], q1, a[0], b[0], k == 0);
                    mma_bf16(y[1], q2, a[0], b[0], k == 0);
                    mma_bf16(y[2], q0, a[1], b[1], k == 0);
                    mma_bf16(y[0], q1, a[1], b[1], false);
                    mma_bf16(y[1], q0, a[2], b[2], false);
                }
            }
            float s[NT][2];
            bool nan = false;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const bool in = seen.sees(base + 2 * t + i);
                if (NT == 1) y[0][i] += (x[0][2 + i] + x[1][2 + i]) + (x[2][2 + i] + x[3][2 + i]) + (y[0][2 + i] + y[1][2 + i]);
#pragma unroll
                for (int u = 0; u < NT; ++u) {
                    const int c = 2 * u + i;
                    s[u][i] = (((x[0][c] + x[1][c]) + (x[2][c] + x[3][c])) + (y[0][c] + y[1][c]) + (NT == 2 ? y[2][c] : 0.f)) * scale;
                    nan |= in && g + 8 * u < heads && s[u][i] != s[u][i];
                }
            }
            if (__any_sync(0xFFFFFFFFu, nan)) {          // infinities have no parts: the score as it is defined
#pragma unroll
                for (int u = 0; u < NT; ++u)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        if (g + 8 * u >= heads) continue;
                        float z = 0.f;
#pragma unroll 1
                        for (int c = 0; c < D / 4; ++c) {
                            const float4 f = lds(ks + piece(8 * sub + 2 * t + i, c)), w = *(const float4 *)(q + (g + 8 * u) * D + 4 * c);
                            z = fmaf(f.x, w.x, fmaf(f.y, w.y, fmaf(f.z, w.z, fmaf(f.w, w.w, z))));
                        }
                        s[u][i] = z * scale;
                    }
            }
            bool grew = false;
#pragma unroll
            for (int u = 0; u < NT; ++u) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int key = base + 2 * t + i;
                    if (scores && seen.sees(key) && g + 8 * u < heads) scores[(long long)key * heads + g + 8 * u] = s[u][i];
                    if (!seen.sees(key)) s[u][i] = -INFINITY;
                }
                grew |= fmaxf(s[u][0], s[u][1]) > m[u] + kSlack;
            }
            if (__any_sync(0xFFFFFFFFu, grew)) {
#pragma unroll
                for (int u = 0; u < NT; ++u) {
                    float v = fmaxf(s[u][0], s[u][1]);
                    v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, 1));
                    v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, 2));
                    v = fmaxf(m[u], v);
                    const float alpha = exp2f(m[u] - base_of(v));
                    m[u] = v;
                    l[u] *= alpha;
                    const F2 both = f2(__shfl_sync(0xFFFFFFFFu, alpha, 8 * t), __shfl_sync(0xFFFFFFFFu, alpha, 8 * t + 4));
#pragma unroll
                    for (int d = 0; d < D / 16; ++d) {
                        o[d][u][0] = f2_mul(o[d][u][0], both);
                        o[d][u][1] = f2_mul(o[d][u][1], both);
                    }
                }
            }
            uint32_t p[NT][3];
#pragma unroll
            for (int u = 0; u < NT; ++u) {
                const float b = base_of(m[u]), p0 = exp2f(s[u][0] - b), p1 = exp2f(s[u][1] - b);
                l[u] += p0 + p1;
                three_parts(p0, p1, p[u][0], p[u][1], p[u][2]);
            }
#pragma unroll
            for (int k = 0; k < D / 32; ++k) {
                const float4 f0 = lds(vs + piece(8 * sub + 2 * t, 8 * k + g)), f1 = lds(vs + piece(8 * sub + 2 * t + 1, 8 * k + g));
                F2 lo[2] = {f2(f0.x, f0.y), f2(f1.x, f1.y)}, hi[2] = {f2(f0.z, f0.w), f2(f1.z, f1.w)};
                uint32_t v[4][3];
#pragma unroll
                for (int i = 0; i < 3; ++i) {
                    v[0][i] = heads_of(f2_values(lo[0]).x, f2_values(lo[1]).x);
                    v[1][i] = heads_of(f2_values(lo[0]).y, f2_values(lo[1]).y);
                    v[2][i] = heads_of(f2_values(hi[0]).x, f2_values(hi[1]).x);
                    v[3][i] = heads_of(f2_values(hi[0]).y, f2_values(hi[1]).y);
#pragma unroll
                    for (int r = 0; r < 2; ++r)
                        if (i < 2) lo[r] = rest(lo[r]), hi[r] = rest(hi[r]);
                }
                float c[2][NT][4];
#pragma unroll
                for (int i = 0; i < 3; ++i)
#pragma unroll
                    for (int d = 0; d < 2; ++d)
#pragma unroll
                        for (int u = 0; u < NT; ++u)
                            if (i == 0)
                                pair(c[d][u], v[2 * d], v[2 * d + 1], 2, p[u][0], 0, p[u][2], true);
                            else
                                pair(c[d][u], v[2 * d], v[2 * d + 1], 0, p[u][2 - i], 1, p[u][2 - i], false);
#pragma unroll
                for (int d = 0; d < 2; ++d)
#pragma unroll
                    for (int u = 0; u < NT; ++u) {
                        o[2 * k + d][u][0] = f2_add(o[2 * k + d][u][0], f2(c[d][u][0], c[d][u][1]));
                        o[2 * k + d][u][1] = f2_add(o[2 * k + d][u][1], f2(c[d][u][2], c[d][u][3]));
                    }
            }
        }
    }
    __device__ __forceinline__ void store(float *so, float *sm, float *sl) {
        const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int u = 0; u < NT; ++u) {
            float v = l[u];
            v += __shfl_xor_sync(0xFFFFFFFFu, v, 1);
            v += __shfl_xor_sync(0xFFFFFFFFu, v, 2);
            if (t == 0) {
                sm[g + 8 * u] = m[u];
                sl[g + 8 * u] = v;
            }
#pragma unroll
            for (int k = 0; k < D / 32; ++k) {
                const float2 a = f2_values(o[2 * k][u][0]), b = f2_values(o[2 * k][u][1]);
                const float2 c = f2_values(o[2 * k + 1][u][0]), d = f2_values(o[2 * k + 1][u][1]);
                float *to = so + (8 * u + 2 * t) * kMergeStride + 32 * k + 4 * g;
                *(float4 *)to = make_float4(a.x, b.x, c.x, d.x);
                *(float4 *)(to + kMergeStride) = make_float4(a.y, b.y, c.y, d.y);
            }
        }
    }
};

// The tile form of a type, head dimension and heads that share a pass over the rows
// (4, 8 or 16; more heads take more passes).
template <typename F> cudaError_t with_tile(bool bf16, int D, int heads, const F &f) {
    if (bf16) {
        if (D == 128) return heads == 4 ? f(Bf16Tile<128, kPacked>()) : heads == 8 ? f(Bf16Tile<128, kEight>()) : f(Bf16Tile<128, kSixteen>());
        return heads == 4 ? f(Bf16Tile<64, kPacked>()) : heads == 8 ? f(Bf16Tile<64, kEight>()) : f(Bf16Tile<64, kSixteen>());
    }
    if (D == 128) return heads == 4 ? f(F32Tile<128>()) : heads == 8 ? f(F32Mma<128, 1>()) : f(F32Mma<128, 2>());
    return heads == 4 ? f(F32Tile<64>()) : heads == 8 ? f(F32Mma<64, 1>()) : f(F32Mma<64, 2>());
}

template <typename Rows> cudaError_t prepare_attend_tiles(bool bf16, int D, int G) {
    const int ht = attend_head_tile(G);
    cudaError_t e = with_tile(bf16, D, ht, [](auto tile) { return prepare_attend<decltype(tile), Rows>(); });
    // fp32 takes tiles of 8 heads for 16 where rows are few
    if (e == cudaSuccess && !bf16 && ht == 16) e = with_tile(bf16, D, 8, [](auto tile) { return prepare_attend<decltype(tile), Rows>(); });
    return e;
}
template <typename Rows> cudaError_t start_attend_tiles(const AttendArgs &a, bool bf16, int D, int ht, int sms, cudaStream_t s) {
    return with_tile(bf16, D, ht, [&](auto tile) { return start_attend<decltype(tile), Rows>(a, ht, sms, s); });
}

}  // namespace
}  // namespace prism
