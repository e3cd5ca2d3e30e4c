// Attention of one new token per sequence over a paged key-value cache.
//
//   z_j = scale * q_h . k_j,  p_j = exp(z_j) / sum_i exp(z_i),  out_h = sum_j p_j v_j
//
// over the rows j < kv_len[b] + added of sequence b, for the G = Hq / Hkv query
// heads h of each KV head; optionally lse_h = log sum_j exp(z_j), and the
// accumulated weights w_j += sum_h p_j that eviction ranks by.
//
// Bound by the bytes of K and V, read once up to G = 16 (more query heads read them
// once for every 16, fp32 tables of few rows once for every 8): 4 D bytes per row and
// KV head in bf16 against 4 G D operations (G a byte: far below what the tensor cores'
// warp-level products give at N = 8 or 16, too few columns for a 128-row tensor-memory
// tile).  Measured, bf16, D = 128: 64 sequences of 6001 to 16384 rows, G = 8, 427 to 433
// us (6.8 TB/s, the rate of a plain copy); one of 131071 rows, G = 4, 85 us (6.3 TB/s);
// 8 multi-head ones of 2048 to 4096 rows 65 us (6.2); 16 of 1 to 8192 rows with weights
// 53 us (5.2); one of 517 rows 5.9 us, a chain of length, table and row loads and the
// join; 16 of 56800 rows with one KV head, G = 16, 90 us (5.2); the same of D = 64, G = 32,
// 95 us (4.9 TB/s of rows read twice).  fp32: one of 131071 rows, G = 4, 160 us (6.7
// TB/s).  A large call costs some 8 us beside its bytes: 4 until the first rows arrive,
// the rest the spread of the SMs' speeds (6% by their place on the chip) and the last join.
#include "paged.cuh"
#include "paged_scores.h"

namespace prism {
namespace {

constexpr int kPaWarps = 4;
constexpr int kPaThreads = 32 * kPaWarps;
constexpr int kPaStage = 8192;           // bytes of one warp's stage: KT rows of K, then of V
constexpr int kPaCtasPerSm = 2;
constexpr float kLn2 = 0.693147180559945309f;

__device__ __forceinline__ void lds_x4(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void lds_x4_t(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
// c += a b, or a b on its own.
__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, bool fresh) {
    if (fresh)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
            : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Two values as three bf16 parts each, rounded: their sum is the value.
__device__ __forceinline__ void three_parts(float x, float y, uint32_t &p0, uint32_t &p1, uint32_t &p2) {
    p0 = cvt_bf16x2(x, y);
    x -= bf16lo(p0), y -= bf16hi(p0);
    p1 = cvt_bf16x2(x, y);
    p2 = cvt_bf16x2(x - bf16lo(p1), y - bf16hi(p1));
}

// What a warp subtracts from its scores is a maximum it has met, renewed (and its sums
// rescaled) only when a score passes it by more than this: probabilities stay below
// 2^8 times the largest, and most tiles need no exchange between lanes.
constexpr float kSlack = 8.f;
// The maximum to subtract: 0 where no score is above -inf (every exp2 is then 0).
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.f : m; }

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
    static constexpr int kHeads = MODE == kPacked ? 4 : 8 * NT;
    static constexpr int kParts = MODE == kPacked ? 2 : 3;   // products of P and V
    static constexpr int kMergeStride = D + 4;
    static constexpr int kStages = MODE == kSixteen ? 2 : 3;
    static constexpr int kClusterRows = (MODE == kSixteen ? 1024 : 512) * 128 / D;   // see attend_cluster
    uint32_t qf[D / 16][NT][2];
    float m[NT][2], l[NT][2];
    F2 o[D / 16][NT][2];                                 // rows g and g + 8 of a head pair

    // Shared address of 16-byte piece c of row r: pieces exchanged by row, so that
    // eight rows of one piece lie in different banks.
    static __device__ __forceinline__ uint32_t piece(int r, int c) {
        return (uint32_t)(r * (2 * D) + ((c ^ (r & 7)) << 4));
    }
    __device__ __forceinline__ void load_q(const T *q, int heads) {
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
    // One stage: rows key0 .. key0 + KT - 1, of which those below len count.
    __device__ __forceinline__ void tile(uint32_t ks, uint32_t vs, float *, int key0, int len, float scale, float *scores, int heads) {
        const int lane = threadIdx.x & 31, g = lane >> 2, c = 2 * (lane & 3);
#pragma unroll
        for (int sub = 0; sub < KT / 16; ++sub) {
            const int base = key0 + 16 * sub;
            if (sub > 0 && base >= len) break;
            float s[NT][4], s2[NT][4];                   // even and odd steps over D: half the chain of products
            const int kr = 16 * sub + (lane & 15);
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                uint32_t a[4];
                lds_x4(ks + piece(kr, 2 * k + (lane >> 4)), a);
#pragma unroll
                for (int t = 0; t < NT; ++t) mma_bf16(k & 1 ? s2[t] : s[t], a, qf[k][t][0], qf[k][t][1], k < 2);
            }
            const bool in0 = base + g < len, in1 = base + g + 8 < len;
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
    static constexpr int kHeads = 4;
    static constexpr int kMergeStride = D + 4;
    static constexpr int kStages = 3;
    static constexpr int kClusterRows = 128 * 128 / D;
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
    __device__ __forceinline__ void load_q(const T *src, int heads) {
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
    __device__ __forceinline__ void tile(uint32_t ks, uint32_t vs, float *pad, int key0, int len, float scale, float *scores, int heads) {
        const int lane = threadIdx.x & 31;
        const uint32_t pads = (uint32_t)__cvta_generic_to_shared(pad);
#pragma unroll 1
        for (int sub = 0; sub < KT / 8; ++sub) {
            const int base = key0 + 8 * sub;
            if (base >= len) break;
            const bool in = base + (lane >> 2) < len;
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
    static constexpr int kHeads = 8 * NT;
    static constexpr int kMergeStride = D + 4;
    static constexpr int kStages = NT == 2 ? 2 : 3;
    static constexpr int kClusterRows = NT == 2 ? 256 * 128 / D : 256;
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
    __device__ __forceinline__ void load_q(const T *src, int heads) {
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
    __device__ __forceinline__ void tile(uint32_t ks, uint32_t vs, float *, int key0, int len, float scale, float *scores, int heads) {
        const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll 1
        for (int sub = 0; sub < KT / 8; ++sub) {
            const int base = key0 + 8 * sub;
            if (base >= len) break;
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
                const bool in = base + 2 * t + i < len;
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
                    if (scores && key < len && g + 8 * u < heads) scores[(long long)key * heads + g + 8 * u] = s[u][i];
                    if (key >= len) s[u][i] = -INFINITY;
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

// A segment is one (sequence, KV head, head tile): blocks of kAttendUnit keys, and
// before them kAttendCost units without keys that stand for what a segment costs
// beside its rows (its queries, merge and result).
__device__ __forceinline__ int blocks_of(int len) { return max(1, (len + kAttendUnit - 1) / kAttendUnit); }
__device__ __forceinline__ int units_of(int len) { return kAttendCost + blocks_of(len); }

// Walk over the pieces of a CTA's share: the blocks [blk0, blk1) of nblk of one
// segment after the other; parts of a segment without blocks are passed over.  Each
// lane keeps the length of one of the next 32 sequences, so that a step waits for
// no load.
struct Pieces {
    int u, u1, seg, b, h, heads, blk0, blk1, nblk, len;   // seg: the segment's first unit
    int base, lens;                      // lane i: rows of sequence base + i
    __device__ __forceinline__ void fetch(const AttendArgs &a) {
        const int at = b + (int)(threadIdx.x & 31);
        base = b;
        lens = at < a.B ? paged_len(a.cache, at, a.added, a.err) : 0;
    }
    __device__ __forceinline__ void sequence() {
        len = __shfl_sync(0xFFFFFFFFu, lens, b - base);
        nblk = blocks_of(len);
    }
    __device__ __forceinline__ bool cut() {
        blk0 = max(u - seg - kAttendCost, 0);
        u = min(seg + kAttendCost + nblk, u1);
        blk1 = max(u - seg - kAttendCost, 0);
        return blk0 < blk1;
    }
    __device__ __forceinline__ bool begin(const AttendArgs &a, const UnitRange &r, int n_heads) {
        u = r.u0;
        u1 = r.u1;
        b = r.b;
        heads = n_heads;
        if (a.B <= 32) {
            base = 0;
            lens = r.lens;
        } else {
            fetch(a);
        }
        sequence();
        h = (u - r.first) / (kAttendCost + nblk);
        seg = r.first + h * (kAttendCost + nblk);
        return cut() || next(a);
    }
    // A cluster's rank takes its run of the blocks of segment i, and no other piece.
    __device__ __forceinline__ void only(const AttendArgs &a, int i, int rank, int n_heads) {
        u = u1 = seg = base = lens = 0;
        heads = n_heads;
        b = i / heads;
        h = i - b * heads;
        len = paged_len(a.cache, b, a.added, a.err);
        nblk = blocks_of(len);
        const int share = (nblk + a.cluster - 1) / a.cluster;
        blk0 = min(nblk, rank * share);
        blk1 = min(nblk, blk0 + share);
    }
    __device__ __forceinline__ bool next(const AttendArgs &a) {
        while (u < u1) {
            seg = u;
            if (++h == heads) {
                h = 0;
                if (++b - base == 32) fetch(a);
                sequence();
            }
            if (cut()) return true;
        }
        return false;
    }
    __device__ __forceinline__ int rows() const { return min(blk1 * kAttendUnit, len) - blk0 * kAttendUnit; }
};

// Writes the result of heads h0 .. of one segment from its sums, maxima and totals.
template <typename T, int D>
__device__ __forceinline__ void write_out(const AttendArgs &a, long long hq, int d, const float (&x)[4], float m, float l) {
    const float inv = l == 0.f ? 0.f : 1.f / l;          // no rows (or none above -inf): zeros
    T *o = (T *)a.out + hq * D + d;
    if (sizeof(T) == 2) {
        *(uint2 *)o = make_uint2(cvt_bf16x2(x[0] * inv, x[1] * inv), cvt_bf16x2(x[2] * inv, x[3] * inv));
    } else {
        *(float4 *)o = make_float4(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
    }
    if (d == 0) {
        if (a.lse) a.lse[hq] = l == 0.f ? -INFINITY : base_of(m) * kLn2 + logf(l);
        if (a.stat) a.stat[hq] = make_float2(base_of(m), inv);
    }
}

// A segment cut between CTAs c0, c0 + 1, ...: piece i lies in CTA c0 + i's slot (its
// second for the segment's first piece, a CTA's last piece; else its first).  Pieces
// are joined in groups, groups in one more step.
struct Cut {
    int b, h, c0, pieces;
    __device__ __forceinline__ int slot(int i) const { return i == 0 ? 2 * c0 + 1 : 2 * (c0 + i); }
    __device__ __forceinline__ int in_group(int g, int size) const { return min(size, pieces - g * size); }
};

// Pieces added in their order: thread t has columns t, t + kPaThreads, ... of the
// [H][D / 4] float4 sums, with their heads' maxima and sums.
template <typename P> struct Joined {
    static constexpr int D = P::D, H = P::kHeads, kPart = H * (D + 2);
    static constexpr int kRound = kPaWarps * P::kStages * kPaStage / (4 * kPart);   // pieces that the rings hold
    static constexpr int kGroup = kRound > 16 ? kRound : 16;
    static constexpr int kCols = H * D / 4 / kPaThreads > 0 ? H * D / 4 / kPaThreads : 1;
    float x[kCols][4], M[kCols], L[kCols];

    template <typename Slot>
    __device__ __forceinline__ void add(unsigned char *rings, const float *part, int n, int pieces, const Slot &slot) {
        const int tid = threadIdx.x;
        const uint32_t buf = (uint32_t)__cvta_generic_to_shared(rings);
        const float *got = (const float *)rings;
#pragma unroll
        for (int c = 0; c < kCols; ++c) {
            M[c] = -INFINITY;
            L[c] = x[c][0] = x[c][1] = x[c][2] = x[c][3] = 0.f;
        }
        for (int i0 = 0; i0 < pieces; i0 += kRound) {
            const int count = min(kRound, pieces - i0);
            for (int e = tid; e < count * (kPart / 4); e += kPaThreads) {
                const int i = e / (kPart / 4);
                cp16(buf + e * 16, part + (long long)slot(i0 + i) * kPart + (e - i * (kPart / 4)) * 4, true);
            }
            cp_group();
            cp_wait_group<0>();
            __syncthreads();
#pragma unroll
            for (int c = 0; c < kCols; ++c) {
                const int e = tid + c * kPaThreads, h = e / (D / 4);
                if (h >= n) continue;
                float top = M[c];
                for (int i = 0; i < count; ++i) top = fmaxf(top, got[i * kPart + H * D + 2 * h]);
                const float base = base_of(top), old = exp2f(M[c] - base);
                M[c] = top;
                L[c] *= old;
#pragma unroll
                for (int d = 0; d < 4; ++d) x[c][d] *= old;
#pragma unroll 4
                for (int i = 0; i < count; ++i) {
                    const float2 ml = *(const float2 *)(got + i * kPart + H * D + 2 * h);
                    const float4 y = *(const float4 *)(got + i * kPart + e * 4);
                    const float f = exp2f(ml.x - base);
                    L[c] = fmaf(f, ml.y, L[c]);
                    x[c][0] = fmaf(f, y.x, x[c][0]);
                    x[c][1] = fmaf(f, y.y, x[c][1]);
                    x[c][2] = fmaf(f, y.z, x[c][2]);
                    x[c][3] = fmaf(f, y.w, x[c][3]);
                }
            }
            __syncthreads();                             // the pieces were read
        }
    }
    __device__ __forceinline__ void store(float *part, int n) const {
#pragma unroll
        for (int c = 0; c < kCols; ++c) {
            const int e = threadIdx.x + c * kPaThreads, h = e / (D / 4);
            if (h >= n) continue;
            __stcg((float4 *)part + e, make_float4(x[c][0], x[c][1], x[c][2], x[c][3]));
            if (e % (D / 4) == 0) __stcg((float2 *)(part + H * D + 2 * h), make_float2(M[c], L[c]));
        }
    }
    __device__ __forceinline__ void write(const AttendArgs &a, long long hq, int n) const {
#pragma unroll
        for (int c = 0; c < kCols; ++c) {
            const int e = threadIdx.x + c * kPaThreads, h = e / (D / 4);
            if (h < n) write_out<typename P::T, D>(a, hq + h, 4 * (e % (D / 4)), x[c], M[c], L[c]);
        }
    }
};

template <typename P> constexpr size_t attend_smem() {
    return (size_t)kPaWarps * (P::kStages * kPaStage + 4 * P::kHeads * (P::kMergeStride + 2));
}

// Persistent CTAs of four warps, two per SM.  The ragged (sequence, KV head,
// block of 64 keys) units are cut into equal contiguous shares, one per CTA, so
// that long and short sequences keep every SM equally busy; a segment cut between
// CTAs is joined by the last of them to finish (in CTA order: the result does not
// depend on which that is).  Within a CTA the tiles of KT keys go to the warps in
// turn, each with its own ring of stages filled by cp.async, its own online
// softmax and no barrier until the segment's end; the ring runs on across
// segments, so loads never stop.
//
// CLUSTER, for few short segments: a cluster of a.cluster CTAs takes one segment,
// each an equal run of its blocks, and joins through distributed shared memory
// instead of tickets and loads from L2.
template <typename P, bool CLUSTER>
__global__ void __launch_bounds__(kPaThreads, kPaCtasPerSm) paged_attend_kernel(AttendArgs a) {
    using T = typename P::T;
    constexpr int D = P::D, KT = P::KT, S = P::kStages, H = P::kHeads;
    constexpr int kPart = Joined<P>::kPart, kGroup = Joined<P>::kGroup;   // kPart: sums [H][D], then (maximum, sum) [H]
    constexpr int kRow = D * (int)sizeof(T), kChunks = kRow / 16, kRowsPer = 32 / kChunks;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ Cut joins[2];
    __shared__ int join_group[2], last;
    int pending = 0;                                     // of thread 0
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    pdl_wait();
    pdl_trigger();

    const int G = a.Hq / a.Hkv, tiles = (G + H - 1) / H, heads = a.Hkv * tiles;
    UnitRange r;
    Pieces p;                                            // the piece being computed
    const int rank = CLUSTER ? (int)blockIdx.x % a.cluster : 0;
    if (CLUSTER) {
        p.only(a, blockIdx.x / a.cluster, rank, heads);
    } else {
        if (!unit_range<kPaThreads>(r, a.B, heads,
                                    [&](int b) { return paged_len(a.cache, b, a.added, a.err); }, units_of))
            return;
        if (!p.begin(a, r, heads)) return;
    }

    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + warp * (S * kPaStage);
    float *merge = (float *)(smem + kPaWarps * S * kPaStage);                       // [warps][H][stride]
    float *sm = merge + kPaWarps * H * P::kMergeStride, *sl = sm + kPaWarps * H;    // [warps][H]
    float *own = merge + warp * H * P::kMergeStride;     // this warp's share, scratch until the segment's end

    // Loads run ahead of the computation: their own walk, and the pool place of each
    // lane's row of the next two tiles, so that no load waits for a block-table entry.
    Pieces f = p;
    int ft = warp;
    bool more = true;
    while (more && ft * KT >= f.rows()) more = f.next(a);
    struct Place {
        int page, row, head;
        bool in, live;
    };
    auto look_up = [&]() {                               // lane's row of the walk's tile (lanes past KT repeat), then on
        Place w{0, 0, f.h / tiles, false, more};
        if (!more) return w;
        const int key = f.blk0 * kAttendUnit + ft * KT + (lane % KT);
        const int slot = (unsigned)key / (unsigned)a.cache.page_size;
        w.in = key < f.len;
        w.row = key - slot * a.cache.page_size;
        if (w.in) w.page = a.cache.table[(long long)f.b * a.cache.table_pages + slot];
        ft += kPaWarps;
        while (more && ft * KT >= f.rows()) {
            more = f.next(a);
            ft = warp;
        }
        return w;
    };
    Place next0 = look_up(), next1 = look_up();
    int stage_in = 0;
    // K and V leave L2 first, so that scores, weights and pieces stay for the next reader
    // (up to 16 query heads a KV head read them once; the next head tile of more reads them again)
    const uint64_t once = l2_evict_first_policy();
    auto issue = [&]() {
        if (next0.live) {
            const bool known = (unsigned)next0.page < (unsigned)a.cache.n_pages;
            if (next0.in && !known) set_err(a.err, kErrPage);
            const int ok = next0.in && known;
            const long long off = ok ? next0.page * a.cache.page_stride + next0.head * a.cache.head_stride + next0.row * a.cache.row_stride : 0;
            const uint32_t ks = ring + stage_in * kPaStage, vs = ks + kPaStage / 2;
            const int c = lane % kChunks;
#pragma unroll
            for (int i = 0; i < KT / kRowsPer; ++i) {
                const int row = i * kRowsPer + lane / kChunks;
                const long long at = __shfl_sync(0xFFFFFFFFu, off, row) + 16 * c;
                const bool in = __shfl_sync(0xFFFFFFFFu, ok, row);
                cp16_once(ks + P::piece(row, c), a.cache.k + at, in, once);
                cp16_once(vs + P::piece(row, c), a.cache.v + at, in, once);
            }
        }
        cp_group();
        next0 = next1;
        next1 = look_up();
        stage_in = stage_in + 1 == S ? 0 : stage_in + 1;
    };
#pragma unroll
    for (int i = 0; i < S - 1; ++i) issue();

    int stage = 0;
    P state;
    bool go = true;
    auto first_head = [&](const Pieces &w) { return (long long)w.b * a.Hq + w.h / tiles * G + w.h % tiles * H; };
    auto head_count = [&](const Pieces &w) { return min(H, G - w.h % tiles * H); };
    state.load_q((const T *)a.q + first_head(p) * D, head_count(p));
    while (go) {
        const int kvh = p.h / tiles, h0 = (p.h % tiles) * H, n = head_count(p);
        const long long hq = first_head(p);
        state.reset();
        float *scores = a.scores ? a.scores + score_place(p.b, kvh, h0, a.Hkv, G, (long long)a.cache.table_pages * a.cache.page_size) : nullptr;
        const int rows = p.rows();
        for (int t = warp; t * KT < rows; t += kPaWarps) {
            cp_wait_group<S - 2>();
            __syncwarp();
            issue();
            const uint32_t ks = ring + stage * kPaStage;
            state.tile(ks, ks + kPaStage / 2, own, p.blk0 * kAttendUnit + t * KT, p.len, a.scale_log2, scores, n);
            stage = stage + 1 == S ? 0 : stage + 1;
        }
        Pieces after = p;
        go = after.next(a);
        if (go) state.load_q((const T *)a.q + first_head(after) * D, head_count(after));   // on its way during the merge
        state.store(own, sm + warp * H, sl + warp * H);
        __syncthreads();
        const bool whole = p.blk0 == 0 && p.blk1 == p.nblk;
        const int first = p.seg + kAttendCost;           // unit of the segment's first block
        const int c0 = CLUSTER ? 0 : first / r.per, c1 = CLUSTER ? 0 : (first + p.nblk - 1) / r.per;
        const int slot = 2 * blockIdx.x + (p.blk0 == 0 ? 1 : 0);
        float *part = a.part + (long long)slot * kPart;
        for (int e = tid; e < n * (D / 4); e += kPaThreads) {
            const int h = e / (D / 4), d = 4 * (e % (D / 4));
            float M = -INFINITY;
#pragma unroll
            for (int w = 0; w < kPaWarps; ++w) M = fmaxf(M, sm[w * H + h]);
            const float base = base_of(M);
            float x[4] = {0.f, 0.f, 0.f, 0.f}, L = 0.f;
#pragma unroll
            for (int w = 0; w < kPaWarps; ++w) {
                const float k = exp2f(sm[w * H + h] - base);
                const float4 y = *(const float4 *)(merge + (w * H + h) * P::kMergeStride + d);
                L = fmaf(k, sl[w * H + h], L);
                x[0] = fmaf(k, y.x, x[0]);
                x[1] = fmaf(k, y.y, x[1]);
                x[2] = fmaf(k, y.z, x[2]);
                x[3] = fmaf(k, y.w, x[3]);
            }
            if (!CLUSTER && whole) {
                write_out<T, D>(a, hq + h, d, x, M, L);
            } else if (CLUSTER) {                        // for the other ranks, where the rings were
                *(float4 *)((float *)smem + h * D + d) = make_float4(x[0], x[1], x[2], x[3]);
                if (d == 0) *(float2 *)((float *)smem + H * D + 2 * h) = make_float2(M, L);
            } else {
                __stcg((float4 *)(part + h * D + d), make_float4(x[0], x[1], x[2], x[3]));
                if (d == 0) {
                    __stcg(part + H * D + 2 * h, M);
                    __stcg(part + H * D + 2 * h + 1, L);
                }
            }
        }
        if (CLUSTER) {
            cluster_sync_all();
            // each rank joins its columns, the ranks' sums in their order
            for (int e = rank + a.cluster * tid; e < n * (D / 4); e += a.cluster * kPaThreads) {
                const int h = e / (D / 4), d = 4 * (e % (D / 4));
                float4 y[8];
                float2 ml[8];
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (k < a.cluster) {
                        dsmem_ld((float *)smem + h * D + d, k, y[k]);
                        dsmem_ld((float *)smem + H * D + 2 * h, k, ml[k]);
                    }
                float M = -INFINITY, x[4] = {0.f, 0.f, 0.f, 0.f}, L = 0.f;
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (k < a.cluster) M = fmaxf(M, ml[k].x);
                const float base = base_of(M);
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (k < a.cluster) {
                        const float f = exp2f(ml[k].x - base);
                        L = fmaf(f, ml[k].y, L);
                        x[0] = fmaf(f, y[k].x, x[0]);
                        x[1] = fmaf(f, y[k].y, x[1]);
                        x[2] = fmaf(f, y[k].z, x[2]);
                        x[3] = fmaf(f, y[k].w, x[3]);
                    }
                write_out<T, D>(a, hq + h, d, x, M, L);
            }
            cluster_sync_all();                          // no CTA leaves while another reads its sums
            return;
        }
        __syncthreads();                                 // the piece is written; the merge area is free again
        if (!whole && tid == 0) {
            const Cut cut{p.b, p.h, c0, c1 - c0 + 1};
            const int g = (blockIdx.x - c0) / kGroup;
            __threadfence();
            int *ticket = a.group_counter + cut.slot(g * kGroup);
            if (atomicAdd(ticket, 1) == cut.in_group(g, kGroup) - 1) {
                __threadfence();
                *ticket = 0;
                joins[pending] = cut;
                join_group[pending++] = g;
            }
        }
        p = after;
    }
    // Groups of which this CTA finished the last piece (of its first and its last
    // segment at most), joined now that the rings are free to take the pieces, all of
    // them on their way at once; the last group of a segment joins the groups.
    cp_wait_group<0>();
    if (tid == 0 && pending < 2) join_group[pending] = -1;
    __syncthreads();
    for (int k = 0; k < 2 && join_group[k] >= 0; ++k) {
        const Cut cut = joins[k];
        const int g = join_group[k], groups = (cut.pieces + kGroup - 1) / kGroup;
        const int h0 = cut.h % tiles * H, n = min(H, G - h0);
        const long long hq = (long long)cut.b * a.Hq + cut.h / tiles * G + h0;
        Joined<P> sum;
        // first the group's pieces, then, by the last group, the groups' sums (one
        // instance of the code: what a launch fetches of it counts for short calls)
        int first = g * kGroup, step = 1, count = cut.in_group(g, kGroup);
        while (true) {
            sum.add(smem, a.part, n, count, [&](int i) { return cut.slot(first + i * step); });
            if (step > 1 || groups == 1) {
                sum.write(a, hq, n);
                break;
            }
            sum.store(a.part + (long long)cut.slot(first) * kPart, n);
            __syncthreads();
            if (tid == 0) {
                int *ticket = a.counter + cut.b * heads + cut.h;
                __threadfence();
                last = atomicAdd(ticket, 1) == groups - 1;
                __threadfence();
                if (last) *ticket = 0;
            }
            __syncthreads();
            if (!last) break;
            first = 0, step = kGroup, count = groups;
        }
    }
}

// weights[j] += sum_h 2^(s_jh - M_h) / L_h from the scores the attention kernel
// left, heads in order; one row of a KV head per thread.  V: float4 of scores per
// row (0: any group).  One row a thread and eight CTAs an SM beat two or four rows
// and fewer CTAs (16 sequences of up to 8192 rows, both kernels, before the attention
// kept P in three parts: 52.1, 52.3 and 53.3 us): what bounds it is the chain of a row's loads, not their bytes.
constexpr int kWtThreads = 256;
constexpr int kWtCtasPerSm = 8;
template <int V>
__global__ void __launch_bounds__(kWtThreads, kWtCtasPerSm) paged_weights_kernel(AttendArgs a, int head_tile) {
    // Before the wait: the attention kernel lets this one start once its own wait is
    // over, so lengths, table and weights are final; scores and stat are not.
    pdl_trigger();
    auto rows = [&](int b) { return paged_len(a.cache, b, a.added, nullptr); };
    auto blocks = [](int n) { return max(1, (n + kWtThreads - 1) / kWtThreads); };
    UnitRange r;
    if (!unit_range<kWtThreads>(r, a.B, a.Hkv, rows, blocks)) {
        pdl_wait();
        return;
    }
    const int G = a.Hq / a.Hkv;
    const long long cap = (long long)a.cache.table_pages * a.cache.page_size;
    int b = r.b, len = rows(b), nblk = blocks(len);
    int h = (r.u0 - r.first) / nblk, blk = (r.u0 - r.first) % nblk;
    for (int u = r.u0; u < r.u1; ++u) {
        const int j = blk * kWtThreads + threadIdx.x;
        const int page = j < len ? a.cache.table[(long long)b * a.cache.table_pages + j / a.cache.page_size] : -1;
        if (u == r.u0) pdl_wait();
        if ((unsigned)page < (unsigned)a.cache.n_pages) {   // else past the rows, or reported by the attention
            const float *s = a.scores + score_place(b, h, 0, a.Hkv, G, cap);
            const float2 *st = a.stat + (long long)b * a.Hq + h * G;
            float *to = a.cache.weights + ((long long)page * a.Hkv + h) * a.cache.page_size + j % a.cache.page_size;
            float w = 0.f;
            auto add = [&](float z, const float2 &ml) { w = fmaf(exp2f(z - ml.x), ml.y, w); };
            if (V > 0) {
                float4 z[V > 0 ? V : 1];
#pragma unroll
                for (int k = 0; k < V; ++k) z[k] = ((const float4 *)s)[(long long)j * V + k];
                const float was = *to;
#pragma unroll
                for (int k = 0; k < V; ++k)
                    add(z[k].x, st[4 * k]), add(z[k].y, st[4 * k + 1]), add(z[k].z, st[4 * k + 2]), add(z[k].w, st[4 * k + 3]);
                *to = was + w;
            } else {
                for (int t = 0; t < G; t += head_tile) {
                    const int n = min(head_tile, G - t);
                    const float *z = s + t * cap + (long long)j * n;
                    for (int k = 0; k < n; ++k) add(z[k], st[t + k]);
                }
                *to += w;
            }
        }
        if (++blk == nblk && u + 1 < r.u1) {
            blk = 0;
            if (++h == a.Hkv) {
                h = 0;
                len = rows(++b);
                nblk = blocks(len);
            }
        }
    }
}

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

}  // namespace

static int attend_head_tile(int G) { return G <= 4 ? 4 : G <= 8 ? 8 : 16; }

int attend_head_tiles(int G) { return (G + 7) / 8; }

int attend_ctas(int sms) { return sms * kPaCtasPerSm; }

size_t attend_part_floats(int D, int G, int sms) {
    return (size_t)2 * attend_ctas(sms) * attend_head_tile(G) * (D + 2);
}

cudaError_t prepare_attend_kernels() {
    for (const bool bf16 : {false, true})
        for (const int D : {64, 128})
            for (const int heads : {4, 8, 16}) {
                const cudaError_t e = with_tile(bf16, D, heads, [](auto tile) {
                    using P = decltype(tile);
                    const cudaError_t e = cudaFuncSetAttribute(paged_attend_kernel<P, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)attend_smem<P>());
                    return e != cudaSuccess ? e : cudaFuncSetAttribute(paged_attend_kernel<P, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)attend_smem<P>());
                });
                if (e != cudaSuccess) return e;
            }
    return cudaSuccess;
}

// CTAs of a cluster per segment, or 1: the shares of a persistent grid.  Clusters
// where all of them run at once and a table's rows are few for each CTA: at most
// `rows` (bf16 at D = 128: 512, with 9 to 16 query heads 1024; fp32 128,
// with 5 to 16 query heads 256).  The rows are the table's, all that a launch knows: a
// table far wider than its sequences takes the shares.  Measured, 8 KV
// heads of 128 and 4 query heads each, cluster against shares: one sequence of 100
// rows 4.8 and 6.6 us, of 1000 5.9 and 8.0, of 4000 10.1 and 10.1; four of 4000 14.8 and
// 17.3; fp32 of 1000 rows 7.8 and 8.7, of 2000 11.2 and 9.7; 4 KV heads with 16 query
// heads each, 1000 rows 7.6 and 14.3, 4000 rows 13.0 and 18.9.
static int attend_cluster(long long segments, long long cap, int rows, int sms) {
    int cs = 1;
    while (cs < 8 && cs * (long long)kAttendUnit < cap && 2 * cs * segments <= attend_ctas(sms)) cs *= 2;
    return cap <= cs * (long long)rows ? cs : 1;
}

cudaError_t launch_paged_attend(const AttendArgs &args, bool bf16, int D, int sms, cudaStream_t s) {
    AttendArgs a = args;
    const int G = a.Hq / a.Hkv;
    const long long cap = (long long)a.cache.table_pages * a.cache.page_size, groups = a.B * (long long)a.Hkv;
    int ht = attend_head_tile(G);
    // fp32 tables of few rows: a tile of 16 heads takes longer than the second pass of
    // two of 8.  Measured, D = 128, 8 against 16: 4 KV heads of 1000 rows 9.6 and 12.3
    // us, of 8000 24 and 26, of 16000 35 and 36; 32 sequences of 500 rows 34 and 24;
    // D = 64: 4000 rows 11.7 and 17.1, 8 sequences of 1000 rows 11.9 and 10.5.
    if (!bf16 && ht == 16 && groups * ((G + 15) / 16) * cap <= 256 * D) ht = 8;
    const long long segments = groups * ((G + ht - 1) / ht);
    const long long most = segments * (kAttendCost + (cap + kAttendUnit - 1) / kAttendUnit);
    cudaError_t e = with_tile(bf16, D, ht, [&](auto tile) {
        using P = decltype(tile);
        a.cluster = attend_cluster(segments, cap, P::kClusterRows, sms);
        if (a.cluster > 1)
            return launch_cluster(paged_attend_kernel<P, true>, dim3((unsigned)segments * a.cluster), dim3(kPaThreads), attend_smem<P>(), a.cluster, s, a);
        const int grid = (int)(most < attend_ctas(sms) ? most : attend_ctas(sms));
        return launch_k(paged_attend_kernel<P, false>, dim3(grid), dim3(kPaThreads), attend_smem<P>(), s, true, a);
    });
    if (e != cudaSuccess || !a.scores) return e;
    const long long chunks = a.B * (long long)a.Hkv * ((cap + kWtThreads - 1) / kWtThreads);
    const dim3 wt((unsigned)(chunks < sms * kWtCtasPerSm ? chunks : sms * kWtCtasPerSm));
    auto go = [&](auto k) { return launch_k(k, wt, dim3(kWtThreads), 0, s, true, a, ht); };
    // 4, 8 or 16 heads of one tile: a row's scores are one, two or four float4
    if (G <= ht && G == 4) return go(paged_weights_kernel<1>);
    if (G <= ht && G == 8) return go(paged_weights_kernel<2>);
    if (G <= ht && G == 16) return go(paged_weights_kernel<4>);
    return go(paged_weights_kernel<0>);
}

}  // namespace prism
