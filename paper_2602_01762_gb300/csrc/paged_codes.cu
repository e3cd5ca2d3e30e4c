// Rows quantised as they are written to a paged cache held in 8 bits, and read back.
//
// A block is `scale_rows` rows of a page and KV head and has one scale s for K and one
// for V; a row's value is its code times s.  Of the new rows x of a block (keys normed
// and rotated, values as they are) and with M the largest code (448 for e4m3, 127 for
// int8):
//
//   s = max(s of the block's earlier rows, 2^ceil(log2(max |x| / M))),  code = rn(x / s)
//
// and where s grows, the earlier rows' codes become rn(code s_before / s).  Scales are
// powers of two: dividing by one is exact, so that a code has one rounding, and a row's
// codes are rounded anew at most as often as its block's largest value doubles (int8:
// its errors add up to less than one step; e4m3: none but below 2^-6 steps).  An e4m3
// code has the same relative precision wherever in its range it lies, so that a closer
// scale would give it nothing; to int8 it would give half a bit on average, and lose
// more than that where one more row a block has every code rounded again.
#include "paged_rope.cuh"

#include <type_traits>

namespace prism {
namespace {

constexpr int kScThreads = 128;
constexpr int kScKeep = 4;               // rows of a lane group kept in registers between a block's maximum and its codes

__device__ __forceinline__ void e4m3_values(uint32_t codes, float (&f)[4]) {
    uint32_t lo, hi;
    asm("{.reg .b16 l, u;\n mov.b32 {l, u}, %2;\n cvt.rn.f16x2.e4m3x2 %0, l;\n cvt.rn.f16x2.e4m3x2 %1, u;}" : "=r"(lo), "=r"(hi) : "r"(codes));
    asm("{.reg .b16 l, u;\n mov.b32 {l, u}, %2;\n cvt.f32.f16 %0, l;\n cvt.f32.f16 %1, u;}" : "=f"(f[0]), "=f"(f[1]) : "r"(lo));
    asm("{.reg .b16 l, u;\n mov.b32 {l, u}, %2;\n cvt.f32.f16 %0, l;\n cvt.f32.f16 %1, u;}" : "=f"(f[2]), "=f"(f[3]) : "r"(hi));
}
// Four codes as values, and four values within the codes' range (or NaN, e4m3) as codes.
template <int FORMAT> __device__ __forceinline__ void decode(uint32_t codes, float (&f)[4]) {
    if (FORMAT == kE4m3) {
        e4m3_values(codes, f);
    } else {
        // the low byte of 2^23 + 128 + code
        const uint32_t c = codes ^ 0x80808080u;
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(__byte_perm(c, 0x4B000000u, 0x7540 + i)) - 8388736.f;
    }
}
template <int FORMAT> __device__ __forceinline__ uint32_t encode(float x0, float x1, float x2, float x3) {
    if (FORMAT == kE4m3) {
        uint32_t r;
        asm("{.reg .b16 l, u;\n cvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\n cvt.rn.satfinite.e4m3x2.f32 u, %4, %3;\n mov.b32 %0, {l, u};}"
            : "=r"(r) : "f"(x0), "f"(x1), "f"(x2), "f"(x3));
        return r;
    }
    // added to 1.5 2^23, a value's nearest whole number (ties to even) is the low byte
    const float big = 12582912.f;
    const uint32_t lo = __byte_perm(__float_as_uint(x0 + big), __float_as_uint(x1 + big), 0x0040);
    const uint32_t hi = __byte_perm(__float_as_uint(x2 + big), __float_as_uint(x3 + big), 0x0040);
    return __byte_perm(lo, hi, 0x5410);
}

// The smallest power of two, from 2^-126 on, that holds magnitudes up to that of bits
// `top` (finite) in the codes' range; 0 for 0.
template <int FORMAT> __device__ __forceinline__ float power_of_two(uint32_t top) {
    // 448 = 1.75 2^8, 127 = 1.984375 2^6
    const int e = (int)(top >> 23) - (FORMAT == kE4m3 ? 8 : 6) + ((top & 0x7FFFFFu) > (FORMAT == kE4m3 ? 0x600000u : 0x7E0000u) ? 1 : 0);
    return top == 0 ? 0.f : __uint_as_float((uint32_t)max(e, 1) << 23);
}

// A team of a.team warps, or with a.per > 1 a part of a warp, per block, head and K or
// V: rows of lanes as in the norm (E values at j and at j + D/2 each), the block's
// largest value over the team, then the codes.  Up to kScKeep rows a lane group stay in
// registers; longer blocks' further rows are read (from L2) and computed again.
template <typename T, int D, int FORMAT>
__global__ void __launch_bounds__(kScThreads) store_codes_kernel(StoreCodesArgs a) {
    using R = Rope<T, D>;
    constexpr int N = R::N, E = R::E, kRows = R::kHeads;   // rows a warp has at a time
    __shared__ uint32_t tops[kScThreads / 32];
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane % R::kLanes, group = lane / R::kLanes;
    const unsigned task = blockIdx.x * (kScThreads / 32 / a.team) + warp / a.team;
    const unsigned run = task / (2u * a.Hkv), b = run / (unsigned)a.tasks;
    if (b >= (unsigned)a.B) return;                      // whole teams
    const int which = (int)(task - run * (2u * a.Hkv));
    const bool is_k = which < a.Hkv;
    const int h = is_k ? which : which - a.Hkv;
    const int block = (int)(run - b * a.tasks) * a.per + (a.per > 1 ? group / a.scale_rows : 0);
    const int step = kRows * a.team;                     // rows of the team at a time
    const int j0 = a.per > 1 ? group % a.scale_rows : warp % a.team * kRows + group;
    // the block's rows are slots first + j, 0 <= j < scale_rows; new ones from j_new on, up to j_end
    const int len = a.cache.kv_len[b], n = row_count(a.n_new, b, a.max_new, a.err);
    const long long first = ((long long)(len < 0 ? 0 : len) / a.scale_rows + block) * a.scale_rows;
    const int j_new = first < len ? (int)(len - first) : 0;
    long long end = len + (long long)n - first;
    int j_end = (int)(end < 0 ? 0 : end > a.scale_rows ? a.scale_rows : end);
    int page = 0, row = 0;
    if (j_new < j_end) {
        if (len < 0 || first >= (long long)a.cache.table_pages * a.cache.page_size) {
            set_err(a.err, kErrCache);
            j_end = 0;
        } else {
            const int slot = (int)(first / a.cache.page_size);
            row = (int)(first - (long long)slot * a.cache.page_size);
            page = a.cache.table[(long long)b * a.cache.table_pages + slot];
            if ((unsigned)page >= (unsigned)a.cache.n_pages) {
                set_err(a.err, kErrPage);
                j_end = 0;
            }
        }
    }
    if (len < 0 && n > 0) set_err(a.err, kErrCache);
    const bool live = j_new < j_end;
    if (a.per > 1 ? !__any_sync(0xFFFFFFFFu, live) : !live) return;

    const HeadsView &from = is_k ? a.k : a.v;
    const char *src = from.p + (long long)b * from.sb + h * from.sh + sub * 16;
    const int shift = (int)(first - len);                // row j is new row j + shift
    Gain<T, D> gain;
    const bool norm = is_k && a.g_k != nullptr;
    if (norm) gain.load(a.g_k);
    // Row j's values, zeros where it is none of the new ones.
    auto load = [&](int j, F2 (&x)[N], F2 (&y)[N]) {
        const bool in = live && j >= j_new && j < j_end;
        const int i = in ? j + shift : 0;
        uint4 l = make_uint4(0u, 0u, 0u, 0u), r = l;
        if (in) {
            l = *(const uint4 *)(src + i * from.st);
            r = *(const uint4 *)(src + i * from.st + D / 2 * sizeof(T));
        }
        Pairs<T>::unpack(l, x);
        Pairs<T>::unpack(r, y);
        if (!is_k) return;
        R rope;
        rope.load(a.rope, in ? row_position(a.pos, b, i, a.rope_len, a.err) : 0);
        if (norm) {
            F2 s = f2_mul(x[0], x[0]);
#pragma unroll
            for (int e = 1; e < N; ++e) s = f2_fma(x[e], x[e], s);
#pragma unroll
            for (int e = 0; e < N; ++e) s = f2_fma(y[e], y[e], s);
            const float f = in ? rsqrtf(lanes_sum<R::kLanes>(f2_sum(s)) * (1.f / D) + a.eps) : (lanes_sum<R::kLanes>(f2_sum(s)), 0.f);
            const F2 ff = f2(f, f);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                x[e] = f2_mul(f2_mul(x[e], ff), gain.x[e]);
                y[e] = f2_mul(f2_mul(y[e], ff), gain.y[e]);
            }
        }
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const F2 p = f2_sub(f2_mul(x[e], rope.cs[e]), f2_mul(y[e], rope.sn[e]));
            y[e] = f2_fma(y[e], rope.cs[e], f2_mul(x[e], rope.sn[e]));
            x[e] = p;
        }
        if (!in)
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = y[e] = 0ull;
    };
    uint32_t top = 0, odd = 0;                           // bits of the largest finite magnitude; whether any is not finite
    auto look = [&](const F2 (&x)[N], const F2 (&y)[N]) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float2 u = f2_values(x[e]), v = f2_values(y[e]);
            const float f[4] = {u.x, u.y, v.x, v.y};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t bits = __float_as_uint(f[i]) & 0x7FFFFFFFu;
                if (bits < 0x7F800000u) top = max(top, bits);
                else odd = 1;
            }
        }
    };
    F2 x[kScKeep][N], y[kScKeep][N];
#pragma unroll
    for (int c = 0; c < kScKeep; ++c) {
        // whole warps: a team's rows of one turn
        const int turn = c * step + (a.per > 1 ? 0 : warp % a.team * kRows);
        if (a.per > 1 ? c == 0 : turn < j_end && turn + kRows > j_new) {
            load(c * step + j0, x[c], y[c]);
            look(x[c], y[c]);
        }
    }
    if (a.per == 1)
        for (int c = kScKeep; c * step < j_end; ++c) {
            F2 u[N], v[N];
            load(c * step + j0, u, v);
            look(u, v);
        }
    const int width = a.per > 1 ? R::kLanes * a.scale_rows : 32;   // lanes of a block
    top |= odd << 31;                                    // the maximum carries both
    {
        uint32_t any = top >> 31, most = top & 0x7FFFFFFFu;
        for (int o = width / 2; o > 0; o >>= 1) {
            most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
            any |= __shfl_xor_sync(0xFFFFFFFFu, any, o);
        }
        top = most | any << 31;
    }
    if (a.team > 1) {
        if (lane == 0) tops[warp] = top;
        asm volatile("bar.sync %0, %1;" ::"r"(1 + warp / a.team), "r"(32 * a.team) : "memory");
        const int base = warp / a.team * a.team;
        for (int w = 0; w < a.team; ++w) {
            const uint32_t t = tops[base + w];
            top = max(top & 0x7FFFFFFFu, t & 0x7FFFFFFFu) | ((top | t) & 0x80000000u);
        }
    }
    const bool any_odd = top >> 31;
    float *scale_at = (is_k ? a.k_scales : a.v_scales) + ((long long)page * a.Hkv + h) * a.scale_blocks + row / a.scale_rows;
    const float before = live && j_new > 0 ? *scale_at : 0.f;
    // every thread has read the scale before it is written
    if (a.team > 1) asm volatile("bar.sync %0, %1;" ::"r"(1 + warp / a.team), "r"(32 * a.team) : "memory");
    else __syncwarp();
    if (!live) return;
    float s = power_of_two<FORMAT>(top & 0x7FFFFFFFu);
    if (FORMAT == kInt8 && any_odd) s = __int_as_float(0x7FFFFFFF);   // int8 has no code for it: the block reads as NaN
    if (!(before < s) && !(s != s)) s = before;          // a NaN stays one
    const float per_s = s > 0.f ? 1.f / s : 0.f;
    char *to = (is_k ? a.cache.k : a.cache.v) + page * a.cache.page_stride + h * a.cache.head_stride + row * a.cache.row_stride;
    const int in_team = a.per > 1 ? lane % width : warp % a.team * 32 + lane, threads = a.per > 1 ? width : 32 * a.team;
    if (in_team == 0 && (j_new == 0 || s != before)) *scale_at = s;
    if (j_new > 0 && before < s) {                       // earlier rows in the grown scale
        const float f = before / s;
#pragma unroll 4
        for (int e = in_team; e < j_new * (D / 4); e += threads) {
            uint32_t *p = (uint32_t *)(to + e / (D / 4) * a.cache.row_stride) + e % (D / 4);
            float v[4];
            decode<FORMAT>(*p, v);
            *p = encode<FORMAT>(v[0] * f, v[1] * f, v[2] * f, v[3] * f);
        }
    }
    auto put = [&](int j, const F2 (&x)[N], const F2 (&y)[N]) {
        if (j < j_new || j >= j_end) return;
        float f[2][E];
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float2 u = f2_values(x[e]), v = f2_values(y[e]);
            f[0][2 * e] = u.x, f[0][2 * e + 1] = u.y, f[1][2 * e] = v.x, f[1][2 * e + 1] = v.y;
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            uint32_t w[E / 4];
            if (any_odd) {                               // e4m3: infinities become NaN
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (!(fabsf(f[i][e]) < INFINITY)) f[i][e] = FORMAT == kE4m3 ? __int_as_float(0x7FFFFFFF) : 0.f;
            }
#pragma unroll
            for (int e = 0; e < E / 4; ++e)
                w[e] = encode<FORMAT>(f[i][4 * e] * per_s, f[i][4 * e + 1] * per_s, f[i][4 * e + 2] * per_s, f[i][4 * e + 3] * per_s);
            char *at = to + j * a.cache.row_stride + i * (D / 2) + sub * E;
            if (E == 8) *(uint2 *)at = make_uint2(w[0], w[E / 4 - 1]);
            else *(uint32_t *)at = w[0];
        }
    };
#pragma unroll
    for (int c = 0; c < kScKeep; ++c)
        if (a.per > 1 ? c == 0 : c * step < j_end) put(c * step + j0, x[c], y[c]);
    if (a.per == 1)
        for (int c = kScKeep; c * step < j_end; ++c) {
            F2 u[N], v[N];
            load(c * step + j0, u, v);
            put(c * step + j0, u, v);
        }
}

// Rows read back, 16 bytes of the result a lane: a CTA takes kRcRows rows of a
// sequence and walks over their heads.
constexpr int kRcThreads = 256;
constexpr int kRcRows = 16;
template <typename T, int D, int FORMAT>
__global__ void __launch_bounds__(kRcThreads) read_codes_kernel(ReadCodesArgs a) {
    constexpr int E = Vec16<T>::E, kLanes = D / E, kGroups = kRcThreads / kLanes;
    constexpr int kAhead = 4;            // rows and heads of a lane at a time, K and V of each
    pdl_wait();
    pdl_trigger();
    const unsigned chunks = (a.max_rows + kRcRows - 1) / (unsigned)kRcRows, b = blockIdx.x / chunks;
    const int i0 = (int)(blockIdx.x - b * chunks) * kRcRows;
    const int n = min(row_count(a.n_rows, b, a.max_rows, a.err), i0 + kRcRows) - i0;
    if (n <= 0) return;
    const long long start = (a.start ? a.start[b] : 0) + (long long)i0, cap = (long long)a.cache.table_pages * a.cache.page_size;
    const int sub = threadIdx.x % kLanes;
    for (int e0 = threadIdx.x / kLanes; e0 < kRcRows * a.Hkv; e0 += kAhead * kGroups) {
        uint32_t c[kAhead][2][E / 4];
        float s[kAhead][2];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int e = e0 + u * kGroups, r = e % kRcRows, h = e / kRcRows;
            s[u][0] = s[u][1] = 0.f;
#pragma unroll
            for (int w = 0; w < E / 4; ++w) c[u][0][w] = c[u][1][w] = 0u;
            if (h >= a.Hkv || r >= n) continue;
            const long long slot = start + r;
            if (slot < 0 || slot >= cap) {
                set_err(a.err, kErrCache);
                continue;
            }
            const int idx = (int)slot / a.cache.page_size, row = (int)slot - idx * a.cache.page_size;
            const int page = a.cache.table[(long long)b * a.cache.table_pages + idx];
            if ((unsigned)page >= (unsigned)a.cache.n_pages) {
                set_err(a.err, kErrPage);
                continue;
            }
            const long long at = page * a.cache.page_stride + h * a.cache.head_stride + row * a.cache.row_stride + sub * E;
            const long long scale = ((long long)page * a.Hkv + h) * a.scale_blocks + row / a.scale_rows;
#pragma unroll
            for (int kv = 0; kv < 2; ++kv) {
                const char *p = (kv ? a.cache.v : a.cache.k) + at;
                if (E == 8) {
                    const uint2 w = *(const uint2 *)p;
                    c[u][kv][0] = w.x, c[u][kv][E / 4 - 1] = w.y;
                } else {
                    c[u][kv][0] = *(const uint32_t *)p;
                }
                s[u][kv] = (kv ? a.v_scales : a.k_scales)[scale];
            }
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int e = e0 + u * kGroups, r = e % kRcRows, h = e / kRcRows;
            if (h >= a.Hkv || r >= n) continue;
#pragma unroll
            for (int kv = 0; kv < 2; ++kv) {
                float f[E];
#pragma unroll
                for (int w = 0; w < E / 4; ++w) {
                    float v[4];
                    decode<FORMAT>(c[u][kv][w], v);
#pragma unroll
                    for (int i = 0; i < 4; ++i) f[4 * w + i] = v[i] * s[u][kv];
                }
                const HeadsView &o = kv ? a.v_out : a.k_out;
                *(uint4 *)(o.p + (long long)b * o.sb + (i0 + r) * o.st + h * o.sh + sub * 16) = Vec16<T>::pack(f);
            }
        }
    }
}

template <typename F> cudaError_t with_codes(CodeFormat format, bool bf16, int D, const F &f) {
    const std::integral_constant<int, 64> small;
    const std::integral_constant<int, 128> large;
    const std::integral_constant<int, kE4m3> e4m3;
    const std::integral_constant<int, kInt8> int8;
    auto type = [&](auto t) {
        if (format == kE4m3) return D == 128 ? f(t, large, e4m3) : f(t, small, e4m3);
        return D == 128 ? f(t, large, int8) : f(t, small, int8);
    };
    return bf16 ? type(uint16_t()) : type(0.f);
}

}  // namespace

cudaError_t launch_store_codes(const StoreCodesArgs &args, CodeFormat format, bool bf16, int D, int, cudaStream_t s) {
    StoreCodesArgs a = args;
    const int rows = 32 / (D / 2 / (bf16 ? 8 : 4)), R = a.scale_rows;   // rows a warp has at a time
    a.per = R < rows && rows % R == 0 ? rows / R : 1;
    a.team = R <= kScKeep * rows ? 1 : R <= 2 * kScKeep * rows ? 2 : 4;
    const long long blocks = (a.max_new + 2LL * R - 2) / R;              // that a sequence's new rows may touch
    a.tasks = (int)((blocks + a.per - 1) / a.per);
    const long long warps = (long long)a.B * a.tasks * 2 * a.Hkv * a.team;
    const dim3 grid((unsigned)((warps + kScThreads / 32 - 1) / (kScThreads / 32)));
    return with_codes(format, bf16, D, [&](auto t, auto d, auto form) {
        return launch_k(store_codes_kernel<decltype(t), d, form>, grid, dim3(kScThreads), 0, s, true, a);
    });
}

cudaError_t launch_read_codes(const ReadCodesArgs &a, CodeFormat format, bool bf16, int D, cudaStream_t s) {
    const dim3 grid((unsigned)a.B * ((a.max_rows + kRcRows - 1) / kRcRows));
    return with_codes(format, bf16, D, [&](auto t, auto d, auto form) {
        return launch_k(read_codes_kernel<decltype(t), d, form>, grid, dim3(kRcThreads), 0, s, true, a);
    });
}

}  // namespace prism
