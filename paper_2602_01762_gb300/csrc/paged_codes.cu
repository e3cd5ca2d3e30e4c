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
//
// Bound by bytes, but a block's codes wait for its largest value and that for the rows'
// loads. Measured, 32 query and 8 KV heads of 128, bf16, blocks of 16: 8 prompts of 1021 to
// 2048 rows 58 us (277 MB, 4.8 TB/s: the queries' kernel 33, keys and values mostly behind
// it), 16 tokens 3.6 us; read back, 4 prefixes of 9001 to 16384 rows 49.5 us (6.3 TB/s).
#include "paged_rope.cuh"

#include <type_traits>

namespace prism {
namespace {

constexpr int kScThreads = 128;
constexpr int kScAngles = 64;            // rows of a tile whose angles are kept in shared memory, at most
constexpr int kScKeep = 4;               // rows of a lane group kept in registers between a block's maximum and its codes
constexpr int kScStage = kScKeep * 1024; // bytes of a warp's rows of one head: two pieces a lane and row
constexpr int kScRing = kScThreads / 32 * 2 * kScStage;

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

// Larger of magnitudes; NaN if one is.
__device__ __forceinline__ float top_of(float a, float b, float c) {
    float d;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// A CTA per tile of rows, a block's or with a.per > 1 those of a.per short blocks that a
// warp has side by side, and a.span of its heads of K or of V; what depends on the rows
// alone (lengths, place, angles) is found once.  A team of a.team warps takes a head:
// rows of lanes as in the norm (E values at j and at j + D/2 each), the block's largest
// value over the team, then the codes, the next head's rows on their way meanwhile.  Up
// to kScKeep rows a lane group stay in registers; longer blocks' further rows are read
// and computed again.
template <typename T, int D, int FORMAT, bool KEYS>
__device__ __forceinline__ void store_tile(const StoreCodesArgs &a, int run, int w0, const HeadsView &rows, char *pages, float *scales, unsigned char *dyn) {
    using R = Rope<T, D>;
    constexpr int N = R::N, E = R::E, kRows = R::kHeads;   // rows a warp has at a time
    __shared__ float tops[2][kScThreads / 32];
    float *const angles = (float *)(dyn + kScRing);      // behind two stages a warp
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane % R::kLanes, group = lane / R::kLanes;
    const int team = warp / a.team, teams = kScThreads / 32 / a.team, in_team = warp - team * a.team;
    const int b = a.by_tasks.of(run), tile = run - b * a.tasks;
    const int w1 = min(w0 + a.span, a.Hkv);
    const int in_warp = a.per > 1 ? a.by_scale.of(group) : 0;    // this lane's block of the warp's
    const int step = kRows * a.team, j0 = a.per > 1 ? group - in_warp * a.scale_rows : in_team * kRows + group;
    // a block's rows are slots first + j, 0 <= j < scale_rows; new ones from j_new on, up to j_end
    const int held = a.cache.kv_len[b], cap = a.cache.table_pages * a.cache.page_size, pos = KEYS ? a.pos[b] : 0;
    const bool fits = held >= 0 && held <= cap;          // no slot beyond a length that does not is a row's
    const int len = fits ? held : 0, n = row_count(a.n_new, b, a.max_new, a.err);
    const int tile_first = (a.by_scale.of(len) + tile * a.per) * a.scale_rows, first = tile_first + in_warp * a.scale_rows;
    const int j_new = max(len - first, 0), j_end = min(max(len + n - first, 0), a.scale_rows);
    const int shift = first - len;                       // row j is new row j + shift
    // turns of the warp with a new row, and this lane's rows in them
    uint32_t turns = 1, mine = 0;
    if (a.per == 1) {
        turns = 0;
#pragma unroll
        for (int c = 0; c < kScKeep; ++c) {
            const int at = c * step + in_team * kRows;
            turns |= (at < j_end && at + kRows > j_new) << c;
        }
    }
#pragma unroll
    for (int c = 0; c < kScKeep; ++c) mine |= (turns >> c & 1 && c * step + j0 >= j_new && c * step + j0 < j_end) << c;
    const char *src = rows.p + (long long)b * rows.sb + (long long)(j0 + shift) * rows.st + sub * 16;
    // this lane's rows of a head, requested before their place is known; each lane copies
    // what it reads itself, so that its own waits are enough
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(dyn) + warp * (2 * kScStage) + lane * 16;
    auto fetch = [&](int w, int stage) {
        if (w < w1) {
            const char *from = src + w * rows.sh;
#pragma unroll
            for (int c = 0; c < kScKeep; ++c) {
                if (mine >> c & 1) {
                    cp16(ring + stage * kScStage + c * 1024, from, true);
                    cp16(ring + stage * kScStage + c * 1024 + 512, from + D / 2 * sizeof(T), true);
                }
                from += step * rows.st;
            }
        }
        cp_group();
    };
    int w = w0 + team;
    // new row i's angles, held to the table; of a tile's first kScAngles rows they are kept
    auto position = [&](int i) {
        const long long at = (long long)pos + i;
        if (at >= 0 && at < a.rope_len) return (int)at;
        set_err(a.err, kErrPosition);
        return at < 0 ? 0 : a.rope_len - 1;
    };
    const uint32_t angles_at = (uint32_t)__cvta_generic_to_shared(angles);
    if (KEYS && fits) {
        const int count = min(a.per > 1 ? kRows : a.scale_rows, kScAngles);
        for (int e = threadIdx.x; e < count * (D / 4); e += kScThreads) {
            const int i = tile_first + e / (D / 4) - len;
            if (i >= 0 && i < n) cp16(angles_at + 16 * e, a.rope + (long long)position(i) * D + 4 * (e % (D / 4)), true);
        }
    }
    fetch(w, 0);
    fetch(w + teams, 1);
    int page = 0, row = 0;
    bool live = j_new < j_end;
    if (live) {
        if (!fits || first >= cap) {
            set_err(a.err, kErrCache);
            live = false;
        } else {
            const int slot = a.by_page.of(first);
            row = first - slot * a.cache.page_size;
            page = a.cache.table[(long long)b * a.cache.table_pages + slot];
            if ((unsigned)page >= (unsigned)a.cache.n_pages) {
                set_err(a.err, kErrPage);
                live = false;
            }
        }
    }
    if (!__any_sync(0xFFFFFFFFu, live)) {                // the same for every warp of the CTA
        cp_wait_group<0>();
        return;
    }
    if (!live) mine = 0;
    float *const scale_at = scales + (long long)page * a.Hkv * a.scale_blocks + a.by_scale.of(row);
    float before = live && j_new > 0 && w < w1 ? scale_at[(long long)w * a.scale_blocks] : 0.f;
    Gain<T, D> gain;
    const bool norm = a.g_k != nullptr;
    if (KEYS) {
        if (norm) gain.load(a.g_k);
        cp_wait_group<1>();
        __syncthreads();                                 // the angles are there
    }
    // Row j's values from what was read of it, before the norm's factor, which is returned.
    // The gain times a bf16 value is exact, and the factor meets a sum that is already
    // turned: two roundings fewer than in the order of the formula, and as many products.
    auto values = [&](int j, bool in, const uint4 &l, const uint4 &r, F2 (&x)[N], F2 (&y)[N]) {
        Pairs<T>::unpack(l, x);
        Pairs<T>::unpack(r, y);
        if (!KEYS) return 1.f;
        R rope;
        const int at = !in ? 0 : a.per > 1 ? group : j;   // a turn's last rows may be past the block's
        if (at < kScAngles) rope.load_shared(angles_at + at * (D * 4));
        else rope.load(a.rope, in ? position(j + shift) : 0);
        float f = 1.f;
        if (norm) {
            F2 s = f2_mul(x[0], x[0]);
#pragma unroll
            for (int e = 1; e < N; ++e) s = f2_fma(x[e], x[e], s);
#pragma unroll
            for (int e = 0; e < N; ++e) s = f2_fma(y[e], y[e], s);
            const float m = lanes_sum<R::kLanes>(f2_sum(s)) * (1.f / D) + a.eps;
            f = rsqrtf(m);
            const float more = fmaf(-(m * f), f, 1.f) * 0.5f;    // one Newton step: within one ulp
            if (fabsf(more) < 1e-3f) f = fmaf(f, more, f);       // but not of 0, infinities and NaN
#pragma unroll
            for (int e = 0; e < N; ++e) {
                x[e] = f2_mul(x[e], gain.x[e]);
                y[e] = f2_mul(y[e], gain.y[e]);
            }
        }
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const F2 p = f2_mul(y[e], rope.sn[e]), q = f2_mul(x[e], rope.sn[e]);
            x[e] = f2_fma(x[e], rope.cs[e], p ^ 0x8000000080000000ull);
            y[e] = f2_fma(y[e], rope.cs[e], q);
        }
        return f;
    };
    auto magnitude = [&](const F2 (&x)[N], const F2 (&y)[N], float f, float top) {
        float row = 0.f;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float2 u = f2_values(x[e]), v = f2_values(y[e]);
            row = top_of(u.x, u.y, top_of(v.x, v.y, row));
        }
        return top_of(top, row * f, 0.f);
    };
    auto finite = [&](const F2 (&x)[N], const F2 (&y)[N], float f, float top) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float2 u = f2_values(x[e]), v = f2_values(y[e]);
            const float z[4] = {u.x * f, u.y * f, v.x * f, v.y * f};
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (fabsf(z[i]) < INFINITY) top = fmaxf(top, fabsf(z[i]));
        }
        return top;
    };
    // further rows of a long block, read and computed once more wherever they are asked for
    auto further = [&](int w, const auto &f) {
        if (a.per == 1)
            for (int c = kScKeep; c * step < j_end; ++c) {
                const bool in = c * step + j0 >= j_new && c * step + j0 < j_end;
                uint4 l = make_uint4(0u, 0u, 0u, 0u), r = l;
                if (in) {
                    const char *from = src + w * rows.sh + c * step * rows.st;
                    l = *(const uint4 *)from;
                    r = *(const uint4 *)(from + D / 2 * sizeof(T));
                }
                F2 u[N], v[N];
                const float factor = values(c * step + j0, in, l, r, u, v);
                if (in) f(c * step + j0, u, v, factor);
            }
    };
    const int width = a.per > 1 ? R::kLanes * a.scale_rows : 32;   // lanes of a block
    const int thread = a.per > 1 ? lane % width : in_team * 32 + lane, threads = a.per > 1 ? width : 32 * a.team;
    const long long page_at = page * a.cache.page_stride + row * a.cache.row_stride;
    for (int turn = 0; w < w1; w += teams, turn ^= 1) {
        const float was = before;
        if (w + teams < w1) before = live && j_new > 0 ? scale_at[(long long)(w + teams) * a.scale_blocks] : 0.f;
        cp_wait_group<1>();
        F2 x[kScKeep][N], y[kScKeep][N];
        float factor[kScKeep], top = 0.f;
#pragma unroll
        for (int c = 0; c < kScKeep; ++c)
            if (turns >> c & 1) {                        // rows that are not new hold anything: their values are not used
                const uint32_t at = ring + turn * kScStage + c * 1024;
                factor[c] = values(c * step + j0, mine >> c & 1, lds16(at), lds16(at + 512), x[c], y[c]);
                if (mine >> c & 1) top = magnitude(x[c], y[c], factor[c], top);
            }
        fetch(w + 2 * teams, turn);                      // what was read makes room
        further(w, [&](int, const F2 (&u)[N], const F2 (&v)[N], float f) { top = magnitude(u, v, f, top); });
        // over the block's lanes, then the team's warps; of a block with a NaN or an infinity
        // the largest finite value, with the sign bit for a mark
        for (int o = width / 2; o > 0; o >>= 1) top = top_of(top, __shfl_xor_sync(0xFFFFFFFFu, top, o), 0.f);
        if (__any_sync(0xFFFFFFFFu, !(top < INFINITY))) {
            const bool odd = !(top < INFINITY);
            float t = 0.f;
#pragma unroll
            for (int c = 0; c < kScKeep; ++c)
                if (mine >> c & 1) t = finite(x[c], y[c], factor[c], t);
            further(w, [&](int, const F2 (&u)[N], const F2 (&v)[N], float f) { t = finite(u, v, f, t); });
            for (int o = width / 2; o > 0; o >>= 1) t = fmaxf(t, __shfl_xor_sync(0xFFFFFFFFu, t, o));
            top = odd ? -t : t;
        }
        if (a.team > 1) {
            if (lane == 0) tops[turn][warp] = top;
            asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "r"(32 * a.team) : "memory");
            uint32_t mark = 0;
            float most = 0.f;
            for (int i = 0; i < a.team; ++i) {
                most = fmaxf(most, fabsf(tops[turn][team * a.team + i]));
                mark |= __float_as_uint(tops[turn][team * a.team + i]) & 0x80000000u;
            }
            top = __uint_as_float(__float_as_uint(most) | mark);
        } else {
            __syncwarp();                                // every lane has read the scale before it is written
        }
        if (!live) continue;
        const bool any_odd = __float_as_uint(top) >> 31;
        float s = power_of_two<FORMAT>(__float_as_uint(top) & 0x7FFFFFFFu);
        if (FORMAT == kInt8 && any_odd) s = __int_as_float(0x7FFFFFFF);   // int8 has no code for it: the block reads as NaN
        if (!(was < s) && !(s != s)) s = was;            // a NaN stays one
        const float per_s = s >= 1.17549435e-38f ? 1.f / s : 0.f;   // of 0 and what is not normal: no code but 0
        char *to = pages + w * a.cache.head_stride + page_at;
        if (thread == 0 && (j_new == 0 || s != was)) scale_at[(long long)w * a.scale_blocks] = s;
        if (j_new > 0 && was < s) {                      // earlier rows in the grown scale
            const float f = was / s;
#pragma unroll 4
            for (int e = thread; e < j_new * (D / 4); e += threads) {
                uint32_t *p = (uint32_t *)(to + e / (D / 4) * a.cache.row_stride) + e % (D / 4);
                float v[4];
                decode<FORMAT>(*p, v);
                *p = encode<FORMAT>(v[0] * f, v[1] * f, v[2] * f, v[3] * f);
            }
        }
        auto put = [&](int j, const F2 (&x)[N], const F2 (&y)[N], float factor) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                uint32_t c[E / 4];
#pragma unroll
                for (int e = 0; e < E / 4; ++e) {
                    F2 u = i ? y[2 * e] : x[2 * e], v = i ? y[2 * e + 1] : x[2 * e + 1];
                    if (KEYS) u = f2_mul(u, f2(factor, factor)), v = f2_mul(v, f2(factor, factor));
                    if (any_odd) {                       // e4m3: infinities become NaN
                        float f[4] = {f2_values(u).x, f2_values(u).y, f2_values(v).x, f2_values(v).y};
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if (!(fabsf(f[k]) < INFINITY)) f[k] = FORMAT == kE4m3 ? __int_as_float(0x7FFFFFFF) : 0.f;
                        u = f2(f[0], f[1]), v = f2(f[2], f[3]);
                    }
                    const float2 p = f2_values(f2_mul(u, f2(per_s, per_s))), q = f2_values(f2_mul(v, f2(per_s, per_s)));
                    c[e] = encode<FORMAT>(p.x, p.y, q.x, q.y);
                }
                char *at = to + j * a.cache.row_stride + i * (D / 2) + sub * E;
                if (E == 8) *(uint2 *)at = make_uint2(c[0], c[E / 4 - 1]);
                else *(uint32_t *)at = c[0];
            }
        };
#pragma unroll
        for (int c = 0; c < kScKeep; ++c)
            if (mine >> c & 1) put(c * step + j0, x[c], y[c], factor[c]);
        further(w, put);
    }
}

// Every a.every-th CTA stores keys or values, a.ctas in all; the others, if any, norm and
// rotate the queries.  With a.beside a kernel of their own does, launched before this
// one, which lets it start once its own wait is over: rows, lengths and cache are final
// then, the two run side by side, and the wait at the end makes this one's end the end of
// both.
template <typename T, int D, int FORMAT, bool ROWS>
__global__ void __launch_bounds__(kScThreads, 3) store_codes_kernel(NormRopeArgs q, StoreCodesArgs a) {
    extern __shared__ __align__(16) unsigned char dyn[];
    if (!a.beside) pdl_wait();
    pdl_trigger();
    const int i = (int)blockIdx.x, turn = a.by_every.of(i);
    if (turn * a.every == i && turn < a.ctas) {
        const int y = a.by_tiles.of(turn), run = turn - y * a.B * a.tasks;   // the keys' CTAs, which take longer, first
        if (y < a.splits) store_tile<T, D, FORMAT, true>(a, run, y * a.span, a.k, a.cache.k, a.k_scales, dyn);
        else store_tile<T, D, FORMAT, false>(a, run, (y - a.splits) * a.span, a.v, a.cache.v, a.v_scales, dyn);
    } else {
        norm_rope_rows<T, D, false, ROWS>(q, (unsigned)(i - min(turn + 1, a.ctas)), dyn);
    }
    if (a.beside) pdl_wait();
}

// Rows read back, 16 bytes of the result a lane: a CTA takes kRcRows rows of a
// sequence and walks over a.span of their heads.
constexpr int kRcThreads = 256;
constexpr int kRcRows = 16;
template <typename T, int D, int FORMAT>
__global__ void __launch_bounds__(kRcThreads) read_codes_kernel(ReadCodesArgs a) {
    constexpr int E = Vec16<T>::E, kLanes = D / E, kGroups = kRcThreads / kLanes;
    constexpr int kAhead = 4;            // rows and heads of a lane at a time, K and V of each
    pdl_wait();
    pdl_trigger();
    const int b = a.by_chunks.of((int)blockIdx.x), i0 = ((int)blockIdx.x - b * (int)a.by_chunks.d) * kRcRows;
    const int h0 = blockIdx.y * a.span, h1 = min(h0 + a.span, a.Hkv);
    const int n = min(row_count(a.n_rows, b, a.max_rows, a.err), i0 + kRcRows) - i0;
    if (n <= 0) return;
    const long long start = (a.start ? a.start[b] : 0) + (long long)i0, cap = (long long)a.cache.table_pages * a.cache.page_size;
    const int sub = threadIdx.x % kLanes;
    for (int e0 = threadIdx.x / kLanes; e0 < kRcRows * (h1 - h0); e0 += kAhead * kGroups) {
        uint32_t c[kAhead][2][E / 4];
        float s[kAhead][2];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int e = e0 + u * kGroups, r = e % kRcRows, h = h0 + e / kRcRows;
            s[u][0] = s[u][1] = 0.f;
#pragma unroll
            for (int w = 0; w < E / 4; ++w) c[u][0][w] = c[u][1][w] = 0u;
            if (h >= h1 || r >= n) continue;
            const long long slot = start + r;
            if (slot < 0 || slot >= cap) {
                set_err(a.err, kErrCache);
                continue;
            }
            const int idx = a.by_page.of((int)slot), row = (int)slot - idx * a.cache.page_size;
            const int page = a.cache.table[(long long)b * a.cache.table_pages + idx];
            if ((unsigned)page >= (unsigned)a.cache.n_pages) {
                set_err(a.err, kErrPage);
                continue;
            }
            const long long at = page * a.cache.page_stride + h * a.cache.head_stride + row * a.cache.row_stride + sub * E;
            const long long scale = ((long long)page * a.Hkv + h) * a.scale_blocks + a.by_scale.of(row);
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
            const int e = e0 + u * kGroups, r = e % kRcRows, h = h0 + e / kRcRows;
            if (h >= h1 || r >= n) continue;
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

cudaError_t prepare_store_codes_kernels(bool bf16, int D) {
    cudaError_t e = cudaSuccess;
    auto set = [&](auto k) {
        return e != cudaSuccess ? e : cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kScRing + 4 * D * kScAngles);
    };
    for (const CodeFormat format : {kE4m3, kInt8})
        e = with_codes(format, bf16, D, [&](auto t, auto d, auto form) {
            e = set(store_codes_kernel<decltype(t), d, form, false>);
            return set(store_codes_kernel<decltype(t), d, form, true>);
        });
    return e;
}

cudaError_t launch_store_codes(const NormRopeArgs &queries, const StoreCodesArgs &args, CodeFormat format, bool bf16, int D, int sms, cudaStream_t s) {
    NormRopeArgs q = queries;
    StoreCodesArgs a = args;
    static_assert(kNrThreads == kScThreads && kNrShared <= kScRing, "one launch");
    unsigned others = plan_norm_rope(q, bf16, D, false, sms);
    const int rows = 32 / (D / 2 / (bf16 ? 8 : 4)), R = a.scale_rows;   // rows a warp has at a time
    a.per = R < rows && rows % R == 0 ? rows / R : 1;
    a.team = 1;
    while (a.team < kScThreads / 32 && a.team * kScKeep * rows < R) a.team *= 2;
    const long long blocks = (a.max_new + 2LL * R - 2) / R;              // that a sequence's new rows may touch
    a.tasks = (int)((blocks + a.per - 1) / a.per);
    // heads of a CTA: fewer than all where the tiles alone give an SM less than four CTAs
    const long long tiles = (long long)a.B * a.tasks;
    const int teams = kScThreads / 32 / a.team;
    int splits = 1;
    while (splits * tiles < 2LL * sms && splits * teams < a.Hkv) splits *= 2;
    a.span = (a.Hkv + splits - 1) / splits;
    a.splits = (a.Hkv + a.span - 1) / a.span;
    a.ctas = (int)(tiles * 2 * a.splits);
    // one launch where all of it runs at once, else the queries' rows on a kernel that takes
    // less of an SM.  Measured, 32 query and 8 KV heads: 16 rows 3.7 and 4.1 us (and 2 us of a
    // launch), 8 prompts of 1021 to 2048 rows 67.5 and 57 us.
    a.beside = a.ctas + (long long)others > 3LL * sms;
    if (a.beside) {
        const cudaError_t e = launch_norm_rope(queries, bf16, D, false, sms, s);
        if (e != cudaSuccess) return e;
        others = 0;
    }
    a.every = (int)((a.ctas + (long long)others) / a.ctas);
    a.by_tasks = Divisor((uint32_t)a.tasks), a.by_tiles = Divisor((uint32_t)tiles), a.by_every = Divisor((uint32_t)a.every);
    a.by_scale = Divisor((uint32_t)R), a.by_page = Divisor((uint32_t)a.cache.page_size);
    const int angles = a.per > 1 ? rows : R < kScAngles ? R : kScAngles;
    const size_t shared = kScRing + sizeof(float) * D * angles;
    const dim3 grid((unsigned)a.ctas + others);
    return with_codes(format, bf16, D, [&](auto t, auto d, auto form) {
        using T = decltype(t);
        return launch_k(q.one_row ? store_codes_kernel<T, d, form, false> : store_codes_kernel<T, d, form, true>, grid, dim3(kScThreads), shared, s, true, q, a);
    });
}

cudaError_t launch_read_codes(const ReadCodesArgs &args, CodeFormat format, bool bf16, int D, int sms, cudaStream_t s) {
    ReadCodesArgs a = args;
    const unsigned chunks = (a.max_rows + kRcRows - 1) / (unsigned)kRcRows;
    // fewer heads a CTA where there would be less than one to an SM
    int splits = 1;
    while (splits < a.Hkv && (long long)a.B * chunks * splits < sms) splits *= 2;
    a.span = (a.Hkv + splits - 1) / splits;
    a.by_chunks = Divisor(chunks), a.by_scale = Divisor((uint32_t)a.scale_rows), a.by_page = Divisor((uint32_t)a.cache.page_size);
    const dim3 grid(a.B * chunks, (unsigned)((a.Hkv + a.span - 1) / a.span));
    return with_codes(format, bf16, D, [&](auto t, auto d, auto form) {
        return launch_k(read_codes_kernel<decltype(t), d, form>, grid, dim3(kRcThreads), 0, s, true, a);
    });
}

}  // namespace prism
