// Rows quantised as they are written to a paged cache held in 8 bits.
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
// 2048 rows 56 us (277 MB, 5.0 TB/s: the queries' kernel 33, keys and values mostly behind
// it), 16 tokens 3.3 us, 16 sequences of 4 rows 5.2, of 16 rows 6.4.
#pragma once

#include "paged_rope.cuh"

#include <type_traits>

namespace prism {
namespace {

constexpr int kScThreads = 128;
constexpr int kScAngles = 64;            // rows of a tile whose angles are kept in shared memory, at most
// Rows of a lane group kept in registers between a block's maximum and its codes: KEEP.
template <int KEEP> constexpr int kScStage = KEEP * 1024;    // bytes of a warp's rows of one head: two pieces a lane and row
template <int KEEP> constexpr int kScRing = kScThreads / 32 * 2 * kScStage<KEEP>;
constexpr int kScChained = 8192;         // bytes of a tile's angles, at most, where tiles are chained: three of them
constexpr size_t kScShared = kScRing<4> + 4 * 128 * kScAngles;   // at most
static_assert(3 * kScChained <= 4 * 128 * kScAngles, "of chained tiles");
template <int KEEP> constexpr int kScCtas = KEEP == 4 ? 3 : KEEP == 2 ? 4 : 5;   // an SM's

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

// A CTA takes a.chain tiles of rows one after the other, a tile being a block's rows or
// with a.per > 1 those of a.per short blocks that a warp has side by side, and a.span of
// their heads of K or of V; what depends on the rows alone (lengths, place, angles) is
// found once a tile.  A team of a.team warps takes a head: rows of lanes as in the norm
// (E values at j and at j + D/2 each), the block's largest value over the team, then the
// codes, the next two heads' or tiles' rows on their way meanwhile.  Up to KEEP rows a
// lane group stay in registers; longer blocks' further rows are read and computed again.
//
// What keeps a warp waiting most is its own code, of which little fits near the
// scheduler: KEEP 1 and 2 (and more CTAs with them) where blocks need no more, and one
// instance of what is rare.  Measured, 8 query heads, 8 prompts, blocks of 1 and 8: 41 and
// 37 us, KEEP 4 64 and 46.
template <typename T, int D, int FORMAT, int KEEP, bool KEYS>
__device__ __forceinline__ void store_tile(const StoreCodesArgs &a, int run, int w0, const HeadsView &rows, char *pages, float *scales, unsigned char *dyn) {
    using R = Rope<T, D>;
    constexpr int N = R::N, E = R::E, kRows = R::kHeads;   // rows a warp has at a time
    constexpr int kStage = kScStage<KEEP>, kRing = kScRing<KEEP>;
    // the warps' maxima, of two turns: what a warp writes in one, its team has read before
    // the barrier of the turn between
    __shared__ float tops[2][kScThreads / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane % R::kLanes, group = lane / R::kLanes;
    const int team = warp / a.team, teams = kScThreads / 32 / a.team, in_team = warp - team * a.team;
    const int b = a.by_tasks.of(run), t0 = (run - b * a.tasks) * a.chain;
    const int w1 = min(w0 + a.span, a.Hkv), items = (w1 - w0 + teams - 1) / teams;   // heads of a team, at most
    const int in_warp = a.per > 1 ? a.by_scale.of(group) : 0;    // this lane's block of the warp's
    const int step = kRows * a.team;
    const int held = a.cache.kv_len[b], cap = a.cache.table_pages * a.cache.page_size, pos = KEYS ? a.pos[b] : 0;
    const bool fits = held >= 0 && held <= cap;          // no slot beyond a length that does not is a row's
    const int len = fits ? held : 0, n = row_count(a.n_new, b, a.max_new, a.err);
    const int block0 = a.by_scale.of(len);
    // A tile's rows: a block's are slots first + j, 0 <= j < scale_rows; new ones from j_new
    // on, up to j_end.  This lane's rows are j0 + c step: turns c of the warp with a new row,
    // and those in which this lane's is one.
    struct Tile {
        int first, j_new, j_end, j0;
        uint32_t turns, mine;
    };
    auto tile_at = [&](int t) {
        Tile x;
        x.first = (block0 + t * a.per + in_warp) * a.scale_rows;
        x.j_new = max(len - x.first, 0), x.j_end = min(max(len + n - x.first, 0), a.scale_rows);
        x.j0 = a.per > 1 ? group - in_warp * a.scale_rows : (KEEP == 1 ? x.j_new / kRows : in_team) * kRows + group;
        x.turns = 1, x.mine = 0;
        if (KEEP > 1) {
            x.turns = 0;
#pragma unroll
            for (int c = 0; c < KEEP; ++c) {
                const int at = c * step + in_team * kRows;
                x.turns |= (at < x.j_end && at + kRows > x.j_new) << c;
            }
        }
#pragma unroll
        for (int c = 0; c < KEEP; ++c) x.mine |= (x.turns >> c & 1 && c * step + x.j0 >= x.j_new && c * step + x.j0 < x.j_end) << c;
        return x;
    };
    auto source = [&](const Tile &x) { return rows.p + (long long)b * rows.sb + (long long)(x.j0 + x.first - len) * rows.st + sub * 16; };
    // new row i's angles, held to the table; of a tile's first kScAngles rows they are kept
    auto position = [&](int i) {
        const long long at = (long long)pos + i;
        if (at >= 0 && at < a.rope_len) return (int)at;
        set_err(a.err, kErrPosition);
        return at < 0 ? 0 : a.rope_len - 1;
    };
    // This lane's rows of a head, requested two heads ahead, of the next tile too, and before
    // their place is known; each lane copies what it reads itself, so that its own waits are
    // enough.  A tile's angles, which the CTA shares, come with its first rows, to one of three
    // places: the tile computed and the two ahead.
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(dyn) + warp * (2 * kStage) + lane * 16;
    const uint32_t angles_at = (uint32_t)__cvta_generic_to_shared(dyn + kRing);
    const int kept = a.per > 1 ? kRows : min(a.scale_rows, kScAngles), angle_bytes = kept * (D * 4);
    int ahead_t = 0, ahead_i = 0;
    uint32_t ahead_angles = angles_at;
    Tile ahead = tile_at(t0);
    auto fetch = [&](int stage) {
        if (ahead_t < a.chain) {
            if (KEYS && ahead_i == 0 && fits) {
                const int i0 = (block0 + (t0 + ahead_t) * a.per) * a.scale_rows - len;
                for (int e = threadIdx.x; e < kept * (D / 4); e += kScThreads) {
                    const int i = i0 + e / (D / 4);
                    if (i >= 0 && i < n) cp16(ahead_angles + 16 * e, a.rope + (long long)position(i) * D + 4 * (e % (D / 4)), true);
                }
            }
            const int w = w0 + team + ahead_i * teams;
            if (w < w1) {
                const char *from = source(ahead) + w * rows.sh;
#pragma unroll
                for (int c = 0; c < KEEP; ++c) {
                    if (ahead.mine >> c & 1) {
                        cp16(ring + stage * kStage + c * 1024, from, true);
                        cp16(ring + stage * kStage + c * 1024 + 512, from + D / 2 * sizeof(T), true);
                    }
                    from += step * rows.st;
                }
            }
            if (++ahead_i == items) {
                ahead_i = 0;
                ++ahead_t;
                ahead_angles += angle_bytes;
                if (ahead_angles == angles_at + 3 * angle_bytes) ahead_angles = angles_at;
                ahead = tile_at(t0 + ahead_t);
            }
        }
        cp_group();
    };
    fetch(0);
    fetch(1);
    Gain<T, D> gain;
    const bool norm = a.g_k != nullptr;
    if (KEYS && norm) gain.load(a.g_k);
    Tile at{};                                           // the tile computed
    uint32_t angles = angles_at;
    // Row j's values from what was read of it, before the norm's factor, which is returned.
    // The gain times a bf16 value is exact, and the factor meets a sum that is already
    // turned: two roundings fewer than in the order of the formula, and as many products.
    auto values = [&](int j, bool in, const uint4 &l, const uint4 &r, F2 (&x)[N], F2 (&y)[N]) {
        Pairs<T>::unpack(l, x);
        Pairs<T>::unpack(r, y);
        if (!KEYS) return 1.f;
        R rope;
        const int own = !in ? 0 : a.per > 1 ? group : j;  // a turn's last rows may be past the block's
        if (own < kScAngles) rope.load_shared(angles + own * (D * 4));
        else rope.load(a.rope, in ? position(j + at.first - len) : 0);
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
            const F2 q = f2_mul(x[e], rope.sn[e]);
            const float2 u = f2_values(x[e]), c = f2_values(rope.cs[e]), p = f2_values(f2_mul(y[e], rope.sn[e]));
            x[e] = f2(fmaf(u.x, c.x, -p.x), fmaf(u.y, c.y, -p.y));   // a pair has no negated operand
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
        if (KEEP == 4 && a.per == 1)
            for (int c = KEEP; c * step < at.j_end; ++c) {
                const int j = c * step + at.j0;
                const bool in = j >= at.j_new && j < at.j_end;
                uint4 l = make_uint4(0u, 0u, 0u, 0u), r = l;
                if (in) {
                    const char *from = source(at) + w * rows.sh + c * step * rows.st;
                    l = *(const uint4 *)from;
                    r = *(const uint4 *)(from + D / 2 * sizeof(T));
                }
                F2 u[N], v[N];
                const float factor = values(j, in, l, r, u, v);
                if (in) f(j, u, v, factor);
            }
    };
    auto team_barrier = [&]() { asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "r"(32 * a.team) : "memory"); };
    const int width = a.per > 1 ? R::kLanes * a.scale_rows : 32;   // lanes of a block
    const int thread = a.per > 1 ? lane % width : in_team * 32 + lane, threads = a.per > 1 ? width : 32 * a.team;
    int page = 0, row = 0, item = items, tile = t0 - 1;
    bool placed = false;                                 // a new row, and a place for its block
    for (int turn = 0;; turn ^= 1, ++item) {
        if (item == items) {                             // the next tile
            item = 0;
            if (++tile == t0 + a.chain) break;
            at = tile_at(tile);
            placed = at.j_new < at.j_end;
            if (!__any_sync(0xFFFFFFFFu, placed)) break; // the same for every warp of the CTA
            if (placed && (!fits || at.first >= cap)) {
                set_err(a.err, kErrCache);
                placed = false;
            }
            if (placed) {
                const int slot = a.by_page.of(at.first);
                row = at.first - slot * a.cache.page_size;
                page = a.cache.table[(long long)b * a.cache.table_pages + slot];
            }
        }
        const int w = w0 + team + item * teams;
        cp_wait_group<1>();
        if (KEYS && item == 0) {
            __syncthreads();                             // the angles are there
            if (tile > t0) {
                angles += angle_bytes;
                if (angles == angles_at + 3 * angle_bytes) angles = angles_at;
            }
        }
        if (w >= w1) {                                   // a team without a head passes its barrier too: see tops
            if (KEEP == 4 && a.team > 1) team_barrier();
            fetch(turn);
            continue;
        }
        const bool live = placed && (unsigned)page < (unsigned)a.cache.n_pages;
        float *const scale_at = scales + ((long long)page * a.Hkv + w) * a.scale_blocks + a.by_scale.of(row);
        const float was = live && at.j_new > 0 ? *scale_at : 0.f;
        F2 x[KEEP][N], y[KEEP][N];
        float factor[KEEP], top = 0.f;
#pragma unroll
        for (int c = 0; c < KEEP; ++c)
            if (at.turns >> c & 1) {                     // rows that are not new hold anything: their values are not used
                const uint32_t from = ring + turn * kStage + c * 1024;
                factor[c] = values(c * step + at.j0, at.mine >> c & 1, lds16(from), lds16(from + 512), x[c], y[c]);
                const float more = magnitude(x[c], y[c], factor[c], top);
                top = at.mine >> c & 1 ? more : top;
            }
        fetch(turn);                                     // what was read makes room
        // over the block's lanes, then the team's warps; of a block with a NaN or an infinity
        // the largest finite value, with the sign bit for a mark
        bool odd = false;
        for (int pass = 0;; ++pass) {
            further(w, [&](int, const F2 (&u)[N], const F2 (&v)[N], float f) { top = pass ? finite(u, v, f, top) : magnitude(u, v, f, top); });
            for (int o = width / 2; o > 0; o >>= 1) top = top_of(top, __shfl_xor_sync(0xFFFFFFFFu, top, o), 0.f);
            if (pass) break;
            odd = !(top < INFINITY);
            if (!__any_sync(0xFFFFFFFFu, odd)) break;
            top = 0.f;
#pragma unroll
            for (int c = 0; c < KEEP; ++c)
                if (at.mine >> c & 1) top = finite(x[c], y[c], factor[c], top);
        }
        if (odd) top = -top;
        if (KEEP == 4 && a.team > 1) {
            if (lane == 0) tops[turn][warp] = top;
            team_barrier();
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
        if (placed && !live) set_err(a.err, kErrPage);
        if (!live) continue;
        const bool any_odd = __float_as_uint(top) >> 31;
        float s = power_of_two<FORMAT>(__float_as_uint(top) & 0x7FFFFFFFu);
        if (FORMAT == kInt8 && any_odd) s = __int_as_float(0x7FFFFFFF);   // int8 has no code for it: the block reads as NaN
        if (!(was < s) && !(s != s)) s = was;            // a NaN stays one
        const float per_s = s >= 1.17549435e-38f ? 1.f / s : 0.f;   // of 0 and what is not normal: no code but 0
        char *to = pages + w * a.cache.head_stride + page * a.cache.page_stride + row * a.cache.row_stride;
        if (thread == 0 && (at.j_new == 0 || s != was)) *scale_at = s;
        if (at.j_new > 0 && was < s) {                      // earlier rows in the grown scale
            const float f = was / s;
#pragma unroll (KEEP == 1 ? 4 : 1)
            for (int e = thread; e < at.j_new * (D / 16); e += threads) {
                uint4 *p = (uint4 *)(to + e / (D / 16) * a.cache.row_stride) + e % (D / 16);
                uint4 c = *p;
                uint32_t *word = &c.x;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float v[4];
                    decode<FORMAT>(word[i], v);
                    word[i] = encode<FORMAT>(v[0] * f, v[1] * f, v[2] * f, v[3] * f);
                }
                *p = c;
            }
        }
        // a block's with what has no code: e4m3's NaN, or 0
        auto mended = [&](F2 (&x)[N], F2 (&y)[N], float &factor) {
            auto one = [&](float z) { return fabsf(z * factor) < INFINITY ? z * factor : FORMAT == kE4m3 ? __int_as_float(0x7FFFFFFF) : 0.f; };
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float2 u = f2_values(x[e]), v = f2_values(y[e]);
                x[e] = f2(one(u.x), one(u.y)), y[e] = f2(one(v.x), one(v.y));
            }
            factor = 1.f;
        };
        if (any_odd) {
#pragma unroll
            for (int c = 0; c < KEEP; ++c)
                if (at.mine >> c & 1) mended(x[c], y[c], factor[c]);
        }
        auto put = [&](char *row, bool in, const F2 (&x)[N], const F2 (&y)[N], float factor) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                uint32_t c[E / 4];
#pragma unroll
                for (int e = 0; e < E / 4; ++e) {
                    F2 u = i ? y[2 * e] : x[2 * e], v = i ? y[2 * e + 1] : x[2 * e + 1];
                    if (KEYS) u = f2_mul(u, f2(factor, factor)), v = f2_mul(v, f2(factor, factor));
                    const float2 p = f2_values(f2_mul(u, f2(per_s, per_s))), q = f2_values(f2_mul(v, f2(per_s, per_s)));
                    c[e] = encode<FORMAT>(p.x, p.y, q.x, q.y);
                }
                char *p = row + i * (D / 2);
                if (in) {
                    if (E == 8) *(uint2 *)p = make_uint2(c[0], c[E / 4 - 1]);
                    else *(uint32_t *)p = c[0];
                }
            }
        };
        char *own = to + at.j0 * a.cache.row_stride + sub * E;
        const long long next = step * a.cache.row_stride;
#pragma unroll
        for (int c = 0; c < KEEP; ++c, own += next)
            if (at.turns >> c & 1) put(own, at.mine >> c & 1, x[c], y[c], factor[c]);
        further(w, [&](int j, F2 (&u)[N], F2 (&v)[N], float f) {
            if (any_odd) mended(u, v, f);
            put(to + j * a.cache.row_stride + sub * E, true, u, v, f);
        });
    }
    cp_wait_group<0>();
}

// Every a.every-th CTA stores keys or values, a.ctas in all; the others, if any, norm and
// rotate the queries.  With a.beside a kernel of their own does, launched before this
// one, which lets it start once its own wait is over: rows, lengths and cache are final
// then, this one's CTAs run where the other's leave room (most of them when those end: 33
// us and 22 more), and the wait at the end makes this one's end the end of both.
template <typename T, int D, int FORMAT, int KEEP>
__global__ void __launch_bounds__(kScThreads, kScCtas<KEEP>) store_codes_kernel(NormRopeArgs q, StoreCodesArgs a) {
    extern __shared__ __align__(16) unsigned char dyn[];
    if (!a.beside) pdl_wait();
    pdl_trigger();
    const int i = (int)blockIdx.x, turn = a.by_every.of(i);
    if (turn * a.every == i && turn < a.ctas) {
        const int y = a.by_tiles.of(turn), run = turn - y * a.B * a.tasks;   // the keys' CTAs, which take longer, first
        if (y < a.splits) store_tile<T, D, FORMAT, KEEP, true>(a, run, y * a.span, a.k, a.cache.k, a.k_scales, dyn);
        else store_tile<T, D, FORMAT, KEEP, false>(a, run, (y - a.splits) * a.span, a.v, a.cache.v, a.v_scales, dyn);
    } else {
        norm_rope_rows<T, D, false, false>(q, (unsigned)(i - min(turn + 1, a.ctas)), dyn);
    }
    if (a.beside) pdl_wait();
}

template <typename F> cudaError_t with_rows(bool bf16, int D, const F &f) {
    const std::integral_constant<int, 64> small;
    const std::integral_constant<int, 128> large;
    if (bf16) return D == 128 ? f(uint16_t(), large) : f(uint16_t(), small);
    return D == 128 ? f(0.f, large) : f(0.f, small);
}
template <int FORMAT> cudaError_t prepare_store(bool bf16, int D) {
    return with_rows(bf16, D, [&](auto t, auto d) {
        return cudaFuncSetAttribute(store_codes_kernel<decltype(t), d, FORMAT, 4>, cudaFuncAttributeMaxDynamicSharedMemorySize, kScShared);
    });
}
template <int FORMAT> cudaError_t start_store(const NormRopeArgs &q, const StoreCodesArgs &a, bool bf16, int D, unsigned ctas, size_t shared, cudaStream_t s) {
    return with_rows(bf16, D, [&](auto t, auto d) {
        using T = decltype(t);
        auto go = [&](auto k) {
            return launch_k(store_codes_kernel<T, d, FORMAT, k>, dim3(ctas), dim3(kScThreads), shared, s, true, q, a);
        };
        return a.keep == 4 ? go(std::integral_constant<int, 4>()) : a.keep == 2 ? go(std::integral_constant<int, 2>()) : go(std::integral_constant<int, 1>());
    });
}

}  // namespace
}  // namespace prism
