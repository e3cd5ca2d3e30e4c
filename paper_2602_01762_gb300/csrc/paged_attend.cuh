// Attention of one new token over a paged cache: the kernel, apart from what a tile
// of rows does (paged_attend_tiles.cuh, paged_attend_codes.cuh).
#pragma once

#include "paged.cuh"
#include "paged_scores.h"

namespace prism {
namespace {

constexpr int kPaWarps = 4;
constexpr int kPaThreads = 32 * kPaWarps;
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

// A segment is one (sequence, KV head, head tile): blocks of kAttendUnit keys, and
// before them P::kCost units without keys that stand for what a segment costs
// beside its rows (its queries, merge and result).
__device__ __forceinline__ int blocks_of(int len) { return max(1, (len + kAttendUnit - 1) / kAttendUnit); }

// The rows of a sequence that are attended to (paged_rows.h).
struct AllRows {
    int len;
    __device__ __forceinline__ void set(const AttendArgs &, int n) { len = n; }
    __device__ __forceinline__ int count() const { return len; }
    __device__ __forceinline__ int key(int r) const { return r; }
    __device__ __forceinline__ bool sees(int key) const { return key < len; }
};
struct WindowRows : SeenRows {
    __device__ __forceinline__ void set(const AttendArgs &a, int n) { SeenRows::set(n, a.window, a.sinks); }
};
template <typename Rows> __device__ __forceinline__ int seen_rows(const AttendArgs &a, int len) {
    Rows r;
    r.set(a, len);
    return r.count();
}

// Walk over the pieces of a CTA's share: the blocks [blk0, blk1) of nblk of one
// segment after the other; parts of a segment without blocks are passed over.  Each
// lane keeps the length of one of the next 32 sequences, so that a step waits for
// no load.
template <typename Rows, int COST> struct Pieces {
    int u, u1, seg, b, h, heads, blk0, blk1, nblk;   // seg: the segment's first unit
    Rows seen;
    int base, lens;                      // lane i: rows of sequence base + i
    __device__ __forceinline__ void fetch(const AttendArgs &a) {
        const int at = b + (int)(threadIdx.x & 31);
        base = b;
        lens = at < a.B ? paged_len(a.cache, at, a.added, a.err) : 0;
    }
    __device__ __forceinline__ void sequence(const AttendArgs &a) {
        seen.set(a, __shfl_sync(0xFFFFFFFFu, lens, b - base));
        nblk = blocks_of(seen.count());
    }
    __device__ __forceinline__ bool cut() {
        blk0 = max(u - seg - COST, 0);
        u = min(seg + COST + nblk, u1);
        blk1 = max(u - seg - COST, 0);
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
        sequence(a);
        h = (u - r.first) / (COST + nblk);
        seg = r.first + h * (COST + nblk);
        return cut() || next(a);
    }
    // A cluster's rank takes its run of the blocks of segment i, and no other piece.
    __device__ __forceinline__ void only(const AttendArgs &a, int i, int rank, int n_heads) {
        u = u1 = seg = base = lens = 0;
        heads = n_heads;
        b = i / heads;
        h = i - b * heads;
        seen.set(a, paged_len(a.cache, b, a.added, a.err));
        nblk = blocks_of(seen.count());
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
                sequence(a);
            }
            if (cut()) return true;
        }
        return false;
    }
    __device__ __forceinline__ int rows() const { return min(blk1 * kAttendUnit, seen.count()) - blk0 * kAttendUnit; }
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
    static constexpr int kRound = kPaWarps * P::kStages * P::kStage / (4 * kPart);   // pieces that the rings hold
    static constexpr int kGroup = kRound > 16 && !P::kScaled ? kRound : 16;
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

// The loads of a warp: a walk over the pieces of its own, and the pool place of each
// lane's row of the next two tiles.
template <typename P, typename Rows> struct RowFeed {
    static constexpr int KT = P::KT, S = P::kStages, kStage = P::kStage, kRow = P::kRow, kChunks = kRow / 16, kRowsPer = 32 / kChunks;
    struct Place {
        int page, row, head;
        bool in, live;                                   // a row that counts; a tile at all
    };
    Pieces<Rows, P::kCost> f;
    Place next0, next1;
    uint64_t once;
    uint32_t ring;
    int ft, warp, tiles, stage_in;
    bool more;
    __device__ __forceinline__ uint32_t free_stage() const { return ring + stage_in * kStage; }
    __device__ __forceinline__ void begin(const AttendArgs &a, const Pieces<Rows, P::kCost> &p, uint32_t at, int w, int n_tiles) {
        f = p;
        ft = warp = w;
        tiles = n_tiles;
        ring = at;
        stage_in = 0;
        // K and V leave L2 first, so that scores, weights and pieces stay for the next reader
        // (up to 16 query heads a KV head read them once; the next head tile of more reads them again)
        once = l2_evict_first_policy();
        more = true;
        while (more && ft * KT >= f.rows()) more = f.next(a);
        next0 = look_up(a);
        next1 = look_up(a);
    }
    __device__ __forceinline__ Place look_up(const AttendArgs &a) {   // lane's row of the walk's tile (lanes past KT repeat), then on
        Place w{0, 0, f.h / tiles, false, more};
        if (!more) return w;
        const int key = f.seen.key(f.blk0 * kAttendUnit + ft * KT) + (int)(threadIdx.x & 31) % KT;
        const int slot = (unsigned)key / (unsigned)a.cache.page_size;
        w.in = f.seen.sees(key);
        w.row = key - slot * a.cache.page_size;
        if (w.in) w.page = a.cache.table[(long long)f.b * a.cache.table_pages + slot];
        ft += kPaWarps;
        while (more && ft * KT >= f.rows()) {
            more = f.next(a);
            ft = warp;
        }
        return w;
    }
    __device__ __forceinline__ void issue(const AttendArgs &a) {
        if (next0.live) {
            const int lane = threadIdx.x & 31;
            const bool known = (unsigned)next0.page < (unsigned)a.cache.n_pages;
            if (next0.in && !known) set_err(a.err, kErrPage);
            const int ok = next0.in && known;
            const long long off = ok ? next0.page * a.cache.page_stride + next0.head * a.cache.head_stride + next0.row * a.cache.row_stride : 0;
            const uint32_t ks = ring + stage_in * kStage, vs = ks + KT * kRow;
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
        next1 = look_up(a);
        stage_in = stage_in + 1 == S ? 0 : stage_in + 1;
    }
};

// The same for 8-bit rows and their scales, one tile of one or two runs of kRunRows rows
// ahead.
// Where runs divide pages and offsets are short (a.run), a run lies in one page and all
// but its page and row is known from the piece or from the launch.
constexpr int kRunRows = 16;
template <typename P, typename Rows> struct CodeFeed {
    static constexpr int KT = P::KT, S = P::kStages, kStage = P::kStage, kRow = P::kRow, kChunks = kRow / 16, kRowsPer = 32 / kChunks;
    static constexpr int kStep = kPaWarps * KT, kCopies = kRunRows / kRowsPer, kAll = (1 << kCopies) - 1;
    static constexpr int kRuns = KT / kRunRows;
    static_assert(KT == kRuns * kRunRows && (kRuns == 1 || kRuns == 2), "a lane's scale is that of its row");
    Pieces<Rows, P::kCost> f;
    const int32_t *table;                                // of the sequence
    const char *k_at, *v_at;                             // of the head and of this lane's part of a run
    const float *scales;                                 // K's of the head (of one run: V's in the upper lanes)
    uint64_t once;
    uint32_t to, ring_end;                               // the next stage, which is free; the last one's end
    uint32_t piece[2];                                   // of this lane's copies, even and odd ones
    int place, end, warp, tiles;
    int page[kRuns], row[kRuns], in[kRuns];              // next tile's runs: bit i: this lane's row of copy i counts
    int own;                                             // and whether row lane % KT of the tile does
    bool more, live;
    __device__ __forceinline__ uint32_t free_stage() const { return to; }
    __device__ __forceinline__ void begin(const CodeAttendArgs &a, const Pieces<Rows, P::kCost> &p, uint32_t at, int w, int n_tiles) {
        const int lane = threadIdx.x & 31;
        f = p;
        warp = w;
        tiles = n_tiles;
        to = at;
        ring_end = at + S * kStage;
        once = l2_evict_first_policy();                  // see RowFeed
#pragma unroll
        for (int i = 0; i < 2; ++i) piece[i] = P::piece(i * kRowsPer + lane / kChunks, lane % kChunks);
        enter(a);
        more = true;
        walk(a);
        look_up(a);
    }
    __device__ __forceinline__ void enter(const CodeAttendArgs &a) {
        const int lane = threadIdx.x & 31, head = tiles == 1 ? f.h : f.h / tiles;
        const long long at = head * a.cache.head_stride + (a.run ? lane / kChunks * a.cache.row_stride : 0) + lane % kChunks * 16;
        table = a.cache.table + (long long)f.b * a.cache.table_pages;
        k_at = a.cache.k + at;
        v_at = a.cache.v + at;
        scales = (kRuns == 2 || lane < KT ? a.k_scales : a.v_scales) + (long long)head * a.scale_blocks;
        place = f.blk0 * kAttendUnit + warp * KT;
        end = f.blk0 * kAttendUnit + f.rows();
    }
    __device__ __forceinline__ void walk(const CodeAttendArgs &a) {
        while (place >= end) {
            more = f.next(a);
            if (!more) break;
            enter(a);
        }
    }
    __device__ __forceinline__ void look_up(const CodeAttendArgs &a) {
        live = more;
        if (!more) return;
        const int lane = threadIdx.x & 31, key = f.seen.key(place);
        const bool all = f.seen.sees_all(key, KT);
        own = all || f.seen.sees(key + lane % KT);
        if (a.run) {
#pragma unroll
            for (int j = 0; j < kRuns; ++j) {
                const int k = key + j * kRunRows, slot = a.by_page.of(k);
                row[j] = k - slot * a.cache.page_size;
                in[j] = kAll;
                page[j] = 0;
                if (all || f.seen.sees_any(k, kRunRows)) page[j] = table[slot];
                if (!all) {
                    in[j] = 0;
#pragma unroll
                    for (int i = 0; i < kCopies; ++i) in[j] |= f.seen.sees(k + i * kRowsPer + lane / kChunks) << i;
                }
            }
        } else {                                         // this lane's row (lanes past KT repeat)
            const int slot = a.by_page.of(key + lane % KT);
            row[0] = key + lane % KT - slot * a.cache.page_size;
            page[0] = own ? table[slot] : 0;
        }
    }
    // Shared address of this lane's copy i: rows come back to the same banks every other copy.
    __device__ __forceinline__ uint32_t place_of(int i) const { return to + piece[i & 1] + (i >> 1) * (2 * kRowsPer * kRow); }
    // One run's. STEP: bytes from a copy's row to the next one's, 0 unless they are dense.
    template <int STEP> __device__ __forceinline__ void copies(const CodeAttendArgs &a, int j, bool known) {
        const long long at = (long long)page[j] * a.short_page + (long long)row[j] * a.short_row;
        const char *kp = k_at + at, *vp = v_at + at;
        if (known && in[j] == kAll) {
#pragma unroll
            for (int i = 0; i < kCopies; ++i) {
                cp16_once(place_of(j * kCopies + i), kp + i * STEP, once);
                cp16_once(place_of(j * kCopies + i) + KT * kRow, vp + i * STEP, once);
                if (!STEP) kp += kRowsPer * a.short_row, vp += kRowsPer * a.short_row;
            }
        } else {
#pragma unroll
            for (int i = 0; i < kCopies; ++i) {
                const bool ok = known && (in[j] >> i & 1);
                cp16_once(place_of(j * kCopies + i), kp + i * STEP, ok, once);
                cp16_once(place_of(j * kCopies + i) + KT * kRow, vp + i * STEP, ok, once);
                if (!STEP) kp += kRowsPer * a.short_row, vp += kRowsPer * a.short_row;
            }
        }
    }
    __device__ __forceinline__ void issue(const CodeAttendArgs &a) {
        if (live) {
            const int lane = threadIdx.x & 31;
            const float *s;
            bool ok = own;
            if (a.run) {
                bool known[kRuns];
#pragma unroll
                for (int j = 0; j < kRuns; ++j) {
                    known[j] = (unsigned)page[j] < (unsigned)a.cache.n_pages;
                    if (!known[j]) {
                        set_err(a.err, kErrPage);        // an unseen run has page 0
                        page[j] = 0;
                    }
                    if (a.run == 2) copies<kRowsPer * kRow>(a, j, known[j]);
                    else copies<0>(a, j, known[j]);
                }
                constexpr int last = kRuns - 1;
                ok = ok && (lane < kRunRows ? known[0] : known[last]);
                const int p = lane < kRunRows ? page[0] : page[last], r = lane < kRunRows ? row[0] : row[last];
                s = scales + (p * a.page_scales + a.by_scale.of(r + lane % kRunRows));
            } else {
                if ((unsigned)page[0] >= (unsigned)a.cache.n_pages) {
                    set_err(a.err, kErrPage);
                    ok = false;
                    page[0] = 0;
                }
                const long long off = page[0] * a.cache.page_stride + row[0] * a.cache.row_stride;
#pragma unroll
                for (int i = 0; i < KT / kRowsPer; ++i) {
                    const int r = i * kRowsPer + lane / kChunks;
                    const long long at = __shfl_sync(0xFFFFFFFFu, off, r);
                    const bool in_r = __shfl_sync(0xFFFFFFFFu, (int)ok, r);
                    cp16_once(place_of(i), k_at + at, in_r, once);
                    cp16_once(place_of(i) + KT * kRow, v_at + at, in_r, once);
                }
                s = scales + (page[0] * (long long)a.Hkv * a.scale_blocks + a.by_scale.of(row[0]));
            }
            // the rows' scales behind them, K's, then V's
            const uint32_t st = to + 2 * KT * kRow + 4 * lane;
            cp4(st, s, ok);
            if (kRuns == 2) cp4(st + 4 * KT, s + (a.v_scales - a.k_scales), ok);
            place += kStep;
            if (place >= end) walk(a);
            look_up(a);
        }
        cp_group();
        to += kStage;
        if (to == ring_end) to -= S * kStage;
    }
};
template <typename P, typename Rows, bool SCALED = P::kScaled> struct FeedOf { using type = RowFeed<P, Rows>; };
template <typename P, typename Rows> struct FeedOf<P, Rows, true> { using type = CodeFeed<P, Rows>; };

// Rings, then a sum area (P::kScaled: one for a cluster's sums, a warp's own goes to its
// ring's free stage; else one for each warp), then maxima and sums.
template <typename P> constexpr int kAttendSums = P::kScaled ? 4 * P::kHeads * (P::D + 2) : kPaWarps * 4 * P::kHeads * P::kMergeStride;
template <typename P> constexpr size_t attend_smem() {
    static_assert(!P::kScaled || 4 * P::kHeads * P::kMergeStride <= P::kStage, "a stage holds a warp's sums");
    return (size_t)kPaWarps * (P::kStages * P::kStage + 8 * P::kHeads) + kAttendSums<P>;
}

// Persistent CTAs of four warps, P::kCtas per SM.  The ragged (sequence, KV head,
// block of 64 keys) units are cut into equal contiguous shares, one per CTA, so
// that long and short sequences keep every SM equally busy; a segment cut between
// CTAs is joined by the last of them to finish (in CTA order: the result does not
// depend on which that is).  Within a CTA the tiles of KT keys go to the warps in
// turn, each with its own ring of stages filled by cp.async, its own online
// softmax and no barrier until the segment's end; the ring runs on across
// segments, so loads never stop.
//
// CLUSTER, for few short segments: a cluster of a.cluster CTAs (or one CTA) takes one
// segment, each an equal run of its blocks, and joins through distributed shared memory
// instead of tickets and loads from L2.
//
// Rows says which rows of a sequence are seen; the others are not read, and their
// block-table entries neither.  P::kScaled: 8-bit rows with a scale for each.
template <typename P, bool CLUSTER, typename Rows>
__global__ void __launch_bounds__(kPaThreads, P::kCtas) paged_attend_kernel(const typename P::Args a) {
    using T = typename P::T;
    constexpr int D = P::D, KT = P::KT, S = P::kStages, H = P::kHeads, kStage = P::kStage;
    constexpr int kPart = Joined<P>::kPart, kGroup = Joined<P>::kGroup;   // kPart: sums [H][D], then (maximum, sum) [H]
    constexpr int kRow = P::kRow;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ Cut joins[2];
    __shared__ int join_group[2], last;
    int pending = 0;                                     // of thread 0
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    pdl_wait();
    pdl_trigger();

    const int G = a.Hq / a.Hkv, tiles = (G + H - 1) / H, heads = a.Hkv * tiles;
    UnitRange r;
    Pieces<Rows, P::kCost> p;                                      // the piece being computed
    const int rank = CLUSTER ? (int)blockIdx.x % a.cluster : 0;
    if (CLUSTER) {
        p.only(a, blockIdx.x / a.cluster, rank, heads);
    } else {
        if (!unit_range<kPaThreads>(r, a.B, heads,
                                    [&](int b) { return paged_len(a.cache, b, a.added, a.err); },
                                    [&](int len) { return P::kCost + blocks_of(seen_rows<Rows>(a, len)); }))
            return;
        if (!p.begin(a, r, heads)) return;
    }

    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + warp * (S * kStage);
    float *merge = (float *)(smem + kPaWarps * S * kStage);                       // [warps][H][stride]
    float *sm = merge + kAttendSums<P> / 4, *sl = sm + kPaWarps * H;                // [warps][H]
    float *own = merge + warp * H * P::kMergeStride;     // this warp's share, scratch until the segment's end
    float *sums = P::kScaled ? merge : (float *)smem;    // a cluster's, for its other ranks
    __shared__ uint32_t own_at[kPaWarps];                // P::kScaled: where the warps' shares are

    // Loads run ahead of the computation: their own walk, and the pool place of the next
    // tiles' rows, so that no load waits for a block-table entry.
    using Feed = typename FeedOf<P, Rows>::type;
    Feed feed;
    feed.begin(a, p, ring, warp, tiles);
    if constexpr (P::kScaled) {
#pragma unroll 1
        for (int i = 0; i < S - 1; ++i) feed.issue(a);   // one instance: what a launch fetches of the code counts
    } else {
#pragma unroll
        for (int i = 0; i < S - 1; ++i) feed.issue(a);
    }

    int stage = 0;
    P state;
    bool go = true;
    auto first_head = [&](const Pieces<Rows, P::kCost> &w) { return (long long)w.b * a.Hq + w.h / tiles * G + w.h % tiles * H; };
    auto head_count = [&](const Pieces<Rows, P::kCost> &w) { return min(H, G - w.h % tiles * H); };
    state.load_q((const T *)a.q + first_head(p) * D, head_count(p), a.scale_log2);
    while (go) {
        const int kvh = p.h / tiles, h0 = (p.h % tiles) * H, n = head_count(p);
        const long long hq = first_head(p);
        state.reset();
        float *scores = a.scores ? a.scores + score_place(p.b, kvh, h0, a.Hkv, G, (long long)a.cache.table_pages * a.cache.page_size) : nullptr;
        const int rows = p.rows();
        for (int t = warp; t * KT < rows; t += kPaWarps) {
            cp_wait_group<S - 2>();
            __syncwarp();
            feed.issue(a);
            const uint32_t ks = ring + stage * kStage;
            state.tile(ks, ks + KT * kRow, own, p.seen.key(p.blk0 * kAttendUnit + t * KT), p.seen, a.scale_log2, scores, n);
            stage = stage + 1 == S ? 0 : stage + 1;
        }
        Pieces<Rows, P::kCost> after = p;
        go = after.next(a);
        if (go) state.load_q((const T *)a.q + first_head(after) * D, head_count(after), a.scale_log2);   // on its way during the merge
        if (P::kScaled) {
            __syncwarp();                                // the stage was read
            own = (float *)(smem + (feed.free_stage() - (uint32_t)__cvta_generic_to_shared(smem)));
            if (lane == 0) own_at[warp] = (uint32_t)(own - (float *)smem);
        }
        state.store(own, sm + warp * H, sl + warp * H);
        __syncthreads();
        const bool whole = p.blk0 == 0 && p.blk1 == p.nblk;
        const int first = p.seg + P::kCost;           // unit of the segment's first block
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
                float4 y;
                if constexpr (P::kScaled) y = *(const float4 *)((const float *)smem + own_at[w] + h * P::kMergeStride + d);
                else y = *(const float4 *)(merge + (w * H + h) * P::kMergeStride + d);
                L = fmaf(k, sl[w * H + h], L);
                x[0] = fmaf(k, y.x, x[0]);
                x[1] = fmaf(k, y.y, x[1]);
                x[2] = fmaf(k, y.z, x[2]);
                x[3] = fmaf(k, y.w, x[3]);
            }
            if (!CLUSTER && whole) {
                write_out<T, D>(a, hq + h, d, x, M, L);
            } else if (CLUSTER) {                        // for the other ranks
                *(float4 *)(sums + h * D + d) = make_float4(x[0], x[1], x[2], x[3]);
                if (d == 0) *(float2 *)(sums + H * D + 2 * h) = make_float2(M, L);
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
                        dsmem_ld(sums + h * D + d, k, y[k]);
                        dsmem_ld(sums + H * D + 2 * h, k, ml[k]);
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

// Rows that a sequence can have to read: the table's, or the window's and the sinks'
// with what their blocks hold besides.
inline long long attend_rows(const AttendArgs &a) {
    const long long cap = (long long)a.cache.table_pages * a.cache.page_size;
    if (a.window < 0) return cap;
    auto up = [](long long n) { return (n + kAttendUnit - 1) / kAttendUnit * kAttendUnit; };
    const long long most = up(a.window) + kAttendUnit + up(a.sinks);
    return cap < most ? cap : most;
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
inline int attend_cluster(long long segments, long long cap, int rows, int sms) {
    int cs = 1;
    while (cs < 8 && cs * (long long)kAttendUnit < cap && cs * segments <= sms) cs *= 2;
    return cap <= cs * (long long)rows ? cs : 1;
}

// The same where a window bounds the rows: most sequences have outgrown it, and segments
// are as long as each other.  Then a cluster, or a CTA of its own, to a segment also where
// there are as many as CTAs, and with more rows to each (P::kWindowRows, clusters up to
// P::kWindowCluster); 0: shares.  Measured, 8 KV heads of 128 and 4 query heads each,
// sequences of 5000 to 20000 rows and 4 sinks, shares against this: bf16, 32 sequences with a window of 256 rows 13.7 and 9.5 us, of
// 1024 26.9 and 24.6, 16 of 1024 17.6 and 14.5, of 2048 26.7 and 24.1; fp32, 16 of 256
// 13.7 and 10.7, of 1024 27.4 and 25.0; e4m3, 32 of 256 15.9 and 12.0, 16 of 1024 16.7 and
// 15.6, 8 of 2048 (four CTAs each) 14.5 and 15.6, 16 of 2048 21.7 and 23.1.
inline int window_cluster(long long segments, long long cap, int rows, int most, long long ctas) {
    int cs = 1;
    while (2 * cs <= most && 2 * cs * segments <= ctas) cs *= 2;
    return segments <= ctas && cap <= cs * (long long)rows ? cs : 0;
}

// ht: heads of a tile.
template <typename P, typename Rows> cudaError_t start_attend(typename P::Args a, int ht, int sms, cudaStream_t s) {
    static_assert(P::kCost <= kAttendMaxCost, "units are counted when a handle is made");
    const int G = a.Hq / a.Hkv;
    const long long cap = attend_rows(a), segments = a.B * (long long)a.Hkv * ((G + ht - 1) / ht);
    const long long most = segments * (P::kCost + (cap + kAttendUnit - 1) / kAttendUnit);
    const long long ctas = (long long)P::kCtas * sms;
    a.cluster = attend_cluster(segments, cap, P::kClusterRows, sms);
    bool whole = a.cluster > 1;
    if (!whole && cap < (long long)a.cache.table_pages * a.cache.page_size) {
        a.cluster = window_cluster(segments, cap, P::kWindowRows, P::kWindowCluster, ctas);
        whole = a.cluster > 0;
    }
    auto clusters = [&](auto tile) {
        using C = decltype(tile);
        return launch_cluster(paged_attend_kernel<C, true, Rows>, dim3((unsigned)segments * a.cluster), dim3(kPaThreads), attend_smem<C>(), a.cluster, s, a);
    };
    if (whole) return cap <= 2LL * kAttendUnit * a.cluster ? clusters(typename P::Short()) : clusters(P());
    const int grid = (int)(most < ctas ? most : ctas);
    return launch_k(paged_attend_kernel<P, false, Rows>, dim3(grid), dim3(kPaThreads), attend_smem<P>(), s, true, a);
}
template <typename P, typename Rows> cudaError_t prepare_attend() {
    using C = typename P::Short;
    cudaError_t e = cudaFuncSetAttribute(paged_attend_kernel<P, false, Rows>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)attend_smem<P>());
    if (e == cudaSuccess) e = cudaFuncSetAttribute(paged_attend_kernel<P, true, Rows>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)attend_smem<P>());
    if (e == cudaSuccess) e = cudaFuncSetAttribute(paged_attend_kernel<C, true, Rows>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)attend_smem<C>());
    return e;
}

}  // namespace
}  // namespace prism
