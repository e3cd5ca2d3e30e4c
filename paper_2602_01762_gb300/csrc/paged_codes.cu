// Rows of a cache held in 8 bits: the launch of their writing (paged_codes.cuh), and
// reading them back: 4 prefixes of 9001 to 16384 rows, 8 KV heads of 128, bf16, 49.5 us
// (6.3 TB/s).
#include "paged_codes.cuh"

namespace prism {
namespace {

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

}  // namespace

cudaError_t prepare_store_codes_kernels(bool bf16, int D) {
    const cudaError_t e = prepare_e4m3_store(bf16, D);
    return e != cudaSuccess ? e : prepare_int8_store(bf16, D);
}

cudaError_t launch_store_codes(const NormRopeArgs &queries, const StoreCodesArgs &args, CodeFormat format, bool bf16, int D, int sms, cudaStream_t s) {
    NormRopeArgs q = queries;
    StoreCodesArgs a = args;
    static_assert(kNrThreads == kScThreads, "one launch");
    unsigned others = plan_norm_rope(q, bf16, D, false, sms);
    const int rows = 32 / (D / 2 / (bf16 ? 8 : 4)), R = a.scale_rows;   // rows a warp has at a time
    a.per = R < rows && rows % R == 0 ? rows / R : 1;
    a.team = 1;
    // one row a lane group for a token too, where the block's earlier rows are few for a warp:
    // 16 tokens in blocks of 16, 32 and 64 rows 3.3, 3.5 and 3.7 us, by KEEP 4 4.3, 4.5 and 5.4
    a.keep = R <= rows || (a.max_new == 1 && R * D <= 8192) ? 1 : R <= 2 * rows ? 2 : 4;
    const long long wave = (a.keep == 4 ? kScCtas<4> : a.keep == 2 ? kScCtas<2> : kScCtas<1>) * (long long)sms;
    while (a.keep == 4 && a.team < kScThreads / 32 && a.team * 4 * rows < R) a.team *= 2;
    const long long blocks = (a.max_new + 2LL * R - 2) / R;              // that a sequence's new rows may touch
    const int angles = a.per > 1 ? rows : R < kScAngles ? R : kScAngles;
    a.tasks = (int)((blocks + a.per - 1) / a.per);
    a.chain = 1;
    // heads of a CTA: fewer than all where the tiles alone give an SM less than four CTAs
    long long tiles = (long long)a.B * a.tasks;
    const int teams = kScThreads / 32 / a.team;
    int splits = 1;
    while (splits * tiles < 2LL * sms && splits * teams < a.Hkv) splits *= 2;
    a.span = (a.Hkv + splits - 1) / splits;
    a.splits = (a.Hkv + a.span - 1) / a.span;
    a.ctas = (int)(tiles * 2 * a.splits);
    // one launch where all of it runs at once, else the queries' rows on a kernel that takes
    // less of an SM.  Measured, 32 query and 8 KV heads: 16 rows 3.3 and 3.9 us (and 2 us of a
    // launch), 8 prompts of 1021 to 2048 rows 59 and 56 us.
    a.beside = a.ctas + (long long)others > wave || !q.one_row;   // that launch takes a row a warp
    if (a.beside) {
        const cudaError_t e = launch_norm_rope(queries, bf16, D, false, sms, s);
        if (e != cudaSuccess) return e;
        others = 0;
    }
    // Tiles a CTA takes one after the other, the next one's rows on their way meanwhile: as
    // many as leave two waves of CTAs, where three tiles' angles fit the CTAs' shared memory.
    // Measured, 8 query heads: 8 prompts (4.5 waves) with 1, 2, 3 and 8 tiles 43, 41, 44 and 74
    // us, 32 prompts 147, 139, 136 and 139, 8 in blocks of one row 76, 66, 64 and 65.
    if (a.beside && 4 * D * angles <= kScChained) {
        const long long most = a.ctas / (2 * wave);
        a.chain = (int)(most < 1 ? 1 : most < 4 ? most : 4);
        a.tasks = (a.tasks + a.chain - 1) / a.chain;
        tiles = (long long)a.B * a.tasks;
        a.ctas = (int)(tiles * 2 * a.splits);
    }
    a.every = (int)((a.ctas + (long long)others) / a.ctas);
    a.by_tasks = Divisor((uint32_t)a.tasks), a.by_tiles = Divisor((uint32_t)tiles), a.by_every = Divisor((uint32_t)a.every);
    a.by_scale = Divisor((uint32_t)R), a.by_page = Divisor((uint32_t)a.cache.page_size);
    const size_t stored = a.keep * kScRing<1> + 4 * (size_t)D * angles * (a.chain < 3 ? a.chain : 3);
    const size_t shared = !a.beside && stored < kNrShared ? kNrShared : stored;
    const unsigned grid = (unsigned)a.ctas + others;
    return format == kE4m3 ? start_e4m3_store(q, a, bf16, D, grid, shared, s) : start_int8_store(q, a, bf16, D, grid, shared, s);
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
    return with_rows(bf16, D, [&](auto t, auto d) {
        return launch_k(format == kE4m3 ? read_codes_kernel<decltype(t), d, kE4m3> : read_codes_kernel<decltype(t), d, kInt8>, grid, dim3(kRcThreads), 0, s, true, a);
    });
}

}  // namespace prism
