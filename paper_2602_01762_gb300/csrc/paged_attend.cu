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
#include "paged_attend_tiles.cuh"

namespace prism {
namespace {

// weights[j] += sum_h 2^(s_jh - M_h) / L_h from the scores the attention kernel
// left, heads in order; one row of a KV head per thread.  V: float4 of scores per
// row (0: any group).  One row a thread and eight CTAs an SM beat two or four rows
// and fewer CTAs (16 sequences of up to 8192 rows, both kernels, before the attention
// kept P in three parts: 52.1, 52.3 and 53.3 us): what bounds it is the chain of a row's loads, not their bytes.
constexpr int kWtThreads = 256;
constexpr int kWtCtasPerSm = 8;
template <int V, bool WINDOW>
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
        const bool seen = j < len && (!WINDOW || j < a.sinks || j >= len - a.window);
        const int page = seen ? a.cache.table[(long long)b * a.cache.table_pages + j / a.cache.page_size] : -1;
        if (u == r.u0) pdl_wait();
        if ((unsigned)page < (unsigned)a.cache.n_pages) {   // else not seen, or reported by the attention
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

}  // namespace

int attend_head_tiles(int G) { return (G + 7) / 8; }

size_t attend_part_floats(int D, int G, int sms) {
    return (size_t)2 * kAttendMaxCtas * sms * attend_head_tile(G) * (D + 2);
}

cudaError_t prepare_attend_kernels(bool bf16, int D, int G) { return prepare_attend_tiles<AllRows>(bf16, D, G); }

cudaError_t launch_paged_attend(const AttendArgs &args, bool bf16, int D, int sms, cudaStream_t s) {
    AttendArgs a = args;
    const int G = a.Hq / a.Hkv;
    const long long cap = attend_rows(a), groups = a.B * (long long)a.Hkv;
    int ht = attend_head_tile(G);
    // fp32 tables of few rows: a tile of 16 heads takes longer than the second pass of
    // two of 8.  Measured, D = 128, 8 against 16: 4 KV heads of 1000 rows 9.6 and 12.3
    // us, of 8000 24 and 26, of 16000 35 and 36; 32 sequences of 500 rows 34 and 24;
    // D = 64: 4000 rows 11.7 and 17.1, 8 sequences of 1000 rows 11.9 and 10.5.
    if (!bf16 && ht == 16 && groups * ((G + 15) / 16) * cap <= 256 * D) ht = 8;
    cudaError_t e = a.window < 0 ? start_attend_tiles<AllRows>(a, bf16, D, ht, sms, s) : start_window_attend(a, bf16, D, ht, sms, s);
    if (e != cudaSuccess || !a.scores) return e;
    const long long rows = (long long)a.cache.table_pages * a.cache.page_size;
    const long long chunks = a.B * (long long)a.Hkv * ((rows + kWtThreads - 1) / kWtThreads);
    const dim3 wt((unsigned)(chunks < sms * kWtCtasPerSm ? chunks : sms * kWtCtasPerSm));
    auto go = [&](auto all, auto window) { return launch_k(a.window < 0 ? all : window, wt, dim3(kWtThreads), 0, s, true, a, ht); };
    // 4, 8 or 16 heads of one tile: a row's scores are one, two or four float4
    if (G <= ht && G == 4) return go(paged_weights_kernel<1, false>, paged_weights_kernel<1, true>);
    if (G <= ht && G == 8) return go(paged_weights_kernel<2, false>, paged_weights_kernel<2, true>);
    if (G <= ht && G == 16) return go(paged_weights_kernel<4, false>, paged_weights_kernel<4, true>);
    return go(paged_weights_kernel<0, false>, paged_weights_kernel<0, true>);
}

}  // namespace prism
