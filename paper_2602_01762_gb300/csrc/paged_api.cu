// C ABI of the paged-cache operators: handle, workspace, checks, launches.  See
// include/prism.h.
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <new>

#include "../../include/prism.h"
#include "paged.cuh"

using namespace prism;

struct prism_paged {
    prism_paged_config cfg{};
    int device = 0, sms = 0;
    bool bf16 = true;
    void *ws = nullptr;
    float *part = nullptr;       // attention pieces
    float *scores = nullptr;     // [max_batch, Hq, max_pages * page_size] (track_weights)
    float2 *stat = nullptr;      // [max_batch, Hq] (track_weights)
    float *grad_part = nullptr;  // [CTAs, 2, D]
    // tickets, all left at zero: the attention's segments, then its CTAs', the gradient's, the eviction's
    int *counter = nullptr;
    int segments = 0, cta_tickets = 0;
    int *grad_ticket() const { return counter + segments + cta_tickets; }
    int *evict_ticket() const { return grad_ticket() + 1; }
    int *err = nullptr;
    char error[256] = "";
};

namespace {

prism_status fail(prism_paged *p, prism_status s, const char *fmt, ...) {
    char msg[256];
    va_list ap;
    va_start(ap, fmt);
    std::vsnprintf(msg, sizeof msg, fmt, ap);
    va_end(ap);
    if (p) std::snprintf(p->error, sizeof p->error, "%s", msg);
    try {
        set_global_error(msg);
    } catch (...) {
    }
    return s;
}
prism_status cuda_status(prism_paged *p, cudaError_t e, const char *what) {
    return e == cudaSuccess ? PRISM_OK : fail(p, PRISM_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

// Makes the handle's device current for one call.
struct OnDevice {
    int was = -1;
    cudaError_t e;
    explicit OnDevice(int d) {
        e = cudaGetDevice(&was);
        if (e == cudaSuccess && was != d) e = cudaSetDevice(d);
        else was = -1;
    }
    ~OnDevice() {
        if (was >= 0) cudaSetDevice(was);
    }
};

bool misaligned(const void *p) { return ((uintptr_t)p & 15u) != 0; }

struct Check {
    prism_paged *p;
    prism_status s = PRISM_OK;
    // Reports the first condition that does not hold.
    void need(bool ok, prism_status st, const char *what) {
        if (!ok && s == PRISM_OK) s = fail(p, st, "%s", what);
    }
    int es() const { return p->bf16 ? 2 : 4; }
    // The stride of a dimension of one element is not used, whatever it is.
    long long stride(long long elements, int n) const { return n > 1 ? elements * es() : 0; }
    HeadsView heads(const prism_heads &h, const prism_rows &r, int n_heads, const char *name) {
        const HeadsView v = {(char *)h.data, stride(h.batch_stride, r.batch), stride(h.row_stride, r.max_new), stride(h.head_stride, n_heads)};
        if (s != PRISM_OK) return v;
        if (!v.p) s = fail(p, PRISM_ERR_INVALID_ARG, "%s is null", name);
        else if (misaligned(v.p) || ((v.sb | v.st | v.sh) & 15))
            s = fail(p, PRISM_ERR_INVALID_ARG, "%s: base and strides must be multiples of 16 bytes", name);
        return v;
    }
    // An output: rows and heads of their own (a stride of 0 would have them written over each other).
    HeadsView out(const prism_heads &h, const prism_rows &r, int n_heads, const char *name) {
        const HeadsView v = heads(h, r, n_heads, name);
        if (s == PRISM_OK && ((v.sb == 0 && r.batch > 1) || (v.st == 0 && r.max_new > 1) || (v.sh == 0 && n_heads > 1)))
            s = fail(p, PRISM_ERR_INVALID_ARG, "%s: an output stride is 0", name);
        return v;
    }
    PagedView cache(const prism_paged_cache *c, const char *name, bool codes = false) {
        const int es = codes ? 1 : this->es();
        auto stride = [&](long long elements, int n) { return n > 1 ? elements * es : 0; };
        PagedView v{};
        if (!c || !c->k_pages || !c->v_pages || !c->block_table || !c->kv_len) {
            if (s == PRISM_OK) s = fail(p, PRISM_ERR_INVALID_ARG, "%s: null cache, pages, block table or kv_len", name);
            return v;
        }
        v = {(char *)c->k_pages, (char *)c->v_pages, stride(c->page_stride, c->n_pages), stride(c->head_stride, p->cfg.n_kv_heads),
             stride(c->row_stride, p->cfg.page_size), c->weights, c->block_table, c->kv_len, c->n_pages, c->table_pages, p->cfg.page_size};
        if (s != PRISM_OK) return v;
        if (misaligned(c->k_pages) || misaligned(c->v_pages) || ((v.page_stride | v.head_stride | v.row_stride) & 15))
            s = fail(p, PRISM_ERR_INVALID_ARG, "%s: bases and strides must be multiples of 16 bytes", name);
        else if ((v.page_stride == 0 && c->n_pages > 1) || (v.head_stride == 0 && p->cfg.n_kv_heads > 1) || (v.row_stride == 0 && v.page_size > 1))
            s = fail(p, PRISM_ERR_INVALID_ARG, "%s: a stride is 0", name);
        else if (c->n_pages < 1 || c->table_pages < 1)
            s = fail(p, PRISM_ERR_SHAPE, "%s: no pages", name);
        else if (c->batch < 1)
            s = fail(p, PRISM_ERR_SHAPE, "%s: batch %d", name, c->batch);
        else if (c->batch > p->cfg.max_batch || c->table_pages > p->cfg.max_pages)
            s = fail(p, PRISM_ERR_CAPACITY, "%s: batch %d and %d pages a sequence exceed the handle's %d and %d", name, c->batch,
                     c->table_pages, p->cfg.max_batch, p->cfg.max_pages);
        return v;
    }
    // A cache held in 8 bits, its scales to `a`.
    template <typename A> void codes(A &a, const prism_paged_cache *c, const prism_paged_scales *q) {
        a.cache = cache(c, "cache", true);
        need(q && q->k_scales && q->v_scales, PRISM_ERR_INVALID_ARG, "scales: null");
        if (s != PRISM_OK) return;
        need((((uintptr_t)q->k_scales | (uintptr_t)q->v_scales) & 3u) == 0, PRISM_ERR_INVALID_ARG, "scales: not aligned to their type");
        need(q->format == PRISM_E4M3 || q->format == PRISM_INT8, PRISM_ERR_INVALID_ARG, "scales: format must be PRISM_E4M3 or PRISM_INT8");
        need(q->scale_rows >= 1 && q->scale_rows <= p->cfg.page_size && p->cfg.page_size % q->scale_rows == 0, PRISM_ERR_SHAPE,
             "scales: scale_rows must divide page_size");
        need(!c->weights, PRISM_ERR_INVALID_ARG, "a cache held in 8 bits has no weights");
        if (s != PRISM_OK) return;
        a.k_scales = q->k_scales, a.v_scales = q->v_scales, a.scale_rows = q->scale_rows;
        a.scale_blocks = p->cfg.page_size / q->scale_rows;
    }
    // An attention's arguments but its cache.
    void attend(AttendArgs &a, const prism_paged_cache *c, int added, int window, int sinks, const void *q, void *out, float *lse) {
        need(q && out, PRISM_ERR_INVALID_ARG, "q or out is null");
        need(!misaligned(q) && !misaligned(out), PRISM_ERR_INVALID_ARG, "q and out must be 16-byte aligned");
        need(added >= 0, PRISM_ERR_INVALID_ARG, "added is negative");
        need(sinks >= 0, PRISM_ERR_INVALID_ARG, "sinks is negative");
        need(!a.cache.weights || p->scores, PRISM_ERR_INVALID_ARG, "the cache has weights: the handle needs track_weights");
        if (s != PRISM_OK) return;
        a.q = q, a.out = out, a.lse = lse;
        if (a.cache.weights) a.scores = p->scores, a.stat = p->stat;
        a.part = p->part, a.counter = p->counter, a.group_counter = p->counter + p->segments, a.err = p->err;
        a.B = c->batch, a.Hq = p->cfg.n_q_heads, a.Hkv = p->cfg.n_kv_heads, a.added = added, a.window = window, a.sinks = sinks;
        a.scale_log2 = (float)(p->cfg.softmax_scale * 1.4426950408889634);
    }
    // What the forward, the append and the gradient have in common.
    template <typename A> A rows(const prism_rows &r) {
        A a{};
        a.q = heads(r.q, r, p->cfg.n_q_heads, "q");
        a.k = heads(r.k, r, p->cfg.n_kv_heads, "k");
        a.g_q = r.g_q, a.g_k = r.g_k, a.rope = r.rope, a.pos = r.pos, a.n_new = r.n_new, a.rope_len = r.rope_len;
        a.B = r.batch, a.max_new = r.max_new, a.Hq = p->cfg.n_q_heads, a.Hkv = p->cfg.n_kv_heads, a.eps = p->cfg.rms_eps, a.err = p->err;
        need(r.batch >= 1 && r.max_new >= 1, PRISM_ERR_SHAPE, "batch and max_new must be at least 1");
        need((long long)r.batch * r.max_new <= (1LL << 24), PRISM_ERR_CAPACITY, "batch * max_new exceeds 2^24 rows");
        need(r.rope != nullptr, PRISM_ERR_INVALID_ARG, "rope is null");
        need(!misaligned(r.rope), PRISM_ERR_INVALID_ARG, "rope must be 16-byte aligned");
        need(r.rope_len >= 1, PRISM_ERR_SHAPE, "rope_len must be at least 1");
        need(!r.g_q == !r.g_k, PRISM_ERR_INVALID_ARG, "g_q and g_k are given together or not at all");
        need(!misaligned(r.g_q) && !misaligned(r.g_k), PRISM_ERR_INVALID_ARG, "gains must be 16-byte aligned");
        return a;
    }
};

}  // namespace

extern "C" {

prism_status prism_paged_create(const prism_paged_config *cfg, int32_t device, prism_paged **out) {
    if (!cfg || !out) return fail(nullptr, PRISM_ERR_INVALID_ARG, "prism_paged_create: null argument");
    *out = nullptr;
    const prism_paged_config &c = *cfg;
    if (c.head_dim != 64 && c.head_dim != 128) return fail(nullptr, PRISM_ERR_INVALID_ARG, "head_dim must be 64 or 128");
    if (c.n_kv_heads < 1 || c.n_q_heads < 1 || c.n_q_heads % c.n_kv_heads || c.n_q_heads > 1024)
        return fail(nullptr, PRISM_ERR_INVALID_ARG, "n_q_heads must be a multiple of n_kv_heads, at most 1024");
    if (c.dtype != PRISM_BF16 && c.dtype != PRISM_F32) return fail(nullptr, PRISM_ERR_INVALID_ARG, "dtype must be PRISM_F32 or PRISM_BF16");
    if (c.page_size < 1 || c.max_batch < 1 || c.max_pages < 1)
        return fail(nullptr, PRISM_ERR_INVALID_ARG, "page_size, max_batch and max_pages must be at least 1");
    if (!(c.softmax_scale >= 0.f) || std::isinf(c.softmax_scale) || !(c.rms_eps >= 0.f) || std::isinf(c.rms_eps))
        return fail(nullptr, PRISM_ERR_INVALID_ARG, "softmax_scale and rms_eps must be finite and not negative");
    const long long rows = (long long)c.max_pages * c.page_size;
    // work units and row numbers are 32-bit: 2^30 units where each segment costs one, and with at least 64 units to a
    // segment there (no more than 2^24 of them) below 2^31 where it costs two
    static_assert(kAttendMaxCost <= 32, "units of a handle's largest call");
    if (rows > (1LL << 30) || (long long)c.max_batch * c.n_q_heads > (1LL << 24) ||
        (long long)c.max_batch * c.n_q_heads * (rows / kAttendUnit + 2) > (1LL << 30))
        return fail(nullptr, PRISM_ERR_CAPACITY, "max_batch * n_q_heads * max_pages * page_size is too large");

    prism_paged *p = new (std::nothrow) prism_paged;
    if (!p) return fail(nullptr, PRISM_ERR_OOM, "host memory");
    p->cfg = c;
    p->device = device;
    p->bf16 = c.dtype == PRISM_BF16;
    if (p->cfg.softmax_scale == 0.f) p->cfg.softmax_scale = (float)(1.0 / std::sqrt((double)c.head_dim));
    OnDevice on(device);
    cudaError_t e = on.e;
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&p->sms, cudaDevAttrMultiProcessorCount, device);
    const int G = c.n_q_heads / c.n_kv_heads;
    if (e == cudaSuccess) e = prepare_attend_kernels(p->bf16, c.head_dim, G);
    if (e == cudaSuccess) e = prepare_window_attend_kernels(p->bf16, c.head_dim, G);
    if (e == cudaSuccess) e = prepare_code_attend_kernels(p->bf16, c.head_dim, G);
    if (e == cudaSuccess) e = prepare_store_codes_kernels(p->bf16, c.head_dim);
    if (e == cudaSuccess) e = prepare_evict_kernels();
    if (e == cudaSuccess) e = prepare_rope_kernels();
    if (e != cudaSuccess) {
        delete p;
        return cuda_status(nullptr, e, "prism_paged_create");
    }
    p->segments = c.max_batch * c.n_kv_heads * attend_head_tiles(G);
    p->cta_tickets = 2 * kAttendMaxCtas * p->sms;
    size_t bytes = 0;
    auto take = [&](size_t n) {
        const size_t at = bytes;
        bytes = (bytes + n + 255) & ~(size_t)255;
        return at;
    };
    const size_t err = take(sizeof(int)), counter = take(sizeof(int) * ((size_t)p->segments + p->cta_tickets + 2));
    const size_t zeroed = bytes;
    const size_t part = take(sizeof(float) * attend_part_floats(c.head_dim, G, p->sms));
    const size_t grad = take(sizeof(float) * 2 * c.head_dim * norm_rope_grad_ctas(p->sms));
    const size_t stat = take(c.track_weights ? sizeof(float2) * (size_t)c.max_batch * c.n_q_heads : 0);
    const size_t scores = take(c.track_weights ? sizeof(float) * (size_t)c.max_batch * c.n_q_heads * rows : 0);
    e = cudaMalloc(&p->ws, bytes);
    if (e != cudaSuccess) {
        cudaGetLastError();
        delete p;
        return fail(nullptr, PRISM_ERR_OOM, "workspace of %zu bytes: %s", bytes, cudaGetErrorString(e));
    }
    char *w = (char *)p->ws;
    p->err = (int *)(w + err);
    p->counter = (int *)(w + counter);
    p->part = (float *)(w + part);
    p->grad_part = (float *)(w + grad);
    if (c.track_weights) {
        p->stat = (float2 *)(w + stat);
        p->scores = (float *)(w + scores);
    }
    e = cudaMemset(p->ws, 0, zeroed);
    if (e == cudaSuccess) e = cudaDeviceSynchronize();
    if (e != cudaSuccess) {
        cudaFree(p->ws);
        delete p;
        return cuda_status(nullptr, e, "prism_paged_create");
    }
    *out = p;
    return PRISM_OK;
}

prism_status prism_paged_destroy(prism_paged *p) {
    if (!p) return PRISM_OK;
    OnDevice on(p->device);
    const cudaError_t e = cudaFree(p->ws);   // waits for the device's work
    delete p;
    return cuda_status(nullptr, e, "prism_paged_destroy");
}

prism_status prism_qk_norm_rope(prism_paged *p, const prism_rows *rows, void *stream) {
    if (!p || !rows) return fail(p, PRISM_ERR_INVALID_ARG, "prism_qk_norm_rope: null argument");
    Check c{p};
    NormRopeArgs a = c.rows<NormRopeArgs>(*rows);
    a.q_out = c.out(rows->q_out, *rows, p->cfg.n_q_heads, "q_out");
    a.k_out = c.out(rows->k_out, *rows, p->cfg.n_kv_heads, "k_out");
    c.need(a.pos != nullptr, PRISM_ERR_INVALID_ARG, "pos is null");
    if (c.s != PRISM_OK) return c.s;
    OnDevice on(p->device);
    if (on.e != cudaSuccess) return cuda_status(p, on.e, "cudaSetDevice");
    return cuda_status(p, launch_norm_rope(a, p->bf16, p->cfg.head_dim, false, p->sms, (cudaStream_t)stream), "prism_qk_norm_rope");
}

prism_status prism_qk_norm_rope_backward(prism_paged *p, const prism_rows *rows, const prism_row_grads *grads, void *stream) {
    if (!p || !rows || !grads) return fail(p, PRISM_ERR_INVALID_ARG, "prism_qk_norm_rope_backward: null argument");
    Check c{p};
    NormRopeGradArgs a = c.rows<NormRopeGradArgs>(*rows);
    a.dq_out = c.heads(grads->dq_out, *rows, p->cfg.n_q_heads, "dq_out");
    a.dk_out = c.heads(grads->dk_out, *rows, p->cfg.n_kv_heads, "dk_out");
    a.dq = c.out(grads->dq, *rows, p->cfg.n_q_heads, "dq");
    a.dk = c.out(grads->dk, *rows, p->cfg.n_kv_heads, "dk");
    a.dg_q = grads->dg_q, a.dg_k = grads->dg_k, a.part = p->grad_part, a.counter = p->grad_ticket();
    c.need(a.pos != nullptr, PRISM_ERR_INVALID_ARG, "pos is null");
    c.need(!a.g_q == !a.dg_q && !a.g_q == !a.dg_k, PRISM_ERR_INVALID_ARG, "dg_q and dg_k are given with the gains and only then");
    if (c.s != PRISM_OK) return c.s;
    OnDevice on(p->device);
    if (on.e != cudaSuccess) return cuda_status(p, on.e, "cudaSetDevice");
    return cuda_status(p, launch_norm_rope_grad(a, p->bf16, p->cfg.head_dim, p->sms, (cudaStream_t)stream), "prism_qk_norm_rope_backward");
}

prism_status prism_paged_append(prism_paged *p, const prism_paged_cache *cache, const prism_rows *rows, void *stream) {
    if (!p || !rows) return fail(p, PRISM_ERR_INVALID_ARG, "prism_paged_append: null argument");
    Check c{p};
    NormRopeArgs a = c.rows<NormRopeArgs>(*rows);
    a.cache = c.cache(cache, "cache");
    a.v = c.heads(rows->v, *rows, p->cfg.n_kv_heads, "v");
    a.q_out = c.out(rows->q_out, *rows, p->cfg.n_q_heads, "q_out");
    if (c.s != PRISM_OK) return c.s;
    c.need(rows->batch == cache->batch, PRISM_ERR_SHAPE, "the rows and the cache differ in batch");
    if (c.s != PRISM_OK) return c.s;
    if (!a.pos) a.pos = cache->kv_len;
    OnDevice on(p->device);
    if (on.e != cudaSuccess) return cuda_status(p, on.e, "cudaSetDevice");
    return cuda_status(p, launch_norm_rope(a, p->bf16, p->cfg.head_dim, true, p->sms, (cudaStream_t)stream), "prism_paged_append");
}

prism_status prism_paged_append_codes(prism_paged *p, const prism_paged_cache *cache, const prism_paged_scales *scales,
                                      const prism_rows *rows, void *stream) {
    if (!p || !rows) return fail(p, PRISM_ERR_INVALID_ARG, "prism_paged_append_codes: null argument");
    Check c{p};
    NormRopeArgs q = c.rows<NormRopeArgs>(*rows);
    StoreCodesArgs a{};
    c.codes(a, cache, scales);
    a.k = q.k;
    a.v = c.heads(rows->v, *rows, p->cfg.n_kv_heads, "v");
    q.q_out = c.out(rows->q_out, *rows, p->cfg.n_q_heads, "q_out");
    if (c.s != PRISM_OK) return c.s;
    c.need(rows->batch == cache->batch, PRISM_ERR_SHAPE, "the rows and the cache differ in batch");
    c.need(rows->batch * (((long long)rows->max_new + 2 * a.scale_rows) / a.scale_rows) * p->cfg.n_kv_heads <= (1LL << 28), PRISM_ERR_CAPACITY,
           "batch * max_new * n_kv_heads is too large");
    if (c.s != PRISM_OK) return c.s;
    if (!q.pos) q.pos = cache->kv_len;
    a.g_k = q.g_k, a.rope = q.rope, a.pos = q.pos, a.n_new = q.n_new, a.rope_len = q.rope_len, a.B = q.B, a.max_new = q.max_new, a.Hkv = q.Hkv;
    a.eps = q.eps, a.err = p->err;
    q.Hkv = 0;                                   // the queries' part, the queries alone
    OnDevice on(p->device);
    if (on.e != cudaSuccess) return cuda_status(p, on.e, "cudaSetDevice");
    return cuda_status(p, launch_store_codes(q, a, (CodeFormat)scales->format, p->bf16, p->cfg.head_dim, p->sms, (cudaStream_t)stream),
                       "prism_paged_append_codes");
}

prism_status prism_paged_read_codes(prism_paged *p, const prism_paged_cache *cache, const prism_paged_scales *scales,
                                    const int32_t *start, const int32_t *n_rows, int32_t max_rows, const prism_heads *k_out,
                                    const prism_heads *v_out, void *stream) {
    if (!p || !k_out || !v_out) return fail(p, PRISM_ERR_INVALID_ARG, "prism_paged_read_codes: null argument");
    Check c{p};
    ReadCodesArgs a{};
    c.codes(a, cache, scales);
    c.need(max_rows >= 1, PRISM_ERR_SHAPE, "max_rows must be at least 1");
    if (c.s != PRISM_OK) return c.s;
    c.need((long long)cache->batch * max_rows <= (1LL << 24), PRISM_ERR_CAPACITY, "batch * max_rows exceeds 2^24 rows");
    prism_rows shape{};
    shape.batch = cache->batch, shape.max_new = max_rows;
    a.k_out = c.out(*k_out, shape, p->cfg.n_kv_heads, "k_out");
    a.v_out = c.out(*v_out, shape, p->cfg.n_kv_heads, "v_out");
    if (c.s != PRISM_OK) return c.s;
    a.start = start, a.n_rows = n_rows, a.B = cache->batch, a.max_rows = max_rows, a.Hkv = p->cfg.n_kv_heads, a.err = p->err;
    OnDevice on(p->device);
    if (on.e != cudaSuccess) return cuda_status(p, on.e, "cudaSetDevice");
    return cuda_status(p, launch_read_codes(a, (CodeFormat)scales->format, p->bf16, p->cfg.head_dim, p->sms, (cudaStream_t)stream), "prism_paged_read_codes");
}

prism_status prism_paged_attend(prism_paged *p, const prism_paged_cache *cache, int32_t added, const void *q, void *out,
                                float *lse, void *stream) {
    return prism_paged_attend_window(p, cache, added, -1, 0, q, out, lse, stream);
}

prism_status prism_paged_attend_window(prism_paged *p, const prism_paged_cache *cache, int32_t added, int32_t window, int32_t sinks,
                                       const void *q, void *out, float *lse, void *stream) {
    if (!p) return fail(nullptr, PRISM_ERR_INVALID_ARG, "prism_paged_attend: null handle");
    Check c{p};
    AttendArgs a{};
    a.cache = c.cache(cache, "cache");
    c.attend(a, cache, added, window, sinks, q, out, lse);
    if (c.s != PRISM_OK) return c.s;
    OnDevice on(p->device);
    if (on.e != cudaSuccess) return cuda_status(p, on.e, "cudaSetDevice");
    return cuda_status(p, launch_paged_attend(a, p->bf16, p->cfg.head_dim, p->sms, (cudaStream_t)stream), "prism_paged_attend");
}

prism_status prism_paged_attend_codes(prism_paged *p, const prism_paged_cache *cache, const prism_paged_scales *scales, int32_t added,
                                      int32_t window, int32_t sinks, const void *q, void *out, float *lse, void *stream) {
    if (!p) return fail(nullptr, PRISM_ERR_INVALID_ARG, "prism_paged_attend_codes: null handle");
    Check c{p};
    CodeAttendArgs a{};
    c.codes(a, cache, scales);
    c.attend(a, cache, added, window, sinks, q, out, lse);
    if (c.s != PRISM_OK) return c.s;
    OnDevice on(p->device);
    if (on.e != cudaSuccess) return cuda_status(p, on.e, "cudaSetDevice");
    return cuda_status(p, launch_code_attend(a, (CodeFormat)scales->format, p->bf16, p->cfg.head_dim, p->sms, (cudaStream_t)stream),
                       "prism_paged_attend_codes");
}

prism_status prism_paged_evict(prism_paged *p, const prism_paged_cache *src, const prism_paged_cache *dst, int32_t budget,
                               int32_t sinks, int32_t recent, int32_t *kept, void *stream) {
    if (!p) return fail(nullptr, PRISM_ERR_INVALID_ARG, "prism_paged_evict: null handle");
    Check c{p};
    EvictArgs a{};
    a.src = c.cache(src, "src");
    a.dst = c.cache(dst, "dst");
    if (c.s == PRISM_OK) {
        c.need(src->batch == dst->batch, PRISM_ERR_SHAPE, "src and dst differ in batch");
        c.need(src->weights != nullptr, PRISM_ERR_INVALID_ARG, "src has no weights");
        c.need(src->block_table != dst->block_table, PRISM_ERR_INVALID_ARG, "src and dst share their block table");
        c.need(kept != nullptr, PRISM_ERR_INVALID_ARG, "kept is null");
        c.need(budget >= 1 && sinks >= 0 && recent >= 0 && (long long)sinks + recent <= budget, PRISM_ERR_INVALID_ARG,
               "budget must be at least 1 and at least sinks + recent, neither negative");
        const long long page = p->cfg.page_size, most = src->table_pages * page;
        c.need((budget < most ? budget : most) <= dst->table_pages * page, PRISM_ERR_SHAPE, "dst has fewer rows than the budget");
        c.need((long long)src->batch * p->cfg.n_kv_heads * ((long long)budget / 8 + 1) <= (1LL << 30), PRISM_ERR_CAPACITY,
               "batch * n_kv_heads * budget is too large");
    }
    if (c.s != PRISM_OK) return c.s;
    a.kept = kept, a.counter = p->evict_ticket(), a.B = src->batch, a.Hkv = p->cfg.n_kv_heads, a.budget = budget, a.sinks = sinks, a.recent = recent, a.err = p->err;
    OnDevice on(p->device);
    if (on.e != cudaSuccess) return cuda_status(p, on.e, "cudaSetDevice");
    return cuda_status(p, launch_paged_evict(a, p->cfg.head_dim * c.es(), p->sms, (cudaStream_t)stream), "prism_paged_evict");
}

prism_status prism_paged_status(prism_paged *p, void *stream, int32_t *flags) {
    if (!p) return fail(nullptr, PRISM_ERR_INVALID_ARG, "prism_paged_status: null handle");
    if (flags) *flags = 0;
    OnDevice on(p->device);
    cudaError_t e = on.e;
    int word = 0;
    if (e == cudaSuccess) e = cudaMemcpyAsync(&word, p->err, sizeof word, cudaMemcpyDeviceToHost, (cudaStream_t)stream);
    if (e == cudaSuccess) e = cudaMemsetAsync(p->err, 0, sizeof word, (cudaStream_t)stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize((cudaStream_t)stream);
    if (e != cudaSuccess) return cuda_status(p, e, "prism_paged_status");
    if (flags) *flags = word;
    return word ? fail(p, PRISM_ERR_DEVICE_FLAG, "device error word 0x%x", word) : PRISM_OK;
}

const char *prism_paged_error(const prism_paged *p) { return p ? p->error : prism_get_error(nullptr); }

}  // extern "C"
