// C-ABI of the paged cache (include/longlive.h: ll_paged_*): argument checks, rotary tables, launches.
#include <new>

#include "api_common.h"
#include "paged.h"

using namespace ll;
using namespace ll_api;

struct ll_paged {
    int layers, q_heads, kv_heads, D, page_tokens, n_pages, fmt, k_exp, v_exp;
    int rope, rope_pairs, axis1, axis2;
    char* dev;                  // null for an index-only handle
    int64_t layer_bytes;
    const double* turns;        // [rope_pairs], behind the pool
};

namespace {

constexpr int MAX_TOKENS = 1 << 24, MAX_SEQS = 1 << 20, MAX_STRIDE = 1 << 28;

bool paged_shapes_ok(int layers, int kv_heads, int D, int page_tokens, int n_pages, int fmt) {
    if (layers < 1 || layers > 65536 || kv_heads < 1 || kv_heads > 1024 || (D != 64 && D != 128) || page_tokens < PAGED_GRANULE ||
        page_tokens > 65536 || page_tokens % PAGED_GRANULE != 0 || n_pages < 1 || (fmt != 0 && fmt != 1))
        return false;
    const int64_t page = paged_page_bytes(kv_heads, page_tokens, D, fmt);        // at most 2^35
    return n_pages <= (int64_t(1) << 46) / page && layers <= (int64_t(1) << 46) / (page * n_pages);
}
int64_t paged_pool_bytes(int layers, int kv_heads, int D, int page_tokens, int n_pages, int fmt) {
    return layers * (n_pages * paged_page_bytes(kv_heads, page_tokens, D, fmt));  // a multiple of 2 * 16 * 64
}

// The batch of a call, as the kernels take it; the checks both calls share.
ll_status batch_of(const ll_paged* c, int layer, int n_seqs, int n_tokens, const int* cu, const int* lens, const int* table, int cols,
                   int64_t table_stride, PagedSeqs* out) {
    if (!c) return fail(LL_ERR_INVALID_ARG, "cache is null");
    if (layer < 0 || layer >= c->layers) return fail(LL_ERR_INVALID_ARG, "layer %d out of range [0, %d)", layer, c->layers);
    if (n_seqs < 1 || n_seqs > MAX_SEQS) return fail(LL_ERR_INVALID_ARG, "n_seqs %d outside [1, 2^20]", n_seqs);
    if (n_tokens < 0 || n_tokens > MAX_TOKENS) return fail(LL_ERR_INVALID_ARG, "n_tokens %d outside [0, 2^24]", n_tokens);
    if (cols < 1 || int64_t(cols) * c->page_tokens > PAGED_MAX_KEYS)
        return fail(LL_ERR_INVALID_ARG, "table_cols %d: 1 .. 2^30 / page_tokens", cols);
    if (table_stride < cols || table_stride > PAGED_MAX_KEYS) return fail(LL_ERR_INVALID_ARG, "table_stride is below table_cols or above 2^30");
    if (c->dev) {
        if (!lens || !table) return fail(LL_ERR_INVALID_ARG, "null seq_lens or page_table");
        if (!cu && n_tokens != n_seqs) return fail(LL_ERR_INVALID_ARG, "without cu_tokens n_tokens (%d) must be n_seqs (%d)", n_tokens, n_seqs);
        if ((reinterpret_cast<uintptr_t>(cu) | reinterpret_cast<uintptr_t>(lens) | reinterpret_cast<uintptr_t>(table)) & 3)
            return fail(LL_ERR_INVALID_ARG, "int32 arrays must be 4-byte aligned");
    } else if (cu || lens || table) {
        return fail(LL_ERR_INVALID_ARG, "index-only handle takes null tensors");
    }
    *out = PagedSeqs{lens, cu, table, table_stride, cols, n_seqs, n_tokens, c->page_tokens, c->n_pages, paged_div(c->page_tokens)};
    return LL_OK;
}

bool stride_ok(int64_t stride, int64_t row) { return stride >= row && stride <= MAX_STRIDE && stride % 8 == 0; }

// The split of the keys over workgroups, and the partial results' sizes in floats.
struct AttnSizes { PagedPlan plan; int64_t rows; };
bool attn_sizes(const ll_paged* c, int n_seqs, int max_new, int64_t max_len, int sink, int window, AttnSizes* out) {
    const int64_t units = int64_t(n_seqs) * c->kv_heads * paged_row_tiles(c->q_heads / c->kv_heads, max_new);
    out->plan = paged_plan(units, paged_most_steps(max_len, max_new, sink, window, paged_step_keys(c->D)));
    out->rows = out->plan.splits > 1 ? units * out->plan.splits * 16 : 0;
    return units * out->plan.splits <= PAGED_MAX_GROUPS && (out->plan.splits == 1 || units * 16 <= PAGED_MAX_GROUPS);
}
bool attn_args_ok(int n_seqs, int max_new, int64_t max_len, int sink, int window) {
    return n_seqs >= 1 && n_seqs <= MAX_SEQS && max_new >= 1 && max_new <= PAGED_MAX_NEW && max_len >= 1 && max_len <= PAGED_MAX_KEYS && sink >= 0 &&
           window >= 0 && (window > 0 || sink == 0) && sink <= PAGED_MAX_KEYS && window <= PAGED_MAX_KEYS;
}

}  // namespace

extern "C" {

size_t ll_paged_bytes(int layers, int kv_heads, int head_dim, int page_tokens, int n_pages, int kv_format) {
    if (!paged_shapes_ok(layers, kv_heads, head_dim, page_tokens, n_pages, kv_format)) return 0;
    return size_t(paged_pool_bytes(layers, kv_heads, head_dim, page_tokens, n_pages, kv_format)) + size_t(head_dim / 2) * sizeof(double);
}

ll_status ll_paged_create(int layers, int q_heads, int kv_heads, int head_dim, int page_tokens, int n_pages, int kv_format, int k_exp, int v_exp,
                          int rope, int rope_dim, float rope_theta, void* dev_buffer, size_t dev_bytes, ll_paged** out) {
    if (!out) return fail(LL_ERR_INVALID_ARG, "out is null");
    *out = nullptr;
    if (!paged_shapes_ok(layers, kv_heads, head_dim, page_tokens, n_pages, kv_format))
        return fail(head_dim != 64 && head_dim != 128 && head_dim > 0 ? LL_ERR_UNSUPPORTED : LL_ERR_INVALID_ARG,
                    "bad shape: layers %d kv_heads %d head_dim %d (64 or 128) page_tokens %d (a multiple of 16) n_pages %d kv_format %d", layers,
                    kv_heads, head_dim, page_tokens, n_pages, kv_format);
    if (q_heads < kv_heads || q_heads > 1024 || q_heads % kv_heads != 0)
        return fail(LL_ERR_INVALID_ARG, "q_heads %d is no multiple of kv_heads %d up to 1024", q_heads, kv_heads);
    if (k_exp < -16 || k_exp > 16 || v_exp < -16 || v_exp > 16 || (kv_format == 0 && (k_exp != 0 || v_exp != 0)))
        return fail(LL_ERR_INVALID_ARG, "k_exp %d, v_exp %d: -16 .. 16, and 0 without 8 bits", k_exp, v_exp);
    if (rope < LL_ROPE_NONE || rope > LL_ROPE_GRID) return fail(LL_ERR_INVALID_ARG, "rope %d", rope);
    const bool dims_ok = rope == LL_ROPE_NONE   ? rope_dim == 0
                         : rope == LL_ROPE_GRID ? rope_dim == head_dim
                                                : rope_dim >= 16 && rope_dim <= head_dim && rope_dim % 16 == 0;
    if (!dims_ok) return fail(LL_ERR_INVALID_ARG, "rope_dim %d does not fit rope %d and head_dim %d", rope_dim, rope, head_dim);
    if (rope != LL_ROPE_NONE && !(rope_theta > 0.0f && std::isfinite(rope_theta))) return fail(LL_ERR_INVALID_ARG, "rope_theta must be positive");
    const bool index_only = dev_buffer == nullptr && dev_bytes == 0;
    const int64_t pool = paged_pool_bytes(layers, kv_heads, head_dim, page_tokens, n_pages, kv_format);
    const size_t total = ll_paged_bytes(layers, kv_heads, head_dim, page_tokens, n_pages, kv_format);

    ll_paged c{};
    c.layers = layers; c.q_heads = q_heads; c.kv_heads = kv_heads; c.D = head_dim; c.page_tokens = page_tokens; c.n_pages = n_pages;
    c.fmt = kv_format; c.k_exp = k_exp; c.v_exp = v_exp; c.rope = rope; c.rope_pairs = rope_dim / 2;
    c.layer_bytes = pool / layers;
    double turns[64] = {};
    const double circle = 6.283185307179586476925;
    if (rope == LL_ROPE_GRID) {                        // frame | row | column, as the rolling cache divides them
        const int n_x = head_dim / 6, n_t = head_dim / 2 - 2 * n_x;
        c.axis1 = n_t; c.axis2 = n_t + n_x;
        for (int i = 0; i < c.rope_pairs; ++i) {
            const int in = i < n_t ? i : (i - n_t) % n_x, of = i < n_t ? n_t : n_x;
            turns[i] = std::pow(double(rope_theta), -double(in) / of) / circle;
        }
    } else {
        for (int i = 0; i < c.rope_pairs; ++i) turns[i] = std::pow(double(rope_theta), -2.0 * i / rope_dim) / circle;
    }
    if (!index_only) {
        if (!dev_buffer) return fail(LL_ERR_INVALID_ARG, "dev_buffer is null");
        if (reinterpret_cast<uintptr_t>(dev_buffer) & 255) return fail(LL_ERR_INVALID_ARG, "dev_buffer is not 256-byte aligned");
        if (dev_bytes < total) return fail(LL_ERR_BUFFER_TOO_SMALL, "dev_buffer has %zu bytes, %zu needed", dev_bytes, total);
        c.dev = static_cast<char*>(dev_buffer);
        c.turns = reinterpret_cast<const double*>(c.dev + pool);
        hipError_t e = hipDeviceSynchronize();         // whatever another stream still does with that memory
        if (e == hipSuccess) e = hipMemset(dev_buffer, 0, size_t(pool));
        if (e == hipSuccess) e = hipMemcpy(c.dev + pool, turns, sizeof(double) * size_t(head_dim / 2), hipMemcpyHostToDevice);
        if (e == hipSuccess) e = hipDeviceSynchronize();
        if (e != hipSuccess) return hip_fail(e, "ll_paged_create: clearing the buffer");
    }
    ll_paged* made = new (std::nothrow) ll_paged(c);
    if (!made) return fail(LL_ERR_INVALID_ARG, "out of host memory");
    *out = made;
    return LL_OK;
}

ll_status ll_paged_destroy(ll_paged* cache) {
    delete cache;
    return LL_OK;
}

ll_status ll_paged_append(const ll_paged* cache, int layer, int n_seqs, int n_tokens, const int* cu_tokens, const int* seq_lens,
                          const int* page_table, int table_cols, int64_t table_stride, const int* positions, const void* q, int64_t q_stride,
                          const void* k, int64_t k_stride, const void* v, int64_t v_stride, void* q_out, int64_t q_out_stride, void* stream) {
    PagedAppendParams p{};
    ll_status st = batch_of(cache, layer, n_seqs, n_tokens, cu_tokens, seq_lens, page_table, table_cols, table_stride, &p.s);
    if (st != LL_OK) return st;
    if (!cache->dev) {
        if (positions || q || k || v || q_out) return fail(LL_ERR_INVALID_ARG, "index-only handle takes null tensors");
        return LL_OK;
    }
    if ((q == nullptr) != (q_out == nullptr)) return fail(LL_ERR_INVALID_ARG, "q and q_out come together");
    if (cache->rope == LL_ROPE_GRID && !positions && n_tokens > 0) return fail(LL_ERR_INVALID_ARG, "frame, row and column need positions");
    if (cache->rope == LL_ROPE_NONE && positions) return fail(LL_ERR_INVALID_ARG, "positions without a rotary embedding");
    if (reinterpret_cast<uintptr_t>(positions) & 3) return fail(LL_ERR_INVALID_ARG, "int32 arrays must be 4-byte aligned");
    const int64_t q_row = int64_t(cache->q_heads) * cache->D, kv_row = int64_t(cache->kv_heads) * cache->D;
    if (!stride_ok(k_stride, kv_row) || !stride_ok(v_stride, kv_row) || (q && (!stride_ok(q_stride, q_row) || !stride_ok(q_out_stride, q_row))))
        return fail(LL_ERR_INVALID_ARG, "strides must be multiples of 8, at least a row and at most 2^28");
    if (n_tokens == 0) return LL_OK;
    if (!k || !v) return fail(LL_ERR_INVALID_ARG, "null tensor");
    if (!aligned16(q, k, v, q_out)) return fail(LL_ERR_INVALID_ARG, "tensors must be 16-byte aligned");
    if (q_out && (q_out == k || q_out == v || (q_out == q && q_stride != q_out_stride)))
        return fail(LL_ERR_INVALID_ARG, "q_out must not overlap k or v, and may be q only with its stride");
    p.q = static_cast<const uint16_t*>(q); p.k = static_cast<const uint16_t*>(k); p.v = static_cast<const uint16_t*>(v);
    p.q_out = static_cast<uint16_t*>(q_out);
    p.q_stride = q_stride; p.k_stride = k_stride; p.v_stride = v_stride; p.q_out_stride = q_out_stride;
    p.pool = cache->dev + layer * cache->layer_bytes;
    p.positions = positions;
    p.turns = cache->turns;
    p.q_heads = cache->q_heads; p.kv_heads = cache->kv_heads; p.D = cache->D; p.fmt = cache->fmt;
    p.halves = cache->rope == LL_ROPE_HALVES;
    p.rope_pairs = cache->rope_pairs;
    p.axes = cache->rope == LL_ROPE_GRID ? 3 : 1;
    p.axis1 = cache->axis1; p.axis2 = cache->axis2;
    p.q_scale = float(1.4426950408889634 / std::sqrt(double(cache->D)));
    p.k_scale = std::ldexp(1.0f, -cache->k_exp); p.v_scale = std::ldexp(1.0f, -cache->v_exp);
    hipError_t e = launch_paged_append(p, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "paged cache-write kernel launch");
    return LL_OK;
}

size_t ll_paged_attn_workspace_bytes(const ll_paged* cache, int n_seqs, int max_new, int64_t max_len, int sink_tokens, int window_tokens) {
    if (!cache || !attn_args_ok(n_seqs, max_new, max_len, sink_tokens, window_tokens)) return 0;
    AttnSizes z;
    if (!attn_sizes(cache, n_seqs, max_new, max_len, sink_tokens, window_tokens, &z)) return 0;
    return size_t(z.rows) * size_t(cache->D + 2) * sizeof(float);
}

ll_status ll_paged_attn(const ll_paged* cache, int layer, int n_seqs, int n_tokens, int max_new, int64_t max_len, const int* cu_tokens,
                        const int* seq_lens, const int* page_table, int table_cols, int64_t table_stride, int sink_tokens, int window_tokens,
                        const void* q, int64_t q_stride, void* out, int64_t out_stride, void* workspace, size_t workspace_bytes, void* stream) {
    PagedAttnParams p{};
    ll_status st = batch_of(cache, layer, n_seqs, n_tokens, cu_tokens, seq_lens, page_table, table_cols, table_stride, &p.s);
    if (st != LL_OK) return st;
    if (!attn_args_ok(n_seqs, max_new, max_len, sink_tokens, window_tokens))
        return fail(LL_ERR_INVALID_ARG, "max_new %d (1 .. 65536), max_len %lld (1 .. 2^30), sink_tokens %d, window_tokens %d (a sink needs a window)", max_new,
                    static_cast<long long>(max_len), sink_tokens, window_tokens);
    AttnSizes z;
    if (!attn_sizes(cache, n_seqs, max_new, max_len, sink_tokens, window_tokens, &z)) return fail(LL_ERR_UNSUPPORTED, "too many row tiles for one call");
    if (!cache->dev) {
        if (q || out || workspace) return fail(LL_ERR_INVALID_ARG, "index-only handle takes null tensors");
        return LL_OK;
    }
    if (!cu_tokens && max_new != 1) return fail(LL_ERR_INVALID_ARG, "max_new %d without cu_tokens", max_new);
    const int64_t row = int64_t(cache->q_heads) * cache->D;
    if (!stride_ok(q_stride, row) || !stride_ok(out_stride, row)) return fail(LL_ERR_INVALID_ARG, "strides must be multiples of 8, at least a row and at most 2^28");
    if (n_tokens == 0) return LL_OK;
    if (!q || !out) return fail(LL_ERR_INVALID_ARG, "null tensor");
    if (!aligned16(q, out, workspace)) return fail(LL_ERR_INVALID_ARG, "tensors must be 16-byte aligned");
    if (q == out) return fail(LL_ERR_INVALID_ARG, "out must not overlap q");
    const size_t needed = size_t(z.rows) * size_t(cache->D + 2) * sizeof(float);
    if (needed > 0 && !workspace) return fail(LL_ERR_INVALID_ARG, "workspace is null, %zu bytes needed", needed);
    if (workspace_bytes < needed) return fail(LL_ERR_BUFFER_TOO_SMALL, "workspace has %zu bytes, %zu needed", workspace_bytes, needed);
    if (needed > 0 && (workspace == q || workspace == out)) return fail(LL_ERR_INVALID_ARG, "workspace must not overlap q or out");
    p.q = static_cast<const uint16_t*>(q); p.out = static_cast<uint16_t*>(out);
    p.q_stride = q_stride; p.out_stride = out_stride;
    p.pool = cache->dev + layer * cache->layer_bytes;
    p.partial = static_cast<float*>(workspace);
    p.partial_ms = p.partial ? p.partial + z.rows * cache->D : nullptr;
    p.q_heads = cache->q_heads; p.kv_heads = cache->kv_heads; p.D = cache->D; p.fmt = cache->fmt;
    p.max_new = max_new; p.sink = sink_tokens; p.window = window_tokens;
    p.k_scale = std::ldexp(1.0f, cache->k_exp); p.v_scale = std::ldexp(1.0f, cache->v_exp);
    p.plan = z.plan;
    const int group = cache->q_heads / cache->kv_heads;
    p.by_group = paged_div(group); p.by_tiles = paged_div(paged_row_tiles(group, max_new)); p.by_kv_heads = paged_div(cache->kv_heads);
    p.by_splits = paged_div(z.plan.splits); p.by_rows = paged_div(std::min<int64_t>(16, int64_t(group) * max_new));
    hipError_t e = launch_paged_attn(p, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "paged attention kernel launch");
    return LL_OK;
}

}  // extern "C"
