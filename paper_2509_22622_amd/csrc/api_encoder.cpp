// C-ABI of the attention to an encoder's states (include/longlive.h: ll_encoder_attn*): argument checks and launches.
#include "api_common.h"
#include "encoder_attn.h"
#include "overlap.h"

using namespace ll;
using namespace ll_api;

namespace {

constexpr int64_t MAX_TILE_ROWS = 1 << 30;             // query rows of a sequence and kv head

bool heads_ok(int q_heads, int kv_heads, int head_dim) {
    return kv_heads >= 1 && q_heads >= kv_heads && q_heads <= ENC_MAX_HEADS && q_heads % kv_heads == 0 && (head_dim == 64 || head_dim == 128);
}
bool most_ok(int n_seqs, int max_q, int max_k) {
    return n_seqs >= 1 && n_seqs <= ENC_MAX_SEQS && max_q >= 1 && max_q <= ENC_MAX_ROWS && max_k >= 1 && max_k <= ENC_MAX_ROWS;
}
bool rows_ok(int n) { return n >= 0 && n <= ENC_MAX_ROWS; }
bool plan_ok(int n_seqs, int q_heads, int kv_heads, int max_q, const EncPlan& p) {
    const int64_t heads = int64_t(n_seqs) * kv_heads, most = ENC_MAX_GROUPS / 2;      // rounded up to 8 tiles, or to 8 units, of which there is at least one of each
    return int64_t(q_heads / kv_heads) * max_q <= MAX_TILE_ROWS && heads * p.tiles * p.splits <= most && heads * p.q_tiles * p.q_splits <= most &&
           heads * p.k_tiles * p.k_splits <= most;
}
int64_t side_numbers(int q_heads, int n_q) { return (int64_t(q_heads) * n_q * 2 + 3) / 4 * 4; }

// The checks that both directions share, and what the kernels are given of the batch.
ll_status batch_of(EncParams& p, int n_seqs, int q_heads, int kv_heads, int head_dim, float scale, int n_q, int n_k, int max_q, int max_k, const int* cu_q,
                   const int* cu_k, const int* k_lens) {
    if (!heads_ok(q_heads, kv_heads, head_dim))
        return fail(head_dim != 64 && head_dim != 128 && head_dim > 0 ? LL_ERR_UNSUPPORTED : LL_ERR_INVALID_ARG,
                    "q_heads %d (a multiple of kv_heads up to 1024), kv_heads %d, head_dim %d (64 or 128)", q_heads, kv_heads, head_dim);
    if (!most_ok(n_seqs, max_q, max_k))
        return fail(LL_ERR_INVALID_ARG, "n_seqs %d (1 .. 2^20), max_q %d, max_k %d (1 .. 2^24)", n_seqs, max_q, max_k);
    if (!rows_ok(n_q) || !rows_ok(n_k)) return fail(LL_ERR_INVALID_ARG, "n_q %d, n_k %d outside [0, 2^24]", n_q, n_k);
    if (!(scale > 0.f && std::isfinite(scale * 1.4426950408889634f))) return fail(LL_ERR_INVALID_ARG, "scale must be positive, and times log2(e) finite");
    if ((!cu_q && n_q % n_seqs != 0) || (!cu_k && n_k % n_seqs != 0))
        return fail(LL_ERR_INVALID_ARG, "without cu_q or cu_k the rows (%d, %d) must be a multiple of n_seqs (%d)", n_q, n_k, n_seqs);
    if ((reinterpret_cast<uintptr_t>(cu_q) | reinterpret_cast<uintptr_t>(cu_k) | reinterpret_cast<uintptr_t>(k_lens)) & 3)
        return fail(LL_ERR_INVALID_ARG, "int32 arrays must be 4-byte aligned");
    p.plan = enc_plan(n_seqs, q_heads, kv_heads, max_q, max_k);
    if (!plan_ok(n_seqs, q_heads, kv_heads, max_q, p.plan)) return fail(LL_ERR_UNSUPPORTED, "too many tiles for one call");
    p.cu_q = cu_q; p.cu_k = cu_k; p.k_lens = k_lens;
    p.n_seqs = n_seqs; p.n_q = n_q; p.n_k = n_k; p.max_q = max_q; p.max_k = max_k;
    p.q_heads = q_heads; p.kv_heads = kv_heads; p.D = head_dim;
    p.scale = scale;
    p.scale_log2 = scale * 1.4426950408889634f;
    p.by_group = paged_div(q_heads / kv_heads);
    p.by_kv_heads = paged_div(kv_heads);
    return LL_OK;
}

// A tensor of a call: `n` rows of `row` numbers, 0 where the call does not touch it.
struct Rows { const void* at; int64_t stride, row; int n; };
Extent bytes_of(const Rows& t) { return Extent{t.at, t.n, t.stride * 2, t.row * 2}; }
ll_status check_rows(const Rows* t, int n) {
    for (int i = 0; i < n; ++i)
        if (t[i].stride < t[i].row || t[i].stride > ENC_MAX_STRIDE || t[i].stride % 8 != 0)
            return fail(LL_ERR_INVALID_ARG, "strides must be multiples of 8, at least a row and at most 2^21");
    for (int i = 0; i < n; ++i) {
        if (t[i].n == 0) continue;
        if (!t[i].at) return fail(LL_ERR_INVALID_ARG, "null tensor");
        if (!aligned16(t[i].at)) return fail(LL_ERR_INVALID_ARG, "tensors must be 16-byte aligned");
    }
    return LL_OK;
}
constexpr const char* OVERLAP = "what a call writes must not overlap its other tensors";
ll_status check_workspace(const void* workspace, size_t bytes, size_t needed) {
    if (needed > 0 && !workspace) return fail(LL_ERR_INVALID_ARG, "workspace is null, %zu bytes needed", needed);
    if (bytes < needed) return fail(LL_ERR_BUFFER_TOO_SMALL, "workspace has %zu bytes, %zu needed", bytes, needed);
    if (!aligned16(workspace)) return fail(LL_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
    return LL_OK;
}

}  // namespace

extern "C" {

size_t ll_encoder_attn_workspace_bytes(int n_seqs, int q_heads, int kv_heads, int head_dim, int max_q, int max_k) {
    if (!heads_ok(q_heads, kv_heads, head_dim) || !most_ok(n_seqs, max_q, max_k)) return 0;
    const EncPlan p = enc_plan(n_seqs, q_heads, kv_heads, max_q, max_k);
    return plan_ok(n_seqs, q_heads, kv_heads, max_q, p) ? size_t(enc_forward_numbers(p, int64_t(n_seqs) * kv_heads, head_dim)) * sizeof(float) : 0;
}

ll_status ll_encoder_attn(int n_seqs, int q_heads, int kv_heads, int head_dim, float scale, int n_q, int n_k, int max_q, int max_k, const int* cu_q,
                          const int* cu_k, const int* k_lens, const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                          int64_t v_stride, void* out, int64_t out_stride, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    EncParams p{};
    ll_status st = batch_of(p, n_seqs, q_heads, kv_heads, head_dim, scale, n_q, n_k, max_q, max_k, cu_q, cu_k, k_lens);
    if (st != LL_OK) return st;
    const int64_t q_row = int64_t(q_heads) * head_dim, k_row = int64_t(kv_heads) * head_dim, heads = int64_t(n_seqs) * kv_heads;
    const bool run = n_q > 0;
    const Rows t[] = {{q, q_stride, q_row, n_q}, {k, k_stride, k_row, run ? n_k : 0}, {v, v_stride, k_row, run ? n_k : 0}, {out, out_stride, q_row, n_q}};
    st = check_rows(t, 4);
    if (st != LL_OK) return st;
    if (!run) return LL_OK;
    if (reinterpret_cast<uintptr_t>(lse) & 3) return fail(LL_ERR_INVALID_ARG, "lse must be 4-byte aligned");
    const int64_t numbers = enc_forward_numbers(p.plan, heads, head_dim);
    st = check_workspace(workspace, workspace_bytes, size_t(numbers) * sizeof(float));
    if (st != LL_OK) return st;
    const Extent all[] = {bytes_of(t[3]), extent(lse, int64_t(q_heads) * n_q * 4), extent(workspace, std::max(numbers * 4, int64_t(1))), bytes_of(t[0]), bytes_of(t[1]), bytes_of(t[2]),
                          extent(cu_q, (int64_t(n_seqs) + 1) * 4), extent(cu_k, (int64_t(n_seqs) + 1) * 4), extent(k_lens, int64_t(n_seqs) * 4)};
    if (any_overlap(all, 9, 3)) return fail(LL_ERR_INVALID_ARG, OVERLAP);
    p.q = static_cast<const uint16_t*>(q); p.k = static_cast<const uint16_t*>(k); p.v = static_cast<const uint16_t*>(v);
    p.out = static_cast<uint16_t*>(out);
    p.q_stride = q_stride; p.k_stride = k_stride; p.v_stride = v_stride; p.out_stride = out_stride;
    p.lse = lse;
    p.part = static_cast<float*>(workspace);
    p.part_ms = p.part ? p.part + numbers / (head_dim + 2) * head_dim : nullptr;
    hipError_t e = launch_encoder_forward(p, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "encoder attention kernel launch");
    return LL_OK;
}

size_t ll_encoder_attn_backward_workspace_bytes(int n_seqs, int q_heads, int kv_heads, int head_dim, int n_q, int max_q, int max_k) {
    if (!heads_ok(q_heads, kv_heads, head_dim) || !most_ok(n_seqs, max_q, max_k) || !rows_ok(n_q)) return 0;
    const EncPlan p = enc_plan(n_seqs, q_heads, kv_heads, max_q, max_k);
    if (!plan_ok(n_seqs, q_heads, kv_heads, max_q, p)) return 0;
    const int64_t heads = int64_t(n_seqs) * kv_heads;
    return size_t(side_numbers(q_heads, n_q) + enc_dq_numbers(p, heads, head_dim) + enc_dkv_numbers(p, heads, head_dim)) * sizeof(float);
}

ll_status ll_encoder_attn_backward(int n_seqs, int q_heads, int kv_heads, int head_dim, float scale, int n_q, int n_k, int max_q, int max_k, const int* cu_q,
                                   const int* cu_k, const int* k_lens, const void* dout, int64_t dout_stride, const void* q, int64_t q_stride, const void* k,
                                   int64_t k_stride, const void* v, int64_t v_stride, const void* out, int64_t out_stride, const float* lse, void* dq,
                                   int64_t dq_stride, void* dk, int64_t dk_stride, void* dv, int64_t dv_stride, void* workspace, size_t workspace_bytes,
                                   void* stream) {
    EncParams p{};
    ll_status st = batch_of(p, n_seqs, q_heads, kv_heads, head_dim, scale, n_q, n_k, max_q, max_k, cu_q, cu_k, k_lens);
    if (st != LL_OK) return st;
    const int64_t q_row = int64_t(q_heads) * head_dim, k_row = int64_t(kv_heads) * head_dim, heads = int64_t(n_seqs) * kv_heads;
    const bool rows = n_q > 0, states = n_k > 0;
    const Rows t[] = {{dq, dq_stride, q_row, n_q}, {dk, dk_stride, k_row, n_k}, {dv, dv_stride, k_row, n_k}, {dout, dout_stride, q_row, n_q}, {q, q_stride, q_row, n_q},
                      {out, out_stride, q_row, n_q}, {k, k_stride, k_row, n_k}, {v, v_stride, k_row, n_k}};
    st = check_rows(t, 8);
    if (st != LL_OK) return st;
    if (!rows && !states) return LL_OK;
    if (rows && !lse) return fail(LL_ERR_INVALID_ARG, "null tensor");
    if (reinterpret_cast<uintptr_t>(lse) & 3) return fail(LL_ERR_INVALID_ARG, "lse must be 4-byte aligned");
    const int64_t side = side_numbers(q_heads, n_q), dqn = enc_dq_numbers(p.plan, heads, head_dim), dkvn = enc_dkv_numbers(p.plan, heads, head_dim);
    st = check_workspace(workspace, workspace_bytes, size_t(side + dqn + dkvn) * sizeof(float));
    if (st != LL_OK) return st;
    const Extent all[] = {bytes_of(t[0]), bytes_of(t[1]), bytes_of(t[2]), extent(workspace, std::max((side + dqn + dkvn) * 4, int64_t(1))), bytes_of(t[3]), bytes_of(t[4]), bytes_of(t[5]),
                          bytes_of(t[6]), bytes_of(t[7]), extent(lse, int64_t(q_heads) * n_q * 4), extent(cu_q, (int64_t(n_seqs) + 1) * 4), extent(cu_k, (int64_t(n_seqs) + 1) * 4),
                          extent(k_lens, int64_t(n_seqs) * 4)};
    if (any_overlap(all, 13, 4)) return fail(LL_ERR_INVALID_ARG, OVERLAP);
    p.dout = static_cast<const uint16_t*>(dout); p.q = static_cast<const uint16_t*>(q); p.k = static_cast<const uint16_t*>(k);
    p.v = static_cast<const uint16_t*>(v); p.o = static_cast<const uint16_t*>(out);
    p.dq = static_cast<uint16_t*>(dq); p.dk = static_cast<uint16_t*>(dk); p.dv = static_cast<uint16_t*>(dv);
    p.dout_stride = dout_stride; p.q_stride = q_stride; p.k_stride = k_stride; p.v_stride = v_stride; p.out_stride = out_stride;
    p.dq_stride = dq_stride; p.dk_stride = dk_stride; p.dv_stride = dv_stride;
    p.lse = const_cast<float*>(lse);
    p.side = static_cast<float*>(workspace);
    p.part_q = p.side ? p.side + side : nullptr;
    p.part_d = p.part_q ? p.part_q + dqn / (head_dim + 1) * head_dim : nullptr;
    p.part_kv = p.part_q ? p.part_q + dqn : nullptr;
    hipError_t e = launch_encoder_backward(p, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "encoder attention backward kernel launch");
    return LL_OK;
}

}  // extern "C"
