// C-ABI of the layer norm (include/longlive.h: ll_layer_norm*): argument checks and launches.
#include "api_common.h"
#include "layer_norm.h"
#include "overlap.h"

using namespace ll;
using namespace ll_api;

namespace {

bool types_ok(int x_type, int y_type, int w_type) {
    const auto known = [](int t) { return t == LL_BF16 || t == LL_F32; };
    return known(x_type) && known(y_type) && known(w_type) && (x_type == LL_F32 || y_type == LL_BF16);
}
bool sizes_ok(int m, int n, int group_rows) { return m >= 0 && m <= NORM_MAX_ROWS && n >= 1 && n <= NORM_MAX_FEATURES && group_rows >= 0; }
bool stride_ok(int64_t stride, int n) { return stride >= n && stride <= NORM_MAX_STRIDE; }
int size_of(int type) { return type == LL_F32 ? 4 : 2; }
Extent rows_of(const void* p, int m, int n, int64_t stride, int type) { return Extent{p, m, stride * size_of(type), int64_t(n) * size_of(type)}; }
bool aligned_to(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & uintptr_t(bytes - 1)) == 0; }
// rows whose pieces of 8 features are whole and 16-byte aligned
bool wide_rows(const void* p, int64_t stride, int type, int n) { return n % 8 == 0 && aligned_to(p, 16) && (stride * size_of(type)) % 16 == 0; }

constexpr const char* SIZES = "m %d (0 .. 2^24), n %d (1 .. 16384), group_rows %d (0 or more)";
constexpr const char* TYPES = "x_type %d, y_type %d, w_type %d: bfloat16 or 32 bits, y in 32 bits only with x";
constexpr const char* STRIDES = "strides must be at least a row and at most 2^21";

}  // namespace

extern "C" {

ll_status ll_layer_norm(int m, int n, int group_rows, float eps, int x_type, const void* x, int64_t x_stride, int w_type, const void* weight,
                        const void* bias, int y_type, void* y, int64_t y_stride, float* stats, void* stream) {
    if (!sizes_ok(m, n, group_rows)) return fail(LL_ERR_INVALID_ARG, SIZES, m, n, group_rows);
    if (!types_ok(x_type, y_type, w_type)) return fail(LL_ERR_INVALID_ARG, TYPES, x_type, y_type, w_type);
    if (!(eps > 0.f && std::isfinite(eps))) return fail(LL_ERR_INVALID_ARG, "eps must be positive");
    if (!stride_ok(x_stride, n) || !stride_ok(y_stride, n)) return fail(LL_ERR_INVALID_ARG, STRIDES);
    if (m == 0) return LL_OK;
    if (!x || !y) return fail(LL_ERR_INVALID_ARG, "null tensor");
    if (!aligned_to(x, size_of(x_type)) || !aligned_to(y, size_of(y_type)) || !aligned_to(weight, size_of(w_type)) || !aligned_to(bias, size_of(w_type)) ||
        !aligned_to(stats, 8))
        return fail(LL_ERR_INVALID_ARG, "tensors must be aligned to their numbers, stats to 8 bytes");
    const int64_t shared = int64_t(group_rows ? (int64_t(m) + group_rows - 1) / group_rows : 1) * n * size_of(w_type);
    const bool same = y == x && x_type == y_type && x_stride == y_stride;
    const Extent t[] = {rows_of(y, m, n, y_stride, y_type), extent(stats, int64_t(m) * 8), extent(weight, shared), extent(bias, shared), rows_of(same ? nullptr : x, m, n, x_stride, x_type)};
    if (any_overlap(t, 5, 2) || overlap(t[1], rows_of(x, m, n, x_stride, x_type)))
        return fail(LL_ERR_INVALID_ARG, "y may be x only with its type and stride, and y and stats must not overlap anything else");
    NormParams p{};
    p.x = x; p.weight = weight; p.bias = bias; p.y = y; p.stats = stats;
    p.x_stride = x_stride; p.y_stride = y_stride;
    p.m = m; p.n = n; p.group_rows = group_rows ? group_rows : m;
    p.x_f32 = x_type == LL_F32; p.y_f32 = y_type == LL_F32; p.w_f32 = w_type == LL_F32;
    p.wide = wide_rows(x, x_stride, x_type, n) && wide_rows(y, y_stride, y_type, n) && wide_rows(weight, n, w_type, n) && wide_rows(bias, n, w_type, n);
    p.eps = eps;
    hipError_t e = launch_norm_forward(p, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "layer norm kernel launch");
    return LL_OK;
}

size_t ll_layer_norm_backward_workspace_bytes(int m, int n, int group_rows) {
    return sizes_ok(m, n, group_rows) ? size_t(norm_numbers(norm_plan(m, n, group_rows), n)) * sizeof(float) : 0;
}

ll_status ll_layer_norm_backward(int m, int n, int group_rows, int y_type, const void* dy, int64_t dy_stride, int x_type, const void* x,
                                 int64_t x_stride, int w_type, const void* weight, const float* stats, const void* residual, int64_t residual_stride,
                                 void* dx, int64_t dx_stride, float* dweight, float* dbias, void* workspace, size_t workspace_bytes, void* stream) {
    if (!sizes_ok(m, n, group_rows)) return fail(LL_ERR_INVALID_ARG, SIZES, m, n, group_rows);
    if (!types_ok(x_type, y_type, w_type)) return fail(LL_ERR_INVALID_ARG, TYPES, x_type, y_type, w_type);
    if (!stride_ok(dy_stride, n) || !stride_ok(x_stride, n) || !stride_ok(dx_stride, n) || (residual && !stride_ok(residual_stride, n)))
        return fail(LL_ERR_INVALID_ARG, STRIDES);
    NormParams p{};
    p.plan = norm_plan(m, n, group_rows);
    if (p.plan.groups == 0 || (m == 0 && !dweight && !dbias)) return LL_OK;
    if (m > 0 && (!dy || !x || !stats || !dx)) return fail(LL_ERR_INVALID_ARG, "null tensor");
    if (!aligned_to(dy, size_of(y_type)) || !aligned_to(x, size_of(x_type)) || !aligned_to(dx, size_of(x_type)) || !aligned_to(residual, size_of(x_type)) ||
        !aligned_to(weight, size_of(w_type)) || !aligned_to(stats, 8))
        return fail(LL_ERR_INVALID_ARG, "tensors must be aligned to their numbers, stats to 8 bytes");
    if (!aligned16(dweight, dbias, workspace)) return fail(LL_ERR_INVALID_ARG, "dweight, dbias and workspace must be 16-byte aligned");
    const size_t needed = dweight || dbias ? size_t(norm_numbers(p.plan, n)) * sizeof(float) : 0;
    if (needed > 0 && !workspace) return fail(LL_ERR_INVALID_ARG, "workspace is null, %zu bytes needed", needed);
    if (workspace_bytes < needed) return fail(LL_ERR_BUFFER_TOO_SMALL, "workspace has %zu bytes, %zu needed", workspace_bytes, needed);
    const int64_t shared = int64_t(p.plan.groups) * n;
    const Extent whole[] = {rows_of(dy, m, n, dy_stride, y_type), rows_of(x, m, n, x_stride, x_type), rows_of(residual, m, n, residual_stride, x_type)};
    Extent t[] = {rows_of(dx, m, n, dx_stride, x_type), extent(dweight, shared * 4), extent(dbias, shared * 4), extent(workspace, int64_t(needed)), extent(stats, int64_t(m) * 8),
                  extent(weight, shared * size_of(w_type)), whole[0], whole[1], whole[2]};
    bool bad = false;
    for (int i = 0; i < 3; ++i) {
        for (int j = 1; j < 4; ++j) bad |= overlap(t[j], whole[i]);
        if (whole[i].at == dx && whole[i].stride == t[0].stride && whole[i].row == t[0].row) t[6 + i].at = nullptr;      // dx in its place
    }
    if (bad || any_overlap(t, 9, 4))
        return fail(LL_ERR_INVALID_ARG, "dx may be dy, x or residual only with its type and stride; dx, dweight, dbias and workspace must not overlap anything else");
    p.dy = dy; p.x = x; p.weight = weight; p.residual = residual; p.dx = dx;
    p.stats = const_cast<float*>(stats);
    p.dweight = dweight; p.dbias = dbias; p.part = static_cast<float*>(workspace);
    p.dy_stride = dy_stride; p.x_stride = x_stride; p.dx_stride = dx_stride; p.residual_stride = residual_stride;
    p.m = m; p.n = n; p.group_rows = group_rows ? group_rows : m;
    p.x_f32 = x_type == LL_F32; p.y_f32 = y_type == LL_F32; p.w_f32 = w_type == LL_F32;
    p.wide = wide_rows(dy, dy_stride, y_type, n) && wide_rows(x, x_stride, x_type, n) && wide_rows(dx, dx_stride, x_type, n) &&
             (!residual || wide_rows(residual, residual_stride, x_type, n)) && wide_rows(weight, n, w_type, n);
    hipError_t e = launch_norm_backward(p, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "layer norm backward kernel launch");
    return LL_OK;
}

}  // extern "C"
