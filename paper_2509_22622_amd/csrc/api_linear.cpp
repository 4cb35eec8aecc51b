// C-ABI of the linear layer (include/longlive.h: ll_linear*): argument checks and launches.
#include "api_common.h"
#include "linear.h"

using namespace ll;
using namespace ll_api;

constexpr int MAX_ROWS = 1 << 24, MAX_STRIDE = 1 << 28;

extern "C" {

static bool linear_shape_ok(int n, int k) {
    return n >= 1 && n <= LINEAR_MAX_N && k >= 8 && k <= LINEAR_MAX_K && k % 8 == 0 && linear_padded_n(n) * linear_padded_k(k) <= LINEAR_MAX_NUMBERS;
}

size_t ll_linear_packed_bytes(int n, int k) { return linear_shape_ok(n, k) ? size_t(linear_padded_n(n) * linear_padded_k(k) * 2) : 0; }

ll_status ll_linear_pack_weight(int n, int k, const void* w, int64_t w_stride, void* w_packed, void* stream) {
    if (!linear_shape_ok(n, k)) return fail(LL_ERR_INVALID_ARG, "n %d (1 .. 2^20), k %d (a multiple of 8, 8 .. 2^20), at most 2^34 numbers", n, k);
    if (!w || !w_packed) return fail(LL_ERR_INVALID_ARG, "null tensor");
    if (w_stride < k || w_stride % 8 != 0 || w_stride > MAX_STRIDE) return fail(LL_ERR_INVALID_ARG, "w_stride must be a multiple of 8, at least k and at most 2^28");
    if (!aligned16(w, w_packed)) return fail(LL_ERR_INVALID_ARG, "tensors must be 16-byte aligned");
    if (w == w_packed) return fail(LL_ERR_INVALID_ARG, "w_packed must not overlap w");
    hipError_t e = launch_linear_pack(static_cast<const uint16_t*>(w), w_stride, static_cast<uint16_t*>(w_packed), n, k, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "weight packing kernel launch");
    return LL_OK;
}

ll_status ll_linear(int m, int n, int k, const void* x, int64_t x_stride, const void* w_packed, const void* bias, int act, const void* residual,
                    int64_t residual_stride, void* y, int64_t y_stride, void* stream) {
    if (!linear_shape_ok(n, k)) return fail(LL_ERR_INVALID_ARG, "n %d (1 .. 2^20), k %d (a multiple of 8, 8 .. 2^20), at most 2^34 numbers", n, k);
    if (m < 0 || m > MAX_ROWS) return fail(LL_ERR_INVALID_ARG, "m %d outside [0, 2^24]", m);
    if (act < LL_ACT_NONE || act > LL_ACT_SILU) return fail(LL_ERR_INVALID_ARG, "act %d", act);
    if (x_stride < k || x_stride > LINEAR_MAX_STRIDE || x_stride % 8 != 0 || y_stride < n || y_stride > LINEAR_MAX_STRIDE ||
        (residual && (residual_stride < n || residual_stride > LINEAR_MAX_STRIDE)))
        return fail(LL_ERR_INVALID_ARG, "strides must be at least a row and at most 2^21, x_stride a multiple of 8");
    if (m == 0) return LL_OK;
    if (!x || !w_packed || !y) return fail(LL_ERR_INVALID_ARG, "null tensor");
    if (!aligned16(x, w_packed, y) || !aligned16(bias, residual)) return fail(LL_ERR_INVALID_ARG, "tensors must be 16-byte aligned");
    if (y == x || y == w_packed || y == bias || (y == residual && y_stride != residual_stride))
        return fail(LL_ERR_INVALID_ARG, "y must not overlap x, w_packed or bias, and may be the residual only with its stride");
    if (linear_blocks(LINEAR_SHAPES[linear_choose(m, n, k)], m, n) > LINEAR_MAX_BLOCKS - 7) return fail(LL_ERR_UNSUPPORTED, "too many blocks of outputs for one call");
    LinearParams p{};
    p.x = static_cast<const uint16_t*>(x); p.w_frag = static_cast<const uint16_t*>(w_packed);
    p.bias = static_cast<const uint16_t*>(bias); p.residual = static_cast<const uint16_t*>(residual);
    p.y = static_cast<uint16_t*>(y);
    p.x_stride = x_stride; p.residual_stride = residual_stride; p.y_stride = y_stride;
    p.M = m; p.N = n; p.K = k; p.act = act;
    p.wide = y_stride % 4 == 0 && (!residual || residual_stride % 4 == 0);
    p.wide8 = y_stride % 8 == 0 && (!residual || residual_stride % 8 == 0);
    hipError_t e = launch_linear(p, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "linear layer kernel launch");
    return LL_OK;
}

}  // extern "C"
