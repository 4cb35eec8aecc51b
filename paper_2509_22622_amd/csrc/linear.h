// y = act(x w^T + bias) + residual (include/longlive.h, ll_linear): the launches, and what w looks like once it is packed.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace ll {

// Packed weight: [n block of 16][k step of 32][64 lanes][8], lane 16 g + r: w[16 nb + r][32 ks + 8 g + 0..7]; zeros where n or k lies
// past the end.  k steps come in pairs.
inline int64_t linear_padded_n(int n) { return (int64_t(n) + 15) / 16 * 16; }
inline int64_t linear_padded_k(int k) { return (int64_t(k) + 63) / 64 * 64; }
constexpr int LINEAR_MAX_N = 1 << 20, LINEAR_MAX_K = 1 << 20, LINEAR_MAX_STRIDE = 1 << 21;   // offsets inside a tile stay below 2^31

struct LinearParams {
    const uint16_t *x, *w_frag, *bias, *residual;   // bias, residual: null if there is none
    uint16_t* y;
    int64_t x_stride, residual_stride, y_stride;
    int M, N, K;
    int act;                                        // ll_activation
    int wide;                                       // groups of four features of y and the residual are 8-byte aligned
};
hipError_t launch_linear_pack(const uint16_t* w, int64_t w_stride, uint16_t* w_frag, int N, int K, hipStream_t s);
hipError_t launch_linear(const LinearParams& p, hipStream_t s);

}  // namespace ll
