// Layer norm, forward and backward (layer_norm.h):
//     h = (x - mean) / sqrt(var + eps),  y = h w + b;
//     g = dy w,  dx = (g - mean(g) - h mean(g h)) / sqrt(var + eps) + residual,  dw = sum of dy h over the rows that share w,  db = sum of dy.
// Bound by memory: a row is read once into registers, 8 features a piece, and everything is computed from there in fp32; the variance is that of what is left when the mean is
// taken off, so nothing cancels.  In the backward pass a thread owns the same features of every row of its workgroup and keeps their sums of dy h and dy in registers; the
// workgroups' sums meet in a second kernel, in a fixed order.
#include "layer_norm.h"

#include <algorithm>

namespace ll {

typedef __bf16 nm_bf16x2 __attribute__((ext_vector_type(2)));
typedef float nm_f32x4 __attribute__((ext_vector_type(4)));
typedef float nm_f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned nm_u32x4 __attribute__((ext_vector_type(4)));

struct NmBf16 { uint16_t bits; };

__device__ __forceinline__ float nm_float(uint16_t bits) { return __builtin_bit_cast(float, unsigned(bits) << 16); }
__device__ __forceinline__ unsigned nm_pack(float a, float b) {
    const nm_f32x2 v = {a, b};
    return __builtin_bit_cast(unsigned, __builtin_convertvector(v, nm_bf16x2));
}

// Features col .. col + 7 of a row; zeros behind the last.
__device__ __forceinline__ void nm_load(float (&f)[8], const NmBf16* row, int col, int n, bool wide) {
    if (wide) {
        nm_u32x4 x = {0, 0, 0, 0};
        if (col < n) x = *reinterpret_cast<const nm_u32x4*>(row + col);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __builtin_bit_cast(float, x[i] << 16);
            f[2 * i + 1] = __builtin_bit_cast(float, x[i] & 0xFFFF0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = col + i < n ? nm_float(row[col + i].bits) : 0.f;
    }
}
__device__ __forceinline__ void nm_load(float (&f)[8], const float* row, int col, int n, bool wide) {
    if (wide) {
        nm_f32x4 a = {0.f, 0.f, 0.f, 0.f}, b = a;
        if (col < n) {
            a = *reinterpret_cast<const nm_f32x4*>(row + col);
            b = *reinterpret_cast<const nm_f32x4*>(row + col + 4);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[i] = a[i];
            f[4 + i] = b[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = col + i < n ? row[col + i] : 0.f;
    }
}
__device__ __forceinline__ void nm_store(const float (&f)[8], NmBf16* row, int col, int n, bool wide) {
    if (wide) {
        if (col < n) *reinterpret_cast<nm_u32x4*>(row + col) = nm_u32x4{nm_pack(f[0], f[1]), nm_pack(f[2], f[3]), nm_pack(f[4], f[5]), nm_pack(f[6], f[7])};
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (col + i < n) row[col + i].bits = uint16_t(nm_pack(f[i], 0.f));
    }
}
__device__ __forceinline__ void nm_store(const float (&f)[8], float* row, int col, int n, bool wide) {
    if (wide) {
        if (col < n) {
            *reinterpret_cast<nm_f32x4*>(row + col) = nm_f32x4{f[0], f[1], f[2], f[3]};
            *reinterpret_cast<nm_f32x4*>(row + col + 4) = nm_f32x4{f[4], f[5], f[6], f[7]};
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (col + i < n) row[col + i] = f[i];
    }
}
// Weight or bias of a group, which may be of either type.
__device__ __forceinline__ void nm_load_shared(float (&f)[8], const void* base, int64_t at, int col, const NormParams& p) {
    if (p.w_f32) nm_load(f, static_cast<const float*>(base) + at, col, p.n, p.w_wide);
    else nm_load(f, static_cast<const NmBf16*>(base) + at, col, p.n, p.w_wide);
}

// Sums over the THREADS threads that hold a row, the same in all of them.  Rows of more than a wave are a workgroup each.
template <int THREADS, int N>
__device__ __forceinline__ void nm_sum(float (&x)[N], float* lds) {
#pragma unroll
    for (int d = (THREADS < 64 ? THREADS : 64) / 2; d; d >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] += __shfl_xor(x[i], d);
    if constexpr (THREADS > 64) {
        constexpr int WAVES = THREADS / 64;
        __syncthreads();                                              // the sums before these were read
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) lds[(threadIdx.x >> 6) * N + i] = x[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            x[i] = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) x[i] += lds[w * N + i];
        }
    }
}

template <int THREADS, int PIECES, typename X, typename Y>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void ll_norm_forward_kernel(const NormParams p) {
    constexpr int ROWS = (THREADS < 256 ? 256 : THREADS) / THREADS;
    __shared__ float lds[16];
    const int t = threadIdx.x % THREADS;
    for (int64_t at = int64_t(blockIdx.x) * ROWS; at < p.m; at += int64_t(gridDim.x) * ROWS) {
        const bool there = at + threadIdx.x / THREADS < p.m;
        const int64_t row = there ? at + threadIdx.x / THREADS : p.m - 1;
        const X* x = static_cast<const X*>(p.x) + row * p.x_stride;
        float f[PIECES][8];
#pragma unroll
        for (int j = 0; j < PIECES; ++j) nm_load(f[j], x, 8 * (j * THREADS + t), p.n, p.wide);
        float sum[1] = {0.f};
#pragma unroll
        for (int j = 0; j < PIECES; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[0] += f[j][i];
        nm_sum<THREADS, 1>(sum, lds);
        const float mean = sum[0] / p.n;
        sum[0] = 0.f;
#pragma unroll
        for (int j = 0; j < PIECES; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                f[j][i] -= mean;
                if (8 * (j * THREADS + t) + i < p.n) sum[0] = __builtin_fmaf(f[j][i], f[j][i], sum[0]);
            }
        nm_sum<THREADS, 1>(sum, lds);
        const float rstd = 1.f / sqrtf(sum[0] / p.n + p.eps);
        if (!there) continue;
        if (p.stats && t == 0) *reinterpret_cast<nm_f32x2*>(p.stats + 2 * row) = nm_f32x2{mean, rstd};
        const int64_t shared = int64_t(int(row) / p.group_rows) * p.n;
        Y* y = static_cast<Y*>(p.y) + row * p.y_stride;
#pragma unroll
        for (int j = 0; j < PIECES; ++j) {
            const int col = 8 * (j * THREADS + t);
            float w[8], b[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                w[i] = 1.f;
                b[i] = 0.f;
            }
            if (p.weight) nm_load_shared(w, p.weight, shared, col, p);
            if (p.bias) nm_load_shared(b, p.bias, shared, col, p);
#pragma unroll
            for (int i = 0; i < 8; ++i) f[j][i] = __builtin_fmaf(f[j][i] * rstd, w[i], b[i]);
            nm_store(f[j], y, col, p.n, p.wide);
        }
    }
}

template <int THREADS, int PIECES, typename X, typename Y>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void ll_norm_backward_kernel(const NormParams p) {
    constexpr int ROWS = (THREADS < 256 ? 256 : THREADS) / THREADS, FEATURES = THREADS * PIECES * 8;
    __shared__ __attribute__((aligned(16))) float lds[ROWS > 1 ? 2 * FEATURES : 16];
    const int t = threadIdx.x % THREADS, part = threadIdx.x / THREADS, items = p.plan.groups * p.plan.chunks;
    for (int item = blockIdx.x; item < items; item += gridDim.x) {
        const int group = item / p.plan.chunks, chunk = item - group * p.plan.chunks;
        const int64_t first = int64_t(group) * p.group_rows + int64_t(chunk) * p.plan.rows;
        const int64_t end = min(min(first + p.plan.rows, int64_t(group + 1) * p.group_rows), int64_t(p.m));
        float w[PIECES][8], dw[PIECES][8], db[PIECES][8];
#pragma unroll
        for (int j = 0; j < PIECES; ++j) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                w[j][i] = 1.f;
                dw[j][i] = db[j][i] = 0.f;
            }
            if (p.weight) nm_load_shared(w[j], p.weight, int64_t(group) * p.n, 8 * (j * THREADS + t), p);
        }
        for (int64_t at = first; at < end; at += ROWS) {                  // the same number of rounds in all of a workgroup: rows of a wave and more synchronise
            const int64_t row = min(at + part, end - 1);
            const bool there = at + part < end;
            const X* x = static_cast<const X*>(p.x) + row * p.x_stride;
            const Y* dy = static_cast<const Y*>(p.dy) + row * p.dy_stride;
            const nm_f32x2 ms = *reinterpret_cast<const nm_f32x2*>(p.stats + 2 * row);
            float h[PIECES][8], g[PIECES][8], s[2] = {0.f, 0.f};
#pragma unroll
            for (int j = 0; j < PIECES; ++j) {
                nm_load(h[j], x, 8 * (j * THREADS + t), p.n, p.wide);
                nm_load(g[j], dy, 8 * (j * THREADS + t), p.n, p.wide);
            }
#pragma unroll
            for (int j = 0; j < PIECES; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    h[j][i] = (h[j][i] - ms[0]) * ms[1];
                    if (there) {
                        dw[j][i] = __builtin_fmaf(g[j][i], h[j][i], dw[j][i]);
                        db[j][i] += g[j][i];
                    }
                    g[j][i] *= w[j][i];
                    s[0] += g[j][i];                                      // behind the last feature dy is 0, and so is g
                    s[1] = __builtin_fmaf(g[j][i], h[j][i], s[1]);
                }
            nm_sum<THREADS, 2>(s, lds);
            if (!there) continue;
            const float a = s[0] / p.n, b = s[1] / p.n;
            X* dx = static_cast<X*>(p.dx) + row * p.dx_stride;
#pragma unroll
            for (int j = 0; j < PIECES; ++j) {
                const int col = 8 * (j * THREADS + t);
                float past[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) past[i] = 0.f;
                if (p.residual) nm_load(past, static_cast<const X*>(p.residual) + row * p.residual_stride, col, p.n, p.wide);
#pragma unroll
                for (int i = 0; i < 8; ++i) g[j][i] = __builtin_fmaf(g[j][i] - a - h[j][i] * b, ms[1], past[i]);
                nm_store(g[j], dx, col, p.n, p.wide);
            }
        }
        if (!p.dweight && !p.dbias) continue;
        if constexpr (ROWS > 1) {                                         // the parts of the workgroup add up, one after the other
            for (int r = 0; r < ROWS; ++r) {
                if (part == r)
#pragma unroll
                    for (int j = 0; j < PIECES; ++j)
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            float* to = lds + 8 * (j * THREADS + t) + i;
                            to[0] = r ? to[0] + dw[j][i] : dw[j][i];
                            to[FEATURES] = r ? to[FEATURES] + db[j][i] : db[j][i];
                        }
                __syncthreads();
            }
#pragma unroll
            for (int j = 0; j < PIECES; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    dw[j][i] = lds[8 * (j * THREADS + t) + i];
                    db[j][i] = lds[FEATURES + 8 * (j * THREADS + t) + i];
                }
            __syncthreads();
        }
        const bool whole = p.plan.chunks == 1;
        float* to_w = whole ? (p.dweight ? p.dweight + int64_t(group) * p.n : nullptr) : p.part + int64_t(item) * 2 * p.n;
        float* to_b = whole ? (p.dbias ? p.dbias + int64_t(group) * p.n : nullptr) : p.part + (int64_t(item) * 2 + 1) * p.n;
        const bool wide = p.n % 8 == 0;
#pragma unroll
        for (int j = 0; j < PIECES; ++j) {
            if (to_w && part == 0) nm_store(dw[j], to_w, 8 * (j * THREADS + t), p.n, wide);
            if (to_b && part == 0) nm_store(db[j], to_b, 8 * (j * THREADS + t), p.n, wide);
        }
    }
}

// Adds up the chunks' sums: 32 features a workgroup, every eighth chunk a thread.
__global__ __launch_bounds__(256) void ll_norm_sum_kernel(const NormParams p) {
    __shared__ float lds[8][33];
    float* out = blockIdx.y ? p.dbias : p.dweight;
    if (!out) return;
    const int blocks = (p.n + 31) / 32, group = blockIdx.x / blocks, c = threadIdx.x & 31, strand = threadIdx.x >> 5;
    const int col = (blockIdx.x - group * blocks) * 32 + c;
    float sum = 0.f;
    if (col < p.n) {
        const float* from = p.part + (int64_t(group) * p.plan.chunks * 2 + blockIdx.y) * p.n + col;
#pragma unroll 4
        for (int i = strand; i < p.plan.chunks; i += 8) sum += from[int64_t(i) * 2 * p.n];
    }
    lds[strand][c] = sum;
    __syncthreads();
    if (strand == 0 && col < p.n) {
#pragma unroll
        for (int i = 1; i < 8; ++i) sum += lds[i][c];
        out[int64_t(group) * p.n + col] = sum;
    }
}

// One kernel for each shape and pair of types.
template <int THREADS, int PIECES, typename X, typename Y>
static void nm_launch(const NormParams& p, bool backward, unsigned grid, hipStream_t s) {
    constexpr int WG = THREADS < 256 ? 256 : THREADS;
    if (backward) hipLaunchKernelGGL((ll_norm_backward_kernel<THREADS, PIECES, X, Y>), dim3(grid), dim3(WG), 0, s, p);
    else hipLaunchKernelGGL((ll_norm_forward_kernel<THREADS, PIECES, X, Y>), dim3(grid), dim3(WG), 0, s, p);
}
template <int THREADS, int PIECES>
static void nm_types(const NormParams& p, bool backward, unsigned grid, hipStream_t s) {
    if (!p.x_f32) nm_launch<THREADS, PIECES, NmBf16, NmBf16>(p, backward, grid, s);
    else if (!p.y_f32) nm_launch<THREADS, PIECES, float, NmBf16>(p, backward, grid, s);
    else nm_launch<THREADS, PIECES, float, float>(p, backward, grid, s);
}
static hipError_t nm_shapes(const NormParams& p, bool backward, unsigned grid, hipStream_t s) {
    switch (norm_shape(p.n)) {
        case 0: nm_types<16, 1>(p, backward, grid, s); break;
        case 1: nm_types<16, 2>(p, backward, grid, s); break;
        case 2: nm_types<16, 4>(p, backward, grid, s); break;
        case 3: nm_types<64, 2>(p, backward, grid, s); break;
        case 4: nm_types<64, 3>(p, backward, grid, s); break;
        case 5: nm_types<64, 4>(p, backward, grid, s); break;
        case 6: nm_types<256, 2>(p, backward, grid, s); break;
        case 7: nm_types<256, 3>(p, backward, grid, s); break;
        case 8: nm_types<256, 4>(p, backward, grid, s); break;
        case 9: nm_types<512, 3>(p, backward, grid, s); break;
        default: nm_types<512, 4>(p, backward, grid, s); break;
    }
    return hipGetLastError();
}
static_assert(NORM_SHAPE_COUNT == 11, "a case for each shape");

constexpr int64_t NM_MAX_GRID = 1 << 20;          // a workgroup takes several rows behind that

hipError_t launch_norm_forward(const NormParams& p, hipStream_t s) {
    const int rows = NORM_SHAPES[norm_shape(p.n)].rows();
    return nm_shapes(p, false, unsigned(std::min((int64_t(p.m) + rows - 1) / rows, NM_MAX_GRID)), s);
}
hipError_t launch_norm_backward(const NormParams& p, hipStream_t s) {
    hipError_t e = nm_shapes(p, true, unsigned(std::min(int64_t(p.plan.groups) * p.plan.chunks, NM_MAX_GRID)), s);
    if (e != hipSuccess || p.plan.chunks == 1 || (!p.dweight && !p.dbias)) return e;
    hipLaunchKernelGGL(ll_norm_sum_kernel, dim3(unsigned(p.plan.groups) * unsigned((p.n + 31) / 32), 2), dim3(256), 0, s, p);
    return hipGetLastError();
}

}  // namespace ll
