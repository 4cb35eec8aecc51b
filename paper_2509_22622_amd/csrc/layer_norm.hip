// Layer norm, forward and backward (layer_norm.h):
//     h = (x - mean) / sqrt(var + eps),  y = h w + b;
//     g = dy w,  dx = (g - mean(g) - h mean(g h)) / sqrt(var + eps) + residual,  dw = sum of dy h over the rows that share w,  db = sum of dy.
// Bound by memory: a row is read once into registers and everything is computed from there in fp32; the variance is that of what is left when the mean is
// taken off, so nothing cancels.  A team of threads holds one or two rows at a time, so that enough of them are on the way.  In the backward pass a thread owns the same features of every
// row of its workgroup and keeps their sums of dy h and dy in registers; the workgroups' sums meet in a second kernel, in a fixed order.
// 32760 rows of 1536 in bfloat16: forward 42.8 us (201 MB, 4.7 TB/s: a copy reaches 4.85), backward with a residual 82 (403 MB, 4.9) and 5.3 for the sums; 2100 of 8192, x in 32 bits:
// 20.6 (103 MB, 5.0), 42 (241 MB, 5.7: part of what the forward pass left is still in the cache) and 5.  One row of 1536: 2.8 us, a launch.
#include "layer_norm.h"

#include <algorithm>

namespace ll {

typedef __bf16 nm_bf16x2 __attribute__((ext_vector_type(2)));
typedef float nm_f32x4 __attribute__((ext_vector_type(4)));
typedef float nm_f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned nm_u32x4 __attribute__((ext_vector_type(4)));
typedef nm_u32x4 nm_u32x4_any __attribute__((aligned(2)));            // at any number's address
typedef nm_f32x4 nm_f32x4_any __attribute__((aligned(4)));

struct NmBf16 { uint16_t bits; };

__device__ __forceinline__ unsigned nm_pack(float a, float b) {
    const nm_f32x2 v = {a, b};
    return __builtin_bit_cast(unsigned, __builtin_convertvector(v, nm_bf16x2));
}

// Eight features of a row as they came from memory.  again(): what is made of them is made anew behind it; kept over a sum it would take twice their registers.
template <typename T>
struct NmPiece;
template <>
struct NmPiece<NmBf16> {
    nm_u32x4 x;
    __device__ __forceinline__ float at(int i) const { return __builtin_bit_cast(float, i & 1 ? x[i / 2] & 0xFFFF0000u : x[i / 2] << 16); }
    __device__ __forceinline__ void wide(const NmBf16* p) { x = *reinterpret_cast<const nm_u32x4*>(p); }
    __device__ __forceinline__ void any(const NmBf16* p) { x = *reinterpret_cast<const nm_u32x4_any*>(p); }
    __device__ __forceinline__ void one(int i, const NmBf16* p) { x[i / 2] |= unsigned(p->bits) << (16 * (i & 1)); }
    __device__ __forceinline__ void clear() { x = nm_u32x4{0, 0, 0, 0}; }
    __device__ __forceinline__ void again() { asm volatile("" : "+v"(x)); }
};
template <>
struct NmPiece<float> {
    nm_f32x4 a, b;
    __device__ __forceinline__ float at(int i) const { return i < 4 ? a[i] : b[i - 4]; }
    __device__ __forceinline__ void wide(const float* p) {
        a = *reinterpret_cast<const nm_f32x4*>(p);
        b = *reinterpret_cast<const nm_f32x4*>(p + 4);
    }
    __device__ __forceinline__ void any(const float* p) {
        a = *reinterpret_cast<const nm_f32x4_any*>(p);
        b = *reinterpret_cast<const nm_f32x4_any*>(p + 4);
    }
    __device__ __forceinline__ void one(int i, const float* p) {
        if (i < 4) a[i] = *p;
        else b[i - 4] = *p;
    }
    __device__ __forceinline__ void clear() { a = b = nm_f32x4{0.f, 0.f, 0.f, 0.f}; }
    __device__ __forceinline__ void again() { asm volatile("" : "+v"(a), "+v"(b)); }
};

// The features of piece j of thread t of a team of `threads`.  WIDE: whole and 16-byte aligned in everything that a call touches.  Otherwise the loads and stores are as wide, which the
// hardware does at any address, but for the last features of a row whose width is no multiple of 8.
template <bool WIDE>
struct NmPlace {
    int t, threads, n;
    __device__ __forceinline__ int col(int j) const { return 8 * (j * threads + t); }
    __device__ __forceinline__ bool there(int j, int i) const { return col(j) + (WIDE ? 0 : i) < n; }
    __device__ __forceinline__ bool whole(int j) const { return WIDE ? col(j) < n : col(j) + 8 <= n; }
};
// Piece j of a row; zeros where there are no features.
template <bool WIDE, typename T>
__device__ __forceinline__ void nm_load(NmPiece<T>& f, const T* row, const NmPlace<WIDE>& at, int j) {
    const T* p = row + at.col(j);
    f.clear();
    if (at.whole(j)) {
        if constexpr (WIDE) f.wide(p);
        else f.any(p);
    } else if constexpr (!WIDE) {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (at.there(j, i)) f.one(i, p + i);
    }
}
template <bool WIDE>
__device__ __forceinline__ void nm_store(const float (&f)[8], NmBf16* row, const NmPlace<WIDE>& at, int j) {
    NmBf16* p = row + at.col(j);
    if (at.whole(j)) {
        const nm_u32x4 x = {nm_pack(f[0], f[1]), nm_pack(f[2], f[3]), nm_pack(f[4], f[5]), nm_pack(f[6], f[7])};
        if constexpr (WIDE) *reinterpret_cast<nm_u32x4*>(p) = x;
        else *reinterpret_cast<nm_u32x4_any*>(p) = x;
    } else if constexpr (!WIDE) {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (at.there(j, i)) p[i].bits = uint16_t(nm_pack(f[i], 0.f));
    }
}
template <bool WIDE>
__device__ __forceinline__ void nm_store(const float (&f)[8], float* row, const NmPlace<WIDE>& at, int j) {
    float* p = row + at.col(j);
    if (at.whole(j)) {
        const nm_f32x4 a = {f[0], f[1], f[2], f[3]}, b = {f[4], f[5], f[6], f[7]};
        if constexpr (WIDE) {
            *reinterpret_cast<nm_f32x4*>(p) = a;
            *reinterpret_cast<nm_f32x4*>(p + 4) = b;
        } else {
            *reinterpret_cast<nm_f32x4_any*>(p) = a;
            *reinterpret_cast<nm_f32x4_any*>(p + 4) = b;
        }
    } else if constexpr (!WIDE) {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (at.there(j, i)) p[i] = f[i];
    }
}
// Weight or bias of a group, which may be of either type.
template <bool WIDE>
__device__ __forceinline__ void nm_load_shared(float (&f)[8], const void* base, int64_t first, const NmPlace<WIDE>& at, int j, bool f32) {
    if (f32) {
        NmPiece<float> x;
        nm_load(x, static_cast<const float*>(base) + first, at, j);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = x.at(i);
    } else {
        NmPiece<NmBf16> x;
        nm_load(x, static_cast<const NmBf16*>(base) + first, at, j);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = x.at(i);
    }
}

// x of this lane and of the lane that `control` of the data-parallel move names.
template <int CONTROL>
__device__ __forceinline__ float nm_with(float x) {
    return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CONTROL, 0xF, 0xF, true));
}
__device__ __forceinline__ float nm_across16(float x) {              // the other 16 of 32 lanes
    const auto p = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    return __builtin_bit_cast(float, unsigned(p[0])) + __builtin_bit_cast(float, unsigned(p[1]));
}
__device__ __forceinline__ float nm_across32(float x) {              // the other half of the wave
    const auto p = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    return __builtin_bit_cast(float, unsigned(p[0])) + __builtin_bit_cast(float, unsigned(p[1]));
}
constexpr int NM_MAX_WAVES = 16;
// A row is added up as so much of itself, and its differences from the mean are taken as half of themselves, so that neither overflows while its numbers are finite: powers of two, which
// change no bit (but of numbers near the smallest), in the additions' own instructions.  Squares may: 1 / sqrt(variance) is 0 then, and so is h.
constexpr float NM_PART = 1.f / NORM_MAX_FEATURES;
// Sums over a team's threads, the same in all of them.  Teams of several waves meet in LDS, in one of two places in turn: whoever writes one again has passed the barrier
// behind the other, which nobody reaches in front of its reads of the first.
template <bool WAVES, int N>
__device__ __forceinline__ void nm_sum(float (&x)[N], float (*lds)[NM_MAX_WAVES][8], int& turn, int first_wave, int waves) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = nm_with<0x140>(nm_with<0x141>(nm_with<0x4E>(nm_with<0xB1>(x[i]))));      // neighbours, pairs, half a row, a row of 16 lanes
    if constexpr (WAVES) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = nm_across32(nm_across16(x[i]));
        if (waves > 1) {
            float(*to)[8] = lds[turn];
            turn ^= 1;
            if ((threadIdx.x & 63) == 0)
#pragma unroll
                for (int i = 0; i < N; ++i) to[threadIdx.x >> 6][i] = x[i];
            __syncthreads();
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = 0.f;
            for (int w = first_wave; w < first_wave + waves; ++w)
#pragma unroll
                for (int i = 0; i < N; ++i) x[i] += to[w][i];
        }
    }
}

// MOST: the most threads of a workgroup.  WAVES: teams of whole waves; otherwise of 16 lanes.
template <int MOST, bool WAVES, bool WIDE, int PIECES, int ROWS, typename X, typename Y>
__global__ __launch_bounds__(MOST) void ll_norm_forward_kernel(const NormParams p, int threads) {
    __shared__ float lds[2][NM_MAX_WAVES][8];
    int team = threadIdx.x / threads;
    if constexpr (WAVES) team = __builtin_amdgcn_readfirstlane(team);
    const int teams = blockDim.x / threads, waves = threads / 64;
    const NmPlace<WIDE> at{int(threadIdx.x) - team * threads, threads, p.n};
    int turn = 0;
    for (int64_t first = int64_t(blockIdx.x) * (teams * ROWS); first < p.m; first += int64_t(gridDim.x) * (teams * ROWS)) {
        int64_t row[ROWS];
        NmPiece<X> x[ROWS][PIECES];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            row[r] = first + team * ROWS + r;
            const X* from = static_cast<const X*>(p.x) + min(row[r], int64_t(p.m - 1)) * p.x_stride;
#pragma unroll
            for (int j = 0; j < PIECES; ++j) nm_load(x[r][j], from, at, j);
        }
        float mean[ROWS], var[ROWS];                                              // half the mean, a quarter of the squares
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            mean[r] = 0.f;
#pragma unroll
            for (int j = 0; j < PIECES; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) mean[r] = __builtin_fmaf(x[r][j].at(i), NM_PART, mean[r]);
        }
        nm_sum<WAVES, ROWS>(mean, lds, turn, team * waves, waves);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            mean[r] /= 2 * (p.n * NM_PART);
            var[r] = 0.f;
#pragma unroll
            for (int j = 0; j < PIECES; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float d = __builtin_fmaf(x[r][j].at(i), 0.5f, -mean[r]);
                    if (at.there(j, i)) var[r] = __builtin_fmaf(d, d, var[r]);
                }
        }
        nm_sum<WAVES, ROWS>(var, lds, turn, team * waves, waves);
        float w[PIECES][8], b[PIECES][8];
        int64_t of = -1;
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            if (row[r] >= p.m) break;
            const float rstd = 1.f / sqrtf(4.f * var[r] / p.n + p.eps);
            if (p.stats && at.t == 0) *reinterpret_cast<nm_f32x2*>(p.stats + 2 * row[r]) = nm_f32x2{2.f * mean[r], rstd};
            const int64_t group = int(row[r]) / p.group_rows;
            if (group != of) {
                of = group;
#pragma unroll
                for (int j = 0; j < PIECES; ++j) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        w[j][i] = 1.f;
                        b[j][i] = 0.f;
                    }
                    if (p.weight) nm_load_shared(w[j], p.weight, group * p.n, at, j, p.w_f32);
                    if (p.bias) nm_load_shared(b[j], p.bias, group * p.n, at, j, p.w_f32);
                }
            }
            Y* y = static_cast<Y*>(p.y) + row[r] * p.y_stride;
#pragma unroll
            for (int j = 0; j < PIECES; ++j) {
                float f[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = __builtin_fmaf(__builtin_fmaf(x[r][j].at(i), 0.5f, -mean[r]) * (2.f * rstd), w[j][i], b[j][i]);
                nm_store(f, y, at, j);
            }
        }
    }
}

template <int MOST, bool WAVES, bool WIDE, int PIECES, typename X, typename Y>
__global__ __launch_bounds__(MOST) void ll_norm_backward_kernel(const NormParams p, int threads) {
    __shared__ float lds[2][NM_MAX_WAVES][8];
    __shared__ float meet[WAVES ? (PIECES == 1 ? 4 * 512 : 1) : 4 * 16 * PIECES * 8];      // of the teams or waves that share features: one of their two sums
    int team = threadIdx.x / threads;
    if constexpr (WAVES) team = __builtin_amdgcn_readfirstlane(team);
    const int teams = blockDim.x / threads, waves = threads / 64;
    const NmPlace<WIDE> at{int(threadIdx.x) - team * threads, threads, p.n};
    const int items = p.plan.groups * p.plan.chunks;
    int turn = 0;
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
            if (p.weight) nm_load_shared(w[j], p.weight, int64_t(group) * p.n, at, j, p.w_f32);
        }
        // A team's rows one after the other, the next one on its way; the same rounds in all of a workgroup.  A row that is not there: the last one, with a gradient of zeros.
        struct { NmPiece<X> x[PIECES], past[PIECES]; NmPiece<Y> dy[PIECES]; nm_f32x2 ms; } now, next;
        const auto load = [&](int64_t want) {
            const int64_t row = min(want, end - 1);
            const X* xr = static_cast<const X*>(p.x) + row * p.x_stride;
            const Y* dyr = static_cast<const Y*>(p.dy) + row * p.dy_stride;
            const X* pr = static_cast<const X*>(p.residual) + row * p.residual_stride;
#pragma unroll
            for (int j = 0; j < PIECES; ++j) {
                nm_load(next.x[j], xr, at, j);
                if (want < end) nm_load(next.dy[j], dyr, at, j);
                else next.dy[j].clear();
                if (p.residual) nm_load(next.past[j], pr, at, j);
                else next.past[j].clear();
            }
            next.ms = *reinterpret_cast<const nm_f32x2*>(p.stats + 2 * row);
        };
        constexpr bool AHEAD = MOST < 1024;                                       // 16 waves have no registers for another row
        if (AHEAD && first < end) load(first + team);
        for (int64_t from = first; from < end; from += teams) {
            const int64_t row = from + team;
            if constexpr (!AHEAD) load(row);
            now = next;
            if (now.ms[1] == 0.f) now.ms[0] = 0.f;                                // the squares were too large: h is 0, also where x - mean is infinite
            if (AHEAD && from + teams < end) load(row + teams);
            float s[2] = {0.f, 0.f};
#pragma unroll
            for (int j = 0; j < PIECES; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float h = (now.x[j].at(i) - now.ms[0]) * now.ms[1], d = now.dy[j].at(i), g = d * w[j][i];
                    if (row < end) dw[j][i] = __builtin_fmaf(d, h, dw[j][i]);
                    db[j][i] += d;
                    s[0] += g;                                                    // where there is no feature dy is 0, and so is g
                    s[1] = __builtin_fmaf(g, h, s[1]);
                }
            nm_sum<WAVES, 2>(s, lds, turn, team * waves, waves);
            if (row >= end) continue;
            const float a = s[0] / p.n, b = s[1] / p.n;
            X* dx = static_cast<X*>(p.dx) + row * p.dx_stride;
#pragma unroll
            for (int j = 0; j < PIECES; ++j) {
                now.x[j].again();
                now.dy[j].again();
                float f[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float h = (now.x[j].at(i) - now.ms[0]) * now.ms[1], g = now.dy[j].at(i) * w[j][i];
                    f[i] = __builtin_fmaf(g - a - h * b, now.ms[1], now.past[j].at(i));
                }
                nm_store(f, dx, at, j);
            }
        }
        if (!p.dweight && !p.dbias) continue;
        // those that own the same features add up: the four teams of 16 lanes of a wave, then teams or waves, in LDS, one sum after the other
        if constexpr (!WAVES) {
#pragma unroll
            for (int j = 0; j < PIECES; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    dw[j][i] = nm_across32(nm_across16(dw[j][i]));
                    db[j][i] = nm_across32(nm_across16(db[j][i]));
                }
        }
        const int parts = WAVES ? teams : blockDim.x / 64, part = WAVES ? team : threadIdx.x / 64;
        if constexpr (!WAVES || PIECES == 1) {
            if (parts > 1) {
                const int each = threads * PIECES * 8;                            // parts * each is at most the size of `meet`
                for (int which = 0; which < 2; ++which) {
                    __syncthreads();                                              // the sum before, or the item before, was read
#pragma unroll
                    for (int j = 0; j < PIECES; ++j)
#pragma unroll
                        for (int i = 0; i < 8; ++i) meet[part * each + (j * 8 + i) * threads + at.t] = which ? db[j][i] : dw[j][i];
                    __syncthreads();
                    if (part == 0)
#pragma unroll
                        for (int j = 0; j < PIECES; ++j)
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                for (int o = 1; o < parts; ++o) {
                                    const float y = meet[o * each + (j * 8 + i) * threads + at.t];
                                    if (which) db[j][i] += y;
                                    else dw[j][i] += y;
                                }
                }
            }
        }
        if (part != 0 || (!WAVES && threadIdx.x >= 16)) continue;
        const bool whole = p.plan.chunks == 1;
        float* to_w = whole ? p.dweight + int64_t(group) * p.n : p.part + int64_t(item) * 2 * p.n;
        float* to_b = whole ? p.dbias + int64_t(group) * p.n : p.part + (int64_t(item) * 2 + 1) * p.n;
#pragma unroll
        for (int j = 0; j < PIECES; ++j) {
            if (p.dweight) nm_store(dw[j], to_w, at, j);
            if (p.dbias) nm_store(db[j], to_b, at, j);
        }
    }
}

// Adds up the chunks' sums: 32 features a workgroup, every STRANDS-th chunk a thread: bound by the way to memory and back.  1000 chunks of 512 features 9.4 us with 8 strands, 5.4 with 32.
template <int STRANDS>
__global__ __launch_bounds__(32 * STRANDS) void ll_norm_sum_kernel(const NormParams p) {
    __shared__ float lds[STRANDS][33];
    float* out = blockIdx.y ? p.dbias : p.dweight;
    if (!out) return;
    const int blocks = (p.n + 31) / 32, group = blockIdx.x / blocks, c = threadIdx.x & 31, strand = threadIdx.x >> 5;
    const int col = (blockIdx.x - group * blocks) * 32 + c;
    float sum = 0.f;
    if (col < p.n) {
        const float* from = p.part + (int64_t(group) * p.plan.chunks * 2 + blockIdx.y) * p.n + col;
#pragma unroll 8
        for (int i = strand; i < p.plan.chunks; i += STRANDS) sum += from[int64_t(i) * 2 * p.n];
    }
    lds[strand][c] = sum;
    __syncthreads();
    if (strand == 0 && col < p.n) {
#pragma unroll
        for (int i = 1; i < STRANDS; ++i) sum += lds[i][c];
        out[int64_t(group) * p.n + col] = sum;
    }
}
constexpr int NM_FEW_CHUNKS = 64;

constexpr int64_t NM_MAX_GRID = 1 << 20;          // a workgroup takes several items behind that

// One kernel for each shape, kind of loads and pair of types.
template <int MOST, bool WAVES, bool WIDE, int PIECES, int ROWS, typename X, typename Y>
static void nm_launch(const NormParams& p, bool backward, hipStream_t s) {
    const NormShape z = norm_shape(p.n);
    const dim3 wg(z.threads * z.teams);
    const int64_t items = backward ? int64_t(p.plan.groups) * p.plan.chunks : (int64_t(p.m) + z.teams * z.rows - 1) / (z.teams * z.rows);
    const dim3 grid(unsigned(std::min(items, NM_MAX_GRID)));
    if (backward) hipLaunchKernelGGL((ll_norm_backward_kernel<MOST, WAVES, WIDE, PIECES, X, Y>), grid, wg, 0, s, p, z.threads);
    else hipLaunchKernelGGL((ll_norm_forward_kernel<MOST, WAVES, WIDE, PIECES, ROWS, X, Y>), grid, wg, 0, s, p, z.threads);
}
template <int MOST, bool WAVES, bool WIDE, int PIECES, int ROWS>
static void nm_types(const NormParams& p, bool backward, hipStream_t s) {
    if (!p.x_f32) nm_launch<MOST, WAVES, WIDE, PIECES, ROWS, NmBf16, NmBf16>(p, backward, s);
    else if (!p.y_f32) nm_launch<MOST, WAVES, WIDE, PIECES, ROWS, float, NmBf16>(p, backward, s);
    else nm_launch<MOST, WAVES, WIDE, PIECES, ROWS, float, float>(p, backward, s);
}
template <bool WIDE>
static hipError_t nm_shapes(const NormParams& p, bool backward, hipStream_t s) {
    const NormShape z = norm_shape(p.n);
    if (z.threads == 16 && z.pieces == 1) nm_types<256, false, WIDE, 1, 2>(p, backward, s);
    else if (z.threads == 16) nm_types<256, false, WIDE, 2, 1>(p, backward, s);
    else if (z.pieces == 1) nm_types<512, true, WIDE, 1, 2>(p, backward, s);
    else if (z.threads <= 512) nm_types<512, true, WIDE, 2, 1>(p, backward, s);
    else nm_types<1024, true, WIDE, 2, 1>(p, backward, s);
    return hipGetLastError();
}

hipError_t launch_norm_forward(const NormParams& p, hipStream_t s) { return p.wide ? nm_shapes<true>(p, false, s) : nm_shapes<false>(p, false, s); }
hipError_t launch_norm_backward(const NormParams& p, hipStream_t s) {
    hipError_t e = p.wide ? nm_shapes<true>(p, true, s) : nm_shapes<false>(p, true, s);
    if (e != hipSuccess || p.plan.chunks == 1 || (!p.dweight && !p.dbias)) return e;
    const dim3 grid(unsigned(p.plan.groups) * unsigned((p.n + 31) / 32), 2);
    if (p.plan.chunks <= NM_FEW_CHUNKS) hipLaunchKernelGGL(ll_norm_sum_kernel<8>, grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL(ll_norm_sum_kernel<32>, grid, dim3(1024), 0, s, p);
    return hipGetLastError();
}

}  // namespace ll
