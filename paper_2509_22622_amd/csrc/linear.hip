// ll_linear: y = act(x w^T + bias) + residual, x [M, K] and y [M, N] row-major, w [N, K] packed once (linear.h); bf16 in and out, fp32 sums,
// one rounding at the end.  Both kernels compute the transposed product y^T = w x^T on 16x16x32 MFMAs: A = w, B = x; lane (g, c) register j of a
// block is y[m0 + c][n0 + 4 g + j], four neighbouring features, one 8-byte store.
//
// What bounds them is how fast a CU takes in operands: 50 to 54 GB/s each, 13.8 TB/s all together, wherever the bytes come from (L2, LDS-direct or
// registers, 96 KB or 144 KB on the way).  A block of BM x BN outputs takes in (BM + BN) 2 K bytes, so few rows want small blocks on
// many CUs and many rows large ones.
//
// ll_linear_few_kernel: blocks of 16 to 64 rows x 16 or 32 features.  A workgroup's eight waves split K, each streams its operands straight into
//   registers, and they join in LDS in a fixed order: no barrier before that, and w passes by in contiguous 1 KB loads.  us with weights that are in no
//   cache: 1 row, 1536 -> 1536 4.0, 4096 -> 4096 9.5 (3.5 TB/s of w); 48 rows 4.8 and 13.6; 300 rows, 6144 -> 1536 20.
// ll_linear_kernel: blocks of 64 x 64 to 256 x 256 through a ring of LDS stages, as the output projection of the cross-attention block
//   (out_proj.hip) has them; x is row-major here, since it comes from the caller.  A stage holds 64 features: a load instruction takes the 128 bytes of
//   each of 8 rows, whole cache lines, and leaves the eight 16-byte pieces of row r in the order piece ^ (r & 7), so that the 16 rows
//   of a fragment read lie in different banks (no conflicts counted; 0.3 % of the cycles since results go out through LDS).  4680 rows, 6144 -> 1536 with bias and residual 96 us = 920 TFLOP/s, and 83 = 1060 where
//   only the weights change from call to call, so that x, y and the residual are in the last-level cache; 8192 rows, 4096 -> 4096 likewise 202 us =
//   1360 TFLOP/s, of which the products alone, with nothing loaded, would take 180.
//   Tried there, and no faster: w two and x three stages ahead (160 KB); five stages of 32 features; four waves of 128 x 128 (a third fewer LDS
//   reads); loads of a step all at its beginning; waves in two groups that take every other
//   64 features (64 x 64: 28.8 -> 29.1 us at K = 6144), nine stages instead of six.
#include "linear.h"

#include <atomic>
#include <type_traits>

#include "../../include/longlive.h"

namespace ll {

typedef __bf16 ln_bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 ln_bf16x2 __attribute__((ext_vector_type(2)));
typedef float ln_f32x4 __attribute__((ext_vector_type(4)));
typedef float ln_f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned ln_u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned ln_u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ ln_f32x4 ln_mfma(ln_u32x4 a, ln_u32x4 b, ln_f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(ln_bf16x8, a), __builtin_bit_cast(ln_bf16x8, b), c, 0, 0, 0);
}

__device__ __forceinline__ float ln_widen(unsigned bits) { return __uint_as_float(bits << 16); }

// erfc(x), x >= 0, as t exp(-x^2 + P(t)), t = 2 / (2 + x), the form that Press, Teukolsky, Vetterling and Flannery give it (Numerical Recipes, section 6.2);
// P is this file's own Chebyshev fit of degree 8 of log(erfc(x) exp(x^2) / t) over x in [0, 13],
// where erfc ends in fp32; relative error 6e-7 and the exponential's.  A fifth of the code of erfcf, which every block of a tile needs.
__device__ __forceinline__ float ln_erfc(float x) {
    const float t = 2.0f * __builtin_amdgcn_rcpf(2.0f + x);
    float e = 0.05331777036190033f;
    e = __builtin_fmaf(e, t, -0.4333844482898712f);
    e = __builtin_fmaf(e, t, 1.2271937131881714f);
    e = __builtin_fmaf(e, t, -1.5042093992233276f);
    e = __builtin_fmaf(e, t, 0.6660377979278564f);
    e = __builtin_fmaf(e, t, -0.15973040461540222f);
    e = __builtin_fmaf(e, t, 0.42068466544151306f);
    e = __builtin_fmaf(e, t, 0.9954137206077576f);
    e = __builtin_fmaf(e, t, -1.2653236389160156f);
    return t * __builtin_amdgcn_exp2f(1.4426950408889634f * __builtin_fmaf(-x, x, e));
}

// The activations.  In the form y * sigmoid(..) or y * erfc(..) nothing is lost to cancellation where y is far below zero.  v_exp_f32 and v_rcp_f32 are
// good to 1 ulp each; they are a quarter as fast as other instructions, and a tile's activations overlap with no other work: 28.8 million of them
// (4680 x 6144) take 6 us on top of the product's 96, with an exact quotient 24.
__device__ __forceinline__ float ln_gelu(float y) {
    const float e = 0.5f * ln_erfc(fabsf(y) * 0.70710678118654752f);
    return y * (y < 0.f ? e : 1.0f - e);
}
// y / (1 + 2^z), as 2^-8 y / (2^-8 + 2^(z - 8)) with z - 8 given: where the quotient ends, its parts are no numbers yet that the unit takes for 0.
__device__ __forceinline__ float ln_gate(float y, float z8) {
    return (0.00390625f * y) * __builtin_amdgcn_rcpf(0.00390625f + __builtin_amdgcn_exp2f(z8));
}
__device__ __forceinline__ float ln_silu(float y) { return ln_gate(y, __builtin_fmaf(-1.4426950408889634f, y, -8.0f)); }
// sigmoid's argument is 2 sqrt(2 / pi) (y + 0.044715 y^3)
__device__ __forceinline__ float ln_gelu_tanh(float y) { return ln_gate(y, __builtin_fmaf(y, __builtin_fmaf(-0.10294324f * y, y, -2.3022082f), -8.0f)); }

// Four neighbouring numbers, features n .. n + 3 of a row that begins at `from`; what lies past the row's end counts as 0.
__device__ __forceinline__ ln_u32x2 ln_four(const LinearParams& p, const uint16_t* from, int n) {
    ln_u32x2 b = {0, 0};
    if (p.wide && n + 4 <= p.N) return *reinterpret_cast<const ln_u32x2*>(from + n);
    if (n < p.N) b[0] = from[n];
    if (n + 1 < p.N) b[0] |= unsigned(from[n + 1]) << 16;
    if (n + 2 < p.N) b[1] = from[n + 2];
    if (n + 3 < p.N) b[1] |= unsigned(from[n + 3]) << 16;
    return b;
}
__device__ __forceinline__ ln_f32x4 ln_floats(ln_u32x2 b) {
    return ln_f32x4{ln_widen(b[0]), __uint_as_float(b[0] & 0xFFFF0000u), ln_widen(b[1]), __uint_as_float(b[1] & 0xFFFF0000u)};
}
// The residual's features n .. n + 3 of row m, and of the bias; zeros where there is none.
__device__ __forceinline__ ln_u32x2 ln_residual(const LinearParams& p, int m, int n) {
    return p.residual && m < p.M ? ln_four(p, p.residual + m * p.residual_stride, n) : ln_u32x2{0, 0};
}
__device__ __forceinline__ ln_u32x2 ln_bias(const LinearParams& p, int n) { return p.bias ? ln_four(p, p.bias, n) : ln_u32x2{0, 0}; }

// ACT: the activation, where the kernel knows it
template <int ACT = -1>
__device__ __forceinline__ ln_f32x4 ln_activated(const LinearParams& p, ln_f32x4 v, ln_u32x2 bias) {
    if (p.bias) v += ln_floats(bias);
    switch (ACT < 0 ? p.act : ACT) {
    case LL_ACT_GELU_TANH: return ln_f32x4{ln_gelu_tanh(v[0]), ln_gelu_tanh(v[1]), ln_gelu_tanh(v[2]), ln_gelu_tanh(v[3])};
    case LL_ACT_GELU: return ln_f32x4{ln_gelu(v[0]), ln_gelu(v[1]), ln_gelu(v[2]), ln_gelu(v[3])};
    case LL_ACT_SILU: return ln_f32x4{ln_silu(v[0]), ln_silu(v[1]), ln_silu(v[2]), ln_silu(v[3])};
    default: return v;
    }
}
__device__ __forceinline__ ln_u32x2 ln_rounded(ln_f32x4 v) {
    const ln_f32x2 lo = {v[0], v[1]}, hi = {v[2], v[3]};
    return ln_u32x2{__builtin_bit_cast(unsigned, __builtin_convertvector(lo, ln_bf16x2)), __builtin_bit_cast(unsigned, __builtin_convertvector(hi, ln_bf16x2))};
}
// Stores features n .. n + 3 of a row that begins at `to`, those that there are.
__device__ __forceinline__ void ln_store4(const LinearParams& p, uint16_t* to, int n, ln_u32x2 o) {
    if (p.wide && n + 4 <= p.N) {
        *reinterpret_cast<ln_u32x2*>(to + n) = o;
        return;
    }
    if (n < p.N) to[n] = uint16_t(o[0]);
    if (n + 1 < p.N) to[n + 1] = uint16_t(o[0] >> 16);
    if (n + 2 < p.N) to[n + 2] = uint16_t(o[1]);
    if (n + 3 < p.N) to[n + 3] = uint16_t(o[1] >> 16);
}
// Features n .. n + 3 of row m: bias, activation, residual, rounding, store.
__device__ __forceinline__ void ln_finish(const LinearParams& p, int m, int n, ln_f32x4 v, ln_u32x2 bias, ln_u32x2 residual) {
    if (m >= p.M || n >= p.N) return;
    v = ln_activated(p, v, bias);
    if (p.residual) v += ln_floats(residual);
    ln_store4(p, p.y + m * p.y_stride, n, ln_rounded(v));
}
// Eight features of row m: the residual's, and the sum with it, rounded and stored.  WHOLE: there are eight, 16-byte aligned.
template <bool WHOLE>
__device__ __forceinline__ ln_u32x4 ln_residual8(const LinearParams& p, int m, int n) {
    if (WHOLE && !(p.residual && m < p.M)) return ln_u32x4{0, 0, 0, 0};
    if (WHOLE || (p.wide8 && p.residual && m < p.M && n + 8 <= p.N)) return *reinterpret_cast<const ln_u32x4*>(p.residual + m * p.residual_stride + n);
    const ln_u32x2 lo = ln_residual(p, m, n), hi = ln_residual(p, m, n + 4);
    return ln_u32x4{lo[0], lo[1], hi[0], hi[1]};
}
template <bool WHOLE>
__device__ __forceinline__ void ln_store8(const LinearParams& p, int m, int n, ln_f32x4 lo, ln_f32x4 hi, ln_u32x4 residual) {
    if (m >= p.M) return;
    if (p.residual) {
        lo += ln_floats(ln_u32x2{residual[0], residual[1]});
        hi += ln_floats(ln_u32x2{residual[2], residual[3]});
    }
    const ln_u32x2 a = ln_rounded(lo), b = ln_rounded(hi);
    uint16_t* const to = p.y + m * p.y_stride;
    if (WHOLE || (p.wide8 && n + 8 <= p.N)) {
        *reinterpret_cast<ln_u32x4*>(to + n) = ln_u32x4{a[0], a[1], b[0], b[1]};
    } else {
        ln_store4(p, to, n, a);
        ln_store4(p, to, n + 4, b);
    }
}

// ---- few rows ----------------------------------------------------------------------------------------------------
constexpr int LN_WAVES = 8;

// A wave takes every eighth 64 features.  Its loads of x have the 128 bytes of each of 8 rows, whole cache lines (the 16 bytes that a lane's operand
// takes, one row a lane, come at a quarter of the rate), and turn into operands through LDS that is the wave's own: no barrier.
// Two batches of U are in registers, one arriving while the other is worked on.
template <int MB, int NB>
constexpr int ln_few_batch() { return 10 / (MB + NB) < 1 ? 1 : 10 / (MB + NB); }

template <int MB, int NB>
__global__ __launch_bounds__(64 * LN_WAVES) void ll_linear_few_kernel(const LinearParams p) {
    constexpr int U = ln_few_batch<MB, NB>(), X_BYTES = LN_WAVES * MB * 2048, JOIN_BYTES = LN_WAVES * NB * MB * 1024;
    __shared__ __attribute__((aligned(16))) char lds[X_BYTES > JOIN_BYTES ? X_BYTES : JOIN_BYTES];
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n_parts = (p.K + 63) / 64, last_nb = (p.N + 15) / 16 - 1, n_runs = last_nb / NB + 1;
    const int nb0 = blockIdx.x % n_runs * NB, m0 = blockIdx.x / n_runs * (16 * MB);
    const uint16_t* w[NB];
#pragma unroll
    for (int a = 0; a < NB; ++a) w[a] = p.w_frag + int64_t(min(nb0 + a, last_nb)) * n_parts * 1024 + lane * 8;
    const int x_row = lane >> 3, x_piece = lane & 7;
    const uint16_t* x[2 * MB];
#pragma unroll
    for (int b = 0; b < 2 * MB; ++b) x[b] = p.x + min(m0 + 8 * b + x_row, p.M - 1) * p.x_stride;
    const int x_loads = (min(p.M - m0, 16 * MB) + 7) >> 3;       // whose eight rows there are
    // piece q of row i of a block of 16 lies at 1024 (i / 8) + 128 (i % 8) + 16 (q ^ (i % 8)): neither side meets a bank twice
    char* const own = lds + wave * (MB * 2048);
    char* const x_to = own + x_row * 128 + (x_piece ^ x_row) * 16;
    const char* const x_from = own + (r >> 3) * 1024 + (r & 7) * 128;
    ln_f32x4 acc[NB * MB];
#pragma unroll
    for (int i = 0; i < NB * MB; ++i) acc[i] = ln_f32x4{0.f, 0.f, 0.f, 0.f};
    struct Batch { ln_u32x4 w[U][NB][2], x[U][2 * MB]; };
    // Parts past the end are the last one again, and not multiplied; features past K are zeros.
    auto load = [&](int first, Batch& f) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int part = min(first + LN_WAVES * u, n_parts - 1), k = 64 * part + 8 * x_piece;
#pragma unroll
            for (int a = 0; a < NB; ++a) {
                f.w[u][a][0] = *reinterpret_cast<const ln_u32x4*>(w[a] + part * 1024);
                f.w[u][a][1] = *reinterpret_cast<const ln_u32x4*>(w[a] + part * 1024 + 512);
            }
#pragma unroll
            for (int b = 0; b < 2 * MB; ++b) {
                f.x[u][b] = ln_u32x4{0, 0, 0, 0};
                if (b < x_loads && k < p.K) f.x[u][b] = *reinterpret_cast<const ln_u32x4*>(x[b] + k);
            }
        }
    };
    auto multiply = [&](int first, const Batch& f) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (first + LN_WAVES * u < n_parts) {
#pragma unroll
                for (int b = 0; b < 2 * MB; ++b) *reinterpret_cast<ln_u32x4*>(x_to + 1024 * b) = f.x[u][b];
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");      // the wave's lanes read what its other lanes wrote: LDS keeps their order
                __builtin_amdgcn_wave_barrier();
                __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int b = 0; b < MB; ++b) {
                        const ln_u32x4 v = *reinterpret_cast<const ln_u32x4*>(x_from + 2048 * b + ((4 * s + g) ^ (r & 7)) * 16);
#pragma unroll
                        for (int a = 0; a < NB; ++a) acc[a * MB + b] = ln_mfma(f.w[u][a][s], v, acc[a * MB + b]);
                    }
                __builtin_amdgcn_wave_barrier();
            }
    };
    constexpr int TURN = LN_WAVES * U;
    Batch f0, f1;
    load(wave, f0);
    for (int first = wave; first < n_parts; first += 2 * TURN) {
        if (first + TURN < n_parts) load(first + TURN, f1);
        multiply(first, f0);
        if (first + TURN >= n_parts) break;
        if (first + 2 * TURN < n_parts) load(first + 2 * TURN, f0);
        multiply(first + TURN, f1);
    }
    __syncthreads();                              // every wave is done with its part of LDS
    ln_f32x4* const join = reinterpret_cast<ln_f32x4*>(lds) + lane;
#pragma unroll
    for (int i = 0; i < NB * MB; ++i) join[(wave * NB * MB + i) * 64] = acc[i];
    __syncthreads();
    for (int i = wave; i < NB * MB; i += LN_WAVES) {
        ln_f32x4 v = join[i * 64];
#pragma unroll
        for (int k = 1; k < LN_WAVES; ++k) v += join[(k * NB * MB + i) * 64];
        const int m = m0 + 16 * (i % MB) + r, n = 16 * (nb0 + i / MB) + 4 * g;
        ln_finish(p, m, n, v, ln_bias(p, n), ln_residual(p, m, n));
    }
}

// ---- many rows ---------------------------------------------------------------------------------------------------
constexpr int LN_BAND = 6;                     // row blocks that an XCD's tiles go through together

// A tile shape: BM x BN outputs per workgroup of 8 waves, WM x WN of them, K in steps of 64 through STAGES stages.
template <int BM_, int BN_, int STAGES_, int WM_, int WN_>
struct LnTile {
    static constexpr int BM = BM_, BN = BN_, STAGES = STAGES_, WM = WM_, WN = WN_;
    static constexpr int WPIECES = BN / 16 * 2, PIECES = WPIECES + BM / 8;      // 1 KB pieces of a stage: of w, then of x (8 rows each)
    static constexpr int LPW = PIECES / LN_WAVES;
    static constexpr int MB = BM / 16 / WM, NB = BN / 16 / WN;
    // results on their way out: a wave's 16 rows of them, and how many such it has room for in LDS
    static constexpr int OUT_PITCH = 16 * NB + 4, OUT_BLOCK = LN_WAVES * 16 * OUT_PITCH * 4;
    static constexpr int OUT_BLOCKS = OUT_BLOCK * MB <= 160 * 1024 ? MB : MB % 2 == 0 ? MB / 2 : 1;
    static constexpr int STAGE_BYTES = PIECES * 1024, LDS_BYTES = STAGES * STAGE_BYTES > OUT_BLOCK * OUT_BLOCKS ? STAGES * STAGE_BYTES : OUT_BLOCK * OUT_BLOCKS;
    static_assert(WM * WN == LN_WAVES && WPIECES % LN_WAVES == 0 && PIECES % LN_WAVES == 0 && STAGES * LPW < 64 && LDS_BYTES <= 160 * 1024 &&
                  BM % (16 * WM) == 0 && BN % (16 * WN) == 0, "tile of the linear layer");
};

template <int N>
__device__ __forceinline__ void ln_wait_vmcnt() {
    __builtin_amdgcn_s_waitcnt((N & 0xF) | ((N >> 4) << 14) | (0x7 << 4) | (0xF << 8));
}
// LDS reads the compiler does not see: `dst` is pending until ln_lds_wait, which waits for all of them.
__device__ __forceinline__ void ln_lds_read(ln_u32x4& dst, unsigned addr, int offset) {
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(dst) : "v"(addr), "n"(offset));
}
template <int N>
__device__ __forceinline__ void ln_lds_wait(ln_u32x4 (&x)[N]) {
    asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(x[0]));
#pragma unroll
    for (int i = 1; i < N; ++i) asm volatile("" : "+v"(x[i]));
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t ln_region(const uint16_t* base) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(base), 0, 0x7FFFFFFF, 0x00020000);   // raw buffer of dwords
}
__device__ __forceinline__ void ln_load_lds16(__amdgpu_buffer_rsrc_t r, char* to, int lane_off, int uniform_off) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(to), 16, lane_off, uniform_off, 0, 0);
}

template <typename Tile>
__global__ __launch_bounds__(64 * LN_WAVES) __attribute__((amdgpu_waves_per_eu(2, 2)))
void ll_linear_kernel(const LinearParams p) {
    constexpr int BM = Tile::BM, BN = Tile::BN, STAGES = Tile::STAGES, STAGE_BYTES = Tile::STAGE_BYTES, LPW = Tile::LPW;
    constexpr int MB = Tile::MB, NB = Tile::NB, WPIECES = Tile::WPIECES;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % Tile::WM, wn = wave / Tile::WM;
    // Workgroup b runs on XCD b % 8: every XCD takes one contiguous run of tiles.  They go through bands of up to 6 row blocks, row blocks fastest, so that
    // the 32 tiles an XCD has in work are about as many blocks of x as of w, which its L2 takes in once: 8192 rows, 4096 -> 8192 524 -> 412 us
    // (with weight blocks fastest a round of tiles reads all of w); bands of 4 and of 8 the same within 2 %.
    const int n_nt = (p.N + BN - 1) / BN, n_mt = (p.M + BM - 1) / BM;
    const int64_t total = int64_t(n_nt) * n_mt;
    const int xcd = blockIdx.x & 7;
    const int64_t tile = ((xcd * total + 7) >> 3) + (blockIdx.x >> 3);
    if (tile >= (((xcd + 1) * total + 7) >> 3)) return;          // uniform over the workgroup
    const int band = int(tile / (LN_BAND * n_nt)), in_band = int(tile % (LN_BAND * n_nt)), rows_of_band = min(LN_BAND, n_mt - band * LN_BAND);
    const int mt = band * LN_BAND + in_band % rows_of_band, nt = in_band / rows_of_band;
    // The last tile of rows begins where it is whole (there are BM rows at least); rows that the one before has are not stored twice.
    const int m_own = mt * BM, m0 = min(m_own, p.M - BM), n0 = nt * BN;
    const int KT = (p.K + 63) / 64, n_steps = 2 * KT;
    const int last_nb = (p.N + 15) / 16 - 1 - (n0 >> 4);

    // The pieces this wave loads per stage: pieces wave + 8 l of [w: (n block, half step) | x: 8 rows].  Blocks past the end are clamped to the
    // last one (their products are never stored).  In the last step the features past K are not read, but the row's first ones in their
    // place, and cleared once they have arrived.  What differs between lanes is one offset; the rest stays in scalar registers.
    const __amdgpu_buffer_rsrc_t w_from = ln_region(p.w_frag + int64_t(n0 >> 4) * n_steps * 512), x_from = ln_region(p.x + m0 * p.x_stride);
    const int piece = (lane & 7) ^ (lane >> 3);                  // of a row's 128 bytes
    const bool past = (KT - 1) * 64 + 8 * piece >= p.K;
    const int x_lane = (lane >> 3) * int(p.x_stride) * 2 + piece * 16;
    const int x_lane_last = past ? x_lane - piece * 16 : x_lane + (KT - 1) * 128;
    int src[LPW];                                                // wave-uniform
#pragma unroll
    for (int l = 0; l < LPW; ++l) {
        const int f = wave + LN_WAVES * l;
        src[l] = LN_WAVES * l < WPIECES ? (min(f / 2, last_nb) * n_steps + f % 2) * 1024 : (f - WPIECES) * 8 * int(p.x_stride) * 2;
    }
    auto issue = [&](int kt, int to, int l) {
        const bool last = kt >= KT - 1;                          // past the end the last step is fetched again, never used
        char* const at = lds + to * STAGE_BYTES + (wave + LN_WAVES * l) * 1024;
        if (LN_WAVES * l < WPIECES) ln_load_lds16(w_from, at, lane * 16, src[l] + (last ? KT - 1 : kt) * 2048);
        else ln_load_lds16(x_from, at, last ? x_lane_last : x_lane, src[l] + (last ? 0 : kt * 128));
    };
    // clears what this wave fetched in place of features past K; its own loads of that stage have arrived, and no wave has read it yet
    const unsigned lds_at = (unsigned)(size_t)(__attribute__((address_space(3))) char*)lds;
    auto clear_past = [&](int stage) {
        if (p.K % 64 == 0) return;
#pragma unroll
        for (int l = 0; l < LPW; ++l)
            if (LN_WAVES * l >= WPIECES && past) {
                const ln_u32x4 zero = {0, 0, 0, 0};
                asm volatile("ds_write_b128 %0, %1" ::"v"(lds_at + stage * STAGE_BYTES + (wave + LN_WAVES * l) * 1024 + lane * 16), "v"(zero) : "memory");
            }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    };

    ln_f32x4 acc[NB][MB];
#pragma unroll
    for (int a = 0; a < NB; ++a)
#pragma unroll
        for (int b = 0; b < MB; ++b) acc[a][b] = ln_f32x4{0.f, 0.f, 0.f, 0.f};

    // Fragment i of half step `sub` of a stage: the wave's NB of w, then its MB of x.  Two register sets: while the MFMAs of one half step run
    // from the one, the next one's fragments are read into the other (out_proj.hip).
    constexpr int NFR = NB + MB, NMFMA = NB * MB;
    ln_u32x4 fr[2][NFR];
    const unsigned w_at = lds_at + lane * 16 + wn * NB * 2048;
    const unsigned x_row = lds_at + WPIECES * 1024 + wm * MB * 2048 + (r >> 3) * 1024 + (r & 7) * 128;
    const unsigned x_at[2] = {x_row + ((g ^ (r & 7)) * 16), x_row + (((4 + g) ^ (r & 7)) * 16)};
    auto read_frag = [&](ln_u32x4& dst, unsigned stage_at, int sub, int i) {
        if (i < NB) ln_lds_read(dst, w_at + stage_at, (i * 2 + sub) * 1024);
        else ln_lds_read(dst, x_at[sub] + stage_at, (i - NB) * 2048);
    };
#pragma unroll
    for (int j = 0; j < STAGES; ++j)
#pragma unroll
        for (int l = 0; l < LPW; ++l) issue(j, j, l);
    ln_wait_vmcnt<(STAGES - 1) * LPW>();
    if (KT == 1) clear_past(0);
    asm volatile("s_barrier" ::: "memory");
#pragma unroll
    for (int i = 0; i < NFR; ++i) read_frag(fr[0][i], 0, 0, i);
    int stage = 0;                               // kt mod STAGES
    for (int kt = 0; kt < KT; ++kt) {
        const int next = stage + 1 == STAGES ? 0 : stage + 1;
#pragma unroll
        for (int sub = 0; sub < 2; ++sub) {
            ln_lds_wait(fr[sub]);
            if (sub == 1) {
                // every read of this step's stage has returned here, and this wave's loads of the next step have landed: behind the barrier that
                // holds for every wave, the stage is loaded anew and the next one read
                ln_wait_vmcnt<(STAGES - 2) * LPW>();
                if (kt + 2 == KT) clear_past(next);
                asm volatile("s_barrier" ::: "memory");
            }
            const unsigned from = unsigned(sub == 1 ? next : stage) * STAGE_BYTES;
#pragma unroll
            for (int m = 0; m < NMFMA; ++m) {
                const int a = m / MB, b = m % MB;
                acc[a][b] = ln_mfma(fr[sub][a], fr[sub][NB + b], acc[a][b]);
                constexpr int SPAN = (NMFMA + 1) / 2;            // reads over the first half of the products, loads over all of them
#pragma unroll
                for (int i = (m * NFR + SPAN - 1) / SPAN; i < NFR && i * SPAN < (m + 1) * NFR; ++i) read_frag(fr[1 - sub][i], from, 1 - sub, i);
                if (sub == 1)
#pragma unroll
                    for (int l = (m * LPW + NMFMA - 1) / NMFMA; l * NMFMA < (m + 1) * LPW; ++l) issue(kt + STAGES, stage, l);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        stage = next;
    }
    ln_lds_wait(fr[0]);                          // no load may still be writing registers or LDS past this point
    ln_wait_vmcnt<0>();

    // Out through LDS, each wave through a part of its own: a lane then has 8 neighbouring features, and 2 NB lanes the whole of the wave's part of a
    // row (128 bytes and more), where straight from the accumulators every lane would store 8 bytes of a row of its own.
    // The residual comes the same way, 16 rows ahead.  The loop over 16 rows stays one: 4680 rows, 1536 -> 6144 with GELU 112 -> 109 us against
    // all of it unrolled, whose instructions come from memory once a tile.
    asm volatile("s_barrier" ::: "memory");      // no wave reads its operands any more
    constexpr int ROW_LANES = 2 * NB, ROWS = 64 / ROW_LANES, PASSES = 16 / ROWS, PITCH = Tile::OUT_PITCH, AT_ONCE = Tile::OUT_BLOCKS;
    float* const own = reinterpret_cast<float*>(lds) + wave * (AT_ONCE * 16 * PITCH);
    const int own_row = lane / ROW_LANES, n = n0 + wn * NB * 16 + lane % ROW_LANES * 8;
    auto row = [&](int b, int pass) {
        const int m = m0 + (wm * MB + b) * 16 + pass * ROWS + own_row;
        return m < m_own ? p.M : m;
    };
    const ln_u32x2 bias[2] = {ln_bias(p, n), ln_bias(p, n + 4)};
    const bool whole = p.wide8 && n0 + BN <= p.N;                // m has a bound of its own in any case
#pragma unroll
    for (int b0 = 0; b0 < MB; b0 += AT_ONCE) {
#pragma unroll
        for (int b = 0; b < AT_ONCE; ++b)
#pragma unroll
            for (int a = 0; a < NB; ++a) *reinterpret_cast<ln_f32x4*>(own + (16 * b + r) * PITCH + 16 * a + 4 * g) = acc[a][b0 + b];
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();         // lanes read what other lanes of the wave wrote: LDS keeps their order
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        auto out = [&](auto whole_, auto act) {
            constexpr bool WHOLE = decltype(whole_)::value;
            ln_u32x4 residual[PASSES];
            auto ask = [&](int b) {
#pragma unroll
                for (int s = 0; s < PASSES; ++s) residual[s] = ln_residual8<WHOLE>(p, row(b0 + b, s), n);
            };
            ask(0);
#pragma nounroll
            for (int b = 0; b < AT_ONCE; ++b) {
                ln_u32x4 here[PASSES];
#pragma unroll
                for (int s = 0; s < PASSES; ++s) here[s] = residual[s];
                if (b + 1 < AT_ONCE) ask(b + 1);
#pragma unroll
                for (int s = 0; s < PASSES; ++s) {
                    const float* const from = own + (16 * b + s * ROWS + own_row) * PITCH + lane % ROW_LANES * 8;
                    ln_store8<WHOLE>(p, row(b0 + b, s), n, ln_activated<decltype(act)::value>(p, *reinterpret_cast<const ln_f32x4*>(from), bias[0]),
                                     ln_activated<decltype(act)::value>(p, *reinterpret_cast<const ln_f32x4*>(from + 4), bias[1]), here[s]);
                }
            }
        };
        if (whole && p.act == LL_ACT_NONE) out(std::true_type{}, std::integral_constant<int, LL_ACT_NONE>{});
        else if (whole) out(std::true_type{}, std::integral_constant<int, -1>{});
        else out(std::false_type{}, std::integral_constant<int, -1>{});
        __builtin_amdgcn_wave_barrier();
    }
}

// One thread per 16-byte unit of the packed weight.
__global__ __launch_bounds__(256) void ll_linear_pack_kernel(const uint16_t* w, int64_t w_stride, uint16_t* w_frag, int N, int K, int64_t units, int n_steps) {
    const int64_t unit = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (unit >= units) return;
    const int lane = int(unit & 63), r = lane & 15, g = lane >> 4;
    const int ks = int((unit >> 6) % n_steps), nb = int((unit >> 6) / n_steps);
    const int n = 16 * nb + r, k = 32 * ks + 8 * g;
    ln_u32x4 o = {0, 0, 0, 0};
    if (n < N && k < K) o = *reinterpret_cast<const ln_u32x4*>(w + n * w_stride + k);       // K is a multiple of 8
    *reinterpret_cast<ln_u32x4*>(w_frag + unit * 8) = o;
}

hipError_t launch_linear_pack(const uint16_t* w, int64_t w_stride, uint16_t* w_frag, int N, int K, hipStream_t s) {
    const int64_t units = linear_padded_n(N) * linear_padded_k(K) / 8;
    if (units * 8 > LINEAR_MAX_NUMBERS) return hipErrorInvalidValue;
    hipLaunchKernelGGL(ll_linear_pack_kernel, dim3(unsigned((units + 255) / 256)), dim3(256), 0, s, w, w_stride, w_frag, N, K, units, int(linear_padded_k(K) / 32));
    return hipGetLastError();
}

template <typename Tile>
static hipError_t launch_tile(const LinearParams& p, hipStream_t s) {
    const int64_t tiles = int64_t((p.M + Tile::BM - 1) / Tile::BM) * ((p.N + Tile::BN - 1) / Tile::BN);
    if (tiles > LINEAR_MAX_BLOCKS - 7) return hipErrorInvalidValue;
    static std::atomic<uint64_t> done{0};                        // GPUs on which the kernel has been given its LDS (the first 64 remember it)
    int device = 0;
    hipError_t e = hipGetDevice(&device);
    if (e != hipSuccess) return e;
    const uint64_t bit = device < 64 ? uint64_t(1) << device : 0;
    if (!(done.load(std::memory_order_relaxed) & bit)) {
        e = hipFuncSetAttribute(reinterpret_cast<const void*>(ll_linear_kernel<Tile>), hipFuncAttributeMaxDynamicSharedMemorySize, Tile::LDS_BYTES);
        if (e != hipSuccess) return e;
        done.fetch_or(bit, std::memory_order_relaxed);
    }
    hipLaunchKernelGGL(ll_linear_kernel<Tile>, dim3(unsigned((tiles + 7) / 8 * 8)), dim3(64 * LN_WAVES), Tile::LDS_BYTES, s, p);
    return hipGetLastError();
}

template <int MB, int NB>
static hipError_t launch_few(const LinearParams& p, hipStream_t s) {
    const int64_t blocks = linear_blocks(LinearShape{16 * MB, 16 * NB}, p.M, p.N);
    if (blocks > LINEAR_MAX_BLOCKS) return hipErrorInvalidValue;
    hipLaunchKernelGGL((ll_linear_few_kernel<MB, NB>), dim3(unsigned(blocks)), dim3(64 * LN_WAVES), 0, s, p);
    return hipGetLastError();
}

hipError_t launch_linear(const LinearParams& p, hipStream_t s) {
    switch (linear_choose(p.M, p.N, p.K)) {
    case 0: return launch_few<1, 1>(p, s);
    case 1: return launch_few<1, 2>(p, s);
    case 2: return launch_few<2, 1>(p, s);
    case 3: return launch_few<2, 2>(p, s);
    case 4: return launch_few<3, 1>(p, s);
    case 5: return launch_few<3, 2>(p, s);
    case 6: return launch_few<4, 1>(p, s);
    case 7: return launch_few<4, 2>(p, s);
    case 8: return launch_tile<LnTile<64, 64, 6, 4, 2>>(p, s);
    case 9: return launch_tile<LnTile<128, 64, 5, 4, 2>>(p, s);
    case 10: return launch_tile<LnTile<128, 128, 3, 4, 2>>(p, s);
    case 11: return launch_tile<LnTile<192, 128, 4, 4, 2>>(p, s);
    case 12: return launch_tile<LnTile<192, 256, 2, 4, 2>>(p, s);
    case 13: return launch_tile<LnTile<256, 128, 3, 4, 2>>(p, s);
    default: return launch_tile<LnTile<256, 256, 2, 4, 2>>(p, s);
    }
}

}  // namespace ll
