// ll_linear: y = act(x w^T + bias) + residual, x [M, K] and y [M, N] row-major, w [N, K] packed once (linear.h); bf16 in and out, fp32 sums,
// one rounding at the end.  Two kernels:
//
// ll_linear_few_kernel, up to 64 rows: bound by the weight's way from memory (2 N K bytes; 64 rows are 64 flops a byte, the chip has some 400).
//   A workgroup owns 16 (or 32) features and every row, its eight waves split K, and join in LDS in a fixed order: no workgroup
//   waits for another, and w passes by once, in contiguous 1 KB loads.
// ll_linear_kernel, more rows: bound by the matrix instructions and, before that, by L2.  Tiles of y through a ring of LDS stages, as the output
//   projection of the cross-attention block (out_proj.hip) has them; x is row-major here, since it comes from the caller.
//   A stage holds 64 features: a load instruction takes the 128 bytes of each of 8 rows, whole cache lines, and leaves the eight 16-byte pieces of row r
//   in the order piece ^ (r & 7), so that the 16 rows of a fragment read lie in different banks.
//
// Both compute the transposed product y^T = w x^T on 16x16x32 MFMAs: A = w, B = x; lane (g, c) register j of a block is y[m0 + c][n0 + 4 g + j],
// four neighbouring features, one 8-byte store.
#include "linear.h"

#include <algorithm>
#include <atomic>

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

// The activations.  In the form y * sigmoid(..) or y * erfc(..) nothing is lost to cancellation where y is far below zero.
__device__ __forceinline__ float ln_act(float y, int act) {
    switch (act) {
    case LL_ACT_GELU_TANH: return y / (1.0f + __expf(-1.5957691216057308f * (y + 0.044715f * y * y * y)));
    case LL_ACT_GELU: return 0.5f * y * erfcf(-0.70710678118654752f * y);
    case LL_ACT_SILU: return y / (1.0f + __expf(-y));
    default: return y;
    }
}

// Features n .. n + 3 of row m: bias, activation, residual, rounding, store.
__device__ __forceinline__ void ln_finish(const LinearParams& p, int m, int n, ln_f32x4 v) {
    if (m >= p.M || n >= p.N) return;
    const uint16_t* const r = p.residual ? p.residual + m * p.residual_stride + n : nullptr;
    uint16_t* const y = p.y + m * p.y_stride + n;
    if (p.wide && n + 4 <= p.N) {
        if (p.bias) {
            const ln_u32x2 b = *reinterpret_cast<const ln_u32x2*>(p.bias + n);
            v += ln_f32x4{ln_widen(b[0]), __uint_as_float(b[0] & 0xFFFF0000u), ln_widen(b[1]), __uint_as_float(b[1] & 0xFFFF0000u)};
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = ln_act(v[j], p.act);
        if (r) {
            const ln_u32x2 b = *reinterpret_cast<const ln_u32x2*>(r);
            v += ln_f32x4{ln_widen(b[0]), __uint_as_float(b[0] & 0xFFFF0000u), ln_widen(b[1]), __uint_as_float(b[1] & 0xFFFF0000u)};
        }
        const ln_f32x2 lo = {v[0], v[1]}, hi = {v[2], v[3]};
        *reinterpret_cast<ln_u32x2*>(y) = ln_u32x2{__builtin_bit_cast(unsigned, __builtin_convertvector(lo, ln_bf16x2)),
                                                   __builtin_bit_cast(unsigned, __builtin_convertvector(hi, ln_bf16x2))};
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (n + j >= p.N) break;
        float x = v[j] + (p.bias ? ln_widen(p.bias[n + j]) : 0.f);
        x = ln_act(x, p.act);
        if (r) x += ln_widen(r[j]);
        y[j] = __builtin_bit_cast(uint16_t, __bf16(x));
    }
}

// ---- few rows ----------------------------------------------------------------------------------------------------
constexpr int LN_WAVES = 8;

template <int MB, int NB>
__global__ __launch_bounds__(64 * LN_WAVES) void ll_linear_few_kernel(const LinearParams p) {
    constexpr int U = MB >= 4 ? 3 : 6;            // k steps of a wave on their way at once
    __shared__ __attribute__((aligned(16))) ln_f32x4 join[LN_WAVES][NB * MB][64];
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n_steps = (p.K + 63) / 64 * 2, last_nb = (p.N + 15) / 16 - 1, nb0 = blockIdx.x * NB;
    const uint16_t* w[NB];
#pragma unroll
    for (int a = 0; a < NB; ++a) w[a] = p.w_frag + int64_t(min(nb0 + a, last_nb)) * n_steps * 512 + lane * 8;
    const uint16_t* x[MB];
#pragma unroll
    for (int b = 0; b < MB; ++b) x[b] = p.x + min(16 * b + r, p.M - 1) * p.x_stride + 8 * g;
    ln_f32x4 acc[NB * MB];
#pragma unroll
    for (int i = 0; i < NB * MB; ++i) acc[i] = ln_f32x4{0.f, 0.f, 0.f, 0.f};
    for (int first = wave; first < n_steps; first += LN_WAVES * U) {
        ln_u32x4 wf[U][NB], xf[U][MB];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int ks = min(first + LN_WAVES * u, n_steps - 1);
#pragma unroll
            for (int a = 0; a < NB; ++a) wf[u][a] = *reinterpret_cast<const ln_u32x4*>(w[a] + ks * 512);
#pragma unroll
            for (int b = 0; b < MB; ++b)
                xf[u][b] = 32 * ks + 8 * g < p.K ? *reinterpret_cast<const ln_u32x4*>(x[b] + 32 * ks) : ln_u32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (first + LN_WAVES * u < n_steps)
#pragma unroll
                for (int a = 0; a < NB; ++a)
#pragma unroll
                    for (int b = 0; b < MB; ++b) acc[a * MB + b] = ln_mfma(wf[u][a], xf[u][b], acc[a * MB + b]);
    }
#pragma unroll
    for (int i = 0; i < NB * MB; ++i) join[wave][i][lane] = acc[i];
    __syncthreads();
    for (int i = wave; i < NB * MB; i += LN_WAVES) {
        ln_f32x4 v = join[0][i][lane];
#pragma unroll
        for (int k = 1; k < LN_WAVES; ++k) v += join[k][i][lane];
        ln_finish(p, 16 * (i % MB) + r, 16 * (nb0 + i / MB) + 4 * g, v);
    }
}

// ---- many rows ---------------------------------------------------------------------------------------------------
// A tile shape: BM x BN outputs per workgroup of 8 waves, WM x WN of them, K in steps of 64 through STAGES stages.
template <int BM_, int BN_, int STAGES_, int WM_, int WN_>
struct LnTile {
    static constexpr int BM = BM_, BN = BN_, STAGES = STAGES_, WM = WM_, WN = WN_;
    static constexpr int WPIECES = BN / 16 * 2, PIECES = WPIECES + BM / 8;      // 1 KB pieces of a stage: of w, then of x (8 rows each)
    static constexpr int STAGE_BYTES = PIECES * 1024, LDS_BYTES = STAGES * STAGE_BYTES;
    static constexpr int LPW = PIECES / LN_WAVES;
    static constexpr int MB = BM / 16 / WM, NB = BN / 16 / WN;
    static_assert(WM * WN == LN_WAVES && WPIECES % LN_WAVES == 0 && PIECES % LN_WAVES == 0 && STAGES * LPW < 64 && LDS_BYTES <= 160 * 1024 && MB >= 1 && NB >= 1,
                  "tile of the linear layer");
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
    // Workgroup b runs on XCD b % 8: every XCD takes one contiguous run of tiles, weight blocks fastest, and with it a few row blocks of x.
    const int n_nt = (p.N + BN - 1) / BN, n_mt = (p.M + BM - 1) / BM;
    const int64_t total = int64_t(n_nt) * n_mt;
    const int xcd = blockIdx.x & 7;
    const int64_t tile = ((xcd * total + 7) >> 3) + (blockIdx.x >> 3);
    if (tile >= (((xcd + 1) * total + 7) >> 3)) return;          // uniform over the workgroup
    const int mt = int(tile / n_nt), nt = int(tile % n_nt);
    const int m0 = mt * BM, n0 = nt * BN;
    const int KT = (p.K + 63) / 64, n_steps = 2 * KT;
    const int last_nb = (p.N + 15) / 16 - 1, last_row = p.M - 1;

    // The pieces this wave loads per stage: pieces wave + 8 l of [w: (n block, half step) | x: 8 rows].  Blocks and rows past the end are
    // clamped to the last one (their products are never stored).  In the last step the features past K are not read, but the row's
    // first ones in their place, and cleared once they have arrived.
    const __amdgpu_buffer_rsrc_t w_from = ln_region(p.w_frag + int64_t(n0 >> 4) * n_steps * 512), x_from = ln_region(p.x + m0 * p.x_stride);
    int src[LPW], src_last[LPW];
    const int piece = (lane & 7) ^ (lane >> 3);                  // of a row's 128 bytes
    const bool past = (KT - 1) * 64 + 8 * piece >= p.K;
#pragma unroll
    for (int l = 0; l < LPW; ++l) {
        const int f = wave + LN_WAVES * l;                       // wave-uniform
        if (LN_WAVES * l < WPIECES) {
            src[l] = (min(f / 2, last_nb - (n0 >> 4)) * n_steps + f % 2) * 1024 + lane * 16;
            src_last[l] = src[l];
        } else {
            const int row = min(m0 + (f - WPIECES) * 8 + (lane >> 3), last_row) - m0;
            src[l] = int(row * p.x_stride) * 2 + piece * 16;
            src_last[l] = past ? src[l] - piece * 16 : src[l] + (KT - 1) * 128;
        }
    }
    auto issue = [&](int kt, int to, int l) {
        const bool last = kt >= KT - 1;                          // past the end the last step is fetched again, never used
        const int kc = last ? KT - 1 : kt;
        const bool of_w = LN_WAVES * l < WPIECES;
        ln_load_lds16(of_w ? w_from : x_from, lds + to * STAGE_BYTES + (wave + LN_WAVES * l) * 1024, last ? src_last[l] : src[l],
                      of_w ? kc * 2048 : last ? 0 : kc * 128);
    };
    // clears what this wave fetched in place of features past K; its own loads of that stage have arrived
    auto clear_past = [&](int stage) {
        if (p.K % 64 == 0) return;
#pragma unroll
        for (int l = 0; l < LPW; ++l)
            if (LN_WAVES * l >= WPIECES && past) {
                const unsigned at = (unsigned)(size_t)(__attribute__((address_space(3))) char*)lds + stage * STAGE_BYTES + (wave + LN_WAVES * l) * 1024 + lane * 16;
                const ln_u32x4 zero = {0, 0, 0, 0};
                asm volatile("ds_write_b128 %0, %1" ::"v"(at), "v"(zero) : "memory");
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
    const unsigned lds_at = (unsigned)(size_t)(__attribute__((address_space(3))) char*)lds;
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
#pragma unroll
                for (int i = 0; i < NFR; ++i)
                    if (i * ((NMFMA + 1) / 2) / NFR == m) read_frag(fr[1 - sub][i], from, 1 - sub, i);
                if (sub == 1)
#pragma unroll
                    for (int l = 0; l < LPW; ++l)
                        if (l * NMFMA / LPW == m) issue(kt + STAGES, stage, l);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        stage = next;
    }
    ln_lds_wait(fr[0]);                          // no load may still be writing registers or LDS past this point
    ln_wait_vmcnt<0>();

#pragma unroll
    for (int b = 0; b < MB; ++b)
#pragma unroll
        for (int a = 0; a < NB; ++a) ln_finish(p, m0 + (wm * MB + b) * 16 + r, n0 + (wn * NB + a) * 16 + 4 * g, acc[a][b]);
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
    if ((units + 255) / 256 > 0x7FFFFFFF) return hipErrorInvalidValue;
    hipLaunchKernelGGL(ll_linear_pack_kernel, dim3(unsigned((units + 255) / 256)), dim3(256), 0, s, w, w_stride, w_frag, N, K, units, int(linear_padded_k(K) / 32));
    return hipGetLastError();
}

template <typename Tile>
static hipError_t launch_tile(const LinearParams& p, hipStream_t s) {
    const int64_t tiles = int64_t((p.M + Tile::BM - 1) / Tile::BM) * ((p.N + Tile::BN - 1) / Tile::BN);
    if (tiles > 0x7FFFFF00) return hipErrorInvalidValue;
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
    hipLaunchKernelGGL((ll_linear_few_kernel<MB, NB>), dim3(unsigned(((p.N + 15) / 16 + NB - 1) / NB)), dim3(64 * LN_WAVES), 0, s, p);
    return hipGetLastError();
}

using LnTile256x128 = LnTile<256, 128, 3, 4, 2>;
using LnTile128x128 = LnTile<128, 128, 3, 4, 2>;
using LnTile128x64 = LnTile<128, 64, 5, 4, 2>;
using LnTile64x64 = LnTile<64, 64, 6, 4, 2>;

// Time of a launch in us: rounds of workgroups over the CUs, each `around` and a walk over K whose step takes `alone` with few workgroups
// on the chip and `more` longer with all CUs at work (out_proj.hip).
template <typename Tile>
static double tile_us(const LinearParams& p, double launch, double around, double alone, double more) {
    const int64_t tiles = int64_t((p.M + Tile::BM - 1) / Tile::BM) * ((p.N + Tile::BN - 1) / Tile::BN);
    return launch + double((tiles + 255) / 256) * (around + double((p.K + 63) / 64) * (alone + more * double(std::min<int64_t>(tiles, 256)) / 256));
}

hipError_t launch_linear(const LinearParams& p, hipStream_t s) {
    if (p.M <= 64) {
        const bool two = (p.N + 15) / 16 >= 256;                 // 32 features a workgroup where there are workgroups enough
        if (p.M <= 16) return two ? launch_few<1, 2>(p, s) : launch_few<1, 1>(p, s);
        if (p.M <= 32) return two ? launch_few<2, 2>(p, s) : launch_few<2, 1>(p, s);
        return two ? launch_few<4, 2>(p, s) : launch_few<4, 1>(p, s);
    }
    const double t0 = tile_us<LnTile256x128>(p, 2.3, 3.85, 0.626, 0.257), t1 = tile_us<LnTile128x128>(p, 2.0, 2.36, 0.367, 0.136);
    const double t2 = tile_us<LnTile128x64>(p, 1.7, 2.13, 0.216, 0.098), t3 = tile_us<LnTile64x64>(p, 1.8, 1.38, 0.151, 0.103);
    const double best = std::min(std::min(t0, t1), std::min(t2, t3));
    if (best == t0) return launch_tile<LnTile256x128>(p, s);
    if (best == t1) return launch_tile<LnTile128x128>(p, s);
    if (best == t2) return launch_tile<LnTile128x64>(p, s);
    return launch_tile<LnTile64x64>(p, s);
}

}  // namespace ll
