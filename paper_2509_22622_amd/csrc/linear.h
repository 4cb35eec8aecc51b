// y = act(x w^T + bias) + residual (include/longlive.h, ll_linear): what w looks like once it is packed, the choice of a kernel by the sizes (plain
// C++, checked on the host), the launches.
#pragma once

#include <cstdint>

namespace ll {

// Packed weight: [n block of 16][k step of 32][64 lanes][8], lane 16 g + r: w[16 nb + r][32 ks + 8 g + 0..7]; zeros where n or k lies
// past the end.  k steps come in pairs.
inline int64_t linear_padded_n(int n) { return (int64_t(n) + 15) / 16 * 16; }
inline int64_t linear_padded_k(int k) { return (int64_t(k) + 63) / 64 * 64; }
constexpr int64_t LINEAR_MAX_NUMBERS = int64_t(1) << 34;        // of a packed weight: a thread packs 8, and a launch has less than 2^32
constexpr int64_t LINEAR_MAX_BLOCKS = (int64_t(1) << 23) - 1;   // workgroups of 512 threads of a launch, likewise
constexpr int LINEAR_MAX_N = 1 << 20, LINEAR_MAX_K = 1 << 20, LINEAR_MAX_STRIDE = 1 << 21;   // offsets inside a tile stay below 2^31

// The blocks of outputs a workgroup can take, and the time of a launch with them: launch + rounds of workgroups over the CUs x (round + steps of 64
// features x (step, and `full` more the more CUs are at work)).  Fitted to 1400 timings (1 to 8192 rows, 300 to 8192 features out, 1024 to 6144 in), off by
// 10 % (rms); the shape it picks is the fastest one or within 0.5 % of it on average.  Without 48-row blocks the picks are 2 % slower on
// average, without those of 192 rows 1.6 % (2400 rows, 4096 -> 4096 84 us, without them 92).
struct LinearShape { int rows, cols; double launch, round, step, full; };
constexpr LinearShape LINEAR_SHAPES[] = {
    {16, 16, 1.86, 0.62, 0.0415, 0.0722},  {16, 32, 1.99, 0.0, 0.0782, 0.1303},   {32, 16, 1.23, 0.83, 0.0975, 0.0235},  {32, 32, 2.25, 0.05, 0.1046, 0.0755},
    {48, 16, 1.66, 0.80, 0.1101, 0.0185},  {48, 32, 1.79, 0.92, 0.1299, 0.0372},  {64, 16, 1.88, 0.93, 0.1241, 0.0229},  {64, 32, 1.68, 1.52, 0.1511, 0.0156},
    {64, 64, 2.09, 1.49, 0.2063, 0.0289},  {128, 64, 2.14, 1.68, 0.3041, 0.0436}, {128, 128, 1.04, 2.75, 0.4501, 0.0591}, {192, 128, 0.0, 5.40, 0.5623, 0.0729},
    {192, 256, 0.0, 4.68, 1.0635, 0.1125}, {256, 128, 0.0, 6.44, 0.6568, 0.1338}, {256, 256, 0.0, 7.54, 1.1827, 0.2294},
};
constexpr int LINEAR_FEW = 8;                  // the first of the LDS-ring tiles: these need a tile's rows at least, the others a row in each 16

inline int64_t linear_blocks(const LinearShape& s, int m, int n) { return (int64_t(m) + s.rows - 1) / s.rows * ((int64_t(n) + s.cols - 1) / s.cols); }
inline int linear_choose(int m, int n, int k) {
    int best = 0;
    double least = 0;
    for (int i = 0; i < int(sizeof(LINEAR_SHAPES) / sizeof(LINEAR_SHAPES[0])); ++i) {
        const LinearShape& s = LINEAR_SHAPES[i];
        if (m < (i < LINEAR_FEW ? s.rows - 15 : s.rows)) break;               // those behind it are no smaller
        const int64_t blocks = linear_blocks(s, m, n);
        const double at_work = blocks < 256 ? double(blocks) / 256 : 1.0;
        const double us = s.launch + double((blocks + 255) / 256) * (s.round + double((int64_t(k) + 63) / 64) * (s.step + s.full * at_work));
        if (i == 0 || us < least) {
            least = us;
            best = i;
        }
    }
    return best;
}

}  // namespace ll

#if defined(__HIPCC__)
#include <hip/hip_runtime.h>

namespace ll {

struct LinearParams {
    const uint16_t *x, *w_frag, *bias, *residual;   // bias, residual: null if there is none
    uint16_t* y;
    int64_t x_stride, residual_stride, y_stride;
    int M, N, K;
    int act;                                        // ll_activation
    int wide, wide8;                                // groups of four, of eight features of y and the residual are 8-, 16-byte aligned
};
hipError_t launch_linear_pack(const uint16_t* w, int64_t w_stride, uint16_t* w_frag, int N, int K, hipStream_t s);
hipError_t launch_linear(const LinearParams& p, hipStream_t s);

}  // namespace ll
#endif
