// Layer norm, forward and backward (include/longlive.h, ll_layer_norm*): how rows are dealt to threads (plain C++, checked on the host by
// tests/check_norm_rules.cpp), and the launches.
#pragma once

#include <cstdint>

namespace ll {

constexpr int NORM_MAX_ROWS = 1 << 24, NORM_MAX_FEATURES = 16384, NORM_MAX_STRIDE = 1 << 21;

// A row is held in the registers of `threads` threads (16 of a wave, or whole waves), `pieces` of 8 features each.  A workgroup has `teams` of so many threads, and a team
// of the forward pass works on `rows` rows at a time: two pieces a thread, which keep enough bytes on the way and leave registers for other waves.  us for one, two and four pieces a
// thread, bfloat16: 1111 x 1536 4.7, 5.0, 5.6; 4680 x 1536 9.6, 9.0, 9.3; 16000 x 4096 60, 48, 49; and for one row of two pieces and two rows 16000 x 8192 100 and 110.
struct NormShape { int threads, pieces, teams, rows; };
inline NormShape norm_shape(int features) {
    if (features <= 128) return {16, 1, 16, 2};
    if (features <= 256) return {16, 2, 16, 1};
    const int pieces = features <= 4096 ? 1 : 2, waves = (features + 512 * pieces - 1) / (512 * pieces);
    return {64 * waves, pieces, waves >= 4 ? 1 : 4 / waves, 2 / pieces};
}

// The backward pass: rows that share a weight go to `chunks` workgroups, `rows` rows each.  Each chunk leaves sums of 2 x features in 32 bits, which have to be written and
// read again: at least 4 rows a chunk, and no more workgroups than the 256 CUs hold at once (`slots`: 16 waves a CU, 8 where a thread has two pieces, whose registers allow no more), which then need no second
// round.  That is so in bfloat16; in 32 bits, and of 16-lane teams with x in 32 bits, registers hold 12 waves, and of workgroups of four waves a quarter comes behind the others (8000 x 1024 31 us, 8000 x 2048 54,
// 131 and 262 MB; 32000 x 128 23).  In bfloat16: us in one and in up to 1024 workgroups, 2100 x 8192 30 and 41, 8000 x 5120 65 and 83, 8000 x 4096 45 and 52, 32000 x 200 23 and 32; 32000 x 8192 323 and 332.
// More than 1024 cost more than they give (32760 of 1536, forward and backward: 132, with up to 2048 139).
constexpr int NORM_ONE = 4;            // rows a team that one workgroup takes by itself: a launch less (with 10, 77 x 512 took 15 us, against 7 + 3 for the sum kernel)
struct NormPlan { int groups, chunks, rows; };
inline NormPlan norm_plan(int m, int features, int group_rows) {
    const NormShape s = norm_shape(features);
    NormPlan p;
    const int each = group_rows ? (group_rows < m ? group_rows : m) : m;             // rows of a group
    p.groups = group_rows ? int((int64_t(m) + group_rows - 1) / group_rows) : 1;
    const int round = s.teams, least = round > 4 ? round : 4;
    const int waves = s.threads * s.teams / 64, resident = s.pieces == 1 || s.threads > 512 ? 16 : 8;
    const int slots = 256 * (resident / waves < 4 ? resident / waves : 4);
    int64_t chunks = p.groups ? slots / p.groups : 1;
    if (chunks > (each + least - 1) / least) chunks = (each + least - 1) / least;
    if (each <= NORM_ONE * s.teams) chunks = 1;
    if (chunks < 1) chunks = 1;
    p.rows = int((each + chunks - 1) / chunks);
    if (chunks > 1) p.rows = (p.rows + round - 1) / round * round;
    p.chunks = p.rows ? (each + p.rows - 1) / p.rows : 1;
    return p;
}
// Numbers (fp32) of the partial sums of the weight's and the bias's gradient.
inline int64_t norm_numbers(const NormPlan& p, int features) { return p.chunks > 1 ? int64_t(p.groups) * p.chunks * 2 * features : 0; }

}  // namespace ll

#if defined(__HIPCC__)
#include <hip/hip_runtime.h>

namespace ll {

struct NormParams {
    const void *x, *dy, *residual, *weight, *bias;
    void *y, *dx;
    float *stats;                           // [m][2]: mean, 1 / sqrt(variance + eps); forward: null where not wanted
    float *dweight, *dbias;                 // [groups][n]; null where not wanted
    float* part;                            // [group][chunk][2][n]
    int64_t x_stride, y_stride, dy_stride, dx_stride, residual_stride;
    int m, n, group_rows;                   // group_rows: m where all rows share a weight
    int x_f32, y_f32, w_f32;
    int wide;                               // pieces of 8 features of everything are whole and 16-byte aligned
    float eps;
    NormPlan plan;
};
hipError_t launch_norm_forward(const NormParams& p, hipStream_t s);
hipError_t launch_norm_backward(const NormParams& p, hipStream_t s);

}  // namespace ll
#endif
