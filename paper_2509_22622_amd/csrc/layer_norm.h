// Layer norm, forward and backward (include/longlive.h, ll_layer_norm*): how rows are dealt to threads (plain C++, checked on the host by
// tests/check_norm_rules.cpp), and the launches.
#pragma once

#include <cstdint>

namespace ll {

constexpr int NORM_MAX_ROWS = 1 << 24, NORM_MAX_FEATURES = 16384, NORM_MAX_STRIDE = 1 << 21;

// A row is held in the registers of `threads` threads, `pieces` of 8 features each; a workgroup has 256 threads (512 for the widest) and so one row or more.
struct NormShape {
    int threads, pieces;
    int workgroup() const { return threads < 256 ? 256 : threads; }
    int rows() const { return workgroup() / threads; }
};
constexpr NormShape NORM_SHAPES[] = {{16, 1}, {16, 2}, {16, 4}, {64, 2}, {64, 3}, {64, 4}, {256, 2}, {256, 3}, {256, 4}, {512, 3}, {512, 4}};
constexpr int NORM_SHAPE_COUNT = int(sizeof(NORM_SHAPES) / sizeof(NORM_SHAPES[0]));
inline int norm_shape(int features) {
    int i = 0;
    while (NORM_SHAPES[i].threads * NORM_SHAPES[i].pieces * 8 < features) ++i;
    return i;
}

// The backward pass: rows that share a weight go to `chunks` workgroups, `rows` rows each.
struct NormPlan { int groups, chunks, rows; };
inline NormPlan norm_plan(int m, int features, int group_rows) {
    const NormShape& s = NORM_SHAPES[norm_shape(features)];
    NormPlan p;
    const int each = group_rows ? (group_rows < m ? group_rows : m) : m;             // rows of a group
    p.groups = group_rows ? int((int64_t(m) + group_rows - 1) / group_rows) : 1;
    const int most = (each + s.rows() - 1) / s.rows();                                // a row of each part of a workgroup
    int64_t chunks = p.groups ? (1024 + p.groups - 1) / p.groups : 1;
    if (chunks > most) chunks = most;
    if (chunks < 1) chunks = 1;
    p.rows = int((each + chunks - 1) / chunks);
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
    int wide, w_wide;                       // pieces of 8 features of the rows, of weight and bias, are 16-byte aligned and whole
    float eps;
    NormPlan plan;
};
hipError_t launch_norm_forward(const NormParams& p, hipStream_t s);
hipError_t launch_norm_backward(const NormParams& p, hipStream_t s);

}  // namespace ll
#endif
