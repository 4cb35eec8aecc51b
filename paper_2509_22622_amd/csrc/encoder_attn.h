// Attention to an encoder's states (include/longlive.h, ll_encoder_attn*): the integer rules that the kernels and the host follow alike (plain C++,
// checked on the host by tests/check_encoder_rules.cpp), and the launches.
#pragma once

#include <cstdint>

#include "paged.h"

namespace ll {

constexpr int ENC_MAX_SEQS = 1 << 20, ENC_MAX_ROWS = 1 << 24, ENC_MAX_HEADS = 1024, ENC_MAX_STRIDE = 1 << 21;
constexpr int64_t ENC_MAX_GROUPS = (1 << 24) - 1;      // workgroups of 256 threads of a launch: below 2^32 threads
constexpr int ENC_ROWS = 128, ENC_FEW_ROWS = 32;       // query rows of a tile; of a tile of few rows
constexpr int ENC_KEYS = 32, ENC_FEW_KEYS = 128;       // keys of a step; of a step of few rows (32 a wave)
constexpr int ENC_MAX_SPLITS = 512;
constexpr int ENC_COLS = 128, ENC_BLOCK = 32;          // keys of a dK/dV tile; query rows of its steps

// The rows of one sequence among a tensor's `total`: begin .. begin + n - 1 are seen, begin + n .. end - 1 are its padding.
struct EncSpan { int begin, n, end; };
LL_PAGED_RULE EncSpan enc_span(const int* cu, const int* lens, int seq, int n_seqs, int total, int most) {
    EncSpan s;
    if (cu) {
        const int b = cu[seq], e = cu[seq + 1];
        s.begin = b < 0 ? 0 : b > total ? total : b;
        s.end = e < s.begin ? s.begin : e > total ? total : e;
    } else {
        const int each = total / n_seqs;
        s.begin = seq * each;
        s.end = s.begin + each;
    }
    s.n = s.end - s.begin;
    if (lens) {
        const int l = lens[seq];
        s.n = l < 0 ? 0 : l < s.n ? l : s.n;
    }
    if (s.n > most) s.n = most;
    return s;
}

// How a call's work is dealt to workgroups.  A unit is a tile of one sequence and kv head; its steps go to `splits` workgroups in equal runs.
struct EncPlan {
    int few;                    // forward: tiles of few rows, whose keys go to the waves
    int tiles, splits, each;    // forward; each: of a unit's tiles to each XCD, 0: all to one
    int q_tiles, q_splits, q_each;      // dQ
    int k_tiles, k_splits, k_each;      // dK/dV
};
// The number of runs: for 1 to 8 workgroups a CU, the time by the CU that has most of them, in steps of a workgroup that shares its CU with another.  A workgroup costs `fixed` steps around
// its own, and where its results are partial each step is `more` and `extra` steps write them and add them up; one by itself on its CU is 0.6 of two.
// The same costs for both head sizes, and as if two workgroups shared a CU (the forward pass of 64 features has three).  Fitted by eye to measurements of 8 and 12 heads, us for so many runs (the rule's in brackets; the backward passes dQ and dK/dV one after the other):
//   forward    12 heads x 4096 x 4096: [1] 130, 2 136, 4 145;  8 x 1000 x 1000: 1 24, 3 21, [4] 21.5, 8 28;  8 x 300 x 2000: 1 41, 4 21, 8 19.6, [10] 21.6, 16 24
//   backward   the same, dQ in so many: [1] 401, 2 507;  1 63, [4] 62, 8 74;  1 78, 4 60, [7] 54, 16 61
//   and dK/dV  12 heads x 4096 x 4096: 1 412, [2] 401;  8 x 1000 x 1000: 1 77, [4] 62;  12 x 32760 x 512: 1 1229, 5 469, [10] 441, 16 451;  x 4096: 1 2809, [2] 2626, 5 2695
struct EncCost { double fixed, more, extra; };
inline int enc_splits(int64_t units, int64_t steps, int least, EncCost c) {
    int best = 1;
    double time = 0;
    for (int k = 0; k <= 8; ++k) {
        int64_t s = k == 0 ? 1 : 256 * k / units;
        if (s > steps / least) s = steps / least;
        if (s > ENC_MAX_SPLITS) s = ENC_MAX_SPLITS;
        if (s < 1 || (k > 0 && s == 1)) continue;
        const double each = double((steps + s - 1) / s) * (s > 1 ? c.more : 1) + c.fixed + (s > 1 ? c.extra : 0);
        const int64_t on = (units * s + 255) / 256;
        const double t = (on == 1 ? 0.6 : 0.5 * double(on)) * each + (s > 1 ? 4 : 0);
        if (k == 0 || t < time) {
            time = t;
            best = int(s);
        }
    }
    return best;
}
inline EncPlan enc_plan(int n_seqs, int q_heads, int kv_heads, int64_t max_q, int64_t max_k) {
    EncPlan p;
    const int group = q_heads / kv_heads;
    const int64_t rows = group * max_q, heads = int64_t(n_seqs) * kv_heads;
    p.few = rows <= ENC_FEW_ROWS;
    p.tiles = p.q_tiles = int((rows + ENC_ROWS - 1) / ENC_ROWS);
    const int64_t key_steps = (max_k + ENC_KEYS - 1) / ENC_KEYS, few_steps = (max_k + ENC_FEW_KEYS - 1) / ENC_FEW_KEYS;
    if (p.few) {                        // bound by memory, which a workgroup a CU keeps busy (24 tokens over up to 1500 states, 32 / 8 heads: 21 us, in 384 workgroups and joined 25)
        const int64_t s = heads < 256 ? 256 / heads : 1;
        p.splits = int(s < few_steps ? s : few_steps);
    } else {
        p.splits = enc_splits(heads * p.tiles, key_steps, 4, EncCost{6, 1, 17});
    }
    p.each = p.tiles >= 8 ? (p.tiles + 7) / 8 : 0;
    p.q_each = p.q_tiles >= 8 ? (p.q_tiles + 7) / 8 : 0;
    p.q_splits = enc_splits(heads * p.q_tiles, key_steps, 8, EncCost{6, 1.6, 8});
    p.k_tiles = int((max_k + ENC_COLS - 1) / ENC_COLS);
    p.k_splits = enc_splits(heads * p.k_tiles, group * ((max_q + ENC_BLOCK - 1) / ENC_BLOCK), 4, EncCost{6, 1, 14});
    p.k_each = heads * p.k_splits < 32 && p.k_tiles >= 8 ? (p.k_tiles + 7) / 8 : 0;
    return p;
}
// How the backward pass is launched.  Small: dQ and dK/dV in one launch, where a sequence and kv head is one tile of each.  Together: delta first, then both side by side, where either has
// no more workgroups than a CU each.  Otherwise dQ, then dK/dV; dQ begins with delta from the forward pass's output and may sweep a tile again, but for sequences of up to ENC_DELTA_FIRST keys,
// and but for dQ in runs, whose delta comes first.
constexpr int ENC_TOGETHER = 256, ENC_DELTA_FIRST = 256;
enum EncWay { ENC_WAY_SMALL, ENC_WAY_TOGETHER, ENC_WAY_IN_TURN };
inline EncWay enc_backward_way(const EncPlan& p, int64_t heads, int n_q, int n_k) {
    if (n_q <= 0 || n_k <= 0) return ENC_WAY_IN_TURN;
    if (p.q_tiles == 1 && p.k_tiles == 1 && p.q_splits == 1 && p.k_splits == 1) return ENC_WAY_SMALL;
    return heads * p.q_tiles * p.q_splits <= ENC_TOGETHER && heads * p.k_tiles * p.k_splits <= ENC_TOGETHER ? ENC_WAY_TOGETHER : ENC_WAY_IN_TURN;
}
// The steps first .. end - 1 of split `i`.
LL_PAGED_RULE void enc_run(int steps, int splits, int i, int& first, int& end) {
    const int each = (steps + splits - 1) / splits;
    first = i * each;
    end = first + each < steps ? first + each : steps;
}

// Numbers (fp32) of the partial results.
inline int64_t enc_forward_numbers(const EncPlan& p, int64_t heads, int D) {
    return p.splits > 1 ? heads * p.tiles * p.splits * (p.few ? ENC_FEW_ROWS : ENC_ROWS) * (D + 2) : 0;
}
inline int64_t enc_dq_numbers(const EncPlan& p, int64_t heads, int D) { return p.q_splits > 1 ? heads * p.q_tiles * p.q_splits * ENC_ROWS * (D + 1) : 0; }
inline int64_t enc_dkv_numbers(const EncPlan& p, int64_t heads, int D) { return p.k_splits > 1 ? heads * p.k_tiles * p.k_splits * ENC_COLS * D * 2 : 0; }

}  // namespace ll

#if defined(__HIPCC__)
#include <hip/hip_runtime.h>

namespace ll {

struct EncParams {
    const uint16_t *q, *k, *v, *dout;
    const uint16_t* o;                       // backward: the forward's output
    uint16_t *out, *dq, *dk, *dv;
    int64_t q_stride, k_stride, v_stride, out_stride, dout_stride, dq_stride, dk_stride, dv_stride;
    const int *cu_q, *cu_k, *k_lens;
    float* lse;                              // [q_heads][n_q]; null where not wanted
    float* side;                             // [q_heads][n_q][2]: lse in log2 units and delta, from the dQ kernel to the dK/dV kernel
    float *part, *part_ms;                   // forward: [unit][split][row][D], [unit][split][row][2]
    float *part_q, *part_d;                  // dQ: [unit][split][row][D], [unit][split][row]
    float* part_kv;                          // dK/dV: [unit][split][2][key][D]
    int n_seqs, n_q, n_k, max_q, max_k, q_heads, kv_heads, D;
    float scale, scale_log2;                 // of the scores; times log2(e)
    EncPlan plan;
    PagedDiv by_group, by_kv_heads;
};
hipError_t launch_encoder_forward(const EncParams& p, hipStream_t s);
hipError_t launch_encoder_backward(const EncParams& p, hipStream_t s);

}  // namespace ll
#endif
