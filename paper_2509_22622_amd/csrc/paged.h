// The paged cache: a pool of pages that many sequences share (include/longlive.h, ll_paged_*).  Layout, the integer rules that the
// kernels and the host follow alike (plain C++, checked on the host by tests/check_paged_rules.cpp), and the launches.
//
// Layout.  Pool [layer][page][kv head][K | V][granule], a granule being 16 consecutive tokens of one head, D * 16 numbers, stored as the
// register images of the 16x16x32 MFMA's first operand so that a wave's 16-byte loads are contiguous 1 KB pieces that need no
// exchange between lanes (lane = 16 g + r):
//   bf16  K [D/32][64 lanes][8]      lane (g, r) of piece c: token r,            features 32 c + 8 g + 0..7
//         V [D/32][64 lanes][2][4]   lane (g, r) of piece c: tokens 4 g + 0..3,  features 32 c + r and 32 c + 16 + r
//   E4M3  K [D/64][64 lanes][2][8]   lane (g, r) of piece c: token r,            features 64 c + 8 g + 0..7 and 64 c + 32 + 8 g + 0..7
//         V [D/64][64 lanes][4][4]   lane (g, r) of piece c: tokens 4 g + 0..3,  features 64 c + 16 i + r, i = 0..3
// Granules of 16 and not blocks of 32 as in the ring caches: a page may then be 16 tokens, and two granules from any two pages make up
// the 32 keys of one MFMA of the second product, because S^T = K q^T leaves lane (g, n) with the scores of keys 4 g + 0..3 of each
// granule for query n, which is the order in which V's lane (g, r) holds them.
#pragma once

#include <cstdint>

#if defined(__HIPCC__)
#define LL_PAGED_RULE __host__ __device__ inline
#else
#define LL_PAGED_RULE inline
#endif

namespace ll {

constexpr int PAGED_GRANULE = 16;              // tokens
constexpr int PAGED_MAX_NEW = 1 << 16;         // query tokens of one sequence in one attention call
constexpr int64_t PAGED_MAX_KEYS = 1 << 30;    // tokens a page table's row may name
constexpr int64_t PAGED_MAX_GROUPS = (1 << 24) - 1;    // workgroups of 256 threads of a launch: below 2^32 threads
constexpr int PAGED_WAVES = 4;                 // waves of an attention workgroup, each with keys of its own

LL_PAGED_RULE int paged_number_bytes(int fmt) { return fmt == 0 ? 2 : 1; }
LL_PAGED_RULE int64_t paged_page_bytes(int kv_heads, int page_tokens, int D, int fmt) {
    return int64_t(kv_heads) * 2 * page_tokens * D * paged_number_bytes(fmt);
}

// Where a number of a granule lies, in numbers from the granule's K or V image (`token` 0..15, `d` 0..D-1).
LL_PAGED_RULE int paged_k_at(int fmt, int token, int d) {
    if (fmt == 0) return (d / 32) * 512 + ((d / 8 % 4) * 16 + token) * 8 + d % 8;
    return (d / 64) * 1024 + ((d / 8 % 4) * 16 + token) * 16 + (d / 32 % 2) * 8 + d % 8;
}
LL_PAGED_RULE int paged_v_at(int fmt, int token, int d) {
    if (fmt == 0) return (d / 32) * 512 + ((token / 4) * 16 + d % 16) * 8 + (d / 16 % 2) * 4 + token % 4;
    return (d / 64) * 1024 + ((token / 4) * 16 + d % 16) * 16 + (d / 16 % 4) * 4 + token % 4;
}

// Division of n < 2^31 by a d that a launch knows, without a divide: with 2^s >= d and m = floor(2^(31 + s) / d) + 1 the product n m is too large by
// less than 2^(31 + s) / d, so that its quotient is exact.
struct PagedDiv {
    uint32_t d, m, shift;
    LL_PAGED_RULE uint32_t of(uint32_t n) const { return uint32_t(uint64_t(n) * m >> shift); }
};
inline PagedDiv paged_div(int64_t d) {
    uint32_t s = 0;
    while ((int64_t(1) << s) < d) ++s;
    return PagedDiv{uint32_t(d), uint32_t((uint64_t(1) << (31 + s)) / uint64_t(d) + 1), 31 + s};
}

// The batch of a call: device arrays, read by the kernels only.  Nothing in them can lead a kernel out of bounds: lengths, offsets and
// pages out of range make a token or a key absent.
struct PagedSeqs {
    const int* lens;            // [n_seqs] tokens of each sequence, the call's own included
    const int* cu;              // [n_seqs + 1] first row of each sequence among the call's rows; null: row i is sequence i's only one
    const int* table;           // [n_seqs][cols], rows table_stride apart: pages
    int64_t table_stride;
    int cols, n_seqs, n_tokens;
    int page_tokens, n_pages;
    PagedDiv by_page;           // page_tokens
};

// Keys a query at position `i` sees: j <= i, and with a window those of the sink or of the last `window` positions.
LL_PAGED_RULE bool paged_sees(int64_t i, int64_t j, int sink, int window) {
    return j <= i && (window == 0 || j < sink || j > i - window);
}

// The key steps of one row tile.  The tile's queries lie at positions i_lo..i_hi; `keys` is how many keys are stored at all.  Steps of
// `step` keys cover the union of their key sets: sink_steps steps from key 0, then steps from first_step on.
struct PagedSteps {
    int total, sink_steps, first_step;
    LL_PAGED_RULE int at(int v) const { return v < sink_steps ? v : v - sink_steps + first_step; }   // the step of visit v
};
LL_PAGED_RULE PagedSteps paged_steps(int64_t i_lo, int64_t i_hi, int64_t keys, int sink, int window, int step) {
    PagedSteps s;
    s.total = s.sink_steps = s.first_step = 0;
    const int64_t end = i_hi + 1 < keys ? i_hi + 1 : keys;
    if (end <= 0) return s;
    if (window != 0) {
        const int64_t sink_end = sink < end ? sink : end;
        s.sink_steps = int((sink_end + step - 1) / step);
        const int64_t begin = i_lo - window + 1;
        s.first_step = begin > 0 ? int(begin / step) : 0;
        if (s.first_step < s.sink_steps) s.first_step = s.sink_steps;
    }
    const int rest = int((end + step - 1) / step) - s.first_step;
    s.total = s.sink_steps + (rest > 0 ? rest : 0);
    return s;
}

// A tile's steps are dealt to the call's `splits` workgroups in runs: `chunk` steps each, or more where the sequence is longer than the
// call was sized for.  A workgroup's run is dealt to its waves likewise.
LL_PAGED_RULE int paged_run(int total, int chunk, int splits) {
    const int even = (total + splits - 1) / splits;
    return even > chunk ? even : chunk;
}

// Keys of one step of a wave: 32 at head_dim 128, 64 at 64; 8 KB of K and as much of V in bfloat16, half of that in 8 bits.
LL_PAGED_RULE int paged_step_keys(int D) { return 4096 / D; }

// Rows of one sequence and kv head: its query heads that share the kv head, for each of its query tokens; tiles of 16.
LL_PAGED_RULE int paged_row_tiles(int group, int max_new) { return (group * max_new + 15) / 16; }

// Rows of the append's tiles, `most` at most: eight at least (whole quads of a granule), and so few only while that brings the launch no more than
// a workgroup or two a CU.  What a tile of a decoding step takes longest for is its values, which go out number by number: 96 rows of 24 units in 8 bits
// 7.6 us in tiles of 32, 5.4 in tiles of 8.
inline int paged_tile_rows(int tokens, int units, int most) {
    int rows = most;
    while (rows > 8 && (int64_t(tokens) + rows / 2 - 1) / (rows / 2) * units <= 512) rows /= 2;
    return rows;
}

// Units (a kv head's K and V, or two query heads) that a workgroup of the append takes, of a tile's `units`: as few as keep the launch in one round of
// the 1024 workgroups that fit the chip at once, and where even whole tiles fill it more than half, as many rounds as make the last one small.  us for
// 391 tiles of 24 units: 12 each (782 workgroups) 77, 8 each (1173) 95, 6 each 84, 2 each 79; for 147 tiles of 18 in 8 bits: 3 each (882) 22, 6 each 24, 2
// each 26, 1 each 31.
inline int paged_units_per_group(int tiles, int units) {
    const int groups = tiles <= 512 ? 1024 / tiles : (4096 + tiles - 1) / tiles;
    return groups >= units ? 1 : (units + groups - 1) / groups;
}

// How a call's keys are dealt out: a workgroup takes `chunk` steps, a tile `splits` of them, for `units` row tiles of at most `steps` steps each.
// One workgroup takes in keys about as fast as a CU can (60 GB/s; 0.27 us a step in bfloat16 at head_dim 128), so one a CU is what few tiles are dealt
// out to, in runs of six steps at least, and only where that takes 24 steps off the walk: the partial results' way through memory and the join cost
// 4 us and more.  us with 1 and with the splits taken: 8 tiles of 4096 steps 1114 and 100 (32), of 128 steps 27 and 13 (21); 1 tile of 1024 steps 165 and
// 16 (64; 170 would take 20); 128 tiles of 128 steps 51 and 42 (2); of 32 steps 13.7 and not the 17.2 of 2.
// From a third of the CUs on the tiles end unevenly, all the more where they are equally long, or leave CUs with one workgroup where two run side by side:
// there long keys go in five runs, or three.  Unequal tiles, us with what the rule above gives and with five: 88 of 450 steps, 8 bits, 53 and 45; 136
// of 250 88 and 72; 208 of 450 194 and 176; 256 of 1000 494 and 468; 320 of 94 72 and 61; but 160 of 150 44 and not the 48 of 5, 448 of 80 42 and not
// 47.  288 equal tiles of 587 steps 588 and 487; 512 of up to 512 steps 502 and 477; 1536 of 94 steps 270 and not the 277 of 3.
struct PagedPlan { int chunk, splits; };
constexpr int PAGED_CUS = 256, PAGED_MAX_SPLITS = 256;
inline PagedPlan paged_plan(int64_t units, int64_t steps) {
    if (steps < 1) steps = 1;
    int64_t splits = 1;
    if (units > PAGED_CUS / 3 && units <= 2 * PAGED_CUS && steps >= (units <= PAGED_CUS ? 200 : units <= PAGED_CUS * 3 / 2 ? 80 : 96)) {
        splits = 5;
    } else if (units <= PAGED_CUS) {
        const int64_t most = steps / 16 > 64 ? steps / 16 : 64;
        splits = PAGED_CUS / units;
        if (splits > steps / 6) splits = steps / 6;
        if (splits > most) splits = most;
        if (splits < 1 || steps - (steps + splits - 1) / splits < 24) splits = 1;
    } else if (units > 2 * PAGED_CUS && units <= 8 * PAGED_CUS && steps >= 256) {
        splits = 3;
    }
    const int64_t chunk = (steps + splits - 1) / splits;
    return PagedPlan{int(chunk), int((steps + chunk - 1) / chunk)};
}
// Most steps of a tile whose sequence has at most max_len tokens.
inline int64_t paged_most_steps(int64_t max_len, int max_new, int sink, int window, int step) {
    const int64_t all = (max_len + step - 1) / step;
    if (window == 0) return all;
    const int64_t seen = (int64_t(sink) + step - 1) / step + (int64_t(window) + max_new + step - 1) / step + 1;
    return seen < all ? seen : all;
}

}  // namespace ll

#if defined(__HIPCC__)
#include <hip/hip_runtime.h>

namespace ll {

struct PagedAppendParams {
    PagedSeqs s;
    const uint16_t *q, *k, *v;     // q null: keys and values only
    uint16_t* q_out;
    int64_t q_stride, k_stride, v_stride, q_out_stride;
    char* pool;                    // of the layer
    const int* positions;          // null: a token's place in its sequence
    const double* turns;           // [rope_pairs] revolutions of the full circle per position
    int q_heads, kv_heads, D, fmt;
    int halves;                    // pairs (i, i + rope_pairs) instead of (2 i, 2 i + 1)
    int rope_pairs, axes;          // axes 3: pairs [0, axis1) turn by positions[3 t], [axis1, axis2) by [3 t + 1], the others by [3 t + 2]
    int axis1, axis2;
    float q_scale, k_scale, v_scale;
    int heads_per_group, tile_rows;   // set by the launch
};
hipError_t launch_paged_append(const PagedAppendParams& p, hipStream_t s);

struct PagedAttnParams {
    PagedSeqs s;
    const uint16_t* q;
    uint16_t* out;
    int64_t q_stride, out_stride;
    const char* pool;              // of the layer
    float* partial;                // [tile][split][16 rows][D], then [tile][split][16][2] (reference, sum)
    float* partial_ms;
    int q_heads, kv_heads, D, fmt;
    int max_new, sink, window;
    float k_scale, v_scale;        // 8-bit cache: what a stored key and value are multiplied by
    PagedPlan plan;
    PagedDiv by_group, by_tiles, by_kv_heads, by_splits, by_rows;   // query heads a kv head, row tiles, kv heads, plan.splits, rows of the fullest tile
};
hipError_t launch_paged_attn(const PagedAttnParams& p, hipStream_t s);

}  // namespace ll
#endif
