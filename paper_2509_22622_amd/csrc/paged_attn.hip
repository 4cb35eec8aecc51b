// ll_paged_attn: attention of each sequence's last token, or last few, over its pages (paged.h):
//     out_i = sum_j 2^(q'_i . k_j) v_j / sum_j 2^(q'_i . k_j)   over the keys j that position i sees; no key: 0.
// q' carries log2(e) / sqrt(D) (ll_paged_append).  Every key and value is read once per kv head and used for at most 16 rows (the query heads
// of the group, times the query tokens): bound by memory, 16 rows x 4 flops per number read against some 400 the chip could do.
//
// So the matrix instructions are there to keep the vector unit out of the way, and everything else serves the stream of loads.
//   S^T = K q^T   16x16x32 MFMAs, A = a granule's K piece as it lies in memory, B = the rows' queries, held in registers;
//   softmax       per row, one pass with the running maximum; lane (g, n) holds row n's scores of keys 4 g + 0..3 of each granule;
//   O^T += V^T P  A = the V pieces of two granules as they lie in memory, B = the weights, in the lane that computed them.
// No number crosses lanes but the row maxima, and nothing goes through LDS: each wave streams keys of its own straight into registers,
// 16 KB a step (8 KB of 8-bit numbers), with the next step's on the way.  A workgroup's four waves take consecutive runs of steps and join at the end, in LDS;
// the keys of a tile are dealt to several workgroups where that fills the chip, and a second kernel joins their results.
// 8-bit numbers become bfloat16 in registers (exact: E4M3 has 4 significant bits); queries and weights stay bfloat16.
#include "paged.h"

#include <algorithm>

namespace ll {

typedef __bf16 pg_bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 pg_bf16x2 __attribute__((ext_vector_type(2)));
typedef float pg_f32x4 __attribute__((ext_vector_type(4)));
typedef float pg_f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned pg_u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned pg_u32x2 __attribute__((ext_vector_type(2)));

// What a tile of rows works on, the same for the attention kernel and the one that joins its results.
struct PgTile {
    int seq, head, tile;            // kv head; tile of 16 rows among the sequence's
    int64_t first_row;              // row of the call's q of the sequence's first token
    int n_new, rows;                // query tokens (at most max_new), valid rows of the tile
    int i0;                         // position of the sequence's first query token
    PagedSteps steps;
    int i_lo, i_hi, keys;
};

__device__ __forceinline__ PgTile pg_tile(const PagedAttnParams& p, int unit, int step) {
    PgTile t;
    const int group = p.by_group.d;
    const int heads = p.by_tiles.of(unit);                                // kv heads of the sequences in front
    t.tile = unit - heads * int(p.by_tiles.d);
    t.seq = p.by_kv_heads.of(heads);
    t.head = heads - t.seq * p.kv_heads;
    t.keys = int(int64_t(p.s.cols) * p.s.page_tokens);                    // at most 2^30
    const int len = max(p.s.lens[t.seq], 0);                              // may be more than the table names: places behind it are none
    int64_t n_new = 1;
    t.first_row = t.seq;
    if (p.s.cu) {
        t.first_row = p.s.cu[t.seq];
        n_new = max(int64_t(p.s.cu[t.seq + 1]) - t.first_row, int64_t(0));   // may be more rows than the call has: those there are keep their places
    }
    t.i0 = int(max(len - n_new, int64_t(-PAGED_MAX_KEYS)));               // so far below 0 max_new rows are all in front of the sequence
    t.n_new = int(min(n_new, int64_t(p.max_new)));
    t.rows = min(max(t.n_new * group - 16 * t.tile, 0), 16);
    t.i_lo = t.i0 + int(p.by_group.of(16 * t.tile));
    t.i_hi = t.i0 + int(p.by_group.of(16 * t.tile + max(t.rows, 1) - 1));
    if (t.rows) t.steps = paged_steps(t.i_lo, t.i_hi, t.keys, p.sink, p.window, step);
    else t.steps = PagedSteps{0, 0, 0};
    return t;
}

// Which tile and which of its workgroups a workgroup is.  Workgroup b runs on XCD b % 8, and the row tiles of one sequence and kv head read the same
// keys: they are 8 apart, so that all but the first find them in that XCD's L2.
__device__ __forceinline__ void pg_place(const PagedAttnParams& p, unsigned block, int& unit, int& split) {
    const unsigned tiles = p.by_tiles.d;
    unsigned run = block, tile = 0;                                     // run: (sequence, kv head, split)
    if (tiles > 1) {
        const unsigned runs = unsigned(p.s.n_seqs) * p.kv_heads * p.plan.splits, set = block / (8 * tiles), in = block % (8 * tiles);
        const unsigned wide = min(8u, runs - 8 * set);                  // the last set may be narrower
        tile = in / wide;
        run = 8 * set + in % wide;
    }
    const unsigned of = p.by_splits.of(run);
    unit = int(of * tiles + tile);
    split = int(run - of * p.plan.splits);
}

// Offset of row n of the tile in q or out, in numbers; -1 if there is no such row.
__device__ __forceinline__ int64_t pg_row_at(const PagedAttnParams& p, const PgTile& t, int n, int64_t stride) {
    const int group = p.by_group.d, r = 16 * t.tile + n, token = p.by_group.of(r);
    const int64_t row = t.first_row + token;
    if (n >= t.rows || row < 0 || row >= p.s.n_tokens) return -1;
    return row * stride + (t.head * group + r - token * group) * p.D;
}

// Four features of a row of out.  A row that has seen no key (sum 0) is zeros.
__device__ __forceinline__ void pg_store(const PagedAttnParams& p, int64_t at, pg_f32x4 x, float sum) {
    const float scale = sum == 0.f ? 0.f : p.v_scale / sum;
    const pg_f32x2 lo = {x[0] * scale, x[1] * scale}, hi = {x[2] * scale, x[3] * scale};
    *reinterpret_cast<pg_u32x2*>(p.out + at) = pg_u32x2{__builtin_bit_cast(unsigned, __builtin_convertvector(lo, pg_bf16x2)),
                                                        __builtin_bit_cast(unsigned, __builtin_convertvector(hi, pg_bf16x2))};
}

// Four E4M3 numbers -> bfloat16.
__device__ __forceinline__ pg_u32x2 pg_widen(unsigned w) {
    return pg_u32x2{__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false)),
                    __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true))};
}

__device__ __forceinline__ pg_f32x4 pg_mfma(pg_u32x4 a, pg_u32x4 b, pg_f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(pg_bf16x8, a), __builtin_bit_cast(pg_bf16x8, b), c, 0, 0, 0);
}

// Largest of a row's values over the four lanes that hold them.
__device__ __forceinline__ float pg_row_max(float x) {
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}

template <int D, int FMT>
struct PgShape {
    static constexpr int NB = FMT == 0 ? 2 : 1;
    static constexpr int GP = D * NB / 64;              // 1 KB pieces of a granule's K, and of its V
    static constexpr int GPS = 256 / D;                 // granules of a step
    static constexpr int STEP = GPS * PAGED_GRANULE;    // keys of a step (paged_step_keys)
    static constexpr int PIECES = GP * GPS;             // 1 KB pieces of a step's K, and of its V
    static constexpr int QF = D / 32;                   // 16-byte pieces of a lane's queries
    static constexpr int OB = D / 16;                   // blocks of 16 features of the output
};

// One step's keys and values in registers.
template <int D, int FMT>
struct PgStep {
    pg_u32x4 k[PgShape<D, FMT>::PIECES], v[PgShape<D, FMT>::PIECES];
};

template <int D, int FMT>
__global__ __launch_bounds__(64 * PAGED_WAVES) __attribute__((amdgpu_waves_per_eu(2, 2)))
void ll_paged_attn_kernel(const PagedAttnParams p) {
    using S = PgShape<D, FMT>;
    constexpr int GP = S::GP, GPS = S::GPS, STEP = S::STEP, QF = S::QF, OB = S::OB;
    __shared__ __attribute__((aligned(16))) float o_join[PAGED_WAVES][16][D + 4];
    __shared__ float m_join[PAGED_WAVES][16], l_join[PAGED_WAVES][16];

    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int unit, split;
    pg_place(p, blockIdx.x, unit, split);
    const PgTile t = pg_tile(p, unit, STEP);
    if (t.rows == 0) return;                                            // uniform over the workgroup
    const int run = paged_run(t.steps.total, p.plan.chunk, p.plan.splits);
    const int begin = split * run, end = min(t.steps.total, begin + run);
    if (begin >= end && split != 0) return;
    const int per_wave = (max(end - begin, 0) + PAGED_WAVES - 1) / PAGED_WAVES;
    const int v0 = begin + wave * per_wave, v1 = min(end, v0 + per_wave);

    const int64_t q_at = pg_row_at(p, t, n, p.q_stride);
    pg_u32x4 q[QF];
#pragma unroll
    for (int c = 0; c < QF; ++c) q[c] = q_at < 0 ? pg_u32x4{0, 0, 0, 0} : *reinterpret_cast<const pg_u32x4*>(p.q + q_at + 32 * c + 8 * g);
    const int my_i = t.i0 + int(p.by_group.of(16 * t.tile + n));        // position of row n

    // Pages of the next 64 granules of this wave, one a lane: where the granule begins, -1 if no page holds it.
    const int64_t page_bytes = paged_page_bytes(p.kv_heads, p.s.page_tokens, D, FMT);
    const int64_t v_region = int64_t(p.s.page_tokens) * D * S::NB;
    const char* const pool = p.pool + int64_t(t.head) * 2 * v_region;
    constexpr int BATCH = 64 / GPS;                                     // steps whose pages are looked up at once
    int at_lo = -1, at_hi = -1;
    auto look_up = [&](int v) {
        const int visit = v + lane / GPS;
        int64_t at = -1;
        if (visit < v1) {
            const int64_t key = int64_t(t.steps.at(visit)) * STEP + lane % GPS * PAGED_GRANULE;
            if (key < t.keys) {
                const int col = p.s.by_page.of(uint32_t(key)), in = int(key) - col * p.s.page_tokens;
                const int page = p.s.table[t.seq * p.s.table_stride + col];
                if (page >= 0 && page < p.s.n_pages) at = page * page_bytes + int64_t(in) * (D * S::NB);
            }
        }
        at_lo = int(at);
        at_hi = int(at >> 32);
    };
    // Loads of step v, and which of its granules lie in a page.  A granule without a page is read from the pool's start and masked.
    auto load = [&](int v, PgStep<D, FMT>& s) -> unsigned {
        unsigned there = 0;
        const int from = (v - v0) % BATCH * GPS;
#pragma unroll
        for (int i = 0; i < GPS; ++i) {
            const int lo = __builtin_amdgcn_readlane(at_lo, from + i), hi = __builtin_amdgcn_readlane(at_hi, from + i);
            if (hi >= 0) there |= 1u << i;
            const char* const at = pool + (hi >= 0 ? (int64_t(hi) << 32 | unsigned(lo)) : 0) + lane * 16;
#pragma unroll
            for (int c = 0; c < GP; ++c) {
                s.k[i * GP + c] = *reinterpret_cast<const pg_u32x4*>(at + 1024 * c);
                s.v[i * GP + c] = *reinterpret_cast<const pg_u32x4*>(at + v_region + 1024 * c);
            }
        }
        return there;
    };

    pg_f32x4 o[OB];
#pragma unroll
    for (int b = 0; b < OB; ++b) o[b] = pg_f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;                                       // row n's reference, and this lane's share of its sum

    auto compute = [&](int v, const PgStep<D, FMT>& s, unsigned there) {
        const int key0 = t.steps.at(v) * STEP;
        const bool whole = there == (1u << GPS) - 1 && key0 + STEP - 1 <= t.i_lo &&
                           (p.window == 0 || key0 + STEP <= p.sink || key0 > t.i_hi - p.window);
        float sc[GPS][4];
#pragma unroll
        for (int i = 0; i < GPS; ++i) {
            pg_f32x4 a = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < QF; ++c) {
                if constexpr (FMT == 0) {
                    a = pg_mfma(s.k[i * GP + c], q[c], a);
                } else {
                    const pg_u32x4 w = s.k[i * GP + c / 2];
                    const pg_u32x2 x = pg_widen(w[c % 2 * 2]), y = pg_widen(w[c % 2 * 2 + 1]);
                    a = pg_mfma(pg_u32x4{x[0], x[1], y[0], y[1]}, q[c], a);
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) sc[i][e] = FMT == 0 ? a[e] : a[e] * p.k_scale;
        }
        if (!whole)
#pragma unroll
            for (int i = 0; i < GPS; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (!(there >> i & 1) || !paged_sees(my_i, key0 + PAGED_GRANULE * i + 4 * g + e, p.sink, p.window)) sc[i][e] = -INFINITY;
        float top = sc[0][0];
#pragma unroll
        for (int i = 0; i < GPS; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) top = fmaxf(top, sc[i][e]);
        // A row's reference moves only if one of its scores is 2^8 times above it: the weights are up to 2^8 then instead of 1, which floating point does
        // not mind, and most steps need no largest score over the row's four lanes (two exchanges, each waiting for the one before).
        if (__any(top > m + 8.0f)) {
            const float to = fmaxf(m, pg_row_max(top)), f = to == m ? 1.0f : __builtin_amdgcn_exp2f(m - to);
            m = to;
            l *= f;
#pragma unroll
            for (int b = 0; b < OB; ++b) o[b] *= f;
        }
        const float ref = m == -INFINITY ? 0.f : m;                     // no key so far: the weights are zeros, not NaN
        pg_u32x4 w[GPS / 2];                                            // weights, in the order of V's pieces
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < GPS; ++i) {
            float e[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                e[j] = __builtin_amdgcn_exp2f(sc[i][j] - ref);
                sum[j] += e[j];
            }
            // The weights go to bfloat16 for the product, as in all of the library's attention (up to 2^-8 of each, at random; the sum above keeps them as they are).
            // That moves an output by 0.0016 of its norm, as much as its own rounding to bfloat16 does; 0.0023 both together, in the middle.
            // Weights in two terms would double the second product.
            w[i / 2][i % 2 * 2] = __builtin_bit_cast(unsigned, __builtin_convertvector((pg_f32x2{e[0], e[1]}), pg_bf16x2));
            w[i / 2][i % 2 * 2 + 1] = __builtin_bit_cast(unsigned, __builtin_convertvector((pg_f32x2{e[2], e[3]}), pg_bf16x2));
        }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        // V^T for block b of 16 features and granules 2 i, 2 i + 1
        auto value = [&](int i, int b) {
            pg_u32x2 x, y;
            if constexpr (FMT == 0) {
                const pg_u32x4 a = s.v[2 * i * GP + b / 2], c = s.v[(2 * i + 1) * GP + b / 2];
                x = pg_u32x2{a[b % 2 * 2], a[b % 2 * 2 + 1]};
                y = pg_u32x2{c[b % 2 * 2], c[b % 2 * 2 + 1]};
            } else {
                x = pg_widen(s.v[2 * i * GP + b / 4][b % 4]);
                y = pg_widen(s.v[(2 * i + 1) * GP + b / 4][b % 4]);
            }
            return pg_u32x4{x[0], x[1], y[0], y[1]};
        };
        if (whole) {
#pragma unroll
            for (int i = 0; i < GPS / 2; ++i)
#pragma unroll
                for (int b = 0; b < OB; ++b) o[b] = pg_mfma(value(i, b), w[i], o[b]);
        } else {
            // A key that some row does not see: its value may be anything, and 0 * NaN is no 0.  Values that none of the tile's tokens sees are cleared.
            // If what comes out has only numbers in it, the values that some of them see were numbers too, and 0 times those is 0.
            // (The tokens one by one in every such step: 16 sequences of 60 tokens, 4 of them new, 8.5 us and not 6.7; 4 prompts of 700 tokens 68 and not 52.)
            const bool one = t.i_lo == t.i_hi;
            auto kept = [&](auto sees) {
                unsigned keep[GPS][2];                                  // for the two pairs of this lane's four keys
#pragma unroll
                for (int i = 0; i < GPS; ++i)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int j = key0 + PAGED_GRANULE * i + 4 * g + 2 * e;
                        keep[i][e] = (there >> i & 1) ? (sees(j) ? 0xFFFFu : 0u) | (sees(j + 1) ? 0xFFFF0000u : 0u) : 0u;
                    }
                return [=, &value](int i, int b) {
                    pg_u32x4 x = value(i, b);
                    x[0] &= keep[2 * i][0];
                    x[1] &= keep[2 * i][1];
                    x[2] &= keep[2 * i + 1][0];
                    x[3] &= keep[2 * i + 1][1];
                    return x;
                };
            };
            const int behind = p.window == 0 ? -1 : int(max(int64_t(t.i_lo) - p.window, int64_t(-1)));     // what no window reaches any more
            const auto some = kept([&](int j) { return j <= t.i_hi && (j < p.sink || j > behind); });
            pg_f32x4 a[OB];
            float none = 0.f;
#pragma unroll
            for (int b = 0; b < OB; ++b) {
                a[b] = o[b];
#pragma unroll
                for (int i = 0; i < GPS / 2; ++i) a[b] = pg_mfma(some(i, b), w[i], a[b]);
#pragma unroll
                for (int e = 0; e < 4; ++e) none = __builtin_fmaf(a[b][e], 0.f, none);
            }
            if (!one && __any(none != 0.f))                             // NaN is not 0 either
                // The query tokens one by one: values that a token does not see are cleared, and that token's rows take what comes out.
                for (int i_tok = t.i_lo; i_tok <= t.i_hi; ++i_tok) {
                    const auto own = kept([&](int j) { return paged_sees(i_tok, j, p.sink, p.window); });
#pragma unroll
                    for (int b = 0; b < OB; ++b) {
                        pg_f32x4 x = o[b];
#pragma unroll
                        for (int i = 0; i < GPS / 2; ++i) x = pg_mfma(own(i, b), w[i], x);
                        if (my_i == i_tok) a[b] = x;
                    }
                }
#pragma unroll
            for (int b = 0; b < OB; ++b) o[b] = a[b];
        }
    };

    if (v0 < v1) {
        PgStep<D, FMT> a, b;
        look_up(v0);
        unsigned there_a = load(v0, a), there_b = 0;
        // Two steps a turn, so that neither's registers move; pages are looked up for whole turns.  Past the end the last step is loaded again and not used.
        static_assert(BATCH % 2 == 0, "a batch of pages begins with a turn's first step");
        for (int v = v0; v < v1; v += 2) {
            there_b = load(min(v + 1, v1 - 1), b);
            compute(v, a, there_a);
            if ((v + 2 - v0) % BATCH == 0 && v + 2 < v1) look_up(v + 2);
            there_a = load(min(v + 2, v1 - 1), a);
            if (v + 1 < v1) compute(v + 1, b, there_b);
        }
    }

    // Join the waves: each row's reference is the largest of theirs.
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (g == 0) {
        m_join[wave][n] = m;
        l_join[wave][n] = l;
    }
#pragma unroll
    for (int b = 0; b < OB; ++b) *reinterpret_cast<pg_f32x4*>(&o_join[wave][n][16 * b + 4 * g]) = o[b];
    __syncthreads();
    const bool only = t.steps.total <= run;                             // nothing to join with other workgroups
    constexpr int LANES = D / 4;                                        // threads of a row
    for (int i = threadIdx.x; i < t.rows * LANES; i += 64 * PAGED_WAVES) {
        const int row = i / LANES, part = i % LANES;
        float top = m_join[0][row];
#pragma unroll
        for (int w = 1; w < PAGED_WAVES; ++w) top = fmaxf(top, m_join[w][row]);
        float sum = 0.f;
        pg_f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < PAGED_WAVES; ++w) {
            const float f = m_join[w][row] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_join[w][row] - top);
            sum += l_join[w][row] * f;                                  // a sum that is no number stays none
            if (f != 0.f) x += *reinterpret_cast<const pg_f32x4*>(&o_join[w][row][4 * part]) * f;
        }
        if (only) {
            const int64_t out_at = pg_row_at(p, t, row, p.out_stride);
            if (out_at >= 0) pg_store(p, out_at + 4 * part, x, sum);
        } else {
            const int64_t result = (int64_t(unit) * p.plan.splits + split) * 16 + row;
            *reinterpret_cast<pg_f32x4*>(p.partial + result * D + 4 * part) = x;
            if (part == 0) {
                p.partial_ms[result * 2] = top;
                p.partial_ms[result * 2 + 1] = sum;
            }
        }
    }
}

// What a row's join works on.  False: no such row, or its only workgroup has written it.
struct PgJoin {
    int used;                       // partial results
    int64_t first, out_at;          // row of the first of them (the next ones 16 further each); where the row of out begins
};
__device__ __forceinline__ bool pg_join(const PagedAttnParams& p, unsigned at, int step, PgJoin& j) {
    const int unit = p.by_rows.of(at), row = int(at) - unit * int(p.by_rows.d);
    const PgTile t = pg_tile(p, unit, step);
    const int run = paged_run(t.steps.total, p.plan.chunk, p.plan.splits);
    if (row >= t.rows || t.steps.total <= run) return false;
    j.used = (t.steps.total + run - 1) / run;
    j.first = int64_t(unit) * p.plan.splits * 16 + row;
    j.out_at = pg_row_at(p, t, row, p.out_stride);
    return j.out_at >= 0;
}
// Joins the results of a row's workgroups, in their order.  The weights of the partial results come first, by themselves, so that the loads of the
// results do not wait for one another.  A wave a row, four rows a workgroup; n_rows of them in all.
constexpr int PG_JOIN_FEW = 16;     // partial results up to which a wave does
template <int D>
__global__ __launch_bounds__(256) void ll_paged_join_few_kernel(const PagedAttnParams p, int step, unsigned n_rows) {
    constexpr int LANES = D / 4, SIDE = 64 / LANES;
    const int lane = threadIdx.x & 63;
    const unsigned at = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    PgJoin j;
    if (at >= n_rows || !pg_join(p, at, step, j)) return;
    const float m = lane < j.used ? p.partial_ms[(j.first + lane * 16) * 2] : -INFINITY;
    float sum = lane < j.used ? p.partial_ms[(j.first + lane * 16) * 2 + 1] : 0.f;
    const int part = lane % LANES, side = lane / LANES;
    const float* const from = p.partial + j.first * D + 4 * part;
    float top = m;
#pragma unroll
    for (int x = 1; x < PG_JOIN_FEW; x *= 2) top = fmaxf(top, __shfl_xor(top, x));
    top = __shfl(top, 0);
    const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
    sum *= f;                                                           // a sum that is no number stays none
#pragma unroll
    for (int x = 1; x < PG_JOIN_FEW; x *= 2) sum += __shfl_xor(sum, x);
    sum = __shfl(sum, 0);
    pg_f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = 0; s < j.used; s += SIDE) {
        const int mine = min(s + side, j.used - 1);
        const pg_f32x4 a = *reinterpret_cast<const pg_f32x4*>(from + int64_t(mine) * (16 * D));
        const float w = __shfl(f, s + side);                            // 0 past the end
        if (w != 0.f) x += a * w;
    }
#pragma unroll
    for (int y = LANES; y < 64; y *= 2)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] += __shfl_xor(x[e], y);
    if (side == 0) pg_store(p, j.out_at + 4 * part, x, sum);
}

// The same with a workgroup a row.  Where the partial results are does not depend on the sequence's length: it asks for all that the call has room for and
// takes those that there are, which makes one trip to memory of three.  131072 tokens, 8 bits, 32 query heads: the call 55.4 -> 53.7 us; one sequence of
// 32000 tokens, 8 query heads on one: 16.5 -> 11.4.  (With a wave a row, above, it gains nothing.)
template <int D>
__global__ __launch_bounds__(256) void ll_paged_join_kernel(const PagedAttnParams p, int step) {
    constexpr int LANES = D / 4, SIDE = 256 / LANES, AHEAD = 8;
    static_assert(PAGED_MAX_SPLITS <= 256, "a thread a partial result");
    __shared__ __attribute__((aligned(16))) float o_join[SIDE][D];
    __shared__ float weight[256], wave_top[4], wave_sum[4];
    const int unit = p.by_rows.of(blockIdx.x), row = int(blockIdx.x) - unit * int(p.by_rows.d);
    const int64_t first = int64_t(unit) * p.plan.splits * 16 + row;
    const int tid = threadIdx.x, wave = tid >> 6, part = tid % LANES, side = tid / LANES;
    float m = -INFINITY, sum = 0.f;
    if (tid < p.plan.splits) {
        m = p.partial_ms[(first + tid * 16) * 2];
        sum = p.partial_ms[(first + tid * 16) * 2 + 1];
    }
    const float* const from = p.partial + first * D + 4 * part;
    auto result = [&](int s) { return *reinterpret_cast<const pg_f32x4*>(from + int64_t(min(s, p.plan.splits - 1)) * (16 * D)); };
    pg_f32x4 a[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) a[i] = result(SIDE * i + side);
    PgJoin j;
    if (!pg_join(p, blockIdx.x, step, j)) return;
    if (tid >= j.used) {
        m = -INFINITY;
        sum = 0.f;
    }
    float top = m;
#pragma unroll
    for (int x = 1; x < 64; x *= 2) top = fmaxf(top, __shfl_xor(top, x));
    if ((tid & 63) == 0) wave_top[wave] = top;
    __syncthreads();
    top = fmaxf(fmaxf(wave_top[0], wave_top[1]), fmaxf(wave_top[2], wave_top[3]));
    const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
    weight[tid] = f;
    sum *= f;
#pragma unroll
    for (int x = 1; x < 64; x *= 2) sum += __shfl_xor(sum, x);
    if ((tid & 63) == 0) wave_sum[wave] = sum;
    __syncthreads();
    pg_f32x4 x = {0.f, 0.f, 0.f, 0.f};
    for (int s = side; s < j.used; s += SIDE * AHEAD) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const float w = s + SIDE * i < 256 ? weight[s + SIDE * i] : 0.f;    // 0 where there is no result
            if (w != 0.f) x += a[i] * w;
        }
        if (s + SIDE * AHEAD < j.used)
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) a[i] = result(s + SIDE * (AHEAD + i));
    }
    *reinterpret_cast<pg_f32x4*>(&o_join[side][4 * part]) = x;
    __syncthreads();
    if (side != 0) return;
#pragma unroll
    for (int s = 1; s < SIDE; ++s) x += *reinterpret_cast<const pg_f32x4*>(&o_join[s][4 * part]);
    pg_store(p, j.out_at + 4 * part, x, (wave_sum[0] + wave_sum[1]) + (wave_sum[2] + wave_sum[3]));
}

template <int D, int FMT>
static hipError_t launch(const PagedAttnParams& p, hipStream_t s) {
    const int64_t units = int64_t(p.s.n_seqs) * p.kv_heads * p.by_tiles.d;
    if (units * p.plan.splits > PAGED_MAX_GROUPS || (p.plan.splits > 1 && units * 16 > PAGED_MAX_GROUPS)) return hipErrorInvalidValue;
    static_assert(PgShape<D, FMT>::STEP == 4096 / D, "paged_step_keys");
    hipLaunchKernelGGL((ll_paged_attn_kernel<D, FMT>), dim3(unsigned(units * p.plan.splits)), dim3(64 * PAGED_WAVES), 0, s, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.plan.splits == 1) return e;
    const unsigned rows = unsigned(units * p.by_rows.d);
    if (p.plan.splits <= PG_JOIN_FEW) hipLaunchKernelGGL((ll_paged_join_few_kernel<D>), dim3((rows + 3) / 4), dim3(256), 0, s, p, PgShape<D, FMT>::STEP, rows);
    else hipLaunchKernelGGL((ll_paged_join_kernel<D>), dim3(rows), dim3(256), 0, s, p, PgShape<D, FMT>::STEP);
    return hipGetLastError();
}

hipError_t launch_paged_attn(const PagedAttnParams& p, hipStream_t s) {
    if (p.fmt == 0) return p.D == 128 ? launch<128, 0>(p, s) : launch<64, 0>(p, s);
    return p.D == 128 ? launch<128, 1>(p, s) : launch<64, 1>(p, s);
}

}  // namespace ll
