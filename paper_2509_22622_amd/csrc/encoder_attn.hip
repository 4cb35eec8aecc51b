// Attention to an encoder's states, forward and backward (encoder_attn.h): per sequence and head
//     P = softmax(c q k^T),  O = P v,  lse = log of the row sums;
//     dV = P^T dO,  dP = dO v^T,  delta = rowsum(P dP),  dS = P (dP - delta),  dQ = c dS k,  dK = c dS^T q.
//
// All products are 32x32x16 MFMAs in one formulation: a wave owns 32 columns (query rows, or keys), every lane one column and half of what is contracted, and
// the other side streams past in blocks of 32 rows through LDS, row-major as it lies in memory.
//   A product over features takes the block's rows as A: lane (half, i) reads 16 bytes of row swap23(i), so that accumulator register r of the lane stands for
//   block row 16 (r / 8) + 8 half + r % 8: the order in which the next product's B operand wants its rows, and the weights stay in their lane.
//   A product over the block's rows takes the block transposed as A: ds_read_b64_tr_b16, where 16 lanes read 4 rows x 16 features and each receives one feature's
//   4 rows.
// A block's 16-byte pieces are stored at piece ^ ((row & 3) << 1 | (row >> 3 & 1)): eight lanes of either read then find eight different bank groups.
#include "encoder_attn.h"

#include <algorithm>

namespace ll {

typedef __bf16 ea_bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 ea_bf16x2 __attribute__((ext_vector_type(2)));
typedef float ea_f32x16 __attribute__((ext_vector_type(16)));
typedef float ea_f32x4 __attribute__((ext_vector_type(4)));
typedef float ea_f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned ea_u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned ea_u32x2 __attribute__((ext_vector_type(2)));
typedef short ea_s16x4 __attribute__((ext_vector_type(4)));

constexpr float EA_LN2 = 0.69314718055994530942f, EA_LOG2E = 1.4426950408889634074f;
constexpr float EA_SLACK = 8.f;                  // a row's reference moves where a score is 2^8 times above it

__device__ __forceinline__ unsigned ea_pack(float a, float b) {
    const ea_f32x2 v = {a, b};
    return __builtin_bit_cast(unsigned, __builtin_convertvector(v, ea_bf16x2));
}
__device__ __forceinline__ ea_f32x16 ea_mfma(ea_u32x4 a, ea_u32x4 b, ea_f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(ea_bf16x8, a), __builtin_bit_cast(ea_bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ ea_f32x16 ea_zero() {
    ea_f32x16 z;
#pragma unroll
    for (int r = 0; r < 16; ++r) z[r] = 0.f;
    return z;
}
// The other half's value of the same column.
__device__ __forceinline__ float ea_other(float x, int half) {
    const auto p = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    return __builtin_bit_cast(float, half ? p[0] : p[1]);
}
__device__ __forceinline__ float ea_max2(float x, int half) { return fmaxf(x, ea_other(x, half)); }
__device__ __forceinline__ float ea_sum2(float x, int half) {        // the same order in both halves
    const float y = ea_other(x, half);
    return half ? y + x : x + y;
}

// ---- LDS blocks ---------------------------------------------------------------------------------------------------
// Byte offset of 16-byte piece `c` of row `r`.
template <int D>
__device__ __forceinline__ int ea_at(int r, int c) { return r * (2 * D) + ((c ^ ((r & 3) << 1 | (r >> 3 & 1))) << 4); }

// A operand of a product over features: this lane's row of 32, features 16 ks + 8 half ..
template <int D>
__device__ __forceinline__ ea_u32x4 ea_row_piece(const char* block, int lane, int ks) {
    const int i = lane & 31, r = (i & 0x13) | (i & 4) << 1 | (i & 8) >> 1;
    return *reinterpret_cast<const ea_u32x4*>(block + ea_at<D>(r, 2 * ks + (lane >> 5)));
}
// A operand of a product over rows: this lane's feature 32 db + lane % 32, rows 16 t + 8 half + 0..7.
template <int D>
__device__ __forceinline__ ea_u32x4 ea_col_piece(const char* block, int lane, int t, int db) {
    typedef __attribute__((address_space(3))) ea_s16x4 lds_s16x4;
    const int s = lane & 15, r = 16 * t + 8 * (lane >> 5) + (s >> 2), c = 4 * db + 2 * (lane >> 4 & 1) + (s >> 1 & 1);
    const char* at = block + ea_at<D>(r, c) + 8 * (s & 1);
    const ea_s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at));
    const ea_s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 4 * 2 * D));        // row + 4: the same piece
    const ea_u32x2 a = __builtin_bit_cast(ea_u32x2, lo), b = __builtin_bit_cast(ea_u32x2, hi);
    return ea_u32x4{a[0], a[1], b[0], b[1]};
}

// A thread's pieces of a block of ROWS rows brought by THREADS threads: from memory into registers, from there into LDS.  Rows behind the last are zeros.
template <int D, int ROWS, int THREADS>
struct EaPieces {
    static constexpr int ACROSS = D / 8, STEP = THREADS / ACROSS, N = ROWS / STEP;
    static_assert(ROWS % STEP == 0 && STEP % 4 == 0, "the place of a piece depends on its row");
    ea_u32x4 x[N];
    __device__ __forceinline__ void load(const uint16_t* base, int64_t stride, int rows, int id) {
        const uint16_t* p = base + (id / ACROSS) * stride + (id % ACROSS) * 8;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            x[j] = ea_u32x4{0, 0, 0, 0};
            if (id / ACROSS + j * STEP < rows) x[j] = *reinterpret_cast<const ea_u32x4*>(p + j * STEP * stride);
        }
    }
    __device__ __forceinline__ void store(char* block, int id) const {
#pragma unroll
        for (int j = 0; j < N; ++j) *reinterpret_cast<ea_u32x4*>(block + ea_at<D>(id / ACROSS + j * STEP, id % ACROSS)) = x[j];
    }
};

// Which item of `items` a workgroup takes, or -1: workgroup b runs on XCD b % 8, and an XCD takes neighbouring items, which read the same keys.
__device__ __forceinline__ int64_t ea_item(int64_t items) {
    const int64_t per_xcd = (items + 7) >> 3, i = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    return int64_t(blockIdx.x >> 3) < per_xcd && i < items ? i : -1;
}
static int64_t ea_grid(int64_t items) { return (items + 7) / 8 * 8; }

// A column that is a query row: (token, query head of the kv head's group).
struct EaRow { bool there; int64_t token; int head; };
__device__ __forceinline__ EaRow ea_query_row(const EncParams& p, const EncSpan& q, int kv_head, int r) {
    const int group = p.by_group.d, token = p.by_group.of(r);
    return EaRow{token < q.n, int64_t(q.begin) + token, kv_head * group + (r - token * group)};
}
template <int D>
__device__ __forceinline__ void ea_load_column(ea_u32x4 (&f)[D / 16], const uint16_t* x, int64_t stride, const EaRow& row, int half) {
    const uint16_t* at = x + row.token * stride + row.head * D + half * 8;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
        f[ks] = ea_u32x4{0, 0, 0, 0};
        if (row.there) f[ks] = *reinterpret_cast<const ea_u32x4*>(at + 16 * ks);
    }
}
// Accumulators of a column [feature 32 db + 8 g + 4 half + i] as bfloat16, times `scale`.
template <int D>
__device__ __forceinline__ void ea_store_column(uint16_t* at, const ea_f32x16 (&acc)[D / 32], float scale, int half) {
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *reinterpret_cast<ea_u32x2*>(at + 32 * db + 8 * g + 4 * half) =
                ea_u32x2{ea_pack(acc[db][4 * g] * scale, acc[db][4 * g + 1] * scale), ea_pack(acc[db][4 * g + 2] * scale, acc[db][4 * g + 3] * scale)};
}
template <int D>
__device__ __forceinline__ void ea_store_part(float* at, const ea_f32x16 (&acc)[D / 32], int half) {
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *reinterpret_cast<ea_f32x4*>(at + 32 * db + 8 * g + 4 * half) = ea_f32x4{acc[db][4 * g], acc[db][4 * g + 1], acc[db][4 * g + 2], acc[db][4 * g + 3]};
}

// ---- forward ------------------------------------------------------------------------------------------------------
// The running softmax of a wave's 32 rows over blocks of 32 keys.
template <int D>
struct EaSoftmax {
    ea_f32x16 acc[D / 32];
    float ref, sum;                              // reference in log2 units, the same in both halves; this half's part of the row sum
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int db = 0; db < D / 32; ++db) acc[db] = ea_zero();
        ref = -INFINITY;
        sum = 0.f;
    }
    // NB blocks of 32 keys, of which `keys` are there.
    template <int NB>
    __device__ __forceinline__ void step(const char* k_block, const char* v_block, const ea_u32x4 (&q)[D / 16], int keys, float scale_log2, int lane) {
        const int half = lane >> 5;
        ea_f32x16 s[NB];
        float top = -INFINITY;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            s[b] = ea_zero();
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) s[b] = ea_mfma(ea_row_piece<D>(k_block + b * 64 * D, lane, ks), q[ks], s[b]);
        }
        if (keys < 32 * NB) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (32 * b + 16 * (r >> 3) + 8 * half + (r & 7) >= keys) s[b][r] = -INFINITY;
        }
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, s[b][r]);
        top = ea_max2(top, half) * scale_log2;
        if (__any(top > ref + EA_SLACK)) {
            const float next = fmaxf(ref, top), down = next == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ref - next);
            ref = next;
            sum *= down;
#pragma unroll
            for (int db = 0; db < D / 32; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[db][r] *= down;
        }
        const float from = ref == -INFINITY ? 0.f : ref;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                float w[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    w[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][8 * t + e], scale_log2, -from));
                    sum += w[e];
                }
                const ea_u32x4 pw = {ea_pack(w[0], w[1]), ea_pack(w[2], w[3]), ea_pack(w[4], w[5]), ea_pack(w[6], w[7])};
#pragma unroll
                for (int db = 0; db < D / 32; ++db) acc[db] = ea_mfma(ea_col_piece<D>(v_block + b * 64 * D, lane, t, db), pw, acc[db]);
            }
    }
};

template <int D>
__device__ __forceinline__ void ea_finish_row(const EncParams& p, const EaRow& row, const ea_f32x16 (&acc)[D / 32], float ref, float sum, int half) {
    if (!row.there) return;
    ea_store_column<D>(p.out + row.token * p.out_stride + row.head * D, acc, sum == 0.f ? 0.f : 1.f / sum, half);
    if (p.lse && half == 0) p.lse[int64_t(row.head) * p.n_q + row.token] = sum == 0.f ? -INFINITY : (ref + __builtin_amdgcn_logf(sum)) * EA_LN2;
}

struct EaForwardItem { int64_t unit; int tile, split, seq, head; };
__device__ __forceinline__ EaForwardItem ea_forward_item(int64_t item, int tiles, int splits, const PagedDiv& by_heads) {
    EaForwardItem i;                                                  // neighbours: the tiles of one run of keys
    const unsigned per = unsigned(tiles) * splits, of = unsigned(item) / per, in = unsigned(item) - of * per;
    i.split = in / tiles;
    i.tile = in - i.split * tiles;
    i.seq = by_heads.of(of);
    i.head = of - i.seq * by_heads.d;
    i.unit = int64_t(of) * tiles + i.tile;
    return i;
}

// 128 query rows, 32 a wave; steps of 64 keys, which the workgroup brings together and every wave reads.
template <int D>
__global__ __launch_bounds__(256, 2) void ll_encoder_forward_kernel(const EncParams p) {
    constexpr int BLOCK = ENC_KEYS * D * 2;
    __shared__ __attribute__((aligned(16))) char lds[2][2][BLOCK];    // [stage][K, V]
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
    const int64_t at = ea_item(int64_t(p.n_seqs) * p.kv_heads * p.plan.tiles * p.plan.splits);
    if (at < 0) return;
    const EaForwardItem it = ea_forward_item(at, p.plan.tiles, p.plan.splits, p.by_kv_heads);
    const EncSpan qs = enc_span(p.cu_q, nullptr, it.seq, p.n_seqs, p.n_q, p.max_q), ks = enc_span(p.cu_k, p.k_lens, it.seq, p.n_seqs, p.n_k, p.max_k);
    if (int64_t(it.tile) * ENC_ROWS >= int64_t(qs.n) * p.by_group.d) return;
    const EaRow row = ea_query_row(p, qs, it.head, it.tile * ENC_ROWS + wave * 32 + (lane & 31));
    ea_u32x4 q[D / 16];
    ea_load_column<D>(q, p.q, p.q_stride, row, half);
    int step, end;
    enc_run((ks.n + ENC_KEYS - 1) / ENC_KEYS, p.plan.splits, it.split, step, end);
    EaSoftmax<D> sm;
    sm.clear();
    EaPieces<D, ENC_KEYS, 256> kp, vp;
    const auto load = [&](int s) {
        const int64_t first = int64_t(ks.begin) + s * ENC_KEYS;
        kp.load(p.k + first * p.k_stride + it.head * D, p.k_stride, ks.n - s * ENC_KEYS, tid);
        vp.load(p.v + first * p.v_stride + it.head * D, p.v_stride, ks.n - s * ENC_KEYS, tid);
    };
    if (step < end) load(step);
    for (int stage = 0; step < end; ++step, stage ^= 1) {
        kp.store(lds[stage][0], tid);
        vp.store(lds[stage][1], tid);
        __syncthreads();                                              // the other stage was read in front of the barrier before this one
        if (step + 1 < end) load(step + 1);
        sm.template step<2>(lds[stage][0], lds[stage][1], q, ks.n - step * ENC_KEYS, p.scale_log2, lane);
    }
    const float sum = ea_sum2(sm.sum, half);
    if (p.plan.splits == 1) {
        ea_finish_row<D>(p, row, sm.acc, sm.ref, sum, half);
    } else if (row.there) {
        const int64_t r = (it.unit * p.plan.splits + it.split) * ENC_ROWS + wave * 32 + (lane & 31);
        ea_store_part<D>(p.part + r * D, sm.acc, half);
        if (half == 0) *reinterpret_cast<ea_f32x2*>(p.part_ms + 2 * r) = ea_f32x2{sm.ref, sum};
    }
}

// Up to 32 query rows; steps of 128 keys, 32 of them each wave's own: nothing is shared until the waves join.
template <int D>
__global__ __launch_bounds__(256, 2) void ll_encoder_few_kernel(const EncParams p) {
    constexpr int BLOCK = 32 * D * 2, JOIN = 32 * (D + 4);           // bytes; floats of a wave's results
    constexpr int BYTES = 4 * 2 * BLOCK > 4 * JOIN * 4 ? 4 * 2 * BLOCK : 4 * JOIN * 4;
    __shared__ __attribute__((aligned(16))) char lds[BYTES];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5, col = lane & 31;
    const int64_t at = ea_item(int64_t(p.n_seqs) * p.kv_heads * p.plan.tiles * p.plan.splits);
    if (at < 0) return;
    const EaForwardItem it = ea_forward_item(at, p.plan.tiles, p.plan.splits, p.by_kv_heads);
    const EncSpan qs = enc_span(p.cu_q, nullptr, it.seq, p.n_seqs, p.n_q, p.max_q), ks = enc_span(p.cu_k, p.k_lens, it.seq, p.n_seqs, p.n_k, p.max_k);
    if (int64_t(it.tile) * ENC_FEW_ROWS >= int64_t(qs.n) * p.by_group.d) return;
    const EaRow row = ea_query_row(p, qs, it.head, it.tile * ENC_FEW_ROWS + col);
    int step, end;
    enc_run((ks.n + ENC_FEW_KEYS - 1) / ENC_FEW_KEYS, p.plan.splits, it.split, step, end);
    EaSoftmax<D> sm;
    sm.clear();
    EaPieces<D, 32, 64> kp, vp;
    const auto load = [&](int s) {
        const int first = s * ENC_FEW_KEYS + wave * 32, left = ks.n - first;
        kp.load(p.k + (int64_t(ks.begin) + first) * p.k_stride + it.head * D, p.k_stride, left, lane);
        vp.load(p.v + (int64_t(ks.begin) + first) * p.v_stride + it.head * D, p.v_stride, left, lane);
    };
    if (step < end) load(step);
    ea_u32x4 q[D / 16];
    ea_load_column<D>(q, p.q, p.q_stride, row, half);
    char* const k_block = lds + wave * 2 * BLOCK;
    for (; step < end; ++step) {
        __builtin_amdgcn_wave_barrier();
        kp.store(k_block, lane);
        vp.store(k_block + BLOCK, lane);
        if (step + 1 < end) load(step + 1);
        const int left = ks.n - step * ENC_FEW_KEYS - wave * 32;
        __builtin_amdgcn_wave_barrier();
        if (left > 0) sm.template step<1>(k_block, k_block + BLOCK, q, left, p.scale_log2, lane);
    }
    // the four waves' results meet in LDS: wave w adds up features D / 4 w ..
    const float sum = ea_sum2(sm.sum, half);
    __syncthreads();
    float* const mine = reinterpret_cast<float*>(lds) + wave * JOIN + col * (D + 4);
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *reinterpret_cast<ea_f32x4*>(mine + 32 * db + 8 * g + 4 * half) = ea_f32x4{sm.acc[db][4 * g], sm.acc[db][4 * g + 1], sm.acc[db][4 * g + 2], sm.acc[db][4 * g + 3]};
    if (half == 0) *reinterpret_cast<ea_f32x2*>(mine + D) = ea_f32x2{sm.ref, sum};
    __syncthreads();
    const float* const rows = reinterpret_cast<const float*>(lds) + col * (D + 4);
    float ref = -INFINITY, total = 0.f, w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) ref = fmaxf(ref, rows[i * JOIN + D]);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float r = rows[i * JOIN + D];
        w[i] = r == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(r - ref);
        total += rows[i * JOIN + D + 1] * w[i];
    }
    if (!row.there) return;
    const int from = wave * (D / 4) + half * (D / 8);                 // this lane's D / 8 features
    float x[D / 8];
#pragma unroll
    for (int f = 0; f < D / 8; f += 4) {
        ea_f32x4 a = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const ea_f32x4 y = *reinterpret_cast<const ea_f32x4*>(rows + i * JOIN + from + f);
#pragma unroll
            for (int j = 0; j < 4; ++j) a[j] += y[j] * w[i];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) x[f + j] = a[j];
    }
    if (p.plan.splits == 1) {
        const float scale = total == 0.f ? 0.f : 1.f / total;
        uint16_t* o = p.out + row.token * p.out_stride + row.head * D + from;
#pragma unroll
        for (int f = 0; f < D / 8; f += 8)
            *reinterpret_cast<ea_u32x4*>(o + f) = ea_u32x4{ea_pack(x[f] * scale, x[f + 1] * scale), ea_pack(x[f + 2] * scale, x[f + 3] * scale),
                                                           ea_pack(x[f + 4] * scale, x[f + 5] * scale), ea_pack(x[f + 6] * scale, x[f + 7] * scale)};
        if (p.lse && tid < 32) p.lse[int64_t(row.head) * p.n_q + row.token] = total == 0.f ? -INFINITY : (ref + __builtin_amdgcn_logf(total)) * EA_LN2;
    } else {
        const int64_t r = (it.unit * p.plan.splits + it.split) * ENC_FEW_ROWS + col;
#pragma unroll
        for (int f = 0; f < D / 8; f += 4) *reinterpret_cast<ea_f32x4*>(p.part + r * D + from + f) = ea_f32x4{x[f], x[f + 1], x[f + 2], x[f + 3]};
        if (tid < 32) *reinterpret_cast<ea_f32x2*>(p.part_ms + 2 * r) = ea_f32x2{ref, total};
    }
}

// Joins the splits of a row: one wave a row, D / 64 features a lane.
template <int D>
__global__ __launch_bounds__(256) void ll_encoder_join_kernel(const EncParams p) {
    const int tile_rows = p.plan.few ? ENC_FEW_ROWS : ENC_ROWS, lane = threadIdx.x & 63;
    const int64_t at = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
    const unsigned unit = unsigned(at / tile_rows), in = unsigned(at % tile_rows), of = unit / unsigned(p.plan.tiles);
    const int tile = int(unit - of * p.plan.tiles), seq = p.by_kv_heads.of(of), head = of - seq * p.kv_heads;
    if (seq >= p.n_seqs) return;
    const EncSpan qs = enc_span(p.cu_q, nullptr, seq, p.n_seqs, p.n_q, p.max_q);
    const int64_t r = int64_t(tile) * tile_rows + in;
    if (r >= int64_t(qs.n) * p.by_group.d) return;
    const EaRow row = ea_query_row(p, qs, head, int(r));
    const int splits = p.plan.splits;
    const int64_t first = int64_t(unit) * splits * tile_rows + in;
    float ref = -INFINITY;
    for (int s = lane; s < splits; s += 64) ref = fmaxf(ref, p.part_ms[2 * (first + int64_t(s) * tile_rows)]);
#pragma unroll
    for (int d = 32; d; d >>= 1) ref = fmaxf(ref, __shfl_xor(ref, d));
    float total = 0.f, x[D / 64] = {};
    for (int s = 0; s < splits; ++s) {
        const int64_t i = first + int64_t(s) * tile_rows;
        const ea_f32x2 ms = *reinterpret_cast<const ea_f32x2*>(p.part_ms + 2 * i);
        const float w = ms[0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ms[0] - ref);
        total += ms[1] * w;
#pragma unroll
        for (int j = 0; j < D / 64; ++j) x[j] += p.part[i * D + lane * (D / 64) + j] * w;
    }
    const float scale = total == 0.f ? 0.f : 1.f / total;
    uint16_t* o = p.out + row.token * p.out_stride + row.head * D + lane * (D / 64);
    if constexpr (D == 128) *reinterpret_cast<unsigned*>(o) = ea_pack(x[0] * scale, x[1] * scale);
    else *o = uint16_t(ea_pack(x[0] * scale, 0.f));
    if (p.lse && lane == 0) p.lse[int64_t(row.head) * p.n_q + row.token] = total == 0.f ? -INFINITY : (ref + __builtin_amdgcn_logf(total)) * EA_LN2;
}

// ---- backward: dQ -------------------------------------------------------------------------------------------------
// 128 query rows, 32 a wave, as the forward pass.  delta_i = sum_j P_ij dP_ij is wanted to 32 bits: dP - delta cancels where a row's weights lie on few keys, and delta from the
// rounded output moves gradients by up to 2.7 times their own rounding there.  So the sweep over the keys adds it up beside its work, begun with dO . O; where the two
// differ by enough to be seen (2^-10 of the row's sum of P |dP - delta|) the sweep is done again with the better one.  Where the keys are few the first sweep only adds it up, and where
// they are dealt to several workgroups that is a launch of its own (PASS 1, then 2).
constexpr int EA_DELTA_FIRST = 256;              // up to so many keys delta comes first
constexpr float EA_DELTA_OFF = 0x1p-10f;

template <int D, int PASS>                       // 0: whole; 1: delta of a run of keys; 2: dQ of a run of keys
__global__ __launch_bounds__(256, 2) void ll_encoder_dq_kernel(const EncParams p) {
    constexpr int BLOCK = ENC_KEYS * D * 2, KS = D / 16, DB = D / 32;
    __shared__ __attribute__((aligned(16))) char lds[2][2][BLOCK];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
    const int tiles = p.plan.q_tiles, splits = PASS == 0 ? 1 : p.plan.q_splits;
    const int64_t at = ea_item(int64_t(p.n_seqs) * p.kv_heads * tiles * splits);
    if (at < 0) return;
    const EaForwardItem it = ea_forward_item(at, tiles, splits, p.by_kv_heads);
    const EncSpan qs = enc_span(p.cu_q, nullptr, it.seq, p.n_seqs, p.n_q, p.max_q), ks = enc_span(p.cu_k, p.k_lens, it.seq, p.n_seqs, p.n_k, p.max_k);
    if (int64_t(it.tile) * ENC_ROWS >= int64_t(qs.n) * p.by_group.d) return;
    const int in = wave * 32 + (lane & 31);
    const EaRow row = ea_query_row(p, qs, it.head, it.tile * ENC_ROWS + in);
    ea_u32x4 q[KS], dout[KS];
    ea_load_column<D>(q, p.q, p.q_stride, row, half);
    ea_load_column<D>(dout, p.dout, p.dout_stride, row, half);
    const int64_t row_at = int64_t(row.head) * p.n_q + row.token;
    const float lse = row.there ? p.lse[row_at] * EA_LOG2E : INFINITY;
    int begin, end;
    enc_run((ks.n + ENC_KEYS - 1) / ENC_KEYS, splits, it.split, begin, end);

    bool sums_only = PASS == 1 || (PASS == 0 && ks.n <= EA_DELTA_FIRST);
    bool known = sums_only;                       // delta is, or will be after the first sweep
    float delta = 0.f;
    if constexpr (PASS == 2) {
        if (row.there)
            for (int s = 0; s < splits; ++s) delta += p.part_d[(it.unit * splits + s) * ENC_ROWS + in];
        known = true;
        if (it.split == 0 && half == 0 && row.there) p.delta[row_at] = delta;
    } else if (!sums_only && row.there) {
        const uint16_t* o = p.o + row.token * p.out_stride + row.head * D + half * 8;
#pragma unroll
        for (int i = 0; i < KS; ++i) {
            const ea_u32x4 x = *reinterpret_cast<const ea_u32x4*>(o + 16 * i);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                delta = __builtin_fmaf(__builtin_bit_cast(float, x[e] << 16), __builtin_bit_cast(float, dout[i][e] << 16), delta);
                delta = __builtin_fmaf(__builtin_bit_cast(float, x[e] & 0xFFFF0000u), __builtin_bit_cast(float, dout[i][e] & 0xFFFF0000u), delta);
            }
        }
        delta = ea_sum2(delta, half);
    }
    const float keep = ks.n == 1 ? 0.f : 1.f;     // the softmax of one key is 1 whatever its score
    ea_f32x16 acc[DB];
    EaPieces<D, ENC_KEYS, 256> kp, vp;
    const auto load = [&](int s) {
        const int64_t first = int64_t(ks.begin) + s * ENC_KEYS;
        kp.load(p.k + first * p.k_stride + it.head * D, p.k_stride, ks.n - s * ENC_KEYS, tid);
        vp.load(p.v + first * p.v_stride + it.head * D, p.v_stride, ks.n - s * ENC_KEYS, tid);
    };
    for (;;) {                                    // at most two sweeps
#pragma unroll
        for (int db = 0; db < DB; ++db) acc[db] = ea_zero();
        float exact = 0.f, apart = 0.f;           // this half's sums of P dP and of P |dP - delta|
        if (begin < end) load(begin);
        int stage = 0;
        for (int step = begin; step < end; ++step, stage ^= 1) {
            kp.store(lds[stage][0], tid);
            vp.store(lds[stage][1], tid);
            __syncthreads();
            if (step + 1 < end) load(step + 1);
            const int left = ks.n - step * ENC_KEYS;
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const char* kb = lds[stage][0] + b * 64 * D;
                const char* vb = lds[stage][1] + b * 64 * D;
                ea_f32x16 s = ea_zero(), dp = ea_zero();
#pragma unroll
                for (int i = 0; i < KS; ++i) {
                    s = ea_mfma(ea_row_piece<D>(kb, lane, i), q[i], s);
                    dp = ea_mfma(ea_row_piece<D>(vb, lane, i), dout[i], dp);
                }
                if (left < 32 * (b + 1)) {
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (32 * b + 16 * (r >> 3) + 8 * half + (r & 7) >= left) s[r] = -INFINITY;
                }
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    float z[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[8 * t + e], p.scale_log2, -lse)), d = dp[8 * t + e];
                        exact = __builtin_fmaf(w, d, exact);
                        z[e] = w * (d - delta);
                        if constexpr (PASS == 0) apart += __builtin_fabsf(z[e]);
                    }
                    if (PASS != 1 && !sums_only) {
                        const ea_u32x4 zw = {ea_pack(z[0], z[1]), ea_pack(z[2], z[3]), ea_pack(z[4], z[5]), ea_pack(z[6], z[7])};
#pragma unroll
                        for (int db = 0; db < DB; ++db) acc[db] = ea_mfma(ea_col_piece<D>(kb, lane, t, db), zw, acc[db]);
                    }
                }
            }
        }
        if constexpr (PASS == 2) break;
        exact = ea_sum2(exact, half);
        if constexpr (PASS == 1) {
            if (half == 0) p.part_d[(it.unit * splits + it.split) * ENC_ROWS + in] = exact;
            return;
        }
        if (known && !sums_only) break;
        apart = ea_sum2(apart, half);
        const bool again = sums_only || (row.there && !(__builtin_fabsf(exact - delta) <= EA_DELTA_OFF * apart));
        delta = exact;
        sums_only = false;
        known = true;
        if (!__syncthreads_or(again)) break;      // also: no wave reads LDS any more
    }
    if (PASS == 0 && half == 0 && row.there) p.delta[row_at] = delta;
    if (PASS == 0) {
        if (row.there) ea_store_column<D>(p.dq + row.token * p.dq_stride + row.head * D, acc, p.scale * keep, half);
    } else if (row.there) {
        ea_store_part<D>(p.part_q + ((it.unit * splits + it.split) * ENC_ROWS + in) * D, acc, half);
    }
}

// ---- backward: dK, dV ---------------------------------------------------------------------------------------------
// 128 keys, 32 a wave; steps of 32 tokens of one query head, the heads of the group one after the other.
template <int D>
__global__ __launch_bounds__(256, 2) void ll_encoder_dkv_kernel(const EncParams p) {
    constexpr int BLOCK = ENC_BLOCK * D * 2, KS = D / 16, DB = D / 32;
    __shared__ __attribute__((aligned(16))) char lds[2][2][BLOCK];    // [stage][q, dO]
    __shared__ float aux[2][2][ENC_BLOCK];                            // [stage][lse, delta]
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
    const int tiles = p.plan.k_tiles, splits = p.plan.k_splits, group = p.by_group.d;
    const int64_t at = ea_item(int64_t(p.n_seqs) * p.kv_heads * tiles * splits);
    if (at < 0) return;
    const EaForwardItem it = ea_forward_item(at, tiles, splits, p.by_kv_heads);
    const EncSpan qs = enc_span(p.cu_q, nullptr, it.seq, p.n_seqs, p.n_q, p.max_q), ks = enc_span(p.cu_k, p.k_lens, it.seq, p.n_seqs, p.n_k, p.max_k);
    const int key0 = it.tile * ENC_COLS, key = key0 + wave * 32 + (lane & 31);
    // rows of the tile that are padding, and behind the last tile all that are left, get zeros
    if (it.split == 0) {
        const int from = max(key0, ks.n), to = it.tile == tiles - 1 ? ks.end - ks.begin : min(key0 + ENC_COLS, ks.end - ks.begin);
        for (int r = from + tid / (D / 8); r < to; r += 256 / (D / 8)) {
            const int64_t tok = int64_t(ks.begin) + r;
            const int f = it.head * D + tid % (D / 8) * 8;
            *reinterpret_cast<ea_u32x4*>(p.dk + tok * p.dk_stride + f) = ea_u32x4{0, 0, 0, 0};
            *reinterpret_cast<ea_u32x4*>(p.dv + tok * p.dv_stride + f) = ea_u32x4{0, 0, 0, 0};
        }
    }
    if (key0 >= ks.n) return;
    const EaRow col{key < ks.n, int64_t(ks.begin) + key, it.head};
    ea_u32x4 k[KS], v[KS];
    ea_load_column<D>(k, p.k, p.k_stride, col, half);
    ea_load_column<D>(v, p.v, p.v_stride, col, half);
    ea_f32x16 acc_k[DB], acc_v[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) acc_k[db] = acc_v[db] = ea_zero();
    const float keep = ks.n == 1 ? 0.f : 1.f;

    const int per_head = (qs.n + ENC_BLOCK - 1) / ENC_BLOCK;
    int step, end;
    enc_run(per_head * group, splits, it.split, step, end);
    int g = per_head ? step / per_head : 0, block = step - g * per_head;      // head of the group, block of its tokens: of the step to load next
    EaPieces<D, ENC_BLOCK, 256> qp, op;
    float side = 0.f;
    const auto load = [&]() {
        const int head = it.head * group + g, first = block * ENC_BLOCK, left = qs.n - first;
        const int64_t tok = int64_t(qs.begin) + first;
        qp.load(p.q + tok * p.q_stride + head * D, p.q_stride, left, tid);
        op.load(p.dout + tok * p.dout_stride + head * D, p.dout_stride, left, tid);
        if (tid < 64) {
            const int r = tid & 31;
            const int64_t i = int64_t(head) * p.n_q + tok + r;
            side = tid < 32 ? INFINITY : 0.f;                         // a row that is not there: P = 2^-inf
            if (r < left) side = tid < 32 ? p.lse[i] * EA_LOG2E : p.delta[i];
        }
        if (++block == per_head) {
            block = 0;
            ++g;
        }
    };
    if (step < end) load();
    for (int stage = 0; step < end; ++step, stage ^= 1) {
        qp.store(lds[stage][0], tid);
        op.store(lds[stage][1], tid);
        if (tid < 64) aux[stage][tid >> 5][tid & 31] = side;
        __syncthreads();
        if (step + 1 < end) load();
        const char* qb = lds[stage][0];
        const char* ob = lds[stage][1];
        ea_f32x16 s = ea_zero(), dp = ea_zero();
#pragma unroll
        for (int i = 0; i < KS; ++i) {
            s = ea_mfma(ea_row_piece<D>(qb, lane, i), k[i], s);
            dp = ea_mfma(ea_row_piece<D>(ob, lane, i), v[i], dp);
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const float* l = aux[stage][0] + 16 * t + 8 * half;
            const float* d = aux[stage][1] + 16 * t + 8 * half;
            float w[8], z[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                w[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[8 * t + e], p.scale_log2, -l[e]));
                z[e] = w[e] * (dp[8 * t + e] - d[e]);
            }
            const ea_u32x4 pw = {ea_pack(w[0], w[1]), ea_pack(w[2], w[3]), ea_pack(w[4], w[5]), ea_pack(w[6], w[7])};
            const ea_u32x4 zw = {ea_pack(z[0], z[1]), ea_pack(z[2], z[3]), ea_pack(z[4], z[5]), ea_pack(z[6], z[7])};
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                acc_v[db] = ea_mfma(ea_col_piece<D>(ob, lane, t, db), pw, acc_v[db]);
                acc_k[db] = ea_mfma(ea_col_piece<D>(qb, lane, t, db), zw, acc_k[db]);
            }
        }
    }
    if (!col.there) return;
    if (splits == 1) {
        ea_store_column<D>(p.dk + col.token * p.dk_stride + it.head * D, acc_k, p.scale * keep, half);
        ea_store_column<D>(p.dv + col.token * p.dv_stride + it.head * D, acc_v, 1.f, half);
    } else {
        float* to = p.part_kv + (it.unit * splits + it.split) * (2 * ENC_COLS * D) + (key - key0) * D;
        ea_store_part<D>(to, acc_k, half);
        ea_store_part<D>(to + ENC_COLS * D, acc_v, half);
    }
}

// Adds up the runs of dQ, dK and dV: 8 numbers of a row a thread.  Items: dQ's rows, then dK's and dV's.
template <int D>
__global__ __launch_bounds__(256) void ll_encoder_sum_kernel(const EncParams p) {
    constexpr int ACROSS = D / 8;
    const int64_t heads = int64_t(p.n_seqs) * p.kv_heads;
    const int64_t q_rows = p.plan.q_splits > 1 ? heads * p.plan.q_tiles * ENC_ROWS : 0, k_rows = p.plan.k_splits > 1 ? heads * p.plan.k_tiles * ENC_COLS : 0;
    int64_t r = (int64_t(blockIdx.x) * 256 + threadIdx.x) / ACROSS;
    const int f = threadIdx.x % ACROSS * 8;
    const bool is_q = r < q_rows;
    if (!is_q) r -= q_rows;
    const bool is_k = !is_q && r < k_rows;
    if (!is_q && !is_k) r -= k_rows;
    if (!is_q && r >= k_rows) return;
    const int tiles = is_q ? p.plan.q_tiles : p.plan.k_tiles, splits = is_q ? p.plan.q_splits : p.plan.k_splits;
    const unsigned unit = unsigned(r >> 7), of = unit / unsigned(tiles);
    const int in = int(r & 127), tile = int(unit - of * tiles), seq = p.by_kv_heads.of(of), head = of - seq * p.kv_heads;
    static_assert(ENC_ROWS == 128 && ENC_COLS == 128, "tiles of 128 rows");
    const EncSpan ks = enc_span(p.cu_k, p.k_lens, seq, p.n_seqs, p.n_k, p.max_k);
    const float* from;
    int64_t apart;
    uint16_t* to;
    float scale = ks.n == 1 ? 0.f : p.scale;
    if (is_q) {
        const EncSpan qs = enc_span(p.cu_q, nullptr, seq, p.n_seqs, p.n_q, p.max_q);
        if (int64_t(tile) * ENC_ROWS + in >= int64_t(qs.n) * p.by_group.d) return;
        const EaRow row = ea_query_row(p, qs, head, tile * ENC_ROWS + in);
        to = p.dq + row.token * p.dq_stride + row.head * D;
        from = p.part_q + (int64_t(unit) * splits * ENC_ROWS + in) * D;
        apart = ENC_ROWS * D;
    } else {
        const int key = tile * ENC_COLS + in;
        if (key >= ks.n) return;
        const int64_t tok = int64_t(ks.begin) + key;
        to = is_k ? p.dk + tok * p.dk_stride + head * D : p.dv + tok * p.dv_stride + head * D;
        if (!is_k) scale = 1.f;
        from = p.part_kv + int64_t(unit) * splits * (2 * ENC_COLS * D) + (is_k ? 0 : ENC_COLS * D) + in * D;
        apart = 2 * ENC_COLS * D;
    }
    ea_f32x4 a = {0.f, 0.f, 0.f, 0.f}, b = a;
    for (int s = 0; s < splits; ++s) {
        a += *reinterpret_cast<const ea_f32x4*>(from + s * apart + f);
        b += *reinterpret_cast<const ea_f32x4*>(from + s * apart + f + 4);
    }
    a *= scale;
    b *= scale;
    *reinterpret_cast<ea_u32x4*>(to + f) = ea_u32x4{ea_pack(a[0], a[1]), ea_pack(a[2], a[3]), ea_pack(b[0], b[1]), ea_pack(b[2], b[3])};
}

// ---- launches -----------------------------------------------------------------------------------------------------
template <int D>
static hipError_t ea_forward(const EncParams& p, hipStream_t s) {
    const int64_t heads = int64_t(p.n_seqs) * p.kv_heads, items = heads * p.plan.tiles * p.plan.splits;
    if (p.plan.few) hipLaunchKernelGGL(ll_encoder_few_kernel<D>, dim3(unsigned(ea_grid(items))), dim3(256), 0, s, p);
    else hipLaunchKernelGGL(ll_encoder_forward_kernel<D>, dim3(unsigned(ea_grid(items))), dim3(256), 0, s, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.plan.splits == 1) return e;
    const int64_t rows = heads * p.plan.tiles * (p.plan.few ? ENC_FEW_ROWS : ENC_ROWS);
    hipLaunchKernelGGL(ll_encoder_join_kernel<D>, dim3(unsigned(rows / 4)), dim3(256), 0, s, p);
    return hipGetLastError();
}
hipError_t launch_encoder_forward(const EncParams& p, hipStream_t s) { return p.D == 128 ? ea_forward<128>(p, s) : ea_forward<64>(p, s); }

template <int D>
static hipError_t ea_backward(const EncParams& p, hipStream_t s) {
    const int64_t heads = int64_t(p.n_seqs) * p.kv_heads;
    const unsigned q_grid = unsigned(ea_grid(heads * p.plan.q_tiles * p.plan.q_splits)), k_grid = unsigned(ea_grid(heads * p.plan.k_tiles * p.plan.k_splits));
    hipError_t e = hipSuccess;
    if (p.n_q > 0) {
        if (p.plan.q_splits == 1) {
            hipLaunchKernelGGL((ll_encoder_dq_kernel<D, 0>), dim3(q_grid), dim3(256), 0, s, p);
            e = hipGetLastError();
        } else {
            hipLaunchKernelGGL((ll_encoder_dq_kernel<D, 1>), dim3(q_grid), dim3(256), 0, s, p);
            e = hipGetLastError();
            if (e != hipSuccess) return e;
            hipLaunchKernelGGL((ll_encoder_dq_kernel<D, 2>), dim3(q_grid), dim3(256), 0, s, p);
            e = hipGetLastError();
        }
        if (e != hipSuccess) return e;
    }
    if (p.n_k > 0) {
        hipLaunchKernelGGL(ll_encoder_dkv_kernel<D>, dim3(k_grid), dim3(256), 0, s, p);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const int64_t rows = heads * ((p.plan.q_splits > 1 ? p.plan.q_tiles * ENC_ROWS : 0) + (p.plan.k_splits > 1 ? 2 * p.plan.k_tiles * ENC_COLS : 0));
    if (rows == 0) return e;
    hipLaunchKernelGGL(ll_encoder_sum_kernel<D>, dim3(unsigned(rows / (256 / (D / 8)))), dim3(256), 0, s, p);
    return hipGetLastError();
}
hipError_t launch_encoder_backward(const EncParams& p, hipStream_t s) { return p.D == 128 ? ea_backward<128>(p, s) : ea_backward<64>(p, s); }

}  // namespace ll
