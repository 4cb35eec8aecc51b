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
// A block's 16-byte pieces are stored in an order that turns with the row (ea_turn), so that the 16 lanes of a 16-byte read, and the 32 of a transposed one, find 64 different banks.
#include "encoder_attn.h"

#include <algorithm>
#include <type_traits>

namespace ll {

typedef __bf16 ea_bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 ea_bf16x2 __attribute__((ext_vector_type(2)));
typedef float ea_f32x16 __attribute__((ext_vector_type(16)));
typedef float ea_f32x4 __attribute__((ext_vector_type(4)));
typedef float ea_f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned ea_u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned ea_u32x2 __attribute__((ext_vector_type(2)));
typedef short ea_s16x4 __attribute__((ext_vector_type(4)));

constexpr int EA_AHEAD = 3;                        // fragments read in front of their matrix instruction (when they came in, dQ went from 287 us to 248; it is at 225 since)
constexpr float EA_LN2 = 0.69314718055994530942f, EA_LOG2E = 1.4426950408889634074f;
constexpr float EA_LOWEST = -3.402823466e38f;      // a row's reference before it has seen a key: finite, so that no difference is of two infinities
constexpr float EA_FAR = 0x1p32f;
constexpr float EA_LARGE = 0x1p118f;               // of a run's sums over the values: those of ENC_MAX_SPLITS runs add up to less than 32 bits hold
constexpr int EA_APART = 256;                    // sequences and kv heads: one for each CU
constexpr int EA_FEW_SPLITS = 16;                // of a row: joined by a few threads
constexpr float EA_SLACK = 8.f, EA_MOST = 0x1p8f; // a row's reference moves where a score is 2^8 times above it: the most that a weight is

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
// The two halves' values of a column, joined in the same order in both.
__device__ __forceinline__ ea_f32x2 ea_halves(float x) {
    const auto p = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    return ea_f32x2{__builtin_bit_cast(float, unsigned(p[0])), __builtin_bit_cast(float, unsigned(p[1]))};
}
__device__ __forceinline__ float ea_max2(float x) {
    const ea_f32x2 p = ea_halves(x);
    return fmaxf(p[0], p[1]);
}
__device__ __forceinline__ float ea_sum2(float x) {
    const ea_f32x2 p = ea_halves(x);
    return p[0] + p[1];
}

// ---- LDS blocks ---------------------------------------------------------------------------------------------------
// Piece c of row r lies at piece c ^ ea_turn(r) of that row.  Four rows one below the other turn by different 64-byte steps, rows four apart by different pieces in them (rows of
// 128 bytes: two rows are the 64 banks, and a pair turns together).
template <int D>
__device__ __forceinline__ int ea_turn(int r) { return D == 128 ? (r & 3) << 2 | (r >> 2 & 3) : (r >> 1 & 1) << 2 | (r >> 2 & 3); }
template <int D>
__device__ __forceinline__ int ea_at(int r, int c) { return r * (2 * D) + ((c ^ ea_turn<D>(r)) << 4); }

// Where in a block a lane reads; which piece, block or 16 rows is a constant more.  Blocks lie at multiples of 256 bytes.
template <int D>
struct EaLane {
    unsigned row, col, col4;
    __device__ __forceinline__ explicit EaLane(int lane) {
        const int i = lane & 31, half = lane >> 5, r = (i & 0x13) | (i & 4) << 1 | (i & 8) >> 1;
        row = ea_at<D>(r, half);
        const int s = lane & 15, first = 8 * half + (s >> 2), c = 2 * (lane >> 4 & 1) + (s >> 1 & 1);
        col = ea_at<D>(first, c) + 8 * (s & 1);
        col4 = ea_at<D>(first + 4, c) + 8 * (s & 1);
    }
    // A operand of a product over features: this lane's row of 32, features 16 ks + 8 half ..
    __device__ __forceinline__ ea_u32x4 row_piece(unsigned block, int ks, int on) const {          // `on`: bytes further, a constant
        typedef const __attribute__((address_space(3))) ea_u32x4 lds_u32x4;
        return *reinterpret_cast<lds_u32x4*>(((block + row) ^ (32 * ks)) + on);
    }
    // A operand of a product over rows: this lane's feature 32 db + lane % 32, rows 16 t + 8 half + 0..7.
    __device__ __forceinline__ ea_u32x4 col_piece(unsigned block, int t, int db, int on) const {
        typedef __attribute__((address_space(3))) ea_s16x4 lds_s16x4;
        const ea_s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_s16x4*>(((block + col) ^ (64 * db)) + (on + 16 * t * 2 * D)));
        const ea_s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_s16x4*>(((block + col4) ^ (64 * db)) + (on + 16 * t * 2 * D)));
        const ea_u32x2 a = __builtin_bit_cast(ea_u32x2, lo), b = __builtin_bit_cast(ea_u32x2, hi);
        return ea_u32x4{a[0], a[1], b[0], b[1]};
    }
};
__device__ __forceinline__ unsigned ea_lds(const char* x) { return (unsigned)(size_t)(const __attribute__((address_space(3))) char*)x; }

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
// What was loaded is there: the compiler would wait for it where it is first used, in the loop, and there for everything that is on its way.
template <int N>
__device__ __forceinline__ void ea_arrived(ea_u32x4 (&f)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(f[i]));
}
// Accumulators of a column [feature 32 db + 8 g + 4 half + i] as bfloat16, times `scale`: the halves exchange every other four features, so that each has eight in a
// row to store (a clip's forward pass, when it stored so: 165 us with eight bytes a store, 156 with sixteen).
__device__ __forceinline__ ea_u32x4 ea_pack_column(const ea_f32x16& acc, int g, float scale) {
    ea_u32x4 x;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const unsigned a = ea_pack(acc[4 * g + 2 * j] * scale, acc[4 * g + 2 * j + 1] * scale);
        const unsigned c = ea_pack(acc[4 * g + 4 + 2 * j] * scale, acc[4 * g + 5 + 2 * j] * scale);
        const auto p = __builtin_amdgcn_permlane32_swap(a, c, false, false);
        x[j] = p[0];
        x[2 + j] = p[1];
    }
    return x;
}
template <int D>
__device__ __forceinline__ void ea_store_column(uint16_t* at, const ea_f32x16 (&acc)[D / 32], float scale, int half) {
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int g = 0; g < 4; g += 2) *reinterpret_cast<ea_u32x4*>(at + 32 * db + 8 * g + 8 * half) = ea_pack_column(acc[db], g, scale);
}
// The same for a wave's 32 query rows by way of `lds`, 32 rows that nobody else uses any more: a row's numbers leave side by side, whole lines at a time. 7680 queries of 40 heads over
// 512 states: 55.5 us with a lane to a row, 53.6 so. (dQ, which has no registers for it, 225 and 230.)
template <int D>
__device__ __forceinline__ void ea_store_rows(const EncParams& p, uint16_t* x, int64_t stride, const EncSpan& q, int kv_head, int first, unsigned lds, const ea_f32x16 (&acc)[D / 32], float scale, int lane) {
    typedef __attribute__((address_space(3))) ea_u32x4 lds_u32x4;
    constexpr int ACROSS = D / 8, PER = 64 / ACROSS;
    const int half = lane >> 5;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int g = 0; g < 4; g += 2) *reinterpret_cast<lds_u32x4*>(lds + ea_at<D>(lane & 31, 4 * db + g + half)) = ea_pack_column(acc[db], g, scale);
    const int in = lane / ACROSS, c = lane % ACROSS;
#pragma unroll
    for (int i = 0; i < 32 / PER; ++i) {
        const EaRow row = ea_query_row(p, q, kv_head, first + PER * i + in);
        const ea_u32x4 y = *reinterpret_cast<lds_u32x4*>(lds + ea_at<D>(PER * i + in, c));
        if (row.there) *reinterpret_cast<ea_u32x4*>(x + row.token * stride + row.head * D + 8 * c) = y;
    }
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
// Scores of a block of 32 rows against this lane's column.
template <int D>
__device__ __forceinline__ ea_f32x16 ea_scores(const EaLane<D>& at, unsigned block, int on, const ea_u32x4 (&col)[D / 16]) {
    ea_f32x16 s = ea_zero();
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) s = ea_mfma(at.row_piece(block, ks, on), col[ks], s);
    return s;
}
// The order of a part of a loop's body: AHEAD fragments are read in front of the first matrix instruction, then READS reads and VECTOR vector instructions stand behind each of the N
// matrix instructions.  Left to itself the compiler, where registers are short, puts each read right in front of its use.
template <int N, int READS, int AHEAD, int VECTOR>
__device__ __forceinline__ void ea_order() {
    __builtin_amdgcn_sched_group_barrier(0x100, AHEAD * READS, 0);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if (i + AHEAD < N) __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
        if (VECTOR) __builtin_amdgcn_sched_group_barrier(0x002, VECTOR, 0);
    }
}
// The rows behind the first `rows` of a block are not there.
__device__ __forceinline__ void ea_mask(ea_f32x16& s, int rows, int half) {
#pragma unroll
    for (int r = 0; r < 16; ++r)
        if (16 * (r >> 3) + 8 * half + (r & 7) >= rows) s[r] = -INFINITY;
}
// The running softmax of a wave's 32 rows over blocks of 32 keys.
template <int D>
struct EaSoftmax {
    ea_f32x16 acc[D / 32];
    float ref, sum;                              // reference in log2 units, the same in both halves; this half's part of the row sum
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int db = 0; db < D / 32; ++db) acc[db] = ea_zero();
        ref = EA_LOWEST;
        sum = 0.f;
    }
    __device__ __forceinline__ void follow(const ea_f32x16& s, float scale_log2) {
        float top = s[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) top = fmaxf(top, s[r]);
        top = ea_max2(top) * scale_log2;
        if (__any(top > ref + EA_SLACK)) {
            const float next = fmaxf(ref, top), down = __builtin_amdgcn_exp2f(ref - next);
            ref = next;
            sum *= down;
#pragma unroll
            for (int db = 0; db < D / 32; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[db][r] *= down;
        }
    }
    __device__ __forceinline__ void weigh(const ea_f32x16& s, ea_u32x4 (&pw)[2], float scale_log2) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            float w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                w[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[8 * t + e], scale_log2, -ref));
                sum += w[e];
            }
            pw[t] = ea_u32x4{ea_pack(w[0], w[1]), ea_pack(w[2], w[3]), ea_pack(w[4], w[5]), ea_pack(w[6], w[7])};
        }
    }
    __device__ __forceinline__ void add(const EaLane<D>& at, unsigned block, int on, const ea_u32x4 (&pw)[2]) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int db = 0; db < D / 32; ++db) acc[db] = ea_mfma(at.col_piece(block, t, db, on), pw[t], acc[db]);
    }
};

// Which tile a workgroup takes, of units of `tiles` tiles and `splits` runs each.  Workgroup b runs on XCD b % 8, and the tiles of a unit's run read the same keys (or rows): they go to one XCD, unit
// after unit in turn; or, with `each`, so many of them to each XCD, from one more on with every unit, which evens out units of unequal length.
struct EaTile { int64_t unit; int tile, split, seq, head; };
__device__ __forceinline__ bool ea_place(const EncParams& p, int tiles, int splits, int each, EaTile& i, unsigned b = blockIdx.x) {
    const unsigned xcd = b & 7, at = b >> 3, per = each ? each : tiles, turn = at / per, in = at - turn * per;
    const unsigned u = each ? turn : xcd + 8 * turn;                  // unit and split
    i.tile = int(each ? ((xcd - u) & 7) * each + in : in);
    const unsigned of = u / unsigned(splits);
    i.split = int(u - of * splits);
    i.seq = p.by_kv_heads.of(of);
    i.head = int(of) - i.seq * p.kv_heads;
    i.unit = int64_t(of) * tiles + i.tile;
    return i.seq < p.n_seqs && i.tile < tiles;
}
static int64_t ea_grid(int64_t units, int tiles, int splits, int each) { return 8 * (each ? units * splits * each : (units * splits + 7) / 8 * tiles); }

// A buffer of everything from `base` on; the same base in all lanes.
__device__ __forceinline__ ea_u32x4 ea_rsrc(const void* base) {
    const uint64_t at = reinterpret_cast<uint64_t>(base);
    const unsigned lo = unsigned(__builtin_amdgcn_readfirstlane(int(unsigned(at)))), hi = unsigned(__builtin_amdgcn_readfirstlane(int(unsigned(at >> 32))));
    return ea_u32x4{lo, hi & 0xFFFFu, 0x7FFFFFFFu, 0x00020000u};
}

// A ring of NS blocks of 32 rows of two tensors, which the workgroup brings together, straight from memory into LDS, and every wave reads.  A wave brings the same
// 1 KB pieces of every block, and so knows by its own count of loads when they are there; behind the barrier all are.  The loads are written as instructions because the compiler, where it knows of them,
// lets every LDS read wait for all of them.
// Rows behind a sequence's last are the last row again (nothing is read that is not there) and then cleared by the wave that brought them, so that a weight of 0 meets no NaN.
template <int D, int STAGES>
struct EaRing {
    static constexpr int NS = STAGES, BLOCK = 32 * D * 2, STAGE = 2 * BLOCK, PIECES = D / 64, LOADS = 2 * PIECES;      // LOADS: of a wave and block
    unsigned lds;                                // of stage 0; a multiple of 256
    int row, feature;                            // this lane's, in the wave's first piece of each tensor; the second one is 16 rows on
    unsigned wave_at;
    __device__ __forceinline__ EaRing(const char* at, int lane, int wave) : lds(ea_lds(at)) {
        wave = __builtin_amdgcn_readfirstlane(wave);
        row = D == 128 ? 4 * wave + (lane >> 4) : 8 * wave + (lane >> 3);
        feature = ((lane & (D / 8 - 1)) ^ ea_turn<D>(row)) * 8;
        wave_at = wave * 1024;
    }
    __device__ __forceinline__ static int after(int stage, int n) { return stage + n >= NS ? stage + n - NS : stage + n; }
    __device__ __forceinline__ unsigned at(int stage) const { return lds + stage * STAGE; }
    // Rows base[0], base[stride] .. of one tensor, `left` of them at least one.
    __device__ __forceinline__ void bring(const uint16_t* base, int64_t stride, int left, unsigned to) const {
        const ea_u32x4 rsrc = ea_rsrc(base);
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const unsigned off = unsigned(min(row + 16 * i, left - 1)) * unsigned(2 * stride) + 2 * feature;
            unsigned keep;                       // m0, which is the compiler's
            asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds\n\ts_mov_b32 m0, %0"
                         : "=&s"(keep) : "s"(to + wave_at + i * 4096), "v"(off), "s"(rsrc) : "memory");
        }
    }
    __device__ __forceinline__ void issue(int stage, const uint16_t* a, int64_t a_stride, const uint16_t* b, int64_t b_stride, int left) const {
        const unsigned to = unsigned(__builtin_amdgcn_readfirstlane(int(at(stage))));
        bring(a, a_stride, left, to);
        bring(b, b_stride, left, to + BLOCK);
    }
    // Behind the wait for this wave's pieces of a block, in front of the barrier.
    __device__ __forceinline__ void clear(int stage, int left, int lane) const {
        typedef __attribute__((address_space(3))) ea_u32x4 lds_u32x4;
        if (left >= 32) return;
#pragma unroll
        for (int i = 0; i < PIECES; ++i)
            if (row + 16 * i >= left) {
                const unsigned to = at(stage) + wave_at + i * 4096 + lane * 16;
                *reinterpret_cast<lds_u32x4*>(to) = ea_u32x4{0, 0, 0, 0};
                *reinterpret_cast<lds_u32x4*>(to + BLOCK) = ea_u32x4{0, 0, 0, 0};
            }
    }
};
// The keys and values of one run, block after block.
template <int D, int STAGES>
struct EaKeys : EaRing<D, STAGES> {
    typedef EaRing<D, STAGES> Ring;
    const uint16_t *k, *v;                       // of the block to issue next
    int64_t k_stride, v_stride;
    int left;                                    // rows from there to the sequence's last
    int to;                                      // its stage
    __device__ __forceinline__ EaKeys(const char* at, int lane, int wave) : Ring(at, lane, wave) {}
    __device__ __forceinline__ void start(const EncParams& p, const EncSpan& ks, int head, int first) {
        const int64_t row = int64_t(ks.begin) + first * ENC_KEYS;
        k_stride = p.k_stride;
        v_stride = p.v_stride;
        k = p.k + row * k_stride + head * D;
        v = p.v + row * v_stride + head * D;
        left = ks.n - first * ENC_KEYS;
        to = 0;
    }
    __device__ __forceinline__ void issue() {
        Ring::issue(to, k, k_stride, v, v_stride, left);
        k += ENC_KEYS * k_stride;
        v += ENC_KEYS * v_stride;
        left -= ENC_KEYS;
        to = Ring::after(to, 1);
    }
};
// At most N of this wave's loads are outstanding.
template <int N>
__device__ __forceinline__ void ea_wait() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
// Every wave's LDS accesses in front of it are done.
__device__ __forceinline__ void ea_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// 128 query rows, 32 a wave; blocks of 32 keys.  In round i block i + 1 is there already: its scores are computed beside the vector work of block i, which does not
// depend on them.  A row's reference is the largest score of its first block: weights have the exponents of 32 bits, so that nothing is lost by one too low while sums stay finite, and
// following the largest score is work in every round (32760 queries of 12 heads x 128 over 4096 keys: 827 us, and 785 without).  Where a sum comes out above 2^32, or as no number, the
// tile is done again, following; and where weights are above what following leaves them and the sums over the values too large to be added up over all runs.  So n states of size |v| are
// summed as long as 2^8 n |v| < 2^127, as in the kernel for few rows.  A tile that is done again costs both sweeps: q of standard deviation 8 and keys of 1, 32760 queries of 12 heads over 4096 keys
// 1690 us, where 1 to 4 take 810 to 830 in the same run; over 512 keys 204, and 142 to 148.
// Bound by the matrix units, which the vector work of the two waves of a SIMD keeps from more: 785 us are 1050 TFLOP/s.  Over few keys the queries' and the outputs' way is as long: over 512
// 143 us, of which 95 are the rounds' (720 TFLOP/s; 100 MB in, 100 MB out).
template <int D>
__global__ __launch_bounds__(256, D == 128 ? 2 : 3) void ll_encoder_forward_kernel(const EncParams p) {
    typedef EaKeys<D, 4> Keys;
    __shared__ __attribute__((aligned(256))) char lds[Keys::NS * Keys::STAGE];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
    EaTile it;
    if (!ea_place(p, p.plan.tiles, p.plan.splits, p.plan.each, it)) return;
    const EncSpan qs = enc_span(p.cu_q, nullptr, it.seq, p.n_seqs, p.n_q, p.max_q), ks = enc_span(p.cu_k, p.k_lens, it.seq, p.n_seqs, p.n_k, p.max_k);
    if (int64_t(it.tile) * ENC_ROWS >= int64_t(qs.n) * p.by_group.d) return;
    int step, end;
    enc_run((ks.n + ENC_KEYS - 1) / ENC_KEYS, p.plan.splits, it.split, step, end);
    const EaRow row = ea_query_row(p, qs, it.head, it.tile * ENC_ROWS + wave * 32 + (lane & 31));
    const EaLane<D> where(lane);
    EaSoftmax<D> sm;
    sm.clear();
    float sum = 0.f;
    if (step < end) {
        Keys keys(lds, lane, wave);
        ea_u32x4 q[D / 16];
        const auto sweep = [&](auto every) {
            keys.start(p, ks, it.head, step);
            int left = keys.left, blocks = end - step;
            for (int i = 0; i < min(blocks, Keys::NS - 1); ++i) keys.issue();
            if constexpr (!decltype(every)::value) {
                ea_load_column<D>(q, p.q, p.q_stride, row, half);
                ea_arrived(q);
            }
            ea_wait<0>();
            for (int i = 0; i < min(blocks, Keys::NS - 1); ++i) keys.clear(i, left - i * ENC_KEYS, lane);
            ea_barrier();
            ea_f32x16 s = ea_scores<D>(where, keys.at(0), 0, q);
            if (left < ENC_KEYS) ea_mask(s, left, half);
            if constexpr (!decltype(every)::value) sm.follow(s, p.scale_log2);
            for (int stage = 0; blocks > 0; --blocks, left -= ENC_KEYS) {
                const int next = Keys::after(stage, 1);
                if (blocks > 2) ea_wait<(Keys::NS - 3) * Keys::LOADS>();      // the block after this one is there
                else ea_wait<0>();
                if (blocks > 1) keys.clear(next, left - ENC_KEYS, lane);
                ea_barrier();                                         // and nobody reads the block before this one any more
                if (blocks > Keys::NS - 1) keys.issue();
                if constexpr (decltype(every)::value) sm.follow(s, p.scale_log2);
                ea_f32x16 s_next = ea_scores<D>(where, keys.at(next), 0, q);      // behind the last block: of none
                ea_u32x4 pw[2];
                sm.weigh(s, pw, p.scale_log2);
                sm.add(where, keys.at(stage), Keys::BLOCK, pw);
                if (left - ENC_KEYS < ENC_KEYS) ea_mask(s_next, left - ENC_KEYS, half);
                s = s_next;
                stage = next;
            }
            sum = ea_sum2(sm.sum);
        };
        sweep(std::false_type{});
        bool again = !(sum < EA_FAR);
        if (__any(sum >= EA_MOST * float(min(ks.n - step * ENC_KEYS, (end - step) * ENC_KEYS)))) {
            float size = 0.f;
#pragma unroll
            for (int db = 0; db < D / 32; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r) size += __builtin_fabsf(sm.acc[db][r]);
            again |= !(size < EA_LARGE);
        }
        if (__syncthreads_or(again)) {
            sm.clear();
            sweep(std::true_type{});
            __syncthreads();                                          // nobody reads the last blocks any more: the output leaves by way of them
        }
    }
    if (p.plan.splits == 1) {
        int id = tid;
        asm volatile("" : "+v"(id));
        ea_store_rows<D>(p, p.out, p.out_stride, qs, it.head, it.tile * ENC_ROWS + wave * 32, ea_lds(lds) + wave * (64 * D), sm.acc, sum == 0.f ? 0.f : 1.f / sum, id & 63);
        if (p.lse && half == 0 && row.there) p.lse[int64_t(row.head) * p.n_q + row.token] = sum == 0.f ? -INFINITY : (sm.ref + __builtin_amdgcn_logf(sum)) * EA_LN2;
    } else if (row.there) {
        const int64_t r = (it.unit * p.plan.splits + it.split) * ENC_ROWS + wave * 32 + (lane & 31);
        ea_store_part<D>(p.part + r * D, sm.acc, half);
        if (half == 0) *reinterpret_cast<ea_f32x2*>(p.part_ms + 2 * r) = ea_f32x2{sm.ref, sum};
    }
}

// Up to 32 query rows; steps of 128 keys, 32 of them each wave's own: nothing is shared until the waves join.  Bound by memory, so a wave asks for its next keys as soon as
// the scores have read these, and for its next values as soon as the sums have.  24 tokens of 32 heads over up to 1500 states of 8, 98.7 MB: 21.3 us, 4.6 TB/s; one of 32 heads over 32000: 131 MB in
// 22.8 us, 5.7 TB/s, and 3.9 us to join 32 runs.
template <int D>
struct EaOwn {
    static constexpr int BLOCK = 32 * D * 2, PIECES = D / 16, PER = 512 / D;      // 1 KB pieces of a block; rows of one
    unsigned lds;
    int row, piece;                              // this lane's row and 16 bytes of the first 1 KB
    __device__ __forceinline__ EaOwn(unsigned at, int lane) : lds(unsigned(__builtin_amdgcn_readfirstlane(int(at)))) {
        row = lane / (D / 8);
        piece = (lane % (D / 8)) ^ ea_turn<D>(row);
    }
    __device__ __forceinline__ void bring(const uint16_t* base, int64_t stride, int left, int on) const {
        const ea_u32x4 rsrc = ea_rsrc(base);
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {       // the rows' turns differ by what i adds to the row
            const unsigned off = unsigned(min(row + PER * i, left - 1)) * unsigned(2 * stride) + unsigned(piece ^ ea_turn<D>(PER * i)) * 16;
            unsigned keep;
            asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds\n\ts_mov_b32 m0, %0"
                         : "=&s"(keep) : "s"(lds + on + i * 1024), "v"(off), "s"(rsrc) : "memory");
        }
    }
    __device__ __forceinline__ void clear(int left, int on, int lane) const {
        typedef __attribute__((address_space(3))) ea_u32x4 lds_u32x4;
        if (left >= 32) return;
#pragma unroll
        for (int i = 0; i < PIECES; ++i)
            if (row + PER * i >= left) *reinterpret_cast<lds_u32x4*>(lds + on + i * 1024 + lane * 16) = ea_u32x4{0, 0, 0, 0};
    }
};
template <int D>
__global__ __launch_bounds__(256, 2) void ll_encoder_few_kernel(const EncParams p) {
    typedef EaOwn<D> Own;
    constexpr int BLOCK = Own::BLOCK, JOIN = 32 * (D + 4);           // bytes; floats of a wave's results
    constexpr int BYTES = 4 * 2 * BLOCK > 4 * JOIN * 4 ? 4 * 2 * BLOCK : 4 * JOIN * 4;
    __shared__ __attribute__((aligned(256))) char lds[BYTES];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5, col = lane & 31;
    EaTile it;                                                        // one tile a sequence and kv head; heads first, which lie side by side in memory
    const unsigned run = p.by_kv_heads.of(blockIdx.x);
    it.tile = 0;
    it.head = int(blockIdx.x - run * p.kv_heads);
    it.seq = run / unsigned(p.plan.splits);
    it.split = int(run - unsigned(it.seq) * p.plan.splits);
    it.unit = int64_t(it.seq) * p.kv_heads + it.head;
    const EncSpan qs = enc_span(p.cu_q, nullptr, it.seq, p.n_seqs, p.n_q, p.max_q), ks = enc_span(p.cu_k, p.k_lens, it.seq, p.n_seqs, p.n_k, p.max_k);
    if (qs.n == 0) return;
    const EaRow row = ea_query_row(p, qs, it.head, col);
    int step, end;
    enc_run((ks.n + ENC_FEW_KEYS - 1) / ENC_FEW_KEYS, p.plan.splits, it.split, step, end);
    EaSoftmax<D> sm;
    sm.clear();
    const Own own(ea_lds(lds) + wave * 2 * BLOCK, lane);
    int left = ks.n - step * ENC_FEW_KEYS - wave * 32, blocks = left > 0 && step < end ? min((left + ENC_FEW_KEYS - 1) / ENC_FEW_KEYS, end - step) : 0;
    left = __builtin_amdgcn_readfirstlane(left);
    blocks = __builtin_amdgcn_readfirstlane(blocks);
    if (blocks > 0) {
        const int64_t first = int64_t(ks.begin) + (ks.n - left);
        const uint16_t *k = p.k + first * p.k_stride + it.head * D, *v = p.v + first * p.v_stride + it.head * D;
        own.bring(k, p.k_stride, left, 0);
        own.bring(v, p.v_stride, left, BLOCK);
        ea_u32x4 q[D / 16];
        ea_load_column<D>(q, p.q, p.q_stride, row, half);
        ea_arrived(q);
        const EaLane<D> where(lane);
        for (; blocks > 0; --blocks, left -= ENC_FEW_KEYS) {
            ea_wait<Own::PIECES>();                                   // the keys are there
            ea_f32x16 s = ea_scores<D>(where, own.lds, 0, q);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");        // and read
            k += ENC_FEW_KEYS * p.k_stride;
            if (blocks > 1) own.bring(k, p.k_stride, left - ENC_FEW_KEYS, 0);
            if (left < 32) ea_mask(s, left, half);
            sm.follow(s, p.scale_log2);
            ea_u32x4 pw[2];
            sm.weigh(s, pw, p.scale_log2);
            if (blocks > 1) ea_wait<Own::PIECES>();                   // the values are there
            else ea_wait<0>();
            own.clear(left, BLOCK, lane);
            sm.add(where, own.lds, BLOCK, pw);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            v += ENC_FEW_KEYS * p.v_stride;
            if (blocks > 1) own.bring(v, p.v_stride, left - ENC_FEW_KEYS, BLOCK);
        }
    }
    // the four waves' results meet in LDS: wave w adds up features D / 4 w ..
    const float sum = ea_sum2(sm.sum);
    __syncthreads();                                                  // every wave is done with its blocks
    float* const mine = reinterpret_cast<float*>(lds) + wave * JOIN + col * (D + 4);
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *reinterpret_cast<ea_f32x4*>(mine + 32 * db + 8 * g + 4 * half) = ea_f32x4{sm.acc[db][4 * g], sm.acc[db][4 * g + 1], sm.acc[db][4 * g + 2], sm.acc[db][4 * g + 3]};
    if (half == 0) *reinterpret_cast<ea_f32x2*>(mine + D) = ea_f32x2{sm.ref, sum};
    __syncthreads();
    const float* const rows = reinterpret_cast<const float*>(lds) + col * (D + 4);
    float ref = EA_LOWEST, total = 0.f, w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) ref = fmaxf(ref, rows[i * JOIN + D]);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        w[i] = __builtin_amdgcn_exp2f(rows[i * JOIN + D] - ref);
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

// Joins the splits of a row, a workgroup each: its splits' weights first, then 16 bytes of every 256 / (D / 4)-th split a thread.  Bound by the way there and back: 32 rows of 32 splits 4.0 us.
template <int D>
__global__ __launch_bounds__(256) void ll_encoder_join_kernel(const EncParams p, int rows) {
    constexpr int ACROSS = D / 4, STRANDS = 256 / ACROSS;
    __shared__ float weight[ENC_MAX_SPLITS];
    __shared__ __attribute__((aligned(16))) float part[STRANDS][D];
    __shared__ float wave_top[4], wave_sum[4];
    const int tile_rows = p.plan.few ? ENC_FEW_ROWS : ENC_ROWS, tid = threadIdx.x, splits = p.plan.splits;
    const unsigned unit = blockIdx.x / unsigned(rows), in = blockIdx.x - unit * rows, of = unit / unsigned(p.plan.tiles);
    const int tile = int(unit - of * p.plan.tiles), seq = p.by_kv_heads.of(of), head = of - seq * p.kv_heads;
    const EncSpan qs = enc_span(p.cu_q, nullptr, seq, p.n_seqs, p.n_q, p.max_q);
    const int64_t r = int64_t(tile) * tile_rows + in;
    if (r >= int64_t(qs.n) * p.by_group.d) return;
    const EaRow row = ea_query_row(p, qs, head, int(r));
    const int64_t first = int64_t(unit) * splits * tile_rows + in;
    ea_f32x2 ms[ENC_MAX_SPLITS / 256];
    float top = EA_LOWEST;
#pragma unroll
    for (int i = 0; i < ENC_MAX_SPLITS / 256; ++i) {
        ms[i] = ea_f32x2{EA_LOWEST, 0.f};
        if (tid + 256 * i < splits) ms[i] = *reinterpret_cast<const ea_f32x2*>(p.part_ms + 2 * (first + int64_t(tid + 256 * i) * tile_rows));
        top = fmaxf(top, ms[i][0]);
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    if ((tid & 63) == 0) wave_top[tid >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(wave_top[0], wave_top[1]), fmaxf(wave_top[2], wave_top[3]));
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < ENC_MAX_SPLITS / 256; ++i) {
        const float w = __builtin_amdgcn_exp2f(ms[i][0] - top);
        weight[tid + 256 * i] = w;
        sum += ms[i][1] * w;
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
    if ((tid & 63) == 0) wave_sum[tid >> 6] = sum;
    __syncthreads();
    ea_f32x4 x = {0.f, 0.f, 0.f, 0.f};
    const int f = tid % ACROSS * 4, strand = tid / ACROSS;
#pragma unroll 4
    for (int s = strand; s < splits; s += STRANDS) {
        const ea_f32x4 y = *reinterpret_cast<const ea_f32x4*>(p.part + (first + int64_t(s) * tile_rows) * D + f);
        const float w = weight[s];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = __builtin_fmaf(y[j], w, x[j]);
    }
    *reinterpret_cast<ea_f32x4*>(&part[strand][f]) = x;
    __syncthreads();
    if (strand != 0) return;
#pragma unroll
    for (int i = 1; i < STRANDS; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] += part[i][f + j];
    const float total = (wave_sum[0] + wave_sum[1]) + (wave_sum[2] + wave_sum[3]), scale = total == 0.f ? 0.f : 1.f / total;
    *reinterpret_cast<ea_u32x2*>(p.out + row.token * p.out_stride + row.head * D + f) = ea_u32x2{ea_pack(x[0] * scale, x[1] * scale), ea_pack(x[2] * scale, x[3] * scale)};
    if (p.lse && tid == 0) p.lse[int64_t(row.head) * p.n_q + row.token] = total == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * EA_LN2;
}

// The same for a few splits of many rows: 8 numbers of a row a thread.  8000 rows of 4 splits 4.8 us, and 11.9 a workgroup each; 128 rows of 16 splits 4.0 and 3.8, 32 of 32 8.0 and 4.0.
template <int D>
__global__ __launch_bounds__(256) void ll_encoder_join_rows_kernel(const EncParams p, int rows) {
    constexpr int ACROSS = D / 8;
    const int tile_rows = p.plan.few ? ENC_FEW_ROWS : ENC_ROWS, splits = p.plan.splits;
    const unsigned at = (blockIdx.x * 256 + threadIdx.x) / ACROSS, unit = at / unsigned(rows), in = at - unit * rows, of = unit / unsigned(p.plan.tiles);
    const int tile = int(unit - of * p.plan.tiles), seq = p.by_kv_heads.of(of), head = of - seq * p.kv_heads, f = threadIdx.x % ACROSS * 8;
    if (seq >= p.n_seqs) return;
    const EncSpan qs = enc_span(p.cu_q, nullptr, seq, p.n_seqs, p.n_q, p.max_q);
    const int64_t r = int64_t(tile) * tile_rows + in;
    if (r >= int64_t(qs.n) * p.by_group.d) return;
    const EaRow row = ea_query_row(p, qs, head, int(r));
    const int64_t first = int64_t(unit) * splits * tile_rows + in;
    float top = EA_LOWEST;
#pragma unroll 4
    for (int s = 0; s < splits; ++s) top = fmaxf(top, p.part_ms[2 * (first + int64_t(s) * tile_rows)]);
    ea_f32x4 a = {0.f, 0.f, 0.f, 0.f}, b = a;
    float total = 0.f;
#pragma unroll 4
    for (int s = 0; s < splits; ++s) {
        const int64_t i = first + int64_t(s) * tile_rows;
        const ea_f32x2 ms = *reinterpret_cast<const ea_f32x2*>(p.part_ms + 2 * i);
        const ea_f32x4 x = *reinterpret_cast<const ea_f32x4*>(p.part + i * D + f), y = *reinterpret_cast<const ea_f32x4*>(p.part + i * D + f + 4);
        const float w = __builtin_amdgcn_exp2f(ms[0] - top);
        total = __builtin_fmaf(ms[1], w, total);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            a[j] = __builtin_fmaf(x[j], w, a[j]);
            b[j] = __builtin_fmaf(y[j], w, b[j]);
        }
    }
    const float scale = total == 0.f ? 0.f : 1.f / total;
    a *= scale;
    b *= scale;
    *reinterpret_cast<ea_u32x4*>(p.out + row.token * p.out_stride + row.head * D + f) = ea_u32x4{ea_pack(a[0], a[1]), ea_pack(a[2], a[3]), ea_pack(b[0], b[1]), ea_pack(b[2], b[3])};
    if (p.lse && f == 0) p.lse[int64_t(row.head) * p.n_q + row.token] = total == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(total)) * EA_LN2;
}

// ---- backward: dQ -------------------------------------------------------------------------------------------------
// 128 query rows, 32 a wave, as the forward pass.  delta_i = sum_j P_ij dP_ij is wanted to 32 bits: dP - delta cancels where a row's weights lie on few keys, and delta from the
// rounded output moves gradients by up to 2.7 times their own rounding there.  So the sweep over the keys adds it up beside its work, begun with dO . O; where the two
// differ by enough to be seen (2^-10 of the row's sum of P |dP - delta|) the sweep is done again with the better one.  Where the keys are few the first sweep only adds it up, and where
// they are dealt to several workgroups that is a launch of its own (PASS 1, then 2).
// Bound as the forward pass: 32760 queries of 12 heads over 512 keys 225 us, of which about 140 are three products' (155 GFLOP) and the rest the way of 400 MB, which nothing stands beside: asking
// for the next tile's rows while a tile is worked on made it 230 (through the cache).
// The second sweep is no rarity: it comes where a row has about half its weight on one key.  The same with q of standard deviation 1, 2, 4 and 8 and keys of 1: 235, 373, 378 and 370 us over 512
// keys; over 4096 1186, 2096, 2289 and 2290.
constexpr float EA_DELTA_OFF = 0x1p-10f;

template <int D, int PASS>                       // 0: whole; 1: delta of a run of keys; 2: dQ of a run of keys; 3: delta; 4: dQ, delta once more; 5: dQ, delta there; 6: of a run
__device__ __forceinline__ void ea_dq(const EncParams& p, const EaTile& it, char* lds) {
    constexpr int KS = D / 16, DB = D / 32;
    typedef EaKeys<D, 4> Keys;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
    const int splits = PASS == 1 || PASS == 2 || PASS == 6 ? p.plan.q_splits : 1;
    const EncSpan qs = enc_span(p.cu_q, nullptr, it.seq, p.n_seqs, p.n_q, p.max_q), ks = enc_span(p.cu_k, p.k_lens, it.seq, p.n_seqs, p.n_k, p.max_k);
    if (int64_t(it.tile) * ENC_ROWS >= int64_t(qs.n) * p.by_group.d) return;
    const int in = wave * 32 + (lane & 31);
    const EaRow row = ea_query_row(p, qs, it.head, it.tile * ENC_ROWS + in);
    ea_u32x4 q[KS], dout[KS];
    ea_load_column<D>(q, p.q, p.q_stride, row, half);
    ea_load_column<D>(dout, p.dout, p.dout_stride, row, half);
    const int64_t row_at = int64_t(row.head) * p.n_q + row.token;
    const float lse = row.there ? p.lse[row_at] * EA_LOG2E : INFINITY;       // a row that is not there: P = 2^-inf
    int begin, end;
    enc_run((ks.n + ENC_KEYS - 1) / ENC_KEYS, splits, it.split, begin, end);

    const bool first = PASS == 1 || PASS == 3 || PASS == 4 || (PASS == 0 && ks.n <= ENC_DELTA_FIRST);        // delta first
    float delta = 0.f;
    if constexpr (PASS == 2) {
        if (row.there)
            for (int s = 0; s < splits; ++s) delta += p.part_d[(it.unit * splits + s) * ENC_ROWS + in];
        if (it.split == 0 && half == 0 && row.there) *reinterpret_cast<ea_f32x2*>(p.side + 2 * row_at) = ea_f32x2{lse, delta};
    } else if constexpr (PASS >= 5) {
        if (row.there) delta = p.side[2 * row_at + 1];
    } else if (!first && row.there) {
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
        delta = ea_sum2(delta);
    }
    const float keep = ks.n == 1 ? 0.f : 1.f;     // the softmax of one key is 1 whatever its score
    const EaLane<D> where(lane);
    ea_arrived(q);
    ea_arrived(dout);
    Keys keys(lds, lane, wave);
    const int all = end - begin, length = ks.n - begin * ENC_KEYS;
    ea_f32x16 acc[DB];
    float exact, apart;                           // this half's sums of P dP and of P |dP - delta|
    bool there = false;                           // up to three blocks stay in LDS
    // FULL: with dQ; otherwise only the sum of P dP
    const auto sweep = [&](auto full) {
        constexpr bool FULL = decltype(full)::value;
#pragma unroll
        for (int db = 0; db < DB; ++db) acc[db] = ea_zero();
        exact = apart = 0.f;
        int left = length, blocks = all;
        if (blocks <= 0) return;
        if (!there || blocks > 3) {
            keys.start(p, ks, it.head, begin);
            for (int i = 0; i < min(blocks, 3); ++i) keys.issue();
            ea_wait<0>();
            for (int i = 0; i < min(blocks, 3); ++i) keys.clear(i, left - i * ENC_KEYS, lane);
            ea_barrier();
            there = true;
        }
        ea_f32x16 s = ea_scores<D>(where, keys.at(0), 0, q), dp = ea_scores<D>(where, keys.at(0), Keys::BLOCK, dout);
        for (int stage = 0; blocks > 0; --blocks, left -= ENC_KEYS) {
            const int next = Keys::after(stage, 1);
            if (blocks > 2) ea_wait<Keys::LOADS>();                   // the block after this one is there
            else ea_wait<0>();
            if (blocks > 1) keys.clear(next, left - ENC_KEYS, lane);
            ea_barrier();                                             // and nobody reads the block before this one any more
            if (blocks > 3) keys.issue();
            if (left < ENC_KEYS) ea_mask(s, left, half);
            // in three parts, for the registers' sake: scores of the next block beside the weights of this one, its dP beside this one's dS, then dQ
            const ea_f32x16 s_next = ea_scores<D>(where, keys.at(next), 0, q);
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], p.scale_log2, -lse));
                if constexpr (PASS != 2 && PASS < 5) exact = __builtin_fmaf(s[r], dp[r], exact);
            }
            ea_order<KS, 1, EA_AHEAD, 6>();
            __builtin_amdgcn_sched_barrier(0);
            const ea_f32x16 dp_next = ea_scores<D>(where, keys.at(next), Keys::BLOCK, dout);
            if constexpr (FULL) {
                ea_u32x4 zw[2];
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    float z[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        z[e] = s[8 * t + e] * (dp[8 * t + e] - delta);
                        if constexpr (PASS == 0) apart += __builtin_fabsf(z[e]);
                    }
                    zw[t] = ea_u32x4{ea_pack(z[0], z[1]), ea_pack(z[2], z[3]), ea_pack(z[4], z[5]), ea_pack(z[6], z[7])};
                }
                ea_order<KS, 1, EA_AHEAD, 7>();
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int db = 0; db < DB; ++db) acc[db] = ea_mfma(where.col_piece(keys.at(stage), t, db, 0), zw[t], acc[db]);
                ea_order<2 * DB, 2, EA_AHEAD, 0>();
                __builtin_amdgcn_sched_barrier(0);
            }
            s = s_next;
            dp = dp_next;
            stage = next;
        }
    };
    if (first) {
        sweep(std::false_type{});
        delta = ea_sum2(exact);
        __syncthreads();                          // nobody reads the last blocks any more
    }
    if constexpr (PASS == 1) {
        if (half == 0) p.part_d[(it.unit * splits + it.split) * ENC_ROWS + in] = delta;
        return;
    } else if constexpr (PASS == 3) {
        if (half == 0 && row.there) *reinterpret_cast<ea_f32x2*>(p.side + 2 * row_at) = ea_f32x2{lse, delta};
        return;
    } else {
        for (bool known = PASS == 2 || PASS >= 5 || first;; known = true) {        // at most twice
            sweep(std::true_type{});
            if (known) break;
            exact = ea_sum2(exact);
            const bool again = !(__builtin_fabsf(exact - delta) <= EA_DELTA_OFF * ea_sum2(apart));      // a row that is not there: 0 <= 0
            delta = exact;
            if (!__syncthreads_or(again)) break;
        }
    }
    int id = threadIdx.x;                        // the row once more: kept through the loop it would cost registers that there are none of
    asm volatile("" : "+v"(id));
    const int mine = (id >> 6) * 32 + (id & 31), of_half = id >> 5 & 1;
    const EaRow at_end = ea_query_row(p, qs, it.head, it.tile * ENC_ROWS + mine);
    if (!at_end.there) return;
    if constexpr (PASS == 0 || PASS == 4 || PASS == 5) {
        if (PASS == 0 && of_half == 0) *reinterpret_cast<ea_f32x2*>(p.side + 2 * (int64_t(at_end.head) * p.n_q + at_end.token)) = ea_f32x2{lse, delta};
        ea_store_column<D>(p.dq + at_end.token * p.dq_stride + at_end.head * D, acc, p.scale * keep, of_half);
    } else {
        ea_store_part<D>(p.part_q + ((it.unit * splits + it.split) * ENC_ROWS + mine) * D, acc, of_half);
    }
}

template <int D, int PASS>
__global__ __launch_bounds__(256, 2) void ll_encoder_dq_kernel(const EncParams p) {
    __shared__ __attribute__((aligned(256))) char lds[EaKeys<D, 4>::NS * EaKeys<D, 4>::STAGE];
    const int splits = PASS == 0 ? 1 : p.plan.q_splits;
    EaTile it;
    if (ea_place(p, p.plan.q_tiles, splits, p.plan.q_each, it)) ea_dq<D, PASS>(p, it, lds);
}

// ---- backward: dK, dV ---------------------------------------------------------------------------------------------
// 128 keys, 32 a wave; blocks of 32 tokens of one query head, the heads of the group one after the other.  The rows' lse and delta come beside their block.  Bound by the matrix
// units: 32760 queries of 12 heads x 128 over 512 keys, four products of 51.5 GFLOP: 218 us, 945 TFLOP/s (the products alone 137), and 11.6 us to add up ten runs.
// At 128 features a register is spilled here, 2 in ll_encoder_both_kernel, 12 and 3 (apart and in one) in ll_encoder_small_backward_kernel; the counted waits stand that: an access more makes one longer.
template <int D>
constexpr int EA_DKV_LDS = EaRing<D, 4>::NS * (EaRing<D, 4>::STAGE + 256);
template <int D>
__device__ __forceinline__ void ea_dkv(const EncParams& p, const EaTile& it, char* lds) {
    typedef EaRing<D, 4> Ring;
    constexpr int KS = D / 16, DB = D / 32, LOADS = Ring::LOADS + 1;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
    const int tiles = p.plan.k_tiles, splits = p.plan.k_splits, group = p.by_group.d;
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
    ea_f32x16 acc_k[DB], acc_v[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) acc_k[db] = acc_v[db] = ea_zero();
    const float keep = ks.n == 1 ? 0.f : 1.f;
    const EaLane<D> where(lane);

    const int per_head = (qs.n + ENC_BLOCK - 1) / ENC_BLOCK;
    int step, end;
    enc_run(per_head * group, splits, it.split, step, end);
    const Ring ring(lds, lane, wave);
    const unsigned sides = ring.lds + Ring::NS * Ring::STAGE;
    // of the step to issue next: head of the group, rows from its block to the sequence's last, where they lie, its stage
    int g = per_head ? step / per_head : 0, to_left = qs.n - (step - g * per_head) * ENC_BLOCK, to = 0;
    const uint16_t *q_at = nullptr, *o_at = nullptr;
    const float* side_at = nullptr;
    const auto place = [&]() {
        const int head = it.head * group + g;
        const int64_t tok = int64_t(qs.begin) + (qs.n - to_left);
        q_at = p.q + tok * p.q_stride + head * D;
        o_at = p.dout + tok * p.dout_stride + head * D;
        side_at = p.side + 2 * (int64_t(head) * p.n_q + tok);
    };
    const auto issue = [&]() {
        ring.issue(to, q_at, p.q_stride, o_at, p.dout_stride, to_left);
        const unsigned side_to = unsigned(__builtin_amdgcn_readfirstlane(int(sides + to * 256))), off = 8 * min(lane & 31, to_left - 1) + 4 * half;
        unsigned keep;
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dword %2, %3, 0 offen lds\n\ts_mov_b32 m0, %0"      // by all waves, the same numbers
                     : "=&s"(keep) : "s"(side_to), "v"(off), "s"(ea_rsrc(side_at)) : "memory");
        to = Ring::after(to, 1);
        to_left -= ENC_BLOCK;
        if (to_left > 0) {
            q_at += ENC_BLOCK * p.q_stride;
            o_at += ENC_BLOCK * p.dout_stride;
            side_at += 2 * ENC_BLOCK;
        } else {
            ++g;
            to_left = qs.n;
            place();
        }
    };
    int blocks = end - step, left = to_left, stage = 0;
    if (blocks > 0) place();
    for (int i = 0; i < min(blocks, 3); ++i) issue();
    ea_u32x4 k[KS], v[KS];
    ea_load_column<D>(k, p.k, p.k_stride, col, half);
    ea_load_column<D>(v, p.v, p.v_stride, col, half);
    ea_arrived(k);
    ea_arrived(v);
    for (; blocks > 0; --blocks) {
        if (blocks > 2) ea_wait<2 * LOADS>();                         // this block is there
        else if (blocks > 1) ea_wait<LOADS>();
        else ea_wait<0>();
        ring.clear(stage, left, lane);
        ea_barrier();                                                 // and nobody reads the block before it any more
        if (blocks > 3) issue();
        const unsigned qb = ring.at(stage);
        ea_f32x16 s = ea_scores<D>(where, qb, 0, k);
        ea_order<KS, 1, EA_AHEAD, 0>();
        if (left < ENC_BLOCK) ea_mask(s, left, half);
        __builtin_amdgcn_sched_barrier(0);
        typedef const __attribute__((address_space(3))) ea_f32x4 lds_f32x4;
        const unsigned side = sides + stage * 256 + half * 32;         // lse of the block's rows, then their delta
        const ea_f32x16 dp = ea_scores<D>(where, qb, Ring::BLOCK, v);             // beside it the weights
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const ea_f32x4 x = *reinterpret_cast<lds_f32x4*>(side + (r >> 3) * 64 + (r & 7) * 4);
#pragma unroll
            for (int j = 0; j < 4; ++j) s[r + j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r + j], p.scale_log2, -x[j]));
        }
        ea_order<KS, 1, EA_AHEAD, 5>();
        __builtin_amdgcn_sched_barrier(0);
        ea_u32x4 pw[2], zw[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            float z[8];
#pragma unroll
            for (int e = 0; e < 8; e += 4) {
                const ea_f32x4 x = *reinterpret_cast<lds_f32x4*>(side + 128 + t * 64 + e * 4);
#pragma unroll
                for (int j = 0; j < 4; ++j) z[e + j] = s[8 * t + e + j] * (dp[8 * t + e + j] - x[j]);
            }
            pw[t] = ea_u32x4{ea_pack(s[8 * t], s[8 * t + 1]), ea_pack(s[8 * t + 2], s[8 * t + 3]), ea_pack(s[8 * t + 4], s[8 * t + 5]), ea_pack(s[8 * t + 6], s[8 * t + 7])};
            zw[t] = ea_u32x4{ea_pack(z[0], z[1]), ea_pack(z[2], z[3]), ea_pack(z[4], z[5]), ea_pack(z[6], z[7])};
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                acc_v[db] = ea_mfma(where.col_piece(qb, t, db, Ring::BLOCK), pw[t], acc_v[db]);
                acc_k[db] = ea_mfma(where.col_piece(qb, t, db, 0), zw[t], acc_k[db]);
            }
        ea_order<4 * DB, 2, EA_AHEAD, 0>();
        __builtin_amdgcn_sched_barrier(0);
        stage = Ring::after(stage, 1);
        left = left > ENC_BLOCK ? left - ENC_BLOCK : qs.n;
    }
    int id = threadIdx.x;                        // the column once more, as the row above
    asm volatile("" : "+v"(id));
    const int mine = it.tile * ENC_COLS + (id >> 6) * 32 + (id & 31), of_half = id >> 5 & 1;
    if (mine >= ks.n) return;
    if (splits == 1) {
        ea_store_column<D>(p.dk + (int64_t(ks.begin) + mine) * p.dk_stride + it.head * D, acc_k, p.scale * keep, of_half);
        ea_store_column<D>(p.dv + (int64_t(ks.begin) + mine) * p.dv_stride + it.head * D, acc_v, 1.f, of_half);
    } else {
        float* to = p.part_kv + (it.unit * splits + it.split) * (2 * ENC_COLS * D) + (mine - it.tile * ENC_COLS) * D;
        ea_store_part<D>(to, acc_k, of_half);
        ea_store_part<D>(to + ENC_COLS * D, acc_v, of_half);
    }
}

template <int D>
__global__ __launch_bounds__(256, 2) void ll_encoder_dkv_kernel(const EncParams p) {
    __shared__ __attribute__((aligned(256))) char lds[EA_DKV_LDS<D>];
    EaTile it;
    if (ea_place(p, p.plan.k_tiles, p.plan.k_splits, p.plan.k_each, it)) ea_dkv<D>(p, it, lds);
}
// Both, where a sequence and kv head is one tile of each.  APART: two workgroups for one, of which the second makes the rows' delta for itself; otherwise one, dQ first.
// A chain of waits while CUs are free, and work once they are not: us apart and in one, 8, 256 and 512 of them, 77 queries over 33 keys of 64 features 9.7 / 12.5, 12.3 / 13.3, 19.3 / 16.8; 128 over 128 of
// 128 features 17.4 / 23.2, 26.8 / 28.1, 49.4 / 42.5.  (A launch each, the first of these forward and backward: 26.2 us, and 24.3 in one.)
template <int D, bool APART>
__global__ __launch_bounds__(256, 2) void ll_encoder_small_backward_kernel(const EncParams p) {
    __shared__ __attribute__((aligned(256))) char lds[EA_DKV_LDS<D>];
    EaTile it;
    if (!ea_place(p, 1, 1, 0, it)) return;
    if constexpr (APART) {
        if (blockIdx.y == 0) {
            ea_dq<D, 4>(p, it, lds);
            return;
        }
        ea_dq<D, 3>(p, it, lds);
    } else {
        ea_dq<D, 0>(p, it, lds);
    }
    ea_wait<0>();                                // lse and delta are on their way to the cache that this workgroup's waves share
    __syncthreads();
    ea_dkv<D>(p, it, lds);
}

// Both in one launch, side by side, behind one that left the rows' delta: two products more, and no dK/dV that waits for dQ on a chip that is half empty.  us so and one after the other (workgroups of dQ and dK/dV without
// splits), 64 features: 8 heads of 1000 over 400 (64 + 32) 32 / 42, 64 of 300 over 300 (192 + 192) 25 / 31, 16 of 1000 over 1000 (128 + 128) 50 / 55, 12 of 3000 over 512 (288 + 48) 58 / 55, 24 of 2000 over 2000
// (384 + 384) 151 / 136; 128 features: 43 / 55, 36 / 44, 71 / 75, 89 / 79, 241 / 208.  Where delta has runs, with the launch that adds them up: 128 features, 8 heads of 1000 over 1000 55 / 62, 2 of 500 over 10000
// 60 / 77.
template <int D, int PASS>
__global__ __launch_bounds__(256, 2) void ll_encoder_both_kernel(const EncParams p, unsigned q_grid) {
    __shared__ __attribute__((aligned(256))) char lds[EA_DKV_LDS<D>];
    EaTile it;
    if (blockIdx.x < q_grid) {
        if (ea_place(p, p.plan.q_tiles, p.plan.q_splits, p.plan.q_each, it)) ea_dq<D, PASS>(p, it, lds);
    } else {
        if (ea_place(p, p.plan.k_tiles, p.plan.k_splits, p.plan.k_each, it, blockIdx.x - q_grid)) ea_dkv<D>(p, it, lds);
    }
}

// Adds up the rows' delta of several runs: a thread a row.
__global__ __launch_bounds__(256) void ll_encoder_delta_kernel(const EncParams p) {
    const unsigned r = blockIdx.x * 256 + threadIdx.x, unit = r / ENC_ROWS, in = r - unit * ENC_ROWS, of = unit / unsigned(p.plan.q_tiles);
    const int tile = int(unit - of * p.plan.q_tiles), seq = p.by_kv_heads.of(of), head = int(of) - seq * p.kv_heads;
    if (seq >= p.n_seqs) return;
    const EncSpan qs = enc_span(p.cu_q, nullptr, seq, p.n_seqs, p.n_q, p.max_q);
    if (int64_t(tile) * ENC_ROWS + in >= int64_t(qs.n) * p.by_group.d) return;
    const EaRow row = ea_query_row(p, qs, head, tile * ENC_ROWS + in);
    const int64_t at = int64_t(row.head) * p.n_q + row.token;
    float delta = 0.f;
#pragma unroll 8
    for (int s = 0; s < p.plan.q_splits; ++s) delta += p.part_d[(int64_t(unit) * p.plan.q_splits + s) * ENC_ROWS + in];
    *reinterpret_cast<ea_f32x2*>(p.side + 2 * at) = ea_f32x2{p.lse[at] * EA_LOG2E, delta};
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
    const int64_t heads = int64_t(p.n_seqs) * p.kv_heads;
    if (p.plan.few) hipLaunchKernelGGL(ll_encoder_few_kernel<D>, dim3(unsigned(heads * p.plan.splits)), dim3(256), 0, s, p);
    else hipLaunchKernelGGL(ll_encoder_forward_kernel<D>, dim3(unsigned(ea_grid(heads, p.plan.tiles, p.plan.splits, p.plan.each))), dim3(256), 0, s, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.plan.splits == 1) return e;
    const int64_t tile = p.plan.few ? ENC_FEW_ROWS : ENC_ROWS, rows = std::min(tile, int64_t(p.by_group.d) * p.max_q);
    if (p.plan.splits <= EA_FEW_SPLITS) {
        const int64_t groups = (heads * p.plan.tiles * rows * (D / 8) + 255) / 256;
        hipLaunchKernelGGL(ll_encoder_join_rows_kernel<D>, dim3(unsigned(groups)), dim3(256), 0, s, p, int(rows));
    } else {
        hipLaunchKernelGGL(ll_encoder_join_kernel<D>, dim3(unsigned(heads * p.plan.tiles * rows)), dim3(256), 0, s, p, int(rows));
    }
    return hipGetLastError();
}
hipError_t launch_encoder_forward(const EncParams& p, hipStream_t s) { return p.D == 128 ? ea_forward<128>(p, s) : ea_forward<64>(p, s); }

template <int D>
static hipError_t ea_backward(const EncParams& p, hipStream_t s) {
    const int64_t heads = int64_t(p.n_seqs) * p.kv_heads;
    const EncWay way = enc_backward_way(p.plan, heads, p.n_q, p.n_k);
    if (way == ENC_WAY_SMALL) {
        const unsigned grid = unsigned(ea_grid(heads, 1, 1, 0));
        if (heads <= EA_APART) hipLaunchKernelGGL((ll_encoder_small_backward_kernel<D, true>), dim3(grid, 2), dim3(256), 0, s, p);
        else hipLaunchKernelGGL((ll_encoder_small_backward_kernel<D, false>), dim3(grid), dim3(256), 0, s, p);
        return hipGetLastError();
    }
    const unsigned q_grid = unsigned(ea_grid(heads, p.plan.q_tiles, p.plan.q_splits, p.plan.q_each));
    const unsigned k_grid = unsigned(ea_grid(heads, p.plan.k_tiles, p.plan.k_splits, p.plan.k_each));
    const bool together = way == ENC_WAY_TOGETHER;
    hipError_t e = hipSuccess;
    if (together) {
        const bool whole = p.plan.q_splits == 1;
        if (whole) hipLaunchKernelGGL((ll_encoder_dq_kernel<D, 3>), dim3(q_grid), dim3(256), 0, s, p);
        else hipLaunchKernelGGL((ll_encoder_dq_kernel<D, 1>), dim3(q_grid), dim3(256), 0, s, p);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
        if (!whole) {
            hipLaunchKernelGGL(ll_encoder_delta_kernel, dim3(unsigned((heads * p.plan.q_tiles * ENC_ROWS + 255) / 256)), dim3(256), 0, s, p);
            e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        if (whole) hipLaunchKernelGGL((ll_encoder_both_kernel<D, 5>), dim3(q_grid + k_grid), dim3(256), 0, s, p, q_grid);
        else hipLaunchKernelGGL((ll_encoder_both_kernel<D, 6>), dim3(q_grid + k_grid), dim3(256), 0, s, p, q_grid);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (p.n_q > 0 && !together) {
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
    if (p.n_k > 0 && !together) {
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
