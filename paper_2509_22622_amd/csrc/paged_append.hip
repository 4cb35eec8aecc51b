// ll_paged_append: the new tokens of many sequences, turned by the rotary embedding and written into their pages (paged.h), and their
// queries, turned and scaled, beside them.  Per pair (a, b) of features and angle t = position * theta^(-2 i / rope_dim):
//     a' = a cos t - b sin t,  b' = b cos t + a sin t;   q' = bf16(R q * log2(e) / sqrt(D)),  K' = R k,  V = v.
// One pass over q, k, v: bound by memory where there are tokens enough, by the chain of loads that finds a token's place (offsets,
// length, page: three round trips, taken while the rows themselves are on their way) where there are few.
//
// A workgroup takes a tile of 256 / (D / 16) tokens and some heads.  A thread has one token and 16 of its features, in two 16-byte pieces
// that hold eight whole pairs in either order of pairs.  Lanes run over a token's threads first, so that eight neighbouring lanes take (and, of the
// queries, store) 128 bytes of one row: with lanes over 16 tokens first, whose stores of K are contiguous instead, every load asks for 64
// pieces of 16 bytes by themselves (12284 rows x (32 + 2 x 8) heads x 128: 86 us, and 77 now, 3.9 TB/s).  Angles are made once per workgroup, in
// revolutions and in double (position * frequency passes 2^24 in long contexts; what remains after the whole turns are taken off is
// good to 2^-24), then sine and cosine in float.
// V is transposed through LDS: four tokens that make up one quad of a granule go out as 16-byte stores; at a sequence's ends, where a quad
// is shared with tokens of another call, number by number.
#include "paged.h"

namespace ll {

typedef unsigned short pa_u16x8 __attribute__((ext_vector_type(8)));
typedef unsigned pa_u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned pa_u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 pa_bf16x8 __attribute__((ext_vector_type(8)));
typedef float pa_f32x8 __attribute__((ext_vector_type(8)));

// Largest s with cu[s] <= row; the caller checks that the row is one of sequence s.
__device__ __forceinline__ int pa_sequence_of(const int* cu, int n_seqs, int row) {
    int lo = 0, hi = n_seqs;                 // the answer lies in [lo, hi)
    while (hi - lo > 1) {
        const int mid = lo + (hi - lo) / 2;
        if (cu[mid] <= row) lo = mid;
        else hi = mid;
    }
    return lo;
}

// To E4M3: to nearest, clamped to the largest number (beyond it the conversion makes NaN); NaN stays NaN.
__device__ __forceinline__ float pa_clamp8(float x) { return x != x ? x : fminf(fmaxf(x, -448.0f), 448.0f); }
__device__ __forceinline__ unsigned pa_pack8(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(pa_clamp8(a), pa_clamp8(b), 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(pa_clamp8(c), pa_clamp8(d), w, true);
    return unsigned(w);
}

template <int D, int FMT>
__global__ __launch_bounds__(256) void ll_paged_append_kernel(const PagedAppendParams p) {
    constexpr int ITEMS = D / 16;                     // threads per token
    constexpr int TT = 256 / ITEMS;                   // tokens per tile
    constexpr int NB = FMT == 0 ? 2 : 1;
    constexpr int VROW = D * NB + 16;                 // bytes of a row of V in LDS
    constexpr int CU_NEAR = 256;                      // offsets that are searched in LDS: one round trip instead of one a halving
    __shared__ float2 cs[TT][D / 2 + 1];              // cosine and sine: thread `item` of a token has [ITEMS e + item], e = 0..7
    __shared__ __attribute__((aligned(16))) unsigned char v_rows[TT * VROW];
    __shared__ int64_t base[TT];                      // granule's byte offset in the layer's pool (kv head 0); -1: not stored
    __shared__ int slot[TT];                          // token inside the granule
    __shared__ signed char quad[TT];                  // 1: first of a whole quad of this tile, -2: no row of the call's, -1: any other
    __shared__ signed char task[TT];                  // tokens that stand for a store of V: whole quads' first ones, and those on their own
    __shared__ int n_tasks;
    __shared__ double turns[D / 2];
    __shared__ int cu_near[CU_NEAR];

    const int tid = threadIdx.x;
    const int row0 = blockIdx.x * p.tile_rows, rows = min(p.tile_rows, p.s.n_tokens - row0);   // of the tile's TT at most
    const int tok = tid / ITEMS, item = tid % ITEMS;
    const int row = row0 + tok;
    const bool live = tok < rows;
    const int n_units = p.q ? p.kv_heads + (p.q_heads + 1) / 2 : p.kv_heads;   // a kv head's K and V, or two heads of q
    const int unit0 = blockIdx.y * p.heads_per_group, unit1 = min(unit0 + p.heads_per_group, n_units);
    // The thread's two pieces of 8 features, and whether they are turned: pieces ITEMS apart, or where pairs are halves apart those that hold
    // the two features of its eight pairs.
    const int rot_items = p.rope_pairs / 8;
    int p0 = item, p1 = item + ITEMS;
    bool turned0 = 4 * p0 < p.rope_pairs, turned1 = 4 * p1 < p.rope_pairs;
    if (p.halves) {
        turned0 = turned1 = item < rot_items;
        p0 = turned0 ? item : 2 * item;
        p1 = turned0 ? item + rot_items : p0 + 1;
    }

    auto load = [&](int unit, pa_u16x8 (&x)[4]) {
        const uint16_t *a, *b;
        bool has_b = true;
        if (unit < p.kv_heads) {
            a = p.k + row * p.k_stride + unit * D;
            b = p.v + row * p.v_stride + unit * D;
        } else {
            const int h = 2 * (unit - p.kv_heads);
            a = p.q + row * p.q_stride + h * D;
            b = a + D;
            has_b = h + 1 < p.q_heads;
        }
        x[0] = *reinterpret_cast<const pa_u16x8*>(a + 8 * p0);
        x[1] = *reinterpret_cast<const pa_u16x8*>(a + 8 * p1);
        if (has_b) {
            x[2] = *reinterpret_cast<const pa_u16x8*>(b + 8 * p0);
            x[3] = *reinterpret_cast<const pa_u16x8*>(b + 8 * p1);
        }
    };
    pa_u16x8 x[4] = {};
    if (live) load(unit0, x);
    if (tid < p.rope_pairs) turns[tid] = p.turns[tid];
    const bool near = p.s.cu && p.s.n_seqs < CU_NEAR;
    if (near) {
        if (tid <= p.s.n_seqs) cu_near[tid] = p.s.cu[tid];
        __syncthreads();
    }

    // Where each token goes: its place, and its page, which is on its way while the angles are made.
    int page = -1;
    int64_t place = -1;
    bool of_none = false;                             // a row of no sequence: nothing of it is stored
    if (tid < rows) {
        const int r = row0 + tid;
        int seq = r;
        int64_t from_end = 1;
        if (p.s.cu) {
            seq = near ? pa_sequence_of(cu_near, p.s.n_seqs, r) : pa_sequence_of(p.s.cu, p.s.n_seqs, r);
            const int first = near ? cu_near[seq] : p.s.cu[seq], end = near ? cu_near[seq + 1] : p.s.cu[seq + 1];
            of_none = r < first || r >= end;
            from_end = int64_t(end) - r;
        }
        if (!of_none) {
            place = int64_t(p.s.lens[seq]) - from_end;
            if (place >= 0 && place < int64_t(p.s.cols) * p.s.page_tokens) page = p.s.table[seq * p.s.table_stride + p.s.by_page.of(uint32_t(place))];
        }
        // its angle's source, behind its cosines and sines
        if (p.rope_pairs) {
            int pos[3] = {int(place), 0, 0};
            if (p.positions && !of_none)
                for (int a = 0; a < p.axes; ++a) pos[a] = p.positions[int64_t(r) * p.axes + a];
            cs[tid][D / 2] = make_float2(__int_as_float(pos[0]), __int_as_float(pos[1]));
            reinterpret_cast<int*>(&v_rows[tid * 16])[0] = pos[2];
        }
    }
    __syncthreads();
    for (int i = tid; i < TT * p.rope_pairs; i += 256) {
        const int t = i / p.rope_pairs, pair = i - t * p.rope_pairs;
        if (t >= rows) break;
        int pos = __float_as_int(cs[t][D / 2].x);
        if (p.axes == 3 && pair >= p.axis1) pos = pair < p.axis2 ? __float_as_int(cs[t][D / 2].y) : reinterpret_cast<const int*>(&v_rows[t * 16])[0];
        const double circles = double(pos) * turns[pair];
        float s, c;
        sincospif(2.0f * float(circles - rint(circles)), &s, &c);
        const int slot_of = p.halves ? pair % 8 * ITEMS + pair / 8 : (pair % 4 + (pair / 4 < ITEMS ? 0 : 4)) * ITEMS + pair / 4 % ITEMS;
        cs[t][slot_of] = make_float2(c, s);
    }
    if (tid < 64) {                                   // the first wave has all the tile's tokens
        int64_t at = -1;
        if (page >= 0 && page < p.s.n_pages)
            at = page * paged_page_bytes(p.kv_heads, p.s.page_tokens, D, FMT) + int64_t((int(place) - int(p.s.by_page.of(uint32_t(place))) * p.s.page_tokens) / PAGED_GRANULE) * (PAGED_GRANULE * D * NB);
        // A quad is whole if its four tokens are consecutive rows of this tile in consecutive places of one granule (pages are whole granules).
        const int in = int(place & 15);
        bool whole = at >= 0 && (in & 3) == 0 && tid + 3 < TT;
#pragma unroll
        for (int e = 1; e < 4; ++e) {
            const int64_t next = __shfl_down(at, e);
            const int next_in = __shfl_down(in, e);
            whole = whole && next == at && next_in == in + e;
        }
        const uint64_t first = __ballot(whole), inside = first << 1 | first << 2 | first << 3;
        const uint64_t tasks = __ballot(at >= 0) & ~inside;
        if (tid < TT) {
            base[tid] = at;
            slot[tid] = in;
            quad[tid] = whole ? 1 : of_none ? -2 : -1;
            if (tasks >> tid & 1) task[__popcll(tasks & ((uint64_t(1) << tid) - 1))] = (signed char)tid;
        }
        if (tid == 0) n_tasks = __popcll(tasks);
    }
    __syncthreads();
    const bool mine = live && quad[tok] != -2;

    auto turn = [&](const pa_u16x8& a, const pa_u16x8& b, float scale, float (&oa)[8], float (&ob)[8]) {
        float fa[8], fb[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            fa[e] = __uint_as_float(unsigned(a[e]) << 16);
            fb[e] = __uint_as_float(unsigned(b[e]) << 16);
        }
        if (p.halves ? turned0 : turned0 || turned1) {
            float2 w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = cs[tok][ITEMS * e + item];
            if (p.halves) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float re = fa[e], im = fb[e];
                    fa[e] = __builtin_fmaf(re, w[e].x, -(im * w[e].y));
                    fb[e] = __builtin_fmaf(im, w[e].x, re * w[e].y);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float re = fa[2 * e], im = fa[2 * e + 1];
                    if (turned0) {
                        fa[2 * e] = __builtin_fmaf(re, w[e].x, -(im * w[e].y));
                        fa[2 * e + 1] = __builtin_fmaf(im, w[e].x, re * w[e].y);
                    }
                    re = fb[2 * e], im = fb[2 * e + 1];
                    if (turned1) {
                        fb[2 * e] = __builtin_fmaf(re, w[4 + e].x, -(im * w[4 + e].y));
                        fb[2 * e + 1] = __builtin_fmaf(im, w[4 + e].x, re * w[4 + e].y);
                    }
                }
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            oa[e] = fa[e] * scale;
            ob[e] = fb[e] * scale;
        }
    };
    auto rounded = [](const float (&f)[8]) {
        pa_f32x8 v;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = f[e];
        return __builtin_bit_cast(pa_u32x4, __builtin_convertvector(v, pa_bf16x8));
    };

    const int64_t v_region = int64_t(p.s.page_tokens) * D * NB;
    for (int unit = unit0; unit < unit1; ++unit) {
        pa_u16x8 y[4] = {};
        if (live && unit + 1 < unit1) load(unit + 1, y);
        if (unit < p.kv_heads) {
            char* const k_image = p.pool + unit * 2 * v_region;
            float a[8], b[8];
            turn(x[0], x[1], FMT == 0 ? 1.0f : p.k_scale, a, b);
            if (mine && base[tok] >= 0) {
                char* const to = k_image + base[tok];
                if constexpr (FMT == 0) {
                    *reinterpret_cast<pa_u32x4*>(to + 2 * paged_k_at(0, slot[tok], 8 * p0)) = rounded(a);
                    *reinterpret_cast<pa_u32x4*>(to + 2 * paged_k_at(0, slot[tok], 8 * p1)) = rounded(b);
                } else {
                    *reinterpret_cast<pa_u32x2*>(to + paged_k_at(1, slot[tok], 8 * p0)) = pa_u32x2{pa_pack8(a[0], a[1], a[2], a[3]), pa_pack8(a[4], a[5], a[6], a[7])};
                    *reinterpret_cast<pa_u32x2*>(to + paged_k_at(1, slot[tok], 8 * p1)) = pa_u32x2{pa_pack8(b[0], b[1], b[2], b[3]), pa_pack8(b[4], b[5], b[6], b[7])};
                }
            }
            __syncthreads();                          // the last head's rows of V have been read
            unsigned char* const mine_at = v_rows + tok * VROW;
            if constexpr (FMT == 0) {
                *reinterpret_cast<pa_u16x8*>(mine_at + 16 * p0) = x[2];
                *reinterpret_cast<pa_u16x8*>(mine_at + 16 * p1) = x[3];
            } else {
                float f[16];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    f[e] = __uint_as_float(unsigned(x[2][e]) << 16) * p.v_scale;
                    f[8 + e] = __uint_as_float(unsigned(x[3][e]) << 16) * p.v_scale;
                }
                *reinterpret_cast<pa_u32x2*>(mine_at + 8 * p0) = pa_u32x2{pa_pack8(f[0], f[1], f[2], f[3]), pa_pack8(f[4], f[5], f[6], f[7])};
                *reinterpret_cast<pa_u32x2*>(mine_at + 8 * p1) = pa_u32x2{pa_pack8(f[8], f[9], f[10], f[11]), pa_pack8(f[12], f[13], f[14], f[15])};
            }
            __syncthreads();
            // 16 bytes of V's image: quad of token t, piece c, lane r
            constexpr int PIECES = D * NB / 64, EACH = 4 / NB;     // features of a lane and piece
            for (int i = tid; i < n_tasks * PIECES * 16; i += 256) {
                const int r = i & 15, c = i / 16 % PIECES, t = task[i / (16 * PIECES)];
                char* const to = k_image + v_region + base[t] + NB * paged_v_at(FMT, slot[t] & ~3, c * 16 * EACH + r);
                if (quad[t] == 1) {
                    pa_u32x4 o;
                    if constexpr (FMT == 0) {
                        const unsigned char* from = v_rows + t * VROW + 2 * (32 * c + r);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const unsigned char* f = from + (e & 1) * 2 * VROW + (e >> 1) * 32;
                            o[e] = *reinterpret_cast<const unsigned short*>(f) | unsigned(*reinterpret_cast<const unsigned short*>(f + VROW)) << 16;
                        }
                    } else {
                        const unsigned char* from = v_rows + t * VROW + 64 * c + r;
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            o[e] = unsigned(from[16 * e]) | unsigned(from[16 * e + VROW]) << 8 | unsigned(from[16 * e + 2 * VROW]) << 16 |
                                   unsigned(from[16 * e + 3 * VROW]) << 24;
                    }
                    *reinterpret_cast<pa_u32x4*>(to) = o;
                } else {
                    const int j = slot[t] & 3;
#pragma unroll
                    for (int e = 0; e < EACH; ++e) {
                        if constexpr (FMT == 0)
                            reinterpret_cast<unsigned short*>(to)[4 * e + j] = *reinterpret_cast<const unsigned short*>(v_rows + t * VROW + 2 * (32 * c + 16 * e + r));
                        else
                            reinterpret_cast<unsigned char*>(to)[4 * e + j] = v_rows[t * VROW + 64 * c + 16 * e + r];
                    }
                }
            }
        } else if (mine) {
            const int h = 2 * (unit - p.kv_heads);
            uint16_t* const to = p.q_out + row * p.q_out_stride + h * D;
            float a[8], b[8];
            turn(x[0], x[1], p.q_scale, a, b);
            *reinterpret_cast<pa_u32x4*>(to + 8 * p0) = rounded(a);
            *reinterpret_cast<pa_u32x4*>(to + 8 * p1) = rounded(b);
            if (h + 1 < p.q_heads) {
                turn(x[2], x[3], p.q_scale, a, b);
                *reinterpret_cast<pa_u32x4*>(to + D + 8 * p0) = rounded(a);
                *reinterpret_cast<pa_u32x4*>(to + D + 8 * p1) = rounded(b);
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = y[e];
    }
}

template <int D, int FMT>
static hipError_t launch(PagedAppendParams p, hipStream_t s) {
    constexpr int TT = 256 / (D / 16);
    const int units = p.q ? p.kv_heads + (p.q_heads + 1) / 2 : p.kv_heads;
    p.tile_rows = paged_tile_rows(p.s.n_tokens, units, TT);
    const int tiles = (p.s.n_tokens + p.tile_rows - 1) / p.tile_rows;
    p.heads_per_group = paged_units_per_group(tiles, units);
    hipLaunchKernelGGL((ll_paged_append_kernel<D, FMT>), dim3(unsigned(tiles), unsigned((units + p.heads_per_group - 1) / p.heads_per_group)), dim3(256), 0, s, p);
    return hipGetLastError();
}

hipError_t launch_paged_append(const PagedAppendParams& p, hipStream_t s) {
    if (p.s.n_tokens < 1) return hipSuccess;
    if (p.fmt == 0) return p.D == 128 ? launch<128, 0>(p, s) : launch<64, 0>(p, s);
    return p.D == 128 ? launch<128, 1>(p, s) : launch<64, 1>(p, s);
}

}  // namespace ll
