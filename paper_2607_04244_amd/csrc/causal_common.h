// Device-side parts that the causal attentions share (causal.hip over the bf16 cache, kv4.hip
// over the 4-bit one): a workgroup's work, key ranges, partial results and output rows.
// Header-only, inline.
#pragma once

#include "target_common.h"

namespace qlin {

typedef float v16f __attribute__((ext_vector_type(16)));

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));

constexpr float kNegInf = -__builtin_huge_valf();
constexpr uint32_t kBf16OnePair = 0x3F803F80u;       // bf16 (1.0, 1.0)

// Both lanes of the pair {l, l ^ 16} (l ^ 32) get the same result.
__device__ inline float pair16_max(float v) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float pair32_max(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float pair16_sum(float v) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ inline float pair32_sum(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// As load_lds_x16 (device_common.h) from a scalar address plus a 32-bit offset in bytes, to an
// LDS byte address.
__device__ inline void load_lds_s16(const uint16_t *base, uint32_t off, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(lds), "v"(off), "s"(base) : "memory", "m0");
}
__device__ inline void load_lds_v16(const uint16_t *src, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" :: "s"(lds), "v"(src) : "memory", "m0");
}
__device__ inline void load_lds_s16_nt(const uint16_t *base, uint32_t off, uint32_t lds) {      // for data a call reads once
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" :: "s"(lds), "v"(off), "s"(base) : "memory", "m0");
}

__device__ inline uint32_t cvt_pk_f16(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f{lo, hi}), v2h));       // round to nearest even
}
__device__ inline float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
__device__ inline int exponent_of(float x) { return (int)(__float_as_uint(x) >> 23 & 0xFFu) - 127; }
// Exponent of the largest value of what is brought below 2^15, in f16's range: products of two
// such scales, and their inverses, are powers that fp32 has.
__device__ inline int f16_exponent(float top) { return min(max(exponent_of(top), -56), 56); }

__device__ inline float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// The row tile (of R packed rows) that work item idx is, among all sequences' tiles: its
// sequence and its number in it; false past the last.  The tiles that see the most keys come
// first, in kClasses classes of equal steps of keys up to max_len (a tile with the longest
// walk that starts late ends late: packed prompts of 1 to 2048 tokens 125 us in the order of
// the rows, 113 in this one).  By the whole wave: a class's tiles of 64 sequences at a time are
// summed up.
constexpr int kClasses = 8;

// Inclusive sum over the lanes by DPP: within rows of 16, then across them.
__device__ inline int lanes_upto(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);     // row_shr 1, 2, 4, 8
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);     // lane 15 to the next row: rows 1, 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);     // lane 31 to rows 2, 3
    return v;
}
__device__ inline bool find_tile(const CausalArgs &a, int idx, int R, int lane, Seq &s, int &tile) {
    if (a.b.n_seq == 1) {                                // no order to find out
        s = load_seq(a.b, 0);
        tile = (s.rows * a.G + R - 1) / R - 1 - idx;
        return tile >= 0;
    }
    for (int i = 0; i < a.b.n_seq; i += 64) {
        Seq own{};
        int tiles = 0;
        if (i + lane < a.b.n_seq) {                      // the sequences' data, a lane each
            own = load_seq(a.b, i + lane);
            tiles = (own.rows * a.G + R - 1) / R;
        }
        // tiles whose first token is at class c's lower bound or later, and not in class c + 1
        int upper = tiles;
        const float per_token = (float)a.G / (float)R, step = (float)a.max_len / kClasses;
        for (int c = kClasses - 1; c >= 0; --c) {
            const float at = ((float)c * step - (float)own.p0) * per_token;
            const int lower = c == 0 ? 0 : min(max((int)fminf(at, 1e9f), 0), upper);
            const int sum = lanes_upto(upper - lower), total = __builtin_amdgcn_readlane(sum, 63);
            if (idx < total) {
                const int l = __popcll(__ballot(sum <= idx));
                // the class's last tile of the sequence first
                tile = __builtin_amdgcn_readlane(upper, l) - 1 - (idx - __builtin_amdgcn_readlane(sum - (upper - lower), l));
                s = lane_value(own, l);
                return true;
            }
            idx -= total;
            upper = lower;
        }
    }
    return false;
}

// A row tile's part of the work, the same in every kernel.
struct Work {
    Seq s;
    int h, split;
    int r0, rows;               // packed rows [r0, r0 + rows) of the sequence
    int i0, rem;                // r0 = i0 G + rem
    int hi;                     // keys [0, hi) that some row of the tile sees
    int64_t at;                 // token 0 of head h: elements, or rows of a 4-bit cache
    const uint16_t *k, *v;      // there, in a cache of bf16
};

// x / G for the x < 64 + 128 that a tile's rows reach (exact for x G < 2^32)
__device__ inline int token_of(const CausalArgs &a, int x) { return a.G == 1 ? x : (int)__umulhi((uint32_t)x, a.inv_g); }

__device__ inline int64_t uniform(int64_t v) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
    return (int64_t)((uint64_t)hi << 32 | lo);
}

// Workgroup (x, y): key range y of item x = tile number * heads + head.  Workgroups go to the 8 XCDs
// in turn, x first: with a multiple of 8 heads all work on one head is on one XCD, and its
// keys are shared in that XCD's L2.  SEVERAL: one_tile may be more than 1 (the division takes the
// kernels that cannot have that 0.1 to 0.2 us).
template <int R, bool SEVERAL = false>
__device__ inline bool find_work(const CausalArgs &a, int lane, int split, Work &w) {
    const int item = gn_chunk(blockIdx.x, a.Hkv, a.inv_heads, a.heads_shift);
    w.h = blockIdx.x - item * a.Hkv;
    w.split = split;
    int tile = 0;
    if (a.one_tile) {
        int b = item;
        if (SEVERAL && a.one_tile > 1) {
            b = item / a.one_tile;
            tile = a.one_tile - 1 - (item - b * a.one_tile);
        }
        if (b >= a.b.n_seq) return false;
        w.s = load_seq(a.b, b);
    } else {
        // where all workgroups run at once, two a compute unit, a long one goes with a short one
        const int half = (a.tiles + 1) / 2, idx = a.pairs && item >= half ? a.tiles - 1 - (item - half) : item;
        if (!find_tile(a, idx, R, lane, w.s, tile)) return false;
    }
    w.r0 = tile * R;
    w.rows = min(R, w.s.rows * a.G - w.r0);
    if (w.rows <= 0) return false;
    w.i0 = w.r0 / a.G;
    w.rem = w.r0 - w.i0 * a.G;
    w.hi = w.s.L > 0 ? max(w.s.p0 + w.i0 + token_of(a, w.rem + w.rows - 1) + 1, 0) : 0;
    // the same in every lane: scalars
    w.s.slot0 = uniform(w.s.slot0);
    w.s.row0 = __builtin_amdgcn_readfirstlane(w.s.row0);
    w.s.p0 = __builtin_amdgcn_readfirstlane(w.s.p0);
    w.s.L = __builtin_amdgcn_readfirstlane(w.s.L);
    w.r0 = __builtin_amdgcn_readfirstlane(w.r0);
    w.rows = __builtin_amdgcn_readfirstlane(w.rows);
    w.hi = __builtin_amdgcn_readfirstlane(w.hi);
    w.i0 = __builtin_amdgcn_readfirstlane(w.i0);
    w.rem = __builtin_amdgcn_readfirstlane(w.rem);
    w.at = w.s.slot0 * a.b.tok + (int64_t)w.h * a.b.head;
    w.k = a.k + w.at;
    w.v = a.v + w.at;
    return true;
}

// Packed row x of the tile: its token in the sequence and its query head.
struct RowOf { int i, hq; };
__device__ inline RowOf row_of(const CausalArgs &a, const Work &w, int x) {
    const int t = token_of(a, w.rem + x);
    return RowOf{w.i0 + t, w.h * a.G + w.rem + x - t * a.G};
}
__device__ inline int64_t row_at(const Work &w, const RowOf &r, int64_t stride) {
    return (int64_t)(w.s.row0 + r.i) * stride + r.hq * kHeadDim;
}
// The steps [first, end) of a key range, of `all` steps in ranges of at least a.least: as few
// ranges as hold them (used), the last ones of a.S empty.
struct Range { int first, end, used; };
__device__ inline Range range_of(const CausalArgs &a, int all, int split) {
    const int per = max((all + a.S - 1) / a.S, a.least);
    return Range{split * per, min((split + 1) * per, all), (all + per - 1) / per};
}

// log2 of a step's keys, for the join, which a division by them would take 0.15 to 0.4 us.
constexpr int shift_of(int keys) { return keys > 1 ? 1 + shift_of(keys / 2) : 0; }

// Partial results: for each item and range the tile's sums as the matrix cores leave them, in
// units of 64 lanes x 4 values (1 KiB, one store of a wave), and (maximum, sum of weights) of
// its rows.
template <int R>
__device__ inline float *unit_at(const CausalArgs &a, int split, int unit) {
    return a.ws_o + (((int64_t)blockIdx.x * a.S + split) * (R / 2) + unit) * 256;
}
template <int R>
__device__ inline float2 *row_ml(const CausalArgs &a, int split, int row) {
    return (float2 *)a.ws_ml + ((int64_t)blockIdx.x * a.S + split) * R + row;
}

// A row's sums are rescaled only when its maximum has grown by more than a factor 2^kLazy of
// the weights: up to there the weights just exceed 1, with the same relative rounding.  Each row
// goes by its own maximum, and a careful pass by the same steps, so that not a bit of a row
// depends on what lies behind its token.
constexpr float kLazy = 8.0f;

// E of a row whose weights p are multiplied by a size s of each key and rounded to f16: they are
// held as p 2^-E, so that p s stays in range (p at most 2^kLazy, s 2^-E below 2^7).  limit: the
// size from which E has to grow.  E is at least -80, so that the sum of 2^28 weights stays in
// fp32; sizes below 2^-94 lose bits.
struct StepScale {
    float e = 0.0f, limit = 0.0f;
    // What the row's sums are multiplied by for a size `most` above the limit.
    __device__ inline float raise(float most) {
        if (!(most > limit)) return 1.0f;
        const int to = min(max(exponent_of(most) - 4, -80), 100), from = (int)e;
        e = (float)to;
        limit = power_of_two(to + 7);
        return __builtin_ldexpf(1.0f, from - to);
    }
};

// The sums of W waves, each relative to its own maximum, as one: returns (maximum, sum of
// weights) and the values in acc.
template <int W>
__device__ inline float2 merged(const float2 *ml, int ml_stride, const v4f *sums, int stride, float c, v4f &acc) {
    float M = kNegInf;
#pragma unroll
    for (int i = 0; i < W; ++i) M = fmaxf(M, ml[i * ml_stride].x);
    const float mu = M == kNegInf ? 0.0f : M;
    float l = 0.0f;
    acc = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < W; ++i) {
        const float2 e = ml[i * ml_stride];
        const float f = exp2_hw((e.x - mu) * c);
        l += e.y * f;
        acc += sums[i * stride] * f;
    }
    return make_float2(M, l);
}

// Four dimensions of an output row from their sums and the sum of weights.
__device__ inline void store_out(const CausalArgs &a, const Work &w, const RowOf &row, int d, const v4f &acc, float l) {
    uint2 y = {};
    if (w.s.L > 0 && w.s.p0 + row.i >= 0) {
        const float inv = 1.0f / l;
        y = make_uint2(cvt_pk_bf16(acc[0] * inv, acc[1] * inv), cvt_pk_bf16(acc[2] * inv, acc[3] * inv));
    }
    *(uint2 *)(a.out + row_at(w, row, a.out_stride) + d) = y;
}

}  // namespace qlin
