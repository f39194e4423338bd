// Causal attention with grouped heads over the key/value cache
// (qlin_causal_attention in include/qlin_target.h).
//
// The G query heads of a key/value head share its keys, so the rows of a matrix product
// are (new token i, head g) packed as r = i G + g: a tile of rows spans few tokens, the
// keys are read once for all G heads, and a single token still fills G rows.  Row r sees
// the keys j <= p0 + r / G.  Scores come out transposed, S^T = K Q^T, with a row's keys
// down the registers of a lane (pair): the softmax needs one or two lane exchanges, and
// the weights are already the B operand of O^T += V^T P^T, whose A operand the
// transposing LDS read takes from V as it lies in the cache.
//
//   k_causal_few<RT>   up to 16 RT rows (RT = 1, 2, 4: one token, draft blocks): bound by
//       the cache's bytes.  Four waves, each with units of 32 keys and LDS of its own, two
//       units in flight, no barrier until the waves' sums are merged.
//   k_causal_prompt    128 rows, 32 a wave, 64-key tiles shared by four waves: bound by
//       the matrix cores and the softmax between them.
//   k_causal_combine   joins key ranges, in order.
//
// Softmax statistics are fp32.  Weights are rounded to bf16 once (the operand) and the
// sum adds the rounded weights.
//
// Values behind a row's token are multiplied by a weight of zero, which an infinity or
// NaN among them survives.  A pass whose sums come out not finite is therefore repeated
// with every row's own keys only (`careful`): the values of later keys as zeros, one token
// of the tile at a time.  The usual pass pays a test of its sums at the end.
#include "target_common.h"

#include <type_traits>

namespace qlin {

namespace {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef short v4s_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4s_t lds_v4s;

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

// Transposing LDS read: within 16 lanes, lane i receives element i & 3 of the 8-byte
// chunks that lanes 4 j + (i >> 2), j = 0 .. 3, address.
__device__ inline v4s_t lds_read_tr(const void *p) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s *)(const __attribute__((address_space(3))) void *)p);
}

// K and V in LDS: 16-byte unit c of key kk at kk * 16 + (c ^ (kk & 15)); reads of one
// unit of 16 keys, and the transposing reads, meet different banks.
__device__ inline int key_unit(int kk, int c) { return kk * 16 + (c ^ (kk & 15)); }

// As load_lds_x16 (device_common.h) from a scalar address plus a 32-bit offset in bytes.
__device__ inline void load_lds_s16(const uint16_t *base, uint32_t off, const uint4 *lds_dst) {
    asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(lds_addr(lds_dst)), "v"(off), "s"(base) : "memory", "m0");
}
__device__ inline void load_lds_s16_nt(const uint16_t *base, uint32_t off, const uint4 *lds_dst) {
    asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, %2 nt" :: "s"(lds_addr(lds_dst)), "v"(off), "s"(base) : "memory", "m0");
}

__device__ inline float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// The row tile (of R packed rows) that work item idx is, among all sequences' tiles in
// order: its sequence (-1: past the last) and its number in it.  By the whole wave: tiles
// of 64 sequences at a time are summed up.
struct Tile { int b, t; };
__device__ inline Tile find_tile(const CausalArgs &a, int idx, int R, int lane) {
    for (int i = 0; i < a.b.n_seq; i += 64) {
        int own = 0;
        if (i + lane < a.b.n_seq) {
            const int r0 = min(max(a.b.new_start[i + lane], 0), a.b.rows);
            const int n = min(max(a.b.new_start[i + lane + 1], r0), a.b.rows) - r0;
            own = (min(n, a.b.max_new) * a.G + R - 1) / R;
        }
        int sum = own;                                   // inclusive sum over the lanes
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int v = __shfl_up(sum, o);
            sum += lane >= o ? v : 0;
        }
        const int total = __shfl(sum, 63);
        if (idx < total) {
            const int at = __popcll(__ballot(sum <= idx));
            return Tile{i + at, idx - (__shfl(sum, at) - __shfl(own, at))};
        }
        idx -= total;
    }
    return Tile{-1, 0};
}

// Work item -> (key/value head, rest).  Workgroup b runs on XCD b % 8: with a multiple of 8
// heads, all work on one head is on one XCD and shares the head's keys in its L2.
__device__ inline void split_item(int blk, int Hkv, int &h, int &rest) {
    if ((Hkv & 7) == 0) {
        const int q = blk >> 3, n = Hkv >> 3;
        rest = q / n;
        h = (blk & 7) + 8 * (q - rest * n);
    } else {
        rest = blk / Hkv;
        h = blk - rest * Hkv;
    }
}

// A row tile's part of the work, the same in both kernels.
struct Work {
    Seq s;
    int h, split;
    int r0, rows;               // packed rows [r0, r0 + rows) of the sequence
    int hi;                     // keys [0, hi) that some row of the tile sees
    const uint16_t *k, *v;      // token 0 of head h
};

__device__ inline int64_t uniform(int64_t v) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
    return (int64_t)((uint64_t)hi << 32 | lo);
}

template <int R>
__device__ inline bool find_work(const CausalArgs &a, int item, int lane, Work &w) {
    int rest;
    split_item(item, a.Hkv, w.h, rest);
    const int idx = rest / a.S;
    w.split = rest - idx * a.S;
    Tile t{idx, 0};
    if (a.one_tile) {                                     // one tile a sequence
        if (idx >= a.b.n_seq) return false;
    } else {
        t = find_tile(a, a.tiles - 1 - idx, R, lane);     // late tiles, which see the most keys, first
        if (t.b < 0) return false;
    }
    w.s = load_seq(a.b, t.b);
    w.r0 = t.t * R;
    w.rows = min(R, w.s.rows * a.G - w.r0);
    if (w.rows <= 0) return false;
    w.hi = w.s.L > 0 ? max(w.s.p0 + (w.r0 + w.rows - 1) / a.G + 1, 0) : 0;
    // the same in every lane: scalars
    w.s.slot0 = uniform(w.s.slot0);
    w.s.row0 = __builtin_amdgcn_readfirstlane(w.s.row0);
    w.s.p0 = __builtin_amdgcn_readfirstlane(w.s.p0);
    w.s.L = __builtin_amdgcn_readfirstlane(w.s.L);
    w.r0 = __builtin_amdgcn_readfirstlane(w.r0);
    w.rows = __builtin_amdgcn_readfirstlane(w.rows);
    w.hi = __builtin_amdgcn_readfirstlane(w.hi);
    const int64_t at = w.s.slot0 * a.b.tok + (int64_t)w.h * a.b.head;
    w.k = a.k + at;
    w.v = a.v + at;
    return true;
}

// Element offset of packed row r's query (stride a.q_stride) or output.
__device__ inline int64_t row_at(const CausalArgs &a, const Work &w, int r, int64_t stride) {
    const int i = r / a.G;
    return (int64_t)(w.s.row0 + i) * stride + (int64_t)(w.h * a.G + r - i * a.G) * kHeadDim;
}
// Index of packed row r among all rows and heads (partial results).
__device__ inline int64_t row_index(const CausalArgs &a, const Work &w, int r) {
    const int i = r / a.G;
    return (int64_t)(w.s.row0 + i) * a.Hq + w.h * a.G + (r - i * a.G);
}

// The values of keys [key, key + 4) and [key2, key2 + 4), without those behind `last`.
__device__ inline v8bf values_up_to(v4s_t lo, v4s_t hi, int key, int key2, int last) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (key + e > last) lo[e] = 0;
        if (key2 + e > last) hi[e] = 0;
    }
    return __builtin_bit_cast(v8bf, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// ---------------------------------------------------------------- few rows

constexpr int kFewWaves = 4, kFewKeys = 32, kFewStages = 2;
constexpr int kFewUnits = kFewKeys * kHeadDim / 8;        // 16-byte units of one unit's K or V (512)

template <int RT>
__global__ __launch_bounds__(kFewWaves * 64, 1) void k_causal_few(CausalArgs a) {
    constexpr int R = 16 * RT;
    __shared__ __attribute__((aligned(16))) uint4 ring[kFewWaves][kFewStages][2][kFewUnits];   // then the waves' sums
    __shared__ float2 ml[kFewWaves][R];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int g = lane >> 4, r = lane & 15;
    Work w;
    if (!find_work<R>(a, blockIdx.x, lane, w)) return;

    // units of this key range, and of this wave: u0 + wave, u0 + wave + 4, ...
    const int units = (w.hi + kFewKeys - 1) / kFewKeys;
    const int per = max((units + a.S - 1) / a.S, kFewWaves);
    const int u0 = w.split * per, u1 = min(u0 + per, units);

    // byte offsets of a lane in four keys, for each of the four swizzles
    uint32_t off[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) off[j] = 2u * ((uint32_t)g * (uint32_t)a.b.tok + 8u * (r ^ (4 * j + g)));
    auto issue = [&](int u, int st) {
        if ((u + 1) * kFewKeys <= w.hi) {
            const int64_t at = (int64_t)u * kFewKeys * a.b.tok;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                load_lds_s16_nt(w.k + at + 4 * j * a.b.tok, off[j & 3], &ring[wave][st][0][j * 64]);
                load_lds_s16_nt(w.v + at + 4 * j * a.b.tok, off[j & 3], &ring[wave][st][1][j * 64]);
            }
            return;
        }
#pragma unroll 1
        for (int j = 0; j < 8; ++j) {                    // the last, partial unit: its last key again
            const int x = j * 64 + lane, kk = x >> 4, c = (x & 15) ^ (kk & 15);
            const int64_t off = (int64_t)min(u * kFewKeys + kk, w.hi - 1) * a.b.tok + 8 * c;
            load_lds_x16_nt(w.k + off, &ring[wave][st][0][j * 64]);
            load_lds_x16_nt(w.v + off, &ring[wave][st][1][j * 64]);
        }
    };

    // queries: B operand, row r of row tile t
    v8bf qf[RT][4];
    int last[RT];                                             // last key that the row sees
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        const int rr = w.r0 + min(16 * t + r, w.rows - 1);
        last[t] = w.s.p0 + rr / a.G;
        const uint16_t *qp = a.q + row_at(a, w, rr, a.q_stride) + 8 * g;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) qf[t][ks] = *(const v8bf *)(qp + 32 * ks);
    }
    const int first_last = w.s.p0 + w.r0 / a.G;               // keys up to here are seen by every row

    float m[RT], l[RT];
    v4f o[RT][8];
    auto run = [&](auto mode) {                               // whether the sums came out finite
        constexpr bool careful = decltype(mode)::value;
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            m[t] = kNegInf;
            l[t] = 0.0f;
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) o[t][dt] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        }
        int st = 0;
        if (u0 + wave < u1) issue(u0 + wave, 0);
        if (u0 + wave + kFewWaves < u1) issue(u0 + wave + kFewWaves, 1);
        for (int u = u0 + wave; u < u1; u += kFewWaves, st ^= 1) {
            // this unit's 16 loads have landed; the next unit's may be in flight
            if (u + kFewWaves < u1) asm volatile("s_waitcnt vmcnt(16)" ::: "memory");
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            const uint4 *kb = ring[wave][st][0], *vb = ring[wave][st][1];
            const int key0 = u * kFewKeys;
            const bool masked = key0 + kFewKeys - 1 > first_last;
            v4f sc[RT][2];
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
                for (int t = 0; t < RT; ++t) sc[t][kt] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int ks = 0; ks < 4; ++ks) {
                    const v8bf kf = *(const v8bf *)&kb[key_unit(16 * kt + r, 4 * ks + g)];
#pragma unroll
                    for (int t = 0; t < RT; ++t)
                        sc[t][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[t][ks], sc[t][kt], 0, 0, 0);
                }
            }
            v8bf pb[RT];
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                if (masked) {
#pragma unroll
                    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            sc[t][kt][i] = key0 + 16 * kt + 4 * g + i <= last[t] ? sc[t][kt][i] : kNegInf;
                }
                float mt = fmaxf(fmaxf(fmaxf(sc[t][0][0], sc[t][0][1]), fmaxf(sc[t][0][2], sc[t][0][3])),
                                 fmaxf(fmaxf(sc[t][1][0], sc[t][1][1]), fmaxf(sc[t][1][2], sc[t][1][3])));
                mt = pair32_max(pair16_max(mt));
                const float mn = fmaxf(m[t], mt);
                const float muc = (mn == kNegInf ? 0.0f : mn) * a.c;
                if (__ballot(mn != m[t])) {
                    const float alpha = exp2_hw(__builtin_fmaf(m[t], a.c, -muc));
                    l[t] *= alpha;
#pragma unroll
                    for (int dt = 0; dt < 8; ++dt) o[t][dt] *= alpha;
                    m[t] = mn;
                }
                uint32_t pw[4];
                float ls = 0.0f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float e0 = exp2_hw(__builtin_fmaf(sc[t][i >> 1][2 * (i & 1)], a.c, -muc));
                    const float e1 = exp2_hw(__builtin_fmaf(sc[t][i >> 1][2 * (i & 1) + 1], a.c, -muc));
                    pw[i] = cvt_pk_bf16(e0, e1);
                    ls = dot2(pw[i], kBf16OnePair, ls);
                }
                l[t] += ls;
                pb[t] = __builtin_bit_cast(v8bf, v4u{pw[0], pw[1], pw[2], pw[3]});
            }
            const int q = r & 3, kr = 4 * g + (r >> 2);        // keys of elements 0..3; + 16 for 4..7
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) {
                const int c = 2 * dt + (q >> 1), off = 8 * (q & 1);
                const v4s_t lo4 = lds_read_tr((const char *)&vb[key_unit(kr, c)] + off);
                const v4s_t hi4 = lds_read_tr((const char *)&vb[key_unit(kr + 16, c)] + off);
                if (careful && masked) {
#pragma unroll
                    for (int t = 0; t < RT; ++t) {
                        const int i0 = (w.r0 + min(16 * t, w.rows - 1)) / a.G, i1 = (w.r0 + min(16 * t + 15, w.rows - 1)) / a.G;
                        v4f sum = o[t][dt];
                        for (int i = i0; i <= i1; ++i) {
                            const int p = w.s.p0 + i;
                            const v4f x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(values_up_to(lo4, hi4, key0 + 4 * g, key0 + 16 + 4 * g, p),
                                                                                  pb[t], o[t][dt], 0, 0, 0);
                            sum = last[t] == p ? x : sum;
                        }
                        o[t][dt] = sum;
                    }
                } else {
                    const v8bf vf = __builtin_bit_cast(v8bf, __builtin_shufflevector(lo4, hi4, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                    for (int t = 0; t < RT; ++t) o[t][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pb[t], o[t][dt], 0, 0, 0);
                }
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // this slot has been read
            if (u + 2 * kFewWaves < u1) issue(u + 2 * kFewWaves, st);
        }
        float bad = 0.0f;                                        // NaN if any sum is not finite
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int dt = 0; dt < 8; ++dt)
#pragma unroll
                for (int i = 0; i < 4; ++i) bad = __builtin_fmaf(o[t][dt][i], 0.0f, bad);
        return !__ballot(bad != 0.0f);
    };
    if (!run(std::false_type{})) run(std::true_type{});
#pragma unroll
    for (int t = 0; t < RT; ++t) l[t] = pair32_sum(pair16_sum(l[t]));

    // the waves' sums through LDS, in the matrix cores' order
    __syncthreads();
    v4f *sums = (v4f *)&ring[0][0][0][0];
    static_assert(sizeof(ring) >= sizeof(v4f) * kFewWaves * RT * 8 * 64, "the sums fit the ring");
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        if (g == 0) ml[wave][16 * t + r] = make_float2(m[t], l[t]);
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) sums[((wave * RT + t) * 8 + dt) * 64 + lane] = o[t][dt];
    }
    __syncthreads();
    for (int x = wave; x < RT * 8; x += kFewWaves) {
        const int t = x >> 3, dt = x & 7, row = 16 * t + r;
        if (row >= w.rows) continue;
        float M = kNegInf;
#pragma unroll
        for (int i = 0; i < kFewWaves; ++i) M = fmaxf(M, ml[i][row].x);
        const float mu = M == kNegInf ? 0.0f : M;
        float ls = 0.0f;
        v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < kFewWaves; ++i) {
            const float2 e = ml[i][row];
            const float f = exp2_hw((e.x - mu) * a.c);
            ls += e.y * f;
            acc += sums[((i * RT + t) * 8 + dt) * 64 + lane] * f;
        }
        const int rr = w.r0 + row, d = 16 * dt + 4 * g;
        if (a.S == 1) {
            const bool none = w.s.L == 0 || w.s.p0 + rr / a.G < 0;
            uint2 y = {};
            if (!none) y = make_uint2(cvt_pk_bf16(acc[0] / ls, acc[1] / ls), cvt_pk_bf16(acc[2] / ls, acc[3] / ls));
            *(uint2 *)(a.out + row_at(a, w, rr, a.out_stride) + d) = y;
        } else {
            const int64_t at = row_index(a, w, rr) * a.S + w.split;
            *(v4f *)(a.ws_o + at * kHeadDim + d) = acc;
            if (dt == 0 && g == 0) *(float2 *)(a.ws_ml + 2 * at) = make_float2(M, ls);
        }
    }
}

// ---------------------------------------------------------------- many rows

constexpr int kPromptWaves = 4, kPromptRows = 32 * kPromptWaves, kPromptKeys = 64, kPromptStages = 2;
constexpr int kPromptUnits = kPromptKeys * kHeadDim / 8;      // 16-byte units of a K or V tile (1024)
constexpr float kLazy = 8.0f;                                 // see below

__global__ __launch_bounds__(kPromptWaves * 64, 2) void k_causal_prompt(CausalArgs a) {
    __shared__ __attribute__((aligned(16))) uint4 ring[kPromptStages][2][kPromptUnits];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int hi = lane >> 5, r = lane & 31;
    Work w;
    if (!find_work<kPromptRows>(a, blockIdx.x, lane, w)) return;

    const int tiles = (w.hi + kPromptKeys - 1) / kPromptKeys;
    const int per = (tiles + a.S - 1) / a.S;
    const int t0 = w.split * per, t1 = min(t0 + per, tiles);

    const uint32_t off = 2u * ((uint32_t)(lane >> 4) * (uint32_t)a.b.tok + 8u * ((lane & 15) ^ ((4 * wave + (lane >> 4)) & 15)));
    auto issue = [&](int t) {
        const int st = t & 1;
        if ((t + 1) * kPromptKeys <= w.hi) {
            const int64_t at = ((int64_t)t * kPromptKeys + 4 * wave) * a.b.tok;
#pragma unroll
            for (int j = 0; j < kPromptUnits / (kPromptWaves * 64); ++j) {
                load_lds_s16(w.k + at + 16 * j * a.b.tok, off, &ring[st][0][(j * kPromptWaves + wave) * 64]);
                load_lds_s16(w.v + at + 16 * j * a.b.tok, off, &ring[st][1][(j * kPromptWaves + wave) * 64]);
            }
            return;
        }
#pragma unroll 1
        for (int j = 0; j < kPromptUnits / (kPromptWaves * 64); ++j) {
            const int x = (j * kPromptWaves + wave) * 64 + lane, kk = x >> 4, c = (x & 15) ^ (kk & 15);
            const int64_t off = (int64_t)min(t * kPromptKeys + kk, w.hi - 1) * a.b.tok + 8 * c;
            load_lds_x16(w.k + off, &ring[st][0][(j * kPromptWaves + wave) * 64]);
            load_lds_x16(w.v + off, &ring[st][1][(j * kPromptWaves + wave) * 64]);
        }
    };

    const int rw0 = min(32 * wave, w.rows - 1), rw1 = min(32 * wave + 31, w.rows - 1);
    const int rr = w.r0 + min(32 * wave + r, w.rows - 1);
    const int last = w.s.p0 + rr / a.G;                                   // last key this row sees
    const int wave_first = w.s.p0 + (w.r0 + rw0) / a.G, wave_last = w.s.p0 + (w.r0 + rw1) / a.G;
    const bool live = 32 * wave < w.rows;                                 // this wave has rows
    v8bf qf[8];
    {
        const uint16_t *qp = a.q + row_at(a, w, rr, a.q_stride) + 8 * hi;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) qf[ks] = *(const v8bf *)(qp + 16 * ks);
    }

    float m, l;
    v16f o[4];
    auto run = [&](auto mode) {                                  // whether the sums came out finite
        constexpr bool careful = decltype(mode)::value;
        m = kNegInf;
        l = 0.0f;
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[dt][i] = 0.0f;
        if (t0 < t1) issue(t0);
        for (int t = t0; t < t1; ++t) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            lds_barrier();                    // tile t is in LDS, and every wave is done with tile t - 1
            if (t + 1 < t1) issue(t + 1);
            const int key0 = t * kPromptKeys;
            if (!live || key0 > wave_last) continue;
            const bool masked = key0 + kPromptKeys - 1 > wave_first;
            const uint4 *kb = ring[t & 1][0], *vb = ring[t & 1][1];
            v16f sc[2];
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[kt][i] = 0.0f;
#pragma unroll
                for (int ks = 0; ks < 8; ++ks) {
                    const v8bf kf = *(const v8bf *)&kb[key_unit(32 * kt + r, 2 * ks + hi)];
                    sc[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[ks], sc[kt], 0, 0, 0);
                }
            }
            if (masked) {
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        sc[kt][i] = key0 + 32 * kt + 8 * (i >> 2) + 4 * hi + (i & 3) <= last ? sc[kt][i] : kNegInf;
            }
            float mt = kNegInf;
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int i = 0; i < 16; ++i) mt = fmaxf(mt, sc[kt][i]);
            mt = pair32_max(mt);
            // The sums are rescaled only when a maximum has grown by more than 2^kLazy: up to
            // there the weights just exceed 1, with the same relative rounding.
            if (__ballot(mt * a.c > __builtin_fmaf(m, a.c, kLazy))) {
                const float mn = fmaxf(m, mt);
                const float alpha = exp2_hw((m - (mn == kNegInf ? 0.0f : mn)) * a.c);
                l *= alpha;
#pragma unroll
                for (int dt = 0; dt < 4; ++dt) o[dt] *= alpha;
                m = mn;
            }
            const float muc = (m == kNegInf ? 0.0f : m) * a.c;
            uint32_t pw[2][8];
            float ls = 0.0f;
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float e0 = exp2_hw(__builtin_fmaf(sc[kt][2 * i], a.c, -muc));
                    const float e1 = exp2_hw(__builtin_fmaf(sc[kt][2 * i + 1], a.c, -muc));
                    pw[kt][i] = cvt_pk_bf16(e0, e1);
                    ls = dot2(pw[kt][i], kBf16OnePair, ls);
                }
            l += ls;
            const int q = lane & 3, kr = 4 * hi + ((lane >> 2) & 3), c0 = 2 * ((lane >> 4) & 1) + (q >> 1), off = 8 * (q & 1);
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const uint32_t *ps = &pw[s >> 1][4 * (s & 1)];
                const v8bf pb = __builtin_bit_cast(v8bf, v4u{ps[0], ps[1], ps[2], ps[3]});
#pragma unroll
                for (int dt = 0; dt < 4; ++dt) {
                    const v4s_t lo4 = lds_read_tr((const char *)&vb[key_unit(16 * s + kr, 4 * dt + c0)] + off);
                    const v4s_t hi4 = lds_read_tr((const char *)&vb[key_unit(16 * s + 8 + kr, 4 * dt + c0)] + off);
                    if (careful && masked) {
                        v16f sum = o[dt];
                        for (int p = wave_first; p <= wave_last; ++p) {
                            const v16f x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                                values_up_to(lo4, hi4, key0 + 16 * s + 4 * hi, key0 + 16 * s + 8 + 4 * hi, p), pb, o[dt], 0, 0, 0);
#pragma unroll
                            for (int i = 0; i < 16; ++i) sum[i] = last == p ? x[i] : sum[i];
                        }
                        o[dt] = sum;
                    } else {
                        const v8bf vf = __builtin_bit_cast(v8bf, __builtin_shufflevector(lo4, hi4, 0, 1, 2, 3, 4, 5, 6, 7));
                        o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pb, o[dt], 0, 0, 0);
                    }
                }
            }
        }
        float bad = 0.0f;                                        // NaN if any sum is not finite
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int i = 0; i < 16; ++i) bad = __builtin_fmaf(o[dt][i], 0.0f, bad);
        return !__syncthreads_or(bad != 0.0f);                   // also: every wave is done with the ring
    };
    if (!run(std::false_type{})) run(std::true_type{});
    l = pair32_sum(l);
    if (32 * wave + r >= w.rows) return;
    if (a.S == 1) {
        const bool none = w.s.L == 0 || last < 0;
        uint16_t *op = a.out + row_at(a, w, rr, a.out_stride);
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {                        // dimensions 32 dt + 8 i + 4 hi .. + 3
                uint2 y = {};
                if (!none) y = make_uint2(cvt_pk_bf16(o[dt][4 * i] / l, o[dt][4 * i + 1] / l),
                                          cvt_pk_bf16(o[dt][4 * i + 2] / l, o[dt][4 * i + 3] / l));
                *(uint2 *)(op + 32 * dt + 8 * i + 4 * hi) = y;
            }
    } else {
        const int64_t at = row_index(a, w, rr) * a.S + w.split;
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *(v4f *)(a.ws_o + at * kHeadDim + 32 * dt + 8 * i + 4 * hi) =
                    v4f{o[dt][4 * i], o[dt][4 * i + 1], o[dt][4 * i + 2], o[dt][4 * i + 3]};
        if (hi == 0) *(float2 *)(a.ws_ml + 2 * at) = make_float2(m, l);
    }
}

// ---------------------------------------------------------------- joining key ranges

// Eight groups of 32 lanes, four dimensions a lane; P groups share a row, each every P-th
// range, and are merged through LDS in group order.
template <int P>
__global__ __launch_bounds__(256) void k_causal_combine(CausalArgs a) {
    constexpr int kBatch = 4;
    __shared__ float2 gml[8];
    __shared__ float4 go[8][32];
    static_assert(P >= 2, "the two groups of a wave share a row");
    const int grp = threadIdx.x >> 5, l = threadIdx.x & 31, lane = threadIdx.x & 63;
    const int part = grp % P;
    int h, rest;                                      // the XCD that wrote the head's partials
    split_item(blockIdx.x, a.Hkv, h, rest);
    const int64_t x = (int64_t)rest * (8 / P) + grp / P;            // (row, head of the group)
    const int64_t mrow = x / a.G;
    const int b = find_seq(a.b, (int)min(mrow, (int64_t)a.b.rows), lane);      // one row a wave
    bool on = mrow < a.b.rows && b < a.b.n_seq;
    Seq s = {};
    if (on) {
        s = load_seq(a.b, b);
        on = mrow >= s.row0 && mrow < s.row0 + s.rows;
    }
    const int hq = h * a.G + (int)(x - mrow * a.G);
    const int64_t at = (mrow * a.Hq + hq) * a.S;
    float m = kNegInf, ls = 0.0f;
    float4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    auto fold = [&](float m2, float l2, const float4 &v) {
        const float M = fmaxf(m, m2), mu = M == kNegInf ? 0.0f : M;
        const float f1 = exp2_hw((m - mu) * a.c), f2 = exp2_hw((m2 - mu) * a.c);
        m = M;
        ls = ls * f1 + l2 * f2;
        acc.x = acc.x * f1 + v.x * f2;
        acc.y = acc.y * f1 + v.y * f2;
        acc.z = acc.z * f1 + v.z * f2;
        acc.w = acc.w * f1 + v.w * f2;
    };
    if (on) {
        for (int s0 = part; s0 < a.S; s0 += P * kBatch) {
            float2 e[kBatch];
            float4 v[kBatch];
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                const int si = s0 + P * i;
                e[i] = si < a.S ? *(const float2 *)(a.ws_ml + 2 * (at + si)) : make_float2(kNegInf, 0.0f);
                v[i] = si < a.S ? *(const float4 *)(a.ws_o + (at + si) * kHeadDim + 4 * l) : float4{0.0f, 0.0f, 0.0f, 0.0f};
            }
#pragma unroll
            for (int i = 0; i < kBatch; ++i) fold(e[i].x, e[i].y, v[i]);
        }
    }
    if (l == 0) gml[grp] = make_float2(m, ls);
    go[grp][l] = acc;
    __syncthreads();
    if (part != 0 || !on) return;
#pragma unroll
    for (int i = 1; i < P; ++i) fold(gml[grp + i].x, gml[grp + i].y, go[grp + i][l]);
    const bool none = s.L == 0 || s.p0 + (mrow - s.row0) < 0;
    uint2 y = {};
    if (!none) y = make_uint2(cvt_pk_bf16(acc.x / ls, acc.y / ls), cvt_pk_bf16(acc.z / ls, acc.w / ls));
    *(uint2 *)(a.out + mrow * a.out_stride + (int64_t)hq * kHeadDim + 4 * l) = y;
}

}  // namespace

const char *causal_kernel_name(int rt) {
    return rt == 1 ? "k_causal_few<1>" : rt == 2 ? "k_causal_few<2>" : rt == 4 ? "k_causal_few<4>" : "k_causal_prompt";
}

hipError_t launch_causal(const CausalArgs &a, int rt, hipStream_t st) {
    const dim3 grid((unsigned)((int64_t)a.tiles * a.Hkv * a.S));
    if (rt == 1) hipLaunchKernelGGL(k_causal_few<1>, grid, dim3(kFewWaves * 64), 0, st, a);
    else if (rt == 2) hipLaunchKernelGGL(k_causal_few<2>, grid, dim3(kFewWaves * 64), 0, st, a);
    else if (rt == 4) hipLaunchKernelGGL(k_causal_few<4>, grid, dim3(kFewWaves * 64), 0, st, a);
    else hipLaunchKernelGGL(k_causal_prompt, grid, dim3(kPromptWaves * 64), 0, st, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.S == 1) return e;
    const int64_t pairs = (int64_t)a.b.rows * a.G;                 // (row, head of a group)
    const int P = a.S >= 5 ? 8 : a.S >= 3 ? 4 : 2;
    const dim3 cgrid((unsigned)((pairs * P + 7) / 8 * a.Hkv));
    if (P == 8) hipLaunchKernelGGL(k_causal_combine<8>, cgrid, dim3(256), 0, st, a);
    else if (P == 4) hipLaunchKernelGGL(k_causal_combine<4>, cgrid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL(k_causal_combine<2>, cgrid, dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace qlin
