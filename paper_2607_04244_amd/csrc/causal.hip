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
//   k_causal_few       up to 16 rows (single tokens): bound by the cache's bytes.  Four waves,
//       each with units of 32 keys and LDS of its own, two units in flight, no barrier until
//       the waves' sums are merged.  64 tokens of 32 / 8 heads over 4096 keys each: 174 to
//       180 us, 6.0 to 6.2 TB/s; one token over 8192 keys 7.1 us and 2.9 for the join.
//   k_causal_mid<NR>   up to 32 NR rows (draft blocks): the cache's bytes, then the products.
//       16 tokens over 8192 keys: 12.2 to 12.5 us in a trace of kernels (10.8 by its own clock, from
//       its first instruction to its last store), of which the keys take 5.4 at that rate; 3.9
//       for the join, and 14.0 to 15.1 the call in a graph.
//   k_causal_prompt<H> 128 rows, 32 a wave, 32 keys a step for four waves: bound by the matrix
//       cores and the softmax between them.  8192 tokens: 509 to 550 us on different cards,
//       1000 to 1080 TFLOP/s, where the library's large bf16 product reaches 1194.
//   k_causal_join      joins key ranges, in order: bound by the partial results' bytes.
// The kernel goes by the rows of the longest sequence (max_new G): a larger tile leaves more of
// the matrix cores' work unused, a smaller one reads the keys again for each tile.  Through few /
// mid<1> / mid<2> / prompt, 32 / 8 heads, us with the join: one sequence of 8192 keys, 1 new token
// 10.4 / 12.8 / 13.2 / 14.2, 4 tokens 11.6 / 12.3 / 12.7 / 14.0, 8 - / 13.1 / 13.3 / 14.6, 16
// - / - / 15.1 / 16.0; 32 sequences of 4096, 1 token 84 / 84 / 81 / 95, 8 - / 87 / 83 / 97, 16
// - / - / 90 / 98.  Between mid<1> and mid<2> the rows alone do not decide: at 8 tokens mid<1> is
// ahead where a workgroup walks up to 256 keys (1000 keys 9.0 / 9.7, 8 sequences of 1000 12.0 /
// 12.7) and behind where it walks more (2 of 8192 18.6 / 17.5, 8 of 4096 29.6 / 27.1).
//
// Softmax statistics are fp32.  Weights are rounded to bf16 once (the operand) and the
// sum adds the rounded weights.
//
// Values behind a row's token are multiplied by a weight of zero, which an infinity or
// NaN among them survives.  A pass whose sums come out not finite is therefore repeated
// with every row's own keys only (`careful`): the values of later keys as zeros, one token
// of the tile at a time.  The usual pass pays a test of its sums at the end.
#include "causal_common.h"

#include <type_traits>

namespace qlin {

namespace {

typedef short v4s_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4s_t lds_v4s;

// Transposing LDS read: within 16 lanes, lane i receives element i & 3 of the 8-byte
// chunks that lanes 4 j + (i >> 2), j = 0 .. 3, address.
__device__ inline v4s_t lds_read_tr(const void *p) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s *)(const __attribute__((address_space(3))) void *)p);
}

// K and V in LDS: the 16 units (16 bytes) of a key's row in an order that changes from key
// to key, so that what lanes read together meets different banks: for K, one unit of 16
// keys; for V by transposing reads, two units of 8 keys (16-wide products) or four of 4 keys
// (32-wide).  With K's order for V, 60 % of the prompt kernel's LDS cycles were conflicts.
__device__ inline int key_unit(int kk, int c) { return kk * 16 + (c ^ (kk & 15)); }
__device__ inline int few_value_unit(int kk, int c) { return kk * 16 + (c ^ (2 * (kk & 7))); }
__device__ inline int value_unit(int kk, int c) { return kk * 16 + (c ^ (4 * (kk & 3))); }

// The two 16-bit types of a cache: bf16, or f16 as a 4-bit cache is unpacked to.
struct InBf16 {
    typedef v8bf v8;
    static constexpr uint32_t kOnes = kBf16OnePair;
    static __device__ inline v16f product(v8 a, v8 b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
    static __device__ inline uint32_t pair(float lo, float hi) { return cvt_pk_bf16(lo, hi); }
    static __device__ inline float add(uint32_t p, float s) { return dot2(p, kOnes, s); }
};
struct InF16 {
    typedef v8h v8;
    static constexpr uint32_t kOnes = 0x3C003C00u;
    static __device__ inline v16f product(v8 a, v8 b, v16f c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
    static __device__ inline uint32_t pair(float lo, float hi) { return cvt_pk_f16(lo, hi); }
    static __device__ inline float add(uint32_t p, float s) {
        return __builtin_amdgcn_fdot2(__builtin_bit_cast(v2h, p), __builtin_bit_cast(v2h, kOnes), s, false);
    }
};

// The values of keys [key, key + 4) and [key2, key2 + 4), without those behind `last`.
__device__ inline v8bf values_up_to(v4s_t lo, v4s_t hi, int key, int key2, int last) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (key + e > last) lo[e] = 0;
        if (key2 + e > last) hi[e] = 0;
    }
    return __builtin_bit_cast(v8bf, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Whether a lane's sums are all finite: 0 x is 0 only then.  Four chains: one of 64 products in a
// row takes as long as a dozen matrix products.
template <int N, typename V>
__device__ inline bool all_finite(const V (&o)[N]) {
    constexpr int E = sizeof(V) / sizeof(float);
    float z[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int dt = 0; dt < N; ++dt)
#pragma unroll
        for (int i = 0; i < E; ++i) z[i & 3] = __builtin_fmaf(o[dt][i], 0.0f, z[i & 3]);
    return (z[0] + z[1]) + (z[2] + z[3]) == 0.0f;
}

// The weights' exponents s c - m c are fused products less a rounded m c: its rounding is in all of a
// row's weights alike and cancels, while |m c| is at most kFar and it is at most 1.  Above, where it
// could take all weights past their range, a careful pass takes (s - m) c, at the steps of the rows
// where that is so; a row that ever is there sends its tile through one, whatever lies behind it.
constexpr float kFar = 16777216.0f;

__device__ inline float exponent(float s, float c, float mu, float muc, bool far) {
    return far ? (s - mu) * c : __builtin_fmaf(s, c, -muc);
}

// ---------------------------------------------------------------- few rows

constexpr int kFewRows = 16, kFewWaves = 4, kFewKeys = 32, kFewStages = 2;
constexpr int kFewUnits = kFewKeys * kHeadDim / 8;        // 16-byte units of one unit's K or V (512)

__global__ __launch_bounds__(kFewWaves * 64, 1) void k_causal_few(CausalArgs a) {
    constexpr int R = kFewRows;
    __shared__ __attribute__((aligned(16))) uint4 ring[kFewWaves][kFewStages][2][kFewUnits];   // then the waves' sums
    __shared__ float2 ml[kFewWaves][R];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int g = lane >> 4, r = lane & 15;
    Work w;
    if (!find_work<R>(a, lane, blockIdx.y, w)) return;

    // units of this key range, and of this wave: u0 + wave, u0 + wave + 4, ...
    const Range range = range_of(a, (w.hi + kFewKeys - 1) / kFewKeys, w.split);
    if (a.S > 1 && w.split >= range.used) return;
    const int u0 = range.first, u1 = range.end;

    // byte offsets of a lane in four keys, for each order of their units
    uint32_t koff[4], voff[2];
#pragma unroll
    for (int j = 0; j < 4; ++j) koff[j] = 2u * ((uint32_t)g * (uint32_t)a.b.tok + 8u * (r ^ (4 * j + g)));
#pragma unroll
    for (int j = 0; j < 2; ++j) voff[j] = 2u * ((uint32_t)g * (uint32_t)a.b.tok + 8u * (r ^ (2 * (4 * j + g))));
    const uint32_t lds = lds_addr(ring[wave]);
    auto issue = [&](int u, int st) {
        const uint32_t to = lds + st * (2 * kFewUnits * 16);
        if ((u + 1) * kFewKeys <= w.hi) {
            const int64_t at = (int64_t)u * kFewKeys * a.b.tok;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                load_lds_s16_nt(w.k + at + 4 * j * a.b.tok, koff[j & 3], to + j * 1024);
                load_lds_s16_nt(w.v + at + 4 * j * a.b.tok, voff[j & 1], to + kFewUnits * 16 + j * 1024);
            }
            return;
        }
#pragma unroll 1
        for (int j = 0; j < 8; ++j) {                    // the last, partial unit: its last key again
            const int kk = 4 * j + g;
            const int64_t at = (int64_t)min(u * kFewKeys + kk, w.hi - 1) * a.b.tok;
            load_lds_v16(w.k + at + 8 * (r ^ (kk & 15)), to + j * 1024);
            load_lds_v16(w.v + at + 8 * (r ^ (2 * (kk & 7))), to + kFewUnits * 16 + j * 1024);
        }
    };

    // queries: B operand, row r
    const RowOf row = row_of(a, w, min(r, w.rows - 1));
    const int last = w.s.p0 + row.i;                          // last key that the row sees
    v8bf qf[4];
    {
        const uint16_t *qp = a.q + row_at(w, row, a.q_stride) + 8 * g;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) qf[ks] = *(const v8bf *)(qp + 32 * ks);
    }
    const int first_last = w.s.p0 + w.i0;                     // keys up to here are seen by every row

    float m, l;
    v4f o[8];
    auto run = [&](auto mode) {                               // whether the sums came out finite
        constexpr bool careful = decltype(mode)::value;
        m = kNegInf;
        l = 0.0f;
        uint64_t gone_far = 0;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) o[dt] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
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
            v4f sc[2];
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
                sc[kt] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int ks = 0; ks < 4; ++ks)
                    sc[kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*(const v8bf *)&kb[key_unit(16 * kt + r, 4 * ks + g)], qf[ks], sc[kt], 0, 0, 0);
            }
            if (masked) {
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) sc[kt][i] = key0 + 16 * kt + 4 * g + i <= last ? sc[kt][i] : kNegInf;
            }
            float mt = fmaxf(fmaxf(fmaxf(sc[0][0], sc[0][1]), fmaxf(sc[0][2], sc[0][3])),
                             fmaxf(fmaxf(sc[1][0], sc[1][1]), fmaxf(sc[1][2], sc[1][3])));
            mt = pair32_max(pair16_max(mt));
            const bool own = (mt - m) * a.c > kLazy;
            if (__ballot(own)) {
                const float mn = own ? mt : m;
                const float alpha = exp2_hw((m - (mn == kNegInf ? 0.0f : mn)) * a.c);
                l *= alpha;
#pragma unroll
                for (int dt = 0; dt < 8; ++dt) o[dt] *= alpha;
                m = mn;
                gone_far |= __ballot(m != kNegInf && fabsf(m * a.c) > kFar);
            }
            const float mu = m == kNegInf ? 0.0f : m, muc = mu * a.c;
            const bool far = careful && fabsf(muc) > kFar;
            uint32_t pw[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float e0 = exp2_hw(exponent(sc[i >> 1][2 * (i & 1)], a.c, mu, muc, far));
                const float e1 = exp2_hw(exponent(sc[i >> 1][2 * (i & 1) + 1], a.c, mu, muc, far));
                pw[i] = cvt_pk_bf16(e0, e1);
                l = dot2(pw[i], kBf16OnePair, l);
            }
            const v8bf pb = __builtin_bit_cast(v8bf, v4u{pw[0], pw[1], pw[2], pw[3]});
            const int q = r & 3, kr = 4 * g + (r >> 2);        // keys of elements 0..3; + 16 for 4..7
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) {
                const int c = 2 * dt + (q >> 1), off = 8 * (q & 1);
                const v4s_t lo4 = lds_read_tr((const char *)&vb[few_value_unit(kr, c)] + off);
                const v4s_t hi4 = lds_read_tr((const char *)&vb[few_value_unit(kr + 16, c)] + off);
                if (careful && masked) {
                    const int p1 = w.s.p0 + row_of(a, w, w.rows - 1).i;
                    v4f sum = o[dt];
                    for (int p = first_last; p <= p1; ++p) {
                        const v4f x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(values_up_to(lo4, hi4, key0 + 4 * g, key0 + 16 + 4 * g, p),
                                                                              pb, o[dt], 0, 0, 0);
                        sum = last == p ? x : sum;
                    }
                    o[dt] = sum;
                } else {
                    o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                        __builtin_bit_cast(v8bf, __builtin_shufflevector(lo4, hi4, 0, 1, 2, 3, 4, 5, 6, 7)), pb, o[dt], 0, 0, 0);
                }
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // this slot has been read
            if (u + 2 * kFewWaves < u1) issue(u + 2 * kFewWaves, st);
        }
        return !__ballot(!all_finite(o)) && !gone_far;
    };
    if (!run(std::false_type{})) run(std::true_type{});
    l = pair32_sum(pair16_sum(l));

    // the waves' sums through LDS, in the matrix cores' order
    __syncthreads();
    v4f *sums = (v4f *)&ring[0][0][0][0];
    static_assert(sizeof(ring) >= sizeof(v4f) * kFewWaves * 8 * 64, "the sums fit the ring");
    if (g == 0) ml[wave][r] = make_float2(m, l);
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) sums[(wave * 8 + dt) * 64 + lane] = o[dt];
    __syncthreads();
    if (r >= w.rows) return;
#pragma unroll
    for (int dt = wave; dt < 8; dt += kFewWaves) {
        v4f acc;
        const float2 e = merged<kFewWaves>(&ml[0][r], R, sums + dt * 64 + lane, 8 * 64, a.c, acc);
        const int d = 16 * dt + 4 * g;
        if (a.S == 1) {
            store_out(a, w, row, d, acc, e.y);
        } else {
            *(v4f *)(unit_at<R>(a, w.split, dt) + 4 * lane) = acc;
            if (dt == 0 && g == 0) *row_ml<R>(a, w.split, r) = e;
        }
    }
}

// ---------------------------------------------------------------- draft blocks

// 32 NR rows, NR = 1, 2: four waves for each 32 rows, a quarter of a step's 128 keys each, so
// that a key range of 256 keys (a 16-token block over 8192 keys on all compute units) is two
// steps, requested at once.  With four 16-row tiles in each of four waves the kernel took 15.0 us
// in a trace (12.4 so): its products waited for one another, with one wave a SIMD.
constexpr int kMidKeys = 128, kMidUnits = kMidKeys * kHeadDim / 8;

template <int NR>
__global__ __launch_bounds__(NR * 256, NR) void k_causal_mid(CausalArgs a) {
    constexpr int W = 4 * NR, R = 32 * NR;
    __shared__ __attribute__((aligned(16))) uint4 ring[2][2][kMidUnits];      // [stage][K, V], then the waves' sums
    __shared__ float2 ml[W][32];
    __shared__ int not_finite[W];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int hi = lane >> 5, r = lane & 31, rt = wave >> 2, ku = wave & 3;
    Work w;
    if (!find_work<R>(a, lane, blockIdx.y, w)) return;
    const Range range = range_of(a, (w.hi + kMidKeys - 1) / kMidKeys, w.split);
    if (a.S > 1 && w.split >= range.used) return;

    // a wave loads 4 keys at a time, W waves 4 W of a step
    const uint32_t koff = 2u * ((uint32_t)(lane >> 4) * (uint32_t)a.b.tok + 8u * ((lane & 15) ^ ((4 * wave + (lane >> 4)) & 15)));
    const uint32_t voff = 2u * ((uint32_t)(lane >> 4) * (uint32_t)a.b.tok + 8u * ((lane & 15) ^ (4 * (lane >> 4))));
    const uint32_t lds = lds_addr(ring) + wave * 1024;
    auto issue = [&](int t) {
        const uint32_t to = lds + (t & 1) * (2 * kMidUnits * 16);
        const int64_t at = ((int64_t)t * kMidKeys + 4 * wave) * a.b.tok;
        if ((t + 1) * kMidKeys <= w.hi) {
#pragma unroll
            for (int j = 0; j < kMidKeys / (4 * W); ++j) {
                load_lds_s16_nt(w.k + at + 4 * W * j * a.b.tok, koff, to + j * W * 1024);
                load_lds_s16_nt(w.v + at + 4 * W * j * a.b.tok, voff, to + kMidUnits * 16 + j * W * 1024);
            }
            return;
        }
#pragma unroll 1
        for (int j = 0; j < kMidKeys / (4 * W); ++j) {                // the last, partial step: its last key again
            const int kk = 4 * (j * W + wave) + (lane >> 4);
            const int64_t key = (int64_t)min(t * kMidKeys + kk, w.hi - 1) * a.b.tok;
            load_lds_v16(w.k + key + 8 * ((lane & 15) ^ (kk & 15)), to + j * W * 1024);
            load_lds_v16(w.v + key + 8 * ((lane & 15) ^ (4 * (kk & 3))), to + kMidUnits * 16 + j * W * 1024);
        }
    };

    const RowOf row = row_of(a, w, min(32 * rt + r, w.rows - 1));
    const int last = w.s.p0 + row.i;                                       // last key this row sees
    const int tile_first = __builtin_amdgcn_readfirstlane(w.s.p0 + row_of(a, w, min(32 * rt, w.rows - 1)).i);
    const int tile_last = __builtin_amdgcn_readfirstlane(w.s.p0 + row_of(a, w, min(32 * rt + 31, w.rows - 1)).i);
    v8bf qf[8];
    {
        const uint16_t *qp = a.q + row_at(w, row, a.q_stride) + 8 * hi;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) qf[ks] = *(const v8bf *)(qp + 16 * ks);
    }
    const int vk = 4 * hi + ((lane >> 2) & 3), vc = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);

    float m, l;
    v16f o[4];
    v4f *const sums = (v4f *)&ring[0][0][0];
    static_assert(sizeof(ring) >= sizeof(v4f) * W * 16 * 64, "the sums fit the ring");
    auto run = [&](auto mode) {                                  // whether the sums came out finite
        constexpr bool careful = decltype(mode)::value;
        m = kNegInf;
        l = 0.0f;
        uint64_t gone_far = 0;
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[dt][i] = 0.0f;
        if (range.first < range.end) issue(range.first);
        if (range.first + 1 < range.end) issue(range.first + 1);
        for (int t = range.first; t < range.end; ++t) {
            // this step's loads have landed; the next step's may be in flight
            if (t + 1 < range.end) asm volatile("s_waitcnt vmcnt(%0)" :: "n"(2 * kMidKeys / (4 * W)) : "memory");
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            lds_barrier();
            const int key0 = t * kMidKeys + 32 * ku;             // this wave's 32 keys
            if (key0 < w.hi && 32 * rt < w.rows) {
                const char *kb = (const char *)ring[t & 1][0] + ku * 8192, *vb = (const char *)ring[t & 1][1] + ku * 8192;
                v16f s;
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = 0.0f;
#pragma unroll
                for (int ks = 0; ks < 8; ++ks)
                    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const v8bf *)(kb + 16 * key_unit(r, 2 * ks + hi)), qf[ks], s, 0, 0, 0);
                const bool masked = key0 + 31 > tile_first;
                if (masked) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[i] = key0 + 8 * (i >> 2) + 4 * hi + (i & 3) <= last ? s[i] : kNegInf;
                }
                float mt = kNegInf;
#pragma unroll
                for (int i = 0; i < 16; ++i) mt = fmaxf(mt, s[i]);
                mt = pair32_max(mt);
                const bool own = (mt - m) * a.c > kLazy;
                if (__ballot(own)) {
                    const float mn = own ? mt : m;
                    const float alpha = exp2_hw((m - (mn == kNegInf ? 0.0f : mn)) * a.c);
                    l *= alpha;
#pragma unroll
                    for (int dt = 0; dt < 4; ++dt) o[dt] *= alpha;
                    m = mn;
                    gone_far |= __ballot(m != kNegInf && fabsf(m * a.c) > kFar);
                }
                const float mu = m == kNegInf ? 0.0f : m, muc = mu * a.c;
                const bool far = careful && fabsf(muc) > kFar;
                uint32_t p[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    p[i] = cvt_pk_bf16(exp2_hw(exponent(s[2 * i], a.c, mu, muc, far)), exp2_hw(exponent(s[2 * i + 1], a.c, mu, muc, far)));
                    l = dot2(p[i], kBf16OnePair, l);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int h = i >> 2, dt = i & 3;
                    const char *vp = vb + 16 * value_unit(16 * h + vk, 4 * dt + vc) + 8 * (lane & 1);
                    const v4s_t lo4 = lds_read_tr(vp), hi4 = lds_read_tr(vp + 8 * 256);
                    const v8bf pb = __builtin_bit_cast(v8bf, v4u{p[4 * h], p[4 * h + 1], p[4 * h + 2], p[4 * h + 3]});
                    if (careful && masked) {
                        v16f sum = o[dt];
#pragma unroll 1
                        for (int x = tile_first; x <= tile_last; ++x) {
                            const v16f y = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                                values_up_to(lo4, hi4, key0 + 16 * h + 4 * hi, key0 + 16 * h + 8 + 4 * hi, x), pb, o[dt], 0, 0, 0);
#pragma unroll
                            for (int j = 0; j < 16; ++j) sum[j] = last == x ? y[j] : sum[j];
                        }
                        o[dt] = sum;
                    } else {
                        o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                            __builtin_bit_cast(v8bf, __builtin_shufflevector(lo4, hi4, 0, 1, 2, 3, 4, 5, 6, 7)), pb, o[dt], 0, 0, 0);
                    }
                }
            }
            if (t + 2 < range.end) {
                lds_barrier();                                   // every wave is done with this stage
                issue(t + 2);
            }
        }
        lds_barrier();                                           // every wave is done with the ring
        // the four waves' sums of each 32 rows through LDS, in the matrix cores' order
        l = pair32_sum(l);
        if (hi == 0) ml[wave][r] = make_float2(m, l);
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                sums[(wave * 16 + dt * 4 + i) * 64 + lane] = v4f{o[dt][4 * i], o[dt][4 * i + 1], o[dt][4 * i + 2], o[dt][4 * i + 3]};
        const uint64_t bad = __ballot(!all_finite(o)) | gone_far;
        if (lane == 0) not_finite[wave] = bad != 0;
        lds_barrier();
        int any = 0;
#pragma unroll
        for (int i = 0; i < W; ++i) any |= not_finite[i];
        return any == 0;
    };
    if (!run(std::false_type{})) run(std::true_type{});
    if (32 * rt + r >= w.rows) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int x = 4 * ku + j;                                // unit of this row tile: dimensions 8 x + 4 hi .. + 3
        v4f acc;
        const float2 e = merged<4>(&ml[4 * rt][r], 32, sums + (rt * 64 + x) * 64 + lane, 16 * 64, a.c, acc);
        if (a.S == 1) {
            store_out(a, w, row, 8 * x + 4 * hi, acc, e.y);
        } else {
            *(v4f *)(unit_at<R>(a, w.split, rt * 16 + x) + 4 * lane) = acc;
            if (x == 0 && hi == 0) *row_ml<R>(a, w.split, 32 * rt + r) = e;
        }
    }
}

// ---------------------------------------------------------------- many rows

// Steps of 32 keys in a pipeline over three steps: while the softmax of step u runs on the
// vector unit, the matrix cores take the scores of step u + 1 and the weighted sums of step
// u - 1.  K and V each have a ring of four steps in LDS, filled by direct-to-LDS loads two
// steps ahead; one barrier for two steps.  Two workgroups a compute unit (64 KiB of LDS and
// 218 registers each), or, HALVES = 2, one of eight waves, four for each half of the keys, whose
// sums meet in LDS: where there is work for one workgroup a unit but not for two, that saves a
// split and its join (a prompt of 1185 tokens 35.0 us in two ranges, 26.8 so).
//
// A step has 16 products of 32 cycles and about 80 vector instructions of 5 cycles, which fit
// between the products (a product with 4 fma and 1 exp: 33.4 cycles at two waves a SIMD).
// Measured over 8192 tokens: matrix cores busy 52 % of the cycles, vector unit 38 %, LDS 25 %
// without conflicts, at 1.8 to 1.9 GHz: the clock of dense products, not the nominal 2.4.
// One step after the other, a barrier each: 567 us; as here 539, and 521 with the searches and
// divisions before the first step shortened.  Other orders of products, vector instructions
// and LDS reads, and raised wave priorities, were equal or slower.
// InF16: the cache is the workspace that a 4-bit one was unpacked to, each head of a sequence
// times a power of two of its own (shifts), and the queries' rows times one of theirs.  A head
// whose rows are too far apart for one power has one for each key, and its tiles go through
// the careful pass.
constexpr int kPromptWaves = 4, kPromptRows = 32 * kPromptWaves, kStepKeys = 32, kStepSlots = 4;
constexpr int kStepUnits = kStepKeys * kHeadDim / 8;          // 16-byte units of a step's K or V (512)

// A row's queries (its lanes: l, l ^ 32) from bf16 to f16 times a power of two, and that power's inverse.
__device__ inline float row_in_f16(v8h *qf) {
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const v4u x = __builtin_bit_cast(v4u, qf[i]);
#pragma unroll
        for (int j = 0; j < 4; ++j) top = fmaxf(top, fmaxf(fabsf(bf16_lo_to_f32(x[j])), fabsf(bf16_hi_to_f32(x[j]))));
    }
    const int e = f16_exponent(pair32_max(top));
    const float f = power_of_two(14 - e);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        v4u x = __builtin_bit_cast(v4u, qf[i]);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = cvt_pk_f16(bf16_lo_to_f32(x[j]) * f, bf16_hi_to_f32(x[j]) * f);
        qf[i] = __builtin_bit_cast(v8h, x);
    }
    return power_of_two(e - 14);
}

template <int HALVES, typename E>
__global__ __launch_bounds__(HALVES * kPromptWaves * 64, 2 / HALVES) void k_causal_prompt(CausalArgs a) {
    __shared__ __attribute__((aligned(16))) uint4 rings[HALVES][2][kStepSlots][kStepUnits];    // K, V
    __shared__ int not_finite[HALVES * kPromptWaves];
    __shared__ float2 second[HALVES == 2 ? kPromptRows : 1];       // (maximum, sum of weights) of the second half
    const int wave = __builtin_amdgcn_readfirstlane((threadIdx.x >> 6) % kPromptWaves), lane = threadIdx.x & 63;
    const int part = HALVES == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / (kPromptWaves * 64));
    const int hi = lane >> 5, r = lane & 31;
    uint4 (*const kring)[kStepUnits] = rings[part][0], (*const vring)[kStepUnits] = rings[part][1];
    Work w;
    if (!find_work<kPromptRows>(a, lane, blockIdx.y, w)) return;

    const Range range = range_of(a, (w.hi + kStepKeys - 1) / kStepKeys, w.split);
    if (a.S > 1 && w.split >= range.used) return;
    // steps [u0, u0 + n); an odd number of steps leaves the second half one without keys
    const int n = HALVES == 1 ? range.end - range.first : (range.end - range.first + 1) / 2, u0 = range.first + part * n;
    const int most = range.end * kStepKeys - 1;                   // the range's last key
    const uint16_t *kp = w.k + (int64_t)u0 * kStepKeys * a.b.tok, *vp = w.v + (int64_t)u0 * kStepKeys * a.b.tok;
    const int first_key = u0 * kStepKeys;

    // wave w loads keys 4 (w + 4 j) .. + 3 of a step, j = 0, 1, into slot u mod 4
    const int lk = 4 * wave + (lane >> 4);
    const uint32_t koff = 2u * ((uint32_t)(lane >> 4) * (uint32_t)a.b.tok + 8u * ((lane & 15) ^ lk));
    const uint32_t voff = 2u * ((uint32_t)(lane >> 4) * (uint32_t)a.b.tok + 8u * ((lane & 15) ^ (4 * (lane >> 4))));
    const uint32_t klds = lds_addr(kring) + wave * 1024, vlds = lds_addr(vring) + wave * 1024;
    const int full = (w.hi - first_key) / kStepKeys;              // steps without keys past the last
    const int64_t half = 16 * a.b.tok, whole = 32 * a.b.tok;
    const uint16_t *kn = kp + 4 * wave * a.b.tok, *vn = vp + 4 * wave * a.b.tok;   // next steps to load
    auto load = [&](const uint16_t *&next, const uint16_t *src, uint32_t lds, int u, uint32_t off, int swz) {
        if (u < full) {
            load_lds_s16(next, off, lds);
            load_lds_s16(next + half, off, lds + 4096);
        } else {                                                  // the last, partial step: its last key again
#pragma unroll 1
            for (int j = 0; j < 2; ++j) {
                const int key = min(u * kStepKeys + lk + 16 * j, w.hi - 1 - first_key);
                load_lds_v16(src + (int64_t)key * a.b.tok + 8 * ((lane & 15) ^ swz), lds + 4096 * j);
            }
        }
        next += whole;
    };
    auto load_k = [&](int u) { load(kn, kp, klds + (u & (kStepSlots - 1)) * 8192, u, koff, lk); };
    auto load_v = [&](int u) { load(vn, vp, vlds + (u & (kStepSlots - 1)) * 8192, u, voff, 4 * (lane >> 4)); };

    const RowOf row = row_of(a, w, min(32 * wave + r, w.rows - 1));
    const int last = min(w.s.p0 + row.i, most);                            // last key this row sees
    const int wave_first = __builtin_amdgcn_readfirstlane(min(w.s.p0 + row_of(a, w, min(32 * wave, w.rows - 1)).i, most));
    const int wave_last = __builtin_amdgcn_readfirstlane(min(w.s.p0 + row_of(a, w, min(32 * wave + 31, w.rows - 1)).i, most));
    typedef typename E::v8 v8;
    constexpr bool kScaled = std::is_same<E, InF16>::value;
    v8 qf[8];
    float c = a.c, back = 1.0f, v_back = 1.0f;                    // f16: scores come out over `back`, sums over v_back
    const short2 *row_shifts = nullptr;                           // or besides over a power of two of each key
    {
        const uint16_t *qp = a.q + row_at(w, row, a.q_stride) + 8 * hi;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) qf[ks] = *(const v8 *)(qp + 16 * ks);
        if constexpr (kScaled) {
            const int64_t head = w.s.slot0 / a.b.seq_slots * a.Hkv + w.h;
            const HeadShift shift = a.shifts[head];
            back = row_in_f16(qf) * power_of_two(shift.k);
            v_back = power_of_two(shift.v);
            c *= back;
            if (shift.by_row) row_shifts = a.row_shifts + head * a.b.capacity;
        }
    }

    // operands from LDS: row r of the scores' A operand; of V, what the transposing read needs.
    // Their places in a slot, so that a slot and a key only add a constant.
    uint32_t kat[8], vat[4];
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) kat[ks] = 16u * key_unit(r, 2 * ks + hi);
    {
        const int vq = lane & 3, vk = 4 * hi + ((lane >> 2) & 3), vc = 2 * ((lane >> 4) & 1) + (vq >> 1);
#pragma unroll
        for (int dt = 0; dt < 4; ++dt) vat[dt] = 16u * value_unit(vk, 4 * dt + vc) + 8 * (vq & 1);
    }
    auto k_frag = [&](int slot, int ks) { return *(const v8 *)((const char *)kring + kat[ks] + slot * 8192); };
    auto v_half = [&](int slot, int key, int dt) { return lds_read_tr((const char *)vring + vat[dt] + slot * 8192 + key * 256); };
    auto v_frag = [&](int slot, int h, int dt) {
        return __builtin_bit_cast(v8, __builtin_shufflevector(v_half(slot, 16 * h, dt), v_half(slot, 16 * h + 8, dt), 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto zero = [](v16f &x) {
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = 0.0f;
    };
    auto mask = [&](v16f &s, int key0) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = key0 + 8 * (i >> 2) + 4 * hi + (i & 3) <= last ? s[i] : kNegInf;
    };
    auto row_max = [&](const v16f &s) {
        float x = kNegInf;
#pragma unroll
        for (int i = 0; i < 16; ++i) x = fmaxf(x, s[i]);
        return pair32_max(x);
    };
    auto operand = [](const uint32_t *p) { return __builtin_bit_cast(v8, v4u{p[0], p[1], p[2], p[3]}); };

    float m = kNegInf, l = 0.0f;
    uint64_t gone_far = 0;
    v16f o[4];
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) zero(o[dt]);

    if (n > 0) {
        load_k(0);
        if (n > 1) load_k(1);
        if (n > 2) load_k(2);
        load_v(0);
        v16f s0, s1;
        uint32_t p0[8], p1[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) p1[i] = 0;                       // there is no step -1: zeros, also in its slot
#pragma unroll
        for (int i = 0; i < kStepUnits; i += kPromptWaves * 64) vring[3][i + threadIdx.x % (kPromptWaves * 64)] = uint4{};
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        lds_barrier();
        zero(s0);
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) s0 = E::product(k_frag(0, ks), qf[ks], s0);

        // step u (u mod 4 = SLOT): softmax of s into p; scores of u + 1 into sn; sums of u - 1 with pp
        auto step = [&](auto slot, int u, v16f &s, v16f &sn, uint32_t *p, const uint32_t *pp) {
            constexpr int SLOT = decltype(slot)::value, KS = (SLOT + 1) & 3, VS = (SLOT + 3) & 3;
            v8 kf[4], vf[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) kf[i] = k_frag(KS, i);
#pragma unroll
            for (int i = 0; i < 4; ++i) vf[i] = v_frag(VS, 0, i);
            const int key0 = first_key + u * kStepKeys;
            if (key0 + kStepKeys - 1 > wave_first) mask(s, key0);
            const float mt = row_max(s);
            const bool own = (mt - m) * c > kLazy, grown = __ballot(own) != 0;
            const float mn = own ? mt : m;
            const float mu = mn == kNegInf ? 0.0f : mn, muc = mu * c;
            float ls = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (i == 0) zero(sn);
                sn = E::product(kf[i & 3], qf[i], sn);
                if (i < 4) kf[i] = k_frag(KS, i + 4);
                o[i & 3] = E::product(vf[i & 3], operand(pp + 4 * (i >> 2)), o[i & 3]);
                if (i < 4) vf[i] = v_frag(VS, 1, i);
                const float e0 = exp2_hw(__builtin_fmaf(s[2 * i], c, -muc)), e1 = exp2_hw(__builtin_fmaf(s[2 * i + 1], c, -muc));
                p[i] = E::pair(e0, e1);
                ls = E::add(p[i], ls);
            }
            // the weights here, between the products, not behind the branch below
#pragma unroll
            for (int i = 0; i < 8; ++i) asm volatile("" : "+v"(p[i]));
            asm volatile("" : "+v"(ls));
#pragma unroll
            for (int i = 0; i < 4; ++i) {                                // two products, six vector instructions, three LDS reads
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x002, 3, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x002, 3, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x002, 3, 0);
            }
            if (grown) {                                             // the sums so far, up to step u - 1
                const float alpha = exp2_hw((m - mu) * c);
                m = mn;
                l *= alpha;
#pragma unroll
                for (int dt = 0; dt < 4; ++dt) o[dt] *= alpha;
                gone_far |= __ballot(fabsf(muc) > kFar);
            }
            l += ls;
        };
        // Before steps u and u + 1 (u even): what they read, K of u + 1 and u + 2 and V of u - 1 and
        // u, was loaded during the two steps before; what is loaded now takes the places of K of
        // u - 1 and u and V of u - 3 and u - 2, which every wave is done with.
        auto advance = [&](int u) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            lds_barrier();
            if (u + 3 < n) load_k(u + 3);
            if (u + 1 < n) load_v(u + 1);
            if (u + 4 < n) load_k(u + 4);
            if (u + 2 < n) load_v(u + 2);
        };
        for (int u = 0; u < n; u += 4) {
            advance(u);
            step(std::integral_constant<int, 0>{}, u, s0, s1, p0, p1);
            if (u + 1 >= n) break;
            step(std::integral_constant<int, 1>{}, u + 1, s1, s0, p1, p0);
            if (u + 2 >= n) break;
            advance(u + 2);
            step(std::integral_constant<int, 2>{}, u + 2, s0, s1, p0, p1);
            if (u + 3 >= n) break;
            step(std::integral_constant<int, 3>{}, u + 3, s1, s0, p1, p0);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        lds_barrier();
#pragma unroll
        for (int i = 0; i < 8; ++i)
            o[i & 3] = E::product(v_frag((n - 1) & 3, i >> 2, i & 3), operand((n & 1 ? p0 : p1) + 4 * (i >> 2)),
                                                               o[i & 3]);
    }
    const uint64_t bad = __ballot(!all_finite(o)) | gone_far;
    if (lane == 0) not_finite[part * kPromptWaves + wave] = bad != 0;
    lds_barrier();
    int any = 0;
#pragma unroll
    for (int i = 0; i < HALVES * kPromptWaves; ++i) any |= not_finite[i];
    if (any || row_shifts) {
        // careful: once more, step by step, every row with the values of its own keys only
        StepScale scale;                                             // of the values' own powers
        m = kNegInf;
        l = 0.0f;
        kn = kp + 4 * wave * a.b.tok;
        vn = vp + 4 * wave * a.b.tok;
#pragma unroll
        for (int dt = 0; dt < 4; ++dt) zero(o[dt]);
#pragma unroll 1
        for (int u = 0; u < n; ++u) {
            lds_barrier();
            load_k(u);                                               // into slot u mod 4
            load_v(u);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            lds_barrier();
            const int slot = u & (kStepSlots - 1), key0 = first_key + u * kStepKeys;
            v16f s;
            zero(s);
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) s = E::product(k_frag(slot, ks), qf[ks], s);
            float value[16];                                         // the values' powers
            if (row_shifts) {
                float most = 0.0f;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int key = key0 + 8 * (i >> 2) + 4 * hi + (i & 3);
                    const short2 shift = row_shifts[min(key, w.hi - 1)];
                    s[i] *= power_of_two(shift.x);
                    value[i] = power_of_two(shift.y);
                    most = fmaxf(most, key <= last ? value[i] : 0.0f);
                }
                const float by = scale.raise(pair32_max(most));
                l *= by;
#pragma unroll
                for (int dt = 0; dt < 4; ++dt) o[dt] *= by;
            }
            mask(s, key0);
            const float mt = row_max(s);
            const bool own = (mt - m) * c > kLazy;
            const float mn = own ? mt : m, mu = mn == kNegInf ? 0.0f : mn, muc = mu * c;
            if (__ballot(own)) {
                const float alpha = exp2_hw((m - mu) * c);
                m = mn;
                l *= alpha;
#pragma unroll
                for (int dt = 0; dt < 4; ++dt) o[dt] *= alpha;
            }
            const bool far = fabsf(muc) > kFar;
            float ls = 0.0f;
            uint32_t p[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float e0 = exp2_hw(exponent(s[2 * i], c, mu, muc, far) - scale.e), e1 = exp2_hw(exponent(s[2 * i + 1], c, mu, muc, far) - scale.e);
                if (row_shifts) {
                    p[i] = E::pair(e0 * value[2 * i], e1 * value[2 * i + 1]);
                    ls += e0 + e1;
                } else {
                    p[i] = E::pair(e0, e1);
                    ls = E::add(p[i], ls);
                }
            }
            l += ls;
            const int t0 = min(wave_first, key0 + kStepKeys - 1), t1 = min(wave_last, key0 + kStepKeys - 1);   // later tokens see all
#pragma unroll
            for (int dt = 0; dt < 4; ++dt) {
                const v16f before = o[dt];
#pragma unroll 1
                for (int t = t0; t <= t1; ++t) {
                    v16f x = before;
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        x = E::product(
                            __builtin_bit_cast(v8, values_up_to(v_half(slot, 16 * h, dt), v_half(slot, 16 * h + 8, dt), key0 + 16 * h + 4 * hi, key0 + 16 * h + 8 + 4 * hi, t)),
                            operand(p + 4 * h), x);
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[dt][i] = min(last, key0 + kStepKeys - 1) == t ? x[i] : o[dt][i];
                }
            }
        }
        lds_barrier();                                               // the rings are free
        if (row_shifts) {
            const float up = power_of_two((int)scale.e);
            l *= up;
#pragma unroll
            for (int dt = 0; dt < 4; ++dt) o[dt] *= up;
        }
    }
    l = pair32_sum(l);
    if constexpr (HALVES == 2) {
        // the second half's sums through its rings, which nothing reads any more
        v4f *const sums = (v4f *)rings[1];
        if (part == 1) {
#pragma unroll
            for (int dt = 0; dt < 4; ++dt)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    sums[((4 * wave + dt) * 4 + i) * 64 + lane] = v4f{o[dt][4 * i], o[dt][4 * i + 1], o[dt][4 * i + 2], o[dt][4 * i + 3]};
            if (hi == 0) second[32 * wave + r] = make_float2(m, l);
        }
        lds_barrier();
        if (part == 1) return;
        const float2 e = second[32 * wave + r];
        const float M = fmaxf(m, e.x), mu = M == kNegInf ? 0.0f : M;
        const float f1 = exp2_hw((m - mu) * c), f2 = exp2_hw((e.x - mu) * c);
        m = M;
        l = l * f1 + e.y * f2;
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const v4f x = sums[((4 * wave + dt) * 4 + i) * 64 + lane];
#pragma unroll
                for (int k = 0; k < 4; ++k) o[dt][4 * i + k] = o[dt][4 * i + k] * f1 + x[k] * f2;
            }
    }
    if (a.S == 1) {
        // through LDS of the wave's own (the keys' ring, which nothing reads any more), so that 16
        // lanes store a row (packed prompts 114.4 us with 8 bytes of 32 rows a store, 110.8 so): unit
        // 4 dt + i has dimensions 32 dt + 8 i .. + 7, 4 of them a lane
        char *const rows = (char *)kring + wave * 8192;
        const bool sees = w.s.L > 0 && last >= 0;
        const float inv = kScaled ? v_back / l : 1.0f / l;
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint2 y = make_uint2(cvt_pk_bf16(o[dt][4 * i] * inv, o[dt][4 * i + 1] * inv),
                                           cvt_pk_bf16(o[dt][4 * i + 2] * inv, o[dt][4 * i + 3] * inv));
                *(uint2 *)(rows + 16 * key_unit(r, 4 * dt + i) + 8 * hi) = sees ? y : uint2{};
            }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int x = 4 * j + (lane >> 4), c = lane & 15;
            if (32 * wave + x >= w.rows) break;
            *(uint4 *)(a.out + row_at(w, row_of(a, w, 32 * wave + x), a.out_stride) + 8 * c) = *(const uint4 *)(rows + 16 * key_unit(x, c));
        }
    } else if (32 * wave + r < w.rows) {
        if constexpr (kScaled) {
#pragma unroll
            for (int dt = 0; dt < 4; ++dt) o[dt] *= v_back;
        }
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *(v4f *)(unit_at<kPromptRows>(a, w.split, (4 * wave + dt) * 4 + i) + 4 * lane) =
                    v4f{o[dt][4 * i], o[dt][4 * i + 1], o[dt][4 * i + 2], o[dt][4 * i + 3]};
        if (hi == 0) *row_ml<kPromptRows>(a, w.split, 32 * wave + r) = make_float2(kScaled ? m * back : m, l);
    }
}

// ---------------------------------------------------------------- joining key ranges

// A wave takes one unit of an item (or every P-th range of it, P waves together, merged through
// LDS in wave order), a lane 4 dimensions of a row.  Bound by the partial results' bytes, or
// with few rows by one trip to memory for the lengths and one for all ranges.
constexpr int kJoinBatch = 8;      // ranges requested together

template <int RT, int P, bool SEVERAL>
__global__ __launch_bounds__(256) void k_causal_join(CausalArgs a) {
    constexpr int R = causal_tile_rows(RT);
    __shared__ float2 gml[4][64];
    __shared__ v4f go[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, part = wave % P;
    const int unit = (blockIdx.y * 4 + wave) / P;
    Work w;
    if (!find_work<R, SEVERAL>(a, lane, 0, w)) return;
    int row, d;                                                    // of this lane
    if (RT == 1) {
        row = 16 * (unit >> 3) + (lane & 15);
        d = 16 * (unit & 7) + 4 * (lane >> 4);
    } else {
        row = 32 * (unit >> 4) + (lane & 31);
        d = 8 * (unit & 15) + 4 * (lane >> 5);
    }
    const int used = w.hi > 0 ? range_of(a, (w.hi + (1 << a.step_shift) - 1) >> a.step_shift, 0).used : 0;
    const bool on = row < w.rows;
    float m = kNegInf, ls = 0.0f;
    v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
    auto fold = [&](const float2 &e, const v4f &v) {
        const float M = fmaxf(m, e.x), mu = M == kNegInf ? 0.0f : M;
        const float f1 = exp2_hw((m - mu) * a.c), f2 = exp2_hw((e.x - mu) * a.c);
        m = M;
        ls = ls * f1 + e.y * f2;
        acc = acc * f1 + v * f2;
    };
    if (on) {
        for (int s0 = part; s0 < used; s0 += P * kJoinBatch) {
            float2 e[kJoinBatch];
            v4f v[kJoinBatch];
#pragma unroll
            for (int i = 0; i < kJoinBatch; ++i) {
                const int s = s0 + P * i;
                e[i] = make_float2(kNegInf, 0.0f);
                v[i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
                if (s < used) {
                    e[i] = *row_ml<R>(a, s, row);
                    v[i] = *(const v4f *)(unit_at<R>(a, s, unit) + 4 * lane);
                }
            }
#pragma unroll
            for (int i = 0; i < kJoinBatch; ++i)
                if (s0 + P * i < used) fold(e[i], v[i]);
        }
    }
    if (P > 1) {
        gml[wave][lane] = make_float2(m, ls);
        go[wave][lane] = acc;
        __syncthreads();
        if (part != 0) return;
#pragma unroll
        for (int i = 1; i < P; ++i) fold(gml[wave + i][lane], go[wave + i][lane]);
    }
    if (!on) return;
    store_out(a, w, row_of(a, w, row), d, acc, ls);
}

template <int RT, bool SEVERAL = false>
void launch_join(const CausalArgs &a, hipStream_t st) {
    constexpr int units = causal_tile_rows(RT) / 2;                // of an item
    if (a.S > 4) hipLaunchKernelGGL((k_causal_join<RT, 4, SEVERAL>), dim3((unsigned)(a.tiles * a.Hkv), units), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_causal_join<RT, 1, SEVERAL>), dim3((unsigned)(a.tiles * a.Hkv), units / 4), dim3(256), 0, st, a);
}

}  // namespace

const char *causal_kernel_name(int rt, int halves) {
    return rt == 1 ? "k_causal_few" : rt == 2 ? "k_causal_mid<1>" : rt == 4 ? "k_causal_mid<2>" : halves == 2 ? "k_causal_prompt<2>" : "k_causal_prompt<1>";
}

hipError_t launch_kv4_join(const CausalArgs &a, int rt, hipStream_t st) {
    if (rt == 1) launch_join<1>(a, st);
    else launch_join<2, true>(a, st);
    return hipGetLastError();
}

hipError_t launch_causal(const CausalArgs &args, int rt, int halves, hipStream_t st) {
    CausalArgs a = args;
    a.step_shift = shift_of(rt == 1 ? kFewKeys : rt ? kMidKeys : kStepKeys);
    const dim3 grid((unsigned)(a.tiles * a.Hkv), (unsigned)a.S);
    if (rt == 1) hipLaunchKernelGGL(k_causal_few, grid, dim3(kFewWaves * 64), 0, st, a);
    else if (rt == 2) hipLaunchKernelGGL(k_causal_mid<1>, grid, dim3(256), 0, st, a);
    else if (rt == 4) hipLaunchKernelGGL(k_causal_mid<2>, grid, dim3(512), 0, st, a);
    else if (a.shifts && halves == 2) hipLaunchKernelGGL((k_causal_prompt<2, InF16>), grid, dim3(2 * kPromptWaves * 64), 0, st, a);
    else if (a.shifts) hipLaunchKernelGGL((k_causal_prompt<1, InF16>), grid, dim3(kPromptWaves * 64), 0, st, a);
    else if (halves == 2) hipLaunchKernelGGL((k_causal_prompt<2, InBf16>), grid, dim3(2 * kPromptWaves * 64), 0, st, a);
    else hipLaunchKernelGGL((k_causal_prompt<1, InBf16>), grid, dim3(kPromptWaves * 64), 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.S == 1) return e;
    if (rt == 1) launch_join<1>(a, st);
    else if (rt == 2) launch_join<2>(a, st);
    else if (rt == 4) launch_join<4>(a, st);
    else launch_join<0>(a, st);
    return hipGetLastError();
}

}  // namespace qlin
