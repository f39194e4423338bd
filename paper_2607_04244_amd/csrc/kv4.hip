// Causal attention with grouped heads over the 4-bit key/value cache, and the cache's
// unpacking to bf16 (qlin_causal_attention_four_bit, qlin_unpack_four_bit in include/qlin_lowbit.h).
//
// Rows are packed as in causal.hip (new token i, head g of a group: r = i G + g) and the
// products the same, S^T = K Q^T and O^T += V^T P^T, in f16, whose operands are made from the
// codes: a nibble c at bits 0-3 of a 16-bit half is the f16 subnormal c 2^-24, at bits 4-7 it
// is c 2^-20, and the matrix cores take both exactly, so a word of eight codes costs one shift
// and four ANDs.  What a row's step s and offset o add is one product for each key and row,
// not one for each value:
//   q . k = s (q . c) + o sum(q),   sum_j p_j v_j = sum_j (p_j s_j) c_j + sum_j p_j o_j
// with p_j s_j rounded to f16 once, its operand (11 bits: against 64 bits an output's error is 1.75e-3 in
// the 2-norm, of which its own rounding to bf16 is 1.65e-3).  Queries are brought into f16's range by a
// power of two for each row; weights by 2^-E for each row, E from the largest size of step that
// the row has seen, raised as the maximum is, so weights times steps keep their 11 bits down to
// 2^-15 of the largest.
// The contraction's order is free: a lane's K words are 32 (64) dimensions in a row, whose
// queries are brought into the extraction's order once, and V comes transposed from LDS, 16
// keys of a dimension a lane.  Codes are finite whatever lies behind a row's token, and a
// hidden key's step and offset are taken as zeros, so no pass has to be repeated.
//
//   k_kv4_few      up to 16 rows (single tokens): bound by the cache's bytes where many sequences
//       are read, 64 of 4096 keys 48.3 to 50.4 us, 5.7 to 5.9 TB/s, and 64 of 130 to 8190 64 to 67, by
//       the longest; one token over 8191 keys 7.2 us and 3.2 for the join, its latency.
//   k_kv4_rows     tiles of 32 rows (blocks, chunks, short prompts): about 350 vector instructions for
//       16 products of 32 keys and rows, 16 exponentials among them.  They bound it where all units
//       work: 32 sequences of 16 tokens over 4096 keys 65 to 69 us, the vector unit busy for 73 % of
//       them, the matrix cores for 25.  Few blocks leave both idle: five of 517 to 8192 keys 38 and 10 %
//       of 23 us, in which a wave has four steps at most, behind its start and before the sums of
//       four waves are merged.  16 tokens over 8192 keys 15.4, 512 without a prefix 13.3.  Tiles of
//       64 rows with one extraction for both, alone on a compute unit: 78 and 19.0 us.
//   k_kv4_peaks, k_unpack_kv4   the cache in 16 bits, bf16 for a caller and f16 for
//       k_causal_prompt, which long chunks go through (causal.hip): its 11 bits keep the result as
//       exact as above, where bf16's 8 would take its error from 1.7e-3 to 4.1e-3.  8192 tokens of 8
//       heads 8.2 to 9.9 us, 4.3 to 5 TB/s; packed prompts of 1 to 2048 4.9 and 13.7 of 130 in all.
//       Heads whose rows have a power each go through that kernel's careful pass, behind a first one
//       that is thrown away: with one row 2^13 below the others a prompt of 2048 takes 254 us for 63.
#include "causal_common.h"
#include "lowbit_internal.h"

#include <type_traits>

namespace qlin {

namespace {

typedef int v2i __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) v2i lds_v2i;

// Transposing LDS read: lane i of 16 receives nibble i of the 8-byte chunks that lanes
// 0 .. 15 address, in their order.
__device__ inline v2i lds_read_tr4(const void *p) {
    return __builtin_amdgcn_ds_read_tr4_b64_v2i32((lds_v2i *)(const __attribute__((address_space(3))) void *)p);
}
__device__ inline v8h operand(const Pairs &p) { return __builtin_bit_cast(v8h, v4u{p.a0, p.a1, p.a2, p.a3}); }
__device__ inline v8h operand(const uint32_t *p) { return __builtin_bit_cast(v8h, v4u{p[0], p[1], p[2], p[3]}); }
// A row's queries, N units of 8 dimensions of it a lane (`over`: reduction over the row's
// lanes): the f16 operands in the extraction's order (pairs (0, 4), (1, 5), (2, 6), (3, 7),
// odd ones over 16), and their sum.  Scores come out divided by `back`.
template <int N, typename M, typename S>
__device__ inline void load_queries(const uint16_t *qp, v8h *qf, float &qs, float &back, M max_over, S sum_over) {
    uint4 q[N];
    float top = 0.0f;
    qs = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        q[i] = *(const uint4 *)(qp + 8 * i);
        const uint32_t w[4] = {q[i].x, q[i].y, q[i].z, q[i].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            top = fmaxf(top, fmaxf(fabsf(bf16_lo_to_f32(w[j])), fabsf(bf16_hi_to_f32(w[j]))));
            qs = dot2(w[j], kBf16OnePair, qs);
        }
    }
    const int e = min(max(exponent_of(max_over(top)), -100), 100);
    const float f = power_of_two(14 - e), f16th = power_of_two(10 - e);
    back = power_of_two(10 + e);                                     // 2^24 (the codes) over f
    qs = sum_over(qs) / back;
#pragma unroll
    for (int i = 0; i < N; ++i)
        qf[i] = __builtin_bit_cast(v8h, v4u{cvt_pk_f16(bf16_lo_to_f32(q[i].x) * f, bf16_lo_to_f32(q[i].z) * f),
                                            cvt_pk_f16(bf16_hi_to_f32(q[i].x) * f16th, bf16_hi_to_f32(q[i].z) * f16th),
                                            cvt_pk_f16(bf16_lo_to_f32(q[i].y) * f, bf16_lo_to_f32(q[i].w) * f),
                                            cvt_pk_f16(bf16_hi_to_f32(q[i].y) * f16th, bf16_hi_to_f32(q[i].w) * f16th)});
}
__device__ inline float grid_step(uint32_t g) { return bf16_lo_to_f32(g); }
__device__ inline float grid_offset(uint32_t g) { return bf16_hi_to_f32(g); }
// What StepScale goes by: steps of either sign, and offsets, which the same weights are multiplied by
// in fp32: p 2^-E |o| stays below 2^55.  Beside an offset a step of 2^-40 of it is nothing.  The
// step's bits behind the offset's make that larger by less than a bf16 step.
constexpr float kOffsetSize = 0x1p-40f;
__device__ inline float offset_bound(uint32_t g) { return fabsf(__uint_as_float(g)); }
__device__ inline float grid_size(uint32_t g) { return fmaxf(fabsf(grid_step(g)), offset_bound(g) * kOffsetSize); }

// Smallest value over the wave.
__device__ inline float wave_min(float v) {
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v = fminf(v, __shfl_xor(v, d));
    return v;
}

__device__ inline void load_lds_s4(const uint32_t *base, uint32_t off, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" :: "s"(lds), "v"(off), "s"(base) : "memory", "m0");
}
__device__ inline void load_lds_v4(const uint32_t *src, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" :: "s"(lds), "v"(src) : "memory", "m0");
}

// 16 scores of a row to weights 2^((s - m) c - E).  Where |m c| is small enough that its rounding
// leaves weights as exact as they are anyway, they are one fused product each.  By the row, not
// the wave: not a bit of a row depends on others.
constexpr float kNear = 256.0f;
__device__ inline void weights(float e[16], float m, float c, float E) {
    const float mu = m == kNegInf ? 0.0f : m, mc = mu * c;
    if (fabsf(mc) <= kNear) {
        const float sub = mc + E;
#pragma unroll
        for (int i = 0; i < 16; ++i) e[i] = __builtin_fmaf(e[i], c, -sub);
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) e[i] = __builtin_fmaf(e[i] - mu, c, -E);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) e[i] = exp2_hw(e[i]);
}
// The weights' sums (l of p, z of p o) and p s as the operand: pairs of keys 8 h + i, 8 h + 4 + i in
// word 4 h + i, odd keys' over 16.
__device__ inline void weigh(const float e[16], const uint32_t grid[16], float &l, float &z, uint32_t *p) {
    float ps[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        l += e[i];
        z = __builtin_fmaf(e[i], grid_offset(grid[i]), z);
        ps[i] = e[i] * (grid_step(grid[i]) * (i & 1 ? 0.0625f : 1.0f));
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) p[4 * h + i] = cvt_pk_f16(ps[8 * h + i], ps[8 * h + 4 + i]);
}

// Steps of 64 keys, a wave's own: K and V codes (4 KiB each), then their grids (256 bytes
// each), two steps of each wave in flight by direct-to-LDS loads.
constexpr int kKvWaves = 4, kKvStages = 2, kStepBytes = 2 * kKv4Keys * 64 + 2 * kKv4Keys * 4, kStepLoads = 10;
constexpr float kCodes = 16777216.0f;     // 2^24: codes are c 2^-24
constexpr int kVAt = kKv4Keys * 64, kKGridAt = 2 * kKv4Keys * 64, kVGridAt = kKGridAt + kKv4Keys * 4;

// A row's four 16-byte units lie in an order that changes from key to key, so that what 16 lanes
// read together meets different banks: V, and K where 16 consecutive lanes read keys that
// differ in the bits that `k_order` folds.
__device__ inline int v_order(int key) { return (key >> 2) & 3; }
template <int RT>
__device__ inline int k_order(int key) {
    return RT == 1 ? (key >> 4) & 3 : ((key >> 2) & 1) | ((key >> 4) & 1) << 1;
}

// What a wave needs to request a step.
template <int RT>
struct Loader {
    const uint32_t *k, *v, *kg, *vg;     // the head's row of token 0
    int64_t tok;
    uint32_t koff[4], voff, goff, lds;
    int hi, lane;
    __device__ inline Loader(const CausalKv4Args &x, const Work &w, int lane_, uint32_t lds_) : tok(x.a.b.tok), lds(lds_), hi(w.hi), lane(lane_) {
        k = x.c.k + 16 * w.at;
        v = x.c.v + 16 * w.at;
        kg = x.c.k_grid + w.at;
        vg = x.c.v_grid + w.at;
        const uint32_t row = (uint32_t)(lane >> 2) * (uint32_t)tok * 64u;
#pragma unroll
        for (int j = 0; j < 4; ++j) koff[j] = row + 16u * ((lane & 3) ^ k_order<RT>(16 * j + (lane >> 2)));
        voff = row + 16u * ((lane & 3) ^ v_order(lane >> 2));
        goff = (uint32_t)lane * (uint32_t)tok * 4u;
    }
    __device__ inline void issue(int u, int st) const {
        const uint32_t to = lds + st * kStepBytes;
        if ((u + 1) * kKv4Keys <= hi) {
            const int64_t row = (int64_t)u * kKv4Keys * tok;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                load_lds_s16_nt((const uint16_t *)(k + 16 * (row + 16 * j * tok)), koff[j], to + j * 1024);
                load_lds_s16_nt((const uint16_t *)(v + 16 * (row + 16 * j * tok)), voff, to + kVAt + j * 1024);
            }
            load_lds_s4(kg + row, goff, to + kKGridAt);
            load_lds_s4(vg + row, goff, to + kVGridAt);
            return;
        }
        // the last, partial step: its last key again
#pragma unroll 1
        for (int j = 0; j < 4; ++j) {
            const int kk = 16 * j + (lane >> 2);
            const int64_t row = (int64_t)min(u * kKv4Keys + kk, hi - 1) * tok;
            load_lds_v16((const uint16_t *)(k + 16 * row + 4 * ((lane & 3) ^ k_order<RT>(kk))), to + j * 1024);
            load_lds_v16((const uint16_t *)(v + 16 * row + 4 * ((lane & 3) ^ v_order(kk))), to + kVAt + j * 1024);
        }
        const int64_t row = (int64_t)min(u * kKv4Keys + lane, hi - 1) * tok;
        load_lds_v4(kg + row, to + kKGridAt);
        load_lds_v4(vg + row, to + kVGridAt);
    }
    // This step's loads have landed; the next one's may be in flight.
    __device__ inline void wait(bool more) const {
        if (more) asm volatile("s_waitcnt vmcnt(%0)" :: "n"(kStepLoads) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
};

// ---------------------------------------------------------------- few rows

__global__ __launch_bounds__(kKvWaves * 64, 2) void k_kv4_few(CausalKv4Args x) {
    constexpr int R = 16;
    const CausalArgs &a = x.a;
    __shared__ __attribute__((aligned(16))) char ring[kKvWaves][kKvStages][kStepBytes];     // then the waves' sums
    __shared__ float2 ml[kKvWaves][R];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int g = lane >> 4, r = lane & 15;
    Work w;
    if (!find_work<R>(a, lane, blockIdx.y, w)) return;
    const Range range = range_of(a, (w.hi + kKv4Keys - 1) / kKv4Keys, w.split);
    if (a.S > 1 && w.split >= range.used) return;
    const int u0 = range.first, u1 = range.end;
    const Loader<1> load(x, w, lane, lds_addr(ring[wave]));
    if (u0 + wave < u1) load.issue(u0 + wave, 0);
    if (u0 + wave + kKvWaves < u1) load.issue(u0 + wave + kKvWaves, 1);

    // queries: B operand, row r; K's word ks of lane group g is dimensions 32 g + 8 ks .. + 7
    const RowOf row = row_of(a, w, min(r, w.rows - 1));
    const int last = w.s.p0 + row.i;                          // last key that the row sees
    const int first_last = w.s.p0 + w.i0;                     // keys up to here are seen by every row
    v8h qf[4];
    float qs, back;
    load_queries<4>(a.q + row_at(w, row, a.q_stride) + 32 * g, qf, qs, back, [](float v) { return pair32_max(pair16_max(v)); },
                    [](float v) { return pair32_sum(pair16_sum(v)); });
    const float c = a.c * back;
    const ExtractConsts<true> extract;

    // places in a step: K of key 16 (r >> 2) + 4 kt + (r & 3); V of key 16 g + r; grids of keys 16 g ..
    const int kat = (16 * (r >> 2) + (r & 3)) * 64 + 16 * (g ^ (r >> 2));
    int vat[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) vat[i] = kVAt + (16 * g + r) * 64 + 16 * (i ^ v_order(r));
    float m = kNegInf, l = 0.0f, z = 0.0f;                    // maximum; sums of p and p o
    StepScale scale;
    float least_limit = 0.0f;                                 // of the wave's rows
    v4f o[8];
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) o[dt] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    auto rescale = [&](float by) {
        l *= by;
        z *= by;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) o[dt] *= by;
    };
    int st = 0;
    for (int u = u0 + wave; u < u1; u += kKvWaves, st ^= 1) {
        load.wait(u + kKvWaves < u1);
        const char *step = ring[wave][st];
        const int key0 = u * kKv4Keys + 16 * g;               // this lane's keys: key0 + 4 kt + i
        const bool masked = (u + 1) * kKv4Keys - 1 > first_last;
        auto grids = [&](int at, int kt) { return *(const uint4 *)(step + at + 4 * (16 * g + 4 * kt)); };
        v4f sc[4];
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) {
            const uint4 kw = *(const uint4 *)(step + kat + kt * 256), kg = grids(kKGridAt, kt);
            const uint32_t word[4] = {kw.x, kw.y, kw.z, kw.w}, grid[4] = {kg.x, kg.y, kg.z, kg.w};
            v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
                acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(operand(extract.pairs(word[ks])), qf[ks], acc, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) sc[kt][i] = __builtin_fmaf(grid_step(grid[i]), acc[i], grid_offset(grid[i]) * qs);
        }
        uint32_t vg[16];                                      // V's grids of the same keys
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) {
            const uint4 x = grids(kVGridAt, kt);
            vg[4 * kt] = x.x;
            vg[4 * kt + 1] = x.y;
            vg[4 * kt + 2] = x.z;
            vg[4 * kt + 3] = x.w;
        }
        float most = 0.0f;                                    // the largest step, where E has to grow
        if (masked) {
            float offset = 0.0f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const bool seen = key0 + i <= last;
                sc[i >> 2][i & 3] = seen ? sc[i >> 2][i & 3] : kNegInf;
                vg[i] = seen ? vg[i] : 0u;
                most = fmaxf(most, fabsf(grid_step(vg[i])));
                offset = fmaxf(offset, offset_bound(vg[i]));
            }
            most = pair32_max(pair16_max(fmaxf(most, offset * kOffsetSize)));
        } else {
            const float own = grid_size(*(const uint32_t *)(step + kVGridAt + 4 * lane));
            if (__ballot(own > least_limit)) most = -wave_min(-own);
        }
        float mt = kNegInf;
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) mt = fmaxf(mt, fmaxf(fmaxf(sc[kt][0], sc[kt][1]), fmaxf(sc[kt][2], sc[kt][3])));
        mt = pair32_max(pair16_max(mt));
        const bool own = (mt - m) * c > kLazy;
        if (__ballot(own || most > scale.limit)) {
            const float mn = own ? mt : m;
            rescale(exp2_hw((m - (mn == kNegInf ? 0.0f : mn)) * c));
            m = mn;
            if (__ballot(most > scale.limit)) {
                rescale(scale.raise(most));
                least_limit = wave_min(scale.limit);
            }
        }
        float e[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) e[i] = sc[i >> 2][i & 3];
        weights(e, m, c, scale.e);
        uint32_t p[8];
        weigh(e, vg, l, z, p);
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) {
            const v2i t = lds_read_tr4(step + vat[dt >> 1] + 8 * (dt & 1));
            o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(operand(extract.pairs(t[0])), operand(p), o[dt], 0, 0, 0);
            o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(operand(extract.pairs(t[1])), operand(p + 4), o[dt], 0, 0, 0);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");    // this stage has been read
        if (u + 2 * kKvWaves < u1) load.issue(u + 2 * kKvWaves, st);
    }
    const float up = power_of_two((int)scale.e);
    l = pair32_sum(pair16_sum(l)) * up;
    z = pair32_sum(pair16_sum(z));
    m *= back;

    // the waves' sums through LDS, in the matrix cores' order
    __syncthreads();
    v4f *sums = (v4f *)&ring[0][0][0];
    static_assert(sizeof(ring) >= sizeof(v4f) * kKvWaves * 8 * 64, "the sums fit the ring");
    if (g == 0) ml[wave][r] = make_float2(m, l);
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) sums[(wave * 8 + dt) * 64 + lane] = (o[dt] * kCodes + z) * up;
    __syncthreads();
    if (r >= w.rows) return;
#pragma unroll
    for (int dt = wave; dt < 8; dt += kKvWaves) {
        v4f acc;
        const float2 e = merged<kKvWaves>(&ml[0][r], R, sums + dt * 64 + lane, 8 * 64, a.c, acc);
        const int d = 16 * dt + 4 * g;
        if (a.S == 1) {
            store_out(a, w, row, d, acc, e.y);
        } else {
            *(v4f *)(unit_at<R>(a, w.split, dt) + 4 * lane) = acc;
            if (dt == 0 && g == 0) *row_ml<R>(a, w.split, r) = e;
        }
    }
}

// ---------------------------------------------------------------- more rows

// Tiles of 32 rows, every wave with its own steps.
__global__ __launch_bounds__(kKvWaves * 64, 2) void k_kv4_rows(CausalKv4Args x) {
    constexpr int R = 32;
    const CausalArgs &a = x.a;
    __shared__ __attribute__((aligned(16))) char ring[kKvWaves][kKvStages][kStepBytes];     // then the waves' sums
    __shared__ float2 ml[kKvWaves][R];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int hi = lane >> 5, r = lane & 31;
    Work w;
    if (!find_work<R, true>(a, lane, blockIdx.y, w)) return;
    const Range range = range_of(a, (w.hi + kKv4Keys - 1) / kKv4Keys, w.split);
    if (a.S > 1 && w.split >= range.used) return;
    const int u0 = range.first, u1 = range.end;
    const Loader<2> load(x, w, lane, lds_addr(ring[wave]));
    if (u0 + wave < u1) load.issue(u0 + wave, 0);
    if (u0 + wave + kKvWaves < u1) load.issue(u0 + wave + kKvWaves, 1);

    // queries: B operand, row r; K's word ks of lane half hi is dimensions 64 hi + 8 ks .. + 7
    const RowOf row = row_of(a, w, min(r, w.rows - 1));
    const int last = w.s.p0 + row.i;                          // last key that the row sees
    const int first_last = w.s.p0 + w.i0;                     // keys up to here are seen by every row
    v8h qf[8];
    float qs, back;
    load_queries<8>(a.q + row_at(w, row, a.q_stride) + 64 * hi, qf, qs, back, pair32_max, pair32_sum);
    const float c = a.c * back;
    const ExtractConsts<true> extract;

    // places in half a step (32 keys): K of key 16 ((r >> 2) & 1) + 4 (r >> 3) + (r & 3), V of key
    // 16 hi + (lane & 15), grids of keys 16 hi ..
    const int kkey = 16 * ((r >> 2) & 1) + 4 * (r >> 3) + (r & 3), kor = k_order<2>(kkey);
    const int kat0 = kkey * 64 + 16 * ((2 * hi) ^ kor), kat1 = kkey * 64 + 16 * ((2 * hi + 1) ^ kor);
    int vat[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) vat[i] = kVAt + (16 * hi + (lane & 15)) * 64 + 16 * (i ^ v_order(lane & 15)) + 8 * ((lane >> 4) & 1);
    float m = kNegInf, l = 0.0f, z = 0.0f;                    // maximum; sums of p and p o
    StepScale scale;
    float least_limit = 0.0f;                                 // of the wave's rows
    v16f o[4];
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[dt][i] = 0.0f;
    auto rescale = [&](float by) {
        l *= by;
        z *= by;
#pragma unroll
        for (int dt = 0; dt < 4; ++dt) o[dt] *= by;
    };
    int st = 0;
    for (int u = u0 + wave; u < u1; u += kKvWaves, st ^= 1) {
        load.wait(u + kKvWaves < u1);
        const bool masked = (u + 1) * kKv4Keys - 1 > first_last;
        const char *const stage = ring[wave][st];
        float most_all = 0.0f;                                // the largest step, where some row's E has to grow
        if (!masked) {
            const float own = grid_size(*(const uint32_t *)(stage + kVGridAt + 4 * lane));
            if (__ballot(own > least_limit)) most_all = -wave_min(-own);
        }
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
            if (u * kKv4Keys + 32 * half >= w.hi) break;
            const char *step = stage + half * 32 * 64, *grids = stage + half * 32 * 4;
            const int key0 = u * kKv4Keys + 32 * half + 16 * hi;          // this lane's keys: key0 + i
            const uint4 k0 = *(const uint4 *)(step + kat0), k1 = *(const uint4 *)(step + kat1);
            const uint32_t word[8] = {k0.x, k0.y, k0.z, k0.w, k1.x, k1.y, k1.z, k1.w};
            v16f sc;
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[i] = 0.0f;
#pragma unroll
            for (int ks = 0; ks < 8; ++ks)
                sc = __builtin_amdgcn_mfma_f32_32x32x16_f16(operand(extract.pairs(word[ks])), qf[ks], sc, 0, 0, 0);
            uint32_t vg[16];
            float e[16];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint4 kg = *(const uint4 *)(grids + kKGridAt + 4 * (16 * hi + 4 * j));
                const uint4 g = *(const uint4 *)(grids + kVGridAt + 4 * (16 * hi + 4 * j));
                const uint32_t grid[4] = {kg.x, kg.y, kg.z, kg.w};
                vg[4 * j] = g.x;
                vg[4 * j + 1] = g.y;
                vg[4 * j + 2] = g.z;
                vg[4 * j + 3] = g.w;
#pragma unroll
                for (int i = 0; i < 4; ++i) e[4 * j + i] = __builtin_fmaf(grid_step(grid[i]), sc[4 * j + i], grid_offset(grid[i]) * qs);
            }
            float most = most_all;
            if (masked) {
                float offset = 0.0f;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const bool seen = key0 + i <= last;
                    e[i] = seen ? e[i] : kNegInf;
                    vg[i] = seen ? vg[i] : 0u;
                    most = fmaxf(most, fabsf(grid_step(vg[i])));
                    offset = fmaxf(offset, offset_bound(vg[i]));
                }
                most = pair32_max(fmaxf(most, offset * kOffsetSize));
            }
            float mt = kNegInf;
#pragma unroll
            for (int i = 0; i < 16; ++i) mt = fmaxf(mt, e[i]);
            mt = pair32_max(mt);
            const bool own = (mt - m) * c > kLazy;
            if (__ballot(own || most > scale.limit)) {
                const float mn = own ? mt : m;
                rescale(exp2_hw((m - (mn == kNegInf ? 0.0f : mn)) * c));
                m = mn;
                if (__ballot(most > scale.limit)) {
                    rescale(scale.raise(most));
                    least_limit = wave_min(scale.limit);
                }
            }
            weights(e, m, c, scale.e);
            uint32_t p[8];
            weigh(e, vg, l, z, p);
#pragma unroll
            for (int dt = 0; dt < 4; ++dt) {
                const v2i v = lds_read_tr4(step + vat[dt]);
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(operand(extract.pairs(v[h])), operand(p + 4 * h), o[dt], 0, 0, 0);
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");    // this stage has been read
        if (u + 2 * kKvWaves < u1) load.issue(u + 2 * kKvWaves, st);
    }
    // the waves' sums through LDS, in the matrix cores' order
    const float up = power_of_two((int)scale.e);
    l = pair32_sum(l) * up;
    z = pair32_sum(z);
    __syncthreads();
    v4f *const sums = (v4f *)&ring[0][0][0];
    static_assert(sizeof(ring) >= sizeof(v4f) * kKvWaves * 16 * 64, "the sums fit the ring");
    if (hi == 0) ml[wave][r] = make_float2(m * back, l);
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const v4f y = {o[dt][4 * i], o[dt][4 * i + 1], o[dt][4 * i + 2], o[dt][4 * i + 3]};
            sums[(wave * 16 + dt * 4 + i) * 64 + lane] = (y * kCodes + z) * up;
        }
    __syncthreads();
    if (r >= w.rows) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int unit = 4 * wave + j;                        // dimensions 8 unit + 4 hi .. + 3
        v4f acc;
        const float2 e = merged<kKvWaves>(&ml[0][r], R, sums + unit * 64 + lane, 16 * 64, a.c, acc);
        if (a.S == 1) {
            store_out(a, w, row, 8 * unit + 4 * hi, acc, e.y);
        } else {
            *(v4f *)(unit_at<R>(a, w.split, unit) + 4 * lane) = acc;
            if (unit == 0 && hi == 0) *row_ml<R>(a, w.split, r) = e;
        }
    }
}

// ---------------------------------------------------------------- unpacking

// Where a sequence's tokens [first, end) of a tile go; false: nowhere.
__device__ inline bool unpack_range(const UnpackArgs &a, int64_t item, Seq &s, int &b, int &h, int &tile, int64_t &to0, int &first, int &end) {
    const int64_t at = item / a.tiles;
    tile = (int)(item - at * a.tiles);
    b = (int)(at / a.heads);
    h = (int)(at - (int64_t)b * a.heads);
    s = load_seq(a.b, b);
    to0 = a.shifts ? (int64_t)b * a.to_seq_slots : s.slot0;
    if (s.L == 0 || (a.shifts && s.rows == 0)) return false;
    if (!a.shifts) {
        int64_t room = a.to_capacity ? a.to_capacity : a.to_slots;
        if (a.to_capacity && a.to_seq_slots) room -= to0 % a.to_seq_slots;
        if (to0 > a.to_slots - s.L || s.L > room) return false;
    }
    first = a.new_only ? max(s.p0, 0) : 0;
    end = a.new_only ? min(s.p0 + s.rows, s.L) : s.L;
    return true;
}

// The largest |value| of each row of keys and of values: the largest and smallest of them in each
// kPeakTokens tokens of a sequence's head, without zeros, infinities and NaN.  A code's value
// lies between offset and offset + 15 step.
__global__ __launch_bounds__(256) void k_kv4_peaks(UnpackArgs a) {
    __shared__ float4 part[4];
    Seq s;
    int b, h, tile, first, end;
    int64_t to0;
    if (!unpack_range(a, blockIdx.x, s, b, h, tile, to0, first, end)) return;
    constexpr float kNone = __builtin_huge_valf();
    float4 p = make_float4(0.0f, 0.0f, kNone, kNone);
    auto peak = [](uint32_t g) { return fmaxf(fabsf(grid_offset(g)), fabsf(__builtin_fmaf(15.0f, grid_step(g), grid_offset(g)))); };
    auto join = [](const float4 &x, const float4 &y) { return make_float4(fmaxf(x.x, y.x), fmaxf(x.y, y.y), fminf(x.z, y.z), fminf(x.w, y.w)); };
#pragma unroll
    for (int i = 0; i < kPeakTokens; i += 256) {
        const int j = tile * kPeakTokens + i + (int)threadIdx.x;
        if (j >= end) continue;
        const int64_t row = (s.slot0 + j) * a.b.tok + (int64_t)h * a.b.head;
        const float k = peak(a.c.k_grid[row]), v = peak(a.c.v_grid[row]);
        const bool on_k = k > 0.0f && k < kNone, on_v = v > 0.0f && v < kNone;
        p = join(p, make_float4(on_k ? k : 0.0f, on_v ? v : 0.0f, on_k ? k : kNone, on_v ? v : kNone));
    }
    p = make_float4(-wave_min(-p.x), -wave_min(-p.y), wave_min(p.z), wave_min(p.w));
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = p;
    __syncthreads();
    if (threadIdx.x == 0) a.peaks[blockIdx.x] = join(join(part[0], part[1]), join(part[2], part[3]));
}

// 16 lanes a row, a word of codes and 16 bytes of bf16 a lane; workgroups walk the tiles of
// tokens of all sequences and heads.  Bound by the 16-bit values written.  SCALED: for
// k_causal_prompt in f16, whose 11 bits keep what bf16's 8 would lose, each head of a
// sequence times a power of two that brings it into f16's range; where its rows are further
// apart than 2^12, each row times one of its own.
template <bool SCALED>
__global__ __launch_bounds__(256) void k_unpack_kv4(UnpackArgs a) {
    const int l = threadIdx.x & 15, grp = threadIdx.x >> 4, lane = threadIdx.x & 63;
    for (int64_t item = blockIdx.x; item < a.items; item += gridDim.x) {
        Seq s;
        int b, h, tile, first, end;
        int64_t to0;
        const bool on = unpack_range(a, item, s, b, h, tile, to0, first, end);
        if (SCALED && tile == 0 && h == 0 && threadIdx.x == 0) a.length[b] = s.L;
        if (!on || first + tile * kUnpackTokens >= end) continue;
        float f[2] = {1.0f, 1.0f};
        bool by_row = false;
        if constexpr (SCALED) {
            // the same in every lane: scalar loads, and no exchange across lanes while there are few
            float4 p = make_float4(0.0f, 0.0f, __builtin_huge_valf(), __builtin_huge_valf());
            const float4 *peaks = a.peaks + ((int64_t)b * a.heads + h) * a.peak_tiles;
            const int n = (end + kPeakTokens - 1) / kPeakTokens;
            auto add = [&](const float4 &x) { p = make_float4(fmaxf(p.x, x.x), fmaxf(p.y, x.y), fminf(p.z, x.z), fminf(p.w, x.w)); };
            if (n <= 8) {
                for (int i = 0; i < n; ++i) add(peaks[i]);
            } else {
                for (int i = lane; i < n; i += 64) add(peaks[i]);
                p = make_float4(-wave_min(-p.x), -wave_min(-p.y), wave_min(p.z), wave_min(p.w));
            }
            by_row = p.z < p.x * (1.0f / 4096.0f) || p.w < p.y * (1.0f / 4096.0f);
            const int k = by_row ? 0 : f16_exponent(p.x) - 14, v = by_row ? 0 : f16_exponent(p.y) - 14;
            if (tile == 0 && threadIdx.x == 0) a.shifts[(int64_t)b * a.heads + h] = HeadShift{(short)k, (short)v, by_row};
            f[0] = power_of_two(-k);
            f[1] = power_of_two(-v);
        }
        constexpr int kRows = kUnpackTokens / 16;             // of a group of 16 lanes, requested together
        uint32_t w[kRows][2], g[kRows][2];
        const int j0 = first + tile * kUnpackTokens + grp;
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int64_t row = (s.slot0 + min(j0 + 16 * i, end - 1)) * a.b.tok + (int64_t)h * a.b.head;
            w[i][0] = a.c.k[16 * row + l];
            w[i][1] = a.c.v[16 * row + l];
            g[i][0] = a.c.k_grid[row];
            g[i][1] = a.c.v_grid[row];
        }
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int j = j0 + 16 * i;
            if (j >= end) break;
            const int64_t to = (to0 + j) * a.to_tok + (int64_t)h * a.to_head + 8 * l;
            if (SCALED && by_row) {
                auto shift = [](uint32_t g) {
                    return f16_exponent(fmaxf(fabsf(grid_offset(g)), fabsf(__builtin_fmaf(15.0f, grid_step(g), grid_offset(g))))) - 14;
                };
                const int k = shift(g[i][0]), v = shift(g[i][1]);
                if (l == 0) a.row_shifts[((int64_t)b * a.heads + h) * a.to_capacity + j] = make_short2((short)k, (short)v);
                f[0] = power_of_two(-k);
                f[1] = power_of_two(-v);
            }
#pragma unroll
            for (int kv = 0; kv < 2; ++kv) {
                const float st = grid_step(g[i][kv]) * f[kv], of = grid_offset(g[i][kv]) * f[kv];
                uint32_t y[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x0 = __builtin_fmaf(st, (float)(w[i][kv] >> 8 * e & 15u), of), x1 = __builtin_fmaf(st, (float)(w[i][kv] >> (8 * e + 4) & 15u), of);
                    y[e] = SCALED ? cvt_pk_f16(x0, x1) : cvt_pk_bf16(x0, x1);
                }
                *(uint4 *)((kv ? a.v : a.k) + to) = make_uint4(y[0], y[1], y[2], y[3]);
            }
        }
    }
}

}  // namespace

const char *causal_kv4_kernel_name(int rt) { return rt == 1 ? "k_kv4_few" : "k_kv4_rows"; }

hipError_t launch_causal_kv4(const CausalKv4Args &args, int rt, hipStream_t st) {
    CausalKv4Args x = args;
    x.a.step_shift = shift_of(kKv4Keys);
    const dim3 grid((unsigned)(x.a.tiles * x.a.Hkv), (unsigned)x.a.S), threads(kKvWaves * 64);
    if (rt == 1) hipLaunchKernelGGL(k_kv4_few, grid, threads, 0, st, x);
    else hipLaunchKernelGGL(k_kv4_rows, grid, threads, 0, st, x);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess || x.a.S == 1 ? e : launch_kv4_join(x.a, rt, st);
}

hipError_t launch_unpack_kv4(const UnpackArgs &a, hipStream_t st) {
    if (a.items == 0) return hipSuccess;
    const dim3 grid((unsigned)(a.items < 65536 ? a.items : 65536));
    if (!a.shifts) {
        hipLaunchKernelGGL(k_unpack_kv4<false>, grid, dim3(256), 0, st, a);
        return hipGetLastError();
    }
    UnpackArgs peaks = a;
    peaks.tiles = a.peak_tiles;
    hipLaunchKernelGGL(k_kv4_peaks, dim3((unsigned)(a.items / a.tiles * a.peak_tiles)), dim3(256), 0, st, peaks);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_unpack_kv4<true>, grid, dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace qlin
