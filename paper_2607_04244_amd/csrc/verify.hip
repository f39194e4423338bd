// The decision on drafted tokens (qlin_verify_draft in include/qlin_target.h).
//
// Bound by the bytes of the logits and the 64-bit exponentials of all of them:
//   k_verify_stats   (row, chunk of 4096 tokens): maximum, its lowest index, and the sum of
//       the weights e^((x - maximum) / T).
//   k_verify_decide  (sequence): whether the first rows already refuse a token.  Large calls
//       only: the statistics of the other rows are then taken where they can still matter.
//   k_verify_weigh   (sequence, chunks), with draft logits: the accepted prefix from the rows'
//       statistics, and, if a token was refused, the chunk's sum of max(P - Q, 0).
//   k_verify_pick    (sequence): the chunk, then the token, that the running sum passes the
//       uniform number in.  Without draft logits the chunks' sums follow from the statistics,
//       and the accepted prefix is found here.
//
// Weights are 64-bit numbers with a relative error of 4.7e-11 (Pow2 below: about 34 bits), their sums
// 64-bit: a running sum over a vocabulary of 10^5 has a boundary every 10^-5 of it or closer, and
// 32-bit weights (off by up to 6e-8 each) would put a few of a thousand choices on the wrong
// side of one.  At 4.7e-11 it is one of 10^5.
// 64-bit products run at the rate of 32-bit ones here, and 32-bit exponentials at a half of
// it, so the accuracy costs about twice the time of 32-bit weights.  A table of 2^(j/32) or
// 2^(j/64) in LDS or lanes with a polynomial of degree 3 took 32 sequences from 84 to 81 us and
// one from 14.3 to 14.9; not taken.
//
// 16 tokens over 151936: 11.2 to 11.6 us in a graph, of which the statistics 5.4 (one trip to memory,
// 38 chunks a row over all compute units) and the token 6.6, a workgroup's dependent steps: decision
// 3.2, chunk 1.2, its logits 1, token 1.  Handing the decision what it reads again later, or the
// drafted tokens' logits with the statistics, took trips to memory away but no time: it is the
// latency of the instructions.  32 sequences of 16 with draft logits: 80 to 103 us on different cards
// and orders of memory (statistics 38 + 20, decision 4.6, sums 16, token 6.3), where the 5 TB/s of
// a copy would read all the logits in 63; the statistics are bound by their 64-bit
// instructions, 14 a logit.
#include "device_common.h"
#include "target_internal.h"

namespace qlin {

namespace {

constexpr float kNegInf = -__builtin_huge_valf(), kPosInf = __builtin_huge_valf();
constexpr int kChunkVecs = kVerifyChunk / 8;             // vectors of 8 logits
constexpr int kPickThreads = 1024, kPickWaves = kPickThreads / 64, kWeighThreads = kChunkVecs;
static_assert(kChunkVecs <= kPickThreads, "a chunk's vectors");

// 2^t, relative error 4.7e-11: (2^f - 1) / f on [-1/2, 1/2] as the polynomial of degree 6 whose
// largest weighted error is smallest.  The coefficients are opaque scalars:
// of constants the compiler makes copies into the accumulator, two moves a product.
struct Pow2 {
    double c[6];
    __device__ inline Pow2() : c{0.6931471807045319, 0.2402265106656167, 0.05550410365990573, 0.009618038132000921,
                                 0.0013333935056283428, 0.00015466756333052078} {
#pragma unroll
        for (int i = 0; i < 6; ++i) asm("" : "+s"(c[i]));
    }
    __device__ inline double fraction(double f) const {
        double p = __builtin_fma(f, 1.5196156371520414e-05, c[5]);
#pragma unroll
        for (int i = 4; i >= 0; --i) p = __builtin_fma(p, f, c[i]);
        return __builtin_fma(p, f, 1.0);
    }
    // -1100 <= t < 1000; 0 below the smallest number.  Rounding by the sum with 1.5 2^52, whose low
    // word is the integer.
    static constexpr double kRound = 6755399441055744.0;
    __device__ inline double operator()(double t) const {
        const double n = t + kRound;
        return __builtin_amdgcn_ldexp(fraction(t - (n - kRound)), (int)(uint32_t)__builtin_bit_cast(uint64_t, n));
    }
    // -1000 <= t < 1000: the exponent by a sum of the upper words, kept from the compiler, which
    // adds both words in four instructions (32 sequences 88.2 us a call, 84.1 so)
    __device__ inline double within(double t) const {
        const double n = t + kRound;
        const uint64_t p = __builtin_bit_cast(uint64_t, fraction(t - (n - kRound)));
        uint32_t hi = (uint32_t)(p >> 32);
        asm("" : "+v"(hi));
        hi += (uint32_t)__builtin_bit_cast(uint64_t, n) << 20;
        return __builtin_bit_cast(double, (uint64_t)hi << 32 | (uint32_t)p);
    }
};

// log2(e) / T, in 45 bits (relative error 2^-45): its product with a bf16 number, of 8 bits, is
// exact in 64, so that k x - k m is rounded once, as a difference, and is 0 for the maximum
// however large |m| / T is.  (With k in 53 bits the rounding of k m stays in every exponent, and
// from |m| / T = 10^19 it exceeds the range of the weights.)
__device__ inline double exponent_scale(float T) {
    const uint64_t u = __builtin_bit_cast(uint64_t, 1.4426950408889634 / (double)T);
    return __builtin_bit_cast(double, (u + 0x80) & ~(uint64_t)0xFF);
}

// Weights of a row or chunk: 2^(k x - n), k = exponent_scale(T), n = ceil(k m), m its maximum.
// With a whole n the weights of the same logit relative to two maxima differ by a power of two
// exactly, so that sums over chunks cut differently, of two rows with the same logits, agree to
// the rounding of the sums.  -infinity and NaN give 0 (2^-1100 is below the smallest number);
// where m is infinite, its equals have weight 1 and all others none.
struct Scale {
    double k, n;
    bool inf;
    Pow2 pow2;
    __device__ inline Scale(double k_, float m) : k(k_), n(ceil(k_ * (double)m)), inf(m == kPosInf) {}
    __device__ inline double operator()(float x) const {
        return inf ? (x == kPosInf ? 1.0 : 0.0) : pow2(fmax(__builtin_fma((double)x, k, -n), -1100.0));
    }
    // of eight logits: one branch
    __device__ inline void weights(const float x[8], double w[8]) const {
        if (inf) {
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = x[e] == kPosInf ? 1.0 : 0.0;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = pow2(fmax(__builtin_fma((double)x[e], k, -n), -1100.0));
        }
    }
    // their sum, where weights below 2^-1000 may count as that: next to the maximum's, 1/2 to 1,
    // they are no part of a 64-bit sum
    __device__ inline double sum(const float x[8]) const {
        double s[2] = {0.0, 0.0};
        if (inf) {
#pragma unroll
            for (int e = 0; e < 8; ++e) s[0] += x[e] == kPosInf ? 1.0 : 0.0;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e & 1] += pow2.within(fmax(__builtin_fma((double)x[e], k, -n), -1000.0));
        }
        return s[0] + s[1];
    }
};
// The factor from weights relative to m to weights relative to the larger M: a power of two.
__device__ inline double rescale(double k, float m, float M) {
    return m == M ? 1.0 : m == kNegInf || M == kPosInf ? 0.0 : __builtin_amdgcn_ldexp(1.0, (int)fmax(ceil(k * (double)m) - ceil(k * (double)M), -1100.0));
}

// Sums, maxima and minima over the lanes by DPP: within rows of 16 (row_shr 1, 2, 4, 8), then
// lane 15 of a row to the next and lane 31 to the upper half; lane 63 has them all.  Lanes
// without a partner keep `old`.  (Shuffles go through LDS: 12 of them in a row, for a 64-bit
// sum, cost a microsecond.)
template <int CTRL, int ROWS>
__device__ inline int dpp(int old, int v) { return __builtin_amdgcn_update_dpp(old, v, CTRL, ROWS, 0xF, false); }
template <int CTRL, int ROWS>
__device__ inline double dpp(double v) {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = dpp<CTRL, ROWS>(0, (int)(uint32_t)u), hi = dpp<CTRL, ROWS>(0, (int)(uint32_t)(u >> 32));
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// Inclusive sum over the lanes.
__device__ inline double lanes_upto(double v) {
    v += dpp<0x111, 0xF>(v);
    v += dpp<0x112, 0xF>(v);
    v += dpp<0x114, 0xF>(v);
    v += dpp<0x118, 0xF>(v);
    v += dpp<0x142, 0xA>(v);
    v += dpp<0x143, 0xC>(v);
    return v;
}
__device__ inline double from_lane(double v, int l) {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)u, l), hi = __builtin_amdgcn_readlane((uint32_t)(u >> 32), l);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ inline double wave_sum(double v) { return from_lane(lanes_upto(v), 63); }
template <int CTRL, int ROWS>
__device__ inline float dpp_max(float v) { return fmaxf(v, __int_as_float(dpp<CTRL, ROWS>(__float_as_int(v), __float_as_int(v)))); }
__device__ inline float wave_max(float v) {
    v = dpp_max<0x111, 0xF>(v);
    v = dpp_max<0x112, 0xF>(v);
    v = dpp_max<0x114, 0xF>(v);
    v = dpp_max<0x118, 0xF>(v);
    v = dpp_max<0x142, 0xA>(v);
    v = dpp_max<0x143, 0xC>(v);
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
__device__ inline int wave_min(int v) {
    v = min(v, dpp<0x111, 0xF>(v, v));
    v = min(v, dpp<0x112, 0xF>(v, v));
    v = min(v, dpp<0x114, 0xF>(v, v));
    v = min(v, dpp<0x118, 0xF>(v, v));
    v = min(v, dpp<0x142, 0xA>(v, v));
    v = min(v, dpp<0x143, 0xC>(v, v));
    return __builtin_amdgcn_readlane(v, 63);
}

// What a sequence asks for.
struct Request {
    int count;
    bool greedy;
    double k;               // exponent_scale(T)
};
__device__ inline Request load_request(const VerifyArgs &a, int b) {
    Request r;
    r.count = a.count ? min(max(a.count[b], 0), a.n) : a.n;
    const float T = a.temperature ? a.temperature[b] : 1.0f;
    r.greedy = !(T > 0.0f);
    r.k = r.greedy ? 1.0 : exponent_scale(T);
    return r;
}

// A row of logits in vectors of 8: its first logit is element `off` of the first vector, which
// is 16-byte aligned.
struct Row {
    int off;
    const uint16_t *base;   // of the first vector
    __device__ inline Row(const uint16_t *p) : off((int)((uintptr_t)p & 15) / 2), base(p - off) {}
};
// Logits 8 v - off .. + 7 of a row, -infinity outside it.  A vector that ends past the row is
// read logit by logit: the row may be the last of its memory.  (One that starts before it
// starts in the row before.)
__device__ inline void load_logits(const Row &r, int v, int V, float x[8]) {
    const int j0 = 8 * v - r.off;
    if (j0 + 8 <= V) {
        const uint4 w = *(const uint4 *)(r.base + 8 * (int64_t)v);
        const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = bf16_lo_to_f32(ww[i]);
            x[2 * i + 1] = bf16_hi_to_f32(ww[i]);
        }
        if (v == 0)
#pragma unroll
            for (int i = 0; i < 7; ++i) x[i] = i < r.off ? kNegInf : x[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = j0 + i >= 0 && j0 + i < V ? __uint_as_float((uint32_t)r.base[8 * (int64_t)v + i] << 16) : kNegInf;
    }
}

// The rows of sequence b: target rows 0 .. n, then draft rows 0 .. n - 1 (`which` in this order).
__device__ inline const uint16_t *target_row(const VerifyArgs &a, int b, int i) { return a.target + ((int64_t)b * (a.n + 1) + i) * a.target_stride; }
__device__ inline const uint16_t *draft_row(const VerifyArgs &a, int b, int i) { return a.draft + ((int64_t)b * a.n + i) * a.draft_stride; }

// One workgroup of T threads a (row, chunk); each thread holds its logits in registers between
// the maximum and the weights.
template <int T>
__global__ __launch_bounds__(T) void k_verify_stats(VerifyArgs a) {
    constexpr int kStatsThreads = T, kStatsVecs = kChunkVecs / T;
    __shared__ VerifyStat part[kStatsThreads / 64];
    __shared__ float wave_m[kStatsThreads / 64];
    // this launch's rows: targets [row0, row1), then drafts [row0, row1) that there are
    const int b = blockIdx.y, x_row = blockIdx.x / a.chunks, c = blockIdx.x - x_row * a.chunks;
    const bool is_draft = x_row >= a.row1 - a.row0;
    const int i = a.row0 + (is_draft ? x_row - (a.row1 - a.row0) : x_row), which = is_draft ? a.n + 1 + i : i;
    const Request rq = load_request(a, b);
    if (is_draft ? i >= rq.count || rq.greedy : i > rq.count) return;
    if (a.row0 > 0 && a.decisions[b].done) return;               // the first rows sufficed
    const Row row(is_draft ? draft_row(a, b, i) : target_row(a, b, i));
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float x[kStatsVecs][8];
    const int v0 = c * kChunkVecs + threadIdx.x;
#pragma unroll
    for (int k = 0; k < kStatsVecs; ++k) load_logits(row, v0 + k * kStatsThreads, a.V, x[k]);
    float m = kNegInf;
#pragma unroll
    for (int k = 0; k < kStatsVecs; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) m = fmaxf(m, x[k][e]);           // ignores NaN
    m = wave_max(m);
    // the chunk's maximum, so that all its weights are relative to one
    if (lane == 0) wave_m[wave] = m;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kStatsThreads / 64; ++k) m = fmaxf(m, wave_m[k]);
    VerifyStat st{m, 0x7FFFFFFF, 0.0};
    if (rq.greedy) {
#pragma unroll
        for (int k = kStatsVecs - 1; k >= 0; --k)
#pragma unroll
            for (int e = 7; e >= 0; --e)
                if (x[k][e] == m) st.at = 8 * (v0 + k * kStatsThreads) - row.off + e;
        st.at = wave_min(st.at);
    } else if (m != kNegInf) {
        const Scale w(rq.k, m);
        double s = 0.0;
#pragma unroll
        for (int k = 0; k < kStatsVecs; ++k) s += w.sum(x[k]);
        st.z = wave_sum(s);
    }
    if (lane == 0) part[wave] = st;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int k = 1; k < kStatsThreads / 64; ++k) {
            st.at = min(st.at, part[k].at);
            st.z += part[k].z;
        }
        a.stats[((int64_t)b * a.all_rows + which) * a.chunks + c] = st;
    }
}

// A row's statistics from its chunks', by a wave; `own` is its lane's chunk, loaded before.
__device__ inline const VerifyStat *row_stats(const VerifyArgs &a, int b, int which) {
    return a.stats + ((int64_t)b * a.all_rows + which) * a.chunks;
}
__device__ inline VerifyStat row_stat(const VerifyArgs &a, int b, int which, const VerifyStat &own, double k, int lane) {
    const VerifyStat *p = row_stats(a, b, which);
    VerifyStat st = own;
    for (int c = lane + 64; c < a.chunks; c += 64) {
        const VerifyStat e = p[c];
        const float M = fmaxf(st.m, e.m);
        st.z = st.z * rescale(k, st.m, M) + e.z * rescale(k, e.m, M);
        st.at = e.m > st.m ? e.at : e.m == st.m ? min(st.at, e.at) : st.at;
        st.m = M;
    }
    const float M = wave_max(st.m);
    const double z = wave_sum(st.z * rescale(k, st.m, M));
    return VerifyStat{M, wave_min(st.m == M ? st.at : 0x7FFFFFFF), z};
}

// The probability of a token with logit x in a row with these statistics.
__device__ inline double probability(float x, const VerifyStat &st, double k) {
    return st.z > 0.0 ? Scale(k, st.m)(x) / st.z : 0.0;
}

// P and Q closer than this, relative to P, are equal: the weights of equal logits are equal, so P and
// Q of equal rows differ by the rounding of two sums of up to 90 steps one after the other (9 in a
// thread, 9 over a workgroup, 65 chunks in a lane, 6 over the lanes) and of two quotients, below
// 190 2^-53.  Without it the next token would be drawn from that rounding.  Subnormal probabilities
// are rounded more coarsely; differences of that size count as none too.
constexpr double kSame = 0x1p-44, kNone = 0x1p-960;

// A chunk whose largest weight is below this, relative to the row's, holds no token to draw.  So a
// chunk with any mass has a token whose probability is a number: without a refused token its
// largest one, above 2^-901 2^-24; and what is left of a sum after a refused token's weight is
// taken out, if anything is, was at least 2^-54 of it, over 4096 tokens.
constexpr double kLeast = 0x1p-900;

// The weights that the next token is drawn by, in 8 tokens of a chunk: those of the target's
// row, less the draft's (or the drafted token's) if `rest`.
struct Choice {
    Row row;
    const uint16_t *q;      // draft row, or null
    int x;                  // drafted token that has all the draft's mass, or -1
    double k, zp, zq;
    float mp, mq;
    __device__ inline void weights(int v, int V, bool rest, double w[8]) const {
        float l[8];
        load_logits(row, v, V, l);
        const Scale p(k, mp);
        const double inv_p = 1.0 / zp;
        p.weights(l, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] *= inv_p;
        if (!rest) return;
        const int j0 = 8 * v - row.off;
        if (q) {
            const Scale s(k, mq);
            const double inv_q = zq > 0.0 ? 1.0 / zq : 0.0;
            const Row qr(q);
            float d[8];
            if (qr.off == row.off) {
                load_logits(qr, v, V, d);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) d[e] = j0 + e >= 0 && j0 + e < V ? __uint_as_float((uint32_t)q[j0 + e] << 16) : kNegInf;
            }
            double we[8];
            s.weights(d, we);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const double d = __builtin_fma(-we[e], inv_q, w[e]);
                w[e] = d > __builtin_fma(kSame, w[e], kNone) ? d : 0.0;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (j0 + e == x) w[e] = 0.0;
        }
    }
};

__device__ inline Choice choice_of(const VerifyArgs &a, int b, const VerifyDecision &d, double k) {
    const bool q = d.rejected && a.draft;
    return Choice{Row(target_row(a, b, d.accepted)), q ? draft_row(a, b, d.accepted) : nullptr,
                  d.rejected && !a.draft ? a.drafted[b * a.n + d.accepted] : -1, k, d.p.z, d.q.z, d.p.m, d.q.m};
}

// The decision of a sequence from the statistics of its rows below `limit`, a wave a row: the
// first refused token, or all accepted (done only if row `count` is below the limit too).
struct Rows { VerifyStat p[kVerifyMaxDraft + 1], q[kVerifyMaxDraft + 1]; int keep[kVerifyMaxDraft + 1]; };
__device__ inline VerifyDecision decide(const VerifyArgs &a, int b, int limit, Rows &rows, Request &rq) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const VerifyStat none{kNegInf, 0x7FFFFFFF, 0.0};
    // everything but the drafted token's logits in one trip to memory, a row ahead and also for rows
    // that turn out to be behind the last (their statistics are not used)
    struct Ahead { VerifyStat own_p, own_q; int x; float u; };
    auto request = [&](int i) {
        Ahead r{none, none, -1, 0.0f};
        if (i > a.n || i >= limit) return r;
        if (lane < a.chunks) r.own_p = row_stats(a, b, i)[lane];
        if (a.draft && i < a.n && lane < a.chunks) r.own_q = row_stats(a, b, a.n + 1 + i)[lane];
        if (i < a.n) r.x = a.drafted[b * a.n + i];
        r.u = a.uniform[b * (a.n + 1) + i];
        return r;
    };
    const int waves = blockDim.x >> 6;
    Ahead next = request(wave);
    rq = load_request(a, b);                    // waves without a row too
    for (int i = wave; i <= rq.count && i < limit; i += waves) {
        const Ahead own = next;
        const int x = own.x;
        const bool in = x >= 0 && x < a.V;
        const float xp = in ? __uint_as_float((uint32_t)target_row(a, b, i)[x] << 16) : kNegInf;
        const float xq = in && a.draft ? __uint_as_float((uint32_t)draft_row(a, b, i)[x] << 16) : kNegInf;
        next = request(i + waves);
        const bool draft = a.draft && !rq.greedy;
        const VerifyStat p = row_stat(a, b, i, own.own_p, rq.k, lane);
        VerifyStat q{0.0f, 0, 0.0};
        if (draft && i < rq.count) q = row_stat(a, b, a.n + 1 + i, own.own_q, rq.k, lane);
        double px = 0.0, qx = 1.0;
        if (in) px = rq.greedy ? (p.m != kNegInf && x == p.at ? 1.0 : 0.0) : probability(xp, p, rq.k);
        if (draft) qx = in ? probability(xq, q, rq.k) : 0.0;
        if (lane == 0) {
            rows.p[i] = p;
            rows.q[i] = q;
            rows.keep[i] = (double)own.u * qx < px;
        }
    }
    __syncthreads();
    const int end = min(rq.count, limit);
    VerifyDecision d{};
    const uint64_t refused = __ballot(lane < end && !rows.keep[min(lane, end)]);     // at most 64 drafted tokens
    d.accepted = refused ? __builtin_ctzll(refused) : end;
    d.rejected = d.accepted < end;
    d.done = d.rejected || rq.count < limit;
    if (d.done) {
        d.p = rows.p[d.accepted];
        d.q = rows.q[d.accepted];
    }
    return d;
}

__global__ __launch_bounds__(kPickThreads) void k_verify_decide(VerifyArgs a) {
    __shared__ Rows rows;
    const int b = blockIdx.x;
    Request rq;
    const VerifyDecision d = decide(a, b, a.first_rows, rows, rq);
    if (threadIdx.x == 0) a.decisions[b] = d;
}

// One workgroup a (sequence, C chunks).  Every workgroup of a sequence finds its decision by
// itself, where the first rows have not: cheaper than a kernel for it.
template <int C>
__global__ __launch_bounds__(kWeighThreads) void k_verify_weigh(VerifyArgs a) {
    __shared__ Rows rows;
    __shared__ double part[C][kWeighThreads / 64];
    const int b = blockIdx.y, c = blockIdx.x * C, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Request rq;
    VerifyDecision d;
    if (a.first_rows && a.decisions[b].done) {
        d = a.decisions[b];
        rq = load_request(a, b);
    } else {
        d = decide(a, b, a.n + 1, rows, rq);
        if (c == 0 && threadIdx.x == 0) a.final_decisions[b] = d;
    }
    if (rq.greedy || !d.rejected || !(d.p.z > 0.0)) return;      // the rows' statistics suffice
    const Choice ch = choice_of(a, b, d, rq.k);
#pragma unroll
    for (int k = 0; k < C; ++k) {
        double w[8], s = 0.0;
        ch.weights((c + k) * kChunkVecs + threadIdx.x, a.V, true, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) s += w[e];
        s = wave_sum(s);
        if (lane == 0) part[k][wave] = s;
    }
    __syncthreads();
    if (threadIdx.x < C && c + threadIdx.x < a.chunks) {
        double t = 0.0;
        for (int i = 0; i < kWeighThreads / 64; ++i) t += part[threadIdx.x][i];
        a.sums[(int64_t)b * a.chunks + c + threadIdx.x] = t;
    }
}

// One workgroup a sequence.  Its chunk is found by every wave for itself, 64 chunks at a time;
// the token by the running sum of its 4096, eight a thread of half the waves.
__global__ __launch_bounds__(kPickThreads) void k_verify_pick(VerifyArgs a) {
    __shared__ Rows rows;
    __shared__ double part[kPickWaves];
    __shared__ int chosen, last_of[kPickWaves];
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    Request rq;
    const float u = a.uniform[b * (a.n + 1) + a.n];
    const bool weighed = a.draft;
    const double *sums = a.sums + (int64_t)b * a.chunks;
    const double early = weighed && lane < a.chunks ? sums[lane] : 0.0;      // with the decision, not after it
    VerifyDecision d;
    if (a.draft || a.first_rows) rq = load_request(a, b);
    if (a.first_rows && a.decisions[b].done) d = a.decisions[b];
    else if (a.draft) d = a.final_decisions[b];
    else d = decide(a, b, a.n + 1, rows, rq);
    if (tid == 0) a.accepted[b] = d.accepted;
    if (tid <= a.n && tid != d.accepted) a.tokens[b * (a.n + 1) + tid] = tid < d.accepted ? a.drafted[b * a.n + tid] : -1;
    int *out = a.tokens + b * (a.n + 1) + d.accepted;
    if (rq.greedy || !(d.p.z > 0.0)) {
        if (tid == 0) *out = rq.greedy && d.p.m != kNegInf ? d.p.at : -1;
        return;
    }
    // A chunk's mass: what was weighed; or the target's from its statistics, relative to the row's
    // maximum, less the drafted token's where it was refused (in the chunk's own scale that
    // weight is a term of the sum, bit for bit); without any mass left, the target's alone.
    const VerifyStat *stats = row_stats(a, b, d.accepted);
    bool rest = d.rejected;
    const Choice ch = choice_of(a, b, d, rq.k);
    float gone = kNegInf;
    int gone_chunk = -1;
    if (rest && !weighed && ch.x >= 0 && ch.x < a.V) {
        gone = __uint_as_float((uint32_t)target_row(a, b, d.accepted)[ch.x] << 16);
        gone_chunk = (ch.x + ch.row.off) / kVerifyChunk;
    }
    auto mass = [&](int c) {
        if (c >= a.chunks) return 0.0;
        if (rest && weighed) return c == lane ? early : sums[c];
        const VerifyStat st = stats[c];
        double z = st.z;
        if (rest && c == gone_chunk && st.m != kNegInf) z = fmax(z - Scale(rq.k, st.m)(gone), 0.0);
        const double f = rescale(rq.k, st.m, d.p.m);
        return f < kLeast ? 0.0 : z * f;
    };
    // the first chunk whose running sum passes r = u total, and the last with any mass
    int chunk = -1, any = 0;
    double at = 0.0, r = 0.0;
    auto find = [&](int c, double own, double upto) {
        const uint64_t over = __ballot(own > 0.0 && upto > r), some = __ballot(own > 0.0);
        if (some) any = c + 63 - __builtin_clzll(some);
        if (!over) return;
        const int l = __builtin_ctzll(over);
        chunk = c + l;
        at = from_lane(upto, l) - from_lane(own, l);
    };
    for (int again = 0; again < 2; ++again) {
        double own = mass(lane), upto = lanes_upto(own), total = from_lane(upto, 63);
        for (int c = 64; c < a.chunks; c += 64) total += wave_sum(mass(c + lane));
        if (rest && !(total > 0.0)) {                        // nothing is left of the difference
            rest = false;
            continue;
        }
        r = (double)u * total;
        find(0, own, upto);
        double run = from_lane(upto, 63);
        for (int c = 64; c < a.chunks && chunk < 0; c += 64) {
            own = mass(c + lane);
            upto = run + lanes_upto(own);
            find(c, own, upto);
            run = from_lane(upto, 63);
        }
        break;
    }
    const bool past = chunk < 0;                            // rounding left none: the last token of all
    if (past) chunk = any;
    double w[8] = {}, own = 0.0;
    const int v = chunk * kChunkVecs + tid, j0 = 8 * v - ch.row.off;
    if (tid < kChunkVecs) ch.weights(v, a.V, rest, w);
    int end = -1;                                           // this thread's last token of any weight
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        own += w[e];
        if (w[e] > 0.0) end = j0 + e;
    }
    const double upto = lanes_upto(own);
    const int wave_end = -wave_min(-end);
    if (lane == 63) part[wave] = upto;
    if (lane == 0) last_of[wave] = wave_end;
    if (tid == 0) chosen = 0x7FFFFFFF;
    __syncthreads();
    const double need = rest && weighed ? r - at : (r - at) / d.p.z;     // weights are relative to the sum
    const double waves = lanes_upto(lane < kPickWaves ? part[lane] : 0.0);
    double sum = (wave ? from_lane(waves, wave - 1) : 0.0) + (upto - own);
    int hit = 0x7FFFFFFF;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        sum += w[e];
        if (hit == 0x7FFFFFFF && w[e] > 0.0 && !past && sum > need) hit = j0 + e;
    }
    const uint64_t hits = __ballot(hit != 0x7FFFFFFF);      // the lowest lane's token is the wave's first
    if (hits && lane == __builtin_ctzll(hits)) atomicMin(&chosen, hit);
    __syncthreads();
    if (tid == 0) {
        int next = chosen;
        if (next == 0x7FFFFFFF) {
            next = -1;
            for (int i = 0; i < kPickWaves; ++i) next = last_of[i] >= 0 ? last_of[i] : next;
        }
        *out = next;
    }
}

}  // namespace

// Few logits go to many small workgroups, many to larger ones, by the call's logits (small / large
// form, graph replays when the rule was chosen): 2.4 million 12.3 / 13.4 us, with draft logits 3.9 million 18.2 / 20.5, 9.4
// 24.1 / 26.0, 26.7 37.5 / 40.2, 37.7 48.0 / 45.8, 65.9 70.3 / 65.1.  Chunks of 8192 and 2048 tokens
// took 14.0 and 13.6 us for the first, 22.2 and 17.6 for the second.
hipError_t launch_verify(VerifyArgs a, int n_seq, bool many, hipStream_t st) {
    auto stats = [&](int row0, int row1) {
        a.row0 = row0;
        a.row1 = row1;
        const int rows = row1 - row0 + (a.draft ? (row1 < a.n ? row1 : a.n) - row0 : 0);
        const dim3 grid((unsigned)(a.chunks * rows), (unsigned)n_seq);
        if (many) hipLaunchKernelGGL(k_verify_stats<128>, grid, dim3(128), 0, st, a);
        else hipLaunchKernelGGL(k_verify_stats<256>, grid, dim3(256), 0, st, a);
        return hipGetLastError();
    };
    hipError_t e;
    if (a.first_rows) {
        if ((e = stats(0, a.first_rows)) != hipSuccess) return e;
        hipLaunchKernelGGL(k_verify_decide, dim3((unsigned)n_seq), dim3(kPickThreads), 0, st, a);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if ((e = stats(a.first_rows, a.n + 1)) != hipSuccess) return e;
    if (a.draft) {
        if (many) hipLaunchKernelGGL(k_verify_weigh<2>, dim3((unsigned)(a.chunks + 1) / 2, (unsigned)n_seq), dim3(kWeighThreads), 0, st, a);
        else hipLaunchKernelGGL(k_verify_weigh<1>, dim3((unsigned)a.chunks, (unsigned)n_seq), dim3(kWeighThreads), 0, st, a);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    hipLaunchKernelGGL(k_verify_pick, dim3((unsigned)n_seq), dim3(kPickThreads), 0, st, a);
    return hipGetLastError();
}

}  // namespace qlin
