// The decision on drafted tokens (qlin_verify_draft in include/qlin_target.h).
//
// Three kernels, bound by the bytes of the logits and the 64-bit exponentials of all of them:
//   k_verify_stats   (row, chunk of 8192 tokens): maximum, its lowest index, and the sum of
//       the weights e^((x - maximum) / T), for every row that a decision can need.
//   k_verify_weigh   (sequence, chunk): the accepted prefix from the rows' statistics, and, if a
//       token was refused, the chunk's sum of max(P - Q, 0).
//   k_verify_pick    (sequence): the chunk, then the token, that the running sum passes the
//       uniform number in.
// Each later kernel reads one or two rows a sequence.
//
// Weights and sums are 64-bit: a running sum over a vocabulary of 10^5 has a boundary every
// 10^-5 of it or closer, and 32-bit weights (off by up to 6e-8 each) would put a few of a
// thousand choices on the wrong side of one.  At an error of 5e-11 it is one of 10^5.
// 64-bit products run at the rate of 32-bit ones here, and 32-bit exponentials at a half of
// it, so the accuracy costs about twice the time of 32-bit weights.
#include "device_common.h"
#include "target_internal.h"

namespace qlin {

namespace {

constexpr float kNegInf = -__builtin_huge_valf(), kPosInf = __builtin_huge_valf();
constexpr int kStatsThreads = 256, kStatsVecs = kVerifyChunk / (8 * kStatsThreads);
constexpr int kPickThreads = kVerifyChunk / 8, kPickWaves = kPickThreads / 64;

// 2^t, t >= -1100, relative error 4.7e-11: (2^f - 1) / f on [-1/2, 1/2] as the polynomial of
// degree 6 whose largest weighted error is smallest; 2^0 is 1 exactly.
__device__ inline double pow2(double t) {
    const double n = rint(t), f = t - n;
    double p = 1.5196156371520414e-05;
    p = __builtin_fma(p, f, 0.00015466756333052078);
    p = __builtin_fma(p, f, 0.0013333935056283428);
    p = __builtin_fma(p, f, 0.009618038132000921);
    p = __builtin_fma(p, f, 0.05550410365990573);
    p = __builtin_fma(p, f, 0.2402265106656167);
    p = __builtin_fma(p, f, 0.6931471807045319);
    p = __builtin_fma(p, f, 1.0);
    return __builtin_amdgcn_ldexp(p, (int)n);
}

// Weights of a row: 2^(k x - k m), k = log2(e) / T, m its maximum.  -infinity and NaN give 0
// (2^-1100 is below the smallest number), an infinite maximum 1 to its equals alone.
struct Scale {
    double k, km;
    float m;
    __device__ inline Scale(double k_, float m_) : k(k_), km(k_ * (double)m_), m(m_) {}
    __device__ inline double operator()(float x) const {
        if (m == kPosInf) return x == kPosInf ? 1.0 : 0.0;
        return pow2(fmax(__builtin_fma((double)x, k, -km), -1100.0));
    }
};
// The factor from weights relative to m to weights relative to the larger M.
__device__ inline double rescale(double k, float m, float M) {
    return m == M ? 1.0 : m == kNegInf || M == kPosInf ? 0.0 : pow2(fmax(((double)m - (double)M) * k, -1100.0));
}

__device__ inline double wave_sum(double v) {
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// What a sequence asks for.
struct Request {
    int count;
    bool greedy;
    double k;               // log2(e) / T
};
__device__ inline Request load_request(const VerifyArgs &a, int b) {
    Request r;
    r.count = a.count ? min(max(a.count[b], 0), a.n) : a.n;
    const float T = a.temperature ? a.temperature[b] : 1.0f;
    r.greedy = !(T > 0.0f);
    r.k = r.greedy ? 1.0 : 1.4426950408889634 / (double)T;
    return r;
}

// A row of logits in vectors of 8: its first logit is element `off` of the first vector, which
// is 16-byte aligned.
struct Row {
    const uint16_t *base;   // of the first vector
    int off;
    __device__ inline Row(const uint16_t *p) : base((const uint16_t *)((uintptr_t)p & ~(uintptr_t)15)), off((int)((uintptr_t)p & 15) / 2) {}
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

// The rows of sequence b: target rows 0 .. n, then draft rows 0 .. n - 1.
__device__ inline const uint16_t *target_row(const VerifyArgs &a, int b, int i) { return a.target + ((int64_t)b * (a.n + 1) + i) * a.target_stride; }
__device__ inline const uint16_t *draft_row(const VerifyArgs &a, int b, int i) { return a.draft + ((int64_t)b * a.n + i) * a.draft_stride; }

// One workgroup a (row, chunk); each thread holds its 32 logits in registers between the
// maximum and the weights.
__global__ __launch_bounds__(kStatsThreads) void k_verify_stats(VerifyArgs a) {
    __shared__ VerifyStat part[kStatsThreads / 64];
    const int b = blockIdx.y, which = blockIdx.x / a.chunks, c = blockIdx.x - which * a.chunks;
    const bool is_draft = which > a.n;
    const int i = is_draft ? which - a.n - 1 : which;
    const Request rq = load_request(a, b);
    if (is_draft ? i >= rq.count || rq.greedy : i > rq.count) return;
    const Row row(is_draft ? draft_row(a, b, i) : target_row(a, b, i));
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float x[kStatsVecs][8];
    const int v0 = c * (kVerifyChunk / 8) + threadIdx.x;
#pragma unroll
    for (int k = 0; k < kStatsVecs; ++k) load_logits(row, v0 + k * kStatsThreads, a.V, x[k]);
    float m = kNegInf;
#pragma unroll
    for (int k = 0; k < kStatsVecs; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) m = fmaxf(m, x[k][e]);           // ignores NaN
#pragma unroll
    for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    VerifyStat st{m, 0x7FFFFFFF, 0.0};
    if (rq.greedy) {
        int at = 0x7FFFFFFF;
#pragma unroll
        for (int k = kStatsVecs - 1; k >= 0; --k)
#pragma unroll
            for (int e = 7; e >= 0; --e)
                if (x[k][e] == m) at = 8 * (v0 + k * kStatsThreads) - row.off + e;
#pragma unroll
        for (int o = 32; o; o >>= 1) at = min(at, __shfl_xor(at, o));
        st.at = at;
    } else if (m != kNegInf) {
        const Scale w(rq.k, m);
        double s = 0.0;
#pragma unroll
        for (int k = 0; k < kStatsVecs; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) s += w(x[k][e]);
        st.z = wave_sum(s);
    }
    if (lane == 0) part[wave] = st;
    __syncthreads();
    if (threadIdx.x == 0) {
        float M = kNegInf;
        for (int k = 0; k < kStatsThreads / 64; ++k) M = fmaxf(M, part[k].m);
        VerifyStat all{M, 0x7FFFFFFF, 0.0};
        for (int k = 0; k < kStatsThreads / 64; ++k) {
            if (part[k].m == M) all.at = min(all.at, part[k].at);
            all.z += part[k].z * rescale(rq.k, part[k].m, M);
        }
        a.stats[((int64_t)b * a.all_rows + which) * a.chunks + c] = all;
    }
}

// A row's statistics from its chunks', by a wave.
__device__ inline VerifyStat row_stat(const VerifyArgs &a, int b, int which, double k, int lane) {
    const VerifyStat *p = a.stats + ((int64_t)b * a.all_rows + which) * a.chunks;
    VerifyStat st{kNegInf, 0x7FFFFFFF, 0.0};
    for (int c = lane; c < a.chunks; c += 64) {
        const VerifyStat e = p[c];
        const float M = fmaxf(st.m, e.m);
        st.z = st.z * rescale(k, st.m, M) + e.z * rescale(k, e.m, M);
        st.at = e.m > st.m ? e.at : e.m == st.m ? min(st.at, e.at) : st.at;
        st.m = M;
    }
    float M = st.m;
#pragma unroll
    for (int o = 32; o; o >>= 1) M = fmaxf(M, __shfl_xor(M, o));
    st.z = wave_sum(st.z * rescale(k, st.m, M));
    int at = st.m == M ? st.at : 0x7FFFFFFF;
#pragma unroll
    for (int o = 32; o; o >>= 1) at = min(at, __shfl_xor(at, o));
    return VerifyStat{M, at, st.z};
}

// The probability of token x in a row with these statistics.
__device__ inline double probability(const uint16_t *row, int x, const VerifyStat &st, double k) {
    return st.z > 0.0 ? Scale(k, st.m)(__uint_as_float((uint32_t)row[x] << 16)) / st.z : 0.0;
}

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
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = p(l[e]) * inv_p;
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
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = fmax(w[e] - s(d[e]) * inv_q, 0.0);
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

// One workgroup a (sequence, chunk).  Every workgroup of a sequence finds its decision by
// itself, a wave a drafted token: cheaper than a kernel for it.
__global__ __launch_bounds__(kPickThreads) void k_verify_weigh(VerifyArgs a) {
    __shared__ VerifyStat ps[kVerifyMaxDraft + 1], qs[kVerifyMaxDraft + 1];
    __shared__ int keeps[kVerifyMaxDraft + 1];
    __shared__ double part[kPickWaves];
    const int b = blockIdx.y, c = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Request rq = load_request(a, b);
    const bool draft = a.draft && !rq.greedy;
    for (int i = wave; i <= rq.count; i += kPickWaves) {
        const VerifyStat p = row_stat(a, b, i, rq.k, lane);
        VerifyStat q{0.0f, 0, 0.0};
        bool keep = false;
        if (i < rq.count) {
            const int x = a.drafted[b * a.n + i];
            const bool in = x >= 0 && x < a.V;
            double px = 0.0, qx = 1.0;
            if (in) px = rq.greedy ? (p.m != kNegInf && x == p.at ? 1.0 : 0.0) : probability(target_row(a, b, i), x, p, rq.k);
            if (draft) {
                q = row_stat(a, b, a.n + 1 + i, rq.k, lane);
                qx = in ? probability(draft_row(a, b, i), x, q, rq.k) : 0.0;
            }
            keep = (double)a.uniform[b * (a.n + 1) + i] * qx < px;
        }
        if (lane == 0) {
            ps[i] = p;
            qs[i] = q;
            keeps[i] = keep;
        }
    }
    __syncthreads();
    VerifyDecision d;
    d.accepted = 0;
    while (d.accepted < rq.count && keeps[d.accepted]) ++d.accepted;
    d.rejected = d.accepted < rq.count;
    d.p = ps[d.accepted];
    d.q = qs[d.accepted];
    if (c == 0 && threadIdx.x == 0) a.decisions[b] = d;
    if (rq.greedy || !d.rejected || !(d.p.z > 0.0)) return;      // the rows' statistics suffice
    double w[8], s = 0.0;
    choice_of(a, b, d, rq.k).weights(c * (kVerifyChunk / 8) + threadIdx.x, a.V, true, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) s += w[e];
    s = wave_sum(s);
    if (lane == 0) part[wave] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        double t = 0.0;
        for (int i = 0; i < kPickWaves; ++i) t += part[i];
        a.sums[(int64_t)b * a.chunks + c] = t;
    }
}

// Sum over the threads before this one, and over all, in a fixed order.
__device__ inline double before_of(double own, double *buf, double *total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    double s = own;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const double v = __shfl_up(s, o);
        s += lane >= o ? v : 0.0;
    }
    __syncthreads();
    if (lane == 63) buf[wave] = s;
    __syncthreads();
    double t = 0.0, at = 0.0;
    for (int i = 0; i < kPickWaves; ++i) {
        if (i == wave) at = t;
        t += buf[i];
    }
    *total = t;
    return at + (s - own);
}

__global__ __launch_bounds__(kPickThreads) void k_verify_pick(VerifyArgs a) {
    __shared__ double buf[kPickWaves], base;
    __shared__ int first, last;
    const int b = blockIdx.x, tid = threadIdx.x;
    const Request rq = load_request(a, b);
    const VerifyDecision d = a.decisions[b];
    int next = -1;
    if (rq.greedy) {
        next = d.p.m != kNegInf ? d.p.at : -1;
    } else if (d.p.z > 0.0) {
        // a chunk's sum: what was weighed, or if nothing is left of the difference, the target's
        const double *sums = a.sums + (int64_t)b * a.chunks;
        const VerifyStat *stats = a.stats + ((int64_t)b * a.all_rows + d.accepted) * a.chunks;
        const int per = (a.chunks + kPickThreads - 1) / kPickThreads, c0 = min(tid * per, a.chunks), c1 = min(c0 + per, a.chunks);
        bool rest = d.rejected;
        auto mass = [&](int c) { return rest ? sums[c] : stats[c].z * rescale(rq.k, stats[c].m, d.p.m); };
        double own = 0.0, total, before;
        for (int c = c0; c < c1; ++c) own += mass(c);
        before = before_of(own, buf, &total);
        if (rest && !(total > 0.0)) {                       // the same in every thread
            rest = false;
            own = 0.0;
            for (int c = c0; c < c1; ++c) own += mass(c);
            before = before_of(own, buf, &total);
        }
        const double r = (double)a.uniform[b * (a.n + 1) + a.n] * total;
        if (tid == 0) {
            first = 0x7FFFFFFF;
            last = -1;
        }
        __syncthreads();
        double run = before;
        int mine = -1;
        double mine_base = 0.0;
        for (int c = c0; c < c1; ++c) {
            const double s = mass(c);
            if (s > 0.0) {
                atomicMax(&last, c);
                if (mine < 0 && run + s > r) {
                    mine = c;
                    mine_base = run;
                    atomicMin(&first, c);
                }
            }
            run += s;
        }
        __syncthreads();
        const int chunk = first != 0x7FFFFFFF ? first : last;
        const bool past = first == 0x7FFFFFFF;              // rounding left none: the last token of all
        if (!past && mine == chunk) base = mine_base;
        __syncthreads();
        const double at = past ? 0.0 : base;
        if (tid == 0) {
            first = 0x7FFFFFFF;
            last = -1;
        }
        double w[8];
        const Choice ch = choice_of(a, b, d, rq.k);
        const int v = chunk * (kVerifyChunk / 8) + tid;
        ch.weights(v, a.V, rest, w);
        own = 0.0;
#pragma unroll
        for (int e = 0; e < 8; ++e) own += w[e];
        run = before_of(own, buf, &total);
        // a chunk's mass from the statistics is relative to the row's maximum, weights to its sum
        const double need = rest ? r - at : (r - at) / d.p.z;
        int hit = 0x7FFFFFFF, end = -1;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            run += w[e];
            const int j = 8 * v - ch.row.off + e;
            if (w[e] > 0.0) {
                end = j;
                if (hit == 0x7FFFFFFF && !past && run > need) hit = j;
            }
        }
        if (hit != 0x7FFFFFFF) atomicMin(&first, hit);
        if (end >= 0) atomicMax(&last, end);
        __syncthreads();
        next = first != 0x7FFFFFFF ? first : last;
    }
    if (tid == 0) a.accepted[b] = d.accepted;
    if (tid <= a.n) a.tokens[b * (a.n + 1) + tid] = tid < d.accepted ? a.drafted[b * a.n + tid] : tid == d.accepted ? next : -1;
}

}  // namespace

hipError_t launch_verify(const VerifyArgs &a, int n_seq, hipStream_t st) {
    hipLaunchKernelGGL(k_verify_stats, dim3((unsigned)(a.chunks * a.all_rows), (unsigned)n_seq), dim3(kStatsThreads), 0, st, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_verify_weigh, dim3((unsigned)a.chunks, (unsigned)n_seq), dim3(kPickThreads), 0, st, a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_verify_pick, dim3((unsigned)n_seq), dim3(kPickThreads), 0, st, a);
    return hipGetLastError();
}

}  // namespace qlin
