// The decision on drafted tokens (qlin_verify_draft in include/qlin_target.h).
//
// The plain kernel: one workgroup a sequence, which walks the drafted tokens in order.
// Weights e^((x - max) / T) and their sums are 64-bit: a running sum over a vocabulary
// has a boundary every 1e-5 of it or closer, and 32-bit weights (off by 6e-8 each)
// would move a boundary past the uniform number in a few of a thousand choices.
#include "device_common.h"
#include "target_internal.h"

namespace qlin {

namespace {

constexpr int kThreads1 = 1024, kWaves1 = kThreads1 / 64;
constexpr float kNegInf = -__builtin_huge_valf();

__device__ inline float logit(const uint16_t *row, int i) {
    const float x = __uint_as_float((uint32_t)row[i] << 16);
    return x == x ? x : kNegInf;
}

// Weight of a logit in a row of maximum m: 1 at the maximum, 0 where masked.
__device__ inline double weight(float x, float m, double inv_t) {
    const float d = x - m;                  // -infinity where x is, or where only m is infinite
    return x == m ? (x == kNegInf ? 0.0 : 1.0) : d == kNegInf ? 0.0 : exp(((double)x - (double)m) * inv_t);
}

__device__ inline double block_sum(double v, double *buf) {
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
    __syncthreads();
    double t = 0.0;
    for (int i = 0; i < kWaves1; ++i) t += buf[i];
    return t;
}

struct Row { float m; int at; double z; };

__device__ Row row_stats(const uint16_t *row, int V, double inv_t, double *buf, int *ibuf) {
    float m = kNegInf;
    int at = 0x7FFFFFFF;
    for (int i = threadIdx.x; i < V; i += kThreads1) {
        const float x = logit(row, i);
        if (x > m) { m = x; at = i; }
    }
    for (int o = 32; o; o >>= 1) {
        const float m2 = __shfl_xor(m, o);
        const int a2 = __shfl_xor(at, o);
        if (m2 > m || (m2 == m && a2 < at)) { m = m2; at = a2; }
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) { buf[threadIdx.x >> 6] = m; ibuf[threadIdx.x >> 6] = at; }
    __syncthreads();
    for (int i = 0; i < kWaves1; ++i) {
        const float m2 = (float)buf[i];
        if (m2 > m || (m2 == m && ibuf[i] < at)) { m = m2; at = ibuf[i]; }
    }
    double z = 0.0;
    for (int i = threadIdx.x; i < V; i += kThreads1) z += weight(logit(row, i), m, inv_t);
    return Row{m, at, block_sum(z, buf)};
}

__global__ __launch_bounds__(kThreads1) void k_verify_plain(VerifyArgs a) {
    __shared__ double buf[kWaves1], part[kThreads1];
    __shared__ int ibuf[kWaves1], found[2];
    const int b = blockIdx.x, V = a.V, n = a.n;
    const int count = a.count ? min(max(a.count[b], 0), n) : n;
    const float T = a.temperature ? a.temperature[b] : 1.0f;
    const bool greedy = !(T > 0.0f);
    const double inv_t = greedy ? 1.0 : 1.0 / (double)T;
    const uint16_t *tb = a.target + (int64_t)b * (n + 1) * a.target_stride;
    const uint16_t *db = a.draft ? a.draft + (int64_t)b * n * a.draft_stride : nullptr;
    int i = 0;
    Row p, q;
    bool rejected = false;
    for (;; ++i) {
        p = row_stats(tb + i * a.target_stride, V, inv_t, buf, ibuf);
        if (i == count) break;
        const int x = a.drafted[b * n + i];
        const bool in = x >= 0 && x < V;
        double px = 0.0, qx = 1.0;
        if (in && p.z > 0.0) px = greedy ? (x == p.at ? 1.0 : 0.0) : weight(logit(tb + i * a.target_stride, x), p.m, inv_t) / p.z;
        if (db && !greedy) {
            q = row_stats(db + i * a.draft_stride, V, inv_t, buf, ibuf);
            qx = in && q.z > 0.0 ? weight(logit(db + i * a.draft_stride, x), q.m, inv_t) / q.z : 0.0;
        }
        if (!((double)a.uniform[b * (n + 1) + i] * qx < px)) { rejected = true; break; }
    }
    const uint16_t *tr = tb + i * a.target_stride, *dr = db && !greedy ? db + i * a.draft_stride : nullptr;
    const int x = rejected ? a.drafted[b * n + i] : -1;
    int next = -1;
    if (greedy) {
        next = p.z > 0.0 ? p.at : -1;
    } else if (p.z > 0.0) {
        const int chunk = (V + kThreads1 - 1) / kThreads1;
        const int lo = min(V, (int)threadIdx.x * chunk), hi = min(V, lo + chunk);
        for (int pass = rejected ? 0 : 1; pass < 2; ++pass) {
            auto w = [&](int j) {
                const double pj = weight(logit(tr, j), p.m, inv_t) / p.z;
                if (pass == 1) return pj;
                const double qj = dr ? (q.z > 0.0 ? weight(logit(dr, j), q.m, inv_t) / q.z : 0.0) : (j == x ? 1.0 : 0.0);
                return pj > qj ? pj - qj : 0.0;
            };
            double s = 0.0;
            for (int j = lo; j < hi; ++j) s += w(j);
            __syncthreads();
            part[threadIdx.x] = s;
            if (threadIdx.x == 0) { found[0] = 0x7FFFFFFF; found[1] = -1; }
            __syncthreads();
            double before = 0.0, total = 0.0;
            for (int t = 0; t < kThreads1; ++t) {
                if (t == (int)threadIdx.x) before = total;
                total += part[t];
            }
            if (!(total > 0.0)) continue;
            const double r = (double)a.uniform[b * (n + 1) + n] * total;
            for (int j = lo; j < hi; ++j) {
                const double wj = w(j);
                before += wj;
                if (wj > 0.0) atomicMax(&found[1], j);
                if (wj > 0.0 && before > r) { atomicMin(&found[0], j); break; }
            }
            __syncthreads();
            next = found[0] != 0x7FFFFFFF ? found[0] : found[1];
            break;
        }
    }
    if (threadIdx.x == 0) a.accepted[b] = i;
    for (int j = threadIdx.x; j <= n; j += kThreads1)
        a.tokens[b * (n + 1) + j] = j < i ? a.drafted[b * n + j] : j == i ? next : -1;
}

}  // namespace

hipError_t launch_verify(const VerifyArgs &a, int n_seq, hipStream_t st) {
    hipLaunchKernelGGL(k_verify_plain, dim3(n_seq), dim3(kThreads1), 0, st, a);
    return hipGetLastError();
}

}  // namespace qlin
