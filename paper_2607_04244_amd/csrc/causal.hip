// Causal attention with grouped heads over the key/value cache
// (qlin_causal_attention in include/qlin_target.h).
//
// The plain kernel: one wave a (row, query head), 64 keys at a time, one lane a key
// for the scores, two dimensions a lane for the weighted sum, with the running maximum
// and sum of the softmax in fp32.
#include "target_common.h"

namespace qlin {

namespace {

constexpr float kNegInf = -__builtin_huge_valf();

__device__ inline float wave_max(float v) {
    for (int o = 32; o; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
    return v;
}
__device__ inline float wave_sum(float v) {
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

__global__ __launch_bounds__(64) void k_causal_row(CausalArgs a) {
    const int m = blockIdx.x, h = blockIdx.y, lane = threadIdx.x;
    const int b = find_seq(a.b, m, lane);
    if (b >= a.b.n_seq) return;
    const Seq s = load_seq(a.b, b);
    if (m < s.row0 || m >= s.row0 + s.rows) return;
    const int keys = s.L > 0 ? s.p0 + (m - s.row0) + 1 : 0;     // visible: j < keys
    const uint16_t *kb = a.k + s.slot0 * a.b.tok + (int64_t)(h / a.G) * a.b.head;
    const uint16_t *vb = a.v + s.slot0 * a.b.tok + (int64_t)(h / a.G) * a.b.head;
    const uint16_t *qr = a.q + (int64_t)m * a.q_stride + h * kHeadDim;
    float mx = kNegInf, l = 0.0f, o0 = 0.0f, o1 = 0.0f;
    for (int j0 = 0; j0 < keys; j0 += 64) {
        const int j = j0 + lane;
        float sc = kNegInf;
        if (j < keys) {
            const uint4 *kr = (const uint4 *)(kb + (int64_t)j * a.b.tok);
            const uint4 *q4 = (const uint4 *)qr;
            sc = 0.0f;
            for (int u = 0; u < kHeadDim / 8; ++u) {
                const uint4 x = kr[u], y = q4[u];
                sc = dot2(x.x, y.x, sc);
                sc = dot2(x.y, y.y, sc);
                sc = dot2(x.z, y.z, sc);
                sc = dot2(x.w, y.w, sc);
            }
        }
        const float mn = fmaxf(mx, wave_max(sc)), muc = (mn == kNegInf ? 0.0f : mn) * a.c;
        const float alpha = exp2f(fmaf(mx, a.c, -muc));
        const float p = bf16_lo_to_f32(cvt_bf16(exp2f(fmaf(sc, a.c, -muc))));
        l = l * alpha + p;
        o0 *= alpha;
        o1 *= alpha;
        mx = mn;
        const int n = min(64, keys - j0);
        for (int i = 0; i < n; ++i) {
            const float w = __shfl(p, i);
            const uint32_t v2 = *(const uint32_t *)(vb + (int64_t)(j0 + i) * a.b.tok + 2 * lane);
            o0 = fmaf(w, bf16_lo_to_f32(v2), o0);
            o1 = fmaf(w, bf16_hi_to_f32(v2), o1);
        }
    }
    l = wave_sum(l);
    *(uint32_t *)(a.out + (int64_t)m * a.out_stride + h * kHeadDim + 2 * lane) = keys > 0 ? cvt_pk_bf16(o0 / l, o1 / l) : 0u;
}

}  // namespace

hipError_t launch_causal(const CausalArgs &a, hipStream_t st) {
    if (a.b.rows == 0) return hipSuccess;
    hipLaunchKernelGGL(k_causal_row, dim3(a.b.rows, a.Hq), dim3(64), 0, st, a);
    return hipGetLastError();
}

}  // namespace qlin
