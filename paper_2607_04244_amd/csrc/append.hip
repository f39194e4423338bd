// Norms and rotation of queries and keys with the append to the key/value cache
// (qlin_norm_rope_append in include/qlin_target.h).
//
// Bound by memory: every head row of 256 bytes is read and written once.  A group of
// 16 lanes holds one head row, 16 bytes a lane; a workgroup takes R tokens and as
// many of their q, k and v heads at a time as it has groups.  The R x half angles of
// its tokens are computed once, by its first threads, into LDS: p * inv_freq in turns
// is reduced in 64 bits, where 2^28 positions leave 30 bits of a turn, and only the
// rest of at most half a turn goes through 32-bit sine and cosine.  One token a workgroup for
// few tokens (a single one takes 3.5 us, of which a launch is 1.6), four for many: 512 rows
// of 32 / 8 heads 7.2 against 7.7 us, 768 rows 10.2 against 8.3, 2048 rows 21.3 against 13.3
// (in the last-level cache 5.7 / 7.6, 7.8 / 7.8, 16.6 / 11.1).  Two and eight tokens: 54.8
// and 51.2 us against 49.8 of four (8192 tokens, without the hint below).
#include "target_common.h"

#include <type_traits>

namespace qlin {

namespace {

constexpr int kGroupLanes = 16;          // lanes of a head row
constexpr int kAppendThreads = 1024;
constexpr int kManyRows = 640;           // R = 4 from here on

// Sum over the 16 lanes of a DPP row, in every lane.
__device__ inline float row_sum(float v) {
    auto ror = [](float x, auto n) {
        return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x120 + decltype(n)::value, 0xF, 0xF, false));
    };
    v += ror(v, std::integral_constant<int, 8>{});
    v += ror(v, std::integral_constant<int, 4>{});
    v += ror(v, std::integral_constant<int, 2>{});
    v += ror(v, std::integral_constant<int, 1>{});
    return v;
}

// Many tokens stream through: with the non-temporal hint both ways 8192 tokens from and to
// memory that no cache holds take 43.0 us against 49.8, 1500 tokens 12.3 against 14.7 (with
// it on the loads alone 47.7 and 13.1; where the last-level cache holds all, 41.6 against
// 39.3).  Few tokens stay in the caches for the attention behind.
template <int R>
__device__ inline uint4 load_row(const uint16_t *p) {
    if constexpr (R > 1) return __builtin_bit_cast(uint4, __builtin_nontemporal_load((const v4u *)p));
    else return *(const uint4 *)p;
}
template <int R>
__device__ inline void store_row(uint16_t *p, const uint4 &y) {
    if constexpr (R > 1) __builtin_nontemporal_store(__builtin_bit_cast(v4u, y), (v4u *)p);
    else *(uint4 *)p = y;
}

template <int R>
__global__ __launch_bounds__(kAppendThreads) void k_norm_rope_append(AppendArgs a) {
    __shared__ float2 cs[R][kHeadDim / 2];   // (cos, sin) of each token's angles
    __shared__ int64_t slot[R];              // cache slot of each token, -1: not stored
    __shared__ int live[R];                  // a new token of some sequence
    const int lane = threadIdx.x & 63, l = threadIdx.x & 15;
    const int groups = blockDim.x / kGroupLanes, grp = threadIdx.x / kGroupLanes;
    const int m0 = blockIdx.x * R;

    for (int r = threadIdx.x >> 6; r < R; r += blockDim.x >> 6) {      // a wave a token
        const int m = m0 + r;
        const int b = m < a.b.rows ? find_seq(a.b, m, lane) : a.b.n_seq;
        int p = 0;
        int64_t sl = -1;
        bool on = false;
        if (b < a.b.n_seq) {
            const Seq s = load_seq(a.b, b);
            on = m >= s.row0 && m < s.row0 + s.rows;
            p = s.p0 + (m - s.row0);
            if (on && p >= 0 && s.L > 0) sl = s.slot0 + p;
        }
        if (lane == 0) {
            slot[r] = sl;
            live[r] = on;
        }
        if (lane < a.half) {
            const double t = (double)p * (a.inv_freq[lane] * 0.15915494309189535);   // turns
            float sn, cn;
            sincospif(2.0f * (float)(t - rint(t)), &sn, &cn);
            cs[r][lane] = make_float2(cn, sn);
        }
    }
    __syncthreads();

    const int heads = a.Hq + 2 * a.Hkv;
    for (int h0 = 0; h0 < heads; h0 += groups) {
        const int h = h0 + grp;
        if (h >= heads) continue;
        const bool is_q = h < a.Hq, is_k = !is_q && h < a.Hq + a.Hkv;
        const int hh = is_q ? h : is_k ? h - a.Hq : h - a.Hq - a.Hkv;
        const uint16_t *src = is_q ? a.q : is_k ? a.k : a.v;
        const int64_t stride = is_q ? a.q_stride : is_k ? a.k_stride : a.v_stride;
        uint4 x[R];
#pragma unroll
        for (int r = 0; r < R; ++r)
            x[r] = live[r] ? load_row<R>(src + (int64_t)(m0 + r) * stride + hh * kHeadDim + 8 * l) : uint4{};
        const uint16_t *w = is_q ? a.q_norm : is_k ? a.k_norm : nullptr;
        uint2 w0 = {}, w1 = {};
        if (w) {
            w0 = *(const uint2 *)(w + 8 * l);
            w1 = *(const uint2 *)(w + 8 * l + 4);
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            uint16_t *dst = is_q ? a.q_out + (int64_t)(m0 + r) * a.q_out_stride + hh * kHeadDim
                                 : (is_k ? a.kc : a.vc) + slot[r] * a.b.tok + hh * a.b.head;
            uint4 y = x[r];
            if (is_q || is_k) {
                float f[8];
                const uint32_t xw[4] = {x[r].x, x[r].y, x[r].z, x[r].w}, ww[4] = {w0.x, w0.y, w1.x, w1.y};
                float ss = 0.0f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    f[2 * i] = bf16_lo_to_f32(xw[i]);
                    f[2 * i + 1] = bf16_hi_to_f32(xw[i]);
                    ss += f[2 * i] * f[2 * i] + f[2 * i + 1] * f[2 * i + 1];
                }
                if (w) {
                    const float inv = 1.0f / sqrtf(row_sum(ss) * (1.0f / kHeadDim) + a.eps);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        f[2 * i] = f[2 * i] * inv * bf16_lo_to_f32(ww[i]);
                        f[2 * i + 1] = f[2 * i + 1] * inv * bf16_hi_to_f32(ww[i]);
                    }
                }
                float o[8];
                if (a.interleaved) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const bool in = 4 * l + i < a.half;
                        const float2 t = cs[r][in ? 4 * l + i : 0];
                        o[2 * i] = in ? f[2 * i] * t.x - f[2 * i + 1] * t.y : f[2 * i];
                        o[2 * i + 1] = in ? f[2 * i] * t.y + f[2 * i + 1] * t.x : f[2 * i + 1];
                    }
                } else {
                    // the partner of a dimension is half / 8 lanes away
                    const int hl = a.half >> 3;
                    const bool lo = l < hl, in = l < 2 * hl;
                    const int from = (lane & 48) | (in ? lo ? l + hl : l - hl : l);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float other = __shfl(f[i], from);
                        const float2 t = cs[r][in ? (lo ? 8 * l : 8 * (l - hl)) + i : 0];
                        o[i] = !in ? f[i] : lo ? f[i] * t.x - other * t.y : other * t.y + f[i] * t.x;
                    }
                }
                y = make_uint4(cvt_pk_bf16(o[0], o[1]), cvt_pk_bf16(o[2], o[3]), cvt_pk_bf16(o[4], o[5]), cvt_pk_bf16(o[6], o[7]));
            }
            if (is_q ? live[r] : slot[r] >= 0) store_row<R>(dst + 8 * l, y);
        }
    }
}

}  // namespace

hipError_t launch_append(const AppendArgs &a, hipStream_t st) {
    const int heads = a.Hq + 2 * a.Hkv;
    const int threads = heads * kGroupLanes > kAppendThreads ? kAppendThreads : (heads * kGroupLanes + 63) / 64 * 64;
    if (a.b.rows == 0) return hipSuccess;
    if (a.b.rows < kManyRows) hipLaunchKernelGGL(k_norm_rope_append<1>, dim3(a.b.rows), dim3(threads), 0, st, a);
    else hipLaunchKernelGGL(k_norm_rope_append<4>, dim3((a.b.rows + 3) / 4), dim3(threads), 0, st, a);
    return hipGetLastError();
}

}  // namespace qlin
