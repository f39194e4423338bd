// Norms and rotation of queries and keys with the append to the key/value cache
// (qlin_norm_rope_append in include/qlin_target.h; qlin_norm_rope_append_four_bit in
// include/qlin_lowbit.h, whose rows of keys and values are laid on 4-bit grids).
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
#include "lowbit_internal.h"

#include <climits>
#include <type_traits>

namespace qlin {

namespace {

constexpr int kGroupLanes = 16;          // lanes of a head row
constexpr int kAppendThreads = 1024;
constexpr int kManyRows = 640;           // R = 4 from here on

// v of the lane N to the right within 16 lanes (a DPP row), around its end.
template <int N>
__device__ inline float rotated(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x120 + N, 0xF, 0xF, false));
}
template <int N>
__device__ inline double rotated(double v) {
    return __hiloint2double(__builtin_amdgcn_update_dpp(0, __double2hiint(v), 0x120 + N, 0xF, 0xF, false),
                            __builtin_amdgcn_update_dpp(0, __double2loint(v), 0x120 + N, 0xF, 0xF, false));
}
// f over the 16 lanes, in every lane.
template <typename T, typename F>
__device__ inline T row_reduce(T v, F f) {
    v = f(v, rotated<8>(v));
    v = f(v, rotated<4>(v));
    v = f(v, rotated<2>(v));
    v = f(v, rotated<1>(v));
    return v;
}
template <typename T>
__device__ inline T row_sum(T v) {
    return row_reduce(v, [](T x, T y) { return x + y; });
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

// Eight dimensions (8 l .. 8 l + 7) of a head row: norm with the weights w (none: null), and the
// rotation by the token's angles cs = (cos, sin).
__device__ inline void norm_rotate(const AppendArgs &a, const uint4 &x, const uint16_t *w, const uint2 &w0, const uint2 &w1, const float2 *cs,
                                   int lane, float o[8]) {
    const int l = lane & 15;
    float f[8];
    const uint32_t xw[4] = {x.x, x.y, x.z, x.w}, ww[4] = {w0.x, w0.y, w1.x, w1.y};
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
    // fused products written out, so that a build's choice cannot change an output's last bit
    if (a.interleaved) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool in = 4 * l + i < a.half;
            const float2 t = cs[in ? 4 * l + i : 0];
            o[2 * i] = in ? __builtin_fmaf(f[2 * i], t.x, -(f[2 * i + 1] * t.y)) : f[2 * i];
            o[2 * i + 1] = in ? __builtin_fmaf(f[2 * i], t.y, f[2 * i + 1] * t.x) : f[2 * i + 1];
        }
    } else {
        // the partner of a dimension is half / 8 lanes away
        const int hl = a.half >> 3;
        const bool lo = l < hl, in = l < 2 * hl;
        const int from = (lane & 48) | (in ? lo ? l + hl : l - hl : l);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float other = __shfl(f[i], from);
            const float2 t = cs[in ? (lo ? 8 * l : 8 * (l - hl)) + i : 0];
            o[i] = in ? __builtin_fmaf(f[i], t.x, lo ? -(other * t.y) : other * t.y) : f[i];
        }
    }
}

// Place of angle i among a token's angles in 64 bits: what 8 lanes read together, angles 8 apart,
// lies side by side.
__device__ inline int angle_at(int i) { return (i & 7) * 8 + (i >> 3); }

// The same in 64 bits, rounded to fp32 and bf16 at the end.  The row is rotated before it is divided by
// its root: x w is exact, with 16 significant bits at most, so a double's high word holds it
// whole, whatever its size, and partners travel in 32 bits.
__device__ inline uint4 norm_rotate_64(const AppendArgs &a, const uint4 &x, const uint16_t *w, const uint2 &w0, const uint2 &w1,
                                       const double2 *cs, int lane) {
    const int l = lane & 15;
    float f[8], y[8];
    int xw_hi[8];
    const uint32_t xw[4] = {x.x, x.y, x.z, x.w}, ww[4] = {w0.x, w0.y, w1.x, w1.y};
    double ss = 0.0, inv = 1.0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = bf16_lo_to_f32(xw[i]);
        f[2 * i + 1] = bf16_hi_to_f32(xw[i]);
    }
    if (w) {
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = __builtin_fma((double)f[i], (double)f[i], ss);
        const double mean = row_sum(ss) * (1.0 / kHeadDim) + (double)a.eps;
        // the hardware's estimate of 1 / sqrt(mean), twice by Newton's rule: past 2^-50
        inv = __builtin_amdgcn_rsq(mean);
#pragma unroll
        for (int i = 0; i < 2; ++i) inv = __builtin_fma(0.5 * inv, __builtin_fma(-mean * inv, inv, 1.0), inv);
        if (!(mean > 0.0)) inv = 1.0 / sqrt(mean);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float by = i & 1 ? bf16_hi_to_f32(ww[i >> 1]) : bf16_lo_to_f32(ww[i >> 1]);
        xw_hi[i] = __double2hiint(w ? (double)f[i] * (double)by : (double)f[i]);
    }
    auto product = [](int hi) { return __hiloint2double(hi, 0); };
    if (a.interleaved) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool in = 4 * l + i < a.half;
            const double2 t = cs[in ? angle_at(4 * l + i) : 0];
            const double x0 = product(xw_hi[2 * i]), x1 = product(xw_hi[2 * i + 1]);
            y[2 * i] = (float)((in ? __builtin_fma(x0, t.x, -(x1 * t.y)) : x0) * inv);
            y[2 * i + 1] = (float)((in ? __builtin_fma(x0, t.y, x1 * t.x) : x1) * inv);
        }
    } else {
        const int hl = a.half >> 3;
        const bool lo = l < hl, in = l < 2 * hl;
        const int from = (lane & 48) | (in ? lo ? l + hl : l - hl : l), sign = lo ? 0 : INT_MIN;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            // what the upper half gets has its sign, what the lower gets the other
            const double x0 = product(xw_hi[i]), other = product(__shfl(xw_hi[i] ^ sign, from));
            const double2 t = cs[in ? angle_at((lo ? 8 * l : 8 * (l - hl)) + i) : 0];
            y[i] = (float)((in ? __builtin_fma(x0, t.x, other * t.y) : x0) * inv);
        }
    }
    return pack8(y);
}

// A row of bf16 values on its 4-bit grid: this lane's word of codes, and the row's (step, offset).
// Quotients are correctly rounded, so a code is that of the exact one, ties included.
__device__ inline uint32_t lay_on_grid(const uint4 &y, int lane, uint32_t &grid) {
    const uint32_t w[4] = {y.x, y.y, y.z, y.w};
    float f[8];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = bf16_lo_to_f32(w[i]);
        f[2 * i + 1] = bf16_hi_to_f32(w[i]);
        top = max(top, max(w[i] << 16 & 0x7FFFFFFFu, w[i] & 0x7FFF0000u));
    }
    const uint64_t without_number = __ballot(top >= 0x7F800000u) >> (lane & 48) & 0xFFFFu;      // in the row's 16 lanes
    float low = f[0], high = f[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) {
        low = fminf(low, f[i]);
        high = fmaxf(high, f[i]);
    }
    low = row_reduce(low, [](float x, float y) { return fminf(x, y); });
    high = row_reduce(high, [](float x, float y) { return fmaxf(x, y); });
    const float range = high - low;
    if (without_number || !(range < __builtin_huge_valf())) {
        grid = 0x7FC07FC0u;
        return 0;
    }
    const uint16_t sb = cvt_bf16(quotient(range, 15.0f, 1.0f / 15.0f));
    const float step = __uint_as_float((uint32_t)sb << 16);
    grid = __float_as_uint(low);             // bf16 in the high half: the offset
    if (sb < 0x0080) return 0;               // below 2^-126
    grid |= sb;
    // of a number of 8 bits, the hardware's estimate (off by one unit at most) and Newton's rule give
    // the correctly rounded reciprocal: so for each of the 128 significands and each estimate
    float inverse = __builtin_amdgcn_rcpf(step);
    inverse = __builtin_fmaf(__builtin_fmaf(-step, inverse, 1.0f), inverse, inverse);
    // added to 1.5 2^23 a quotient is rounded to a whole number, in the sum's low bits
    constexpr uint32_t kWhole = 0x4B400000u;
    uint32_t codes = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t c = __float_as_uint(quotient(f[i] - low, step, inverse) + __uint_as_float(kWhole));
        codes += (min(c, kWhole + 15u) - kWhole) << 4 * i;
    }
    return codes;
}

// The workgroup's tokens m0 .. m0 + R - 1, a wave each: their cache slots (-1: not stored), whether
// they are new tokens of some sequence, and (cos, sin) of their angles, in 64 bits too where
// cs64 is given.
template <int R>
__device__ inline void find_tokens(const AppendArgs &a, int m0, int64_t *slot, int *live, float2 (*cs)[kHeadDim / 2], double2 (*cs64)[kHeadDim / 2]) {
    const int lane = threadIdx.x & 63;
    for (int r = threadIdx.x >> 6; r < R; r += blockDim.x >> 6) {
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
            if (cs64) {
                double sn, cn;
                sincospi(2.0 * (t - rint(t)), &sn, &cn);
                cs64[r][angle_at(lane)] = make_double2(cn, sn);
                cs[r][lane] = make_float2((float)cn, (float)sn);
            } else {
                float sn, cn;
                sincospif(2.0f * (float)(t - rint(t)), &sn, &cn);
                cs[r][lane] = make_float2(cn, sn);
            }
        }
    }
}

template <int R>
__global__ __launch_bounds__(kAppendThreads) void k_norm_rope_append(AppendArgs a) {
    __shared__ float2 cs[R][kHeadDim / 2];
    __shared__ int64_t slot[R];
    __shared__ int live[R];
    const int lane = threadIdx.x & 63, l = threadIdx.x & 15;
    const int groups = blockDim.x / kGroupLanes, grp = threadIdx.x / kGroupLanes;
    const int m0 = blockIdx.x * R;
    find_tokens<R>(a, m0, slot, live, cs, nullptr);
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
                float o[8];
                norm_rotate(a, x[r], w, w0, w1, cs[r], lane, o);
                y = pack8(o);
            }
            if (is_q ? live[r] : slot[r] >= 0) store_row<R>(dst + 8 * l, y);
        }
    }
}

// Into the 4-bit cache.  The keys in 64 bits, so that their codes are those of the definition and
// not those of its rounding errors: several times the instructions of a query's row, so rows
// are dealt out keys first and few waves have those of more than one token.  8192 tokens 52
// us; a wave a head for all four tokens 58.3, of which the keys' 64 bits 17 (the bf16 cache
// 40.6).  80 registers, so that two workgroups of 48 heads share a compute unit: with 88, and
// one, 63.6.  One token a workgroup keeps the order of its heads (368 rows 7.05 us; 7.44 dealt): a launch
// and three trips to memory one after the other, as rows are requested behind the search for
// their sequence; and under the bound of registers meant for four tokens it keeps one in scratch.
template <int R>
__global__ __launch_bounds__(kAppendThreads, 6) void k_norm_rope_append_kv4(AppendKv4Args args) {
    __shared__ float2 cs[R][kHeadDim / 2];
    __shared__ double2 cs64[R][kHeadDim / 2];
    __shared__ int64_t slot[R];
    __shared__ int live[R];
    const AppendArgs &a = args.a;
    const int lane = threadIdx.x & 63, l = threadIdx.x & 15;
    const int groups = blockDim.x / kGroupLanes, grp = threadIdx.x / kGroupLanes;
    const int m0 = blockIdx.x * R;
    find_tokens<R>(a, m0, slot, live, cs, cs64);
    __syncthreads();

    const int keys = R * a.Hkv, all = R * (a.Hq + 2 * a.Hkv);
    // row i: keys of all tokens, then values, then queries
    struct Row { bool is_k, is_q; int r, h; };
    auto row_of = [&](int i) {
        if constexpr (R == 1) {                          // one token: its queries, keys, values
            const int h = i - a.Hq;
            return Row{h >= 0 && h < a.Hkv, h < 0, 0, h < 0 ? i : h < a.Hkv ? h : h - a.Hkv};
        }
        Row t{i < keys, i >= 2 * keys, 0, 0};
        const int in = t.is_q ? i - 2 * keys : t.is_k ? i : i - keys, heads = t.is_q ? a.Hq : a.Hkv;
        const uint32_t inverse = t.is_q ? args.inv_q : args.inv_kv;
        t.r = inverse ? (int)__umulhi((uint32_t)in, inverse) : in;
        t.h = in - t.r * heads;
        return t;
    };
    for (int i0 = grp; i0 < all; i0 += R * groups) {
        uint4 x[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int at = i0 + i * groups;
            x[i] = uint4{};
            if (at >= all) continue;
            const Row t = row_of(at);
            if (!live[t.r]) continue;
            const uint16_t *src = t.is_q ? a.q + (int64_t)(m0 + t.r) * a.q_stride : t.is_k ? a.k + (int64_t)(m0 + t.r) * a.k_stride : a.v + (int64_t)(m0 + t.r) * a.v_stride;
            x[i] = load_row<R>(src + t.h * kHeadDim + 8 * l);
        }
        // one row after the other, so that two workgroups' registers fit a compute unit
#pragma unroll 1
        for (int i = i0; i < min(i0 + R * groups, all); i += groups) {
            const uint4 now = x[0];
#pragma unroll
            for (int k = 0; k + 1 < R; ++k) x[k] = x[k + 1];
            int at = lane;                   // opaque: places in LDS worked out for each row take fewer registers
            asm volatile("" : "+v"(at));
            const Row t = row_of(i);
            const uint16_t *w = t.is_q ? a.q_norm : t.is_k ? a.k_norm : nullptr;
            uint2 w0 = {}, w1 = {};
            if (w) {
                w0 = *(const uint2 *)(w + 8 * l);
                w1 = *(const uint2 *)(w + 8 * l + 4);
            }
            if (t.is_q) {
                float o[8];
                norm_rotate(a, now, w, w0, w1, cs[t.r], at, o);
                if (live[t.r]) store_row<R>(a.q_out + (int64_t)(m0 + t.r) * a.q_out_stride + t.h * kHeadDim + 8 * l, pack8(o));
                continue;
            }
            uint32_t grid;
            const uint32_t codes = lay_on_grid(t.is_k ? norm_rotate_64(a, now, w, w0, w1, cs64[t.r], at) : now, lane, grid);
            if (slot[t.r] < 0) continue;
            const int64_t row = slot[t.r] * a.b.tok + t.h * a.b.head;
            (t.is_k ? args.c.k : args.c.v)[16 * row + l] = codes;
            if (l == 0) (t.is_k ? args.c.k_grid : args.c.v_grid)[row] = grid;
        }
    }
}

// Heads of a token, in threads.
int append_threads(const AppendArgs &a) {
    const int heads = a.Hq + 2 * a.Hkv;
    return heads * kGroupLanes > kAppendThreads ? kAppendThreads : (heads * kGroupLanes + 63) / 64 * 64;
}

}  // namespace

hipError_t launch_append(const AppendArgs &a, hipStream_t st) {
    if (a.b.rows == 0) return hipSuccess;
    const dim3 threads(append_threads(a));
    if (a.b.rows < kManyRows) hipLaunchKernelGGL(k_norm_rope_append<1>, dim3(a.b.rows), threads, 0, st, a);
    else hipLaunchKernelGGL(k_norm_rope_append<4>, dim3((a.b.rows + 3) / 4), threads, 0, st, a);
    return hipGetLastError();
}

hipError_t launch_append_kv4(const AppendKv4Args &args, hipStream_t st) {
    const AppendArgs &a = args.a;
    if (a.b.rows == 0) return hipSuccess;
    AppendKv4Args x = args;
    auto inverse = [](int n) { return n > 1 ? (uint32_t)((((uint64_t)1 << 32) + n - 1) / n) : 0u; };
    x.inv_q = inverse(a.Hq);
    x.inv_kv = inverse(a.Hkv);
    const dim3 threads(append_threads(a));
    if (a.b.rows < kManyRows) hipLaunchKernelGGL(k_norm_rope_append_kv4<1>, dim3(a.b.rows), threads, 0, st, x);
    else hipLaunchKernelGGL(k_norm_rope_append_kv4<4>, dim3((a.b.rows + 3) / 4), threads, 0, st, x);
    return hipGetLastError();
}

}  // namespace qlin
