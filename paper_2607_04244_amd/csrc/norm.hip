// The norms around a block with its gate and the residual, and the quantization of tokens
// to 8 bits (qlin_block_norm, qlin_quantize_tokens in include/qlin_lowbit.h).
//
// Bound by memory: every element is read and written once, rows stay in registers
// between the reductions over a row and what they scale.  A row belongs to a wave, whose
// sums need no barrier, or to a workgroup where there are too few rows for that or they
// are too wide.  As workgroups / waves, us: norms of 2560 with 256, 1024, 2048, 4096, 8192 rows
// 4.6 / 6.5, 7.8 / 8.9, 11.7 / 11.4, 17.8 / 15.8, 30.2 / 29.1; of 4096, where a wave's rows take all
// its registers, with 2048, 8192 15.4 / 16.0, 48.1 / 54.9; tokens of 4096 with 1024, 2048, 8192 6.1 /
// 5.7, 9.1 / 7.9, 24.4 / 18.3.  8192 rows of 2560 with a gate of their own, 210 MB, 42.7 us from
// memory, 4.9 TB/s: a copy's rate.  One row 2.4 to 2.7 us, the launch and two trips to memory.
// Gated tokens are bound by arithmetic, 43 vector instructions an element, with a division and
// an exponential in full: 333 rows of 9728, two on 77 of 256 units, 9.3 to 10.7 us.
#include "target_common.h"
#include "lowbit_internal.h"

#include <type_traits>

namespace qlin {

namespace {

constexpr int kWaveRows = 4;             // rows (waves) of a workgroup where a row is a wave's

// A row's threads: all of a wave (WG = false) or of a workgroup.
template <bool WG>
struct RowThreads {
    int row, at, count;
    __device__ inline RowThreads() {
        if constexpr (WG) {
            row = blockIdx.x;
            at = threadIdx.x;
            count = blockDim.x;
        } else {
            row = blockIdx.x * kWaveRows + (threadIdx.x >> 6);
            at = threadIdx.x & 63;
            count = 64;
        }
    }
};

// Reductions over a row's threads, the result in every one.
template <bool WG, typename T, typename F>
__device__ inline T row_reduce(T v, T *lds, F f) {
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v = f(v, __shfl_xor(v, d));
    if constexpr (WG) {
        __syncthreads();                                     // the last reduction's values have been read
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = lds[0];
        for (int i = 1; i < (int)(blockDim.x >> 6); ++i) v = f(v, lds[i]);
    }
    return v;
}

__device__ inline void unpack8(const uint4 &x, float f[8]) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = bf16_lo_to_f32(w[i]);
        f[2 * i + 1] = bf16_hi_to_f32(w[i]);
    }
}

// CH units of 8 elements a thread.
template <int CH, bool WG>
__global__ __launch_bounds__(WG ? 1024 : 64 * kWaveRows) void k_block_norm(BlockNormArgs a) {
    __shared__ float sums[16];
    const RowThreads<WG> t;
    if (t.row >= a.rows) return;
    const int units = a.width / 8;
    auto unit = [&](int c) { return t.at + c * t.count; };
    auto sum = [](float x, float y) { return x + y; };
    const float per = 1.0f / (float)a.width;
    const uint16_t *res = a.residual + (int64_t)t.row * a.residual_stride;

    uint4 h[CH], y[CH], gate[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        h[c] = y[c] = gate[c] = uint4{};
        if (unit(c) >= units) continue;
        h[c] = *(const uint4 *)(res + 8 * unit(c));
        if (a.y) y[c] = *(const uint4 *)(a.y + (int64_t)t.row * a.y_stride + 8 * unit(c));
        if (a.gate) gate[c] = *(const uint4 *)(a.gate + (int64_t)t.row * a.gate_stride + 8 * unit(c));
    }
    if (a.y) {
        float inv = a.scale;
        if (a.post) {
            float ss = 0.0f;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                float f[8];
                unpack8(y[c], f);
#pragma unroll
                for (int i = 0; i < 8; ++i) ss += f[i] * f[i];
            }
            inv = a.scale / sqrtf(row_reduce<WG>(ss, sums, sum) * per + a.eps);
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if (unit(c) >= units) continue;
            float f[8], r[8];
            unpack8(y[c], f);
            unpack8(h[c], r);
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] *= inv;
            if (a.post) {
                float w[8];
                unpack8(*(const uint4 *)(a.post + 8 * unit(c)), w);
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] *= w[i];
            }
            if (a.gate) {
                float g[8];
                unpack8(gate[c], g);
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] *= a.sigmoid ? 1.0f / (1.0f + __expf(-g[i])) : g[i];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) r[i] += f[i];
            h[c] = pack8(r);
            *(uint4 *)(a.residual_out + (int64_t)t.row * a.residual_out_stride + 8 * unit(c)) = h[c];
        }
    }
    if (!a.pre) return;
    float ss = 0.0f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        float f[8];
        unpack8(h[c], f);
#pragma unroll
        for (int i = 0; i < 8; ++i) ss += f[i] * f[i];
    }
    const float inv = 1.0f / sqrtf(row_reduce<WG>(ss, sums, sum) * per + a.eps);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        if (unit(c) >= units) continue;
        float f[8], w[8];
        unpack8(h[c], f);
        unpack8(*(const uint4 *)(a.pre + 8 * unit(c)), w);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = f[i] * inv * w[i];
        *(uint4 *)(a.out + (int64_t)t.row * a.out_stride + 8 * unit(c)) = pack8(f);
    }
}

template <int CH, bool WG>
__global__ __launch_bounds__(WG ? 1024 : 64 * kWaveRows) void k_quantize_tokens(QuantizeArgs a) {
    __shared__ uint32_t peaks[16];
    const RowThreads<WG> t;
    if (t.row >= a.rows) return;
    const int units = a.width / 8;
    auto unit = [&](int c) { return t.at + c * t.count; };
    const uint16_t *x = a.x + (int64_t)t.row * a.x_stride;
    uint4 u[CH], up[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        u[c] = up[c] = uint4{};
        if (unit(c) >= units) continue;
        u[c] = *(const uint4 *)(x + 8 * unit(c));
        if (a.gated) up[c] = *(const uint4 *)(x + a.width + 8 * unit(c));
    }
    float f[CH][8];
    uint32_t peak = 0;                       // |v|'s bits: an infinity is past all numbers, a NaN past that
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        unpack8(u[c], f[c]);
        if (a.gated) {
            float b[8];
            unpack8(up[c], b);
#pragma unroll
            for (int i = 0; i < 8; ++i) f[c][i] = f[c][i] / (1.0f + expf(-f[c][i])) * b[i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) peak = max(peak, __float_as_uint(f[c][i]) & 0x7FFFFFFFu);
    }
    peak = row_reduce<WG>(peak, peaks, [](uint32_t x, uint32_t y) { return max(x, y); });
    const bool finite = peak < 0x7F800000u, zero = peak < 0x0D800000u;       // 2^-100
    const float scale = finite ? zero ? 0.0f : __uint_as_float(peak) / 127.0f : __builtin_nanf("");
    const float inv = 1.0f / scale;
    if (t.at == 0) a.scale[t.row] = scale;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        if (unit(c) >= units) continue;
        uint32_t w[2] = {0, 0};
        if (finite && !zero) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                w[i >> 2] |= ((uint32_t)(int)rintf(quotient(f[c][i], scale, inv)) & 0xFFu) << 8 * (i & 3);
        }
        *(uint2 *)(a.codes + (int64_t)t.row * a.codes_stride + 8 * unit(c)) = make_uint2(w[0], w[1]);
    }
}

// Calls run(CH, WG, grid, threads).  A wave takes rows of up to Most units a lane.
template <int Most, typename F>
hipError_t for_rows(int rows, int width, F run) {
    static_assert(Most == 5 || Most == 8, "the kernels that there are");
    const int units = width / 8;
    if (rows >= 2048 && units <= 64 * Most) {
        const dim3 grid((rows + kWaveRows - 1) / kWaveRows), threads(64 * kWaveRows);
        const int per = (units + 63) / 64;
        if (per <= 1) run(std::integral_constant<int, 1>{}, std::false_type{}, grid, threads);
        else if (per <= 2) run(std::integral_constant<int, 2>{}, std::false_type{}, grid, threads);
        else if (Most == 5 || per <= 5) run(std::integral_constant<int, 5>{}, std::false_type{}, grid, threads);
        else run(std::integral_constant<int, Most>{}, std::false_type{}, grid, threads);
    } else {
        const int per = (units + 1023) / 1024, n = (units + per - 1) / per;
        const dim3 grid(rows), threads((n + 63) / 64 * 64);
        if (per <= 1) run(std::integral_constant<int, 1>{}, std::true_type{}, grid, threads);
        else if (per <= 2) run(std::integral_constant<int, 2>{}, std::true_type{}, grid, threads);
        else if (per <= 4) run(std::integral_constant<int, 4>{}, std::true_type{}, grid, threads);
        else run(std::integral_constant<int, 8>{}, std::true_type{}, grid, threads);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_block_norm(const BlockNormArgs &a, hipStream_t st) {
    return for_rows<5>(a.rows, a.width, [&](auto ch, auto wg, dim3 grid, dim3 threads) {
        hipLaunchKernelGGL((k_block_norm<decltype(ch)::value, decltype(wg)::value>), grid, threads, 0, st, a);
    });
}

hipError_t launch_quantize_tokens(const QuantizeArgs &a, hipStream_t st) {
    return for_rows<8>(a.rows, a.width, [&](auto ch, auto wg, dim3 grid, dim3 threads) {
        hipLaunchKernelGGL((k_quantize_tokens<decltype(ch)::value, decltype(wg)::value>), grid, threads, 0, st, a);
    });
}

}  // namespace qlin
