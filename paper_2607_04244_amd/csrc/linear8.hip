// The linear of 8-bit integers with a scale for each token and channel (qlin_eight_bit_linear in
// include/qlin_lowbit.h).
//
// y[m][n] = sx[m] sw[n] sum_k x[m][k] w[n][k]; the sums are 32-bit integers from the matrix
// cores, exact in any order, so K is cut freely over waves and workgroups.  The weights are
// the A operand, the tokens B: a lane's results are four channels of one token at a time.
//
//   k_i8_few<MT>   up to 16 MT rows: bound by the weights' bytes.  A workgroup has 16 channels,
//       its waves a part of K each, read straight into the operands' registers.
//   k_i8_tile      128 x 128 outputs, K 128 at a time through LDS: bound by the matrix cores.
//   k_i8_join      adds K ranges' sums and scales them.
#include "target_common.h"
#include "lowbit_internal.h"

namespace qlin {

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v16i __attribute__((ext_vector_type(16)));

__device__ inline v4i load16(const int8_t *p) { return *(const v4i *)p; }
__device__ inline v4i load16_nt(const int8_t *p) { return __builtin_nontemporal_load((const v4i *)p); }

__device__ inline float scaled(int sum, float sx, float sw) { return (float)sum * (sx * sw); }

// ---------------------------------------------------------------- few rows

constexpr int kFewWaves = 8, kFewBatch = 8;          // steps of 64 bytes requested together

template <int MT>
__global__ __launch_bounds__(kFewWaves * 64) void k_i8_few(I8Args a) {
    __shared__ v4i part[kFewWaves][MT][64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int g = lane >> 4, r = lane & 15;
    const int n0 = blockIdx.x * 16, all = (a.K + kI8FewStep - 1) / kI8FewStep;
    const int first = blockIdx.y * a.steps, end = min(first + a.steps, all);
    const int per = (end - first + kFewWaves - 1) / kFewWaves;
    const int s0 = first + wave * per, s1 = min(s0 + per, end);

    const int8_t *wp = a.w + (int64_t)min(n0 + r, a.N - 1) * a.w_stride + 16 * g;
    const int8_t *xp[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) xp[t] = a.x + (int64_t)min(16 * t + r, a.M - 1) * a.x_stride + 16 * g;
    v4i acc[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[t] = v4i{0, 0, 0, 0};
    for (int s = s0; s < s1; s += kFewBatch) {
        v4i wv[kFewBatch], xv[kFewBatch][MT];
#pragma unroll
        for (int i = 0; i < kFewBatch; ++i) {
            const int k = (s + i) * kI8FewStep;
            wv[i] = v4i{0, 0, 0, 0};                 // past the range or K
            if (s + i < s1 && k + 16 * g < a.K) {
                wv[i] = load16_nt(wp + k);
#pragma unroll
                for (int t = 0; t < MT; ++t) xv[i][t] = load16(xp[t] + k);
            } else {
#pragma unroll
                for (int t = 0; t < MT; ++t) xv[i][t] = v4i{0, 0, 0, 0};
            }
        }
#pragma unroll
        for (int i = 0; i < kFewBatch; ++i)
#pragma unroll
            for (int t = 0; t < MT; ++t) acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv[i], xv[i][t], acc[t], 0, 0, 0);
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) part[wave][t][lane] = acc[t];
    __syncthreads();
    // an output a thread: channel fastest
    for (int e = threadIdx.x; e < 256 * MT; e += kFewWaves * 64) {
        const int n = e & 15, m = e >> 4;
        int sum = 0;
#pragma unroll
        for (int i = 0; i < kFewWaves; ++i) sum += ((const int *)&part[i][m >> 4][(m & 15) + 16 * (n >> 2)])[n & 3];
        if (m >= a.M || n0 + n >= a.N) continue;
        if (a.S > 1) a.parts[((int64_t)blockIdx.y * a.M + m) * a.N + n0 + n] = sum;
        else a.y[(int64_t)m * a.y_stride + n0 + n] = cvt_bf16(scaled(sum, a.x_scale[m], a.w_scale[n0 + n]));
    }
}

// ---------------------------------------------------------------- many rows

constexpr int kTileThreads = 256;

// Rows of 128 bytes in LDS, their 16-byte units in an order that changes every two rows: one
// unit of 16 rows, which lanes read together, meets different banks.
__device__ inline int tile_unit(int row, int u) { return row * 8 + (u ^ ((row >> 1) & 7)); }

__global__ __launch_bounds__(kTileThreads, 2) void k_i8_tile(I8Args a) {
    constexpr int T = kI8Tile, U = T * kI8TileStep / 16;                       // units of one operand's stage
    __shared__ __attribute__((aligned(16))) uint4 ring[2][2][U];                // [stage][w, x]
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int hi = lane >> 5, r = lane & 31;
    const int n0 = (int)(blockIdx.x % (unsigned)a.tiles_n) * T, m0 = (int)(blockIdx.x / (unsigned)a.tiles_n) * T;
    const int all = (a.K + kI8TileStep - 1) / kI8TileStep;
    const int first = blockIdx.y * a.steps, end = min(first + a.steps, all);

    // a wave loads 8 rows at a time, 4 times, of each operand
    const int lr = lane >> 3, lu = lane & 7;
    const int8_t *src[2][4];
    int unit[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int row = 8 * (4 * wave + j) + lr;
        unit[j] = lu ^ ((row >> 1) & 7);
        src[0][j] = a.w + (int64_t)min(n0 + row, a.N - 1) * a.w_stride;
        src[1][j] = a.x + (int64_t)min(m0 + row, a.M - 1) * a.x_stride;
    }
    auto issue = [&](int s) {
        const int k = s * kI8TileStep, st = s & 1;
#pragma unroll
        for (int o = 0; o < 2; ++o)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int at = k + 16 * unit[j];                                // past K: its first unit, left out below
                load_lds_x16(src[o][j] + (at < a.K ? at : 0), &ring[st][o][64 * (4 * wave + j)]);
            }
    };
    const int wn = 64 * (wave & 1), wm = 64 * (wave >> 1);
    v16i acc[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;
    if (first < end) issue(first);
    for (int s = first; s < end; ++s) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        lds_barrier();                                                         // this stage is there, the other one read
        if (s + 1 < end) issue(s + 1);
        const uint4 *ws = ring[s & 1][0], *xs = ring[s & 1][1];
        const bool partial = (s + 1) * kI8TileStep > a.K;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            v4i wf[2], xf[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                wf[i] = __builtin_bit_cast(v4i, ws[tile_unit(wn + 32 * i + r, 2 * ks + hi)]);
                xf[i] = __builtin_bit_cast(v4i, xs[tile_unit(wm + 32 * i + r, 2 * ks + hi)]);
                if (partial && s * kI8TileStep + 16 * (2 * ks + hi) >= a.K) wf[i] = v4i{0, 0, 0, 0};
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wf[i], xf[j], acc[i][j], 0, 0, 0);
        }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int m = m0 + wm + 32 * j + r;
        if (m >= a.M) continue;
        const float sx = a.S > 1 ? 0.0f : a.x_scale[m];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int n = n0 + wn + 32 * i + 8 * q + 4 * hi;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (n + e >= a.N) continue;
                    const int sum = acc[i][j][4 * q + e];
                    if (a.S > 1) a.parts[((int64_t)blockIdx.y * a.M + m) * a.N + n + e] = sum;
                    else a.y[(int64_t)m * a.y_stride + n + e] = cvt_bf16(scaled(sum, sx, a.w_scale[n + e]));
                }
            }
    }
}

__global__ __launch_bounds__(256) void k_i8_join(I8Args a) {
    const int64_t all = (int64_t)a.M * a.N;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        int sum = 0;
        for (int s = 0; s < a.S; ++s) sum += a.parts[(int64_t)s * all + i];
        const int m = (int)(i / a.N), n = (int)(i - (int64_t)m * a.N);
        a.y[(int64_t)m * a.y_stride + n] = cvt_bf16(scaled(sum, a.x_scale[m], a.w_scale[n]));
    }
}

}  // namespace

hipError_t launch_i8_linear(const I8Args &a, hipStream_t st) {
    const dim3 few((a.N + 15) / 16, a.S), threads(kFewWaves * 64);
    if (a.M <= 16) hipLaunchKernelGGL(k_i8_few<1>, few, threads, 0, st, a);
    else if (a.M <= 32) hipLaunchKernelGGL(k_i8_few<2>, few, threads, 0, st, a);
    else if (a.M <= kI8FewRows) hipLaunchKernelGGL(k_i8_few<4>, few, threads, 0, st, a);
    else hipLaunchKernelGGL(k_i8_tile, dim3((unsigned)(a.tiles_m * a.tiles_n), a.S), dim3(kTileThreads), 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.S == 1) return e;
    const int64_t blocks = ((int64_t)a.M * a.N + 255) / 256;
    hipLaunchKernelGGL(k_i8_join, dim3((unsigned)(blocks < 16384 ? blocks : 16384)), dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace qlin
