// The linear of 8-bit integers with a scale for each token and channel (qlin_eight_bit_linear in
// include/qlin_lowbit.h).
//
// y[m][n] = sx[m] sw[n] sum_k x[m][k] w[n][k]; the sums are 32-bit integers from the matrix
// cores, exact in any order, so K is cut freely over waves and workgroups.  The weights are
// the A operand, the tokens B: a lane's results are four channels of one token at a time.
//
//   k_i8_few<MT, NS>  up to 16 MT rows: bound by the weights' bytes.  Eight waves share K, each
//       reads its part of 16 channels straight into the operand's registers.  16 x 2560 x 19456
//       (rows, K, channels) 14.2 us, 3.55 TB/s, where a plain read of the weights takes 11.0;
//       1 x 4096 x 2560 4.9 us, the launch and one trip to memory.
//   k_i8_tile      tiles of 64 x 128 to 256 x 320 outputs through LDS: bound by the matrix cores and
//       LDS reads between them, and by the clock, which falls under them.  8192 x 8192 x 8192 501 to 518
//       us, 2120 to 2195 TOP/s (the library's product 2050); 2048 x 2560 x 19456 122 to 124 us,
//       1650 TOP/s (122): 488 tiles on 256 units.
//   k_i8_tile_join, k_i8_join   add K ranges' sums and scale them.
#include "target_common.h"
#include "lowbit_internal.h"

#include <type_traits>

namespace qlin {

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v16i __attribute__((ext_vector_type(16)));

__device__ inline void load_lds_a16(const int8_t *src, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" :: "s"(lds), "v"(src) : "memory", "m0");
}

__device__ inline v4i load16(const int8_t *p) { return *(const v4i *)p; }

__device__ inline float scaled(int sum, float sx, float sw) { return (float)sum * (sx * sw); }

// Four channels of a token.
__device__ inline void store4(const I8Args &a, int m, int n, float sx, const v4i &sum) {
    uint16_t *y = a.y + (int64_t)m * a.y_stride + n;
    if (n + 3 < a.N) {
        *(uint2 *)y = make_uint2(cvt_pk_bf16(scaled(sum[0], sx, a.w_scale[n]), scaled(sum[1], sx, a.w_scale[n + 1])),
                                 cvt_pk_bf16(scaled(sum[2], sx, a.w_scale[n + 2]), scaled(sum[3], sx, a.w_scale[n + 3])));
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (n + e < a.N) y[e] = cvt_bf16(scaled(sum[e], sx, a.w_scale[n + e]));
}

// ---------------------------------------------------------------- few rows

constexpr int kFewWaves = kI8FewWaves, kFewBatch = 8;          // steps of 64 bytes requested together
constexpr int kFewGroups = 256;                      // one a compute unit

// Not read with the hint that data is read once: 15.3 us with it, 14.2 without, as the 64 bytes of a
// row that a load takes are half a cache line.  One workgroup a compute unit walks several
// channel tiles: two units' worth 16.1 us, each tile its own workgroup 18.2.
// NS > 0: a wave's part of K is at most NS steps; its part of the tokens stays in registers
// while the workgroup walks channel tiles, whose weights are requested a tile ahead.  NS = 0:
// any K, both operands in batches.
template <int MT, int NS>
__global__ __launch_bounds__(kFewWaves * 64) void k_i8_few(I8Args a) {
    __shared__ v4i part[2][kFewWaves][MT][64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int g = lane >> 4, r = lane & 15;
    const int all = (a.K + kI8Step - 1) / kI8Step;
    const int first = blockIdx.y * a.steps, end = min(first + a.steps, all);
    const int per = (end - first + kFewWaves - 1) / kFewWaves;
    const int s0 = first + wave * per, s1 = min(s0 + per, end);

    const int8_t *xp[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) xp[t] = a.x + (int64_t)min(16 * t + r, a.M - 1) * a.x_stride + 16 * g;
    auto w_at = [&](int tile) { return a.w + (int64_t)min(16 * tile + r, a.N - 1) * a.w_stride + 16 * g; };
    auto inside = [&](int s) { return s < s1 && s * kI8Step + 16 * g < a.K; };
    constexpr int B = NS ? NS : kFewBatch;
    v4i wv[B], xv[B][MT];
    auto load_w = [&](const int8_t *wp, int s) {
#pragma unroll
        for (int i = 0; i < B; ++i) wv[i] = inside(s + i) ? load16(wp + (s + i) * kI8Step) : v4i{0, 0, 0, 0};
    };
    auto load_x = [&](int s) {
#pragma unroll
        for (int i = 0; i < B; ++i)
#pragma unroll
            for (int t = 0; t < MT; ++t) xv[i][t] = inside(s + i) ? load16(xp[t] + (s + i) * kI8Step) : v4i{0, 0, 0, 0};
    };
    int buffer = 0;
    if (NS) {
        load_w(w_at(blockIdx.x), s0);
        load_x(s0);
    }
    for (int tile = blockIdx.x; tile < a.tiles_n; tile += gridDim.x, buffer ^= 1) {
        v4i acc[MT];
#pragma unroll
        for (int t = 0; t < MT; ++t) acc[t] = v4i{0, 0, 0, 0};
        auto multiply = [&](const v4i *w) {
#pragma unroll
            for (int i = 0; i < B; ++i)
#pragma unroll
                for (int t = 0; t < MT; ++t) acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[i], xv[i][t], acc[t], 0, 0, 0);
        };
        if constexpr (NS > 0) {
            v4i now[B];
#pragma unroll
            for (int i = 0; i < B; ++i) now[i] = wv[i];
            if (tile + (int)gridDim.x < a.tiles_n) load_w(w_at(tile + gridDim.x), s0);
            multiply(now);
        } else {
            for (int s = s0; s < s1; s += B) {
                load_w(w_at(tile), s);
                load_x(s);
                multiply(wv);
            }
        }
#pragma unroll
        for (int t = 0; t < MT; ++t) part[buffer][wave][t][lane] = acc[t];
        lds_barrier();
        // an output a thread: channel fastest
        for (int e = threadIdx.x; e < 256 * MT; e += kFewWaves * 64) {
            const int n = 16 * tile + (e & 15), m = e >> 4;
            int sum = 0;
#pragma unroll
            for (int i = 0; i < kFewWaves; ++i) sum += ((const int *)&part[buffer][i][m >> 4][(m & 15) + 16 * ((e & 15) >> 2)])[e & 3];
            if (m >= a.M || n >= a.N) continue;
            if (a.S > 1) a.parts[((int64_t)blockIdx.y * a.M + m) * a.N + n] = sum;
            else a.y[(int64_t)m * a.y_stride + n] = cvt_bf16(scaled(sum, a.x_scale[m], a.w_scale[n]));
        }
    }
}

template <int MT>
void launch_few(const I8Args &a, int per_wave, hipStream_t st) {
    const dim3 threads(kFewWaves * 64);
    const int rounds = (a.tiles_n * a.S + kFewGroups - 1) / kFewGroups;
    const dim3 grid((a.tiles_n + rounds - 1) / rounds, a.S), each(a.tiles_n, a.S);
    constexpr int most = i8_few_steps(16 * MT);
    if (per_wave <= 5) hipLaunchKernelGGL((k_i8_few<MT, 5>), grid, threads, 0, st, a);
    else if (most >= 8 && per_wave <= 8) hipLaunchKernelGGL((k_i8_few<MT, most >= 8 ? 8 : 0>), grid, threads, 0, st, a);
    else if (per_wave <= most) hipLaunchKernelGGL((k_i8_few<MT, most>), grid, threads, 0, st, a);
    else hipLaunchKernelGGL((k_i8_few<MT, 0>), each, threads, 0, st, a);
}

// ---------------------------------------------------------------- many rows

// Steps of 64 KS bytes of K through a ring of ST stages in LDS, filled ST - 1 steps ahead by
// direct-to-LDS loads; one barrier a step.  WN x WM products of 32 x 32 a wave, GN x GM waves: 4
// waves of 128 x 128 instead of 8 of 128 x 64 read less and wait more (602 us for 8192 x 8192 x 8192
// against 572).  A step's first fragments are read during the last products of the step before, so
// that a wave alone on its SIMD does not wait for them.
// KS = 2: half the barriers, and loads of whole cache lines.  2048 x 2560 x 19456 122 to 124 us in two
// stages against 139 in three of 64 bytes, 8192 x 8192 x 8192 501 to 518 against 542; 128 x 64 outputs 24.4 against
// 28.1 (256 x 2560 x 9728).  128 x 128, where two stages are all that fits two workgroups, 28.4
// against 24.8 (333 x 9728 x 2560).
// The matrix cores alone, operands of random bits in registers, run at 3256 TOP/s on all units (4673
// with zeros: power); with the LDS reads and a barrier beside them 2853, this kernel without its
// loads 2659.  Loads dealt out between the products, a raised priority for them and tiles in bands
// of 4 were equal.
// LDS rows hold their 16-byte units in an order that changes with the row, so that one unit of 16
// rows, which lanes read together, meets different banks.
template <int KS>
__device__ inline int tile_unit(int row, int u) { return KS == 1 ? row * 4 + (u ^ ((row >> 2) & 3)) : row * 8 + (u ^ ((row >> 1) & 7)); }

// Workgroup b's tile.  Workgroups go to the 8 XCDs in turn; each XCD takes a contiguous part of
// the tiles, eight of the tokens' by all of the channels', tokens fastest: what runs at once on
// an XCD shares rows of both operands in its L2.
__device__ inline void tile_of(const I8Args &a, int b, int &tm, int &tn) {
    const int tiles = a.tiles_m * a.tiles_n, x = b & 7, whole = tiles >> 3, rest = tiles & 7;
    const int t = x * whole + min(x, rest) + (b >> 3), band = t / (8 * a.tiles_n), in = t - band * 8 * a.tiles_n;
    const int rows = min(8, a.tiles_m - 8 * band);
    tn = in / rows;
    tm = 8 * band + in - tn * rows;
}

template <int WN, int WM, int GN, int GM, int KS, int ST, int PER_CU>
__global__ __launch_bounds__(GN * GM * 64, GN * GM * PER_CU / 4) void k_i8_tile(I8Args a) {
    constexpr int TN = 32 * WN * GN, TM = 32 * WM * GM, W = GN * GM;
    constexpr int U = 4 * KS, R = 64 / U, Q = 2 * KS, Step = KS * kI8Step;          // units of a row, rows of a load, products' parts of a step
    constexpr int L = ((TN + TM) / R + W - 1) / W;                                  // loads of a wave a step
    static_assert(KS == 1 || (KS == 2 && W % 2 == 0), "a place's unit is the same in each of a wave's loads");
    __shared__ __attribute__((aligned(16))) uint4 ring[ST][L * W * 64];             // rows of w, then of x (the last one again)
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int hi = lane >> 5, r = lane & 31;
    int tm, tn;
    tile_of(a, blockIdx.x, tm, tn);
    const int n0 = tn * TN, m0 = tm * TM;
    const int k0 = blockIdx.y * a.steps * kI8Step, k1 = min(k0 + a.steps * kI8Step, a.K), end = (k1 - k0 + Step - 1) / Step;

    // load i of a wave: rows R (wave + W i) .. + R - 1 of the stage, U lanes a row
    const int8_t *src[L];
    const int unit = KS == 1 ? (lane & 3) ^ ((lane >> 4) & 3) : (lane & 7) ^ (4 * (wave & 1) + (lane >> 4));    // its place's unit
#pragma unroll
    for (int i = 0; i < L; ++i) {
        const int row = R * (wave + W * i) + lane / U;
        src[i] = row < TN ? a.w + (int64_t)min(n0 + row, a.N - 1) * a.w_stride : a.x + (int64_t)min(m0 + row - TN, a.M - 1) * a.x_stride;
    }
    const uint32_t lds = lds_addr(ring) + wave * 1024;
    auto issue = [&](int s) {
        const int at = k0 + s * Step + 16 * unit;                                   // past the range: the row's first unit, left out below
        const uint32_t to = lds + (uint32_t)(s % ST) * (uint32_t)sizeof(ring[0]);
#pragma unroll
        for (int i = 0; i < L; ++i) load_lds_a16(src[i] + (at < k1 ? at : 0), to + i * W * 1024);
    };
    const int wn = 32 * WN * (wave % GN), wm = TN + 32 * WM * (wave / GN);
    v16i acc[WN][WM];
#pragma unroll
    for (int i = 0; i < WN; ++i)
#pragma unroll
        for (int j = 0; j < WM; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;
    v4i wf[2][WN], xf[2][WM];
    auto fragments = [&](int s, auto part) {                                        // 32 bytes of K
        constexpr int q = decltype(part)::value, h = q & 1;
        const uint4 *st = ring[s % ST];
#pragma unroll
        for (int i = 0; i < WN; ++i) wf[h][i] = __builtin_bit_cast(v4i, st[tile_unit<KS>(wn + 32 * i + r, 2 * q + hi)]);
#pragma unroll
        for (int j = 0; j < WM; ++j) xf[h][j] = __builtin_bit_cast(v4i, st[tile_unit<KS>(wm + 32 * j + r, 2 * q + hi)]);
        if (k0 + s * Step + 16 * (2 * q + 1) >= k1) {                               // the last, partial step
            const bool in = k0 + s * Step + 16 * (2 * q + hi) < k1;
#pragma unroll
            for (int i = 0; i < WN; ++i) wf[h][i] = in ? wf[h][i] : v4i{0, 0, 0, 0};
        }
    };
    auto products = [&](auto part) {
        constexpr int h = decltype(part)::value & 1;
#pragma unroll
        for (int i = 0; i < WN; ++i)
#pragma unroll
            for (int j = 0; j < WM; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wf[h][i], xf[h][j], acc[i][j], 0, 0, 0);
    };
    // step s has landed: the loads of the ST - 2 steps behind it may be in flight
    auto landed = [&](int s) {
        if (s + ST - 2 < end) asm volatile("s_waitcnt vmcnt(%0)" :: "n"((ST - 2) * L) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        lds_barrier();
    };
    typedef std::integral_constant<int, 0> First;
    typedef std::integral_constant<int, Q - 1> Last;
    if (end > 0) {
#pragma unroll
        for (int i = 0; i < ST - 1; ++i)
            if (i < end) issue(i);
        landed(0);
        fragments(0, First{});
        for (int s = 0; s < end; ++s) {
            if (s + ST - 1 < end) issue(s + ST - 1);                                // where step s - 1 was, which every wave has read
            fragments(s, std::integral_constant<int, 1>{});
            products(First{});
            if constexpr (KS == 2) {
                fragments(s, std::integral_constant<int, 2>{});
                products(std::integral_constant<int, 1>{});
                fragments(s, Last{});
                products(std::integral_constant<int, 2>{});
            }
            if (s + 1 < end) {
                landed(s + 1);
                fragments(s + 1, First{});
            }
            products(Last{});
        }
    }
    if (a.S > 1) {                                          // in the matrix cores' order
        v4i *to = (v4i *)a.parts + ((int64_t)(blockIdx.y * gridDim.x + blockIdx.x) * W + wave) * (WN * WM * 256) + lane;
#pragma unroll
        for (int i = 0; i < WN; ++i)
#pragma unroll
            for (int j = 0; j < WM; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    to[((i * WM + j) * 4 + q) * 64] = v4i{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        return;
    }
#pragma unroll
    for (int j = 0; j < WM; ++j) {
        const int m = m0 + wm - TN + 32 * j + r;
        if (m >= a.M) continue;
        const float sx = a.x_scale[m];
#pragma unroll
        for (int i = 0; i < WN; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                store4(a, m, n0 + wn + 32 * i + 8 * q + 4 * hi, sx, v4i{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]});
    }
}

// A wave a 32 x 32 product's quarter (1 KiB of each range's sums), four channels of a token a lane.
template <int WN, int WM, int GN, int GM>
__global__ __launch_bounds__(256) void k_i8_tile_join(I8Args a) {
    constexpr int W = GN * GM, P = W * WN * WM * 4;         // quarters of a tile
    const int lane = threadIdx.x & 63, at = blockIdx.x * 4 + (threadIdx.x >> 6);
    const int tile = at / P, p = at - tile * P, wave = p / (WN * WM * 4), ij = p / 4 % (WN * WM), q = p & 3;
    int tm, tn;
    tile_of(a, tile, tm, tn);
    const int n = tn * (32 * WN * GN) + 32 * WN * (wave % GN) + 32 * (ij / WM) + 8 * q + 4 * (lane >> 5);
    const int m = tm * (32 * WM * GM) + 32 * WM * (wave / GN) + 32 * (ij % WM) + (lane & 31);
    if (m >= a.M || n >= a.N) return;
    const v4i *from = (const v4i *)a.parts + (int64_t)at * 64 + lane;
    const int64_t range = (int64_t)a.tiles_m * a.tiles_n * P * 64;
    v4i sum = from[0];
    for (int s = 1; s < a.S; ++s) sum += from[s * range];
    store4(a, m, n, a.x_scale[m], sum);
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

template <int WN, int WM, int GN, int GM, int KS, int ST, int PER_CU>
hipError_t launch_tile(const I8Args &a, hipStream_t st) {
    const unsigned tiles = (unsigned)(a.tiles_m * a.tiles_n);
    hipLaunchKernelGGL((k_i8_tile<WN, WM, GN, GM, KS, ST, PER_CU>), dim3(tiles, a.S), dim3(GN * GM * 64), 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.S == 1) return e;
    hipLaunchKernelGGL((k_i8_tile_join<WN, WM, GN, GM>), dim3(tiles * (GN * GM * WN * WM)), dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_i8_linear(const I8Args &a, hipStream_t st) {
    switch (a.form) {
    case 1: return launch_tile<2, 1, 2, 2, 2, 3, 2>(a, st);
    case 2: return launch_tile<2, 2, 2, 2, 1, 4, 2>(a, st);
    case 3: return launch_tile<2, 2, 4, 2, 1, 3, 2>(a, st);
    case 4: return launch_tile<4, 2, 2, 4, 2, 2, 1>(a, st);
    case 5: return launch_tile<5, 2, 2, 4, 2, 2, 1>(a, st);
    }
    const int per_wave = (a.steps + kFewWaves - 1) / kFewWaves;
    if (a.M <= 16) launch_few<1>(a, per_wave, st);
    else if (a.M <= 32) launch_few<2>(a, per_wave, st);
    else launch_few<4>(a, per_wave, st);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.S == 1) return e;
    const int64_t blocks = ((int64_t)a.M * a.N + 255) / 256;
    hipLaunchKernelGGL(k_i8_join, dim3((unsigned)(blocks < 16384 ? blocks : 16384)), dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace qlin
