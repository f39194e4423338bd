// Internal interface between the C-ABI host code of the layer's operators in fewer bits
// (lowbit_abi.cpp) and their HIP kernels (norm.hip, linear8.hip, append.hip, kv4.hip).
// Not installed; the public ABI is include/qlin_lowbit.h.
#pragma once

#include "target_internal.h"

namespace qlin {

struct BlockNormArgs {
    const uint16_t *y, *residual, *post, *gate, *pre;
    uint16_t *residual_out, *out;
    int64_t y_stride, residual_stride, gate_stride, residual_out_stride, out_stride;
    int rows, width, sigmoid;
    float scale, eps;
};

struct QuantizeArgs {
    const uint16_t *x;
    int8_t *codes;
    float *scale;
    int64_t x_stride, codes_stride;
    int rows, width, gated;
};

// The linear of 8-bit integers.
struct I8Args {
    const int8_t *x, *w;
    const float *x_scale, *w_scale;
    uint16_t *y;
    int32_t *parts;                 // S > 1: the ranges' sums, [S][M][N], or of tiles in the matrix cores' order
    int64_t x_stride, w_stride, y_stride;
    int M, N, K;
    int S, steps;                   // K ranges; steps of one (64 bytes)
    int tiles_m, tiles_n;
    int form;                       // of kI8Forms
};
// Form 0 is k_i8_few, up to kI8FewRows rows; the others k_i8_tile: channels and rows of a tile,
// workgroups of a compute unit.
struct I8Form { int n, m, per_cu; };
constexpr I8Form kI8Forms[] = {{16, 64, 2}, {128, 64, 2}, {128, 128, 2}, {256, 128, 2}, {256, 256, 1}, {320, 256, 1}};
constexpr int kI8FormCount = sizeof kI8Forms / sizeof *kI8Forms;
constexpr int kI8FewRows = 64, kI8Step = 64, kI8FewWaves = 8;
// Steps of the tokens that a wave of k_i8_few holds in registers, for M rows.
constexpr int i8_few_steps(int M) { return M <= 16 ? 19 : M <= 32 ? 8 : 5; }

// The 4-bit cache's arrays beside BatchArgs, whose tok and head are rows here.
struct Kv4Arrays {
    uint32_t *k, *v;                // 16 words a row
    uint32_t *k_grid, *v_grid;      // (step, offset) a row
};

struct AppendKv4Args {
    AppendArgs a;                   // a.kc and a.vc unused
    Kv4Arrays c;
    uint32_t inv_q, inv_kv;         // ceil(2^32 / heads), 0: one head (set by the launch)
};

struct UnpackArgs {
    BatchArgs b;                    // of the 4-bit cache
    Kv4Arrays c;
    uint16_t *k, *v;                // bf16; f16 with shifts
    int64_t to_slots, to_seq_slots, to_capacity, to_tok, to_head;
    int heads, new_only;
    int64_t items;                  // (sequence, head, tile of tokens)
    int tiles;
    // For the attention over a workspace: sequence b begins at slot b * to_seq_slots there, and its
    // head's keys and values are f16 times 2^-shift.  Null: the 4-bit cache's slots, bf16.
    HeadShift *shifts;
    short2 *row_shifts;             // [sequence][head][to_capacity], where a head's shift is by_row
    int32_t *length;                // lengths, 0 where a sequence counts as one without cached tokens
    float4 *peaks;                  // of each kPeakTokens tokens of a sequence's head: see k_kv4_peaks
    int peak_tiles;
};
constexpr int kUnpackTokens = 64;   // tokens of a tile
constexpr int kPeakTokens = 1024;

struct CausalKv4Args {
    CausalArgs a;                   // a.k and a.v unused; a.b.tok and a.b.head in rows
    Kv4Arrays c;
};
constexpr int kKv4Keys = 64;        // keys of a step

hipError_t launch_block_norm(const BlockNormArgs &a, hipStream_t st);
hipError_t launch_quantize_tokens(const QuantizeArgs &a, hipStream_t st);
hipError_t launch_i8_linear(const I8Args &a, hipStream_t st);
hipError_t launch_append_kv4(const AppendKv4Args &a, hipStream_t st);
hipError_t launch_unpack_kv4(const UnpackArgs &a, hipStream_t st);
hipError_t launch_causal_kv4(const CausalKv4Args &a, int rt, hipStream_t st);
const char *causal_kv4_kernel_name(int rt);

}  // namespace qlin
