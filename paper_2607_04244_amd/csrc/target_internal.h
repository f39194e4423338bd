// Internal interface between the C-ABI host code of the target's operators
// (target_abi.cpp) and their HIP kernels (append.hip, causal.hip, verify.hip).
// Not installed; the public ABI is include/qlin_target.h.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace qlin {

constexpr int kHeadDim = 128;

// The batch and the cache as the kernels take them (include/qlin_target.h).
struct BatchArgs {
    const int32_t *new_start, *length;
    const int64_t *cache_start;     // or null: b * seq_slots
    int64_t slots, seq_slots, capacity;
    int64_t tok, head;              // elements between slots, between heads
    int n_seq, rows, max_new;
    int longest;                    // a longer sequence counts as one without cached tokens
};

struct AppendArgs {
    BatchArgs b;
    const uint16_t *q, *k, *v;
    const uint16_t *q_norm, *k_norm;
    const double *inv_freq;
    uint16_t *q_out, *kc, *vc;
    int64_t q_stride, k_stride, v_stride, q_out_stride;
    float eps;
    int Hq, Hkv, half, interleaved;
};

struct HeadShift { short k, v; int by_row; };

struct CausalArgs {
    BatchArgs b;
    const uint16_t *q, *k, *v;
    uint16_t *out;
    int64_t q_stride, out_stride;
    int Hq, Hkv, G;
    float *ws_o, *ws_ml;            // S > 1: sums and (maximum, sum of weights) of each item, range and row
    int tiles;                      // row tiles, at least those there are
    int one_tile;                   // this many tiles a sequence (1: tile i is sequence i); 0: as many as its rows need
    int pairs;                      // at most two workgroups a compute unit
    int S, least;                   // key ranges; least steps of one
    int step_shift;                 // a step has 2^step_shift keys (set by the launch)
    int max_len;                    // bound of the sequences' lengths (orders the tiles)
    uint32_t inv_heads, inv_g;      // x / Hkv by gn_chunk; ceil(2^32 / G) (0: G = 1)
    int heads_shift;
    float c;                        // scale log2(e): scores to base-2 exponents
    const HeadShift *shifts;        // k and v are f16 times 2^-shift, of each sequence and head; null: bf16
    const short2 *row_shifts;       // where it is by_row: (k's, v's) shift of each sequence, head and token
};

// Rows (tokens x heads of a group) of a tile of k_causal_few (rt = 1), of k_causal_mid (2, 4) or
// of k_causal_prompt (0).
constexpr int causal_tile_rows(int rt) { return rt ? 16 * rt : 128; }

// Verification.  A row of logits is cut into chunks of kVerifyChunk from the 16-byte boundary at
// or before it (up to 7 logits earlier).
constexpr int kVerifyChunk = 4096, kVerifyMaxDraft = 64;
struct VerifyStat { float m; int at; double z; };      // maximum, its lowest index (greedy), sum of the weights
// done: known from the rows looked at; p and q are then the statistics of the row that decides
struct VerifyDecision { int accepted, rejected, done; VerifyStat p, q; };

struct VerifyArgs {
    const uint16_t *target, *draft;
    const int32_t *drafted, *count;
    const float *temperature, *uniform;
    int32_t *accepted, *tokens;
    int64_t target_stride, draft_stride;
    int n, V;
    int chunks, all_rows;           // chunks of a row; rows of a sequence (targets, then drafts)
    VerifyStat *stats;              // [sequence][all_rows][chunks]
    double *sums;                   // [sequence][chunks]
    VerifyDecision *decisions, *final_decisions;   // [sequence] from the first rows (if first_rows), from all
    int first_rows;                 // rows whose statistics come first, 0: all together
    int row0, row1;                 // rows of this launch of k_verify_stats
};

hipError_t launch_append(const AppendArgs &a, hipStream_t st);
hipError_t launch_causal(const CausalArgs &a, int rt, int halves, hipStream_t st);
hipError_t launch_kv4_join(const CausalArgs &a, int rt, hipStream_t st);      // rt 1, 2
const char *causal_kernel_name(int rt, int halves);
hipError_t launch_verify(VerifyArgs a, int n_seq, bool many, hipStream_t st);

}  // namespace qlin
