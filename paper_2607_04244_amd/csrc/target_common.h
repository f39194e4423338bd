// Device-side helpers shared by the target's kernels: a sequence's rows and slots, with
// every bound clamped, and arithmetic of rows.  Header-only, inline.
#pragma once

#include "device_common.h"
#include "target_internal.h"

namespace qlin {

// Sequence b: its rows [row0, row0 + n), of which the first `rows` are computed, its
// cached tokens L and the slot of token 0.  Whatever the arrays hold, rows stay in
// [0, a.rows), and L is 0 unless slots [slot0, slot0 + L) are inside the cache and, with a
// capacity, inside one sequence's room.
struct Seq {
    int row0, n, rows, p0, L;
    int64_t slot0;
};

__device__ inline Seq load_seq(const BatchArgs &a, int b) {
    Seq s;
    s.row0 = min(max(a.new_start[b], 0), a.rows);
    s.n = min(max(a.new_start[b + 1], s.row0), a.rows) - s.row0;
    s.rows = min(s.n, a.max_new);
    const int L = max(a.length[b], 0);
    s.p0 = L - s.n;                         // position of its first new token
    s.slot0 = a.cache_start ? a.cache_start[b] : (int64_t)b * a.seq_slots;
    int64_t room = a.capacity ? a.capacity : a.slots;
    if (a.capacity && a.cache_start && a.seq_slots) room -= s.slot0 % a.seq_slots;
    s.L = s.slot0 >= 0 && s.slot0 <= a.slots - L && L <= room && L <= a.longest ? L : 0;
    return s;
}

// Value of lane l, the same in every lane.
__device__ inline int lane_value(int v, int l) { return __builtin_amdgcn_readlane(v, l); }
__device__ inline int64_t lane_value(int64_t v, int l) {
    const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)v, l), hi = __builtin_amdgcn_readlane((uint32_t)(v >> 32), l);
    return (int64_t)((uint64_t)hi << 32 | lo);
}
__device__ inline Seq lane_value(const Seq &s, int l) {
    return Seq{lane_value(s.row0, l), lane_value(s.n, l), lane_value(s.rows, l), lane_value(s.p0, l), lane_value(s.L, l),
               lane_value(s.slot0, l)};
}

// The sequence that row m belongs to (n_seq: padding), by the whole wave: the
// number of sequences that end at or before m.
__device__ inline int find_seq(const BatchArgs &a, int m, int lane) {
    int b = 0;
    for (int i = 0; i < a.n_seq; i += 64)
        b += __popcll(__ballot(i + lane < a.n_seq && a.new_start[min(i + lane, a.n_seq - 1) + 1] <= m));
    return b;
}

// Eight values rounded to bf16.
__device__ inline uint4 pack8(const float f[8]) {
    return make_uint4(cvt_pk_bf16(f[0], f[1]), cvt_pk_bf16(f[2], f[3]), cvt_pk_bf16(f[4], f[5]), cvt_pk_bf16(f[6], f[7]));
}

// A quotient of fp32 numbers, correctly rounded, from the divisor's correctly rounded
// reciprocal (Markstein): the remainder of the first quotient is exact in a fused product.
__device__ inline float quotient(float x, float d, float inv) {
    const float q = x * inv;
    return __builtin_fmaf(__builtin_fmaf(-q, d, x), inv, q);
}

}  // namespace qlin
