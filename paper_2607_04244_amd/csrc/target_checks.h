// Argument checks that the C ABIs of the target's operators share (target_abi.cpp,
// lowbit_abi.cpp): address ranges, batches, caches and row arrays.
#pragma once

#include "../../include/qlin_target.h"

#include <hip/hip_runtime.h>

#include <atomic>
#include <climits>
#include <cmath>

#include "qlin_internal.h"
#include "target_internal.h"

namespace qlin {

constexpr int64_t kMaxSeq = 65536, kMaxRows = (int64_t)1 << 22, kMaxLen = (int64_t)1 << 28, kMaxSlots = (int64_t)1 << 40;
constexpr int64_t kMaxHeads = 4096, kMaxGroup = 64, kMaxSplits = 256, kMaxStride = (int64_t)1 << 40;
constexpr int64_t kMaxTokenStride = (int64_t)1 << 28;       // 32-bit byte offsets over four tokens
constexpr int64_t kMaxRowStride = (int64_t)1 << 32;
constexpr int64_t kMaxExtent = (int64_t)1 << 60;      // elements of one strided array

// An address range, in bytes.
struct Range { uintptr_t lo; size_t bytes; };

inline bool overlap(const Range &a, const Range &b) { return a.bytes && b.bytes && a.lo < b.lo + b.bytes && b.lo < a.lo + a.bytes; }

inline Range rows_range(const void *p, int64_t rows, int64_t stride, int64_t width) {
    return Range{(uintptr_t)p, rows > 0 ? (size_t)((rows - 1) * stride + width) * 2 : 0};
}

// Whether two arrays of rows share an element.  Slices of the rows of one array do not, though
// their ranges overlap.
inline bool rows_meet(const void *p, int64_t stride, int64_t width, const void *q, int64_t q_stride, int64_t q_width, int64_t rows) {
    if (!overlap(rows_range(p, rows, stride, width), rows_range(q, rows, q_stride, q_width))) return false;
    if (stride != q_stride) return true;
    const int64_t d = ((int64_t)((uintptr_t)q - (uintptr_t)p) / 2 % stride + stride) % stride;   // 16-byte aligned both
    return d < width || d + q_width > stride;
}

inline Range cache_range(const void *p, const qlin_kv_cache *c) {
    return Range{(uintptr_t)p, (size_t)((c->slots - 1) * c->token_stride + (c->heads - 1) * c->head_stride + kHeadDim) * 2};
}

inline bool aligned(const void *p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

inline int check_batch(const qlin_batch *b) {
    if (!b) return fail(QLIN_ERR_INVALID, "NULL batch");
    if (b->n_seq < 1 || b->rows < 0 || b->max_new < 0 || b->max_new > b->rows || b->max_len < 0)
        return fail(QLIN_ERR_INVALID, "n_seq must be positive, rows >= 0, max_new in [0, rows], max_len >= 0");
    if (b->n_seq > kMaxSeq || b->rows > kMaxRows || b->max_len > kMaxLen)
        return fail(QLIN_ERR_UNSUPPORTED, "at most 65536 sequences, 2^22 rows and 2^28 cached tokens");
    return QLIN_OK;
}

inline int check_batch_arrays(const qlin_batch *b) {
    if (!b->new_start || !b->length) return fail(QLIN_ERR_INVALID, "NULL new_start or length");
    if (!aligned(b->new_start, 4) || !aligned(b->length, 4) || !aligned(b->cache_start, 8))
        return fail(QLIN_ERR_ALIGN, "new_start and length must be 4-byte aligned, cache_start 8");
    return QLIN_OK;
}

inline int check_heads(int64_t q_heads, int64_t kv_heads, int64_t head_dim) {
    if (q_heads <= 0 || kv_heads <= 0 || q_heads % kv_heads)
        return fail(QLIN_ERR_INVALID, "query and key/value heads must be positive, the first a multiple of the second");
    if (head_dim != kHeadDim) return fail(QLIN_ERR_UNSUPPORTED, "head_dim must be 128 (got %lld)", (long long)head_dim);
    if (q_heads > kMaxHeads) return fail(QLIN_ERR_UNSUPPORTED, "at most 4096 query heads");
    if (q_heads / kv_heads > kMaxGroup) return fail(QLIN_ERR_UNSUPPORTED, "at most 64 query heads per key/value head");
    return QLIN_OK;
}

inline int check_cache(const qlin_kv_cache *c) {
    if (!c) return fail(QLIN_ERR_INVALID, "NULL cache");
    if (c->slots < 1 || c->seq_slots < 0 || c->capacity < 0 || c->token_stride < kHeadDim || c->head_stride < kHeadDim)
        return fail(QLIN_ERR_INVALID, "cache: slots must be positive, seq_slots and capacity >= 0, strides >= 128");
    if (c->token_stride % 8 || c->head_stride % 8) return fail(QLIN_ERR_ALIGN, "cache strides must be multiples of 8");
    if (c->slots > kMaxSlots || c->seq_slots > kMaxSlots || c->capacity > kMaxSlots || c->token_stride > kMaxTokenStride || c->head_stride > kMaxStride ||
        (double)c->slots * (double)c->token_stride + (double)c->heads * (double)c->head_stride > (double)kMaxExtent)
        return fail(QLIN_ERR_UNSUPPORTED, "cache too large");
    if (!c->k || !c->v) return fail(QLIN_ERR_INVALID, "NULL cache");
    if (!aligned(c->k, 16) || !aligned(c->v, 16)) return fail(QLIN_ERR_ALIGN, "the cache must be 16-byte aligned");
    return QLIN_OK;
}

// Whether the arrays that describe a batch share an element with a range.
inline bool batch_meets(const qlin_batch *b, const Range &r) {
    const size_t n = (size_t)b->n_seq;
    return overlap(r, Range{(uintptr_t)b->new_start, (n + 1) * 4}) || overlap(r, Range{(uintptr_t)b->length, n * 4}) ||
           overlap(r, Range{(uintptr_t)b->cache_start, b->cache_start ? n * 8 : 0});
}

// Row arrays of `width` elements: stride and alignment.
inline int check_rows(const void *p, int64_t stride, int64_t width, const char *name) {
    if (!p) return fail(QLIN_ERR_INVALID, "NULL %s", name);
    if (stride < width || stride > kMaxRowStride) return fail(QLIN_ERR_INVALID, "%s: stride must be at least %lld", name, (long long)width);
    if (stride % 8 || !aligned(p, 16)) return fail(QLIN_ERR_ALIGN, "%s must be 16-byte aligned, its stride a multiple of 8", name);
    return QLIN_OK;
}

inline BatchArgs batch_args(const qlin_batch *b, const qlin_kv_cache *c) {
    BatchArgs a;
    a.new_start = b->new_start;
    a.length = b->length;
    a.cache_start = b->cache_start;
    a.slots = c->slots;
    a.seq_slots = c->seq_slots;
    a.capacity = c->capacity;
    a.tok = c->token_stride;
    a.head = c->head_stride;
    a.n_seq = (int)b->n_seq;
    a.rows = (int)b->rows;
    a.max_new = (int)b->max_new;
    a.longest = INT_MAX;
    return a;
}

// What the appends take beside batch and cache.
struct AppendRows {
    const uint16_t *q;
    int64_t q_stride;
    const uint16_t *k;
    int64_t k_stride;
    const uint16_t *v;
    int64_t v_stride;
    const uint16_t *q_norm, *k_norm;
    float eps;
    const double *inv_freq;
    int64_t rotary_dim;
    uint16_t *q_out;
    int64_t q_out_stride;
};

inline int check_append_values(const AppendRows &r) {
    if (r.rotary_dim < 0 || r.rotary_dim > kHeadDim || r.rotary_dim % 16)
        return fail(QLIN_ERR_INVALID, "rotary_dim must be a multiple of 16 in [0, 128]");
    if (!(r.eps >= 0.0f) || std::isinf(r.eps)) return fail(QLIN_ERR_INVALID, "eps must be >= 0");
    return QLIN_OK;
}

// `cache`: the n address ranges of its arrays.
inline int check_append_arrays(const qlin_batch *batch, int64_t q_heads, int64_t heads, const AppendRows &r, const Range *cache, int n) {
    if (check_batch_arrays(batch) != QLIN_OK) return last_status();
    const int64_t wq = q_heads * kHeadDim, wk = heads * kHeadDim, M = batch->rows;
    if (check_rows(r.q, r.q_stride, wq, "q") != QLIN_OK || check_rows(r.k, r.k_stride, wk, "k") != QLIN_OK ||
        check_rows(r.v, r.v_stride, wk, "v") != QLIN_OK || check_rows(r.q_out, r.q_out_stride, wq, "q_out") != QLIN_OK)
        return last_status();
    if (r.rotary_dim && !r.inv_freq) return fail(QLIN_ERR_INVALID, "NULL inv_freq");
    if (!aligned(r.q_norm, 8) || !aligned(r.k_norm, 8) || !aligned(r.inv_freq, 8))
        return fail(QLIN_ERR_ALIGN, "norm weights and inv_freq must be 8-byte aligned");
    const Range in[] = {rows_range(r.q, M, r.q_stride, wq), rows_range(r.k, M, r.k_stride, wk), rows_range(r.v, M, r.v_stride, wk)};
    const Range ro = rows_range(r.q_out, M, r.q_out_stride, wq);
    if (!(r.q_out == r.q && r.q_out_stride == r.q_stride) && rows_meet(r.q, r.q_stride, wq, r.q_out, r.q_out_stride, wq, M))
        return fail(QLIN_ERR_INVALID, "q_out overlaps q without being it");
    if (rows_meet(r.k, r.k_stride, wk, r.q_out, r.q_out_stride, wq, M) || rows_meet(r.v, r.v_stride, wk, r.q_out, r.q_out_stride, wq, M))
        return fail(QLIN_ERR_INVALID, "q_out overlaps k or v");
    for (int i = 0; i < n; ++i) {
        if (overlap(ro, cache[i])) return fail(QLIN_ERR_INVALID, "q_out overlaps the cache");
        for (const Range &x : in)
            if (overlap(x, cache[i])) return fail(QLIN_ERR_INVALID, "q, k or v overlaps the cache");
    }
    const Range small[] = {{(uintptr_t)r.q_norm, r.q_norm ? (size_t)kHeadDim * 2 : 0}, {(uintptr_t)r.k_norm, r.k_norm ? (size_t)kHeadDim * 2 : 0},
                           {(uintptr_t)r.inv_freq, (size_t)r.rotary_dim / 2 * 8}};
    for (int i = -1; i < n; ++i) {
        const Range &w = i < 0 ? ro : cache[i];
        if (batch_meets(batch, w)) return fail(QLIN_ERR_INVALID, "q_out or the cache overlaps new_start, length or cache_start");
        for (const Range &x : small)
            if (overlap(w, x)) return fail(QLIN_ERR_INVALID, "q_out or the cache overlaps norm weights or inv_freq");
    }
    return QLIN_OK;
}

// All but the cache's arrays.
inline AppendArgs append_args(const BatchArgs &b, int64_t q_heads, int64_t heads, const AppendRows &r, int interleaved) {
    AppendArgs a;
    a.b = b;
    a.q = r.q;
    a.k = r.k;
    a.v = r.v;
    a.q_norm = r.q_norm;
    a.k_norm = r.k_norm;
    a.inv_freq = r.inv_freq;
    a.q_out = r.q_out;
    a.q_stride = r.q_stride;
    a.k_stride = r.k_stride;
    a.v_stride = r.v_stride;
    a.q_out_stride = r.q_out_stride;
    a.eps = r.eps;
    a.Hq = (int)q_heads;
    a.Hkv = (int)heads;
    a.half = (int)r.rotary_dim / 2;
    a.interleaved = interleaved != 0;
    return a;
}

// factor: scores to base-2 exponents
inline int check_attention_values(float scale, int64_t splits, int64_t workspace_bytes, float *factor) {
    if (splits < 0 || splits > kMaxSplits) return fail(QLIN_ERR_INVALID, "splits must be in [0, 256]");
    *factor = (float)(1.4426950408889634 * (scale > 0.0f ? (double)scale : 1.0 / std::sqrt((double)kHeadDim)));
    if (!(scale >= 0.0f) || std::isinf(*factor)) return fail(QLIN_ERR_INVALID, "scale must be positive (or 0), scale log2(e) a finite float");
    if (workspace_bytes < 0) return fail(QLIN_ERR_INVALID, "workspace_bytes must be >= 0");
    return QLIN_OK;
}

// Compute units of the current device.
inline int compute_units(int64_t *cus) {
    constexpr int kDevices = 64;
    static std::atomic<int> known[kDevices];
    int dev = 0, n = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e == hipSuccess && dev >= 0 && dev < kDevices) n = known[dev].load(std::memory_order_relaxed);
    if (e == hipSuccess && n == 0) {
        e = hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev);
        if (e == hipSuccess && dev >= 0 && dev < kDevices) known[dev].store(n, std::memory_order_relaxed);
    }
    if (e != hipSuccess) return hip_fail(e, "device query");
    *cus = n;
    return QLIN_OK;
}

// qlin_causal_attention of long chunks over a cache in f16 with `shifts` (CausalArgs), after its
// checks, in a workspace of its size (target_abi.cpp).
int attend_in_f16(const qlin_batch *batch, const qlin_kv_cache *cache, const HeadShift *shifts, const short2 *row_shifts,
                  int64_t q_heads, float factor, int64_t splits, const uint16_t *q, int64_t q_stride, uint16_t *out,
                  int64_t out_stride, void *workspace, hipStream_t stream);

}  // namespace qlin
