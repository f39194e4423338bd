// C ABI of the target's operators (include/qlin_target.h): argument checks,
// plans and launches.

#include "../../include/qlin_target.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdio>
#include <cstring>

#include "qlin_internal.h"
#include "target_internal.h"

using namespace qlin;

namespace {

constexpr int64_t kMaxSeq = 65536, kMaxRows = (int64_t)1 << 22, kMaxLen = (int64_t)1 << 28, kMaxSlots = (int64_t)1 << 40;
constexpr int64_t kMaxHeads = 4096, kMaxGroup = 64, kMaxSplits = 256, kMaxStride = (int64_t)1 << 40;
constexpr int64_t kMaxDraft = kVerifyMaxDraft, kMaxVocab = (int64_t)1 << 24, kMaxVerifySeq = 65535;   // sequences: a grid's y
constexpr int64_t kMaxTokenStride = (int64_t)1 << 28;       // 32-bit byte offsets over four tokens
constexpr int64_t kMaxRowStride = (int64_t)1 << 32;
constexpr int64_t kVerifyTwoParts = (int64_t)1 << 26, kVerifyMany = (int64_t)1 << 25;     // logits of a call: see qlin_verify_draft
constexpr int64_t kMaxExtent = (int64_t)1 << 60;      // elements of one strided array

// An address range, in bytes.
struct Range { uintptr_t lo; size_t bytes; };

bool overlap(const Range &a, const Range &b) { return a.bytes && b.bytes && a.lo < b.lo + b.bytes && b.lo < a.lo + a.bytes; }

Range rows_range(const void *p, int64_t rows, int64_t stride, int64_t width) {
    return Range{(uintptr_t)p, rows > 0 ? (size_t)((rows - 1) * stride + width) * 2 : 0};
}

// Whether two arrays of rows share an element.  Slices of the rows of one array do not, though
// their ranges overlap.
bool rows_meet(const void *p, int64_t stride, int64_t width, const void *q, int64_t q_stride, int64_t q_width, int64_t rows) {
    if (!overlap(rows_range(p, rows, stride, width), rows_range(q, rows, q_stride, q_width))) return false;
    if (stride != q_stride) return true;
    const int64_t d = ((int64_t)((uintptr_t)q - (uintptr_t)p) / 2 % stride + stride) % stride;   // 16-byte aligned both
    return d < width || d + q_width > stride;
}

Range cache_range(const void *p, const qlin_kv_cache *c) {
    return Range{(uintptr_t)p, (size_t)((c->slots - 1) * c->token_stride + (c->heads - 1) * c->head_stride + kHeadDim) * 2};
}

bool aligned(const void *p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

int check_batch(const qlin_batch *b) {
    if (!b) return fail(QLIN_ERR_INVALID, "NULL batch");
    if (b->n_seq < 1 || b->rows < 0 || b->max_new < 0 || b->max_new > b->rows || b->max_len < 0)
        return fail(QLIN_ERR_INVALID, "n_seq must be positive, rows >= 0, max_new in [0, rows], max_len >= 0");
    if (b->n_seq > kMaxSeq || b->rows > kMaxRows || b->max_len > kMaxLen)
        return fail(QLIN_ERR_UNSUPPORTED, "at most 65536 sequences, 2^22 rows and 2^28 cached tokens");
    return QLIN_OK;
}

int check_batch_arrays(const qlin_batch *b) {
    if (!b->new_start || !b->length) return fail(QLIN_ERR_INVALID, "NULL new_start or length");
    if (!aligned(b->new_start, 4) || !aligned(b->length, 4) || !aligned(b->cache_start, 8))
        return fail(QLIN_ERR_ALIGN, "new_start and length must be 4-byte aligned, cache_start 8");
    return QLIN_OK;
}

int check_heads(int64_t q_heads, int64_t kv_heads, int64_t head_dim) {
    if (q_heads <= 0 || kv_heads <= 0 || q_heads % kv_heads)
        return fail(QLIN_ERR_INVALID, "query and key/value heads must be positive, the first a multiple of the second");
    if (head_dim != kHeadDim) return fail(QLIN_ERR_UNSUPPORTED, "head_dim must be 128 (got %lld)", (long long)head_dim);
    if (q_heads > kMaxHeads) return fail(QLIN_ERR_UNSUPPORTED, "at most 4096 query heads");
    if (q_heads / kv_heads > kMaxGroup) return fail(QLIN_ERR_UNSUPPORTED, "at most 64 query heads per key/value head");
    return QLIN_OK;
}

int check_cache(const qlin_kv_cache *c) {
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
bool batch_meets(const qlin_batch *b, const Range &r) {
    const size_t n = (size_t)b->n_seq;
    return overlap(r, Range{(uintptr_t)b->new_start, (n + 1) * 4}) || overlap(r, Range{(uintptr_t)b->length, n * 4}) ||
           overlap(r, Range{(uintptr_t)b->cache_start, b->cache_start ? n * 8 : 0});
}

// Row arrays of `width` elements: stride and alignment.
int check_rows(const void *p, int64_t stride, int64_t width, const char *name) {
    if (!p) return fail(QLIN_ERR_INVALID, "NULL %s", name);
    if (stride < width || stride > kMaxRowStride) return fail(QLIN_ERR_INVALID, "%s: stride must be at least %lld", name, (long long)width);
    if (stride % 8 || !aligned(p, 16)) return fail(QLIN_ERR_ALIGN, "%s must be 16-byte aligned, its stride a multiple of 8", name);
    return QLIN_OK;
}

BatchArgs batch_args(const qlin_batch *b, const qlin_kv_cache *c) {
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
    return a;
}

// The kernel and split of one causal attention, from the host's bounds.
struct CausalPlan { int rt = 0, halves = 1, tiles = 0, one_tile = 0, pairs = 0, S = 1, least = 1; int64_t ws_bytes = 0; };

// Estimated microseconds of a call whose `blocks` (tile, head) items walk L keys in S ranges, in
// k_causal_prompt by workgroups of one or two `halves`.  Fitted to graph replays of 32 / 8 heads.
// A workgroup has some time without keys and then takes a key (of 4 rows or of 128) in, for few
// rows, 0.026 us (every compute unit reads the cache); for prompts, alone on its compute unit,
// 0.017 us as one half and 0.0125 as two, and 0.004 more where all units work (their clock
// falls); of two on a unit 0.033.  More workgroups than run at once keep the units busy up to a
// part of the last one's time: a half for few rows, whose sequences come in any order, less for
// prompts, whose longest tiles come first, and least where two share a unit (the last ones have
// it alone).  Where one sequence may be much longer than the others (`ragged`) two halves of all
// its keys end late.
//
// Measured (halves/ranges: us).  64 sequences of 130 to 8190 keys, few rows: 1 range 187, 2 179,
// 4 177, 6 188; one token over 8191 keys: 16 ranges 11.9, 32 10.2, 64 over 13.  500 tokens behind
// 7400, 128 items: 1/1 154, 1/2 91, 1/3 86, 1/4 79, 1/6 92, 2/1 111, 2/2 79, 2/4 85; 200 behind
// 1800, 56 items: 1/2 27.9, 1/4 20.9, 2/2 26.4, 2/4 22.1; prompts of 512: 1/1 16.1, 2/1 16.7; 1185:
// 1/2 35.0, 2/1 26.8; 1500: 1/1 39.7, 1/2 44.2, 2/1 33.9; 4000: 1/1 136, 2/1 151; 56 new tokens of
// 7940 and 1649 of 2412: 1/3 76, 2/1 118.  Over 360 random batches the choice of halves takes the
// 71 calls that it makes faster to 0.88 of their time; 14 are slower, the worst 1.16.
double causal_cost(int rt, int halves, double ragged, double blocks, double L, double S, double cus) {
    const double W = blocks * S, slots = rt || halves == 2 ? cus : 2 * cus, busy = std::min(W / cus, 1.0);
    const double key = rt ? 0.026 : halves == 2 ? 0.0125 + 0.0043 * busy : W <= cus ? 0.017 + 0.004 * busy : 0.033;
    const double one = L / S * key + (rt ? 4.0 : halves == 2 ? 8.3 : W <= cus ? 5.4 : 8.0);
    const double join = S > 1 ? 3.0 + W * causal_tile_rows(rt) * (kHeadDim + 2) * 4 / 8e6 : 0.0;
    return join + (halves == 2 ? ragged * one : 0.0) + (W <= slots ? one : W * one / slots + (rt ? 0.5 : 0.1 * halves) * one);
}

// What a plan depends on; compared bit by bit.
struct CausalKey { int64_t n_seq, rows, max_new, max_len, Hq, Hkv, splits, cus; };

int make_causal_plan(const CausalKey &k, CausalPlan *p) {
    const CausalKey *const b = &k;
    const int64_t Hq = k.Hq, Hkv = k.Hkv, splits = k.splits, cus = k.cus;
    const int64_t G = Hq / Hkv, most = b->max_new * G;
    p->rt = most <= 16 ? 1 : most <= 32 ? 2 : most <= 64 ? 4 : 0;
    const int64_t R = causal_tile_rows(p->rt), per = (most + R - 1) / R;
    p->one_tile = per <= 1;
    const int64_t tiles = p->one_tile ? b->n_seq : std::min(b->n_seq * per, b->rows * G / R + b->n_seq);
    const int64_t blocks = std::max<int64_t>(tiles * Hkv, 1);
    const int64_t least = p->rt ? 128 : 256;     // keys of a range: a step of each wave, eight of a prompt
    int64_t S = std::max<int64_t>(splits, 1);
    // of several sequences behind cached tokens, maybe a few only have the most keys
    const double ragged = b->n_seq > 1 && b->max_len > b->max_new ? 0.07 * (double)(b->max_len - b->max_new) / (double)b->max_len : 0.0;
    auto cost = [&](int halves, int64_t s) {
        return causal_cost(p->rt, halves, ragged, (double)blocks, (double)b->max_len, (double)s, (double)cus);
    };
    double best = cost(1, S);
    for (int halves = 1; halves <= (p->rt ? 1 : 2); ++halves) {
        auto consider = [&](int64_t ranges) {
            const double t = cost(halves, ranges);
            if (t >= best) return;
            best = t;
            S = ranges;
            p->halves = halves;
        };
        const int64_t most_S = std::min<int64_t>((b->max_len + halves * least - 1) / (halves * least), kMaxSplits);
        if (splits) consider(splits);
        else
            for (const int64_t s : {(int64_t)1, (int64_t)2, (int64_t)3, (int64_t)4, (int64_t)6, (int64_t)8, cus / blocks, 2 * cus / blocks})
                if (s >= 1 && s <= most_S) consider(s);
    }
    // work items of up to 512 threads in a 32-bit grid, also those that join the ranges
    if (tiles * Hkv * std::max(S, S > 1 ? R / 2 : 0) >= (int64_t)1 << 23)
        return fail(QLIN_ERR_UNSUPPORTED, "too many rows, heads and key ranges for one call");
    p->tiles = (int)tiles;
    p->S = (int)S;
    p->pairs = p->halves == 1 && blocks * S <= 2 * cus;
    // ranges that only balance sequences of different lengths leave the short ones whole
    const int64_t keys = splits == 0 && p->halves == 1 && blocks * S > (p->rt ? cus : 2 * cus) ? 4 * 128 : p->halves * least;
    p->least = (int)(keys / (p->rt == 0 ? 32 : p->rt == 1 ? 32 : 128));
    p->ws_bytes = S > 1 ? tiles * Hkv * S * R * (kHeadDim + 2) * 4 : 0;
    return QLIN_OK;
}

// Compute units of the current device.
int compute_units(int64_t *cus) {
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

// The plan of a call.  Each thread remembers 64, directly mapped: the layers of a model ask for
// the same one, and weighing the choices takes longer than all the checks.
int causal_plan(const qlin_batch *b, int64_t Hq, int64_t Hkv, int64_t splits, CausalPlan *p) {
    CausalKey k{b->n_seq, b->rows, b->max_new, b->max_len, Hq, Hkv, splits, 256};   // forced ranges: arithmetic
    if (splits == 0 && compute_units(&k.cus) != QLIN_OK) return last_status();
    struct Entry { CausalKey key; CausalPlan plan; bool used; };
    static thread_local Entry memory[64];
    uint64_t words[sizeof k / 8], h = 0;
    memcpy(words, &k, sizeof k);
    for (const uint64_t w : words) h = (h ^ w) * 0x9E3779B97F4A7C15ull;
    Entry &e = memory[h >> 58];
    if (!e.used || memcmp(&e.key, &k, sizeof k)) {
        CausalPlan made;
        if (make_causal_plan(k, &made) != QLIN_OK) return last_status();
        e = Entry{k, made, true};
    }
    *p = e.plan;
    return QLIN_OK;
}

// Workspace of the verification: the rows' statistics, then the chunks' sums, then the decisions.
struct VerifyLayout { int64_t chunks, rows, sums, decisions, bytes; };

VerifyLayout verify_layout(int64_t n_seq, int64_t n_draft, int64_t vocab) {
    VerifyLayout l;
    l.chunks = (vocab + 7 + kVerifyChunk - 1) / kVerifyChunk;
    l.rows = 2 * n_draft + 1;
    l.sums = n_seq * l.rows * l.chunks * (int64_t)sizeof(VerifyStat);
    l.decisions = l.sums + (n_seq * l.chunks * 8 + 15) / 16 * 16;
    l.bytes = l.decisions + 2 * n_seq * (int64_t)sizeof(VerifyDecision);
    return l;
}

}  // namespace

extern "C" {

int qlin_norm_rope_append(const qlin_batch *batch, const qlin_kv_cache *cache, int64_t q_heads, int64_t head_dim,
                          const uint16_t *q, int64_t q_stride, const uint16_t *k, int64_t k_stride,
                          const uint16_t *v, int64_t v_stride, const uint16_t *q_norm, const uint16_t *k_norm,
                          float eps, const double *inv_freq, int64_t rotary_dim, int interleaved, uint16_t *q_out,
                          int64_t q_out_stride, void *stream) {
    clear_err();
    if (check_batch(batch) != QLIN_OK) return last_status();
    if (!cache) return fail(QLIN_ERR_INVALID, "NULL cache");
    if (check_heads(q_heads, cache->heads, head_dim) != QLIN_OK) return last_status();
    if (check_cache(cache) != QLIN_OK) return last_status();
    if (rotary_dim < 0 || rotary_dim > kHeadDim || rotary_dim % 16)
        return fail(QLIN_ERR_INVALID, "rotary_dim must be a multiple of 16 in [0, 128]");
    if (!(eps >= 0.0f) || std::isinf(eps)) return fail(QLIN_ERR_INVALID, "eps must be >= 0");
    if (batch->rows == 0) return QLIN_OK;
    if (check_batch_arrays(batch) != QLIN_OK) return last_status();
    const int64_t wq = q_heads * kHeadDim, wk = cache->heads * kHeadDim, M = batch->rows;
    if (check_rows(q, q_stride, wq, "q") != QLIN_OK || check_rows(k, k_stride, wk, "k") != QLIN_OK ||
        check_rows(v, v_stride, wk, "v") != QLIN_OK || check_rows(q_out, q_out_stride, wq, "q_out") != QLIN_OK)
        return last_status();
    if (rotary_dim && !inv_freq) return fail(QLIN_ERR_INVALID, "NULL inv_freq");
    if (!aligned(q_norm, 8) || !aligned(k_norm, 8) || !aligned(inv_freq, 8))
        return fail(QLIN_ERR_ALIGN, "norm weights and inv_freq must be 8-byte aligned");
    const Range rq = rows_range(q, M, q_stride, wq), rk = rows_range(k, M, k_stride, wk), rv = rows_range(v, M, v_stride, wk);
    const Range ro = rows_range(q_out, M, q_out_stride, wq), ck = cache_range(cache->k, cache), cv = cache_range(cache->v, cache);
    if (!(q_out == q && q_out_stride == q_stride) && rows_meet(q, q_stride, wq, q_out, q_out_stride, wq, M))
        return fail(QLIN_ERR_INVALID, "q_out overlaps q without being it");
    if (rows_meet(k, k_stride, wk, q_out, q_out_stride, wq, M) || rows_meet(v, v_stride, wk, q_out, q_out_stride, wq, M))
        return fail(QLIN_ERR_INVALID, "q_out overlaps k or v");
    if (overlap(ro, ck) || overlap(ro, cv)) return fail(QLIN_ERR_INVALID, "q_out overlaps the cache");
    for (const Range &r : {rq, rk, rv})
        if (overlap(r, ck) || overlap(r, cv)) return fail(QLIN_ERR_INVALID, "q, k or v overlaps the cache");
    const Range small[] = {{(uintptr_t)q_norm, q_norm ? (size_t)kHeadDim * 2 : 0}, {(uintptr_t)k_norm, k_norm ? (size_t)kHeadDim * 2 : 0},
                           {(uintptr_t)inv_freq, (size_t)rotary_dim / 2 * 8}};
    for (const Range &w : {ro, ck, cv}) {
        if (batch_meets(batch, w)) return fail(QLIN_ERR_INVALID, "q_out or the cache overlaps new_start, length or cache_start");
        for (const Range &r : small)
            if (overlap(w, r)) return fail(QLIN_ERR_INVALID, "q_out or the cache overlaps norm weights or inv_freq");
    }

    AppendArgs a;
    a.b = batch_args(batch, cache);
    a.q = q;
    a.k = k;
    a.v = v;
    a.q_norm = q_norm;
    a.k_norm = k_norm;
    a.inv_freq = inv_freq;
    a.q_out = q_out;
    a.kc = cache->k;
    a.vc = cache->v;
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.q_out_stride = q_out_stride;
    a.eps = eps;
    a.Hq = (int)q_heads;
    a.Hkv = (int)cache->heads;
    a.half = (int)rotary_dim / 2;
    a.interleaved = interleaved != 0;
    const hipError_t e = launch_append(a, (hipStream_t)stream);
    return e == hipSuccess ? QLIN_OK : hip_fail(e, "append launch");
}

int qlin_causal_plan(const qlin_batch *batch, int64_t q_heads, int64_t kv_heads, int64_t head_dim, int64_t splits,
                     int64_t *splits_out, int64_t *workspace_bytes, char *buf, int64_t buflen) {
    clear_err();
    if (check_batch(batch) != QLIN_OK || check_heads(q_heads, kv_heads, head_dim) != QLIN_OK) return last_status();
    if (splits < 0 || splits > kMaxSplits) return fail(QLIN_ERR_INVALID, "splits must be in [0, 256]");
    CausalPlan p;
    if (causal_plan(batch, q_heads, kv_heads, splits, &p) != QLIN_OK) return last_status();
    if (splits_out) *splits_out = p.S;
    if (workspace_bytes) *workspace_bytes = p.ws_bytes;
    if (buf && buflen > 0)
        snprintf(buf, (size_t)buflen, "kernel=%s splits=%d grid=%lld combine=%d", causal_kernel_name(p.rt, p.halves), p.S,
                 (long long)p.tiles * kv_heads * p.S, p.S > 1 ? 1 : 0);
    return QLIN_OK;
}

int qlin_causal_attention(const qlin_batch *batch, const qlin_kv_cache *cache, int64_t q_heads, int64_t head_dim,
                          float scale, int64_t splits, const uint16_t *q, int64_t q_stride, uint16_t *out,
                          int64_t out_stride, void *workspace, int64_t workspace_bytes, void *stream) {
    clear_err();
    if (check_batch(batch) != QLIN_OK) return last_status();
    if (!cache) return fail(QLIN_ERR_INVALID, "NULL cache");
    if (check_heads(q_heads, cache->heads, head_dim) != QLIN_OK) return last_status();
    if (check_cache(cache) != QLIN_OK) return last_status();
    if (splits < 0 || splits > kMaxSplits) return fail(QLIN_ERR_INVALID, "splits must be in [0, 256]");
    // scores to base-2 exponents
    const float factor = (float)(1.4426950408889634 * (scale > 0.0f ? (double)scale : 1.0 / std::sqrt((double)kHeadDim)));
    if (!(scale >= 0.0f) || std::isinf(factor)) return fail(QLIN_ERR_INVALID, "scale must be positive (or 0), scale log2(e) a finite float");
    if (workspace_bytes < 0) return fail(QLIN_ERR_INVALID, "workspace_bytes must be >= 0");
    if (batch->rows == 0) return QLIN_OK;
    if (check_batch_arrays(batch) != QLIN_OK) return last_status();
    const int64_t w = q_heads * kHeadDim, M = batch->rows;
    if (check_rows(q, q_stride, w, "q") != QLIN_OK || check_rows(out, out_stride, w, "out") != QLIN_OK) return last_status();
    if (!aligned(workspace, 16)) return fail(QLIN_ERR_ALIGN, "workspace must be 16-byte aligned");
    const Range ro = rows_range(out, M, out_stride, w);
    if (rows_meet(q, q_stride, w, out, out_stride, w, M) || overlap(ro, cache_range(cache->k, cache)) || overlap(ro, cache_range(cache->v, cache)))
        return fail(QLIN_ERR_INVALID, "out overlaps q or the cache");
    if (batch_meets(batch, ro)) return fail(QLIN_ERR_INVALID, "out overlaps new_start, length or cache_start");
    CausalPlan p;
    if (causal_plan(batch, q_heads, cache->heads, splits, &p) != QLIN_OK) return last_status();
    if (p.ws_bytes > 0 && (!workspace || workspace_bytes < p.ws_bytes))
        return fail(QLIN_ERR_INVALID, "workspace of %lld bytes needed (%lld given)", (long long)p.ws_bytes,
                    (long long)(workspace ? workspace_bytes : 0));
    const Range ws{(uintptr_t)workspace, (size_t)p.ws_bytes};
    for (const Range &r : {ro, rows_range(q, M, q_stride, w), cache_range(cache->k, cache), cache_range(cache->v, cache)})
        if (overlap(r, ws)) return fail(QLIN_ERR_INVALID, "the workspace overlaps q, out or the cache");
    if (batch_meets(batch, ws)) return fail(QLIN_ERR_INVALID, "the workspace overlaps new_start, length or cache_start");
    if (batch->max_new == 0) return QLIN_OK;

    CausalArgs a;
    a.b = batch_args(batch, cache);
    a.q = q;
    a.k = cache->k;
    a.v = cache->v;
    a.out = out;
    a.q_stride = q_stride;
    a.out_stride = out_stride;
    a.Hq = (int)q_heads;
    a.Hkv = (int)cache->heads;
    a.G = (int)(q_heads / cache->heads);
    a.ws_o = (float *)workspace;
    a.ws_ml = a.ws_o + (size_t)p.tiles * a.Hkv * p.S * causal_tile_rows(p.rt) * kHeadDim;
    a.tiles = p.tiles;
    a.one_tile = p.one_tile;
    a.pairs = p.pairs;
    a.least = p.least;
    a.S = p.S;
    a.max_len = (int)batch->max_len;
    gn_reciprocal(a.Hkv, &a.inv_heads, &a.heads_shift);
    a.inv_g = a.G > 1 ? (uint32_t)((((uint64_t)1 << 32) + a.G - 1) / a.G) : 0u;
    a.c = factor;
    const hipError_t e = launch_causal(a, p.rt, p.halves, (hipStream_t)stream);
    return e == hipSuccess ? QLIN_OK : hip_fail(e, "causal attention launch");
}

int qlin_verify_plan(int64_t n_seq, int64_t n_draft, int64_t vocab, int64_t *workspace_bytes) {
    clear_err();
    if (n_seq < 0 || n_draft < 0 || vocab < 1) return fail(QLIN_ERR_INVALID, "n_seq and n_draft must be >= 0, vocab positive");
    if (n_seq > kMaxVerifySeq || n_draft > kMaxDraft || vocab > kMaxVocab)
        return fail(QLIN_ERR_UNSUPPORTED, "at most 65535 sequences, 64 drafted tokens and 2^24 tokens of vocabulary");
    if (workspace_bytes) *workspace_bytes = verify_layout(n_seq, n_draft, vocab).bytes;
    return QLIN_OK;
}

int qlin_verify_draft(int64_t n_seq, int64_t n_draft, int64_t vocab, const uint16_t *target, int64_t target_stride,
                      const uint16_t *draft, int64_t draft_stride, const int32_t *drafted, const int32_t *count,
                      const float *temperature, const float *uniform, int32_t *accepted, int32_t *tokens,
                      void *workspace, int64_t workspace_bytes, void *stream) {
    int64_t need = 0;
    if (qlin_verify_plan(n_seq, n_draft, vocab, &need) != QLIN_OK) return last_status();
    if (workspace_bytes < 0) return fail(QLIN_ERR_INVALID, "workspace_bytes must be >= 0");
    if (n_seq == 0) return QLIN_OK;
    if (!target || !uniform || !accepted || !tokens || (n_draft > 0 && !drafted))
        return fail(QLIN_ERR_INVALID, "NULL target, drafted, uniform, accepted or tokens");
    if (target_stride < vocab || target_stride > kMaxRowStride || (draft && (draft_stride < vocab || draft_stride > kMaxRowStride)))
        return fail(QLIN_ERR_INVALID, "row strides must be at least vocab");
    if (!aligned(target, 16) || !aligned(draft, 16) || !aligned(workspace, 16))
        return fail(QLIN_ERR_ALIGN, "target, draft and workspace must be 16-byte aligned");
    for (const void *p : {(const void *)drafted, (const void *)count, (const void *)temperature, (const void *)uniform,
                          (const void *)accepted, (const void *)tokens})
        if (!aligned(p, 4)) return fail(QLIN_ERR_ALIGN, "int32 and float arrays must be 4-byte aligned");
    if (need > 0 && (!workspace || workspace_bytes < need))
        return fail(QLIN_ERR_INVALID, "workspace of %lld bytes needed (%lld given)", (long long)need,
                    (long long)(workspace ? workspace_bytes : 0));
    const size_t per = (size_t)n_seq * 4;
    const Range outs[2] = {{(uintptr_t)accepted, per}, {(uintptr_t)tokens, per * (size_t)(n_draft + 1)}};
    const Range ins[] = {rows_range(target, n_seq * (n_draft + 1), target_stride, vocab),
                         rows_range(draft, draft ? n_seq * n_draft : 0, draft_stride, vocab),
                         {(uintptr_t)drafted, per * (size_t)n_draft},
                         {(uintptr_t)count, count ? per : 0},
                         {(uintptr_t)temperature, temperature ? per : 0},
                         {(uintptr_t)uniform, per * (size_t)(n_draft + 1)}};
    const Range ws{(uintptr_t)workspace, (size_t)need};
    for (const Range &i : ins) {
        for (const Range &o : outs)
            if (overlap(o, i)) return fail(QLIN_ERR_INVALID, "accepted or tokens overlaps an input");
        if (overlap(i, ws)) return fail(QLIN_ERR_INVALID, "the workspace overlaps an input");
    }
    for (const Range &o : outs)
        if (overlap(o, ws)) return fail(QLIN_ERR_INVALID, "the workspace overlaps accepted or tokens");
    if (overlap(outs[0], outs[1])) return fail(QLIN_ERR_INVALID, "accepted overlaps tokens");

    VerifyArgs a;
    a.target = target;
    a.draft = draft;
    a.drafted = drafted;
    a.count = count;
    a.temperature = temperature;
    a.uniform = uniform;
    a.accepted = accepted;
    a.tokens = tokens;
    a.target_stride = target_stride;
    a.draft_stride = draft_stride;
    a.n = (int)n_draft;
    a.V = (int)vocab;
    const VerifyLayout l = verify_layout(n_seq, n_draft, vocab);
    a.chunks = (int)l.chunks;
    a.all_rows = (int)(draft ? l.rows : n_draft + 1);
    a.stats = (VerifyStat *)workspace;
    a.sums = (double *)((char *)workspace + l.sums);
    a.decisions = (VerifyDecision *)((char *)workspace + l.decisions);
    a.final_decisions = a.decisions + n_seq;
    // Large calls look at a third of the rows first: a sequence that refuses a token there, as
    // most do at 3 of 4 tokens kept, needs no more.
    const int64_t logits = n_seq * (n_draft + 1 + (draft ? n_draft : 0)) * vocab;
    a.first_rows = logits >= kVerifyTwoParts && n_draft >= 3 ? (int)(n_draft + 1) / 3 : 0;
    a.row0 = a.row1 = 0;
    const hipError_t e = launch_verify(a, (int)n_seq, logits >= kVerifyMany, (hipStream_t)stream);
    return e == hipSuccess ? QLIN_OK : hip_fail(e, "verify launch");
}

}  // extern "C"
