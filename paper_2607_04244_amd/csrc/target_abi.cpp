// C ABI of the target's operators (include/qlin_target.h): argument checks,
// plans and launches.

#include "../../include/qlin_target.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstring>

#include "target_checks.h"

using namespace qlin;

namespace {

constexpr int64_t kMaxDraft = kVerifyMaxDraft, kMaxVocab = (int64_t)1 << 24, kMaxVerifySeq = 65535;   // sequences: a grid's y
constexpr int64_t kVerifyTwoParts = (int64_t)1 << 26, kVerifyMany = (int64_t)1 << 25;     // logits of a call: see qlin_verify_draft

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

// The launches of a checked call.
int launch_attention(const qlin_batch *batch, const qlin_kv_cache *cache, const HeadShift *shifts, const short2 *row_shifts,
                     const CausalPlan &p, int64_t q_heads, float factor, const uint16_t *q, int64_t q_stride, uint16_t *out, int64_t out_stride, void *workspace,
                     hipStream_t stream) {
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
    a.shifts = shifts;
    a.row_shifts = row_shifts;
    const hipError_t e = launch_causal(a, p.rt, p.halves, stream);
    return e == hipSuccess ? QLIN_OK : hip_fail(e, "causal attention launch");
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

namespace qlin {

int attend_in_f16(const qlin_batch *batch, const qlin_kv_cache *cache, const HeadShift *shifts, const short2 *row_shifts,
                  int64_t q_heads, float factor, int64_t splits, const uint16_t *q, int64_t q_stride, uint16_t *out,
                  int64_t out_stride, void *workspace, hipStream_t stream) {
    CausalPlan p;
    if (causal_plan(batch, q_heads, cache->heads, splits, &p) != QLIN_OK) return last_status();
    return launch_attention(batch, cache, shifts, row_shifts, p, q_heads, factor, q, q_stride, out, out_stride, workspace, stream);
}

}  // namespace qlin

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
    const AppendRows r{q, q_stride, k, k_stride, v, v_stride, q_norm, k_norm, eps, inv_freq, rotary_dim, q_out, q_out_stride};
    if (check_append_values(r) != QLIN_OK) return last_status();
    if (batch->rows == 0) return QLIN_OK;
    const Range c[] = {cache_range(cache->k, cache), cache_range(cache->v, cache)};
    if (check_append_arrays(batch, q_heads, cache->heads, r, c, 2) != QLIN_OK) return last_status();

    AppendArgs a = append_args(batch_args(batch, cache), q_heads, cache->heads, r, interleaved);
    a.kc = cache->k;
    a.vc = cache->v;
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
    float factor;
    if (check_attention_values(scale, splits, workspace_bytes, &factor) != QLIN_OK) return last_status();
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

    return launch_attention(batch, cache, nullptr, nullptr, p, q_heads, factor, q, q_stride, out, out_stride, workspace, (hipStream_t)stream);
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
