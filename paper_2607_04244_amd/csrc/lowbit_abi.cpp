// C ABI of a layer's operators in fewer bits (include/qlin_lowbit.h): argument checks,
// plans and launches.

#include "../../include/qlin_lowbit.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdio>
#include <cstring>

#include "lowbit_internal.h"
#include "target_checks.h"

using namespace qlin;

namespace {

constexpr int64_t kMaxWidth = 65536, kMaxChannels = (int64_t)1 << 22, kMaxK = 131056, kMaxKSplits = 64;
constexpr int64_t kMaxRowTokens = (int64_t)1 << 20;          // 32-bit byte offsets over 64 tokens
constexpr int64_t kMaxRowHeads = (int64_t)1 << 36;
constexpr int64_t kMaxCacheRows = (int64_t)1 << 53;          // 64-bit byte offsets
constexpr int64_t kKv4FewRows = 64;                        // a sequence's rows from which unpacking is weighed
constexpr int64_t kMaxUnpacked = (int64_t)1 << 34;           // bytes of an unpacked cache: beyond, codes are read, which takes no such scratch

Range bytes_range(const void *p, int64_t rows, int64_t stride, int64_t width) {
    return Range{(uintptr_t)p, p && rows > 0 ? (size_t)((rows - 1) * stride + width) : 0};
}

bool meets_any(const Range &r, std::initializer_list<Range> others) {
    for (const Range &o : others)
        if (overlap(r, o)) return true;
    return false;
}

// Whether two row arrays share an element without being the same.
bool clash(const void *p, int64_t stride, const void *q, int64_t q_stride, int64_t rows, int64_t width) {
    return !(p == q && stride == q_stride) && rows_meet(p, stride, width, q, q_stride, width, rows);
}

int check_kv4(const qlin_kv4_cache *c) {
    if (!c) return fail(QLIN_ERR_INVALID, "NULL cache");
    if (c->slots < 1 || c->seq_slots < 0 || c->capacity < 0 || c->token_stride < 1 || c->head_stride < 1)
        return fail(QLIN_ERR_INVALID, "cache: slots and strides must be positive, seq_slots and capacity >= 0");
    if (c->slots > kMaxSlots || c->seq_slots > kMaxSlots || c->capacity > kMaxSlots || c->token_stride > kMaxRowTokens ||
        c->head_stride > kMaxRowHeads || (double)c->slots * (double)c->token_stride + (double)c->heads * (double)c->head_stride > (double)kMaxCacheRows)
        return fail(QLIN_ERR_UNSUPPORTED, "cache too large");
    if (!c->k || !c->v || !c->k_grid || !c->v_grid) return fail(QLIN_ERR_INVALID, "NULL cache");
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->k_grid, 4) || !aligned(c->v_grid, 4))
        return fail(QLIN_ERR_ALIGN, "the cache's codes must be 16-byte aligned, its grids 4");
    return QLIN_OK;
}

// The address ranges of a cache: codes and grids of keys and of values.
struct Kv4Ranges {
    Range r[4];
    explicit Kv4Ranges(const qlin_kv4_cache *c) {
        const size_t rows = (size_t)((c->slots - 1) * c->token_stride + (c->heads - 1) * c->head_stride + 1);
        r[0] = Range{(uintptr_t)c->k, rows * 64};
        r[1] = Range{(uintptr_t)c->v, rows * 64};
        r[2] = Range{(uintptr_t)c->k_grid, rows * 4};
        r[3] = Range{(uintptr_t)c->v_grid, rows * 4};
    }
    bool meet(const Range &o) const { return overlap(r[0], o) || overlap(r[1], o) || overlap(r[2], o) || overlap(r[3], o); }
    bool meet_each_other() const {
        for (int i = 0; i < 4; ++i)
            for (int j = i + 1; j < 4; ++j)
                if (overlap(r[i], r[j])) return true;
        return false;
    }
};

BatchArgs batch_args(const qlin_batch *b, const qlin_kv4_cache *c) {
    qlin_kv_cache rows = {};
    rows.capacity = c->capacity;
    rows.slots = c->slots;
    rows.token_stride = c->token_stride;
    rows.head_stride = c->head_stride;
    rows.seq_slots = c->seq_slots;
    return qlin::batch_args(b, &rows);
}

Kv4Arrays kv4_arrays(const qlin_kv4_cache *c) { return Kv4Arrays{c->k, c->v, (uint32_t *)c->k_grid, (uint32_t *)c->v_grid}; }

UnpackArgs unpack_args(const qlin_batch *b, const qlin_kv4_cache *c, bool new_only) {
    UnpackArgs a = {};
    a.b = batch_args(b, c);
    a.b.longest = (int)b->max_len;
    a.c = kv4_arrays(c);
    a.heads = (int)c->heads;
    a.new_only = new_only;
    a.tiles = (int)(((new_only ? b->max_new : b->max_len) + kUnpackTokens - 1) / kUnpackTokens);
    a.items = b->n_seq * c->heads * a.tiles;
    return a;
}

// ---- the linear

struct I8Plan { int form = 0, tiles_m = 0, tiles_n = 0, S = 1, steps = 0; int64_t ws_bytes = 0; };

int check_i8(int64_t M, int64_t N, int64_t K, int64_t splits) {
    if (M < 0 || N < 1 || K < 16 || K % 16 || splits < 0 || splits > kMaxKSplits)
        return fail(QLIN_ERR_INVALID, "M must be >= 0, N positive, K a positive multiple of 16, splits in [0, 64]");
    if (M > kMaxRows || N > kMaxChannels || K > kMaxK) return fail(QLIN_ERR_UNSUPPORTED, "at most 2^22 rows and channels, K up to 131056");
    return QLIN_OK;
}

constexpr const char *kI8Names[] = {"k_i8_few", "k_i8_tile<128x64>", "k_i8_tile<128x128>", "k_i8_tile<256x128>", "k_i8_tile<256x256>", "k_i8_tile<320x256>"};

// Estimated microseconds of a call in a tile form with S ranges of K, fitted to graph replays
// (K steps of 64 bytes; weights of several layers in turn).  A step takes `alone` where a
// workgroup has its compute unit to itself and few work, `full` where all units do or it shares
// one (for both; their clock falls), and a workgroup some time for its first loads and its
// stores.  Measured / estimated, forms 1 to 5: 512 x 19456 x 2560 (rows, channels, K) 55.6 / 56.3 /
// 60.0 / 49.5 / 56.9 and 52.0 / 59.2 / 55.8 / 45.5 / 52.0 us; 1500 x 2560 x 2560 18.1 / 19.8 / 26.8 /
// 40.0 / 48.8 and 20.7 / 19.4 / 33.4 / 42.8 / 45.8; 333 x 2560 x 9728 in form 2 with 1, 2, 3, 4 ranges
// 57.0 / 33.7 / 26.5 / 23.5 and 54.1 / 33.7 / 26.5 / 23.1.  Over 14 sizes that times of all forms were
// taken of, its choice is the fastest measured or up to 9 % slower.
struct I8Time { double alone, full, fixed; };
constexpr I8Time kI8Times[] = {{}, {0.22, 0.38, 5.5}, {0.31, 0.62, 7.0}, {0.61, 1.17, 9.0}, {0.80, 0.99, 9.0}, {0.82, 1.35, 9.0}};

double i8_cost(int form, double tiles, double tiles_m, double steps, double S, double weights, double cus) {
    const I8Form &f = kI8Forms[form];
    const I8Time &t = kI8Times[form];
    const double slots = cus * f.per_cu, rounds = std::floor(tiles * S / slots), rest = (tiles * S - rounds * slots) / cus;
    // of two workgroups a unit, the units that have both end last, however few
    const double range = std::ceil(steps / S), load = f.per_cu == 1 ? rest : std::min(std::max(rest - 1.0, 0.0) * 5.0, 1.0);
    const double time = rounds * (range * t.full + t.fixed) + (rest > 0.0 ? range * (t.alone + (t.full - t.alone) * load) + t.fixed : 0.0);
    const double join = S > 1.0 ? 1.8 + S * tiles * f.n * f.m * 8.0 / 1.2e7 : 0.0;
    return std::max(time, std::min(tiles_m, 2.0) * weights / 4e6) + join;        // two tiles of rows read the weights twice
}

int i8_plan(int64_t M, int64_t N, int64_t K, int64_t splits, I8Plan *p) {
    if (check_i8(M, N, K, splits) != QLIN_OK) return last_status();
    int64_t cus = 256;                               // forced ranges: arithmetic
    if (splits == 0 && compute_units(&cus) != QLIN_OK) return last_status();
    const bool few = M <= kI8FewRows;
    const int64_t steps = (K + kI8Step - 1) / kI8Step;
    int64_t S = 1;
    if (few) {
        // as few ranges as let each wave keep its part of the tokens in registers: 64 x 9728 x 2560
        // (rows, K, channels) 26.9 us in one range, 17.3 in four; 32 rows 17.9, 13.8 in three
        const int64_t held = kI8FewWaves * i8_few_steps((int)M);
        S = splits ? splits : (steps + held - 1) / held;
    } else {
        double best = 0.0;
        for (int form = 1; form < kI8FormCount; ++form) {
            const I8Form &f = kI8Forms[form];
            const int64_t tiles_m = (M + f.m - 1) / f.m, tiles = tiles_m * ((N + f.n - 1) / f.n);
            auto consider = [&](int64_t ranges) {
                const double t = i8_cost(form, (double)tiles, (double)tiles_m, (double)steps, (double)ranges, (double)N * (double)K, (double)cus);
                if (best > 0.0 && t >= best) return;
                best = t;
                p->form = form;
                S = ranges;
            };
            if (splits) consider(splits);
            else
                for (const int64_t s : {1, 2, 3, 4, 6, 8})
                    if (s <= std::max<int64_t>(steps / 4, 1)) consider(s);
        }
    }
    const I8Form &f = kI8Forms[p->form];
    p->tiles_m = (int)((M + f.m - 1) / f.m);
    p->tiles_n = (int)((N + f.n - 1) / f.n);
    const int64_t tiles = (int64_t)std::max(p->tiles_m, 1) * p->tiles_n;
    if (tiles >= (int64_t)1 << 23) return fail(QLIN_ERR_UNSUPPORTED, "too many rows and channels for one call");
    S = std::max<int64_t>(1, std::min(S, std::min(steps, kMaxKSplits)));
    p->steps = (int)((steps + S - 1) / S);
    p->S = (int)((steps + p->steps - 1) / p->steps);
    if (p->S > 1 && !few && tiles * f.n * f.m >= (int64_t)1 << 34)       // the joining kernel's grid
        return fail(QLIN_ERR_UNSUPPORTED, "too many rows and channels for K ranges");
    p->ws_bytes = p->S == 1 ? 0 : (int64_t)p->S * 4 * (few ? M * N : tiles * f.n * f.m);
    return QLIN_OK;
}

// ---- attention over the 4-bit cache

// rt: 1, 2 as causal_tile_rows; 0: unpacked to the workspace, then qlin_causal_attention
struct Kv4Plan { int rt = 0, tiles = 0, one_tile = 0, S = 1, least = 1; int64_t ws_bytes = 0, unpacked = 0; };

// Where the parts of the unpack form's workspace begin: keys, values, lengths, shifts of heads and of
// rows, peaks, attention.
struct Unpacked {
    int64_t v, length, shifts, row_shifts, peaks, peak_tiles, attention;
    Unpacked(int64_t n_seq, int64_t heads, int64_t max_len) {
        auto whole = [](int64_t n) { return (n + 15) / 16 * 16; };
        v = n_seq * heads * max_len * kHeadDim * 2;
        length = 2 * v;
        shifts = length + whole(n_seq * 4);
        row_shifts = shifts + whole(n_seq * heads * (int64_t)sizeof(HeadShift));
        peaks = row_shifts + whole(n_seq * heads * max_len * 4);
        peak_tiles = (max_len + kPeakTokens - 1) / kPeakTokens;
        attention = peaks + n_seq * heads * peak_tiles * 16;
    }
};

// The workspace's cache of 16-bit values.
qlin_kv_cache unpacked_cache(const qlin_batch *b, int64_t heads, void *workspace) {
    const Unpacked u(b->n_seq, heads, b->max_len);
    qlin_kv_cache c;
    c.capacity = b->max_len;
    c.k = (uint16_t *)workspace;
    c.v = (uint16_t *)((char *)workspace + u.v);
    c.heads = heads;
    c.slots = (b->n_seq - 1) * heads * b->max_len + b->max_len;
    c.token_stride = kHeadDim;
    c.head_stride = b->max_len * kHeadDim;
    c.seq_slots = heads * b->max_len;
    return c;
}

// Estimated microseconds of the kernels that read codes (rt 1, 2): `blocks` (tile, head) items,
// sequences of up to `most` keys, in S ranges of equal size.  Fitted to graph replays of 32 / 8
// heads.  A workgroup has some time without keys, then a step of 64 keys a wave takes `alone` where
// it has its compute unit to itself and `paired` where two share one; ranges of several sequences
// are assumed half as many as of the longest in each.  Measured / estimated: 32 tokens of 4096
// keys in 1 and 2 ranges 31.3, 32.3 / 31.7, 36.4; 8 of 4000 in 2, 4, 8 20.5, 16.5, 17.5 / 21.2, 14.5, 11.5;
// 16 tokens over 8192 in 8, 16, 32 18.2, 15.3, 16.7 / 17.2, 13.3, 13.4; 5 x 16 over 517 to 8192 in 4, 8, 12
// 26.8, 27.3, 25.0 / 27.5, 24.9, 25.6.
double kv4_cost(int rt, double blocks, double most, double S, bool several, double cus) {
    const double fixed = rt == 1 ? 4.5 : 6.0, alone = rt == 1 ? 1.7 : 2.0, paired = rt == 1 ? 2.8 : 3.6;
    const double W = blocks * (several ? 0.5 * (S + 1.0) : S), slots = 2.0 * cus;
    const double load = std::min(std::max(W / cus - 1.0, 0.0), 1.0), steps = std::ceil(most / S / (4.0 * kKv4Keys));
    const double one = fixed + steps * (alone + (paired - alone) * load);
    return (W <= slots ? one : W * one / slots + 0.5 * one) + (S > 1.0 ? 3.0 + W * causal_tile_rows(rt) * (kHeadDim + 2) * 4 / 8e6 : 0.0);
}

// The same of the unpack form: two kernels that write the cache in 16 bits, then tiles of 128 rows.
// Measured / estimated: 300 tokens behind 3700 51.9 / 46, 500 behind 7400 99 / 102, 16 x 128 behind 2872
// 169 / 190 us.  What it cannot know: heads that go by a power for each row (cached rows more than 2^12
// apart) take up to four times as long, 500 behind 7400 348 us.
double unpack_cost(double tiles, double rows, double mean, double cus) { return 18.0 + rows * 1.5e-4 + 1.15 * tiles * mean * 0.033 / (2.0 * cus); }

int kv4_plan(const qlin_batch *b, int64_t Hq, int64_t Hkv, int64_t splits, Kv4Plan *p) {
    int64_t cus = 256;                                            // forced ranges: arithmetic
    if (splits == 0 && compute_units(&cus) != QLIN_OK) return last_status();
    const int64_t G = Hq / Hkv, most = b->max_new * G;
    p->rt = most <= 16 ? 1 : 2;
    const int64_t R = causal_tile_rows(p->rt), per = (most + R - 1) / R;
    // of sequences with about as many new tokens each, a tile is found without a walk over them (the
    // first microseconds of a workgroup)
    p->one_tile = (int)(per <= 1 ? 1 : b->n_seq * per <= 2 * (b->rows * G / R + 1) ? per : 0);
    const int64_t tiles = p->one_tile ? b->n_seq * per : std::min(b->n_seq * per, b->rows * G / R + b->n_seq);
    const int64_t blocks = std::max<int64_t>(tiles * Hkv, 1), steps = (b->max_len + kKv4Keys - 1) / kKv4Keys;
    // a tile's keys: of a prompt's tiles half of it on average
    const double mean = (double)b->max_len - 0.5 * (double)std::min(b->max_new, b->max_len);
    int64_t S = std::max<int64_t>(splits, 1);
    double best = kv4_cost(p->rt, (double)blocks, mean, (double)S, b->n_seq > 1, (double)cus);
    if (splits == 0 && blocks < 2 * cus)                          // more ranges of them cost more than late tails
        for (const int64_t s : {(int64_t)2, (int64_t)3, (int64_t)4, (int64_t)6, (int64_t)8, (int64_t)12, (int64_t)16, (int64_t)24, cus / blocks, 2 * cus / blocks}) {
            if (s < 2 || s > std::min((steps + 3) / 4, kMaxSplits)) continue;      // a step of each wave
            const double t = kv4_cost(p->rt, (double)blocks, mean, (double)s, b->n_seq > 1, (double)cus);
            if (t >= best) continue;
            best = t;
            S = s;
        }
    const int64_t tiles128 = std::min(b->n_seq * ((most + 127) / 128), b->rows * G / 128 + b->n_seq);
    const double rows16 = (double)b->n_seq * (double)Hkv * (double)b->max_len;
    if (most > kKv4FewRows && b->max_len > 0 && unpack_cost((double)(tiles128 * Hkv), rows16, mean, (double)cus) < best &&
        rows16 * 4.0 * kHeadDim <= (double)kMaxUnpacked) {
        int64_t attention = 0;
        if (qlin_causal_plan(b, Hq, Hkv, kHeadDim, splits, nullptr, &attention, nullptr, 0) != QLIN_OK) return last_status();
        p->rt = 0;
        p->unpacked = Unpacked(b->n_seq, Hkv, b->max_len).attention;
        p->ws_bytes = p->unpacked + attention;
        return QLIN_OK;
    }
    if (tiles * Hkv * std::max(S, S > 1 ? R / 2 : 0) >= (int64_t)1 << 23)
        return fail(QLIN_ERR_UNSUPPORTED, "too many rows, heads and key ranges for one call");
    p->tiles = (int)tiles;
    p->S = (int)S;
    p->least = (int)std::max<int64_t>(splits ? 4 : (steps + S - 1) / S, 4);        // ranges of one size: short sequences stay whole
    p->ws_bytes = S > 1 ? tiles * Hkv * S * R * (kHeadDim + 2) * 4 : 0;
    return QLIN_OK;
}

}  // namespace

extern "C" {

int qlin_block_norm(int64_t rows, int64_t width, const uint16_t *y, int64_t y_stride, const uint16_t *residual,
                    int64_t residual_stride, const uint16_t *post_norm, const uint16_t *gate, int64_t gate_stride,
                    int gate_sigmoid, float scale, const uint16_t *pre_norm, float eps, uint16_t *residual_out,
                    int64_t residual_out_stride, uint16_t *out, int64_t out_stride, void *stream) {
    clear_err();
    if (rows < 0 || width < 8 || width % 8) return fail(QLIN_ERR_INVALID, "rows must be >= 0, width a positive multiple of 8");
    if (rows >= kMaxRows || width > kMaxWidth) return fail(QLIN_ERR_UNSUPPORTED, "fewer than 2^22 rows of up to 65536");
    if (!(eps >= 0.0f) || std::isinf(eps)) return fail(QLIN_ERR_INVALID, "eps must be >= 0");
    if (!std::isfinite(scale)) return fail(QLIN_ERR_INVALID, "scale must be finite");
    if (rows == 0) return QLIN_OK;
    if (!y && (post_norm || gate || residual_out)) return fail(QLIN_ERR_INVALID, "post_norm, gate and residual_out need y");
    if ((pre_norm != nullptr) != (out != nullptr)) return fail(QLIN_ERR_INVALID, "pre_norm and out go together");
    if (!y && !out) return fail(QLIN_ERR_INVALID, "neither y nor out given");
    if (check_rows(residual, residual_stride, width, "residual") != QLIN_OK) return last_status();
    if (y && (check_rows(y, y_stride, width, "y") != QLIN_OK || check_rows(residual_out, residual_out_stride, width, "residual_out") != QLIN_OK))
        return last_status();
    if (out && check_rows(out, out_stride, width, "out") != QLIN_OK) return last_status();
    if (gate && gate_stride != 0 && check_rows(gate, gate_stride, width, "gate") != QLIN_OK) return last_status();
    if (!aligned(gate, 16) || !aligned(post_norm, 16) || !aligned(pre_norm, 16))
        return fail(QLIN_ERR_ALIGN, "gate and norm weights must be 16-byte aligned");
    const Range weights[] = {{(uintptr_t)post_norm, post_norm ? (size_t)width * 2 : 0}, {(uintptr_t)pre_norm, pre_norm ? (size_t)width * 2 : 0},
                             {(uintptr_t)gate, gate && gate_stride == 0 ? (size_t)width * 2 : 0}};
    const struct { const uint16_t *p; int64_t stride; } outs[] = {{residual_out, residual_out_stride}, {out, out_stride}};
    for (const auto &o : outs) {
        if (!o.p) continue;
        if (clash(o.p, o.stride, residual, residual_stride, rows, width) || (y && clash(o.p, o.stride, y, y_stride, rows, width)))
            return fail(QLIN_ERR_INVALID, "an output overlaps y or residual without being it");
        if (gate && gate_stride != 0 && rows_meet(o.p, o.stride, width, gate, gate_stride, width, rows))
            return fail(QLIN_ERR_INVALID, "an output overlaps the gate");
        for (const Range &r : weights)
            if (overlap(rows_range(o.p, rows, o.stride, width), r)) return fail(QLIN_ERR_INVALID, "an output overlaps norm weights or the gate");
    }
    if (residual_out && out && rows_meet(residual_out, residual_out_stride, width, out, out_stride, width, rows))
        return fail(QLIN_ERR_INVALID, "residual_out overlaps out");

    BlockNormArgs a;
    a.y = y;
    a.residual = residual;
    a.post = post_norm;
    a.gate = gate;
    a.pre = pre_norm;
    a.residual_out = residual_out;
    a.out = out;
    a.y_stride = y_stride;
    a.residual_stride = residual_stride;
    a.gate_stride = gate_stride;
    a.residual_out_stride = residual_out_stride;
    a.out_stride = out_stride;
    a.rows = (int)rows;
    a.width = (int)width;
    a.sigmoid = gate_sigmoid != 0;
    a.scale = scale;
    a.eps = eps;
    const hipError_t e = launch_block_norm(a, (hipStream_t)stream);
    return e == hipSuccess ? QLIN_OK : hip_fail(e, "block norm launch");
}

int qlin_quantize_tokens(int64_t rows, int64_t width, const uint16_t *x, int64_t x_stride, int gated, int8_t *codes,
                         int64_t codes_stride, float *scale, void *stream) {
    clear_err();
    if (rows < 0 || width < 16 || width % 16) return fail(QLIN_ERR_INVALID, "rows must be >= 0, width a positive multiple of 16");
    if (rows >= kMaxRows || width > kMaxWidth) return fail(QLIN_ERR_UNSUPPORTED, "fewer than 2^22 rows of up to 65536");
    if (rows == 0) return QLIN_OK;
    const int64_t in = gated ? 2 * width : width;
    if (check_rows(x, x_stride, in, "x") != QLIN_OK) return last_status();
    if (!codes || !scale) return fail(QLIN_ERR_INVALID, "NULL codes or scale");
    if (codes_stride < width || codes_stride > kMaxRowStride) return fail(QLIN_ERR_INVALID, "codes: stride must be at least %lld", (long long)width);
    if (!aligned(codes, 16) || codes_stride % 16 || !aligned(scale, 4))
        return fail(QLIN_ERR_ALIGN, "codes must be 16-byte aligned, its stride a multiple of 16, scale 4-byte aligned");
    const Range rx = rows_range(x, rows, x_stride, in), rc = bytes_range(codes, rows, codes_stride, width), rs{(uintptr_t)scale, (size_t)rows * 4};
    if (overlap(rc, rx) || overlap(rs, rx) || overlap(rc, rs)) return fail(QLIN_ERR_INVALID, "codes or scale overlaps x or each other");
    const hipError_t e = launch_quantize_tokens(QuantizeArgs{x, codes, scale, x_stride, codes_stride, (int)rows, (int)width, gated != 0}, (hipStream_t)stream);
    return e == hipSuccess ? QLIN_OK : hip_fail(e, "token quantization launch");
}

int qlin_eight_bit_plan(int64_t M, int64_t N, int64_t K, int64_t splits, int64_t *splits_out, int64_t *workspace_bytes, char *buf, int64_t buflen) {
    clear_err();
    I8Plan p;
    if (i8_plan(M, N, K, splits, &p) != QLIN_OK) return last_status();
    if (splits_out) *splits_out = p.S;
    if (workspace_bytes) *workspace_bytes = p.ws_bytes;
    if (buf && buflen > 0)
        snprintf(buf, (size_t)buflen, "kernel=%s splits=%d grid=%lld combine=%d", kI8Names[p.form], p.S,
                 (long long)p.tiles_m * p.tiles_n * p.S, p.S > 1 ? 1 : 0);
    return QLIN_OK;
}

int qlin_eight_bit_linear(int64_t M, int64_t N, int64_t K, int64_t splits, const int8_t *x, int64_t x_stride, const float *x_scale,
                   const int8_t *w, int64_t w_stride, const float *w_scale, uint16_t *y, int64_t y_stride, void *workspace,
                   int64_t workspace_bytes, void *stream) {
    clear_err();
    I8Plan p;
    if (i8_plan(M, N, K, splits, &p) != QLIN_OK) return last_status();
    if (workspace_bytes < 0) return fail(QLIN_ERR_INVALID, "workspace_bytes must be >= 0");
    if (M == 0) return QLIN_OK;
    if (!x || !w || !x_scale || !w_scale) return fail(QLIN_ERR_INVALID, "NULL x, w or scales");
    if (x_stride < K || w_stride < K || x_stride > kMaxRowStride || w_stride > kMaxRowStride)
        return fail(QLIN_ERR_INVALID, "x and w: strides must be at least %lld", (long long)K);
    if (!aligned(x, 16) || !aligned(w, 16) || x_stride % 16 || w_stride % 16)
        return fail(QLIN_ERR_ALIGN, "x and w must be 16-byte aligned, their strides multiples of 16");
    if (!aligned(x_scale, 4) || !aligned(w_scale, 4)) return fail(QLIN_ERR_ALIGN, "scales must be 4-byte aligned");
    if (check_rows(y, y_stride, N, "y") != QLIN_OK) return last_status();
    if (!aligned(workspace, 16)) return fail(QLIN_ERR_ALIGN, "workspace must be 16-byte aligned");
    if (p.ws_bytes > 0 && (!workspace || workspace_bytes < p.ws_bytes))
        return fail(QLIN_ERR_INVALID, "workspace of %lld bytes needed (%lld given)", (long long)p.ws_bytes,
                    (long long)(workspace ? workspace_bytes : 0));
    const Range rx = bytes_range(x, M, x_stride, K), rw = bytes_range(w, N, w_stride, K), sx{(uintptr_t)x_scale, (size_t)M * 4},
                sw{(uintptr_t)w_scale, (size_t)N * 4}, ry = rows_range(y, M, y_stride, N), ws{(uintptr_t)workspace, (size_t)p.ws_bytes};
    if (meets_any(ry, {rx, rw, sx, sw})) return fail(QLIN_ERR_INVALID, "y overlaps an input");
    if (meets_any(ws, {rx, rw, sx, sw, ry})) return fail(QLIN_ERR_INVALID, "the workspace overlaps an input or y");

    I8Args a;
    a.x = x;
    a.w = w;
    a.x_scale = x_scale;
    a.w_scale = w_scale;
    a.y = y;
    a.parts = (int32_t *)workspace;
    a.x_stride = x_stride;
    a.w_stride = w_stride;
    a.y_stride = y_stride;
    a.M = (int)M;
    a.N = (int)N;
    a.K = (int)K;
    a.S = p.S;
    a.steps = p.steps;
    a.tiles_m = p.tiles_m;
    a.tiles_n = p.tiles_n;
    a.form = p.form;
    const hipError_t e = launch_i8_linear(a, (hipStream_t)stream);
    return e == hipSuccess ? QLIN_OK : hip_fail(e, "8-bit linear launch");
}

int qlin_norm_rope_append_four_bit(const qlin_batch *batch, const qlin_kv4_cache *cache, int64_t q_heads, int64_t head_dim,
                              const uint16_t *q, int64_t q_stride, const uint16_t *k, int64_t k_stride, const uint16_t *v,
                              int64_t v_stride, const uint16_t *q_norm, const uint16_t *k_norm, float eps,
                              const double *inv_freq, int64_t rotary_dim, int interleaved, uint16_t *q_out,
                              int64_t q_out_stride, void *stream) {
    clear_err();
    if (check_batch(batch) != QLIN_OK) return last_status();
    if (!cache) return fail(QLIN_ERR_INVALID, "NULL cache");
    if (check_heads(q_heads, cache->heads, head_dim) != QLIN_OK || check_kv4(cache) != QLIN_OK) return last_status();
    const AppendRows rows{q, q_stride, k, k_stride, v, v_stride, q_norm, k_norm, eps, inv_freq, rotary_dim, q_out, q_out_stride};
    if (check_append_values(rows) != QLIN_OK) return last_status();
    if (batch->rows == 0) return QLIN_OK;
    const Kv4Ranges c(cache);
    if (check_append_arrays(batch, q_heads, cache->heads, rows, c.r, 4) != QLIN_OK) return last_status();
    if (c.meet_each_other()) return fail(QLIN_ERR_INVALID, "the cache's arrays overlap each other");

    AppendKv4Args x;
    x.a = append_args(batch_args(batch, cache), q_heads, cache->heads, rows, interleaved);
    x.a.kc = x.a.vc = nullptr;
    x.c = kv4_arrays(cache);
    const hipError_t e = launch_append_kv4(x, (hipStream_t)stream);
    return e == hipSuccess ? QLIN_OK : hip_fail(e, "append launch");
}

int qlin_unpack_four_bit(const qlin_batch *batch, const qlin_kv4_cache *cache, const qlin_kv_cache *to, int64_t head_dim, int new_only,
                    void *stream) {
    clear_err();
    if (check_batch(batch) != QLIN_OK) return last_status();
    if (!cache || !to) return fail(QLIN_ERR_INVALID, "NULL cache");
    if (cache->heads < 1 || to->heads != cache->heads) return fail(QLIN_ERR_INVALID, "the caches must have the same, positive number of heads");
    if (head_dim != kHeadDim) return fail(QLIN_ERR_UNSUPPORTED, "head_dim must be 128 (got %lld)", (long long)head_dim);
    if (cache->heads > kMaxHeads) return fail(QLIN_ERR_UNSUPPORTED, "at most 4096 heads");
    if (check_kv4(cache) != QLIN_OK || check_cache(to) != QLIN_OK) return last_status();
    if (new_only && batch->max_new == 0) return QLIN_OK;
    if (check_batch_arrays(batch) != QLIN_OK) return last_status();
    const Kv4Ranges c(cache);
    const Range tk = cache_range(to->k, to), tv = cache_range(to->v, to);
    if (c.meet(tk) || c.meet(tv) || overlap(tk, tv)) return fail(QLIN_ERR_INVALID, "the caches overlap");
    if (batch_meets(batch, tk) || batch_meets(batch, tv)) return fail(QLIN_ERR_INVALID, "the cache overlaps new_start, length or cache_start");

    UnpackArgs a = unpack_args(batch, cache, new_only != 0);
    a.k = to->k;
    a.v = to->v;
    a.to_slots = to->slots;
    a.to_seq_slots = to->seq_slots;
    a.to_capacity = to->capacity;
    a.to_tok = to->token_stride;
    a.to_head = to->head_stride;
    const hipError_t e = launch_unpack_kv4(a, (hipStream_t)stream);
    return e == hipSuccess ? QLIN_OK : hip_fail(e, "unpack launch");
}

int qlin_causal_four_bit_plan(const qlin_batch *batch, int64_t q_heads, int64_t kv_heads, int64_t head_dim, int64_t splits,
                         int64_t *splits_out, int64_t *workspace_bytes, char *buf, int64_t buflen) {
    clear_err();
    if (check_batch(batch) != QLIN_OK || check_heads(q_heads, kv_heads, head_dim) != QLIN_OK) return last_status();
    if (splits < 0 || splits > kMaxSplits) return fail(QLIN_ERR_INVALID, "splits must be in [0, 256]");
    Kv4Plan p;
    if (kv4_plan(batch, q_heads, kv_heads, splits, &p) != QLIN_OK) return last_status();
    if (workspace_bytes) *workspace_bytes = p.ws_bytes;
    if (p.rt == 0) {
        char inner[200];
        int64_t S = 1;
        if (qlin_causal_plan(batch, q_heads, kv_heads, head_dim, splits, &S, nullptr, inner, sizeof inner) != QLIN_OK) return last_status();
        if (splits_out) *splits_out = S;
        if (buf && buflen > 0) snprintf(buf, (size_t)buflen, "unpack=%lld %s", (long long)p.unpacked, inner);
        return QLIN_OK;
    }
    if (splits_out) *splits_out = p.S;
    if (buf && buflen > 0)
        snprintf(buf, (size_t)buflen, "kernel=%s splits=%d grid=%lld combine=%d", causal_kv4_kernel_name(p.rt), p.S,
                 (long long)p.tiles * kv_heads * p.S, p.S > 1 ? 1 : 0);
    return QLIN_OK;
}

int qlin_causal_attention_four_bit(const qlin_batch *batch, const qlin_kv4_cache *cache, int64_t q_heads, int64_t head_dim,
                              float scale, int64_t splits, const uint16_t *q, int64_t q_stride, uint16_t *out,
                              int64_t out_stride, void *workspace, int64_t workspace_bytes, void *stream) {
    clear_err();
    if (check_batch(batch) != QLIN_OK) return last_status();
    if (!cache) return fail(QLIN_ERR_INVALID, "NULL cache");
    if (check_heads(q_heads, cache->heads, head_dim) != QLIN_OK || check_kv4(cache) != QLIN_OK) return last_status();
    float factor;
    if (check_attention_values(scale, splits, workspace_bytes, &factor) != QLIN_OK) return last_status();
    if (batch->rows == 0) return QLIN_OK;
    const int64_t w = q_heads * kHeadDim, M = batch->rows;
    if (check_batch_arrays(batch) != QLIN_OK || check_rows(q, q_stride, w, "q") != QLIN_OK || check_rows(out, out_stride, w, "out") != QLIN_OK)
        return last_status();
    if (!aligned(workspace, 16)) return fail(QLIN_ERR_ALIGN, "workspace must be 16-byte aligned");
    const Range ro = rows_range(out, M, out_stride, w);
    const Kv4Ranges c(cache);
    if (rows_meet(q, q_stride, w, out, out_stride, w, M) || c.meet(ro)) return fail(QLIN_ERR_INVALID, "out overlaps q or the cache");
    if (batch_meets(batch, ro)) return fail(QLIN_ERR_INVALID, "out overlaps new_start, length or cache_start");
    Kv4Plan p;
    if (kv4_plan(batch, q_heads, cache->heads, splits, &p) != QLIN_OK) return last_status();
    if (p.ws_bytes > 0 && (!workspace || workspace_bytes < p.ws_bytes))
        return fail(QLIN_ERR_INVALID, "workspace of %lld bytes needed (%lld given)", (long long)p.ws_bytes,
                    (long long)(workspace ? workspace_bytes : 0));
    const Range ws{(uintptr_t)workspace, (size_t)p.ws_bytes};
    if (overlap(ro, ws) || overlap(rows_range(q, M, q_stride, w), ws) || c.meet(ws))
        return fail(QLIN_ERR_INVALID, "the workspace overlaps q, out or the cache");
    if (batch_meets(batch, ws)) return fail(QLIN_ERR_INVALID, "the workspace overlaps new_start, length or cache_start");
    if (batch->max_new == 0) return QLIN_OK;

    if (p.rt == 0) {
        // the cache in f16 first; sequences that count as without cached tokens have length 0 there
        const qlin_kv_cache to = unpacked_cache(batch, cache->heads, workspace);
        const Unpacked at(batch->n_seq, cache->heads, batch->max_len);
        UnpackArgs a = unpack_args(batch, cache, false);
        a.k = to.k;
        a.v = to.v;
        a.to_slots = to.slots;
        a.to_seq_slots = to.seq_slots;
        a.to_capacity = to.capacity;
        a.to_tok = to.token_stride;
        a.to_head = to.head_stride;
        a.length = (int32_t *)((char *)workspace + at.length);
        a.shifts = (HeadShift *)((char *)workspace + at.shifts);
        a.row_shifts = (short2 *)((char *)workspace + at.row_shifts);
        a.peaks = (float4 *)((char *)workspace + at.peaks);
        a.peak_tiles = (int)at.peak_tiles;
        const hipError_t e = launch_unpack_kv4(a, (hipStream_t)stream);
        if (e != hipSuccess) return hip_fail(e, "unpack launch");
        qlin_batch b = *batch;
        b.length = a.length;
        b.cache_start = nullptr;
        return attend_in_f16(&b, &to, a.shifts, a.row_shifts, q_heads, factor, splits, q, q_stride, out, out_stride, (char *)workspace + at.attention, (hipStream_t)stream);
    }
    CausalKv4Args x;
    x.a = CausalArgs{};
    x.a.b = batch_args(batch, cache);
    x.a.b.longest = (int)batch->max_len;
    x.a.q = q;
    x.a.out = out;
    x.a.q_stride = q_stride;
    x.a.out_stride = out_stride;
    x.a.Hq = (int)q_heads;
    x.a.Hkv = (int)cache->heads;
    x.a.G = (int)(q_heads / cache->heads);
    x.a.ws_o = (float *)workspace;
    x.a.ws_ml = x.a.ws_o + (size_t)p.tiles * x.a.Hkv * p.S * causal_tile_rows(p.rt) * kHeadDim;
    x.a.tiles = p.tiles;
    x.a.one_tile = p.one_tile;
    x.a.least = p.least;
    x.a.S = p.S;
    x.a.max_len = (int)batch->max_len;
    gn_reciprocal(x.a.Hkv, &x.a.inv_heads, &x.a.heads_shift);
    x.a.inv_g = x.a.G > 1 ? (uint32_t)((((uint64_t)1 << 32) + x.a.G - 1) / x.a.G) : 0u;
    x.a.c = factor;
    x.c = kv4_arrays(cache);
    const hipError_t e = launch_causal_kv4(x, p.rt, (hipStream_t)stream);
    return e == hipSuccess ? QLIN_OK : hip_fail(e, "causal attention launch");
}

}  // extern "C"
