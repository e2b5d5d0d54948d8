// Attention of the training model's Transformer layers and its backward pass (include/egeria.h has the definition).
#include "attention.hpp"

namespace egeria {

namespace {

bool valid_desc(const egeria_attention_desc *d)
{
    if (!d || (d->dtype != EGERIA_F32 && d->dtype != EGERIA_BF16)) return false;
    if (d->batch < 0 || d->heads < 1 || d->kv_heads < 1 || d->heads % d->kv_heads != 0 || d->q_len < 0 || d->k_len < 0 || d->head_dim < 1) return false;
    if (!(d->scale >= -3.402823466e+38f && d->scale <= 3.402823466e+38f)) return false;
    if (((uintptr_t)d->q_lens & 3u) || ((uintptr_t)d->k_lens & 3u)) return false;
    return !d->bias || valid_position_table(d->bias);
}

// sizes that the kernels' 32-bit counters and the workspace's 64-bit ones hold
bool covered(const egeria_attention_desc *d)
{
    if (d->head_dim > 128 || d->heads > 65535 || d->q_len > (1 << 29) || d->k_len > (1 << 29)) return false;
    const int64_t pairs = (int64_t)d->batch * d->heads;
    return pairs < (1LL << 31) && pairs * d->q_len < (1LL << 38) && pairs * d->k_len < (1LL << 38);
}

// A tensor [batch, len, heads, dim]: 0 as it should be, else the error.  Elements of an output must not overlap: taken by rising
// stride, every dimension's step has to clear what the ones below span.
egeria_status check_view(const egeria_heads *t, const egeria_attention_desc *d, int len, int heads, bool output)
{
    if (!t) return EGERIA_ERR_INVALID_ARG;
    if (t->batch_stride < 0 || t->token_stride < 0 || t->head_stride < 0) return EGERIA_ERR_INVALID_ARG;
    if (d->batch == 0 || len == 0) return EGERIA_OK;
    const size_t size = d->dtype == EGERIA_F32 ? 4 : 2;
    if (!t->data || ((uintptr_t)t->data & (size - 1))) return EGERIA_ERR_INVALID_ARG;
    int64_t n[3] = {d->batch, len, heads}, s[3] = {t->batch_stride, t->token_stride, t->head_stride};
    for (int i = 0; i < 2; ++i)
        for (int k = 0; k < 2 - i; ++k)
            if (s[k] > s[k + 1]) {
                const int64_t u = s[k], w = n[k];
                s[k] = s[k + 1], n[k] = n[k + 1];
                s[k + 1] = u, n[k + 1] = w;
            }
    unsigned __int128 span = (unsigned)d->head_dim;
    for (int i = 0; i < 3; ++i) {
        if (n[i] == 1) continue;
        if (output && (unsigned __int128)s[i] < span) return EGERIA_ERR_INVALID_ARG;
        span += (unsigned __int128)(n[i] - 1) * (unsigned __int128)s[i];
    }
    return span * size < ((unsigned __int128)1 << 62) ? EGERIA_OK : EGERIA_ERR_UNSUPPORTED;
}

View view_of(const egeria_heads *t) { return {(char *)t->data, t->batch_stride, t->token_stride, t->head_stride}; }

AttnArgs make_args(const egeria_attention_desc *d)
{
    AttnArgs a = {};
    a.q_lens = d->q_lens;
    a.k_lens = d->k_lens;
    a.batch = d->batch;
    a.heads = d->heads;
    a.kv_heads = d->kv_heads;
    a.group = d->heads / d->kv_heads;
    a.q_len = d->q_len;
    a.k_len = d->k_len;
    a.dim = d->head_dim;
    a.causal = d->causal ? 1 : 0;
    a.scale = d->scale;
    if (d->bias) {
        a.table = d->bias->table;
        a.table_rows = d->bias->buckets;
        a.b = make_buckets(d->bias);
    }
    return a;
}

int64_t row_tiles(const egeria_attention_desc *d) { return ((int64_t)d->q_len + kRowTile - 1) / kRowTile; }

// Whether every row of a tensor starts on 16 bytes, holds whole units of 16, rows do not overlap and as many as a tile
// has at most span less than 2 GiB.
bool wide_rows(const egeria_heads *t, const egeria_attention_desc *d)
{
    if (t->token_stride < d->head_dim) return false;
    const int64_t size = d->dtype == EGERIA_F32 ? 4 : 2;
    return !((uintptr_t)t->data & 15u) && t->batch_stride * size % 16 == 0 && t->token_stride * size % 16 == 0 && t->head_stride * size % 16 == 0 &&
           d->head_dim * size % 16 == 0 && t->token_stride * size < (0x7fffffffLL - 1024) / (kOnePassKeys > kRowTile ? kOnePassKeys : kRowTile);
}

int64_t few_tiles(const egeria_attention_desc *d)
{
    const int64_t rows = (int64_t)(d->heads / d->kv_heads) * d->q_len;
    return (rows + kFewRows - 1) / kFewRows * d->batch * d->kv_heads;
}

// The forward kernel for few rows, and how many workgroups share a row tile's keys there (0: the other kernel).  A tile of 128 queries
// leaves most of its waves without rows up to 32 queries; and where there are few such tiles, tiles of 32 rows and a share of the
// keys for each wave occupy more of the device.  The border lies between what was measured, 128-row tiles / this way, us: below 48 tiles
// fp32 1 x 512 x 6 x 64 39 / 16, 1 x 130 x 8 x 128 36 / 19, bf16 1 x 1000 x 4 x 128 26 / 18, but 2 x 512 x 5 x 64 12.4 / 15.2; with 48
// bf16 1 x 2048 x 3 x 128 46 / 50, 2 x 512 x 6 x 64 causal 13.0 / 14.8, but fp32 2 x 512 x 6 x 64 39 / 18.  Splits have at least 256
// keys.
int few_splits(const egeria_attention_desc *d)
{
    const int64_t blocks = (int64_t)d->batch * d->heads * (((int64_t)d->q_len + kRowTile - 1) / kRowTile);
    const int64_t tiles = few_tiles(d);
    if (d->q_len > 32 && !(blocks < 48 && d->k_len >= (d->dtype == EGERIA_F32 ? 64 : 512))) return 0;
    if (tiles == 0) return 0;
    // a round of workgroups, if their keys are few; else two, since the sequences' lengths may differ
    const int64_t slots = (int64_t)compute_units() * (d->dtype == EGERIA_BF16 && d->head_dim <= 64 ? 2 : 1);
    int64_t n = slots / tiles;
    if (n < 1 || d->k_len / n > 1024) n = (2 * slots + tiles - 1) / tiles;
    const int64_t most = ((int64_t)d->k_len + 255) / 256;
    n = n > most ? most : n;
    return n < 1 ? 1 : (int)n;
}

// Parts that the steps of a backward kernel's workgroups are dealt in, each a sum in fp32 that a last launch adds up: the number, at
// most 16 and of two steps at least, that ends first when `slots` workgroups run at a time.  A workgroup costs two steps more than it
// has and, to write and join its part, `more`; the last launch half of that.  Causal: half the steps in all, but the longest workgroup
// has all of its own.  (As many parts as one round of two workgroups for each compute unit holds / this count, us, backward: bf16
// causal 1 x 4096 x 9 x 64 203 / 156 and 16384 x 2 (1) x 128 579 / 537, fp32 the former 1196 / 831, 2 x 1049 x 710 keys x 16 (8) x 128 544 /
// 497; but bf16 8 x 512 x 8 x 75 94 / 102.  Without `more`, bf16 causal 6 x 1024 x 12 x 64 takes 109 instead of 86.)
int parts_of(int64_t blocks, int64_t steps, int64_t slots, double more, bool causal)
{
    int best = 1;
    double least = 0.0;
    for (int n = 1; n <= 16 && (n == 1 || 2 * n <= steps); ++n) {
        const double rounds = (double)((blocks * n + slots - 1) / slots), each = (double)((steps + n - 1) / n), all = 0.5 * (double)blocks * (double)steps / (double)slots;
        const double one = 2.0 + (n > 1 ? more : 0.0);
        const double cost = (causal ? (all > each ? all : each) + one * rounds : rounds * (each + one)) + (n > 1 ? 0.5 * more : 0.0);
        if (n == 1 || cost < least) {
            best = n;
            least = cost;
        }
    }
    return best;
}

// The backward kernel that makes everything in one pass: where its keys and LDS fit and a workgroup for each key head of the batch
// gives half the compute units work (two kernels / this one, us: fp32 24 x 197 x 12 x 64 180 / 124, bf16 200 x 128 x 8 x 64 78 / 64; at 130 x
// 100 x 4 x 32 causal 22 / 23).
bool one_pass(const egeria_attention_desc *d)
{
    return d->k_len <= kOnePassKeys && d->head_dim <= 64 && (int64_t)d->batch * d->kv_heads >= 128 && one_pass_lds(d, true) <= kMostLds;
}

struct Plan {
    bool one = false;
    size_t off_delta = 0, off_part = 0, off_o = 0, off_ml = 0, off_q = 0, off_kv = 0, total = 0;
    int splits = 0, q_parts = 1, kv_parts = 1, whole = 0;
    int64_t blocks = 0;                     // workgroups of the largest backward launch
};
Plan make_plan(const egeria_attention_desc *d, bool backward)
{
    Plan p;
    auto take = [&](size_t bytes) { size_t o = p.total; p.total += align_up(bytes, 256); return o; };
    take(256);
    if (backward && one_pass(d)) {
        p.one = true;
        // rounds of as many key heads as run at a time; what the last round would have fewer of is done in parts, so that it is short
        const int64_t units = (int64_t)d->batch * d->kv_heads, slots = (int64_t)compute_units() * (d->k_len <= 128 ? 2 : 1), over = units % slots;
        const int64_t steps = ((int64_t)d->q_len + one_pass_queries(d->dtype) - 1) / one_pass_queries(d->dtype) * (d->heads / d->kv_heads);
        int64_t parts = over ? slots / over : 1;
        const int64_t most = units > slots ? steps : steps / 2;            // (a sum in parts costs a launch: for half a round's steps at least)
        parts = parts > most ? most : parts;
        p.kv_parts = (int)(parts < 1 ? 1 : (parts > 16 ? 16 : parts));
        p.whole = (int)(p.kv_parts > 1 ? units - over : units);
        p.blocks = p.whole + (units - p.whole) * p.kv_parts;
        p.off_part = take((size_t)d->batch * d->heads * p.kv_parts * position_rows(d->bias) * 4);
        if (p.kv_parts > 1) p.off_kv = take((size_t)p.kv_parts * over * d->k_len * padded_dim(d->head_dim) * 8);
        return p;
    }
    if (backward) {
        p.off_delta = take((size_t)d->batch * d->heads * d->q_len * 4);
        const int64_t key_tiles = ((int64_t)d->k_len + kRowTile - 1) / kRowTile, wide = padded_dim(d->head_dim), cu = compute_units();
        // workgroups of the two kernels that a compute unit holds, by their LDS and registers
        const bool f32 = d->dtype == EGERIA_F32, long_rows = d->head_dim > 64;
        const int64_t q_slots = cu * (f32 ? (long_rows ? 1 : 2) : (long_rows ? 2 : 3)), kv_slots = cu * (f32 && long_rows ? 1 : 2);
        const int64_t q_steps = ((int64_t)d->k_len + kKeyTile - 1) / kKeyTile, kv_step = long_rows ? kKeyTile / 2 : kKeyTile;
        const double more = f32 ? 0.9 : 3.5;                                // a part's bytes, written and read again, in steps
        p.q_parts = parts_of((int64_t)d->batch * d->heads * row_tiles(d), q_steps, q_slots, more, d->causal != 0);
        p.kv_parts = parts_of((int64_t)d->batch * d->kv_heads * key_tiles, ((int64_t)d->q_len + kv_step - 1) / kv_step * (d->heads / d->kv_heads), kv_slots,
                              more, d->causal != 0);
        const int64_t q_blocks = (int64_t)d->batch * d->heads * row_tiles(d) * p.q_parts, kv_blocks = (int64_t)d->batch * d->kv_heads * key_tiles * p.kv_parts + d->heads;
        p.blocks = q_blocks > kv_blocks ? q_blocks : kv_blocks;
        p.off_part = take((size_t)q_blocks * position_rows(d->bias) * 4);
        if (p.q_parts > 1) p.off_q = take((size_t)p.q_parts * d->batch * d->heads * d->q_len * wide * 4);
        if (p.kv_parts > 1) p.off_kv = take((size_t)p.kv_parts * d->batch * d->kv_heads * d->k_len * wide * 8);
        return p;
    }
    p.splits = few_splits(d);
    if (p.splits > 1) {
        const size_t rows = (size_t)few_tiles(d) * kFewRows * p.splits;
        p.off_o = take(rows * padded_dim(d->head_dim) * 4);
        p.off_ml = take(rows * 8);
    }
    return p;
}

}  // namespace

}  // namespace egeria

using namespace egeria;

#define EG_TRY(expr)                                       \
    do {                                                   \
        const egeria_status s__ = (expr);                  \
        if (s__ != EGERIA_OK) return s__;                  \
    } while (0)
#define EG_HIP(expr)                                   \
    do {                                               \
        if ((expr) != hipSuccess) return EGERIA_ERR_HIP; \
    } while (0)

extern "C" {

size_t egeria_attention_workspace_bytes(const egeria_attention_desc *desc, int32_t backward)
{
    return valid_desc(desc) && covered(desc) ? make_plan(desc, backward != 0).total : 0;
}

egeria_status egeria_attention(const egeria_attention_desc *desc, const egeria_heads *q, const egeria_heads *k, const egeria_heads *v,
                               const egeria_heads *out, float *lse, void *ws, size_t ws_bytes, void *stream)
{
    if (!valid_desc(desc)) return EGERIA_ERR_INVALID_ARG;
    if (!covered(desc)) return EGERIA_ERR_UNSUPPORTED;
    EG_TRY(check_view(q, desc, desc->q_len, desc->heads, false));
    EG_TRY(check_view(k, desc, desc->k_len, desc->kv_heads, false));
    EG_TRY(check_view(v, desc, desc->k_len, desc->kv_heads, false));
    EG_TRY(check_view(out, desc, desc->q_len, desc->heads, true));
    const int64_t rows = (int64_t)desc->batch * desc->heads * desc->q_len;
    if ((rows > 0 && !lse) || ((uintptr_t)lse & 15u) || !ws || ((uintptr_t)ws & 15u)) return EGERIA_ERR_INVALID_ARG;
    const Plan p = make_plan(desc, false);
    if (ws_bytes < p.total) return EGERIA_ERR_WORKSPACE_TOO_SMALL;
    if (rows == 0) return EGERIA_OK;
    // (the launch that joins splits has fewer threads: 8 for a row of its tiles at most 32, and there are splits where tiles are few)
    if ((p.splits ? few_tiles(desc) * p.splits : row_tiles(desc) * desc->batch * desc->heads) * 256 > kMostThreads) return EGERIA_ERR_UNSUPPORTED;
    AttnArgs a = make_args(desc);
    a.q = view_of(q), a.k = view_of(k), a.v = view_of(v), a.o = view_of(out);
    a.lse = lse;
    a.splits = p.splits;
    a.split_o = (float *)((char *)ws + p.off_o);
    a.split_ml = (float *)((char *)ws + p.off_ml);
    const bool vec = wide_rows(q, desc) && wide_rows(k, desc) && wide_rows(v, desc) && wide_rows(out, desc);
    EG_HIP((p.splits ? launch_attention_few : launch_attention_forward)(a, (egeria_dtype)desc->dtype, vec, (hipStream_t)stream));
    return EGERIA_OK;
}

egeria_status egeria_attention_backward(const egeria_attention_desc *desc, const egeria_heads *dout, const egeria_heads *q,
                                        const egeria_heads *k, const egeria_heads *v, const egeria_heads *out, const float *lse,
                                        const egeria_heads *dq, const egeria_heads *dk, const egeria_heads *dv, float *dtable, void *ws,
                                        size_t ws_bytes, void *stream)
{
    if (!valid_desc(desc)) return EGERIA_ERR_INVALID_ARG;
    if (!covered(desc)) return EGERIA_ERR_UNSUPPORTED;
    for (const egeria_heads *t : {dout, q, out}) EG_TRY(check_view(t, desc, desc->q_len, desc->heads, false));
    for (const egeria_heads *t : {k, v}) EG_TRY(check_view(t, desc, desc->k_len, desc->kv_heads, false));
    EG_TRY(check_view(dq, desc, desc->q_len, desc->heads, true));
    for (const egeria_heads *t : {dk, dv}) EG_TRY(check_view(t, desc, desc->k_len, desc->kv_heads, true));
    const int64_t rows = (int64_t)desc->batch * desc->heads * desc->q_len;
    if ((rows > 0 && !lse) || ((uintptr_t)lse & 15u) || !ws || ((uintptr_t)ws & 15u)) return EGERIA_ERR_INVALID_ARG;
    if ((dtable && !desc->bias) || ((uintptr_t)dtable & 15u)) return EGERIA_ERR_INVALID_ARG;
    const Plan p = make_plan(desc, true);
    if (ws_bytes < p.total) return EGERIA_ERR_WORKSPACE_TOO_SMALL;
    if (p.blocks * (p.one && desc->k_len > 128 ? 512 : 256) > kMostThreads) return EGERIA_ERR_UNSUPPORTED;      // (a wave for 32 keys, four or eight of them)
    AttnArgs a = make_args(desc);
    a.d_o = view_of(dout), a.q = view_of(q), a.k = view_of(k), a.v = view_of(v), a.o = view_of(out);
    a.dq = view_of(dq), a.dk = view_of(dk), a.dv = view_of(dv);
    a.lse = const_cast<float *>(lse);
    a.delta = (float *)((char *)ws + p.off_delta);
    a.partials = dtable ? (float *)((char *)ws + p.off_part) : nullptr;
    a.dtable = dtable;
    a.q_parts = p.q_parts, a.kv_parts = p.kv_parts;
    a.part_q = (float *)((char *)ws + p.off_q), a.part_kv = (float *)((char *)ws + p.off_kv);
    hipStream_t st = (hipStream_t)stream;
    bool vec = true;
    for (const egeria_heads *t : {dout, q, k, v, out, dq, dk, dv}) vec = vec && wide_rows(t, desc);
    a.whole = p.whole;
    a.table_parts = (int64_t)a.batch * (p.one ? a.kv_parts : a.q_parts * row_tiles(desc));
    EG_HIP((p.one ? launch_attention_one_pass : launch_attention_backward)(a, (egeria_dtype)desc->dtype, vec, st));
    return EGERIA_OK;
}

}  // extern "C"
