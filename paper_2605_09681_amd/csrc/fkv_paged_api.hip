// fkv_paged_api.hip -- the entry points of the paged cache of many sequences: checks of
// every argument before anything is enqueued, and the plan of the launches.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>
#include <limits>

#include "paged.h"

namespace {

using fkv::PagedArgs;

fkv_status fail(fkv_status st, const char *fmt, ...) {
    char text[400];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(text, sizeof text, fmt, ap);
    va_end(ap);
    return fkv::api_error(st, text);
}

bool aligned(const void *p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

// floor(2^64 / P) + 1 as two words (0, 0 for P = 1), for j / P by multiplication
void magic_of(int32_t P, uint32_t *hi, uint32_t *lo) {
    *hi = *lo = 0;
    if (P <= 1) return;
    const unsigned __int128 m = (((unsigned __int128)1) << 64) / (uint64_t)P + 1;
    *hi = (uint32_t)(uint64_t)(m >> 32);
    *lo = (uint32_t)(uint64_t)m;
}

// sizes: the workspace queries read no pointers.
fkv_status check_batch(const fkv_batch *b, int32_t n_kv_heads, bool sizes) {
    if (!b) return fail(FKV_ERR_ARG, "batch is NULL");
    if (b->n_seqs < 1 || b->n_seqs > FKV_MAX_SEQS) return fail(FKV_ERR_SHAPE, "n_seqs %d outside [1, %d]", b->n_seqs, FKV_MAX_SEQS);
    if (b->n_tokens < 0 || b->n_tokens > 1 << 24) return fail(FKV_ERR_SHAPE, "n_tokens %d outside [0, 2^24]", b->n_tokens);
    if (b->page_tokens < 1 || b->page_tokens > 1 << 20) return fail(FKV_ERR_SHAPE, "page_tokens %d outside [1, 2^20]", b->page_tokens);
    if (b->n_pages < 1 || b->max_pages < 1) return fail(FKV_ERR_SHAPE, "n_pages %d or max_pages %d below 1", b->n_pages, b->max_pages);
    if ((int64_t)b->n_pages * b->page_tokens > (((int64_t)1 << 31) - 1) / n_kv_heads)
        return fail(FKV_ERR_SHAPE, "%d pages of %d tokens and %d heads: 2^31 rows or more", b->n_pages, b->page_tokens, n_kv_heads);
    if (b->max_new < 1) return fail(FKV_ERR_ARG, "max_new %d below 1", b->max_new);
    if (b->sum_len < 0) return fail(FKV_ERR_ARG, "sum_len %lld below 0", (long long)b->sum_len);
    if (sizes || b->n_tokens == 0) return FKV_OK;
    if (!b->page_table || !b->seq_len || !b->q_start) return fail(FKV_ERR_ARG, "page_table, seq_len or q_start is NULL");
    if (!aligned(b->page_table, 4) || !aligned(b->seq_len, 4) || !aligned(b->q_start, 4))
        return fail(FKV_ERR_ARG, "page_table, seq_len or q_start is not 4-byte aligned");
    return FKV_OK;
}

fkv_status check_heads(int32_t n_heads, int32_t n_kv_heads, int32_t head_dim) {
    if (n_heads < 1 || n_heads > FKV_MAX_HEADS || n_kv_heads < 1 || n_kv_heads > n_heads || n_heads % n_kv_heads)
        return fail(FKV_ERR_SHAPE, "%d heads over %d key heads: at most %d, a whole number to each key head", n_heads, n_kv_heads,
                    FKV_MAX_HEADS);
    if (head_dim != 64 && head_dim != 128) return fail(FKV_ERR_SHAPE, "head_dim %d is not 64 or 128", head_dim);
    return FKV_OK;
}

// Whether rows h * head + t * token of `width` elements share some.
bool overlap(int64_t heads, int64_t tokens, int64_t head, int64_t token, int64_t width) {
    if ((heads > 1 && head < width) || (tokens > 1 && token < width)) return true;
    if (heads == 1 || tokens == 1 || head >= (tokens - 1) * token + width || token >= (heads - 1) * head + width) return false;
    for (int64_t h = 1; h < heads; ++h)                   // the nearest of the tokens before and after
        for (int64_t t = h * head / token; t <= h * head / token + 1; ++t)
            if (t < tokens && std::abs(h * head - t * token) < width) return true;
    return false;
}

// out_width: of rows that are written.
fkv_status check_rows(const fkv_rows *r, int elem, const char *name, int n_heads, int n_tokens, int out_width = 0) {
    if (!r || !r->data) return fail(FKV_ERR_ARG, "%s: NULL tensor pointer", name);
    if (!aligned(r->data, 16)) return fail(FKV_ERR_ARG, "%s is not 16-byte aligned", name);
    const int64_t per = 16 / elem, most = (int64_t)1 << 36;
    if (r->head_stride < 0 || r->token_stride < 0 || r->head_stride % per || r->token_stride % per || r->head_stride > most ||
        r->token_stride > most)
        return fail(FKV_ERR_ARG, "%s: strides %lld and %lld must be multiples of %lld elements in [0, 2^36]", name,
                    (long long)r->head_stride, (long long)r->token_stride, (long long)per);
    if (out_width && overlap(n_heads, n_tokens, r->head_stride, r->token_stride, out_width))
        return fail(FKV_ERR_ARG, "%s: rows of %d elements overlap at strides %lld and %lld", name, out_width,
                    (long long)r->head_stride, (long long)r->token_stride);
    return FKV_OK;
}

fkv_status check_scale(float scale, int32_t causal, const fkv_span *spans, int n) {
    if (!(scale > 0.f) || !isfinite(scale)) return fail(FKV_ERR_ARG, "scale %g must be positive and finite", (double)scale);
    if (causal != 0 && causal != 1) return fail(FKV_ERR_ARG, "causal %d is not 0 or 1", causal);
    for (int y = 0; spans && y < n; ++y)
        if (spans[y].sink_tokens < 0 || spans[y].recent_tokens < -1)
            return fail(FKV_ERR_ARG, "spans[%d]: sink_tokens %d below 0 or recent_tokens %d below -1", y, spans[y].sink_tokens,
                        spans[y].recent_tokens);
    return FKV_OK;
}

void set_batch(PagedArgs *a, const fkv_batch *b) {
    a->table = b->page_table;
    a->seq_len = b->seq_len;
    a->q_start = b->q_start;
    a->n_seqs = b->n_seqs;
    a->max_pages = b->max_pages;
    a->page_tokens = b->page_tokens;
    a->n_pages = b->n_pages;
    a->n_tokens = b->n_tokens;
    a->max_new = std::min(b->max_new, std::max(b->n_tokens, 1));
    a->cap = (int32_t)std::min((int64_t)b->max_pages * b->page_tokens, (int64_t)1 << 30);
    magic_of(b->page_tokens, &a->mp_hi, &a->mp_lo);
    a->lo = 1;
    a->hi = std::numeric_limits<int32_t>::max();
}

void set_span(PagedArgs *a, const fkv_span *spans, int n, bool one) {
    const int32_t most = 1 << 30;
    a->wide = 0;
    a->one_span = 1;
    for (int y = 1; spans && !one && y < n; ++y)
        if (spans[y].sink_tokens != spans[0].sink_tokens || spans[y].recent_tokens != spans[0].recent_tokens) a->one_span = 0;
    for (int y = 0; y < n; ++y) {
        a->sink[y] = spans ? std::min(spans[one ? 0 : y].sink_tokens, most) : 0;
        a->recent[y] = spans ? std::min(spans[one ? 0 : y].recent_tokens, most) : -1;
        if (a->recent[y] < 0) a->wide = -1;
        else if (a->wide >= 0) a->wide = std::max(a->wide, std::min(a->sink[y] + std::min(a->recent[y], most - 1), most));
    }
}

// One attention launch: sequences of lo .. hi new tokens in tiles of `rows` query rows (n * group of
// them to a sequence and key head), split for `target` workgroups.
struct Launch {
    int32_t lo, hi, rows, target, min_tiles;
    int64_t n_items, n_work, n_slots, n_joins;   // items at the most; workgroups, slots, cut items where items are cut
    size_t part_bytes;
};

// few: of the launch for few rows (see few_groups), 0: of the other.
Launch plan(const fkv_batch *b, int kv, int group, int32_t lo, int32_t hi, int rows, int cus, int few, int width) {
    // the workgroups that the device holds at once; a part is worth 128 keys, or 512 to the larger tiles
    const int target = cus * (few ? fkv::few_groups(few, rows) : rows == 256 ? 1 : 2), min_tiles = few ? 4 : 8;
    Launch l;
    l.lo = lo;
    l.hi = hi;
    l.rows = rows;
    l.target = target;
    l.min_tiles = min_tiles;
    // row tiles: one for every `rows` rows of the batch, and one more a sequence; no more than the longest sequence's of each
    const int64_t most = std::min(std::min(b->max_new, b->n_tokens), hi), seqs = std::min(b->n_seqs, b->n_tokens);
    const int64_t tiles = std::min((int64_t)b->n_tokens * group / rows + seqs, seqs * ((most * group + rows - 1) / rows));
    // few rows: the items, and the parts that cuts add; a sequence is cut only if its tiles are more than one
    // part's, so parts of cut ones are at most twice the target.  Many rows: a share and two slots to a workgroup.
    l.n_items = tiles * kv;
    l.n_work = few ? l.n_items + target + 8 : target;
    l.n_slots = 2 * (int64_t)target + (few ? 64 : 0);
    l.n_joins = few ? std::min(l.n_items, l.n_slots / 2) : target;
    l.part_bytes = l.n_joins * sizeof(fkv::JoinItem) + (size_t)l.n_slots * rows * fkv::part_width(width) * 4;
    return l;
}

void set_launch(PagedArgs *a, const Launch &l, void *part, bool split) {
    a->lo = l.lo;
    a->hi = l.hi;
    a->target = split ? l.target : 0;
    a->min_tiles = l.min_tiles;
    a->n_work = (int32_t)(split ? l.n_work : l.n_items);
    a->n_slots = (int32_t)l.n_slots;
    a->joins = (fkv::JoinItem *)part;
    a->n_joins = (int32_t)l.n_joins;
    a->part = (float *)((char *)part + l.n_joins * sizeof(fkv::JoinItem));
    magic_of(a->group, &a->g_hi, &a->g_lo);
}

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

// Query rows of a sequence and key head up to which the launch for few rows takes it: a tile of its own, or, where the
// batch's keys are known to be few, four.  The other launch reaches three times its rate, once there is work for the
// device (us, few / many): 12 heads of 128, 3000 tokens, 128 new 26 / 50; 20000 tokens, 192 new 80 / 101, 384 new 137 /
// 106; 16 heads over 4, 20000 tokens, 48 new 40 / 83; 16 sequences of 4000 tokens, 12 heads, 128 new 204 / 144.
int few_rows(const fkv_batch *b, int kv) { return b->sum_len > 0 && b->sum_len <= ((int64_t)1 << 18) / kv ? 256 : 64; }

// Query rows of a tile of the launch for many rows, by the most rows of a sequence and key head.
int tile_rows(int64_t rows) { return rows > 512 ? 256 : 128; }

struct AttendPlan {
    bool few, many;
    Launch f, m;
    size_t bytes;
};

AttendPlan attend_plan(const fkv_batch *b, int n_heads, int kv, int head_dim, int cus) {
    AttendPlan p;
    memset(&p, 0, sizeof p);
    const int group = n_heads / kv, edge = few_rows(b, kv) / group;   // new tokens of a sequence: few up to edge
    const int most = std::min(b->max_new, std::max(b->n_tokens, 1));
    p.many = most > edge;
    p.few = !p.many || b->n_seqs > 1;
    if (p.few)
        p.f = plan(b, kv, group, 1, edge, fkv::paged_row_tile((int)std::min((int64_t)std::min(most, edge) * group, (int64_t)64)), cus, -head_dim, head_dim);
    if (p.many)
        p.m = plan(b, kv, group, p.few ? edge + 1 : 1, std::numeric_limits<int32_t>::max(), tile_rows((int64_t)most * group), cus, 0, head_dim);
    p.bytes = std::max(p.f.part_bytes, p.m.part_bytes);
    return p;
}

struct LatentPlan {
    bool absorbed, expanded;
    Launch f, m;
    int64_t head_rows;
    size_t owned_at, q_at, o_at, k_at, v_at, part_at, bytes;
};

LatentPlan latent_plan(const fkv_batch *b, int n_heads, int d, int R, int form, int cus) {
    LatentPlan p;
    memset(&p, 0, sizeof p);
    const int most = std::min(b->max_new, std::max(b->n_tokens, 1)), all = std::numeric_limits<int32_t>::max();
    // (expanded copies have room for sum_len tokens: where that is not known, the other form serves them all)
    p.expanded = form == FKV_LATENT_EXPANDED || (form == FKV_LATENT_AUTO && most >= FKV_LATENT_FEW && b->sum_len > 0);
    p.absorbed = form == FKV_LATENT_ABSORBED || (form == FKV_LATENT_AUTO && (!p.expanded || b->n_seqs > 1));
    size_t at = 0;
    auto take = [&](size_t n) {
        const size_t here = at;
        at += round256(n);
        return here;
    };
    const size_t rows = (size_t)b->n_tokens * n_heads;
    if (p.absorbed) {
        const int hi = p.expanded ? FKV_LATENT_FEW - 1 : all;
        p.f = plan(b, 1, n_heads, 1, hi, fkv::paged_row_tile((int)std::min<int64_t>((int64_t)std::min(most, hi) * n_heads, 64)), cus, R, R);
        p.owned_at = take((size_t)b->n_tokens * 4);
        p.q_at = take(rows * (R + FKV_LATENT_ROT) * 2);
        p.o_at = take(rows * R * 4);
    }
    if (p.expanded) {
        p.m = plan(b, n_heads, 1, p.absorbed ? FKV_LATENT_FEW : 1, all, 256, cus, 0, d);
        const int64_t block = fkv::paged::kSeqRows;
        p.head_rows = ((b->sum_len + block - 1) / block + b->n_seqs) * block;
        p.k_at = take((size_t)n_heads * p.head_rows * (d + FKV_LATENT_ROT) * 2);
        p.v_at = take((size_t)n_heads * p.head_rows * d * 2);
    }
    p.part_at = take(std::max(p.f.part_bytes, p.m.part_bytes));
    p.bytes = at;
    return p;
}

fkv_status check_work(const Launch &l) {
    // (a launch holds fewer than 2^32 threads, at most 512 in a workgroup)
    return l.n_items >= (int64_t)1 << 22 ? fail(FKV_ERR_SHAPE, "%lld tiles of query rows are too many for one call", (long long)l.n_items)
                                        : FKV_OK;
}

fkv_status done(hipError_t e, const char *what) {
    return e == hipSuccess ? fkv::api_ok() : fail(FKV_ERR_DEVICE, "%s: %s", what, hipGetErrorString(e));
}

fkv_status check_latent(const fkv_batch *b, int32_t n_heads, int32_t head_dim, int32_t latent_dim, int32_t form, bool sizes) {
    fkv_status st;
    if ((st = check_heads(n_heads, 1, head_dim)) != FKV_OK) return st;
    if (latent_dim != 256 && latent_dim != 512) return fail(FKV_ERR_SHAPE, "latent_dim %d is not 256 or 512", latent_dim);
    if (form < FKV_LATENT_AUTO || form > FKV_LATENT_EXPANDED) return fail(FKV_ERR_ARG, "form %d is not an fkv_latent_form", form);
    if ((st = check_batch(b, 1, sizes)) != FKV_OK) return st;
    if (b->sum_len > (int64_t)1 << 30) return fail(FKV_ERR_SHAPE, "sum_len %lld above 2^30", (long long)b->sum_len);
    const LatentPlan p = latent_plan(b, n_heads, head_dim, latent_dim, form, 8);
    if (p.head_rows / fkv::paged::kSeqRows > 65535 || p.head_rows * (head_dim + FKV_LATENT_ROT) * 2 >= (int64_t)1 << 32)
        return fail(FKV_ERR_SHAPE, "sum_len %lld is too large for the expanded form", (long long)b->sum_len);
    return FKV_OK;
}

}  // namespace

extern "C" {

fkv_status fkv_append_paged(const fkv_batch *batch, int32_t n_heads, int32_t head_dim, int32_t dtype, const fkv_rows *K_new,
                            const fkv_rows *V_new, void *K_pages, void *V_pages, void *stream) {
    fkv_status st;
    if (dtype != FKV_BF16 && dtype != FKV_F32) return fail(FKV_ERR_ARG, "dtype %d is not FKV_BF16 or FKV_F32", dtype);
    if (n_heads < 1 || n_heads > FKV_MAX_HEADS) return fail(FKV_ERR_SHAPE, "n_heads %d outside [1, %d]", n_heads, FKV_MAX_HEADS);
    const int es = dtype == FKV_BF16 ? 2 : 4;
    if (head_dim < 1 || head_dim > 16384 / es || head_dim * es % 16)
        return fail(FKV_ERR_SHAPE, "rows of %d elements: a multiple of 16 bytes, at most 16384, are taken", head_dim);
    if ((st = check_batch(batch, n_heads, false)) != FKV_OK) return st;
    if (batch->n_tokens == 0) return fkv::api_ok();
    if ((V_new == nullptr) != (V_pages == nullptr)) return fail(FKV_ERR_ARG, "V_new and V_pages must both be given or both be NULL");
    if ((st = check_rows(K_new, es, "K_new", n_heads, batch->n_tokens)) != FKV_OK) return st;
    if (V_new && (st = check_rows(V_new, es, "V_new", n_heads, batch->n_tokens)) != FKV_OK) return st;
    if (!K_pages) return fail(FKV_ERR_ARG, "K_pages is NULL");
    if (!aligned(K_pages, 16) || !aligned(V_pages, 16)) return fail(FKV_ERR_ARG, "K_pages or V_pages is not 16-byte aligned");
    fkv::PagedAppendArgs a;
    memset(&a, 0, sizeof a);
    set_batch(&a.batch, batch);
    const fkv_rows *rows[2] = {K_new, V_new};
    void *pages[2] = {K_pages, V_pages};
    for (int w = 0; w < 2; ++w) {
        if (!rows[w]) continue;
        a.src[w] = (const uint8_t *)rows[w]->data;
        a.dst[w] = (uint8_t *)pages[w];
        a.tok[w] = rows[w]->token_stride * es;
        a.head[w] = rows[w]->head_stride * es;
    }
    a.heads = n_heads;
    a.chunks = head_dim * es / 16;
    magic_of(a.chunks, &a.chunks_hi, &a.chunks_lo);
    magic_of(a.heads, &a.heads_hi, &a.heads_lo);
    // (a launch holds fewer than 2^32 threads)
    a.block_tokens = std::max(batch->n_tokens < 1 << 23 ? 1 : 2, std::min(64, 1024 / (a.heads * a.chunks)));
    (void)hipGetLastError();
    return done(fkv::launch_paged_append(a, (hipStream_t)stream), "fkv_append_paged launch");
}

fkv_status fkv_paged_attention_workspace_size(const fkv_batch *batch, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                                              size_t *bytes) {
    fkv_status st;
    if ((st = check_heads(n_heads, n_kv_heads, head_dim)) != FKV_OK) return st;
    if ((st = check_batch(batch, n_kv_heads, true)) != FKV_OK) return st;
    if (!bytes) return fail(FKV_ERR_ARG, "bytes is NULL");
    int cus = 0;
    if ((st = fkv::api_compute_units(&cus)) != FKV_OK) return st;
    *bytes = attend_plan(batch, n_heads, n_kv_heads, head_dim, cus).bytes;
    return fkv::api_ok();
}

fkv_status fkv_paged_attention(const fkv_batch *batch, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, const fkv_rows *Q,
                               const void *K_pages, const void *V_pages, int32_t causal, const fkv_span *spans, float scale,
                               const fkv_rows *O, float *lse, void *workspace, size_t workspace_bytes, void *stream) {
    fkv_status st;
    if ((st = check_heads(n_heads, n_kv_heads, head_dim)) != FKV_OK) return st;
    if ((st = check_batch(batch, n_kv_heads, false)) != FKV_OK) return st;
    if ((st = check_scale(scale, causal, spans, n_kv_heads)) != FKV_OK) return st;
    if (batch->n_tokens == 0) return fkv::api_ok();
    if ((st = check_rows(Q, 2, "Q", n_heads, batch->n_tokens)) != FKV_OK) return st;
    if ((st = check_rows(O, 2, "O", n_heads, batch->n_tokens, head_dim)) != FKV_OK) return st;
    if (!K_pages || !V_pages) return fail(FKV_ERR_ARG, "K_pages or V_pages is NULL");
    if (!aligned(K_pages, 16) || !aligned(V_pages, 16) || !aligned(workspace, 16) || !aligned(lse, 4))
        return fail(FKV_ERR_ARG, "K_pages, V_pages, the workspace or lse is not aligned");
    int cus = 8;
    if (workspace && (st = fkv::api_compute_units(&cus)) != FKV_OK) return st;
    const AttendPlan p = attend_plan(batch, n_heads, n_kv_heads, head_dim, cus);
    if (workspace && workspace_bytes < p.bytes)
        return fail(FKV_ERR_CAPACITY, "workspace of %zu bytes, %zu needed", workspace_bytes, p.bytes);
    if ((st = check_work(p.f)) != FKV_OK || (st = check_work(p.m)) != FKV_OK) return st;
    PagedArgs a;
    memset(&a, 0, sizeof a);
    set_batch(&a, batch);
    a.Q = (const uint16_t *)Q->data;
    a.q_tok = Q->token_stride;
    a.q_head = Q->head_stride;
    a.K = (const uint16_t *)K_pages;
    a.V = (const uint16_t *)V_pages;
    a.O = (uint16_t *)O->data;
    a.o_tok = O->token_stride;
    a.o_head = O->head_stride;
    a.lse = lse;
    a.n_heads = n_heads;
    a.kv = n_kv_heads;
    a.group = n_heads / n_kv_heads;
    a.causal = causal;
    a.scale_log2 = std::min(scale * 1.4426950408889634f, std::numeric_limits<float>::max());
    set_span(&a, spans, n_kv_heads, false);
    (void)hipGetLastError();
    hipError_t e = hipSuccess;
    if (p.few) {
        set_launch(&a, p.f, workspace, workspace != nullptr);
        e = fkv::launch_paged_attention(a, head_dim, p.f.rows, (hipStream_t)stream);
    }
    if (e == hipSuccess && p.many) {
        set_launch(&a, p.m, workspace, workspace != nullptr);
        e = fkv::launch_paged_tiles(a, head_dim, p.m.rows, (hipStream_t)stream);
    }
    return done(e, "fkv_paged_attention launch");
}

fkv_status fkv_latent_attention_workspace_size(const fkv_batch *batch, int32_t n_heads, int32_t head_dim, int32_t latent_dim,
                                               int32_t form, size_t *bytes) {
    fkv_status st;
    if ((st = check_latent(batch, n_heads, head_dim, latent_dim, form, true)) != FKV_OK) return st;
    if (!bytes) return fail(FKV_ERR_ARG, "bytes is NULL");
    int cus = 0;
    if ((st = fkv::api_compute_units(&cus)) != FKV_OK) return st;
    *bytes = latent_plan(batch, n_heads, head_dim, latent_dim, form, cus).bytes;
    return fkv::api_ok();
}

fkv_status fkv_latent_attention(const fkv_batch *batch, int32_t n_heads, int32_t head_dim, int32_t latent_dim, const fkv_rows *Q,
                                const void *pages, const void *W_k, const void *W_v, int32_t causal, const fkv_span *span,
                                float scale, const fkv_rows *O, int32_t form, void *workspace, size_t workspace_bytes,
                                void *stream) {
    fkv_status st;
    if ((st = check_latent(batch, n_heads, head_dim, latent_dim, form, false)) != FKV_OK) return st;
    if ((st = check_scale(scale, causal, span, 1)) != FKV_OK) return st;
    if (batch->n_tokens == 0) return fkv::api_ok();
    if ((st = check_rows(Q, 2, "Q", n_heads, batch->n_tokens)) != FKV_OK) return st;
    if ((st = check_rows(O, 2, "O", n_heads, batch->n_tokens, head_dim)) != FKV_OK) return st;
    if (!pages || !W_k || !W_v || !workspace) return fail(FKV_ERR_ARG, "pages, W_k, W_v or the workspace is NULL");
    if (!aligned(pages, 16) || !aligned(W_k, 16) || !aligned(W_v, 16) || !aligned(workspace, 256))
        return fail(FKV_ERR_ARG, "pages, W_k or W_v is not 16-byte aligned, or the workspace not 256-byte aligned");
    int cus = 0;
    if ((st = fkv::api_compute_units(&cus)) != FKV_OK) return st;
    const LatentPlan p = latent_plan(batch, n_heads, head_dim, latent_dim, form, cus);
    if (workspace_bytes < p.bytes) return fail(FKV_ERR_CAPACITY, "workspace of %zu bytes, %zu needed", workspace_bytes, p.bytes);
    if ((st = check_work(p.f)) != FKV_OK || (st = check_work(p.m)) != FKV_OK) return st;
    char *ws = (char *)workspace;
    fkv::LatentArgs a;
    memset(&a, 0, sizeof a);
    set_batch(&a.p, batch);
    a.p.Q = (const uint16_t *)Q->data;
    a.p.q_tok = Q->token_stride;
    a.p.q_head = Q->head_stride;
    a.p.K = (const uint16_t *)pages;
    a.p.O = (uint16_t *)O->data;
    a.p.o_tok = O->token_stride;
    a.p.o_head = O->head_stride;
    a.p.n_heads = n_heads;
    a.p.causal = causal;
    a.p.scale_log2 = std::min(scale * 1.4426950408889634f, std::numeric_limits<float>::max());
    a.W_k = (const uint16_t *)W_k;
    a.W_v = (const uint16_t *)W_v;
    a.R = latent_dim;
    a.p.kv = 1;
    a.p.group = n_heads;
    set_span(&a.p, span, 1, true);
    const hipStream_t s = (hipStream_t)stream;
    (void)hipGetLastError();
    hipError_t e = hipSuccess;
    if (p.absorbed) {
        a.owned = (int32_t *)(ws + p.owned_at);
        a.q_abs = (uint16_t *)(ws + p.q_at);
        a.o_abs = (float *)(ws + p.o_at);
        set_launch(&a.p, p.f, ws + p.part_at, true);
        PagedArgs rows = a.p;
        rows.Q = a.q_abs;
        rows.q_head = latent_dim + FKV_LATENT_ROT;
        rows.q_tok = n_heads * rows.q_head;
        rows.O = (uint16_t *)a.o_abs;                      // (fp32 rows)
        rows.o_head = latent_dim;
        rows.o_tok = (int64_t)n_heads * latent_dim;
        e = fkv::launch_latent_absorb(a, head_dim, s);
        if (e == hipSuccess) e = fkv::launch_latent_rows(rows, latent_dim, p.f.rows, s);
        if (e == hipSuccess) e = fkv::launch_latent_unabsorb(a, head_dim, s);
    }
    if (e == hipSuccess && p.expanded) {
        a.K_exp = (uint16_t *)(ws + p.k_at);
        a.V_exp = (uint16_t *)(ws + p.v_at);
        set_launch(&a.p, p.m, ws + p.part_at, true);
        a.p.head_rows = p.head_rows;
        e = fkv::launch_latent_expand(a, head_dim, s);
        PagedArgs tiles = a.p;
        tiles.K = a.K_exp;
        tiles.V = a.V_exp;
        tiles.kv = n_heads;
        tiles.group = 1;
        magic_of(1, &tiles.g_hi, &tiles.g_lo);
        set_span(&tiles, span, n_heads, true);
        if (e == hipSuccess) e = fkv::launch_expanded_tiles(tiles, head_dim, s);
    }
    return done(e, "fkv_latent_attention launch");
}

}  // extern "C"
