// paged.h -- the paged cache of many sequences as the kernels see it: the batch,
// which keys a query row sees, and how the work is split over the workgroups.
//
// Sequence i has len tokens in the cache; its last n are new, rows start ..
// start + n - 1 of the batch's tensors.  With `group` query heads to a key head, the
// query rows of one key head are r = token * group + (head within the group), so heads
// that share keys share tiles.  Lengths, starts and the page table are device data that
// a captured graph may change between replays: every value is held to its range here, and
// the split over workgroups is worked out from them by every wave (two or three passes over
// the sequences, 64 a step: 2 us for up to 64 of them, some 20 for 1024), not on the host.
#pragma once

#include "fkv_internal.h"

namespace fkv {

// A cut item, as the launch that computes its parts leaves it for the one that joins them.
struct JoinItem {
    int32_t rows;                   // query rows; 0: none
    int32_t start, len, first;      // of its sequence
    int32_t y, row0;                // key head, first query row
    int32_t parts, slot, step;      // few rows: slots slot + step * part; many rows: `parts` workgroups from slot's on
    int32_t goes_on;                // many rows: this workgroup's share begins with a part of an item (its slot 2 r)
    int32_t count;                  // few rows, in the first: cut items of the launch
    int32_t pad[5];
};

// Every tensor that the paged kernels take; also the launch's plan.
struct PagedArgs {
    const uint16_t *Q, *K, *V;      // rows; page pools [n_pages][kv][page_tokens][d] (or the expanded copies)
    uint16_t *O;
    float *lse;                     // [n_heads][n_tokens], may be NULL
    int64_t q_tok, q_head, o_tok, o_head;   // elements
    const int32_t *table, *seq_len, *q_start;
    int32_t n_seqs, max_pages, page_tokens, n_pages, n_tokens, max_new, cap;   // cap: tokens that a table row holds
    uint32_t mp_hi, mp_lo;          // floor(2^64 / page_tokens) + 1 (0 for 1)
    int32_t n_heads, kv, group;
    uint32_t g_hi, g_lo;            // magic of group
    int32_t causal;
    float scale_log2;               // scale * log2(e), finite
    // The launch takes the sequences with lo <= new tokens <= hi.
    int32_t lo, hi;
    int32_t target;                 // workgroups to split for; 0: no workspace, no split
    int32_t min_tiles;              // key tiles that a part is worth
    int32_t n_work, n_slots;        // workgroups launched, slots in `part`
    float *part;
    JoinItem *joins;                // few rows: [n_joins] cut items; many rows: one a workgroup
    int32_t n_joins;
    int32_t one_span;               // every key head has the same span
    int32_t wide;                   // the most keys outside the new tokens that a head sees; < 0: all
    int64_t head_rows;              // expanded copies: rows per head
    int32_t sink[FKV_MAX_HEADS], recent[FKV_MAX_HEADS];   // per key head; recent < 0: every key
};

constexpr int kLatentRot = FKV_LATENT_ROT;

// Attention of rows-per-tile (16, 32, 48, 64) query rows, its parts joined (k_paged_attn.hip).
hipError_t launch_paged_attention(const PagedArgs &a, int head_dim, int rows, hipStream_t s);
hipError_t launch_latent_rows(const PagedArgs &a, int latent_dim, int rows, hipStream_t s);
// Attention of tiles of 128 or 256 query rows, its parts joined (k_paged_tile.hip).
hipError_t launch_paged_tiles(const PagedArgs &a, int head_dim, int rows, hipStream_t s);
hipError_t launch_expanded_tiles(const PagedArgs &a, int head_dim, hipStream_t s);   // 256
// Workgroups of that kernel that share a CU, by its registers and LDS: head_dim 64 or 128, negative, or latent_dim.
constexpr int few_groups(int dim, int rows) {
    return dim == -64 ? (rows <= 16 ? 5 : rows <= 32 ? 4 : 3) : dim == -128 ? (rows <= 32 ? 3 : 2) : dim == 256 && rows <= 32 ? 2 : 1;
}
constexpr int few_waves(int dim, int rows) { return few_groups(dim, rows) * (dim < 0 ? 1 : 2); }   // per SIMD
// Floats of a row of a part's slot: its output, its reference, the sum of its weights as they weigh the values, and as
// they are (for lse).  A slot holds all rows' outputs, then their references and sums.
constexpr int part_width(int d) { return d + 3; }
inline int paged_row_tile(int rows) { return rows <= 64 ? (rows + 15) / 16 * 16 : 64; }

// Rows into the pages (k_paged_append.hip).
struct PagedAppendArgs {
    const uint8_t *src[2];          // keys, values (NULL: left out)
    uint8_t *dst[2];                // pools [n_pages][heads][page_tokens][row]
    int64_t tok[2], head[2];        // bytes
    int32_t heads, chunks;          // 16-byte chunks per row
    uint32_t chunks_hi, chunks_lo, heads_hi, heads_lo;   // magic, as mp_hi, mp_lo
    int32_t block_tokens;           // tokens per workgroup, at most 64
    PagedArgs batch;                // its batch fields
};
hipError_t launch_paged_append(const PagedAppendArgs &a, hipStream_t s);

// Latent attention's products (k_latent.hip).
struct LatentArgs {
    PagedArgs p;                    // Q: the caller's rows, K: the latent pool, O: the caller's output
    const uint16_t *W_k, *W_v;      // [n_heads][d][R]
    int32_t R;
    uint16_t *q_abs;                // absorbed: [n_tokens][n_heads][R + 64]
    float *o_abs;                   // absorbed: [n_tokens][n_heads][R]
    int32_t *owned;                 // absorbed: [n_tokens], 1 where a sequence of the launch holds the token
    uint16_t *K_exp, *V_exp;        // expanded: [n_heads][head_rows][d + 64], [n_heads][head_rows][d]
};
hipError_t launch_latent_absorb(const LatentArgs &a, int head_dim, hipStream_t s);
hipError_t launch_latent_unabsorb(const LatentArgs &a, int head_dim, hipStream_t s);
hipError_t launch_latent_expand(const LatentArgs &a, int head_dim, hipStream_t s);

namespace paged {

constexpr int kSeqRows = 256;       // rows of the expanded copies are dealt to sequences in these

__device__ __forceinline__ float neg_inf() { return -__builtin_inff(); }

// j / P for 0 <= j < 2^31 with floor(2^64 / P) + 1 = hi * 2^32 + lo (0 for P = 1).
__device__ __forceinline__ int div_magic(int j, uint32_t hi, uint32_t lo) {
    if (hi == 0 && lo == 0) return j;
    return (int)(((uint64_t)(uint32_t)j * hi + __umulhi((uint32_t)j, lo)) >> 32);
}

// Sums over the lanes of a wave before and at each (DPP: no trip through LDS); the last lane's is the sum of all.
__device__ __forceinline__ int scan_sum(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);   // row_shr 1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // row_bcast 15, 31
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
    return x;
}
// The largest of the lanes before and at each, of values >= 0.
__device__ __forceinline__ int scan_max(int x) {
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));
    return x;
}
__device__ __forceinline__ float sum_of(float x) {
    auto add = [&](float y, int bits) { return y + __int_as_float(bits); };
    x = add(x, __builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x111, 0xf, 0xf, false));
    x = add(x, __builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x112, 0xf, 0xf, false));
    x = add(x, __builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x114, 0xf, 0xf, false));
    x = add(x, __builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x118, 0xf, 0xf, false));
    x = add(x, __builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x142, 0xa, 0xf, false));
    x = add(x, __builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x143, 0xc, 0xf, false));
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}

struct Seq {
    int len, start, n, first;       // first: position of the first new token (negative: more new tokens than tokens)
};

// This lane's of the sequences i0 .. i0 + 63; every lane of a wave calls it, for i0 = 0, 64, ... in turn.  *held: the
// largest start before i0 (0 at first), then the largest before i0 + 64.  A start is held to the largest before
// it, so that a row belongs to one sequence at most and all sequences' rows are no more than the batch has, which
// the host's bounds on items, slots and joins rest on.
__device__ __forceinline__ Seq sequence(const PagedArgs &a, int i0, int *held) {
    const int i = i0 + (threadIdx.x & 63), k = min(i, a.n_seqs - 1);
    const int len = a.seq_len[k], from = a.q_start[k], to = a.q_start[k + 1];
    // (lanes behind the last sequence: its end)
    int end = min(max(to, 0), a.n_tokens), start = i < a.n_seqs ? min(max(from, 0), a.n_tokens) : end;
    // A branch: with the maximum taken in any case and loads between its steps, attention of one token each of 1024
    // sequences of 100 took 147 us instead of 103.
    if (__ballot(end < start || start < *held) != 0) {
        start = max(scan_max(start), *held);
        end = max(end, start);
    }
    *held = __builtin_amdgcn_readlane(end, 63);
    Seq s = {0, 0, 0, 0};
    if (i < a.n_seqs) {
        s.len = min(max(len, 0), a.cap);
        s.start = start;
        s.n = min(end - start, a.max_new);
        s.first = s.len - (end - start);
    }
    return s;
}

// Token of query row r (of a sequence and key head).
__device__ __forceinline__ int token_of(const PagedArgs &a, int r) { return div_magic(r, a.g_hi, a.g_lo); }

// Which keys of a sequence the query rows of a token see: j < end and (j < sink or j >= low).
struct Sight {
    int end, low;
};
__device__ __forceinline__ Sight sight(const PagedArgs &a, const Seq &s, int recent, int token) {
    const int p = a.causal ? s.first + token : s.first;
    return Sight{a.causal ? min(p + 1, s.len) : s.len, recent < 0 ? 0 : p - recent};
}
__device__ __forceinline__ bool sees(const Sight &v, int sink, int j) { return j < v.end && (j < sink || j >= v.low); }
// No key at all (a sequence without tokens, a position before 0, or an expanded copy that ends before what the row sees).
__device__ __forceinline__ bool blind(const Sight &v, int sink) { return v.end <= 0 || (sink <= 0 && v.low >= v.end); }

// The key tiles that tokens t0 .. t1 of a sequence visit: [0, a_tiles) and, from tile
// b_first on, the others; KT keys each.
struct Tiles {
    int a_tiles, b_first, n;
    Sight least, most;              // what every row of the tile sees at the least, and some row at the most
    __device__ __forceinline__ int key(int t, int kt) const { return (t < a_tiles ? t : b_first + t - a_tiles) * kt; }
};
template <int KT>
__device__ __forceinline__ Tiles tiles_of(const PagedArgs &a, const Seq &s, int sink, int recent, int t0, int t1) {
    const Sight f = sight(a, s, recent, t0), l = sight(a, s, recent, t1);
    Tiles x;
    x.least = Sight{f.end, l.low};
    x.most = Sight{l.end, f.low};
    const int end = (max(l.end, 0) + KT - 1) / KT, low = min(max(f.low, 0) / KT, end);
    x.b_first = low;
    x.a_tiles = min((min(sink, max(l.end, 0)) + KT - 1) / KT, low);
    x.n = x.a_tiles + end - low;
    return x;
}
// Keys j0 .. j0 + KT - 1 are seen by every row.
template <int KT>
__device__ __forceinline__ bool all_seen(const Tiles &x, int sink, int j0) {
    return j0 + KT <= x.least.end && (j0 + KT <= sink || j0 >= x.least.low);
}

// One workgroup's work: part `part` of `parts` of row tile rt of key head y of a sequence.
struct Work {
    Seq s;
    int i;                          // the sequence
    int y, rt, part, parts;
    int slot;                       // of the item's part 0; the next part's is `step` further
    int step;
    int join;                       // number of the item among the cut ones
    bool ok;
};

// a / b for 0 <= a < 2^24, b >= 1 (an integer division is some 40 instructions).
__device__ __forceinline__ int quotient(int a, int b) {
    const int q = (int)((float)a * __builtin_amdgcn_rcpf((float)b)), r = a - q * b;
    return q + (r >= b) - (r < 0);
}

// The launch's split: keys are dealt in parts of some tiles.  That is the least size, from an
// equal share of all tiles for `target` workgroups up to twice the share, in kSizes steps, with which
// the parts are no more than `target`: a workgroup too many would start when the others have ended.  Where
// there are more items than that, only those of more than twice the share are cut.  A sequence's items are all
// cut alike, its parts dealt evenly over each item's tiles.
template <int ROWS, int KT>
struct Split {
    static constexpr int kSizes = 8;
    float per_tile;                 // parts a tile; 0: nothing is cut
    Seq first;                      // this lane's sequence of the first 64
    int first_held;                 // the largest start of those (see sequence)

    // Row tiles of this lane's sequence, 0 if the launch does not take it; the most key tiles of an item.
    static __device__ __forceinline__ void counts(const PagedArgs &a, const Seq &s, int *rts, int *tiles) {
        const bool mine = s.n > 0 && s.n >= a.lo && s.n <= a.hi;
        *rts = mine ? (int)(((uint32_t)s.n * (uint32_t)a.group + ROWS - 1) / ROWS) : 0;    // (n, group: 24 and 7 bits)
        const int keys = a.wide < 0 ? s.len : (int)min((int64_t)s.len, (int64_t)a.wide + s.n + 2 * KT);
        *tiles = max((keys + KT - 1) / KT, 1);
    }
    __device__ __forceinline__ Seq of(const PagedArgs &a, int i0, int *held) const {
        if (i0 > 0) return sequence(a, i0, held);
        *held = first_held;
        return first;
    }
    __device__ __forceinline__ int parts(int tiles) const { return max((int)ceilf((float)tiles * per_tile), 1); }

    __device__ __forceinline__ explicit Split(const PagedArgs &a) {
        first_held = 0;
        first = sequence(a, 0, &first_held);
        per_tile = 0.f;
        if (a.target <= 0) return;
        float sum = 0.f;
        for (int i0 = 0, held = 0; i0 < a.n_seqs; i0 += 64) {
            int rts, tiles;
            counts(a, of(a, i0, &held), &rts, &tiles);
            sum += (float)rts * (float)tiles;
        }
        const float share = sum_of(sum) * (float)a.kv / (float)a.target;
        float per[kSizes], total[kSizes];
#pragma unroll
        for (int k = 0; k < kSizes; ++k) {
            per[k] = __builtin_amdgcn_rcpf(fmaxf((float)a.min_tiles, ceilf(share * (1.f + (float)(k * k) / ((kSizes - 1) * (kSizes - 1))))));
            total[k] = 0.f;
        }
        per_tile = per[kSizes - 1];
        if ((int64_t)a.n_seqs * a.kv > a.target) return;      // (more items than that, or sequences that take no part)
        for (int i0 = 0, held = 0; i0 < a.n_seqs; i0 += 64) {
            int rts, tiles;
            counts(a, of(a, i0, &held), &rts, &tiles);
#pragma unroll
            for (int k = 0; k < kSizes; ++k) total[k] += (float)rts * fmaxf(ceilf((float)tiles * per[k]), 1.f);
        }
#pragma unroll
        for (int k = kSizes - 2; k >= 0; --k)
            if (sum_of(total[k]) * (float)a.kv <= (float)a.target) per_tile = per[k];
    }

    // Work item `want`.  Every lane of a wave calls it; the result is the same in all.
    __device__ __forceinline__ Work locate(const PagedArgs &a, int want) const {
        Work w;
        w.ok = false;
        int done = 0, slots = 0, joins = 0;
        for (int i0 = 0, held = 0; i0 < a.n_seqs; i0 += 64) {
            const Seq s = of(a, i0, &held);
            int rts, tiles;
            counts(a, s, &rts, &tiles);
            const int n = parts(tiles), c = a.kv * rts * n, cut = n > 1 ? c : 0, items = n > 1 ? a.kv * rts : 0;
            const int ic = scan_sum(c), is = scan_sum(cut), ij = scan_sum(items);
            const uint64_t found = __ballot(done + ic > want);
            if (found) {
                const int l = __builtin_ctzll(found);
                auto at = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
                w.i = i0 + l;
                w.s = Seq{at(s.len), at(s.start), at(s.n), at(s.first)};
                const int rt = at(rts), local = want - (done + at(ic) - at(c));
                w.parts = at(n);
                w.step = a.kv * rt;
                w.part = w.parts > 1 ? quotient(local, w.step) : 0;
                const int u = local - w.part * w.step;
                w.y = quotient(u, rt);
                w.rt = rt - 1 - (u - w.y * rt);              // the longest rows of a causal chunk first
                w.slot = slots + at(is) - at(cut) + u;
                w.join = joins + at(ij) - at(items) + u;
                w.ok = true;
                return w;
            }
            done += __builtin_amdgcn_readlane(ic, 63);
            slots += __builtin_amdgcn_readlane(is, 63);
            joins += __builtin_amdgcn_readlane(ij, 63);
        }
        return w;
    }
    // Cut items of the launch.
    __device__ __forceinline__ int cut_items(const PagedArgs &a) const {
        int sum = 0;
        for (int i0 = 0, held = 0; i0 < a.n_seqs; i0 += 64) {
            int rts, tiles;
            counts(a, of(a, i0, &held), &rts, &tiles);
            sum += __builtin_amdgcn_readlane(scan_sum(parts(tiles) > 1 ? a.kv * rts : 0), 63);
        }
        return sum;
    }
};

// Equal shares for launches of many rows: all items (sequence, key head, row tile, in this order) lie on a line,
// each as long as its key tiles, and workgroup r takes what lies in [r, r + 1) shares, so that a device full of workgroups
// ends at once whatever the lengths.  The tiles of a head's row tiles are taken to grow evenly from the first
// to the last row tile's, which makes every place on the line a closed form (in 64 bits; that they are not quite so
// costs balance alone), and an item costs kFixed tiles beside its own (the first loads, the first tile's references, the
// output: 10 us, a tile 2).  An item whose stretch a share ends in is cut there: workgroup r's first part of a cut item
// lies in slot 2 r if the item began before it, in slot 2 r + 1 otherwise.
template <int ROWS, int KT>
struct Shares {
    static constexpr int kFixed = 5;
    double total, each;             // of the line
    int groups;                     // workgroups that have a share
    Seq lane_seq;                   // this lane's sequence of the first 64
    int lane_held;                  // the largest start of those (see sequence)

    // A sequence on the line, and a key head of it; uniform.
    struct Place {
        Seq s;
        int i, rts, y;
        double begin, end;          // of the sequence
        double y_begin, y_long;     // of the key head: begin and length
        double first, grow;         // its first row tile's length, growth from one to the next
        bool ok;
    };

    static __device__ __forceinline__ int row_tiles(const PagedArgs &a, const Seq &s) {
        return s.n > 0 && s.n >= a.lo && s.n <= a.hi ? (int)(((uint32_t)s.n * (uint32_t)a.group + ROWS - 1) / ROWS) : 0;
    }
    static __device__ __forceinline__ void lengths(const PagedArgs &a, const Seq &s, int rts, int y, double *first, double *grow, double *all) {
        const int last = (rts - 1) * ROWS, rows = s.n * a.group;
        const int f = max(tiles_of<KT>(a, s, a.sink[y], a.recent[y], 0, token_of(a, min(ROWS, rows) - 1)).n, 1) + kFixed;
        const int l = max(tiles_of<KT>(a, s, a.sink[y], a.recent[y], token_of(a, last), token_of(a, rows - 1)).n, 1) + kFixed;
        *first = f;
        *grow = rts > 1 ? (double)(l - f) / (double)(rts - 1) : 0.;
        *all = 0.5 * (double)rts * (double)(f + l);
    }
    static __device__ __forceinline__ double length(const PagedArgs &a, const Seq &s, int rts) {
        if (rts == 0) return 0.;
        double f, g, all, sum = 0.;
        if (a.one_span) {
            lengths(a, s, rts, 0, &f, &g, &all);
            return all * (double)a.kv;
        }
        for (int y = 0; y < a.kv; ++y) {
            lengths(a, s, rts, y, &f, &g, &all);
            sum += all;
        }
        return sum;
    }
    template <int CTRL, int MASK>
    static __device__ __forceinline__ double moved(double v) {
        const uint64_t u = __builtin_bit_cast(uint64_t, v);
        const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, MASK, 0xf, false);
        const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, MASK, 0xf, false);
        return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
    }
    static __device__ __forceinline__ double scan(double x) {     // as scan_sum
        x += moved<0x111, 0xf>(x);
        x += moved<0x112, 0xf>(x);
        x += moved<0x114, 0xf>(x);
        x += moved<0x118, 0xf>(x);
        x += moved<0x142, 0xa>(x);
        x += moved<0x143, 0xc>(x);
        return x;
    }
    static __device__ __forceinline__ double lane_of(double v, int l) {
        const uint64_t u = __builtin_bit_cast(uint64_t, v);
        const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)u, l), hi = __builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), l);
        return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
    }
    __device__ __forceinline__ Seq of(const PagedArgs &a, int i0, int *held) const {
        if (i0 > 0) return sequence(a, i0, held);
        *held = lane_held;
        return lane_seq;
    }

    __device__ __forceinline__ explicit Shares(const PagedArgs &a) {
        lane_held = 0;
        lane_seq = sequence(a, 0, &lane_held);
        total = 0.;
        for (int i0 = 0, held = 0; i0 < a.n_seqs; i0 += 64) {
            const Seq s = of(a, i0, &held);
            total += lane_of(scan(length(a, s, row_tiles(a, s))), 63);
        }
        groups = max((int)fmin((double)a.target, total / (double)a.min_tiles), 1);
        each = total / (double)groups;
    }
    __device__ __forceinline__ double start(int r) const { return r >= groups ? total : each * (double)r; }

    static __device__ __forceinline__ void set_head(const PagedArgs &a, Place *p, int y, double begin) {
        p->y = y;
        p->y_begin = begin;
        lengths(a, p->s, p->rts, y, &p->first, &p->grow, &p->y_long);
    }
    static __device__ __forceinline__ void next_head(const PagedArgs &a, Place *p) { set_head(a, p, p->y + 1, p->y_begin + p->y_long); }
    // Where row tile k of the place's head begins (k = rts: where the head ends).
    static __device__ __forceinline__ double at(const PagedArgs &a, const Place &p, int k) {
        if (k == p.rts) return p.y + 1 == a.kv ? p.end : p.y_begin + p.y_long;
        return p.y_begin + (double)k * (p.first + 0.5 * p.grow * (double)(k - 1));
    }
    // The key tile at which x cuts an item of n tiles that lies in [from, to).
    static __device__ __forceinline__ int cut(double x, double from, double to, int n) {
        return x <= from ? 0 : x >= to ? n : min(max((int)((x - from) / (to - from) * (double)(n + kFixed) + 0.5) - kFixed, 0), n);
    }
    // The sequence at x of the line; key head 0.
    __device__ __forceinline__ Place find(const PagedArgs &a, double x) const {
        Place p;
        p.ok = false;
        double done = 0.;
        for (int i0 = 0, held = 0; i0 < a.n_seqs; i0 += 64) {
            const Seq s = of(a, i0, &held);
            const int rts = row_tiles(a, s);
            const double sum = scan(length(a, s, rts));
            const uint64_t found = __ballot(rts > 0 && done + sum > x);
            if (found) {
                const int l = __builtin_ctzll(found);
                auto at = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
                p.i = i0 + l;
                p.s = Seq{at(s.len), at(s.start), at(s.n), at(s.first)};
                p.rts = at(rts);
                p.begin = l > 0 ? done + lane_of(sum, l - 1) : done;
                p.end = done + lane_of(sum, l);
                set_head(a, &p, 0, p.begin);
                p.ok = true;
                return p;
            }
            done += lane_of(sum, 63);
        }
        return p;
    }
    // Row tile of the place's head in which x lies.
    static __device__ __forceinline__ int row_tile_at(const PagedArgs &a, const Place &p, double x) {
        const double u = x - p.y_begin, b = p.first - 0.5 * p.grow;        // u = b k + grow / 2 k^2
        double k = p.grow == 0. ? u / p.first : (sqrt(fmax(b * b + 2. * p.grow * u, 0.)) - b) / p.grow;
        int i = (int)fmin(fmax(k, 0.), (double)(p.rts - 1));
        while (i > 0 && at(a, p, i) > x) --i;
        while (i + 1 < p.rts && at(a, p, i + 1) <= x) ++i;
        return i;
    }
};

// The sequence that holds this lane's batch row `token`, one of t0 .. t1 - 1 (-1: none, or not one of the
// launch's), and in *held what is known of it.  Every lane of a wave calls it.
__device__ __forceinline__ int owner_of(const PagedArgs &a, int token, int t0, int t1, Seq *held) {
    int owner = -1;
    for (int i0 = 0, before = 0; i0 < a.n_seqs; i0 += 64) {
        const Seq s = sequence(a, i0, &before);
        const int n = s.n >= a.lo && s.n <= a.hi ? s.n : 0;
        for (uint64_t some = __ballot(n > 0 && s.start < t1 && s.start + n > t0); some; some &= some - 1) {
            const int l = __builtin_ctzll(some);
            auto at = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
            // (read by all lanes: within the branch, lane l may take no part, nor have worked its values out)
            const Seq x = {at(s.len), at(s.start), at(n), at(s.first)};
            if (owner < 0 && token >= x.start && token - x.start < x.n) {
                owner = i0 + l;
                *held = x;
            }
        }
    }
    return owner;
}

// First row of sequence i in the expanded copies.
__device__ __forceinline__ int64_t first_row(const PagedArgs &a, int i) {
    const int lane = threadIdx.x & 63;
    int64_t done = 0;                // (lengths may say more than the copies have room for)
    for (int i0 = 0, held = 0; i0 < i; i0 += 64) {
        const Seq s = sequence(a, i0, &held);
        const bool mine = i0 + lane < i && s.n > 0 && s.n >= a.lo && s.n <= a.hi;
        done += __builtin_amdgcn_readlane(scan_sum(mine ? (s.len + kSeqRows - 1) / kSeqRows : 0), 63);
    }
    return done * kSeqRows;
}

// Block `want` of kSeqRows rows of the expanded copies: the sequence, its number in *seq, and the
// block's first key (-1: no such block).
__device__ __forceinline__ int locate_block(const PagedArgs &a, int want, Seq *held, int *seq) {
    int done = 0;
    for (int i0 = 0, before = 0; i0 < a.n_seqs; i0 += 64) {
        const Seq s = sequence(a, i0, &before);
        const int blocks = s.n > 0 && s.n >= a.lo && s.n <= a.hi ? (s.len + kSeqRows - 1) / kSeqRows : 0;
        const int ib = scan_sum(blocks);
        const uint64_t found = __ballot(done + ib > want);
        if (found) {
            const int l = __builtin_ctzll(found);
            auto at = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
            *held = Seq{at(s.len), at(s.start), at(s.n), at(s.first)};
            *seq = i0 + l;
            return (want - done - at(ib) + at(blocks)) * kSeqRows;
        }
        done += __builtin_amdgcn_readlane(ib, 63);
    }
    return -1;
}

// Row of the page pools that holds key j of sequence i (0 <= j < len); a page outside the pool
// is held to it.
__device__ __forceinline__ int pool_row(const PagedArgs &a, const int32_t *pages, int y, int j) {
    const int b = div_magic(j, a.mp_hi, a.mp_lo);
    const int page = min(max(pages[b], 0), a.n_pages - 1);
    return (page * a.kv + y) * a.page_tokens + (j - b * a.page_tokens);
}

// Chunk (16 bytes) c of row k of a tile in LDS lies at chunk place(k, c) of the row: rows that
// are read together then fall into distinct banks.  CH: chunks per row.  KEYS: rows read one to a
// lane, the same chunk of each (the score operand, and rows that serve both products);
// otherwise read four at a time, transposed (the value operand).
template <int CH, bool KEYS>
__device__ __forceinline__ int place(int k, int c) {
    if (CH % 16 == 0) return c ^ (KEYS ? (k & 15) : ((k & 3) << 2 | (k >> 2 & 3)));
    return c ^ (KEYS ? (k >> 1 & 7) : ((k >> 1 & 1) << 2 | (k >> 2 & 3)));
}

// sum + the two bf16 of a word, one rounding.
__device__ __forceinline__ float add_two(uint32_t word, float sum) {
    typedef __bf16 pair_t __attribute__((ext_vector_type(2)));
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(pair_t, word), __builtin_bit_cast(pair_t, 0x3f803f80), sum, false);
}

// Any of the 8 bf16 of v is an infinity or a NaN.
__device__ __forceinline__ bool special(const u32x4 &v) {
    bool s = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) s |= (v[i] & 0x7f80u) == 0x7f80u || (v[i] & 0x7f800000u) == 0x7f800000u;
    return s;
}

// The 8 bf16 of v with 0 for infinities and NaNs; and the reverse, for one value.
__device__ __forceinline__ u32x4 finite_only(u32x4 v) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
        v[i] = ((v[i] & 0x7f80u) == 0x7f80u ? 0u : v[i] & 0xffffu) | ((v[i] & 0x7f800000u) == 0x7f800000u ? 0u : v[i] & 0xffff0000u);
    return v;
}
__device__ __forceinline__ float special_only(uint32_t bits) { return (bits & 0x7f80u) == 0x7f80u ? __uint_as_float(bits << 16) : 0.f; }

// A part's sum far from 1 (its reference far from its largest score) moves into its reference by a power of two,
// so that joining it with other parts' loses nothing; the factor for its outputs.  (Where that power would leave the
// range of a score the parts' references are too near one another to need it.)
__device__ __forceinline__ float moderate(float *m, float *l, float *exact, float scale_log2) {
    if (!(*l > 0.f) || (*l > 0x1p-20f && *l < 0x1p20f) || !(*l < __builtin_inff()) || scale_log2 < 0x1p-100f) return 1.f;
    const int k = __builtin_amdgcn_frexp_expf(*l);
    *m += (float)k / scale_log2;
    const float by = __builtin_amdgcn_ldexpf(1.f, -k);
    *l *= by;
    *exact *= by;
    return by;
}

// Whether any thread of the workgroup says so; every thread calls it.  flag: LDS that is otherwise free
// (__syncthreads_or takes LDS of its own, with which two workgroups no longer share a CU).
__device__ __forceinline__ bool any_of(bool mine, int *flag) {
    __syncthreads();
    if (threadIdx.x == 0) *flag = 0;
    __syncthreads();
    if (mine) *flag = 1;
    __syncthreads();
    const bool any = *flag != 0;
    __syncthreads();
    return any;
}

}  // namespace paged
}  // namespace fkv
