// k_paged_tile.hip -- attention of chunks and prompts of many sequences over paged caches
// (or, EXPANDED, over the keys and values made from latent rows), gfx950 MFMA.
//
// An item is a sequence, a key head and a tile of 32 NW query rows (the query heads of a key
// head share a tile).  A workgroup of NW waves computes its share of the line of all items
// (Shares), walking the keys of each 64 at a time.  Per wave, 32 query rows and
// v_mfma_f32_32x32x16_bf16:
//   S^T = K Q^T    (A = K rows from LDS, B = the wave's queries in registers),
//   softmax        per query column, fp32, with a reference that is not the maximum but the
//                  largest score of the part's first tile: any reference cancels in the
//                  quotient, and probabilities above one are as exact as those below,
//   O^T += V^T P^T (A = V^T through the LDS transpose read, P straight from S^T).
// Where a row's sum leaves [2^-64, 2^100] (weights below 2^-126 are lost, and would count) or an output is not
// finite, and where an infinity or a NaN lies among values that only some rows see, the part is
// computed again, tile by tile with a running maximum.  The sum adds the rounded probabilities that
// weight the values, two at a time; lse takes another one of the probabilities as they are.
//
// The matrix units bound it, so everything is arranged around their stream: the products of a
// tile are one pinned sequence (scores of key block 1, values of block 0, scores of the next
// tile's block 0, values of block 1) with the exponentials of a block spread over the 16 products behind its scores, a few
// VALU instructions each, and operands read four products ahead.  LDS rows are padded so that
// every read is one address and a constant (with chunks placed by exclusive-or instead, 24
// VALU instructions a tile more).  At 480P (12 heads of 128, 4680 rows over 37440 keys, 1.08
// TFLOP) 1.04 to 1.20 ms as the card is cool or hot, 0.9 to 1.04 PFLOP/s; products in 57% of
// the cycles.  Attention over one history in place (k_attn.hip) does the same sums in 0.97 ms where this takes
// 1.07, in turn on one card: it transposes values on their way into LDS, this reads two transposed halves for
// each value product (1.6 LDS instructions a product in place of 1.2).  Steps: running maxima and 128 rows, two workgroups a CU 1510 us; the pinned
// stream with 256 rows 1250; padded rows, rotating buffers, contiguous rows read from one
// address 1210; equal shares 1130 (228 items leave 28 CUs idle otherwise; with 14 heads, 266
// items, 1970 without and 1270 with); results stored under the next item's first loads 1070.  An item
// costs some 10 us beside its tiles (4 the first loads, 1 the reference, 3 the output);
// prompts of 1700 to 3500 tokens, 40 heads over 8, five items a workgroup, reach 0.73 PFLOP/s
// for that (242 GFLOP, 347 us, 0.70 on a hot card), one prompt of 8192 tokens and 16 heads 0.83.  Measured beside it,
// slower: 128 rows and two workgroups a CU in the same stream (1270 us, prompts 490 against
// 440), tiles loaded through four unrolled buffers (spills in the loop over tiles).  Registers: at head_dim 128
// 24 values and more do not fit (41 with lse, 32 over expanded copies, 52 and 68 with 128 rows).  They are stored and
// loaded in an item's setup and output; in the loop over tiles 3 are, with 128 rows and lse.
#include <type_traits>
#include <utility>

#include "paged_join.h"

namespace fkv {
namespace {

using namespace paged;

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) bf16x4_t lds_bf16x4_t;

constexpr int KT = 64;
constexpr float kFar = 0x1p10f;     // log2 units from which scores are subtracted before they are scaled
constexpr float kLn2 = 0.69314718055994530942f;

__device__ __forceinline__ bf16x8_t frag(const u32x4 &v) { return __builtin_bit_cast(bf16x8_t, v); }

__device__ __forceinline__ uint2 pack4(float x0, float x1, float x2, float x3) {
    const uint32_t b0 = __builtin_bit_cast(uint16_t, (__bf16)x0), b1 = __builtin_bit_cast(uint16_t, (__bf16)x1);
    const uint32_t b2 = __builtin_bit_cast(uint16_t, (__bf16)x2), b3 = __builtin_bit_cast(uint16_t, (__bf16)x3);
    return make_uint2(b0 | (b1 << 16), b2 | (b3 << 16));
}

// The larger of a value and that of the lane 32 further.
__device__ __forceinline__ float across_max(float v) { return fmaxf(v, __shfl_xor(v, 32)); }

// f(0), f(1), ... with constants.
template <int... I, class F>
__device__ __forceinline__ void each(std::integer_sequence<int, I...>, F &&f) {
    (f(std::integral_constant<int, I>{}), ...);
}

template <int DQK, int DV, bool EXPANDED, int NW, bool LSE>
__global__ __launch_bounds__(64 * NW, NW == 4 ? 2 : 1) void paged_tile_kernel(PagedArgs a) {
    constexpr int ROWS = 32 * NW, NT = 64 * NW;
    constexpr int CK = DQK / 8, CV = DV / 8, KS = DQK / 16, MB = DV / 32;
    constexpr int NK = KT * CK / NT, NV = KT * CV / NT;
    // Key tiles t and t + 1 are read while t + 2 is written: more than two buffers, or two and another
    // barrier (NW 4: two workgroups share a CU's LDS).
    constexpr int KB = NW == 8 ? 3 : 2;
    // Rows in LDS are padded: 16 keys' chunks (the score operand), and the 8 rows of 64 bytes that a
    // transpose read covers, then fall into distinct banks, and every read of a tile is one address
    // and a constant.
    constexpr int SK = DQK + 8, SV = DV + 32;
    __shared__ __attribute__((aligned(16))) uint16_t kts[KB * KT * SK], vts[2 * KT * SV];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), hh = lane >> 5, c = lane & 31;

    // A share of the line of all items, or (no workspace) one item.
    using Line = Shares<ROWS, KT>;
    const bool shared = a.target > 0;
    const int number = shared ? (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3) : blockIdx.x;   // (neighbours on one XCD)
    typename Line::Place at;
    int rt = 0;
    int64_t base = 0;                             // the sequence's first row in the expanded copies
    double from = 0., until = 0., stride = 0.;
    if (shared) {
        if (tid == 0) {
            a.joins[number].rows = 0;
            a.joins[number].goes_on = 0;
        }
        const Line line(a);
        if (number >= line.groups || line.total == 0.) return;
        from = line.start(number);
        until = line.start(number + 1);
        stride = line.each;
        at = line.find(a, from);
        if (!at.ok) return;
        while (at.y + 1 < a.kv && at.y_begin + at.y_long <= from) Line::next_head(a, &at);
        rt = Line::row_tile_at(a, at, from);
    } else {
        const Work item = Split<ROWS, KT>(a).locate(a, number);
        if (!item.ok) return;
        at.s = item.s;
        at.i = item.i;
        at.y = item.y;
        rt = item.rt;
    }
    if (EXPANDED) base = first_row(a, at.i);
    f32x16_t o[MB];
    float m = neg_inf(), l = 0.f, exact = 0.f;    // exact (LSE): the sum of the weights as they are, not as they are rounded
    // This lane's row of the item before, whose results are stored while the next one's first tiles are on their way.
    int pending = 0;                              // 1: an output row, 2: a part of one
    bool none = false;                            // the row sees no key
    int64_t out_at = 0, lse_at = 0;               // where it goes: in O and lse, or (a part) in `part`
    auto clear = [&]() {
        m = neg_inf();
        l = exact = 0.f;
#pragma unroll
        for (int b = 0; b < MB; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[b][r] = 0.f;
    };
    auto flush = [&]() {
        if (pending == 1) {
            const float inv = none ? 0.f : 1.f / l;
            uint16_t *to = a.O + out_at;
#pragma unroll
            for (int b = 0; b < MB; ++b)
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    *(uint2 *)(to + 32 * b + 8 * u) = pack4(o[b][4 * u] * inv, o[b][4 * u + 1] * inv, o[b][4 * u + 2] * inv, o[b][4 * u + 3] * inv);
            if (LSE && hh == 0) a.lse[lse_at] = none ? neg_inf() : fmaf(m * kLn2, a.scale_log2, logf(exact));
        } else if (pending == 2) {
            float *to = a.part + out_at;
            const float by = moderate(&m, &l, &exact, a.scale_log2);
#pragma unroll
            for (int b = 0; b < MB; ++b)
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    *(f32x4_t *)(to + 32 * b + 8 * u) = f32x4_t{o[b][4 * u], o[b][4 * u + 1], o[b][4 * u + 2], o[b][4 * u + 3]} * by;
            if (hh == 0) {
                a.part[lse_at] = m;
                a.part[lse_at + ROWS] = l;
                if (LSE) a.part[lse_at + 2 * ROWS] = exact;
            }
        }
        pending = 0;
    };
#pragma unroll 1
    for (;;) {                                    // (the body ends with the workgroup past its reads of LDS)
        Seq s = at.s;
        if (EXPANDED) s.len = (int)min((int64_t)s.len, max(a.head_rows - base, (int64_t)0));
        const int y = at.y, r0 = rt * ROWS, rows = min(ROWS, s.n * a.group - r0);
        const int sink = a.sink[y], recent = a.recent[y];
        const int t_first = token_of(a, r0), t_last = token_of(a, r0 + rows - 1);
        const Tiles x = tiles_of<KT>(a, s, sink, recent, t_first, t_last);
        const double item_at = shared ? Line::at(a, at, rt) : 0., item_end = shared ? Line::at(a, at, rt + 1) : 0.;
        const int tb = shared ? Line::cut(from, item_at, item_end, x.n) : 0, te = shared ? Line::cut(until, item_at, item_end, x.n) : x.n;
        const bool whole = tb == 0 && te == x.n;
        const int32_t *pages = a.table + (int64_t)at.i * a.max_pages;

        // This lane's query row.
        const int row = min(32 * w + c, rows - 1) + r0, tok = token_of(a, row), head = y * a.group + row - tok * a.group;
        const bool live = 32 * w + c < rows;
        const Sight seen = sight(a, s, recent, tok);
        bf16x8_t q[KS];
        // Rows of a tile's keys, one to a lane (past the part's last tile, that one's); EXPANDED: the first one's.
        const int j_last = x.most.end - 1;
        const uint16_t *K = a.K, *V = a.V;
        if (EXPANDED) {
            K += (y * a.head_rows + base) * DQK;
            V += (y * a.head_rows + base) * DV;
        }
        auto rows_of = [&](int t) {
            const int j = x.key(min(t, te - 1), KT);
            return EXPANDED ? j : pool_row(a, pages, y, min(j + lane, j_last));
        };
        u32x4 kr[NK], vr[NV];
        bool odd = false;                             // an infinity or a NaN among values that not every row sees
        // EXPANDED: a tile's rows lie together; a row past the sequence's last is read as zeros.  (Offsets are unsigned: a
        // head's copies have fewer than 2^32 bytes.  A buffer of its own for every tile: 620 us against 600 at 480P.)
        auto rsrc = [](const uint16_t *p, int64_t bytes) {
            return __builtin_amdgcn_make_buffer_rsrc((void *)p, 0, (int)(uint32_t)bytes, 0x00020000);
        };
        const auto k_buf = rsrc(K, EXPANDED ? (int64_t)s.len * DQK * 2 : 0), v_buf = rsrc(V, EXPANDED ? (int64_t)s.len * DV * 2 : 0);
        // N chunks of the rows of a pool; rows that follow one another are read from one address.
        auto load = [&](const uint16_t *pool, int row_of_lane, auto width, auto &to) __attribute__((always_inline)) {
            constexpr int W = width, CH = W / 8, N = KT * CH / NT;
            const int first = __builtin_amdgcn_readfirstlane(row_of_lane);
            if (__ballot(row_of_lane == first + lane) == ~0ull) {
                const char *at = (const char *)(pool + (int64_t)first * W);
#pragma unroll
                for (int i = 0; i < N; ++i) to[i] = *(const u32x4 *)(at + i * (NT * 16) + (uint32_t)(tid * 16));
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int id = tid + i * NT, k = id / CH;
                    to[i] = *(const u32x4 *)(pool + (int64_t)__shfl(row_of_lane, k) * W + (id - k * CH) * 8);
                }
            }
        };
        auto load_k_to = [&](int row_of_lane, auto &kr) __attribute__((always_inline)) {
            if constexpr (EXPANDED) {
#pragma unroll
                for (int i = 0; i < NK; ++i)
                    kr[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(k_buf, (tid + i * NT) * 16, (int)((uint32_t)row_of_lane * (DQK * 2)), 0));
            } else {
                load(K, row_of_lane, std::integral_constant<int, DQK>{}, kr);
            }
        };
        auto load_k = [&](int row_of_lane) __attribute__((always_inline)) { load_k_to(row_of_lane, kr); };
        auto load_v = [&](int row_of_lane) __attribute__((always_inline)) {
            if constexpr (EXPANDED) {
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    vr[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(v_buf, (tid + i * NT) * 16, (int)((uint32_t)row_of_lane * (DV * 2)), 0));
            } else {
                load(V, row_of_lane, std::integral_constant<int, DV>{}, vr);
            }
        };
        auto store_k_from = [&](uint16_t *kt, const auto &kr) {
#pragma unroll
            for (int i = 0; i < NK; ++i) {
                const int id = tid + i * NT, k = id / CK;
                *(u32x4 *)(kt + k * SK + (id - k * CK) * 8) = kr[i];
            }
        };
        auto store_k = [&](uint16_t *kt) { store_k_from(kt, kr); };
        auto store_v = [&](uint16_t *vt, int j0, bool edge) {
            if (edge) {
                // (values of keys that no row sees are cleared: a probability of zero would not silence a NaN)
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    if (!sees(x.most, sink, j0 + (tid + i * NT) / CV)) vr[i] = u32x4{0, 0, 0, 0};
                    odd |= special(vr[i]);
                }
            }
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int id = tid + i * NT, k = id / CV;
                *(u32x4 *)(vt + k * SV + (id - k * CV) * 8) = vr[i];
            }
        };
        // Where this lane reads a tile: key c, chunk hh of K (then + 32 kb keys, + 2 k chunks); keys 4 hh + 0..3
        // of V (+ 8, + 16 k), channels 16 (lane / 16 % 2) + 4 (lane % 4) (+ 32 b).
        const uint16_t *k_lane = kts + c * SK + 8 * hh;
        const uint16_t *v_lane = vts + (4 * hh + ((lane & 15) >> 2)) * SV + 16 * (lane >> 4 & 1) + 4 * (lane & 3);

        // Scores of key block kb (32 keys).
        auto score = [&](const uint16_t *kt, int kb, f32x16_t &z) {
#pragma unroll
            for (int r = 0; r < 16; ++r) z[r] = 0.f;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const bf16x8_t f = frag(*(const u32x4 *)(kt + 32 * kb * SK + 16 * k));
                z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, q[k], z, 0, 0, 0);
            }
        };
        auto hide = [&](int j0, int kb, f32x16_t &z) {
            const int j = j0 + 32 * kb + 4 * hh, end = seen.end - j, first = sink - j, low = seen.low - j;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int k = 8 * (r >> 2) + (r & 3);
                z[r] = k < end && (k < first || k >= low) ? z[r] : neg_inf();
            }
        };
        // V^T of keys 16 k + 4 hh + 0..3 and + 8, channels 32 b + (lane % 32).
        auto value = [&](const uint16_t *vt, int k, int b) {
            const uint16_t *at = vt + 16 * k * SV + 32 * b;
            const bf16x4_t u = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_t *)at);
            const bf16x4_t v = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_t *)(at + 8 * SV));
            return __builtin_shufflevector(u, v, 0, 1, 2, 3, 4, 5, 6, 7);
        };

        if (tb >= te) {
            flush();
            clear();
        } else {
            int next_v = rows_of(tb + 1), next_k = rows_of(tb + 2);   // pool rows of the tiles to load next
            int j0 = x.key(tb, KT);
            bool edge = !all_seen<KT>(x, sink, j0);   // not every row sees every key of the tile
            {
                const int first = rows_of(tb);
                u32x4 k2[NK];
                load_k(first);
                load_v(first);
                load_k_to(next_v, k2);
                {
                    const uint16_t *from = a.Q + (int64_t)(s.start + tok) * a.q_tok + (int64_t)head * a.q_head + 8 * hh;
#pragma unroll
                    for (int k = 0; k < KS; ++k) q[k] = frag(live ? *(const u32x4 *)(from + 16 * k) : u32x4{0, 0, 0, 0});
                }
                __builtin_amdgcn_sched_barrier(0);
                flush();
                clear();
                store_k(kts);
                store_v(vts, j0, edge);
                load_v(next_v);
                store_k_from(kts + KT * SK, k2);
            }
            __syncthreads();
            f32x16_t z[2];
            score(k_lane, 0, z[0]);
            {                                         // the reference: the row's largest score in the first tile, masked keys too
                score(k_lane, 1, z[1]);
                float top = neg_inf();
#pragma unroll
                for (int r = 0; r < 16; ++r) top = fmaxf(top, fmaxf(z[0][r], z[1][r]));
                top = across_max(top);
                m = fabsf(top) < __builtin_inff() ? top : 0.f;
            }
            // 2^(c (z - m)): the product c m is rounded on its own, by 2^-14 log2 units at most below kFar;
            // beyond, scores are subtracted before they are scaled (of nearby scores the difference is exact)
            const bool far = __ballot(!(fabsf(m * a.scale_log2) < kFar)) != 0;
            const float cm = far ? 0.f : m * a.scale_log2;
            bool met = false;
            float sum[2] = {0.f, 0.f}, all_sum[2] = {0.f, 0.f}, v[2];
            u32x4 p[2][2];                            // probabilities, two bf16 a word: key block, 16 keys
            auto ready = [&](int j, int kb) {         // a key block's scores are complete, and not those of an ordinary tile
                hide(j, kb, z[kb]);
                if (far) z[kb] -= m;
#pragma unroll
                for (int r = 0; r < 16; ++r) met |= z[kb][r] != neg_inf();
            };
            // Half of the work on scores 2 i and 2 i + 1 of key block kb.
            auto step = [&](int kb, int i, int half) __attribute__((always_inline)) {
                if (half == 0) {
                    v[0] = fmaf(z[kb][2 * i], a.scale_log2, -cm);
                    v[1] = fmaf(z[kb][2 * i + 1], a.scale_log2, -cm);
                    v[0] = __builtin_amdgcn_exp2f(v[0]);
                } else {
                    v[1] = __builtin_amdgcn_exp2f(v[1]);
                    if (LSE) {
                        all_sum[0] += v[0];
                        all_sum[1] += v[1];
                    }
                    uint32_t word = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{v[0], v[1]}, bf16x2_t));
                    asm volatile("" : "+v"(word));     // (not moved to its use)
                    sum[i & 1] = add_two(word, sum[i & 1]);
                    p[kb][i >> 2][i & 3] = word;
                }
            };
            edge |= far;
            if (edge) ready(j0, 0);
            else met = true;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                step(0, i, 0);
                step(0, i, 1);
            }
            // One pinned stream a tile: (C) the scores of its second key block, (D) the values of its first, (A)
            // the scores of the next tile's first, (B) the values of its second; the exponentials of a key block run
            // behind the 16 and more products after its scores, operands are read kAhead products ahead.
            constexpr int kAhead = 4, NV4 = 2 * MB, kD = KS, kA = KS + NV4, kB = 2 * KS + NV4, kN = 2 * KS + 2 * NV4;
            int k_this = 0, k_next = KT * SK, k_free = KB == 3 ? 2 * KT * SK : 0, v_this = 0;   // the buffers
#pragma unroll 1
            for (int t = tb; t < te; ++t) {
                const uint16_t *k0 = k_lane + k_this, *k1 = k_lane + k_next, *vt = v_lane + v_this;
                const int jn = x.key(min(t + 1, te - 1), KT);
                const bool edge_n = !all_seen<KT>(x, sink, jn);
                // over tile t - 1, which every wave has weighted; past the part's last tile that one again
                store_v(vts + (KT * SV - v_this), jn, edge_n);
                load_k(next_k);
                next_v = next_k;
                next_k = rows_of(t + 3);
                bf16x8_t f[kAhead];
                auto fetch = [&](auto index) __attribute__((always_inline)) {
                    constexpr int i = index;
                    if constexpr (i < kD) f[i % kAhead] = frag(*(const u32x4 *)(k0 + 32 * SK + 16 * i));
                    else if constexpr (i < kA) f[i % kAhead] = value(vt, (i - kD) / MB, (i - kD) % MB);
                    else if constexpr (i < kB) f[i % kAhead] = frag(*(const u32x4 *)(k1 + 16 * (i - kA)));
                    else if constexpr (i < kN) f[i % kAhead] = value(vt, 2 + (i - kB) / MB, (i - kB) % MB);
                };
                each(std::make_integer_sequence<int, kAhead>{}, fetch);
                each(std::make_integer_sequence<int, kN>{}, [&](auto index) __attribute__((always_inline)) {
                    constexpr int i = index;
                    constexpr bool scores = i < kD || (i >= kA && i < kB);
                    constexpr int kb = i < kD || i >= kB ? 1 : 0;                 // key block of the product
                    constexpr int at = i < kD ? i : i < kA ? i - kD : i < kB ? i - kA : i - kB, n = scores ? KS : NV4;
                    if constexpr (scores) {
                        if constexpr (at == 0) {
#pragma unroll
                            for (int r = 0; r < 16; ++r) z[kb][r] = 0.f;
                        }
                        z[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % kAhead], q[at], z[kb], 0, 0, 0);
                    } else {
                        o[at % MB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i % kAhead], frag(p[kb][at / MB]), o[at % MB], 0, 0, 0);
                    }
                    fetch(std::integral_constant<int, i + kAhead>{});
                    // behind (C) and (B) key block 0, behind (D) and (A) key block 1; the first 8 scores behind values
                    constexpr int h0 = 8 * at / n, h1 = 8 * (at + 1) / n, of = i < kD || i >= kB ? 0 : 1, first = scores ? 4 : 0;
#pragma unroll
                    for (int h = h0; h < h1; ++h) step(of, first + h / 2, h & 1);
                    __builtin_amdgcn_sched_barrier(0);
                    if constexpr (i == kD - 1) {
                        if (edge) ready(j0, 1);
                        if (KB == 2) __syncthreads();  // (every wave has read tile t's keys)
                    }
                    if constexpr (i == kA - 1) {
                        store_k(kts + k_free);
                        load_v(next_v);
                    }
                    if constexpr (i == kB - 1) {
                        l = sum[0] + sum[1];           // (the last time without the tile after the last)
                        if (LSE) exact = all_sum[0] + all_sum[1];
                        j0 = jn;
                        edge = edge_n || far;
                        if (edge) ready(j0, 0);
                        else met = true;
                    }
                });
                __syncthreads();
                const int used = k_this;
                k_this = k_next;
                k_next = k_free;
                k_free = KB == 3 ? used : k_this;
                v_this = KT * SV - v_this;
            }
            met = (__ballot(met) >> c | __ballot(met) >> (32 + c)) & 1;
            const float all = l + __shfl_xor(l, 32);
            bool again = odd;
            if (live && met) {
                again |= !(all > 0x1p-64f && all < 0x1p100f);
#pragma unroll
                for (int b = 0; b < MB; ++b)
#pragma unroll
                    for (int r = 0; r < 16; ++r) again |= !(fabsf(o[b][r]) < __builtin_inff());
            }
            if (!met) m = neg_inf();                  // (no key of the part's)
            if (any_of(again, (int *)kts)) {
                // Tile by tile with a running maximum; an infinity or a NaN among the values goes to the rows that
                // see it alone.
                clear();
#pragma unroll 1
                for (int t = tb; t < te; ++t) {
                    const int j = x.key(t, KT);
                    const uint16_t *kt = k_lane, *vt = v_lane;
                    load_k(rows_of(t));
                    load_v(rows_of(t));
                    store_k(kts);
                    store_v(vts, j, !all_seen<KT>(x, sink, j));
                    __syncthreads();
#pragma unroll 1
                    for (int kb = 0; kb < 2; ++kb) {
                        f32x16_t z;
                        score(kt, kb, z);
                        hide(j, kb, z);
                        float top = neg_inf(), sum = 0.f, rounded = 0.f;
#pragma unroll
                        for (int r = 0; r < 16; ++r) top = fmaxf(top, z[r]);
                        const float up = fmaxf(m, across_max(top)), base = up == neg_inf() ? 0.f : up;
                        const float alpha = up == m ? 1.f : __builtin_amdgcn_exp2f((m - up) * a.scale_log2);
                        m = up;
                        bf16x8_t p[2];
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const float v = __builtin_amdgcn_exp2f((z[r] - base) * a.scale_log2);
                            sum += v;
                            p[r >> 3][r & 7] = (__bf16)v;
                            rounded += (float)p[r >> 3][r & 7];
                        }
                        l = l * alpha + rounded;
                        exact = exact * alpha + sum;
#pragma unroll
                        for (int b = 0; b < MB; ++b) {
                            o[b] *= alpha;
#pragma unroll
                            for (int k = 0; k < 2; ++k)
                                o[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag(finite_only(__builtin_bit_cast(u32x4, value(vt + 32 * kb * SV, k, b)))),
                                                                               p[k], o[b], 0, 0, 0);
                        }
#pragma unroll 1
                        for (int k = 32 * kb; k < 32 * kb + 32; ++k) {    // (any weight leaves them as they are)
                            if (!sees(seen, sink, j + k)) continue;
#pragma unroll
                            for (int u = 0; u < 4 * MB; ++u) {            // channels 8 u + 4 hh + 0..3
                                const uint2 v = *(const uint2 *)(vts + k * SV + 8 * u + 4 * hh);
                                o[u >> 2][4 * (u & 3) + 0] += special_only(v.x & 0xffffu);
                                o[u >> 2][4 * (u & 3) + 1] += special_only(v.x >> 16);
                                o[u >> 2][4 * (u & 3) + 2] += special_only(v.y & 0xffffu);
                                o[u >> 2][4 * (u & 3) + 3] += special_only(v.y >> 16);
                            }
                        }
                    }
                    __syncthreads();
                }
            }
        }

        l += __shfl_xor(l, 32);
        if (LSE) exact += __shfl_xor(exact, 32);
        none = blind(seen, sink);
        if (live && whole && (tb < te || !shared || (item_at >= from && item_at < until))) {   // (no key: who has the item's begin)
            pending = 1;
            out_at = (int64_t)(s.start + tok) * a.o_tok + (int64_t)head * a.o_head + 4 * hh;
            lse_at = (int64_t)head * a.n_tokens + s.start + tok;
        } else if (live && !whole && tb < te) {
            if (tid == 0) {
                JoinItem &j = a.joins[number];
                if (tb > 0) {
                    j.goes_on = 1;
                } else {
                    j.rows = rows;
                    j.start = s.start;
                    j.len = s.len;
                    j.first = s.first;
                    j.y = y;
                    j.row0 = r0;
                    // the workgroups whose shares begin before the item ends
                    int n = min((int)((item_end - from) / stride), (int)gridDim.x - 1 - number);
                    while (n > 0 && stride * (double)(number + n) >= item_end) --n;
                    while (number + n + 1 < (int)gridDim.x && stride * (double)(number + n + 1) < item_end) ++n;
                    j.parts = n + 1;
                }
            }
            pending = 2;
            const int64_t slot = (int64_t)(2 * number + (tb == 0)) * (ROWS * part_width(DV));
            out_at = slot + (32 * w + c) * DV + 4 * hh;
            lse_at = slot + ROWS * DV + 32 * w + c;
        }
        // The next item of the share.
        if (!shared || item_end >= until) break;
        if (++rt == at.rts) {
            rt = 0;
            if (at.y + 1 < a.kv) {
                Line::next_head(a, &at);
            } else {
                const Line line(a);
                at = line.find(a, at.end);
                if (!at.ok) break;
                if (EXPANDED) base = first_row(a, at.i);
            }
        }
    }
    flush();
}

// One workgroup joins some rows of the cut item that workgroup x's share ends in: its own part lies in slot
// 2 x + 1, those of the workgroups after it in slots 2 g, of some that have none in no slot.  D / 4 threads take 4
// channels each of a row, and one row alone: bound by latency, 40 cut items of 6 parts of 256 rows of 64 channels 8.2 us, with
// 2 rows in turn 13.8.  grid: x = workgroup, y = rows.
template <int D>
constexpr int join_rows() { return kJoinThreads / (D / 4); }

template <int D, int ROWS>
__global__ __launch_bounds__(kJoinThreads) void paged_share_join_kernel(PagedArgs a) {
    constexpr int64_t kSlot = ROWS * part_width(D);
    const JoinItem j = a.joins[blockIdx.x];
    const int d = threadIdx.x % (D / 4), r = blockIdx.y * join_rows<D>() + threadIdx.x / (D / 4);
    if (r >= j.rows) return;
    Joined x;
    constexpr int kAtOnce = 4;
    for (int k0 = 0; k0 < j.parts; k0 += kAtOnce) {
        float m[kAtOnce], l[kAtOnce], e[kAtOnce];
        join_f32x4 o[kAtOnce];
        int on[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {               // (a slot that nobody wrote is read and left out)
            const int g = blockIdx.x + min(k0 + k, j.parts - 1);
            const float *p = a.part + (2 * g + (k0 + k == 0)) * kSlot;
            on[k] = a.joins[g].goes_on;
            m[k] = p[ROWS * D + r];
            l[k] = p[ROWS * D + ROWS + r];
            e[k] = p[ROWS * D + 2 * ROWS + r];            // (only written and used for lse)
            o[k] = *(const join_f32x4 *)(p + r * D + 4 * d);
        }
        __builtin_amdgcn_sched_barrier(0);                // (all loads before the first use)
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k)
            if (k0 + k == 0 || (k0 + k < j.parts && on[k])) x.add(m[k], l[k], e[k], o[k], a.scale_log2);
    }
    x.put(a, j, r, 4 * d);
}

template <int DQK, int DV, bool EXPANDED, int NW, bool LSE>
void launch_as(const PagedArgs &a, hipStream_t s) {
    hipLaunchKernelGGL((paged_tile_kernel<DQK, DV, EXPANDED, NW, LSE>), dim3((unsigned)a.n_work), dim3(64 * NW), 0, s, a);
    if (a.target == 0) return;
    hipLaunchKernelGGL((paged_share_join_kernel<DV, 32 * NW>), dim3((unsigned)a.n_work, 32 * NW / join_rows<DV>()), dim3(kJoinThreads), 0, s, a);
}

template <int DQK, int DV, bool EXPANDED, int NW>
void launch(const PagedArgs &a, hipStream_t s) {
    if (!EXPANDED && a.lse) launch_as<DQK, DV, EXPANDED, NW, !EXPANDED>(a, s);
    else launch_as<DQK, DV, EXPANDED, NW, false>(a, s);
}

}  // namespace

hipError_t launch_paged_tiles(const PagedArgs &a, int head_dim, int rows, hipStream_t s) {
    if (head_dim == 64) {
        if (rows == 128) launch<64, 64, false, 4>(a, s);
        else launch<64, 64, false, 8>(a, s);
    } else {
        if (rows == 128) launch<128, 128, false, 4>(a, s);
        else launch<128, 128, false, 8>(a, s);
    }
    return hipGetLastError();
}

hipError_t launch_expanded_tiles(const PagedArgs &a, int head_dim, hipStream_t s) {
    if (head_dim == 64) launch<64 + kLatentRot, 64, true, 8>(a, s);
    else launch<128 + kLatentRot, 128, true, 8>(a, s);
    return hipGetLastError();
}

}  // namespace fkv
