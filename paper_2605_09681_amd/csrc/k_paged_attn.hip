// k_paged_attn.hip -- attention of few new tokens of many sequences over paged caches,
// gfx950 MFMA: single tokens and short chunks (up to 64 query rows of a sequence and key
// head, 256 where the batch's keys are known to be few, or any number over latent rows), with
// keys and values of their own or, SHARED, with values that are the first DV channels of the
// key rows (latent rows: all heads read one row).
//
//   o = sum_j 2^(c (s_j - m)) v_j / sum_j 2^(c (s_j - m)),  s_j = q . k_j,  c = scale log2 e
//
// A workgroup takes one part of an item (sequence, key head, tile of 16 MT query rows)
// and walks its keys 32 at a time.  The NW waves share each tile of keys, which is read
// once for the item's up to 64 rows and lies in LDS, three tiles deep:
//   scores   S^T = K Q^T (v_mfma_f32_16x16x32_bf16): the tile's 2 x MT blocks of 16 keys
//            and 16 rows are dealt to the waves, which turn theirs into probabilities
//            and put those into LDS (bf16; the sum that divides the output adds them as they
//            are rounded, lse's as they are);
//   values   O^T += V^T P^T: each wave owns DV / NW output channels of all rows (V^T
//            through the LDS transpose read).  SHARED leaves its outputs in fp32 to the product that follows.
// The scores of tile t + 1 and the values of tile t run in the same stretch between two
// barriers, one barrier a tile; tile t + 3 is on its way from HBM meanwhile.
//
// m is not the maximum but the largest score of the part's first tile: any reference
// cancels in the quotient, and probabilities above one are as exact in fp32 and bf16 as
// those below (down to 2^-126: what a sum of 2^-64 and more loses with each weight below it is under
// 2^-62 of it), so nothing waits for other waves' scores.  Where a row's sum leaves
// [2^-64, 2^100] or an output is not finite, and where an infinity or a NaN lies among
// values that only some rows see, the part is computed again, tile by tile with a running
// maximum (`careful`).
//
// Why so: few rows are bound by the bytes of their keys, so the keys of a sequence are split
// over the device (Split), a tile is read once for 64 rows (more rows are more items, each of which
// reads the keys again, from the caches where they are few), and each CU has 16 to 48 KB of them
// on their way.  480P, one token over 32761 keys of 12 heads (201 MB): 34 us and 4 for the
// join; 16 sequences of up to 7800 tokens, 16 heads over 4 key heads (76 MB): 18.5 and 4 us, 4.1
// TB/s; the same over latent rows of 576, 40 heads (54 MB): 25 and 8.5 us.  Of the last, 2 us are the
// split, 6 the first two tiles and the queries, 6 five tiles, 3 the output (82 KB a workgroup).
// Measured beside it: every wave forming all probabilities from scores in LDS (40 heads 67 us), parts of
// 256 keys instead of 128 (latent rows: 16.2 against 12.9 us for one token).
// Registers: latent rows of 320 channels with 16 and 32 query rows have 18 and 59 fewer than they would use in the
// 128 that two workgroups a CU leave (2 and 7 reloads a tile), those of 576 with 64 rows 31.
#include <type_traits>

#include "paged_join.h"

namespace fkv {
namespace {

using namespace paged;

typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) bf16x4_t lds_bf16x4_t;

constexpr int KT = 32;              // keys per tile
constexpr float kFar = 0x1p10f;     // log2 units from which scores are subtracted before they are scaled
constexpr float kLn2 = 0.69314718055994530942f;


__device__ __forceinline__ bf16x8_t frag(const u32x4 &v) { return __builtin_bit_cast(bf16x8_t, v); }

__device__ __forceinline__ uint2 pack4(const f32x4_t &x) {
    uint32_t b[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) b[k] = __builtin_bit_cast(uint16_t, (__bf16)x[k]);
    return make_uint2(b[0] | (b[1] << 16), b[2] | (b[3] << 16));
}

template <int DQK, int DV, bool SHARED, int MT, int NW>
struct Cfg {
    static constexpr int ROWS = 16 * MT, NT = 64 * NW;
    static constexpr int CK = DQK / 8, CV = DV / 8;                  // 16-byte chunks per row
    static constexpr int BLOCKS = 2 * MT;                            // 16 x 16 score blocks of a tile
    static constexpr int PER = (BLOCKS + NW - 1) / NW;               // of a wave: w, w + NW (all of one key block)
    static constexpr int KS = DQK / 32;                              // steps of the score product
    static constexpr int NB = DV / 16 / NW;                          // 16-channel blocks of a wave's output
    static constexpr int NK = (KT * CK + NT - 1) / NT, NV = SHARED ? 0 : (KT * CV + NT - 1) / NT;   // chunks per thread
    static constexpr int TILE = KT * (DQK + (SHARED ? 0 : DV));      // elements
    // Probabilities as one bf16, or (SHARED: the queries were rounded to bf16 once more, and the outputs go through
    // another product) as the sum of two, of which nothing is lost.
    static constexpr int PL = SHARED ? 2 : 1;
    static constexpr int P_FLOATS = 2 * PL * MT * 64 * 4;            // [2][PL][MT][lane][key block] x 4 bf16
    static constexpr int SS = KT + 4;                                // careful: floats per row of scores (16 rows in distinct banks)
    static_assert(DV % (16 * NW) == 0 && KT * CV % NT == 0 && NW % 2 == 0, "whole blocks and chunks");
};

template <int DQK, int DV, bool SHARED, int MT, int NW>
__global__ __launch_bounds__(64 * NW, few_waves(SHARED ? DV : -DV, 16 * MT)) void paged_attn_kernel(PagedArgs a) {
    using C = Cfg<DQK, DV, SHARED, MT, NW>;
    __shared__ __attribute__((aligned(16))) uint16_t tiles[3][C::TILE];
    // probabilities; careful: scores [row][SS]
    __shared__ __attribute__((aligned(16))) float mix[C::P_FLOATS > C::ROWS * C::SS ? C::P_FLOATS : C::ROWS * C::SS];
    // per row and key block: first tile's largest scores, sums of the weights as they weigh the values, and as they are (-1: no
    // key was seen)
    __shared__ float ends[3][MT][2][16];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, c = lane & 15;

    const Split<C::ROWS, KT> split(a);
    const Work item = split.locate(a, blockIdx.x);
    if (blockIdx.x == 0 && a.target > 0) {
        const int n = split.cut_items(a);
        if (tid == 0) a.joins[0].count = n;
    }
    if (!item.ok) return;
    const Seq s = item.s;
    const int y = item.y, r0 = item.rt * C::ROWS, rows = min(C::ROWS, s.n * a.group - r0);
    const int sink = a.sink[y], recent = a.recent[y];
    const int t_first = token_of(a, r0), t_last = token_of(a, r0 + rows - 1);
    const Tiles x = tiles_of<KT>(a, s, sink, recent, t_first, t_last);
    const int tb = (int)((int64_t)x.n * item.part / item.parts), te = (int)((int64_t)x.n * (item.part + 1) / item.parts);
    const int32_t *pages = a.table + (int64_t)item.i * a.max_pages;
    if (item.parts > 1 && item.part == 0 && tid == 0 && item.join < a.n_joins) {
        JoinItem &j = a.joins[item.join];
        j.rows = rows;
        j.start = s.start;
        j.len = s.len;
        j.first = s.first;
        j.y = y;
        j.row0 = r0;
        j.parts = item.parts;
        j.slot = item.slot;
        j.step = item.step;
    }
    auto row_of = [&](int r) { return min(r, rows - 1) + r0; };

    // Score blocks of this wave: key block kb of row tiles mt_of(0), mt_of(1).
    const int kb = w & 1;
    auto mt_of = [&](int i) { return (w + NW * i) >> 1; };
    auto mine = [&](int i) { return C::BLOCKS % NW == 0 || w + NW * i < C::BLOCKS; };
    bf16x8_t q[C::PER][C::KS];
    Sight seen[C::PER];
    f32x4_t o[MT][C::NB];
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int b = 0; b < C::NB; ++b) o[t][b] = f32x4_t{0.f, 0.f, 0.f, 0.f};

    // Pool rows of a tile's keys, one to a lane (both halves of the wave hold the same 32);
    // keys past the last that a row sees take its place.
    const int j_last = x.most.end - 1;
    auto rows_of = [&](int t) { return t < te ? pool_row(a, pages, y, min(x.key(t, KT) + (lane & 31), j_last)) : 0; };
    u32x4 kr[C::NK], vr[C::NV > 0 ? C::NV : 1];
    auto load_to = [&](int row_of_lane, auto &kr, auto &vr) {
#pragma unroll
        for (int i = 0; i < C::NK; ++i) {
            const int id = min(tid + i * C::NT, KT * C::CK - 1), k = id / C::CK;
            kr[i] = *(const u32x4 *)(a.K + (int64_t)__shfl(row_of_lane, k) * DQK + (id - k * C::CK) * 8);
        }
#pragma unroll
        for (int i = 0; i < C::NV; ++i) {
            const int id = tid + i * C::NT, k = id / C::CV;
            vr[i] = *(const u32x4 *)(a.V + (int64_t)__shfl(row_of_lane, k) * DV + (id - k * C::CV) * 8);
        }
    };
    auto load = [&](int row_of_lane) { load_to(row_of_lane, kr, vr); };
    bool odd = false;                            // an infinity or a NaN among values that not every row sees
    auto store_from = [&](int t, auto &kr, auto &vr) {
        const int j0 = x.key(t, KT);
        uint16_t *kt = tiles[t % 3], *vt = kt + KT * DQK;
        if (!all_seen<KT>(x, sink, j0)) {
            // (values of keys that no row sees are cleared: a probability of zero would not silence a NaN)
            if (SHARED) {
#pragma unroll
                for (int i = 0; i < C::NK; ++i) {
                    if (!sees(x.most, sink, j0 + (tid + i * C::NT) / C::CK)) kr[i] = u32x4{0, 0, 0, 0};
                    odd |= special(kr[i]);
                }
            }
#pragma unroll
            for (int i = 0; i < C::NV; ++i) {
                if (!sees(x.most, sink, j0 + (tid + i * C::NT) / C::CV)) vr[i] = u32x4{0, 0, 0, 0};
                odd |= special(vr[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < C::NK; ++i) {
            const int id = tid + i * C::NT, k = id / C::CK;
            if (KT * C::CK % C::NT == 0 || id < KT * C::CK) *(u32x4 *)(kt + k * DQK + place<C::CK, true>(k, id - k * C::CK) * 8) = kr[i];
        }
#pragma unroll
        for (int i = 0; i < C::NV; ++i) {
            const int id = tid + i * C::NT, k = id / C::CV;
            *(u32x4 *)(vt + k * DV + place<C::CV, false>(k, id - k * C::CV) * 8) = vr[i];
        }
    };
    auto store = [&](int t) { store_from(t, kr, vr); };
    // This wave's blocks of a tile's scores, two sums each so that half as many products wait for one another.
    f32x4_t z[C::PER];
    const bool busy = C::BLOCKS >= NW || w < C::BLOCKS;
    auto score = [&](int t) {
        if (!busy) return;
        const uint16_t *kt = tiles[t % 3] + (16 * kb + c) * DQK;
        f32x4_t u[C::PER];
#pragma unroll
        for (int i = 0; i < C::PER; ++i) z[i] = u[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < C::KS; ++k) {
            const bf16x8_t f = frag(*(const u32x4 *)(kt + place<C::CK, true>(16 * kb + c, 4 * k + g) * 8));
#pragma unroll
            for (int i = 0; i < C::PER; ++i) {
                f32x4_t &to = k & 1 ? u[i] : z[i];
                to = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, q[i][k], to, 0, 0, 0);
            }
        }
#pragma unroll
        for (int i = 0; i < C::PER; ++i) z[i] += u[i];
    };
    // The reference, times scale_log2 (0: taken from the scores before); the sums of the weights as they weigh the values, and,
    // where those are rounded, as they are.
    float ref[C::PER], cm[C::PER], l[C::PER], exact[C::PER];
    bool far = false, met[C::PER];               // met: a key of the row's was seen
    auto probabilities = [&](int t) {
        if (!busy) return;
        const int j0 = x.key(t, KT) + 16 * kb + 4 * g;
        const bool edge = !all_seen<KT>(x, sink, x.key(t, KT));
#pragma unroll
        for (int i = 0; i < C::PER; ++i) {
            if (far) z[i] -= ref[i];
            f32x4_t e;
#pragma unroll
            for (int r = 0; r < 4; ++r) e[r] = __builtin_amdgcn_exp2f(fmaf(z[i][r], a.scale_log2, -cm[i]));
            if (edge) {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const bool see = sees(seen[i], sink, j0 + r);
                    e[r] = see ? e[r] : 0.f;
                    met[i] |= see;
                }
            } else {
                met[i] = true;
            }
            const uint2 hi = pack4(e);
            const float four = (e[0] + e[1]) + (e[2] + e[3]);
            if (C::PL == 2) l[i] += four;
            else {
                l[i] = add_two(hi.y, add_two(hi.x, l[i]));
                exact[i] += four;
            }
            if (!mine(i)) continue;
            ((uint2 *)mix)[(((t & 1) * C::PL * MT + mt_of(i)) * 64 + lane) * 2 + kb] = hi;
            if (C::PL == 2) {
                const f32x4_t rest = {e[0] - __uint_as_float(hi.x << 16), e[1] - __uint_as_float(hi.x & 0xffff0000u),
                                      e[2] - __uint_as_float(hi.y << 16), e[3] - __uint_as_float(hi.y & 0xffff0000u)};
                ((uint2 *)mix)[((((t & 1) * C::PL + 1) * MT + mt_of(i)) * 64 + lane) * 2 + kb] = pack4(rest);
            }
        }
    };
    // V^T of keys 4 g + 0..3 and + 16, 16 channels: the places of this lane's reads.
    constexpr int D = SHARED ? DQK : DV, CH = D / 8;
    const int ka = 4 * g + (c >> 2);
    auto value = [&](int t, int b) {
        const uint16_t *vt = tiles[t % 3] + (SHARED ? 0 : KT * DQK);
        const int ch = 2 * (w * C::NB + b) + ((c & 3) >> 1);
        const bf16x4_t u = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_t *)(vt + ka * D + place<CH, SHARED>(ka, ch) * 8 + 4 * (c & 1)));
        const bf16x4_t v = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_t *)(vt + (ka + 16) * D + place<CH, SHARED>(ka + 16, ch) * 8 + 4 * (c & 1)));
        return __builtin_shufflevector(u, v, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    auto values = [&](int t) {
        bf16x8_t p[C::PL * MT];
#pragma unroll
        for (int i = 0; i < C::PL * MT; ++i) p[i] = frag(((const u32x4 *)mix)[((t & 1) * C::PL * MT + i) * 64 + lane]);
#pragma unroll
        for (int b = 0; b < C::NB; ++b) {
            const bf16x8_t f = value(t, b);
#pragma unroll
            for (int i = 0; i < C::PL * MT; ++i) o[i % MT][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, p[i], o[i % MT][b], 0, 0, 0);
        }
    };

    float m_row[MT], l_row[MT], exact_row[MT];   // of rows 16 t + c, in every wave
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        m_row[t] = neg_inf();
        l_row[t] = exact_row[t] = 0.f;
    }
    if (tb < te) {
        int next;
        {                                        // the first two tiles in flight together
            const int at0 = rows_of(tb), at1 = rows_of(tb + 1);
            u32x4 k2[C::NK], v2[C::NV > 0 ? C::NV : 1];
            next = rows_of(tb + 2);
            load(at0);
            if (tb + 1 < te) load_to(at1, k2, v2);
#pragma unroll
            for (int i = 0; i < C::PER; ++i) {
                const int r = row_of(16 * mt_of(i) + c), tok = token_of(a, r), head = y * a.group + r - tok * a.group;
                const uint16_t *from = a.Q + (int64_t)(s.start + tok) * a.q_tok + (int64_t)head * a.q_head + 8 * g;
                seen[i] = sight(a, s, recent, tok);
#pragma unroll
                for (int k = 0; k < C::KS; ++k)
                    q[i][k] = frag(mine(i) && 16 * mt_of(i) + c < rows ? *(const u32x4 *)(from + 32 * k) : u32x4{0, 0, 0, 0});
            }
            store(tb);
            if (tb + 2 < te) load(next);
            next = rows_of(tb + 3);
            if (tb + 1 < te) store_from(tb + 1, k2, v2);
        }
        __syncthreads();
        score(tb);
#pragma unroll
        for (int i = 0; i < C::PER; ++i) {       // (masked keys too: any score is a reference)
            float top = fmaxf(fmaxf(z[i][0], z[i][1]), fmaxf(z[i][2], z[i][3]));
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            if (g == 0 && mine(i)) ends[0][mt_of(i)][kb][c] = top;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < C::PER; ++i) {
            const int mt = mine(i) ? mt_of(i) : 0;
            ref[i] = fmaxf(ends[0][mt][0][c], ends[0][mt][1][c]);
            ref[i] = fabsf(ref[i]) < __builtin_inff() ? ref[i] : 0.f;
            cm[i] = ref[i] * a.scale_log2;
            // below kFar the rounding of cm is 2^-14 log2 units at most; beyond, scores are subtracted before they
            // are scaled (of nearby scores the difference is exact)
            far |= __ballot(!(fabsf(cm[i]) < kFar)) != 0;
            l[i] = exact[i] = 0.f;
            met[i] = false;
        }
#pragma unroll
        for (int i = 0; i < C::PER; ++i) cm[i] = far ? 0.f : cm[i];
        probabilities(tb);
        __syncthreads();
        for (int t = tb; t < te; ++t) {
            if (t + 1 < te) score(t + 1);
            if (t + 2 < te) store(t + 2);        // (over tile t - 1, which every wave has weighted)
            if (t + 3 < te) load(next);
            next = rows_of(t + 4);
            if (t + 1 < te) probabilities(t + 1);
            values(t);
            __syncthreads();
        }
#pragma unroll
        for (int i = 0; i < C::PER; ++i) {
            l[i] += __shfl_xor(l[i], 16);
            l[i] += __shfl_xor(l[i], 32);
            exact[i] += __shfl_xor(exact[i], 16);
            exact[i] += __shfl_xor(exact[i], 32);
            const uint64_t any = __ballot(met[i]);
            if (g == 0 && mine(i)) {
                ends[1][mt_of(i)][kb][c] = l[i];
                ends[2][mt_of(i)][kb][c] = (any >> c | any >> (16 + c) | any >> (32 + c) | any >> (48 + c)) & 1 ? exact[i] : -1.f;
            }
        }
        __syncthreads();
        bool again = odd && t_last > t_first;
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            const float top = fmaxf(ends[0][t][0][c], ends[0][t][1][c]);
            m_row[t] = fabsf(top) < __builtin_inff() ? top : 0.f;
            l_row[t] = ends[1][t][0][c] + ends[1][t][1][c];
            const float exact0 = ends[2][t][0][c], exact1 = ends[2][t][1][c];
            exact_row[t] = (exact0 < 0.f ? 0.f : exact0) + (exact1 < 0.f ? 0.f : exact1);
            if (16 * t + c >= rows) continue;
            if (exact0 < 0.f && exact1 < 0.f) {
                m_row[t] = neg_inf();            // (no key of the part's)
                continue;
            }
            again |= !(l_row[t] > 0x1p-64f && l_row[t] < 0x1p100f);
#pragma unroll
            for (int b = 0; b < C::NB; ++b)
#pragma unroll
                for (int r = 0; r < 4; ++r) again |= !(fabsf(o[t][b][r]) < __builtin_inff());
        }
        if (any_of(again, (int *)tiles)) {
            // Tile by tile: every wave forms the probabilities of all rows, with a running maximum.
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                m_row[t] = neg_inf();
                l_row[t] = exact_row[t] = 0.f;
#pragma unroll
                for (int b = 0; b < C::NB; ++b) o[t][b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            }
#pragma unroll 1
            for (int t = tb; t < te; ++t) {
                const int j0 = x.key(t, KT);
                load(rows_of(t));
                store(t);
                __syncthreads();
                score(t);
#pragma unroll
                for (int i = 0; i < C::PER; ++i)
                    if (mine(i)) *(f32x4_t *)(mix + (16 * mt_of(i) + c) * C::SS + 16 * kb + 4 * g) = z[i];
                __syncthreads();
                const uint16_t *vt = tiles[t % 3] + (SHARED ? 0 : KT * DQK);
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    const Sight see = sight(a, s, recent, token_of(a, row_of(16 * i + c)));
                    float e[8], top = neg_inf(), sum = 0.f, rounded = 0.f;
#pragma unroll
                    for (int r = 0; r < 8; ++r) {
                        const int k = 16 * (r >> 2) + 4 * g + (r & 3);
                        e[r] = sees(see, sink, j0 + k) ? mix[(16 * i + c) * C::SS + k] : neg_inf();
                        top = fmaxf(top, e[r]);
                    }
                    top = fmaxf(top, __shfl_xor(top, 16));
                    top = fmaxf(top, __shfl_xor(top, 32));
                    const float up = fmaxf(m_row[i], top), base = up == neg_inf() ? 0.f : up;
                    const float alpha = up == m_row[i] ? 1.f : __builtin_amdgcn_exp2f((m_row[i] - up) * a.scale_log2);
                    m_row[i] = up;
                    bf16x8_t p, rest;
#pragma unroll
                    for (int r = 0; r < 8; ++r) {
                        const float v = __builtin_amdgcn_exp2f((e[r] - base) * a.scale_log2);
                        sum += v;
                        p[r] = (__bf16)v;
                        rest[r] = (__bf16)(v - (float)p[r]);
                        rounded += (float)p[r];
                    }
                    l_row[i] = l_row[i] * alpha + (C::PL == 2 ? sum : rounded);
                    exact_row[i] = exact_row[i] * alpha + sum;
#pragma unroll
                    for (int b = 0; b < C::NB; ++b) {
                        const bf16x8_t f = frag(finite_only(__builtin_bit_cast(u32x4, value(t, b))));
                        o[i][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, p, o[i][b] * alpha, 0, 0, 0);
                        if (C::PL == 2) o[i][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, rest, o[i][b], 0, 0, 0);
                    }
                    // infinities and NaNs for the rows that see them (any weight leaves them as they are)
#pragma unroll 1
                    for (int k = 0; k < KT; ++k) {
                        if (!sees(see, sink, j0 + k)) continue;
#pragma unroll
                        for (int b = 0; b < C::NB; ++b) {
                            const uint2 v = *(const uint2 *)(vt + k * D + place<CH, SHARED>(k, 2 * (w * C::NB + b) + (g >> 1)) * 8 + 4 * (g & 1));
                            o[i][b] += f32x4_t{special_only(v.x & 0xffffu), special_only(v.x >> 16), special_only(v.y & 0xffffu), special_only(v.y >> 16)};
                        }
                    }
                }
                __syncthreads();
            }
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                l_row[t] += __shfl_xor(l_row[t], 16);
                l_row[t] += __shfl_xor(l_row[t], 32);
                exact_row[t] += __shfl_xor(exact_row[t], 16);
                exact_row[t] += __shfl_xor(exact_row[t], 32);
            }
        }
    }

    // Results: to the output, or to the part's slot.
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int r = 16 * t + c;
        if (r >= rows) continue;
        if (item.parts == 1) {
            const int tok = token_of(a, r0 + r), head = y * a.group + r0 + r - tok * a.group;
            const bool none = blind(sight(a, s, recent, tok), sink);
            const float inv = none ? 0.f : 1.f / l_row[t];
            const int64_t to = (int64_t)(s.start + tok) * a.o_tok + (int64_t)head * a.o_head + 4 * g;
#pragma unroll
            for (int b = 0; b < C::NB; ++b) {
                if (SHARED) *(f32x4_t *)((float *)a.O + to + 16 * (w * C::NB + b)) = o[t][b] * inv;
                else *(uint2 *)(a.O + to + 16 * (w * C::NB + b)) = pack4(o[t][b] * inv);
            }
            if (a.lse && w == 0 && g == 0)
                a.lse[(int64_t)head * a.n_tokens + s.start + tok] =
                    none ? neg_inf() : fmaf(m_row[t] * kLn2, a.scale_log2, logf(exact_row[t]));
        } else {
            float *slot = a.part + (int64_t)(item.slot + item.part * item.step) * (C::ROWS * part_width(DV));
            const float by = moderate(&m_row[t], &l_row[t], &exact_row[t], a.scale_log2);
#pragma unroll
            for (int b = 0; b < C::NB; ++b) *(f32x4_t *)(slot + r * DV + 16 * (w * C::NB + b) + 4 * g) = o[t][b] * by;
            if (w == 0 && g == 0) {
                slot[C::ROWS * DV + r] = m_row[t];
                slot[C::ROWS * DV + C::ROWS + r] = l_row[t];
                if (!SHARED) slot[C::ROWS * DV + 2 * C::ROWS + r] = exact_row[t];
            }
        }
    }
}

// One workgroup joins CH channels of a row of a cut item: CH / 4 threads take 4 each, kLanes of them every
// kLanes'th part, and their sums meet in LDS in a fixed order.  WIDE: the output is fp32.  grid: x = cut item, y = row, z = channels.
template <int D, int ROWS, bool WIDE, int CH>
__global__ __launch_bounds__(kJoinThreads) void paged_join_kernel(PagedArgs a) {
    constexpr int kLanes = kJoinThreads / (CH / 4), kAtOnce = 4;
    __shared__ join_f32x4 sum[kLanes][CH / 4];
    __shared__ float top[kLanes], total[kLanes], exact[kLanes];
    if ((int)blockIdx.x >= a.joins[0].count) return;
    const JoinItem j = a.joins[blockIdx.x];
    const int r = blockIdx.y, d = threadIdx.x % (CH / 4), lane = threadIdx.x / (CH / 4), ch = CH * blockIdx.z + 4 * d;
    if (r >= j.rows) return;
    const int64_t step = (int64_t)j.step * (ROWS * part_width(D));
    const float *p = a.part + (int64_t)j.slot * (ROWS * part_width(D)), *po = p + r * D + ch, *pm = p + ROWS * D + r, *pl = pm + ROWS;
    Joined x;
    for (int k0 = lane; k0 < j.parts; k0 += kAtOnce * kLanes) {
        float m[kAtOnce], l[kAtOnce], e[kAtOnce];
        join_f32x4 o[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const int64_t at = min(k0 + k * kLanes, j.parts - 1) * step;
            m[k] = pm[at];
            l[k] = pl[at];
            e[k] = WIDE ? 0.f : pl[at + ROWS];
            o[k] = *(const join_f32x4 *)(po + at);
        }
        // (all loads before the first use: one memory latency, not one each)
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k)
            if (k0 + k * kLanes < j.parts) x.add(m[k], l[k], e[k], o[k], a.scale_log2);
    }
    sum[lane][d] = x.acc;
    if (d == 0) {
        top[lane] = x.M;
        total[lane] = x.L;
        exact[lane] = x.E;
    }
    __syncthreads();
    if (lane > 0) return;
    for (int i = 1; i < kLanes; ++i) x.add(top[i], total[i], exact[i], sum[i][d], a.scale_log2);
    x.put<WIDE>(a, j, r, ch);
}

template <int DQK, int DV, bool SHARED, int NW>
void launch_rows(const PagedArgs &a, int rows, hipStream_t s) {
    auto go = [&](auto mt) {
        constexpr int MT = decltype(mt)::value, kCh = DV == 512 ? 128 : DV == 256 ? 64 : DV;
        hipLaunchKernelGGL((paged_attn_kernel<DQK, DV, SHARED, MT, NW>), dim3((unsigned)a.n_work), dim3(64 * NW), 0, s, a);
        if (a.target > 0) hipLaunchKernelGGL((paged_join_kernel<DV, 16 * MT, SHARED, kCh>), dim3((unsigned)a.n_joins, 16 * MT, DV / kCh), dim3(kJoinThreads), 0, s, a);
    };
    if (rows <= 16) go(std::integral_constant<int, 1>{});
    else if (rows <= 32) go(std::integral_constant<int, 2>{});
    else if (rows <= 48) go(std::integral_constant<int, 3>{});
    else go(std::integral_constant<int, 4>{});
}

}  // namespace

hipError_t launch_paged_attention(const PagedArgs &a, int head_dim, int rows, hipStream_t s) {
    if (head_dim == 64) launch_rows<64, 64, false, 4>(a, rows, s);
    else launch_rows<128, 128, false, 4>(a, rows, s);
    return hipGetLastError();
}

hipError_t launch_latent_rows(const PagedArgs &a, int latent_dim, int rows, hipStream_t s) {
    if (latent_dim == 256) launch_rows<256 + kLatentRot, 256, true, 8>(a, rows, s);
    else launch_rows<512 + kLatentRot, 512, true, 8>(a, rows, s);
    return hipGetLastError();
}

}  // namespace fkv
