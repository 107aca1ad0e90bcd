// k_paged_attn.hip -- attention of few new tokens of many sequences over paged caches,
// gfx950 MFMA: single tokens and short chunks (up to 64 query rows of a sequence and key
// head), with keys and values of their own or, SHARED, with values that are the first DV
// channels of the key rows (latent rows: all heads read one row).
//
//   o = sum_j 2^(c (s_j - m)) v_j / sum_j 2^(c (s_j - m)),  s_j = q . k_j,  c = scale log2 e
//
// A workgroup takes one part of an item (sequence, key head, tile of 16 MT query rows)
// and walks its keys 32 at a time.  The NW waves share each tile of keys, which is read
// from HBM once and lies in LDS, three tiles deep:
//   scores   S^T = K Q^T (v_mfma_f32_16x16x32_bf16): the tile's 2 x MT blocks, and
//            shares of the channels where there are more waves than blocks, are dealt to
//            the waves; the blocks meet in LDS as fp32;
//   softmax  every wave forms the probabilities of all rows from there, so that no wave
//            waits for another's: running maximum and sum in fp32;
//   values   O^T += V^T P^T: each wave owns DV / NW output channels of all rows (V^T
//            through the LDS transpose read, P straight from the softmax's registers).
// The scores of tile t + 1 and the values of tile t run in the same stretch between two
// barriers, one barrier a tile; tile t + 3 is on its way from HBM meanwhile.
// Probabilities are rounded to bf16 for the value product, the sum adds them before.
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
constexpr float kSlack = 8.f;       // log2 units that the softmax's reference may lag behind
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
    static constexpr int KS = DQK / 32;                              // steps of the score product
    static constexpr int SHARES = NW > BLOCKS ? NW / BLOCKS : 1;     // of the channels, per block
    static constexpr int PER = BLOCKS > NW ? BLOCKS / NW : 1;        // blocks per wave
    static constexpr int STEPS = (KS + SHARES - 1) / SHARES;
    static constexpr int NB = DV / 16 / NW;                          // 16-channel blocks of a wave's output
    static constexpr int NK = (KT * CK + NT - 1) / NT, NV = SHARED ? 0 : (KT * CV + NT - 1) / NT;   // chunks per thread
    static constexpr int TILE = KT * (DQK + (SHARED ? 0 : DV));      // elements
    static constexpr int SS = KT + 4;                                // floats per row of scores: 16 rows in distinct banks
    static constexpr int SCORES = SHARES * ROWS * SS;
    static_assert(DV % (16 * NW) == 0 && KT * CV % NT == 0, "whole blocks and chunks");
};

template <int DQK, int DV, bool SHARED, int MT, int NW>
__global__ __launch_bounds__(64 * NW) void paged_attn_kernel(PagedArgs a) {
    using C = Cfg<DQK, DV, SHARED, MT, NW>;
    __shared__ __attribute__((aligned(16))) uint16_t tiles[3][C::TILE];
    __shared__ __attribute__((aligned(16))) float scores[2][C::SCORES];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, c = lane & 15;

    const Work item = locate<C::ROWS, KT>(a, blockIdx.x, -1);
    if (!item.ok) return;
    const Seq s = item.s;
    const int y = item.y, r0 = item.rt * C::ROWS, rows = min(C::ROWS, s.n * a.group - r0);
    const int sink = a.sink[y], recent = a.recent[y];
    const int t_first = r0 / a.group, t_last = (r0 + rows - 1) / a.group;
    const Tiles x = tiles_of<KT>(a, s, sink, recent, t_first, t_last);
    const int tb = (int)((int64_t)x.n * item.part / item.parts), te = (int)((int64_t)x.n * (item.part + 1) / item.parts);
    const int32_t *pages = a.table + (int64_t)item.i * a.max_pages;

    // This lane's query rows (row 16 t + c).
    Sight seen[MT];
    int64_t q_at[MT], o_at[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int r = min(16 * t + c, rows - 1) + r0, tok = r / a.group, head = y * a.group + r - tok * a.group;
        seen[t] = sight(a, s, recent, tok);
        q_at[t] = (int64_t)(s.start + tok) * a.q_tok + (int64_t)head * a.q_head;
        o_at[t] = (int64_t)(s.start + tok) * a.o_tok + (int64_t)head * a.o_head;
    }

    // Score blocks of this wave: key block kb of row tiles mt0 + (NW / 2) i, channel steps k0 .. k1 - 1.
    const int kb = w & 1, mt0 = C::SHARES > 1 ? (w >> 1) % MT : w >> 1, share = C::SHARES > 1 ? (w >> 1) / MT : 0;
    const int k0 = C::KS * share / C::SHARES, k1 = C::KS * (share + 1) / C::SHARES;
    bf16x8_t q[C::PER][C::STEPS];
#pragma unroll
    for (int i = 0; i < C::PER; ++i) {
        const int mt = mt0 + NW / 2 * i;
        int64_t at = q_at[0];
#pragma unroll
        for (int t = 1; t < MT; ++t) at = mt == t ? q_at[t] : at;
#pragma unroll
        for (int k = 0; k < C::STEPS; ++k)
            q[i][k] = frag(k0 + k < k1 && 16 * mt + c < rows ? *(const u32x4 *)(a.Q + at + 32 * (k0 + k) + 8 * g) : u32x4{0, 0, 0, 0});
    }

    f32x4_t o[MT][C::NB];
    float m[MT], l[MT];
    auto clear = [&]() {
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            m[t] = neg_inf();
            l[t] = 0.f;
#pragma unroll
            for (int b = 0; b < C::NB; ++b) o[t][b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }
    };
    clear();
    bool odd = false;                            // an infinity or a NaN among values that not every row sees

    // Pool rows of a tile's keys, one to a lane (both halves of the wave hold the same 32);
    // keys past the last that a row sees take its place.
    const int j_last = x.most.end - 1;
    auto rows_of = [&](int t) { return t < te ? pool_row(a, pages, y, min(x.key(t, KT) + (lane & 31), j_last)) : 0; };
    u32x4 kr[C::NK], vr[C::NV > 0 ? C::NV : 1];
    auto load = [&](int row_of_lane) {
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
    auto store = [&](int t) {
        const int j0 = x.key(t, KT);
        const bool edge = !all_seen<KT>(x, sink, j0);
        uint16_t *kt = tiles[t % 3], *vt = kt + KT * DQK;
        // (values of keys that no row sees are cleared, a probability of zero would not silence a NaN)
        auto clean = [&](u32x4 &v, int k) {
            if (!sees(x.most, sink, j0 + k)) v = u32x4{0, 0, 0, 0};
            odd |= special(v);
        };
#pragma unroll
        for (int i = 0; i < C::NK; ++i) {
            const int id = tid + i * C::NT, k = id / C::CK;
            if (SHARED && edge) clean(kr[i], k);
            if (id < KT * C::CK) *(u32x4 *)(kt + k * DQK + place<C::CK, true>(k, id - k * C::CK) * 8) = kr[i];
        }
#pragma unroll
        for (int i = 0; i < C::NV; ++i) {
            const int id = tid + i * C::NT, k = id / C::CV;
            if (edge) clean(vr[i], k);
            *(u32x4 *)(vt + k * DV + place<C::CV, false>(k, id - k * C::CV) * 8) = vr[i];
        }
    };
    auto score = [&](int t) {
        const uint16_t *kt = tiles[t % 3] + (16 * kb + c) * DQK;
        f32x4_t z[C::PER];
#pragma unroll
        for (int i = 0; i < C::PER; ++i) z[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < C::STEPS; ++k) {
            if (C::KS % C::SHARES && k0 + k >= k1) break;
            const bf16x8_t f = frag(*(const u32x4 *)(kt + place<C::CK, true>(16 * kb + c, 4 * (k0 + k) + g) * 8));
#pragma unroll
            for (int i = 0; i < C::PER; ++i) z[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, q[i][k], z[i], 0, 0, 0);
        }
        float *to = scores[t & 1] + share * (C::ROWS * C::SS) + c * C::SS + 16 * kb + 4 * g;
#pragma unroll
        for (int i = 0; i < C::PER; ++i) *(f32x4_t *)(to + 16 * (mt0 + NW / 2 * i) * C::SS) = z[i];
    };
    // CAREFUL: where a value is an infinity or a NaN, only the rows that see it get it (a probability of
    // zero times it would be a NaN).
    auto values = [&](int t, auto careful) {
        constexpr bool CAREFUL = decltype(careful)::value;
        const int j0 = x.key(t, KT);
        const bool edge = !all_seen<KT>(x, sink, j0);
        bf16x8_t p[MT];
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            f32x4_t z[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const float *from = scores[t & 1] + (16 * i + c) * C::SS + 16 * u + 4 * g;
                z[u] = *(const f32x4_t *)from;
#pragma unroll
                for (int h = 1; h < C::SHARES; ++h) z[u] += *(const f32x4_t *)(from + h * (C::ROWS * C::SS));
                if (edge) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) z[u][r] = sees(seen[i], sink, j0 + 16 * u + 4 * g + r) ? z[u][r] : neg_inf();
                }
            }
            float top = neg_inf();
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int r = 0; r < 4; ++r) top = fmaxf(top, z[u][r]);
            // The reference moves only where a score passes it by more than kSlack (probabilities up
            // to 2^kSlack lose no digit).  Scores are subtracted before they are scaled: the difference of
            // nearby scores is exact whatever their size.
            if (__ballot((top - m[i]) * a.scale_log2 > kSlack)) {
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                const float next = (top - m[i]) * a.scale_log2 > kSlack ? top : m[i];
                const float alpha = next == m[i] ? 1.f : __builtin_amdgcn_exp2f((m[i] - next) * a.scale_log2);
                m[i] = next;
                l[i] *= alpha;
#pragma unroll
                for (int b = 0; b < C::NB; ++b) o[i][b] *= alpha;
            }
            const float base = m[i] == neg_inf() ? 0.f : m[i];
            float sum = 0.f;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float e = __builtin_amdgcn_exp2f((z[u][r] - base) * a.scale_log2);
                    sum += e;
                    p[i][4 * u + r] = (__bf16)e;
                }
            l[i] += sum;
        }
        const uint16_t *vt = tiles[t % 3] + (SHARED ? 0 : KT * DQK);
        constexpr int D = SHARED ? DQK : DV, CH = D / 8;
        const int ka = 4 * g + (c >> 2), kc = ka + 16;
#pragma unroll
        for (int b = 0; b < C::NB; ++b) {
            const int ch = 2 * (w * C::NB + b) + ((c & 3) >> 1);
            const bf16x4_t u = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_t *)(vt + ka * D + place<CH, SHARED>(ka, ch) * 8 + 4 * (c & 1)));
            const bf16x4_t v = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_t *)(vt + kc * D + place<CH, SHARED>(kc, ch) * 8 + 4 * (c & 1)));
            bf16x8_t f = __builtin_shufflevector(u, v, 0, 1, 2, 3, 4, 5, 6, 7);
            if (CAREFUL) f = frag(finite_only(__builtin_bit_cast(u32x4, f)));
#pragma unroll
            for (int i = 0; i < MT; ++i) o[i][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, p[i], o[i][b], 0, 0, 0);
        }
        if (CAREFUL) {                           // (any weight leaves them as they are)
#pragma unroll 1
            for (int k = 0; k < KT; ++k) {
#pragma unroll
                for (int b = 0; b < C::NB; ++b) {
                    const uint2 v = *(const uint2 *)(vt + k * D + place<CH, SHARED>(k, 2 * (w * C::NB + b) + (g >> 1)) * 8 + 4 * (g & 1));
                    const f32x4_t add = {special_only(v.x & 0xffffu), special_only(v.x >> 16), special_only(v.y & 0xffffu), special_only(v.y >> 16)};
#pragma unroll
                    for (int i = 0; i < MT; ++i)
                        if (sees(seen[i], sink, j0 + k)) o[i][b] += add;
                }
            }
        }
    };

    auto walk = [&](auto careful) {
        int next = rows_of(tb);
        load(next);
        next = rows_of(tb + 1);
        store(tb);
        if (tb + 1 < te) load(next);
        next = rows_of(tb + 2);
        __syncthreads();
        score(tb);
        if (tb + 1 < te) store(tb + 1);
        if (tb + 2 < te) load(next);
        next = rows_of(tb + 3);
        __syncthreads();
        for (int t = tb; t < te; ++t) {
            if (t + 1 < te) score(t + 1);
            if (t + 2 < te) store(t + 2);         // (over tile t - 1, which every wave has weighted)
            if (t + 3 < te) load(next);
            next = rows_of(t + 4);
            values(t, careful);
            __syncthreads();
        }
    };
    if (tb < te) {
        walk(std::false_type{});
        if (t_last > t_first && any_of(odd, (int *)tiles)) {
            clear();
            walk(std::true_type{});
        }
    }

    // Results: to the output, or to the part's slot.
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        l[t] += __shfl_xor(l[t], 16);
        l[t] += __shfl_xor(l[t], 32);
        const int r = 16 * t + c;
        if (r >= rows) continue;
        if (item.parts == 1) {
            const bool none = seen[t].end <= 0;
            const float inv = none ? 0.f : 1.f / l[t];
#pragma unroll
            for (int b = 0; b < C::NB; ++b)
                *(uint2 *)(a.O + o_at[t] + 16 * (w * C::NB + b) + 4 * g) = pack4(o[t][b] * inv);
            if (a.lse && w == 0 && g == 0) {
                const int tok = (r0 + r) / a.group, head = y * a.group + r0 + r - tok * a.group;
                a.lse[(int64_t)head * a.n_tokens + s.start + tok] =
                    none ? neg_inf() : fmaf(m[t] * kLn2, a.scale_log2, logf(l[t]));
            }
        } else {
            float *slot = a.part + (int64_t)(item.slot + item.part * item.step) * (C::ROWS * (DV + 2));
#pragma unroll
            for (int b = 0; b < C::NB; ++b) *(f32x4_t *)(slot + r * DV + 16 * (w * C::NB + b) + 4 * g) = o[t][b];
            if (w == 0 && g == 0) {
                slot[C::ROWS * DV + r] = m[t];
                slot[C::ROWS * DV + C::ROWS + r] = l[t];
            }
        }
    }
}

template <int DQK, int DV, bool SHARED, int NW>
void launch_rows(const PagedArgs &a, int rows, hipStream_t s) {
    auto go = [&](auto mt) {
        constexpr int MT = decltype(mt)::value;
        hipLaunchKernelGGL((paged_attn_kernel<DQK, DV, SHARED, MT, NW>), dim3((unsigned)a.n_work), dim3(64 * NW), 0, s, a);
        if (a.target > 0) launch_join<DV, 16 * MT, KT>(a, s);
    };
    if (rows <= 16) go(std::integral_constant<int, 1>{});
    else if (rows <= 32) go(std::integral_constant<int, 2>{});
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
