// k_paged_tile.hip -- attention of chunks and prompts of many sequences over paged caches
// (or, EXPANDED, over the keys and values made from latent rows), gfx950 MFMA.
//
// A workgroup of 4 waves takes one part of an item (sequence, key head, tile of 128 query
// rows; the query heads of a key head share a tile) and walks its keys 64 at a time
// through two LDS buffers.  Per wave, 32 query rows and v_mfma_f32_32x32x16_bf16:
//   S^T = K Q^T    (A = K rows from LDS, B = the wave's queries in registers),
//   softmax        per query column, fp32, a running maximum that moves only where a
//                  score passes it by kSlack,
//   O^T += V^T P^T (A = V^T through the LDS transpose read, P straight from S^T).
#include <type_traits>

#include "paged_join.h"

namespace fkv {
namespace {

using namespace paged;

typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) bf16x4_t lds_bf16x4_t;

constexpr int KT = 64, ROWS = kPagedTileRows, NT = 256;
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

template <int DQK, int DV, bool EXPANDED>
__global__ __launch_bounds__(NT, 2) void paged_tile_kernel(PagedArgs a) {
    constexpr int CK = DQK / 8, CV = DV / 8, KS = DQK / 16, MB = DV / 32;
    constexpr int NK = KT * CK / NT, NV = KT * CV / NT;
    __shared__ __attribute__((aligned(16))) uint16_t kts[2][KT * DQK], vts[2][KT * DV];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), hh = lane >> 5, c = lane & 31;

    Work item = locate<ROWS, KT>(a, blockIdx.x, -1);
    if (!item.ok) return;
    Seq s = item.s;
    if (EXPANDED) s.len = (int)min((int64_t)s.len, max(a.head_rows - item.base, (int64_t)0));
    const int y = item.y, r0 = item.rt * ROWS, rows = min(ROWS, s.n * a.group - r0);
    const int sink = a.sink[y], recent = a.recent[y];
    const int t_first = r0 / a.group, t_last = (r0 + rows - 1) / a.group;
    const Tiles x = tiles_of<KT>(a, s, sink, recent, t_first, t_last);
    const int tb = (int)((int64_t)x.n * item.part / item.parts), te = (int)((int64_t)x.n * (item.part + 1) / item.parts);
    const int32_t *pages = a.table + (int64_t)item.i * a.max_pages;

    // This lane's query row.
    const int row = min(32 * w + c, rows - 1) + r0, tok = row / a.group, head = y * a.group + row - tok * a.group;
    const bool live = 32 * w + c < rows;
    const Sight seen = sight(a, s, recent, tok);
    bf16x8_t q[KS];
    {
        const uint16_t *from = a.Q + (int64_t)(s.start + tok) * a.q_tok + (int64_t)head * a.q_head + 8 * hh;
#pragma unroll
        for (int k = 0; k < KS; ++k) q[k] = frag(live ? *(const u32x4 *)(from + 16 * k) : u32x4{0, 0, 0, 0});
    }
    f32x16_t o[MB];
    float m, l;

    // Rows of a tile's keys, one to a lane (past the part's last tile, that one's).
    const int j_last = x.most.end - 1;
    const uint16_t *K = a.K, *V = a.V;
    if (EXPANDED) {
        K += (y * a.head_rows + item.base) * DQK;
        V += (y * a.head_rows + item.base) * DV;
    }
    auto rows_of = [&](int t) {
        const int j = min(x.key(min(t, te - 1), KT) + lane, j_last);
        return EXPANDED ? j : pool_row(a, pages, y, j);
    };
    u32x4 kr[NK], vr[NV];
    bool odd = false;                             // an infinity or a NaN among values that not every row sees
    auto load_k = [&](int row_of_lane) {
#pragma unroll
        for (int i = 0; i < NK; ++i) {
            const int id = tid + i * NT, k = id / CK;
            kr[i] = *(const u32x4 *)(K + (int64_t)__shfl(row_of_lane, k) * DQK + (id - k * CK) * 8);
        }
    };
    auto load_v = [&](int row_of_lane) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int id = tid + i * NT, k = id / CV;
            vr[i] = *(const u32x4 *)(V + (int64_t)__shfl(row_of_lane, k) * DV + (id - k * CV) * 8);
        }
    };
    auto store_k = [&](int t) {
        uint16_t *kt = kts[t & 1];
#pragma unroll
        for (int i = 0; i < NK; ++i) {
            const int id = tid + i * NT, k = id / CK;
            *(u32x4 *)(kt + k * DQK + place<CK, true>(k, id - k * CK) * 8) = kr[i];
        }
    };
    auto store_v = [&](int t) {
        const int j0 = x.key(min(t, te - 1), KT);
        uint16_t *vt = vts[t & 1];
        if (!all_seen<KT>(x, sink, j0)) {
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
            *(u32x4 *)(vt + k * DV + place<CV, false>(k, id - k * CV) * 8) = vr[i];
        }
    };

    // Where this lane reads the tiles: key c (and c + 32) of K, chunk 2 k + hh (the pattern of
    // place() repeats every GK steps); keys 4 hh + 0..3 (and
    // + 8) of V, channels 32 b + 16 (lane / 16 % 2) + 4 (lane % 4) of each four.
    constexpr int GK = (CK % 16 == 0 ? 16 : 8) / 2;
    int ka[GK], va[MB], vb[MB];
    {
        const int vk = 4 * hh + ((lane & 15) >> 2), vc = 2 * (lane >> 4 & 1) + ((lane & 3) >> 1), vh = 4 * (lane & 1);
#pragma unroll
        for (int k = 0; k < GK; ++k) ka[k] = c * DQK + place<CK, true>(c, 2 * k + hh) * 8;
#pragma unroll
        for (int b = 0; b < MB; ++b) {
            va[b] = vk * DV + place<CV, false>(vk, 4 * b + vc) * 8 + vh;
            vb[b] = (vk + 8) * DV + place<CV, false>(vk + 8, 4 * b + vc) * 8 + vh;
        }
    }
    auto clear = [&]() {
        l = 0.f;
#pragma unroll
        for (int b = 0; b < MB; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[b][r] = 0.f;
    };
    // Scores of key block kb (32 keys).
    auto score = [&](const uint16_t *kt, int kb, f32x16_t &z) {
#pragma unroll
        for (int r = 0; r < 16; ++r) z[r] = 0.f;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            const bf16x8_t f = frag(*(const u32x4 *)(kt + 32 * kb * DQK + ka[k % GK] + k / GK * GK * 16));
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
        const uint16_t *at = vt + 16 * k * DV;
        const bf16x4_t u = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_t *)(at + va[b]));
        const bf16x4_t v = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_t *)(at + vb[b]));
        return __builtin_shufflevector(u, v, 0, 1, 2, 3, 4, 5, 6, 7);
    };

    m = neg_inf();
    clear();
    if (tb < te) {
        int next_v = rows_of(tb), next_k = rows_of(tb + 1);   // pool rows of the tiles to load next
        load_k(next_v);
        load_v(next_v);
        store_k(tb);
        load_k(next_k);
        store_v(tb);
        next_v = next_k;
        next_k = rows_of(tb + 2);
        __syncthreads();
        {                                         // the reference: the row's largest score in the first tile, masked keys too
            float top = neg_inf();
#pragma unroll 1
            for (int kb = 0; kb < 2; ++kb) {
                f32x16_t z;
                score(kts[tb & 1], kb, z);
#pragma unroll
                for (int r = 0; r < 16; ++r) top = fmaxf(top, z[r]);
            }
            top = across_max(top);
            m = fabsf(top) < __builtin_inff() ? top : 0.f;
        }
        // 2^(c (z - m)): the product c m is rounded on its own, by 2^-14 log2 units at most below kFar;
        // beyond, scores are subtracted before they are scaled (of nearby scores the difference is exact)
        const bool far = __ballot(!(fabsf(m * a.scale_log2) < kFar)) != 0;
        const float cm = far ? 0.f : m * a.scale_log2;
        bool met = false;
        for (int t = tb; t < te; ++t) {
            if (t > tb) __syncthreads();
            // the next tile's keys, then its values: over tile t - 1, which every wave has weighted (past the
            // end the last tile again)
            store_k(t + 1);
            load_v(next_v);
            const int j0 = x.key(t, KT);
            const uint16_t *kt = kts[t & 1], *vt = vts[t & 1];
            f32x16_t z[2];
            score(kt, 0, z[0]);
            score(kt, 1, z[1]);
            if (far || !all_seen<KT>(x, sink, j0)) {
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) {
                    hide(j0, kb, z[kb]);
                    if (far) z[kb] -= m;
#pragma unroll
                    for (int r = 0; r < 16; ++r) met |= z[kb][r] != neg_inf();
                }
            } else {
                met = true;
            }
            store_v(t + 1);
            load_k(next_k);
            next_v = next_k;
            next_k = rows_of(t + 3);
            float sum[2] = {0.f, 0.f};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                bf16x8_t p;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float v = __builtin_amdgcn_exp2f(fmaf(z[k >> 1][8 * (k & 1) + e], a.scale_log2, -cm));
                    sum[e & 1] += v;
                    p[e] = (__bf16)v;
                }
#pragma unroll
                for (int b = 0; b < MB; ++b) o[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(value(vt, k, b), p, o[b], 0, 0, 0);
            }
            l += sum[0] + sum[1];
        }
        met = (__ballot(met) >> c | __ballot(met) >> (32 + c)) & 1;
        const float all = l + __shfl_xor(l, 32);
        bool again = odd;
        if (live && met) {
            again |= !(all > 0x1p-100f && all < 0x1p100f);
#pragma unroll
            for (int b = 0; b < MB; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) again |= !(fabsf(o[b][r]) < __builtin_inff());
        }
        if (!met) m = neg_inf();                  // (no key of the part's)
        if (any_of(again, (int *)kts)) {
            // Tile by tile with a running maximum; an infinity or a NaN among the values goes to the rows that
            // see it alone.
            m = neg_inf();
            clear();
#pragma unroll 1
            for (int t = tb; t < te; ++t) {
                const int j0 = x.key(t, KT);
                load_k(rows_of(t));
                load_v(rows_of(t));
                store_k(t);
                store_v(t);
                __syncthreads();
                const uint16_t *kt = kts[t & 1], *vt = vts[t & 1];
#pragma unroll 1
                for (int kb = 0; kb < 2; ++kb) {
                    f32x16_t z;
                    score(kt, kb, z);
                    hide(j0, kb, z);
                    float top = neg_inf(), sum = 0.f;
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
                    }
                    l = l * alpha + sum;
#pragma unroll
                    for (int b = 0; b < MB; ++b) {
                        o[b] *= alpha;
#pragma unroll
                        for (int k = 0; k < 2; ++k)
                            o[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag(finite_only(__builtin_bit_cast(u32x4, value(vt + 32 * kb * DV, k, b)))),
                                                                           p[k], o[b], 0, 0, 0);
                    }
#pragma unroll 1
                    for (int k = 32 * kb; k < 32 * kb + 32; ++k) {    // (any weight leaves them as they are)
                        if (!sees(seen, sink, j0 + k)) continue;
#pragma unroll
                        for (int u = 0; u < 4 * MB; ++u) {            // channels 8 u + 4 hh + 0..3
                            const uint2 v = *(const uint2 *)(vt + k * DV + place<CV, false>(k, u) * 8 + 4 * hh);
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
    if (!live) return;
    if (item.parts == 1) {
        const bool none = seen.end <= 0;
        const float inv = none ? 0.f : 1.f / l;
        uint16_t *to = a.O + (int64_t)(s.start + tok) * a.o_tok + (int64_t)head * a.o_head + 4 * hh;
#pragma unroll
        for (int b = 0; b < MB; ++b)
#pragma unroll
            for (int u = 0; u < 4; ++u)
                *(uint2 *)(to + 32 * b + 8 * u) = pack4(o[b][4 * u] * inv, o[b][4 * u + 1] * inv, o[b][4 * u + 2] * inv, o[b][4 * u + 3] * inv);
        if (a.lse && hh == 0)
            a.lse[(int64_t)head * a.n_tokens + s.start + tok] = none ? neg_inf() : fmaf(m * kLn2, a.scale_log2, logf(l));
    } else {
        float *slot = a.part + (int64_t)(item.slot + item.part * item.step) * (ROWS * (DV + 2));
        float *to = slot + (32 * w + c) * DV + 4 * hh;
        const float by = moderate(&m, &l, a.scale_log2);
#pragma unroll
        for (int b = 0; b < MB; ++b)
#pragma unroll
            for (int u = 0; u < 4; ++u)
                *(f32x4_t *)(to + 32 * b + 8 * u) = f32x4_t{o[b][4 * u], o[b][4 * u + 1], o[b][4 * u + 2], o[b][4 * u + 3]} * by;
        if (hh == 0) {
            slot[ROWS * DV + 32 * w + c] = m;
            slot[ROWS * DV + ROWS + 32 * w + c] = l;
        }
    }
}

template <int DQK, int DV, bool EXPANDED>
void launch(const PagedArgs &a, hipStream_t s) {
    hipLaunchKernelGGL((paged_tile_kernel<DQK, DV, EXPANDED>), dim3((unsigned)a.n_work), dim3(NT), 0, s, a);
    if (a.target > 0) launch_join<DV, ROWS, KT, true>(a, s);
}

}  // namespace

hipError_t launch_paged_tiles(const PagedArgs &a, int head_dim, hipStream_t s) {
    if (head_dim == 64) launch<64, 64, false>(a, s);
    else launch<128, 128, false>(a, s);
    return hipGetLastError();
}

hipError_t launch_expanded_tiles(const PagedArgs &a, int head_dim, hipStream_t s) {
    if (head_dim == 64) launch<64 + kLatentRot, 64, true>(a, s);
    else launch<128 + kLatentRot, 128, true>(a, s);
    return hipGetLastError();
}

}  // namespace fkv
