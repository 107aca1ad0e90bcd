// k_attn_q8.hip -- attention over a rolling cache held in 8 bits (E4M3 codes, a
// power-of-two scale for each head and block of tokens), any number of query
// tokens, gfx950 MFMA.
//
// For head h the keys are its kept history tokens (the frames of a static
// head's budget, Eq. 2; the kept segments of a dynamic head, Eq. 3/4), read in
// place from the 8-bit cache, then the n_cur current tokens in bf16; every query
// row attends to all of them.  v_cvt_scalef32_pk_bf16_fp8 turns two codes and
// their block's scale into two bf16 values exactly, so after the conversion the
// arithmetic is that of a bf16 cache.
//
// One wave works on its own: it takes every 8th tile of 64 keys of its
// workgroup's part, keeps its own running maximum, sum and output, and meets the
// other waves once, at the end.  With v_mfma_f32_16x16x32_bf16, for 16 query rows:
//   S^T = K Q^T   (A = 16 key rows straight from global memory: lane l holds
//                 channels 64u + 16(l/16) .. + 16 of key l%16, u = 0.., in the
//                 order in which the products consume them; the queries'
//                 fragments are loaded in the same order),
//   softmax       per query column, fp32, in log2 units, running maximum;
//   O^T += V^T P^T (A = V^T through the LDS transpose read: the wave stores its
//                 64 value rows as bf16 and reads 4 keys of 16 channels at a
//                 time, B = P straight from the S^T accumulators).
// The sum adds the probabilities before they are rounded to bf16 for the value
// product.  Parts of an item (head, query tile) meet in fp32 slots of the
// workspace; the workgroup that arrives last joins them in order.
#include "handover.h"
#include "fkv_internal.h"

namespace fkv {
namespace {

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr int kThreads = 512, kWaves = 8;
constexpr int kTile = 64;                 // keys per tile
constexpr int kRows = kAttnQ8Rows;        // query rows per tile
constexpr float kLn2 = 0.69314718055994530942f;

__device__ __forceinline__ float neg_inf() { return -__builtin_inff(); }

// j / P for 0 <= j < 2^31 with floor(2^64 / P) + 1 = hi * 2^32 + lo (0 for P = 1).
__device__ __forceinline__ int div_magic(int j, uint32_t hi, uint32_t lo) {
    if (hi == 0 && lo == 0) return j;
    return (int)(((uint64_t)(uint32_t)j * hi + __umulhi((uint32_t)j, lo)) >> 32);
}

// LDS written by other lanes of the wave is read after this (and the reverse): a
// wave's LDS operations finish in order, so it only keeps the compiler's order.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// One head's kept history: its length and where its tokens lie.
struct History {
    int kvl, kept, first, gap;
    const int32_t *segs;      // kept_seg row (dynamic)
};
__device__ __forceinline__ History history_of(const AttnQ8Args &a, int h) {
    History x;
    x.kept = a.st_kept[h];
    x.first = a.st_first[h];
    x.gap = a.st_gap[h];
    x.segs = a.kept_seg + (int64_t)h * a.n_seg;
    if (x.kept >= 0) {
        x.kvl = x.kept * a.F;
    } else {
        const int n = a.kv_len[h], most = a.H * a.F;
        x.kvl = n < 0 ? 0 : n > most ? most : n;
    }
    return x;
}

// Kept token j (0 <= j < kvl): its slot and its row within the frame.  A kept_seg
// row and kv_len that disagree must not address outside the head's cache: ids
// and tokens are clamped.
struct Place {
    int slot, p;
};
__device__ __forceinline__ Place place_of(const AttnQ8Args &a, const History &x, const int *slots, int j) {
    int t, p;
    if (x.kept >= 0) {
        const int y = div_magic(j, a.mf_hi, a.mf_lo);
        p = j - y * a.F;
        t = y < x.first ? y : y + x.gap;
    } else {
        const int q = div_magic(j, a.ml_hi, a.ml_lo);
        const int g = min(max(x.segs[q], 0), a.n_seg - 1);
        const int tok = min(g * a.L + (j - q * a.L), a.H * a.F - 1);
        t = div_magic(tok, a.mf_hi, a.mf_lo);
        p = tok - t * a.F;
    }
    return Place{slots[t], p};
}

// Two codes and their scale as bf16 (exact).
template <bool HI>
__device__ __forceinline__ uint32_t widen2(uint32_t codes, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, HI));
}
__device__ __forceinline__ u32x4 widen8(uint32_t c0, uint32_t c1, float scale) {
    return u32x4{widen2<false>(c0, scale), widen2<true>(c0, scale), widen2<false>(c1, scale), widen2<true>(c1, scale)};
}
__device__ __forceinline__ bf16x8_t frag(const u32x4 &v) { return __builtin_bit_cast(bf16x8_t, v); }

template <int D>
struct Cfg {
    static constexpr int U = D / 64;              // 64-channel halves of a row
    static constexpr int KS = D / 32;             // steps of the score product
    static constexpr int MB = D / 16;             // 16-channel blocks of the output
    // Value rows in LDS, padded by 32 bytes: the four rows that a transpose read
    // covers, and the eight that a 16-byte store covers, then fall into distinct banks.
    static constexpr int VS = D + 16;
    static constexpr int REGION = kTile * VS;     // elements per wave
    static constexpr int OS = D + 4;              // a wave's output rows in LDS (floats)
    static_assert(kRows * OS * 4 + 2 * kRows * 4 <= REGION * 2, "a wave's result fits its value rows");
};

typedef __attribute__((address_space(3))) bf16x4_t lds_bf16x4_t;

template <int D>
struct Wave {
    using C = Cfg<D>;
    bf16x8_t q[C::KS];
    f32x4_t o[C::MB];
    float m, l;             // running maximum (log2 units) and this lane's share of the sum

    // The tile's scores s[i] (keys 16i + 4(lane/16) + r of column lane%16) become
    // probabilities; keys from `valid` on do not exist.
    __device__ __forceinline__ void softmax(f32x4_t (&s)[4], float scale_log2, int valid, int g) {
        float top = neg_inf();
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float z = s[i][r] * scale_log2;
                s[i][r] = 16 * i + 4 * g + r < valid ? z : neg_inf();
                top = fmaxf(top, s[i][r]);
            }
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float mn = fmaxf(m, top), base = mn == neg_inf() ? 0.f : mn;
        const float alpha = __builtin_amdgcn_exp2f(m - base);
        m = mn;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                s[i][r] = __builtin_amdgcn_exp2f(s[i][r] - base);
                sum += s[i][r];
            }
        l = l * alpha + sum;
        if (__ballot(alpha != 1.f)) {
#pragma unroll
            for (int mb = 0; mb < C::MB; ++mb) o[mb] *= alpha;
        }
    }

    // O^T += V^T P^T with the tile's value rows in LDS.
    __device__ __forceinline__ void values(const f32x4_t (&p)[4], uint16_t *v, int lane) {
        const int g = lane >> 4, c = lane & 15;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            bf16x8_t b;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                b[r] = (__bf16)p[2 * t][r];
                b[4 + r] = (__bf16)p[2 * t + 1][r];
            }
            uint16_t *row = v + (32 * t + 4 * g + (c >> 2)) * C::VS + 4 * (c & 3);
#pragma unroll
            for (int mb = 0; mb < C::MB; ++mb) {
                const bf16x4_t x = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_t *)(row + 16 * mb));
                const bf16x4_t y = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_t *)(row + 16 * C::VS + 16 * mb));
                const bf16x8_t f = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
                o[mb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, b, o[mb], 0, 0, 0);
            }
        }
    }
};

// grid: (head, query tile, part), part innermost.
template <int D>
__global__ __launch_bounds__(kThreads) void attn_q8_kernel(AttnQ8Args a) {
    using C = Cfg<D>;
    __shared__ __attribute__((aligned(16))) uint16_t lds[kWaves * C::REGION];
    __shared__ int slots[FKV_MAX_FRAMES];
    __shared__ uint32_t flag;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, g = lane >> 4, c = lane & 15;
    const int part = blockIdx.x % a.n_split, item = blockIdx.x / a.n_split;
    const int h = item / a.n_qtiles, q0 = (item - h * a.n_qtiles) * kRows;
    if (tid < a.H) slots[tid] = a.slots.slot[tid];
    __syncthreads();

    const History x = history_of(a, h);
    const int th = (x.kvl + kTile - 1) / kTile, T = th + (a.n_cur + kTile - 1) / kTile;
    const int t0 = (int)((int64_t)T * part / a.n_split), t1 = (int)((int64_t)T * (part + 1) / a.n_split);

    Wave<D> s;
    s.m = neg_inf();
    s.l = 0.f;
#pragma unroll
    for (int mb = 0; mb < C::MB; ++mb) s.o[mb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    const bool row_ok = q0 + c < a.n_q;
#pragma unroll
    for (int k = 0; k < C::KS; ++k) {
        const int d = (k >> 1) * 64 + g * 16 + (k & 1) * 8;
        s.q[k] = frag(row_ok ? *(const u32x4 *)(a.Q + ((int64_t)h * a.n_q + q0 + c) * D + d) : u32x4{0, 0, 0, 0});
    }
    uint16_t *vt = lds + w * C::REGION;
    const uint8_t *K8 = a.K8 + (int64_t)h * a.cap * a.F * D, *V8 = a.V8 + (int64_t)h * a.cap * a.F * D;
    const float *ks = a.k_scale + (int64_t)h * a.cap * a.n_blocks, *vs = a.v_scale + (int64_t)h * a.cap * a.n_blocks;
    const uint16_t *Kn = a.K_cur + (int64_t)h * a.n_cur * D, *Vn = a.V_cur + (int64_t)h * a.n_cur * D;

    for (int t = t0 + w; t < t1; t += kWaves) {
        f32x4_t z[4];
        const bool hist = t < th;
        const int j0 = (hist ? t : t - th) * kTile, valid = (hist ? x.kvl : a.n_cur) - j0;
        if (hist) {
            const Place at = place_of(a, x, slots, min(j0 + lane, x.kvl - 1));
            const int row = at.slot * a.F + at.p, blk = at.slot * a.n_blocks + (at.p >> a.block_shift);
            const float sk = ks[blk], sv = vs[blk];
            u32x4 kr[4][C::U], vr[4][C::U];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t off = (uint32_t)__shfl(row, 16 * i + c) * D + g * 16;
#pragma unroll
                for (int u = 0; u < C::U; ++u) {
                    kr[i][u] = *(const u32x4 *)(K8 + off + 64 * u);
                    vr[i][u] = *(const u32x4 *)(V8 + off + 64 * u);
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float sc = __shfl(sk, 16 * i + c);
                z[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < C::KS; ++k) {
                    const u32x4 r = kr[i][k >> 1];
                    z[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(frag(widen8(r[2 * (k & 1)], r[2 * (k & 1) + 1], sc)),
                                                                   s.q[k], z[i], 0, 0, 0);
                }
            }
            wave_sync();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float sc = __shfl(sv, 16 * i + c);
                const bool ok = 16 * i + c < valid;
#pragma unroll
                for (int u = 0; u < C::U; ++u) {
                    const u32x4 r = ok ? vr[i][u] : u32x4{0, 0, 0, 0};   // no NaN of a row past the end
                    u32x4 *dst = (u32x4 *)(vt + (16 * i + c) * C::VS + 64 * u + 16 * g);
                    dst[0] = widen8(r[0], r[1], sc);
                    dst[1] = widen8(r[2], r[3], sc);
                }
            }
        } else {
            wave_sync();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int key = 16 * i + c;
                const bool ok = key < valid;
                const int64_t off = (int64_t)(j0 + (ok ? key : 0)) * D + g * 16;
                z[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < C::KS; ++k) {
                    const u32x4 r = *(const u32x4 *)(Kn + off + 64 * (k >> 1) + 8 * (k & 1));
                    z[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(frag(r), s.q[k], z[i], 0, 0, 0);
                }
#pragma unroll
                for (int u = 0; u < C::U; ++u) {
                    u32x4 *dst = (u32x4 *)(vt + key * C::VS + 64 * u + 16 * g);
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        dst[e] = ok ? *(const u32x4 *)(Vn + off + 64 * u + 8 * e) : u32x4{0, 0, 0, 0};
                }
            }
        }
        s.softmax(z, a.scale_log2, valid, g);
        wave_sync();
        s.values(z, vt, lane);
    }

    // the wave's result into its region of LDS: output rows, maxima, sums
    s.l += __shfl_xor(s.l, 16);
    s.l += __shfl_xor(s.l, 32);
    wave_sync();
    float *mine = (float *)vt;
#pragma unroll
    for (int mb = 0; mb < C::MB; ++mb) *(f32x4_t *)(mine + c * C::OS + 16 * mb + 4 * g) = s.o[mb];
    if (lane < kRows) {
        mine[kRows * C::OS + lane] = s.m;
        mine[kRows * C::OS + kRows + lane] = s.l;
    }
    __syncthreads();

    // thread -> row r, channels d .. d + 3
    const int r = tid / (D / 4), d = tid % (D / 4) * 4;
    const bool active = r < kRows && q0 + r < a.n_q;
    float M = neg_inf(), L = 0.f;
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
    if (active) {
        const float *base = (const float *)lds;
        constexpr int RF = C::REGION / 2;                 // floats per region
        for (int i = 0; i < kWaves; ++i) M = fmaxf(M, base[i * RF + kRows * C::OS + r]);
        const float ref = M == neg_inf() ? 0.f : M;
        for (int i = 0; i < kWaves; ++i) {
            const float wt = __builtin_amdgcn_exp2f(base[i * RF + kRows * C::OS + r] - ref);
            L += wt * base[i * RF + kRows * C::OS + kRows + r];
            acc += wt * *(const f32x4_t *)(base + i * RF + r * C::OS + d);
        }
    }
    const int64_t out_row = (int64_t)h * a.n_q + q0 + r;
    if (a.n_split > 1) {
        float *slots_of = a.part + (size_t)item * a.n_split * (kRows * (D + 2));
        float *slot = slots_of + (size_t)part * (kRows * (D + 2));
        if (active) {
            uint64_t *dst = (uint64_t *)(slot + r * D + d);
            put_shared((unsigned long long *)dst, make_uint2(__float_as_uint(acc[0]), __float_as_uint(acc[1])));
            put_shared((unsigned long long *)dst + 1, make_uint2(__float_as_uint(acc[2]), __float_as_uint(acc[3])));
            if (d == 0) {
                put_shared(slot + kRows * D + r, M);
                put_shared(slot + kRows * D + kRows + r, L);
            }
        }
        if (!arrive_last(a.counters + (size_t)item * kItemCounterStride, (uint32_t)a.n_split, &flag)) return;
        M = neg_inf();
        L = 0.f;
        acc = f32x4_t{0.f, 0.f, 0.f, 0.f};
        if (active) {
            for (int j = 0; j < a.n_split; ++j) {
                const float *p = slots_of + (size_t)j * (kRows * (D + 2));
                const float mj = get_shared(p + kRows * D + r), lj = get_shared(p + kRows * D + kRows + r);
                const uint2 u = get_shared((const uint2 *)(p + r * D + d)), v = get_shared((const uint2 *)(p + r * D + d) + 1);
                const float Mn = fmaxf(M, mj), ref = Mn == neg_inf() ? 0.f : Mn;
                const float so = __builtin_amdgcn_exp2f(M - ref), sn = __builtin_amdgcn_exp2f(mj - ref);
                M = Mn;
                L = L * so + lj * sn;
                acc[0] = acc[0] * so + __uint_as_float(u.x) * sn;
                acc[1] = acc[1] * so + __uint_as_float(u.y) * sn;
                acc[2] = acc[2] * so + __uint_as_float(v.x) * sn;
                acc[3] = acc[3] * so + __uint_as_float(v.y) * sn;
            }
        }
    }
    if (!active) return;
    if (T == 0) {                                          // no key at all
        *(uint2 *)(a.O + out_row * D + d) = make_uint2(0, 0);
        if (a.lse && d == 0) a.lse[out_row] = neg_inf();
        return;
    }
    const float inv = 1.f / L;
    uint32_t b[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) b[e] = __builtin_bit_cast(uint16_t, (__bf16)(acc[e] * inv));
    *(uint2 *)(a.O + out_row * D + d) = make_uint2(b[0] | (b[1] << 16), b[2] | (b[3] << 16));
    if (a.lse && d == 0) a.lse[out_row] = fmaf(M, kLn2, logf(L));
}

// Large chunks: the kept history as a bf16 copy [n_heads][slab][d] for the chunk
// attention's kernel.  A workgroup widens kExpandRows rows of K and V; 16 bytes
// of codes per thread and row.  grid: x = row group, y = head.
constexpr int kExpandThreads = 256, kExpandRows = 128;
template <int D>
__global__ __launch_bounds__(kExpandThreads) void expand_q8_kernel(AttnQ8Args a) {
    constexpr int TPR = D / 16, RPP = kExpandThreads / TPR, N = kExpandRows / RPP;   // threads per row, rows per pass
    __shared__ int slots[FKV_MAX_FRAMES];
    const int tid = threadIdx.x, h = blockIdx.y;
    if (tid < a.H) slots[tid] = a.slots.slot[tid];
    __syncthreads();
    const History x = history_of(a, h);
    if (blockIdx.x == 0 && tid == 0) a.kv_out[h] = x.kvl;
    // the arrival counters of the attention launch that follows
    const int64_t n_threads = (int64_t)gridDim.x * gridDim.y * kExpandThreads;
    for (int64_t i = ((int64_t)h * gridDim.x + blockIdx.x) * kExpandThreads + tid; i < a.n_counters; i += n_threads)
        a.counters[i * kItemCounterStride] = 0;
    const int j0 = blockIdx.x * kExpandRows + tid / TPR, c = tid % TPR * 16;
    const uint8_t *K8 = a.K8 + (int64_t)h * a.cap * a.F * D, *V8 = a.V8 + (int64_t)h * a.cap * a.F * D;
    const float *ks = a.k_scale + (int64_t)h * a.cap * a.n_blocks, *vs = a.v_scale + (int64_t)h * a.cap * a.n_blocks;
    u32x4 k[N], v[N];
    float sk[N], sv[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int j = j0 + i * RPP;
        if (j < x.kvl) {
            const Place at = place_of(a, x, slots, j);
            const uint32_t off = (uint32_t)(at.slot * a.F + at.p) * D + c, blk = at.slot * a.n_blocks + (at.p >> a.block_shift);
            k[i] = __builtin_nontemporal_load((const u32x4 *)(K8 + off));
            v[i] = __builtin_nontemporal_load((const u32x4 *)(V8 + off));
            sk[i] = ks[blk];
            sv[i] = vs[blk];
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int j = j0 + i * RPP;
        if (j < x.kvl) {
            const int64_t off = ((int64_t)h * a.slab + j) * D + c;
            u32x4 *dk = (u32x4 *)(a.Kc + off), *dv = (u32x4 *)(a.Vc + off);
            dk[0] = widen8(k[i][0], k[i][1], sk[i]);
            dk[1] = widen8(k[i][2], k[i][3], sk[i]);
            dv[0] = widen8(v[i][0], v[i][1], sv[i]);
            dv[1] = widen8(v[i][2], v[i][3], sv[i]);
        }
    }
}

}  // namespace

hipError_t launch_expand_q8(const AttnQ8Args &a, int head_dim, hipStream_t s) {
    const int64_t groups = (a.slab + kExpandRows - 1) / kExpandRows;
    const dim3 grid((unsigned)(groups > 0 ? groups : 1), (unsigned)a.n_heads);
    if (head_dim == 64) hipLaunchKernelGGL(expand_q8_kernel<64>, grid, dim3(kExpandThreads), 0, s, a);
    else hipLaunchKernelGGL(expand_q8_kernel<128>, grid, dim3(kExpandThreads), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_attention_q8(const AttnQ8Args &a, int head_dim, hipStream_t s) {
    const dim3 grid((unsigned)((int64_t)a.n_heads * a.n_qtiles * a.n_split));
    if (head_dim == 64) hipLaunchKernelGGL(attn_q8_kernel<64>, grid, dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL(attn_q8_kernel<128>, grid, dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace fkv
