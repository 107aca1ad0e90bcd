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
// One wave works on its own: the keys are split in units of 16 over the waves of all
// parts of an item; a wave takes 64 keys a step, keeps its own running maximum, sum
// and output, and meets the other waves once, at the end.  With v_mfma_f32_16x16x32_bf16, for 16 query rows:
//   S^T = K Q^T   (A = 16 key rows straight from global memory: lane l holds
//                 channels 64u + 16(l/16) .. + 16 of key l%16, u = 0.., in the
//                 order in which the products consume them; the queries'
//                 fragments are loaded in the same order),
//   softmax       per query column, fp32, in log2 units, running maximum;
//   O^T += V^T P^T (A = V^T through the LDS transpose read: the wave stores its
//                 64 value rows as bf16 and reads 4 keys of 16 channels at a
//                 time, B = P straight from the S^T accumulators).
// The sum adds the probabilities before they are rounded to bf16 for the value
// product (a rounding of half a bf16 step each, unbiased: 1.6e-3 of the output in the
// 2-norm, as much as the output's own).  Parts of an item (head, query tile) meet in
// fp32 slots of the workspace, which a second launch joins in order.
//
// Why so: with few query tokens the bytes of the cache bound the work, and a wave
// that waits for nobody keeps its rows in flight: the next step's keys are requested
// as soon as this step's are consumed, its values after this step's are in LDS.  K
// needs no LDS at all.  480P, one query token, all 21 frames kept (101 MB): 28.3 us,
// 25 of them this launch; with the arithmetic taken out the loads alone take 24, 4.6
// TB/s beside the launch (a 1 GiB copy reaches 5.1).  More query tokens share a
// conversion and a row's trip through LDS, 16 to 48 rows a wave: 128 tokens 42.0 us,
// 512 140 us (0.33 PFLOP/s): bound by the latency of a step, two waves per SIMD with
// 200 and more registers each (256 at d = 128 and 32 rows, where five more are spilled
// before the history's loop and come back after it, none within a loop).  Measured beside it, neutral or slower: 4 waves per
// workgroup (512 tokens 180 us), 128 registers and twice the waves for d = 64 (spills),
// the running maximum taken in every step (3 to 8% slower), 12 waves per workgroup for
// d = 64 (168 registers spill: 666 tokens of 16 heads 21 to 55 us; one token 11.1 to 10.8).
#include "fkv_internal.h"

namespace fkv {
namespace {

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr int kThreads = 512, kWaves = 8;
constexpr int kTile = 64;                 // keys per step of a wave
constexpr int kUnit = 16;                 // keys: the grain of the split over waves
constexpr int kJoinThreads = 256, kJoin = 4;  // joining: threads of a workgroup, parts loaded at a time
constexpr float kSlack = 8.f;             // log2 units that the softmax's reference may lag behind
constexpr float kFar = 0x1p24f;           // log2 units from which a reference is kept as a score
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

// MT: query tiles of 16 rows that a wave holds.
template <int D, int MT>
struct Cfg {
    static constexpr int ROWS = 16 * MT;          // query rows of an item
    static constexpr int U = D / 64;              // 64-channel halves of a row
    static constexpr int KS = D / 32;             // steps of the score product
    static constexpr int MB = D / 16;             // 16-channel blocks of the output
    // Value rows in LDS, padded by 32 bytes: the four rows that a transpose read
    // covers, and the eight that a 16-byte store covers, then fall into distinct banks
    // by the layout (the conflict counter still reads 0.3 of the LDS cycles).
    static constexpr int VS = D + 16;
    static constexpr int REGION = kTile * VS;     // elements per wave
    // A wave's results meet the others' in its region, PT tiles at a time: output rows,
    // maxima and sums (floats).
    static constexpr int OS = D + 4, PT = MT < 2 ? MT : 2, PROWS = 16 * PT;
    static_assert(PROWS * OS * 4 + 2 * PROWS * 4 <= REGION * 2, "the results fit the value rows");
};

typedef __attribute__((address_space(3))) bf16x4_t lds_bf16x4_t;

template <int D, int MT>
struct Wave {
    using C = Cfg<D, MT>;
    bf16x8_t q[MT][C::KS];
    f32x4_t o[MT][C::MB];
    // The softmax's reference is the score *shift plus m log2 units (shift in LDS, read
    // once a row of the wave is far); l: this lane's share of the sum.
    float m[MT], l[MT], *shift;
    bool far;

    __device__ __forceinline__ void init(const uint16_t *Q, int q0, int n_q, int lane, float *lds) {
        const int g = lane >> 4, c = lane & 15;
        shift = lds + lane;
        far = false;
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            m[t] = neg_inf();
            l[t] = 0.f;
            shift[64 * t] = 0.f;
            const int row = q0 + 16 * t + c;
#pragma unroll
            for (int mb = 0; mb < C::MB; ++mb) o[t][mb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < C::KS; ++k)
                q[t][k] = frag(row < n_q ? *(const u32x4 *)(Q + (int64_t)row * D + (k >> 1) * 64 + g * 16 + (k & 1) * 8)
                                         : u32x4{0, 0, 0, 0});
        }
    }

    // Tile t's scores s[i] (keys 16i + 4(lane/16) + r of column lane%16) become
    // probabilities; keys from `valid` on do not exist.  The reference moves only
    // where a score passes it by more than kSlack: probabilities then reach 2^kSlack,
    // which costs no digit in fp32 or bf16, and a step without such a score needs
    // neither the other lanes' maxima nor a new scale for the outputs.
    // Far rows: m rounds its score times scale_log2, and the exponent keeps the
    // difference, half a step of m at most; of scores of 1e13 or -1e30 that is more than
    // an exponent holds.  From kFar on the reference is the score itself, subtracted
    // from the others before they are scaled: of nearby scores the difference is exact.
    // (Every score so: 480P, 512 rows 161 us instead of 140.)
    __device__ __forceinline__ void softmax(int t, f32x4_t (&s)[4], float scale_log2, int valid, int g) {
        if (valid < kTile) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) s[i][r] = 16 * i + 4 * g + r < valid ? s[i][r] : neg_inf();
        }
        float top = neg_inf();
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) top = fmaxf(top, s[i][r]);
        float sh = far ? shift[64 * t] : 0.f;
        if (__ballot((top - sh) * scale_log2 > m[t] + kSlack)) {
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float z = top * scale_log2;
            const bool move = (top - sh) * scale_log2 > m[t] + kSlack, to_far = move && !(fabsf(z) < kFar);
            float mn = move ? z : m[t], alpha = mn == m[t] ? 1.f : __builtin_amdgcn_exp2f(m[t] - mn);
            if (far || __ballot(to_far)) {
                const float next = to_far ? top : move ? 0.f : sh;
                mn = to_far ? 0.f : mn;
                const float rise = (next - sh) * scale_log2 + (mn - m[t]);
                alpha = !move ? 1.f : m[t] == neg_inf() ? 0.f : __builtin_amdgcn_exp2f(-rise);
                far = true;
                shift[64 * t] = sh = next;
            }
            m[t] = mn;
            l[t] *= alpha;
#pragma unroll
            for (int mb = 0; mb < C::MB; ++mb) o[t][mb] *= alpha;
        }
        if (far) {
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] -= sh;
        }
        const float base = m[t] == neg_inf() ? 0.f : m[t];
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                s[i][r] = __builtin_amdgcn_exp2f(fmaf(s[i][r], scale_log2, -base));
                sum += s[i][r];
            }
        l[t] += sum;
    }

    // Tile t's reference as a score (a far row's m is 0).
    __device__ __forceinline__ float reference(int t, float scale_log2) const {
        return (far ? shift[64 * t] : 0.f) + m[t] / scale_log2;
    }

    // O^T += V^T P^T with the step's value rows in LDS.
    __device__ __forceinline__ void values(const f32x4_t (&p)[MT][4], uint16_t *v, int lane) {
        const int g = lane >> 4, c = lane & 15;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            bf16x8_t b[MT];
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    b[t][r] = (__bf16)p[t][2 * k][r];
                    b[t][4 + r] = (__bf16)p[t][2 * k + 1][r];
                }
            uint16_t *row = v + (32 * k + 4 * g + (c >> 2)) * C::VS + 4 * (c & 3);
#pragma unroll
            for (int mb = 0; mb < C::MB; ++mb) {
                const bf16x4_t x = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_t *)(row + 16 * mb));
                const bf16x4_t y = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_t *)(row + 16 * C::VS + 16 * mb));
                const bf16x8_t f = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
                for (int t = 0; t < MT; ++t) o[t][mb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, b[t], o[t][mb], 0, 0, 0);
            }
        }
    }
};

// Channels d .. d + 3 of an output row from its sums; empty: the row's head has no key.
template <int D>
__device__ __forceinline__ void put_row(const AttnQ8Args &a, int64_t row, int d, const f32x4_t &acc, float M, float L, bool empty) {
    const float inv = empty ? 0.f : 1.f / L;
    uint32_t b[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) b[k] = __builtin_bit_cast(uint16_t, (__bf16)(acc[k] * inv));
    *(uint2 *)(a.O + row * D + d) = make_uint2(b[0] | (b[1] << 16), b[2] | (b[3] << 16));
    if (a.lse && d == 0) a.lse[row] = empty ? neg_inf() : fmaf(M * kLn2, a.scale_log2, logf(L));
}

// Workgroups go to the 8 XCDs in turn: each XCD takes a contiguous run of the list
// (head, part, query tile), tiles innermost, so the tiles that read the same keys
// mostly share an L2.
template <int D, int MT>
__global__ __launch_bounds__(kThreads) void attn_q8_kernel(AttnQ8Args a) {
    using C = Cfg<D, MT>;
    constexpr int kRows = C::ROWS;
    __shared__ __attribute__((aligned(16))) uint16_t lds[kWaves * C::REGION];
    __shared__ int slots[FKV_MAX_FRAMES];
    __shared__ float shifts[kWaves][MT * 64];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, g = lane >> 4, c = lane & 15;
    const int place = (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);
    const int group = place / a.n_qtiles, qt = place - group * a.n_qtiles;
    const int h = group / a.n_split, part = group - h * a.n_split;
    if (h >= a.n_heads) return;
    const int item = h * a.n_qtiles + qt, q0 = qt * kRows;
    if (tid < a.H) slots[tid] = a.slots.slot[tid];
    __syncthreads();

    // The keys in units of 16: uh of the history, then those of the current tokens,
    // split evenly over the waves of all parts.
    const History x = history_of(a, h);
    const int uh = (x.kvl + kUnit - 1) / kUnit, units = uh + (a.n_cur + kUnit - 1) / kUnit;
    const int n_waves = a.n_split * kWaves, wi = part * kWaves + w;
    const int u0 = (int)((int64_t)units * wi / n_waves), u1 = (int)((int64_t)units * (wi + 1) / n_waves);

    Wave<D, MT> s;
    s.init(a.Q + (int64_t)h * a.n_q * D, q0, a.n_q, lane, shifts[w]);
    uint16_t *vt = lds + w * C::REGION;

    // History: a step's rows are in flight while the step before weights its values.
    const int jend = min(u1 * kUnit, x.kvl);
    if (u0 * kUnit < jend) {
        const uint8_t *K8 = a.K8 + (int64_t)h * a.cap * a.F * D, *V8 = a.V8 + (int64_t)h * a.cap * a.F * D;
        const float *ks = a.k_scale + (int64_t)h * a.cap * a.n_blocks, *vs = a.v_scale + (int64_t)h * a.cap * a.n_blocks;
        u32x4 kr[4][C::U], vr[4][C::U];
        float sk, sv;
        // Rows of 64 keys whose places the lanes hold, one each (past the wave's last key
        // the last one again: its line is there already).
        auto load = [&](const uint8_t *base, const float *scale, int2 at, u32x4 (&r)[4][C::U], float &sc) {
            sc = scale[at.y];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t off = (uint32_t)__shfl(at.x, 16 * i + c) * D + g * 16;
#pragma unroll
                for (int u = 0; u < C::U; ++u) r[i][u] = *(const u32x4 *)(base + off + 64 * u);
            }
        };
        auto row_of = [&](int j) {
            const Place at = place_of(a, x, slots, min(j + lane, jend - 1));
            return make_int2(at.slot * a.F + at.p, at.slot * a.n_blocks + (at.p >> a.block_shift));
        };
        int j0 = u0 * kUnit;
        int2 at = row_of(j0);
        load(K8, ks, at, kr, sk);
        load(V8, vs, at, vr, sv);
        for (; j0 < jend; j0 += kTile) {
            const int next = j0 + kTile, valid = jend - j0;
            // (the next step's places first: a look-up in kept_seg returns with this step's rows)
            at = row_of(next);
            f32x4_t z[MT][4];
            float sc[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) sc[i] = __shfl(sk, 16 * i + c);
#pragma unroll
            for (int k = 0; k < C::KS; ++k) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const u32x4 r = kr[i][k >> 1];
                    const bf16x8_t f = frag(widen8(r[2 * (k & 1)], r[2 * (k & 1) + 1], sc[i]));
#pragma unroll
                    for (int t = 0; t < MT; ++t)
                        z[t][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, s.q[t][k], k ? z[t][i] : f32x4_t{0.f, 0.f, 0.f, 0.f},
                                                                          0, 0, 0);
                }
            }
            if (next < jend) load(K8, ks, at, kr, sk);
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
            if (next < jend) load(V8, vs, at, vr, sv);
#pragma unroll
            for (int t = 0; t < MT; ++t) s.softmax(t, z[t], a.scale_log2, valid, g);
            wave_sync();
            s.values(z, vt, lane);
        }
    }
    // Current tokens, bf16.
    const int cend = min((u1 - uh) * kUnit, a.n_cur);
    for (int j0 = max(u0 - uh, 0) * kUnit; j0 < cend; j0 += kTile) {
        const uint16_t *Kn = a.K_cur + (int64_t)h * a.n_cur * D, *Vn = a.V_cur + (int64_t)h * a.n_cur * D;
        const int valid = cend - j0;
        // all the step's key rows and half of its value rows in flight at once, the other
        // half as the key rows' registers come free
        u32x4 kq[4][C::KS], vq[2][2][2 * C::U];
        uint32_t off[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            off[i] = (uint32_t)(j0 + min(16 * i + c, valid - 1)) * D + g * 16;
#pragma unroll
            for (int k = 0; k < C::KS; ++k) kq[i][k] = *(const u32x4 *)(Kn + off[i] + 64 * (k >> 1) + 8 * (k & 1));
        }
        auto load_values = [&](int half) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int u = 0; u < 2 * C::U; ++u)
                    vq[half][i][u] = *(const u32x4 *)(Vn + off[2 * half + i] + 64 * (u >> 1) + 8 * (u & 1));
        };
        load_values(0);
        f32x4_t z[MT][4];
#pragma unroll
        for (int k = 0; k < C::KS; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int t = 0; t < MT; ++t)
                    z[t][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(frag(kq[i][k]), s.q[t][k],
                                                                      k ? z[t][i] : f32x4_t{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
        load_values(1);
        wave_sync();
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int key = 16 * (2 * half + i) + c;
#pragma unroll
                for (int u = 0; u < 2 * C::U; ++u)
                    *(u32x4 *)(vt + key * C::VS + 64 * (u >> 1) + 16 * g + 8 * (u & 1)) =
                        key < valid ? vq[half][i][u] : u32x4{0, 0, 0, 0};
            }
#pragma unroll
        for (int t = 0; t < MT; ++t) s.softmax(t, z[t], a.scale_log2, valid, g);
        wave_sync();
        s.values(z, vt, lane);
    }

    // The waves' results, PT tiles at a time: into the regions of LDS, then joined by
    // the workgroup's threads, 4 channels of a row each.  References meet as scores, their
    // differences scaled: nothing but the rounding of a score, also for far rows.
    float *mine = (float *)vt;
    constexpr int kPRows = C::PROWS, RF = C::REGION / 2;      // RF: floats per region
#pragma unroll
    for (int t0 = 0; t0 < MT; t0 += C::PT) {
        if (t0 > 0) __syncthreads();                          // (the tiles before are read)
        wave_sync();
#pragma unroll
        for (int k = 0; k < C::PT; ++k) {
            const int t = t0 + k;
            if (t >= MT) break;
            s.l[t] += __shfl_xor(s.l[t], 16);
            s.l[t] += __shfl_xor(s.l[t], 32);
#pragma unroll
            for (int mb = 0; mb < C::MB; ++mb) *(f32x4_t *)(mine + (16 * k + c) * C::OS + 16 * mb + 4 * g) = s.o[t][mb];
            const float ref = s.reference(t, a.scale_log2);
            if (lane < 16) {
                mine[kPRows * C::OS + 16 * k + lane] = ref;
                mine[kPRows * C::OS + kPRows + 16 * k + lane] = s.l[t];
            }
        }
        __syncthreads();
        const int rows = min(min(kPRows, kRows - 16 * t0), a.n_q - q0 - 16 * t0);
        for (int x = tid; x < rows * (D / 4); x += kThreads) {
            const int r = x / (D / 4), d = x % (D / 4) * 4;
            const float *base = (const float *)lds;
            float M = neg_inf(), L = 0.f;
            f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < kWaves; ++i) M = fmaxf(M, base[i * RF + kPRows * C::OS + r]);
            const float ref = M == neg_inf() ? 0.f : M;
#pragma unroll
            for (int i = 0; i < kWaves; ++i) {
                const float wt = __builtin_amdgcn_exp2f((base[i * RF + kPRows * C::OS + r] - ref) * a.scale_log2);
                L += wt * base[i * RF + kPRows * C::OS + kPRows + r];
                acc += wt * *(const f32x4_t *)(base + i * RF + r * C::OS + d);
            }
            if (a.n_split > 1) {                              // joined by join_q8_kernel
                float *slot = a.part + ((size_t)item * a.n_split + part) * (kRows * (D + 2));
                *(f32x4_t *)(slot + (16 * t0 + r) * D + d) = acc;
                if (d == 0) {
                    slot[kRows * D + 16 * t0 + r] = M;
                    slot[kRows * D + kRows + 16 * t0 + r] = L;
                }
            } else {
                put_row<D>(a, (int64_t)h * a.n_q + q0 + 16 * t0 + r, d, acc, M, L, units == 0);
            }
        }
    }
}

// Joins the parts of the items: M = max_j m_j, L = sum_j 2^((m_j - M) scale_log2) l_j and
// likewise the outputs.  A launch of its own: the parts then cross as ordinary cached stores
// and loads, every row has a workgroup, and the workspace holds no counters.  (Joined
// by the part that arrives last, 480P: one query token 29.2 us, 16 tokens 24.0, 32
// tokens 32.7; so 29.7, 21.8 and 26.0.)  One workgroup per row and head: D/4 threads
// take 4 channels each, kLanes of them every kLanes'th part, then the lanes' sums meet
// in LDS, always in the same order.  grid: x = row, y = head.
template <int D>
__global__ __launch_bounds__(kJoinThreads) void join_q8_kernel(AttnQ8Args a) {
    constexpr int kLanes = kJoinThreads / (D / 4);
    __shared__ f32x4_t sum[kLanes][D / 4];
    __shared__ float top[kLanes], total[kLanes];
    const int h = blockIdx.y, row = blockIdx.x, t = threadIdx.x % (D / 4), lane = threadIdx.x / (D / 4);
    const int qt = row / a.q_tile, r = row - qt * a.q_tile;
    const size_t slot = (size_t)a.q_tile * (D + 2);
    const float *p = a.part + ((size_t)h * a.n_qtiles + qt) * a.n_split * slot;
    const float *pm = p + (size_t)a.q_tile * D + r, *pl = pm + a.q_tile, *po = p + (size_t)r * D + 4 * t;
    float M = neg_inf(), L = 0.f;
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
    auto add = [&](float m, float l, const f32x4_t &o) {
        const float Mn = fmaxf(M, m), ref = Mn == neg_inf() ? 0.f : Mn;
        const float so = __builtin_amdgcn_exp2f((M - ref) * a.scale_log2), sn = __builtin_amdgcn_exp2f((m - ref) * a.scale_log2);
        M = Mn;
        L = L * so + l * sn;
        acc = acc * so + o * sn;
    };
    for (int j0 = lane; j0 < a.n_split; j0 += kJoin * kLanes) {
        float mj[kJoin], lj[kJoin];
        f32x4_t o[kJoin];
#pragma unroll
        for (int j = 0; j < kJoin; ++j) {
            const size_t at = (size_t)min(j0 + j * kLanes, a.n_split - 1) * slot;
            mj[j] = pm[at];
            lj[j] = pl[at];
            o[j] = *(const f32x4_t *)(po + at);
        }
        // (all loads before the first use, and no branch that they could sink behind: one
        // memory latency, not one each)
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < kJoin; ++j) {
            const bool ok = j0 + j * kLanes < a.n_split;
            add(ok ? mj[j] : neg_inf(), ok ? lj[j] : 0.f, ok ? o[j] : f32x4_t{0.f, 0.f, 0.f, 0.f});
        }
    }
    sum[lane][t] = acc;
    if (t == 0) {
        top[lane] = M;
        total[lane] = L;
    }
    __syncthreads();
    if (lane > 0) return;
    for (int i = 1; i < kLanes; ++i) add(top[i], total[i], sum[i][t]);
    const History hist = history_of(a, h);
    put_row<D>(a, (int64_t)h * a.n_q + row, 4 * t, acc, M, L, hist.kvl + a.n_cur == 0);
}

// Large chunks: the kept history as a bf16 copy [n_heads][slab][d] for the chunk
// attention's kernel.  A workgroup widens kExpandRows rows of K and V; 16 bytes
// of codes per thread and row.  grid: x = row group, y = head.
constexpr int kExpandThreads = 256, kExpandRows = 64;
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
    const dim3 grid((unsigned)(((int64_t)a.n_heads * a.n_split * a.n_qtiles + 7) / 8 * 8));
    auto launch = [&](auto *kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, s, a); };
    if (head_dim == 64) {
        switch (a.q_tile) {
        case 16: launch(attn_q8_kernel<64, 1>); break;
        case 32: launch(attn_q8_kernel<64, 2>); break;
        default: launch(attn_q8_kernel<64, 3>); break;
        }
    } else if (a.q_tile == 16) {
        launch(attn_q8_kernel<128, 1>);
    } else {
        launch(attn_q8_kernel<128, 2>);
    }
    if (a.n_split > 1) {
        const dim3 join((unsigned)a.n_q, (unsigned)a.n_heads);
        if (head_dim == 64) hipLaunchKernelGGL(join_q8_kernel<64>, join, dim3(kJoinThreads), 0, s, a);
        else hipLaunchKernelGGL(join_q8_kernel<128>, join, dim3(kJoinThreads), 0, s, a);
    }
    return hipGetLastError();
}

}  // namespace fkv
