// k_rope.hip -- position rotation of queries and keys, and the rolling cache's
// write with the rotation on the way: into a bf16 or fp32 cache, or quantised
// into a cache held in 8 bits with a scale for each head and block of tokens.
//
// Channel pair j of a rotated row, (x, y), becomes (x cos a - y sin a, x sin a +
// y cos a) with a = position * theta^(-i/n).  Positions reach 2^24, where fp32
// would keep no digit of the angle.  The host passes theta^(-i/n) / (2 pi), turns
// per position, as a 64-bit fixed-point fraction; position * turns modulo one turn
// is then an integer product that wraps by itself, of which the kernel keeps the
// top 32 bits.  Its two top bits give the quadrant, the rest an angle within +-pi/4
// whose sine and cosine are polynomials in fp32 (Chebyshev fits; with every rounding
// from the angle on, off by at most 0.85 and 1.05 times 2^-23).
//
// An item is one token and 8 + 8 channels: [8v, 8v + 8) and the 8 channels d/2
// further on, which are each other's partners under FKV_PAIR_HALVES and two
// runs of four adjacent pairs otherwise: 8 pairs either way, 8 items per row of
// 128.  A thread computes the sines and cosines of its item once and walks the
// heads of its workgroup with them: they depend on the token alone, and they are
// the costly part.
//
// Bound by memory at chunk sizes: rotating a 480P chunk's Q, K and V (86 MB) takes
// 18.9 us and appending a 1080P chunk (301 MB) 65 us, 4.6 TB/s (a 1 GiB copy reaches
// 5.1); loads are streamed past the caches (with ordinary ones 22.0 us).  Appending a
// 480P chunk to 8 bits (43 MB) takes 12.2 us, 1080P 46 us: short of the larger one's 4.9
// TB/s by the launch and the one wait of a block for its maximum.  Magnitudes as
// integers, conversions that scale, and keys and values in workgroups of their own
// brought it there from 17.0.
#include "fkv_internal.h"

namespace fkv {
namespace {

constexpr int kThreads = 256;
constexpr int kAppendThreads = 512;      // largest workgroup of the 8-bit append: a block of 64 x 128
constexpr float kE4M3Max = 448.f;

__device__ __forceinline__ uint32_t pack_bf16(float x, float y) {
    return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x) | ((uint32_t)__builtin_bit_cast(uint16_t, (__bf16)y) << 16);
}
__device__ __forceinline__ float lo_bf16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_bf16(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// 8 adjacent elements as they lie in memory: one 16-byte vector of bf16, two of fp32.
template <bool F32>
struct Raw8 {
    u32x4 v[F32 ? 2 : 1];
    __device__ __forceinline__ void load(const uint8_t *p) {
#pragma unroll
        for (int i = 0; i < (F32 ? 2 : 1); ++i) v[i] = __builtin_nontemporal_load((const u32x4 *)p + i);
    }
    __device__ __forceinline__ void store(uint8_t *p) const {
#pragma unroll
        for (int i = 0; i < (F32 ? 2 : 1); ++i) ((u32x4 *)p)[i] = v[i];
    }
    __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if constexpr (F32) x[e] = __uint_as_float(v[e >> 2][e & 3]);
            else x[e] = (e & 1) ? hi_bf16(v[0][e >> 1]) : lo_bf16(v[0][e >> 1]);
        }
    }
    __device__ __forceinline__ void set(const float (&x)[8]) {
        if constexpr (F32) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e >> 2][e & 3] = __float_as_uint(x[e]);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[0][e] = pack_bf16(x[2 * e], x[2 * e + 1]);
        }
    }
};

// Sines and cosines of an item's 8 pairs: pair e is channels (e, e of the second
// run) under FKV_PAIR_HALVES; otherwise pairs 0..3 are the first run's adjacent
// pairs and 4..7 the second run's.
struct Turn {
    float c[8], s[8];
};

// Sine and cosine of `turns` / 2^32 turns.
__device__ __forceinline__ void sin_cos(int32_t turns, float *sn, float *cs) {
    const int32_t q = (int32_t)((uint32_t)turns + 0x20000000u) >> 30;     // quadrant, -2..1
    const int32_t r = (int32_t)((uint32_t)turns - ((uint32_t)q << 30));   // within 1/8 turn of it
    const float x = (float)r * 0x1.921fb6p-30f;                           // 2 pi / 2^32
    const float y = x * x;
    const float s = fmaf(y * x, fmaf(y, fmaf(y, -0x1.9acap-13f, 0x1.110c2ap-7f), -0x1.555552p-3f), x);
    const float c = fmaf(y * y, fmaf(y, fmaf(y, 0x1.9bd8eep-16f, -0x1.6c12d4p-10f), 0x1.555554p-5f), fmaf(y, -0.5f, 1.f));
    const bool odd = q & 1;
    const float a = odd ? c : s, b = odd ? s : c;
    *sn = q & 2 ? -a : a;                                                 // s, c, -s, -c by quadrant
    *cs = (q + 1) & 2 ? -b : b;                                           // c, -s, -c, s
}

// Pair e of item v within its row of D channels.
template <int D>
__device__ __forceinline__ int pair_of(bool halves, int v, int e) {
    return halves ? 8 * v + e : 4 * v + (e & 3) + (e >> 2) * (D / 4);
}

// turns: the table in LDS (a per-lane index into the launch arguments would copy
// them to scratch).
template <int D>
__device__ __forceinline__ Turn turn_of(const RopeTable &r, const uint2 *turns, int frame_pos, int p, int v) {
    const int row = p / r.row_tokens, col = p - row * r.row_tokens;
    const int t = frame_pos + (r.token_step ? p : 0);
    const int e0 = r.end_frame, e1 = r.end_row, e2 = r.end_col, halves = r.halves;
    Turn w;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int j = pair_of<D>(halves, v, e);
        const int pos = j < e0 ? t : j < e1 ? row : j < e2 ? col : 0;
        // the high word of pos * (hi 2^32 + lo) mod 2^64, pos signed
        const uint2 f = turns[j];
        const uint32_t hi = (uint32_t)pos * f.y + __umulhi((uint32_t)pos, f.x) - (pos < 0 ? f.x : 0u);
        sin_cos((int32_t)hi, &w.s[e], &w.c[e]);
    }
    return w;
}

// The item's pairs turned.  STILL: the axes leave pairs over, which are left as they
// are (x * 1 - y * 0 would not be x beside an infinity or a NaN).  A kernel of its own:
// choosing pair by pair takes the 8-bit append of 480P from 12.5 to 14.0 us.
template <int D, bool STILL>
__device__ __forceinline__ void turn(const Turn &w, const RopeTable &r, int v, float (&x)[8], float (&y)[8]) {
    const bool halves = r.halves;
    auto put = [&](int e, float &to, float turned) {
        if (!STILL || pair_of<D>(halves, v, e) < r.end_col) to = turned;
    };
    if (halves) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float a = x[e], b = y[e];
            put(e, x[e], a * w.c[e] - b * w.s[e]);
            put(e, y[e], a * w.s[e] + b * w.c[e]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float a = x[2 * e], b = x[2 * e + 1], c = y[2 * e], d = y[2 * e + 1];
            put(e, x[2 * e], a * w.c[e] - b * w.s[e]);
            put(e, x[2 * e + 1], a * w.s[e] + b * w.c[e]);
            put(4 + e, y[2 * e], c * w.c[4 + e] - d * w.s[4 + e]);
            put(4 + e, y[2 * e + 1], c * w.s[4 + e] + d * w.c[4 + e]);
        }
    }
}

__device__ __forceinline__ void load_turns(const RopeTable &r, uint2 *turns) {
    if (threadIdx.x < 64) turns[threadIdx.x] = make_uint2(r.turns[threadIdx.x].lo, r.turns[threadIdx.x].hi);
    __syncthreads();
}

// grid: x = token group of a frame, y = new frame, z = group of heads.
template <int D, bool F32, bool STILL>
__global__ __launch_bounds__(kThreads) void rotate_kernel(RotateArgs a) {
    constexpr int ES = F32 ? 4 : 2, IPR = D / 16;         // items per row
    __shared__ uint2 turns[64];
    load_turns(a.rope, turns);
    const int f = blockIdx.y, v = threadIdx.x % IPR;
    const int p = blockIdx.x * (kThreads / IPR) + threadIdx.x / IPR;
    if (p >= a.F) return;
    const Turn w = turn_of<D>(a.rope, turns, a.pos.slot[f], p, v);
    const int h0 = blockIdx.z * a.heads_per_wg, h1 = min(h0 + a.heads_per_wg, a.n_heads);
    const int64_t tok = (int64_t)f * a.F + p;
    const int64_t out = ((int64_t)a.slots.slot[f] * a.F + p) * (D * ES) + v * 8 * ES;
    for (int h = h0; h < h1; ++h) {
        Raw8<F32> r[3][2];
#pragma unroll
        for (int t = 0; t < 3; ++t)
            if (a.src[t]) {
                const uint8_t *s = a.src[t] + h * a.src_head[t] + tok * a.src_tok[t] + v * 8 * ES;
                r[t][0].load(s);
                r[t][1].load(s + D / 2 * ES);
            }
#pragma unroll
        for (int t = 0; t < 3; ++t)
            if (a.src[t]) {
                uint8_t *d = a.dst[t] + h * a.dst_head + out;
                if (t < 2) {
                    float x[8], y[8];
                    r[t][0].get(x);
                    r[t][1].get(y);
                    turn<D, STILL>(w, a.rope, v, x, y);
                    r[t][0].set(x);
                    r[t][1].set(y);
                }
                r[t][0].store(d);
                r[t][1].store(d + D / 2 * ES);
            }
    }
}

typedef short i16x2_t __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

// Magnitudes are compared as integers: the bits of |x| grow with |x|, infinities
// and NaN above all numbers.  Beyond kPlainBits -- 448 * 2^119, the largest that
// the scales reach -- a block takes the careful way: its scale from the finite
// elements alone, its codes clamped, NaN for what is not finite.
constexpr uint32_t kPlainBits = 0x7f600000u;

__device__ __forceinline__ uint32_t max_bits8(const float (&x)[8], uint32_t m) {
#pragma unroll
    for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(x[e]) & 0x7fffffffu);
    return m;
}
// The same of 8 elements as they lie in memory (bf16: two at a time).
template <bool F32>
__device__ __forceinline__ uint32_t max_bits8(const Raw8<F32> &r, uint32_t m) {
    if constexpr (F32) {
#pragma unroll
        for (int e = 0; e < 8; ++e) m = max(m, r.v[e >> 2][e & 3] & 0x7fffffffu);
    } else {
        u16x2_t t = __builtin_bit_cast(u16x2_t, (uint32_t)(r.v[0][0] & 0x7fff7fffu));
#pragma unroll
        for (int e = 1; e < 4; ++e)
            t = __builtin_elementwise_max(t, __builtin_bit_cast(u16x2_t, (uint32_t)(r.v[0][e] & 0x7fff7fffu)));
        m = max(m, (uint32_t)max(t[0], t[1]) << 16);
    }
    return m;
}

// Largest finite magnitude of 8 elements and m.
__device__ __forceinline__ float finite_max8(const float (&x)[8], float m) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float b = fabsf(x[e]);
        m = fmaxf(m, b < __builtin_inff() ? b : 0.f);
    }
    return m;
}

// Exponent k of the scale of a block with largest magnitude `bits`: the smallest
// with amax <= 448 * 2^k, in [-100, 119]; 0 for an all-zero block.
__device__ __forceinline__ int scale_exponent(uint32_t bits) {
    if (bits == 0) return 0;
    const int e = (int)(bits >> 23) - 127;                       // (a subnormal amax is far below the clamp)
    const int k = (bits & 0x7fffffu) <= 0x600000u ? e - 8 : e - 7;  // 448 = 1.75 * 2^8
    return min(max(k, -100), 119);
}

// 8 codes of x / scale (v_cvt_scalef32_pk_fp8: one rounding, to nearest even).
__device__ __forceinline__ uint2 codes8(const float (&x)[8], float scale) {
    uint2 c;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        i16x2_t w = {0, 0};
        w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, x[4 * i], x[4 * i + 1], scale, false);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, x[4 * i + 2], x[4 * i + 3], scale, true);
        (i ? c.y : c.x) = __builtin_bit_cast(uint32_t, w);
    }
    return c;
}
template <bool F32>
__device__ __forceinline__ uint2 codes8(const Raw8<F32> &r, float scale) {
    if constexpr (F32) {
        float x[8];
        r.get(x);
        return codes8(x, scale);
    } else {
        uint2 c;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            i16x2_t w = {0, 0};
            w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2_t, (uint32_t)r.v[0][2 * i]), scale, false);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2_t, (uint32_t)r.v[0][2 * i + 1]), scale, true);
            (i ? c.y : c.x) = __builtin_bit_cast(uint32_t, w);
        }
        return c;
    }
}
// The careful way: at most 448 in magnitude, NaN for what is not finite.
__device__ __forceinline__ uint2 careful_codes8(const float (&x)[8], float scale) {
    const float most = kE4M3Max * scale;
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
        y[e] = fabsf(x[e]) < __builtin_inff() ? __builtin_amdgcn_fmed3f(x[e], -most, most) : __builtin_nanf("");
    return codes8(y, scale);
}

// Largest m of the workgroup; r: its waves' words of LDS, used again two calls later.
__device__ __forceinline__ uint32_t block_max(uint32_t m, uint32_t *r) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o));
    const int n = blockDim.x >> 6;
    if (n > 1) {
        if ((threadIdx.x & 63) == 0) r[threadIdx.x >> 6] = m;
        __syncthreads();
        for (int i = 0; i < n; ++i) m = max(m, r[i]);
    }
    return m;
}

// One workgroup: one block of tokens of one frame, its keys or its values
// (ROTATE: keys that turn; otherwise rows as they are), for heads_per_wg heads;
// IPT items per thread.
template <int D, bool F32, int IPT, bool ROTATE, bool STILL>
__device__ __forceinline__ void append_block(const AppendQ8Args &a, bool values, int h0, int h1, const uint2 *turns,
                                             uint32_t (*red)[2][kAppendThreads / 64]) {
    constexpr int ES = F32 ? 4 : 2, IPR = D / 16;
    const int f = blockIdx.y, b = blockIdx.x, v = threadIdx.x % IPR;
    const int step = blockDim.x / IPR, p0 = b * a.block_tokens + threadIdx.x / IPR;
    const int slot = a.slots.slot[f];
    const uint8_t *src = values ? a.V : a.K;
    const int64_t src_head = values ? a.v_head : a.k_head, src_tok = values ? a.v_tok : a.k_tok;
    uint8_t *dst = values ? a.V8 : a.K8;
    float *scales = values ? a.v_scale : a.k_scale;
    Turn w[IPT];
    for (int h = h0; h < h1; ++h) {
        const uint8_t *X = src + h * src_head + v * 8 * ES;
        Raw8<F32> r[IPT][2];
#pragma unroll
        for (int i = 0; i < IPT; ++i) {
            const int p = p0 + i * step;
            r[i][0] = r[i][1] = Raw8<F32>{};
            if (p < a.F) {
                const int64_t tok = (int64_t)f * a.F + p;
                r[i][0].load(X + tok * src_tok);
                r[i][1].load(X + tok * src_tok + D / 2 * ES);
            }
        }
        if (ROTATE && h == h0) {                         // (while the first rows are on their way)
#pragma unroll
            for (int i = 0; i < IPT; ++i) w[i] = turn_of<D>(a.rope, turns, a.pos.slot[f], p0 + i * step, v);
        }
        float x[IPT][2][8];
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < IPT; ++i) {
            if constexpr (ROTATE) {
                r[i][0].get(x[i][0]);
                r[i][1].get(x[i][1]);
                turn<D, STILL>(w[i], a.rope, v, x[i][0], x[i][1]);
                m = max_bits8(x[i][1], max_bits8(x[i][0], m));
            } else {
                m = max_bits8(r[i][1], max_bits8(r[i][0], m));
            }
        }
        m = block_max(m, red[0][h & 1]);
        const bool careful = m > kPlainBits;             // (the same in every thread)
        if (careful) {
            float top = 0.f;
#pragma unroll
            for (int i = 0; i < IPT; ++i)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    if constexpr (!ROTATE) r[i][k].get(x[i][k]);
                    top = finite_max8(x[i][k], top);
                }
            m = block_max(__float_as_uint(top), red[1][h & 1]);
        }
        const float scale = __uint_as_float((uint32_t)(127 + scale_exponent(m)) << 23);
        if (threadIdx.x == 0) scales[((int64_t)h * a.cap + slot) * a.n_blocks + b] = scale;
#pragma unroll
        for (int i = 0; i < IPT; ++i) {
            const int p = p0 + i * step;
            if (p < a.F) {
                uint8_t *row = dst + (((int64_t)h * a.cap + slot) * a.F + p) * D + v * 8;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    uint2 c;
                    if (careful) c = careful_codes8(x[i][k], scale);
                    else if constexpr (ROTATE) c = codes8(x[i][k], scale);
                    else c = codes8(r[i][k], scale);
                    *(uint2 *)(row + k * (D / 2)) = c;
                }
            }
        }
    }
}

// Keys and values in workgroups of their own: half the registers, twice the
// workgroups to hide the loads, the barrier and the stores of one behind the
// others.  grid: x = block of the frame, y = new frame, z = 2 * (group of heads) +
// (1: values).
template <int D, bool F32, int IPT, bool STILL>
__global__ __launch_bounds__(kAppendThreads) void append_q8_kernel(AppendQ8Args a) {
    __shared__ uint2 turns[64];
    __shared__ uint32_t red[2][2][kAppendThreads / 64];  // [plain, careful][parity of the head][wave]
    const bool values = blockIdx.z & 1;
    const int h0 = (blockIdx.z >> 1) * a.heads_per_wg, h1 = min(h0 + a.heads_per_wg, a.n_heads);
    if (a.rope.on && !values) {
        load_turns(a.rope, turns);
        append_block<D, F32, IPT, true, STILL>(a, values, h0, h1, turns, red);
    } else {
        append_block<D, F32, IPT, false, false>(a, values, h0, h1, turns, red);
    }
}

// Heads that one workgroup walks: the sines and cosines of its tokens serve all
// of them, so as many as leave the device `wanted` workgroups.  Rotating, 480P:
// 1024 18.9 us, 512 19.4, 256 23.3.  Appending to 8 bits (and as many for the values),
// 480P: 768 12.2 us, 256 12.4, one head each 13.5; blocks of 16 tokens 12.4, 20.5, 11.8.
constexpr int kRotateGroups = 1024, kAppendGroups = 768;
int heads_per_workgroup(int64_t token_groups, int n_heads, int wanted) {
    const int64_t groups = (wanted + token_groups - 1) / token_groups;   // groups of heads wanted
    return groups >= n_heads ? 1 : (int)((n_heads + groups - 1) / groups);
}

template <int D, bool F32, bool STILL>
hipError_t append_q8(AppendQ8Args &a, hipStream_t s) {
    const int items = a.block_tokens * (D / 16), threads = items < kAppendThreads ? items : kAppendThreads;
    a.heads_per_wg = heads_per_workgroup((int64_t)a.n_blocks * a.n_frames, a.n_heads, kAppendGroups);
    const dim3 grid((unsigned)a.n_blocks, (unsigned)a.n_frames, 2 * (unsigned)((a.n_heads + a.heads_per_wg - 1) / a.heads_per_wg));
    if (items == threads) hipLaunchKernelGGL((append_q8_kernel<D, F32, 1, STILL>), grid, dim3(threads), 0, s, a);
    else hipLaunchKernelGGL((append_q8_kernel<D, F32, 2, STILL>), grid, dim3(threads), 0, s, a);
    return hipGetLastError();
}

template <int D, bool F32, bool STILL>
hipError_t rotate(RotateArgs &a, hipStream_t s) {
    const int per = kThreads / (D / 16), groups = (a.F + per - 1) / per;
    a.heads_per_wg = heads_per_workgroup((int64_t)groups * a.n_frames, a.n_heads, kRotateGroups);
    const dim3 grid((unsigned)groups, (unsigned)a.n_frames, (unsigned)((a.n_heads + a.heads_per_wg - 1) / a.heads_per_wg));
    hipLaunchKernelGGL((rotate_kernel<D, F32, STILL>), grid, dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

bool leaves_pairs(const RopeTable &r, int head_dim) { return r.on && r.end_col < head_dim / 2; }

}  // namespace

hipError_t launch_rotate(const RotateArgs &a0, int head_dim, bool f32, hipStream_t s) {
    RotateArgs a = a0;
    if (a.n_frames == 0) return hipSuccess;
    if (leaves_pairs(a.rope, head_dim)) {
        if (head_dim == 64) return f32 ? rotate<64, true, true>(a, s) : rotate<64, false, true>(a, s);
        return f32 ? rotate<128, true, true>(a, s) : rotate<128, false, true>(a, s);
    }
    if (head_dim == 64) return f32 ? rotate<64, true, false>(a, s) : rotate<64, false, false>(a, s);
    return f32 ? rotate<128, true, false>(a, s) : rotate<128, false, false>(a, s);
}

hipError_t launch_append_q8(const AppendQ8Args &a0, int head_dim, bool f32, hipStream_t s) {
    AppendQ8Args a = a0;
    if (a.n_frames == 0) return hipSuccess;
    if (leaves_pairs(a.rope, head_dim)) {
        if (head_dim == 64) return f32 ? append_q8<64, true, true>(a, s) : append_q8<64, false, true>(a, s);
        return f32 ? append_q8<128, true, true>(a, s) : append_q8<128, false, true>(a, s);
    }
    if (head_dim == 64) return f32 ? append_q8<64, true, false>(a, s) : append_q8<64, false, false>(a, s);
    return f32 ? append_q8<128, true, false>(a, s) : append_q8<128, false, false>(a, s);
}

}  // namespace fkv
