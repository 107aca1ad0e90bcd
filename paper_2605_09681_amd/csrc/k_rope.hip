// k_rope.hip -- position rotation of queries and keys, and the rolling cache's
// write with the rotation on the way: into a bf16 or fp32 cache, or quantised
// into a cache held in 8 bits with a scale for each head and block of tokens.
//
// Channel pair j of a rotated row, (x, y), becomes (x cos a - y sin a, x sin a +
// y cos a) with a = position * theta^(-i/n).  The host passes theta^(-i/n) /
// (2 pi) in fp64 (turns per position); position * turns is formed in fp64 and
// reduced to [-1/2, 1/2] turns there -- positions reach 2^24, where fp32 would
// keep no digit of the angle -- and only the remainder is rounded to fp32 for
// the sine and cosine.
//
// An item is one token and 8 + 8 channels: [8v, 8v + 8) and the 8 channels d/2
// further on, which are each other's partners under FKV_PAIR_HALVES and two
// runs of four adjacent pairs otherwise: 8 pairs either way, 8 items per row of
// 128.  A thread computes the sines and cosines of its item once and walks the
// heads of its workgroup with them: they depend on the token alone, and they are
// the costly part (fp64 reduction and about 40 instructions per pair).
#include "fkv_internal.h"

namespace fkv {
namespace {

constexpr int kThreads = 256;
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

// turns: the table in LDS (a per-lane index into the launch arguments would copy
// them to scratch).  v: the item within its row of D channels.
template <int D>
__device__ __forceinline__ Turn turn_of(const RopeTable &r, const double *turns, int frame_pos, int p, int v) {
    const int row = p / r.row_tokens, col = p - row * r.row_tokens;
    const int t = frame_pos + (r.token_step ? p : 0);
    const int e0 = r.end_frame, e1 = r.end_row, e2 = r.end_col, halves = r.halves;
    Turn w;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int j = halves ? 8 * v + e : 4 * v + (e & 3) + (e >> 2) * (D / 4);
        const int pos = j < e0 ? t : j < e1 ? row : j < e2 ? col : 0;
        const double a = (double)pos * turns[j];
        const float f = (float)(a - rint(a));
        sincospif(2.f * f, &w.s[e], &w.c[e]);
    }
    return w;
}

__device__ __forceinline__ void turn(const Turn &w, bool halves, float (&x)[8], float (&y)[8]) {
    if (halves) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float a = x[e], b = y[e];
            x[e] = a * w.c[e] - b * w.s[e];
            y[e] = a * w.s[e] + b * w.c[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float a = x[2 * e], b = x[2 * e + 1], c = y[2 * e], d = y[2 * e + 1];
            x[2 * e] = a * w.c[e] - b * w.s[e];
            x[2 * e + 1] = a * w.s[e] + b * w.c[e];
            y[2 * e] = c * w.c[4 + e] - d * w.s[4 + e];
            y[2 * e + 1] = c * w.s[4 + e] + d * w.c[4 + e];
        }
    }
}

__device__ __forceinline__ void load_turns(const RopeTable &r, double *turns) {
    if (threadIdx.x < 64) turns[threadIdx.x] = r.turns[threadIdx.x];
    __syncthreads();
}

// grid: x = token group of a frame, y = new frame, z = group of heads.
template <int D, bool F32>
__global__ __launch_bounds__(kThreads) void rotate_kernel(RotateArgs a) {
    constexpr int ES = F32 ? 4 : 2, IPR = D / 16;         // items per row
    __shared__ double turns[64];
    load_turns(a.rope, turns);
    const int f = blockIdx.y, v = threadIdx.x % IPR;
    const int p = blockIdx.x * (kThreads / IPR) + threadIdx.x / IPR;
    if (p >= a.F) return;
    const bool halves = a.rope.halves;
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
                    turn(w, halves, x, y);
                    r[t][0].set(x);
                    r[t][1].set(y);
                }
                r[t][0].store(d);
                r[t][1].store(d + D / 2 * ES);
            }
    }
}

// Largest finite magnitude of 8 elements and m.
__device__ __forceinline__ float amax8(const float (&x)[8], float m) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float b = fabsf(x[e]);
        m = fmaxf(m, b < __builtin_inff() ? b : 0.f);
    }
    return m;
}

// Exponent k of a block's scale: the smallest with amax <= 448 * 2^k, in [-100, 119]; 0 for an all-zero block.
__device__ __forceinline__ int scale_exponent(float amax) {
    const uint32_t b = __float_as_uint(amax);
    if (b == 0) return 0;
    const int e = (int)(b >> 23) - 127;                       // (a subnormal amax is far below the clamp)
    const int k = (b & 0x7fffffu) <= 0x600000u ? e - 8 : e - 7;  // 448 = 1.75 * 2^8
    return min(max(k, -100), 119);
}

// 8 codes of x * 2^-k.
__device__ __forceinline__ uint2 codes8(const float (&x)[8], float inv) {
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float z = __builtin_amdgcn_fmed3f(x[e] * inv, -kE4M3Max, kE4M3Max);
        y[e] = fabsf(x[e]) < __builtin_inff() ? z : __builtin_nanf("");
    }
    uint2 c;
    c.x = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false), true);
    c.y = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], 0, false), true);
    return c;
}

// One workgroup: one block of tokens of one frame, for heads_per_wg heads; IPT
// items per thread.  grid: x = block of the frame, y = new frame, z = group of heads.
template <int D, bool F32, int IPT>
__global__ __launch_bounds__(kThreads) void append_q8_kernel(AppendQ8Args a) {
    constexpr int ES = F32 ? 4 : 2, IPR = D / 16;
    __shared__ double turns[64];
    __shared__ float red[2][2][kThreads / 64];           // [parity][K, V][wave]
    const bool rope = a.rope.on;
    if (rope) load_turns(a.rope, turns);
    const int f = blockIdx.y, b = blockIdx.x, v = threadIdx.x % IPR;
    const int step = blockDim.x / IPR, p0 = b * a.block_tokens + threadIdx.x / IPR;
    const bool halves = a.rope.halves;
    const int n_waves = blockDim.x >> 6, wave = threadIdx.x >> 6;
    const int slot = a.slots.slot[f];
    Turn w[IPT];
    if (rope) {
#pragma unroll
        for (int i = 0; i < IPT; ++i) w[i] = turn_of<D>(a.rope, turns, a.pos.slot[f], p0 + i * step, v);
    }
    const int h0 = blockIdx.z * a.heads_per_wg, h1 = min(h0 + a.heads_per_wg, a.n_heads);
    for (int h = h0; h < h1; ++h) {
        const uint8_t *K = a.K + h * a.k_head + v * 8 * ES, *V = a.V + h * a.v_head + v * 8 * ES;
        Raw8<F32> kr[IPT][2], vr[IPT][2];
#pragma unroll
        for (int i = 0; i < IPT; ++i) {
            const int p = p0 + i * step;
            kr[i][0] = kr[i][1] = vr[i][0] = vr[i][1] = Raw8<F32>{};
            if (p < a.F) {
                const int64_t tok = (int64_t)f * a.F + p;
                kr[i][0].load(K + tok * a.k_tok);
                kr[i][1].load(K + tok * a.k_tok + D / 2 * ES);
                vr[i][0].load(V + tok * a.v_tok);
                vr[i][1].load(V + tok * a.v_tok + D / 2 * ES);
            }
        }
        float kx[IPT][2][8], mk = 0.f, mv = 0.f;
#pragma unroll
        for (int i = 0; i < IPT; ++i) {
            kr[i][0].get(kx[i][0]);
            kr[i][1].get(kx[i][1]);
            if (rope) turn(w[i], halves, kx[i][0], kx[i][1]);
            mk = amax8(kx[i][1], amax8(kx[i][0], mk));
            float x[8];
            vr[i][0].get(x);
            mv = amax8(x, mv);
            vr[i][1].get(x);
            mv = amax8(x, mv);
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            mk = fmaxf(mk, __shfl_xor(mk, o));
            mv = fmaxf(mv, __shfl_xor(mv, o));
        }
        if (n_waves > 1) {
            float(&r)[2][kThreads / 64] = red[h & 1];    // the other half is read by slower waves of the head before
            if ((threadIdx.x & 63) == 0) {
                r[0][wave] = mk;
                r[1][wave] = mv;
            }
            __syncthreads();
            for (int i = 0; i < n_waves; ++i) {
                mk = fmaxf(mk, r[0][i]);
                mv = fmaxf(mv, r[1][i]);
            }
        }
        const int ek = scale_exponent(mk), ev = scale_exponent(mv);
        const float ik = __uint_as_float((uint32_t)(127 - ek) << 23), iv = __uint_as_float((uint32_t)(127 - ev) << 23);
        const int64_t at = ((int64_t)h * a.cap + slot) * a.n_blocks + b;
        if (threadIdx.x == 0) {
            a.k_scale[at] = __uint_as_float((uint32_t)(127 + ek) << 23);
            a.v_scale[at] = __uint_as_float((uint32_t)(127 + ev) << 23);
        }
#pragma unroll
        for (int i = 0; i < IPT; ++i) {
            const int p = p0 + i * step;
            if (p < a.F) {
                const int64_t row = (((int64_t)h * a.cap + slot) * a.F + p) * D + v * 8;
                *(uint2 *)(a.K8 + row) = codes8(kx[i][0], ik);
                *(uint2 *)(a.K8 + row + D / 2) = codes8(kx[i][1], ik);
                float x[8];
                vr[i][0].get(x);
                *(uint2 *)(a.V8 + row) = codes8(x, iv);
                vr[i][1].get(x);
                *(uint2 *)(a.V8 + row + D / 2) = codes8(x, iv);
            }
        }
    }
}

// Heads that one workgroup walks: the sines and cosines of its tokens serve all
// of them, so as many as leave about four workgroups per compute unit.
int heads_per_workgroup(int64_t token_groups, int n_heads) {
    const int64_t groups = (1024 + token_groups - 1) / token_groups;   // groups of heads wanted
    return groups >= n_heads ? 1 : (int)((n_heads + groups - 1) / groups);
}

template <int D, bool F32>
hipError_t append_q8(AppendQ8Args &a, hipStream_t s) {
    const int items = a.block_tokens * (D / 16), threads = items < kThreads ? items : kThreads;
    a.heads_per_wg = heads_per_workgroup((int64_t)a.n_blocks * a.n_frames, a.n_heads);
    const dim3 grid((unsigned)a.n_blocks, (unsigned)a.n_frames, (unsigned)((a.n_heads + a.heads_per_wg - 1) / a.heads_per_wg));
    switch (items / threads) {
    case 1: hipLaunchKernelGGL((append_q8_kernel<D, F32, 1>), grid, dim3(threads), 0, s, a); break;
    case 2: hipLaunchKernelGGL((append_q8_kernel<D, F32, 2>), grid, dim3(threads), 0, s, a); break;
    default: hipLaunchKernelGGL((append_q8_kernel<D, F32, 4>), grid, dim3(threads), 0, s, a); break;
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rotate(const RotateArgs &a0, int head_dim, bool f32, hipStream_t s) {
    RotateArgs a = a0;
    if (a.n_frames == 0) return hipSuccess;
    const int per = kThreads / (head_dim / 16), groups = (a.F + per - 1) / per;
    a.heads_per_wg = heads_per_workgroup((int64_t)groups * a.n_frames, a.n_heads);
    const dim3 grid((unsigned)groups, (unsigned)a.n_frames, (unsigned)((a.n_heads + a.heads_per_wg - 1) / a.heads_per_wg));
    if (head_dim == 64 && f32) hipLaunchKernelGGL((rotate_kernel<64, true>), grid, dim3(kThreads), 0, s, a);
    else if (head_dim == 64) hipLaunchKernelGGL((rotate_kernel<64, false>), grid, dim3(kThreads), 0, s, a);
    else if (f32) hipLaunchKernelGGL((rotate_kernel<128, true>), grid, dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL((rotate_kernel<128, false>), grid, dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_append_q8(const AppendQ8Args &a0, int head_dim, bool f32, hipStream_t s) {
    AppendQ8Args a = a0;
    if (a.n_frames == 0) return hipSuccess;
    if (head_dim == 64) return f32 ? append_q8<64, true>(a, s) : append_q8<64, false>(a, s);
    return f32 ? append_q8<128, true>(a, s) : append_q8<128, false>(a, s);
}

}  // namespace fkv
