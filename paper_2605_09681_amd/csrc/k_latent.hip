// k_latent.hip -- the matrix products around attention over latent rows, gfx950 MFMA.
//
// Absorbed form: q'_h = W_k,h^T q_h before the attention, rounded to bf16 for the matrix units as the
// queries themselves are, and o_h = W_v,h o'_h after it, o' in fp32 as the sum of two bf16.
// Expanded form: k_h = W_k,h c and v_h = W_v,h c of every cached token, rounded to bf16
// as a cache of its own keys and values would hold them.  With the probabilities and the output that
// makes four roundings to bf16 of 1.4e-3 to 1.7e-3 each, 3.1e-3 together at the most (measured 1.9e-3 to
// 3.0e-3, relative 2-norm against 64 bits), where the absorbed form has 2.3e-3.  Keys, values or
// probabilities as the sum of two bf16 would take 1.4 to 1.6 times the products each and save one of the
// four; fp16 has the digits but not the range of the latent rows.
#include <algorithm>

#include "paged.h"

namespace fkv {
namespace {

using namespace paged;

typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) bf16x4_t lds_bf16x4_t;

constexpr int NT = 256;

__device__ __forceinline__ bf16x8_t frag(const u32x4 &v) { return __builtin_bit_cast(bf16x8_t, v); }

__device__ __forceinline__ uint2 pack4(float x0, float x1, float x2, float x3) {
    const uint32_t b0 = __builtin_bit_cast(uint16_t, (__bf16)x0), b1 = __builtin_bit_cast(uint16_t, (__bf16)x1);
    const uint32_t b2 = __builtin_bit_cast(uint16_t, (__bf16)x2), b3 = __builtin_bit_cast(uint16_t, (__bf16)x3);
    return make_uint2(b0 | (b1 << 16), b2 | (b3 << 16));
}

// q'[t][h][r] = sum_c W_k[h][c][r] q[t][h][c]: 64 latent channels of a head and 16 TM tokens a
// workgroup, 16 channels a wave; the weights' 64 columns lie in LDS and are read transposed.  The last
// column block copies the queries' rotated channels.  grid: x = token tile, y = head, z = column block.
template <int D, int TM>
__global__ __launch_bounds__(NT) void latent_absorb_kernel(LatentArgs a) {
    __shared__ __attribute__((aligned(16))) uint16_t wt[D * 64];
    const PagedArgs &p = a.p;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, g = lane >> 4, c = lane & 15;
    const int x = blockIdx.z, h = blockIdx.y, t0 = blockIdx.x * (16 * TM), width = a.R + kLatentRot;
    const uint16_t *Q = p.Q + (int64_t)h * p.q_head;
    uint16_t *out = a.q_abs + (int64_t)h * width + 64 * x;
    if (x == 0 && h == 0 && w == 0) {
        Seq s;
        const bool mine = owner_of(p, lane < 16 * TM && t0 + lane < p.n_tokens ? t0 + lane : -1, t0, t0 + 16 * TM, &s) >= 0;
        if (lane < 16 * TM && t0 + lane < p.n_tokens) a.owned[t0 + lane] = mine;
    }
    if (64 * x == a.R) {
        for (int id = tid; id < 16 * TM * 8; id += NT) {
            const int t = t0 + id / 8;
            if (t < p.n_tokens)
                *(u32x4 *)(out + (int64_t)t * p.n_heads * width + id % 8 * 8) = *(const u32x4 *)(Q + (int64_t)t * p.q_tok + D + id % 8 * 8);
        }
        return;
    }
    const uint16_t *W = a.W_k + (int64_t)h * D * a.R + 64 * x;
#pragma unroll
    for (int i = 0; i < D * 8 / NT; ++i) {
        const int id = tid + i * NT, k = id / 8;
        *(u32x4 *)(wt + k * 64 + place<8, false>(k, id % 8) * 8) = *(const u32x4 *)(W + (int64_t)k * a.R + id % 8 * 8);
    }
    uint2 q[TM][D / 16];
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const uint16_t *row = Q + (int64_t)min(t0 + 16 * i + c, p.n_tokens - 1) * p.q_tok + 4 * g;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) q[i][k] = *(const uint2 *)(row + 16 * k);
    }
    __syncthreads();
    f32x4_t acc[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) acc[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    const int ch = 2 * w + ((c & 3) >> 1);
#pragma unroll
    for (int k = 0; k < D / 32; ++k) {
        const int ka = 32 * k + 4 * g + (c >> 2), kc = ka + 16;
        const bf16x4_t u = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_t *)(wt + ka * 64 + place<8, false>(ka, ch) * 8 + 4 * (c & 1)));
        const bf16x4_t v = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4_t *)(wt + kc * 64 + place<8, false>(kc, ch) * 8 + 4 * (c & 1)));
        const bf16x8_t f = __builtin_shufflevector(u, v, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const u32x4 b = {q[i][2 * k].x, q[i][2 * k].y, q[i][2 * k + 1].x, q[i][2 * k + 1].y};
            acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, frag(b), acc[i], 0, 0, 0);
        }
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int t = t0 + 16 * i + c;
        if (t < p.n_tokens)
            *(uint2 *)(out + (int64_t)t * p.n_heads * width + 16 * w + 4 * g) = pack4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
    }
}

// fp32 values as the sum of two bf16.
__device__ __forceinline__ void two_bf16(const f32x4_t &v0, const f32x4_t &v1, bf16x8_t *hi, bf16x8_t *lo) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float v = e < 4 ? v0[e] : v1[e - 4];
        (*hi)[e] = (__bf16)v;
        (*lo)[e] = (__bf16)(v - (float)(*hi)[e]);
    }
}

// o[t][h][c] = sum_r W_v[h][c][r] o'[t][h][r], for the tokens that a sequence of the launch holds:
// 16 channels a wave and 16 TM tokens, both operands straight from memory.  grid: x = token tile, y = head, z = 64 channels.
template <int R, int TM>
__global__ __launch_bounds__(NT) void latent_unabsorb_kernel(LatentArgs a, int D) {
    const PagedArgs &p = a.p;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, g = lane >> 4, c = lane & 15;
    const int h = blockIdx.y, t0 = blockIdx.x * (16 * TM), c0 = 64 * blockIdx.z + 16 * w;
    const uint16_t *W = a.W_v + ((int64_t)h * D + c0 + c) * R + 8 * g;
    const float *row[TM];
    f32x4_t acc[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        row[i] = a.o_abs + ((int64_t)min(t0 + 16 * i + c, p.n_tokens - 1) * p.n_heads + h) * R + 8 * g;
        acc[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll 2
    for (int k = 0; k < R / 32; ++k) {
        const bf16x8_t f = frag(*(const u32x4 *)(W + 32 * k));
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            bf16x8_t hi, lo;
            two_bf16(*(const f32x4_t *)(row[i] + 32 * k), *(const f32x4_t *)(row[i] + 32 * k + 4), &hi, &lo);
            acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, hi, acc[i], 0, 0, 0);
            acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, lo, acc[i], 0, 0, 0);
        }
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int t = t0 + 16 * i + c;
        if (t < p.n_tokens && a.owned[t])
            *(uint2 *)(p.O + (int64_t)t * p.o_tok + (int64_t)h * p.o_head + c0 + 4 * g) = pack4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
    }
}

// The same for few tokens, bound by the latency of its loads and by how many CUs read the weights: 16 channels and 16
// tokens a workgroup, the latent channels dealt to its 4 waves, whose every load is on its way before the first product;
// their sums meet in LDS in order.  16 tokens of 40 heads, 512 latent channels (10.5 MB of weights) 5.0 us; a wave to all latent
// channels, 64 channels a workgroup, 7.4.  grid: x = token tile, y = head, z = 16 channels.
template <int R>
__global__ __launch_bounds__(NT) void latent_unabsorb_few_kernel(LatentArgs a, int D) {
    constexpr int S = R / 128;
    __shared__ f32x4_t sums[3][64];
    const PagedArgs &p = a.p;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, g = lane >> 4, c = lane & 15;
    const int h = blockIdx.y, t = blockIdx.x * 16 + c, c0 = 16 * blockIdx.z, r0 = w * (R / 4) + 8 * g;
    const uint16_t *W = a.W_v + ((int64_t)h * D + c0 + c) * R + r0;
    const float *row = a.o_abs + ((int64_t)min(t, p.n_tokens - 1) * p.n_heads + h) * R + r0;
    u32x4 f[S];
    f32x4_t v[S][2];
#pragma unroll
    for (int k = 0; k < S; ++k) {
        f[k] = *(const u32x4 *)(W + 32 * k);
        v[k][0] = *(const f32x4_t *)(row + 32 * k);
        v[k][1] = *(const f32x4_t *)(row + 32 * k + 4);
    }
    const bool owned = w == 0 && t < p.n_tokens && a.owned[t];
    __builtin_amdgcn_sched_barrier(0);
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < S; ++k) {
        bf16x8_t hi, lo;
        two_bf16(v[k][0], v[k][1], &hi, &lo);
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(frag(f[k]), hi, acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(frag(f[k]), lo, acc, 0, 0, 0);
    }
    if (w > 0) sums[w - 1][lane] = acc;
    __syncthreads();
    if (!owned) return;
#pragma unroll
    for (int i = 0; i < 3; ++i) acc += sums[i][lane];
    *(uint2 *)(p.O + (int64_t)t * p.o_tok + (int64_t)h * p.o_head + c0 + 4 * g) = pack4(acc[0], acc[1], acc[2], acc[3]);
}

// Keys and values of 256 cached tokens of a sequence, blocks of 256 of the heads' 2 D channels in turn: 8
// waves of 64 channels and 128 tokens, latent channels 64 at a time through two LDS buffers; the next block's
// first operands are on their way while a block's results are stored.  The first workgroup of a token block copies its
// rotated keys to every head.  Bound by latency between its few steps and by its 120 MB of results: 15600 tokens, 12 heads of
// 128, 512 latent channels (49 GFLOP) 75 to 95 us; with blocks of 128 x 128 95 to 120, stored 8 bytes a token and lane 90 to
// 114.  Two registers (14 at D 64) do not fit and are stored outside the products.  grid: x = every gridDim.x'th channel
// block, y = token block.
template <int D, int R>
__global__ __launch_bounds__(512, 2) void latent_expand_kernel(LatentArgs a) {
    constexpr int NT = 512, STEP = 64, N = 256 * STEP / 8 / NT;      // chunks per thread and operand
    constexpr int HEADS = 128 / D;                         // heads per channel block
    __shared__ __attribute__((aligned(16))) uint16_t lat[2][256 * STEP], wts[2][256 * STEP];
    const PagedArgs &p = a.p;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, hh = lane >> 5, c = lane & 31;
    Seq s;
    int i = 0;
    const int j0 = locate_block(p, blockIdx.y, &s, &i);
    if (j0 < 0) return;
    const int64_t base = (int64_t)blockIdx.y * kSeqRows;
    const int n = (int)min((int64_t)min(s.len - j0, kSeqRows), p.head_rows - base);
    if (n <= 0) return;
    // no new token sees these keys
    if (p.recent[0] >= 0 && j0 >= p.sink[0] && j0 + n <= s.first - p.recent[0]) return;
    const int32_t *pages = p.table + (int64_t)i * p.max_pages;
    const int width = R + kLatentRot;
    constexpr int W = D + kLatentRot;
    const int cols = (p.n_heads + HEADS - 1) / HEADS;
    // Where this thread's N chunks of a token row come from: tokens tid / 8 + 64 u.
    const uint16_t *from_l[N];
#pragma unroll
    for (int u = 0; u < N; ++u)
        from_l[u] = p.K + (int64_t)pool_row(p, pages, 0, min(j0 + tid / 8 + 64 * u, j0 + n - 1)) * width + tid % 8 * 8;
    if (blockIdx.x == 0) {
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const int k = tid / 8 + 64 * u;
            const u32x4 v = *(const u32x4 *)(from_l[u] + R);
            if (k >= n) continue;
            for (int h = 0; h < p.n_heads; ++h) *(u32x4 *)(a.K_exp + (h * p.head_rows + base + k) * W + D + tid % 8 * 8) = v;
        }
    }
    // Channel rows of a block, 64 at a time: of head h its keys', then its values', (D = 64) then the next head's.
    auto channels = [&](int x, int u) {                    // u: which 64
        const int h = min(x * HEADS + (D == 64 ? u >> 1 : 0), p.n_heads - 1);
        const bool value = D == 64 ? u & 1 : u >> 1;
        return (value ? a.W_v : a.W_k) + ((int64_t)h * D + (D == 64 ? 0 : 64 * (u & 1))) * R;
    };
    u32x4 lr[N], wr[N];
    auto load = [&](int x, int k) {
#pragma unroll
        for (int u = 0; u < N; ++u) {
            lr[u] = *(const u32x4 *)(from_l[u] + k * STEP);
            wr[u] = *(const u32x4 *)(channels(x, u) + (uint32_t)((tid / 8) * R + tid % 8 * 8) + k * STEP);
        }
    };
    auto store = [&](int buf) {
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const int k = tid / 8 + 64 * u, at = k * STEP + place<8, true>(k, tid % 8) * 8;
            *(u32x4 *)(lat[buf] + at) = lr[u];
            *(u32x4 *)(wts[buf] + at) = wr[u];
        }
    };
    const int wc = w & 3, wk = w >> 2;                     // this wave's 64 channels and 128 tokens
    load(blockIdx.x, 0);
#pragma unroll 1
    for (int x = blockIdx.x; x < cols; x += gridDim.x) {
        f32x16_t acc[2][4];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int v = 0; v < 4; ++v)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[u][v][r] = 0.f;
        store(0);
        load(x, 1);
#pragma unroll 1
        for (int k = 0; k < R / STEP; ++k) {
            __syncthreads();
            const int buf = k & 1;
            if (k + 1 < R / STEP) store(buf ^ 1);
            if (k + 2 < R / STEP) load(x, k + 2);
#pragma unroll
            for (int u = 0; u < STEP / 16; ++u) {
                bf16x8_t fa[2], fb[4];
#pragma unroll
                for (int v = 0; v < 2; ++v)
                    fa[v] = frag(*(const u32x4 *)(wts[buf] + (64 * wc + 32 * v + c) * STEP + place<8, true>(c, 2 * u + hh) * 8));
#pragma unroll
                for (int v = 0; v < 4; ++v)
                    fb[v] = frag(*(const u32x4 *)(lat[buf] + (128 * wk + 32 * v + c) * STEP + place<8, true>(c, 2 * u + hh) * 8));
#pragma unroll
                for (int v = 0; v < 4; ++v)
#pragma unroll
                    for (int y = 0; y < 2; ++y) acc[y][v] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[y], fb[v], acc[y][v], 0, 0, 0);
            }
        }
        static_assert(R / STEP % 2 == 0, "the last step reads buffer 1, the next block's first goes to buffer 0");
        if (x + (int)gridDim.x < cols) load(x + gridDim.x, 0);
        const int h = x * HEADS + (D == 64 ? wc >> 1 : 0);
        const bool value = D == 64 ? wc & 1 : wc >> 1;
        uint16_t *out = value ? a.V_exp : a.K_exp;
        const int stride = value ? D : W, c0 = D == 64 ? 0 : 64 * (wc & 1);
        // Through LDS (buffer 0, which every wave has read; 64 tokens at a time, 8 KB a wave), so that 8 lanes store a
        // token's 64 channels together.
        uint16_t *mine = (w < 4 ? lat[0] : wts[0]) + (w & 3) * 4096;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");      // (a wave's LDS operations finish in order)
#pragma unroll
            for (int v = 0; v < 2; ++v)
#pragma unroll
                for (int y = 0; y < 2; ++y)
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        *(uint2 *)(mine + (32 * v + c) * 64 + ((4 * y + u) ^ (c & 7)) * 8 + 4 * hh) =
                            pack4(acc[y][2 * half + v][4 * u], acc[y][2 * half + v][4 * u + 1], acc[y][2 * half + v][4 * u + 2],
                                  acc[y][2 * half + v][4 * u + 3]);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int row = 8 * u + (lane >> 3), k = 128 * wk + 64 * half + row;
                const u32x4 v = *(const u32x4 *)(mine + row * 64 + ((lane & 7) ^ (row & 7)) * 8);
                if (k < n && h < p.n_heads) *(u32x4 *)(out + (h * p.head_rows + base + k) * stride + c0 + (lane & 7) * 8) = v;
            }
        }
        __syncthreads();                                   // (the next block's first operands go there)
    }
}

}  // namespace

hipError_t launch_latent_absorb(const LatentArgs &a, int head_dim, hipStream_t s) {
    const bool few = a.p.n_tokens <= 32;
    const int tile = few ? 16 : 64;
    const dim3 grid((a.p.n_tokens + tile - 1) / tile, a.p.n_heads, a.R / 64 + 1);
    if (head_dim == 64) {
        if (few) hipLaunchKernelGGL((latent_absorb_kernel<64, 1>), grid, dim3(NT), 0, s, a);
        else hipLaunchKernelGGL((latent_absorb_kernel<64, 4>), grid, dim3(NT), 0, s, a);
    } else {
        if (few) hipLaunchKernelGGL((latent_absorb_kernel<128, 1>), grid, dim3(NT), 0, s, a);
        else hipLaunchKernelGGL((latent_absorb_kernel<128, 4>), grid, dim3(NT), 0, s, a);
    }
    return hipGetLastError();
}

hipError_t launch_latent_unabsorb(const LatentArgs &a, int head_dim, hipStream_t s) {
    if (a.p.n_tokens <= 32) {
        const dim3 grid((a.p.n_tokens + 15) / 16, a.p.n_heads, head_dim / 16);
        if (a.R == 256) hipLaunchKernelGGL((latent_unabsorb_few_kernel<256>), grid, dim3(NT), 0, s, a, head_dim);
        else hipLaunchKernelGGL((latent_unabsorb_few_kernel<512>), grid, dim3(NT), 0, s, a, head_dim);
    } else {
        const dim3 grid((a.p.n_tokens + 63) / 64, a.p.n_heads, head_dim / 64);
        if (a.R == 256) hipLaunchKernelGGL((latent_unabsorb_kernel<256, 4>), grid, dim3(NT), 0, s, a, head_dim);
        else hipLaunchKernelGGL((latent_unabsorb_kernel<512, 4>), grid, dim3(NT), 0, s, a, head_dim);
    }
    return hipGetLastError();
}

hipError_t launch_latent_expand(const LatentArgs &a, int head_dim, hipStream_t s) {
    // a round of workgroups: each pays for its first loads and its place in the batch once
    const int cols = (a.p.n_heads * head_dim + 127) / 128, blocks = (int)(a.p.head_rows / kSeqRows);
    const dim3 grid((unsigned)std::min(std::max(256 / blocks, 1), cols), (unsigned)blocks), threads(512);
    if (head_dim == 64) {
        if (a.R == 256) hipLaunchKernelGGL((latent_expand_kernel<64, 256>), grid, threads, 0, s, a);
        else hipLaunchKernelGGL((latent_expand_kernel<64, 512>), grid, threads, 0, s, a);
    } else {
        if (a.R == 256) hipLaunchKernelGGL((latent_expand_kernel<128, 256>), grid, threads, 0, s, a);
        else hipLaunchKernelGGL((latent_expand_kernel<128, 512>), grid, threads, 0, s, a);
    }
    return hipGetLastError();
}

}  // namespace fkv
