// paged_join.h -- joins the parts of split items: M = max_j m_j,
// L = sum_j 2^(c (m_j - M)) l_j, O = sum_j 2^(c (m_j - M)) o_j / L.  A launch of its own: the
// parts cross as ordinary stores and loads, and the workspace holds no counters.
// A workgroup takes 64 channels of join_tokens tokens of a query head, 16 threads 4 channels
// each.  WIDE (few parts of many rows): every 16 threads take rows of their own; otherwise
// they share a row, each taking every kLanes'th part, and their sums meet in LDS in a fixed
// order.  Tokens of items that were not split are left alone.
#pragma once

#include "paged.h"

namespace fkv {
namespace paged {

constexpr int kJoinThreads = 256, kJoin = 4;   // threads of a workgroup, parts loaded at a time
typedef float join_f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 join_bf16x4 __attribute__((ext_vector_type(4)));

// grid: x = tokens, y = query head, z = 64 channels.  ROWS, KT: of the kernel that wrote the parts.
template <int D, int ROWS, int KT, bool WIDE>
__global__ __launch_bounds__(kJoinThreads) void paged_join_kernel(PagedArgs a) {
    constexpr int kLanes = kJoinThreads / 16;
    constexpr int64_t kSlot = ROWS * (D + 2);
    __shared__ join_f32x4 sum[kLanes][16];
    __shared__ float top[kLanes], total[kLanes];
    const int head = blockIdx.y, y = head / a.group, d = threadIdx.x % 16, lane = threadIdx.x / 16;
    const int ch = 64 * blockIdx.z + 4 * d;
    const int end = min((int)(blockIdx.x + 1) * a.join_tokens, a.n_tokens);
    const Split<ROWS, KT> split(a);
    for (int token = blockIdx.x * a.join_tokens; token < end;) {
        const Work w = split.locate(a, 0, token, end);   // (the same in the whole workgroup)
        if (!w.ok) return;
        const int from = max(token, w.s.start), last = min(end, w.s.start + w.s.n);   // the sequence's tokens of the workgroup
        const int rts = w.step / a.kv;
        const int64_t step = w.step * kSlot;
        for (int t = from + (WIDE ? lane : 0); t < last; t += WIDE ? kLanes : 1) {
            const int tok = t - w.s.start, r = tok * a.group + head - y * a.group, rt = r / ROWS;
            const float *p = a.part + (int64_t)(w.slot + y * rts + rts - 1 - rt) * kSlot;
            const float *po = p + (r - rt * ROWS) * D + ch, *pm = p + ROWS * D + r - rt * ROWS, *pl = pm + ROWS;
            float M = neg_inf(), L = 0.f;
            join_f32x4 acc = {0.f, 0.f, 0.f, 0.f};
            auto add = [&](float m, float l, const join_f32x4 &o) {
                const float Mn = fmaxf(M, m), ref = Mn == neg_inf() ? 0.f : Mn;
                const float so = __builtin_amdgcn_exp2f((M - ref) * a.scale_log2), sn = __builtin_amdgcn_exp2f((m - ref) * a.scale_log2);
                M = Mn;
                L = L * so + l * sn;
                acc = acc * so + o * sn;
            };
            constexpr int kStep = WIDE ? 1 : kLanes;
            for (int j0 = WIDE ? 0 : lane; j0 < w.parts; j0 += kJoin * kStep) {
                float mj[kJoin], lj[kJoin];
                join_f32x4 o[kJoin];
#pragma unroll
                for (int j = 0; j < kJoin; ++j) {
                    const int64_t at = min(j0 + j * kStep, w.parts - 1) * step;
                    mj[j] = pm[at];
                    lj[j] = pl[at];
                    o[j] = *(const join_f32x4 *)(po + at);
                }
                // (all loads before the first use: one memory latency, not one each)
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int j = 0; j < kJoin; ++j)
                    if (j0 + j * kStep < w.parts) add(mj[j], lj[j], o[j]);
            }
            if (!WIDE) {
                __syncthreads();                         // (the row before is read)
                sum[lane][d] = acc;
                if (d == 0) {
                    top[lane] = M;
                    total[lane] = L;
                }
                __syncthreads();
                if (lane > 0) continue;
                for (int i = 1; i < kLanes; ++i) add(top[i], total[i], sum[i][d]);
            }
            const bool none = sight(a, w.s, a.recent[y], tok).end <= 0;
            const float inv = none ? 0.f : 1.f / L;
            join_bf16x4 out;
#pragma unroll
            for (int k = 0; k < 4; ++k) out[k] = (__bf16)(acc[k] * inv);
            *(join_bf16x4 *)(a.O + (int64_t)t * a.o_tok + (int64_t)head * a.o_head + ch) = out;
            if (a.lse && ch == 0)
                a.lse[(int64_t)head * a.n_tokens + t] = none ? neg_inf() : fmaf(M * 0.69314718055994530942f, a.scale_log2, logf(L));
        }
        token = last;
    }
}

template <int D, int ROWS, int KT, bool WIDE>
inline void launch_join(const PagedArgs &a, hipStream_t s) {
    const dim3 grid((unsigned)((a.n_tokens + a.join_tokens - 1) / a.join_tokens), (unsigned)a.n_heads, D / 64);
    hipLaunchKernelGGL((paged_join_kernel<D, ROWS, KT, WIDE>), grid, dim3(kJoinThreads), 0, s, a);
}

}  // namespace paged
}  // namespace fkv
