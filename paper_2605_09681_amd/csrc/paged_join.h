// paged_join.h -- joins the parts of cut items: M = max_j m_j,
// L = sum_j 2^(c (m_j - M)) l_j, O = sum_j 2^(c (m_j - M)) o_j / L, l_j the sum of the weights as they weigh
// the values, rounded to bf16; lse takes that of the weights themselves.  A launch of its own: the
// parts cross as ordinary stores and loads, and the workspace holds no counters.  The
// launch that writes the parts leaves a JoinItem for every cut item, so that this one works
// nothing out again (each workgroup finding its items from the lengths took 5 to 10 us, and
// whole launches of them 10 to 60).
#pragma once

#include "paged.h"

namespace fkv {
namespace paged {

constexpr int kJoinThreads = 256;
typedef float join_f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 join_bf16x4 __attribute__((ext_vector_type(4)));

struct Joined {
    float M = neg_inf(), L = 0.f, E = 0.f;        // E: of the exact sums
    join_f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    __device__ __forceinline__ void add(float m, float l, float exact, const join_f32x4 &o, float scale_log2) {
        const float Mn = fmaxf(M, m), ref = Mn == neg_inf() ? 0.f : Mn;
        const float so = __builtin_amdgcn_exp2f((M - ref) * scale_log2), sn = __builtin_amdgcn_exp2f((m - ref) * scale_log2);
        M = Mn;
        L = L * so + l * sn;
        E = E * so + exact * sn;
        acc = acc * so + o * sn;
    }
    // Channels ch .. ch + 3 of the item's row r.  WIDE: of fp32.
    template <bool WIDE = false>
    __device__ __forceinline__ void put(const PagedArgs &a, const JoinItem &j, int r, int ch) const {
        const int row = j.row0 + r, tok = token_of(a, row), head = j.y * a.group + row - tok * a.group, t = j.start + tok;
        const bool none = blind(sight(a, Seq{j.len, j.start, 0, j.first}, a.recent[j.y], tok), a.sink[j.y]);
        const float inv = none ? 0.f : 1.f / L;
        join_bf16x4 out;
#pragma unroll
        for (int k = 0; k < 4; ++k) out[k] = (__bf16)(acc[k] * inv);
        const int64_t to = (int64_t)t * a.o_tok + (int64_t)head * a.o_head + ch;
        if (WIDE) *(join_f32x4 *)((float *)a.O + to) = acc * inv;
        else *(join_bf16x4 *)(a.O + to) = out;
        if (a.lse && ch == 0)
            a.lse[(int64_t)head * a.n_tokens + t] = none ? neg_inf() : fmaf(M * 0.69314718055994530942f, a.scale_log2, logf(E));
    }
};

}  // namespace paged
}  // namespace fkv
