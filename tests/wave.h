// wave.h -- one 64-lane wave on the host, for tests of device code that works something out
// with cross-lane operations: each lane runs as a context of its own up to its next such
// operation, where all lanes meet.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <setjmp.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <ucontext.h>

#include <algorithm>
#include <functional>
#include <vector>

namespace wave {

constexpr int kLanes = 64;
struct State {
    ucontext_t back, lane[kLanes];
    jmp_buf resume, at[kLanes];      // (once a lane has begun: without swapcontext's system calls)
    int now, ended;
    uint64_t value[2][kLanes];
    int op[2][kLanes], turn[kLanes];
    std::function<void(int)> body;
};
inline State &state() {
    static State s;
    return s;
}

inline void entry() {
    State &s = state();
    s.body(s.now);
    ++s.ended;
    _longjmp(s.resume, 1);
}

// body(lane) in all lanes.
inline void run(std::function<void(int)> body) {
    static std::vector<char> stacks((size_t)kLanes << 17);
    State &s = state();
    s.body = body;
    s.ended = 0;
    for (int i = 0; i < kLanes; ++i) {
        getcontext(&s.lane[i]);
        s.lane[i].uc_stack.ss_sp = stacks.data() + ((size_t)i << 17);
        s.lane[i].uc_stack.ss_size = (size_t)1 << 17;
        s.lane[i].uc_link = nullptr;
        makecontext(&s.lane[i], entry, 0);
        s.turn[i] = 0;
    }
    for (bool begun = false; s.ended == 0; begun = true) {
        for (s.now = 0; s.now < kLanes; ++s.now)
            if (!_setjmp(s.resume)) {
                if (begun) _longjmp(s.at[s.now], 1);
                else swapcontext(&s.back, &s.lane[s.now]);
            }
        if (s.ended != 0 && s.ended != kLanes) {
            fprintf(stderr, "%d of 64 lanes ended\n", s.ended);
            abort();
        }
    }
}

// This lane's value, and what all lanes brought to the same operation.
inline const uint64_t *meet(int op, uint64_t v) {
    State &s = state();
    const int i = s.now, t = s.turn[i]++ & 1;
    s.value[t][i] = v;
    s.op[t][i] = op;
    if (!_setjmp(s.at[i])) _longjmp(s.resume, 1);
    for (int k = 0; k < kLanes; ++k)
        if (s.op[t][k] != op) {
            fprintf(stderr, "lane %d is at operation %d, lane %d at %d\n", i, op, k, s.op[t][k]);
            abort();
        }
    return s.value[t];
}

struct Index {
    operator int() const { return state().now; }
};
struct Dim {
    Index x;
};

}  // namespace wave

static const wave::Dim threadIdx;

inline uint64_t __ballot(int p) {
    const uint64_t *v = wave::meet(1, p != 0);
    uint64_t b = 0;
    for (int i = 0; i < wave::kLanes; ++i) b |= v[i] << i;
    return b;
}
inline int __builtin_amdgcn_readlane(int x, int lane) { return (int)(uint32_t)wave::meet(2, (uint32_t)x)[lane & 63]; }
inline int __builtin_amdgcn_update_dpp(int old, int x, int ctrl, int rows, int, bool) {
    const uint64_t *v = wave::meet(ctrl, (uint32_t)x);
    const int i = wave::state().now, row = i >> 4;
    int from = -1;
    if (ctrl > 0x110 && ctrl <= 0x11f) from = (i & 15) >= (ctrl & 15) ? i - (ctrl & 15) : -1;
    else if (ctrl == 0x142) from = row > 0 ? 16 * row - 1 : -1;
    else if (ctrl == 0x143) from = row > 1 ? 31 : -1;
    else abort();
    return from < 0 || !(rows >> row & 1) ? old : (int)(uint32_t)v[from];
}
inline uint32_t __umulhi(uint32_t a, uint32_t b) { return (uint32_t)((uint64_t)a * b >> 32); }
inline float __builtin_amdgcn_rcpf(float x) { return 1.f / x; }
inline int __builtin_amdgcn_frexp_expf(float x) {
    int e;
    frexpf(x, &e);
    return e;
}
template <class T>
inline float __builtin_amdgcn_fdot2_f32_bf16(T a, T b, float c, bool) {
    return (float)((double)(float)a[0] * (float)b[0] + (double)(float)a[1] * (float)b[1] + c);
}
inline float __builtin_amdgcn_ldexpf(float x, int e) { return ldexpf(x, e); }
inline float __builtin_amdgcn_exp2f(float x) { return exp2f(x); }
inline int __float_as_int(float x) { return __builtin_bit_cast(int, x); }
inline float __int_as_float(int x) { return __builtin_bit_cast(float, x); }
inline float __uint_as_float(uint32_t x) { return __builtin_bit_cast(float, x); }
inline void __syncthreads() { wave::meet(3, 0); }
using std::max;
using std::min;
