// The 64 lanes of a wavefront on the host: device code whose control flow is the same in all of them runs as 64 fibers, which meet at each exchange between lanes.
#pragma once
#include <math.h>
#include <setjmp.h>
#include <stddef.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>
#include <ucontext.h>
#include <functional>
#include <type_traits>
#include <vector>

#define __device__
#define __host__
#define __global__
#define __shared__ static
#define __forceinline__ inline
#define __launch_bounds__(...)
#define __align__(n) alignas(n)
#define asm                          // inline assembly does nothing here: none of what is tested has any
#define volatile(...)

typedef int hipError_t;
typedef void *hipStream_t;
enum { hipSuccess = 0, hipErrorInvalidValue = 1 };
struct uint2 { uint32_t x, y; };
struct dim3 { unsigned x, y, z; };

namespace lanes {
constexpr int kLanes = 64;
struct Fiber { ucontext_t start; jmp_buf at; bool begun, done; std::vector<char> stack; };
inline Fiber fiber[kLanes];
inline jmp_buf scheduler;
inline int now;                      // the running lane
inline uint32_t sent[2][kLanes];
inline std::function<void()> body;
inline int exchanges[kLanes];

inline void entry() {
    body();
    fiber[now].done = true;
    _longjmp(scheduler, 1);
}
// Lane `now` stops here until all others have come as far.
inline void meet() {
    ++exchanges[now];
    if (!_setjmp(fiber[now].at)) _longjmp(scheduler, 1);
}
inline void run(std::function<void()> f) {
    body = std::move(f);
    for (int i = 0; i < kLanes; ++i) { fiber[i].begun = fiber[i].done = false; exchanges[i] = 0; }
    for (bool more = true; more;) {
        more = false;
        for (now = 0; now < kLanes; ++now) {
            Fiber &f = fiber[now];
            if (f.done) continue;
            if (!_setjmp(scheduler)) {
                if (f.begun) _longjmp(f.at, 1);
                f.begun = true;
                if (f.stack.empty()) f.stack.resize(1 << 16);
                getcontext(&f.start);
                f.start.uc_stack.ss_sp = f.stack.data();
                f.start.uc_stack.ss_size = f.stack.size();
                makecontext(&f.start, entry, 0);
                setcontext(&f.start);
            }
            more = more || !fiber[now].done;
        }
        for (int i = 1; i < kLanes; ++i)
            if (exchanges[i] != exchanges[0] || fiber[i].done != fiber[0].done) { fprintf(stderr, "lanes went different ways\n"); abort(); }
    }
}
// Everyone's value.
inline const uint32_t *everyone(uint32_t v) {
    const int turn = exchanges[now] & 1;                 // the last exchange's values may still be read
    sent[turn][now] = v;
    meet();
    return sent[turn];
}
struct Pair { uint32_t v[2]; uint32_t operator[](int i) const { return v[i]; } };
struct Index { operator unsigned() const { return (unsigned)now; } };
struct Three { Index x; };
}  // namespace lanes

static lanes::Three threadIdx;
static struct { unsigned x; } blockIdx, blockDim, gridDim;

inline unsigned long long __ballot(bool b) {
    const uint32_t *all = lanes::everyone(b);
    unsigned long long r = 0;
    for (int i = 0; i < 64; ++i) r |= (unsigned long long)(all[i] != 0) << i;
    return r;
}
inline int emulated_readlane(int v, int lane) { return (int)lanes::everyone((uint32_t)v)[lane & 63]; }
inline int emulated_readfirstlane(int v) { return emulated_readlane(v, 0); }
inline int emulated_dpp(int, int v, int ctrl, int, int, bool) {
    const uint32_t *all = lanes::everyone((uint32_t)v);
    const int l = lanes::now;
    switch (ctrl) {
    case 0xB1: return (int)all[l ^ 1];                   // quad_perm 1,0,3,2
    case 0x4E: return (int)all[l ^ 2];                   // quad_perm 2,3,0,1
    case 0x140: return (int)all[l ^ 15];                 // row_mirror
    case 0x141: return (int)all[l ^ 7];                  // row_half_mirror
    default: abort();
    }
}
inline lanes::Pair emulated_permlane_swap(uint32_t a, uint32_t b, int n) {       // a's odd groups of n lanes change places with b's even ones
    const int l = lanes::now;
    const uint32_t x = lanes::everyone(a)[l & ~n], y = lanes::everyone(b)[l & ~n];
    const uint32_t z = lanes::everyone(a)[l | n], w = lanes::everyone(b)[l | n];
    return l & n ? lanes::Pair{{y, w}} : lanes::Pair{{x, z}};
}
inline lanes::Pair emulated_permlane16_swap(uint32_t a, uint32_t b, bool, bool) { return emulated_permlane_swap(a, b, 16); }
inline lanes::Pair emulated_permlane32_swap(uint32_t a, uint32_t b, bool, bool) { return emulated_permlane_swap(a, b, 32); }
#define __builtin_amdgcn_readlane emulated_readlane
#define __builtin_amdgcn_readfirstlane emulated_readfirstlane
#define __builtin_amdgcn_update_dpp emulated_dpp
#define __builtin_amdgcn_permlane16_swap emulated_permlane16_swap
#define __builtin_amdgcn_permlane32_swap emulated_permlane32_swap
inline int max(int a, int b) { return a > b ? a : b; }
inline uint32_t max(uint32_t a, uint32_t b) { return a > b ? a : b; }
inline int __umulhi(uint32_t a, uint32_t b) { return (int)((uint64_t)a * b >> 32); }

// What the headers name beside, for the compiler's sake.
inline uint32_t __float_as_uint(float f) { uint32_t u; memcpy(&u, &f, 4); return u; }
inline float __uint_as_float(uint32_t u) { float f; memcpy(&f, &u, 4); return f; }
inline float __builtin_amdgcn_rcpf(float v) { return 1.0f / v; }
inline float __builtin_amdgcn_exp2f(float v) { return exp2f(v); }
template <typename... T> inline short __attribute__((ext_vector_type(4))) __builtin_amdgcn_ds_read_tr16_b64_v4i16(T...) { abort(); }
template <typename A, typename B, typename C> inline C __builtin_amdgcn_mfma_f32_32x32x16_bf16(A, B, C, int, int, int) { abort(); }
