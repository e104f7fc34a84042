// What the kernels over rows of channels share (layer normalisation, checkpoints, embedding): eight channels of a row in registers, and sums over the
// lanes of a wavefront.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace delta {
namespace rows {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
struct bf16 { uint16_t bits; };

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    const f32x2 v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

// Eight neighbouring channels as they lie in memory, 16 bytes (bf16) or 32 (fp32).
template <typename T> struct Eight;
template <> struct Eight<bf16> {
    u32x4 raw;
    __device__ __forceinline__ void zero() { raw = u32x4{0u, 0u, 0u, 0u}; }
    __device__ __forceinline__ void load(const unsigned char *p) { raw = *reinterpret_cast<const u32x4 *>(p); }
    __device__ __forceinline__ void to(float (&v)[8]) const {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[2 * e] = __uint_as_float(raw[e] << 16);
            v[2 * e + 1] = __uint_as_float(raw[e] & 0xFFFF0000u);
        }
    }
    static __device__ __forceinline__ void store(unsigned char *p, const float (&v)[8]) {
        *reinterpret_cast<u32x4 *>(p) = u32x4{pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7])};
    }
};
template <> struct Eight<float> {
    f32x4 a, b;
    __device__ __forceinline__ void zero() { a = b = f32x4{0.f, 0.f, 0.f, 0.f}; }
    __device__ __forceinline__ void load(const unsigned char *p) {
        a = reinterpret_cast<const f32x4 *>(p)[0];
        b = reinterpret_cast<const f32x4 *>(p)[1];
    }
    __device__ __forceinline__ void to(float (&v)[8]) const {
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[4 + e] = b[e]; }
    }
    static __device__ __forceinline__ void store(unsigned char *p, const float (&v)[8]) {
        reinterpret_cast<f32x4 *>(p)[0] = f32x4{v[0], v[1], v[2], v[3]};
        reinterpret_cast<f32x4 *>(p)[1] = f32x4{v[4], v[5], v[6], v[7]};
    }
};

// A lane's value from another lane of its row of 16, without a trip through LDS.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, false); }
template <int CTRL>
__device__ __forceinline__ float dpp(float v) { return __uint_as_float(dpp<CTRL>(__float_as_uint(v))); }
__device__ __forceinline__ uint32_t quad_xor1(uint32_t v) { return dpp<0xB1>(v); }     // quad_perm 1,0,3,2
__device__ __forceinline__ uint32_t quad_xor2(uint32_t v) { return dpp<0x4E>(v); }     // quad_perm 2,3,0,1

// v plus its value in the other row of 16 of each half (the other half) of the wavefront: the swap hands a register's odd rows (upper half) to a copy's
// even ones (lower half).
__device__ __forceinline__ float row_pairs(float v) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float halves(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// The sum of v over the 32 lanes of half a wavefront, over all 64, the same in each: within the rows of 16 by quad permutations and mirrors, then by the
// swaps.  All lanes of the half (of the wavefront) active.
__device__ __forceinline__ float half_sum(float v) {
    v += dpp<0xB1>(v);
    v += dpp<0x4E>(v);
    v += dpp<0x141>(v);                                                    // row_half_mirror: the other quad of a lane's eight
    v += dpp<0x140>(v);                                                    // row_mirror: the other eight
    return row_pairs(v);
}
__device__ __forceinline__ float wave_sum(float v) { return halves(half_sum(v)); }

}  // namespace rows
}  // namespace delta
