// Activation checkpoints in 8 bits: the format, and how eight channels of it are written and read.
//
// A tensor of [rows, C] values (bf16 or fp32) is held as rows * C bytes, one a value, padded to 16 bytes, then one scale byte for each
// block of 32 channels of a row (the last block of a row may be shorter), [rows][ceil(C / 32)], padded to 16 bytes.
//   A block's scale is 2^e with e the smallest integer in [-120, 122] for which no value of the block exceeds MAX * 2^e; its byte is e + 127.
//   A value is round(x / 2^e), ties to even:
//     int8   a whole number q in [-127, 127] (MAX = 127); the byte is q in two's complement
//     e4m3   an OCP E4M3 number (MAX = 448); the byte is its code
//   A block that holds an infinity or a NaN has the scale byte 255 and reads back as NaN throughout: an overflow stays visible.
// The scale is a power of two, so that x / 2^e and q * 2^e are exact: packing rounds once, unpacking not at all (q * 2^e has at most 8 significant bits
// and its lowest is 2^-129 or more, which bf16 and fp32 both hold), and a kernel that reads the checkpoint works on the same values as
// one that reads the unpacked tensor.  Against x the rounding is off by at most 2^e / 2 <= max|x| / 127 (int8; half of that at best) or 2^-4 |x| (e4m3, in
// its normal range).  8.25 bits a value: 0.516 of bf16, 0.258 of fp32.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace delta {

enum { PACK_NONE = 0, PACK_INT8 = 1, PACK_E4M3 = 2 };

constexpr int kPackBlock = 32;
inline uint64_t packed_scale_offset(uint64_t rows, uint64_t C) { return (rows * C + 15) / 16 * 16; }
inline uint64_t packed_bytes(uint64_t rows, uint64_t C) {
    return packed_scale_offset(rows, C) + (rows * ((C + kPackBlock - 1) / kPackBlock) + 15) / 16 * 16;
}

namespace packed {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// The scale byte of a block from the bits of its largest magnitude.  Compared as integers: a NaN's lie above infinity's.
template <int FMT>
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax) {
    constexpr uint32_t kTop = FMT == PACK_INT8 ? 6 : 8;                    // MAX = kFrac * 2^kTop, 1.984375 and 1.75
    constexpr uint32_t kFrac = FMT == PACK_INT8 ? 0x7E0000u : 0x600000u;   // its fraction bits
    const int b = (int)(amax >> 23) - (int)kTop + ((amax & 0x7FFFFFu) > kFrac ? 1 : 0);
    return amax >= 0x7F800000u ? 255u : (uint32_t)(b < 7 ? 7 : b);
}
__device__ __forceinline__ float scale_of(uint32_t byte) { return byte == 255u ? __builtin_nanf("") : __uint_as_float(byte << 23); }
__device__ __forceinline__ float inverse_of(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }   // 2^-e; of 255: anything

// Eight values into eight bytes.  int8: 3 * 2^22 + x / 2^e rounds to a whole number in fp32, ties to even, and its low byte is q.
template <int FMT>
__device__ __forceinline__ u32x2 encode(const float (&v)[8], float inv) {
    u32x2 o;
    if constexpr (FMT == PACK_INT8) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t w = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                w |= (__float_as_uint(__builtin_fmaf(v[4 * h + i], inv, 12582912.f)) & 0xFFu) << (8 * i);
            o[h] = w;
        }
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h] * inv, v[4 * h + 1] * inv, 0, false);
            o[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h + 2] * inv, v[4 * h + 3] * inv, w, true);
        }
    }
    return o;
}
// Byte N of a word, signed, as fp32: one instruction, where the compiler often makes three (layer normalisation's gradients from int8, 768 channels, 16384 rows:
// 21.3 us, 17 with it).
template <int N>
__device__ __forceinline__ float signed_byte(uint32_t w) {
    float f;
    if constexpr (N == 0) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_0" : "=v"(f) : "v"(w));
    if constexpr (N == 1) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_1" : "=v"(f) : "v"(w));
    if constexpr (N == 2) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_2" : "=v"(f) : "v"(w));
    if constexpr (N == 3) asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_3" : "=v"(f) : "v"(w));
    return f;
}
// Two of a word's four values (the upper two if `hi`), times a scale each.
template <int FMT>
__device__ __forceinline__ void decode2(uint32_t w, bool hi, float s0, float s1, float *v) {
    if constexpr (FMT == PACK_INT8) {
        v[0] = (hi ? signed_byte<2>(w) : signed_byte<0>(w)) * s0;
        v[1] = (hi ? signed_byte<3>(w) : signed_byte<1>(w)) * s1;
    } else {
        const f32x2 a = hi ? __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true) : __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
        v[0] = a.x * s0;
        v[1] = a.y * s1;
    }
}
// Eight values of one block.
template <int FMT>
__device__ __forceinline__ void decode(u32x2 w, float s, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) decode2<FMT>(w[i >> 1], i & 1, s, s, v + 2 * i);
}

}  // namespace packed
}  // namespace delta
