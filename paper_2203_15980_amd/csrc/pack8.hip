// DELTA_OP_PACK8 and DELTA_OP_UNPACK8 for gfx950: an activation into its 8-bit checkpoint (packed.hpp) and back.
// Beside Evict and Offload (DELTA Table 1) a third way to make an activation small between the forward and the backward pass.
//
// Bound by memory: 3.03 bytes a value in bf16, 5.03 in fp32, one read and one write of each.  A thread owns eight channels (16 or 32 bytes on one side,
// 8 on the other), the four threads of a block of 32 find its largest magnitude with two exchanges inside the quad, and each thread has
// kAhead such pieces in flight.  us for 16384 x 768, pack and unpack, with 1, 2, 4, 8 pieces: bf16 (38 MB each) 7.7 + 7.6, 6.6 + 6.8 (5.7 TB/s),
// 9.0 + 7.9, 10.3 + 9.7; fp32 (63 MB) 14.9 + 13.2 (11 + 13 on tensors that the caches partly hold), 16.3 + 13.1, 17.0 + 13.1, 18.4 + 14.5.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.hpp"
#include "packed.hpp"
#include "rows.hpp"

namespace delta {
namespace pk8 {

using packed::u32x2;

constexpr int kThreads = 256;
template <typename T> constexpr int kAhead = sizeof(T) == 2 ? 2 : 1;

struct Args {
    const unsigned char *x;
    unsigned char *y;
    uint64_t scales;             // byte offset of the scale bytes in the checkpoint
    uint32_t blocks;             // rows * ceil(C / 32)
    uint32_t nb, C;              // blocks of a row, channels
    Divisor per_row;             // nb
};

// Where piece `at` (a quarter of a block) lies: its block, its first element in the tensor, and whether it is inside its row.
struct Place { uint32_t block; uint64_t element; bool live; };
__device__ __forceinline__ Place place(const Args &a, uint64_t at) {
    Place p;
    p.block = (uint32_t)(at >> 2);
    const uint32_t row = (uint32_t)divide((int)p.block, a.per_row), col = (p.block - row * a.nb) * 32 + ((uint32_t)at & 3) * 8;
    p.element = (uint64_t)row * a.C + col;
    p.live = p.block < a.blocks && col < a.C;
    return p;
}

template <typename T, int FMT>
__global__ __launch_bounds__(kThreads) void pack_kernel(Args a) {
    const uint64_t first = (uint64_t)blockIdx.x * (kThreads * kAhead<T>) + threadIdx.x;
    rows::Eight<T> raw[kAhead<T>];
    Place p[kAhead<T>];
#pragma unroll
    for (int i = 0; i < kAhead<T>; ++i) {
        p[i] = place(a, first + i * kThreads);
        raw[i].zero();
        if (p[i].live) raw[i].load(a.x + p[i].element * sizeof(T));
    }
#pragma unroll
    for (int i = 0; i < kAhead<T>; ++i) {
        float v[8];
        raw[i].to(v);
        uint32_t amax = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) amax = max(amax, __float_as_uint(v[e]) & 0x7FFFFFFFu);
        amax = max(amax, rows::quad_xor1(amax));
        amax = max(amax, rows::quad_xor2(amax));
        const uint32_t byte = packed::scale_byte<FMT>(amax);
        if (p[i].live) *reinterpret_cast<u32x2 *>(a.y + p[i].element) = packed::encode<FMT>(v, packed::inverse_of(byte));
        if ((threadIdx.x & 3) == 0 && p[i].block < a.blocks) a.y[a.scales + p[i].block] = (unsigned char)byte;
    }
}

template <typename T, int FMT>
__global__ __launch_bounds__(kThreads) void unpack_kernel(Args a) {
    const uint64_t first = (uint64_t)blockIdx.x * (kThreads * kAhead<T>) + threadIdx.x;
    u32x2 raw[kAhead<T>];
    uint32_t byte[kAhead<T>];
    Place p[kAhead<T>];
#pragma unroll
    for (int i = 0; i < kAhead<T>; ++i) {
        p[i] = place(a, first + i * kThreads);
        if (p[i].live) {
            raw[i] = *reinterpret_cast<const u32x2 *>(a.x + p[i].element);
            byte[i] = a.x[a.scales + p[i].block];
        }
    }
#pragma unroll
    for (int i = 0; i < kAhead<T>; ++i) {
        if (!p[i].live) continue;
        float v[8];
        packed::decode<FMT>(raw[i], packed::scale_of(byte[i]), v);
        rows::Eight<T>::store(a.y + p[i].element * sizeof(T), v);
    }
}

}  // namespace pk8

const char *pack8_check(const void *x, const void *y, long long rows, int C, int fmt) {
    if (fmt != PACK_INT8 && fmt != PACK_E4M3) return "a checkpoint is DELTA_PACK_INT8 or DELTA_PACK_E4M3";
    if (rows <= 0 || rows > 0x7FFFFFFFLL || C <= 0 || C % 8) return "channels must be a multiple of 8";
    if (rows * ((C + kPackBlock - 1LL) / kPackBlock) > 0x7FFFFFFFLL / 4) return "too many rows for a checkpoint";
    if (!x || !y || (((uintptr_t)x | (uintptr_t)y) & 15)) return "pointers must be non-null and 16-byte aligned";
    return nullptr;
}

// x [rows, C] in bf16 or fp32 and its checkpoint y (pack), or a checkpoint x and the tensor y.
hipError_t launch_pack8(const void *x, void *y, long long rows, int C, int bf16, int fmt, bool pack, hipStream_t stream) {
    if (pack8_check(x, y, rows, C, fmt)) return hipErrorInvalidValue;
    pk8::Args a;
    a.x = static_cast<const unsigned char *>(x); a.y = static_cast<unsigned char *>(y);
    a.scales = packed_scale_offset(rows, C);
    a.nb = (uint32_t)((C + kPackBlock - 1) / kPackBlock); a.C = (uint32_t)C;
    a.blocks = (uint32_t)(rows * a.nb);
    a.per_row = make_divisor(a.nb);
    const uint32_t each = pk8::kThreads * (bf16 ? pk8::kAhead<rows::bf16> : pk8::kAhead<float>), grid = (a.blocks * 4 + each - 1) / each;
    auto run = [&](auto kernel) { kernel<<<dim3(grid), dim3(pk8::kThreads), 0, stream>>>(a); };
    if (pack) {
        if (bf16) fmt == PACK_INT8 ? run(pk8::pack_kernel<rows::bf16, PACK_INT8>) : run(pk8::pack_kernel<rows::bf16, PACK_E4M3>);
        else fmt == PACK_INT8 ? run(pk8::pack_kernel<float, PACK_INT8>) : run(pk8::pack_kernel<float, PACK_E4M3>);
    } else {
        if (bf16) fmt == PACK_INT8 ? run(pk8::unpack_kernel<rows::bf16, PACK_INT8>) : run(pk8::unpack_kernel<rows::bf16, PACK_E4M3>);
        else fmt == PACK_INT8 ? run(pk8::unpack_kernel<float, PACK_INT8>) : run(pk8::unpack_kernel<float, PACK_E4M3>);
    }
    return hipGetLastError();
}

}  // namespace delta
