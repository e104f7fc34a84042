// What the kernels of attention over packed sequences share: where a workgroup's rows lie, tiles on their way to LDS, operands out of it.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.hpp"
#include "rows.hpp"

namespace delta {
namespace pat {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
using rows::f32x4;
using rows::u32x4;

struct Args {
    const unsigned char *x;                              // [M][(heads + 2 kv) D]: queries, keys, values
    const long long *off;                                // [seqs + 1]
    unsigned char *y;                                    // [M][heads D]: forward's output (backward: read)
    float *lse;                                          // [heads][M], natural; null: not stored
    const unsigned char *gy;                             // [M][heads D]
    unsigned char *gx;                                   // as x
    float *delta;                                        // [heads][M], sum over a row's channels of y gy
    int M, seqs, heads, kv, slots;
    float scale, scale_log2e;                            // 1 / sqrt(D), times log2 e
};

// Rows of a workgroup: `tile` of the segment [start, start + len).  Segments: the rows before the first sequence, the sequences, the rows behind the last
// (the first and the last belong to no sequence: `alone`).  Boundaries are held in [0, M], so that no offset leads out of the tensors.
//
// The lengths are known to the device alone, so a launch has a slot for every tile there may be: segment j's tiles take the slots from
// floor(start_j / Q) + j on.  They have room, as ceil(len / Q) <= floor((start + len) / Q) - floor(start / Q) + 1; slots left over end at once.
struct Rows { int start, len, tile; bool alone; };

__device__ __forceinline__ int boundary(const Args &a, int j) {                    // of segment j's first row; j = seqs + 2: M
    if (j == 0) return 0;
    if (j == a.seqs + 2) return a.M;
    const long long o = a.off[j - 1];
    return o < 0 ? 0 : o > a.M ? a.M : (int)o;
}
inline int slots_of(int M, int seqs, int Q) { return M / Q + seqs + 2; }

// The segment whose slots hold `slot`: a wavefront looks at 64 boundaries at a time.  False: no tile there.
template <int Q>
__device__ __forceinline__ bool find_rows(const Args &a, int slot, Rows &r) {
    const int lane = threadIdx.x & 63;
    int lo = 0, n = a.seqs + 2;
    while (n > 1) {
        const int step = (n + 63) / 64, j = lo + lane * step;
        const bool before = lane * step < n && boundary(a, j) / Q + j <= slot;
        const int k = __builtin_popcountll(__ballot(before)) - 1;                  // lane 0's segment begins at or before the slot
        const int at = k < 0 ? 0 : k;
        lo += at * step;
        n = n - at * step < step ? n - at * step : step;
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    const int b = __builtin_amdgcn_readfirstlane(boundary(a, lo)), e = __builtin_amdgcn_readfirstlane(boundary(a, lo + 1));
    r.start = b;
    r.len = e - b;
    r.tile = slot - (b / Q + lo);
    r.alone = lo == 0 || lo == a.seqs + 1;
    return r.tile >= 0 && r.tile * (long long)Q < r.len;
}

// Consecutive workgroups go to the 8 XCDs in turn, each with an L2 of its own: numbered like this, an XCD's heads are neighbours, which share keys and values.
__device__ __forceinline__ int head_of(int i, int heads) { return heads % 8 ? i : (i & 7) * (heads >> 3) + (i >> 3); }

// Rows of D bf16 channels in LDS: a pitch of an odd number of 16 bytes, so that neighbouring rows' pieces lie in different banks.
template <int D> constexpr int kPitch = D * 2 + 16;

// A tile of 64 rows on its way from memory through registers to LDS, by THREADS threads; rows from `limit` on come as zeros.
template <int D, int ROWS, int THREADS>
struct Tile {
    static constexpr int kPieces = ROWS * (D / 8) / THREADS;
    static_assert(ROWS * (D / 8) % THREADS == 0, "whole pieces");
    u32x4 v[kPieces];
    __device__ __forceinline__ void fetch(const unsigned char *base, size_t pitch, int first, int limit) {
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
            const int i = (int)threadIdx.x + p * THREADS, r = first + i / (D / 8), seg = i % (D / 8);
            v[p] = u32x4{0u, 0u, 0u, 0u};
            if (r < limit) v[p] = *reinterpret_cast<const u32x4 *>(base + (size_t)r * pitch + seg * 16);
        }
    }
    __device__ __forceinline__ void store(unsigned char *lds) const {
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
            const int i = (int)threadIdx.x + p * THREADS;
            *reinterpret_cast<u32x4 *>(lds + (i / (D / 8)) * kPitch<D> + (i % (D / 8)) * 16) = v[p];
        }
    }
};

// Operand of a 32 x 32 x 16 product out of LDS: row `row` + lane % 32, channels 16 step + 8 (lane / 32) ..
template <int D>
__device__ __forceinline__ bf16x8 rows_of(const unsigned char *tile, int row, int step) {
    const int lane = threadIdx.x & 63;
    return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(tile + (row + (lane & 31)) * kPitch<D> + step * 32 + (lane >> 5) * 16));
}
// The same of the transposed tile: channel 32 block + lane % 32, and the eight rows row + 4 (lane / 32) + {0 .. 3, 8 .. 11}: the rows that a lane's eight
// accumulators of one 32 x 32 product stand for.  ds_read_b64_tr_b16: within 16 lanes, lane j points at row j / 4 and columns 4 (j % 4) .. of a 4 x 16 block and
// receives column j of its four rows.
template <int D>
__device__ __forceinline__ bf16x8 columns_of(const unsigned char *tile, int row, int block) {
    typedef s16x4 __attribute__((address_space(3))) * lds_ptr;
    const int lane = threadIdx.x & 63;
    const unsigned char *p = tile + (row + 4 * (lane >> 5) + ((lane & 15) >> 2)) * kPitch<D> + (32 * block + 16 * ((lane >> 4) & 1) + 4 * (lane & 3)) * 2;
    const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p));
    const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p + 8 * kPitch<D>));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Accumulators 8 j .. 8 j + 7 of a 32 x 32 product, rounded to bf16, as an operand whose reduction runs over the product's rows.
__device__ __forceinline__ bf16x8 as_operand(const f32x16 &s, int j) {
    const u32x4 v = {rows::pack2(s[8 * j], s[8 * j + 1]), rows::pack2(s[8 * j + 2], s[8 * j + 3]), rows::pack2(s[8 * j + 4], s[8 * j + 5]),
                     rows::pack2(s[8 * j + 6], s[8 * j + 7])};
    return __builtin_bit_cast(bf16x8, v);
}
// Row of a 32 x 32 product that accumulator e stands for, in lanes 0 .. 31 (4 more in the others).
__device__ __forceinline__ constexpr int row_of(int e) { return 8 * (e >> 2) + (e & 3); }

__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ float halves_max(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// A lane's column of a transposed product over BLOCKS * 32 channels, times `by`, as bf16 to `out` (channels 32 block + row_of + 4 half).
template <int BLOCKS>
__device__ __forceinline__ void store_column(unsigned char *out, const f32x16 (&o)[BLOCKS], float by) {
    const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int t = 0; t < BLOCKS; ++t)
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
            uint2 w;
            w.x = rows::pack2(o[t][4 * e4 + 0] * by, o[t][4 * e4 + 1] * by);
            w.y = rows::pack2(o[t][4 * e4 + 2] * by, o[t][4 * e4 + 3] * by);
            *reinterpret_cast<uint2 *>(out + (32 * t + 8 * e4 + 4 * half) * 2) = w;
        }
}

// Zeros to `n` rows of `bytes` (a multiple of 16) each.
__device__ __forceinline__ void zero_rows(unsigned char *p, size_t pitch, int n, int bytes) {
    const int per = bytes / 16;
    for (int i = threadIdx.x; i < n * per; i += blockDim.x) *reinterpret_cast<u32x4 *>(p + (size_t)(i / per) * pitch + (i % per) * 16) = u32x4{0u, 0u, 0u, 0u};
}

}  // namespace pat
}  // namespace delta
