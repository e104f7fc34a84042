// Weight gradient of a linear layer (1x1, stride 1, bf16) whose input is held as an 8-bit checkpoint (packed.hpp), for gfx950:
//   gw[k,c] = scale_k * sum_m gpre[m,k] * x[m,c],   x[m,c] = q[m,c] * 2^e[m, c / 32]
// The product, its tiles, the swizzle of the LDS rows and the partial sums are wgrad1x1.hip's, whose reduction kernel finishes it: a workgroup of 8
// wavefronts owns 64 KT x 64 CT of (k, c) and is persistent over slices of pixels.  x is exact in bf16, so the sums are of the same products as after
// DELTA_OP_UNPACK8, whose tensor (2 bytes a value written and read again) is not needed.
//  * gpre, the bytes of x and its scale bytes go from memory straight into LDS through a ring of S slices of 128 pixels (64 beside four k tiles), 48 KB a
//    slice of 128 x 128 where bf16 needs 64; one barrier a slice.
//  * x stays in 8 bits as far as the registers: gfx950's transposing read of bytes (ds_read_b64_tr_b8: 16 lanes point at 8 rows of 16 channels, each
//    gets one channel's 8 values along the rows) gives a lane the 8 pixels of one MFMA operand, which it converts, two values and their two scales with
//    7 instructions in int8, 6 in E4M3: 28 and 24 for 8 values.  A wavefront owns 128 x 64 of (k, c) where K allows, so that a step is 8 MFMAs (256
//    cycles) beside the next step's 56 conversions (224).  The first step of a slice is converted before its first product, with nothing beside it: with two
//    steps a slice (128 x 128) that is half of all conversions, with one (64 channels of x) all.  The pixels' scales are turned into bf16 once a slice,
//    a slice ahead, and read by whole wavefronts at once (in fp32 these reads were half of all LDS reads).
//    With x converted by the whole workgroup into a bf16 tile a slice ahead instead, and 64 x 64 to a wavefront, a slice's steps waited for one
//    another: 43 us for 768 -> 768 on 16384 tokens.
//  * Workgroups are numbered so that those of one split, which read the same pixels, are on one XCD and share its L2: a third of the misses.
//  * The wavefronts that share a tile add their sums through LDS, in a fixed tree.
// us, and the reduction's beside them: 768 -> 768 on 16384 tokens, int8, 35 + 5.4 (550 TFLOP/s; E4M3 33; wgrad1x1.hip on the unpacked tensor 40 + 5.5), on 333
// tokens 1024 -> 256 9 + 3.4.  Bound by neither memory (38 MB, 6 us) nor the matrix units (8) alone: a slice's waits, LDS reads, and the conversions that
// stand before the products or between them.
// Rows past the last pixel are fetched from the last pixel and overwritten with zeros in LDS; their scales are zeros.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.hpp"
#include "packed.hpp"
#include "rows.hpp"

namespace delta {
namespace wgp {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));

struct Args {
    const unsigned char *x, *g;     // checkpoint of [M,C]; [M,K] bf16
    float *partial;                 // as wgrad1x1_kernel's
    uint64_t scales;                // byte offset of the scale bytes in x
    int M, C, K, nslices, nsplit;
};

template <int KT, int CT> struct Shape {
    static constexpr int kF = KT == 1 ? 2 : 4;                                                   // 32-channel pieces of k that a wavefront owns; of c: 2
    static constexpr int kAlong = KT * 2 / kF, kTiles = kAlong * CT, kQS = 8 / kTiles;           // wavefronts along k; wavefront tiles; wavefronts on each
    static constexpr int kPixels = KT == 4 ? 64 : 128;                                           // of a slice
    static constexpr int kG = kPixels * KT * 128, kX = kPixels * CT * 64;                        // bytes of a slice: gpre, bytes of x
    static constexpr int kScaleWords = CT == 4 ? 2 : 1, kScales = kPixels * kScaleWords * 4;     // 4-byte words of scale bytes a pixel
    static constexpr int kSlice = kG + kX + kScales, kMade = CT * 2 * kPixels * 2;               // of the ring; of a slice's scales in bf16
    static constexpr int kFit = (160 * 1024 - 2 * kMade) / kSlice, kStages = kFit < 5 ? kFit : 5;
    static constexpr int kGL = kG / 8192, kXB = kX / 1024, kXL = kXB < 8 ? 1 : kXB / 8;          // loads per wavefront; 1 KB blocks of x
    static constexpr int kSB = kScales / 256, kLoads = kGL + kXL + 1;                            // 256-byte blocks of scales
    static constexpr int kSums = kQS / 2 * kTiles * kF * 8192;
    static constexpr int kRing = kStages * kSlice + 2 * kMade, kLds = kRing > kSums ? kRing : kSums;
    static_assert(kStages >= 3 && kLds <= 160 * 1024, "one slice multiplied, two in flight");
};

// Which way the 64-byte groups of a row of gpre in LDS are permuted (wgrad1x1.hip says why), and the 16-byte segments of a row of x: the eight rows that a
// transposing read touches at one segment lie in eight different sixteenths of the 64 banks (rows of 64, 128 and 256 bytes lie four, two and one to
// a 256-byte line).
template <int TW>
__device__ __forceinline__ int swizzle(int row) { return TW == 1 ? (row >> 1) & 1 : row & 3; }
template <int CT>
__device__ __forceinline__ int swizzle8(int row) { return CT == 1 ? (row >> 2) & 1 : CT == 2 ? (row >> 1) & 3 : row & 7; }

template <int KT, int CT, int FMT>
__global__ __launch_bounds__(512) void wgrad1x1_packed_kernel(Args a) {
    using T = Shape<KT, CT>;
    constexpr int GP = KT * 128, XP = CT * 64, S = T::kStages, QS = T::kQS, F = T::kF;
    extern __shared__ __align__(16) unsigned char smem[];
    uint16_t *const made = reinterpret_cast<uint16_t *>(smem + S * T::kSlice);   // [2][CT * 2 blocks][kPixels]
    const int tid = threadIdx.x, lane = tid & 63;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int base = wv % T::kTiles, qs = wv / T::kTiles, kw = base % T::kAlong, cw = base / T::kAlong;
    // Workgroups go round the 8 XCDs in order of their number; numbered anew, each XCD's are neighbours.
    const int xcd = blockIdx.x & 7, whole = (int)gridDim.x >> 3, rest = (int)gridDim.x & 7;
    const int number = xcd * whole + (xcd < rest ? xcd : rest) + ((int)blockIdx.x >> 3), ntiles = (int)gridDim.x / a.nsplit;
    const int split = number / ntiles, tile = number % ntiles;
    const int ktiles = a.K / (64 * KT), kt = tile % ktiles, ct = tile / ktiles;
    const uint32_t nb = (uint32_t)a.C / 32;

    // ---- direct loads: the direct load fixes where a lane's 16 bytes land, so the permutations are applied to the address each lane fetches
    // (row, byte) of a lane's part of a slice, and its offset in the tensor for the slice that is fetched next
    int grow[T::kGL], xrow[T::kXL];
    uint32_t gseg[T::kGL], xseg[T::kXL], xlds[T::kXL];
#pragma unroll
    for (int i = 0; i < T::kGL; ++i) {
        const int b = (wv * T::kGL + i) * 1024 + lane * 16, s = (b % GP) >> 4;
        grow[i] = b / GP;
        gseg[i] = (uint32_t)(kt * GP + (((s >> 2) ^ swizzle<KT>(grow[i])) << 6) + (s & 3) * 16);
    }
#pragma unroll
    for (int i = 0; i < T::kXL; ++i) {
        const int blk = T::kXB < 8 ? wv % T::kXB : wv * T::kXL + i, b = blk * 1024 + lane * 16;      // fewer blocks than wavefronts: some bring one twice
        xlds[i] = (uint32_t)blk * 1024;
        xrow[i] = b / XP;
        xseg[i] = (uint32_t)(ct * XP + ((((b % XP) >> 4) ^ swizzle8<CT>(xrow[i])) << 4));
    }
    const int sblk = wv % T::kSB, sword = sblk * 64 + lane, spixel = sword / T::kScaleWords;
    typedef __attribute__((address_space(3))) unsigned char *lptr_t;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lptr_t)smem;
    uint32_t gat[T::kGL], xat[T::kXL];
    uint64_t sat;
    // Where the rows of a slice lie, rows past the last pixel where that pixel's do.  For CT = 1 a pixel's first scale byte is in one of its word's halves.
    auto place = [&](int slice) {
        const int m0 = slice * T::kPixels, last = a.M - 1 - m0;
#pragma unroll
        for (int i = 0; i < T::kGL; ++i) gat[i] = (uint32_t)(m0 + (grow[i] < last ? grow[i] : last)) * (uint32_t)a.K * 2u + gseg[i];
#pragma unroll
        for (int i = 0; i < T::kXL; ++i) xat[i] = (uint32_t)(m0 + (xrow[i] < last ? xrow[i] : last)) * (uint32_t)a.C + xseg[i];
        sat = (uint64_t)(uint32_t)(m0 + (spixel < last ? spixel : last)) * nb + (uint32_t)(ct * CT * 2);
    };
    // Fetches slice `slice`, `nsplit` behind the one before; only the last slice of all has rows past the last pixel.
    const uint32_t gstep = (uint32_t)a.nsplit * T::kPixels * (uint32_t)a.K * 2u, xstep = (uint32_t)a.nsplit * T::kPixels * (uint32_t)a.C;
    const uint64_t sstep = (uint64_t)a.nsplit * T::kPixels * nb;
    auto fetch = [&](int slice, int buf) {
        if ((slice + 1) * (long long)T::kPixels > a.M) place(slice);
        const uint32_t sb = lds0 + (uint32_t)(buf * T::kSlice);
        load_lds_b32(a.x + a.scales + (sat & ~(uint64_t)3) + (sword % T::kScaleWords) * 4, sb + T::kG + T::kX + (uint32_t)sblk * 256);
        sat += sstep;
#pragma unroll
        for (int i = 0; i < T::kGL; ++i) {
            load_lds_b128(a.g, gat[i], sb + (uint32_t)(wv * T::kGL + i) * 1024);
            gat[i] += gstep;
        }
#pragma unroll
        for (int i = 0; i < T::kXL; ++i) {
            load_lds_b128(a.x, xat[i], sb + T::kG + xlds[i]);
            xat[i] += xstep;
        }
    };
    // Direct loads complete in order, and a slice's scales are its first: all but the last `later` slices' loads and the rest of the one before those have
    // landed (later < 0: all).
    auto wait_scales = [&](int later) {
        if (later < 0) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        else if (later == 0) asm volatile("s_waitcnt vmcnt(%0)" :: "n"(T::kLoads - 1) : "memory");
        else if (later == 1) asm volatile("s_waitcnt vmcnt(%0)" :: "n"(2 * T::kLoads - 1) : "memory");
        else asm volatile("s_waitcnt vmcnt(%0)" :: "n"(3 * T::kLoads - 1) : "memory");
    };
    // the scales of a slice in the ring, in bf16 (a power of two, or NaN), [block][pixel]
    auto scales = [&](int slice, int buf, uint16_t *out) {
        const int last = a.M - 1 - slice * T::kPixels;
        const unsigned char *raw = smem + buf * T::kSlice + T::kG + T::kX;
#pragma unroll
        for (int i = 0; i < (T::kMade / 2 + 511) / 512; ++i) {
            const int p = (tid + i * 512) % (T::kMade / 2), block = p / T::kPixels, pixel = p % T::kPixels;      // fewer scales than threads: some make one twice
            uint32_t at = (uint32_t)block;
            if constexpr (CT == 1) at += (uint32_t)(((uint64_t)(uint32_t)(slice * T::kPixels + (pixel < last ? pixel : last)) * nb + (uint32_t)(ct * 2)) & 3);
            const uint32_t byte = raw[pixel * (T::kScaleWords * 4) + at];
            out[p] = (uint16_t)(pixel <= last ? (byte == 255u ? 0x7FC0u : byte << 7) : 0u);
        }
    };

    // ---- transposing reads.  gpre as in wgrad1x1.hip: a lane supplies row 8 (lane / 32) + (lane % 16) / 4 (+ 4) of a 16-pixel step and channels
    // 16 ((lane / 16) % 2) + 4 (lane % 4) .. + 3 of a 32-channel piece; x: row 8 (lane / 32) + (lane % 16) / 2 and channels
    // 16 ((lane / 16) % 2) + 8 (lane % 2) .. + 7.  Adding multiples of 16 to the row keeps the permutations.
    const int srow = 8 * (lane >> 5) + ((lane & 15) >> 2), scol = 32 * ((lane >> 4) & 1) + 8 * (lane & 3);
    const int xsrow = 8 * (lane >> 5) + ((lane & 15) >> 1);
    int goff[F], xoff[2];
#pragma unroll
    for (int f = 0; f < F; ++f) goff[f] = srow * GP + (((kw * F + f) ^ swizzle<KT>(srow)) << 6) + scol;
#pragma unroll
    for (int h = 0; h < 2; ++h)
        xoff[h] = T::kG + xsrow * XP + (((cw * 4 + h * 2 + ((lane >> 4) & 1)) ^ swizzle8<CT>(xsrow)) << 4) + 8 * (lane & 1);
    typedef s16x4 __attribute__((address_space(3))) * lds_ptr;
    typedef i32x2 __attribute__((address_space(3))) * lds_ptr8;
    auto tr_read = [&](const unsigned char *p) { return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p)); };
    auto tr_read8 = [&](const unsigned char *p) { return __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_ptr8)(p)); };

    f32x16 acc[F][2];
#pragma unroll
    for (int i = 0; i < F; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

    const int mine = (a.nslices - split + a.nsplit - 1) / a.nsplit;        // at least 1: nsplit <= nslices
    auto slice_of = [&](int t) { return split + t * a.nsplit; };
    place(slice_of(0));
#pragma unroll
    for (int t = 0; t < S - 1; ++t)
        if (t < mine) fetch(slice_of(t), t);
    wait_scales(mine - 1 < S - 2 ? mine - 1 : S - 2);            // those of slice 0
    __syncthreads();
    scales(slice_of(0), 0, made);
    for (int t = 0, buf = 0; t < mine; ++t) {
        const int later = mine - 2 - t < S - 3 ? mine - 2 - t : S - 3;
        wait_scales(later);                                      // this wavefront's part of slice t and its scales of slice t + 1 have landed
        __syncthreads();                                         // everyone's have; the scales of slice t are converted; the buffers of slice t - 1 are free
        const int nbuf = buf == 0 ? S - 1 : buf - 1, next = buf + 1 == S ? 0 : buf + 1;
        if (t + S - 1 < mine) fetch(slice_of(t + S - 1), nbuf);
        unsigned char *sl = smem + buf * T::kSlice;
        const int valid = a.M - slice_of(t) * T::kPixels;
        if (valid < T::kPixels) {                                // the last slice of all: rows past the last pixel
            for (int i = tid; i < (T::kG + T::kX) / 16; i += 512) {
                const int row = i * 16 < T::kG ? i * 16 / GP : (i * 16 - T::kG) / XP;
                if (row >= valid) *reinterpret_cast<u32x4 *>(sl + i * 16) = u32x4{0u, 0u, 0u, 0u};
            }
            __syncthreads();
        }
        const uint16_t *sc = made + (t & 1) * (T::kMade / 2) + cw * 2 * T::kPixels + 8 * (lane >> 5);
        // Step by step: all reads of a step first, then, pair by pair between two MFMAs of the step before (32 cycles, room for eight other instructions),
        // its conversions.  The compiler is held to this order, or it converts a whole step before it multiplies.
        constexpr int kSteps = T::kPixels / (16 * QS);
        s16x8 af[2][F];
        u32x4 bf[2][2];
        i32x2 raw[2];
        u32x4 sv[2];
        auto read = [&](int q, int to) {
            const int q0 = 16 * (qs + q * QS);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                raw[h] = tr_read8(sl + q0 * XP + xoff[h]);
                sv[h] = *reinterpret_cast<const u32x4 *>(sc + h * T::kPixels + q0);
            }
#pragma unroll
            for (int f = 0; f < F; ++f)
                af[to][f] = __builtin_shufflevector(tr_read(sl + q0 * GP + goff[f]), tr_read(sl + (q0 + 4) * GP + goff[f]), 0, 1, 2, 3, 4, 5, 6, 7);
        };
        auto pair = [&](int p, int to) {                         // of eight: values 2 (p % 4) and the next of piece p / 4
            const int h = p >> 2, e = p & 3;
            float x[2];
            packed::decode2<FMT>((uint32_t)(e & 2 ? raw[h].y : raw[h].x), e & 1, __uint_as_float(sv[h][e] << 16), __uint_as_float(sv[h][e] & 0xFFFF0000u), x);
            bf[to][h][e] = rows::pack2(x[0], x[1]);
        };
        read(0, 0);
#pragma unroll
        for (int p = 0; p < 8; ++p) pair(p, 0);
#pragma unroll
        for (int q = 0; q < kSteps; ++q) {
            if (q + 1 < kSteps) read(q + 1, (q + 1) & 1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < 2 * F; ++i) {
                acc[i % F][i / F] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, af[q & 1][i % F]), __builtin_bit_cast(bf16x8, bf[q & 1][i / F]),
                                                                            acc[i % F][i / F], 0, 0, 0);
                if (q + 1 < kSteps) {
#pragma unroll
                    for (int p = i * 4 / F; p < (i + 1) * 4 / F; ++p) pair(p, (q + 1) & 1);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        // behind the last slice: of a buffer that nothing reads any more
        scales(slice_of(t + 1), next, made + ((t + 1) & 1) * (T::kMade / 2));
        buf = next;
    }

    // ---- the QS sums of a tile: the upper half of the wavefronts on it hands its sums to the lower half, until one is left
    if constexpr (QS > 1) {
#pragma unroll
        for (int n = QS / 2; n; n /= 2) {
            __syncthreads();                                     // the ring is dead, or the sums before are read
            f32x4 *red = reinterpret_cast<f32x4 *>(smem) + lane; // [n][wavefront tiles][F][2][4][64]
            if (qs >= n && qs < 2 * n) {
#pragma unroll
                for (int k = 0; k < F * 8; ++k) {
                    const f32x16 &v = acc[k >> 3][(k >> 2) & 1];
                    red[((qs - n) * T::kTiles + base) * (F * 512) + k * 64] = f32x4{v[4 * (k & 3)], v[4 * (k & 3) + 1], v[4 * (k & 3) + 2], v[4 * (k & 3) + 3]};
                }
            }
            __syncthreads();
            if (qs < n) {
#pragma unroll
                for (int k = 0; k < F * 8; ++k) {
                    const f32x4 v = red[(qs * T::kTiles + base) * (F * 512) + k * 64];
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[k >> 3][(k >> 2) & 1][4 * (k & 3) + e] += v[e];
                }
            }
        }
        if (qs) return;
    }
#pragma unroll
    for (int k = 0; k < F * 8; ++k) {
        const int piece = kw * F + (k >> 3);                     // of the workgroup's 2 KT along k: two to a 64 x 64 tile
        const f32x16 &v = acc[k >> 3][(k >> 2) & 1];
        f32x4 *out = reinterpret_cast<f32x4 *>(a.partial) + (((size_t)split * ntiles + tile) * (KT * CT) + cw * KT + (piece >> 1)) * 1024 +
                     (((piece & 1) * 2 + ((k >> 2) & 1)) * 4 + (k & 3)) * 64 + lane;
        *out = f32x4{v[4 * (k & 3)], v[4 * (k & 3) + 1], v[4 * (k & 3) + 2], v[4 * (k & 3) + 3]};
    }
}

// A workgroup's time per pixel, and what one more split of a 128 x 128 tile costs: wgrad1x1.hip's, taken over as they are, not measured for this kernel.
static constexpr double kPixelNs = 5.5, kSumsNs = 24.;

struct Plan { int kt, ct, tiles, nslices, nsplit; };

const char *plan_for(const ConvArgs &a, Plan &p) {
    if (!a.bf16 || a.R != 1 || a.S != 1 || a.pad != 0 || a.stride != 1) return "weight gradient from a checkpoint: linear layers (1x1, stride 1), bf16";
    if (a.Cin % 64 || a.Cout % 64) return "weight gradient: channel counts must be multiples of 64";
    if ((unsigned long long)a.M * a.Cin * 2ull >= 0x7FFFFFFFull || (unsigned long long)a.M * a.Cout * 2ull >= 0x7FFFFFFFull)
        return "weight gradient: tensors of 2 GiB or more";
    p.kt = a.Cout % 128 == 0 ? 2 : 1;                            // as wgrad1x1.hip's
    p.ct = a.Cin % 128 == 0 ? 2 : 1;
    if (p.kt == 2 && p.ct == 1 && a.Cout % 256 == 0) p.kt = 4;
    if (p.ct == 2 && p.kt == 1 && a.Cin % 256 == 0) p.ct = 4;
    p.tiles = (a.Cout / (64 * p.kt)) * (a.Cin / (64 * p.ct));
    const int pixels = p.kt == 4 ? 64 : 128;
    p.nslices = (a.M + pixels - 1) / pixels;
    p.nsplit = wgrad_splits(a.M, p.tiles, kPixelNs, kSumsNs * p.kt * p.ct / 4);
    if (p.nsplit > p.nslices) p.nsplit = p.nslices;
    return nullptr;
}

template <int KT, int CT, int FMT>
hipError_t launch(const Args &w, const Plan &p, hipStream_t stream) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&wgrad1x1_packed_kernel<KT, CT, FMT>),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, Shape<KT, CT>::kLds);
    if (e != hipSuccess) return e;
    wgrad1x1_packed_kernel<KT, CT, FMT><<<dim3(p.nsplit * p.tiles), dim3(512), Shape<KT, CT>::kLds, stream>>>(w);
    return hipGetLastError();
}
template <int KT, int CT>
hipError_t launch(const Args &w, const Plan &p, int fmt, hipStream_t stream) {
    return fmt == PACK_INT8 ? launch<KT, CT, PACK_INT8>(w, p, stream) : launch<KT, CT, PACK_E4M3>(w, p, stream);
}

}  // namespace wgp

const char *wgrad1x1_packed_check(const ConvArgs &a) {
    wgp::Plan p;
    return wgp::plan_for(a, p);
}

size_t wgrad1x1_packed_workspace_bytes(const ConvArgs &a) {
    wgp::Plan p;
    return wgp::plan_for(a, p) ? 0 : (size_t)p.nsplit * p.tiles * p.kt * p.ct * 16384;
}

// As launch_wgrad1x1, with a.x the checkpoint of [M, Cin].
hipError_t launch_wgrad1x1_packed(const ConvArgs &a, int fmt, const void *g, float *gw, void *workspace, size_t workspace_bytes, hipStream_t stream) {
    wgp::Plan p;
    if (wgp::plan_for(a, p) || (fmt != PACK_INT8 && fmt != PACK_E4M3) || !g || !gw || !workspace || !a.x || !a.scale ||
        workspace_bytes < wgrad1x1_packed_workspace_bytes(a) || ((uintptr_t)workspace | (uintptr_t)g | (uintptr_t)a.x) & 15)
        return hipErrorInvalidValue;
    wgp::Args w;
    w.x = static_cast<const unsigned char *>(a.x); w.g = static_cast<const unsigned char *>(g);
    w.partial = static_cast<float *>(workspace);
    w.scales = packed_scale_offset((uint64_t)a.M, (uint64_t)a.Cin);
    w.M = a.M; w.C = a.Cin; w.K = a.Cout; w.nslices = p.nslices; w.nsplit = p.nsplit;
    hipError_t e;
    switch (p.kt * 10 + p.ct) {
    case 11: e = wgp::launch<1, 1>(w, p, fmt, stream); break;
    case 12: e = wgp::launch<1, 2>(w, p, fmt, stream); break;
    case 14: e = wgp::launch<1, 4>(w, p, fmt, stream); break;
    case 21: e = wgp::launch<2, 1>(w, p, fmt, stream); break;
    case 22: e = wgp::launch<2, 2>(w, p, fmt, stream); break;
    case 41: e = wgp::launch<4, 1>(w, p, fmt, stream); break;
    default: return hipErrorInvalidValue;
    }
    if (e != hipSuccess) return e;
    return launch_wgrad1x1_reduce(w.partial, a.scale, gw, a.Cout, a.Cin, p.kt, p.ct, p.nsplit, stream);
}

}  // namespace delta
