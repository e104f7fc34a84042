// Weight gradient of a linear layer (1x1, stride 1, bf16) whose input is held as an 8-bit checkpoint (packed.hpp), for gfx950:
//   gw[k,c] = scale_k * sum_m gpre[m,k] * x[m,c],   x[m,c] = q[m,c] * 2^e[m, c / 32]
// The product, its tiles, the swizzle of the LDS rows and the partial sums are wgrad1x1.hip's, whose reduction kernel finishes it: a workgroup of 8
// wavefronts owns 64 KT x 64 CT of (k, c) and is persistent over slices of pixels.  x is exact in bf16, so the sums are of the same products as after
// DELTA_OP_UNPACK8, whose tensor (2 bytes a value written and read again) is not needed.
//  * gpre, the bytes of x and its scale bytes go from memory straight into LDS through a ring of S slices, S - 2 of them in flight beside the one
//    multiplied and the one converted: 24 KB a slice of 128 x 128, where bf16 needs 32.
//  * A slice's x is converted into a bf16 tile (two of them in turn) while the slice before is multiplied: one barrier a slice.  16 values a
//    thread: 1 conversion, 1 product and 1/2 packing each.
// Rows past the last pixel are fetched from the last pixel; those of gpre are overwritten with zeros in LDS, those of x converted to zeros.
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
using packed::u32x2;

struct Args {
    const unsigned char *x, *g;     // checkpoint of [M,C]; [M,K] bf16
    float *partial;                 // as wgrad1x1_kernel's
    uint64_t scales;                // byte offset of the scale bytes in x
    int M, C, K, nslices, nsplit;
};

template <int KT, int CT> struct Shape {
    static constexpr int kTiles = KT * CT, kQS = 8 / kTiles, kPixels = kTiles == 1 ? 128 : 64;   // of a slice
    static constexpr int kG = kPixels * KT * 128, kX = kPixels * CT * 64;                        // bytes of a slice: gpre, bytes of x
    static constexpr int kScaleWords = CT == 4 ? 2 : 1, kScales = kPixels * kScaleWords * 4;     // 4-byte words of scale bytes a pixel
    static constexpr int kSlice = kG + kX + kScales, kTile = kPixels * CT * 128;                 // of the ring; of a converted tile
    static constexpr int kFit = (160 * 1024 - 2 * kTile) / kSlice, kStages = kFit < 5 ? kFit : 5;
    static constexpr int kGL = kG / 8192, kXB = kX / 1024, kXL = kXB < 8 ? 1 : kXB / 8;          // loads per wavefront; 1 KB blocks of x
    static constexpr int kSB = kScales / 256, kLoads = kGL + kXL + 1;                            // 256-byte blocks of scales
    static constexpr int kSums = (kQS - 1) * kTiles * 16384;
    static constexpr int kRing = kStages * kSlice + 2 * kTile, kLds = kRing > kSums ? kRing : kSums;
    static_assert(kStages >= 3, "one slice multiplied, one converted, one in flight");
};

template <int TW>
__device__ __forceinline__ int swizzle(int row) { return TW == 1 ? (row >> 1) & 1 : row & 3; }       // wgrad1x1.hip says why

template <int KT, int CT, int FMT>
__global__ __launch_bounds__(512) void wgrad1x1_packed_kernel(Args a) {
    using T = Shape<KT, CT>;
    constexpr int GP = KT * 128, XP = CT * 128, S = T::kStages, QS = T::kQS;
    extern __shared__ __align__(16) unsigned char smem[];
    unsigned char *const tiles = smem + S * T::kSlice;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int base = wv % T::kTiles, qs = wv / T::kTiles, kw = base % KT, cw = base / KT;
    const int ktiles = a.K / (64 * KT), kt = blockIdx.y % ktiles, ct = blockIdx.y / ktiles;
    const uint32_t nb = (uint32_t)a.C / 32;

    // ---- direct loads.  gpre: LDS slot s of row r holds segment s with its 64-byte group permuted; x and its scales as they lie.
    int grow[T::kGL], xrow[T::kXL];
    uint32_t gseg[T::kGL], xat[T::kXL], xlds[T::kXL];
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
        xrow[i] = b / (CT * 64);
        xat[i] = (uint32_t)(ct * CT * 64 + b % (CT * 64));
    }
    const int sblk = wv % T::kSB, sword = sblk * 64 + lane, srow_ = sword / T::kScaleWords;
    typedef __attribute__((address_space(3))) unsigned char *lptr_t;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lptr_t)smem;
    auto fetch = [&](int slice, int buf) {
        const int m0 = slice * T::kPixels, last = a.M - 1 - m0;  // rows past the last pixel: that pixel
        const uint32_t sb = lds0 + (uint32_t)(buf * T::kSlice);
#pragma unroll
        for (int i = 0; i < T::kGL; ++i) {
            const int row = grow[i] < last ? grow[i] : last;
            load_lds_b128(a.g, (uint32_t)(m0 + row) * (uint32_t)a.K * 2u + gseg[i], sb + (uint32_t)(wv * T::kGL + i) * 1024);
        }
#pragma unroll
        for (int i = 0; i < T::kXL; ++i) {
            const int row = xrow[i] < last ? xrow[i] : last;
            load_lds_b128(a.x, (uint32_t)(m0 + row) * (uint32_t)a.C + xat[i], sb + T::kG + xlds[i]);
        }
        // the word that holds the pixel's first scale byte of this tile (CT = 1: in one of its halves)
        const int row = srow_ < last ? srow_ : last;
        const uint64_t at = (uint64_t)(m0 + row) * nb + (uint32_t)(ct * CT * 2);
        load_lds_b32(a.x + a.scales + (at & ~(uint64_t)3) + (sword % T::kScaleWords) * 4, sb + T::kG + T::kX + (uint32_t)sblk * 256);
    };
    // direct loads complete in order: "at most n later slices outstanding" is vmcnt(n * loads per slice)
    auto wait_slices = [&](int later) {
        if (later <= 0) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        else if (later == 1) asm volatile("s_waitcnt vmcnt(%0)" :: "n"(T::kLoads) : "memory");
        else asm volatile("s_waitcnt vmcnt(%0)" :: "n"(2 * T::kLoads) : "memory");
    };
    // x of a slice in the ring into a bf16 tile: 16 channels of a row are 32 neighbouring bytes of it
    auto convert = [&](int slice, int buf, unsigned char *tile) {
        constexpr int kPieces = T::kX / 16;
        const unsigned char *raw = smem + buf * T::kSlice + T::kG;
        const int valid = a.M - slice * T::kPixels;
#pragma unroll
        for (int i = 0; i < (kPieces + 511) / 512; ++i) {
            const int p = tid + i * 512, row = p / (CT * 4), s16 = p % (CT * 4);
            if (kPieces < 512 && p >= kPieces) break;
            const u32x4 q = *reinterpret_cast<const u32x4 *>(raw + p * 16);
            uint32_t at = (uint32_t)(s16 >> 1);
            if constexpr (CT == 1) {
                const int m = row < valid ? row : valid - 1;
                at += (uint32_t)(((uint64_t)(slice * T::kPixels + m) * nb + (uint32_t)(ct * 2)) & 3);
            }
            const float s = packed::scale_of(raw[T::kX + row * (T::kScaleWords * 4) + at]);
            float v[16];
#pragma unroll
            for (int w = 0; w < 4; ++w) packed::decode4<FMT>(q[w], s, v + 4 * w);
            u32x4 o[2];
#pragma unroll
            for (int w = 0; w < 8; ++w) o[w >> 2][w & 3] = row < valid ? rows::pack2(v[2 * w], v[2 * w + 1]) : 0u;
            u32x4 *to = reinterpret_cast<u32x4 *>(tile + row * XP + (((s16 >> 1) ^ swizzle<CT>(row)) << 6) + (s16 & 1) * 32);
            to[0] = o[0];
            to[1] = o[1];
        }
    };

    // ---- transposing reads, as in wgrad1x1.hip
    const int srow = 8 * (lane >> 5) + ((lane & 15) >> 2), scol = 32 * ((lane >> 4) & 1) + 8 * (lane & 3);
    int goff[2], xoff[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        goff[t] = srow * GP + (((kw * 2 + t) ^ swizzle<KT>(srow)) << 6) + scol;
        xoff[t] = srow * XP + (((cw * 2 + t) ^ swizzle<CT>(srow)) << 6) + scol;
    }
    typedef s16x4 __attribute__((address_space(3))) * lds_ptr;
    auto tr_read = [&](const unsigned char *p) { return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p)); };

    f32x16 acc[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

    const int mine = (a.nslices - (int)blockIdx.x + a.nsplit - 1) / a.nsplit;        // at least 1: nsplit <= nslices
    auto slice_of = [&](int t) { return (int)blockIdx.x + t * a.nsplit; };
#pragma unroll
    for (int t = 0; t < S - 1; ++t)
        if (t < mine) fetch(slice_of(t), t);
    wait_slices(mine - 1 < S - 2 ? mine - 1 : S - 2);            // slices 1 .. S - 2 may be outstanding; waits for more where S is 5
    __syncthreads();
    convert(slice_of(0), 0, tiles);
    for (int t = 0, buf = 0; t < mine; ++t) {
        const int later = mine - 2 - t < S - 3 ? mine - 2 - t : S - 3;
        wait_slices(later);                                      // this wavefront's part of slice t + 1 has landed
        __syncthreads();                                         // everyone's has; x of slice t is converted; the buffers of slice t - 1 are free
        const int nbuf = buf == 0 ? S - 1 : buf - 1, next = buf + 1 == S ? 0 : buf + 1;
        if (t + S - 1 < mine) fetch(slice_of(t + S - 1), nbuf);
        unsigned char *sl = smem + buf * T::kSlice;
        const unsigned char *xt = tiles + (t & 1) * T::kTile;
        const int valid = a.M - slice_of(t) * T::kPixels;
        if (valid < T::kPixels) {                                // the last slice of all: rows of gpre past the last pixel
            for (int i = tid; i < T::kG / 16; i += 512)
                if (i * 16 / GP >= valid) *reinterpret_cast<u32x4 *>(sl + i * 16) = u32x4{0u, 0u, 0u, 0u};
            __syncthreads();
        }
        if (t + 1 < mine) convert(slice_of(t + 1), next, tiles + ((t + 1) & 1) * T::kTile);
#pragma unroll
        for (int q = 0; q < T::kPixels / (16 * QS); ++q) {
            const int q0 = 16 * (qs + q * QS);
            s16x8 af[2], bf[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                af[h] = __builtin_shufflevector(tr_read(sl + q0 * GP + goff[h]), tr_read(sl + (q0 + 4) * GP + goff[h]), 0, 1, 2, 3, 4, 5, 6, 7);
                bf[h] = __builtin_shufflevector(tr_read(xt + q0 * XP + xoff[h]), tr_read(xt + (q0 + 4) * XP + xoff[h]), 0, 1, 2, 3, 4, 5, 6, 7);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, af[i]), __builtin_bit_cast(bf16x8, bf[j]),
                                                                        acc[i][j], 0, 0, 0);
        }
        buf = next;
    }

    // ---- the QS sums of a tile, added in the order of qs
    f32x4 sum[16];                                               // [i][j][e4]
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        const f32x16 &v = acc[k >> 3][(k >> 2) & 1];
        sum[k] = f32x4{v[4 * (k & 3)], v[4 * (k & 3) + 1], v[4 * (k & 3) + 2], v[4 * (k & 3) + 3]};
    }
    if constexpr (QS > 1) {
        __syncthreads();                                         // the ring and the tiles are dead
        f32x4 *red = reinterpret_cast<f32x4 *>(smem) + lane;     // [QS - 1][tiles][16][64]
        if (qs) {
#pragma unroll
            for (int k = 0; k < 16; ++k) red[((qs - 1) * T::kTiles + base) * 1024 + k * 64] = sum[k];
        }
        __syncthreads();
        if (qs) return;
#pragma unroll
        for (int g = 0; g < QS - 1; ++g)
#pragma unroll
            for (int k = 0; k < 16; ++k) sum[k] += red[(g * T::kTiles + base) * 1024 + k * 64];
    }
    f32x4 *out = reinterpret_cast<f32x4 *>(a.partial) + (((size_t)blockIdx.x * gridDim.y + blockIdx.y) * T::kTiles + base) * 1024 + lane;
#pragma unroll
    for (int k = 0; k < 16; ++k) out[k * 64] = sum[k];
}

// A workgroup's time per pixel, and what one more split of a 128 x 128 tile costs: wgrad1x1.hip's.
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
    const int pixels = p.kt * p.ct == 1 ? 128 : 64;
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
    wgrad1x1_packed_kernel<KT, CT, FMT><<<dim3(p.nsplit, p.tiles), dim3(512), Shape<KT, CT>::kLds, stream>>>(w);
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
