// Layer normalisation beyond transformer_ops.hip's kernel (bf16, at most 2048 channels, forward) for gfx950: fp32, up to 8192 channels, and the gradients.
//   xh = (x - mean) / sqrt(var + eps),  y = xh * gamma + beta                       (biased variance)
//   g = gy * gamma,  gx = (g - mean(g) - xh * mean(g * xh)) / sqrt(var + eps) (+ gx_add)
//   dgamma = sum over the rows of gy * xh,  dbeta = sum over the rows of gy
// mean and var come from x again: the row is read anyway, and nothing but x has to be kept (DELTA's Assumptions 1-3: the backward pass reads stored
// forward activations).  x may be a checkpoint in 8 bits (packed.hpp), read as it lies.
//
// Bound by memory, 3 reads or writes of the tensor for the gradients (6 bytes a value in bf16, 5.03 with x in 8 bits) and 2 forward.  Up to 1024
// channels, and backward up to 2048 if there are many rows, a wavefront owns a row and keeps it in registers; beyond, a workgroup does, eight channels a
// thread.  Workers are persistent over rows, the next row's loads in flight while one is worked on, and keep their sums of dgamma and dbeta in
// registers: a workgroup writes one partial sum of 2 C values and a second kernel adds those in a fixed order (no atomics: a fixed function of the
// inputs).  All statistics and sums are fp32: the mean first, then the variance of the centred values.
// us, and the second kernel's beside them, with 16384 rows of 768 channels: bf16 17.5 + 4 (75 MB, 4.3 TB/s; from int8 or E4M3, 63 MB, the same), fp32 27 + 4.5
// (151 MB, 5.6 TB/s), forward 21.5 (100 MB, 4.7 TB/s); 8192 rows of 8192 channels with gx_add, bf16 110 + 7 (537 MB, 4.9 TB/s), forward 62 (268 MB, 4.3 TB/s);
// 8192 rows of 2048 channels with gx_add, fp32, 49 + 5 (268 MB, 5.4 TB/s), forward 29 (134 MB, 4.7 TB/s); 77 rows of 768 4.7 + 2.3.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.hpp"
#include "packed.hpp"
#include "rows.hpp"

namespace delta {
namespace ln {

using packed::u32x2;
using rows::f32x4;

// Forward: a wavefront owns a row up to the first.  fp32, a wavefront's and a workgroup's, us: 768 channels, 16384 rows 21 and 25; 2048 channels, 8192
// rows 33 and 31.
constexpr int kRowChannels = 1024, kMostChannels = 8192;
// Backward: whether a wavefront owns a row.  Up to 1024 channels always; up to 2048 if there are rows enough for 128 workgroups of them.  Both kernels, us,
// a wavefront's first, from int8 (E4M3 within 1 us of it) and with gx_add:
//   rows x channels   bf16          with gx_add   from int8     with gx_add   fp32          with gx_add   from int8     with gx_add
//   16384 x 768       22 and 46
//   8192 x 1544       22 and 33     26 and 36     21 and 34     24 and 36     38 and 39     49 and 48     28 and 35     42 and 43
//   8192 x 2048       25 and 34     31 and 41     23 and 34     27 and 38     50 and 47     59 and 57     40 and 40     52 and 49
//   2048 x 1536       24 and 24
//   1024 x 2048       11.6, 13.7    12.5, 14.2    12.2, 14.2    12.3, 14.1    13.6, 15.1    14.7, 16.2    13.2, 14.7    14.9, 15.4
//   200 x 2048        13.4, 12.8
//   77 x 1536         8.1, 6.4
// In fp32 with gx_add a row of 2048 stays in registers because gx_add is fetched late: fetched with the row 24 to 63 registers went to memory, and 85 us
// to the 59.
constexpr bool row_to_wave(long long rows, int C) { return C <= 1024 || (C <= 2048 && rows >= 1024); }
// Wavefronts of its workgroup.  The same for a tensor and its checkpoint, with and without gx_add: the sums' order, and so their bits, do not depend on those.
// us with 8 and 16: 512 channels, 16384 rows 16.2 and 15.8; 768 channels, bf16 21.4 and 20.3, fp32 52 and 56 (forward too), 77 rows 7.0 and 8.2: there 8, as
// bf16 with many rows gains less than the others lose.
template <int R> constexpr int kWaves = R == 1 ? 16 : 8;

// Rows fetched ahead, by a wavefront (1 and 2: 768 channels 21.4 and 21.3 us, fp32 52 and 54) and by a workgroup (1 and 2: 8192 channels, with the
// forward pass, 188 and 178).
constexpr int kDeep = 1, kDeepWide = 2;

struct Args {
    const unsigned char *x, *gy, *add;                   // add: null or [rows, C]
    unsigned char *y, *gx;                               // y: the forward's; gx: null or [rows, C]
    const float *gamma, *beta;
    float *partial;                                      // null or [workgroups][2][C]
    uint64_t scales;                                     // of a checkpoint x: byte offset of the scale bytes
    uint32_t rows, C;
    float eps;
};

// Eight channels of x: as they are, or a checkpoint's.
template <typename T, int FMT> struct Source {
    rows::Eight<T> v;
    __device__ __forceinline__ void zero() { v.zero(); }
    __device__ __forceinline__ void load(const Args &a, uint32_t row, uint32_t ck) { v.load(a.x + (uint64_t)row * a.C * sizeof(T) + ck * (8u * (uint32_t)sizeof(T))); }
    __device__ __forceinline__ void to(float (&f)[8]) const { v.to(f); }
};
template <typename T> struct Packed {
    u32x2 q;
    uint32_t byte;
    __device__ __forceinline__ void zero() { q = u32x2{0u, 0u}; byte = 0; }
    __device__ __forceinline__ void load(const Args &a, uint32_t row, uint32_t ck) {
        q = *reinterpret_cast<const u32x2 *>(a.x + (uint64_t)row * a.C + ck * 8u);
        byte = (a.x + a.scales + (uint64_t)row * ((a.C + 31) / 32))[ck / 4];
    }
};
template <typename T> struct Source<T, PACK_INT8> : Packed<T> {
    __device__ __forceinline__ void to(float (&f)[8]) const { packed::decode<PACK_INT8>(this->q, packed::scale_of(this->byte), f); }
};
template <typename T> struct Source<T, PACK_E4M3> : Packed<T> {
    __device__ __forceinline__ void to(float (&f)[8]) const { packed::decode<PACK_E4M3>(this->q, packed::scale_of(this->byte), f); }
};

__device__ __forceinline__ void load8(const float *p, float (&v)[8]) {
    const f32x4 a = reinterpret_cast<const f32x4 *>(p)[0], b = reinterpret_cast<const f32x4 *>(p)[1];
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[4 + e] = b[e]; }
}
__device__ __forceinline__ void store8(float *p, const float (&v)[8]) {
    reinterpret_cast<f32x4 *>(p)[0] = f32x4{v[0], v[1], v[2], v[3]};
    reinterpret_cast<f32x4 *>(p)[1] = f32x4{v[4], v[5], v[6], v[7]};
}

// Sums over the wavefront (a row to each) or over the workgroup (`slot`: LDS of its own for each sum of a row, a float to a wavefront, rewritten at the
// next row, two barriers later).
struct WaveSum {
    __device__ __forceinline__ float one(float v, float *) const { return rows::wave_sum(v); }
    __device__ __forceinline__ void two(float &a, float &b, float *) const { a = rows::wave_sum(a); b = rows::wave_sum(b); }
};
struct GroupSum {
    int wave, waves;
    __device__ __forceinline__ float one(float v, float *slot) const {
        v = rows::wave_sum(v);
        if ((threadIdx.x & 63) == 0) slot[wave] = v;
        __syncthreads();
        float s = 0.f;
        for (int w = 0; w < waves; ++w) s += slot[w];
        return s;
    }
    __device__ __forceinline__ void two(float &a, float &b, float *slot) const {
        a = rows::wave_sum(a);
        b = rows::wave_sum(b);
        if ((threadIdx.x & 63) == 0) { slot[wave] = a; slot[16 + wave] = b; }
        __syncthreads();
        a = b = 0.f;
        for (int w = 0; w < waves; ++w) { a += slot[w]; b += slot[16 + w]; }
    }
};

// A product that no neighbouring sum takes in: which product of two a sum is fused with is the compiler's choice, and another one from a checkpoint than
// from the tensor would give other bits.
__device__ __forceinline__ float scaled(float v, float by) {
#pragma clang fp contract(off)
    return v * by;
}

// x of a row into x - mean (`over`: 1 / C); returns 1 / sqrt(var + eps).  Channels past the row's end come as zeros and stay zeros.
template <int R, typename SUM>
__device__ __forceinline__ float centre(float (&v)[R][8], const bool (&live)[R], const Args &a, float over, const SUM &sum, float *slots) {
    float s = 0.f;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int e = 0; e < 8; e += 2) s += v[r][e] + v[r][e + 1];
    const float mean = scaled(sum.one(s, slots), over);
    float sq = 0.f;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const float m = live[r] ? mean : 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[r][e] -= m;
            sq += v[r][e] * v[r][e];
        }
    }
    return 1.0f / sqrtf(scaled(sum.one(sq, slots + 16), over) + a.eps);
}

// ---- forward
template <typename T, int R, typename SUM>
__device__ __forceinline__ void forward_rows(const Args &a, uint32_t row, uint32_t step, uint32_t ck0, const SUM &sum, float *slots) {
    bool live[R];
#pragma unroll
    for (int r = 0; r < R; ++r) live[r] = (ck0 + 64 * r) * 8 < a.C;
    const float over = 1.0f / (float)a.C;
    rows::Eight<T> raw[R];
    auto fetch = [&](uint32_t m) {
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (live[r]) raw[r].load(a.x + (uint64_t)m * a.C * sizeof(T) + (ck0 + 64 * r) * (8u * (uint32_t)sizeof(T)));
    };
#pragma unroll
    for (int r = 0; r < R; ++r) raw[r].zero();
    if (row < a.rows) fetch(row);
    for (; row < a.rows; row += step) {
        float v[R][8];
#pragma unroll
        for (int r = 0; r < R; ++r) raw[r].to(v[r]);
        if (row + step < a.rows) fetch(row + step);
        const float rstd = centre<R>(v, live, a, over, sum, slots);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (!live[r]) continue;
            float g[8], b[8];
            load8(a.gamma + (ck0 + 64 * r) * 8, g);
            load8(a.beta + (ck0 + 64 * r) * 8, b);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[r][e] = v[r][e] * rstd * g[e] + b[e];
            rows::Eight<T>::store(a.y + (uint64_t)row * a.C * sizeof(T) + (ck0 + 64 * r) * (8u * (uint32_t)sizeof(T)), v[r]);
        }
    }
}

template <typename T, int R>
__global__ __launch_bounds__(256) void forward_kernel(Args a) {
    forward_rows<T, R>(a, blockIdx.x * 4 + (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), gridDim.x * 4, threadIdx.x & 63, WaveSum(), nullptr);
}
template <typename T>
__global__ __launch_bounds__(1024) void forward_wide_kernel(Args a) {
    __shared__ float slots[48];
    forward_rows<T, 1>(a, blockIdx.x, gridDim.x, threadIdx.x, GroupSum{(int)(threadIdx.x >> 6), (int)(blockDim.x >> 6)}, slots);
}

// ---- backward
// ADD: with gx_add.  STRIDE: pieces (of eight channels) between two of a thread's.  LDS: `gamma` is the whole row's, in
// LDS, zeros behind it; else gamma is kept in registers.  DEEP: rows fetched ahead (not of
// gx_add).
template <typename T, int FMT, bool ADD, bool LDS, int R, int STRIDE, int DEEP, typename SUM>
__device__ __forceinline__ void backward_rows(const Args &a, uint32_t row, uint32_t step, uint32_t ck0, const SUM &sum, float *slots, const float *gamma,
                                              float (&dg)[R][8], float (&db)[R][8]) {
    constexpr bool kLate = R >= 4 && sizeof(T) == 4;     // gx_add is fetched where it is added, or the row does not fit the registers
    bool live[R];
    float kept[8];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        live[r] = (ck0 + STRIDE * r) * 8 < a.C;
#pragma unroll
        for (int e = 0; e < 8; ++e) kept[e] = dg[r][e] = db[r][e] = 0.f;
    }
    if (!LDS && live[0]) load8(a.gamma + ck0 * 8, kept);
    Source<T, FMT> xr[DEEP][R];
    rows::Eight<T> gr[DEEP][R];
    auto fetch = [&](uint32_t m, int d) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (!live[r]) continue;
            xr[d][r].load(a, m, ck0 + STRIDE * r);
            gr[d][r].load(a.gy + (uint64_t)m * a.C * sizeof(T) + (ck0 + STRIDE * r) * (8u * (uint32_t)sizeof(T)));
        }
    };
#pragma unroll
    for (int d = 0; d < DEEP; ++d) {
#pragma unroll
        for (int r = 0; r < R; ++r) { xr[d][r].zero(); gr[d][r].zero(); }
        if (row + d * step < a.rows) fetch(row + d * step, d);
    }
    const float over = 1.0f / (float)a.C;
    auto work = [&](uint32_t row, int d) {
        // gx = g * rstd - mean(g) * rstd - xh * (mean(g * xh) * rstd): rstd never meets itself, so that a row's gradient is finite wherever rstd is (its square
        // leaves fp32 for var + eps below 2^-128), and two multiply-adds a value make it
        float c[R][8], g[R][8];                          // x - mean, then xh
        rows::Eight<T> gc[R], ar[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            xr[d][r].to(c[r]);
            gc[r] = gr[d][r];
            if (ADD && !kLate && live[r]) ar[r].load(a.add + (uint64_t)row * a.C * sizeof(T) + (ck0 + STRIDE * r) * (8u * (uint32_t)sizeof(T)));
        }
        if (row + DEEP * step < a.rows) fetch(row + DEEP * step, d);
        const float rstd = centre<R>(c, live, a, over, sum, slots);
        float s1 = 0.f, s2 = 0.f;
        if (LDS) asm volatile("" ::: "memory");          // gamma is read again for each row: kept in registers it would cost a row in flight
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float gy[8], gm[8];
            gc[r].to(gy);
            if constexpr (LDS) load8(gamma + (ck0 + STRIDE * r) * 8, gm);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                c[r][e] = scaled(c[r][e], rstd);
                dg[r][e] += gy[e] * c[r][e];
                db[r][e] += gy[e];
                g[r][e] = scaled(gy[e], LDS ? gm[e] : kept[e]);
                s1 += g[r][e];
                s2 += g[r][e] * c[r][e];
            }
        }
        sum.two(s1, s2, slots + 32);
        if (!a.gx) return;
        s1 = scaled(scaled(s1, over), rstd);
        s2 = scaled(scaled(s2, over), rstd);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (!live[r]) continue;
            float o[8], add[8];
            if constexpr (ADD && kLate) ar[r].load(a.add + (uint64_t)row * a.C * sizeof(T) + (ck0 + STRIDE * r) * (8u * (uint32_t)sizeof(T)));
            if constexpr (ADD) ar[r].to(add);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                o[e] = __builtin_fmaf(-c[r][e], s2, __builtin_fmaf(g[r][e], rstd, -s1));
                if constexpr (ADD) o[e] += add[e];
            }
            rows::Eight<T>::store(a.gx + (uint64_t)row * a.C * sizeof(T) + (ck0 + STRIDE * r) * (8u * (uint32_t)sizeof(T)), o);
        }
    };
#pragma unroll 1
    for (; row < a.rows; row += DEEP * step)
#pragma unroll
        for (int d = 0; d < DEEP; ++d)
            if (row + d * step < a.rows) work(row + d * step, d);
}

// A row to a wavefront, R * 512 channels; the wavefronts' sums meet in LDS, [wavefronts][C], in their order.
template <typename T, int FMT, bool ADD, int R>
__global__ __launch_bounds__(kWaves<R> * 64) void backward_kernel(Args a) {
    constexpr int W = kWaves<R>;
    extern __shared__ __align__(16) float shared[];
    const uint32_t lane = threadIdx.x & 63, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    for (uint32_t c = threadIdx.x; c < R * 512; c += W * 64) shared[c] = c < a.C ? a.gamma[c] : 0.f;
    __syncthreads();
    float dg[R][8], db[R][8];
    backward_rows<T, FMT, ADD, true, R, 64, kDeep>(a, blockIdx.x * W + wave, gridDim.x * W, lane, WaveSum(), nullptr, shared, dg, db);
    if (!a.partial) return;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        __syncthreads();                                 // gamma, then the first sums, are read
#pragma unroll
        for (int r = 0; r < R; ++r)
            if ((lane + 64 * r) * 8 < a.C) store8(shared + wave * a.C + (lane + 64 * r) * 8, which ? db[r] : dg[r]);
        __syncthreads();
        for (uint32_t c = threadIdx.x; c < a.C; c += W * 64) {
            float s = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) s += shared[w * a.C + c];
            a.partial[((uint64_t)blockIdx.x * 2 + which) * a.C + c] = s;
        }
    }
}
// A row to a workgroup, eight channels to a thread.
template <typename T, int FMT, bool ADD>
__global__ __launch_bounds__(1024) void backward_wide_kernel(Args a) {
    __shared__ float slots[64];
    float dg[1][8], db[1][8];
    backward_rows<T, FMT, ADD, false, 1, 1, kDeepWide>(a, blockIdx.x, gridDim.x, threadIdx.x, GroupSum{(int)(threadIdx.x >> 6), (int)(blockDim.x >> 6)}, slots, nullptr, dg, db);
    if (!a.partial || threadIdx.x * 8 >= a.C) return;
    store8(a.partial + (uint64_t)blockIdx.x * 2 * a.C + threadIdx.x * 8, dg[0]);
    store8(a.partial + ((uint64_t)blockIdx.x * 2 + 1) * a.C + threadIdx.x * 8, db[0]);
}

// out[c] = the sum of n partial sums: 16 columns to a workgroup, 64 threads to a column (thread t adds partials t, t + 64, ..), whose sums meet in a
// fixed tree.
__global__ __launch_bounds__(1024) void partials_kernel(const float *partial, float *out, uint32_t n, uint32_t columns) {
    __shared__ float part[64][17];
    const uint32_t col = threadIdx.x & 15, t = threadIdx.x >> 4, c = blockIdx.x * 16 + col;
    float s = 0.f;
    for (uint32_t i = t; i < n; i += 64) s += partial[(uint64_t)i * columns + c];
    part[t][col] = s;
    __syncthreads();
    if (t < 8) {
#pragma unroll
        for (int i = 1; i < 8; ++i) s += part[t + 8 * i][col];
        part[t][col] = s;                                // its own entry: no other thread reads it before the barrier
    }
    __syncthreads();
    if (t) return;
#pragma unroll
    for (int i = 1; i < 8; ++i) s += part[i][col];
    out[c] = s;
}

// Workgroups of the backward launch: no more than there are rows for, and at most those that measured best, of 128, 256, 512 and 1024, us:
// 512 channels 20, 16, 18, -; 768 channels 30, 20.1, 20.9, -; 1536 channels -, 21, 25, -; 2048 channels, a wavefront's, -, 25, 32, -;
// 4096 channels (to a workgroup, forward too) -, 96, 89, 102; 8192 channels 245, 178, 192, -.
uint32_t workgroups(long long rows, int C) {
    const bool wave = row_to_wave(rows, C);
    const long long per = !wave ? 1 : C <= 512 ? kWaves<1> : kWaves<2>, most = !wave && C <= 4096 ? 512 : 256;
    const long long want = (rows + per - 1) / per;
    return (uint32_t)(want < most ? want : most);
}

}  // namespace ln

// Forward in what transformer_ops.hip's kernel does not take: fp32, or more than 2048 channels.
hipError_t launch_layernorm_more(const void *x, void *y, const float *gamma, const float *beta, long long rows, int C, float eps, int bf16,
                                 hipStream_t stream) {
    ln::Args a = {};
    a.x = static_cast<const unsigned char *>(x); a.y = static_cast<unsigned char *>(y); a.gamma = gamma; a.beta = beta;
    a.rows = (uint32_t)rows; a.C = (uint32_t)C; a.eps = eps;
    if (C > ln::kRowChannels) {
        const dim3 grid((unsigned)(rows < 1024 ? rows : 1024)), block((unsigned)((C / 8 + 63) / 64 * 64));
        if (bf16) ln::forward_wide_kernel<rows::bf16><<<grid, block, 0, stream>>>(a);
        else ln::forward_wide_kernel<float><<<grid, block, 0, stream>>>(a);
        return hipGetLastError();
    }
    const long long groups = (rows + 3) / 4;
    const dim3 grid((unsigned)(groups < 4096 ? groups : 4096)), block(256);
    auto run = [&](auto kernel) { kernel<<<grid, block, 0, stream>>>(a); };
    if (C <= 512) run(ln::forward_kernel<float, 1>);
    else run(ln::forward_kernel<float, 2>);
    return hipGetLastError();
}

size_t layernorm_bwd_workspace_bytes(long long rows, int C) { return (size_t)ln::workgroups(rows, C) * 2 * C * sizeof(float); }

template <typename T, int FMT, bool ADD>
static hipError_t layernorm_bwd(const ln::Args &a, uint32_t grid, hipStream_t stream) {
    if (!ln::row_to_wave(a.rows, (int)a.C)) {
        ln::backward_wide_kernel<T, FMT, ADD><<<dim3(grid), dim3((a.C / 8 + 63) / 64 * 64), 0, stream>>>(a);
        return hipGetLastError();
    }
    auto run = [&](auto kernel, unsigned waves) {
        const size_t sums = a.partial ? (size_t)waves * a.C : 0, gamma = (a.C + 511) / 512 * 512;
        kernel<<<dim3(grid), dim3(waves * 64), (sums > gamma ? sums : gamma) * sizeof(float), stream>>>(a);              // 64 KB at most
    };
    if (a.C <= 512) run(ln::backward_kernel<T, FMT, ADD, 1>, ln::kWaves<1>);
    else if (a.C <= 1024) run(ln::backward_kernel<T, FMT, ADD, 2>, ln::kWaves<2>);
    else if (a.C <= 1536) run(ln::backward_kernel<T, FMT, ADD, 3>, ln::kWaves<3>);
    else run(ln::backward_kernel<T, FMT, ADD, 4>, ln::kWaves<4>);
    return hipGetLastError();
}
template <typename T>
static hipError_t layernorm_bwd(const ln::Args &a, int fmt, uint32_t grid, hipStream_t stream) {
    switch (fmt) {
    case PACK_NONE: return a.add ? layernorm_bwd<T, PACK_NONE, true>(a, grid, stream) : layernorm_bwd<T, PACK_NONE, false>(a, grid, stream);
    case PACK_INT8: return a.add ? layernorm_bwd<T, PACK_INT8, true>(a, grid, stream) : layernorm_bwd<T, PACK_INT8, false>(a, grid, stream);
    case PACK_E4M3: return a.add ? layernorm_bwd<T, PACK_E4M3, true>(a, grid, stream) : layernorm_bwd<T, PACK_E4M3, false>(a, grid, stream);
    default: return hipErrorInvalidValue;
    }
}

// x: [rows, C] or its checkpoint (fmt); gy, add (or null), gx (or null): [rows, C]; gw: null or 2 C values, dgamma then dbeta, with a workspace of
// layernorm_bwd_workspace_bytes, 16-byte aligned.  Shapes as layernorm_check takes them.
hipError_t launch_layernorm_bwd(const void *x, const void *gy, const void *add, void *gx, const float *gamma, float *gw, long long rows, int C, float eps,
                                int bf16, int fmt, void *workspace, size_t workspace_bytes, hipStream_t stream) {
    if (!x || !gy || !gamma || rows <= 0 || rows > 0x7FFFFFFFLL || C <= 0 || C % 8 || C > ln::kMostChannels || (!gx && !gw)) return hipErrorInvalidValue;
    if (gw && (!workspace || workspace_bytes < layernorm_bwd_workspace_bytes(rows, C))) return hipErrorInvalidValue;
    ln::Args a = {};
    a.x = static_cast<const unsigned char *>(x); a.gy = static_cast<const unsigned char *>(gy); a.add = static_cast<const unsigned char *>(add);
    a.gx = static_cast<unsigned char *>(gx); a.gamma = gamma; a.partial = gw ? static_cast<float *>(workspace) : nullptr;
    a.scales = packed_scale_offset(rows, C);
    a.rows = (uint32_t)rows; a.C = (uint32_t)C; a.eps = eps;
    const uint32_t grid = ln::workgroups(rows, C);
    const hipError_t e = bf16 ? layernorm_bwd<rows::bf16>(a, fmt, grid, stream) : layernorm_bwd<float>(a, fmt, grid, stream);
    if (e != hipSuccess || !gw) return e;
    ln::partials_kernel<<<dim3((unsigned)(2 * C / 16)), dim3(1024), 0, stream>>>(a.partial, gw, grid, 2 * (uint32_t)C);
    return hipGetLastError();
}

}  // namespace delta
