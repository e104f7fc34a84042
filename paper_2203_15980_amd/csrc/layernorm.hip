// Layer normalisation beyond transformer_ops.hip's kernel (bf16, at most 2048 channels, forward) for gfx950: fp32, up to 8192 channels, and the gradients.
//   xh = (x - mean) / sqrt(var + eps),  y = xh * gamma + beta                       (biased variance)
//   g = gy * gamma,  gx = (g - mean(g) - xh * mean(g * xh)) / sqrt(var + eps) (+ gx_add)
//   dgamma = sum over the rows of gy * xh,  dbeta = sum over the rows of gy
// mean and var come from x again: the row is read anyway, and nothing but x has to be kept (DELTA's Assumptions 1-3: the backward pass reads stored
// forward activations).  x may be a checkpoint in 8 bits (packed.hpp), read as it lies.
//
// Bound by memory, 3 reads or writes of the tensor for the gradients (6 bytes a value in bf16, 5.03 with x in 8 bits) and 2 forward.  Up to 2048 channels (backward:
// 1024) a wavefront owns a row and keeps it in registers; beyond, a workgroup does, eight channels a thread.  Workers are persistent over rows, the next
// row's loads in flight while one is worked on, and keep their sums of dgamma and dbeta in registers: a workgroup writes one partial sum of 2 C values and
// a second kernel adds those in a fixed order (no atomics: a fixed function of the inputs).  All statistics and sums are fp32: the mean first,
// then the variance of the centred values.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.hpp"
#include "packed.hpp"
#include "rows.hpp"

namespace delta {
namespace ln {

using packed::u32x2;
using rows::f32x4;

constexpr int kWaves = 8;                                // of a workgroup that has a row to each wavefront
constexpr int kRowChannels = 2048, kMostChannels = 8192;          // forward: a wavefront owns a row up to the first
constexpr int kBackwardRowChannels = 1024;               // backward

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
    __device__ __forceinline__ void load(const Args &a, uint32_t row, uint32_t ck) { v.load(a.x + ((uint64_t)row * a.C + ck * 8) * sizeof(T)); }
    __device__ __forceinline__ void to(float (&f)[8]) const { v.to(f); }
};
template <typename T> struct Packed {
    u32x2 q;
    uint32_t byte;
    __device__ __forceinline__ void zero() { q = u32x2{0u, 0u}; byte = 0; }
    __device__ __forceinline__ void load(const Args &a, uint32_t row, uint32_t ck) {
        q = *reinterpret_cast<const u32x2 *>(a.x + (uint64_t)row * a.C + ck * 8);
        byte = a.x[a.scales + (uint64_t)row * ((a.C + 31) / 32) + ck / 4];
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

// x of a row into xh; returns 1 / sqrt(var + eps).  Channels past the row's end come as zeros and stay zeros.
template <int R, typename SUM>
__device__ __forceinline__ float normalise(float (&v)[R][8], const bool (&live)[R], const Args &a, const SUM &sum, float *slots) {
    float s = 0.f;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int e = 0; e < 8; e += 2) s += v[r][e] + v[r][e + 1];
    const float mean = sum.one(s, slots) / (float)a.C;
    float sq = 0.f;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[r][e] = live[r] ? v[r][e] - mean : 0.f;
            sq += v[r][e] * v[r][e];
        }
    const float rstd = 1.0f / sqrtf(sum.one(sq, slots + 16) / (float)a.C + a.eps);
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[r][e] *= rstd;
    return rstd;
}

// ---- forward
template <typename T, int R, typename SUM>
__device__ __forceinline__ void forward_rows(const Args &a, uint32_t row, uint32_t step, uint32_t ck0, const SUM &sum, float *slots) {
    bool live[R];
#pragma unroll
    for (int r = 0; r < R; ++r) live[r] = (ck0 + 64 * r) * 8 < a.C;
    for (; row < a.rows; row += step) {
        float v[R][8];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            rows::Eight<T> raw;
            raw.zero();
            if (live[r]) raw.load(a.x + ((uint64_t)row * a.C + (ck0 + 64 * r) * 8) * sizeof(T));
            raw.to(v[r]);
        }
        normalise<R>(v, live, a, sum, slots);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (!live[r]) continue;
            float g[8], b[8];
            load8(a.gamma + (ck0 + 64 * r) * 8, g);
            load8(a.beta + (ck0 + 64 * r) * 8, b);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[r][e] = v[r][e] * g[e] + b[e];
            rows::Eight<T>::store(a.y + ((uint64_t)row * a.C + (ck0 + 64 * r) * 8) * sizeof(T), v[r]);
        }
    }
}

template <typename T, int R>
__global__ __launch_bounds__(256) void forward_kernel(Args a) {
    forward_rows<T, R>(a, blockIdx.x * 4 + (threadIdx.x >> 6), gridDim.x * 4, threadIdx.x & 63, WaveSum(), nullptr);
}
template <typename T>
__global__ __launch_bounds__(1024) void forward_wide_kernel(Args a) {
    __shared__ float slots[48];
    forward_rows<T, 1>(a, blockIdx.x, gridDim.x, threadIdx.x, GroupSum{(int)(threadIdx.x >> 6), (int)(blockDim.x >> 6)}, slots);
}

// ---- backward
// ADD: with gx_add.  (Its row is not fetched ahead: at two pieces a lane the registers of four wavefronts on a SIMD would not hold it.)
template <typename T, int FMT, bool ADD, int R, typename SUM>
__device__ __forceinline__ void backward_rows(const Args &a, uint32_t row, uint32_t step, uint32_t ck0, const SUM &sum, float *slots,
                                              float (&dg)[R][8], float (&db)[R][8]) {
    bool live[R];
    float gamma[R][8];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        live[r] = (ck0 + 64 * r) * 8 < a.C;
#pragma unroll
        for (int e = 0; e < 8; ++e) gamma[r][e] = dg[r][e] = db[r][e] = 0.f;
        if (live[r]) load8(a.gamma + (ck0 + 64 * r) * 8, gamma[r]);
    }
    Source<T, FMT> xr[R];
    rows::Eight<T> gr[R];
    auto fetch = [&](uint32_t m) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (!live[r]) continue;
            xr[r].load(a, m, ck0 + 64 * r);
            gr[r].load(a.gy + ((uint64_t)m * a.C + (ck0 + 64 * r) * 8) * sizeof(T));
        }
    };
#pragma unroll
    for (int r = 0; r < R; ++r) { xr[r].zero(); gr[r].zero(); }
    if (row < a.rows) fetch(row);
    const float over = 1.0f / (float)a.C;
    for (; row < a.rows; row += step) {
        float x[R][8], gy[R][8];
        rows::Eight<T> ar[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            xr[r].to(x[r]);
            gr[r].to(gy[r]);
            if (ADD && live[r]) ar[r].load(a.add + ((uint64_t)row * a.C + (ck0 + 64 * r) * 8) * sizeof(T));
        }
        if (row + step < a.rows) fetch(row + step);
        const float rstd = normalise<R>(x, live, a, sum, slots);
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                dg[r][e] += gy[r][e] * x[r][e];
                db[r][e] += gy[r][e];
                gy[r][e] *= gamma[r][e];
                s1 += gy[r][e];
                s2 += gy[r][e] * x[r][e];
            }
        sum.two(s1, s2, slots + 32);
        if (!a.gx) continue;
        s1 *= over;
        s2 *= over;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (!live[r]) continue;
            float o[8], add[8];
            if constexpr (ADD) ar[r].to(add);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                o[e] = rstd * (gy[r][e] - s1 - x[r][e] * s2);
                if constexpr (ADD) o[e] += add[e];
            }
            rows::Eight<T>::store(a.gx + ((uint64_t)row * a.C + (ck0 + 64 * r) * 8) * sizeof(T), o);
        }
    }
}

// A row to a wavefront, R * 512 channels; the wavefronts' sums meet in LDS, [kWaves][C], in their order.
template <typename T, int FMT, bool ADD, int R>
__global__ __launch_bounds__(kWaves * 64, R == 1 ? 4 : 2) void backward_kernel(Args a) {
    extern __shared__ __align__(16) float red[];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float dg[R][8], db[R][8];
    backward_rows<T, FMT, ADD, R>(a, blockIdx.x * kWaves + wave, gridDim.x * kWaves, lane, WaveSum(), nullptr, dg, db);
    if (!a.partial) return;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        if (half) __syncthreads();                       // the first half's sums are read
#pragma unroll
        for (int r = 0; r < R; ++r)
            if ((lane + 64 * r) * 8 < a.C) store8(red + wave * a.C + (lane + 64 * r) * 8, half ? db[r] : dg[r]);
        __syncthreads();
        for (uint32_t c = threadIdx.x; c < a.C; c += kWaves * 64) {
            float s = 0.f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) s += red[w * a.C + c];
            a.partial[((uint64_t)blockIdx.x * 2 + half) * a.C + c] = s;
        }
    }
}
// A row to a workgroup, eight channels to a thread.
template <typename T, int FMT, bool ADD>
__global__ __launch_bounds__(1024) void backward_wide_kernel(Args a) {
    __shared__ float slots[64];
    float dg[1][8], db[1][8];
    backward_rows<T, FMT, ADD, 1>(a, blockIdx.x, gridDim.x, threadIdx.x, GroupSum{(int)(threadIdx.x >> 6), (int)(blockDim.x >> 6)}, slots, dg, db);
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

// Workgroups of the backward launch: as many as are resident at once, and no more than there are rows for.
uint32_t workgroups(long long rows, int C) {
    const long long per = C <= kBackwardRowChannels ? kWaves : 1, most = C <= 4096 ? 512 : 256;
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
    switch ((C + 511) / 512) {
    case 1: run(ln::forward_kernel<float, 1>); break;
    case 2: run(ln::forward_kernel<float, 2>); break;
    case 3: run(ln::forward_kernel<float, 3>); break;
    default: run(ln::forward_kernel<float, 4>); break;
    }
    return hipGetLastError();
}

size_t layernorm_bwd_workspace_bytes(long long rows, int C) { return (size_t)ln::workgroups(rows, C) * 2 * C * sizeof(float); }

template <typename T, int FMT, bool ADD>
static hipError_t layernorm_bwd(const ln::Args &a, uint32_t grid, hipStream_t stream) {
    if (a.C > ln::kBackwardRowChannels) {
        ln::backward_wide_kernel<T, FMT, ADD><<<dim3(grid), dim3((a.C / 8 + 63) / 64 * 64), 0, stream>>>(a);
        return hipGetLastError();
    }
    const size_t lds = a.partial ? (size_t)ln::kWaves * a.C * sizeof(float) : 0;         // 32 KB at most
    if (a.C <= 512) ln::backward_kernel<T, FMT, ADD, 1><<<dim3(grid), dim3(ln::kWaves * 64), lds, stream>>>(a);
    else ln::backward_kernel<T, FMT, ADD, 2><<<dim3(grid), dim3(ln::kWaves * 64), lds, stream>>>(a);
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
