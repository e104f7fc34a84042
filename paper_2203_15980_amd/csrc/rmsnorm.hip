// Root-mean-square normalisation over the channels of a row for gfx950, bf16 and fp32: the residual's addition in front, an 8-bit checkpoint of the result
// beside it, and the gradients.
//   s = x + res, rounded to the storage type (s = x without a residual);  r = 1 / sqrt(mean(s^2) + eps);  y = s r gamma
//   checkpoint: y as stored, packed (packed.hpp): the bits that pack8.hip makes of y
//   g = gy gamma,  sh = s r,  gx = r (g - sh mean(g sh)) (+ gx_add);  dgamma = sum over the rows of gy sh
// gx is the gradient of x and of res: both reach the loss through s alone, and what else reads s adds its gradient as gx_add.
// r comes from s again in the backward pass, as in layernorm.hip: nothing but s has to be kept.
//
// Bound by memory: forward with residual and checkpoint 9.03 bytes a value in bf16, backward with gx_add 8.  A wavefront owns a row up to 2048 channels, a
// workgroup beyond (eight channels a thread); the row stays in registers from its load to its store.  us, rows one after another from HBM: 8192 x 4096 in bf16
// forward with residual and int8 checkpoint 52 (303 MB, 5.8 TB/s), gradients with gx_add 60 to 62 (268 MB, 4.3 to 4.5 TB/s; 46 to 49 where calls follow each other and find
// operands in the shared cache); fp32 forward without a checkpoint 87 to 89 (537 MB, 6.1 TB/s), gradients 106 to 108 (5.0 TB/s); 16384 x 768 in bf16 forward 16, gradients 19
// (their operands partly from the shared cache); 77 x 768 3.4 and 6.3: launches.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.hpp"
#include "packed.hpp"
#include "rows.hpp"

namespace delta {
namespace rms {

using packed::u32x2;
using rows::f32x4;

constexpr int kWaveChannels = 2048, kMostChannels = 8192;

struct Args {
    const unsigned char *x, *res, *gy, *add;             // forward: x, res (or null); backward: x is s; gy, add (or null)
    unsigned char *y, *sum, *held, *gx;                  // sum: with res; held: null or the checkpoint; gx: null or [rows, C]
    const float *gamma;
    float *partial;                                      // null or [workgroups][C]
    uint64_t scales;                                     // byte offset of the checkpoint's scale bytes
    uint32_t rows, C;
    float eps;
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

// v as the storage type holds it.
template <typename T> __device__ __forceinline__ void round_to(float (&v)[8]);
template <> __device__ __forceinline__ void round_to<float>(float (&)[8]) {}
template <> __device__ __forceinline__ void round_to<rows::bf16>(float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        const uint32_t p = rows::pack2(v[e], v[e + 1]);
        v[e] = __uint_as_float(p << 16);
        v[e + 1] = __uint_as_float(p & 0xFFFF0000u);
    }
}

// The sum over a row's owners: a wavefront, or a workgroup (`slot`: a float to a wavefront, of this sum's own, rewritten two barriers later).
struct WaveSum {
    __device__ __forceinline__ float operator()(float v, float *) const { return rows::wave_sum(v); }
};
struct GroupSum {
    __device__ __forceinline__ float operator()(float v, float *slot) const {
        v = rows::wave_sum(v);
        if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
        __syncthreads();
        float s = 0.f;
        for (uint32_t w = 0; w < blockDim.x >> 6; ++w) s += slot[w];
        return s;
    }
};

template <int R, typename SUM>
__device__ __forceinline__ float inverse_rms(const float (&s)[R][8], const Args &a, const SUM &sum, float *slot) {
    float q = 0.f;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int e = 0; e < 8; ++e) q += s[r][e] * s[r][e];
    return 1.0f / sqrtf(sum(q, slot) * (1.0f / (float)a.C) + a.eps);
}

// ---- forward.  A block of 32 channels is four neighbouring lanes' (C is a multiple of 8: a short last block's lanes past the end hold zeros).
template <typename T, int FMT, int R, int STRIDE, typename SUM>
__device__ __forceinline__ void forward_rows(const Args &a, uint32_t row, uint32_t step, uint32_t ck0, const SUM &sum, float *slots) {
    constexpr uint32_t kEs = (uint32_t)sizeof(T);
    for (; row < a.rows; row += step) {
        const uint64_t at = (uint64_t)row * a.C * kEs;
        float s[R][8];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const uint32_t ck = ck0 + STRIDE * r;
            rows::Eight<T> v, w;
            v.zero(); w.zero();
            if (ck * 8 < a.C) {
                v.load(a.x + at + ck * 8 * kEs);
                if (a.res) w.load(a.res + at + ck * 8 * kEs);
            }
            v.to(s[r]);
            if (a.res) {
                float b[8];
                w.to(b);
#pragma unroll
                for (int e = 0; e < 8; ++e) s[r][e] += b[e];
                round_to<T>(s[r]);
                if (ck * 8 < a.C) rows::Eight<T>::store(a.sum + at + ck * 8 * kEs, s[r]);
            }
        }
        const float rstd = inverse_rms<R>(s, a, sum, slots);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const uint32_t ck = ck0 + STRIDE * r;
            const bool live = ck * 8 < a.C;
            if (live) {
                float g[8];
                load8(a.gamma + ck * 8, g);
#pragma unroll
                for (int e = 0; e < 8; ++e) s[r][e] = s[r][e] * rstd * g[e];
                rows::Eight<T>::store(a.y + at + ck * 8 * kEs, s[r]);
            }
            if constexpr (FMT != PACK_NONE) {
                round_to<T>(s[r]);
                uint32_t m = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t b = live ? __float_as_uint(s[r][e]) & 0x7FFFFFFFu : 0u;
                    m = b > m ? b : m;
                }
                uint32_t o = rows::quad_xor1(m);
                m = o > m ? o : m;
                o = rows::quad_xor2(m);
                m = o > m ? o : m;
                const uint32_t byte = packed::scale_byte<FMT>(m);
                if (live) {
                    *reinterpret_cast<u32x2 *>(a.held + (uint64_t)row * a.C + ck * 8) = packed::encode<FMT>(s[r], packed::inverse_of(byte));
                    if ((ck & 3) == 0) a.held[a.scales + (uint64_t)row * ((a.C + 31) / 32) + ck / 4] = (unsigned char)byte;
                }
            }
        }
        if (STRIDE == 1) __syncthreads();                // the slots are read
    }
}

template <typename T, int FMT, int R>
__global__ __launch_bounds__(256) void forward_kernel(Args a) {
    forward_rows<T, FMT, R, 64>(a, blockIdx.x * 4 + (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), gridDim.x * 4, threadIdx.x & 63, WaveSum(), nullptr);
}
template <typename T, int FMT>
__global__ __launch_bounds__(1024) void forward_wide_kernel(Args a) {
    __shared__ float slots[16];
    forward_rows<T, FMT, 1, 1>(a, blockIdx.x, gridDim.x, threadIdx.x, GroupSum(), slots);
}

// ---- backward: workers are persistent over rows and keep their sums of dgamma; DEEP rows are on their way while one is worked on
template <typename T, bool ADD, int R, int STRIDE, int DEEP, typename SUM>
__device__ __forceinline__ void backward_rows(const Args &a, uint32_t row, uint32_t step, uint32_t ck0, const SUM &sum, float *slots, float (&dg)[R][8]) {
    constexpr uint32_t kEs = (uint32_t)sizeof(T);
    rows::Eight<T> sr[DEEP][R], gr[DEEP][R];
    auto fetch = [&](uint32_t m, int d) {
        const uint64_t at = (uint64_t)m * a.C * kEs;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const uint32_t ck = ck0 + STRIDE * r;
            if (ck * 8 >= a.C) continue;
            sr[d][r].load(a.x + at + ck * 8 * kEs);
            gr[d][r].load(a.gy + at + ck * 8 * kEs);
        }
    };
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int e = 0; e < 8; ++e) dg[r][e] = 0.f;
#pragma unroll
    for (int d = 0; d < DEEP; ++d) {
#pragma unroll
        for (int r = 0; r < R; ++r) { sr[d][r].zero(); gr[d][r].zero(); }
        if ((uint64_t)row + (uint64_t)d * step < a.rows) fetch(row + d * step, d);
    }
    auto work = [&](uint32_t row, int d) {
        const uint64_t at = (uint64_t)row * a.C * kEs;
        float s[R][8], g[R][8];
        rows::Eight<T> w[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            sr[d][r].to(s[r]);
            gr[d][r].to(g[r]);
            if (ADD && (ck0 + STRIDE * r) * 8 < a.C) w[r].load(a.add + at + (ck0 + STRIDE * r) * 8 * kEs);
        }
        if ((uint64_t)row + (uint64_t)DEEP * step < a.rows) fetch(row + DEEP * step, d);
        const float rstd = inverse_rms<R>(s, a, sum, slots);
        float dot = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const uint32_t ck = ck0 + STRIDE * r;
            if (ck * 8 >= a.C) continue;
            float gm[8];
            load8(a.gamma + ck * 8, gm);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                s[r][e] *= rstd;                         // sh: r never meets itself, so that a row's gradient is finite wherever r is
                dg[r][e] += g[r][e] * s[r][e];
                g[r][e] *= gm[e];
                dot += g[r][e] * s[r][e];
            }
        }
        const float m = sum(dot, slots + 16) * (1.0f / (float)a.C) * rstd;
        if (!a.gx) return;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const uint32_t ck = ck0 + STRIDE * r;
            if (ck * 8 >= a.C) continue;
            float o[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = __builtin_fmaf(-s[r][e], m, g[r][e] * rstd);
            if (ADD) {
                float b[8];
                w[r].to(b);
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] += b[e];
            }
            rows::Eight<T>::store(a.gx + at + ck * 8 * kEs, o);
        }
    };
#pragma unroll 1
    for (uint64_t m = row; m < a.rows; m += (uint64_t)DEEP * step)
#pragma unroll
        for (int d = 0; d < DEEP; ++d)
            if (m + (uint64_t)d * step < a.rows) work((uint32_t)(m + (uint64_t)d * step), d);
}

// A row to a wavefront; the wavefronts' sums meet in LDS, in their order.
template <typename T, bool ADD, int R>
__global__ __launch_bounds__(512) void backward_kernel(Args a) {
    extern __shared__ __align__(16) float shared[];
    const uint32_t lane = threadIdx.x & 63, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    float dg[R][8];
    backward_rows<T, ADD, R, 64, 1>(a, blockIdx.x * 8 + wave, gridDim.x * 8, lane, WaveSum(), nullptr, dg);
    if (!a.partial) return;
#pragma unroll
    for (int r = 0; r < R; ++r)
        if ((lane + 64 * r) * 8 < a.C) store8(shared + wave * a.C + (lane + 64 * r) * 8, dg[r]);
    __syncthreads();
    for (uint32_t c = threadIdx.x; c < a.C; c += 512) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) s += shared[w * a.C + c];
        a.partial[(uint64_t)blockIdx.x * a.C + c] = s;
    }
}
template <typename T, bool ADD>
__global__ __launch_bounds__(1024) void backward_wide_kernel(Args a) {
    __shared__ float slots[32];                          // two sums a row: a slot is rewritten two barriers after it was read
    float dg[1][8];
    backward_rows<T, ADD, 1, 1, 2>(a, blockIdx.x, gridDim.x, threadIdx.x, GroupSum(), slots, dg);
    if (a.partial && threadIdx.x * 8 < a.C) store8(a.partial + (uint64_t)blockIdx.x * a.C + threadIdx.x * 8, dg[0]);
}

// out[c] = the sum of n partial sums: 16 columns to a workgroup, 64 threads to a column (thread t adds partials t, t + 64, ..), whose sums meet in a
// fixed tree.
__global__ __launch_bounds__(1024) void sums_kernel(const float *partial, float *out, uint32_t n, uint32_t columns) {
    __shared__ float part[64][17];
    const uint32_t col = threadIdx.x & 15, t = threadIdx.x >> 4, c = blockIdx.x * 16 + col;
    float s = 0.f;
    if (c < columns)
        for (uint32_t i = t; i < n; i += 64) s += partial[(uint64_t)i * columns + c];
    part[t][col] = s;
    __syncthreads();
    if (t < 8) {
#pragma unroll
        for (int i = 1; i < 8; ++i) s += part[t + 8 * i][col];
        part[t][col] = s;                                // its own entry: no other thread reads it before the barrier
    }
    __syncthreads();
    if (t || c >= columns) return;
#pragma unroll
    for (int i = 1; i < 8; ++i) s += part[i][col];
    out[c] = s;
}

// Few rows: one launch for both gradients.  A workgroup owns 64 channels and needs every row's r and mean(g sh), which it makes for itself: all threads go over all values,
// eight at a time, four threads' sums (a block of 32 channels, never of two rows) go to LDS, eight threads to a row add those; then the same eight make the row's
// gx of the 64 channels, and the rows' terms of dgamma meet in a fixed order.
// r is not known yet where g s is summed: s goes in by its block's own power of two, which multiplies the block's sum in 64 bits, so that only mean(g sh) has to be in range.
constexpr int kFew = 128;
constexpr uint32_t kFewValues = 16384;
template <typename T> constexpr int kAtOnce = sizeof(T) == 2 ? 4 : 2;              // pieces of a thread on their way
template <typename T>
__global__ __launch_bounds__(1024) void few_kernel(Args a, float *gw, Divisor per_row) {
    constexpr uint32_t kEs = (uint32_t)sizeof(T);
    __shared__ float sums[2][kFewValues / 32];
    __shared__ int powers[kFewValues / 32];
    __shared__ __align__(16) float parts[16][64];
    const uint32_t lane = threadIdx.x & 63, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const uint32_t row = threadIdx.x >> 3, ck = blockIdx.x * 8 + (threadIdx.x & 7);
    const bool mine = row < a.rows && ck * 8 < a.C;
    const uint64_t at = ((uint64_t)row * a.C + ck * 8) * kEs;
    rows::Eight<T> sr, gr, ar;
    sr.zero(); gr.zero(); ar.zero();
    if (mine) {                                          // on their way under the first part
        sr.load(a.x + at);
        gr.load(a.gy + at);
        if (a.add) ar.load(a.add + at);
    }
    const uint32_t pieces = a.rows * (a.C / 8);
#pragma unroll 1
    for (uint32_t i0 = threadIdx.x; i0 < pieces; i0 += kAtOnce<T> * 1024) {
        rows::Eight<T> u[kAtOnce<T>], w[kAtOnce<T>];
        float gm[kAtOnce<T>][8];
#pragma unroll
        for (int k = 0; k < kAtOnce<T>; ++k) {
            const uint32_t i = i0 + k * 1024;
            if (i >= pieces) continue;
            u[k].load(a.x + (uint64_t)i * 8 * kEs);
            w[k].load(a.gy + (uint64_t)i * 8 * kEs);
            load8(a.gamma + (i - (uint32_t)divide((int)i, per_row) * (a.C / 8)) * 8, gm[k]);
        }
#pragma unroll
        for (int k = 0; k < kAtOnce<T>; ++k) {
            const uint32_t i = i0 + k * 1024;
            if (i >= pieces) continue;                   // whole fours of threads: C is a multiple of 32
            float s[8], g[8], q = 0.f, dot = 0.f;
            u[k].to(s);
            w[k].to(g);
            uint32_t most = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) most = max(most, __float_as_uint(s[e]) & 0x7FFFFFFFu);
            most = max(most, rows::quad_xor1(most));
            most = max(most, rows::quad_xor2(most));
            const int power = (int)(most >> 23) - 127;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                q += s[e] * s[e];
                dot += g[e] * gm[k][e] * __builtin_ldexpf(s[e], -power);
            }
            q += rows::dpp<0xB1>(q);
            dot += rows::dpp<0xB1>(dot);
            q += rows::dpp<0x4E>(q);
            dot += rows::dpp<0x4E>(dot);
            if ((lane & 3) == 0) { sums[0][i / 4] = q; sums[1][i / 4] = dot; powers[i / 4] = power; }
        }
    }
    __syncthreads();
    float inverse = 0.f, mean = 0.f;
    {
        const uint32_t n = a.C / 32;
        float q = 0.f;
        double all = 0.0;                                // sums of g s, for their range
        if (row < a.rows)
            for (uint32_t i = threadIdx.x & 7; i < n; i += 8) {
                q += sums[0][row * n + i];
                all += __builtin_ldexp((double)sums[1][row * n + i], powers[row * n + i]);
            }
        q += rows::dpp<0xB1>(q);
        q += rows::dpp<0x4E>(q);
        q += rows::dpp<0x141>(q);                        // row_half_mirror: the other quad of a lane's eight
        const float over = 1.0f / (float)a.C;
        inverse = 1.0f / sqrtf(q * over + a.eps);
        float dot = (float)(all * (double)inverse);
        dot += rows::dpp<0xB1>(dot);
        dot += rows::dpp<0x4E>(dot);
        dot += rows::dpp<0x141>(dot);
        mean = dot * over;
    }
    float s[8], g[8], dg[8];
    sr.to(s);
    gr.to(g);
    const float r = mine ? inverse : 0.f, m = mean * r;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        s[e] *= r;
        dg[e] = g[e] * s[e];
    }
    if (mine && a.gx) {
        float gm[8], o[8], b[8];
        load8(a.gamma + ck * 8, gm);
        ar.to(b);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            o[e] = __builtin_fmaf(-s[e], m, g[e] * gm[e] * r);
            if (a.add) o[e] += b[e];
        }
        rows::Eight<T>::store(a.gx + at, o);
    }
    if (!gw) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) {                        // the wavefront's eight rows
        dg[e] += rows::dpp<0x128>(dg[e]);                // row_ror:8
        dg[e] = rows::halves(rows::row_pairs(dg[e]));
    }
    if (lane < 8) store8(&parts[wave][lane * 8], dg);
    __syncthreads();
    const uint32_t c = blockIdx.x * 64 + threadIdx.x;
    if (threadIdx.x >= 64 || c >= a.C) return;
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < 16; ++w) sum += parts[w][threadIdx.x];
    gw[c] = sum;
}
// us with gx_add, bf16: 1 x 4096 4.3, 128 x 64 4.6, two launches 6.2 whatever the size up to 77 x 768, which takes 7.0 like this: a workgroup reads everything.
constexpr bool few_rows(uint64_t rows, uint64_t C) { return rows <= kFew && rows * C <= kFewValues && C % 32 == 0; }

// Workgroups of the backward launch, a partial sum of dgamma to each.  A row to a workgroup: two at least, whose loads go out together, and the partial sums are half as many (us
// with one, two and four: 300 x 8192 17.0, 12.1, 12.6; 500 x 4096 13.9, 10.6, 10.3; 1032 x 3080 in fp32 17.3, 17.2, 17.9).  A row to a wavefront: one (1000 x 2048 7.9,
// 9.4, 13.6).
uint32_t workgroups(long long rows, int C) {
    const long long per = C <= kWaveChannels ? 8 : 2, most = C <= kWaveChannels ? 256 : 512;
    const long long want = (rows + per - 1) / per;
    return (uint32_t)(want < most ? want : most);
}

}  // namespace rms

const char *rmsnorm_check(const float *gamma, long long rows, int C) {
    if (C <= 0 || C % 8 || C > rms::kMostChannels) return "root-mean-square normalisation needs a multiple of 8 channels, up to 8192";
    if (!gamma || ((uintptr_t)gamma & 15)) return "scale must be non-null and 16-byte aligned";
    if (rows > 0x7FFFFFFFLL) return "root-mean-square normalisation takes at most 2147483647 rows";
    return nullptr;
}

template <typename T, int FMT>
static hipError_t rmsnorm_forward(const rms::Args &a, hipStream_t stream) {
    if (a.C > rms::kWaveChannels) {
        rms::forward_wide_kernel<T, FMT><<<dim3(a.rows < 4096 ? a.rows : 4096), dim3((a.C / 8 + 63) / 64 * 64), 0, stream>>>(a);
        return hipGetLastError();
    }
    const uint32_t groups = (a.rows + 3) / 4;
    auto run = [&](auto kernel) { kernel<<<dim3(groups < 8192 ? groups : 8192), dim3(256), 0, stream>>>(a); };
    if (a.C <= 512) run(rms::forward_kernel<T, FMT, 1>);
    else if (a.C <= 1024) run(rms::forward_kernel<T, FMT, 2>);
    else run(rms::forward_kernel<T, FMT, 4>);
    return hipGetLastError();
}
template <typename T>
static hipError_t rmsnorm_forward(const rms::Args &a, int fmt, hipStream_t stream) {
    switch (fmt) {
    case PACK_NONE: return rmsnorm_forward<T, PACK_NONE>(a, stream);
    case PACK_INT8: return rmsnorm_forward<T, PACK_INT8>(a, stream);
    case PACK_E4M3: return rmsnorm_forward<T, PACK_E4M3>(a, stream);
    default: return hipErrorInvalidValue;
    }
}

// res and sum: both or neither; held: the checkpoint's bytes (fmt), or null.
hipError_t launch_rmsnorm(const void *x, const void *res, void *y, void *sum, void *held, const float *gamma, long long rows, int C, float eps, int bf16,
                          int fmt, hipStream_t stream) {
    if (!x || !y || !res != !sum || !held != !fmt || rows <= 0 || rmsnorm_check(gamma, rows, C)) return hipErrorInvalidValue;
    rms::Args a = {};
    a.x = static_cast<const unsigned char *>(x); a.res = static_cast<const unsigned char *>(res);
    a.y = static_cast<unsigned char *>(y); a.sum = static_cast<unsigned char *>(sum); a.held = static_cast<unsigned char *>(held);
    a.gamma = gamma; a.scales = packed_scale_offset((uint64_t)rows, (uint64_t)C);
    a.rows = (uint32_t)rows; a.C = (uint32_t)C; a.eps = eps;
    return bf16 ? rmsnorm_forward<rows::bf16>(a, fmt, stream) : rmsnorm_forward<float>(a, fmt, stream);
}

size_t rmsnorm_bwd_workspace_bytes(long long rows, int C) { return (size_t)rms::workgroups(rows, C) * C * sizeof(float); }

template <typename T, bool ADD>
static hipError_t rmsnorm_backward(const rms::Args &a, uint32_t grid, hipStream_t stream) {
    if (a.C > rms::kWaveChannels) {
        rms::backward_wide_kernel<T, ADD><<<dim3(grid), dim3((a.C / 8 + 63) / 64 * 64), 0, stream>>>(a);
        return hipGetLastError();
    }
    auto run = [&](auto kernel) { kernel<<<dim3(grid), dim3(512), 8 * a.C * sizeof(float), stream>>>(a); };
    if (a.C <= 512) run(rms::backward_kernel<T, ADD, 1>);
    else if (a.C <= 1024) run(rms::backward_kernel<T, ADD, 2>);
    else run(rms::backward_kernel<T, ADD, 4>);
    return hipGetLastError();
}

// s: the normalised tensor; gy, add (or null), gx (or null): [rows, C]; gw: null or C values, with a workspace of rmsnorm_bwd_workspace_bytes.
hipError_t launch_rmsnorm_bwd(const void *s, const void *gy, const void *add, void *gx, const float *gamma, float *gw, long long rows, int C, float eps,
                              int bf16, void *workspace, size_t workspace_bytes, hipStream_t stream) {
    if (!s || !gy || rows <= 0 || rmsnorm_check(gamma, rows, C) || (!gx && !gw)) return hipErrorInvalidValue;
    if (gw && (!workspace || workspace_bytes < rmsnorm_bwd_workspace_bytes(rows, C))) return hipErrorInvalidValue;
    rms::Args a = {};
    a.x = static_cast<const unsigned char *>(s); a.gy = static_cast<const unsigned char *>(gy); a.add = static_cast<const unsigned char *>(add);
    a.gx = static_cast<unsigned char *>(gx); a.gamma = gamma; a.partial = gw ? static_cast<float *>(workspace) : nullptr;
    a.rows = (uint32_t)rows; a.C = (uint32_t)C; a.eps = eps;
    if (rms::few_rows((uint64_t)rows, (uint64_t)C)) {
        const dim3 columns((unsigned)(C + 63) / 64);
        const Divisor per_row = make_divisor((uint32_t)C / 8);
        if (bf16) rms::few_kernel<rows::bf16><<<columns, dim3(1024), 0, stream>>>(a, gw, per_row);
        else rms::few_kernel<float><<<columns, dim3(1024), 0, stream>>>(a, gw, per_row);
        return hipGetLastError();
    }
    const uint32_t grid = rms::workgroups(rows, C);
    const hipError_t e = bf16 ? (add ? rmsnorm_backward<rows::bf16, true>(a, grid, stream) : rmsnorm_backward<rows::bf16, false>(a, grid, stream))
                              : (add ? rmsnorm_backward<float, true>(a, grid, stream) : rmsnorm_backward<float, false>(a, grid, stream));
    if (e != hipSuccess || !gw) return e;
    rms::sums_kernel<<<dim3((unsigned)(C + 15) / 16), dim3(1024), 0, stream>>>(a.partial, gw, grid, (uint32_t)C);
    return hipGetLastError();
}

}  // namespace delta
