// Rotary positions for gfx950, bf16 and fp32, with any number of axes (up to 8), and their gradient.
//   theta[m, i] = sum over the axes a of pos[m, a] * freq[a, i]
//   each rotated head's pair i of channels (u, v) -> (u cos theta - v sin theta, u sin theta + v cos theta); the gradient turns by -theta
// Pair i is (i, i + D / 2), or (2 i, 2 i + 1) with PAIRS.  Heads behind the rotated ones are copied.
//
// Angles.  A position times a frequency is many turns, of which a fraction counts: 64 bits alone are off by 2^-51 of the angle, 1e-6 at 2^31 radians.  The products,
// their sum and the turns are held as two 64-bit numbers, the second what the first one's rounding left (the exact product and sum by fma and by Knuth's two-sum; 1 / (2 pi) in
// two parts), then a fraction of an eighth of a turn at most goes to fp32 and into the Taylor polynomials of sine and cosine (to x^9 and x^10: what is left out is
// below 2e-9).  Sine and cosine are off by 3.5 * 2^-24 at most.  Computed once a token, by the wavefront that turns its row, and read from LDS for each head.
//
// Bound by memory: each value is read and written once.  bf16, 8192 rows of 48 heads of 128, 40 of them rotated, 33 us (201 MB, 6.1 TB/s, part of it from the L2s'
// shared cache; 40 to 45 us, 4.5 to 5.0 TB/s, from HBM); fp32 84 us (403 MB, 4.8 TB/s).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.hpp"
#include "rows.hpp"

namespace delta {
namespace rot {

using rows::f32x4;

constexpr int kMostD = 256, kMostAxes = 8, kWaves = 4;
constexpr uint32_t kAngles = 512;                        // of a wavefront's rows: D / 2 each

struct Args {
    const unsigned char *x;
    unsigned char *y;
    const long long *pos;                                // [rows][axes]
    const float *freq;                                   // [axes][D / 2]
    uint32_t rows, axes, D;
    uint32_t turned, units;                              // pieces of 16 channels of a row: of the rotated heads, all
    uint32_t tokens;                                     // rows of a wavefront at a time
    Divisor per_head, per_half, per_row;                 // by D / 16, by D / 2, by units
    float sign;
};

// A sum of products of whole numbers and fp32 numbers, and what its roundings left.
struct Angle {
    double hi, lo;
    __device__ __forceinline__ Angle(long long pos, double f) {                    // one product
#pragma clang fp contract(off)
        const double top = (double)(int32_t)(pos >> 32) * 4294967296.0, low = (double)(uint32_t)pos;
        const double n = top + low, rest = low - (n - top);                        // pos = n + rest: top is zero or no smaller than low
        hi = n * f;
        lo = __builtin_fma(rest, f, __builtin_fma(n, f, -hi));
    }
    __device__ __forceinline__ void add(const Angle &a) {
#pragma clang fp contract(off)
        const double sum = hi + a.hi, b = sum - hi;
        lo += ((hi - (sum - b)) + (a.hi - b)) + a.lo;
        hi = sum;
    }
    __device__ __forceinline__ void turns(double &t, double &rest) const {          // times 1 / (2 pi)
#pragma clang fp contract(off)
        constexpr double kTurn = 0.15915494309189535, kTurnRest = -9.839338337591243e-18;
        t = hi * kTurn;
        rest = __builtin_fma(lo, kTurn, __builtin_fma(hi, kTurnRest, __builtin_fma(hi, kTurn, -t)));
    }
};

// Cosine and sine of an angle in turns: whole quarters aside, an eighth of a turn at most is left.
__device__ __forceinline__ void turn_of(double t, double rest, float &c, float &s) {
    const double k = rint(4.0 * t);
    const float x = (float)((t - 0.25 * k) + rest) * 6.28318530717958648f, q = x * x;
    const float sn = x * (1.0f + q * (-1.66666666666666667e-1f + q * (8.33333333333333333e-3f + q * (-1.98412698412698413e-4f + q * 2.75573192239858907e-6f))));
    const float cs = 1.0f + q * (-0.5f + q * (4.16666666666666667e-2f + q * (-1.38888888888888889e-3f + q * (2.48015873015873016e-5f + q * -2.75573192239858907e-7f))));
    const int n = (int)((long long)k & 3);
    c = n == 0 ? cs : n == 1 ? -sn : n == 2 ? -cs : sn;
    s = n == 0 ? sn : n == 1 ? cs : n == 2 ? -sn : -cs;
}

// A wavefront takes `tokens` rows at a time: as many as have 64 pieces together (30000 rows of 96 channels 6.6 us; one row at a time 10.4).
template <typename T, bool PAIRS>
__global__ __launch_bounds__(kWaves * 64) void rotary_kernel(Args a) {
    constexpr uint32_t kEs = (uint32_t)sizeof(T);
    __shared__ __align__(16) float table[kWaves][kAngles * 2];                     // a wavefront's own: cosines, then as many sines
    const uint32_t lane = threadIdx.x & 63, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), half = a.D / 2;
    float *cosine = table[wave], *sine = cosine + kAngles;
    const uint64_t step = (uint64_t)gridDim.x * kWaves * a.tokens;
    for (uint64_t row0 = (uint64_t)blockIdx.x * kWaves * a.tokens; row0 < a.rows; row0 += step) {
        const uint64_t first = row0 + (uint64_t)wave * a.tokens;
        const uint32_t here = first >= a.rows ? 0u : a.rows - first < a.tokens ? (uint32_t)(a.rows - first) : a.tokens;
        __syncthreads();                                 // the last rows' angles are read
        for (uint32_t i = lane; i < here * half; i += 64) {
            const uint32_t token = (uint32_t)divide((int)i, a.per_half), pair = i - token * half;
            const long long *pos = a.pos + (first + token) * a.axes;
            Angle angle(pos[0], (double)a.freq[pair]);
            for (uint32_t x = 1; x < a.axes; ++x) angle.add(Angle(pos[x], (double)a.freq[x * half + pair]));
            double t, rest;
            angle.turns(t, rest);
            float c, s;
            turn_of(t, rest, c, s);
            cosine[i] = c;
            sine[i] = a.sign * s;
        }
        __syncthreads();
        const unsigned char *xr = a.x + first * a.units * 16 * kEs;                // the rows lie one behind another
        unsigned char *yr = a.y + first * a.units * 16 * kEs;
        for (uint32_t i = lane; i < here * a.units; i += 64) {
            const uint32_t token = a.tokens == 1 ? 0u : (uint32_t)divide((int)i, a.per_row), u = i - token * a.units;
            const uint32_t head = (uint32_t)divide((int)u, a.per_head), piece = u - head * (a.D / 16);
            const bool turns = u < a.turned;
            // the two halves of 8 channels: eight pairs between them, or four in each
            const uint32_t lo = (PAIRS || !turns ? u * 16 : head * a.D + piece * 8) + token * a.units * 16, hi = PAIRS || !turns ? lo + 8 : lo + half;
            rows::Eight<T> p, q;
            p.load(xr + (uint64_t)lo * kEs);
            q.load(xr + (uint64_t)hi * kEs);
            if (turns) {
                float v[8], w[8], o[8], n[8], c[8], s[8];
                p.to(v);
                q.to(w);
#pragma unroll
                for (int e = 0; e < 8; e += 4) {
                    const f32x4 ct = *reinterpret_cast<const f32x4 *>(cosine + token * half + piece * 8 + e);
                    const f32x4 st = *reinterpret_cast<const f32x4 *>(sine + token * half + piece * 8 + e);
#pragma unroll
                    for (int j = 0; j < 4; ++j) { c[e + j] = ct[j]; s[e + j] = st[j]; }
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if (PAIRS) {
                        const float a0 = e < 4 ? v[2 * (e & 3)] : w[2 * (e & 3)], b0 = e < 4 ? v[2 * (e & 3) + 1] : w[2 * (e & 3) + 1];
                        (e < 4 ? o : n)[2 * (e & 3)] = a0 * c[e] - b0 * s[e];
                        (e < 4 ? o : n)[2 * (e & 3) + 1] = a0 * s[e] + b0 * c[e];
                    } else {
                        o[e] = v[e] * c[e] - w[e] * s[e];
                        n[e] = v[e] * s[e] + w[e] * c[e];
                    }
                }
                rows::Eight<T>::store(yr + (uint64_t)lo * kEs, o);
                rows::Eight<T>::store(yr + (uint64_t)hi * kEs, n);
            } else {
                *reinterpret_cast<rows::Eight<T> *>(yr + (uint64_t)lo * kEs) = p;  // bit for bit
                *reinterpret_cast<rows::Eight<T> *>(yr + (uint64_t)hi * kEs) = q;
            }
        }
    }
}

}  // namespace rot

// `heads` rotated heads and `rest` copied ones, of D channels: channels = (heads + rest) D.
const char *rotary_check(const float *freq, long long rows, int channels, int heads, int rest, long long axes) {
    if (heads <= 0 || rest < 0 || heads > channels || rest > channels - heads || channels % (heads + rest)) return "rotary positions need R rotated heads and S others, (R + S) D channels";
    const int D = channels / (heads + rest);
    if (D % 16 || D > rot::kMostD) return "rotary positions need heads of a multiple of 16 channels, up to 256";
    if (axes < 1 || axes > rot::kMostAxes) return "positions must hold 1 to 8 int64 values for each row";
    if (!freq || ((uintptr_t)freq & 3)) return "scale must hold the frequencies, [axes][D / 2]";
    if (rows > 0x7FFFFFFFLL) return "rotary positions take at most 2147483647 rows";
    return nullptr;
}

hipError_t launch_rotary(const void *x, const void *pos, void *y, const float *freq, long long rows, int channels, int heads, int rest, int axes, int pairs,
                         int backward, int bf16, hipStream_t stream) {
    if (!x || !pos || !y || rows <= 0 || rotary_check(freq, rows, channels, heads, rest, axes)) return hipErrorInvalidValue;
    rot::Args a = {};
    a.x = static_cast<const unsigned char *>(x); a.y = static_cast<unsigned char *>(y); a.pos = static_cast<const long long *>(pos); a.freq = freq;
    a.rows = (uint32_t)rows; a.axes = (uint32_t)axes; a.D = (uint32_t)(channels / (heads + rest));
    a.turned = (uint32_t)heads * (a.D / 16); a.units = (uint32_t)channels / 16;
    a.tokens = a.units >= 64 ? 1 : 64 / a.units;         // of at most 64 pieces, half of each rotated: 512 angles at most
    a.per_head = make_divisor(a.D / 16); a.per_half = make_divisor(a.D / 2); a.per_row = make_divisor(a.units);
    a.sign = backward ? -1.f : 1.f;
    const long long groups = (rows + rot::kWaves * a.tokens - 1) / (rot::kWaves * a.tokens);
    auto run = [&](auto kernel) { kernel<<<dim3((unsigned)(groups < 16384 ? groups : 16384)), dim3(rot::kWaves * 64), 0, stream>>>(a); };
    if (bf16) { if (pairs) run(rot::rotary_kernel<rows::bf16, true>); else run(rot::rotary_kernel<rows::bf16, false>); }
    else { if (pairs) run(rot::rotary_kernel<float, true>); else run(rot::rotary_kernel<float, false>); }
    return hipGetLastError();
}

}  // namespace delta
