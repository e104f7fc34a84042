// Log probabilities of given tokens over a vocabulary of any size for gfx950, bf16 and fp32, with the distribution's entropy, its log-sum-exp and its most
// likely tokens, and the gradients.
//   lse = log sum_j exp z_j,  lp = z[id] - lse,  H = lse - sum_j p_j z_j,  p_j = exp(z_j - lse)
//   gz_j = g_lp ([j = id] - p_j) - g_H p_j (z_j - lse + H) + g_lse p_j
// One pass over the logits: a thread keeps the largest value m so far, s = sum exp(z - m) and w = sum (m - z) exp(z - m), and scales s and w where m
// grows; threads meet through LDS.  lp = (z - m) - log s and H = log s + w / s: no difference of large numbers.
//   The gradient takes z_j - lse, which the rounding of lse moves by 2^-24 |lse| for all j, or, where lp is the smaller number, (z_j - z[id]) + lp, off by 2^-24 of
// |z_j - z[id]| and |lp|: what moves all logits of a row alike moves no probability.  (By lse alone, logits around 500, 10000: p off by 2^-16, 2^-11.)  4 |lp| < |lse|: the two
// subtractions, lp's own rounding and what it was made of are four of its steps against one of lse's.
//   A value of -infinity has no weight (z - m is held above -1e30, so that 0 * infinity is not formed).  Where no value has any, lp = lse = -infinity and
//   H = 0, and the row's gradient is zero.  NaN, or +infinity, makes the row NaN.
//
// Alternatives.  Of 64 groups of threads the K-th largest group maximum is a value that K logits reach at least; the threads whose own maximum reaches it read
// their logits again and put those that do into LDS (about 64 log(64 / (64 - K)), 24 with K = 20), and each finds its place by counting the larger ones.
// Where more than 1024 do (long runs of equal logits) or fewer than K groups hold anything, or the row holds a NaN or +infinity, a sorted list over a
// wavefront's lanes takes the logits one by one instead.  Order: value (a NaN above all, -0 as 0), of equal ones the lowest index: exact, from the logits'
// own bits.
//
// Bound by memory where there are many rows: 4096 x 131072 in bf16 (1.07 GB) forward 185 to 247 us (4.3 to 5.8 TB/s), gradient 355 to 402 us (2.15 GB, 5.3 to
// 6.0 TB/s), the least in calls of one kind after one another, the most where they take turns.  333 x 50001 in fp32 with 5 alternatives 24 us (67 MB), gradient 21 us (logits around
// 10000: 23); one row of 30522 with 20 alternatives 8.1 to 10.4 us: latency.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.hpp"
#include "rows.hpp"

namespace delta {
namespace lpr {

using rows::f32x4;
using rows::u32x4;

constexpr int kMostK = 64;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct Args {
    const unsigned char *z;                              // [rows][V]
    const long long *id;
    float *y;                                            // [3][rows]: lp, H, lse
    float *best;                                         // [rows][K]
    long long *which;
    const float *gy;                                     // [3][rows]
    unsigned char *gz;
    uint32_t rows, V, K;
};

// Eight neighbouring values from any address of the type: rows of odd length begin anywhere.
template <typename T> struct Raw;
template <> struct Raw<rows::bf16> {
    u32x4 raw;
    __device__ __forceinline__ void load(const unsigned char *p) { __builtin_memcpy(&raw, p, 16); }
    __device__ __forceinline__ void to(float (&v)[8]) const {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[2 * e] = __uint_as_float(raw[e] << 16);
            v[2 * e + 1] = __uint_as_float(raw[e] & 0xFFFF0000u);
        }
    }
};
template <> struct Raw<float> {
    f32x4 a, b;
    __device__ __forceinline__ void load(const unsigned char *p) {
        __builtin_memcpy(&a, p, 16);
        __builtin_memcpy(&b, p + 16, 16);
    }
    __device__ __forceinline__ void to(float (&v)[8]) const {
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[4 + e] = b[e]; }
    }
};
template <typename T> __device__ __forceinline__ float load_one(const unsigned char *p) {
    if constexpr (sizeof(T) == 2) return __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t *>(p) << 16);
    else return *reinterpret_cast<const float *>(p);
}
template <typename T> __device__ __forceinline__ void store_any(unsigned char *p, const float (&v)[8]) {
    if constexpr (sizeof(T) == 2) {
        const u32x4 raw = {rows::pack2(v[0], v[1]), rows::pack2(v[2], v[3]), rows::pack2(v[4], v[5]), rows::pack2(v[6], v[7])};
        __builtin_memcpy(p, &raw, 16);
    } else {
        const f32x4 a = {v[0], v[1], v[2], v[3]}, b = {v[4], v[5], v[6], v[7]};
        __builtin_memcpy(p, &a, 16);
        __builtin_memcpy(p + 16, &b, 16);
    }
}
template <typename T> __device__ __forceinline__ void store_one(unsigned char *p, float v) {
    if constexpr (sizeof(T) == 2) *reinterpret_cast<uint16_t *>(p) = (uint16_t)rows::pack2(v, v);
    else *reinterpret_cast<float *>(p) = v;
}

// The running sums of some values.  m is finite from the start (the lowest fp32 number: rows of just that value are uniform), so that no difference of
// infinities is formed; a NaN reaches s through 2^t.
struct Sums {
    float m, s, w;
    __device__ __forceinline__ void none() { m = -3.402823466e38f; s = w = 0.f; }
    // from m to a larger one
    __device__ __forceinline__ void raise(float to) {
        const float d = fmaxf(m - to, -1e30f), f = __builtin_amdgcn_exp2f(d * kLog2e);
        w = f * (w - s * d);
        s *= f;
        m = to;
    }
    __device__ __forceinline__ void add(float v) {
        const float d = v - m, e = __builtin_amdgcn_exp2f(d * kLog2e);
        s += e;
        w = __builtin_fmaf(-fmaxf(d, -1e30f), e, w);
    }
};

// A value's place in the order, as a whole number: NaN above all, -0 as 0.
__device__ __forceinline__ int32_t order_of(float v) {
    if (v != v) return 0x7FC00000;
    const int32_t b = (int32_t)__float_as_uint(v + 0.f);
    return b < 0 ? b ^ 0x7FFFFFFF : b;
}
__device__ __forceinline__ float value_of(int32_t o) { return __uint_as_float((uint32_t)(o < 0 ? o ^ 0x7FFFFFFF : o)); }
// Value, then index: the larger one goes first.
__device__ __forceinline__ unsigned long long key_of(float v, uint32_t j) {
    return (unsigned long long)((uint32_t)order_of(v) ^ 0x80000000u) << 32 | (0xFFFFFFFFu - j);
}
__device__ __forceinline__ unsigned long long lane_of(unsigned long long v, int lane) {
    return (unsigned long long)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane);
}

// A wavefront's K best keys, lane i the i-th; zero where there is none yet (no value has that key).
struct Best {
    unsigned long long key;
    unsigned long long least;                            // the K-th, the same in all lanes
    __device__ __forceinline__ void none() { key = least = 0; }
    __device__ __forceinline__ void insert(unsigned long long k, uint32_t K) {     // k the same in all lanes, above `least`
        const uint32_t lane = threadIdx.x & 63;
        const int at = __builtin_popcountll(__ballot(key > k));
        const uint32_t lo = (uint32_t)__shfl_up((int)(uint32_t)key, 1), hi = (uint32_t)__shfl_up((int)(key >> 32), 1);
        if ((int)lane == at) key = k;
        else if ((int)lane > at) key = (unsigned long long)hi << 32 | lo;
        least = lane_of(key, (int)K - 1);
    }
    // The value of each lane that has one (`there`), at the lane's index.
    __device__ __forceinline__ void offer(float v, uint32_t j, bool there, uint32_t K) {
        const unsigned long long k = there ? key_of(v, j) : 0;
        unsigned long long todo = __ballot(k > least);
        while (todo) {
            const int lane = __builtin_ctzll(todo);
            insert(lane_of(k, lane), K);
            todo &= todo - 1;
            todo &= __ballot(k > least);
        }
    }
};

__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));           // no canonicalising of values that are as they came from memory
    return r;
}
__device__ __forceinline__ float wave_max(float v) {
    v = fmaxf(v, rows::dpp<0xB1>(v));
    v = fmaxf(v, rows::dpp<0x4E>(v));
    v = fmaxf(v, rows::dpp<0x141>(v));
    v = fmaxf(v, rows::dpp<0x140>(v));
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// The thread's pieces of eight values, threadIdx.x + k * blockDim.x, three in flight: f(values, piece).  One copy of f and moves of what is in flight: a launch over few
// rows waits for its instructions to come from memory too.  With it and with eight copies of f in loops of four pieces: 1 x 30522 in fp32 with 20 alternatives 12.0 and 14.9 us, 333 x 50001
// with 5 28.9 and 37.9 us, 4096 x 131072 in bf16 231 and 267 us.
template <typename T>
struct Pieces {
    Raw<T> ahead[3];
    uint32_t n;
    __device__ __forceinline__ void fetch(const unsigned char *z, uint32_t pieces) {     // the first three
        n = pieces;
#pragma unroll
        for (int k = 0; k < 3; ++k)
            if (threadIdx.x + k * blockDim.x < n) ahead[k].load(z + (uint64_t)(threadIdx.x + k * blockDim.x) * 8 * sizeof(T));
    }
    template <typename F>
    __device__ __forceinline__ void each(const unsigned char *z, F &&f) {                // after fetch
        const uint64_t step = blockDim.x;
#pragma unroll 1
        for (uint64_t p = threadIdx.x; p < n; p += step) {
            float v[8];
            ahead[0].to(v);
            ahead[0] = ahead[1];
            ahead[1] = ahead[2];
            if (p + 3 * step < n) ahead[2].load(z + (p + 3 * step) * 8 * sizeof(T));
            f(v, (uint32_t)p);
        }
    }
};

constexpr uint32_t kMostThere = 1024;                    // candidates in LDS

// Lists over the lanes: each wavefront's over its share of the row, then the first one's over all lists.  keys: [wavefronts][64].
template <typename T>
__device__ __forceinline__ void sorted_best(const unsigned char *z, uint32_t V, uint32_t K, unsigned long long *keys, uint32_t wave, uint32_t waves, Best &top) {
    const uint32_t lane = threadIdx.x & 63;
    top.none();
    for (uint32_t j0 = wave * 64; j0 < V; j0 += waves * 64) {
        const uint32_t j = j0 + lane;
        top.offer(j < V ? load_one<T>(z + (uint64_t)j * sizeof(T)) : 0.f, j, j < V, K);
    }
    __syncthreads();                                     // what `keys` held is read
    keys[wave * 64 + lane] = lane < K ? top.key : 0;
    __syncthreads();
    if (wave) return;
    for (uint32_t w = 1; w < waves; ++w) {
        const unsigned long long k = keys[w * 64 + lane];
        unsigned long long todo = __ballot(k > top.least);
        while (todo) {
            top.insert(lane_of(k, __builtin_ctzll(todo)), K);
            todo &= todo - 1;
            todo &= __ballot(k > top.least);
        }
    }
}

template <typename T, bool TOP>
__global__ __launch_bounds__(1024) void forward_kernel(Args a) {
    constexpr uint32_t kEs = (uint32_t)sizeof(T);
    __shared__ __align__(16) Sums part[16];
    __shared__ __align__(16) unsigned long long keys[TOP ? kMostThere : 1];        // also [wavefronts][64]
    __shared__ float most[64];
    __shared__ uint32_t place[64];
    __shared__ uint32_t found;
    const uint32_t lane = threadIdx.x & 63, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), waves = blockDim.x >> 6;
    for (uint32_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const unsigned char *z = a.z + (uint64_t)row * a.V * kEs;
        const uint32_t pieces = a.V / 8, rest = pieces * 8 + threadIdx.x;          // the last V % 8 values go to the first threads
        Pieces<T> in;
        in.fetch(z, pieces);                             // on their way while the id is looked at
        const float last = rest < a.V ? load_one<T>(z + (uint64_t)rest * kEs) : -__builtin_inff();
        const long long id = a.id[row];
        if (id < 0 || id >= a.V) {                       // no token
            if (threadIdx.x < 3) a.y[(uint64_t)threadIdx.x * a.rows + row] = 0.f;
            if (TOP && threadIdx.x < a.K) {
                a.best[(uint64_t)row * a.K + threadIdx.x] = 0.f;
                a.which[(uint64_t)row * a.K + threadIdx.x] = -1;
            }
            continue;
        }
        const float mine = load_one<T>(z + (uint64_t)id * kEs);
        Sums u;
        u.none();
        auto take = [&](const float (&v)[8]) {
            const float mx = max3(max3(v[0], v[1], v[2]), max3(v[3], v[4], v[5]), max3(v[6], v[7], u.m));
            if (mx > u.m) u.raise(mx);
#pragma unroll
            for (int e = 0; e < 8; ++e) u.add(v[e]);
        };
        in.each(z, [&](const float (&v)[8], uint32_t) { take(v); });
        if (rest < a.V) {
            if (last > u.m) u.raise(last);
            u.add(last);
        }
        const float own = u.m;                           // the thread's largest (not of NaN)
        u.raise(wave_max(u.m));
        u.s = rows::wave_sum(u.s);
        u.w = rows::wave_sum(u.w);
        if (lane == 0) part[wave] = u;
        if (TOP) {
            // groups: a row of 16 lanes of 16 wavefronts, a quad of 4, a lane of 1
            float g = own;
            if (waves >= 4) {
                g = fmaxf(g, rows::dpp<0xB1>(g));
                g = fmaxf(g, rows::dpp<0x4E>(g));
            }
            if (waves == 16) {
                g = fmaxf(g, rows::dpp<0x141>(g));
                g = fmaxf(g, rows::dpp<0x140>(g));
            }
            const uint32_t per = waves;                  // lanes of a group
            if ((lane & (per - 1)) == 0) most[threadIdx.x / per] = g;
            if (threadIdx.x < 64) place[threadIdx.x] = 0;
            if (threadIdx.x == 0) found = 0;
        }
        __syncthreads();
        {
            Sums o = part[lane < waves ? lane : 0];
            o.raise(wave_max(o.m));
            u.m = o.m;
            u.s = rows::wave_sum(lane < waves ? o.s : 0.f);
            u.w = rows::wave_sum(lane < waves ? o.w : 0.f);
        }
        const float logs = __builtin_amdgcn_logf(u.s) * kLn2;                      // -infinity where nothing has weight
        auto lp = [&](float v) { return (v - u.m) - logs; };
        const bool none = u.s == 0.f;
        if (threadIdx.x == 0) {
            a.y[row] = none ? -__builtin_inff() : lp(mine);
            a.y[(uint64_t)a.rows + row] = none ? 0.f : logs + u.w / u.s;
            a.y[(uint64_t)2 * a.rows + row] = u.m + logs;
        }
        if (TOP) {
            auto put = [&](uint32_t at, unsigned long long k) {
                const float v = value_of((int32_t)((uint32_t)(k >> 32) ^ 0x80000000u));
                a.best[(uint64_t)row * a.K + at] = none ? -__builtin_inff() : lp(v);
                a.which[(uint64_t)row * a.K + at] = (long long)(0xFFFFFFFFu - (uint32_t)k);
            };
            // the groups' order: each wavefront compares its share of them with all (all 64 in each of 16 wavefronts took 2 us of a row)
            const float g = most[lane];
            const int share = 64 / (int)waves;
            uint32_t above = 0;
#pragma unroll 4
            for (int o = (int)wave * share; o < (int)(wave + 1) * share; ++o) {
                const float h = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(g), o));
                above += h > g || (h == g && o < (int)lane);
            }
            atomicAdd(&place[lane], above);
            __syncthreads();
            above = place[lane];
            const float bar = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(g), __builtin_ctzll(__ballot(above == a.K - 1))));
            bool listed = u.s == u.s && bar > -3.402823466e38f;                    // the lowest number: fewer than K groups hold anything
            if (listed) {
                auto offer = [&](float v, uint32_t j) {
                    if (v >= bar) {
                        const uint32_t at = atomicAdd(&found, 1u);
                        if (at < kMostThere) keys[at] = key_of(v, j);
                    }
                };
                if (own >= bar) {
                    in.fetch(z, pieces);
                    in.each(z, [&](const float (&v)[8], uint32_t q) {
                        if (max3(max3(v[0], v[1], v[2]), max3(v[3], v[4], v[5]), fmaxf(v[6], v[7])) < bar) return;
#pragma unroll
                        for (int e = 0; e < 8; ++e) offer(v[e], q * 8 + e);
                    });
                    if (rest < a.V) offer(last, rest);
                }
                __syncthreads();
                const uint32_t n = found;
                listed = n <= kMostThere;
                if (listed)
                    for (uint32_t i = threadIdx.x; i < n; i += blockDim.x) {
                        const unsigned long long k = keys[i];
                        uint32_t rank = 0;
#pragma unroll 4
                        for (uint32_t o = 0; o < n; ++o) rank += keys[o] > k;
                        if (rank < a.K) put(rank, k);
                    }
            }
            if (!listed) {
                Best top;
                sorted_best<T>(z, a.V, a.K, keys, wave, waves, top);
                if (wave == 0 && lane < a.K) put(lane, top.key);
            }
        }
        __syncthreads();                                 // what is in LDS is read
    }
}

template <typename T>
struct Uniform {
    const __attribute__((address_space(4))) T *p;        // constant memory, as far as the kernel is concerned
    __device__ __forceinline__ explicit Uniform(const T *at) : p((const __attribute__((address_space(4))) T *)(uintptr_t)at) {}
    __device__ __forceinline__ T operator[](uint64_t i) const { return p[i]; }
};

template <typename T>
__global__ __launch_bounds__(256) void backward_kernel(Args a, uint32_t chunks) {
    constexpr uint32_t kEs = (uint32_t)sizeof(T), kChunk = 256 * 8;
    const uint64_t n = (uint64_t)a.rows * chunks;
    for (uint64_t b = blockIdx.x; b < n; b += gridDim.x) {
        const uint32_t row = (uint32_t)(b / chunks), j = (uint32_t)(b - (uint64_t)row * chunks) * kChunk + threadIdx.x * 8;
        if (j >= a.V) continue;
        // The row's numbers, the same for all lanes: nothing here writes them, so scalar loads may bring them.
        const Uniform<float> y(a.y + row), gy(a.gy + row);
        const long long id = Uniform<long long>(a.id + row)[0];
        const float lp = y[0], H = y[a.rows], lse = y[(uint64_t)2 * a.rows], g1 = gy[0], g2 = gy[a.rows], g3 = gy[(uint64_t)2 * a.rows];
        const bool live = id >= 0 && id < a.V && lse != -__builtin_inff();
        asm volatile("" ::"s"(lp));                      // with the others, not behind the branch
        const uint64_t at = ((uint64_t)row * a.V + j) * kEs;
        const bool whole = j + 8 <= a.V;
        float v[8], o[8], from = lse, more = 0.f;        // log p_j = (z_j - from) + more
        if (live) {
            Raw<T> raw;
            if (whole) raw.load(a.z + at);
            if (4.f * fabsf(lp) < fabsf(lse)) {          // not of infinities and NaN; behind the load above (before it: 4096 x 131072 in bf16 450 us)
                from = load_one<T>(a.z + ((uint64_t)row * a.V + id) * kEs);
                more = lp;
            }
            if (whole) raw.to(v);
            else
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = j + e < a.V ? load_one<T>(a.z + at + e * kEs) : 0.f;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float g = 0.f;
            if (live) {
                const float d = (v[e] - from) + more, p = __builtin_amdgcn_exp2f(d * kLog2e);
                if (p != 0.f) g = p * ((g3 - g1) - g2 * (d + H));
                if (j + e == (uint32_t)id) g += g1;
            }
            o[e] = g;
        }
        if (whole) store_any<T>(a.gz + at, o);
        else
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (j + e < a.V) store_one<T>(a.gz + at + e * kEs, o[e]);
    }
}

}  // namespace lpr

const char *logprob_check(long long rows, int V, int K) {
    if (V <= 0 || rows <= 0 || rows > 0x7FFFFFFFLL) return "log probabilities take 1 to 2147483647 rows";
    if (K < 0 || K > lpr::kMostK || K > V) return "log probabilities give 0 to 64 alternatives, no more than there are tokens";
    return nullptr;
}

// y: [3][rows]; best, which: [rows][K], null with K = 0.
hipError_t launch_logprob(const void *z, const void *id, float *y, float *best, long long *which, long long rows, int V, int K, int bf16, hipStream_t stream) {
    if (!z || !id || !y || logprob_check(rows, V, K) || (K && (!best || !which))) return hipErrorInvalidValue;
    lpr::Args a = {};
    a.z = static_cast<const unsigned char *>(z); a.id = static_cast<const long long *>(id); a.y = y; a.best = best; a.which = which;
    a.rows = (uint32_t)rows; a.V = (uint32_t)V; a.K = (uint32_t)K;
    // Wavefronts to a row, by its length alone.  us with 1, 4 and 16 in bf16, without alternatives, then with 5 (fp32: the same order but where all wait for memory):
    //   V        1 row                             333 rows                            4096 rows
    //   2048     3.5, 3.2, 3.2   7.7, 4.8, 4.8     3.9, 3.6, 4.4   8.8, 5.5, 8.5       5.8, 7.8, 18.7    13.3, 15.4, 58
    //   4095     4.3, 3.3, 3.7   9.7, 5.3, 4.7     4.9, 4.1, 4.7   10.7, 6.3, 8.9      9.5, 11.6, 22.5   18.8, 20.7, 65
    //   8191     5.9, 3.6, 3.6   11.9, 6.0, 5.0    6.5, 4.7, 5.1   14.0, 7.8, 9.7      15.1, 19.1, 27.9  27.2, 29.0, 72
    //   16383    9.3, 4.6, 4.3   17.5, 8.2, 6.0    10.1, 5.9, 6.4  20.3, 10.2, 12.2    24.8, 28.2, 40.1  43.1, 39.9, 94
    //   32768    15.8, 6.0, 5.2  27.8, 11.1, 7.6   17.2, 8.3, 8.3  32.3, 14.6, 14.8    44.2, 45.0, 55.2  75.4, 62.4, 118
    // A compromise: few rows would have more wavefronts at each length, thousands of rows fewer, which a rule by rows too could give.
    const uint32_t waves = V >= 16 * 1024 ? 16 : V >= 4096 ? 4 : 1;
    auto run = [&](auto kernel) { kernel<<<dim3(a.rows < 65536u ? a.rows : 65536u), dim3(waves * 64), 0, stream>>>(a); };
    if (bf16) { if (K) run(lpr::forward_kernel<rows::bf16, true>); else run(lpr::forward_kernel<rows::bf16, false>); }
    else { if (K) run(lpr::forward_kernel<float, true>); else run(lpr::forward_kernel<float, false>); }
    return hipGetLastError();
}

// y: what the forward pass left; gy: [3][rows].
hipError_t launch_logprob_bwd(const void *z, const void *id, const float *y, const float *gy, void *gz, long long rows, int V, int bf16, hipStream_t stream) {
    if (!z || !id || !y || !gy || !gz || logprob_check(rows, V, 0)) return hipErrorInvalidValue;
    lpr::Args a = {};
    a.z = static_cast<const unsigned char *>(z); a.id = static_cast<const long long *>(id); a.y = const_cast<float *>(y); a.gy = gy;
    a.gz = static_cast<unsigned char *>(gz); a.rows = (uint32_t)rows; a.V = (uint32_t)V;
    const uint32_t chunks = (a.V + 2047) / 2048;
    const uint64_t n = (uint64_t)a.rows * chunks;
    auto run = [&](auto kernel) { kernel<<<dim3((unsigned)(n < (1u << 20) ? n : 1u << 20)), dim3(256), 0, stream>>>(a, chunks); };
    if (bf16) run(lpr::backward_kernel<rows::bf16>);
    else run(lpr::backward_kernel<float>);
    return hipGetLastError();
}

}  // namespace delta
