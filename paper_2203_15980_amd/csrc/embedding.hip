// Embedding lookup and its gradient for gfx950:
//   y[m] = scale * w[id[m]],   gw[v] = scale * sum over the m with id[m] = v of gy[m]        (scale: a factor per channel)
// An id outside [0, V) stands for no token: its row of y is zero and its row of gy counts for nothing.
//
// Lookup: bound by memory, one read of a table row and one write for each token.  A thread keeps its eight channels' factors and has kAhead rows in flight.
//
// Gradient: every row of gw is written once, by one place, from the tokens in sorted order; no atomics on values, so the sums' order is fixed by
// the ids alone.  What bounds it is the write of gw (4 V C bytes) beside one read of gy.
//   * sort: stable radix sort of (id, position), two digits of half the id's bits each; a workgroup takes kSortItems tokens, ranks them by ballots within a
//     wavefront, and finds its bases from all workgroups' digit counts itself; the first pass leaves the second one's counts (integer atomics: exact).
//     Up to kSmall tokens one workgroup sorts (id, position) pairs in LDS by comparing and exchanging.
//   * bounds: first and last place of each id that occurs; beside that, in the same launch, the sums of every aligned window of sorted places
//     that holds one id only (frequent ids have many), each by a workgroup of its own.
//   * rows: a row of gw adds its places before the first whole window, the windows' sums, and its places behind the last, or is zeros.
// The window has about sqrt(tokens) / 2 places, so that a row's chain, of places and of windows, stays short even if all tokens are the same.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.hpp"
#include "rows.hpp"

namespace delta {
namespace emb {

using rows::f32x4;

constexpr int kAhead = 4;
constexpr uint32_t kSmall = 2048;                        // most tokens that one workgroup sorts
constexpr uint32_t kSortItems = 1024;                    // of a workgroup in the radix sort: 4 wavefronts, 4 rounds of 64 each
constexpr int kMostBits = 22, kMostBins = 1 << ((kMostBits + 1) / 2);
constexpr long long kMostTokens = 1 << 24;

// Threads of a workgroup that works on whole rows: `pieces` (of eight channels) to a row, several rows side by side where they are short.
struct Rows { uint32_t pieces, side, threads; };
inline Rows rows_of(int C) {
    Rows r;
    r.pieces = (uint32_t)C / 8;
    r.side = r.pieces >= 256 ? 1 : 256 / r.pieces;
    r.threads = (r.pieces * r.side + 63) / 64 * 64;
    return r;
}

struct LookupArgs {
    const int64_t *id;
    const unsigned char *w;
    unsigned char *y;
    const float *scale;
    uint32_t n, V, C, pieces, side;
};

__device__ __forceinline__ void factors(const float *scale, uint32_t piece, float (&f)[8]) {
    const f32x4 a = reinterpret_cast<const f32x4 *>(scale)[piece * 2], b = reinterpret_cast<const f32x4 *>(scale)[piece * 2 + 1];
#pragma unroll
    for (int e = 0; e < 4; ++e) { f[e] = a[e]; f[4 + e] = b[e]; }
}

template <typename T>
__global__ __launch_bounds__(1024) void lookup_kernel(LookupArgs a) {
    const uint32_t piece = threadIdx.x % a.pieces, at = threadIdx.x / a.pieces;
    if (at >= a.side) return;
    float f[8];
    factors(a.scale, piece, f);
    const uint32_t step = gridDim.x * a.side;
    for (uint32_t m0 = blockIdx.x * a.side + at; m0 < a.n; m0 += kAhead * step) {
        rows::Eight<T> raw[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const uint32_t m = m0 + i * step;
            raw[i].zero();
            if (m >= a.n) continue;
            const int64_t id = a.id[m];
            if ((uint64_t)id < a.V) raw[i].load(a.w + ((uint64_t)id * a.C + piece * 8) * sizeof(T));
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const uint32_t m = m0 + i * step;
            if (m >= a.n) continue;
            float v[8];
            raw[i].to(v);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= f[e];
            rows::Eight<T>::store(a.y + ((uint64_t)m * a.C + piece * 8) * sizeof(T), v);
        }
    }
}

// ---- gradient
struct Plan {
    uint32_t n, V, C;
    uint32_t bits1, bits2;                               // of the two digits; an id of no token sorts as V, behind all others
    uint32_t blocks, window, windows;
    uint64_t key1, pos1, key2, pos2, hist1, hist2, first, last, sums, bytes;       // workspace: byte offsets and size
};

Plan plan_for(long long n, int V, int C) {
    Plan p;
    p.n = (uint32_t)n; p.V = (uint32_t)V; p.C = (uint32_t)C;
    uint32_t bits = 1;
    while ((1u << bits) <= (uint32_t)V) ++bits;
    p.bits1 = (bits + 1) / 2;
    p.bits2 = bits - p.bits1;
    p.blocks = (p.n + kSortItems - 1) / kSortItems;
    p.window = 32;
    while ((uint64_t)p.window * p.window * 4 < p.n) p.window *= 2;
    p.windows = p.n / p.window;                          // whole ones
    uint64_t at = 0;
    auto take = [&](uint64_t bytes) { const uint64_t o = at; at += (bytes + 255) / 256 * 256; return o; };
    const bool small = p.n <= kSmall;
    p.key1 = take(small ? 0 : 4ull * p.n); p.pos1 = take(small ? 0 : 4ull * p.n);
    p.key2 = take(4ull * p.n); p.pos2 = take(4ull * p.n);
    p.hist1 = take(small ? 0 : (4ull << p.bits1) * p.blocks); p.hist2 = take(small ? 0 : (4ull << p.bits2) * p.blocks);
    p.first = take(4ull * p.V); p.last = take(4ull * p.V);
    p.sums = take(4ull * p.windows * p.C);
    p.bytes = at;
    return p;
}

struct Args {
    const int64_t *id;
    const unsigned char *gy;
    const float *scale;
    float *gw;
    uint32_t *key1, *pos1, *key2, *pos2, *hist1, *hist2, *first, *last;
    float *sums;
    uint32_t n, V, C, bits1, bits2, blocks, window, windows, pieces, side;
};

__device__ __forceinline__ uint32_t key_of(int64_t id, uint32_t V) { return (uint64_t)id < V ? (uint32_t)id : V; }

// Workgroups [from, gridDim.x) write zeros over `count` values.
__device__ __forceinline__ void clear(uint32_t *p, uint64_t count, uint32_t from) {
    for (uint64_t i = (uint64_t)(blockIdx.x - from) * blockDim.x + threadIdx.x; i < count; i += (uint64_t)(gridDim.x - from) * blockDim.x) p[i] = 0;
}

// Workgroup 0 sorts all tokens; the others clear first and last.
__global__ __launch_bounds__(1024) void sort_small_kernel(Args a) {
    if (blockIdx.x) {
        clear(a.first, a.V, 1);
        clear(a.last, a.V, 1);
        return;
    }
    __shared__ uint64_t item[kSmall];
    uint32_t size = 64;
    while (size < a.n) size *= 2;
    for (uint32_t i = threadIdx.x; i < size; i += 1024) item[i] = i < a.n ? (uint64_t)key_of(a.id[i], a.V) << 32 | i : ~0ull;
    __syncthreads();
    for (uint32_t run = 2; run <= size; run *= 2)        // bitonic: all items are different, so any sort is a stable one
        for (uint32_t d = run / 2; d; d /= 2) {
            for (uint32_t t = threadIdx.x; t < size / 2; t += 1024) {
                const uint32_t i = (t / d) * 2 * d + t % d, j = i + d;
                const uint64_t x = item[i], y = item[j];
                if ((x > y) == ((i & run) == 0)) { item[i] = y; item[j] = x; }
            }
            __syncthreads();
        }
    for (uint32_t i = threadIdx.x; i < a.n; i += 1024) {
        a.key2[i] = (uint32_t)(item[i] >> 32);
        a.pos2[i] = (uint32_t)item[i];
    }
}

// Digit counts of the first pass, [block][digit]; the workgroups behind clear the second pass's counts, first and last.
__global__ __launch_bounds__(256) void count_kernel(Args a) {
    if (blockIdx.x >= a.blocks) {
        clear(a.hist2, (uint64_t)a.blocks << a.bits2, a.blocks);
        clear(a.first, a.V, a.blocks);
        clear(a.last, a.V, a.blocks);
        return;
    }
    __shared__ uint32_t bins[kMostBins];
    const uint32_t nbins = 1u << a.bits1;
    for (uint32_t i = threadIdx.x; i < nbins; i += 256) bins[i] = 0;
    __syncthreads();
    const uint32_t i0 = blockIdx.x * kSortItems;
    for (uint32_t i = threadIdx.x; i < kSortItems; i += 256)
        if (i0 + i < a.n) atomicAdd(&bins[key_of(a.id[i0 + i], a.V) & (nbins - 1)], 1u);
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < nbins; i += 256) a.hist1[(uint64_t)blockIdx.x * nbins + i] = bins[i];
}

// One pass of the sort: each token to its place by the digit, in the order the tokens come in.
template <bool FIRST>
__global__ __launch_bounds__(256) void scatter_kernel(Args a) {
    __shared__ uint32_t base[kMostBins];                 // where this workgroup's tokens of a digit begin
    __shared__ uint32_t mine[4][kMostBins];              // tokens of a digit in each wavefront; then in those before it
    __shared__ uint32_t part[256];
    const uint32_t bits = FIRST ? a.bits1 : a.bits2, shift = FIRST ? 0 : a.bits1, nbins = 1u << bits;
    const uint32_t *hist = FIRST ? a.hist1 : a.hist2;
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    for (uint32_t i = tid; i < 4 * nbins; i += 256) mine[i / nbins][i % nbins] = 0;
    // all tokens of smaller digits, and this digit's in the workgroups before: a thread sums its share of the digits, each over the workgroups
    const uint32_t per = (nbins + 255) / 256;
    uint32_t before[kMostBins / 256], sum = 0;
#pragma unroll
    for (int k = 0; k < kMostBins / 256; ++k) before[k] = 0;
    uint32_t all[kMostBins / 256];
#pragma unroll
    for (int k = 0; k < kMostBins / 256; ++k) {
        const uint32_t d = tid * per + k;
        all[k] = 0;
        if ((uint32_t)k >= per || d >= nbins) continue;
        for (uint32_t b = 0; b < a.blocks; ++b) {
            const uint32_t c = hist[(uint64_t)b * nbins + d];
            before[k] += b < blockIdx.x ? c : 0;
            all[k] += c;
        }
        sum += all[k];
    }
    part[tid] = sum;
    __syncthreads();
    for (uint32_t o = 1; o < 256; o *= 2) {              // inclusive sums over the threads
        const uint32_t v = tid >= o ? part[tid - o] : 0;
        __syncthreads();
        part[tid] += v;
        __syncthreads();
    }
    uint32_t run = part[tid] - sum;
#pragma unroll
    for (int k = 0; k < kMostBins / 256; ++k) {
        const uint32_t d = tid * per + k;
        if ((uint32_t)k >= per || d >= nbins) continue;
        base[d] = run + before[k];
        run += all[k];
    }
    // ranks within a wavefront: how many lanes before hold the same digit, after the rounds before
    const uint32_t i0 = blockIdx.x * kSortItems + wave * (kSortItems / 4);
    uint32_t key[kSortItems / 256], pos[kSortItems / 256], rank[kSortItems / 256];
#pragma unroll
    for (int r = 0; r < (int)(kSortItems / 256); ++r) {
        const uint32_t i = i0 + r * 64 + lane;
        const bool live = i < a.n;
        key[r] = 0; pos[r] = i;
        if (live) {
            key[r] = FIRST ? key_of(a.id[i], a.V) : a.key1[i];
            if (!FIRST) pos[r] = a.pos1[i];
        }
        const uint32_t d = (key[r] >> shift) & (nbins - 1);
        uint64_t same = __ballot(live);
        for (uint32_t b = 0; b < bits; ++b) {
            const uint64_t set = __ballot((d >> b) & 1);
            same &= (d >> b) & 1 ? set : ~set;
        }
        const uint32_t lower = (uint32_t)__popcll(same & ((1ull << lane) - 1));
        volatile uint32_t *count = &mine[wave][d];
        const uint32_t had = live ? *count : 0;
        rank[r] = had + lower;
        __builtin_amdgcn_wave_barrier();
        if (live && lower == 0) *count = had + (uint32_t)__popcll(same);
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    for (uint32_t d = tid; d < nbins; d += 256) {        // a digit's tokens in the wavefronts before
        uint32_t s = base[d];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const uint32_t c = mine[w][d];
            mine[w][d] = s;
            s += c;
        }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < (int)(kSortItems / 256); ++r) {
        if (i0 + r * 64 + lane >= a.n) continue;
        const uint32_t to = mine[wave][(key[r] >> shift) & (nbins - 1)] + rank[r];
        if (FIRST) {
            a.key1[to] = key[r];
            a.pos1[to] = pos[r];
            atomicAdd(&a.hist2[((uint64_t)(to / kSortItems) << a.bits2) + (key[r] >> a.bits1)], 1u);
        } else {
            a.key2[to] = key[r];
            a.pos2[to] = pos[r];
        }
    }
}

// sum += rows [from, to) of gy in sorted order, kAhead rows in flight
template <typename T>
__device__ __forceinline__ void add_places(const Args &a, uint32_t from, uint32_t to, uint32_t piece, float (&sum)[8]) {
    for (uint32_t i = from; i < to; i += kAhead) {
        rows::Eight<T> raw[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            raw[k].zero();
            if (i + k < to) raw[k].load(a.gy + ((uint64_t)a.pos2[i + k] * a.C + piece * 8) * sizeof(T));
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            float v[8];
            raw[k].to(v);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += v[e];
        }
    }
}

// Workgroups [0, windows): the sum of a window that holds one id; the others: where each id begins and ends.
template <typename T>
__global__ __launch_bounds__(1024) void bounds_kernel(Args a) {
    if (blockIdx.x >= a.windows) {
        const uint32_t i = (blockIdx.x - a.windows) * blockDim.x + threadIdx.x;
        if (i >= a.n) return;
        const uint32_t k = a.key2[i];
        if (k >= a.V) return;
        if (i == 0 || a.key2[i - 1] != k) a.first[k] = i;
        if (i + 1 == a.n || a.key2[i + 1] != k) a.last[k] = i + 1;
        return;
    }
    const uint32_t from = blockIdx.x * a.window, k = a.key2[from];
    if (k >= a.V || a.key2[from + a.window - 1] != k || threadIdx.x >= a.pieces) return;
    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    add_places<T>(a, from, from + a.window, threadIdx.x, sum);
    float *out = a.sums + (uint64_t)blockIdx.x * a.C + threadIdx.x * 8;
    reinterpret_cast<f32x4 *>(out)[0] = f32x4{sum[0], sum[1], sum[2], sum[3]};
    reinterpret_cast<f32x4 *>(out)[1] = f32x4{sum[4], sum[5], sum[6], sum[7]};
}

template <typename T>
__global__ __launch_bounds__(1024) void rows_kernel(Args a) {
    const uint32_t piece = threadIdx.x % a.pieces, at = threadIdx.x / a.pieces;
    if (at >= a.side) return;
    const uint32_t v = blockIdx.x * a.side + at;
    if (v >= a.V) return;
    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const uint32_t from = a.first[v], to = a.last[v];
    if (from < to) {
        const uint32_t lo = (from + a.window - 1) / a.window, hi = to / a.window;      // whole windows [lo, hi)
        if (lo < hi) {
            add_places<T>(a, from, lo * a.window, piece, sum);
            for (uint32_t j = lo; j < hi; ++j) {
                const f32x4 *p = reinterpret_cast<const f32x4 *>(a.sums + (uint64_t)j * a.C + piece * 8);
                const f32x4 x = p[0], y = p[1];
#pragma unroll
                for (int e = 0; e < 4; ++e) { sum[e] += x[e]; sum[4 + e] += y[e]; }
            }
            add_places<T>(a, hi * a.window, to, piece, sum);
        } else {
            add_places<T>(a, from, to, piece, sum);
        }
        float f[8];
        factors(a.scale, piece, f);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] *= f[e];
    }
    float *out = a.gw + (uint64_t)v * a.C + piece * 8;
    reinterpret_cast<f32x4 *>(out)[0] = f32x4{sum[0], sum[1], sum[2], sum[3]};
    reinterpret_cast<f32x4 *>(out)[1] = f32x4{sum[4], sum[5], sum[6], sum[7]};
}

}  // namespace emb

const char *embedding_check(const void *w, const float *scale, long long n, long long V, int C) {
    if (n <= 0 || n > emb::kMostTokens) return "1 to 16777216 tokens";
    if (V <= 0 || V >= 1ll << emb::kMostBits) return "a vocabulary of 1 to 4194303 rows";
    if (C <= 0 || C % 8 || C > 8192) return "channels must be a multiple of 8, at most 8192";
    if (!w || !scale || (((uintptr_t)w | (uintptr_t)scale) & 15)) return "w and scale must be non-null and 16-byte aligned";
    return nullptr;
}

hipError_t launch_embedding(const void *id, const void *w, const float *scale, void *y, long long n, int V, int C, int bf16, hipStream_t stream) {
    if (embedding_check(w, scale, n, V, C) || !id || !y) return hipErrorInvalidValue;
    const emb::Rows r = emb::rows_of(C);
    emb::LookupArgs a;
    a.id = static_cast<const int64_t *>(id); a.w = static_cast<const unsigned char *>(w); a.y = static_cast<unsigned char *>(y); a.scale = scale;
    a.n = (uint32_t)n; a.V = (uint32_t)V; a.C = (uint32_t)C; a.pieces = r.pieces; a.side = r.side;
    const long long want = (n + r.side - 1) / r.side;
    const dim3 grid((unsigned)(want < 2048 ? want : 2048)), block(r.threads);
    if (bf16) emb::lookup_kernel<rows::bf16><<<grid, block, 0, stream>>>(a);
    else emb::lookup_kernel<float><<<grid, block, 0, stream>>>(a);
    return hipGetLastError();
}

size_t embedding_bwd_workspace_bytes(long long n, int V, int C) { return emb::plan_for(n, V, C).bytes; }

template <typename T>
static hipError_t embedding_bwd(const emb::Args &a, const emb::Rows &r, hipStream_t stream) {
    using namespace emb;
    const uint32_t clearing = a.V / 4096 + 1;
    if (a.n <= kSmall) {
        sort_small_kernel<<<dim3(1 + clearing), dim3(1024), 0, stream>>>(a);
    } else {
        count_kernel<<<dim3(a.blocks + clearing), dim3(256), 0, stream>>>(a);
        scatter_kernel<true><<<dim3(a.blocks), dim3(256), 0, stream>>>(a);
        scatter_kernel<false><<<dim3(a.blocks), dim3(256), 0, stream>>>(a);
    }
    const uint32_t threads = (a.pieces + 63) / 64 * 64;
    bounds_kernel<T><<<dim3(a.windows + (a.n + threads - 1) / threads), dim3(threads), 0, stream>>>(a);
    rows_kernel<T><<<dim3((a.V + a.side - 1) / a.side), dim3(r.threads), 0, stream>>>(a);
    return hipGetLastError();
}

// gw [V][C] fp32, every row written.  gy [n, C] in bf16 or fp32; a workspace of embedding_bwd_workspace_bytes, 16-byte aligned.
hipError_t launch_embedding_bwd(const void *id, const void *gy, const float *scale, float *gw, long long n, int V, int C, int bf16, void *workspace,
                                size_t workspace_bytes, hipStream_t stream) {
    if (embedding_check(gy, scale, n, V, C) || !id || !gw || !workspace || ((uintptr_t)workspace & 15)) return hipErrorInvalidValue;
    const emb::Plan p = emb::plan_for(n, V, C);
    if (workspace_bytes < p.bytes) return hipErrorInvalidValue;
    const emb::Rows r = emb::rows_of(C);
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    auto u32 = [&](uint64_t o) { return reinterpret_cast<uint32_t *>(ws + o); };
    emb::Args a;
    a.id = static_cast<const int64_t *>(id); a.gy = static_cast<const unsigned char *>(gy); a.scale = scale; a.gw = gw;
    a.key1 = u32(p.key1); a.pos1 = u32(p.pos1); a.key2 = u32(p.key2); a.pos2 = u32(p.pos2);
    a.hist1 = u32(p.hist1); a.hist2 = u32(p.hist2); a.first = u32(p.first); a.last = u32(p.last);
    a.sums = reinterpret_cast<float *>(ws + p.sums);
    a.n = p.n; a.V = p.V; a.C = p.C; a.bits1 = p.bits1; a.bits2 = p.bits2; a.blocks = p.blocks;
    a.window = p.window; a.windows = p.windows; a.pieces = r.pieces; a.side = r.side;
    return bf16 ? embedding_bwd<rows::bf16>(a, r, stream) : embedding_bwd<float>(a, r, stream);
}

}  // namespace delta
