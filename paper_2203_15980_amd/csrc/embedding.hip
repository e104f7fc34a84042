// Embedding lookup and its gradient for gfx950:
//   y[m] = scale * w[id[m]],   gw[v] = scale * sum over the m with id[m] = v of gy[m]        (scale: a factor per channel)
// An id outside [0, V) stands for no token: its row of y is zero and its row of gy counts for nothing.
//
// Lookup: bound by memory, one read of a table row and one write for each token.  A thread keeps its eight channels' factors and has kLookups rows in flight.
//
// Gradient: rows of gw from the tokens in sorted order; no atomics on values, so the sums' order is fixed by the ids alone.  What bounds it is the write
// of gw (4 V C bytes) beside one read of gy.
//   * sort, and zeros beside it: gw is filled with zeros by the launches that sort, whose few workgroups leave the memory idle; rows of ids that occur are
//     written once more (never more than there are tokens).  Up to 8192 tokens one workgroup sorts (id, position) pairs in LDS; beyond, a stable
//     radix sort of two digits over all workgroups: each ranks 256 tokens and more by ballots within a wavefront and finds its bases from all
//     workgroups' digit counts itself.  (One workgroup for 16384 tokens, or sixteen with an id's low bits each, took 23 us where the four launches took 20.)
//   * sums: a workgroup owns a chunk of sorted places, whose rows of gy it fetches 8 at a time, and adds up run by run.  A run of one id
//     that begins and ends in the chunk is a row of gw; what a chunk holds of a run that goes on beyond it becomes a partial sum: its first run in slot 0
//     if it came in from the chunk before, its last in slot 1 if it began here.
//   * joins: the chunk in which a run of several chunks begins adds its slot 1 and the following chunks' slots 0 up to the run's end, a row of gw.  Where
//     that may be many, spans of about the square root of their number that lie inside one run are added up before, each by a workgroup of its own: an id that all
//     tokens hold costs a chain of at most 256 chunks, or of four spans, and its sum is rounded that often.
// us for V = 30522, C = 768, bf16, 16384 tokens: lookup 13 (50 MB, 4 TB/s; 8 with the table's rows in the caches), sort with zeros 28.5 (94 MB written,
// 3.3 TB/s), sums 12, joins 4.3; V = 131072, C = 2048, 32768 tokens: 181 (1.07 GB, 5.9 TB/s), 63, spans 4.7, joins 6.  fp32, 16384 tokens: lookup 14.5.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.hpp"
#include "rows.hpp"

namespace delta {
namespace emb {

using rows::f32x4;

constexpr int kLookups = 2, kAhead = 4;                  // rows in flight of the lookup (1, 2, 4: the same within 1 us), chunks of the joins
constexpr uint32_t kCounts = 16;                         // workgroups' counts in flight (8, 16, 32: 16384 tokens 45, 43, 42 us; 40000 119, 116, 117)
constexpr int kPlaces = 8;                               // rows in flight of the sums (4, 8, 16: the same in bf16; fp32, 16384 x 768: 73, 73, 87 us)
// Tokens that one workgroup sorts in LDS, places for 1024, 4096 or 8192; an item is an id above its place, in 32 bits.  The whole gradient, us, so and
// through the four launches of the sort over all workgroups:
//   tokens        1024      1100      4096      8192      9000      16384    | of 64 channels: 2048      6000
//   30522 x 768   28 / 38   25 / 33   26 / 34   32 / 39   36 / 37   52 / 41  | 21 / 23   26 / 25
constexpr uint32_t places_in_lds(uint32_t n, uint32_t bits) {
    return n <= 1024 ? 1024 : n <= 4096 && bits <= 20 ? 4096 : n <= 8192 && bits <= 19 ? 8192 : 0;
}
// Sort over all workgroups: each takes 256 tokens up to the first number, 512 up to the second, 2048 up to the third, 8192 beyond, as each reads the
// counts of all.  The whole gradient, us:
//   tokens, channels   16384, 768 (and the lookup)   16384, 64   32768, 64   65536, 64   131072, 64   1048576, 16   2097152, 64   2097152, 16   8388608, 16
//   256                57                            27          36          46          69
//   512                58                            27          34          39          53                         1688
//   2048                                             39          43          46          49           136           321           305           2139
//   8192                                                                                              153                         230           871
constexpr uint32_t kOneRound = 16384, kTwoRounds = 65536, kEightRounds = 1 << 20;
// Joins: groups of threads that share a run's chunks, and how many chunks to a group are joined at once, by one workgroup; of more, spans of chunks that
// one run covers are joined ahead, in a launch of their own.  At once a run over all tokens takes 64 loads one after the other (half a microsecond each)
// to 256 chunks a group.  The whole gradient, us, at once and by spans:
//   tokens x channels (chunks a group)   16384 x 768 (205)   8192 x 2048 (1024)   32768 x 2048 (1024)   131072 x 64 (512)   16777216 x 16 (65536)
//   ids all different                    46 / 47             60 / 62              113 / 116             50 / 52             1710 / 1711
//   half of the tokens one id            57 / 47             124 / 72             179 / 122             92 / 53             8740 / 1688
//   all of them                          72 / 45             190 / 65             241 / 115             131 / 48            16080 / 1624
inline uint32_t groups_of(uint32_t pieces) { return pieces >= 256 ? 1 : 512 / pieces < 8 ? 512 / pieces : 8; }
constexpr uint32_t kJoinedAtOnce = 256;
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
    for (uint32_t m0 = blockIdx.x * a.side + at; m0 < a.n; m0 += kLookups * step) {
        rows::Eight<T> raw[kLookups];
        bool there[kLookups];
#pragma unroll
        for (int i = 0; i < kLookups; ++i) {
            const uint32_t m = m0 + i * step;
            raw[i].zero();
            there[i] = false;
            if (m >= a.n) continue;
            const int64_t id = a.id[m];
            there[i] = (uint64_t)id < a.V;
            if (there[i]) raw[i].load(a.w + ((uint64_t)id * a.C + piece * 8) * sizeof(T));
        }
#pragma unroll
        for (int i = 0; i < kLookups; ++i) {
            const uint32_t m = m0 + i * step;
            if (m >= a.n) continue;
            float v[8];
            raw[i].to(v);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = there[i] ? v[e] * f[e] : 0.f;       // zero also where the factor is an infinity or a NaN
            rows::Eight<T>::store(a.y + ((uint64_t)m * a.C + piece * 8) * sizeof(T), v);
        }
    }
}

// ---- gradient
struct Plan {
    uint32_t in_lds;                                     // places of the sort in one workgroup, or 0: over all
    uint32_t n, V, C;
    uint32_t bits, bits1, bits2;                         // of a key and its two digits; an id of no token sorts as V, behind all others
    uint32_t rounds, blocks, chunk, chunks;
    uint32_t span;                                       // chunks that are joined ahead where one run covers them all, or 0: none are
    uint64_t key1, pos1, key2, pos2, hist1, hist2, sums, bytes;                    // workspace: byte offsets and size
};

Plan plan_for(long long n, int V, int C) {
    Plan p;
    p.n = (uint32_t)n; p.V = (uint32_t)V; p.C = (uint32_t)C;
    p.bits = 1;
    while ((1u << p.bits) <= (uint32_t)V) ++p.bits;
    p.bits1 = (p.bits + 1) / 2;
    p.bits2 = p.bits - p.bits1;
    p.rounds = p.n <= kOneRound ? 1 : p.n <= kTwoRounds ? 2 : p.n <= kEightRounds ? 8 : 32;
    p.blocks = (p.n + p.rounds * 256 - 1) / (p.rounds * 256);
    // us, 768 channels:  77 tokens   1024   4096   8192   16384   32768   | of 2048 channels: 32768
    //   8 places         21          22.5   25     31     45
    //   16               23          24.4   26.5   31.5   42.5    75.5    | 271
    //   32                           28     30            45      74.5    | 266
    //   64                           37     39            49      77.6    | 269
    p.chunk = p.n <= 8192 ? 8 : p.n <= 16384 ? 16 : 32;
    p.chunks = (p.n + p.chunk - 1) / p.chunk;
    p.span = 0;
    if (p.chunks > kJoinedAtOnce * groups_of(p.C / 8))   // about the square root: as many spans to a table's longest run as chunks to a span
        for (p.span = 2; (uint64_t)p.span * p.span < p.chunks; p.span *= 2) {}
    uint64_t at = 0;
    auto take = [&](uint64_t bytes) { const uint64_t o = at; at += (bytes + 255) / 256 * 256; return o; };
    p.in_lds = places_in_lds(p.n, p.bits);
    p.key1 = take(p.in_lds ? 0 : 4ull * p.n); p.pos1 = take(p.in_lds ? 0 : 4ull * p.n);
    p.key2 = take(4ull * p.n); p.pos2 = take(4ull * p.n);
    p.hist1 = take(p.in_lds ? 0 : (4ull << p.bits1) * p.blocks); p.hist2 = take(p.in_lds ? 0 : (4ull << p.bits2) * p.blocks);
    p.sums = take(8ull * p.chunks * p.C);
    p.bytes = at;
    return p;
}

struct Args {
    const int64_t *id;
    const unsigned char *gy;
    const float *scale;
    float *gw;
    uint32_t *key1, *pos1, *key2, *pos2, *hist1, *hist2;
    float *sums;                                         // [chunks][2][C]
    uint32_t n, V, C, bits, bits1, bits2, in_lds, rounds, blocks, chunk, chunks, span, pieces;
};

__device__ __forceinline__ uint32_t key_of(int64_t id, uint32_t V) { return (uint64_t)id < V ? (uint32_t)id : V; }

// The eighths [lo, hi) of gw filled with zeros by the workgroups from `from` on.
__device__ __forceinline__ void fill(const Args &a, uint32_t from, uint32_t lo, uint32_t hi) {
    const uint64_t pieces = (uint64_t)a.V * a.C / 4, first = pieces * lo / 8, end = pieces * hi / 8;
    f32x4 *p = reinterpret_cast<f32x4 *>(a.gw);
    for (uint64_t i = first + (uint64_t)(blockIdx.x - from) * blockDim.x + threadIdx.x; i < end; i += (uint64_t)(gridDim.x - from) * blockDim.x)
        p[i] = f32x4{0.f, 0.f, 0.f, 0.f};
}

// Ranks of 64 tokens by a digit d of `bits` bits: the lanes that hold the same digit (of those that are live), and how many of them come before this one.
__device__ __forceinline__ uint64_t same_digit(uint32_t d, uint32_t bits, bool live) {
    uint64_t same = __ballot(live);
    for (uint32_t b = 0; b < bits; ++b) {
        const uint64_t set = __ballot((d >> b) & 1);
        same &= (d >> b) & 1 ? set : ~set;
    }
    return same;
}

// LDS of the sort in one workgroup: neighbouring items to a thread.  Every 16th word is followed by an unused one: a thread's words lie side by side.
template <int THREADS, int ITEMS, int WIDTH> struct SortLds {
    uint32_t item[(uint32_t)ITEMS * THREADS * 17 / 16];
    uint32_t count[(1 << WIDTH) * THREADS / 2 * 17 / 16];          // two counts to a word, [digit][thread]
    uint32_t part[THREADS / 64];
};
__device__ __forceinline__ uint32_t spaced(uint32_t i) { return i + (i >> 4); }

// The sum of v over the threads before this one; `part`: a word to a wavefront.
template <int THREADS>
__device__ __forceinline__ uint32_t sum_before(uint32_t v, uint32_t *part) {
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t run = v;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        const uint32_t u = __shfl_up(run, o, 64);
        if ((int)lane >= o) run += u;
    }
    if (lane == 63) part[wave] = run;
    __syncthreads();
    run -= v;
#pragma unroll
    for (int i = 0; i < THREADS / 64; ++i) run += (uint32_t)i < wave ? part[i] : 0;
    return run;
}

// Workgroup 0 sorts all tokens, the others fill gw.  An item is an id above its position, in 32 bits.  A pass (at most WIDTH bits) counts each thread's digits
// in a column of its own, sums the counts by (digit, thread), which is the sorted order of equal digits, and moves each item to its count's sum.
template <int THREADS, int ITEMS, int WIDTH>
__global__ __launch_bounds__(THREADS) void sort_kernel(Args a) {
    constexpr uint32_t kMost = (uint32_t)ITEMS * THREADS, kPlaceBits = kMost == 1024 ? 10 : kMost == 4096 ? 12 : 13;
    static_assert(kMost == 1u << kPlaceBits, "an item is 32 bits");
    if (blockIdx.x) {
        fill(a, 1, 0, 8);
        return;
    }
    __shared__ SortLds<THREADS, ITEMS, WIDTH> l;
    uint16_t *const count = reinterpret_cast<uint16_t *>(l.count);
    const uint32_t tid = threadIdx.x;
#pragma unroll
    for (uint32_t k = 0; k < (uint32_t)ITEMS; ++k) {          // what is behind the last token sorts behind it: all its bits are set, and it comes last
        const uint32_t i = tid + k * THREADS;
        l.item[spaced(i)] = i < a.n ? key_of(a.id[i], a.V) << kPlaceBits | i : ~0u;
    }
    const uint32_t passes = (a.bits + WIDTH - 1) / WIDTH, width = (a.bits + passes - 1) / passes, words = (1u << width) / 2;     // words of counts a thread sums
    const uint32_t column = spaced(tid / 2) * 2 + (tid & 1);
    auto at = [&](uint32_t d) { return d * (THREADS * 17 / 16) + column; };        // spaced(d * THREADS / 2 + tid / 2)
    for (uint32_t p = 0; p < passes; ++p) {
        const uint32_t shift = kPlaceBits + p * width, mask = (1u << width) - 1;
        for (uint32_t i = tid; i < spaced(words * THREADS); i += THREADS) l.count[i] = 0;
        __syncthreads();
        uint32_t item[(uint32_t)ITEMS], rank[(uint32_t)ITEMS];
#pragma unroll
        for (uint32_t k = 0; k < (uint32_t)ITEMS; ++k) item[k] = l.item[spaced(tid * (uint32_t)ITEMS + k)];
#pragma unroll
        for (uint32_t k = 0; k < (uint32_t)ITEMS; ++k) {
            const uint32_t i = at(item[k] >> shift & mask);
            rank[k] = count[i];
            count[i] = (uint16_t)(rank[k] + 1);
        }
        __syncthreads();
        uint32_t w[(1 << WIDTH) / 2], sum = 0;
#pragma unroll
        for (int j = 0; j < (1 << WIDTH) / 2; ++j) {
            w[j] = (uint32_t)j < words ? l.count[spaced(tid * words + j)] : 0;
            sum += (w[j] & 0xFFFFu) + (w[j] >> 16);
        }
        uint32_t run = sum_before<THREADS>(sum, l.part);
#pragma unroll
        for (int j = 0; j < (1 << WIDTH) / 2; ++j) {
            if ((uint32_t)j >= words) break;
            const uint32_t second = run + (w[j] & 0xFFFFu);
            l.count[spaced(tid * words + j)] = run | second << 16;
            run = second + (w[j] >> 16);
        }
        __syncthreads();
#pragma unroll
        for (uint32_t k = 0; k < (uint32_t)ITEMS; ++k) l.item[spaced(count[at(item[k] >> shift & mask)] + rank[k])] = item[k];
        __syncthreads();
    }
    for (uint32_t i = tid; i < a.n; i += THREADS) {
        const uint32_t v = l.item[spaced(i)];
        a.key2[i] = v >> kPlaceBits;
        a.pos2[i] = v & (kMost - 1);
    }
}

// Digit counts of a pass, [block][digit]; the workgroups behind fill gw.
template <bool FIRST, int ROUNDS>
__global__ __launch_bounds__(256) void count_kernel(Args a) {
    if (blockIdx.x >= a.blocks) {
        fill(a, a.blocks, FIRST ? 0 : 4, FIRST ? 1 : 5);           // counting is over in half a scatter's time
        return;
    }
    __shared__ uint32_t bins[kMostBins];
    const uint32_t nbins = 1u << (FIRST ? a.bits1 : a.bits2), i0 = blockIdx.x * (ROUNDS * 256);
    uint32_t *hist = (FIRST ? a.hist1 : a.hist2) + (uint64_t)blockIdx.x * nbins;
    for (uint32_t i = threadIdx.x; i < nbins; i += 256) bins[i] = 0;
    __syncthreads();
#pragma unroll
    for (uint32_t r = 0; r < ROUNDS; ++r) {
        const uint32_t i = i0 + r * 256 + threadIdx.x;
        if (i < a.n) atomicAdd(&bins[FIRST ? key_of(a.id[i], a.V) & (nbins - 1) : a.key1[i] >> a.bits1], 1u);
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < nbins; i += 256) hist[i] = bins[i];
}

// One pass of the sort: each token to its place by the digit, in the order the tokens come in.
template <bool FIRST, int ROUNDS>
__global__ __launch_bounds__(256) void scatter_kernel(Args a) {
    if (blockIdx.x >= a.blocks) {
        fill(a, a.blocks, FIRST ? 1 : 5, FIRST ? 4 : 8);
        return;
    }
    __shared__ uint32_t base[kMostBins];                 // where this workgroup's tokens of a digit begin
    __shared__ uint32_t mine[4][kMostBins];              // tokens of a digit in each wavefront; then in those before it
    __shared__ uint32_t part[4];
    const uint32_t bits = FIRST ? a.bits1 : a.bits2, shift = FIRST ? 0 : a.bits1, nbins = 1u << bits;
    const uint32_t *hist = FIRST ? a.hist1 : a.hist2;
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t i0 = (blockIdx.x * 4 + wave) * (ROUNDS * 64);
    uint32_t key[ROUNDS], pos[ROUNDS], rank[ROUNDS];
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const uint32_t i = i0 + r * 64 + lane;
        key[r] = 0; pos[r] = i;
        if (i >= a.n) continue;
        key[r] = FIRST ? key_of(a.id[i], a.V) : a.key1[i];
        if (!FIRST) pos[r] = a.pos1[i];
    }
    for (uint32_t w = 0; w < 4; ++w)
        for (uint32_t i = tid; i < nbins; i += 256) mine[w][i] = 0;
    // all tokens of smaller digits, and this digit's in the workgroups before: a thread sums its share of the digits, each over the workgroups
    const uint32_t per = (nbins + 255) / 256;
    uint32_t before[kMostBins / 256], all[kMostBins / 256], sum = 0;
#pragma unroll
    for (int k = 0; k < kMostBins / 256; ++k) {
        const uint32_t d = tid * per + k;
        before[k] = all[k] = 0;
        if ((uint32_t)k >= per || d >= nbins) continue;
        uint32_t b = 0;
        for (; b + kCounts <= a.blocks; b += kCounts)
#pragma unroll
            for (uint32_t j = 0; j < kCounts; ++j) {
                const uint32_t c = hist[(uint64_t)(b + j) * nbins + d];
                before[k] += b + j < blockIdx.x ? c : 0;
                all[k] += c;
            }
        if (b < a.blocks) {                              // the rest together too: one by one they took 9 us of 51 for 16000 tokens
            uint32_t c[kCounts];
#pragma unroll
            for (uint32_t j = 0; j < kCounts; ++j) c[j] = b + j < a.blocks ? hist[(uint64_t)(b + j) * nbins + d] : 0;
#pragma unroll
            for (uint32_t j = 0; j < kCounts; ++j) {
                before[k] += b + j < blockIdx.x ? c[j] : 0;
                all[k] += c[j];
            }
        }
        sum += all[k];
    }
    uint32_t run = sum_before<256>(sum, part);
#pragma unroll
    for (int k = 0; k < kMostBins / 256; ++k) {
        const uint32_t d = tid * per + k;
        if ((uint32_t)k >= per || d >= nbins) continue;
        base[d] = run + before[k];
        run += all[k];
    }
    // ranks within a wavefront: how many lanes before hold the same digit, after the rounds before (`mine` is cleared: sum_before has a barrier)
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const bool live = i0 + r * 64 + lane < a.n;
        const uint32_t d = (key[r] >> shift) & (nbins - 1);
        const uint64_t same = same_digit(d, bits, live);
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
    for (int r = 0; r < ROUNDS; ++r) {
        if (i0 + r * 64 + lane >= a.n) continue;
        const uint32_t to = mine[wave][(key[r] >> shift) & (nbins - 1)] + rank[r];
        if (FIRST) {
            a.key1[to] = key[r];
            a.pos1[to] = pos[r];
        } else {
            a.key2[to] = key[r];
            a.pos2[to] = pos[r];
        }
    }
}

__device__ __forceinline__ void put(float *out, const float (&v)[8]) {
    reinterpret_cast<f32x4 *>(out)[0] = f32x4{v[0], v[1], v[2], v[3]};
    reinterpret_cast<f32x4 *>(out)[1] = f32x4{v[4], v[5], v[6], v[7]};
}

// A workgroup's chunk of sorted places, run by run, kPlaces rows in flight.
template <typename T>
__global__ __launch_bounds__(1024) void sums_kernel(Args a) {
    const uint32_t piece = threadIdx.x, lane = piece & 63, from = blockIdx.x * a.chunk, size = from + a.chunk < a.n ? a.chunk : a.n - from;
    const uint32_t mine = from + (lane < size ? lane : size - 1);                  // a lane to a place: chunks have at most 64
    const uint32_t keys = a.key2[mine], places = a.pos2[mine];
    const uint32_t before = from ? a.key2[from - 1] : ~0u, after = from + size < a.n ? a.key2[from + size] : ~0u;
    const bool live = piece < a.pieces;                  // the last wavefront's spare lanes only lend their place
    float f[8], sum[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = sum[e] = 0.f;
    if (live) factors(a.scale, piece, f);
    uint32_t run = (uint32_t)__builtin_amdgcn_readlane((int)keys, 0);              // the run that is being added up
    bool came = run == before;                           // whether it came in from the chunk before
    auto close = [&](bool goes_on) {
        if (run >= a.V || !live) return;
        if (came || goes_on) {
            put(a.sums + ((uint64_t)blockIdx.x * 2 + (came ? 0 : 1)) * a.C + piece * 8, sum);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] *= f[e];
            put(a.gw + (uint64_t)run * a.C + piece * 8, sum);
        }
    };
    for (uint32_t i = 0; i < size; i += kPlaces) {
        rows::Eight<T> raw[kPlaces];
#pragma unroll
        for (int k = 0; k < kPlaces; ++k) {
            const uint32_t m = (uint32_t)__builtin_amdgcn_readlane((int)places, (int)(i + k));         // behind the chunk: its last place
            raw[k].zero();
            if (live && (uint32_t)__builtin_amdgcn_readlane((int)keys, (int)(i + k)) < a.V) raw[k].load(a.gy + (uint64_t)m * a.C * sizeof(T) + piece * 8 * sizeof(T));
        }
#pragma unroll
        for (int k = 0; k < kPlaces; ++k) {
            if (i + k >= size) break;
            const uint32_t key = (uint32_t)__builtin_amdgcn_readlane((int)keys, (int)(i + k));
            if (key != run) {
                close(false);
                run = key;
                came = false;
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] = 0.f;
            }
            float v[8];
            raw[k].to(v);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += v[e];
        }
    }
    close(run == after);
}

// Adds up rows place(0), place(1), .. of the partial sums.  Threads: `side` groups of `pieces`; group g adds every side-th row, kAhead of them in flight, and
// group 0 the groups' sums in their order (`part`: [side][C]).  Only group 0 returns true, and holds the sum.
template <typename PLACE>
__device__ __forceinline__ bool add_up(const Args &a, uint32_t side, uint32_t places, PLACE place, float *part, float (&sum)[8]) {
    const uint32_t piece = threadIdx.x % a.pieces, group = threadIdx.x / a.pieces;
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] = 0.f;
    if (group < side) {
        for (uint32_t j0 = group; j0 < places; j0 += side * kAhead) {
            f32x4 v[kAhead][2];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const uint32_t j = j0 + k * side;
                v[k][0] = v[k][1] = f32x4{0.f, 0.f, 0.f, 0.f};
                if (j >= places) continue;
                const f32x4 *at = reinterpret_cast<const f32x4 *>(a.sums + (uint64_t)place(j) * a.C + piece * 8);
                v[k][0] = at[0];
                v[k][1] = at[1];
            }
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) { sum[e] += v[k][0][e]; sum[4 + e] += v[k][1][e]; }
        }
        put(part + (uint64_t)group * a.C + piece * 8, sum);
    }
    __syncthreads();
    if (group) return false;
    for (uint32_t g = 1; g < side; ++g)
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += part[g * a.C + piece * 8 + e];
    return true;
}

// A span of chunks that lies inside one run: the sum of its slots 0 into slot 1 of its first chunk, which is free, as the run came in.
__global__ __launch_bounds__(1024) void spans_kernel(Args a, uint32_t side) {
    extern __shared__ __align__(16) float part[];
    const uint32_t first = blockIdx.x * a.span, key = a.key2[first * a.chunk];     // whole spans only: all their chunks are there
    if (!first || key >= a.V || a.key2[first * a.chunk - 1] != key || a.key2[(first + a.span - 1) * a.chunk] != key) return;
    float sum[8];
    if (add_up(a, side, a.span, [&](uint32_t j) { return (first + j) * 2; }, part, sum))
        put(a.sums + ((uint64_t)first * 2 + 1) * a.C + threadIdx.x % a.pieces * 8, sum);
}

// The runs that begin in this workgroup's chunk and go on into the next: slot 1 of this chunk, then slots 0 of the following ones that begin with the same id,
// or for a whole span of them slot 1 of its first.
template <bool SPANS>
__global__ __launch_bounds__(1024) void joins_kernel(Args a, uint32_t side) {
    extern __shared__ __align__(16) float part[];
    const uint32_t next = (blockIdx.x + 1) * a.chunk, key = a.key2[next];          // one workgroup fewer than there are chunks
    if (key >= a.V || a.key2[next - 1] != key) return;
    if (blockIdx.x && a.key2[next - a.chunk] == key && a.key2[next - a.chunk - 1] == key) return;      // it began further back
    // Chunks that begin with this id: 64 are looked at together, and if all do, first every 4096th, then every 64th, then each.
    const uint32_t from = blockIdx.x + 1;
    uint32_t following = 0;
    auto look = [&](uint32_t apart) {                    // how many of the next 64 groups of `apart` chunks begin with it to their last
        const uint64_t at = (uint64_t)(from + following + ((threadIdx.x & 63) + 1) * apart - 1) * a.chunk;
        const uint64_t others = __ballot(at >= a.n || a.key2[at] != key);
        const uint32_t groups = others ? (uint32_t)__builtin_ctzll(others) : 64;
        following += groups * apart;
        return groups;
    };
    if (look(1) == 64)
        for (uint32_t apart = 4096; apart; apart /= 64)
            while (look(apart) == 64) {}
    // place 0 is this chunk's slot 1; then `before` chunks, `spans` spans, the rest chunks
    uint32_t before = following, spans = 0, first = 0;
    if constexpr (SPANS) {
        const uint32_t lo = (from + a.span - 1) / a.span, hi = (from + following) / a.span;
        if (lo < hi) {
            before = lo * a.span - from;
            spans = hi - lo;
            first = lo * a.span;
        }
    }
    const uint32_t behind = before + spans, places = SPANS ? 1 + behind + (following - before - spans * a.span) : 1 + following;
    auto place = [&](uint32_t j) {
        if (!j) return blockIdx.x * 2 + 1;
        if (!SPANS || j <= before) return (blockIdx.x + j) * 2;
        if (j <= behind) return (first + (j - before - 1) * a.span) * 2 + 1;
        return (first + spans * a.span + (j - behind - 1)) * 2;
    };
    float sum[8], f[8];
    if (!add_up(a, side, places, place, part, sum)) return;
    const uint32_t piece = threadIdx.x;                  // of group 0
    factors(a.scale, piece, f);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] *= f[e];
    put(a.gw + (uint64_t)key * a.C + piece * 8, sum);
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
    const dim3 grid((unsigned)(want < 4096 ? want : 4096)), block(r.threads);
    if (bf16) emb::lookup_kernel<rows::bf16><<<grid, block, 0, stream>>>(a);
    else emb::lookup_kernel<float><<<grid, block, 0, stream>>>(a);
    return hipGetLastError();
}

size_t embedding_bwd_workspace_bytes(long long n, int V, int C) { return emb::plan_for(n, V, C).bytes; }

// Workgroups that fill gw beside a sort: no more than there is work for, and three to a compute unit.  512 / 768 / 1024 / 2048 for V = 131072, C = 2048: 260 / 248 /
// 264 / 271 us; for V = 30522, C = 768: 58 / 57 / 58 / 57.
static uint32_t fillers(const emb::Args &a, uint32_t eighths, uint32_t threads) {
    const uint64_t want = (uint64_t)a.V * a.C / 4 * eighths / 8 / (threads * 4) + 1, most = threads == 256 ? 768 : 256;        // as many threads
    return (uint32_t)(want < most ? want : most);
}

template <int ROUNDS>
static void sort(const emb::Args &a, hipStream_t stream) {
    const dim3 counting(a.blocks + fillers(a, 1, 256)), scattering(a.blocks + fillers(a, 3, 256)), block(256);
    emb::count_kernel<true, ROUNDS><<<counting, block, 0, stream>>>(a);
    emb::scatter_kernel<true, ROUNDS><<<scattering, block, 0, stream>>>(a);
    emb::count_kernel<false, ROUNDS><<<counting, block, 0, stream>>>(a);
    emb::scatter_kernel<false, ROUNDS><<<scattering, block, 0, stream>>>(a);
}

template <typename T>
static hipError_t embedding_bwd(const emb::Args &a, hipStream_t stream) {
    using namespace emb;
    if (a.in_lds == 1024) {
        sort_kernel<256, 4, 5><<<dim3(1 + fillers(a, 8, 256)), dim3(256), 0, stream>>>(a);
    } else if (a.in_lds == 4096) {
        sort_kernel<1024, 4, 4><<<dim3(1 + fillers(a, 8, 1024)), dim3(1024), 0, stream>>>(a);
    } else if (a.in_lds) {
        sort_kernel<1024, 8, 4><<<dim3(1 + fillers(a, 8, 1024)), dim3(1024), 0, stream>>>(a);
    } else if (a.rounds == 1) {
        sort<1>(a, stream);
    } else if (a.rounds == 2) {
        sort<2>(a, stream);
    } else if (a.rounds == 8) {
        sort<8>(a, stream);
    } else {
        sort<32>(a, stream);
    }
    const uint32_t threads = (a.pieces + 63) / 64 * 64;
    sums_kernel<T><<<dim3(a.chunks), dim3(threads), 0, stream>>>(a);
    if (a.chunks > 1) {
        const uint32_t side = groups_of(a.pieces);
        const dim3 block((a.pieces * side + 63) / 64 * 64);
        const size_t lds = side * a.C * sizeof(float);
        if (a.span) {
            spans_kernel<<<dim3(a.chunks / a.span), block, lds, stream>>>(a, side);
            joins_kernel<true><<<dim3(a.chunks - 1), block, lds, stream>>>(a, side);
        } else {
            joins_kernel<false><<<dim3(a.chunks - 1), block, lds, stream>>>(a, side);
        }
    }
    return hipGetLastError();
}

// gw [V][C] fp32, every row written.  gy [n, C] in bf16 or fp32; a workspace of embedding_bwd_workspace_bytes, 16-byte aligned.
hipError_t launch_embedding_bwd(const void *id, const void *gy, const float *scale, float *gw, long long n, int V, int C, int bf16, void *workspace,
                                size_t workspace_bytes, hipStream_t stream) {
    if (embedding_check(gy, scale, n, V, C) || !id || !gw || !workspace || ((uintptr_t)workspace & 15)) return hipErrorInvalidValue;
    const emb::Plan p = emb::plan_for(n, V, C);
    if (workspace_bytes < p.bytes) return hipErrorInvalidValue;
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    auto u32 = [&](uint64_t o) { return reinterpret_cast<uint32_t *>(ws + o); };
    emb::Args a;
    a.id = static_cast<const int64_t *>(id); a.gy = static_cast<const unsigned char *>(gy); a.scale = scale; a.gw = gw;
    a.key1 = u32(p.key1); a.pos1 = u32(p.pos1); a.key2 = u32(p.key2); a.pos2 = u32(p.pos2);
    a.hist1 = u32(p.hist1); a.hist2 = u32(p.hist2);
    a.sums = reinterpret_cast<float *>(ws + p.sums);
    a.n = p.n; a.V = p.V; a.C = p.C; a.bits = p.bits; a.bits1 = p.bits1; a.bits2 = p.bits2; a.in_lds = p.in_lds; a.rounds = p.rounds; a.blocks = p.blocks;
    a.chunk = p.chunk; a.chunks = p.chunks; a.span = p.span; a.pieces = (uint32_t)C / 8;
    return bf16 ? embedding_bwd<rows::bf16>(a, stream) : embedding_bwd<float>(a, stream);
}

}  // namespace delta
