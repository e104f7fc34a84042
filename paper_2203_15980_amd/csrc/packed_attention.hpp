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
    float *delta;                                        // [heads][M], sum over a row's channels of y gy; then [heads][M] log2-sum-exp
    float *part;                                         // null or [splits][M][2 kv D]: sums of gk and gv over a share of a key head's query heads
    int M, seqs, heads, kv, slots, splits;
    float scale, scale_log2e;                            // 1 / sqrt(D), times log2 e
};

// Keys to a block of a group's: four groups' blocks of 128 channels fit the LDS as half ones only.
template <int D, int G> constexpr int kKeys = D == 128 && G == 4 ? 32 : 64;

// Groups of wavefronts that share a tile's work: a workgroup is 4 wavefronts, each with 32 rows, and with 2 or 4 groups the tile is 64 or 32 rows and a group takes every
// second or fourth block of what the rows meet.  Four groups until the chip has a workgroup to each CU (long sequences: two), two until it has about
// four (heads of 128, whose blocks leave room for one on a CU: two).  us with 1, 2 and 4 groups, forward, then gradients, causal:
//   tokens x heads (key heads) of channels   forward            gradients
//   200 x 12 (12) of 64                      6.3, 5.7, 5.2      19.1, 15.7, 13.6
//   512 x 12 (12) of 64                      9.7, 7.6, 6.4      29.8, 21.5, 16.8
//   4096 x 4 (1) of 64                       50, 34, 28         183, 118, 84
//   2048 x 32 (4) of 64                      32, 32, 65         119, 98, 195
//   1024 x 8 (2) of 128                      24, 16, 14         90, 61, 46
//   1024 x 32 (8) of 128                     25, 23, 37         111, 88, 120
//   2048 x 32 (8) of 128                     51, 66, 107        217, 268, 342
inline int groups_of(long long M, long long seqs, int units, int D) {
    const long long tiles = (M + 31) / 32 * units;
    if (tiles <= 256 || (tiles <= 512 && M >= 1024 * seqs)) return 4;
    return tiles <= (D == 64 ? 2048 : 1024) ? 2 : 1;
}

// Rows of a workgroup: `tile` of the segment [start, start + len).  Segments: the rows before the first sequence, the sequences, the rows behind the last
// (the first and the last belong to no sequence: `alone`).  Boundaries are held in [0, M], so that no offset leads out of the tensors.
//
// The lengths are known to the device alone, so a launch has a slot for every tile there may be, sum of ceil(len / Q) <= M / Q + segments; slots left over end at once.
struct Rows { int start, len, tile; bool alone; };

__device__ __forceinline__ int boundary(const Args &a, int j) {                    // of segment j's first row; j = seqs + 2: M
    if (j == 0) return 0;
    if (j == a.seqs + 2) return a.M;
    const long long o = a.off[j - 1];
    return o < 0 ? 0 : o > a.M ? a.M : (int)o;
}
inline int slots_of(int M, int seqs, int Q) { return M / Q + seqs + 2; }

__device__ __forceinline__ int wave_sum(int v) {
    v += (int)rows::dpp<0xB1>((uint32_t)v);
    v += (int)rows::dpp<0x4E>((uint32_t)v);
    v += (int)rows::dpp<0x141>((uint32_t)v);
    v += (int)rows::dpp<0x140>((uint32_t)v);
    auto r = __builtin_amdgcn_permlane16_swap((uint32_t)v, (uint32_t)v, false, false);
    v = (int)(r[0] + r[1]);
    r = __builtin_amdgcn_permlane32_swap((uint32_t)v, (uint32_t)v, false, false);
    return __builtin_amdgcn_readfirstlane((int)(r[0] + r[1]));
}
// The index of the n-th set bit.
__device__ __forceinline__ int nth_bit(unsigned long long bits, int n) {
    for (; n > 0; --n) bits &= bits - 1;
    return __builtin_ctzll(bits);
}

// The rows of the `slot`-th tile to begin.  False: there is none.
// 2 to 62 sequences, a lane to a segment: the tiles with the most work go first, whichever sequences they are of.  Causal that is the tiles of the highest index (of
// sum max(0, n_j - t) tiles of index t or more, n_j to a sequence, the largest t that still has more than `slot` is looked for); else those of the longest sequences.
// One, or more: segment j's tiles take the slots from floor(start_j / Q) + j on, in order, the last ones first; they have room, as
// ceil(len / Q) <= floor((start + len) / Q) - floor(start / Q) + 1.
// 9 sequences of up to 1531, 16 heads of 128, causal: forward 55 us in the order of the slots, 48 like this.  (One sequence needs none of it: 77 tokens 4.9 and 5.8 us.)
template <int Q, bool CAUSAL>
__device__ __forceinline__ bool find_rows(const Args &a, int slots, int slot, Rows &r) {
    const int lane = threadIdx.x & 63, last = a.seqs + 2;
    int lo = 0, n = last, step, at, mine, next;
    if (a.seqs > 1 && n <= 64) {
        mine = boundary(a, lane < last ? lane : last);
        next = boundary(a, lane + 1 < last ? lane + 1 : last);
        const bool alone = lane == 0 || lane == last - 1;
        const int tiles = next > mine ? (next - mine + Q - 1) / Q : 0, full = alone ? 0 : tiles;
        int most = full;
        most = max(most, (int)rows::dpp<0xB1>((uint32_t)most));
        most = max(most, (int)rows::dpp<0x4E>((uint32_t)most));
        most = max(most, (int)rows::dpp<0x141>((uint32_t)most));
        most = max(most, (int)rows::dpp<0x140>((uint32_t)most));
        most = max(max(__builtin_amdgcn_readlane(most, 0), __builtin_amdgcn_readlane(most, 16)), max(__builtin_amdgcn_readlane(most, 32), __builtin_amdgcn_readlane(most, 48)));
        const int all = wave_sum(full);
        if (slot < all) {
            // the largest v with more than `slot` tiles at or above it; `above`: those above it
            int v = 0, top = most, above = 0;                                      // v has more, top has not
            while (top - v > 1) {
                const int mid = (v + top) / 2, here = wave_sum(CAUSAL ? max(0, full - mid) : full > mid ? full : 0);
                if (here > slot) v = mid;
                else { top = mid; above = here; }
            }
            const int rest = slot - above;
            if (CAUSAL) {                                // the tiles of index v
                at = nth_bit(__ballot(full > v), rest);
                r.tile = v;
            } else {                                     // the sequences of v + 1 tiles
                at = nth_bit(__ballot(full == v + 1), rest / (v + 1));
                r.tile = rest % (v + 1);
            }
            r.alone = false;
        } else {
            const int rest = slot - all, first = __builtin_amdgcn_readlane(tiles, 0);
            at = rest < first ? 0 : last - 1;
            r.tile = rest < first ? rest : rest - first;
            r.alone = true;
        }
        at = __builtin_amdgcn_readfirstlane(at);
    } else {
        slot = slots - 1 - slot;
        do {
            step = (n + 63) / 64;
            const int j = lo + lane * step;
            mine = boundary(a, j < last ? j : last);
            next = boundary(a, j + 1 < last ? j + 1 : last);                       // of use where step is 1
            const bool before = lane * step < n && mine / Q + j <= slot;
            at = __builtin_popcountll(__ballot(before)) - 1;                       // lane 0's segment begins at or before the slot
            at = at < 0 ? 0 : at;
            lo += at * step;
            n = n - at * step < step ? n - at * step : step;
        } while (step > 1);
        lo = __builtin_amdgcn_readfirstlane(lo);
        at = __builtin_amdgcn_readfirstlane(at);
        r.tile = slot - (__builtin_amdgcn_readlane(mine, at) / Q + lo);
        r.alone = lo == 0 || lo == a.seqs + 1;
    }
    r.start = __builtin_amdgcn_readlane(mine, at);
    r.len = __builtin_amdgcn_readlane(next, at) - r.start;
    r.tile = __builtin_amdgcn_readfirstlane(r.tile);
    return r.tile >= 0 && r.tile * (long long)Q < r.len;
}

// Consecutive workgroups go to the 8 XCDs in turn, each with an L2 of its own: numbered like this, an XCD's heads are neighbours, which share keys and values.
__device__ __forceinline__ int head_of(int i, int heads) { return heads % 8 ? i : (i & 7) * (heads >> 3) + (i >> 3); }
// A workgroup's head and slot, of `units` heads.  Not causal, an XCD takes a run of one head's slots after the other's.
template <bool CAUSAL>
__device__ __forceinline__ void place_of(unsigned i, unsigned n, int units, int slots, int &unit, int &slot) {       // workgroup i of n
    if (CAUSAL) {
        unit = head_of((int)(i % (unsigned)units), units);
        slot = (int)(i / (unsigned)units);
    } else {
        const unsigned per = n >> 3, rem = n & 7u, xcd = i & 7u, k = xcd * per + (xcd < rem ? xcd : rem) + (i >> 3);
        unit = (int)(k / (unsigned)slots);
        slot = (int)(k % (unsigned)slots);
    }
}

// A tile of rows of D bf16 channels in LDS, without padding: piece p (16 bytes) of row r lies at piece p ^ twist(r) of its row, so that both ways of
// reading it below meet each bank as seldom as can be: 16 lanes that read one piece of 16 rows, and 32 that read 64 bytes of four rows.
template <int D, int ROWS = 64> constexpr int kTile = ROWS * D * 2;
template <int D>
__device__ __forceinline__ constexpr int twist(int r) {
    return D == 128 ? (r & 3) << 2 | (r >> 2 & 3) : (r >> 1 & 1) << 2 | (r >> 2 & 3);
}

// Rows of memory straight into such a tile, by W wavefronts: `base` is the tile's first row, at most `rows` of its rows are there (the others come as the last of
// those).  Whoever reads the tile waits (arrived) and meets the others' barrier first.
template <int D, int W, int ROWS = 64>
struct Loader {
    static constexpr int kRows = 64 * 16 / (D * 2), kTurns = ROWS / (kRows * W);   // rows of a wavefront's load; loads to a tile
    static_assert(kTurns * kRows * W == ROWS, "whole loads");
    int row, lds;
    __device__ __forceinline__ Loader(int wave) {
        row = wave * kRows + (int)(threadIdx.x & 63) / (D / 8);
        lds = wave * kRows * D * 2;
    }
    __device__ __forceinline__ void load(const unsigned char *base, uint32_t pitch, int rows, uint32_t tile) const {
#pragma unroll W < 4 && kTurns > 2 ? 2 : kTurns
        for (int t = 0; t < kTurns; ++t) {
            const int r = row + t * kRows * W;
            const uint32_t piece = (uint32_t)(((int)(threadIdx.x & 63) % (D / 8)) ^ twist<D>(r)) * 16;
            load_lds_b128(base, (uint32_t)(r < rows ? r : rows - 1) * pitch + piece, tile + (uint32_t)(lds + t * kRows * W * D * 2));
        }
    }
};
__device__ __forceinline__ void arrived() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ uint32_t lds_of(const unsigned char *p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const unsigned char *)p; }

// Operand of a 32 x 32 x 16 product out of a tile: row `row` + lane % 32, channels 16 step + 8 (lane / 32) ..
template <int D>
__device__ __forceinline__ bf16x8 rows_of(const unsigned char *tile, int row, int step) {
    const int lane = threadIdx.x & 63, r = row + (lane & 31);
    return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(tile + r * (D * 2) + ((2 * step + (lane >> 5)) ^ twist<D>(lane & 31)) * 16));
}
// The same of the transposed tile: channel 32 block + lane % 32, and the eight rows row + 4 (lane / 32) + {0 .. 3, 8 .. 11} (row a multiple of 16): the rows that a
// lane's eight accumulators of one 32 x 32 product stand for.  ds_read_b64_tr_b16: within 16 lanes, lane j points at row j / 4 and columns 4 (j % 4) .. of a 4 x 16
// block and receives column j of its four rows.
template <int D>
__device__ __forceinline__ bf16x8 columns_of(const unsigned char *tile, int row, int block) {
    typedef s16x4 __attribute__((address_space(3))) * lds_ptr;
    const int lane = threadIdx.x & 63, r = 4 * (lane >> 5) + ((lane & 15) >> 2), piece = 4 * block + 2 * (lane >> 4 & 1) + (lane >> 1 & 1);
    const unsigned char *p = tile + (row + r) * (D * 2) + (lane & 1) * 8;
    const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p + (piece ^ twist<D>(r)) * 16));
    const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(p + 8 * (D * 2) + (piece ^ twist<D>(r + 8)) * 16));
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

// The same times `by` in fp32, [channel] from `out` on.
template <int BLOCKS>
__device__ __forceinline__ void store_column(float *out, const f32x16 (&o)[BLOCKS], float by) {
    const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int t = 0; t < BLOCKS; ++t)
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4)
            *reinterpret_cast<f32x4 *>(out + 32 * t + 8 * e4 + 4 * half) = f32x4{o[t][4 * e4] * by, o[t][4 * e4 + 1] * by, o[t][4 * e4 + 2] * by, o[t][4 * e4 + 3] * by};
}

// Sums of the W wavefronts of one group on their way through LDS to those of another: register e of a lane at [wavefront][e][lane].
template <int BLOCKS>
__device__ __forceinline__ void hand_over(float *lds, int wave, const f32x16 (&o)[BLOCKS]) {
    float *at = lds + wave * BLOCKS * 16 * 64 + (threadIdx.x & 63);
#pragma unroll
    for (int t = 0; t < BLOCKS; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) at[(t * 16 + e) * 64] = o[t][e];
}
template <int BLOCKS>
__device__ __forceinline__ void take_over(const float *lds, int wave, f32x16 (&o)[BLOCKS], float by) {
    const float *at = lds + wave * BLOCKS * 16 * 64 + (threadIdx.x & 63);
#pragma unroll
    for (int t = 0; t < BLOCKS; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[t][e] += at[(t * 16 + e) * 64] * by;
}

// Zeros to `n` rows of `bytes` (a multiple of 16) each.
__device__ __forceinline__ void zero_rows(unsigned char *p, size_t pitch, int n, int bytes) {
    const int per = bytes / 16;
    for (int i = threadIdx.x; i < n * per; i += blockDim.x) *reinterpret_cast<u32x4 *>(p + (size_t)(i / per) * pitch + (i % per) * 16) = u32x4{0u, 0u, 0u, 0u};
}

}  // namespace pat
}  // namespace delta
