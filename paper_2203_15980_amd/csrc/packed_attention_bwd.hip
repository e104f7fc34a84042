// The gradients of attention over packed sequences (packed_attention.hip) for gfx950.  With p = exp(s - lse), s = q k^T / sqrt D:
//   delta = sum over a row's channels of ctx gctx,  dp = gctx v^T,  ds = p (dp - delta)
//   gq = ds k / sqrt D,  gk = ds^T q / sqrt D,  gv = p^T gctx, gk and gv summed over the query heads of their key head
// Two launches and no atomics: one owns queries (delta, which it leaves for the other, and gq), one owns keys and walks through the queries of all its heads
// in order, so that a gradient's bits depend on its inputs alone.  Scores are formed twice: 7 products where 5 would do, against 32-bit sums of gq that would
// have to meet across workgroups.
//   gq: as the forward kernel, a lane owns a query: S^T = K Q^T, dP^T = V gO^T, gQ^T += K^T dS^T.
//   gk, gv: a lane owns a key: S = Q K^T, dP = gO V^T, gV^T += gO^T P, gK^T += Q^T dS; queries and their gradients come through LDS.
// p and ds are rounded to bf16 before they multiply, and delta reads ctx as it was stored, in bf16: three roundings of about the size of the result's own (0.0017 of the gradient
// each; together 0.0024 to 0.0026 against 64 bits with sequences of hundreds and more, up to 0.0031 with tens, 0.0036 with two rows); all sums are fp32.
//
// Bound by the SIMDs as the forward kernel is.  8192 tokens, 32 heads over 8 of 128, causal: gq 735 to 770 us (825 GFLOP: 1070 to 1120 TFLOP/s, the matrix units 61 to 64 % busy), gk and gv
// 1010 to 1080 us (1100 GFLOP: 1020 to 1090 TFLOP/s) and 25 for the parts; counted as five products 800 TFLOP/s.  32 sequences of up to 512, 12 heads of 64, not causal: 36 and 50 us.
// 77 tokens, 12 heads of 64, one launch: 8 us.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.hpp"
#include "packed_attention.hpp"

namespace delta {
namespace pat {

constexpr float kLog2e = 1.4426950408889634f;
template <int D, int G> constexpr int kPair = 2 * kTile<D, kKeys<D, G>>;           // K and V of a block

// W wavefronts of 32 queries each, G times: the groups take turns at the blocks of keys, and their sums meet in LDS.
template <int D, int W, int G, bool CAUSAL>
__device__ __forceinline__ void gq_tile(const Args &a, unsigned block, unsigned blocks_of_launch, unsigned char *smem) {
    constexpr int Q = W * 32, KS = D / 16, DB = D / 32, kStep = kKeys<D, G>;
    const int lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)) % W, group = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)) / W;
    int head, slot;
    place_of<CAUSAL>(block, blocks_of_launch, a.heads, a.slots, head, slot);
    Rows r;
    if (!find_rows<Q, CAUSAL>(a, a.slots, slot, r)) return;
    const size_t out_pitch = (size_t)a.heads * D * 2, pitch = (size_t)(a.heads + 2 * a.kv) * D * 2;
    const int q0 = r.tile * Q;
    unsigned char *gxb = a.gx + (size_t)r.start * pitch + (size_t)head * D * 2;
    if (r.alone) {
        zero_rows(gxb + (size_t)q0 * pitch, pitch, r.len - q0 < Q ? r.len - q0 : Q, D * 2);
        return;
    }
    const unsigned char *xb = a.x + (size_t)r.start * pitch;
    const int kh = head / (a.heads / a.kv);
    const unsigned char *kb = xb + (size_t)(a.heads + kh) * D * 2, *vb = kb + (size_t)a.kv * D * 2;
    const int w0 = q0 + 32 * wave, q = w0 + l32;
    const bool there = q < r.len;
    const int row = there ? q : r.len - 1;
    bf16x8 qf[KS], gf[KS];
    float delta = 0.f;
    {
        const unsigned char *p = xb + (size_t)row * pitch + (size_t)head * D * 2 + half * 16;
        const size_t at = ((size_t)r.start + row) * out_pitch + (size_t)head * D * 2 + half * 16;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            qf[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(p + s * 32));
            rows::Eight<rows::bf16> g, y;
            g.load(a.gy + at + s * 32);
            y.load(a.y + at + s * 32);
            gf[s] = __builtin_bit_cast(bf16x8, g.raw);
            float u[8], v[8];
            g.to(u);
            y.to(v);
#pragma unroll
            for (int e = 0; e < 8; ++e) delta += u[e] * v[e];
        }
    }
    delta = rows::halves(delta);
    const size_t stat = (size_t)head * a.M + r.start + row;
    const float lse2 = a.lse[stat] * kLog2e;
    if (there && !half && !group) {
        a.delta[stat] = delta;
        a.delta[(size_t)a.heads * a.M + stat] = lse2;
    }
    f32x16 g[DB];
#pragma unroll
    for (int t = 0; t < DB; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) g[t][e] = 0.f;
    const int keys = CAUSAL && q0 + Q < r.len ? q0 + Q : r.len, blocks = (keys + kStep - 1) / kStep;
    const int limit = CAUSAL && q + 1 < r.len ? q + 1 : r.len;
    const Loader<D, W, kStep> loader(wave);
    const uint32_t lds = lds_of(smem) + (uint32_t)group * 2 * kPair<D, G>;
    auto load = [&](int i) {
        const int b = i * G + group;
        if (b >= blocks) return;
        const uint32_t at = lds + (uint32_t)(i & 1) * kPair<D, G>;
        const size_t from = (size_t)b * kStep * pitch;
        loader.load(kb + from, (uint32_t)pitch, r.len - b * kStep, at);
        loader.load(vb + from, (uint32_t)pitch, r.len - b * kStep, at + kTile<D, kStep>);
    };
    load(0);
    for (int i = 0; i * G < blocks; ++i) {
        arrived();
        __syncthreads();                                 // the block is there; the one before is done with
        load(i + 1);
        const unsigned char *ks = smem + (group * 2 + (i & 1)) * kPair<D, G>, *vs = ks + kTile<D, kStep>;
        const int k0 = (i * G + group) * kStep;
        if (k0 < keys && w0 < r.len && (!CAUSAL || k0 <= w0 + 31)) {
            const bool border = k0 + kStep > (CAUSAL ? (w0 + 1 < r.len ? w0 + 1 : r.len) : r.len);
            const int lim = border ? limit - k0 - 4 * half : kStep;
#pragma unroll 1
            for (int t = 0; t < kStep / 32; ++t) {
                __builtin_amdgcn_sched_barrier(0);       // one tile after the other: both at once do not fit the registers
                f32x16 s, dp;
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] = dp[e] = 0.f;
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    s = mfma(rows_of<D>(ks, 32 * t, k), qf[k], s);
                    dp = mfma(rows_of<D>(vs, 32 * t, k), gf[k], dp);
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], a.scale_log2e, -lse2));
                    s[e] = p * (dp[e] - delta);
                }
                if (__builtin_expect(border, 0)) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[e] = 32 * t + row_of(e) < lim ? s[e] : 0.f;
                    asm volatile("" ::: "memory");
                }
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const bf16x8 ds = as_operand(s, j);
#pragma unroll
                    for (int d = 0; d < DB; ++d) g[d] = mfma(columns_of<D>(ks, 32 * t + 16 * j, d), ds, g[d]);
                }
            }
        }
    }
    if constexpr (G > 1) {
        __syncthreads();                                 // the last blocks are done with
        float *sums = reinterpret_cast<float *>(smem);
        if (group) hand_over(sums, (group - 1) * W + wave, g);
        __syncthreads();
        if (group) return;
#pragma unroll
        for (int other = 0; other < G - 1; ++other) take_over(sums, other * W + wave, g, 1.0f);
    }
    if (there) store_column<DB>(gxb + (size_t)q * pitch, g, a.scale);
}

// Heads of 128: a lane's sums of gk and gv, its key and its value would be 192 registers of the 256 that two wavefronts to a SIMD leave: the values stay in LDS, and the order of
// reads is held apart (sched_barrier) where the compiler would fetch ahead of the registers.  On a full chip 8 wavefronts share a block of 64 queries, one workgroup to a CU: 8192 tokens 1010 to
// 1080 us; two workgroups of 4, each with blocks of 32 queries, 1160 to 1260.
template <int D, int W> constexpr int kQueries = D == 128 && W < 8 ? 32 : 64;
template <int D, int W, int G> constexpr int kKvLds = G * 4 * kTile<D, kQueries<D, W>> + (D == 128 ? kTile<D, W * 32> : 0);

// OWN: with delta made here, for all queries that the keys may meet, instead of read: both kernels are one launch then.
constexpr int kOwn = 2048;
template <int D, int W, int G, bool CAUSAL, bool OWN>
__device__ __forceinline__ void gkv_tile(const Args &a, unsigned workgroup, unsigned workgroups, unsigned char *smem) {
    constexpr int K = W * 32, KS = D / 16, DB = D / 32, Q = kQueries<D, W>;
    constexpr bool kValuesInLds = D == 128;
    __shared__ __align__(16) float own[OWN ? kOwn : 4];  // [head of the share][query, to whole blocks]
    __shared__ __align__(16) float stats[G][2][2][Q];    // of a block's queries: log-sum-exp (log2), delta
    const int lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5, thread = (int)threadIdx.x % (W * 64);
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)) % W, group = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)) / W;
    int unit, slot;
    place_of<CAUSAL>(workgroup, workgroups, a.kv * a.splits, a.slots, unit, slot);
    const int kh = unit / a.splits, split = unit % a.splits;
    Rows r;
    if (!find_rows<K, CAUSAL>(a, a.slots, slot, r)) return;
    if (CAUSAL) r.tile = (r.len - 1) / K - r.tile;       // a sequence's first keys have the most queries
    const size_t out_pitch = (size_t)a.heads * D * 2, pitch = (size_t)(a.heads + 2 * a.kv) * D * 2;
    const int first = r.tile * K, share = a.heads / a.kv / a.splits;                // query heads of this workgroup
    unsigned char *gkb = a.gx + (size_t)r.start * pitch + (size_t)(a.heads + kh) * D * 2, *gvb = gkb + (size_t)a.kv * D * 2;
    float *part = a.part ? a.part + (((size_t)split * a.M + r.start) * 2 * a.kv + kh) * D : nullptr;
    if (r.alone) {
        const int n = r.len - first < K ? r.len - first : K;
        if (a.part) {
            unsigned char *at = reinterpret_cast<unsigned char *>(part) + (size_t)first * 2 * a.kv * D * 4;
            zero_rows(at, (size_t)2 * a.kv * D * 4, n, D * 4);
            zero_rows(at + (size_t)a.kv * D * 4, (size_t)2 * a.kv * D * 4, n, D * 4);
        } else {
            zero_rows(gkb + (size_t)first * pitch, pitch, n, D * 2);
            zero_rows(gvb + (size_t)first * pitch, pitch, n, D * 2);
        }
        return;
    }
    const unsigned char *xb = a.x + (size_t)r.start * pitch;
    const int w0 = first + 32 * wave, key = w0 + l32;
    const bool there = key < r.len;
    const uint32_t lds = lds_of(smem) + (uint32_t)group * 4 * kTile<D, Q>;
    const unsigned char *tiles = smem + group * 4 * kTile<D, Q>, *values = smem + G * 4 * kTile<D, Q>;
    bf16x8 kf[KS], vf[kValuesInLds ? 1 : KS];
    {
        const unsigned char *p = xb + (size_t)(there ? key : r.len - 1) * pitch + (size_t)(a.heads + kh) * D * 2 + half * 16;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            kf[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(p + s * 32));
            if constexpr (!kValuesInLds) vf[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(p + (size_t)a.kv * D * 2 + s * 32));
        }
    }
    if constexpr (kValuesInLds) {                        // 64 rows from a base of their own: their offsets stay within 32 bits
        constexpr int kRows = K < 64 ? K : 64;
#pragma unroll
        for (int at = 0; at < K; at += kRows)
            if (first + at < r.len)                      // (the wavefronts of keys behind the last do nothing)
                Loader<D, W * G, kRows>(group * W + wave).load(xb + (size_t)(first + at) * pitch + (size_t)(a.heads + a.kv + kh) * D * 2, (uint32_t)pitch, r.len - first - at,
                                                               lds_of(values) + (uint32_t)(at * D * 2));
    }
    f32x16 gk[DB], gv[DB];
#pragma unroll
    for (int t = 0; t < DB; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) gk[t][e] = gv[t][e] = 0.f;
    const int begin = CAUSAL ? first / Q : 0, per = (r.len + Q - 1) / Q - begin;
    const Loader<D, W, Q> loader(wave);
    const uint32_t lds_stats = lds_of(reinterpret_cast<const unsigned char *>(&stats[group][0][0][0]));
    float lse2 = 0.f;                                    // OWN: of the block on its way, query `thread`
    static_assert(Q <= W * 64, "a query to a thread");
    auto load = [&](int head, int at, int buffer) {
        const uint32_t to = lds + (uint32_t)buffer * 2 * kTile<D, Q>;
        loader.load(xb + (size_t)at * pitch + (size_t)head * D * 2, (uint32_t)pitch, r.len - at, to);
        loader.load(a.gy + ((size_t)r.start + at) * out_pitch + (size_t)head * D * 2, (uint32_t)out_pitch, r.len - at, to + kTile<D, Q>);
        if constexpr (OWN) {
            if (thread < Q) lse2 = a.lse[(size_t)head * a.M + r.start + (at + thread < r.len ? at + thread : r.len - 1)] * kLog2e;
        } else {                                         // 64 numbers to a wavefront's load: the log-sum-exps, then the deltas, of Q queries
#pragma unroll
            for (int part = 0; part < 2 * Q / 64; ++part)
                if (wave == part % W) {
                    const int i = part * 64 + lane, q = at + i % Q;
                    const float *from = a.delta + (i < Q ? (size_t)a.heads * a.M : 0) + (size_t)head * a.M + r.start + (q < r.len ? q : r.len - 1);
                    load_lds_b32(from, lds_stats + (uint32_t)(buffer * 2 * Q + part * 64) * 4);
                }
        }
    };
    // Each head's queries from the last block on backwards: causal, workgroups on an XCD begin at the same block and find it in its L2.  The groups take turns at the
    // blocks of all heads in one row.
    const int end = (kh * a.splits + split + 1) * share;
    int head = end - share, block = per - 1, buffer = 0;
    auto go_on = [&](int n) {
        for (block -= n; block < 0; block += per) ++head;
    };
    go_on(group);
    if (head < end) load(head, (begin + block) * Q, 0);
    const int span = (begin + per) * Q;
    if constexpr (OWN) {
        const int part = (int)threadIdx.x & 3;
        for (int i = (int)threadIdx.x >> 2; i < share * span; i += W * G * 16) {
            const int h = i / span, q = i - h * span;
            float sum = 0.f;
            if (q < r.len) {
                const size_t at = ((size_t)r.start + q) * out_pitch + (size_t)(end - share + h) * D * 2 + part * (D / 2);
#pragma unroll
                for (int c = 0; c < D / 32; ++c) {
                    rows::Eight<rows::bf16> g, y;
                    g.load(a.gy + at + c * 16);
                    y.load(a.y + at + c * 16);
                    float u[8], v[8];
                    g.to(u);
                    y.to(v);
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum += u[e] * v[e];
                }
            }
            sum += rows::dpp<0xB1>(sum);
            sum += rows::dpp<0x4E>(sum);
            if (!part) own[i] = sum;
        }
    }
    for (int i = 0; i * G < per * share; ++i) {
        if (OWN && thread < Q) stats[group][buffer][0][thread] = lse2;
        arrived();
        __syncthreads();                                 // the block is there; the one before is done with
        const int at = (begin + block) * Q;
        const bool some = head < end;
        const float *deltas = OWN ? own + (some ? head - (end - share) : 0) * span + at : stats[group][buffer][1];
        go_on(G);
        if (head < end) load(head, (begin + block) * Q, buffer ^ 1);
        const unsigned char *qs = tiles + buffer * 2 * kTile<D, Q>, *gs = qs + kTile<D, Q>;
        if (some && w0 < r.len && (!CAUSAL || at + Q - 1 >= w0)) {
#pragma unroll D == 128 ? 1 : 2
            for (int t = 0; t < Q / 32; ++t) {
                __builtin_amdgcn_sched_barrier(0);       // one tile after the other
                f32x16 s, dp;
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] = dp[e] = 0.f;
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    s = mfma(rows_of<D>(qs, 32 * t, k), kf[k], s);
                    if constexpr (kValuesInLds) dp = mfma(rows_of<D>(gs, 32 * t, k), rows_of<D>(values, 32 * wave, k), dp);
                    else dp = mfma(rows_of<D>(gs, 32 * t, k), vf[k], dp);
                }
#pragma unroll
                for (int e4 = 0; e4 < 4; ++e4) {
                    const f32x4 l = *reinterpret_cast<const f32x4 *>(&stats[group][buffer][0][32 * t + 8 * e4 + 4 * half]);
                    const f32x4 dl = *reinterpret_cast<const f32x4 *>(deltas + 32 * t + 8 * e4 + 4 * half);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[4 * e4 + e], a.scale_log2e, -l[e]));
                        s[4 * e4 + e] = p;
                        dp[4 * e4 + e] = p * (dp[4 * e4 + e] - dl[e]);
                    }
                }
                if (__builtin_expect((CAUSAL && at + 32 * t < w0 + 31) || at + 32 * t + 32 > r.len, 0)) {
                    // the rows of the product that see this key: causal from its own on, and queries of the sequence
                    const int from = CAUSAL ? key - at - 32 * t - 4 * half : -64, to = r.len - at - 32 * t - 4 * half;
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const bool sees = row_of(e) >= from && row_of(e) < to;
                        s[e] = sees ? s[e] : 0.f;
                        dp[e] = sees ? dp[e] : 0.f;
                    }
                    asm volatile("" ::: "memory");
                }
                if (D == 128) __builtin_amdgcn_sched_barrier(0);                   // nor the products' operands before the weights are bf16
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const bf16x8 p = as_operand(s, j), ds = as_operand(dp, j);
#pragma unroll
                    for (int d = 0; d < DB; ++d) {
                        gv[d] = mfma(columns_of<D>(gs, 32 * t + 16 * j, d), p, gv[d]);
                        gk[d] = mfma(columns_of<D>(qs, 32 * t + 16 * j, d), ds, gk[d]);
                    }
                }
            }
        }
        buffer ^= 1;
    }
    if constexpr (G > 1) {
        float *sums = reinterpret_cast<float *>(smem);
        __syncthreads();                                 // the last blocks are done with
        if (group) hand_over(sums, (group - 1) * W + wave, gk);
        __syncthreads();
        if (!group)
#pragma unroll
            for (int other = 0; other < G - 1; ++other) take_over(sums, other * W + wave, gk, 1.0f);
        __syncthreads();
        if (group) hand_over(sums, (group - 1) * W + wave, gv);
        __syncthreads();
        if (group) return;
#pragma unroll
        for (int other = 0; other < G - 1; ++other) take_over(sums, other * W + wave, gv, 1.0f);
    }
    if (!there) return;
    if (a.part) {
        store_column<DB>(part + (size_t)key * 2 * a.kv * D, gk, a.scale);
        store_column<DB>(part + ((size_t)key * 2 + 1) * a.kv * D, gv, 1.0f);
    } else {
        store_column<DB>(gkb + (size_t)key * pitch, gk, a.scale);
        store_column<DB>(gvb + (size_t)key * pitch, gv, 1.0f);
    }
}

// gk and gv of a row (of `n` channels, a multiple of 8) as the sums of their parts, in order.
__global__ __launch_bounds__(256) void join_kernel(Args a, uint32_t n, uint32_t pitch, uint32_t at) {
    const uint64_t all = (uint64_t)a.M * (n / 8);
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (uint64_t)gridDim.x * 256) {
        const uint64_t row = i / (n / 8), c = (i - row * (n / 8)) * 8;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = 0.f;
        for (int s = 0; s < a.splits; ++s) {
            const f32x4 *p = reinterpret_cast<const f32x4 *>(a.part + ((uint64_t)s * a.M + row) * n + c);
            const f32x4 lo = p[0], hi = p[1];
#pragma unroll
            for (int e = 0; e < 4; ++e) { v[e] += lo[e]; v[4 + e] += hi[e]; }
        }
        rows::Eight<rows::bf16>::store(a.gx + row * pitch + at + c * 2, v);
    }
}

template <int D, int W, int G, bool CAUSAL>
__global__ __launch_bounds__(W * G * 64, 2) void gq_kernel(Args a) {
    extern __shared__ __align__(16) unsigned char smem[];
    gq_tile<D, W, G, CAUSAL>(a, blockIdx.x, gridDim.x, smem);
}
template <int D, int W, int G, bool CAUSAL>
__global__ __launch_bounds__(W * G * 64, 2) void gkv_kernel(Args a) {
    extern __shared__ __align__(16) unsigned char smem[];
    gkv_tile<D, W, G, CAUSAL, false>(a, blockIdx.x, gridDim.x, smem);
}
template <int D, int W, int G, bool CAUSAL>
__global__ __launch_bounds__(W * G * 64, 2) void both_kernel(Args a, unsigned queries) {
    extern __shared__ __align__(16) unsigned char smem[];
    if (blockIdx.x < queries) gq_tile<D, W, G, CAUSAL>(a, blockIdx.x, queries, smem);
    else gkv_tile<D, W, G, CAUSAL, true>(a, blockIdx.x - queries, gridDim.x - queries, smem);
}

template <typename KERNEL>
static hipError_t allow(KERNEL kernel, int lds) {
    return lds > 64 * 1024 ? hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds) : hipSuccess;
}
template <int D, int W, int G, bool CAUSAL>
static hipError_t launch_gq(Args a, hipStream_t stream) {
    constexpr int kLds = G * 2 * kPair<D, G>;
    static_assert((G - 1) * W * D / 32 * 16 * 64 * 4 <= kLds, "the sums fit where the blocks were");
    const hipError_t e = allow(&gq_kernel<D, W, G, CAUSAL>, kLds);
    if (e != hipSuccess) return e;
    a.slots = slots_of(a.M, a.seqs, W * 32);
    gq_kernel<D, W, G, CAUSAL><<<dim3((unsigned)a.slots * (unsigned)a.heads), dim3(W * G * 64), kLds, stream>>>(a);
    return hipGetLastError();
}
template <int D, int W, int G, bool CAUSAL>
static hipError_t launch_gkv(Args a, hipStream_t stream) {
    constexpr int kLds = kKvLds<D, W, G>;
    static_assert((G - 1) * W * D / 32 * 16 * 64 * 4 <= kLds, "the sums fit where the blocks were");
    const hipError_t e = allow(&gkv_kernel<D, W, G, CAUSAL>, kLds);
    if (e != hipSuccess) return e;
    a.slots = slots_of(a.M, a.seqs, W * 32);
    gkv_kernel<D, W, G, CAUSAL><<<dim3((unsigned)a.slots * (unsigned)(a.kv * a.splits)), dim3(W * G * 64), kLds, stream>>>(a);
    return hipGetLastError();
}
template <int D, bool CAUSAL>
static hipError_t launch_both(Args a, hipStream_t stream) {
    constexpr int W = 1, G = 4, kLdsQ = G * 2 * kPair<D, G>, kLds = kLdsQ > kKvLds<D, W, G> ? kLdsQ : kKvLds<D, W, G>;
    const hipError_t e = allow(&both_kernel<D, W, G, CAUSAL>, kLds);
    if (e != hipSuccess) return e;
    a.slots = slots_of(a.M, a.seqs, W * 32);
    const unsigned queries = (unsigned)a.slots * (unsigned)a.heads;
    both_kernel<D, W, G, CAUSAL><<<dim3(queries + (unsigned)a.slots * (unsigned)(a.kv * a.splits)), dim3(W * G * 64), kLds, stream>>>(a, queries);
    return hipGetLastError();
}

template <int D, bool CAUSAL>
static hipError_t backward(const Args &a, hipStream_t stream) {
    hipError_t e;
    const int gq = groups_of(a.M, a.seqs, a.heads, D), gkv = groups_of(a.M, a.seqs, a.kv * a.splits, D);
    // one launch for both while it has at most two workgroups to a CU (1024 tokens, 12 heads of 64: 38.5 us, two launches 31)
    const long long tiles = (long long)(a.M + 31) / 32 * (a.heads + a.kv * a.splits);
    // and where its threads, 256 to a slot of either kind, are fewer than 2^32, the most that a launch takes; apart they always are (packed_attention_check)
    const long long slots = (long long)slots_of(a.M, a.seqs, 32) * (a.heads + a.kv * a.splits);
    if (gq == 4 && gkv == 4 && tiles <= 512 && slots < 1 << 24 && (long long)(a.heads / a.kv / a.splits) * (a.M + 64) <= kOwn) {
        e = launch_both<D, CAUSAL>(a, stream);
    } else {
        e = gq == 4 ? launch_gq<D, 1, 4, CAUSAL>(a, stream) : gq == 2 ? launch_gq<D, 2, 2, CAUSAL>(a, stream) : launch_gq<D, 4, 1, CAUSAL>(a, stream);
        if (e != hipSuccess) return e;
        e = gkv == 4 ? launch_gkv<D, 1, 4, CAUSAL>(a, stream) : gkv == 2 ? launch_gkv<D, 2, 2, CAUSAL>(a, stream) : launch_gkv<D, D == 128 ? 8 : 4, 1, CAUSAL>(a, stream);
    }
    if (e != hipSuccess || a.splits == 1) return e;
    const uint32_t n = (uint32_t)(2 * a.kv * D);
    const uint64_t pieces = ((uint64_t)a.M * (n / 8) + 255) / 256;
    join_kernel<<<dim3((unsigned)(pieces < 4096 ? pieces : 4096)), dim3(256), 0, stream>>>(a, n, (uint32_t)(a.heads * D * 2) + n * 2, (uint32_t)(a.heads * D * 2));
    return hipGetLastError();
}

// In how many shares a key head's query heads go: as few as give the chip two rounds of its 512 workgroups; of short sequences, where a workgroup has little to do and the
// parts' trip through memory counts for more, half a round.  us of the gradients with 1, 2, 4 and 8 shares (as many as there are query heads), causal:
//   8192 tokens, 32 heads over 8 of 128                     2427, 1798, 1836
//   2048 tokens, 8 heads over 1 of 128                      278, 166, 110, 89
//   9 sequences of up to 1531, 16 heads over 2 of 128       416, 236, 227, 181
//   1 x 512, 4 heads over 1 of 64                           28, 21, 15
//   64 sequences of up to 120, 16 heads over 4 of 128       78, 76, 90
//   100 sequences of up to 80, 32 heads over 4 of 64        62, 71, 78, 92
static int splits_of(long long M, long long seqs, int heads, int kv) {
    const int group = heads / kv;
    const long long tiles = (M + 127) / 128, want = M >= 512 * seqs ? 1024 : 256, there = M >= 512 * seqs ? tiles : tiles + seqs;
    int n = 1;
    while (n < group && (group % n || there * kv * n < want)) ++n;
    return n;
}

}  // namespace pat

// delta and the log-sum-exp in powers of two, and behind them the parts of gk and gv where there are several.
static size_t delta_bytes(long long M, int heads) { return ((size_t)M * heads * 2 * sizeof(float) + 255) / 256 * 256; }
size_t packed_attention_bwd_workspace_bytes(long long M, long long seqs, int Cout, int heads, int kv) {
    const int n = pat::splits_of(M, seqs, heads, kv);
    return delta_bytes(M, heads) + (n > 1 ? (size_t)n * M * 2 * kv * (Cout / heads) * sizeof(float) : 0);
}

// y, lse: what the forward pass left; gy as y; gx as x, all of it written (rows of no sequence with zeros).
hipError_t launch_packed_attention_bwd(const void *x, const void *off, const void *y, const float *lse, const void *gy, void *gx, long long M, long long seqs,
                                       int Cin, int Cout, int heads, int kv, int causal, int bf16, void *workspace, size_t workspace_bytes, hipStream_t stream) {
    if (!x || !off || !y || !lse || !gy || !gx || packed_attention_check(M, seqs, Cin, Cout, heads, kv, bf16)) return hipErrorInvalidValue;
    if (!workspace || workspace_bytes < packed_attention_bwd_workspace_bytes(M, seqs, Cout, heads, kv)) return hipErrorInvalidValue;
    pat::Args a = {};
    a.x = static_cast<const unsigned char *>(x); a.off = static_cast<const long long *>(off);
    a.y = static_cast<unsigned char *>(const_cast<void *>(y)); a.lse = const_cast<float *>(lse);
    a.gy = static_cast<const unsigned char *>(gy); a.gx = static_cast<unsigned char *>(gx); a.delta = static_cast<float *>(workspace);
    a.M = (int)M; a.seqs = (int)seqs; a.heads = heads; a.kv = kv;
    a.splits = pat::splits_of(M, seqs, heads, kv);
    a.part = a.splits > 1 ? reinterpret_cast<float *>(static_cast<unsigned char *>(workspace) + delta_bytes(M, heads)) : nullptr;
    a.scale = 1.0f / sqrtf((float)(Cout / heads));
    a.scale_log2e = a.scale * pat::kLog2e;
    if (Cout / heads == 64) return causal ? pat::backward<64, true>(a, stream) : pat::backward<64, false>(a, stream);
    return causal ? pat::backward<128, true>(a, stream) : pat::backward<128, false>(a, stream);
}

}  // namespace delta
