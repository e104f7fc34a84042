// The gradients of attention over packed sequences (packed_attention.hip) for gfx950.  With p = exp(s - lse), s = q k^T / sqrt D:
//   delta = sum over a row's channels of ctx gctx,  dp = gctx v^T,  ds = p (dp - delta)
//   gq = ds k / sqrt D,  gk = ds^T q / sqrt D,  gv = p^T gctx, gk and gv summed over the query heads of their key head
// Two launches and no atomics: one owns queries (delta, which it leaves for the other, and gq), one owns keys and walks through the queries of all its heads
// in order, so that a gradient's bits depend on its inputs alone.  Scores are formed twice: 7 products where 5 would do, against 32-bit sums of gq that would
// have to meet across workgroups.
//   gq: as the forward kernel, a lane owns a query: S^T = K Q^T, dP^T = V gO^T, gQ^T += K^T dS^T.
//   gk, gv: a lane owns a key: S = Q K^T, dP = gO V^T, gV^T += gO^T P, gK^T += Q^T dS; queries and their gradients come through LDS.
// p and ds are rounded to bf16 before they multiply; all sums are fp32.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.hpp"
#include "packed_attention.hpp"

namespace delta {
namespace pat {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kStep = 64;                                // keys (of gq's kernel) or queries (of the other's) to a block

template <int D> constexpr int kPair = 2 * kTile<D>;                               // two tiles

template <int D, int W, bool CAUSAL>
__global__ __launch_bounds__(W * 64, 2) void gq_kernel(Args a) {
    constexpr int Q = W * 32, KS = D / 16, DB = D / 32;
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), l32 = lane & 31, half = lane >> 5;
    int head, slot;
    place_of<CAUSAL>(a.heads, a.slots, head, slot);
    Rows r;
    if (!find_rows<Q>(a, slot, r)) return;
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
    if (there && !half) a.delta[stat] = delta;
    f32x16 g[DB];
#pragma unroll
    for (int t = 0; t < DB; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) g[t][e] = 0.f;
    const int keys = CAUSAL && q0 + Q < r.len ? q0 + Q : r.len, blocks = (keys + kStep - 1) / kStep;
    const int limit = CAUSAL && q + 1 < r.len ? q + 1 : r.len;
    const Loader<D, W> loader(wave);
    const uint32_t lds = lds_of(smem);
    auto load = [&](int b) {
        const uint32_t at = lds + (uint32_t)(b & 1) * kPair<D>;
        const size_t from = (size_t)b * kStep * pitch;
        loader.load(kb + from, (uint32_t)pitch, r.len - b * kStep, at);
        loader.load(vb + from, (uint32_t)pitch, r.len - b * kStep, at + kTile<D>);
    };
    load(0);
    for (int b = 0; b < blocks; ++b) {
        arrived();
        __syncthreads();                                 // block b is there; block b - 1 is done with
        if (b + 1 < blocks) load(b + 1);
        const unsigned char *ks = smem + (b & 1) * kPair<D>, *vs = ks + kTile<D>;
        const int k0 = b * kStep;
        if (w0 < r.len && (!CAUSAL || k0 <= w0 + 31)) {
            const bool border = k0 + kStep > (CAUSAL ? (w0 + 1 < r.len ? w0 + 1 : r.len) : r.len);
            const int lim = border ? limit - k0 - 4 * half : kStep;
#pragma unroll 1
            for (int t = 0; t < 2; ++t) {
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
    if (there) store_column<DB>(gxb + (size_t)q * pitch, g, a.scale);
}

// Heads of 128: a lane's sums of gk and gv, its key and its value would be 192 registers of the 256 that two wavefronts to a SIMD leave: the values stay in LDS, and
// with them (32 KB) and another workgroup's there is room for blocks of 32 queries.
template <int D> constexpr int kQueries = D == 128 ? 32 : 64;
template <int D, int W> constexpr int kKvLds = 4 * kTile<D, kQueries<D>> + (D == 128 ? kTile<D, W * 32> : 0);

template <int D, int W, bool CAUSAL>
__global__ __launch_bounds__(W * 64, 2) void gkv_kernel(Args a) {
    constexpr int K = W * 32, KS = D / 16, DB = D / 32, Q = kQueries<D>;
    constexpr bool kValuesInLds = D == 128;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ __align__(16) float stats[2][2][Q];       // of a block's queries: log-sum-exp (log2), delta
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), l32 = lane & 31, half = lane >> 5;
    int unit, slot;
    place_of<CAUSAL>(a.kv * a.splits, a.slots, unit, slot);
    const int kh = unit / a.splits, split = unit % a.splits;
    if (CAUSAL) slot = a.slots - 1 - slot;               // the first keys have the most queries
    Rows r;
    if (!find_rows<K>(a, slot, r)) return;
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
    const uint32_t lds = lds_of(smem);
    const unsigned char *values = smem + 4 * kTile<D, Q>;
    bf16x8 kf[KS], vf[kValuesInLds ? 1 : KS];
    {
        const unsigned char *p = xb + (size_t)(there ? key : r.len - 1) * pitch + (size_t)(a.heads + kh) * D * 2 + half * 16;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            kf[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(p + s * 32));
            if constexpr (!kValuesInLds) vf[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(p + (size_t)a.kv * D * 2 + s * 32));
        }
    }
    if constexpr (kValuesInLds)
        Loader<D, W, K>(wave).load(xb + (size_t)first * pitch + (size_t)(a.heads + a.kv + kh) * D * 2, (uint32_t)pitch, r.len - first, lds + 4 * kTile<D, Q>);
    f32x16 gk[DB], gv[DB];
#pragma unroll
    for (int t = 0; t < DB; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) gk[t][e] = gv[t][e] = 0.f;
    const int begin = CAUSAL ? first / Q : 0, per = (r.len + Q - 1) / Q - begin;
    const Loader<D, W, Q> loader(wave);
    float st = 0.f;                                      // the thread's statistic of the block on its way: log-sum-exp (the first Q threads), delta (the next Q)
    auto load = [&](int head, int at, int buffer) {
        const uint32_t to = lds + (uint32_t)buffer * 2 * kTile<D, Q>;
        loader.load(xb + (size_t)at * pitch + (size_t)head * D * 2, (uint32_t)pitch, r.len - at, to);
        loader.load(a.gy + ((size_t)r.start + at) * out_pitch + (size_t)head * D * 2, (uint32_t)out_pitch, r.len - at, to + kTile<D, Q>);
        const int q = at + ((int)threadIdx.x & (Q - 1));
        if (threadIdx.x < Q) st = q < r.len ? a.lse[(size_t)head * a.M + r.start + q] * kLog2e : __builtin_inff();      // p = 0 behind the last query
        else if (threadIdx.x < 2 * Q) st = q < r.len ? a.delta[(size_t)head * a.M + r.start + q] : 0.f;
    };
    // Each head's queries from the last block on backwards: causal, workgroups on an XCD begin at the same block and find it in its L2.
    const int end = (kh * a.splits + split + 1) * share;
    int head = end - share, block = per - 1, buffer = 0;
    load(head, (begin + block) * Q, 0);
    for (;;) {
        if (threadIdx.x < 2 * Q) stats[buffer][threadIdx.x / Q][threadIdx.x & (Q - 1)] = st;
        arrived();
        __syncthreads();                                 // the block is there; the one before is done with
        const int at = (begin + block) * Q;
        if (block-- == 0) { block = per - 1; ++head; }
        const bool more = head < end;
        if (more) load(head, (begin + block) * Q, buffer ^ 1);
        const unsigned char *qs = smem + buffer * 2 * kTile<D, Q>, *gs = qs + kTile<D, Q>;
        if (w0 < r.len && (!CAUSAL || at + Q - 1 >= w0)) {
#pragma unroll
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
                    const f32x4 l = *reinterpret_cast<const f32x4 *>(&stats[buffer][0][32 * t + 8 * e4 + 4 * half]);
                    const f32x4 dl = *reinterpret_cast<const f32x4 *>(&stats[buffer][1][32 * t + 8 * e4 + 4 * half]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[4 * e4 + e], a.scale_log2e, -l[e]));
                        s[4 * e4 + e] = p;
                        dp[4 * e4 + e] = p * (dp[4 * e4 + e] - dl[e]);
                    }
                }
                if (CAUSAL && __builtin_expect(at + 32 * t < w0 + 31, 0)) {
                    const int from = key - at - 32 * t - 4 * half;                 // the first row of the product that sees this key
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        s[e] = row_of(e) >= from ? s[e] : 0.f;
                        dp[e] = row_of(e) >= from ? dp[e] : 0.f;
                    }
                    asm volatile("" ::: "memory");
                }
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
        if (!more) break;
        buffer ^= 1;
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

template <int D, int W, bool CAUSAL>
static hipError_t backward(Args a, hipStream_t stream) {
    constexpr int kLds = 2 * kPair<D>, kLdsKv = kKvLds<D, W>;
    static_assert(kLds <= 64 * 1024 && kLdsKv <= 64 * 1024, "what a launch may ask for without more ado");
    a.slots = slots_of(a.M, a.seqs, W * 32);
    gq_kernel<D, W, CAUSAL><<<dim3((unsigned)a.slots * (unsigned)a.heads), dim3(W * 64), kLds, stream>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    gkv_kernel<D, W, CAUSAL><<<dim3((unsigned)a.slots * (unsigned)(a.kv * a.splits)), dim3(W * 64), kLdsKv, stream>>>(a);
    e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    const uint32_t n = (uint32_t)(2 * a.kv * D);
    const uint64_t groups = ((uint64_t)a.M * (n / 8) + 255) / 256;
    join_kernel<<<dim3((unsigned)(groups < 4096 ? groups : 4096)), dim3(256), 0, stream>>>(a, n, (uint32_t)(a.heads * D * 2) + n * 2, (uint32_t)(a.heads * D * 2));
    return hipGetLastError();
}

// In how many shares a key head's query heads go: as few as give the chip two rounds of its 512 workgroups.
static int splits_of(long long M, int heads, int kv) {
    const int group = heads / kv;
    int n = 1;
    while (n < group && (group % n || (M + 127) / 128 * kv * n < 1024)) ++n;
    return n;
}

}  // namespace pat

// delta, and behind it the parts of gk and gv where there are several.
static size_t delta_bytes(long long M, int heads) { return ((size_t)M * heads * sizeof(float) + 255) / 256 * 256; }
size_t packed_attention_bwd_workspace_bytes(long long M, int Cout, int heads, int kv) {
    const int n = pat::splits_of(M, heads, kv);
    return delta_bytes(M, heads) + (n > 1 ? (size_t)n * M * 2 * kv * (Cout / heads) * sizeof(float) : 0);
}

// y, lse: what the forward pass left; gy as y; gx as x, all of it written (rows of no sequence with zeros).
hipError_t launch_packed_attention_bwd(const void *x, const void *off, const void *y, const float *lse, const void *gy, void *gx, long long M, long long seqs,
                                       int Cin, int Cout, int heads, int kv, int causal, int bf16, void *workspace, size_t workspace_bytes, hipStream_t stream) {
    if (!x || !off || !y || !lse || !gy || !gx || packed_attention_check(M, seqs, Cin, Cout, heads, kv, bf16)) return hipErrorInvalidValue;
    if (!workspace || workspace_bytes < packed_attention_bwd_workspace_bytes(M, Cout, heads, kv)) return hipErrorInvalidValue;
    pat::Args a = {};
    a.x = static_cast<const unsigned char *>(x); a.off = static_cast<const long long *>(off);
    a.y = static_cast<unsigned char *>(const_cast<void *>(y)); a.lse = const_cast<float *>(lse);
    a.gy = static_cast<const unsigned char *>(gy); a.gx = static_cast<unsigned char *>(gx); a.delta = static_cast<float *>(workspace);
    a.M = (int)M; a.seqs = (int)seqs; a.heads = heads; a.kv = kv;
    a.splits = pat::splits_of(M, heads, kv);
    a.part = a.splits > 1 ? reinterpret_cast<float *>(static_cast<unsigned char *>(workspace) + delta_bytes(M, heads)) : nullptr;
    a.scale = 1.0f / sqrtf((float)(Cout / heads));
    a.scale_log2e = a.scale * pat::kLog2e;
    if (Cout / heads == 64) return causal ? pat::backward<64, 4, true>(a, stream) : pat::backward<64, 4, false>(a, stream);
    return causal ? pat::backward<128, 4, true>(a, stream) : pat::backward<128, 4, false>(a, stream);
}

}  // namespace delta
