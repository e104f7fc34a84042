// Attention over packed sequences (forward) for gfx950: ctx = softmax(q k^T / sqrt D) v per query head and sequence, causal or not, R query heads over S key
// heads (head h reads key head h / (R / S)), D = 64 or 128, bf16; and the scores' log-sum-exp, which the gradients read.
//
// Layout.  x [M, (R + 2 S) D]: R heads of queries, S of keys, S of values; y [M, R D]; lse [R, M].  Sequence i is rows off[i] .. off[i+1] - 1; rows of
// no sequence are zero in y and lse (packed_attention.hpp: how a workgroup finds its rows).
//
// A workgroup takes one head and 32 queries a wavefront; K and V of its sequence stream through LDS in blocks of 64 keys, two buffers, the next
// block on its way from memory straight to LDS.  Everything is computed transposed, as in attention.hip: S^T = K Q^T, so that a lane owns a query and its softmax statistics are
// the lane's own; O^T += V^T P^T with P straight from the accumulators.  Running maximum and sum in fp32; P is rounded to bf16 before it multiplies V.
// Causal: a workgroup ends at its last query's block, a wavefront skips the blocks behind its own last query, and only blocks that a border crosses are masked.
//
// Bound by the SIMDs: a block of 64 keys takes a wavefront 2 D * 64 * 32 * 2 operations, 1024 cycles of the matrix unit with D = 128, and about as many of the vector unit (an exponential,
// a multiply-add, an addition, half a maximum and half a conversion a score), which overlap little; and by power, as the clock falls to 1.8 to 1.9 GHz.  8192
// tokens, 32 heads over 8 of 128, causal: 540 to 595 us, 920 to 1020 TFLOP/s (a large matrix product reaches 1175 here; the matrix units 54 % busy, no bank conflicts);
// 9 packed sequences of up to 1531, 16 heads over 2 of 128 50 to 54 us (580 to 630 TFLOP/s); 32 of up to 512, 12 heads of 64, not causal 27 us (360 TFLOP/s: the vector unit's work
// is the same for half the products); 77 tokens 4.9 us: latency.
// Tried with heads of 128 and not kept: the next block's scores under this one's exponentials (8192 tokens 552 and 561 us, 4096 157 and 152, 2048 tokens of 8 heads 30 and 29), a
// wavefront's priority raised around its products (the same), two wavefronts' tiles from padded rows through registers (704 us).  Heads of 64, which leave more registers: not measured.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.hpp"
#include "packed_attention.hpp"

namespace delta {
namespace pat {

template <int D, int G> constexpr int kBuffer = 2 * kTile<D, kKeys<D, G>>;         // K and V of a block

// W wavefronts of 32 queries each, G times: group g takes the blocks g, g + G, .. of keys, and the groups' sums meet in LDS.
template <int D, int W, int G, bool CAUSAL>
__global__ __launch_bounds__(W * G * 64, 2) void forward_kernel(Args a) {
    constexpr int Q = W * 32, KS = D / 16, DB = D / 32, kBlock = kKeys<D, G>, T = kBlock / 32;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ float meet[G > 1 ? (G - 1) * W : 1][2][64];
    const int lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)) % W, group = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)) / W;
    int head, slot;
    place_of<CAUSAL>(blockIdx.x, gridDim.x, a.heads, a.slots, head, slot);
    Rows r;
    if (!find_rows<Q, CAUSAL>(a, a.slots, slot, r)) return;
    const size_t out_pitch = (size_t)a.heads * D * 2, pitch = (size_t)(a.heads + 2 * a.kv) * D * 2;
    const int q0 = r.tile * Q;
    unsigned char *yb = a.y + (size_t)r.start * out_pitch + (size_t)head * D * 2;
    float *lse = a.lse ? a.lse + (size_t)head * a.M + r.start : nullptr;
    if (r.alone) {
        const int n = r.len - q0 < Q ? r.len - q0 : Q;
        zero_rows(yb + (size_t)q0 * out_pitch, out_pitch, n, D * 2);
        if (lse && (int)threadIdx.x < n) lse[q0 + threadIdx.x] = 0.f;
        return;
    }
    const unsigned char *xb = a.x + (size_t)r.start * pitch;
    const int kh = head / (a.heads / a.kv);
    const unsigned char *kb = xb + (size_t)(a.heads + kh) * D * 2, *vb = kb + (size_t)a.kv * D * 2;
    const int w0 = q0 + 32 * wave, q = w0 + l32;
    const bool there = q < r.len;
    bf16x8 qf[KS];
    {
        const unsigned char *p = xb + (size_t)(there ? q : r.len - 1) * pitch + (size_t)head * D * 2 + half * 16;
#pragma unroll
        for (int s = 0; s < KS; ++s) qf[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(p + s * 32));
    }
    f32x16 o[DB];
#pragma unroll
    for (int t = 0; t < DB; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[t][e] = 0.f;
    float m_run = -3.402823466e38f, l_run = 0.f;         // finite: a lane's first blocks may hold no key of its own; l_run: this half-wave's share of the sum
    const int keys = CAUSAL && q0 + Q < r.len ? q0 + Q : r.len, blocks = (keys + kBlock - 1) / kBlock;
    const int limit = CAUSAL && q + 1 < r.len ? q + 1 : r.len;                     // the lane's keys
    const Loader<D, W, kBlock> loader(wave);
    const uint32_t lds = lds_of(smem) + (uint32_t)group * 2 * kBuffer<D, G>;
    auto load = [&](int i) {
        const int b = i * G + group;
        if (b >= blocks) return;
        const uint32_t at = lds + (uint32_t)(i & 1) * kBuffer<D, G>;
        const size_t from = (size_t)b * kBlock * pitch;
        loader.load(kb + from, (uint32_t)pitch, r.len - b * kBlock, at);
        loader.load(vb + from, (uint32_t)pitch, r.len - b * kBlock, at + kTile<D, kBlock>);
    };
    load(0);
    for (int i = 0; i * G < blocks; ++i) {
        arrived();
        __syncthreads();                                 // the block is there; the one before is done with
        load(i + 1);
        const unsigned char *ks = smem + (group * 2 + (i & 1)) * kBuffer<D, G>, *vs = ks + kTile<D, kBlock>;
        const int k0 = (i * G + group) * kBlock;
        if (k0 < keys && w0 < r.len && (!CAUSAL || k0 <= w0 + 31)) {
            f32x16 s[T];
#pragma unroll
            for (int t = 0; t < T; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) s[t][e] = 0.f;
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int t = 0; t < T; ++t) s[t] = mfma(rows_of<D>(ks, 32 * t, k), qf[k], s[t]);
            if (__builtin_expect(k0 + kBlock > (CAUSAL ? (w0 + 1 < r.len ? w0 + 1 : r.len) : r.len), 0)) {
                const int lim = limit - k0 - 4 * half;
#pragma unroll
                for (int t = 0; t < T; ++t)
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[t][e] = 32 * t + row_of(e) < lim ? s[t][e] : -__builtin_inff();
                asm volatile("" ::: "memory");           // keeps the masked path a separate block
            }
            float mx = -__builtin_inff();
#pragma unroll
            for (int t = 0; t < T; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[t][e]);
            const float m_new = fmaxf(m_run, halves_max(mx) * a.scale_log2e);
            // Where no lane's maximum grows nothing is scaled.  Scaling later still, once it has grown by 2^8, saved 4 % of long sequences' time, but a row's largest weight is then
            // not exactly one, and y 0.0021 instead of 0.0018 from 64 bits.
            if (__any(m_new > m_run)) {
                const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);         // 0 on the first block
                m_run = m_new;
                l_run *= alpha;
#pragma unroll
                for (int t = 0; t < DB; ++t)
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[t][e] *= alpha;
            }
#pragma unroll
            for (int t = 0; t < T; ++t) {
                float sum = 0.f;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    s[t][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][e], a.scale_log2e, -m_run));
                    sum += s[t][e];
                }
                l_run += sum;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const bf16x8 p = as_operand(s[t], j);
#pragma unroll
                    for (int d = 0; d < DB; ++d) o[d] = mfma(columns_of<D>(vs, 32 * t + 16 * j, d), p, o[d]);
                }
            }
        }
    }
    l_run = rows::halves(l_run);
    if constexpr (G > 1) {
        __syncthreads();                                 // the last blocks are done with
        float *sums = reinterpret_cast<float *>(smem);
        if (group) {
            hand_over(sums, (group - 1) * W + wave, o);
            meet[(group - 1) * W + wave][0][lane] = m_run;
            meet[(group - 1) * W + wave][1][lane] = l_run;
        }
        __syncthreads();
        if (group) return;
        float m = m_run;
#pragma unroll
        for (int g = 0; g < G - 1; ++g) m = fmaxf(m, meet[g * W + wave][0][lane]);
        const float mine = __builtin_amdgcn_exp2f(m_run - m);
        l_run *= mine;
        m_run = m;
#pragma unroll
        for (int t = 0; t < DB; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[t][e] *= mine;
#pragma unroll
        for (int g = 0; g < G - 1; ++g) {
            const float other = __builtin_amdgcn_exp2f(meet[g * W + wave][0][lane] - m);
            l_run += meet[g * W + wave][1][lane] * other;
            take_over(sums, g * W + wave, o, other);
        }
    }
    if (!there) return;
    store_column<DB>(yb + (size_t)q * out_pitch, o, 1.0f / l_run);
    if (lse && !half) lse[q] = (m_run + __builtin_amdgcn_logf(l_run)) * 0.6931471805599453f;
}

template <int D, int W, int G, bool CAUSAL>
static hipError_t forward(Args a, hipStream_t stream) {
    constexpr int kLds = G * 2 * kBuffer<D, G>;
    static_assert((G - 1) * W * D / 32 * 16 * 64 * 4 <= kLds, "the sums fit where the blocks were");
    if (kLds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&forward_kernel<D, W, G, CAUSAL>), hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
        if (e != hipSuccess) return e;
    }
    a.slots = slots_of(a.M, a.seqs, W * 32);
    forward_kernel<D, W, G, CAUSAL><<<dim3((unsigned)a.slots * (unsigned)a.heads), dim3(W * G * 64), kLds, stream>>>(a);
    return hipGetLastError();
}
template <int D, bool CAUSAL>
static hipError_t forward(const Args &a, hipStream_t stream) {
    switch (groups_of(a.M, a.seqs, a.heads, D)) {
    case 4: return forward<D, 1, 4, CAUSAL>(a, stream);
    case 2: return forward<D, 2, 2, CAUSAL>(a, stream);
    default: return forward<D, 4, 1, CAUSAL>(a, stream);
    }
}

}  // namespace pat

// x [M, (heads + 2 kv) D], `seqs` sequences.
const char *packed_attention_check(long long M, long long seqs, int Cin, int Cout, int heads, int kv, int bf16) {
    if (!bf16) return "attention is bf16 only";
    if (heads <= 0 || kv <= 0 || heads % kv) return "attention needs R query heads, a multiple of S key heads";
    if (Cout % heads || (Cout / heads != 64 && Cout / heads != 128) || (long long)Cout / heads * (heads + 2LL * kv) != Cin)
        return "attention needs heads of 64 or 128 channels, Cout = R D, Cin = (R + 2 S) D";
    if (Cin > 1 << 24) return "attention takes rows of at most 16777216 channels";     // 64 of them lie within 32 bits
    if (M <= 0 || M > 0x7FFFFF00LL) return "attention takes 1 to 2147483392 rows";
    if (seqs < 1 || seqs > 0x3FFFFFFFLL) return "offsets must hold one int64 value more than there are sequences";
    // threads of a launch: 128 queries or keys to 256 threads (fewer where the launch is small), and a workgroup to each sequence and each end; with 512 threads to 256
    // keys at most twice as many: below 2^32
    if ((M / 128 + seqs + 2) * heads * 256 > 0x7FFFFFFFLL) return "too many rows, sequences and heads in one launch";
    return nullptr;
}

static pat::Args packed_attention_args(const void *x, const void *off, void *y, float *lse, long long M, long long seqs, int Cout, int heads, int kv) {
    pat::Args a = {};
    a.x = static_cast<const unsigned char *>(x); a.off = static_cast<const long long *>(off); a.y = static_cast<unsigned char *>(y); a.lse = lse;
    a.M = (int)M; a.seqs = (int)seqs; a.heads = heads; a.kv = kv;
    a.scale = 1.0f / sqrtf((float)(Cout / heads));
    a.scale_log2e = a.scale * 1.4426950408889634f;
    return a;
}

hipError_t launch_packed_attention(const void *x, const void *off, void *y, float *lse, long long M, long long seqs, int Cin, int Cout, int heads, int kv,
                                   int causal, int bf16, hipStream_t stream) {
    if (!x || !off || !y || packed_attention_check(M, seqs, Cin, Cout, heads, kv, bf16)) return hipErrorInvalidValue;
    const pat::Args a = packed_attention_args(x, off, y, lse, M, seqs, Cout, heads, kv);
    if (Cout / heads == 64) return causal ? pat::forward<64, true>(a, stream) : pat::forward<64, false>(a, stream);
    return causal ? pat::forward<128, true>(a, stream) : pat::forward<128, false>(a, stream);
}

}  // namespace delta
