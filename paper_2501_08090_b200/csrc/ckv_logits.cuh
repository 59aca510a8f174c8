// Penalties, biases and masks on logits, and the probabilities that follow.
#pragma once

#include <cuda_bf16.h>

#include "ckv_common.cuh"

namespace ckv {

// Row j of a request's logits (j drafted tokens precede it).  With n_v = how often token v was generated (drafts
// before the row among them) and seen_v = whether it was generated or stands in the prompt, in fp32:
//   x = logit;  seen: x > 0 ? x / repetition : x * repetition;  x -= frequency * n;  n > 0: x -= presence;  x += bias
//   excluded where the mask's bit is 0;  p_v = 2^((x_v - max x) log2(e) / temperature) / their sum
//   temperature <= 0: 1 at the first largest, else 0;  nothing allowed, or only minus infinities: all 0
//
// Bound by HBM: a logit is read once and a result written once.  A cluster of CTAs owns a row, a CTA a slice of
// at most 16384 tokens that its threads hold in registers, 32 each, as pieces of 16 aligned bytes.  While they are
// on their way the CTA counts the history's tokens of its slice in shared memory (whole numbers: the order
// of atomics does not show) and looks up the biases.  The CTAs exchange (max, place of it, sum) once through
// distributed shared memory.
struct LogitsParams {
    const void *logits;
    void *out;
    long long stride, out_stride;   // elements between rows
    const float *params;            // [batch][4]: repetition, presence, frequency, temperature; NULL: none
    const int32_t *history;         // [batch][history_stride]: prompt, then generated tokens; NULL: none
    const int32_t *prompt_lens, *history_lens;
    const int32_t *drafts;          // [batch][rows - 1]; NULL: none
    const int32_t *bias_ids;        // [batch][n_bias]; NULL: none
    const float *bias;
    const uint32_t *mask;           // [batch * rows] rows of words; NULL: none
    long long history_stride, mask_stride;
    int32_t rows, vocab, n_bias, probs;
    int32_t pieces;                 // pieces of 16 bytes that a CTA owns
};

constexpr int kLogitsThreads = 512, kLogitsSlice = 16384;
// Sixteen slices, less what a row loses to its place within its first and last piece.
constexpr int kLogitsMaxVocab = 16 * kLogitsSlice - 16;

// The elements of a piece of 16 bytes.
__device__ __forceinline__ void piece_elements(const uint4 &raw, float (&x)[4])
{
    x[0] = __uint_as_float(raw.x); x[1] = __uint_as_float(raw.y); x[2] = __uint_as_float(raw.z); x[3] = __uint_as_float(raw.w);
}

__device__ __forceinline__ void piece_elements(const uint4 &raw, float (&x)[8])
{
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}

template <typename T>
__device__ __forceinline__ T from_float(float x);
template <>
__device__ __forceinline__ float from_float(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float(float x) { return __float2bfloat16_rn(x); }

struct LogitsPeak {
    float m;                        // largest
    int at;                         // its first place
};

__device__ __forceinline__ LogitsPeak higher(LogitsPeak a, LogitsPeak b) { return b.m > a.m || (b.m == a.m && b.at < a.at) ? b : a; }

// Stores E elements x to dst[0 .. E - 1]; `whole`: dst is aligned for as much as one access takes.
template <typename T, int E>
__device__ __forceinline__ void store_elements(T *dst, const float *x, bool whole, int from, int to)
{
    if (whole && from == 0 && to == E) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int e = 0; e < E; e += 4) *(float4 *)(dst + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
        } else if constexpr (E == 8) {
            *(uint4 *)dst = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
        } else {
            *(uint2 *)dst = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
        }
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (e >= from && e < to) dst[e] = from_float<T>(x[e]);
    }
}

template <typename Tin, typename Tout>
__global__ void __launch_bounds__(kLogitsThreads, 2)
logits_process_kernel(const LogitsParams p)
{
    constexpr int E = 16 / sizeof(Tin), K = kLogitsSlice / E / kLogitsThreads;   // elements of a piece, pieces of a thread
    extern __shared__ uint32_t s_count[];         // [slice]: bit 31: in the prompt; below: times generated.  Then entries of the bias
    __shared__ LogitsPeak s_peak[kLogitsThreads / 32];
    __shared__ float s_sum[kLogitsThreads / 32];
    __shared__ float s_share[3];                  // this CTA's (max, its place, sum), read by the cluster
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = (int)cluster_rank(), ctas = (int)cluster_size();
    const int row = blockIdx.x / ctas, b = row / p.rows, j = row % p.rows, V = p.vocab;
    const Tin *in = static_cast<const Tin *>(p.logits) + row * p.stride;
    Tout *out = static_cast<Tout *>(p.out) + row * p.out_stride;
    const int off = (int)(reinterpret_cast<uintptr_t>(in) / sizeof(Tin) % E);    // elements before the row in its first piece
    const int first = rank * p.pieces * E - off, last = min(first + p.pieces * E, V);            // the slice; `first` may lie below 0
    const int used = max(0, last - first);
    grid_dependency_wait();
    grid_launch_dependents();

    float x[K][E];
    {
        uint4 raw[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int at = first + (k * kLogitsThreads + tid) * E;
            raw[k] = make_uint4(0u, 0u, 0u, 0u);
            if (at < last) raw[k] = *(const uint4 *)(in + at);   // up to 15 bytes beside the row, not used
        }
        const float *pr = p.params + 4 * b;
        const float rep = p.params ? __ldg(pr) : 1.f, pres = p.params ? __ldg(pr + 1) : 0.f, freq = p.params ? __ldg(pr + 2) : 0.f;
        const bool counted = p.history != nullptr || p.drafts != nullptr;
        if (counted) {
            for (int i = tid * 4; i < p.pieces * E; i += kLogitsThreads * 4) *(uint4 *)(s_count + i) = make_uint4(0u, 0u, 0u, 0u);
            __syncthreads();
            auto count = [&](int token, bool prompt) {
                const unsigned at = (unsigned)(token - first);
                if (token < 0 || at >= (unsigned)used) return;
                if (prompt) atomicOr(s_count + at, 0x80000000u);
                else atomicAdd(s_count + at, 1u);
            };
            if (p.history != nullptr) {
                const int n = (int)min((long long)max(__ldg(p.history_lens + b), 0), p.history_stride);
                const int prompt = __ldg(p.prompt_lens + b);
                const int32_t *text = p.history + b * p.history_stride;
#pragma unroll 4
                for (int i = tid; i < n; i += kLogitsThreads) count(__ldg(text + i), i < prompt);
            }
            if (p.drafts != nullptr)
                for (int i = tid; i < j; i += kLogitsThreads) count(__ldg(p.drafts + (long long)b * (p.rows - 1) + i), false);
            __syncthreads();
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int at = (k * kLogitsThreads + tid) * E;       // within the slice
            piece_elements(raw[k], x[k]);
            uint32_t c[E];
#pragma unroll
            for (int e = 0; e < E; ++e) c[e] = 0u;
            if (counted && at < used) {
#pragma unroll
                for (int e = 0; e < E; e += 4) *(uint4 *)(c + e) = *(const uint4 *)(s_count + at + e);
            }
#pragma unroll
            for (int e = 0; e < E; ++e) {
                float v = x[k][e];
                if (c[e] != 0u) {                 // rounded step by step, as the formula stands
                    const uint32_t n = c[e] & 0x7fffffffu;
                    v = v > 0.f ? __fdiv_rn(v, rep) : __fmul_rn(v, rep);
                    v = __fsub_rn(v, __fmul_rn(freq, (float)n));
                    if (n > 0u) v = __fsub_rn(v, pres);
                }
                x[k][e] = v;
            }
        }
    }
    if (p.bias_ids != nullptr) {                  // where an id stands twice, the last entry counts
        __syncthreads();
        for (int i = tid * 4; i < p.pieces * E; i += kLogitsThreads * 4) *(uint4 *)(s_count + i) = make_uint4(0u, 0u, 0u, 0u);
        __syncthreads();
        for (int i = tid; i < p.n_bias; i += kLogitsThreads) {
            const int token = __ldg(p.bias_ids + (long long)b * p.n_bias + i);
            const unsigned at = (unsigned)(token - first);
            if (token >= 0 && at < (unsigned)used) atomicMax(s_count + at, (uint32_t)i + 1u);
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int at = (k * kLogitsThreads + tid) * E;
            if (at >= used) continue;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const uint32_t entry = s_count[at + e];
                if (entry != 0u) x[k][e] = __fadd_rn(x[k][e], __ldg(p.bias + (long long)b * p.n_bias + entry - 1));
            }
        }
    }
    // ---- what is outside the row or not allowed is excluded
    LogitsPeak peak = {-INFINITY, 0x7fffffff};
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int v0 = first + (k * kLogitsThreads + tid) * E;
        uint32_t allowed = 0u;
        if (v0 < last) {
            allowed = 0xffffffffu;
            if (p.mask != nullptr) {
                const uint32_t *words = p.mask + row * p.mask_stride;
                const int lo = max(v0, 0), w0 = lo / 32, w1 = min(v0 + E - 1, V - 1) / 32;
                const uint32_t a = __ldg(words + w0), z = w1 != w0 ? __ldg(words + w1) : a;
                // bits from token lo on, moved up to lo's place in the piece
                allowed = __funnelshift_r(a, z, lo % 32) << (lo - v0);
            }
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (v0 + e < 0 || v0 + e >= last || !(allowed >> e & 1u)) x[k][e] = -INFINITY;
            peak = higher(peak, {x[k][e], v0 + e});
        }
    }
    const bool whole = reinterpret_cast<uintptr_t>(out + first) % (sizeof(Tout) * E < 16 ? sizeof(Tout) * E : 16) == 0;
    auto store = [&](int k) {
        const int v0 = first + (k * kLogitsThreads + tid) * E;
        if (v0 < last) store_elements<Tout, E>(out + v0, x[k], whole, max(0, -v0), min(E, last - v0));
    };
    if (!p.probs) {
#pragma unroll
        for (int k = 0; k < K; ++k) store(k);
        return;
    }
    // ---- the row's maximum and sum
    const float temperature = p.params ? __ldg(p.params + 4 * b + 3) : 1.f;
    const bool greedy = !(temperature > 0.f);
    const float scale = greedy ? 1.4426950408889634f : fminf(1.4426950408889634f / temperature, 3e38f);     // 0 * scale has to be 0
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        peak = higher(peak, {__shfl_xor_sync(0xffffffffu, peak.m, o), __shfl_xor_sync(0xffffffffu, peak.at, o)});
    if (lane == 0) s_peak[warp] = peak;
    __syncthreads();
    peak = s_peak[0];
#pragma unroll
    for (int w = 1; w < kLogitsThreads / 32; ++w) peak = higher(peak, s_peak[w]);
    const float ref = peak.m == -INFINITY ? 0.f : peak.m;
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            x[k][e] = fast_exp2((x[k][e] - ref) * scale);
            sum += x[k][e];
        }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) s_sum[warp] = sum;
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < kLogitsThreads / 32; ++w) sum += s_sum[w];
        s_share[0] = peak.m;
        s_share[1] = __int_as_float(peak.at);
        s_share[2] = sum;
    }
    cluster_barrier();
    LogitsPeak top = {-INFINITY, 0x7fffffff};
    for (int c = 0; c < ctas; ++c) {
        float m, at;
        const uint32_t share = cluster_map(smem_u32(s_share), c);
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(m) : "r"(share));
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(at) : "r"(share + 4));
        top = higher(top, {m, __float_as_int(at)});
    }
    const float all = top.m == -INFINITY ? 0.f : top.m;
    float total = 0.f;
    for (int c = 0; c < ctas; ++c) {
        float m, l;
        const uint32_t share = cluster_map(smem_u32(s_share), c);
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(m) : "r"(share));
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(l) : "r"(share + 8));
        total += l * fast_exp2(((m == -INFINITY ? 0.f : m) - all) * scale);      // l = 0 where nothing is allowed
    }
    // a row of NaN where a NaN or an infinity is among what is allowed; zeros where nothing is
    const float f = total == 0.f ? 0.f : fast_exp2((ref - all) * scale) / total;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int v0 = first + (k * kLogitsThreads + tid) * E;
#pragma unroll
        for (int e = 0; e < E; ++e) x[k][e] = greedy && total == total ? (v0 + e == top.at && top.m > -INFINITY ? 1.f : 0.f) : x[k][e] * f;
        store(k);
    }
    cluster_barrier();                            // nobody leaves while others read its share
}

}  // namespace ckv
