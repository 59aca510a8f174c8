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
// at most 8192 tokens that its threads hold in registers, 32 each, as pieces of 16 aligned bytes.  While they are
// on their way the CTA counts the history's tokens of its slice, and looks up the biases' last entries, in arrays in
// shared memory (whole numbers, and the largest of entries: the order of atomics does not show).  Tokens that change
// are few: a bit tells their thread, which takes them out of its registers and handles them one by one.
// The CTAs exchange (max, sum, place of the max) once through distributed shared memory.
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

// Threads of a CTA: 256, in four CTAs an SM, so that some load while others meet (a row of 50257 tokens in 8 CTAs of 256
// 59 us for 512 rows, in 4 of 512 63); 512 where sixteen CTAs of 256 do not hold the row.
constexpr int kLogitsThreads = 256, kLogitsElements = 32;
// Sixteen slices of 512 threads, less what a row loses to its place within its first and last piece.
constexpr int kLogitsMaxVocab = 16 * 512 * kLogitsElements - 16;

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

__device__ __forceinline__ float element(float x) { return x; }
__device__ __forceinline__ float element(__nv_bfloat16 x) { return __bfloat162float(x); }

template <typename T>
__device__ __forceinline__ T from_float(float x);
template <>
__device__ __forceinline__ float from_float(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float(float x) { return __float2bfloat16_rn(x); }

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

template <typename Tin, typename Tout, int T>
__global__ void __launch_bounds__(T, 1024 / T)
logits_process_kernel(const LogitsParams p)
{
    constexpr int E = 16 / sizeof(Tin), K = kLogitsElements / E;                 // elements of a piece, pieces of a thread
    constexpr int kWarps = T / 32;
    extern __shared__ uint32_t s_token[];         // [slice]: times generated, bit 31: in the prompt; then, with biases, [slice]: the entry plus 1
    __shared__ uint32_t s_changes[T];             // a bit per element of a thread: counted or biased
    __shared__ float s_max[kWarps], s_sum[kWarps];
    __shared__ int s_at[kWarps];
    __shared__ uint4 s_share[16];                 // every CTA's maximum, sum and place of the maximum, written by them
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = (int)cluster_rank(), ctas = (int)cluster_size();
    const int row = blockIdx.x / ctas, b = row / p.rows, j = row % p.rows, V = p.vocab;
    const Tin *in = static_cast<const Tin *>(p.logits) + row * p.stride;
    Tout *out = static_cast<Tout *>(p.out) + row * p.out_stride;
    const int off = (int)(reinterpret_cast<uintptr_t>(in) / sizeof(Tin) % E);    // elements before the row in its first piece
    const int first = rank * p.pieces * E - off, last = min(first + p.pieces * E, V);            // the slice; `first` may lie below 0
    const unsigned used = (unsigned)max(0, last - first);
    const bool counted = p.history != nullptr || p.drafts != nullptr, biased = p.bias_ids != nullptr;
    uint32_t *s_count = s_token, *s_entry = s_token + (counted ? p.pieces * E : 0);
    auto place = [&](int i) { return (i / E * T + tid) * E + i % E; };           // of the thread's element i in the slice
    if (counted || biased) {
        for (int i = tid * 4; i < p.pieces * E * ((counted ? 1 : 0) + (biased ? 1 : 0)); i += T * 4) *(uint4 *)(s_token + i) = make_uint4(0u, 0u, 0u, 0u);
        s_changes[tid] = 0u;
    }
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");        // waited for before others' shared memory is written
    grid_dependency_wait();
    grid_launch_dependents();

    float x[K][E];
    uint32_t allowed = 0u;                        // a bit per element of the thread: in the row, and the mask's bit
    uint4 raw[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int v0 = first + (k * T + tid) * E;
        raw[k] = make_uint4(0u, 0u, 0u, 0u);
        if (v0 < last) raw[k] = *(const uint4 *)(in + v0);       // up to 15 bytes beside the row, not used
    }
    // ---- how often its tokens came, and their biases
    if (counted || biased) {
        const int n = p.history != nullptr ? (int)min((long long)max(__ldg(p.history_lens + b), 0), p.history_stride) : 0;
        const int prompt = p.history != nullptr ? __ldg(p.prompt_lens + b) : 0;
        __syncthreads();
        // calls fn(place in the slice, index) for the tokens of a list that lie in the slice; true: the token was not there yet
        auto each = [&](const int32_t *list, int count, auto fn) {
#pragma unroll 4
            for (int i = tid; i < count; i += T) {
                const int token = __ldg(list + i);
                const unsigned at = (unsigned)(token - first);
                if (token < 0 || at >= used || !fn(at, i)) continue;
                const unsigned piece = at / E;                   // piece piece / T of thread piece % T
                atomicOr(s_changes + piece % T, 1u << (piece / T * E + at % E));
            }
        };
        each(p.history + b * p.history_stride, n,
             [&](unsigned at, int i) { return (i < prompt ? atomicOr(s_count + at, 0x80000000u) : atomicAdd(s_count + at, 1u)) == 0u; });
        each(p.drafts + (long long)b * (p.rows - 1), p.drafts != nullptr ? j : 0, [&](unsigned at, int) { return atomicAdd(s_count + at, 1u) == 0u; });
        // where an id stands twice, the last entry counts
        each(p.bias_ids + (long long)b * p.n_bias, p.n_bias, [&](unsigned at, int i) { return atomicMax(s_entry + at, (uint32_t)i + 1u) == 0u; });
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int v0 = first + (k * T + tid) * E;
        const int from = max(0, -v0), to = min(E, last - v0);    // the piece's elements in the slice
        if (to <= from) continue;
        uint32_t bits = (1u << to) - (1u << from);
        if (p.mask != nullptr) {
            const uint32_t *words = p.mask + row * p.mask_stride;
            const int lo = v0 + from, w0 = lo / 32, w1 = (v0 + to - 1) / 32;
            const uint32_t a = __ldg(words + w0), z = w1 != w0 ? __ldg(words + w1) : a;
            bits &= __funnelshift_r(a, z, lo % 32) << from;
        }
        allowed |= bits << (k * E);
    }
    // ---- the tokens that change: their values, rounded step by step as the formula stands, take the counts' places
    uint32_t changed = 0u;
    float most = -INFINITY;
    if (counted || biased) {
        __syncthreads();
        changed = s_changes[tid] & allowed;
        allowed &= ~changed;
        if (changed != 0u) {
            const float *pr = p.params + 4 * b;
            const float rep = counted ? __ldg(pr) : 1.f, pres = counted ? __ldg(pr + 1) : 0.f, freq = counted ? __ldg(pr + 2) : 0.f;
            for (uint32_t left = changed; left != 0u; left &= left - 1u) {
                const int at = place(__ffs(left) - 1);
                float v = element(in[first + at]);
                const uint32_t c = counted ? s_count[at] : 0u, times = c & 0x7fffffffu, entry = biased ? s_entry[at] : 0u;
                if (c != 0u) {
                    v = v > 0.f ? __fdiv_rn(v, rep) : __fmul_rn(v, rep);
                    v = __fsub_rn(v, __fmul_rn(freq, (float)times));
                    if (times > 0u) v = __fsub_rn(v, pres);
                }
                if (entry != 0u) v = __fadd_rn(v, __ldg(p.bias + (long long)b * p.n_bias + entry - 1));
                s_token[at] = __float_as_uint(v);
                most = fmaxf(most, v);
            }
        }
    }
    // calls fn(the token, its place in s_token) for them
    auto each_changed = [&](auto fn) {
        for (uint32_t left = changed; left != 0u; left &= left - 1u) {
            const int at = place(__ffs(left) - 1);
            fn(first + at, s_token[at]);
        }
    };
    // ---- what is outside the row, not allowed or changed is taken out
#pragma unroll
    for (int k = 0; k < K; ++k) piece_elements(raw[k], x[k]);
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        if (!(allowed >> i & 1u)) x[i / E][i % E] = -INFINITY;
        most = fmaxf(most, x[i / E][i % E]);
    }
    const bool whole = reinterpret_cast<uintptr_t>(out + first) % (sizeof(Tout) * E < 16 ? sizeof(Tout) * E : 16) == 0;
    auto store = [&](int k) {
        const int v0 = first + (k * T + tid) * E;
        if (v0 < last) store_elements<Tout, E>(out + v0, x[k], whole, max(0, -v0), min(E, last - v0));
    };
    if (!p.probs) {
#pragma unroll
        for (int k = 0; k < K; ++k) store(k);
        each_changed([&](int v, uint32_t &x) { out[v] = from_float<Tout>(__uint_as_float(x)); });
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        return;
    }
    // ---- the row's maximum and sum
    const float temperature = p.params ? __ldg(p.params + 4 * b + 3) : 1.f;
    const bool greedy = !(temperature > 0.f);
    const float scale = greedy ? 1.4426950408889634f : fminf(1.4426950408889634f / temperature, 3e38f);     // 0 * scale has to be 0
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
    if (lane == 0) s_max[warp] = most;
    __syncthreads();
    most = s_max[lane % kWarps];
#pragma unroll
    for (int o = kWarps / 2; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
    int at = 0x7fffffff;                          // the first place of the slice's maximum
    if (greedy) {
#pragma unroll
        for (int k = K - 1; k >= 0; --k)
#pragma unroll
            for (int e = E - 1; e >= 0; --e)
                if (x[k][e] == most) at = first + (k * T + tid) * E + e;
        each_changed([&](int v, uint32_t &x) {
            if (__uint_as_float(x) == most) at = min(at, v);
        });
        at = (int)__reduce_min_sync(0xffffffffu, (unsigned)at);
        if (lane == 0) s_at[warp] = at;
    }
    const float ref = most == -INFINITY ? 0.f : most;
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            x[k][e] = fast_exp2((x[k][e] - ref) * scale);
            sum += x[k][e];
        }
    each_changed([&](int, uint32_t &x) {
        const float w = fast_exp2((__uint_as_float(x) - ref) * scale);
        sum += w;
        x = __float_as_uint(w);
    });
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) s_sum[warp] = sum;
    __syncthreads();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");          // every CTA of the cluster runs
    if (warp == 0) {
        sum = lane < kWarps ? s_sum[lane] : 0.f;
#pragma unroll
        for (int o = kWarps / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (greedy) at = (int)__reduce_min_sync(0xffffffffu, (unsigned)s_at[lane % kWarps]);
        at = __shfl_sync(0xffffffffu, at, 0);
        sum = __shfl_sync(0xffffffffu, sum, 0);
        if (lane < ctas)                          // to CTA `lane`
            asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(cluster_map(smem_u32(s_share + rank), lane)),
                         "r"(__float_as_uint(most)), "r"(__float_as_uint(sum)), "r"((uint32_t)at), "r"(0u) : "memory");
    }
    cluster_barrier();
    // lane c looks at CTA c's; sums in the same order everywhere
    const bool there = lane < ctas;
    const uint4 share = s_share[there ? lane : 0];
    const float m = there ? __uint_as_float(share.x) : -INFINITY;
    float l = there ? __uint_as_float(share.y) : 0.f;
    float top = m;
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    top = __shfl_sync(0xffffffffu, top, 0);
    const float all = top == -INFINITY ? 0.f : top;
    l *= m == -INFINITY ? 0.f : fast_exp2((m - all) * scale);    // a slice in which nothing is allowed adds nothing
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
    const float total = __shfl_sync(0xffffffffu, l, 0);
    if (greedy && total == total) {               // 1 at the first of the largest
        const unsigned best = __reduce_min_sync(0xffffffffu, there && m == top && top > -INFINITY ? share.z : 0x7fffffffu);
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int e = 0; e < E; ++e) x[k][e] = first + (k * T + tid) * E + e == (int)best ? 1.f : 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) store(k);
    } else {
        // NaN where a NaN or an infinity is among what is allowed; zeros where nothing is
        const float f = total == 0.f ? 0.f : (most == -INFINITY ? 0.f : fast_exp2((most - all) * scale)) / total;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int e = 0; e < E; ++e) x[k][e] *= f;
#pragma unroll
        for (int k = 0; k < K; ++k) store(k);
        each_changed([&](int v, uint32_t &x) { out[v] = from_float<Tout>(__uint_as_float(x) * f); });
    }
}

}  // namespace ckv
