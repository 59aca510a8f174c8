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
// Its floor is HBM's: a logit is read once and a result written once, 32 us for 512 rows of 50257 tokens with everything, of which it takes
// 68 (alone 31 and 43).  It is bound by waiting: of the 13 cycles between two issues of a warp 4.2 are for pieces on their way from L2 and 2.2
// at the barriers between the lists' steps, with 7 of 16 warps a scheduler; neither issue (2.1 of 4) nor DRAM (33 %) is full.
// A cluster of CTAs owns a row, a CTA a slice of it.  The slice is brought into L2 by one bulk prefetch as the CTA starts, and read there twice, as pieces of 16 aligned
// bytes: for the maximum and the sum, and for the results.  (Held in registers between, 32 tokens a thread, it cost 64
// registers and two to four CTAs an SM: 141 us for 512 rows of 50257 tokens with everything, against 68; alone 57 against 43.)
// Tokens that change are few.  Meanwhile the CTA marks them, a bit each; the marks before a token give it a place in short
// arrays in shared memory, where its occurrences are counted and its bias's last entry is found (whole numbers, and
// the largest of entries: the order of atomics does not show), and where the CTA's threads handle them in turn.
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
    int32_t marked;                 // tokens of a CTA that can change
};

// Words of marks that a CTA has room for.
constexpr int kLogitsWords = 1024, kLogitsMaxVocab = 262128;

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
    constexpr int kWarps = T / 32;
    constexpr int E = 16 / sizeof(Tin), U = 16 / E;              // elements of a piece, pieces of a thread at a time
    extern __shared__ uint32_t s_marked[];        // [marked]: the tokens' places in the slice; counts, bit 31: in the prompt, then values; entries plus 1
    __shared__ uint32_t s_marks[kLogitsWords];    // a bit per token of the slice
    __shared__ int s_base[kLogitsWords];          // marks before a word's
    __shared__ int s_total[kWarps];
    __shared__ float s_max[kWarps], s_sum[kWarps];
    __shared__ unsigned s_at[kWarps];
    __shared__ uint4 s_share[16];                 // every CTA's maximum, sum and place of the maximum, written by them
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = (int)cluster_rank(), ctas = (int)cluster_size();
    const int row = blockIdx.x / ctas, b = row / p.rows, j = row % p.rows, V = p.vocab;
    const Tin *in = static_cast<const Tin *>(p.logits) + row * p.stride;
    Tout *out = static_cast<Tout *>(p.out) + row * p.out_stride;
    const uint32_t *words = p.mask != nullptr ? p.mask + row * p.mask_stride : nullptr;
    const int off = (int)(reinterpret_cast<uintptr_t>(in) / sizeof(Tin) % E);    // elements before the row in its first piece
    const int first = rank * p.pieces * E - off, last = min(first + p.pieces * E, V);            // the slice; `first` may lie below 0
    const int pieces = max(0, (last - first + E - 1) / E);
    const bool changes = p.marked > 0;
    uint32_t *s_place = s_marked, *s_count = s_marked + p.marked, *s_entry = s_count + p.marked;
    float *s_value = (float *)s_count;
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");        // waited for before others' shared memory is written
    if (changes) {
#pragma unroll 1
        for (int i = tid; i < (p.bias_ids != nullptr ? 2 : 1) * p.marked; i += T) s_count[i] = 0u;
#pragma unroll 1
        for (int i = tid; i < kLogitsWords; i += T) s_marks[i] = 0u;
    }
    grid_dependency_wait();
    grid_launch_dependents();
    // up to 15 bytes beside the row are read with it, and not used
    if (p.probs && pieces > 0 && tid == 0)
        asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(in + first), "r"(pieces * 16) : "memory");

    // fetched ahead of the marks
    const float *pr = p.params + 4 * b;
    const float rep = p.params ? __ldg(pr) : 1.f, pres = p.params ? __ldg(pr + 1) : 0.f, freq = p.params ? __ldg(pr + 2) : 0.f;
    const float temperature = p.params ? __ldg(pr + 3) : 1.f;
    // ---- the tokens that change
    int marked = 0;
    if (changes) {
        const int32_t *text = p.history + b * p.history_stride, *drafted = p.drafts + (long long)b * (p.rows - 1), *ids = p.bias_ids + (long long)b * p.n_bias;
        const int n_drafts = p.drafts != nullptr ? j : 0;
        const int room = p.history != nullptr ? (int)min(p.history_stride, 0x7fffffffll) : 0;
        const int n = room > 0 ? min(max(__ldg(p.history_lens + b), 0), room) : 0, prompt = room > 0 ? __ldg(p.prompt_lens + b) : 0;
        __syncthreads();                          // the arrays are clear
        // calls fn(place in the slice, index) for the tokens of the lists that lie in the slice
        auto each = [&](auto history, auto bias) {
            auto place_of = [&](int token) { return token >= 0 && token >= first && token < last ? token - first : -1; };
            constexpr int kAhead = 8;             // tokens of a thread on their way together, the first ones before their number is known
#pragma unroll 1
            for (long long i0 = tid; i0 < (i0 == tid ? room : n); i0 += kAhead * T) {
                int token[kAhead];
#pragma unroll
                for (int k = 0; k < kAhead; ++k) token[k] = i0 + k * T < room ? __ldg(text + i0 + k * T) : -1;
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    const int at = i0 + k * T < n ? place_of(token[k]) : -1;
                    if (at >= 0) history(at, i0 + k * T < prompt);
                }
            }
#pragma unroll 1
            for (int i = tid; i < n_drafts; i += T) {
                const int at = place_of(__ldg(drafted + i));
                if (at >= 0) history(at, false);
            }
#pragma unroll 1
            for (int i = tid; i < p.n_bias; i += T) {
                const int at = place_of(__ldg(ids + i));
                if (at >= 0) bias(at, i);
            }
        };
        auto mark = [&](int at, int) { atomicOr(s_marks + at / 32, 1u << at % 32); };
        each(mark, mark);
        __syncthreads();
        constexpr int kOwn = kLogitsWords / T;    // words of a thread, neighbours
        int own_marks = 0;
#pragma unroll
        for (int w = 0; w < kOwn; ++w) own_marks += __popc(s_marks[tid * kOwn + w]);
        int upto = own_marks;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += v;
        }
        if (lane == 31) s_total[warp] = upto;
        __syncthreads();
        upto -= own_marks;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            upto += w < warp ? s_total[w] : 0;
            marked += s_total[w];
        }
#pragma unroll
        for (int w = 0; w < kOwn; ++w) {
            s_base[tid * kOwn + w] = upto;
            upto += __popc(s_marks[tid * kOwn + w]);
        }
        __syncthreads();
        auto index = [&](int at) {
            const int i = s_base[at / 32] + __popc(s_marks[at / 32] & ((1u << at % 32) - 1u));
            s_place[i] = at;                      // the same from whoever writes it
            return i;
        };
        each([&](int at, bool in_prompt) { in_prompt ? atomicOr(s_count + index(at), 0x80000000u) : atomicAdd(s_count + index(at), 1u); },
             [&](int at, int i) { atomicMax(s_entry + index(at), (uint32_t)i + 1u); });          // where an id stands twice, the last entry counts
        __syncthreads();
    }
    // ---- a thread's maximum, and the sum against it
    const bool greedy = !(temperature > 0.f);
    // neither infinite nor 0: 0 * scale has to be 0, and minus infinity times it minus infinity
    const float scale = greedy ? 1.4426950408889634f : fminf(fmaxf(1.4426950408889634f / temperature, 1e-44f), 3e38f);
    float most = -INFINITY, sum = 0.f;
    // Calls fn(i, elements) with this thread's pieces i, i + T, .. of the slice, U at a time, what is outside the row, not
    // allowed or marked at minus infinity.
    constexpr uint32_t kAll = (1u << E) - 1u;
    static_assert(T * E % 32 == 0, "pieces of a thread begin at the same bit of a word");
    auto each_pieces = [&](auto fn) {
        const Tin *at = in + first + tid * E;
        const int shift = (first + tid * E) & 31, mark_shift = tid * E & 31, last_word = (V - 1) >> 5;
#pragma unroll 1
        for (int i = tid; i < pieces; i += U * T, at += U * T * E) {
            const bool inner = i > 0 && i + (U - 1) * T < pieces - 1;            // nothing of these is outside the row
            uint4 raw[U];
            uint32_t bits[U];
#pragma unroll
            for (int k = 0; k < U; ++k) {
                raw[k] = make_uint4(0u, 0u, 0u, 0u);
                if (inner || i + k * T < pieces) raw[k] = *(const uint4 *)(at + k * T * E);
                bits[k] = kAll;
            }
            if (!inner) {
#pragma unroll
                for (int k = 0; k < U; ++k) {
                    const int v = first + (i + k * T) * E, from = max(0, -v), to = min(E, last - v);
                    bits[k] = to > from ? (1u << to) - (1u << from) : 0u;
                }
            }
            if (words != nullptr) {
                const int w = (first + i * E) >> 5;              // -1 for a piece that begins before the row
#pragma unroll
                for (int k = 0; k < U; ++k) {
                    const int n = w + k * (T * E / 32);          // words outside the mask hold nothing of the row
                    const uint32_t lo = __ldg(words + (inner ? n : min(max(n, 0), last_word))), hi = __ldg(words + min(n + 1, last_word));
                    bits[k] &= __funnelshift_r(lo, hi, shift);
                }
            }
            if (changes) {
#pragma unroll
                for (int k = 0; k < U; ++k)
                    if (inner || i + k * T < pieces) bits[k] &= ~(s_marks[i * E / 32 + k * (T * E / 32)] >> mark_shift);
            }
            float x[U][E];
            uint32_t every = kAll;
#pragma unroll
            for (int k = 0; k < U; ++k) {
                piece_elements(raw[k], x[k]);
                every &= bits[k];
            }
            if (every != kAll) {
#pragma unroll
                for (int k = 0; k < U; ++k)
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        if (!(bits[k] >> e & 1u)) x[k][e] = -INFINITY;
            }
            fn(i, x);
        }
    };
    if (changes) {                                // marked tokens, rounded step by step as the formula stands; loops of one step, as everything
                                                  // around them is run once: four at a time 70.2 us instead of 68.4 for 512 rows
#pragma unroll 1
        for (int i = tid; i < marked; i += T) {
            const int at = (int)s_place[i];
            float v = element(in[first + at]);
            const uint32_t c = s_count[i], times = c & 0x7fffffffu, entry = p.bias_ids != nullptr ? s_entry[i] : 0u;
            if (c != 0u) {
                v = v > 0.f ? __fdiv_rn(v, rep) : __fmul_rn(v, rep);
                v = __fsub_rn(v, __fmul_rn(freq, (float)times));
                if (times > 0u) v = __fsub_rn(v, pres);
            }
            if (entry != 0u) v = __fadd_rn(v, __ldg(p.bias + (long long)b * p.n_bias + entry - 1));
            if (words != nullptr && !(__ldg(words + (first + at) / 32) >> (first + at) % 32 & 1u)) v = -INFINITY;
            s_value[i] = v;
            most = fmaxf(most, v);
        }
        const float ref = most == -INFINITY ? 0.f : most;
#pragma unroll 1
        for (int i = tid; i < marked; i += T) sum += fast_exp2((s_value[i] - ref) * scale);
    }
    const bool whole = reinterpret_cast<uintptr_t>(out + first) % (sizeof(Tout) * E < 16 ? sizeof(Tout) * E : 16) == 0;
    auto store = [&](int i, const float *x) {
        const int v = first + i * E;
        if (i < pieces) store_elements<Tout, E>(out + v, x, whole, max(0, -v), min(E, last - v));
    };
    if (!p.probs) {
        __syncthreads();                          // in place: marked logits have been read
        each_pieces([&](int i, float (&x)[U][E]) {
#pragma unroll
            for (int k = 0; k < U; ++k) store(i + k * T, x[k]);
        });
        __syncthreads();
        for (int i = tid; i < marked; i += T) out[first + (int)s_place[i]] = from_float<Tout>(s_value[i]);
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        return;
    }
    each_pieces([&](int, float (&x)[U][E]) {
        float top = x[0][0];
#pragma unroll
        for (int k = 0; k < U; ++k)
#pragma unroll
            for (int e = 0; e < E; ++e) top = fmaxf(top, x[k][e]);
        if (top > most) {
            sum *= fast_exp2((most - top) * scale);
            most = top;
        }
        const float ref = most == -INFINITY ? 0.f : most;
#pragma unroll
        for (int k = 0; k < U; ++k)
#pragma unroll
            for (int e = 0; e < E; ++e) sum += fast_exp2((x[k][e] - ref) * scale);
    });
    // ---- the CTA's, then the row's
    const float own = most;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
    if (lane == 0) s_max[warp] = most;
    __syncthreads();
    most = s_max[lane % kWarps];
#pragma unroll
    for (int o = kWarps / 2; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
    sum *= own == -INFINITY ? 1.f : fast_exp2((own - most) * scale);             // a thread that saw NaN alone keeps it
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) s_sum[warp] = sum;
    if (greedy) {                                 // the first place of the slice's maximum
        unsigned at = 0x7fffffffu;
        each_pieces([&](int i, float (&x)[U][E]) {
#pragma unroll
            for (int k = 0; k < U; ++k)
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (x[k][e] == most) at = min(at, (unsigned)(first + (i + k * T) * E + e));
        });
        for (int i = tid; i < marked; i += T)
            if (s_value[i] == most) at = min(at, (unsigned)(first + (int)s_place[i]));
        at = __reduce_min_sync(0xffffffffu, at);
        if (lane == 0) s_at[warp] = at;
    }
    __syncthreads();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");          // every CTA of the cluster runs
    if (warp == 0) {
        sum = lane < kWarps ? s_sum[lane] : 0.f;
#pragma unroll
        for (int o = kWarps / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        sum = __shfl_sync(0xffffffffu, sum, 0);
        const unsigned at = greedy ? __reduce_min_sync(0xffffffffu, s_at[lane % kWarps]) : 0u;
        if (lane < ctas)                          // to CTA `lane`
            asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(cluster_map(smem_u32(s_share + rank), lane)),
                         "r"(__float_as_uint(most)), "r"(__float_as_uint(sum)), "r"(at), "r"(0u) : "memory");
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
    l *= m == -INFINITY ? 1.f : fast_exp2((m - top) * scale);    // a slice in which nothing is allowed has none, or a NaN
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
    const float total = __shfl_sync(0xffffffffu, l, 0);
    // NaN where a NaN or an infinity is among what is allowed; zeros where nothing is; greedy: 1 at the first of the largest
    const float all = top == -INFINITY ? 0.f : top, f = total == 0.f ? 0.f : 1.f / total;
    const unsigned best = __reduce_min_sync(0xffffffffu, there && m == top && top > -INFINITY ? share.z : 0x7fffffffu);
    const bool one = greedy && total == total;
    if (one) {
        const float none[E] = {};
        for (int i = tid; i < pieces; i += T) store(i, none);
        __syncthreads();
        if (tid == 0 && (int)best >= first && (int)best < last) out[best] = from_float<Tout>(1.f);
        return;
    }
    each_pieces([&](int i, float (&x)[U][E]) {
#pragma unroll
        for (int k = 0; k < U; ++k) {
#pragma unroll
            for (int e = 0; e < E; ++e) x[k][e] = fast_exp2((x[k][e] - all) * scale) * f;
            store(i + k * T, x[k]);
        }
    });
    if (!changes) return;
    __syncthreads();                              // pieces first, then what is marked in them
#pragma unroll 1
    for (int i = tid; i < marked; i += T) {
        out[first + (int)s_place[i]] = from_float<Tout>(fast_exp2((s_value[i] - all) * scale) * f);
    }
}

}  // namespace ckv
