// Verification of drafted tokens against the target model's probabilities.
#pragma once

#include <cuda_bf16.h>

#include "ckv_common.cuh"

namespace ckv {

// For a request with n drafted tokens x_0 .. x_{n-1}, target rows p_0 .. p_n and draft rows q_0 ..
// q_{n-1}: draft j is accepted while u_j q_j(x_j) < p_j(x_j); at the first refusal j the next token is
// drawn from the weights max(p_j - q_j, 0), after n acceptances from p_n.  Drawn means the first token
// whose running sum of weights exceeds u * (sum of all weights).  Without draft rows q_j is a point
// mass at x_j.  If the differences leave nothing (p_j <= q_j everywhere), the weights are p_j.
//
// Products, differences and sums are in 64 bits: over 10^5 tokens a sum in 32 bits moves the borders
// between tokens by more than many tokens' probability.
//
// Bound by reading the one or two rows that decide (4 V bytes each in fp32).  A cluster works on a
// request; every warp owns a contiguous segment of the vocabulary and adds up its weights, the
// segments' sums tell which warp holds the crossing, and that warp walks its segment once more
// (from the cache) to find the token.  All sums are taken in a fixed order.
struct VerifyParams {
    const int32_t *draft_tokens;    // [batch][max_draft]
    const int32_t *draft_lens;      // [batch] or NULL: max_draft each
    const void *target;             // [batch][max_draft + 1] rows of `vocab`, target_stride elements apart
    const void *draft;              // [batch][max_draft] rows, draft_stride elements apart, or NULL
    const float *u_accept;          // [batch][max_draft]
    const float *u_sample;          // [batch]
    int32_t *tokens;                // [batch][max_draft + 1]
    int32_t *accepted;              // [batch]
    long long target_stride, draft_stride;
    int32_t batch, max_draft, vocab;
};

constexpr int kVerifyThreads = 512;
constexpr int kMaxCluster = 16;

__device__ __forceinline__ float prob_of(const float *p) { return __ldg(p); }
__device__ __forceinline__ float prob_of(const __nv_bfloat16 *p)
{
    return __uint_as_float((uint32_t)__ldg((const unsigned short *)p) << 16);
}

template <typename T, int kVec>
__device__ __forceinline__ void load_probs(const T *p, float (&out)[kVec])
{
    if constexpr (kVec == 1) {
        out[0] = prob_of(p);
    } else if constexpr (sizeof(T) == 4) {
        const float4 v = __ldg((const float4 *)p);
        out[0] = v.x; out[1] = v.y; out[2] = v.z; out[3] = v.w;
    } else {
        const uint2 v = __ldg((const uint2 *)p);
        out[0] = __uint_as_float(v.x << 16); out[1] = __uint_as_float(v.x & 0xffff0000u);
        out[2] = __uint_as_float(v.y << 16); out[3] = __uint_as_float(v.y & 0xffff0000u);
    }
}

// max(p - q, 0) in 64 bits; a NaN counts as nothing.
__device__ __forceinline__ double weight_of(float p, float q)
{
    const double w = (double)p - (double)q;
    return w > 0.0 ? w : 0.0;
}

template <typename T, int kVec>
__global__ void __launch_bounds__(kVerifyThreads)
draft_verify_kernel(const VerifyParams p)
{
    constexpr int kWarps = kVerifyThreads / 32;
    constexpr int kStripe = 32 * kVec;           // tokens a warp reads at once
    constexpr int kUnroll = 8;
    __shared__ int s_taken;
    __shared__ double s_warp[kWarps];
    __shared__ double s_cta[2][kMaxCluster];     // every CTA's sum, in every CTA; one set per round
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int rank = (int)cluster_rank(), ctas = (int)cluster_size();
    const int r = blockIdx.x / ctas;
    const T *target = static_cast<const T *>(p.target), *draft = static_cast<const T *>(p.draft);
    grid_dependency_wait();
    grid_launch_dependents();
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");

    const int n = p.draft_lens != nullptr ? min(max(__ldg(p.draft_lens + r), 0), p.max_draft) : p.max_draft;
    if (warp == 0) {
        int taken = n;
        for (int base = 0; base < n; base += 32) {
            const int j = base + lane;
            bool ok = false;
            if (j < n) {
                const int x = __ldg(p.draft_tokens + (size_t)r * p.max_draft + j);
                if (x >= 0 && x < p.vocab) {     // a token outside the vocabulary is refused
                    const double u = __ldg(p.u_accept + (size_t)r * p.max_draft + j);
                    const double px = prob_of(target + ((size_t)r * (p.max_draft + 1) + j) * p.target_stride + x);
                    const double qx = draft != nullptr ? (double)prob_of(draft + ((size_t)r * p.max_draft + j) * p.draft_stride + x) : 1.0;
                    ok = u * qx < px;
                }
            }
            const unsigned refused = __ballot_sync(0xffffffffu, j < n && !ok);
            if (refused) { taken = base + __ffs(refused) - 1; break; }
        }
        if (lane == 0) s_taken = taken;
        if (rank == 0) {
            for (int j = lane; j <= p.max_draft; j += 32)
                if (j != taken)
                    p.tokens[(size_t)r * (p.max_draft + 1) + j] = j < taken ? __ldg(p.draft_tokens + (size_t)r * p.max_draft + j) : -1;
            if (lane == 0) p.accepted[r] = taken;
        }
    }
    __syncthreads();
    const int taken = s_taken;
    const bool refused = taken < n;
    const T *p_row = target + ((size_t)r * (p.max_draft + 1) + taken) * p.target_stride;
    const T *q_row = refused && draft != nullptr ? draft + ((size_t)r * p.max_draft + taken) * p.draft_stride : nullptr;
    int hole = refused && draft == nullptr ? __ldg(p.draft_tokens + (size_t)r * p.max_draft + taken) : -1;
    int32_t *out = p.tokens + (size_t)r * (p.max_draft + 1) + taken;

    // this warp's segment of the vocabulary
    const int segments = ctas * kWarps;
    const int stripes = (p.vocab + kStripe - 1) / kStripe;
    const int per = (stripes + segments - 1) / segments;
    const int from = min((rank * kWarps + warp) * per, stripes), to = min(from + per, stripes);
    auto weights = [&](int stripe, double (&w)[kVec]) {
        const int at = stripe * kStripe + lane * kVec;
        float pv[kVec], qv[kVec];
#pragma unroll
        for (int x = 0; x < kVec; ++x) pv[x] = qv[x] = 0.f;
        if (at < p.vocab) {                      // kVec > 1 only if it divides the vocabulary
            load_probs<T, kVec>(p_row + at, pv);
            if (q_row != nullptr) load_probs<T, kVec>(q_row + at, qv);
        }
#pragma unroll
        for (int x = 0; x < kVec; ++x) w[x] = at + x == hole ? 0.0 : weight_of(pv[x], qv[x]);
    };
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");                // every CTA runs: its memory may be written
    for (int round = 0; round < 2; ++round) {
        double sum = 0.0;
        for (int stripe = from; stripe < to; stripe += kUnroll) {
            double part[kUnroll];
#pragma unroll
            for (int k = 0; k < kUnroll; ++k) {
                double w[kVec];
                part[k] = 0.0;
                if (stripe + k < to) {
                    weights(stripe + k, w);
#pragma unroll
                    for (int x = 0; x < kVec; ++x) part[k] += w[x];
                }
            }
#pragma unroll
            for (int k = 0; k < kUnroll; ++k) sum += part[k];
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (lane == 0) s_warp[warp] = sum;
        __syncthreads();
        if (warp == 0) {
            double mine = 0.0;
            for (int w = 0; w < kWarps; ++w) mine += s_warp[w];
            if (lane < ctas) {
                const uint32_t dst = cluster_map(smem_u32(&s_cta[round][rank]), lane);
                asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(dst), "d"(mine) : "memory");
            }
        }
        cluster_barrier();
        double total = 0.0;
        for (int c = 0; c < ctas; ++c) total += s_cta[round][c];
        if (!(total > 0.0)) {                    // the same in every CTA
            if (round == 0 && (q_row != nullptr || hole >= 0)) {
                q_row = nullptr;
                hole = -1;
                continue;
            }
            if (rank == 0 && threadIdx.x == 0) *out = -1;      // a row without any weight
            return;
        }
        const double goal = (double)__ldg(p.u_sample + r) * total;
        // the CTA, then the warp, whose weights cross the goal; rounding may leave none, then the last
        // one with any weight
        double run = 0.0, before = 0.0;
        int owner = -1;
        for (int c = 0; c < ctas; ++c) {
            const double v = s_cta[round][c];
            if (v > 0.0) { owner = c; before = run; if (run + v > goal) break; }
            run += v;
        }
        if (owner != rank) return;
        run = before;
        owner = -1;
        for (int w = 0; w < kWarps; ++w) {
            const double v = s_warp[w];
            if (v > 0.0) { owner = w; before = run; if (run + v > goal) break; }
            run += v;
        }
        if (owner != warp) return;
        run = before;
        int token = -1;
        for (int stripe = from; stripe < to; ++stripe) {
            double w[kVec], own = 0.0;
            weights(stripe, w);
#pragma unroll
            for (int x = 0; x < kVec; ++x) own += w[x];
            double upto = own;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const double v = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += v;
            }
            const unsigned any = __ballot_sync(0xffffffffu, own > 0.0);
            const unsigned over = __ballot_sync(0xffffffffu, own > 0.0 && run + upto > goal);
            if (any) {
                // the lane that crosses, else (so far) the last lane with any weight
                const int src = over ? __ffs(over) - 1 : 31 - __clz(any);
                int pick = -1;
                double at = run + (upto - own);
#pragma unroll
                for (int x = 0; x < kVec; ++x) {
                    if (w[x] > 0.0 && !(pick >= 0 && at > goal)) pick = x;
                    at += w[x];
                }
                token = stripe * kStripe + src * kVec + __shfl_sync(0xffffffffu, pick, src);
            }
            if (over) break;
            run += __shfl_sync(0xffffffffu, upto, 31);
        }
        if (lane == 0) *out = token;
        return;
    }
}

}  // namespace ckv
