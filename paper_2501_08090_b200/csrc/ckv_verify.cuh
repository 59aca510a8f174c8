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
// Products are formed in 64 bits; weights are summed in pairs of fp32 whose rounding errors are kept, the
// pairs in fp64, their errors and the lower parts of differences in fp32: over 10^5 tokens a sum in 32 bits moves
// the borders between tokens by more than many tokens' probability.  Each error is at most 2^-24 of its
// pair, so a chain's sum of them is at most 2^-23 of its weights and each of its additions is off by 2^-24 of that.
// With one CTA a row a chain has V / 512 additions: 2^-38 of the sum at V = 2^18, 2^-41 in clusters of 8.
//
// Bound by reading the one or two rows that decide (4 V bytes each in fp32).  A cluster works on a
// request; every warp owns a contiguous segment of the vocabulary and adds up its weights, the
// segments' sums tell which warp holds the crossing, and that warp walks its segment once more
// (from the cache) to find the token.  Loads are issued in batches before anything is added, in
// the walk too: one stripe at a time, each waited for, the walk alone took 15 us of a 128256-token row
// split over 32 warps.  All sums are taken in a fixed order.
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

constexpr int kVerifyThreads = 256;
constexpr int kMaxCluster = 16;

__device__ __forceinline__ float prob_of(const float *p) { return __ldg(p); }
__device__ __forceinline__ float prob_of(const __nv_bfloat16 *p)
{
    return __uint_as_float((uint32_t)__ldg((const unsigned short *)p) << 16);
}

// 16 bytes of a row: kVec probabilities.
template <typename T>
struct ProbVec {
    static constexpr int kVec = 16 / sizeof(T);
    uint32_t w[4];

    __device__ __forceinline__ void clear() { w[0] = w[1] = w[2] = w[3] = 0u; }
    __device__ __forceinline__ void load(const void *p)          // 16-byte aligned
    {
        const uint4 v = __ldg((const uint4 *)p);
        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    }
    __device__ __forceinline__ float get(int x) const
    {
        if constexpr (sizeof(T) == 2) return __uint_as_float(x & 1 ? w[x / 2] & 0xffff0000u : w[x / 2] << 16);
        else return __uint_as_float(w[x]);
    }
    __device__ __forceinline__ void drop(int x)
    {
        if constexpr (sizeof(T) == 2) w[x / 2] &= x & 1 ? 0x0000ffffu : 0xffff0000u;
        else w[x] = 0u;
    }
    // bytes `by` .. `by` + 15 of this piece followed by `next` (by: a multiple of the type's size below 16)
    __device__ __forceinline__ void shift(const ProbVec &next, int by)
    {
        uint32_t v[8] = {w[0], w[1], w[2], w[3], next.w[0], next.w[1], next.w[2], next.w[3]};
        if (by & 8) {
#pragma unroll
            for (int x = 0; x < 6; ++x) v[x] = v[x + 2];
        }
        if (by & 4) {
#pragma unroll
            for (int x = 0; x < 5; ++x) v[x] = v[x + 1];
        }
#pragma unroll
        for (int x = 0; x < 4; ++x) w[x] = sizeof(T) == 2 ? __funnelshift_r(v[x], v[x + 1], (by & 2) * 8) : v[x];
    }
};

// A sum of weights: fp64, and in fp32 the rounding errors of the fp32 sums that went into it.
struct WeightSum {
    double hi = 0.0;
    float lo = 0.f;

    // a + b, both >= 0: one conversion to fp64 for two values (conversions, 16 a clock and SM, are what
    // limits a sum in fp64 here; the two-term sum's error is exact)
    __device__ __forceinline__ void add(float a, float b)
    {
        const float s = a + b, bb = s - a;
        lo += (a - (s - bb)) + (b - bb);
        hi += (double)s;
    }
    __device__ __forceinline__ double total() const { return hi + (double)lo; }
};

// A row's weights: max(p - q, 0), with q = 0 where there is no draft row; 0 for the token `hole` and for a
// NaN.  Rows may start anywhere.  A warp reads stripes of 32 pieces that are aligned in the target's
// row (token 0 lies `skip` tokens into stripe 0); the draft's piece is put together from two where
// its row starts at another offset.  A piece is read if it holds a token of the row; what else
// it holds is dropped.
template <typename T, bool kDraft>
struct Weights {
    using Vec = ProbVec<T>;
    static constexpr int kVec = Vec::kVec;
    static constexpr int kStripe = 32 * kVec;
    static constexpr int kBatch = kDraft ? 2 : sizeof(T) == 2 ? 4 : 8;      // stripes whose loads are in flight together
    const T *p, *q;
    int vocab, hole, lane, skip;

    __device__ __forceinline__ Weights(const T *p_, const T *q_, int vocab_, int hole_, int lane_)
        : p(p_), q(q_), vocab(vocab_), hole(hole_), lane(lane_), skip((int)(((uintptr_t)p_ & 15u) / sizeof(T)))
    {
    }
    __device__ __forceinline__ int stripes() const { return (vocab + skip + kStripe - 1) / kStripe; }
    __device__ __forceinline__ int token(int stripe) const { return stripe * kStripe + lane * kVec - skip; }
    __device__ __forceinline__ bool holds(int first) const { return first + kVec > 0 && first < vocab; }

    struct Batch { Vec p[kBatch], q[kDraft ? kBatch : 1]; };
    // the loads of stripes at .. at + kBatch - 1, as far as they lie before `end`
    __device__ __forceinline__ void load(Batch &b, int at, int end) const
    {
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const int first = token(at + k);
            b.p[k].clear();
            if (at + k < end && holds(first)) b.p[k].load(p + first);
        }
        if constexpr (kDraft) {
            const int by = (int)((uintptr_t)(q - skip) & 15u);   // the same for every piece
            Vec next[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const int first = token(at + k), before = first - by / (int)sizeof(T);
                const bool live = at + k < end;
                b.q[k].clear();
                next[k].clear();
                if (live && holds(before)) b.q[k].load(q + before);
                if (live && by != 0 && holds(before + kVec)) next[k].load(q + before + kVec);
            }
            if (by != 0) {
#pragma unroll
                for (int k = 0; k < kBatch; ++k) b.q[k].shift(next[k], by);
            }
        }
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const int first = token(at + k);
            const bool edge = first < 0 || first + kVec > vocab, holed = !kDraft && (unsigned)(hole - first) < (unsigned)kVec;
            if (edge || holed) {
#pragma unroll
                for (int x = 0; x < kVec; ++x)
                    if ((unsigned)(first + x) >= (unsigned)vocab || (!kDraft && first + x == hole)) {
                        b.p[k].drop(x);
                        if constexpr (kDraft) b.q[k].drop(x);
                    }
            }
        }
    }
    // weight = hi + lo exactly (lo = 0 without a draft row)
    __device__ __forceinline__ float weight(const Batch &b, int k, int x, float &lo) const
    {
        const float pv = b.p[k].get(x);
        if constexpr (kDraft) {
            const float qv = b.q[k].get(x);
            const bool more = pv > qv;           // false for a NaN
            const float w = more ? pv - qv : 0.f;
            lo = more ? (pv - w) - qv : 0.f;
            return w;
        } else {
            lo = 0.f;
            return fmaxf(pv, 0.f);
        }
    }
    __device__ __forceinline__ void add(WeightSum &sum, const Batch &b, int k) const
    {
#pragma unroll
        for (int x = 0; x < kVec; x += 2) {
            float l0, l1;
            const float w0 = weight(b, k, x, l0), w1 = weight(b, k, x + 1, l1);
            sum.add(w0, w1);
            if constexpr (kDraft) sum.lo += l0 + l1;
        }
    }
    __device__ double segment_sum(int from, int to) const
    {
        WeightSum sum[2];                        // two chains of additions
        Batch b;
        for (int at = from; at < to; at += kBatch) {
            load(b, at, to);
#pragma unroll
            for (int k = 0; k < kBatch; ++k) add(sum[k & 1], b, k);
        }
        double all = sum[0].total() + sum[1].total();
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
        return all;
    }
    // The first token of the segment whose running sum, `run` before the segment, exceeds `goal`; if
    // rounding leaves none, the last one with any weight.
    __device__ int walk(int from, int to, double run, double goal) const
    {
        constexpr int kAt = kDraft ? 2 : 4;      // stripes at a time: their sums stay in registers
        Batch b;
        int hit = -1;                            // the crossing stripe, or so far the last one with any weight
        double hit_run = run;
        bool found = false;
        for (int at = from; at < to && !found; at += kAt) {
            load(b, at, min(to, at + kAt));
            double sum[kAt];
#pragma unroll
            for (int k = 0; k < kAt; ++k) {
                WeightSum own;
                add(own, b, k);
                sum[k] = own.total();
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1)
#pragma unroll
                for (int k = 0; k < kAt; ++k) sum[k] += __shfl_xor_sync(0xffffffffu, sum[k], o);
#pragma unroll
            for (int k = 0; k < kAt; ++k) {
                if (sum[k] > 0.0 && !found) {
                    hit = at + k;
                    hit_run = run;
                    found = run + sum[k] > goal;
                }
                run += sum[k];
            }
        }
        return hit < 0 ? -1 : in_stripe(hit, hit_run, found ? goal : INFINITY);
    }
    __device__ int in_stripe(int stripe, double run, double goal) const
    {
        Batch b;
        load(b, stripe, stripe + 1);
        WeightSum sum;
        add(sum, b, 0);
        const double own = sum.total();
        double upto = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const double v = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += v;
        }
        const unsigned any = __ballot_sync(0xffffffffu, own > 0.0);
        const unsigned over = __ballot_sync(0xffffffffu, own > 0.0 && run + upto > goal);
        const int src = over ? __ffs(over) - 1 : 31 - __clz(any);        // some lane has weight
        int pick = 0;
        bool found = false;
        double at = run + (upto - own);
#pragma unroll
        for (int x = 0; x < kVec; ++x) {
            float lo;
            const float hi = weight(b, 0, x, lo);
            if (hi > 0.f && !(found && at > goal)) { pick = x; found = true; }
            at += (double)hi + (double)lo;
        }
        return __shfl_sync(0xffffffffu, token(stripe) + pick, src);
    }
};

template <typename T>
__global__ void __launch_bounds__(kVerifyThreads, 4)
draft_verify_kernel(const VerifyParams p)
{
    constexpr int kWarps = kVerifyThreads / 32;
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
    const int hole = refused && draft == nullptr ? __ldg(p.draft_tokens + (size_t)r * p.max_draft + taken) : -1;
    int32_t *out = p.tokens + (size_t)r * (p.max_draft + 1) + taken;
    const Weights<T, true> differences(p_row, q_row, p.vocab, -1, lane);
    Weights<T, false> plain(p_row, nullptr, p.vocab, hole, lane);

    // this warp's segment of the vocabulary, in stripes
    const int segments = ctas * kWarps;
    const int stripes = plain.stripes();
    const int per = (stripes + segments - 1) / segments;
    const int from = min((rank * kWarps + warp) * per, stripes), to = min(from + per, stripes);
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");                // every CTA runs: its memory may be written
    for (int round = 0; round < 2; ++round) {
        const bool by_difference = q_row != nullptr && round == 0;
        const double sum = by_difference ? differences.segment_sum(from, to) : plain.segment_sum(from, to);
        if (lane == 0) s_warp[warp] = sum;
        __syncthreads();
        if (warp == 0) {
            double mine = 0.0;
#pragma unroll
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
            if (round == 0 && (by_difference || hole >= 0)) {
                plain.hole = -1;
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
        const int token = by_difference ? differences.walk(from, to, before, goal) : plain.walk(from, to, before, goal);
        if (lane == 0) *out = token;
        return;
    }
}

}  // namespace ckv
