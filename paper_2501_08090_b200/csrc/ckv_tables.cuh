// Block tables, lengths and slots from request lengths: pages that tokens need are taken from a list of
// free pages, pages that requests give up return to it.
#pragma once

#include "ckv_common.cuh"

namespace ckv {

// The free list is a stack: pages free[0 .. F - 1], taken from its end.  What a call moves is numbered in the
// order of requests and, within one, of its context:
//   release  page k of N goes to place F + N - 1 - k
//   assign   page k comes from place F - 1 - k
// so an assignment that is released again leaves the list as it was, and all places follow from one sum over the
// requests before.  A request is served if it needs no page, or if the needs of all requests up to and including
// it fit F: whoever is refused takes nothing, and nobody after it jumps the queue with a need of its own.
//
// Latency-bound: a few KB move, after lengths, count and pages have been fetched one after another.  Every CTA sums for
// itself, and CTAs share what is to be moved.  Where lengths or count are written in place the grid is one
// cluster, and all of them are read before its barrier.  256 requests that take a token each: assign 4.0 us, release 3.1;
// 64 requests that take prompts of up to 2047 tokens, with their slots: 3.8 and 2.8.
struct TablesParams {
    int32_t *block_tables;
    const int32_t *seq_lens;
    const int32_t *amounts;         // assign: tokens to add; release: lengths to keep
    int32_t *free_pages;
    const int32_t *free_count;
    int32_t *lens_out, *count_out;
    int32_t *step_lens, *new_start; // assign; may be NULL
    long long *slots;               // assign; may be NULL
    uint32_t *status;
    int32_t batch, max_pages_per_req, num_pages, n_slots;
    int32_t in_place;               // lengths or count are written where they are read: the grid is one cluster
};

__host__ __device__ __forceinline__ int pages_of(int tokens) { return tokens / kPageSize + (tokens % kPageSize != 0); }

// What is kept of every request in shared memory: sums of pages up to and including it, of tokens before it,
// and its length (-1: unusable).
constexpr int kTablesWords = 3;

// Exclusive sums over the block of two numbers a thread, and their totals.
__device__ __forceinline__ void block_sums(long long &a, long long &b, long long &total_a, long long &total_b)
{
    __shared__ long long s_a[32], s_b[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    long long ia = a, ib = b;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(0xffffffffu, ia, o), y = __shfl_up_sync(0xffffffffu, ib, o);
        if (lane >= o) { ia += x; ib += y; }
    }
    if (lane == 31) { s_a[warp] = ia; s_b[warp] = ib; }
    __syncthreads();
    long long before_a = 0, before_b = 0;
    total_a = total_b = 0;
#pragma unroll 4
    for (int w = 0; w < warps; ++w) {
        if (w == warp) { before_a = total_a; before_b = total_b; }
        total_a += s_a[w];
        total_b += s_b[w];
    }
    a = before_a + ia - a;
    b = before_b + ib - b;
}

// How many of the `n` sums, which do not decrease, are at most k: the first request whose sum exceeds it.
__device__ __forceinline__ int first_above(const int *sums, int n, int k)
{
    int r = 0;
#pragma unroll 1
    for (int half = 1 << (31 - __clz(n)); half > 0; half >>= 1)
        if (r + half <= n && sums[r + half - 1] <= k) r += half;
    return r;
}

__device__ __forceinline__ int clamp_int(long long x) { return (int)min(x, 0x7fffffffll); }

__device__ __forceinline__ int checked_count(const TablesParams &p)
{
    const int F = *p.free_count;
    if (F >= 0 && F <= p.num_pages) return F;
    if (threadIdx.x == 0) atomicOr(p.status, kStatusBadPage);
    return F < 0 ? 0 : p.num_pages;
}

template <bool kAssign>
__global__ void __launch_bounds__(1024)
pages_kernel(const TablesParams p)
{
    extern __shared__ int s_words[];
    // s_len: assign the length, -1 where the request is not served; release the pages kept, -1 where its length is unusable
    int *s_upto = s_words, *s_tokens = s_upto + p.batch, *s_len = s_tokens + p.batch;
    __shared__ int s_taken;
    const int rank = (int)blockIdx.x, ctas = (int)gridDim.x;
    const int chunk = (p.batch + blockDim.x - 1) / blockDim.x, r0 = min((int)threadIdx.x * chunk, p.batch), r1 = min(r0 + chunk, p.batch);
    const long long room = min((long long)p.max_pages_per_req * kPageSize, 0x7fffffffll);          // tokens that a table can hold
    if (threadIdx.x == 0) s_taken = 0;
    grid_dependency_wait();                       // every input may come from the preceding kernel
    grid_launch_dependents();
    const int F = checked_count(p);
    // ---- what each request moves, summed up
    long long pages = 0, tokens = 0;
    for (int r = r0; r < r1; ++r) {
        const int L = p.seq_lens[r], x = p.amounts[r];
        const bool fits = L >= 0 && L <= room && x >= 0 && (kAssign ? (long long)L + x <= room : x <= L);
        if (!fits && rank == 0) atomicOr(p.status, kStatusBadLength);
        const int moved = !fits ? 0 : kAssign ? pages_of(L + x) - pages_of(L) : pages_of(L) - pages_of(x);
        pages += moved;
        tokens += kAssign ? max(x, 0) : 0;
        s_upto[r] = moved;
        s_tokens[r] = kAssign ? max(x, 0) : 0;
        s_len[r] = !fits ? -1 : kAssign ? L : pages_of(x);
    }
    long long total_pages, total_tokens;
    block_sums(pages, tokens, total_pages, total_tokens);
    int taken = 0;
    for (int r = r0; r < r1; ++r) {
        const int moved = s_upto[r], n = s_tokens[r];
        pages += moved;
        if (pages <= F) taken = clamp_int(pages);
        else if (kAssign && moved > 0) s_len[r] = -1;
        s_upto[r] = clamp_int(pages);
        s_tokens[r] = clamp_int(tokens);
        tokens += n;
    }
    if (kAssign && taken > 0) atomicMax(&s_taken, taken);
    __syncthreads();
    if (p.in_place) cluster_barrier();            // every CTA has read the inputs
    taken = kAssign ? s_taken : clamp_int(total_pages);          // pages that move
    auto upto_before = [&](int r) { return r > 0 ? s_upto[r - 1] : 0; };
    const int at = rank * blockDim.x + threadIdx.x, stride = ctas * blockDim.x;
    if (rank == 0) {
        for (int r = r0; r < r1; ++r) {
            const int L = p.seq_lens[r], x = p.amounts[r];       // this thread alone writes their places
            const bool ok = s_len[r] >= 0;
            p.lens_out[r] = !ok ? L : kAssign ? L + x : x;
            if (kAssign && p.step_lens != nullptr) p.step_lens[r] = ok ? L + x : 0;
            if (kAssign && p.new_start != nullptr) p.new_start[r] = s_tokens[r];
        }
        if (threadIdx.x == 0) {
            if (kAssign && p.new_start != nullptr) p.new_start[p.batch] = clamp_int(total_tokens);
            if (!kAssign && (long long)F + total_pages > p.num_pages) atomicOr(p.status, kStatusBadPage);
            *p.count_out = kAssign ? F - taken : (int)min((long long)F + total_pages, (long long)p.num_pages);
        }
    }
    // (Loops of one step each: the code runs once, cold, and four steps at a time cost 3 us more in fetching it than they saved.)
    if constexpr (kAssign) {
        // the k-th page that is taken; -1 where the list holds none
        auto page_taken = [&](int k) {
            const int id = p.free_pages[F - 1 - k];
            return id >= 0 && id < p.num_pages ? id : -1;
        };
#pragma unroll 1
        for (long long k = at; k < taken; k += stride) {
            const int r = first_above(s_upto, p.batch, (int)k), id = page_taken((int)k);
            if (id < 0) atomicOr(p.status, kStatusBadPage);
            p.block_tables[(size_t)r * p.max_pages_per_req + pages_of(s_len[r]) + (int)k - upto_before(r)] = id;
        }
        const int n = p.slots != nullptr ? (int)min(total_tokens, (long long)p.n_slots) : 0;
#pragma unroll 1
        for (long long t = at; t < n; t += stride) {
            const int r = first_above(s_tokens, p.batch, (int)t) - 1, L = s_len[r];
            long long slot = -1;
            if (L >= 0) {
                const int pos = L + (int)t - s_tokens[r], column = pos / kPageSize, held = pages_of(L);
                const int id = column < held ? p.block_tables[(size_t)r * p.max_pages_per_req + column] : page_taken(upto_before(r) + column - held);
                if (id >= 0 && id < p.num_pages) slot = (long long)id * kPageSize + pos % kPageSize;
                else atomicOr(p.status, kStatusBadPage);
            }
            p.slots[t] = slot;
        }
    } else {
#pragma unroll 1
        for (long long k = at; k < taken; k += stride) {
            const int r = first_above(s_upto, p.batch, (int)k);
            int id = p.block_tables[(size_t)r * p.max_pages_per_req + s_len[r] + (int)k - upto_before(r)];
            if (id < 0 || id >= p.num_pages) {
                atomicOr(p.status, kStatusBadPage);
                id = -1;
            }
            const long long place = (long long)F + taken - 1 - k;
            if (place < p.num_pages) p.free_pages[place] = id;
        }
    }
}

}  // namespace ckv
