// Key bounds of the pages and the selection of pages by them: what the page-sparse attention of long
// contexts needs beside the attention kernel.
#pragma once

#include <cuda_bf16.h>

#include "ckv_common.cuh"

namespace ckv {

// ------------------------------------------------------------------------------------------
// The index.  For every (layer, page, kv head) a record of 2 d bytes, lo[d] then hi[d] (int8), and a
// step (fp32, a power of two): lo[x] * step <= k[x] <= hi[x] * step for each key k of the page that
// the context holds.  With m the largest |k[x]| of the page and head (at least 2^-100), the step is
// 2^(floor(log2 m) - 6), or twice that where m would need more than 127 steps; lo is rounded down
// and hi up.  A power of two makes every quotient exact, so an index is the same bits whoever builds
// it.  A page that holds a key with an infinity or a NaN gets lo = -127, hi = 127 and a step of 2^121, which only
// keys beside bf16's largest exceed (2^122): it is nearly always selected, and attention then shows what a
// full pass would have shown: a NaN, or a weight of 0 where its scores are minus infinity.
// Records come first, all layers, then all steps.
// ------------------------------------------------------------------------------------------
constexpr float kIndexStepOfInvalid = 2.658455991569832e36f;      // 2^121

// Step exponent for a largest magnitude m; 2^-exponent comes back in `inv`.
__device__ __forceinline__ int step_exponent(float m, float &inv)
{
    const int e = (int)(__float_as_uint(fmaxf(m, 7.888609052210118e-31f)) >> 23) - 127 - 6;    // 2^-100
    inv = __uint_as_float((uint32_t)(127 - e) << 23);
    return e;
}

// The stretch of work that each warp of a grid takes when the units of all requests lie on one axis that
// is cut evenly.  Executed by whole CTAs of kThreads: the requests' units are summed once a CTA (once a warp,
// every warp of an SM repeating it, it took 2.6 us of score_pages_kernel's 20).  units_of(r): the units of request
// r.  T counts them.
template <typename T>
struct Stretch {
    T begin, n;                     // first unit of the warp, their number (0: none)
    T before;                       // units of the requests before r
    int r;                          // the request that holds `begin`
};

template <int kThreads, typename T, typename UnitsOf>
__device__ __forceinline__ Stretch<T> find_stretch(UnitsOf units_of, int batch)
{
    constexpr int kWarps = kThreads / 32;
    __shared__ T s_upto[kThreads];
    __shared__ T s_warp[kWarps];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const T warps = (T)gridDim.x * kWarps, warp = (T)blockIdx.x * kWarps + w;
    Stretch<T> s = {0, 0, 0, -1};
    T before = 0, total = 0;
    if (batch > kThreads) {                      // more requests than threads: their sum first
        for (int r = threadIdx.x; r < batch; r += kThreads) total += units_of(r);
#pragma unroll
        for (int x = 16; x > 0; x >>= 1) total += __shfl_xor_sync(0xffffffffu, total, x);
        if (lane == 0) s_warp[w] = total;
        __syncthreads();
        total = 0;
#pragma unroll
        for (int x = 0; x < kWarps; ++x) total += s_warp[x];
    }
    for (int base = 0; base < batch; base += kThreads) {
        const int r = base + threadIdx.x;
        T upto = r < batch ? (T)units_of(r) : (T)0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const T v = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += v;
        }
        __syncthreads();                         // the shared arrays may still be read
        if (lane == 31) s_warp[w] = upto;
        __syncthreads();
        T all = 0;
#pragma unroll
        for (int x = 0; x < kWarps; ++x) {
            if (x < w) upto += s_warp[x];
            all += s_warp[x];
        }
        s_upto[threadIdx.x] = upto;
        __syncthreads();
        if (batch <= kThreads) total = all;
        if (base == 0) {
            const T per = (total + warps - 1) / warps;
            s.begin = warp * per;
            s.n = s.begin < total ? min(per, total - s.begin) : (T)0;
        }
        if (s.n > 0 && s.r < 0 && s.begin < before + all) {
            int at = 0;
            while (s_upto[at + 31] <= s.begin - before) at += 32;
            at += __ffs(__ballot_sync(0xffffffffu, s_upto[at + lane] > s.begin - before)) - 1;
            s.r = base + at;
            s.before = before + (at > 0 ? s_upto[at - 1] : (T)0);
        }
        before += all;
    }
    return s;
}

struct IndexParams {
    const uint16_t *pool_layer;
    const int32_t *block_tables;
    const int32_t *seq_lens;
    uint8_t *records;               // this layer's
    float *steps;
    uint32_t *status;
    int32_t batch, max_pages_per_req, num_pages, num_kv_heads;
    int32_t last;                   // pages that hold one of the last `last` tokens; 0: all pages
};

__device__ __forceinline__ int index_pages(const IndexParams &p, int L, int &first)
{
    first = 0;
    if (tiles_of_length(L, p.max_pages_per_req) == 0) return 0;
    if (p.last > 0) first = max(0, L - p.last) / kPageSize;
    return (L + kPageSize - 1) / kPageSize - first;
}

// bulk_load_1d of data that is read once
__device__ __forceinline__ void bulk_load_once(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar, uint64_t policy)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1], %2, [%3], %4;"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar), "l"(policy) : "memory");
}

constexpr int kIndexWarps = 8;       // two CTAs an SM: 16 warps x 3 stages x 4 KB in flight (head_dim 128)
constexpr int kIndexStages = 3;

template <int D>
struct IndexLayout {
    static constexpr int kStageBytes = kPageSize * D * 2;        // the key rows of one (page, kv head)
    static constexpr int kBarOff = kIndexWarps * kIndexStages * kStageBytes;
    static constexpr int kSmemBytes = kBarOff + kIndexWarps * kIndexStages * 8;
};

// A place among the units (request, page, kv head) of an update, kv heads of a page first: neighbouring
// units are neighbours in memory.
struct IndexCursor {
    int r, page_at, page_end, h, L;

    __device__ __forceinline__ void next(const IndexParams &p)
    {
        if (++h < p.num_kv_heads) return;
        h = 0;
        if (++page_at < page_end) return;
        int n = 0;
        do {
            if (++r >= p.batch) return;
            L = __ldg(p.seq_lens + r);
            n = index_pages(p, L, page_at);
        } while (n == 0);
        page_end = page_at + n;
    }
};

// A warp takes one (page, kv head) at a time: 16 key rows, contiguous in the pool, one bulk copy.  The
// units of all requests lie on one axis that is cut evenly over the warps of the grid, so long and
// short requests balance; the copies of the units ahead fill a ring of the warp's own.  Bound by
// HBM: it reads the key half of the pool once.  (With the rows loaded to registers, one unit ahead, 96
// registers left 16 warps an SM and 4 KB each in flight: 75 us for 8 requests of 4001 to 32768 tokens.)
template <int D>
__global__ void __launch_bounds__(kIndexWarps * 32, 2)
kv_index_update_kernel(const IndexParams p)
{
    using Lay = IndexLayout<D>;
    constexpr int kVecs = D / 8;                 // 16-byte pieces of a row
    constexpr int kRows = 32 / kVecs;            // rows that a warp reads at once
    constexpr int NV = kPageSize / kRows;
    extern __shared__ __align__(128) uint8_t s_ring[];
    const int lane = threadIdx.x & 31;
    const int row0 = lane / kVecs;
    const uint32_t ring = smem_u32(s_ring) + (threadIdx.x >> 5) * kIndexStages * Lay::kStageBytes;
    const uint32_t bars = smem_u32(s_ring) + Lay::kBarOff + (threadIdx.x >> 5) * kIndexStages * 8;
    if (lane == 0) {
        for (int s = 0; s < kIndexStages; ++s) mbar_init(bars + s * 8, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_proxy_async();
    }
    __syncwarp();
    grid_dependency_wait();
    grid_launch_dependents();

    const Stretch<long long> st = find_stretch<kIndexWarps * 32, long long>([&](int r) {
        int first;
        const int n = index_pages(p, __ldg(p.seq_lens + r), first);
        if (blockIdx.x == 0 && n == 0) atomicOr(p.status, kStatusBadLength);
        return (long long)n * p.num_kv_heads;
    }, p.batch);
    const int units = (int)st.n;
    if (units <= 0) return;
    IndexCursor ic;
    ic.r = st.r;
    ic.L = __ldg(p.seq_lens + st.r);
    index_pages(p, ic.L, ic.page_at);
    ic.page_at += (int)((st.begin - st.before) / p.num_kv_heads);
    ic.page_end = (ic.L + kPageSize - 1) / kPageSize;
    ic.h = (int)((st.begin - st.before) % p.num_kv_heads);

    const uint64_t policy = l2_evict_first_policy();             // keys are read once
    // what the compute side needs of the units in flight, oldest first
    int f_page[kIndexStages], f_head[kIndexStages], f_tokens[kIndexStages];
    int next_id = __ldg(p.block_tables + (size_t)ic.r * p.max_pages_per_req + ic.page_at);
    int issued = 0;
    auto issue = [&](int &f_pg, int &f_h, int &f_t) {
        if (issued >= units) return;
        const int slot = issued % kIndexStages;
        f_pg = next_id;
        f_h = ic.h;
        f_t = min(kPageSize, ic.L - ic.page_at * kPageSize);
        if (f_pg < 0 || f_pg >= p.num_pages) {
            if (lane == 0) {
                atomicOr(p.status, kStatusBadPage);
                mbar_arrive_expect_tx(bars + slot * 8, 0);       // nothing to wait for
            }
            f_pg = -1;
        } else if (lane == 0) {
            const uint32_t bytes = f_t * D * 2;
            mbar_arrive_expect_tx(bars + slot * 8, bytes);
            bulk_load_once(ring + slot * Lay::kStageBytes, p.pool_layer + ((size_t)f_pg * p.num_kv_heads + f_h) * 2 * kPageSize * D, bytes, bars + slot * 8, policy);
        }
        if (++issued < units) {
            ic.next(p);
            if (ic.h == 0) next_id = __ldg(p.block_tables + (size_t)ic.r * p.max_pages_per_req + ic.page_at);
        }
    };
#pragma unroll
    for (int s = 0; s < kIndexStages; ++s) issue(f_page[s], f_head[s], f_tokens[s]);

    bool alive = true;
    int landed = 0;
    for (int done = 0; done < units; ++done) {
        const int slot = done % kIndexStages;
        alive = __all_sync(0xffffffffu, mbar_wait_bounded(bars + slot * 8, (done / kIndexStages) & 1, p.status));
        if (!alive) break;
        ++landed;
        const int page = f_page[0], head = f_head[0], tokens = f_tokens[0];
        // minimum and maximum over the rows; a NaN propagates, an infinity is an end of its own
        const __nv_bfloat162 top = __nv_bfloat162(__ushort_as_bfloat16(0x7f80), __ushort_as_bfloat16(0x7f80));
        const __nv_bfloat162 bottom = __nv_bfloat162(__ushort_as_bfloat16(0xff80), __ushort_as_bfloat16(0xff80));
        __nv_bfloat162 lo[4] = {top, top, top, top}, hi[4] = {bottom, bottom, bottom, bottom};
        const uint8_t *stage = s_ring + ((threadIdx.x >> 5) * kIndexStages + slot) * Lay::kStageBytes;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if (k * kRows + row0 < tokens) {
                const uint4 v = *(const uint4 *)(stage + (k * 32 + lane) * 16);
                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const __nv_bfloat162 e = *reinterpret_cast<const __nv_bfloat162 *>(&w[x]);
                    lo[x] = __hmin2_nan(lo[x], e);
                    hi[x] = __hmax2_nan(hi[x], e);
                }
            }
        }
        __syncwarp();                            // the stage has been read
#pragma unroll
        for (int s = 0; s + 1 < kIndexStages; ++s) { f_page[s] = f_page[s + 1]; f_head[s] = f_head[s + 1]; f_tokens[s] = f_tokens[s + 1]; }
        issue(f_page[kIndexStages - 1], f_head[kIndexStages - 1], f_tokens[kIndexStages - 1]);
        if (page < 0) continue;
#pragma unroll
        for (int o = kVecs; o < 32; o <<= 1) {
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                lo[x] = __hmin2_nan(lo[x], __shfl_xor_sync(0xffffffffu, lo[x], o));
                hi[x] = __hmax2_nan(hi[x], __shfl_xor_sync(0xffffffffu, hi[x], o));
            }
        }
        float a[8], b[8], m = 0.f;
        bool finite = true;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const float2 l = __bfloat1622float2(lo[x]), u = __bfloat1622float2(hi[x]);
            a[2 * x] = l.x; a[2 * x + 1] = l.y; b[2 * x] = u.x; b[2 * x + 1] = u.y;
        }
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            const float most = fmaxf(fabsf(a[x]), fabsf(b[x]));
            finite = finite && a[x] > -INFINITY && b[x] < INFINITY;      // false for a NaN
            m = fmaxf(m, most);
        }
        const bool invalid = __any_sync(0xffffffffu, !finite);
#pragma unroll
        for (int o = 1; o < kVecs; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        float inv;
        int e = step_exponent(m, inv);
        if (ceilf(m * inv) > 127.f) { ++e; inv *= 0.5f; }
        uint32_t lo8[2] = {0u, 0u}, hi8[2] = {0u, 0u};
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            const int l = invalid ? -127 : (int)floorf(a[x] * inv), u = invalid ? 127 : (int)ceilf(b[x] * inv);
            lo8[x / 4] |= (uint32_t)(l & 0xff) << (8 * (x & 3));
            hi8[x / 4] |= (uint32_t)(u & 0xff) << (8 * (x & 3));
        }
        const size_t at = (size_t)page * p.num_kv_heads + head;
        if (lane < kVecs) {
            *(uint2 *)(p.records + at * 2 * D + 8 * lane) = make_uint2(lo8[0], lo8[1]);
            *(uint2 *)(p.records + at * 2 * D + D + 8 * lane) = make_uint2(hi8[0], hi8[1]);
        }
        if (lane == 0) p.steps[at] = invalid ? kIndexStepOfInvalid : __uint_as_float((uint32_t)(e + 127) << 23);
    }
    // Do not leave while copies into this warp's ring may still be in flight (only after a wait gave up).
    if (!alive)
        for (int k = landed; k < issued; ++k) mbar_wait_bounded(bars + (k % kIndexStages) * 8, (k / kIndexStages) & 1, p.status);
}

// The bounds as numbers: bf16 [pages][kv heads][2][d] (exact: 7 bits times a power of two).
struct IndexValuesParams {
    const uint2 *records;           // this layer's
    const float *steps;
    uint4 *out;
    long long records_n;            // (page, kv head) records of the layer
};

// A thread turns 8 bounds at a time into 16 bytes, so that a warp's stores fill whole lines (16 bounds a
// thread, two stores 32 bytes apart from lane to lane, took 11.9 us of 9379 pages and 8 heads, where this takes 10.2).
template <int D>
__global__ void __launch_bounds__(256)
kv_index_values_kernel(const IndexValuesParams p)
{
    constexpr int kPieces = 2 * D / 8;           // of a record: a power of two
    constexpr int kUnroll = 4;
    grid_dependency_wait();
    grid_launch_dependents();
    const long long n = p.records_n * kPieces;
    const long long i0 = blockIdx.x * (long long)(blockDim.x * kUnroll) + threadIdx.x;
    uint2 v[kUnroll];
    float step[kUnroll];
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
        const long long i = i0 + k * blockDim.x;
        if (i < n) { v[k] = __ldg(p.records + i); step[k] = __ldg(p.steps + i / kPieces); }
    }
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
        const long long i = i0 + k * blockDim.x;
        if (i >= n) return;
        const uint32_t w[2] = {v[k].x, v[k].y};
        uint32_t o[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const uint32_t two = w[x / 2] >> (16 * (x & 1));
            o[x] = pack_bf16x2((float)(int8_t)(two & 0xff) * step[k], (float)(int8_t)((two >> 8) & 0xff) * step[k]);
        }
        p.out[i] = make_uint4(o[0], o[1], o[2], o[3]);
    }
}

// ------------------------------------------------------------------------------------------
// Selection.  The score of a page for a (request, kv head) bounds every product of a query of the
// group with a key of the page:
//   s = max over the group's query heads g of  2^e_g * step * sum_x max(q8[x] lo[x], q8[x] hi[x]),
// q8 the query in whole steps of 2^e_g (|q8| <= 127), e_g chosen as the index's steps are.  The sum
// splits by the sign of q8 into q8- . lo + q8+ . hi, so it is a product of 8-bit matrices: records
// of 16 pages (A, 2 d wide) times the group's 8 columns (q8-, q8+), in m16n8k32 tiles.  Sums of
// 8-bit products are exact in 32 bits and the steps are powers of two, so a score (but for one so
// small beside the group's largest that fp32 holds it as a denormal) does not depend on the order of
// summation, and the selection is the same whichever way the work is split.
//
// score_pages_kernel: candidate pages are scored in tiles of 16 (the rows of an MMA).  The
// tiles of all (request, kv head) pairs lie on one axis that is cut evenly over the warps of a grid
// that fills the GPU, so that contexts of very different lengths balance.  A warp copies the records
// of the tiles ahead of the one it multiplies into a ring of its own in shared memory (asynchronous
// copies: no registers wait for them, and a new pair's queries are converted while they fly).
// Bound by HBM: 2 d + 4 bytes per page and kv head, once.
// select_pair: a CTA finds the threshold among its keys (the scores as ordered 32-bit
// numbers, in registers) of its pair by counting them in 256 bins over the range still in question, then over
// the bin that holds the threshold, until that bin is wanted whole (usually the second time; bisection,
// one bit a turn, took 2-3 times as long), and writes the chosen pages in context order.  It copies
// the table to shared memory while the scores are still being computed.  The first `sink` and the last `recent`
// pages are always taken; equal scores go to the earlier page.
// ------------------------------------------------------------------------------------------
struct SelectParams {
    const uint8_t *records;
    const float *steps;
    const int32_t *block_tables;
    const int32_t *seq_lens;
    const uint16_t *q;              // [batch][Hq][d]
    int32_t *sel_tables;            // [batch][Hkv][budget]
    int32_t *sel_lens;              // [batch]
    uint32_t *keys;                 // [batch * Hkv][key_stride]
    int32_t key_stride;             // a multiple of 4, at least max_pages_per_req
    uint32_t *status;
    int32_t batch, max_pages_per_req, num_pages, num_kv_heads, group;
    int32_t budget, sink, recent;
    int32_t after_scores;           // select_pages_kernel directly follows score_pages_kernel
};

// Four CTAs an SM: 24 warps x 2 stages x 4 KB in flight (head_dim 128).  Other splits of the same shared
// memory are within 2 % (16 warps x 3, 26 x 2, 18 x 3), 8 warps x 6 is 18 % slower, 48 x 1 50 %.
constexpr int kScoreWarps = 6;
constexpr int kScoreStages = 2;
constexpr int kScoreCtas = 4;
constexpr int kMaxSelectThreads = 1024;

__device__ __forceinline__ void mma_s8_16832(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Candidate pages of a request: those that neither fit the budget with all others nor are kept anyway.
__device__ __forceinline__ int candidates(const SelectParams &p, int L)
{
    if (tiles_of_length(L, p.max_pages_per_req) == 0) return 0;
    const int n = (L + kPageSize - 1) / kPageSize;
    return n > p.budget && p.budget > p.sink + p.recent ? n - p.sink - p.recent : 0;
}

// The group's queries as B fragments: column = lane / 4, this lane's bytes of each piece; step0 and
// step1 are those of the two columns whose sums this lane receives (-1: no such head).
template <int D>
struct QueryFragments {
    static constexpr int kPieces = D / 64;       // 16-byte pieces of 8-bit channels that one lane holds
    uint32_t neg[kPieces][4], pos[kPieces][4];
    float step0, step1;

    // fetch: the loads; convert: what they brought in whole numbers (raw stays live in between)
    __device__ __forceinline__ void load(const uint16_t *q, int group, int lane)
    {
        uint32_t raw[kPieces][8];
        fetch(raw, q, group, lane);
        convert(raw, group, lane);
    }
    static __device__ __forceinline__ void fetch(uint32_t (&raw)[kPieces][8], const uint16_t *q, int group, int lane)
    {
        const int g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            uint4 a = make_uint4(0u, 0u, 0u, 0u), b = a;
            if (g < group) {
                const uint4 *src = (const uint4 *)(q + g * D + i * 64 + t * 16);
                a = __ldg(src);
                b = __ldg(src + 1);
            }
            raw[i][0] = a.x; raw[i][1] = a.y; raw[i][2] = a.z; raw[i][3] = a.w;
            raw[i][4] = b.x; raw[i][5] = b.y; raw[i][6] = b.z; raw[i][7] = b.w;
        }
    }
    __device__ __forceinline__ void convert(uint32_t (&raw)[kPieces][8], int group, int lane)
    {
        const int g = lane >> 2, t = lane & 3;
        // the largest magnitude, two at a time; a NaN would win, as an infinity does
        __nv_bfloat162 most = __nv_bfloat162(__ushort_as_bfloat16(0), __ushort_as_bfloat16(0));
#pragma unroll
        for (int i = 0; i < kPieces; ++i)
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                const uint32_t w = raw[i][x] & 0x7fff7fffu;
                most = __hmax2_nan(most, *reinterpret_cast<const __nv_bfloat162 *>(&w));
            }
        const float2 two = __bfloat1622float2(most);
        if (__any_sync(0xffffffffu, !(two.x < INFINITY && two.y < INFINITY))) {
            // infinities and NaN take no part in the selection: they become zeros
            float m = 0.f;
#pragma unroll 1
            for (int n = 0; n < kPieces * 16; ++n) {
                uint32_t keep = 0u;
#pragma unroll
                for (int i = 0; i < kPieces; ++i)
#pragma unroll
                    for (int x = 0; x < 8; ++x)
                        if (i * 16 + x * 2 == (n & ~1)) {
                            const uint32_t half = n & 1 ? 0xffff0000u : 0x0000ffffu;
                            if ((raw[i][x] & half & 0x7f807f80u) == (half & 0x7f807f80u)) raw[i][x] &= ~half;
                            keep = raw[i][x] & half & 0x7fff7fffu;
                        }
                m = fmaxf(m, __uint_as_float(n & 1 ? keep : keep << 16));
            }
            most = __nv_bfloat162(__float2bfloat16(m), __float2bfloat16(m));
        }
        const float2 pair = __bfloat1622float2(most);
        float m = fmaxf(pair.x, pair.y);
        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
        float inv;
        const int e = step_exponent(m, inv);
        // only the order of a pair's scores matters: steps relative to the group's largest, so that no
        // product overflows
        int e_max = e;
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) e_max = max(e_max, __shfl_xor_sync(0xffffffffu, e_max, x));
        const float step = g < group ? ldexpf(1.f, e - e_max) : -1.f;
        // x * inv is exact; added to 1.5 * 2^23 it is rounded to a whole number (ties to even), which is
        // then the low byte of the sum
        constexpr float kMagic = 12582912.f;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                uint32_t n8[4], p8[4];
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const uint32_t w = raw[i][2 * x + y / 2];
                    const float v = fmaf(__uint_as_float(y & 1 ? w & 0xffff0000u : w << 16), inv, kMagic);
                    n8[y] = __float_as_uint(fmaxf(fminf(v, kMagic), kMagic - 127.f));
                    p8[y] = __float_as_uint(fminf(fmaxf(v, kMagic), kMagic + 127.f));
                }
                neg[i][x] = __byte_perm(__byte_perm(n8[0], n8[1], 0x0040), __byte_perm(n8[2], n8[3], 0x0040), 0x5410);
                pos[i][x] = __byte_perm(__byte_perm(p8[0], p8[1], 0x0040), __byte_perm(p8[2], p8[3], 0x0040), 0x5410);
            }
        }
        step0 = __shfl_sync(0xffffffffu, step, (2 * t) * 4);
        step1 = __shfl_sync(0xffffffffu, step, (2 * t + 1) * 4);
    }
};

// One tile: the keys (ordered scores) of rows g and g + 8 from lane (g, t)'s pieces a and b of their records.
// Lane t = 0 of a row of four gets row g's, t = 1 row g + 8's; row_step is the step of that lane's row.
template <int D>
__device__ __forceinline__ uint32_t tile_key(const uint4 (&a)[2 * D / 64], const uint4 (&b)[2 * D / 64], const QueryFragments<D> &q, float row_step, int t)
{
    constexpr int P = 2 * D / 64;
    int acc[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const uint32_t *q8 = i < P / 2 ? q.neg[i] : q.pos[i - P / 2];
        mma_s8_16832(acc, a[i].x, b[i].x, a[i].y, b[i].y, q8[0], q8[1]);
        mma_s8_16832(acc, a[i].z, b[i].z, a[i].w, b[i].w, q8[2], q8[3]);
    }
    float x0 = fmaxf(q.step0 >= 0.f ? (float)acc[0] * q.step0 : -INFINITY, q.step1 >= 0.f ? (float)acc[1] * q.step1 : -INFINITY);
    float x1 = fmaxf(q.step0 >= 0.f ? (float)acc[2] * q.step0 : -INFINITY, q.step1 >= 0.f ? (float)acc[3] * q.step1 : -INFINITY);
    x0 = fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, 1));
    x1 = fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, 1));
    x0 = fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, 2));
    x1 = fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, 2));
    // 2^-22: sums stay below 2^21, steps below 2^123; + 0 makes a negative zero positive
    const float s = (t == 0 ? x0 : x1) * (row_step * 0x1p-22f) + 0.f;
    const uint32_t bits = __float_as_uint(s);
    return bits ^ ((uint32_t)((int32_t)bits >> 31) | 0x80000000u);
}

template <int D>
struct ScoreLayout {
    static constexpr int kPieces = 2 * D / 64;                   // 16-byte pieces of a record that one lane reads
    static constexpr int kStepsOff = 16 * 2 * D;                 // a stage: 16 records, then their 16 steps
    static constexpr int kStageBytes = kStepsOff + 64;
    static constexpr int kSmemBytes = kScoreWarps * kScoreStages * kStageBytes;
};

__device__ __forceinline__ void cp_async_16(uint32_t dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

__device__ __forceinline__ void cp_async_4(uint32_t dst, const void *src)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}

// A place on the axis of tiles: request, kv head, tile of that pair.  next() is executed by whole warps, and only
// while the warp's stretch goes on: it looks for the next request with candidates, 32 at a time, and behind the
// stretch that may be far (one context of 8000 pages before 7999 of one page: 1292 us, where those before it took 62).
struct TileCursor {
    int r, h, tile, cand, tiles;

    __device__ __forceinline__ void next(const SelectParams &p, int lane)
    {
        if (++tile < tiles) return;
        tile = 0;
        if (++h < p.num_kv_heads) return;
        h = 0;
        unsigned live = 0u;
        int c = 0;
        for (++r; live == 0u && r < p.batch; r += 32) {
            c = r + lane < p.batch ? candidates(p, __ldg(p.seq_lens + r + lane)) : 0;
            live = __ballot_sync(0xffffffffu, c > 0);
        }
        if (live == 0u) { cand = tiles = 0; return; }            // not reached: a stretch ends in a tile
        const int src = __ffs(live) - 1;
        r += src - 32;
        cand = __shfl_sync(0xffffffffu, c, src);
        tiles = (cand + 15) / 16;
    }
};

template <int D>
__global__ void __launch_bounds__(kScoreWarps * 32, kScoreCtas)
score_pages_kernel(const SelectParams p)
{
    using Lay = ScoreLayout<D>;
    constexpr int P = Lay::kPieces;
    extern __shared__ __align__(16) uint8_t s_ring[];
    const int lane = threadIdx.x & 31;
    const int g = lane >> 2, t = lane & 3;
    const uint32_t ring = smem_u32(s_ring) + (threadIdx.x >> 5) * kScoreStages * Lay::kStageBytes;
    grid_dependency_wait();
    grid_launch_dependents();

    const Stretch<int> st = find_stretch<kScoreWarps * 32, int>(
        [&](int r) { return (candidates(p, __ldg(p.seq_lens + r)) + 15) / 16 * p.num_kv_heads; }, p.batch);
    const int n_tiles = st.n;
    if (n_tiles <= 0) return;
    TileCursor ic;
    ic.r = st.r;
    ic.cand = candidates(p, __ldg(p.seq_lens + st.r));
    ic.tiles = (ic.cand + 15) / 16;
    ic.h = (st.begin - st.before) / ic.tiles;
    ic.tile = (st.begin - st.before) % ic.tiles;
    TileCursor cc = ic;

    // ---- the first pair's queries are on their way while the first copies are prepared
    uint32_t q_raw[QueryFragments<D>::kPieces][8];
    QueryFragments<D>::fetch(q_raw, p.q + (size_t)(ic.r * p.num_kv_heads + ic.h) * p.group * D, p.group, lane);

    // ---- issue side: lane (g, t) copies its quarter of the records of rows g and g + 8.  Table entries travel
    // in registers, 32 (two tiles) at a time, fetched one such chunk ahead.
    TileCursor pc = ic;                          // the chunk that is fetched next holds this tile
    int to_fetch = n_tiles;                      // tiles from there to the end of the warp's stretch
    auto fetch_chunk = [&]() -> int {
        if (to_fetch <= 0) return 0;
        const int32_t *table = p.block_tables + (size_t)pc.r * p.max_pages_per_req + p.sink;
        const int c = (pc.tile & ~1) * 16 + lane;
        const int id = c < pc.cand ? __ldg(table + c) : 0;
        const int last = min(pc.tile | 1, pc.tiles - 1);
        to_fetch -= last + 1 - pc.tile;
        pc.tile = last;
        if (to_fetch > 0) pc.next(p, lane);      // on to the next chunk
        return id;
    };
    int cur_ids = fetch_chunk(), next_ids = fetch_chunk();
    int issued = 0;
    auto issue = [&]() {
        if (issued < n_tiles) {
            const uint32_t stage = ring + (issued % kScoreStages) * Lay::kStageBytes;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                int page = __shfl_sync(0xffffffffu, cur_ids, (ic.tile & 1) * 16 + x * 8 + g);
                if (page < 0 || page >= p.num_pages) { atomicOr(p.status, kStatusBadPage); page = 0; }
                const size_t at = (size_t)page * p.num_kv_heads + ic.h;
                const uint8_t *src = p.records + at * 2 * D + t * 16;
#pragma unroll
                for (int i = 0; i < P; ++i) cp_async_16(stage + (x * P + i) * 512 + lane * 16, src + i * 64);
                if (t == x) cp_async_4(stage + Lay::kStepsOff + (x * 8 + g) * 4, p.steps + at);
            }
            if (++issued < n_tiles) {
                const bool last_of_chunk = (ic.tile & 1) || ic.tile + 1 == ic.tiles;
                ic.next(p, lane);
                if (last_of_chunk) {
                    cur_ids = next_ids;
                    next_ids = fetch_chunk();
                }
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int s = 0; s < kScoreStages; ++s) issue();

    // ---- compute side
    QueryFragments<D> q;
    q.convert(q_raw, p.group, lane);
    int q_pair = cc.r * p.num_kv_heads + cc.h;
    for (int done = 0; done < n_tiles; ++done) {
        const int pair = cc.r * p.num_kv_heads + cc.h;
        if (pair != q_pair) {
            q.load(p.q + (size_t)pair * p.group * D, p.group, lane);
            q_pair = pair;
        }
        asm volatile("cp.async.wait_group %0;" ::"n"(kScoreStages - 1) : "memory");
        __syncwarp();
        const uint8_t *stage = s_ring + ((threadIdx.x >> 5) * kScoreStages + done % kScoreStages) * Lay::kStageBytes;
        uint4 a[P], b[P];
#pragma unroll
        for (int i = 0; i < P; ++i) {
            a[i] = *(const uint4 *)(stage + i * 512 + lane * 16);
            b[i] = *(const uint4 *)(stage + (P + i) * 512 + lane * 16);
        }
        const uint32_t key = tile_key<D>(a, b, q, *(const float *)(stage + Lay::kStepsOff + ((t & 1) * 8 + g) * 4), t);
        __syncwarp();                            // the stage has been read
        issue();
        const int c = cc.tile * 16 + g + (t == 0 ? 0 : 8);
        if (t < 2 && c < cc.cand) p.keys[(size_t)pair * p.key_stride + c] = key;
        if (done + 1 < n_tiles) cc.next(p, lane);
    }
}

constexpr int kSelectBins = 256;
constexpr int kSelectRounds = 4;     // 8 bits of the keys' range each

struct SelectScratch {
    uint32_t *words;                // shared memory, 16-byte aligned: [candidates] page ids or keys; kScoreD: ids, then keys
    int (*hist)[kSelectBins];       // [kSelectRounds], 16-byte aligned
    uint32_t (*range)[32];          // [3]
};

// The selection of one (request, kv head) by a whole CTA, the waits for the preceding kernel included;
// emit(place, page id) is called once for each place of its list.  `report`: this CTA writes the
// request's length and flags an unusable one.
//
// kKeys > 0: at most that many keys a thread, in registers, and the table in shared memory; 0: the keys
// are in shared memory.  Few keys a thread and many threads are best, as the code runs once, from a cold
// instruction cache: for 64 requests of 512 to 2048 pages and 8 kv heads scores and selection take 41.5 us
// with 4 keys a thread, 43 with 8, 45.5 with 16, 44 to 51 with the keys in shared memory.
// kScoreD > 0: the CTA scores its pair's pages itself (head_dim kScoreD); score_pages_kernel is not launched.
template <int kKeys, int kScoreD, typename Emit>
__device__ __forceinline__ void select_pair(const SelectParams &p, int pair, const SelectScratch scratch, bool report, Emit emit)
{
    constexpr bool kInRegisters = kKeys > 0;
    constexpr int K = kInRegisters ? kKeys : 1;
    static_assert(K == 1 || K % 4 == 0, "keys are loaded four at a time");
    uint32_t *s_words = scratch.words;
    int (*s_hist)[kSelectBins] = scratch.hist;
    uint32_t (*s_range)[32] = scratch.range;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int r = pair / p.num_kv_heads;
    const int32_t *table = p.block_tables + (size_t)r * p.max_pages_per_req;
    // Right behind score_pages_kernel, the lengths and tables may be read before the wait: that kernel
    // released this one after its own wait, so whatever wrote them has completed.
    if (!p.after_scores) grid_dependency_wait();
    const int L = __ldg(p.seq_lens + r);
    const bool usable = tiles_of_length(L, p.max_pages_per_req) != 0;
    const int n = usable ? (L + kPageSize - 1) / kPageSize : 0;
    const int cand = n - p.sink - p.recent;      // pages sink .. sink + cand - 1 compete for `want` places
    const int want = p.budget - p.sink - p.recent;
    const bool chosen = n > p.budget && want > 0;
    // the pages that are always taken: the first ones and the last ones, or all
    const int ends = n > p.budget ? p.sink + p.recent : p.budget;
    auto end_page = [&](int i, int &place) -> int32_t {
        if (n <= p.budget) { place = i; return i < n ? __ldg(table + i) : -1; }
        const bool head = i < p.sink;
        place = head ? i : p.budget - p.recent + i - p.sink;
        return __ldg(table + (head ? i : n - p.recent + i - p.sink));
    };
    int place0 = 0;
    const int32_t end0 = (int)threadIdx.x < ends ? end_page(threadIdx.x, place0) : 0;
    if (kScoreD == 0 && chosen) {
        for (int i = threadIdx.x; i < kSelectRounds * kSelectBins; i += blockDim.x) (&s_hist[0][0])[i] = 0;
        if constexpr (kInRegisters)
            for (int i = threadIdx.x; i < cand; i += blockDim.x) s_words[i] = (uint32_t)__ldg(table + p.sink + i);
    }
    grid_dependency_wait();
    grid_launch_dependents();

    if (report && threadIdx.x == 0) {
        if (!usable) atomicOr(p.status, kStatusBadLength);
        if (pair % p.num_kv_heads == 0) p.sel_lens[r] = attended_length(L, p.max_pages_per_req, p.budget);
    }
    if ((int)threadIdx.x < ends) emit(place0, end0);
    for (int i = threadIdx.x + blockDim.x; i < ends; i += blockDim.x) {
        int place;
        const int32_t id = end_page(i, place);
        emit(place, id);
    }
    if (!chosen) return;

    if constexpr (kScoreD > 0) {
        constexpr int P = 2 * kScoreD / 64;
        const int g = lane >> 2, t = lane & 3, h = pair % p.num_kv_heads;
        uint32_t *s_keys = s_words + ((cand + 3) & ~3);
        QueryFragments<kScoreD> q;
        for (int base = warp * 16; base < cand; base += warps * 16) {
            const int c0 = base + g, c1 = c0 + 8;
            int page[2] = {c0 < cand ? __ldg(table + p.sink + c0) : 0, c1 < cand ? __ldg(table + p.sink + c1) : 0};
            if (t < 2 && base + g + 8 * t < cand) s_words[base + g + 8 * t] = (uint32_t)(t == 0 ? page[0] : page[1]);
            size_t at[2];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                if (page[x] < 0 || page[x] >= p.num_pages) { atomicOr(p.status, kStatusBadPage); page[x] = 0; }
                at[x] = (size_t)page[x] * p.num_kv_heads + h;
            }
            uint4 a[P], b[P];
#pragma unroll
            for (int i = 0; i < P; ++i) {
                a[i] = __ldg((const uint4 *)(p.records + at[0] * 2 * kScoreD) + i * 4 + t);
                b[i] = __ldg((const uint4 *)(p.records + at[1] * 2 * kScoreD) + i * 4 + t);
            }
            const float row_step = __ldg(p.steps + (t & 1 ? at[1] : at[0]));
            if (base == warp * 16) q.load(p.q + (size_t)pair * p.group * kScoreD, p.group, lane);
            const uint32_t key = tile_key<kScoreD>(a, b, q, row_step, t);
            if (t < 2 && base + g + 8 * t < cand) s_keys[base + g + 8 * t] = key;
        }
        for (int i = threadIdx.x; i < kSelectRounds * kSelectBins; i += blockDim.x) (&s_hist[0][0])[i] = 0;
        __syncthreads();
    }

    // thread x owns the keys first .. last - 1 (contiguous, so that context order is thread order)
    const uint32_t *keys = p.keys + (size_t)pair * p.key_stride;
    const int share = kInRegisters ? K : ((cand + blockDim.x - 1) / blockDim.x) | 1;     // odd: no bank conflicts
    const int first = min(cand, (int)threadIdx.x * share), last = min(cand, first + share);
    uint32_t own[K];
    uint32_t lo = 0xffffffffu, hi = 0u;
    if constexpr (kInRegisters) {
#pragma unroll
        for (int x = 0; x < K; x += 4) {
            uint4 v = make_uint4(0u, 0u, 0u, 0u);
            if (first + x < cand)                                            // the stride is a multiple of 4
                v = kScoreD > 0 ? *(const uint4 *)(s_words + ((cand + 3) & ~3) + first + x) : __ldg((const uint4 *)(keys + first + x));
            own[x] = v.x; own[x + 1] = v.y; own[x + 2] = v.z; own[x + 3] = v.w;
        }
#pragma unroll
        for (int x = 0; x < K; ++x) {
            if (first + x < last) { lo = min(lo, own[x]); hi = max(hi, own[x]); }
            else own[x] = 0u;                    // below every score's key
        }
    } else {
        for (int i = threadIdx.x; i < cand; i += blockDim.x) {
            const uint32_t k = __ldg(keys + i);
            s_words[i] = k;
            lo = min(lo, k);
            hi = max(hi, k);
        }
    }
    // calls f(key) on this thread's keys
    auto each = [&](auto f) {
        if constexpr (kInRegisters) {
#pragma unroll
            for (int x = 0; x < K; ++x) f(own[x]);
        } else {
            for (int i = first; i < last; ++i) f(s_words[i]);
        }
    };
    lo = __reduce_min_sync(0xffffffffu, lo);
    hi = __reduce_max_sync(0xffffffffu, hi);
    if (lane == 0) { s_range[0][warp] = lo; s_range[1][warp] = hi; }
    __syncthreads();
    lo = __reduce_min_sync(0xffffffffu, lane < warps ? s_range[0][lane] : 0xffffffffu);
    hi = __reduce_max_sync(0xffffffffu, lane < warps ? s_range[1][lane] : 0u);

    // The want-th largest key lies in [lo, hi]; `left` places remain for the keys of that range.  Every
    // warp reads the bins and comes to the same conclusion, so a round has one barrier.
    int left = want;
    for (int round = 0; round < kSelectRounds; ++round) {
        const int shift = max(0, 24 - __clz((int)(hi - lo)));              // (hi - lo) >> shift < 256
        int *hist = s_hist[round];
        each([&](uint32_t k) {
            if (k >= lo && k <= hi) atomicAdd(hist + ((k - lo) >> shift), 1);
        });
        __syncthreads();
        // lane x holds the bins 255 - 8 x down to 248 - 8 x
        const int4 b1 = *(const int4 *)(hist + 252 - 8 * lane), b0 = *(const int4 *)(hist + 248 - 8 * lane);
        const int bins[8] = {b1.w, b1.z, b1.y, b1.x, b0.w, b0.z, b0.y, b0.x};
        int sum = 0;
#pragma unroll
        for (int x = 0; x < 8; ++x) sum += bins[x];
        int upto = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += v;
        }
        const int src = __ffs(__ballot_sync(0xffffffffu, upto >= left)) - 1;      // the lane whose bins reach `left`
        int above = upto - sum, bin = 0, held = 0;
        bool found = false;
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            if (!found && above + bins[x] >= left) { found = true; bin = 255 - 8 * lane - x; held = bins[x]; }
            if (!found) above += bins[x];
        }
        bin = __shfl_sync(0xffffffffu, bin, src);
        held = __shfl_sync(0xffffffffu, held, src);
        left -= __shfl_sync(0xffffffffu, above, src);
        lo += (uint32_t)bin << shift;
        hi = min(hi, lo + ((1u << shift) - 1u));
        if (shift == 0 || held == left) break;
    }
    // keys above lo are in; of the keys equal to lo the first ones in context order fill what is left
    unsigned mine = 0;                           // above lo in the upper half, equal in the lower
    each([&](uint32_t k) { mine += k > lo ? 0x10000u : k == lo ? 1u : 0u; });
    unsigned upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned v = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += v;
    }
    if (lane == 31) s_range[2][warp] = upto;
    __syncthreads();
    const unsigned w = lane < warps ? s_range[2][lane] : 0u;
    const unsigned whole = __reduce_add_sync(0xffffffffu, w);
    const unsigned before = __reduce_add_sync(0xffffffffu, lane < warp ? w : 0u) + upto - mine;
    const int equal_places = want - (int)(whole >> 16);
    int above = (int)(before >> 16), equal = (int)(before & 0xffffu), i = first;
    each([&](uint32_t k) {
        if (k > lo || (k == lo && equal < equal_places))
            emit(p.sink + above + min(equal, equal_places), kInRegisters ? (int32_t)s_words[i] : __ldg(table + p.sink + i));
        above += k > lo;
        equal += k == lo;
        ++i;
    });
}

template <int kKeys>
__global__ void __launch_bounds__(kMaxSelectThreads)
select_pages_kernel(const SelectParams p)
{
    extern __shared__ __align__(16) uint32_t s_words[];
    __shared__ __align__(16) int s_hist[kSelectRounds][kSelectBins];
    __shared__ uint32_t s_range[3][32];
    int32_t *out = p.sel_tables + (size_t)blockIdx.x * p.budget;
    select_pair<kKeys, 0>(p, blockIdx.x, SelectScratch{s_words, s_hist, s_range}, true, [&](int place, int32_t id) { out[place] = id; });
}

}  // namespace ckv
