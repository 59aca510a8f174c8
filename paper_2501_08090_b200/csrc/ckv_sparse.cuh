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
// it.  A page that holds a key with an infinity or a NaN gets lo = -127, hi = 127 and the largest
// step: it is nearly always selected, and attention then shows what a full pass would have shown.
// Records come first, all layers, then all steps.
// ------------------------------------------------------------------------------------------
constexpr int kIndexMinExp = -100;
constexpr float kIndexStepOfInvalid = 2.658455991569832e36f;      // 2^121

// Step exponent for a largest magnitude m; 2^-exponent comes back in `inv`.
__device__ __forceinline__ int step_exponent(float m, float &inv)
{
    const int e = (int)(__float_as_uint(fmaxf(m, 7.888609052210118e-31f)) >> 23) - 127 - 6;    // 2^-100
    inv = __uint_as_float((uint32_t)(127 - e) << 23);
    return e;
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

// A warp takes one (page, kv head) at a time: 16 key rows, contiguous in the pool, one 16-byte piece
// of 32 / (D/8) rows per load.  The units of all requests lie on one axis that is cut evenly over
// the warps of the grid, so long and short requests balance; neighbouring units are neighbours in
// memory (kv heads of a page first).  Bound by HBM: it reads the key half of the pool once, and the
// next unit's rows are on their way while one is reduced.
template <int D>
__global__ void __launch_bounds__(256)
kv_index_update_kernel(const IndexParams p)
{
    constexpr int kVecs = D / 8;                 // 16-byte pieces of a row
    constexpr int kRows = 32 / kVecs;            // rows of one load
    constexpr int NV = kPageSize / kRows;
    const int lane = threadIdx.x & 31;
    const int warp = (blockIdx.x * blockDim.x + threadIdx.x) >> 5, warps = (gridDim.x * blockDim.x) >> 5;
    const int vec = lane % kVecs, row0 = lane / kVecs;
    grid_dependency_wait();
    grid_launch_dependents();

    long long pages = 0;
    for (int base = 0; base < p.batch; base += 32) {
        const int r = base + lane;
        int first;
        const int n = r < p.batch ? index_pages(p, __ldg(p.seq_lens + r), first) : 1;
        if (warp == 0 && n == 0) atomicOr(p.status, kStatusBadLength);
        if (r < p.batch) pages += n;
    }
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) pages += __shfl_xor_sync(0xffffffffu, pages, x);
    const long long total = pages * p.num_kv_heads;
    const long long per = (total + warps - 1) / warps;
    const long long begin = warp * per, end = min(begin + per, total);
    if (begin >= end) return;

    // the request that holds unit `begin`
    int r = 0, page_at = 0, page_end = 0, L = 0;
    long long running = 0;
    for (int base = 0; base < p.batch; base += 32) {
        const int rr = base + lane;
        int first = 0;
        const int len = rr < p.batch ? __ldg(p.seq_lens + rr) : 0;
        const int n = rr < p.batch ? index_pages(p, len, first) : 0;
        long long upto = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long v = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += v;
        }
        upto = running + upto * p.num_kv_heads;
        const unsigned hit = __ballot_sync(0xffffffffu, upto > begin);
        if (hit) {
            const int src = __ffs(hit) - 1;
            r = base + src;
            L = __shfl_sync(0xffffffffu, len, src);
            const int n_r = __shfl_sync(0xffffffffu, n, src);
            const long long before = __shfl_sync(0xffffffffu, upto, src) - (long long)n_r * p.num_kv_heads;
            page_at = __shfl_sync(0xffffffffu, first, src) + (int)((begin - before) / p.num_kv_heads);
            page_end = (L + kPageSize - 1) / kPageSize;
            running = before;
            break;
        }
        running = __shfl_sync(0xffffffffu, upto, 31);
    }
    int h = (int)((begin - running) % p.num_kv_heads);

    uint4 rows[NV], next_rows[NV];
    int page, next_page = -1;
    auto fetch = [&](uint4 (&dst)[NV], int &pg) {
        pg = __ldg(p.block_tables + (size_t)r * p.max_pages_per_req + page_at);
        if (pg < 0 || pg >= p.num_pages) {
            if (lane == 0) atomicOr(p.status, kStatusBadPage);
            pg = -1;
            return;
        }
        const int tokens = min(kPageSize, L - page_at * kPageSize);
        const uint4 *src = (const uint4 *)(p.pool_layer + ((size_t)pg * p.num_kv_heads + h) * 2 * kPageSize * D);
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (k * kRows + row0 < tokens) dst[k] = __ldg(src + (k * kRows + row0) * kVecs + vec);
    };
    fetch(rows, page);
    int tokens = min(kPageSize, L - page_at * kPageSize), head = h;
    for (long long unit = begin; unit < end; ++unit) {
        // step to the next unit and start its loads
        int next_tokens = 0, next_head = 0;
        if (unit + 1 < end) {
            if (++h == p.num_kv_heads) {
                h = 0;
                if (++page_at == page_end) {
                    int n, first;
                    do { L = __ldg(p.seq_lens + ++r); n = index_pages(p, L, first); } while (n == 0);
                    page_at = first;
                    page_end = first + n;
                }
            }
            fetch(next_rows, next_page);
            next_tokens = min(kPageSize, L - page_at * kPageSize);
            next_head = h;
        }
        if (page >= 0) {
            const __nv_bfloat162 top = __nv_bfloat162(__ushort_as_bfloat16(0x7f80), __ushort_as_bfloat16(0x7f80));
            const __nv_bfloat162 bottom = __nv_bfloat162(__ushort_as_bfloat16(0xff80), __ushort_as_bfloat16(0xff80));
            __nv_bfloat162 lo[4] = {top, top, top, top}, hi[4] = {bottom, bottom, bottom, bottom};
            bool invalid = false;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                if (k * kRows + row0 < tokens) {
                    const uint32_t w[4] = {rows[k].x, rows[k].y, rows[k].z, rows[k].w};
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const __nv_bfloat162 v = *reinterpret_cast<const __nv_bfloat162 *>(&w[x]);
                        invalid |= (w[x] & 0x7f80u) == 0x7f80u || (w[x] & 0x7f800000u) == 0x7f800000u;
                        lo[x] = __hmin2(lo[x], v);
                        hi[x] = __hmax2(hi[x], v);
                    }
                }
            }
#pragma unroll
            for (int o = kVecs; o < 32; o <<= 1) {
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    lo[x] = __hmin2(lo[x], __shfl_xor_sync(0xffffffffu, lo[x], o));
                    hi[x] = __hmax2(hi[x], __shfl_xor_sync(0xffffffffu, hi[x], o));
                }
            }
            invalid = __any_sync(0xffffffffu, invalid);
            float m = 0.f;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const float2 a = __bfloat1622float2(lo[x]), b = __bfloat1622float2(hi[x]);
                m = fmaxf(m, fmaxf(fmaxf(fabsf(a.x), fabsf(a.y)), fmaxf(fabsf(b.x), fabsf(b.y))));
            }
#pragma unroll
            for (int o = 1; o < kVecs; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
            float inv;
            int e = step_exponent(m, inv);
            if (ceilf(m * inv) > 127.f) { ++e; inv *= 0.5f; }
            uint32_t lo8[2] = {0u, 0u}, hi8[2] = {0u, 0u};
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const float2 a = __bfloat1622float2(lo[x]), b = __bfloat1622float2(hi[x]);
                const int a0 = invalid ? -127 : (int)floorf(a.x * inv), a1 = invalid ? -127 : (int)floorf(a.y * inv);
                const int b0 = invalid ? 127 : (int)ceilf(b.x * inv), b1 = invalid ? 127 : (int)ceilf(b.y * inv);
                lo8[x / 2] |= ((uint32_t)(a0 & 0xff) | (uint32_t)(a1 & 0xff) << 8) << (16 * (x & 1));
                hi8[x / 2] |= ((uint32_t)(b0 & 0xff) | (uint32_t)(b1 & 0xff) << 8) << (16 * (x & 1));
            }
            const size_t at = (size_t)page * p.num_kv_heads + head;
            if (lane < kVecs) {
                *(uint2 *)(p.records + at * 2 * D + 8 * lane) = make_uint2(lo8[0], lo8[1]);
                *(uint2 *)(p.records + at * 2 * D + D + 8 * lane) = make_uint2(hi8[0], hi8[1]);
            }
            if (lane == 0) p.steps[at] = invalid ? kIndexStepOfInvalid : __uint_as_float((uint32_t)(e + 127) << 23);
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) rows[k] = next_rows[k];
        page = next_page;
        tokens = next_tokens;
        head = next_head;
    }
}

// The bounds as numbers: bf16 [pages][kv heads][2][d] (exact: 7 bits times a power of two).
struct IndexValuesParams {
    const uint4 *records;           // this layer's
    const float *steps;
    uint4 *out;
    long long vecs;                 // 16-byte pieces of the layer's records
    int32_t vecs_per_record;
};

__global__ void kv_index_values_kernel(const IndexValuesParams p)
{
    grid_dependency_wait();
    grid_launch_dependents();
    for (long long i = blockIdx.x * (long long)blockDim.x + threadIdx.x; i < p.vecs; i += (long long)gridDim.x * blockDim.x) {
        const uint4 v = p.records[i];
        const float step = p.steps[i / p.vecs_per_record];
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        uint32_t o[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            const uint32_t two = w[x / 2] >> (16 * (x & 1));
            o[x] = pack_bf16x2((float)(int8_t)(two & 0xff) * step, (float)(int8_t)((two >> 8) & 0xff) * step);
        }
        p.out[2 * i] = make_uint4(o[0], o[1], o[2], o[3]);
        p.out[2 * i + 1] = make_uint4(o[4], o[5], o[6], o[7]);
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
// A cluster works on one (request, kv head): its CTAs score a share of the candidate pages each
// and store the scores, as ordered 32-bit keys, into the first CTA's shared memory; that CTA then
// finds the threshold by counting (2048 bins over the range of the keys that are still in question,
// then within the bin that holds the threshold) and writes the chosen pages in context order.
// The first `sink` and the last `recent` pages are always taken; equal scores go to the earlier page.
// ------------------------------------------------------------------------------------------
struct SelectParams {
    const uint8_t *records;
    const float *steps;
    const int32_t *block_tables;
    const int32_t *seq_lens;
    const uint16_t *q;              // [batch][Hq][d]
    int32_t *sel_tables;            // [batch][Hkv][budget]
    int32_t *sel_lens;              // [batch]
    uint32_t *status;
    int32_t batch, max_pages_per_req, num_pages, num_kv_heads, group;
    int32_t budget, sink, recent;
};

constexpr int kSelectThreads = 256;
constexpr int kSelectBins = 2048;

__device__ __forceinline__ void mma_s8_16832(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Inclusive sum over the threads of the CTA (kSelectThreads of them); `total` gets the whole sum.
__device__ __forceinline__ int cta_inclusive_sum(int v, int *s_warp, int &total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += up;
    }
    __syncthreads();                             // s_warp may still be read from the call before
    if (lane == 31) s_warp[warp] = v;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kSelectThreads / 32; ++w) {
        const int x = s_warp[w];
        if (w < warp) before += x;
        total += x;
    }
    return v + before;
}

template <int D>
__global__ void __launch_bounds__(kSelectThreads)
select_pages_kernel(const SelectParams p)
{
    constexpr int P = 2 * D / 64;                // 16-byte pieces of a record that one lane reads
    extern __shared__ uint32_t s_keys[];         // [max candidates] in the first CTA of the cluster
    __shared__ int s_hist[kSelectBins];
    __shared__ int s_warp[kSelectThreads / 32];
    __shared__ uint32_t s_range[2];
    __shared__ int s_found[3];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int rank = (int)cluster_rank(), ctas = (int)cluster_size();
    const int pair = blockIdx.x / ctas;          // (request, kv head)
    const int r = pair / p.num_kv_heads, h = pair % p.num_kv_heads;
    grid_dependency_wait();
    grid_launch_dependents();

    const int L = __ldg(p.seq_lens + r);
    const bool usable = tiles_of_length(L, p.max_pages_per_req) != 0;
    const int n = usable ? (L + kPageSize - 1) / kPageSize : 0;
    const int32_t *table = p.block_tables + (size_t)r * p.max_pages_per_req;
    int32_t *out = p.sel_tables + (size_t)pair * p.budget;
    if (rank == 0 && threadIdx.x == 0) {
        if (!usable) atomicOr(p.status, kStatusBadLength);
        if (h == 0) p.sel_lens[r] = n > p.budget ? L - (n - p.budget) * kPageSize : (usable ? L : 0);
    }
    if (n <= p.budget) {                         // the whole context fits (the same for every CTA of the cluster)
        if (rank == 0)
            for (int i = threadIdx.x; i < p.budget; i += kSelectThreads) out[i] = i < n ? __ldg(table + i) : -1;
        return;
    }
    const int cand = n - p.sink - p.recent;      // pages sink .. sink + cand - 1 compete for `want` places
    const int want = p.budget - p.sink - p.recent;
    if (rank == 0) {
        for (int i = threadIdx.x; i < p.sink; i += kSelectThreads) out[i] = __ldg(table + i);
        for (int i = threadIdx.x; i < p.recent; i += kSelectThreads) out[p.budget - p.recent + i] = __ldg(table + n - p.recent + i);
    }
    if (want == 0) return;
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");      // this CTA runs: others may reach its memory

    // ---- the group's queries as B fragments: column = lane / 4, this lane's bytes of each piece
    const int g = lane >> 2, t = lane & 3;
    uint32_t qneg[P / 2][4], qpos[P / 2][4];
    float qstep = 0.f;
    {
        uint4 raw[P / 2][2];
        float m = 0.f;
#pragma unroll
        for (int i = 0; i < P / 2; ++i) {
            raw[i][0] = raw[i][1] = make_uint4(0u, 0u, 0u, 0u);
            if (g < p.group) {
                const uint4 *src = (const uint4 *)(p.q + ((size_t)r * p.num_kv_heads * p.group + h * p.group + g) * D + i * 64 + t * 16);
                raw[i][0] = __ldg(src);
                raw[i][1] = __ldg(src + 1);
            }
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                const uint32_t w = ((const uint32_t *)raw[i])[x];
                const float a = fabsf(__uint_as_float(w << 16)), b = fabsf(__uint_as_float(w & 0xffff0000u));
                if (a < INFINITY) m = fmaxf(m, a);               // infinities and NaN take no part in the selection
                if (b < INFINITY) m = fmaxf(m, b);
            }
        }
        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
        float inv;
        const int e = step_exponent(m, inv);
        // only the order of a pair's scores matters: steps relative to the group's largest, so that no
        // product overflows
        int e_max = e;
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) e_max = max(e_max, __shfl_xor_sync(0xffffffffu, e_max, x));
        qstep = ldexpf(1.f, e - e_max);
        auto whole = [&](float x) { return fabsf(x) < INFINITY ? (int)fminf(fmaxf(rintf(x * inv), -127.f), 127.f) : 0; };
#pragma unroll
        for (int i = 0; i < P / 2; ++i) {
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                uint32_t neg = 0u, pos = 0u;
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const uint32_t w = ((const uint32_t *)raw[i])[2 * x + y];
                    const int a = whole(__uint_as_float(w << 16)), b = whole(__uint_as_float(w & 0xffff0000u));
                    neg |= ((uint32_t)(min(a, 0) & 0xff) | (uint32_t)(min(b, 0) & 0xff) << 8) << (16 * y);
                    pos |= ((uint32_t)max(a, 0) | (uint32_t)max(b, 0) << 8) << (16 * y);
                }
                qneg[i][x] = neg;
                qpos[i][x] = pos;
            }
        }
    }
    // steps of the two columns whose sums this lane receives
    const float step0 = __shfl_sync(0xffffffffu, qstep, (2 * t) * 4), step1 = __shfl_sync(0xffffffffu, qstep, (2 * t + 1) * 4);
    const bool live0 = 2 * t < p.group, live1 = 2 * t + 1 < p.group;

    // ---- scores of this CTA's share, 16 pages per warp and turn
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    const uint32_t keys0 = cluster_map(smem_u32(s_keys), 0);
    const int tiles = (cand + 15) / 16;
    const int per = (tiles + ctas - 1) / ctas;
    const int tile_end = min(tiles, (rank + 1) * per);
    for (int tile = rank * per + warp; tile < tile_end; tile += kSelectThreads / 32) {
        const int c0 = tile * 16 + g, c1 = c0 + 8;
        int page0 = c0 < cand ? __ldg(table + p.sink + c0) : 0, page1 = c1 < cand ? __ldg(table + p.sink + c1) : 0;
        if (page0 < 0 || page0 >= p.num_pages) { atomicOr(p.status, kStatusBadPage); page0 = 0; }
        if (page1 < 0 || page1 >= p.num_pages) { atomicOr(p.status, kStatusBadPage); page1 = 0; }
        const size_t at0 = (size_t)page0 * p.num_kv_heads + h, at1 = (size_t)page1 * p.num_kv_heads + h;
        uint4 a[P], b[P];
#pragma unroll
        for (int i = 0; i < P; ++i) {
            a[i] = __ldg((const uint4 *)(p.records + at0 * 2 * D) + i * 4 + t);
            b[i] = __ldg((const uint4 *)(p.records + at1 * 2 * D) + i * 4 + t);
        }
        const float s0 = __ldg(p.steps + at0), s1 = __ldg(p.steps + at1);
        int acc[4] = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const uint32_t *q8 = i < P / 2 ? qneg[i] : qpos[i - P / 2];
            mma_s8_16832(acc, a[i].x, b[i].x, a[i].y, b[i].y, q8[0], q8[1]);
            mma_s8_16832(acc, a[i].z, b[i].z, a[i].w, b[i].w, q8[2], q8[3]);
        }
        float x0 = fmaxf(live0 ? (float)acc[0] * step0 : -INFINITY, live1 ? (float)acc[1] * step1 : -INFINITY);
        float x1 = fmaxf(live0 ? (float)acc[2] * step0 : -INFINITY, live1 ? (float)acc[3] * step1 : -INFINITY);
        x0 = fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, 1));
        x1 = fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, 1));
        x0 = fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, 2));
        x1 = fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, 2));
        const int c = t == 0 ? c0 : c1;
        if (t < 2 && c < cand) {
            // 2^-22: sums stay below 2^21, steps below 2^123; + 0 makes a negative zero positive
            const float s = (t == 0 ? x0 * (s0 * 0x1p-22f) : x1 * (s1 * 0x1p-22f)) + 0.f;
            const uint32_t bits = __float_as_uint(s);
            const uint32_t key = bits ^ ((uint32_t)((int32_t)bits >> 31) | 0x80000000u);
            asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(keys0 + 4 * c), "r"(key) : "memory");
        }
    }
    cluster_barrier();
    if (rank != 0) return;

    // ---- the threshold: the want-th largest key.  [lo, hi] always holds it; `left` of the places are
    // still to be filled from the keys in that range (all keys above hi are in).
    const int share = ((cand + kSelectThreads - 1) / kSelectThreads) | 1;        // odd: no bank conflicts
    const int first = min(cand, (int)threadIdx.x * share), last = min(cand, first + share);
    if (threadIdx.x == 0) { s_range[0] = 0xffffffffu; s_range[1] = 0u; }
    __syncthreads();
    uint32_t lo = 0xffffffffu, hi = 0u;
    for (int i = first; i < last; ++i) { lo = min(lo, s_keys[i]); hi = max(hi, s_keys[i]); }
    lo = __reduce_min_sync(0xffffffffu, lo);
    hi = __reduce_max_sync(0xffffffffu, hi);
    if (lane == 0) { atomicMin(&s_range[0], lo); atomicMax(&s_range[1], hi); }
    __syncthreads();
    lo = s_range[0];
    hi = s_range[1];
    int left = want;
    for (;;) {
        const int shift = max(0, 21 - __clz((int)(hi - lo)));              // (hi - lo) >> shift < 2048
        for (int i = threadIdx.x; i < kSelectBins; i += kSelectThreads) s_hist[i] = 0;
        __syncthreads();
        for (int i = first; i < last; ++i) {
            const uint32_t k = s_keys[i];
            if (k >= lo && k <= hi) atomicAdd(&s_hist[(k - lo) >> shift], 1);
        }
        __syncthreads();
        // thread x holds bins from the top: 2047 - 8 x down to 2040 - 8 x
        constexpr int kOwn = kSelectBins / kSelectThreads;
        int own = 0;
#pragma unroll
        for (int x = 0; x < kOwn; ++x) own += s_hist[kSelectBins - 1 - (int)threadIdx.x * kOwn - x];
        int total;
        const int upto = cta_inclusive_sum(own, s_warp, total);
        if (upto >= left && upto - own < left) {                            // exactly one thread
            int above = upto - own;
            int bin = kSelectBins - 1 - (int)threadIdx.x * kOwn;
            while (above + s_hist[bin] < left) above += s_hist[bin--];
            s_found[0] = bin;
            s_found[1] = left - above;
            s_found[2] = s_hist[bin];
        }
        __syncthreads();
        lo += (uint32_t)s_found[0] << shift;
        hi = min(hi, lo + ((1u << shift) - 1u));
        left = s_found[1];
        const int held = s_found[2];
        __syncthreads();
        if (shift == 0 || held == left) break;
    }
    // keys above lo are in; of the keys equal to lo the first `left` in context order (all of them
    // if the whole bin was taken)
    int above = 0, equal = 0;
    for (int i = first; i < last; ++i) {
        above += s_keys[i] > lo;
        equal += s_keys[i] == lo;
    }
    int n_above, n_equal;
    int above_before = cta_inclusive_sum(above, s_warp, n_above) - above;
    int equal_before = cta_inclusive_sum(equal, s_warp, n_equal) - equal;
    const int equal_places = want - n_above;
    for (int i = first; i < last; ++i) {
        const uint32_t k = s_keys[i];
        const bool eq = k == lo;
        if (k > lo || (eq && equal_before < equal_places))
            out[p.sink + above_before + min(equal_before, equal_places)] = __ldg(table + p.sink + i);
        above_before += k > lo;
        equal_before += eq;
    }
}

}  // namespace ckv
