// Decode attention over the whole of a context or over a sliding window and its first tokens, from a
// cache in bf16 or in 8 bits.
#pragma once

#include <cuda_fp16.h>

#include "ckv_common.cuh"

namespace ckv {

// What is computed.  New token i of a request (position p = L - q_len + i) and query head h see token t if
// t <= p and (t > p - window or t < sink):   out = softmax_t(q k_t / sqrt(d)) v_t.
//
// Which pages are read.  Those of the sinks, then those from the earliest new token's window on: `head` pages
// from the front, then a gap of `skip` pages, `count` pages in all.  Within them every token is either
// visible or masked by its position; a tile of 32 tokens (2 pages) that all columns see entirely takes no mask.
//
// How the work is split.  Contexts (and windows longer than many contexts) differ a thousandfold, so the tiles
// of all (request, kv head) pairs lie on one axis, kCacheCost units ahead of each pair for what a piece costs
// besides its tiles, and every warp takes an even span of it, as it reads them: one kernel, no plan on the
// host.  A warp is independent: a ring of kStages tiles of its own, filled by TMA some tiles ahead, mma.sync on
// them, the softmax in the log2 domain with a running maximum.  A pair that lies within one span is finished
// there; of one that spans cut, each span leaves a partial (m, l, O) and cache_attn_fold_kernel joins them.
//
//   S^T[tok 16 x col 8] = K[tok 16 x d] . Q^T[d x col 8],   O^T[d 16 x col 8] += V^T[d 16 x tok 16] . P^T[tok 16 x col 8]
//
// 8-bit records.  value = n * step, n a whole number of magnitude <= 127, a step per (page, head, K | V): a
// block's 16 tokens are one m16 block of the matrix instruction, so a step is one factor for a block's scores, and one
// for its weights.  n is exact in fp16, as 1152 + n - 1152: its byte with the sign bit flipped, under the
// byte 0x64, is the fp16 number 1152 + n (two logic operations a pair of numbers, then a subtraction that is
// exact).  Queries are scaled by a power of two per column so that their largest has magnitude 2^7 to 2^8, and
// rounded to fp16: exact down to 2^-22 of the largest, below that to within 2^-33 of it.
// V's steps: the contribution of token t to O is 2^(s_t - m) step_t n_t, so with e_t = log2(step_t) the weights
// P_t = 2^(s_t + e_t - M), M the running maximum of s + e, are at most 2^8 whatever the steps are, and
// l = sum_t P_t 2^-e_t.  They are rounded to fp16 (2^-11) for P V and summed unrounded in fp32.
// In the bf16 cache weights are rounded to bf16 as everywhere in this library (the instruction takes one type).
//
// Masked values.  A masked score is selected away, and a masked row of the bf16 cache too: its weight is 0, but
// 0 * inf is not, so in a tile that some column does not see entirely the product is formed once a new token,
// with the rows cleared that this token does not see, and its columns taken.  Records are finite; a step that is not (a block that
// holds an infinity or a NaN) makes the scores of the block's visible tokens NaN.
struct CacheAttnParams {
    const int32_t *block_tables;
    const int32_t *seq_lens;
    const uint16_t *q;              // [batch][q_len][Hq][d]
    uint16_t *out;
    const float2 *steps;            // 8-bit cache: [layers][pages][Hkv] (K's, V's)
    float *part;                    // [2 * spans] partials: m[8], l[8], rows [8][D]
    int4 *cuts;                     // [spans] the pair that a span begins and does not end: request, kv head, last span; request -1: none
    uint32_t *status;
    int32_t batch, max_pages_per_req, num_pages, num_kv_heads, group;
    int32_t layer_page_base;        // layer * num_pages
    int32_t num_spans;
    int32_t q_len, q_base, q_pass;  // this launch computes new tokens q_base .. q_base + q_pass - 1; q_pass * group <= 8
    int32_t window, sink;           // window 0: all
    float scale_log2;               // log2(e) / sqrt(d)
};

// Units that a piece costs besides its tiles, and the fewest that a span holds: few short contexts are not cut
// into more partials than their tiles are worth.
constexpr int kCacheCost = 3, kCacheMinUnits = 4;

// The pages of a context that a launch reads.
struct Visited {
    int head, skip, count, tiles;   // tiles 0: the length is unusable
};

__device__ __forceinline__ Visited visited_pages(int L, const CacheAttnParams &p)
{
    Visited v = {0, 0, 0, 0};
    if (tiles_of_length(L, p.max_pages_per_req, p.q_len) == 0) return v;
    const int earliest = L - p.q_len + p.q_base, latest = earliest + p.q_pass - 1;
    const int first = p.window > 0 && earliest >= p.window ? (earliest - p.window + 1) / kPageSize : 0;
    v.head = min(p.sink / kPageSize + (p.sink % kPageSize != 0), first);
    v.skip = first - v.head;
    v.count = latest / kPageSize + 1 - v.skip;
    v.tiles = (v.count + kPagesPerTile - 1) / kPagesPerTile;
    return v;
}

__device__ __forceinline__ int units_of(const Visited &v) { return v.tiles > 0 ? v.tiles + kCacheCost : 0; }

// A place on the axis of units: a tile of a pair.
struct TilePlace {
    int r, h, tile;                 // r = -1: none
    Visited vis;
    int L;
    long long v;                    // the tile's unit
};

__device__ __forceinline__ int warp_sum(int x)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// The units of a span, and the first tile among them.  By one whole warp.
__device__ __forceinline__ long long span_units(const CacheAttnParams &p, int lane)
{
    int sum = 0;
    for (int r = lane; r < p.batch; r += 32) sum += units_of(visited_pages(__ldg(p.seq_lens + r), p));
    const long long total = (long long)warp_sum(sum) * p.num_kv_heads;
    return max((long long)kCacheMinUnits, (total + p.num_spans - 1) / p.num_spans);
}

__device__ __forceinline__ TilePlace span_begin(const CacheAttnParams &p, long long begin, long long end, int lane)
{
    TilePlace at;
    at.r = -1;
    long long running = 0;                       // units (all heads) before request `base`
    for (int base = 0; base < p.batch; base += 32) {
        const int r = base + lane;
        const int L = r < p.batch ? __ldg(p.seq_lens + r) : 0;
        int incl = r < p.batch ? units_of(visited_pages(L, p)) : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += x;
        }
        const long long upto = running + (long long)incl * p.num_kv_heads;
        const unsigned hit = __ballot_sync(0xffffffffu, upto > begin);
        if (hit) {
            const int src = __ffs(hit) - 1;
            at.L = __shfl_sync(0xffffffffu, L, src);
            at.vis = visited_pages(at.L, p);
            const int units = units_of(at.vis);
            const long long before = __shfl_sync(0xffffffffu, upto, src) - (long long)units * p.num_kv_heads;
            const int rem = (int)(begin - before);
            at.h = rem / units;
            at.tile = max(0, rem % units - kCacheCost);
            at.v = before + (long long)at.h * units + kCacheCost + at.tile;
            if (at.v < end) at.r = base + src;   // else the span holds a pair's overhead units only
            return at;
        }
        running = __shfl_sync(0xffffffffu, upto, 31);
    }
    return at;
}

template <int D, bool k8>
struct CacheAttnLayout {
    static constexpr int kWarps = k8 ? 12 : 6;
    static constexpr int kStages = D == 128 ? 2 : 4;
    static constexpr int kPageBytes = 32 * D * (k8 ? 1 : 2);
    static constexpr int kHalfBytes = 32 * 128;                  // bf16: a box of 64 columns
    static constexpr int kBoxes = k8 ? 1 : D / 64;               // TMA boxes of a page
    static constexpr int kTileBytes = kPagesPerTile * kPageBytes;
    static constexpr int kRingBytes = kStages * kTileBytes;
    static constexpr int kStepsOff = kWarps * kRingBytes;        // float2 a page of a stage
    static constexpr int kBarOff = kStepsOff + (k8 ? kWarps * kStages * kPagesPerTile * 8 : 0);
    static constexpr int kSmemBytes = kBarOff + kWarps * kStages * 8 + 1024;     // 1024: alignment of the swizzle's pattern
};

constexpr int kPartHead = 2 * kMaxGroup;         // m[8], l[8] in front of a partial's rows

// l is kept 2^-5 smaller than it is: with steps of 2^-106 to 2^121 it stays a normal number for 2^16 tokens and more.
constexpr int kCacheSumBias = 5;

__device__ __forceinline__ uint32_t sub_1152(uint32_t x)
{
    __half2 h = __hsub2(*reinterpret_cast<__half2 *>(&x), __half2half2(__ushort_as_half(0x6480)));
    return *reinterpret_cast<uint32_t *>(&h);
}

// Bytes 0, 2 and 1, 3 of x as pairs of fp16 numbers.
__device__ __forceinline__ void records_to_half(uint32_t x, uint32_t &even, uint32_t &odd)
{
    even = sub_1152((x & 0x00ff00ffu) ^ 0x64806480u);
    odd = sub_1152(((x >> 8) & 0x00ff00ffu) ^ 0x64806480u);
}

__device__ __forceinline__ void mma_f16_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi)
{
    uint32_t d;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}

template <int D, bool k8>
__global__ void __launch_bounds__(CacheAttnLayout<D, k8>::kWarps * 32, 1)
cache_attn_kernel(const __grid_constant__ CUtensorMap tmap, const CacheAttnParams p)
{
    using Lay = CacheAttnLayout<D, k8>;
    constexpr int W = Lay::kWarps, NS = Lay::kStages, kSteps16 = D / 16;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int span = blockIdx.x * W + warp;
    const int G = p.group, heads = p.num_kv_heads * G, ncols = p.q_pass * G;
    const uint32_t ring = smem_u32(smem) + warp * Lay::kRingBytes;
    const uint32_t step_ring = smem_u32(smem + Lay::kStepsOff) + warp * NS * kPagesPerTile * 8;
    const uint32_t bars = smem_u32(smem + Lay::kBarOff) + warp * NS * 8;
    if (lane == 0) {
        prefetch_tensormap(&tmap);
        // a stage is full when its boxes have landed and, 8-bit, the copies of its steps by lanes 0 and 1
        for (int s = 0; s < NS; ++s) mbar_init(bars + s * 8, k8 ? 1 + kPagesPerTile : 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_proxy_async();
    }
    __syncwarp();
    grid_dependency_wait();                       // every input may come from the preceding kernel
    grid_launch_dependents();

    if (span == 0) {                              // requests of unusable length: rows cleared, status
        const int row_elems = p.q_pass * heads * D;
        for (int base = 0; base < p.batch; base += 32) {
            const int r = base + lane;
            unsigned todo = __ballot_sync(0xffffffffu, r < p.batch && visited_pages(__ldg(p.seq_lens + r), p).tiles == 0);
            if (todo && lane == 0) atomicOr(p.status, kStatusBadLength);
            for (; todo; todo &= todo - 1) {
                uint4 *row = (uint4 *)(p.out + ((size_t)(base + __ffs(todo) - 1) * p.q_len + p.q_base) * heads * D);
                for (int i = lane; i < row_elems / 8; i += 32) row[i] = make_uint4(0u, 0u, 0u, 0u);
            }
        }
    }
    const long long q_units = span_units(p, lane), begin = span * q_units, end = begin + q_units;
    TilePlace ic = span_begin(p, begin, end, lane);
    int4 cut = make_int4(-1, -1, -1, -1);

    const uint64_t policy = l2_evict_first_policy();
    // ---- issue side: the next tile to fetch, and its pages: lane i holds page 32 * chunk + i of the pair's visited ones
    TilePlace cc = ic;                            // compute side
    constexpr int kTilesPerChunk = 32 / kPagesPerTile;
    auto load_chunk = [&](int r, const Visited &vis, int chunk) {
        const int v = chunk * 32 + lane;
        return v < vis.count ? __ldg(p.block_tables + (size_t)r * p.max_pages_per_req + (v < vis.head ? v : v + vis.skip)) : 0;
    };
    int chunk_now = 0, chunk_next = 0;
    if (ic.r >= 0) {
        chunk_now = load_chunk(ic.r, ic.vis, ic.tile / kTilesPerChunk);
        chunk_next = load_chunk(ic.r, ic.vis, ic.tile / kTilesPerChunk + 1);
    }
    int issued = 0;
    // Moves to the next tile of the axis; false at the span's end.
    auto advance = [&](TilePlace &at) {
        ++at.v;
        if (++at.tile < at.vis.tiles) return at.v < end;
        at.tile = 0;
        at.v += kCacheCost;
        if (at.v >= end) return false;
        if (++at.h < p.num_kv_heads) return true;
        at.h = 0;
        do {
            if (++at.r >= p.batch) return false;
            at.L = __ldg(p.seq_lens + at.r);
            at.vis = visited_pages(at.L, p);
        } while (at.vis.tiles == 0);
        return true;
    };
    bool more = ic.r >= 0;
    auto issue_next = [&]() {
        const int stage = issued % NS;
        const int np = min(kPagesPerTile, ic.vis.count - ic.tile * kPagesPerTile);
        const int pg = lane / Lay::kBoxes, box = lane % Lay::kBoxes;
        int page = __shfl_sync(0xffffffffu, chunk_now, (ic.tile % kTilesPerChunk * kPagesPerTile + pg) & 31);
        const uint32_t bar = bars + stage * 8;
        if (lane == 0) mbar_arrive_expect_tx(bar, np * Lay::kPageBytes);
        __syncwarp();
        if (pg < np) {
            if (page < 0 || page >= p.num_pages) {
                atomicOr(p.status, kStatusBadPage);
                page = 0;
            }
            const int block = (p.layer_page_base + page) * p.num_kv_heads + ic.h;
            tma_load_2d(ring + stage * Lay::kTileBytes + pg * Lay::kPageBytes + box * Lay::kHalfBytes, &tmap, box * 64, block * 32, bar, policy);
            if constexpr (k8)
                asm volatile("cp.async.ca.shared.global [%0], [%1], 8;"
                             ::"r"(step_ring + (stage * kPagesPerTile + pg) * 8), "l"(p.steps + block) : "memory");
        }
        if constexpr (k8) {
            if (lane < kPagesPerTile) asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
        }
        ++issued;
        const int r = ic.r, h = ic.h;
        more = advance(ic);
        if (!more) return;
        if (ic.r != r || ic.h != h) {
            chunk_now = load_chunk(ic.r, ic.vis, 0);
            chunk_next = load_chunk(ic.r, ic.vis, 1);
        } else if (ic.tile % kTilesPerChunk == 0) {
            chunk_now = chunk_next;
            chunk_next = load_chunk(ic.r, ic.vis, ic.tile / kTilesPerChunk + 1);
        }
    };
    while (issued < NS && more) issue_next();

    // ---- compute side
    const int g0 = (lane & 3) * 2;               // first of the two columns this lane accumulates
    const int i0 = min(g0 / G, p.q_pass - 1), i1 = min((g0 + 1) / G, p.q_pass - 1);              // their new tokens
    const int row16 = (lane & 7) + ((lane >> 3) & 1) * 8;        // ldmatrix: this lane's row of a page's keys
    auto piece_at = [&](int row, int c) {        // byte offset of the 16 bytes c of a row in a page's box
        if constexpr (!k8) return row * 128 + ((c ^ (row & 7)) << 4);
        else if constexpr (D == 128) return row * 128 + ((c ^ (row & 7)) << 4);
        else return row * 64 + ((c ^ ((row >> 1) & 3)) << 4);
    };
    bool alive = true;
    int done = 0;
    bool go = cc.r >= 0;
    while (go) {
        const int r = cc.r, h = cc.h, L = cc.L, tile0 = cc.tile;
        const Visited vis = cc.vis;
        const int n = (int)min((long long)(vis.tiles - tile0), end - cc.v);
        const long long v0 = cc.v;
        // ---- queries: column c = (new token c / G, head c % G), this lane holds four elements of every 16 of column lane / 4
        uint32_t qf[kSteps16][2];
        float qs0 = p.scale_log2, qs1 = p.scale_log2;
        {
            const int c = lane >> 2, j = lane & 3;
            const uint16_t *row = p.q + (((size_t)r * p.q_len + p.q_base + c / G) * heads + h * G + c % G) * D;
            if constexpr (k8) {
                uint2 raw[kSteps16];
                uint32_t most = 0;
#pragma unroll
                for (int ks = 0; ks < kSteps16; ++ks) {
                    raw[ks] = c < ncols ? __ldg((const uint2 *)(row + ks * 16 + j * 4)) : make_uint2(0u, 0u);
                    most = max(max(most, raw[ks].x & 0x7fffu), max(raw[ks].x >> 16 & 0x7fffu, max(raw[ks].y & 0x7fffu, raw[ks].y >> 16 & 0x7fffu)));
                }
                most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
                most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
                // the largest comes to lie in [2^7, 2^8); infinities stay, and what is left beside them does not matter
                const int e = min(max((int)(most >> 7), 8), 254);                // biased exponent
                const float up = __uint_as_float((uint32_t)(254 + 7 - e) << 23);
                float back = __uint_as_float((uint32_t)max(e - 7, 1) << 23) * p.scale_log2;
#pragma unroll
                for (int ks = 0; ks < kSteps16; ++ks) {
                    const float x0 = __uint_as_float(raw[ks].x << 16), x1 = __uint_as_float(raw[ks].x & 0xffff0000u);
                    const float x2 = __uint_as_float(raw[ks].y << 16), x3 = __uint_as_float(raw[ks].y & 0xffff0000u);
                    qf[ks][0] = pack_f16x2(x0 * up, x2 * up);
                    qf[ks][1] = pack_f16x2(x1 * up, x3 * up);
                }
                qs0 = __shfl_sync(0xffffffffu, back, g0 * 4);
                qs1 = __shfl_sync(0xffffffffu, back, g0 * 4 + 4);
            } else {
#pragma unroll
                for (int ks = 0; ks < kSteps16; ++ks) {
                    qf[ks][0] = c < ncols ? __ldg((const uint32_t *)row + ks * 8 + j) : 0u;
                    qf[ks][1] = c < ncols ? __ldg((const uint32_t *)row + ks * 8 + 4 + j) : 0u;
                }
            }
        }
        const int earliest = L - p.q_len + p.q_base;
        const int pos0 = earliest + i0, pos1 = earliest + i1, latest = earliest + p.q_pass - 1;
        // the first token of each window
        const int from0 = p.window > 0 ? pos0 - p.window + 1 : 0, from1 = p.window > 0 ? pos1 - p.window + 1 : 0;
        const int from_latest = p.window > 0 ? latest - p.window + 1 : 0;
        float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
        float o[kSteps16][4];
#pragma unroll
        for (int c = 0; c < kSteps16; ++c) o[c][0] = o[c][1] = o[c][2] = o[c][3] = 0.f;

#pragma unroll 1
        for (int ti = tile0; ti < tile0 + n; ++ti, ++done) {
            const int stage = done % NS;
            if (alive) alive = __all_sync(0xffffffffu, mbar_wait_bounded(bars + stage * 8, (done / NS) & 1, p.status));
            if (!alive) continue;
            const uint32_t sb = ring + stage * Lay::kTileBytes;
            const int np = min(kPagesPerTile, vis.count - ti * kPagesPerTile);
            int base[kPagesPerTile];             // first token of each page
            bool all_seen = np == kPagesPerTile;
#pragma unroll
            for (int mt = 0; mt < kPagesPerTile; ++mt) {
                const int v = ti * kPagesPerTile + mt;
                base[mt] = (v < vis.head ? v : v + vis.skip) * kPageSize;
                all_seen = all_seen && base[mt] + kPageSize - 1 <= earliest && (base[mt] >= from_latest || base[mt] + kPageSize <= p.sink);
            }
            // ---- S^T = K Q^T
            float s[kPagesPerTile][4];
#pragma unroll
            for (int mt = 0; mt < kPagesPerTile; ++mt) {
                s[mt][0] = s[mt][1] = s[mt][2] = s[mt][3] = 0.f;
                if (mt < np) {
                    const uint32_t kb = sb + mt * Lay::kPageBytes;
                    if constexpr (k8) {
#pragma unroll
                        for (int c = 0; c < kSteps16; c += 2) {
                            uint32_t x[4], lo0, hi0, lo1, hi1;
                            ldmatrix_x4(x, kb + piece_at(row16, c + (lane >> 4)));
                            records_to_half(x[0], lo0, hi0);
                            records_to_half(x[1], lo1, hi1);
                            mma_f16_16816(s[mt], lo0, lo1, hi0, hi1, qf[c][0], qf[c][1]);
                            records_to_half(x[2], lo0, hi0);
                            records_to_half(x[3], lo1, hi1);
                            mma_f16_16816(s[mt], lo0, lo1, hi0, hi1, qf[c + 1][0], qf[c + 1][1]);
                        }
                    } else {
#pragma unroll
                        for (int ks = 0; ks < kSteps16; ++ks) {
                            uint32_t a[4];
                            ldmatrix_x4(a, kb + (ks / 4) * Lay::kHalfBytes + piece_at(row16, ks % 4 * 2 + (lane >> 4)));
                            mma_bf16_16816(s[mt], a, qf[ks][0], qf[ks][1]);
                        }
                    }
                }
            }
            // ---- scores in the log2 domain, V's step among them
            float wl[kPagesPerTile];             // what a weight counts for in l
            float mx0 = -INFINITY, mx1 = -INFINITY;
#pragma unroll
            for (int mt = 0; mt < kPagesPerTile; ++mt) {
                float a0 = qs0, a1 = qs1, add = 0.f;
                wl[mt] = 1.f;
                if constexpr (k8) {
                    float ks, vs;
                    asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(ks), "=f"(vs) : "r"(step_ring + (stage * kPagesPerTile + mt) * 8));
                    const int e = (int)(__float_as_uint(vs) >> 23 & 255u);
                    a0 *= ks;
                    a1 *= ks;
                    add = (float)(e - 127) + (vs - vs);                          // NaN where the block is
                    wl[mt] = __uint_as_float((uint32_t)max(254 - kCacheSumBias - e, 0) << 23);
                }
                s[mt][0] = fmaf(s[mt][0], a0, add);
                s[mt][1] = fmaf(s[mt][1], a1, add);
                s[mt][2] = fmaf(s[mt][2], a0, add);
                s[mt][3] = fmaf(s[mt][3], a1, add);
                if (!all_seen) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int t = base[mt] + (lane >> 2) + (i >= 2 ? 8 : 0);
                        const int pos = i & 1 ? pos1 : pos0, from = i & 1 ? from1 : from0;
                        if (mt >= np || t > pos || (t < from && t >= p.sink)) s[mt][i] = -INFINITY;            // selected, never multiplied
                    }
                }
                mx0 = fmaxf(mx0, fmaxf(s[mt][0], s[mt][2]));
                mx1 = fmaxf(mx1, fmaxf(s[mt][1], s[mt][3]));
            }
            // The reference that a column's exponentials are taken against moves only when a score exceeds it by
            // more than 2^8; a column with nothing above -inf so far takes them against 0: they come out 0.
            if (__any_sync(0xffffffffu, mx0 > m0 + 8.f || mx1 > m1 + 8.f)) {
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) {
                    mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, x));
                    mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, x));
                }
                const float old0 = m0, old1 = m1;
                m0 = fmaxf(m0, mx0);
                m1 = fmaxf(m1, mx1);
                const float al0 = fast_exp2(old0 - (m0 == -INFINITY ? 0.f : m0)), al1 = fast_exp2(old1 - (m1 == -INFINITY ? 0.f : m1));
                l0 *= al0;
                l1 *= al1;
#pragma unroll
                for (int c = 0; c < kSteps16; ++c) { o[c][0] *= al0; o[c][2] *= al0; o[c][1] *= al1; o[c][3] *= al1; }
            }
            const float ref0 = m0 == -INFINITY ? 0.f : m0, ref1 = m1 == -INFINITY ? 0.f : m1;
            uint32_t pb[kPagesPerTile][2];
#pragma unroll
            for (int mt = 0; mt < kPagesPerTile; ++mt) {
                const float p0 = fast_exp2(s[mt][0] - ref0), p1 = fast_exp2(s[mt][1] - ref1);
                const float p2 = fast_exp2(s[mt][2] - ref0), p3 = fast_exp2(s[mt][3] - ref1);
                l0 = fmaf(p0 + p2, wl[mt], l0);
                l1 = fmaf(p1 + p3, wl[mt], l1);
                pb[mt][0] = movmatrix_trans(k8 ? pack_f16x2(p0, p1) : pack_bf16x2(p0, p1));      // tokens 0..7 of the page
                pb[mt][1] = movmatrix_trans(k8 ? pack_f16x2(p2, p3) : pack_bf16x2(p2, p3));      // tokens 8..15
            }
            // ---- O^T += V^T P^T
#pragma unroll
            for (int mt = 0; mt < kPagesPerTile; ++mt) {
                if (mt >= np) continue;
                const uint32_t vb = sb + mt * Lay::kPageBytes;
                if constexpr (k8) {
#pragma unroll
                    for (int c = 0; c < kSteps16; c += 2) {
                        uint32_t x[4], lo0, hi0, lo1, hi1;
                        ldmatrix_x4_trans(x, vb + piece_at(16 + row16, c + (lane >> 4)));
                        records_to_half(x[0], lo0, hi0);
                        records_to_half(x[1], lo1, hi1);
                        mma_f16_16816(o[c], lo0, hi0, lo1, hi1, pb[mt][0], pb[mt][1]);
                        records_to_half(x[2], lo0, hi0);
                        records_to_half(x[3], lo1, hi1);
                        mma_f16_16816(o[c + 1], lo0, hi0, lo1, hi1, pb[mt][0], pb[mt][1]);
                    }
                } else {
                    const int vrow = 16 + (lane & 7) + (lane >> 4) * 8, vsel = (lane >> 3) & 1;
                    if (all_seen) {
#pragma unroll
                        for (int c = 0; c < kSteps16; ++c) {
                            uint32_t a[4];
                            ldmatrix_x4_trans(a, vb + (c / 4) * Lay::kHalfBytes + piece_at(vrow, c % 4 * 2 + vsel));
                            mma_bf16_16816(o[c], a, pb[mt][0], pb[mt][1]);
                        }
                    } else {
#pragma unroll 1
                        for (int i = 0; i < p.q_pass; ++i) {                     // one new token's columns, the rows it sees
                            const int pos = earliest + i, from = p.window > 0 ? pos - p.window + 1 : 0;
                            uint32_t keep[2];
#pragma unroll
                            for (int half = 0; half < 2; ++half) {
                                const int t = base[mt] + half * 8 + (lane & 3) * 2;
                                const bool s0 = t <= pos && (t >= from || t < p.sink), s1 = t + 1 <= pos && (t + 1 >= from || t + 1 < p.sink);
                                keep[half] = (s0 ? 0xffffu : 0u) | (s1 ? 0xffff0000u : 0u);
                            }
#pragma unroll
                            for (int c = 0; c < kSteps16; ++c) {
                                uint32_t a[4];
                                ldmatrix_x4_trans(a, vb + (c / 4) * Lay::kHalfBytes + piece_at(vrow, c % 4 * 2 + vsel));
                                a[0] &= keep[0]; a[1] &= keep[0]; a[2] &= keep[1]; a[3] &= keep[1];
                                float x[4] = {0.f, 0.f, 0.f, 0.f};               // other tokens' columns may hold anything
                                mma_bf16_16816(x, a, pb[mt][0], pb[mt][1]);
                                if (i0 == i) { o[c][0] += x[0]; o[c][2] += x[2]; }
                                if (i1 == i) { o[c][1] += x[1]; o[c][3] += x[3]; }
                            }
                        }
                    }
                }
            }
            __syncwarp();                         // the stage has been read
            if (more) issue_next();               // refill it with the tile NS ahead
        }

        // ---- the piece's end
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) {
            l0 += __shfl_xor_sync(0xffffffffu, l0, x);
            l1 += __shfl_xor_sync(0xffffffffu, l1, x);
        }
        const bool whole = n == vis.tiles;
        // 8-bit: a lane holds elements d, d + 1 (d = 16 c + 2 (lane / 4)) of its two columns; bf16: elements d and d + 8
        // (d = 16 c + lane / 4), and neighbouring lanes trade, so that each has a pair of one column
        const bool odd = (lane >> 2) & 1;
        if (whole) {
            const float bias = k8 ? __uint_as_float((uint32_t)(127 - kCacheSumBias) << 23) : 1.f;
            const float inv0 = 1.f / l0, inv1 = 1.f / l1;
            uint16_t *rows = p.out + ((size_t)r * p.q_len + p.q_base) * heads * D + (size_t)h * G * D;
            auto row_of = [&](int c) { return rows + ((size_t)(c / G) * heads + c % G) * D; };
#pragma unroll
            for (int c = 0; c < kSteps16; ++c) {
                const float x0 = o[c][0] * bias * inv0, x1 = o[c][1] * bias * inv1, y0 = o[c][2] * bias * inv0, y1 = o[c][3] * bias * inv1;
                if constexpr (k8) {
                    const int d = c * 16 + (lane >> 2) * 2;
                    if (alive && g0 < ncols) *(uint32_t *)(row_of(g0) + d) = pack_bf16x2(x0, y0);
                    if (alive && g0 + 1 < ncols) *(uint32_t *)(row_of(g0 + 1) + d) = pack_bf16x2(x1, y1);
                } else {
                    const float tx = __shfl_xor_sync(0xffffffffu, odd ? x0 : x1, 4), ty = __shfl_xor_sync(0xffffffffu, odd ? y0 : y1, 4);
                    const int d = c * 16 + (lane >> 3) * 2, col = g0 + odd;
                    if (alive && col < ncols) {
                        *(uint32_t *)(row_of(col) + d) = odd ? pack_bf16x2(tx, x1) : pack_bf16x2(x0, tx);
                        *(uint32_t *)(row_of(col) + d + 8) = odd ? pack_bf16x2(ty, y1) : pack_bf16x2(y0, ty);
                    }
                }
            }
        } else {
            // a pair's first piece in slot 2 span + 1, any other in slot 2 span: a span has at most one of each
            const int slot = 2 * span + (tile0 == 0 ? 1 : 0);
            float *part = p.part + (size_t)slot * (kPartHead + kMaxGroup * D), *rows = part + kPartHead;
            if (tile0 == 0) cut = make_int4(r, h, (int)((v0 + vis.tiles - 1) / q_units), 0);
            if (lane < 4) {
                // a warp that gave up leaves NaN, not what it had
                *(float2 *)(part + g0) = make_float2(m0, m1);
                *(float2 *)(part + kMaxGroup + g0) = alive ? make_float2(l0, l1) : make_float2(NAN, NAN);
            }
#pragma unroll
            for (int c = 0; c < kSteps16; ++c) {
                if constexpr (k8) {
                    const int d = c * 16 + (lane >> 2) * 2;
                    *(float2 *)(rows + g0 * D + d) = make_float2(o[c][0], o[c][2]);
                    *(float2 *)(rows + (g0 + 1) * D + d) = make_float2(o[c][1], o[c][3]);
                } else {
                    const float tx = __shfl_xor_sync(0xffffffffu, odd ? o[c][0] : o[c][1], 4), ty = __shfl_xor_sync(0xffffffffu, odd ? o[c][2] : o[c][3], 4);
                    const int d = c * 16 + (lane >> 3) * 2, col = g0 + odd;
                    *(float2 *)(rows + col * D + d) = odd ? make_float2(tx, o[c][1]) : make_float2(o[c][0], tx);
                    *(float2 *)(rows + col * D + d + 8) = odd ? make_float2(ty, o[c][3]) : make_float2(o[c][2], ty);
                }
            }
        }
        // on to the next piece
        cc.tile = tile0 + n - 1;
        cc.v = v0 + n - 1;
        go = advance(cc);
    }
    // do not leave while copies may be in flight (only after a wait gave up)
    if (!alive)
        for (int i = max(0, issued - NS); i < issued; ++i) mbar_wait_bounded(bars + (i % NS) * 8, (i / NS) & 1, p.status);
    if (lane == 0) p.cuts[span] = cut;
}

// ------------------------------------------------------------------------------------------
// The partials of the pairs that spans cut:  M = max m_i,  out = sum 2^(m_i - M) O_i / sum 2^(m_i - M) l_i, in the
// spans' order, so results are bit-identical from run to run.  A block looks after the cuts of some spans and
// two of the eight columns; a warp folds a column of few partials, the whole block one of many.
// ------------------------------------------------------------------------------------------
constexpr int kFoldWarps = 8, kFoldFew = 16, kFoldBlocks = 148;

template <int D>
struct FoldSum {
    float m, l;
    float4 acc;                     // elements 4 lane .. 4 lane + 3
};

// Partials first, first + step, ... below n of a pair whose first piece's span is s.
template <int D>
__device__ __forceinline__ FoldSum<D> fold_partials(const float *part, int s, int first, int step, int n, int col, int lane)
{
    constexpr size_t kSlot = kPartHead + kMaxGroup * D;
    FoldSum<D> f = {-INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
    auto slot = [&](int i) { return part + (size_t)(i == 0 ? 2 * s + 1 : 2 * (s + i)) * kSlot; };
    for (int i = first + lane * step; i < n; i += 32 * step) f.m = fmaxf(f.m, slot(i)[col]);
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) f.m = fmaxf(f.m, __shfl_xor_sync(0xffffffffu, f.m, x));
    const float ref = f.m == -INFINITY ? 0.f : f.m;
#pragma unroll 4
    for (int i = first; i < n; i += step) {
        const float *at = slot(i);
        const float w = fast_exp2(at[col] - ref);
        f.l += w * at[kMaxGroup + col];
        if (lane * 4 < D) {
            const float4 a = *(const float4 *)(at + kPartHead + col * D + lane * 4);
            f.acc.x += w * a.x; f.acc.y += w * a.y; f.acc.z += w * a.z; f.acc.w += w * a.w;
        }
    }
    return f;
}

template <int D>
__global__ void __launch_bounds__(kFoldWarps * 32)
cache_attn_fold_kernel(const CacheAttnParams p, const float bias)
{
    __shared__ float s_ml[kFoldWarps][2];
    __shared__ float4 s_acc[kFoldWarps][32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int G = p.group, heads = p.num_kv_heads * G, ncols = p.q_pass * G;
    grid_dependency_wait();
    grid_launch_dependents();
    const int part_of = blockIdx.x / kFoldBlocks;                // columns part_of and part_of + 4
    auto store = [&](const int4 &cut, int col, const FoldSum<D> &f) {
        const float inv = 1.f / f.l;
        uint16_t *row = p.out + ((size_t)cut.x * p.q_len + p.q_base + col / G) * heads * D + (size_t)(cut.y * G + col % G) * D;
        if (lane * 4 < D)
            *(uint2 *)(row + lane * 4) = make_uint2(pack_bf16x2(f.acc.x * bias * inv, f.acc.y * bias * inv), pack_bf16x2(f.acc.z * bias * inv, f.acc.w * bias * inv));
    };
    int turn = 0;
    for (int s = blockIdx.x % kFoldBlocks; s < p.num_spans; s += kFoldBlocks) {
        const int4 cut = p.cuts[s];
        if (cut.x < 0) continue;
        const int n = cut.z - s + 1;
        for (int col = part_of; col < ncols; col += 4) {
            if (n <= kFoldFew) {
                if (turn++ % kFoldWarps == warp) store(cut, col, fold_partials<D>(p.part, s, 0, 1, n, col, lane));
            } else {
                const FoldSum<D> f = fold_partials<D>(p.part, s, warp, kFoldWarps, n, col, lane);
                __syncthreads();                  // the last one has been read
                if (lane == 0) { s_ml[warp][0] = f.m; s_ml[warp][1] = f.l; }
                s_acc[warp][lane] = f.acc;
                __syncthreads();
                if (warp == 0) {
                    FoldSum<D> t = {-INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
                    for (int w = 0; w < kFoldWarps; ++w) t.m = fmaxf(t.m, s_ml[w][0]);
                    const float ref = t.m == -INFINITY ? 0.f : t.m;
                    for (int w = 0; w < kFoldWarps; ++w) {
                        const float x = fast_exp2(s_ml[w][0] - ref);
                        const float4 a = s_acc[w][lane];
                        t.l += x * s_ml[w][1];
                        t.acc.x += x * a.x; t.acc.y += x * a.y; t.acc.z += x * a.z; t.acc.w += x * a.w;
                    }
                    store(cut, col, t);
                }
            }
        }
    }
}

}  // namespace ckv
