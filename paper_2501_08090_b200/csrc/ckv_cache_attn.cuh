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
// How the work is split.  A warp is independent: a ring of tiles of its own, filled by TMA some tiles ahead,
// mma.sync on them, the softmax in the log2 domain with a running maximum; what it has of a pair at the end is a
// partial (m, l, O):   M = max m_i,  out = sum 2^(m_i - M) O_i / sum 2^(m_i - M) l_i.
//   cache_attn_pair_kernel   (windows, short tables: pairs of one length, nearly)  a cluster of CTAs owns a (request, kv
//       head), its warps take the tiles in turn; partials are folded in shared memory, the CTAs' pushed to
//       the one that looks after a column.
//   cache_attn_span_kernel   (contexts that differ a thousandfold)  the tiles of all pairs lie on one axis, kCacheCost
//       units ahead of each pair for what a piece costs besides its tiles, and every warp takes an even span of
//       it: no plan on the host.  A pair within one span is finished there, one within a CTA by the CTA at its end;
//       of a pair that CTAs cut, each CTA leaves one partial, and cache_attn_fold_kernel joins them.
//
//   S^T[tok 16 x col 8] = K[tok 16 x d] . Q^T[d x col 8],   O^T[d 16 x col 8] += V^T[d 16 x tok 16] . P^T[tok 16 x col 8]
//
// 8-bit records.  value = n * step, n a whole number of magnitude <= 127, a step per (page, head, K | V): a
// block's 16 tokens are one m16 block of the matrix instruction, so a step is one factor for a block's scores, and one
// for its weights.
// K is multiplied as it lies, by the 8-bit matrix instruction: a query is scaled by a power of two, so that its largest
// element has magnitude 2^20 to 2^21, rounded to a whole number and cut into three signed bytes (exact down to 2^-13 of
// the largest element, below that to within 2^-21 of it); the three products' sums are exact.
// V meets weights in fp16: n is exact there, as 1152 + n - 1152: its byte with the sign bit flipped, under the
// byte 0x64, is the fp16 number 1152 + n (two logic operations a pair of numbers, then a subtraction that is
// exact).
// V's steps: the contribution of token t to O is 2^(s_t - m) step_t n_t, so with e_t = log2(step_t) the weights
// P_t = 2^(s_t + e_t - M), M the running maximum of s + e, are at most 2^8 whatever the steps are, and
// l = sum_t P_t 2^-e_t, in fp32.
// A warp sums l 2^K, K the e of its first page: the factor is 2^(K - e_t), and while every |e_t - K| <= 30 what P_t loses below 2^-126
// is 2^-66 of l.  With steps further apart it would not do: tokens of a block of zeros, whose step is 2^-106, count in l
// as any others, and their P_t vanish beside a large step's.  From the first such page on (`far` below) l is summed against a reference r
// of its own, the running maximum of s alone.
//
// Weights for P V.  The instruction takes them in V's type, bf16 or fp16, so each goes in as two numbers, its rounding and the rounding
// of what that leaves, in two products: 2^-15 or 2^-22 of a weight is lost (fp16: 2^-25 of the reference where that is more), where
// one product lost 2^-8 or 2^-11 and outputs of values that cancel were off by as much of what was summed.  It costs 1 % of
// the bf16 windows' time and 2 to 4 % of the 8-bit cache's (64 contexts of 1024 to 16384 tokens 176.5 -> 180.6 us).
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
    float *part;                    // partials (PartLayout): two a CTA, then one a span
    int4 *cuts;                     // [CTAs] the pair that a CTA begins and does not end: request, kv head, last CTA; request -1: none
    uint32_t *status;
    int32_t batch, max_pages_per_req, num_pages, num_kv_heads, group;
    int32_t layer_page_base;        // layer * num_pages
    int32_t num_spans;
    int32_t q_len, q_base, q_pass;  // this launch computes new tokens q_base .. q_base + q_pass - 1; q_pass * group <= 8
    int32_t window, sink;           // window 0: all
    float scale_log2;               // log2(e) / sqrt(d)
};

// Units that a piece costs besides its tiles.  Measured with 1, 2, 3, 4, 6, us, 8-bit: 64 contexts of 1 to 4096 tokens 68.9, 59.9, 57.7,
// 56, 59; 400 of 1 to 300 62.7, 54.8, 54, 52, 54; 64 of 1024 to 16384 180 to 182.  Spans may be of one unit: held to 4, so that few short
// contexts are cut into fewer partials, 4 contexts of 1 to 1024 tokens took 14.2 instead of 10.0.
constexpr int kCacheCost = 4;

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

// The units of a span, of all spans, and whether a length is unusable; then the first tile among a span's.  By one whole warp.
__device__ __forceinline__ long long span_units(const CacheAttnParams &p, int lane, long long &total, bool &unusable)
{
    int sum = 0;
    bool none = false;
    for (int r = lane; r < p.batch; r += 32) {
        const int units = units_of(visited_pages(__ldg(p.seq_lens + r), p));
        sum += units;
        none |= units == 0;
    }
    unusable = __any_sync(0xffffffffu, none);
    total = (long long)warp_sum(sum) * p.num_kv_heads;
    return max(1ll, (total + p.num_spans - 1) / p.num_spans);
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

// A partial: m[8], l[8], then eight rows of D floats at a pitch that spreads the banks.
template <int D>
struct PartLayout {
    static constexpr int kHead = 2 * kMaxGroup, kPitch = D + 4, kFloats = kHead + kMaxGroup * kPitch;
};

// W warps a CTA, each with a ring of S tiles.
template <int D, bool k8, int W, int S>
struct CacheAttnLayout {
    static constexpr int kPageBytes = 32 * D * (k8 ? 1 : 2);
    static constexpr int kHalfBytes = 32 * 128;                  // bf16: a box of 64 columns
    static constexpr int kBoxes = k8 ? 1 : D / 64;               // TMA boxes of a page
    static constexpr int kTileBytes = kPagesPerTile * kPageBytes;
    static constexpr int kRingBytes = S * kTileBytes;
    static constexpr int kStepsOff = W * kRingBytes;             // float2 a page of a stage
    static constexpr int kBarOff = kStepsOff + (k8 ? W * S * kPagesPerTile * 8 : 0);
    static constexpr int kSmemBytes = kBarOff + W * S * 8 + 1024;                // 1024: alignment of the swizzle's pattern
    static_assert(PartLayout<D>::kFloats * 4 <= kRingBytes, "a warp's partial takes its ring's place");
};

// A warp's final l, against m as O is, is kept 2^-5 smaller than it is: with steps of 2^-106 to 2^121 it stays a normal number
// for 2^16 tokens and more.
constexpr int kCacheSumBias = 5, kCacheStepRange = 30;

__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }       // -126 <= e <= 127

template <bool k8>
__device__ __forceinline__ float sum_bias()
{
    return k8 ? __uint_as_float((uint32_t)(127 - kCacheSumBias) << 23) : 1.f;
}

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

// D(16x8, fp32) += A(16x16, row) * B(16x8, col), fp16 or bf16.  Not volatile, so that independent products overlap.
template <bool kHalf>
__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    if constexpr (!kHalf)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// D(16x8, int32) += A(16x32, int8, row) * B(32x8, int8, col)
__device__ __forceinline__ void mma_s8_16832(int (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// The same with nothing to add to.
__device__ __forceinline__ void mma_s8_16832_first(int (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=r"(d[0]), "=r"(d[1]), "=r"(d[2]), "=r"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "r"(0));
}

__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi)
{
    uint32_t d;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}

// Two weights as the product with V takes them, and what that leaves of them.
template <bool k8>
__device__ __forceinline__ void split_weights(float p0, float p1, uint32_t &weights, uint32_t &rest)
{
    if constexpr (k8) {
        const uint32_t w = pack_f16x2(p0, p1);
        const float2 x = __half22float2(*reinterpret_cast<const __half2 *>(&w));
        weights = movmatrix_trans(w);
        rest = movmatrix_trans(pack_f16x2(p0 - x.x, p1 - x.y));
    } else {
        // cut, not rounded, and 2^-23 of the weight added to what is left, so that this is above 0 wherever the weight is: an infinite
        // value that is seen has to stay infinite, which times 0 or a negative rest it would not
        constexpr float kMore = 1.f + 0x1p-23f;
        const uint32_t b0 = __float_as_uint(p0), b1 = __float_as_uint(p1);
        weights = movmatrix_trans(__byte_perm(b0, b1, 0x7632));
        rest = movmatrix_trans(pack_bf16x2(fmaf(p0, kMore, -__uint_as_float(b0 & 0xffff0000u)), fmaf(p1, kMore, -__uint_as_float(b1 & 0xffff0000u))));
    }
}

// ldmatrix at addr + kOffset.  Volatile: ordered behind the waits for the tile.
template <int kOffset>
__device__ __forceinline__ void ldmatrix_x4_at(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4+%5];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr), "n"(kOffset));
}

template <int kOffset>
__device__ __forceinline__ void ldmatrix_x4_trans_at(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4+%5];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr), "n"(kOffset));
}

template <int N>
struct Const {
    static constexpr int value = N;
};

// f(Const<0>) .. f(Const<N - 1>), so that an index may be part of a type.
template <int N, typename F>
__device__ __forceinline__ void unrolled(F f)
{
    if constexpr (N > 0) {
        unrolled<N - 1>(f);
        f(Const<N - 1>());
    }
}

// Byte offset of the 16 bytes c of a row within a page's box, as TMA's swizzle lays them.  In a box that begins at a multiple
// of the swizzle's pattern, the offset of pieces 2 k + c (c = 0, 1) is that of piece c with bits 5 and up changed by k << 5.
template <int D, bool k8>
__device__ __forceinline__ int piece_at(int row, int c)
{
    if constexpr (k8 && D == 64) return row * 64 + ((c ^ ((row >> 1) & 3)) << 4);
    else return row * 128 + ((c ^ (row & 7)) << 4);
}

// One warp's part of a pair: its queries, what it sees, and what it has summed.  Columns of the matrix products are
// (new token c / G, head c % G), ncols of the eight live; a lane accumulates columns g0 and g0 + 1.
template <int D, bool k8>
struct PairPart {
    static constexpr int kSteps16 = D / 16, kQueryRegs = k8 ? 3 * D / 32 : D / 16;
    uint32_t qf[kQueryRegs][2];     // B fragments; 8-bit: D / 32 of the queries' high bytes, then of the middle and the low ones
    float qs0, qs1;                 // what a score is multiplied by: scale and, 8-bit, the query's power of two
    int earliest, pos0, pos1;       // position of the launch's first new token, and of the lane's columns' tokens
    int i0, i1;                     // those tokens
    int seen_head, seen_from, seen_to;           // tiles that every column sees entirely: [0, seen_head) and [seen_from, seen_to)
    uint32_t k_off, v_off;          // ldmatrix: this lane's rows of a page's keys and values, piece 0 or 1
    float m0, m1, l0, l1;
    static constexpr int kNoStep = 1 << 20;
    int K;                          // 8-bit: l is 2^K times what it is against m; far: l is against r, and d = 2^(m - r)
    bool far;
    float r0, r1, d0, d1;
    float o[kSteps16][4];

    __device__ __forceinline__ void begin(const CacheAttnParams &p, const Visited &vis, int r, int h, int L, int lane)
    {
        const int G = p.group, heads = p.num_kv_heads * G, ncols = p.q_pass * G;
        const int g0 = (lane & 3) * 2, c = lane >> 2, j = lane & 3;
        i0 = min(g0 / G, p.q_pass - 1);
        i1 = min((g0 + 1) / G, p.q_pass - 1);
        earliest = L - p.q_len + p.q_base;
        pos0 = earliest + i0;
        pos1 = earliest + i1;
        {
            // whole pages up to the first new token's, from the one on that begins behind the last one's window's start
            const int whole = (earliest + 1) / kPageSize, start = earliest + p.q_pass - 1 - p.window;
            const int from = p.window > 0 && start >= 0 ? start / kPageSize + 1 : 0;
            seen_head = min(min(vis.head, p.sink / kPageSize), whole) / kPagesPerTile;
            seen_from = (from - vis.skip + kPagesPerTile - 1) / kPagesPerTile;
            seen_to = (whole - vis.skip) / kPagesPerTile;
            const int row = (lane & 7) + ((lane >> 3) & 1) * 8, row_v = k8 ? 16 + row : 16 + (lane & 7) + (lane >> 4) * 8;
            k_off = piece_at<D, k8>(row, lane >> 4);
            v_off = piece_at<D, k8>(row_v, k8 ? lane >> 4 : (lane >> 3) & 1);
        }
        qs0 = qs1 = p.scale_log2;
        const uint16_t *row = p.q + (((size_t)r * p.q_len + p.q_base + c / G) * heads + h * G + c % G) * D;
        if constexpr (k8) {
            // four elements of every 16 of column lane / 4
            uint2 raw[kSteps16];
            uint32_t most = 0;
#pragma unroll
            for (int ks = 0; ks < kSteps16; ++ks) {
                raw[ks] = c < ncols ? __ldg((const uint2 *)(row + ks * 16 + j * 4)) : make_uint2(0u, 0u);
                most = __vmaxu2(most, __vmaxu2(raw[ks].x & 0x7fff7fffu, raw[ks].y & 0x7fff7fffu));
            }
            most = max(most & 0xffffu, most >> 16);
            most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
            most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
            const int e = max((int)(most >> 7), 21);             // biased exponent of the largest
            const float up = __uint_as_float((uint32_t)(254 + 20 - min(e, 254)) << 23);
            // with an infinity or a NaN in the query every score is infinite or NaN, and so is the row NaN
            const float back = most >= 0x7f80u ? NAN : __uint_as_float((uint32_t)(e - 20) << 23) * p.scale_log2;
#pragma unroll
            for (int ks = 0; ks < kSteps16; ++ks) {
                // x up + 1.5 2^23 + 0x8080, rounded to a whole number: its lowest bytes are the digits, plus 128, 128 and 64
                constexpr float kMagic = 12582912.f + 32896.f;
                const uint32_t f0 = __float_as_uint(fmaf(__uint_as_float(raw[ks].x << 16), up, kMagic));
                const uint32_t f1 = __float_as_uint(fmaf(__uint_as_float(raw[ks].x & 0xffff0000u), up, kMagic));
                const uint32_t f2 = __float_as_uint(fmaf(__uint_as_float(raw[ks].y << 16), up, kMagic));
                const uint32_t f3 = __float_as_uint(fmaf(__uint_as_float(raw[ks].y & 0xffff0000u), up, kMagic));
                const uint32_t a = __byte_perm(f0, f1, 0x5140), b = __byte_perm(f2, f3, 0x5140);
                qf[ks / 2][ks % 2] = (__byte_perm(__byte_perm(f0, f1, 0x0062), __byte_perm(f2, f3, 0x0062), 0x5410) + 0x40404040u) ^ 0x80808080u;
                qf[D / 32 + ks / 2][ks % 2] = __byte_perm(a, b, 0x7632) ^ 0x80808080u;
                qf[2 * (D / 32) + ks / 2][ks % 2] = __byte_perm(a, b, 0x5410) ^ 0x80808080u;
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
        m0 = m1 = -INFINITY;
        l0 = l1 = 0.f;
        K = k8 ? kNoStep : 0;
        far = false;
        r0 = r1 = -INFINITY;
        d0 = d1 = 0.f;
#pragma unroll
        for (int ks = 0; ks < kSteps16; ++ks) o[ks][0] = o[ks][1] = o[ks][2] = o[ks][3] = 0.f;
    }

    __device__ __forceinline__ static bool sees(int pos, int t, const CacheAttnParams &p)
    {
        return t <= pos && (p.window <= 0 || t > pos - p.window || t < p.sink);
    }

    // A tile in shared memory at sb, its steps at steps.
    __device__ __forceinline__ void tile(const CacheAttnParams &p, const Visited &vis, int ti, uint32_t sb, uint32_t steps, int lane)
    {
        if (!far && (ti < seen_head || (ti >= seen_from && ti < seen_to)) && tile_as<true>(p, vis, ti, sb, steps, lane)) return;
        tile_as<false>(p, vis, ti, sb, steps, lane);
    }

    // all_seen: two whole pages, which every column sees entirely.  It is `far` for the other form: false, with nothing done, where
    // the tile's steps are far from 2^K.  (A form of its own for parts that are far cost the others 2 %.)
    template <bool all_seen>
    __device__ __forceinline__ bool tile_as(const CacheAttnParams &p, const Visited &vis, int ti, uint32_t sb, uint32_t steps, int lane)
    {
        constexpr int kPageBytes = 32 * D * (k8 ? 1 : 2), kHalfBytes = 32 * 128;
        const int np = all_seen ? kPagesPerTile : min(kPagesPerTile, vis.count - ti * kPagesPerTile);
        auto first_token = [&](int mt) {
            const int v = ti * kPagesPerTile + mt;
            return (v < vis.head ? v : v + vis.skip) * kPageSize;
        };
        // ---- S^T = K Q^T
        float s[kPagesPerTile][4];
        const uint32_t k_at = sb + k_off, v_at = sb + v_off;
        if constexpr (k8) {
            int d[kPagesPerTile][3][4];
            unrolled<D / 32>([&](auto step) {
                constexpr int ks = decltype(step)::value;
                unrolled<kPagesPerTile>([&](auto page) {
                    constexpr int mt = decltype(page)::value;
                    if (!all_seen && mt >= np && ks > 0) return;                 // what a page that is not there gives is not looked at
                    uint32_t a[4];
                    ldmatrix_x4_at<mt * kPageBytes>(a, k_at ^ (ks << 5));
#pragma unroll
                    for (int digit = 0; digit < 3; ++digit) {
                        const uint32_t b0 = qf[digit * (D / 32) + ks][0], b1 = qf[digit * (D / 32) + ks][1];
                        if constexpr (ks == 0) mma_s8_16832_first(d[mt][digit], a, b0, b1);
                        else mma_s8_16832(d[mt][digit], a, b0, b1);
                    }
                });
            });
#pragma unroll
            for (int mt = 0; mt < kPagesPerTile; ++mt)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[mt][i] = fmaf((float)d[mt][0][i], 65536.f, (float)(d[mt][1][i] * 256 + d[mt][2][i]));
        } else {
#pragma unroll
            for (int mt = 0; mt < kPagesPerTile; ++mt) s[mt][0] = s[mt][1] = s[mt][2] = s[mt][3] = 0.f;
            unrolled<kSteps16>([&](auto step) {
                constexpr int ks = decltype(step)::value;
                unrolled<kPagesPerTile>([&](auto page) {
                    constexpr int mt = decltype(page)::value;
                    if (!all_seen && mt >= np) return;
                    uint32_t a[4];
                    ldmatrix_x4_at<mt * kPageBytes + (ks / 4) * kHalfBytes>(a, k_at ^ (ks % 4 << 5));
                    mma_16816<k8>(s[mt], a[0], a[1], a[2], a[3], qf[ks][0], qf[ks][1]);
                });
            });
        }
        // ---- scores in the log2 domain, V's step among them
        int e[kPagesPerTile] = {};               // log2 of V's step
        float wl[kPagesPerTile];                 // what a weight counts for in l
        bool near = true;
        float mx0 = -INFINITY, mx1 = -INFINITY;
#pragma unroll
        for (int mt = 0; mt < kPagesPerTile; ++mt) {
            float a0 = qs0, a1 = qs1, add = 0.f;
            wl[mt] = 1.f;
            if constexpr (k8) {
                float ks, vs;
                asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(ks), "=f"(vs) : "r"(steps + mt * 8));
                e[mt] = (int)(__float_as_uint(vs) >> 23 & 255u) - 127;           // 128 where the block is NaN
                if (!all_seen && mt >= np) e[mt] = e[0];         // a page that is not there, of masked tokens
                a0 *= ks;
                a1 *= ks;
                add = (float)e[mt] + (vs - vs);
                wl[mt] = power_of_two(K - e[mt]);
                near = near && (unsigned)(K - e[mt] + kCacheStepRange) <= 2u * kCacheStepRange;
            }
            s[mt][0] = fmaf(s[mt][0], a0, add);
            s[mt][1] = fmaf(s[mt][1], a1, add);
            s[mt][2] = fmaf(s[mt][2], a0, add);
            s[mt][3] = fmaf(s[mt][3], a1, add);
            if (!all_seen) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int token = first_token(mt) + (lane >> 2) + (i >= 2 ? 8 : 0);
                    if (mt >= np || !sees(i & 1 ? pos1 : pos0, token, p)) s[mt][i] = -INFINITY;      // selected, never multiplied
                }
            }
            mx0 = fmaxf(mx0, fmaxf(s[mt][0], s[mt][2]));
            mx1 = fmaxf(mx1, fmaxf(s[mt][1], s[mt][3]));
        }
        // The reference that a column's exponentials are taken against moves only when a score exceeds it by
        // more than 2^8; a column with nothing above -inf so far takes them against 0: they come out 0.
        // (Steps that are not near are looked at here too, since a branch is taken anyway.)
        constexpr bool may_be_far = k8 && !all_seen;
        float lim0 = m0, lim1 = m1;
        if (may_be_far && far) {                 // r moves too, where a score may exceed it by as much
            const float low = (float)min(e[0], e[kPagesPerTile - 1]);
            lim0 = fminf(lim0, r0 + low);
            lim1 = fminf(lim1, r1 + low);
        }
        if (__any_sync(0xffffffffu, mx0 > lim0 + 8.f || mx1 > lim1 + 8.f || (k8 && !near))) {
            if (k8 && !near && !(may_be_far && far)) {
                const bool begins = K == kNoStep;
                if (begins) K = e[0];
                if (!begins || abs(K - e[kPagesPerTile - 1]) > kCacheStepRange) {
                    if (all_seen) return false;
                    far = true;
                    r0 = m0 - (float)K;
                    r1 = m1 - (float)K;
                }
#pragma unroll
                for (int mt = 0; mt < kPagesPerTile; ++mt) wl[mt] = power_of_two(K - e[mt]);
            }
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) {
                mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, x));
                mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, x));
            }
            const float old0 = m0, old1 = m1;
            m0 = fmaxf(m0, mx0);
            m1 = fmaxf(m1, mx1);
            const float al0 = fast_exp2(old0 - (m0 == -INFINITY ? 0.f : m0)), al1 = fast_exp2(old1 - (m1 == -INFINITY ? 0.f : m1));
            if (may_be_far && far) {
                float t0 = -INFINITY, t1 = -INFINITY;            // the largest scores, without the steps
#pragma unroll
                for (int mt = 0; mt < kPagesPerTile; ++mt) {
                    t0 = fmaxf(t0, fmaxf(s[mt][0], s[mt][2]) - (float)e[mt]);
                    t1 = fmaxf(t1, fmaxf(s[mt][1], s[mt][3]) - (float)e[mt]);
                }
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) {
                    t0 = fmaxf(t0, __shfl_xor_sync(0xffffffffu, t0, x));
                    t1 = fmaxf(t1, __shfl_xor_sync(0xffffffffu, t1, x));
                }
                const float was0 = r0, was1 = r1;
                r0 = fmaxf(r0, t0);
                r1 = fmaxf(r1, t1);
                l0 *= fast_exp2(was0 - (r0 == -INFINITY ? 0.f : r0));
                l1 *= fast_exp2(was1 - (r1 == -INFINITY ? 0.f : r1));
                d0 = m0 == -INFINITY ? 0.f : fast_exp2(m0 - r0);
                d1 = m1 == -INFINITY ? 0.f : fast_exp2(m1 - r1);
            } else {
                l0 *= al0;
                l1 *= al1;
            }
#pragma unroll
            for (int c = 0; c < kSteps16; ++c) { o[c][0] *= al0; o[c][2] *= al0; o[c][1] *= al1; o[c][3] *= al1; }
        }
        const float ref0 = m0 == -INFINITY ? 0.f : m0, ref1 = m1 == -INFINITY ? 0.f : m1;
        uint32_t pb[kPagesPerTile][2], rest[kPagesPerTile][2];   // weights as the product takes them, and what that rounding leaves
#pragma unroll
        for (int mt = 0; mt < kPagesPerTile; ++mt) {
            const float p0 = fast_exp2(s[mt][0] - ref0), p1 = fast_exp2(s[mt][1] - ref1);
            const float p2 = fast_exp2(s[mt][2] - ref0), p3 = fast_exp2(s[mt][3] - ref1);
            if (may_be_far && far) {
                // P 2^(m - r - e) while that factor is at most 2^64: what P loses is then 2^-62 of l.  (e at most 126 for blocks that are
                // not finite: their tokens are masked, or make the sum NaN, and d, which may be infinite, must not meet 0.)
                const float over = power_of_two(-min(e[mt], 126)), w0 = d0 * over, w1 = d1 * over;
                if (fmaxf(w0, w1) <= 0x1p64f) {
                    l0 = fmaf(p0 + p2, w0, l0);
                    l1 = fmaf(p1 + p3, w1, l1);
                } else {
                    const float z0 = (float)e[mt] + (r0 == -INFINITY ? 0.f : r0), z1 = (float)e[mt] + (r1 == -INFINITY ? 0.f : r1);
                    l0 += fast_exp2(s[mt][0] - z0) + fast_exp2(s[mt][2] - z0);
                    l1 += fast_exp2(s[mt][1] - z1) + fast_exp2(s[mt][3] - z1);
                }
            } else {
                l0 = fmaf(p0 + p2, wl[mt], l0);
                l1 = fmaf(p1 + p3, wl[mt], l1);
            }
            split_weights<k8>(p0, p1, pb[mt][0], rest[mt][0]);   // tokens 0..7 of the page
            split_weights<k8>(p2, p3, pb[mt][1], rest[mt][1]);   // tokens 8..15
        }
        // ---- O^T += V^T P^T
        unrolled<kPagesPerTile>([&](auto page) {
            constexpr int mt = decltype(page)::value;
            if (!all_seen && mt >= np) return;
            if constexpr (k8) {
                unrolled<D / 32>([&](auto step) {
                    constexpr int c = 2 * decltype(step)::value;
                    uint32_t x[4], lo0, hi0, lo1, hi1;
                    ldmatrix_x4_trans_at<mt * kPageBytes>(x, v_at ^ (c << 4));
                    records_to_half(x[0], lo0, hi0);
                    records_to_half(x[1], lo1, hi1);
                    mma_16816<k8>(o[c], lo0, hi0, lo1, hi1, pb[mt][0], pb[mt][1]);
                    mma_16816<k8>(o[c], lo0, hi0, lo1, hi1, rest[mt][0], rest[mt][1]);
                    records_to_half(x[2], lo0, hi0);
                    records_to_half(x[3], lo1, hi1);
                    mma_16816<k8>(o[c + 1], lo0, hi0, lo1, hi1, pb[mt][0], pb[mt][1]);
                    mma_16816<k8>(o[c + 1], lo0, hi0, lo1, hi1, rest[mt][0], rest[mt][1]);
                });
            } else if constexpr (all_seen) {
                unrolled<kSteps16>([&](auto step) {
                    constexpr int c = decltype(step)::value;
                    uint32_t a[4];
                    ldmatrix_x4_trans_at<mt * kPageBytes + (c / 4) * kHalfBytes>(a, v_at ^ (c % 4 << 5));
                    mma_16816<k8>(o[c], a[0], a[1], a[2], a[3], pb[mt][0], pb[mt][1]);
                    mma_16816<k8>(o[c], a[0], a[1], a[2], a[3], rest[mt][0], rest[mt][1]);
                });
            } else {
#pragma unroll 1
                for (int i = 0; i < p.q_pass; ++i) {             // one new token's columns, the rows it sees
                    uint32_t keep[2];
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const int t = first_token(mt) + half * 8 + (lane & 3) * 2;
                        keep[half] = (sees(earliest + i, t, p) ? 0xffffu : 0u) | (sees(earliest + i, t + 1, p) ? 0xffff0000u : 0u);
                    }
                    unrolled<kSteps16>([&](auto step) {
                        constexpr int c = decltype(step)::value;
                        uint32_t a[4];
                        ldmatrix_x4_trans_at<mt * kPageBytes + (c / 4) * kHalfBytes>(a, v_at ^ (c % 4 << 5));
                        a[0] &= keep[0]; a[1] &= keep[0]; a[2] &= keep[1]; a[3] &= keep[1];
                        float x[4] = {0.f, 0.f, 0.f, 0.f};       // other tokens' columns may hold anything
                        mma_16816<k8>(x, a[0], a[1], a[2], a[3], pb[mt][0], pb[mt][1]);
                        mma_16816<k8>(x, a[0], a[1], a[2], a[3], rest[mt][0], rest[mt][1]);
                        if (i0 == i) { o[c][0] += x[0]; o[c][2] += x[2]; }
                        if (i1 == i) { o[c][1] += x[1]; o[c][3] += x[3]; }
                    });
                }
            }
        });
        return true;
    }

    // l against m as O is, 2^-5 of it, and summed over the lanes that share a column.
    __device__ __forceinline__ void finish()
    {
        if constexpr (k8) {
            // in two halves: a factor may lie below fp32's range where l lies as far above
            const float k = K == kNoStep ? 0.f : (float)K;
            const float h0 = fast_exp2(0.5f * ((far && m0 > -INFINITY ? r0 - m0 : -k) - (float)kCacheSumBias));
            const float h1 = fast_exp2(0.5f * ((far && m1 > -INFINITY ? r1 - m1 : -k) - (float)kCacheSumBias));
            l0 = l0 * h0 * h0;
            l1 = l1 * h1 * h1;
        }
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) {
            l0 += __shfl_xor_sync(0xffffffffu, l0, x);
            l1 += __shfl_xor_sync(0xffffffffu, l1, x);
        }
    }

    // Calls put(column, element, x, y) with pairs of neighbouring elements.  8-bit: a lane holds elements d, d + 1
    // (d = 16 c + 2 (lane / 4)) of its two columns; bf16: elements d and d + 8 (d = 16 c + lane / 4), and neighbouring
    // lanes trade, so that each has pairs of one column.
    template <typename Put>
    __device__ __forceinline__ void elements(int lane, float f0, float f1, Put put) const
    {
        const int g0 = (lane & 3) * 2;
        const bool odd = (lane >> 2) & 1;
#pragma unroll
        for (int c = 0; c < kSteps16; ++c) {
            const float x0 = o[c][0] * f0, x1 = o[c][1] * f1, y0 = o[c][2] * f0, y1 = o[c][3] * f1;
            if constexpr (k8) {
                put(g0, c * 16 + (lane >> 2) * 2, x0, y0);
                put(g0 + 1, c * 16 + (lane >> 2) * 2, x1, y1);
            } else {
                const float tx = __shfl_xor_sync(0xffffffffu, odd ? x0 : x1, 4), ty = __shfl_xor_sync(0xffffffffu, odd ? y0 : y1, 4);
                const int d = c * 16 + (lane >> 3) * 2;
                put(g0 + odd, d, odd ? tx : x0, odd ? x1 : tx);
                put(g0 + odd, d + 8, odd ? ty : y0, odd ? y1 : ty);
            }
        }
    }

    // To a partial in shared or global memory.  A warp that gave up leaves NaN.
    __device__ __forceinline__ void store_partial(float *part, int lane, bool alive) const
    {
        using Part = PartLayout<D>;
        const int g0 = (lane & 3) * 2;
        if (lane < 4) {
            *(float2 *)(part + g0) = make_float2(m0, m1);
            *(float2 *)(part + kMaxGroup + g0) = alive ? make_float2(l0, l1) : make_float2(NAN, NAN);
        }
        elements(lane, 1.f, 1.f, [&](int g, int d, float x, float y) { *(float2 *)(part + Part::kHead + g * Part::kPitch + d) = make_float2(x, y); });
    }

    // To the output.  A warp that gave up leaves NaN here too.
    __device__ __forceinline__ void store_out(const CacheAttnParams &p, int r, int h, int lane, bool alive) const
    {
        const int G = p.group, heads = p.num_kv_heads * G, ncols = p.q_pass * G;
        uint16_t *rows = p.out + ((size_t)r * p.q_len + p.q_base) * heads * D + (size_t)h * G * D;
        const float bias = sum_bias<k8>();
        // (O bias) / l: with the largest steps O / l alone would overflow
        elements(lane, bias, bias, [&](int g, int d, float x, float y) {
            const float inv = 1.f / ((g & 1) ? l1 : l0);
            if (g < ncols) *(uint32_t *)(rows + ((size_t)(g / G) * heads + g % G) * D + d) = alive ? pack_bf16x2(x * inv, y * inv) : 0x7fff7fffu;
        });
    }
};

// A column of partials folded by one warp, in their order: the lane's elements are 4 lane .. 4 lane + 3.
struct FoldSum {
    float m, l;
    float4 acc;

    // w = 2^x.  8-bit: in two halves, since a partial of small steps has an l as much larger as the factor is small; its O is small.
    template <bool k8>
    __device__ __forceinline__ void add_l(float l_i, float x, float w)
    {
        if constexpr (k8) {
            const float half = fast_exp2(0.5f * x);
            l += l_i * half * half;
        } else {
            l += w * l_i;
        }
    }
};

// Partial i is at(i), in shared or global memory, for i in the list: list(i) is the one behind i (>= n: none), and
// candidates of the maximum are spread over the lanes.
template <int D, bool k8, typename At, typename Next>
__device__ __forceinline__ FoldSum fold_column(int n, int col, int lane, At at, Next next)
{
    using Part = PartLayout<D>;
    FoldSum f = {-INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
    for (int i = lane; i < n; i += 32)
        if (next(i - 1) == i) f.m = fmaxf(f.m, at(i)[col]);
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) f.m = fmaxf(f.m, __shfl_xor_sync(0xffffffffu, f.m, x));
    const float ref = f.m == -INFINITY ? 0.f : f.m;
#pragma unroll 4
    for (int i = next(-1); i < n; i = next(i)) {
        const float *part = at(i);
        const float w = fast_exp2(part[col] - ref);
        f.add_l<k8>(part[kMaxGroup + col], part[col] - ref, w);
        if (lane * 4 < D) {
            const float4 a = *(const float4 *)(part + Part::kHead + col * Part::kPitch + lane * 4);
            f.acc.x += w * a.x; f.acc.y += w * a.y; f.acc.z += w * a.z; f.acc.w += w * a.w;
        }
    }
    return f;
}

template <int D, bool k8, typename At>
__device__ __forceinline__ FoldSum fold_column(int n, int col, int lane, At at)
{
    return fold_column<D, k8>(n, col, lane, at, [](int i) { return i + 1; });
}

template <int D>
__device__ __forceinline__ void store_fold(const CacheAttnParams &p, int r, int h, int col, const FoldSum &f, float bias, int lane)
{
    const int G = p.group, heads = p.num_kv_heads * G;
    const float inv = 1.f / f.l;
    uint16_t *row = p.out + ((size_t)r * p.q_len + p.q_base + col / G) * heads * D + (size_t)(h * G + col % G) * D;
    if (lane * 4 < D)
        *(uint2 *)(row + lane * 4) = make_uint2(pack_bf16x2(f.acc.x * bias * inv, f.acc.y * bias * inv), pack_bf16x2(f.acc.z * bias * inv, f.acc.w * bias * inv));
}

template <int D>
__device__ __forceinline__ void store_fold_partial(float *part, int col, const FoldSum &f, int lane)
{
    using Part = PartLayout<D>;
    if (lane == 0) { part[col] = f.m; part[kMaxGroup + col] = f.l; }
    if (lane * 4 < D) *(float4 *)(part + Part::kHead + col * Part::kPitch + lane * 4) = f.acc;
}

// Requests of unusable length: rows cleared, status.  By all warps of the grid, a request each in turn: 4000 idle slots of 32 heads x 128
// beside three contexts of 40000 tokens took 666 us by one warp and with requests passed over one by one, 105 so (56 without them).
template <int D>
__device__ __forceinline__ void clear_unusable(const CacheAttnParams &p, int span, int lane)
{
    const int heads = p.num_kv_heads * p.group, row_elems = p.q_pass * heads * D;
    if (span == 0 && lane == 0) atomicOr(p.status, kStatusBadLength);
    int upto = 0;                                // such requests before `base`
    for (int base = 0; base < p.batch; base += 32) {
        const int r = base + lane;
        const unsigned gone = __ballot_sync(0xffffffffu, r < p.batch && visited_pages(__ldg(p.seq_lens + r), p).tiles == 0);
        const int place = upto + __popc(gone & ((1u << lane) - 1u));
        unsigned todo = __ballot_sync(0xffffffffu, (gone >> lane & 1u) && place % p.num_spans == span);
        for (; todo; todo &= todo - 1) {
            uint4 *row = (uint4 *)(p.out + ((size_t)(base + __ffs(todo) - 1) * p.q_len + p.q_base) * heads * D);
            for (int i = lane; i < row_elems / 8; i += 32) row[i] = make_uint4(0u, 0u, 0u, 0u);
        }
        upto += __popc(gone);
    }
}

// A warp's ring of S tiles: barriers, fills, waits.
template <int D, bool k8, int W, int S>
struct TileRing {
    using Lay = CacheAttnLayout<D, k8, W, S>;
    uint32_t ring, steps, bars;
    int issued, done;
    bool alive;

    __device__ __forceinline__ void init(uint8_t *smem, int warp, int lane, const CUtensorMap *tmap)
    {
        ring = smem_u32(smem) + warp * Lay::kRingBytes;
        steps = smem_u32(smem + Lay::kStepsOff) + warp * S * kPagesPerTile * 8;
        bars = smem_u32(smem + Lay::kBarOff) + warp * S * 8;
        issued = done = 0;
        alive = true;
        if (lane == 0) {
            prefetch_tensormap(tmap);
            // a stage is full when its boxes have landed and, 8-bit, the copies of its steps by lanes 0 and 1
            for (int s = 0; s < S; ++s) mbar_init(bars + s * 8, k8 ? 1 + kPagesPerTile : 1);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            fence_proxy_async();
        }
        __syncwarp();
    }

    // Fill the next stage with a tile of np pages of kv head h; lane i holds the id of its page i / kBoxes.
    __device__ __forceinline__ void issue(const CUtensorMap *tmap, const CacheAttnParams &p, int h, int np, int page, uint64_t policy, int lane)
    {
        const int stage = issued % S, pg = lane / Lay::kBoxes, box = lane % Lay::kBoxes;
        const uint32_t bar = bars + stage * 8;
        if (lane == 0) mbar_arrive_expect_tx(bar, np * Lay::kPageBytes);
        __syncwarp();
        if (pg < np) {
            if (page < 0 || page >= p.num_pages) {
                atomicOr(p.status, kStatusBadPage);
                page = 0;
            }
            const int block = (p.layer_page_base + page) * p.num_kv_heads + h;
            tma_load_2d(ring + stage * Lay::kTileBytes + pg * Lay::kPageBytes + box * Lay::kHalfBytes, tmap, box * 64, block * 32, bar, policy);
            if constexpr (k8)
                asm volatile("cp.async.ca.shared.global [%0], [%1], 8;"
                             ::"r"(steps + (stage * kPagesPerTile + pg) * 8), "l"(p.steps + block) : "memory");
        }
        if constexpr (k8) {
            if (lane < kPagesPerTile) asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
        }
        ++issued;
    }

    // Wait for the oldest stage; false once a wait has given up.
    __device__ __forceinline__ bool wait(uint32_t *status)
    {
        if (alive) alive = __all_sync(0xffffffffu, mbar_wait_bounded(bars + done % S * 8, (done / S) & 1, status));
        return alive;
    }
    __device__ __forceinline__ uint32_t tile() const { return ring + done % S * Lay::kTileBytes; }
    __device__ __forceinline__ uint32_t tile_steps() const { return steps + done % S * kPagesPerTile * 8; }
    __device__ __forceinline__ void drain(uint32_t *status) const
    {
        // do not go on while copies may be in flight (only after a wait gave up)
        if (!alive)
            for (int i = max(0, issued - S); i < issued; ++i) mbar_wait_bounded(bars + (i % S) * 8, (i / S) & 1, status);
    }
};

// ------------------------------------------------------------------------------------------
// Even spans of all pairs' tiles.
//
// Warps: what their rings hold is in flight, 128 KB an SM with eight warps of the 8-bit kernel.  More streams at once cost
// bandwidth: 64 contexts of 8700 tokens (1.14 GB) take 181 us with eight warps of two stages (97 % of a copy's rate), 180
// with eight of three (contexts of 1024 to 16384 181 and 182), 190 with ten of two, 191 with twelve of two, 240 with six of two.  In
// long runs the GPU's power limit holds them at 195 to 214 us.
// ------------------------------------------------------------------------------------------
template <int D, bool k8>
struct SpanShape {
    static constexpr int kWarps = k8 ? 8 : 6, kStages = D == 128 ? 2 : 4;
    using Layout = CacheAttnLayout<D, k8, kWarps, kStages>;
};

// What a warp leaves of a pair that its span cuts: [2 w] of its first piece, if others follow it (the partial is
// in global memory, since the ring is still in use), [2 w + 1] of its last piece (in its ring).
struct Contribution {
    int r, h;                       // r = -1: none
    int first, last;                // the CTAs that hold the pair's first and last tiles
};

template <int D, bool k8>
__global__ void __launch_bounds__(SpanShape<D, k8>::kWarps * 32, 1)
cache_attn_span_kernel(const __grid_constant__ CUtensorMap tmap, const CacheAttnParams p)
{
    using Shape = SpanShape<D, k8>;
    using Part = PartLayout<D>;
    constexpr int W = Shape::kWarps, S = Shape::kStages;
    extern __shared__ uint8_t smem_raw[];
    __shared__ Contribution s_left[2 * W];
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int span = blockIdx.x * W + warp;
    TileRing<D, k8, W, S> ring;
    ring.init(smem, warp, lane, &tmap);
    if (lane < 2) s_left[2 * warp + lane].r = -1;
    __syncwarp();
    grid_dependency_wait();                       // every input may come from the preceding kernel
    grid_launch_dependents();
    if (threadIdx.x == 0) p.cuts[blockIdx.x] = make_int4(-1, 0, 0, 0);

    long long total;
    bool unusable;
    const long long q_units = span_units(p, lane, total, unusable), begin = span * q_units, end = min(begin + q_units, total);
    if (unusable) clear_unusable<D>(p, span, lane);
    TilePlace ic = span_begin(p, begin, end, lane);              // the next tile to fetch
    TilePlace cc = ic;                                           // the next to compute

    const uint64_t policy = l2_evict_first_policy();
    // lane i holds page 32 * chunk + i of the pair's visited ones
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
    // Moves to the next tile of the axis; false at the span's end.
    auto advance = [&](TilePlace &at) {
        ++at.v;
        if (++at.tile < at.vis.tiles) return at.v < end;
        at.tile = 0;
        at.v += kCacheCost;
        if (at.v >= end) return false;
        if (++at.h < p.num_kv_heads) return true;
        at.h = 0;
        if (++at.r >= p.batch) return false;
        at.L = __ldg(p.seq_lens + at.r);
        at.vis = visited_pages(at.L, p);
        while (at.vis.tiles == 0) {              // idle slots, 32 at a time
            const int r = at.r + lane, L = r < p.batch ? __ldg(p.seq_lens + r) : 0;
            const unsigned live = __ballot_sync(0xffffffffu, r < p.batch && visited_pages(L, p).tiles != 0);
            if (live == 0u) {
                if ((at.r += 32) >= p.batch) return false;
                continue;
            }
            at.r += __ffs(live) - 1;
            at.L = __shfl_sync(0xffffffffu, L, __ffs(live) - 1);
            at.vis = visited_pages(at.L, p);
        }
        return true;
    };
    bool more = ic.r >= 0;
    auto issue_next = [&]() {
        const int np = min(kPagesPerTile, ic.vis.count - ic.tile * kPagesPerTile);
        const int page = __shfl_sync(0xffffffffu, chunk_now, (ic.tile % kTilesPerChunk * kPagesPerTile + lane / Shape::Layout::kBoxes) & 31);
        ring.issue(&tmap, p, ic.h, np, page, policy, lane);
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
    while (ring.issued < S && more) issue_next();

    float *parked = p.part + (size_t)(2 * gridDim.x + span) * Part::kFloats;
    float *mine = (float *)(smem + warp * Shape::Layout::kRingBytes);
    PairPart<D, k8> part;
    bool go = cc.r >= 0;
    while (go) {
        const int r = cc.r, h = cc.h, tile0 = cc.tile;
        const Visited vis = cc.vis;
        const int n = (int)min((long long)(vis.tiles - tile0), end - cc.v);
        const long long v0 = cc.v;
        part.begin(p, vis, r, h, cc.L, lane);
#pragma unroll 1
        for (int ti = tile0; ti < tile0 + n; ++ti, ++ring.done) {
            if (!ring.wait(p.status)) continue;
            part.tile(p, vis, ti, ring.tile(), ring.tile_steps(), lane);
            __syncwarp();                         // the stage has been read
            if (more) issue_next();               // refill it with the tile S ahead
        }
        part.finish();
        const bool whole = n == vis.tiles;
        cc.tile = tile0 + n - 1;
        cc.v = v0 + n - 1;
        go = advance(cc);
        if (whole) {
            part.store_out(p, r, h, lane, ring.alive);
        } else {
            if (!go) ring.drain(p.status);
            part.store_partial(go ? parked : mine, lane, ring.alive);
            const long long pair0 = v0 - tile0;   // the pair's first tile's unit
            if (lane == 0) s_left[2 * warp + (go ? 0 : 1)] = {r, h, (int)(pair0 / q_units / W), (int)((pair0 + vis.tiles - 1) / q_units / W)};
        }
    }
    ring.drain(p.status);
    __syncthreads();
    // ---- the CTA's fold: consecutive contributions to one pair, a column a warp
    const Contribution left = s_left[min(lane, 2 * W - 1)];
    const unsigned there = __ballot_sync(0xffffffffu, lane < 2 * W && left.r >= 0);
    const unsigned before = there & ((1u << lane) - 1u);
    const int other = before ? 31 - __clz(before) : lane;
    const bool leads = (there >> lane & 1u) &&
                       (before == 0u || s_left[min(other, 2 * W - 1)].r != left.r || s_left[min(other, 2 * W - 1)].h != left.h);
    const int ncols = p.q_pass * p.group;
    int turn = 0;
    for (unsigned leaders = __ballot_sync(0xffffffffu, leads); leaders != 0u; leaders &= leaders - 1u) {
        const int a = __ffs(leaders) - 1;
        const unsigned behind = leaders & (leaders - 1u);        // from the next pair on
        const unsigned mine_too = there & ~((1u << a) - 1u) & (behind ? (behind & -behind) - 1u : 0xffffffffu);
        const Contribution c = s_left[a];
        const bool here = c.first == c.last;     // the whole pair is this CTA's
        float *slot = p.part + (size_t)(2 * blockIdx.x + (c.first == blockIdx.x ? 1 : 0)) * Part::kFloats;
        for (int col = 0; col < ncols; ++col) {
            if (turn++ % W != warp) continue;
            const FoldSum f = fold_column<D, k8>(
                2 * W, col, lane,
                [&](int i) -> const float * {
                    return i & 1 ? (const float *)(smem + i / 2 * Shape::Layout::kRingBytes) : p.part + (size_t)(2 * gridDim.x + blockIdx.x * W + i / 2) * Part::kFloats;
                },
                [&](int i) { const unsigned rest = mine_too >> (i + 1); return rest ? i + __ffs(rest) : 2 * W; });
            if (here) store_fold<D>(p, c.r, c.h, col, f, sum_bias<k8>(), lane);
            else store_fold_partial<D>(slot, col, f, lane);
        }
        if (!here && c.first == blockIdx.x && threadIdx.x == 0) p.cuts[blockIdx.x] = make_int4(c.r, c.h, c.last, 0);
    }
}

// ------------------------------------------------------------------------------------------
// The pairs that CTAs cut: the first CTA's partial lies in its second slot, the others' in their first.  A block
// looks after one CTA's cut; its warps take the eight columns, kFoldGroups warps a column.  (The last CTA to arrive folding
// them in the span kernel saves the launch, and was 1 to 5 us slower in a row of calls: fences and counters at every
// CTA's end, where this kernel starts under the others' tails.)
// ------------------------------------------------------------------------------------------
constexpr int kFoldGroups = 4;

template <int D, bool k8>
__global__ void __launch_bounds__(kMaxGroup * kFoldGroups * 32)
cache_attn_fold_kernel(const CacheAttnParams p)
{
    using Part = PartLayout<D>;
    __shared__ __align__(16) float s_part[kFoldGroups][Part::kFloats];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, col = warp % kMaxGroup, group = warp / kMaxGroup;
    grid_dependency_wait();
    grid_launch_dependents();
    const int first = blockIdx.x;
    const int4 cut = p.cuts[first];
    if (cut.x < 0) return;
    const int n = cut.z - first + 1;
    if (col < p.q_pass * p.group) {
        const FoldSum f = fold_column<D, k8>((n - group + kFoldGroups - 1) / kFoldGroups, col, lane, [&](int i) -> const float * {
            const int cta = first + group + i * kFoldGroups;
            return p.part + (size_t)(2 * cta + (cta == first ? 1 : 0)) * Part::kFloats;
        });
        store_fold_partial<D>(s_part[group], col, f, lane);
    }
    __syncthreads();
    if (group == 0 && col < p.q_pass * p.group)
        store_fold<D>(p, cut.x, cut.y, col, fold_column<D, k8>(kFoldGroups, col, lane, [&](int i) -> const float * { return s_part[i]; }), sum_bias<k8>(), lane);
}

// ------------------------------------------------------------------------------------------
// A cluster of CTAs per pair and block of new tokens; q_pass: new tokens of a block.
//
// Windows of 2048 of 64 requests, 8 kv heads x 128: bf16 (538 MB) 78.7 us, a copy's rate and what neighbours find in L2; 8-bit
// (270 MB) 48.6 us, 85 % of it, the rest start and fold.  Four warps a CTA instead of six: 81.9 and 52.5.  One request's
// window of 512 in 8 bits takes 5.1 us, launch and a chain of look-ups, tiles and folds (with the cluster's CTAs reading each
// other's partials between two barriers, where they push them before one, 0.4 more).
// ------------------------------------------------------------------------------------------
template <int D, bool k8>
struct PairShape {
    static constexpr int kWarps = 6, kStages = (k8 ? 2 : 1) * (D == 128 ? 1 : 2), kCtas = 2;     // CTAs resident on an SM
    using Layout = CacheAttnLayout<D, k8, kWarps, kStages>;
};

template <int D, bool k8>
__global__ void __launch_bounds__(PairShape<D, k8>::kWarps * 32, PairShape<D, k8>::kCtas)
cache_attn_pair_kernel(const __grid_constant__ CUtensorMap tmap, const CacheAttnParams params)
{
    using Shape = PairShape<D, k8>;
    using Part = PartLayout<D>;
    constexpr int W = Shape::kWarps, S = Shape::kStages;
    constexpr int kMostCtas = 16;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(16) float s_fold[kMostCtas][D + 4];     // written by the cluster's CTAs: a column's partial, O, then m and l
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");        // waited for before others' shared memory is written
    const int rank = (int)cluster_rank(), ctas = (int)cluster_size();
    // blocks of new tokens that the columns hold at a time: neighbours, so that they meet in L2
    const int per_pass = params.q_pass, passes = (params.q_len + per_pass - 1) / per_pass;
    CacheAttnParams p = params;
    p.q_base = blockIdx.x / ctas % passes * per_pass;
    p.q_pass = min(per_pass, p.q_len - p.q_base);
    const int pair = blockIdx.x / ctas / passes, r = pair / p.num_kv_heads, h = pair % p.num_kv_heads;
    const int G = p.group, heads = p.num_kv_heads * G, ncols = p.q_pass * G;
    TileRing<D, k8, W, S> ring;
    ring.init(smem, warp, lane, &tmap);
    grid_dependency_wait();                       // every input may come from the preceding kernel
    grid_launch_dependents();
    const int L = __ldg(p.seq_lens + r);
    const Visited vis = visited_pages(L, p);
    if (vis.tiles == 0) {                         // unusable: the same for the whole cluster
        if (rank == 0) {
            for (int i = threadIdx.x; i < ncols * D / 8; i += W * 32) {
                const int c = i / (D / 8);
                uint16_t *row = p.out + ((size_t)r * p.q_len + p.q_base + c / G) * heads * D + (size_t)(h * G + c % G) * D;
                ((uint4 *)row)[i % (D / 8)] = make_uint4(0u, 0u, 0u, 0u);
            }
            if (threadIdx.x == 0) atomicOr(p.status, kStatusBadLength);
        }
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        return;
    }
    const uint64_t policy = l2_evict_first_policy();
    const int step = ctas * W;
    int next = rank * W + warp;                   // the next tile to fetch
    auto page_of = [&](int tile) {
        const int v = tile * kPagesPerTile + lane / Shape::Layout::kBoxes;
        return lane / Shape::Layout::kBoxes < kPagesPerTile && v < vis.count
                   ? __ldg(p.block_tables + (size_t)r * p.max_pages_per_req + (v < vis.head ? v : v + vis.skip)) : 0;
    };
    int page = page_of(next);
    auto issue_next = [&]() {
        const int now = page;
        page = page_of(next + step);
        ring.issue(&tmap, p, h, min(kPagesPerTile, vis.count - next * kPagesPerTile), now, policy, lane);
        next += step;
    };
    while (ring.issued < S && next < vis.tiles) issue_next();
    PairPart<D, k8> part;
    part.begin(p, vis, r, h, L, lane);
#pragma unroll 1
    for (int ti = rank * W + warp; ti < vis.tiles; ti += step, ++ring.done) {
        if (!ring.wait(p.status)) break;
        part.tile(p, vis, ti, ring.tile(), ring.tile_steps(), lane);
        __syncwarp();
        if (next < vis.tiles) issue_next();
    }
    ring.drain(p.status);
    part.finish();
    part.store_partial((float *)(smem + warp * Shape::Layout::kRingBytes), lane, ring.alive);
    __syncthreads();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");          // every CTA of the cluster runs
    // ---- the CTA's fold, a column a warp; the results go to the CTA that looks after the column, column c to CTA c % ctas
    for (int col = warp; col < ncols; col += W) {
        const FoldSum f = fold_column<D, k8>(W, col, lane, [&](int i) -> const float * { return (const float *)(smem + i * Shape::Layout::kRingBytes); });
        if (ctas == 1) {
            store_fold<D>(p, r, h, col, f, sum_bias<k8>(), lane);
            continue;
        }
        const float *slot = s_fold[col / ctas * ctas + rank];
        const int owner = col % ctas;
        if (lane * 4 < D)
            asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};"
                         ::"r"(cluster_map(smem_u32(slot + lane * 4), owner)), "f"(f.acc.x), "f"(f.acc.y), "f"(f.acc.z), "f"(f.acc.w) : "memory");
        if (lane == 0) asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(cluster_map(smem_u32(slot + D), owner)), "f"(f.m), "f"(f.l) : "memory");
    }
    if (ctas == 1) return;
    cluster_barrier();
    // ---- the cluster's fold
    for (int col = rank + warp * ctas; col < ncols; col += W * ctas) {
        const float(*part)[D + 4] = s_fold + col / ctas * ctas;
        FoldSum f = {lane < ctas ? part[lane][D] : -INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
#pragma unroll
        for (int x = kMostCtas / 2; x > 0; x >>= 1) f.m = fmaxf(f.m, __shfl_xor_sync(0xffffffffu, f.m, x));
        f.m = __shfl_sync(0xffffffffu, f.m, 0);
        const float ref = f.m == -INFINITY ? 0.f : f.m;
        for (int c = 0; c < ctas; ++c) {
            const float w = fast_exp2(part[c][D] - ref);
            f.add_l<k8>(part[c][D + 1], part[c][D] - ref, w);
            if (lane * 4 < D) {
                const float4 a = *(const float4 *)(part[c] + lane * 4);
                f.acc.x += w * a.x; f.acc.y += w * a.y; f.acc.z += w * a.z; f.acc.w += w * a.w;
            }
        }
        store_fold<D>(p, r, h, col, f, sum_bias<k8>(), lane);
    }
}

}  // namespace ckv
