// Rotated append: the new queries and keys of a step are turned by their positions, keys and values
// are written to their pages.
#pragma once

#include "ckv_common.cuh"

namespace ckv {

// Rotation.  Pair j of a head (j < rotary/2) at position t is a point of the plane turned by the
// angle t * inv_freq[j]:  x' = x cos - y sin,  y' = y cos + x sin.  The pair is (j, j + rotary/2),
// or (2j, 2j + 1) when interleaved; elements from `rotary` on are copied.
//
// The angle grows with the position: in 32 bits t * inv_freq loses 2^-24 of up to 10^5 radians.  So
// the product is formed in 64 bits, in whole turns, and its fraction (within half a turn) goes to
// sincospif as fp32, what that rounding leaves by one step of the sums of angles: both stay within a few 2^-24 of themselves at any
// position, where they are near 0 too (without that step they were 2^-24 off in absolute terms).  Each product is rounded once to bf16.
//
// Layout of the work.  A CTA owns kTokens consecutive tokens: one where they are few, four in long
// prompts, where finding each token's request, page and sines would otherwise hold up its loads.  A
// unit is 16 elements of one row that share 8 frequencies: two 16-byte pieces, 8 elements apart
// (interleaved, copied) or rotary/2 apart.  A thread keeps its unit index u and walks over rows
// (query heads, key heads, value heads) and tokens, the next row's loads on their way: every load of a row
// is a full 16-byte piece with neighbours in neighbouring lanes, and the 8 cosines and sines are
// read from shared memory once a token.  The first loads are issued before anything is looked up.
struct RopeParams {
    const uint16_t *q, *k, *v;      // [tokens][heads][d], each with its own stride between tokens
    uint16_t *q_out;
    long long q_stride, k_stride, v_stride, q_out_stride;      // elements
    const float *inv_freq;          // [rotary / 2]
    const int32_t *new_start;       // [batch + 1] first token of each request, or NULL: q_len each
    const int32_t *block_tables;
    const int32_t *seq_lens;
    uint16_t *pool_layer;
    uint32_t *status;
    int32_t batch, q_len, max_pages_per_req, num_pages, num_q_heads, num_kv_heads;
    int32_t n_tokens, rotary;
    float scale;                    // multiplies cosines and sines (1 unless a scaled scheme asks for it)
};

// The request that token i belongs to: the last r with new_start[r] <= i, for a non-decreasing list.
// Executed by whole warps; 32 candidates a round.  -1 if i lies outside the list.
__device__ __forceinline__ int request_of_token(const int32_t *__restrict__ new_start, int batch, int i, int lane)
{
    if (i < __ldg(new_start) || i >= __ldg(new_start + batch)) return -1;
    int lo = 0, n = batch;                       // the answer lies in [lo, lo + n)
    while (n > 1) {
        const int step = (n + 31) / 32;
        const int at = lo + lane * step;
        const bool below = at < lo + n && __ldg(new_start + at) <= i;
        const int last = 31 - __clz(__ballot_sync(0xffffffffu, below) | 1u);     // candidate 0 is below by construction
        const int from = lo + last * step;
        n = min(step, lo + n - from);
        lo = from;
    }
    return lo;
}

__device__ __forceinline__ float bf16_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }

// Of an angle in whole turns.
__device__ __forceinline__ void cosine_sine(double turns, float &c, float &s)
{
    const double halves = 2. * (turns - rint(turns));
    const float x = (float)halves, rest = (float)(halves - (double)x) * 3.14159265f;
    float sine, cosine;
    sincospif(x, &sine, &cosine);
    c = fmaf(-rest, sine, cosine);
    s = fmaf(rest, cosine, sine);
}

template <int D, bool kInterleaved, int kTokens>
__global__ void __launch_bounds__(256, kTokens == 1 ? 4 : 5)
kv_append_rope_kernel(const RopeParams p)
{
    constexpr int U = D / 16;                    // units of a row
    __shared__ float s_cos[kTokens][D / 2], s_sin[kTokens][D / 2];
    __shared__ int s_pos[kTokens], s_page[kTokens];              // page -1: nothing is appended; position -1: unusable, -2: no request's
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long token0 = (long long)blockIdx.x * kTokens;
    const int n = kTokens == 1 ? 1 : (int)min((long long)kTokens, p.n_tokens - token0);
    const int u = threadIdx.x % U;
    const int rows = p.num_q_heads + 2 * p.num_kv_heads;
    const int row_step = blockDim.x / U;
    const int half = p.rotary / 2;
    const bool turned_unit = 8 * u < half;
    // the unit's two pieces, in elements from the row's start
    const int e0 = kInterleaved || !turned_unit ? 16 * u : 8 * u;
    const int e1 = kInterleaved || !turned_unit ? 16 * u + 8 : half + 8 * u;
    grid_dependency_wait();                      // inputs may come from the preceding kernel, the pool may still be read by it
    grid_launch_dependents();

    auto fetch = [&](int tok, int row, uint4 &a, uint4 &b) {
        const long long i = token0 + tok;
        const uint16_t *src;
        if (row < p.num_q_heads) src = p.q + i * p.q_stride + row * D;
        else if (row < p.num_q_heads + p.num_kv_heads) src = p.k + i * p.k_stride + (row - p.num_q_heads) * D;
        else src = p.v + i * p.v_stride + (row - p.num_q_heads - p.num_kv_heads) * D;
        a = *(const uint4 *)(src + e0);
        b = *(const uint4 *)(src + e1);
    };
    const int row0 = (p.q != nullptr ? 0 : p.num_q_heads) + threadIdx.x / U;      // without queries only keys and values move
    int row = row0;
    uint4 a = make_uint4(0u, 0u, 0u, 0u), b = a;
    if (row < rows) fetch(0, row, a, b);

    // ---- each token's request, position and page (a warp a token), then all their cosines and sines
    if (warp < n) {
        const int i = (int)token0 + warp;
        int r, idx, n_new;
        if (p.new_start == nullptr) {
            r = i / p.q_len;
            idx = i - r * p.q_len;
            n_new = p.q_len;
        } else {
            r = request_of_token(p.new_start, p.batch, i, lane);
            const int first = r < 0 ? 0 : __ldg(p.new_start + r);
            n_new = r < 0 ? 0 : __ldg(p.new_start + r + 1) - first;
            idx = i - first;
            if (idx < 0 || idx >= n_new) r = -1;         // in a list that is not in order
        }
        int pos = -2, page = -1;
        if (r >= 0) {
            const int L = __ldg(p.seq_lens + r);
            pos = tiles_of_length(L, p.max_pages_per_req, n_new) != 0 ? L - n_new + idx : -1;
            if (pos >= 0) page = __ldg(p.block_tables + (size_t)r * p.max_pages_per_req + pos / kPageSize);
            if (page < 0 || page >= p.num_pages) {
                if (lane == 0) atomicOr(p.status, pos >= 0 ? kStatusBadPage : kStatusBadLength);
                page = -1;
            }
        }
        if (lane == 0) { s_pos[warp] = pos; s_page[warp] = page; }
    }
    __syncthreads();
    for (int j = threadIdx.x; j < n * half; j += blockDim.x) {
        const int tok = kTokens == 1 ? 0 : j / half, f = kTokens == 1 ? j : j % half;
        const double turns = (double)max(s_pos[tok], 0) * (double)__ldg(p.inv_freq + f) * 0.15915494309189533577;     // 1 / (2 pi)
        float c, s;
        cosine_sine(turns, c, s);
        s_cos[tok][f] = c * p.scale;
        s_sin[tok][f] = s * p.scale;
    }
    __syncthreads();

    if (row >= rows) return;
    for (int tok = 0; tok < n; ++tok) {
        const int pos = s_pos[tok], page = s_page[tok];
        float c[8], s[8];
        if (turned_unit) {
#pragma unroll
            for (int x = 0; x < 8; ++x) { c[x] = s_cos[tok][8 * u + x]; s[x] = s_sin[tok][8 * u + x]; }
        }
        for (; row < rows; row += row_step) {
            uint4 na = a, nb = b;
            if (row + row_step < rows) fetch(tok, row + row_step, na, nb);
            else if (kTokens > 1 && tok + 1 < n) fetch(tok + 1, row0, na, nb);
            const bool value_row = row >= p.num_q_heads + p.num_kv_heads;
            if (turned_unit && !value_row) {
                uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
                if (kInterleaved) {
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const float x0 = bf16_lo(x[w]), y0 = bf16_hi(x[w]), x1 = bf16_lo(y[w]), y1 = bf16_hi(y[w]);
                        x[w] = pack_bf16x2(x0 * c[w] - y0 * s[w], y0 * c[w] + x0 * s[w]);
                        y[w] = pack_bf16x2(x1 * c[w + 4] - y1 * s[w + 4], y1 * c[w + 4] + x1 * s[w + 4]);
                    }
                } else {
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const float x0 = bf16_lo(x[w]), x1 = bf16_hi(x[w]), y0 = bf16_lo(y[w]), y1 = bf16_hi(y[w]);
                        x[w] = pack_bf16x2(x0 * c[2 * w] - y0 * s[2 * w], x1 * c[2 * w + 1] - y1 * s[2 * w + 1]);
                        y[w] = pack_bf16x2(y0 * c[2 * w] + x0 * s[2 * w], y1 * c[2 * w + 1] + x1 * s[2 * w + 1]);
                    }
                }
                a = make_uint4(x[0], x[1], x[2], x[3]);
                b = make_uint4(y[0], y[1], y[2], y[3]);
            }
            uint16_t *dst = nullptr;
            if (row < p.num_q_heads) {
                if (pos > -2) dst = p.q_out + (token0 + tok) * p.q_out_stride + row * D;
                if (pos < 0) a = b = make_uint4(0u, 0u, 0u, 0u);
            } else if (page >= 0) {
                const int kv = value_row ? 1 : 0;
                const int h = row - p.num_q_heads - kv * p.num_kv_heads;
                dst = p.pool_layer + ((((size_t)page * p.num_kv_heads + h) * 2 + kv) * kPageSize + pos % kPageSize) * D;
            }
            if (dst != nullptr) {
                *(uint4 *)(dst + e0) = a;
                *(uint4 *)(dst + e1) = b;
            }
            a = na;
            b = nb;
        }
        row = row0;
    }
}

}  // namespace ckv
