// The 8-bit cache: rotated and quantised append, and its values.
#pragma once

#include "ckv_common.cuh"
#include "ckv_rope.cuh"

namespace ckv {

// A block is what one page holds of one kv head, keys or values: 16 rows of d whole numbers n of magnitude <= 127 and
// one step; an element is n * step.  The step is a power of two, so quotients by it are exact: a block has the
// same bits whoever quantises its rows, a value is exact in bf16, and a block that gets a coarser step is
// requantised by a shift.  The price is up to one bit of resolution against a free step.
//
//   m = max |x| of the block's new rows;  need = 2^(floor(log2 max(m, 2^-100)) - 6)  (m / need < 128)
//   step' = need where the rows begin the page, else max(step, need);  n = rint(x / step') within +-127
//   older rows of the page, if step' > step:  n' = rint(n step / step')
//   an infinity or a NaN among the rows: step' = NaN until the page is begun again; the rows' n are 0
//
// bf16 numbers have 8 bits, so x / step' is at most 127.5 and every |n step' - x| <= step' / 2.
//
// A CTA owns a page that new tokens of one request touch, or a part of it where pages are few.  It finds its cosines and
// sines once (as kv_append_rope_kernel, whose rotation this is: rounded to bf16 first, as a bf16 cache would hold the
// key), then its warps take the page's blocks, two per kv head, and after them the query rows.  A warp holds a block's
// new rows in registers, 16 elements a lane and turn, between finding their maximum and quantising them; the first
// block's are on their way before the page is looked up.
//
// Prompts are bound by HBM: 32909 tokens of 32 + 8 + 8 heads x 128 (741 MB) 118 us, 96 % of a copy's rate.  Few tokens by launch,
// look-ups and instructions: one token 2.7 us, five of 96 requests with 64 query heads 7.5, 3.7 without queries.
struct Append8Params {
    RopeParams rope;                // pool_layer unused; inv_freq NULL: nothing is turned; q NULL: no queries
    uint8_t *records;               // the layer's records
    float *steps;                   // the layer's steps
    int32_t parts;                  // CTAs of a page
    uint32_t q_heads_inv;           // inverse_of(query heads)
};

// Quotients of small numbers by a divisor >= 2 that is known at the launch: exact for x < 2^16 and d < 2^16, which
// the rows of a page's tokens are with kCache8MaxHeads query heads.
inline uint32_t inverse_of(uint32_t d) { return (uint32_t)((0x100000000ull + d - 1) / d); }
__device__ __forceinline__ int quotient(int x, uint32_t inverse) { return (int)__umulhi((uint32_t)x, inverse); }

// A page of a request's new tokens.  CTAs of a launch are laid out so that every request has at least as many as
// pages that its tokens can touch: with equally many tokens each, pages_touched of them; else request r's begin with
// CTA first / 16 + 2 r, `first` being its first token's row.
__host__ __device__ inline int pages_touched(int tokens) { return (tokens + kPageSize - 2) / kPageSize + 1; }

struct PageOfTokens {
    int r;                          // -1: none
    int L, n;                       // length, and number of the request's rows by the list
    int first, rows;                // the request's first row, and how many of its rows there are before n_tokens
    int page;                       // of its pages, counted from the one that holds its first new token
};

// By all threads of a CTA, more than the square root of the batch: where the list is short, as it mostly is, each looks at
// one request, its length included, so that nothing is fetched twice on the way to the page.
__device__ __forceinline__ PageOfTokens page_of_tokens(const int32_t *__restrict__ start, int each, int n_tokens, const int32_t *__restrict__ lens,
                                                       int batch, int index)
{
    __shared__ int s_from, s_found[4];
    int r, first, next, L, begin_cta;
    if (start == nullptr) {
        const int of = pages_touched(each);
        r = min(index / of, batch - 1);
        begin_cta = r * of;
        first = r * each;
        next = first + each;
        L = __ldg(lens + r);
    } else {
        const int row0 = __ldg(start);
        auto cta = [&](int begin, int r) { return (begin - row0) / kPageSize + 2 * r; };
        const int threads = blockDim.x, step = (batch + threads - 1) / threads;
        if (threadIdx.x == 0) s_from = s_found[0] = 0;
        if (step > 1) {                          // the stretch of `step` requests that holds it
            const int at = threadIdx.x * step;
            __syncthreads();
            if (at < batch && cta(__ldg(start + at), at) <= index && (at + step >= batch || cta(__ldg(start + at + step), at + step) > index)) s_from = at;
            __syncthreads();
        }
        __syncthreads();
        const int at = s_from + threadIdx.x;
        if (threadIdx.x < (step > 1 ? step : threads) && at < batch) {
            const int begin = __ldg(start + at), end = __ldg(start + at + 1), length = __ldg(lens + at);
            if (cta(begin, at) <= index && (at + 1 >= batch || cta(end, at + 1) > index)) {
                s_found[0] = at;
                s_found[1] = begin;
                s_found[2] = end;
                s_found[3] = length;
            }
        }
        __syncthreads();
        r = s_found[0];
        first = s_found[1];
        next = s_found[2];
        L = s_found[3];
        begin_cta = cta(first, r);
    }
    PageOfTokens t;
    t.r = r;
    t.first = first;
    t.n = next - first;
    t.rows = min(t.n, n_tokens - first);
    t.L = L;
    t.page = index - begin_cta;
    if (first < 0 || t.rows <= 0 || t.page < 0) t.r = -1;        // no rows, or a list that is not in order
    return t;
}

// The step's bits that rows of largest magnitude `most` (bits of a bf16) need.
__device__ __forceinline__ uint32_t step_bits_of(uint32_t most)
{
    if (most >= 0x7f80u) return 0x7fffffffu;                     // NaN
    return (max(most >> 7, 27u) - 6u) << 23;
}

__device__ __forceinline__ uint32_t pack_records(float a, float b, float c, float d)
{
    // nearest, ties to even; a NaN becomes 0; 127.5 becomes 128, cut to 127; -127.5 must not become -128
    const int x = max(__float2int_rn(a), -127), y = max(__float2int_rn(b), -127), z = max(__float2int_rn(c), -127), w = max(__float2int_rn(d), -127);
    uint32_t lo, out;
    asm("cvt.pack.sat.s8.s32.b32 %0, %1, %2, %3;" : "=r"(lo) : "r"(w), "r"(z), "r"(0));
    asm("cvt.pack.sat.s8.s32.b32 %0, %1, %2, %3;" : "=r"(out) : "r"(y), "r"(x), "r"(lo));
    return out;
}

__device__ __forceinline__ uint2 quantise8(const uint4 &x, float inv)
{
    return make_uint2(pack_records(bf16_lo(x.x) * inv, bf16_hi(x.x) * inv, bf16_lo(x.y) * inv, bf16_hi(x.y) * inv),
                      pack_records(bf16_lo(x.z) * inv, bf16_hi(x.z) * inv, bf16_lo(x.w) * inv, bf16_hi(x.w) * inv));
}

// Four records in steps 1 / ratio times as large.
__device__ __forceinline__ uint32_t coarser(uint32_t n, float ratio)
{
    return pack_records((float)(int8_t)n * ratio, (float)(int8_t)(n >> 8) * ratio, (float)(int8_t)(n >> 16) * ratio, (float)(int8_t)(n >> 24) * ratio);
}

// Turn the 16 elements that a lane holds of a row by 8 angles.
template <bool kInterleaved>
__device__ __forceinline__ void turn16(uint4 &a, uint4 &b, const float *__restrict__ c, const float *__restrict__ s)
{
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

constexpr int kAppend8Warps = 8;

template <int D, bool kInterleaved>
__global__ void __launch_bounds__(kAppend8Warps * 32, 3)
kv8_append_kernel(const Append8Params p)
{
    constexpr int U = D / 16, kRows = 32 / U, kTurns = kPageSize / kRows;        // lanes of a row, rows a turn, turns of a block
    __shared__ float s_cos[kPageSize][D / 2], s_sin[kPageSize][D / 2];
    const RopeParams &rp = p.rope;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    grid_dependency_wait();                      // inputs may come from the preceding kernel, the cache may still be read by it
    grid_launch_dependents();
    const int part = (int)(blockIdx.x % p.parts);
    const PageOfTokens t = page_of_tokens(rp.new_start, rp.q_len, rp.n_tokens, rp.seq_lens, rp.batch, blockIdx.x / p.parts);
    if (t.r < 0) return;
    const int u = lane % U, half = rp.inv_freq != nullptr ? rp.rotary / 2 : 0;
    const bool turned = 8 * u < half;
    const int e0 = kInterleaved || !turned ? 16 * u : 8 * u, e1 = kInterleaved || !turned ? 16 * u + 8 : half + 8 * u;
    // who takes query rows: from the last warp on, since the first ones have blocks before (one token 2.7 us instead of 3.3)
    const int row_threads = p.parts * kAppend8Warps * kRows, row_thread = row_threads - 1 - (part * kAppend8Warps * 32 + (int)threadIdx.x) / U;
    if (tiles_of_length(t.L, rp.max_pages_per_req, t.n) == 0) {  // unusable: the request's rows of q_out are cleared, 16 a page's CTAs
        if (threadIdx.x == 0) atomicOr(rp.status, kStatusBadLength);
        if (rp.q == nullptr) return;
        const int rows = min(kPageSize, t.rows - t.page * kPageSize) * rp.num_q_heads;
        for (int i = row_thread; i < rows; i += row_threads) {
            uint16_t *dst = rp.q_out + (long long)(t.first + t.page * kPageSize + i / rp.num_q_heads) * rp.q_out_stride + i % rp.num_q_heads * D + u * 16;
            *(uint4 *)dst = *(uint4 *)(dst + 8) = make_uint4(0u, 0u, 0u, 0u);
        }
        return;
    }
    const int pos0 = t.L - t.n, column = pos0 / kPageSize + t.page;
    const int a = max(pos0, column * kPageSize) - column * kPageSize, b = min(pos0 + t.rows - column * kPageSize, kPageSize);     // slots a .. b - 1
    if (b <= a) return;
    const int n = b - a, row_in_turn = lane / U;
    const long long row0 = t.first + (column * kPageSize + a - pos0);
    int page = __ldg(rp.block_tables + (size_t)t.r * rp.max_pages_per_req + column);
    uint4 x[kTurns][2];
    auto fetch = [&](int item) {                 // a block's new rows
        const bool value = item >= rp.num_kv_heads;
        const long long stride = value ? rp.v_stride : rp.k_stride;
        const uint16_t *src = (value ? rp.v : rp.k) + row0 * stride + (value ? item - rp.num_kv_heads : item) * D;
#pragma unroll
        for (int k = 0; k < kTurns; ++k) {
            const int i = k * kRows + row_in_turn;
            x[k][0] = x[k][1] = make_uint4(0u, 0u, 0u, 0u);
            if (i < n) {
                x[k][0] = *(const uint4 *)(src + i * stride + e0);
                x[k][1] = *(const uint4 *)(src + i * stride + e1);
            }
        }
    };
    const int items = 2 * rp.num_kv_heads, item_step = p.parts * kAppend8Warps;
    int item = part * kAppend8Warps + warp;
    if (item < items) fetch(item);
    for (int i = warp; i < n; i += kAppend8Warps)
        for (int f = lane; f < half; f += 32) {
            const double turns = (double)(column * kPageSize + a + i) * (double)__ldg(rp.inv_freq + f) * 0.15915494309189533577;     // 1 / (2 pi)
            float c, s;
            cosine_sine(turns, c, s);
            s_cos[i][f] = c * rp.scale;
            s_sin[i][f] = s * rp.scale;
        }
    if (page < 0 || page >= rp.num_pages) {
        if (threadIdx.x == 0) atomicOr(rp.status, kStatusBadPage);
        item = items;                            // queries are turned all the same
    }
    __syncthreads();
    for (; item < items; item += item_step) {
        const bool value = item >= rp.num_kv_heads;
        const size_t block = ((size_t)page * rp.num_kv_heads + (value ? item - rp.num_kv_heads : item)) * 2 + value;
        uint8_t *rows = p.records + block * kPageSize * D;
        const float before = a > 0 ? p.steps[block] : 0.f;
        uint32_t most = 0;
#pragma unroll
        for (int k = 0; k < kTurns; ++k) {
            const int i = k * kRows + row_in_turn;
            if (turned && !value && i < n) turn16<kInterleaved>(x[k][0], x[k][1], &s_cos[i][8 * u], &s_sin[i][8 * u]);
            const uint32_t w[8] = {x[k][0].x, x[k][0].y, x[k][0].z, x[k][0].w, x[k][1].x, x[k][1].y, x[k][1].z, x[k][1].w};
#pragma unroll
            for (int e = 0; e < 8; ++e) most = __vmaxu2(most, w[e] & 0x7fff7fffu);
        }
        most = __reduce_max_sync(0xffffffffu, max(most & 0xffffu, most >> 16));
        const uint32_t need = step_bits_of(most);
        // positive numbers and the NaN compare as their bits do
        const uint32_t bits = a > 0 ? max(need, __float_as_uint(before) & 0x7fffffffu) : need;
        const bool finite = bits < 0x7f800000u;
        const float inv = finite ? __uint_as_float((254u << 23) - (bits & 0x7f800000u)) : NAN;
#pragma unroll
        for (int k = 0; k < kTurns; ++k) {
            const int i = k * kRows + row_in_turn;
            if (i < n) {
                *(uint2 *)(rows + (a + i) * D + e0) = quantise8(x[k][0], inv);
                *(uint2 *)(rows + (a + i) * D + e1) = quantise8(x[k][1], inv);
            }
        }
        if (a > 0 && finite && bits != __float_as_uint(before)) {                // older rows get the coarser step: seldom, so fetched only then
            const float ratio = before * inv;
#pragma unroll 1
            for (int i = lane; i < a * D / 16; i += 32) {
                const uint4 old = ((const uint4 *)rows)[i];
                ((uint4 *)rows)[i] = make_uint4(coarser(old.x, ratio), coarser(old.y, ratio), coarser(old.z, ratio), coarser(old.w, ratio));
            }
        }
        if (lane == 0) p.steps[block] = __uint_as_float(bits);
        if (item + item_step < items) fetch(item + item_step);
    }
    if (rp.q == nullptr) return;
    // query rows, kAhead of a thread on their way together (rows are apart, q_out in place of q included)
    constexpr int kAhead = 4;
    const int rows = n * rp.num_q_heads;
#pragma unroll 1
    for (int i0 = row_thread; i0 < rows; i0 += kAhead * row_threads) {
        uint4 lo[kAhead], hi[kAhead];
        int tok[kAhead], head[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int i = min(i0 + k * row_threads, rows - 1);
            tok[k] = rp.num_q_heads > 1 ? quotient(i, p.q_heads_inv) : i;
            head[k] = i - tok[k] * rp.num_q_heads;
            const uint16_t *src = rp.q + (row0 + tok[k]) * rp.q_stride + head[k] * D;
            lo[k] = *(const uint4 *)(src + e0);
            hi[k] = *(const uint4 *)(src + e1);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (i0 + k * row_threads >= rows) break;
            if (turned) turn16<kInterleaved>(lo[k], hi[k], &s_cos[tok[k]][8 * u], &s_sin[tok[k]][8 * u]);
            uint16_t *dst = rp.q_out + (row0 + tok[k]) * rp.q_out_stride + head[k] * D;
            *(uint4 *)(dst + e0) = lo[k];
            *(uint4 *)(dst + e1) = hi[k];
        }
    }
}

// ------------------------------------------------------------------------------------------
// The values of each request's last tokens, as bf16 rows: exact, since n has 7 bits and the step is a power
// of two.  A CTA per page, as in the append; a thread moves 16 elements.  33 000 tokens of 8 heads x 128 (203 MB): 37 us,
// 83 % of a copy's rate, since a page's look-ups stand before 96 KB; one request's last tokens 3.5.
// ------------------------------------------------------------------------------------------
struct Gather8Params {
    const uint8_t *records;         // the layer's
    const float *steps;
    const int32_t *start;           // [batch + 1] first row of each request, or NULL: `each` rows
    const int32_t *block_tables;
    const int32_t *seq_lens;
    uint16_t *k, *v;
    long long k_stride, v_stride;
    uint32_t *status;
    int32_t batch, each, n_tokens, max_pages_per_req, num_pages, num_kv_heads;
    uint32_t per_token_inv;         // inverse_of(rows of a token, 2 * kv heads)
};

template <int D>
__global__ void __launch_bounds__(256)
kv8_gather_kernel(const Gather8Params p)
{
    constexpr int U = D / 16;
    grid_dependency_wait();
    grid_launch_dependents();
    const PageOfTokens t = page_of_tokens(p.start, p.each, p.n_tokens, p.seq_lens, p.batch, blockIdx.x);
    if (t.r < 0) return;
    const bool usable = tiles_of_length(t.L, p.max_pages_per_req, t.n) != 0;
    int a = 0, b = min(kPageSize, t.rows - t.page * kPageSize), page = -1;
    long long row0 = t.first + t.page * kPageSize;               // unusable: the rows are cleared, 16 a CTA
    if (usable) {
        const int pos0 = t.L - t.n, column = pos0 / kPageSize + t.page;
        a = max(pos0, column * kPageSize) - column * kPageSize;
        b = min(pos0 + t.rows - column * kPageSize, kPageSize);
        row0 = t.first + (column * kPageSize + a - pos0);
        if (b <= a) return;
        page = __ldg(p.block_tables + (size_t)t.r * p.max_pages_per_req + column);
    }
    if (page < 0 || page >= p.num_pages) {                       // nothing to read: zeros
        if (threadIdx.x == 0) atomicOr(p.status, usable ? kStatusBadPage : kStatusBadLength);
        page = -1;
    }
    // a thread keeps its 16 elements u of a row and goes through the rows: per token keys of every head, then values
    const int u = threadIdx.x % U, per_token = 2 * p.num_kv_heads, rows = (b - a) * per_token;
    constexpr int kBatch = 4, kStride = 256 / U; // rows of a thread on their way together
#pragma unroll 1
    for (int i0 = threadIdx.x / U; i0 < rows; i0 += kStride * kBatch) {
        uint4 n[kBatch];
        float step[kBatch];
        int tok[kBatch], row[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const int i = i0 + k * kStride;
            tok[k] = quotient(i, p.per_token_inv);
            row[k] = i - tok[k] * per_token;
            n[k] = make_uint4(0u, 0u, 0u, 0u);
            step[k] = 0.f;
            if (page >= 0 && i < rows) {
                const int value = row[k] >= p.num_kv_heads, h = row[k] - value * p.num_kv_heads;
                const size_t block = ((size_t)page * p.num_kv_heads + h) * 2 + value;
                n[k] = __ldg((const uint4 *)(p.records + (block * kPageSize + a + tok[k]) * D) + u);
                step[k] = __ldg(p.steps + block);
            }
        }
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            if (i0 + k * kStride >= rows) break;
            const uint32_t x[4] = {n[k].x, n[k].y, n[k].z, n[k].w};
            uint32_t w[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                w[2 * j] = pack_bf16x2((float)(int8_t)x[j] * step[k], (float)(int8_t)(x[j] >> 8) * step[k]);
                w[2 * j + 1] = pack_bf16x2((float)(int8_t)(x[j] >> 16) * step[k], (float)(int8_t)(x[j] >> 24) * step[k]);
            }
            uint16_t *dst = row[k] >= p.num_kv_heads ? p.v + (row0 + tok[k]) * p.v_stride + (row[k] - p.num_kv_heads) * D : p.k + (row0 + tok[k]) * p.k_stride + row[k] * D;
            *(uint4 *)(dst + u * 16) = make_uint4(w[0], w[1], w[2], w[3]);
            *(uint4 *)(dst + u * 16 + 8) = make_uint4(w[4], w[5], w[6], w[7]);
        }
    }
}

}  // namespace ckv
