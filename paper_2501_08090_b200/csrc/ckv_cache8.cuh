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
// A CTA owns a page that new tokens of one request touch.  It finds its cosines and sines once (as
// kv_append_rope_kernel, whose rotation this is: rounded to bf16 first, as a bf16 cache would hold the key), then
// its warps take the page's blocks, two per kv head, and after them the query rows.  A warp holds a block's new rows
// in registers, 16 elements a lane and turn, between finding their maximum and quantising them.
struct Append8Params {
    RopeParams rope;                // pool_layer unused; inv_freq NULL: nothing is turned; q NULL: no queries
    uint8_t *records;               // the layer's records
    float *steps;                   // the layer's steps
};

// A page of a request's new tokens: CTAs of a launch are laid out so that request r has at least as many as pages
// that its tokens can touch, beginning with CTA first / 16 + 2 r, `first` being its first token's row.
struct PageOfTokens {
    int r;                          // -1: none
    int L, n;                       // length, and number of the request's rows by the list
    int first, rows;                // the request's first row, and how many of its rows there are before n_tokens
    int page;                       // of its pages, counted from the one that holds its first new token
};

__device__ __forceinline__ PageOfTokens page_of_tokens(const int32_t *__restrict__ start, int each, int n_tokens, const int32_t *__restrict__ lens,
                                                       int batch, int index, int lane)
{
    PageOfTokens t;
    auto begin = [&](int r) { return start == nullptr ? r * each : __ldg(start + r); };
    const int row0 = begin(0);
    auto cta = [&](int r) { return (begin(r) - row0) / kPageSize + 2 * r; };
    int lo = 0, n = batch;                       // the request lies in [lo, lo + n)
    while (n > 1) {
        const int step = (n + 31) / 32, at = lo + lane * step;
        const bool below = at < lo + n && cta(at) <= index;
        const int last = 31 - __clz(__ballot_sync(0xffffffffu, below) | 1u);
        const int from = lo + last * step;
        n = min(step, lo + n - from);
        lo = from;
    }
    t.r = lo;
    t.first = begin(lo);
    t.n = begin(lo + 1) - t.first;
    t.rows = min(t.n, n_tokens - t.first);
    t.L = __ldg(lens + lo);
    t.page = index - cta(lo);
    if (t.first < 0 || t.rows <= 0 || t.page < 0) t.r = -1;         // no rows, or a list that is not in order
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
__global__ void __launch_bounds__(kAppend8Warps * 32)
kv8_append_kernel(const Append8Params p)
{
    constexpr int U = D / 16, kRows = 32 / U, kTurns = kPageSize / kRows;        // lanes of a row, rows a turn, turns of a block
    __shared__ float s_cos[kPageSize][D / 2], s_sin[kPageSize][D / 2];
    const RopeParams &rp = p.rope;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    grid_dependency_wait();                      // inputs may come from the preceding kernel, the cache may still be read by it
    grid_launch_dependents();
    const PageOfTokens t = page_of_tokens(rp.new_start, rp.q_len, rp.n_tokens, rp.seq_lens, rp.batch, blockIdx.x, lane);
    if (t.r < 0) return;
    const int u = lane % U, half = rp.inv_freq != nullptr ? rp.rotary / 2 : 0;
    const bool turned = 8 * u < half;
    const int e0 = kInterleaved || !turned ? 16 * u : 8 * u, e1 = kInterleaved || !turned ? 16 * u + 8 : half + 8 * u;
    if (tiles_of_length(t.L, rp.max_pages_per_req, t.n) == 0) {  // unusable: the request's rows of q_out are cleared, 16 a CTA
        if (threadIdx.x == 0) atomicOr(rp.status, kStatusBadLength);
        if (rp.q == nullptr) return;
        const int rows = min(kPageSize, t.rows - t.page * kPageSize) * rp.num_q_heads;
        for (int i = threadIdx.x / U; i < rows; i += blockDim.x / U) {
            uint16_t *dst = rp.q_out + (long long)(t.first + t.page * kPageSize + i / rp.num_q_heads) * rp.q_out_stride + i % rp.num_q_heads * D + u * 16;
            *(uint4 *)dst = *(uint4 *)(dst + 8) = make_uint4(0u, 0u, 0u, 0u);
        }
        return;
    }
    const int pos0 = t.L - t.n, column = pos0 / kPageSize + t.page;
    const int a = max(pos0, column * kPageSize) - column * kPageSize, b = min(pos0 + t.rows - column * kPageSize, kPageSize);     // slots a .. b - 1
    if (b <= a) return;
    const long long row0 = t.first + (column * kPageSize + a - pos0);
    int page = __ldg(rp.block_tables + (size_t)t.r * rp.max_pages_per_req + column);
    if (page < 0 || page >= rp.num_pages) {
        if (threadIdx.x == 0) atomicOr(rp.status, kStatusBadPage);
        page = -1;                               // queries are turned all the same
    }
    for (int j = threadIdx.x; j < (b - a) * half; j += blockDim.x) {
        const int i = j / half, f = j % half;
        const double turns = (double)(column * kPageSize + a + i) * (double)__ldg(rp.inv_freq + f) * 0.15915494309189533577;     // 1 / (2 pi)
        float c, s;
        sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
        s_cos[i][f] = c * rp.scale;
        s_sin[i][f] = s * rp.scale;
    }
    __syncthreads();
    const int row_in_turn = lane / U;
    for (int item = warp; page >= 0 && item < 2 * rp.num_kv_heads; item += kAppend8Warps) {
        const bool value = item >= rp.num_kv_heads;
        const int h = value ? item - rp.num_kv_heads : item;
        const uint16_t *src = (value ? rp.v : rp.k) + row0 * (value ? rp.v_stride : rp.k_stride) + h * D;
        const long long stride = value ? rp.v_stride : rp.k_stride;
        const size_t block = ((size_t)page * rp.num_kv_heads + h) * 2 + value;
        const float before = a > 0 ? p.steps[block] : 0.f;
        uint4 x[kTurns][2];
        uint32_t most = 0;
#pragma unroll
        for (int k = 0; k < kTurns; ++k) {
            const int i = k * kRows + row_in_turn;
            x[k][0] = x[k][1] = make_uint4(0u, 0u, 0u, 0u);
            if (i < b - a) {
                x[k][0] = *(const uint4 *)(src + i * stride + e0);
                x[k][1] = *(const uint4 *)(src + i * stride + e1);
            }
        }
#pragma unroll
        for (int k = 0; k < kTurns; ++k) {
            const int i = k * kRows + row_in_turn;
            if (turned && !value && i < b - a) turn16<kInterleaved>(x[k][0], x[k][1], &s_cos[i][8 * u], &s_sin[i][8 * u]);
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
        uint8_t *rows = p.records + block * kPageSize * D;
        if (a > 0 && finite && bits != __float_as_uint(before)) {                // older rows get the coarser step
            const float ratio = before * inv;
            for (int w = lane; w < a * D / 4; w += 32) {
                uint32_t *at = (uint32_t *)rows + w;
                const uint32_t n = *at;
                *at = pack_records((float)(int8_t)n * ratio, (float)(int8_t)(n >> 8) * ratio, (float)(int8_t)(n >> 16) * ratio, (float)(int8_t)(n >> 24) * ratio);
            }
        }
#pragma unroll
        for (int k = 0; k < kTurns; ++k) {
            const int i = k * kRows + row_in_turn;
            if (i < b - a) {
                *(uint2 *)(rows + (a + i) * D + e0) = quantise8(x[k][0], inv);
                *(uint2 *)(rows + (a + i) * D + e1) = quantise8(x[k][1], inv);
            }
        }
        if (lane == 0) p.steps[block] = __uint_as_float(bits);
    }
    if (rp.q == nullptr) return;
    for (int i = threadIdx.x / U; i < (b - a) * rp.num_q_heads; i += kAppend8Warps * kRows) {
        const int tok = i / rp.num_q_heads, head = i % rp.num_q_heads;
        const uint16_t *src = rp.q + (row0 + tok) * rp.q_stride + head * D;
        uint4 x = *(const uint4 *)(src + e0), y = *(const uint4 *)(src + e1);
        if (turned) turn16<kInterleaved>(x, y, &s_cos[tok][8 * u], &s_sin[tok][8 * u]);
        uint16_t *dst = rp.q_out + (row0 + tok) * rp.q_out_stride + head * D;
        *(uint4 *)(dst + e0) = x;
        *(uint4 *)(dst + e1) = y;
    }
}

// ------------------------------------------------------------------------------------------
// The values of each request's last tokens, as bf16 rows: exact, since n has 7 bits and the step is a power
// of two.  A CTA per page, as in the append; a thread moves 16 elements.
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
};

template <int D>
__global__ void __launch_bounds__(256)
kv8_gather_kernel(const Gather8Params p)
{
    constexpr int U = D / 16;
    const int lane = threadIdx.x & 31;
    grid_dependency_wait();
    grid_launch_dependents();
    const PageOfTokens t = page_of_tokens(p.start, p.each, p.n_tokens, p.seq_lens, p.batch, blockIdx.x, lane);
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
    const int per_token = 2 * p.num_kv_heads * U, units = (b - a) * per_token;
    for (int i = threadIdx.x; i < units; i += 256) {
        const int tok = i / per_token, rem = i % per_token;
        const int value = rem / (p.num_kv_heads * U), h = rem / U % p.num_kv_heads, u = rem % U;
        uint32_t w[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
        if (page >= 0) {
            const size_t block = ((size_t)page * p.num_kv_heads + h) * 2 + value;
            const uint4 n = __ldg((const uint4 *)(p.records + (block * kPageSize + a + tok) * D) + u);
            const float step = __ldg(p.steps + block);
            const uint32_t x[4] = {n.x, n.y, n.z, n.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                w[2 * j] = pack_bf16x2((float)(int8_t)x[j] * step, (float)(int8_t)(x[j] >> 8) * step);
                w[2 * j + 1] = pack_bf16x2((float)(int8_t)(x[j] >> 16) * step, (float)(int8_t)(x[j] >> 24) * step);
            }
        }
        uint16_t *dst = (value ? p.v + (row0 + tok) * p.v_stride : p.k + (row0 + tok) * p.k_stride) + h * D + u * 16;
        *(uint4 *)dst = make_uint4(w[0], w[1], w[2], w[3]);
        *(uint4 *)(dst + 8) = make_uint4(w[4], w[5], w[6], w[7]);
    }
}

}  // namespace ckv
