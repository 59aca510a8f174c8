// Host runtime and C ABI of the operators around a long decode step (include/chiron_kv.h): rotated
// append, key bounds of the pages, page selection, verification of drafted tokens.
#include "chiron_kv.h"

#include <algorithm>

#include "ckv_host.cuh"
#include "ckv_pagelist.cuh"
#include "ckv_rope.cuh"
#include "ckv_sparse.cuh"
#include "ckv_verify.cuh"

using ckv::aligned16;
using ckv::allow;
using ckv::check_call;
using ckv::enqueue;
using ckv::fail;
using ckv::overlap;

namespace {

size_t index_records(const ckv_config &c) { return (size_t)c.num_layers * c.num_pages * c.num_kv_heads; }

// Pages that one request may hold where pages are selected: their scores fit an SM's shared memory.
constexpr int kMaxSelectPages = 49152;

// score_pages_kernel over all candidate pages, then select_pages_kernel; cand: the most candidates a request
// can have.
template <int D>
int32_t launch_select(ckv_pool *pool, ckv::SelectParams &sp, int cand, void *stream)
{
    static thread_local int configured_device = -1;
    auto score = ckv::score_pages_kernel<D>;
    constexpr size_t score_smem = ckv::ScoreLayout<D>::kSmemBytes;
    if (configured_device != pool->device) {
        CKV_CUDA(allow(score, false, score_smem));
        CKV_CUDA(allow(ckv::select_pages_kernel<16>, false, (size_t)ckv::kMaxSelectThreads * 16 * 4));
        CKV_CUDA(allow(ckv::select_pages_kernel<0>, false, (size_t)kMaxSelectPages * 4));
        configured_device = pool->device;
    }
    const long long pairs = (long long)sp.batch * sp.num_kv_heads;
    if (cand > 0) {
        const long long warps = pairs * ((cand + 15) / 16);      // no more than there can be tiles
        const unsigned blocks = (unsigned)std::min<long long>((warps + ckv::kScoreWarps - 1) / ckv::kScoreWarps, (long long)ckv::kScoreCtas * pool->num_sms);
        CKV_CUDA(enqueue(score, blocks, ckv::kScoreWarps * 32, score_smem, pool->overlap, 0, stream, sp));
        pool->launches += 1;
        sp.after_scores = 1;
    }
    const auto select = [&](auto kernel, int keys) {             // `keys` a thread
        const int threads = std::min(ckv::kMaxSelectThreads, std::max(64, (cand + keys * 32 - 1) / (keys * 32) * 32));
        return enqueue(kernel, (unsigned)pairs, threads, (size_t)cand * 4, pool->overlap, 0, stream, sp);
    };
    CKV_CUDA(cand <= 4 * ckv::kMaxSelectThreads    ? select(ckv::select_pages_kernel<4>, 4)
             : cand <= 8 * ckv::kMaxSelectThreads  ? select(ckv::select_pages_kernel<8>, 8)
             : cand <= 16 * ckv::kMaxSelectThreads ? select(ckv::select_pages_kernel<16>, 16)
                                                   : select(ckv::select_pages_kernel<0>, 16));
    pool->launches += 1;
    return CKV_OK;
}

template <int D>
int32_t launch_index_update(ckv_pool *pool, const ckv::IndexParams &ip, unsigned blocks, void *stream)
{
    static thread_local int configured_device = -1;
    auto kernel = ckv::kv_index_update_kernel<D>;
    constexpr size_t smem = ckv::IndexLayout<D>::kSmemBytes;
    if (configured_device != pool->device) {
        CKV_CUDA(allow(kernel, false, smem));
        configured_device = pool->device;
    }
    CKV_CUDA(enqueue(kernel, blocks, ckv::kIndexWarps * 32, smem, pool->overlap, 0, stream, ip));
    pool->launches += 1;
    return CKV_OK;
}

// The smallest power of two that is at least x, within [1, 16].
unsigned cluster_of(long long x)
{
    unsigned c = 1;
    while (c < 16 && c < x) c *= 2;
    return c;
}

// CTAs of a request: enough to fill the GPU (four CTAs an SM), of 2048 tokens or, the number being rounded up to
// a power of two, at least half as many.  256 requests of 128256 tokens: 2 CTAs 42 us, 4 CTAs 36, 8 CTAs 42;
// clusters of 16 start slowly (64 requests of 50257 tokens: 20 us against 10 with 8) and pay only for a few
// requests (one of 128256: 6.2 us against 8.0).
template <typename T>
int32_t launch_verify(const ckv::VerifyParams &vp, void *stream)
{
    static thread_local int configured_device = -1, num_sms = 0;
    auto kernel = ckv::draft_verify_kernel<T>;
    int device = -1;
    CKV_CUDA(cudaGetDevice(&device));
    if (configured_device != device) {
        CKV_CUDA(allow(kernel, true, 0));
        CKV_CUDA(cudaDeviceGetAttribute(&num_sms, cudaDevAttrMultiProcessorCount, device));
        configured_device = device;
    }
    const long long fill = (4ll * num_sms + vp.batch - 1) / vp.batch;
    const unsigned cluster = cluster_of(std::min<long long>(std::min<long long>(fill, vp.vocab / 2048), vp.batch <= 8 ? 16 : 8));
    CKV_CUDA(enqueue(kernel, (unsigned)vp.batch * cluster, ckv::kVerifyThreads, 0, true, cluster, stream, vp));
    return CKV_OK;
}

int32_t check_index(const ckv_pool *pool, const char *fn, const void *d_index, size_t index_bytes)
{
    if (!d_index) return fail(CKV_EINVAL, "%s: NULL index", fn);
    if (!aligned16(d_index)) return fail(CKV_EINVAL, "%s: index not 16-byte aligned", fn);
    const size_t need = index_records(pool->cfg) * (2 * (size_t)pool->cfg.head_dim + 4);
    if (index_bytes < need) return fail(CKV_ENOMEM, "%s: index holds %zu bytes, %zu needed", fn, index_bytes, need);
    return CKV_OK;
}

uint8_t *layer_records(const ckv_pool *pool, const void *d_index, int32_t layer)
{
    const ckv_config &c = pool->cfg;
    return static_cast<uint8_t *>(const_cast<void *>(d_index)) + (size_t)layer * c.num_pages * c.num_kv_heads * 2 * c.head_dim;
}

float *layer_steps(const ckv_pool *pool, const void *d_index, int32_t layer)
{
    const ckv_config &c = pool->cfg;
    return reinterpret_cast<float *>(static_cast<uint8_t *>(const_cast<void *>(d_index)) + index_records(c) * 2 * c.head_dim) +
           (size_t)layer * c.num_pages * c.num_kv_heads;
}

uint16_t *layer_pool(const ckv_pool *pool, int32_t layer)
{
    const ckv_config &c = pool->cfg;
    return reinterpret_cast<uint16_t *>(pool->d_pool) + (size_t)layer * c.num_pages * c.num_kv_heads * 2 * c.page_size * c.head_dim;
}

}  // namespace

namespace ckv {

int32_t select_launch(ckv_pool *pool, const char *fn, int32_t layer, int32_t batch, const int32_t *d_block_tables,
                             const int32_t *d_seq_lens, const void *d_q, const void *d_index, size_t index_bytes,
                             int32_t budget, int32_t sink, int32_t recent, int32_t *d_pages, int32_t *d_lens, bool attend,
                      SelectParams *out_params, bool *selected, void *stream)
{
    if (int32_t rc = check_call(pool, layer, batch, fn)) return rc;
    if (!d_block_tables || !d_seq_lens || !d_q || !d_pages || !d_lens) return fail(CKV_EINVAL, "%s: NULL argument", fn);
    if (!aligned16(d_q)) return fail(CKV_EINVAL, "%s: q not 16-byte aligned", fn);
    if (sink < 0 || recent < 1 || budget < 1 || (long long)sink + recent > budget)
        return fail(CKV_EINVAL, "%s: budget %d must hold sink %d >= 0 and recent %d >= 1 pages", fn, budget, sink, recent);
    if (int32_t rc = ckv::check_budget(budget, fn)) return rc;
    const ckv_config &c = pool->cfg;
    if (c.max_pages_per_req > kMaxSelectPages)
        return fail(CKV_EINVAL, "%s: selection holds at most %d pages of a request, the tables have %d", fn, kMaxSelectPages, c.max_pages_per_req);
    if (int32_t rc = check_index(pool, fn, d_index, index_bytes)) return rc;
    // blocks of one request write its results while others still read its length and pages
    const long long tables_n = (long long)batch * c.max_pages_per_req, pages_n = (long long)batch * c.num_kv_heads * budget;
    if (overlap(d_pages, pages_n, d_block_tables, tables_n) || overlap(d_pages, pages_n, d_seq_lens, batch) ||
        overlap(d_lens, batch, d_block_tables, tables_n) || overlap(d_lens, batch, d_seq_lens, batch) || overlap(d_pages, pages_n, d_lens, batch))
        return fail(CKV_EINVAL, "%s: pages and lens must not overlap the tables, the lengths or one another", fn);
    SelectParams &sp = *out_params;
    sp = SelectParams{};
    sp.records = layer_records(pool, d_index, layer);
    sp.steps = layer_steps(pool, d_index, layer);
    sp.block_tables = d_block_tables;
    sp.seq_lens = d_seq_lens;
    sp.q = static_cast<const uint16_t *>(d_q);
    sp.sel_tables = d_pages;
    sp.sel_lens = d_lens;
    sp.status = pool->wsp<uint32_t>(pool->ws.status);
    sp.batch = batch;
    sp.max_pages_per_req = c.max_pages_per_req;
    sp.num_pages = c.num_pages;
    sp.num_kv_heads = c.num_kv_heads;
    sp.group = c.num_q_heads / c.num_kv_heads;
    sp.budget = budget;
    sp.sink = sink;
    sp.recent = recent;
    sp.key_stride = ckv::key_stride(c);
    const long long keys = (long long)batch * c.num_kv_heads * sp.key_stride;
    if (keys > ckv::kMaxSelectKeys)
        return fail(CKV_ENOMEM, "%s: %d requests of up to %d pages need %lld scores, a selection holds %lld", fn, batch,
                    c.max_pages_per_req, keys, ckv::kMaxSelectKeys);
    const int cand = c.max_pages_per_req > budget && budget > sink + recent ? c.max_pages_per_req - sink - recent : 0;
    // one launch where tables are short and pairs few (measured at page_list_attn_kernel)
    *selected = !(attend && cand <= kListSelectPages && (long long)batch * c.num_kv_heads <= kListSelectPairs && budget <= kMaxListInKernel);
    if (!*selected) return CKV_OK;
    if (cand > 0 && keys > pool->score_room)
        return fail(CKV_ENOMEM, "%s: %d requests of up to %d pages need room for %lld scores, the scratch (ckv_set_select_scratch) holds %lld",
                    fn, batch, c.max_pages_per_req, keys, pool->score_room);
    sp.keys = pool->d_scores;
    return c.head_dim == 128 ? launch_select<128>(pool, sp, cand, stream) : launch_select<64>(pool, sp, cand, stream);
}

}  // namespace ckv

extern "C" {

int32_t kv_append_rope(ckv_pool *pool, int32_t layer, int32_t batch, int32_t n_tokens, const int32_t *d_block_tables,
                       const int32_t *d_seq_lens, const int32_t *d_new_start, const float *d_inv_freq, int32_t rotary_dim,
                       int32_t interleaved, float scale, const void *d_q, int64_t q_stride, const void *d_k_new,
                       int64_t k_stride, const void *d_v_new, int64_t v_stride, void *d_q_out, int64_t q_out_stride,
                       void *stream)
{
    const char *fn = "kv_append_rope";
    if (int32_t rc = check_call(pool, layer, batch, fn)) return rc;
    const ckv_config &c = pool->cfg;
    if (n_tokens < 0) return fail(CKV_EINVAL, "%s: n_tokens < 0", fn);
    if (!d_block_tables || !d_seq_lens || !d_inv_freq) return fail(CKV_EINVAL, "%s: NULL argument", fn);
    if (rotary_dim < 16 || rotary_dim > c.head_dim || rotary_dim % 16 != 0)
        return fail(CKV_EINVAL, "%s: rotary_dim %d is not a multiple of 16 in [16, %d]", fn, rotary_dim, c.head_dim);
    if (!d_new_start && n_tokens % batch != 0)
        return fail(CKV_EINVAL, "%s: %d tokens do not split evenly over %d requests", fn, n_tokens, batch);
    if (n_tokens == 0) return CKV_OK;
    if (!d_k_new || !d_v_new) return fail(CKV_EINVAL, "%s: NULL argument", fn);
    if ((d_q == nullptr) != (d_q_out == nullptr)) return fail(CKV_EINVAL, "%s: q and q_out go together", fn);
    const int64_t q_row = (int64_t)c.num_q_heads * c.head_dim, kv_row = (int64_t)c.num_kv_heads * c.head_dim;
    const struct { const char *name; const void *ptr; int64_t stride, row; } rows[4] = {
        {"q", d_q, q_stride, q_row}, {"k_new", d_k_new, k_stride, kv_row}, {"v_new", d_v_new, v_stride, kv_row},
        {"q_out", d_q_out, q_out_stride, q_row}};
    for (const auto &x : rows) {
        if (!x.ptr) continue;
        if (!aligned16(x.ptr)) return fail(CKV_EINVAL, "%s: %s not 16-byte aligned", fn, x.name);
        if (n_tokens > 1 && (x.stride < x.row || x.stride % 8 != 0))
            return fail(CKV_EINVAL, "%s: %s's stride between tokens, %lld, is below a token's %lld elements or no multiple of 8", fn, x.name,
                        (long long)x.stride, (long long)x.row);
    }
    if (d_q && d_q_out == d_q && n_tokens > 1 && q_out_stride != q_stride)
        return fail(CKV_EINVAL, "%s: q_out in place of q must have its stride", fn);
    ckv::RopeParams rp{};
    rp.q = static_cast<const uint16_t *>(d_q);
    rp.k = static_cast<const uint16_t *>(d_k_new);
    rp.v = static_cast<const uint16_t *>(d_v_new);
    rp.q_out = static_cast<uint16_t *>(d_q_out);
    rp.q_stride = q_stride; rp.k_stride = k_stride; rp.v_stride = v_stride; rp.q_out_stride = q_out_stride;
    rp.inv_freq = d_inv_freq;
    rp.new_start = d_new_start;
    rp.block_tables = d_block_tables;
    rp.seq_lens = d_seq_lens;
    rp.pool_layer = layer_pool(pool, layer);
    rp.status = pool->wsp<uint32_t>(pool->ws.status);
    rp.batch = batch;
    rp.q_len = n_tokens / batch;
    rp.max_pages_per_req = c.max_pages_per_req;
    rp.num_pages = c.num_pages;
    rp.num_q_heads = c.num_q_heads;
    rp.num_kv_heads = c.num_kv_heads;
    rp.rotary = rotary_dim;
    rp.n_tokens = n_tokens;
    rp.scale = scale;
    // as many rows at a time as make equal turns of at most 256 threads; four tokens a CTA where that leaves
    // every SM eight CTAs
    const int units = c.head_dim / 16, row_count = (d_q ? c.num_q_heads : 0) + 2 * c.num_kv_heads;
    const int turns = (row_count * units + 255) / 256;
    const int rows_per_turn = (row_count + turns - 1) / turns;
    const int several = (long long)pool->num_sms * 8 * 4 <= n_tokens ? 4 : 1;
    const unsigned threads = (unsigned)std::max(32 * several, (rows_per_turn * units + 31) / 32 * 32), blocks = (unsigned)((n_tokens + several - 1) / several);
    const auto launch = [&](auto one, auto four) {
        return several == 1 ? enqueue(one, blocks, threads, 0, pool->overlap, 0, stream, rp)
                            : enqueue(four, blocks, threads, 0, pool->overlap, 0, stream, rp);
    };
    cudaError_t e;
    if (c.head_dim == 128)
        e = interleaved ? launch(ckv::kv_append_rope_kernel<128, true, 1>, ckv::kv_append_rope_kernel<128, true, 4>)
                        : launch(ckv::kv_append_rope_kernel<128, false, 1>, ckv::kv_append_rope_kernel<128, false, 4>);
    else
        e = interleaved ? launch(ckv::kv_append_rope_kernel<64, true, 1>, ckv::kv_append_rope_kernel<64, true, 4>)
                        : launch(ckv::kv_append_rope_kernel<64, false, 1>, ckv::kv_append_rope_kernel<64, false, 4>);
    CKV_CUDA(e);
    pool->launches += 1;
    pool->pool_written = true;
    return CKV_OK;
}

size_t kv_index_bytes(const ckv_config *cfg)
{
    if (kv_pool_bytes(cfg) == 0) {               // says why the configuration is invalid
        return 0;
    }
    return index_records(*cfg) * (2 * (size_t)cfg->head_dim + 4);
}

int32_t kv_index_update(ckv_pool *pool, int32_t layer, int32_t batch, const int32_t *d_block_tables,
                        const int32_t *d_seq_lens, int32_t last_tokens, void *d_index, size_t index_bytes, void *stream)
{
    const char *fn = "kv_index_update";
    if (int32_t rc = check_call(pool, layer, batch, fn)) return rc;
    if (!d_block_tables || !d_seq_lens) return fail(CKV_EINVAL, "%s: NULL argument", fn);
    if (last_tokens < 0) return fail(CKV_EINVAL, "%s: last_tokens < 0", fn);
    if (int32_t rc = check_index(pool, fn, d_index, index_bytes)) return rc;
    const ckv_config &c = pool->cfg;
    ckv::IndexParams ip{};
    ip.pool_layer = layer_pool(pool, layer);
    ip.block_tables = d_block_tables;
    ip.seq_lens = d_seq_lens;
    ip.records = layer_records(pool, d_index, layer);
    ip.steps = layer_steps(pool, d_index, layer);
    ip.status = pool->wsp<uint32_t>(pool->ws.status);
    ip.batch = batch;
    ip.max_pages_per_req = c.max_pages_per_req;
    ip.num_pages = c.num_pages;
    ip.num_kv_heads = c.num_kv_heads;
    ip.last = last_tokens;
    // no more warps than there can be units
    const long long pages = last_tokens > 0 ? std::min<long long>(c.max_pages_per_req, last_tokens / c.page_size + 2) : c.max_pages_per_req;
    const long long ctas = (pages * batch * c.num_kv_heads + ckv::kIndexWarps - 1) / ckv::kIndexWarps;
    const unsigned blocks = (unsigned)std::min<long long>(ctas, 2ll * pool->num_sms);
    return c.head_dim == 128 ? launch_index_update<128>(pool, ip, blocks, stream) : launch_index_update<64>(pool, ip, blocks, stream);
}

int32_t kv_index_values(ckv_pool *pool, int32_t layer, const void *d_index, size_t index_bytes, void *d_out, void *stream)
{
    const char *fn = "kv_index_values";
    if (int32_t rc = check_call(pool, layer, 1, fn)) return rc;
    if (int32_t rc = check_index(pool, fn, d_index, index_bytes)) return rc;
    if (!d_out || !aligned16(d_out)) return fail(CKV_EINVAL, "%s: out is NULL or not 16-byte aligned", fn);
    const ckv_config &c = pool->cfg;
    ckv::IndexValuesParams vp{};
    vp.records = reinterpret_cast<const uint2 *>(layer_records(pool, d_index, layer));
    vp.steps = layer_steps(pool, d_index, layer);
    vp.out = static_cast<uint4 *>(d_out);
    vp.records_n = (long long)c.num_pages * c.num_kv_heads;
    const long long pieces = vp.records_n * (2 * c.head_dim / 8);
    const unsigned blocks = (unsigned)((pieces + 1023) / 1024);
    CKV_CUDA(c.head_dim == 128 ? enqueue(ckv::kv_index_values_kernel<128>, blocks, 256, 0, pool->overlap, 0, stream, vp)
                               : enqueue(ckv::kv_index_values_kernel<64>, blocks, 256, 0, pool->overlap, 0, stream, vp));
    pool->launches += 1;
    return CKV_OK;
}

size_t kv_select_bytes(const ckv_config *cfg)
{
    if (kv_pool_bytes(cfg) == 0) return 0;       // says why the configuration is invalid
    return sizeof(uint32_t) * (size_t)std::min((long long)cfg->max_batch * cfg->num_kv_heads * ckv::key_stride(*cfg), ckv::kMaxSelectKeys);
}

int32_t ckv_set_select_scratch(ckv_pool *pool, void *d_scratch, size_t scratch_bytes)
{
    const char *fn = "ckv_set_select_scratch";
    if (!pool) return fail(CKV_EINVAL, "%s: pool is NULL", fn);
    if (!aligned16(d_scratch)) return fail(CKV_EINVAL, "%s: scratch not 16-byte aligned", fn);
    pool->d_scores = static_cast<uint32_t *>(d_scratch);
    pool->score_room = d_scratch ? (long long)(scratch_bytes / sizeof(uint32_t)) : 0;
    return CKV_OK;
}

int32_t decode_select_pages(ckv_pool *pool, int32_t layer, int32_t batch, const int32_t *d_block_tables,
                            const int32_t *d_seq_lens, const void *d_q, const void *d_index, size_t index_bytes,
                            int32_t budget, int32_t sink, int32_t recent, int32_t *d_pages, int32_t *d_lens, void *stream)
{
    ckv::SelectParams sp;
    bool selected;
    return ckv::select_launch(pool, "decode_select_pages", layer, batch, d_block_tables, d_seq_lens, d_q, d_index, index_bytes,
                              budget, sink, recent, d_pages, d_lens, false, &sp, &selected, stream);
}

int32_t draft_verify(int32_t batch, int32_t max_draft, int32_t vocab, int32_t dtype, const int32_t *d_draft_tokens,
                     const int32_t *d_draft_lens, const void *d_target_probs, int64_t target_stride,
                     const void *d_draft_probs, int64_t draft_stride, const float *d_u_accept, const float *d_u_sample,
                     int32_t *d_tokens, int32_t *d_accepted, void *stream)
{
    const char *fn = "draft_verify";
    if (batch < 1 || max_draft < 0 || vocab < 1) return fail(CKV_EINVAL, "%s: batch %d, max_draft %d or vocab %d out of range", fn, batch, max_draft, vocab);
    if ((long long)batch * 16 >= (1ll << 31)) return fail(CKV_EINVAL, "%s: batch %d out of range", fn, batch);
    if (dtype != CKV_PROBS_F32 && dtype != CKV_PROBS_BF16) return fail(CKV_EINVAL, "%s: unknown dtype %d", fn, dtype);
    if (!d_target_probs || !d_u_sample || !d_tokens || !d_accepted || (max_draft > 0 && (!d_draft_tokens || !d_u_accept)))
        return fail(CKV_EINVAL, "%s: NULL argument", fn);
    if (target_stride < vocab || (d_draft_probs && draft_stride < vocab)) return fail(CKV_EINVAL, "%s: a row's stride is below the vocabulary", fn);
    const uintptr_t size = dtype == CKV_PROBS_F32 ? 4 : 2;
    const uintptr_t at = reinterpret_cast<uintptr_t>(d_target_probs) | reinterpret_cast<uintptr_t>(d_draft_probs);
    if (at % size != 0) return fail(CKV_EINVAL, "%s: probabilities not aligned to their type", fn);
    // blocks of one request write its results while others still read its drafts
    const long long drafts_n = (long long)batch * max_draft, tokens_n = drafts_n + batch;
    if (overlap(d_tokens, tokens_n, d_draft_tokens, drafts_n) || overlap(d_tokens, tokens_n, d_draft_lens, batch) ||
        overlap(d_accepted, batch, d_draft_tokens, drafts_n) || overlap(d_accepted, batch, d_draft_lens, batch) ||
        overlap(d_tokens, tokens_n, d_u_sample, batch) || overlap(d_accepted, batch, d_u_sample, batch) ||
        overlap(d_tokens, tokens_n, d_u_accept, drafts_n) || overlap(d_accepted, batch, d_u_accept, drafts_n) || overlap(d_tokens, tokens_n, d_accepted, batch))
        return fail(CKV_EINVAL, "%s: tokens and accepted must not overlap the drafts, their lengths, the random numbers or one another", fn);
    ckv::VerifyParams vp{};
    vp.draft_tokens = d_draft_tokens;
    vp.draft_lens = d_draft_lens;
    vp.target = d_target_probs;
    vp.draft = max_draft > 0 ? d_draft_probs : nullptr;
    vp.u_accept = d_u_accept;
    vp.u_sample = d_u_sample;
    vp.tokens = d_tokens;
    vp.accepted = d_accepted;
    vp.target_stride = target_stride;
    vp.draft_stride = d_draft_probs ? draft_stride : 0;
    vp.batch = batch;
    vp.max_draft = max_draft;
    vp.vocab = vocab;
    return dtype == CKV_PROBS_F32 ? launch_verify<float>(vp, stream) : launch_verify<__nv_bfloat16>(vp, stream);
}

}  // extern "C"
