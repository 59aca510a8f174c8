// Host runtime and C ABI of a decode step whose state stays on the GPU (include/chiron_kv.h): the 8-bit cache,
// windowed attention, page tables, logits.
#include "chiron_kv.h"

#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "ckv_cache8.cuh"
#include "ckv_cache_attn.cuh"
#include "ckv_host.cuh"
#include "ckv_logits.cuh"
#include "ckv_tables.cuh"

using ckv::aligned16;
using ckv::allow;
using ckv::check_call;
using ckv::enqueue;
using ckv::fail;
using ckv::check_apart;
using ckv::overlap;
using ckv::whole;

namespace {

size_t blocks_of(const ckv_config &c) { return (size_t)c.num_pages * c.num_kv_heads * 2; }      // of a layer: a (page, kv head)'s keys or values

uint8_t *layer_records(const ckv_pool *pool, int32_t layer)
{
    return pool->d_pool + (size_t)layer * blocks_of(pool->cfg) * pool->cfg.page_size * pool->cfg.head_dim;
}

float *all_steps(const ckv_pool *pool)
{
    const ckv_config &c = pool->cfg;
    return reinterpret_cast<float *>(pool->d_pool + (size_t)c.num_layers * blocks_of(c) * c.page_size * c.head_dim);
}

// Rows of tokens, each with its own stride: aligned, and apart by at least a token's elements.
struct Rows {
    const char *name;
    const void *ptr;
    int64_t stride, row;
};

int32_t check_rows(const char *fn, int32_t n_tokens, std::initializer_list<Rows> rows)
{
    for (const Rows &x : rows) {
        if (!x.ptr) continue;
        if (!aligned16(x.ptr)) return fail(CKV_EINVAL, "%s: %s not 16-byte aligned", fn, x.name);
        if (n_tokens > 1 && (x.stride < x.row || x.stride % 8 != 0))
            return fail(CKV_EINVAL, "%s: %s's stride between tokens, %lld, is below a token's %lld elements or no multiple of 8", fn, x.name,
                        (long long)x.stride, (long long)x.row);
    }
    return CKV_OK;
}

// CTAs of a launch that has one for every page that a request's last tokens can touch (page_of_tokens).
unsigned page_ctas(const int32_t *d_start, int32_t n_tokens, int32_t batch)
{
    return d_start ? (unsigned)(n_tokens / ckv::kPageSize + 2 * (long long)batch) : (unsigned)(batch * (long long)ckv::pages_touched(n_tokens / batch));
}

template <int D, bool k8>
int32_t launch_cache_attention(ckv_pool *pool, ckv::CacheAttnParams &ap, void *stream)
{
    using Span = ckv::SpanShape<D, k8>;
    using Pair = ckv::PairShape<D, k8>;
    static thread_local int configured_device = -1, resident[5];              // clusters of 1, 2, 4, 8, 16 CTAs
    auto span = ckv::cache_attn_span_kernel<D, k8>;
    auto pair = ckv::cache_attn_pair_kernel<D, k8>;
    if (configured_device != pool->device) {
        CKV_CUDA(allow(span, false, Span::Layout::kSmemBytes));
        CKV_CUDA(allow(pair, true, Pair::Layout::kSmemBytes));
        for (int i = 0; i < 5; ++i) CKV_CUDA(ckv::resident_clusters(pair, Pair::kWarps * 32, Pair::Layout::kSmemBytes, 1u << i, &resident[i]));
        configured_device = pool->device;
    }
    // The most tiles that a pair can have, and the clusters that own pairs: as many CTAs as its tiles feed, while all
    // clusters run at once, with room for those of a call before that have not ended; without that room where a
    // warp would have more than 5 tiles else.  Windows of 2048, 8 kv heads, with 1, 2, 4, 8, 16 CTAs a pair, us: 2 requests, 8-bit, 10.7, 11.6, 8.0,
    // 7.2, 10.8 (16 do not all run at once); 4 requests, bf16, 13.4, 12.4, 10.0 (3 tiles a warp), 11.6, 16.8; 8 requests, bf16, 17.8,
    // 15.0, 14.4, 20.9, 27.9; 16 requests, 8-bit, 21.7, 17.3, 22.6, 32.8, 51.5.  Taken: 8, 4, 4, 2.
    const long long table = ap.max_pages_per_req;
    const long long cut = ((long long)ap.window + ap.q_len + ckv::kPageSize - 2) / ckv::kPageSize + 1 + ckv::pages_of(ap.sink);
    const bool windowed = ap.window > 0 && cut < table;
    const long long tiles = ((windowed ? cut : table) + ckv::kPagesPerTile - 1) / ckv::kPagesPerTile, pairs = (long long)ap.batch * ap.num_kv_heads;
    const int per_pass = std::min(ap.q_len, ckv::kMaxGroup / ap.group), passes = (ap.q_len + per_pass - 1) / per_pass;      // a launch holds 8 columns
    const long long blocks = pairs * passes;
    int size = 0;
    while (size < 4 && ((long long)Pair::kWarps << size) < tiles &&
           (4 * blocks <= 3ll * resident[size + 1] || (blocks <= resident[size + 1] && tiles > (5ll * Pair::kWarps << size))))
        ++size;
    const unsigned cluster = 1u << size;
    // Pairs that a window cuts are of one length, nearly: a cluster owns each, if the clusters fill the GPU.  Otherwise that
    // pays while a warp has few tiles: the even spans cost 4 us before they win.  Measured, us, pairs against spans: windows of
    // 2048 of 64 requests, bf16 78.9 and 90.1, 8-bit 48.8 and 54.6; one request, 8-bit, of 16384 tokens (5 tiles a warp) 15.4
    // and 17.2, of 32000 (10) 23.7 and 21.8; 64 requests of 1 to 1024 tokens (at most 5) 23.4 and 24.7, of 1 to 2048 (11)
    // 37.4 and 35.1; 400 of 1 to 300 57.3 and 52.7 (bf16 57.7 and 53.9), where the rule is on the wrong side.
    // The host knows the table's width and not the lengths: under one of 8192 pages, 64 requests of 1 to 1024 tokens take
    // the spans (25.1), and 4 of them 10.0 instead of 6.5.
    if (tiles <= 8ll * cluster * Pair::kWarps || (windowed && blocks * cluster > pool->num_sms)) {
        ap.q_pass = per_pass;
        CKV_CUDA(enqueue(pair, (unsigned)(blocks * cluster), Pair::kWarps * 32, Pair::Layout::kSmemBytes, pool->overlap, cluster, stream, pool->tmap, ap));
        pool->launches += 1;
        return CKV_OK;
    }
    const unsigned ctas = std::min(pool->num_sms, ckv::kMaxSpans / Span::kWarps);
    ap.num_spans = (int32_t)ctas * Span::kWarps;
    for (ap.q_base = 0; ap.q_base < ap.q_len; ap.q_base += per_pass) {
        ap.q_pass = std::min(per_pass, ap.q_len - ap.q_base);
        CKV_CUDA(enqueue(span, ctas, Span::kWarps * 32, Span::Layout::kSmemBytes, pool->overlap, 0, stream, pool->tmap, ap));
        CKV_CUDA(enqueue(ckv::cache_attn_fold_kernel<D, k8>, ctas, ckv::kMaxGroup * ckv::kFoldGroups * 32, 0, pool->overlap, 0, stream, ap));
        pool->launches += 2;
    }
    return CKV_OK;
}

int32_t cache_attention(ckv_pool *pool, const char *fn, int bits, int32_t layer, int32_t batch, int32_t q_len, const int32_t *d_block_tables,
                        const int32_t *d_seq_lens, const void *d_q, void *d_out, int32_t window, int32_t sink, void *stream)
{
    if (int32_t rc = check_call(pool, layer, batch, fn, bits)) return rc;
    if (q_len < 1 || q_len > ckv::kMaxGroup) return fail(CKV_EINVAL, "%s: q_len %d outside [1, %d]", fn, q_len, ckv::kMaxGroup);
    if (window < (bits == 8 ? 0 : 1) || sink < 0) return fail(CKV_EINVAL, "%s: window %d or sink %d out of range", fn, window, sink);
    if (!d_block_tables || !d_seq_lens || !d_q || !d_out) return fail(CKV_EINVAL, "%s: NULL argument", fn);
    if (!aligned16(d_q) || !aligned16(d_out)) return fail(CKV_EINVAL, "%s: q/out not 16-byte aligned", fn);
    const ckv_config &c = pool->cfg;
    const long long rows = 2ll * batch * q_len * c.num_q_heads * c.head_dim;
    if (int32_t rc = check_apart(fn, {"out", whole(d_out, rows)},
                                 {{"q", d_out == d_q ? ckv::ByteRows{} : whole(d_q, rows)}, {"block_tables", whole(d_block_tables, 4ll * batch * c.max_pages_per_req)},
                                  {"seq_lens", whole(d_seq_lens, 4ll * batch)}}))
        return rc;
    ckv::CacheAttnParams ap{};
    ap.block_tables = d_block_tables;
    ap.seq_lens = d_seq_lens;
    ap.q = static_cast<const uint16_t *>(d_q);
    ap.out = static_cast<uint16_t *>(d_out);
    ap.steps = bits == 8 ? reinterpret_cast<const float2 *>(all_steps(pool)) : nullptr;
    ap.part = pool->wsp<float>(pool->ws.part);
    ap.cuts = pool->wsp<int4>(pool->ws.cuts);
    ap.status = pool->wsp<uint32_t>(pool->ws.status);
    ap.batch = batch;
    ap.max_pages_per_req = c.max_pages_per_req;
    ap.num_pages = c.num_pages;
    ap.num_kv_heads = c.num_kv_heads;
    ap.group = c.num_q_heads / c.num_kv_heads;
    ap.layer_page_base = layer * c.num_pages;
    ap.q_len = q_len;
    ap.window = window;
    ap.sink = window > 0 ? sink : 0;
    ap.scale_log2 = (float)(1.4426950408889634 / std::sqrt((double)c.head_dim));
    return c.head_dim == 128 ? (bits == 8 ? launch_cache_attention<128, true>(pool, ap, stream) : launch_cache_attention<128, false>(pool, ap, stream))
                             : (bits == 8 ? launch_cache_attention<64, true>(pool, ap, stream) : launch_cache_attention<64, false>(pool, ap, stream));
}

// What both page calls check, and their launch.
template <bool kAssign>
int32_t launch_pages(ckv_pool *pool, const char *fn, const ckv::TablesParams &args, int32_t batch, void *stream)
{
    if (int32_t rc = ckv::check_device(pool, fn)) return rc;
    if (batch < 1 || batch > pool->cfg.max_batch) return fail(CKV_EINVAL, "%s: batch %d outside [1, %d]", fn, batch, pool->cfg.max_batch);
    ckv::TablesParams tp = args;
    if (!tp.block_tables || !tp.seq_lens || !tp.amounts || !tp.free_pages || !tp.free_count || !tp.lens_out || !tp.count_out)
        return fail(CKV_EINVAL, "%s: NULL argument", fn);
    if (tp.n_slots < 0 || (tp.n_slots > 0 && !tp.slots)) return fail(CKV_EINVAL, "%s: %d slots, or no array for them", fn, tp.n_slots);
    if (reinterpret_cast<uintptr_t>(tp.slots) % 8 != 0) return fail(CKV_EINVAL, "%s: slots not 8-byte aligned", fn);
    tp.batch = batch;
    tp.max_pages_per_req = pool->cfg.max_pages_per_req;
    tp.num_pages = pool->cfg.num_pages;
    tp.status = pool->wsp<uint32_t>(pool->ws.status);
    // lengths and count may be written in place; everything else that is written lies apart from what is read
    const long long tables_n = (long long)batch * tp.max_pages_per_req;
    const struct { const void *ptr; long long n; } a[] = {
        {tp.lens_out, batch}, {tp.count_out, 1}, {tp.step_lens, batch}, {tp.new_start, batch + 1ll}, {tp.slots, 2ll * tp.n_slots},
        {tp.block_tables, tables_n}, {tp.free_pages, tp.num_pages},
        {tp.lens_out == tp.seq_lens ? nullptr : tp.seq_lens, batch}, {tp.lens_out == tp.amounts ? nullptr : tp.amounts, batch},
        {tp.count_out == tp.free_count ? nullptr : tp.free_count, 1}};
    for (int i = 0; i < 7; ++i)
        for (int k = i + 1; k < 10; ++k)
            if (overlap(a[i].ptr, a[i].n, a[k].ptr, a[k].n)) return fail(CKV_EINVAL, "%s: two of the arrays overlap", fn);
    // the sums of 8192 requests, three words each, fit an SM's shared memory
    static thread_local int configured_device = -1;
    auto kernel = ckv::pages_kernel<kAssign>;
    if (configured_device != pool->device) {
        CKV_CUDA(allow(kernel, true, sizeof(int) * ckv::kTablesWords * ckv::kMaxBatch));
        configured_device = pool->device;
    }
    // A thread for each page or slot that may have to move, in CTAs of few threads, since what a move costs is instructions:
    // 50000 slots by 256 CTAs of 256 threads 3.7 us, by 64 6.0, by 16 16.0.  In place there are no more than a
    // cluster's 16, of 1024 threads where that is too few (9.9 us); so many too where a CTA's own sums are long.
    tp.in_place = tp.lens_out == tp.seq_lens || tp.lens_out == tp.amounts || tp.count_out == tp.free_count;
    const long long moves = kAssign ? std::max<long long>(tp.n_slots, batch) : tables_n;
    const unsigned threads = batch > 1024 || (tp.in_place && moves > 4096) ? 1024 : 256;
    unsigned ctas = 1;
    while (ctas < (tp.in_place ? 16 : 256) && moves > (long long)threads * ctas) ctas *= 2;
    CKV_CUDA(enqueue(kernel, ctas, threads, sizeof(int) * ckv::kTablesWords * batch, pool->overlap, tp.in_place ? ctas : 0, stream, tp));
    pool->launches += 1;
    pool->inputs_from_predecessor = true;        // a decode step that follows directly must not read its tables ahead
    return CKV_OK;
}

template <typename Tin, typename Tout>
int32_t launch_logits(ckv::LogitsParams &lp, int32_t batch, void *stream)
{
    static thread_local int configured_device = -1, num_sms = 0;
    constexpr int kNarrow = 256, kWide = 512;     // threads of a CTA
    auto narrow = ckv::logits_process_kernel<Tin, Tout, kNarrow>, wide = ckv::logits_process_kernel<Tin, Tout, kWide>;
    constexpr int E = 16 / sizeof(Tin);
    constexpr size_t kMostBytes = 200 * 1024;    // of the arrays of changed tokens
    int device = -1;
    CKV_CUDA(cudaGetDevice(&device));
    if (configured_device != device) {
        CKV_CUDA(allow(narrow, true, kMostBytes));
        CKV_CUDA(allow(wide, true, kMostBytes));
        CKV_CUDA(cudaDeviceGetAttribute(&num_sms, cudaDevAttrMultiProcessorCount, device));
        configured_device = device;
    }
    const long long rows = (long long)batch * lp.rows;
    // pieces of a row, wherever in its first one it may begin
    const bool aligned = aligned16(lp.logits) && (lp.stride % E == 0 || rows == 1);
    const int pieces = (lp.vocab + (aligned ? E - 1 : 2 * E - 2)) / E;
    const long long lists = (lp.history ? lp.history_stride : 0) + (lp.drafts ? lp.rows - 1 : 0) + lp.n_bias;
    const size_t arrays = sizeof(uint32_t) * (lp.bias_ids ? 3 : 2);
    // CTAs of a row: few, since each begins with a chain of look-ups, of at most 16384 tokens (32768 with changes, whose chain
    // is longer: 512 rows of 50257 tokens with everything in 2 CTAs 68 us, in 4 75, in 8 103; alone 47, 43, 51), and with their
    // arrays in shared memory; up to 16 where there are few rows
    const long long most = lists > 0 ? 32 * ckv::kLogitsWords : 16 * ckv::kLogitsWords;
    unsigned cluster = 1;
    const auto slice = [&] { return (pieces + (long long)cluster - 1) / cluster * E; };
    while (slice() > most || std::min(lists, slice()) * arrays > kMostBytes) ++cluster;
    while (cluster < 16 && 2 * cluster * rows <= num_sms && slice() > 2048) cluster = std::min(16u, 2 * cluster);
    lp.pieces = (int)(slice() / E);
    lp.marked = (int)std::min(lists, slice());
    // Twice the threads where all CTAs are on their way at once with much to go through: one request's 5 rows of 128256 tokens
    // with a history of 4096 9.0 us instead of 11.5, 64 rows of 50257 with everything 13.8 instead of 18.0, 140 of 16384 alone 5.4
    // instead of 6.2.  With little, fewer warps meet sooner: 16 rows of 50257 with everything 10.2 and 10.3, 8 with a mask
    // 4.2 and 5.4; and many rows go through four narrow CTAs an SM faster: 512 with everything 68 and 75.
    const bool wider = rows * cluster <= 2 * num_sms && lists + slice() >= 8192;
    CKV_CUDA(enqueue(wider ? wide : narrow, (unsigned)(rows * cluster), wider ? kWide : kNarrow, arrays * lp.marked, true, cluster, stream, lp));
    return CKV_OK;
}

}  // namespace

extern "C" {

int32_t kv8_append(ckv_pool *pool, int32_t layer, int32_t batch, int32_t n_tokens, const int32_t *d_block_tables,
                   const int32_t *d_seq_lens, const int32_t *d_new_start, const float *d_inv_freq, int32_t rotary_dim,
                   int32_t interleaved, float scale, const void *d_q, int64_t q_stride, const void *d_k_new,
                   int64_t k_stride, const void *d_v_new, int64_t v_stride, void *d_q_out, int64_t q_out_stride,
                   void *stream)
{
    const char *fn = "kv8_append";
    if (int32_t rc = check_call(pool, layer, batch, fn, 8)) return rc;
    const ckv_config &c = pool->cfg;
    if (n_tokens < 0) return fail(CKV_EINVAL, "%s: n_tokens < 0", fn);
    if (!d_block_tables || !d_seq_lens) return fail(CKV_EINVAL, "%s: NULL argument", fn);
    if (d_inv_freq && (rotary_dim < 16 || rotary_dim > c.head_dim || rotary_dim % 16 != 0))
        return fail(CKV_EINVAL, "%s: rotary_dim %d is not a multiple of 16 in [16, %d]", fn, rotary_dim, c.head_dim);
    if (!d_new_start && n_tokens % batch != 0)
        return fail(CKV_EINVAL, "%s: %d tokens do not split evenly over %d requests", fn, n_tokens, batch);
    if (n_tokens == 0) return CKV_OK;
    if (!d_k_new || !d_v_new) return fail(CKV_EINVAL, "%s: NULL argument", fn);
    if ((d_q == nullptr) != (d_q_out == nullptr)) return fail(CKV_EINVAL, "%s: q and q_out go together", fn);
    if (d_q && !d_inv_freq) return fail(CKV_EINVAL, "%s: queries are only turned, and there is no inv_freq", fn);
    const int64_t q_row = (int64_t)c.num_q_heads * c.head_dim, kv_row = (int64_t)c.num_kv_heads * c.head_dim;
    if (int32_t rc = check_rows(fn, n_tokens, {{"q", d_q, q_stride, q_row}, {"k_new", d_k_new, k_stride, kv_row}, {"v_new", d_v_new, v_stride, kv_row},
                                               {"q_out", d_q_out, q_out_stride, q_row}}))
        return rc;
    if (d_q && d_q_out == d_q && n_tokens > 1 && q_out_stride != q_stride)
        return fail(CKV_EINVAL, "%s: q_out in place of q must have its stride", fn);
    const ckv::ByteRows q_rows = {d_q, 2 * q_row, 2 * q_stride, n_tokens};
    if (int32_t rc = check_apart(fn, {"q_out", {d_q_out, 2 * q_row, 2 * q_out_stride, n_tokens}},
                                 {{"q", d_q_out == d_q ? ckv::ByteRows{} : q_rows}, {"k_new", {d_k_new, 2 * kv_row, 2 * k_stride, n_tokens}},
                                  {"v_new", {d_v_new, 2 * kv_row, 2 * v_stride, n_tokens}}, {"block_tables", whole(d_block_tables, 4ll * batch * c.max_pages_per_req)},
                                  {"seq_lens", whole(d_seq_lens, 4ll * batch)}, {"new_start", whole(d_new_start, 4ll * batch + 4)},
                                  {"inv_freq", whole(d_inv_freq, 2ll * rotary_dim)}}))
        return rc;
    ckv::Append8Params ap{};
    ckv::RopeParams &rp = ap.rope;
    rp.q = static_cast<const uint16_t *>(d_q);
    rp.k = static_cast<const uint16_t *>(d_k_new);
    rp.v = static_cast<const uint16_t *>(d_v_new);
    rp.q_out = static_cast<uint16_t *>(d_q_out);
    rp.q_stride = q_stride; rp.k_stride = k_stride; rp.v_stride = v_stride; rp.q_out_stride = q_out_stride;
    rp.inv_freq = d_inv_freq;
    rp.new_start = d_new_start;
    rp.block_tables = d_block_tables;
    rp.seq_lens = d_seq_lens;
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
    ap.records = layer_records(pool, layer);
    ap.steps = all_steps(pool) + layer * blocks_of(c);
    ap.q_heads_inv = c.num_q_heads > 1 ? ckv::inverse_of(c.num_q_heads) : 0;
    const auto kernel = c.head_dim == 128 ? (interleaved ? ckv::kv8_append_kernel<128, true> : ckv::kv8_append_kernel<128, false>)
                                          : (interleaved ? ckv::kv8_append_kernel<64, true> : ckv::kv8_append_kernel<64, false>);
    // where pages are few, several CTAs a page, as far as they fit the GPU at a time: their blocks and query rows are chains of
    // look-ups and loads (one token 3.4 us in one CTA, 2.7 in several); twice as far with query rows (five tokens of 96 requests:
    // 8.5 us in two CTAs a page, 7.8 in four; without queries 3.9 and 4.7)
    const unsigned pages = page_ctas(d_new_start, n_tokens, batch);
    ap.parts = 1;
    while (ap.parts < 4 && pages * 2u * ap.parts <= (d_q ? 6u : 3u) * pool->num_sms) ap.parts *= 2;
    CKV_CUDA(enqueue(kernel, pages * ap.parts, ckv::kAppend8Warps * 32, 0, pool->overlap, 0, stream, ap));
    pool->launches += 1;
    return CKV_OK;
}

int32_t kv8_gather(ckv_pool *pool, int32_t layer, int32_t batch, int32_t n_tokens, const int32_t *d_block_tables,
                   const int32_t *d_seq_lens, const int32_t *d_start, void *d_k, int64_t k_stride, void *d_v,
                   int64_t v_stride, void *stream)
{
    const char *fn = "kv8_gather";
    if (int32_t rc = check_call(pool, layer, batch, fn, 8)) return rc;
    const ckv_config &c = pool->cfg;
    if (n_tokens < 0) return fail(CKV_EINVAL, "%s: n_tokens < 0", fn);
    if (!d_block_tables || !d_seq_lens) return fail(CKV_EINVAL, "%s: NULL argument", fn);
    if (!d_start && n_tokens % batch != 0)
        return fail(CKV_EINVAL, "%s: %d tokens do not split evenly over %d requests", fn, n_tokens, batch);
    if (n_tokens == 0) return CKV_OK;
    if (!d_k || !d_v) return fail(CKV_EINVAL, "%s: NULL argument", fn);
    const int64_t row = (int64_t)c.num_kv_heads * c.head_dim;
    if (int32_t rc = check_rows(fn, n_tokens, {{"k", d_k, k_stride, row}, {"v", d_v, v_stride, row}})) return rc;
    const ckv::NamedRows k_rows = {"k", {d_k, 2 * row, 2 * k_stride, n_tokens}}, v_rows = {"v", {d_v, 2 * row, 2 * v_stride, n_tokens}};
    const ckv::NamedRows tables = {"block_tables", whole(d_block_tables, 4ll * batch * c.max_pages_per_req)}, lens = {"seq_lens", whole(d_seq_lens, 4ll * batch)},
                         start = {"start", whole(d_start, 4ll * batch + 4)};
    if (int32_t rc = check_apart(fn, k_rows, {v_rows, tables, lens, start})) return rc;
    if (int32_t rc = check_apart(fn, v_rows, {tables, lens, start})) return rc;
    ckv::Gather8Params gp{};
    gp.records = layer_records(pool, layer);
    gp.steps = all_steps(pool) + layer * blocks_of(c);
    gp.start = d_start;
    gp.block_tables = d_block_tables;
    gp.seq_lens = d_seq_lens;
    gp.k = static_cast<uint16_t *>(d_k);
    gp.v = static_cast<uint16_t *>(d_v);
    gp.k_stride = k_stride;
    gp.v_stride = v_stride;
    gp.status = pool->wsp<uint32_t>(pool->ws.status);
    gp.batch = batch;
    gp.each = n_tokens / batch;
    gp.n_tokens = n_tokens;
    gp.max_pages_per_req = c.max_pages_per_req;
    gp.num_pages = c.num_pages;
    gp.num_kv_heads = c.num_kv_heads;
    gp.per_token_inv = ckv::inverse_of(2 * c.num_kv_heads);
    CKV_CUDA(enqueue(c.head_dim == 128 ? ckv::kv8_gather_kernel<128> : ckv::kv8_gather_kernel<64>, page_ctas(d_start, n_tokens, batch), 256, 0, pool->overlap, 0,
                     stream, gp));
    pool->launches += 1;
    return CKV_OK;
}

int32_t kv8_attention(ckv_pool *pool, int32_t layer, int32_t batch, int32_t q_len, const int32_t *d_block_tables, const int32_t *d_seq_lens,
                      const void *d_q, void *d_out, int32_t window, int32_t sink, void *stream)
{
    return cache_attention(pool, "kv8_attention", 8, layer, batch, q_len, d_block_tables, d_seq_lens, d_q, d_out, window, sink, stream);
}

int32_t decode_attention_window(ckv_pool *pool, int32_t layer, int32_t batch, int32_t q_len, const int32_t *d_block_tables,
                                const int32_t *d_seq_lens, const void *d_q, void *d_out, int32_t window, int32_t sink, void *stream)
{
    return cache_attention(pool, "decode_attention_window", 16, layer, batch, q_len, d_block_tables, d_seq_lens, d_q, d_out, window, sink, stream);
}

int32_t kv_pages_assign(ckv_pool *pool, int32_t batch, int32_t *d_block_tables, const int32_t *d_seq_lens, const int32_t *d_new_tokens,
                        const int32_t *d_free_pages, const int32_t *d_free_count, int32_t *d_lens_out, int32_t *d_count_out,
                        int32_t *d_step_lens, int32_t *d_new_start, int64_t *d_slots, int32_t n_slots, void *stream)
{
    ckv::TablesParams tp{};
    tp.block_tables = d_block_tables;
    tp.seq_lens = d_seq_lens;
    tp.amounts = d_new_tokens;
    tp.free_pages = const_cast<int32_t *>(d_free_pages);
    tp.free_count = d_free_count;
    tp.lens_out = d_lens_out;
    tp.count_out = d_count_out;
    tp.step_lens = d_step_lens;
    tp.new_start = d_new_start;
    tp.slots = reinterpret_cast<long long *>(d_slots);
    tp.n_slots = n_slots;
    return launch_pages<true>(pool, "kv_pages_assign", tp, batch, stream);
}

int32_t kv_pages_release(ckv_pool *pool, int32_t batch, const int32_t *d_block_tables, const int32_t *d_seq_lens, const int32_t *d_keep_lens,
                         int32_t *d_free_pages, const int32_t *d_free_count, int32_t *d_lens_out, int32_t *d_count_out, void *stream)
{
    ckv::TablesParams tp{};
    tp.block_tables = const_cast<int32_t *>(d_block_tables);
    tp.seq_lens = d_seq_lens;
    tp.amounts = d_keep_lens;
    tp.free_pages = d_free_pages;
    tp.free_count = d_free_count;
    tp.lens_out = d_lens_out;
    tp.count_out = d_count_out;
    return launch_pages<false>(pool, "kv_pages_release", tp, batch, stream);
}

int32_t logits_process(int32_t batch, int32_t rows, int32_t vocab, int32_t in_dtype, int32_t out_dtype, int32_t probs, const void *d_logits,
                       int64_t logits_stride, const float *d_params, const int32_t *d_history, int64_t history_stride, const int32_t *d_prompt_lens,
                       const int32_t *d_history_lens, const int32_t *d_drafts, const int32_t *d_bias_ids, const float *d_bias, int32_t n_bias,
                       const uint32_t *d_mask, int64_t mask_stride, void *d_out, int64_t out_stride, void *stream)
{
    const char *fn = "logits_process";
    if (batch < 1 || rows < 1 || (long long)batch * rows * 16 >= (1ll << 31)) return fail(CKV_EINVAL, "%s: batch %d or rows %d out of range", fn, batch, rows);
    if (vocab < 1 || vocab > ckv::kLogitsMaxVocab) return fail(CKV_EINVAL, "%s: vocab %d outside [1, %d]", fn, vocab, ckv::kLogitsMaxVocab);
    for (int32_t d : {in_dtype, out_dtype})
        if (d != CKV_PROBS_F32 && d != CKV_PROBS_BF16) return fail(CKV_EINVAL, "%s: unknown dtype %d", fn, d);
    if (!d_logits || !d_out) return fail(CKV_EINVAL, "%s: NULL argument", fn);
    if (d_history && (!d_prompt_lens || !d_history_lens || history_stride < 0))
        return fail(CKV_EINVAL, "%s: the history needs its lengths and a stride of at least 0", fn);
    if ((d_history || d_drafts) && !d_params) return fail(CKV_EINVAL, "%s: the history and the drafts are counted for penalties, and there are no params", fn);
    if (n_bias < 0 || (n_bias > 0 && (!d_bias_ids || !d_bias))) return fail(CKV_EINVAL, "%s: n_bias %d, or no biases", fn, n_bias);
    if (logits_stride < vocab || out_stride < vocab) return fail(CKV_EINVAL, "%s: a row's stride is below the vocabulary", fn);
    if (d_mask && mask_stride < (vocab + 31) / 32) return fail(CKV_EINVAL, "%s: the mask's stride is below the vocabulary's words", fn);
    const uintptr_t in_size = in_dtype == CKV_PROBS_F32 ? 4 : 2, out_size = out_dtype == CKV_PROBS_F32 ? 4 : 2;
    const uintptr_t in_at = reinterpret_cast<uintptr_t>(d_logits), out_at = reinterpret_cast<uintptr_t>(d_out);
    if (in_at % in_size != 0 || out_at % out_size != 0) return fail(CKV_EINVAL, "%s: logits or out not aligned to their type", fn);
    const long long n = (long long)batch * rows, words = (vocab + 31) / 32;
    const ckv::NamedRows out = {"out", {d_out, (long long)(vocab * out_size), (long long)(out_stride * out_size), n}};
    if (!(in_at == out_at && in_dtype == out_dtype && (n == 1 || logits_stride == out_stride)) &&
        overlap(out.rows, {d_logits, (long long)(vocab * in_size), (long long)(logits_stride * in_size), n}))
        return fail(CKV_EINVAL, "%s: out overlaps the logits without being them", fn);
    // what other blocks may still be reading
    if (int32_t rc = check_apart(fn, out, {{"params", whole(d_params, 16ll * batch)}, {"history", whole(d_history, 4ll * batch * history_stride)},
                                           {"prompt_lens", whole(d_history ? d_prompt_lens : nullptr, 4ll * batch)},
                                           {"history_lens", whole(d_history ? d_history_lens : nullptr, 4ll * batch)},
                                           {"drafts", whole(d_drafts, 4ll * batch * (rows - 1))}, {"bias_ids", whole(d_bias_ids, 4ll * batch * n_bias)},
                                           {"bias", whole(d_bias, 4ll * batch * n_bias)}, {"mask", {d_mask, 4 * words, 4 * mask_stride, n}}}))
        return rc;
    ckv::LogitsParams lp{};
    lp.logits = d_logits;
    lp.out = d_out;
    lp.stride = logits_stride;
    lp.out_stride = out_stride;
    lp.params = d_params;
    lp.history = history_stride > 0 ? d_history : nullptr;
    lp.prompt_lens = d_prompt_lens;
    lp.history_lens = d_history_lens;
    lp.drafts = rows > 1 ? d_drafts : nullptr;
    lp.bias_ids = n_bias > 0 ? d_bias_ids : nullptr;
    lp.bias = d_bias;
    lp.mask = d_mask;
    lp.history_stride = history_stride;
    lp.mask_stride = mask_stride;
    lp.rows = rows;
    lp.vocab = vocab;
    lp.n_bias = n_bias;
    lp.probs = probs;
    if (in_dtype == CKV_PROBS_F32)
        return out_dtype == CKV_PROBS_F32 ? launch_logits<float, float>(lp, batch, stream) : launch_logits<float, __nv_bfloat16>(lp, batch, stream);
    return out_dtype == CKV_PROBS_F32 ? launch_logits<__nv_bfloat16, float>(lp, batch, stream) : launch_logits<__nv_bfloat16, __nv_bfloat16>(lp, batch, stream);
}

}  // extern "C"
