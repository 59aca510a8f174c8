// Host side that every translation unit of the library shares: the last error's message, the handle
// and the checks that each call begins with.
#pragma once

#include "chiron_kv.h"

#include <cstdarg>
#include <cstdio>
#include <vector>

#include "ckv_common.cuh"

namespace ckv {

inline thread_local char g_error[512] = "";

inline int32_t fail(int32_t code, const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_error, sizeof g_error, fmt, ap);
    va_end(ap);
    return code;
}

#define CKV_CUDA(call)                                                                        \
    do {                                                                                      \
        cudaError_t e_ = (call);                                                              \
        if (e_ != cudaSuccess)                                                                \
            return ckv::fail(CKV_ECUDA, "%s failed: %s (%s:%d)", #call, cudaGetErrorString(e_),    \
                        __FILE__, __LINE__);                                                  \
    } while (0)

// Scores that one selection may hold: every page of every table, up to this many.
constexpr long long kMaxSelectKeys = 64ll << 20;

// Scores of a (request, kv head), the number rounded up for 16-byte loads.
inline int32_t key_stride(const ckv_config &c) { return (c.max_pages_per_req + 3) & ~3; }

struct WorkspaceLayout {
    size_t status, header, span_start, part, arrivals, trace;
    size_t st_tables, st_lens, st_q, st_k, st_v, st_out;
    size_t total;
};

}  // namespace ckv

struct ckv_pool {
    ckv_config cfg;
    int device;
    int num_sms;
    int num_spans;                   // partition width: one span per warp of the attention kernel
    uint8_t *d_pool;
    uint8_t *d_ws;
    ckv::WorkspaceLayout ws;
    CUtensorMap tmap;
    int64_t launches;
    bool profile;
    bool overlap;                    // launch kernels with programmatic stream serialization
    bool pool_written;               // a kernel other than the fused step wrote the pool since the last attention launch
    bool inputs_from_predecessor;    // the next attention launch reads tables and lengths its predecessor in the stream writes
    int host_route;                  // decode_step_host: CKV_HOST_ROUTE_*
    uint32_t *d_scores;              // ckv_set_select_scratch: room for `score_room` scores of a page selection
    long long score_room;
    std::vector<cudaEvent_t> ev;     // pairs (start, stop)
    int ev_used;

    template <typename T> T *wsp(size_t off) const { return reinterpret_cast<T *>(d_ws + off); }
};

namespace ckv {

inline int32_t check_device(const ckv_pool *pool, const char *fn)
{
    if (!pool) return fail(CKV_EINVAL, "%s: pool is NULL", fn);
    int current = -1;
    if (cudaGetDevice(&current) != cudaSuccess || current != pool->device)
        return fail(CKV_EINVAL, "%s: the pool lives on device %d but device %d is current", fn, pool->device, current);
    return CKV_OK;
}

inline int32_t check_call(ckv_pool *pool, int32_t layer, int32_t batch, const char *fn)
{
    if (int32_t rc = check_device(pool, fn)) return rc;
    if (layer < 0 || layer >= pool->cfg.num_layers)
        return fail(CKV_EINVAL, "%s: layer %d outside [0, %d)", fn, layer, pool->cfg.num_layers);
    if (batch < 1 || batch > pool->cfg.max_batch)
        return fail(CKV_EINVAL, "%s: batch %d outside [1, %d]", fn, batch, pool->cfg.max_batch);
    return CKV_OK;
}

// Pages of a list; their tokens have to be countable in 32 bits.
inline int32_t check_budget(int32_t budget, const char *fn)
{
    if (budget < 1 || budget > 1 << 26) return fail(CKV_EINVAL, "%s: budget %d outside [1, 2^26]", fn, budget);
    return CKV_OK;
}

constexpr int kMaxListInKernel = 2048;           // pages of a list that the attention kernel selects itself

// Checks and launches of decode_select_pages (ckv_ops.cu), for it and for decode_attention_sparse.  `attend`: the
// attention kernel follows and may be left the whole selection; *selected says whether it was done.
struct SelectParams;
int32_t select_launch(ckv_pool *pool, const char *fn, int32_t layer, int32_t batch, const int32_t *d_block_tables,
                      const int32_t *d_seq_lens, const void *d_q, const void *d_index, size_t index_bytes,
                      int32_t budget, int32_t sink, int32_t recent, int32_t *d_pages, int32_t *d_lens, bool attend,
                      SelectParams *out_params, bool *selected, void *stream);

// Whether two arrays of 32-bit entries share memory (NULL: no).
inline bool overlap(const void *a, long long na, const void *b, long long nb)
{
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x && y && x < y + (uintptr_t)nb * 4 && y < x + (uintptr_t)na * 4;
}

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace ckv
