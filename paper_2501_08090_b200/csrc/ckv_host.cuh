// Host side that every translation unit of the library shares: the last error's message, the handle
// and the checks that each call begins with.
#pragma once

#include "chiron_kv.h"

#include <algorithm>
#include <cstdarg>
#include <cstdio>
#include <initializer_list>
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
    size_t cuts;
    size_t total;
};

}  // namespace ckv

struct ckv_pool {
    ckv_config cfg;
    int bits;                        // a cached element's: 16, or 8 (kv8_pool_create)
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

// The handle's cache must be of the type that the call reads or writes.
inline int32_t check_bits(const ckv_pool *pool, int bits, const char *fn)
{
    if (pool->bits != bits) return fail(CKV_EINVAL, "%s: the handle holds a cache of %d bits an element, the call is for %d", fn, pool->bits, bits);
    return CKV_OK;
}

inline int32_t check_call(ckv_pool *pool, int32_t layer, int32_t batch, const char *fn, int bits = 16)
{
    if (int32_t rc = check_device(pool, fn)) return rc;
    if (int32_t rc = check_bits(pool, bits, fn)) return rc;
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

// `n` rows of `row` bytes, `stride` >= row bytes apart where there are several.  NULL: none.
struct ByteRows {
    const void *ptr;
    long long row, stride, n;
};

// Whether a row of one shares a byte with a row of the other: rows of one may lie between the other's.
inline bool overlap(const ByteRows &a, const ByteRows &b)
{
    if (!a.ptr || !b.ptr || a.n < 1 || b.n < 1 || a.row < 1 || b.row < 1) return false;
    const long long at_a = (long long)reinterpret_cast<uintptr_t>(a.ptr), at_b = (long long)reinterpret_cast<uintptr_t>(b.ptr);
    const long long step_a = a.n > 1 ? a.stride : a.row, step_b = b.n > 1 ? b.stride : b.row;
    if (at_a + (a.n - 1) * step_a + a.row <= at_b || at_b + (b.n - 1) * step_b + b.row <= at_a) return false;
    if (a.n > 1 && b.n > 1 && step_a == step_b) {
        // row j of b begins at_b - at_a + (j - i) step behind row i of a: the least difference of rows that lets it begin above -b.row
        const long long d = at_b - at_a, x = -b.row - d;
        const long long k = std::max((x >= 0 ? x / step_a : -((-x + step_a - 1) / step_a)) + 1, 1 - a.n);
        return k <= b.n - 1 && d + k * step_a < a.row;
    }
    // in order of address, from the first row that does not end before the other's begin
    long long i = std::max(0ll, (at_b - at_a - a.row) / step_a), j = std::max(0ll, (at_a - at_b - b.row) / step_b);
    while (i < a.n && j < b.n) {
        const long long p = at_a + i * step_a, q = at_b + j * step_b;
        if (p + a.row <= q) ++i;
        else if (q + b.row <= p) ++j;
        else return true;
    }
    return false;
}

// Memory that a call writes, against what it reads or writes elsewhere.
struct NamedRows {
    const char *name;
    ByteRows rows;
};

inline int32_t check_apart(const char *fn, const NamedRows &written, std::initializer_list<NamedRows> others)
{
    for (const NamedRows &x : others)
        if (overlap(written.rows, x.rows)) return fail(CKV_EINVAL, "%s: %s overlaps %s", fn, written.name, x.name);
    return CKV_OK;
}

inline ByteRows whole(const void *p, long long bytes) { return {p, bytes, bytes, 1}; }

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Enqueue a kernel; `overlap`: its prologue may run under its predecessor's tail; `cluster`: CTAs of a cluster.
template <typename... P, typename... A>
cudaError_t enqueue(void (*kernel)(P...), unsigned blocks, unsigned threads, size_t smem, bool overlap, unsigned cluster, void *stream,
                    const A &...args)
{
    cudaLaunchConfig_t lc{};
    lc.gridDim = dim3(blocks);
    lc.blockDim = dim3(threads);
    lc.dynamicSmemBytes = smem;
    lc.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = overlap ? 1 : 0;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    lc.attrs = attr;
    lc.numAttrs = cluster > 0 ? 2 : 1;
    return cudaLaunchKernelEx(&lc, kernel, args...);
}

// More than 8 CTAs in a cluster and more than 48 KB of shared memory have to be allowed once per
// kernel and device.
template <typename Kernel>
cudaError_t allow(Kernel kernel, bool wide_cluster, size_t smem)
{
    cudaError_t e = cudaSuccess;
    if (wide_cluster) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e == cudaSuccess && smem > 0) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    return e;
}

// How many clusters of this size the GPU holds at a time: less than its CTAs' number says, since a cluster stays within a part
// of the GPU.
template <typename Kernel>
cudaError_t resident_clusters(Kernel kernel, unsigned threads, size_t smem, unsigned cluster, int *clusters)
{
    cudaLaunchConfig_t lc{};
    lc.gridDim = dim3(cluster);
    lc.blockDim = dim3(threads);
    lc.dynamicSmemBytes = smem;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = cluster;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    lc.attrs = &attr;
    lc.numAttrs = 1;
    return cudaOccupancyMaxActiveClusters(clusters, kernel, &lc);
}

// The handle of kv_pool_create and kv8_pool_create (ckv_api.cu).
int32_t create_pool(const char *fn, const ckv_config *cfg, int bits, void *d_pool, size_t pool_bytes, void *d_workspace,
                    size_t workspace_bytes, int32_t device, ckv_pool **out_pool);

}  // namespace ckv
