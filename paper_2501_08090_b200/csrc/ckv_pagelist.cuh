// Attention over a list of pages per (request, kv head): what a page selection is followed by.
#pragma once

#include "ckv_common.cuh"
#include "ckv_sparse.cuh"

namespace ckv {

// A cluster of CTAs per (request, kv head), a tile of 32 tokens (2 pages) per warp and turn, each warp with a
// stage of its own that it fills by TMA.  The arithmetic of a tile is paged_decode_attn_kernel's:
//   S^T[tok 16 x g 8] = K[tok 16 x d] . Q^T[d x g 8],   O^T[d 16 x g 8] += V^T[d 16 x tok 16] . P^T[tok 16 x g 8]
// on mma.sync with the softmax in the log2 domain.  That kernel cuts the tokens of all requests into even
// spans, since contexts differ a thousandfold, and its spans' partials meet in global memory: publish,
// fence, count, fetch, fold, 4 to 8 us.  Lists of a selection are of one length, or shorter, so here a CTA or
// cluster owns a pair and its partials never leave the SMs: they are folded in the CTA's shared memory, a
// warp per column, then across the cluster through distributed shared memory, a CTA per column, in a
// fixed order.
//
//   M = max m_i,  out = sum_i 2^(m_i - M) O_i / sum_i 2^(m_i - M) l_i   over warps, then over CTAs.
//
// Weights are rounded to bf16 for P V, as in paged_decode_attn_kernel (the matrix instruction takes one type, and V is
// bf16), and summed unrounded in fp32: 2^-8 of each weight at most, which averages out over the tokens.  Against 64 bits
// the outputs are off by 1.9e-3 of their size (root of squares) where fp32 weights leave 1.7e-3, the output's own
// rounding.
//
// Bound by HBM where the pairs fill the GPU (512 pairs of 128 pages 80.8 us against 87 in even spans; 768
// of 33 pages 37.8 against 44), by latency where they do not (5 pairs of 24 pages 3.8 us against 8.8).
// Six warps and two CTAs an SM: 296 CTAs at a time.  Of the same 12 warps an SM, 4 x 3 leave 512 pairs a second
// wave that is nearly empty (95 us), 2 x 6 too (91), 12 x 1 folds while nothing is loaded (88).
struct ListParams {
    const int32_t *pages;           // [batch][Hkv][budget]
    const int32_t *lens;            // [batch] tokens in the lists, or (context_pages > 0) of the contexts they were chosen from
    const uint16_t *q;
    uint16_t *out;
    uint32_t *status;
    int32_t batch, budget, num_pages, num_kv_heads, group;
    int32_t layer_page_base;        // layer * num_pages
    int32_t context_pages;          // > 0: a selection over tables of this many pages wrote the lists just before
    float scale_log2;               // log2(e) / sqrt(d)
};

template <int D>
struct ListLayout {
    static constexpr int kWarps = 6;
    static constexpr int kCtas = 2;              // resident on an SM
    static constexpr int kHalves = D / 64;
    static constexpr int kHalfBytes = 32 * 128;                  // one TMA box: 32 rows x 128 B
    static constexpr int kPageBytes = kHalves * kHalfBytes;
    static constexpr int kStageBytes = kPagesPerTile * kPageBytes;
    static constexpr int kPitch = D + 4;                         // floats per row of a partial (bank spread)
    static constexpr int kPartFloats = kMaxGroup * kPitch + 2 * kMaxGroup;       // rows, then m[8], l[8]
    // a warp's partial takes its stage's place once its last tile is done; the CTA's lies in warp 0's second half
    static constexpr int kCtaPartOff = kStageBytes / 2;
    static_assert(kPartFloats * 4 <= kStageBytes / 2, "two partials must fit a stage");
    static constexpr int kBarOff = kWarps * kStageBytes;
    static constexpr int kListOff = kBarOff + kWarps * 8;        // the list, where this kernel selects it
    static constexpr int kSmemBytes = kListOff + 1024;           // and the list
    // a selection's scratch lies where the stages will be
    static constexpr int kHistOff = 16384, kRangeOff = kHistOff + kSelectRounds * kSelectBins * 4;
    static_assert(kRangeOff + 3 * 32 * 4 <= kWarps * kStageBytes, "a selection's scratch must fit the stages");
};

__device__ __forceinline__ float4 ld_cluster_f32x4(uint32_t addr)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr));
    return v;
}

__device__ __forceinline__ float ld_cluster_f32(uint32_t addr)
{
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr));
    return v;
}

// kSelect: the lists are not there yet.  Every CTA of a cluster scores and selects its pair's pages for
// itself (few short tables: kListSelectPages), and the first one writes the list out: one launch in
// place of three.  One launch against three, device time: 8 pairs of 64 pages, 24 kept, 8.1 us against 10.7; 8 of 256
// pages 9.9 against 10.9; 128 of 64 pages 11.9 against 16.8; 128 of 256 pages 14.1 against 17.4, with 128 kept 30.8
// against 33.6 (head_dim 128); 5 of 256 pages 8.4 against 9.6 (64).  A launch is 2.4 us of the caller's time besides.
// (Selecting here behind score_pages_kernel, for any table, was slower than select_pages_kernel: 768 pairs 73 us in
// all against 70, since two CTAs an SM select while nothing is loaded.)
constexpr int kListSelectKeys = 4;               // a thread
constexpr int kListSelectPages = 256, kListSelectPairs = 128;
template <int D, bool kSelect>
__global__ void __launch_bounds__(ListLayout<D>::kWarps * 32, ListLayout<D>::kCtas)
page_list_attn_kernel(const __grid_constant__ CUtensorMap tmap, const ListParams p, const __grid_constant__ SelectParams sp)
{
    using Lay = ListLayout<D>;
    constexpr int W = Lay::kWarps, kKSteps = D / 16, kDTiles = D / 16;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)cluster_rank(), ctas = (int)cluster_size();
    const int pair = blockIdx.x / ctas, r = pair / p.num_kv_heads, h = pair % p.num_kv_heads;
    const int G = p.group;
    const uint32_t stage = smem_u32(smem) + warp * Lay::kStageBytes, bar = smem_u32(smem + Lay::kBarOff) + warp * 8;
    float *part = (float *)(smem + warp * Lay::kStageBytes);
    if (lane == 0) {
        prefetch_tensormap(&tmap);
        mbar_init(bar, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_proxy_async();
    }
    __syncwarp();
    const int heads = p.num_kv_heads * G;
    uint16_t *out_rows = p.out + ((size_t)r * heads + h * G) * D;
    uint32_t qf[kKSteps][2];
    auto load_q = [&]() {
        const int c = lane >> 2;
        const uint32_t *qrow = (const uint32_t *)(p.q + ((size_t)r * heads + h * G + c) * D);
#pragma unroll
        for (int ks = 0; ks < kKSteps; ++ks) {
            qf[ks][0] = c < G ? __ldg(qrow + ks * 8 + (lane & 3)) : 0u;
            qf[ks][1] = c < G ? __ldg(qrow + ks * 8 + 4 + (lane & 3)) : 0u;
        }
    };
    // Right behind a selection, lengths and queries may be read before the wait: that kernel released this
    // one after its own wait, so whatever wrote them has completed; the lists' length follows from the
    // context's.
    if (kSelect || p.context_pages == 0) grid_dependency_wait();
    load_q();
    const int len = __ldg(p.lens + r);
    const int L = p.context_pages > 0 ? attended_length(len, p.context_pages, p.budget) : len;
    const int tiles = tiles_of_length(L, p.budget);
    int32_t *s_list = (int32_t *)(smem + Lay::kListOff);
    if constexpr (kSelect) {
        int32_t *out = sp.sel_tables + (size_t)pair * sp.budget;
        const SelectScratch scratch = {(uint32_t *)smem, (int (*)[kSelectBins])(smem + Lay::kHistOff), (uint32_t (*)[32])(smem + Lay::kRangeOff)};
        select_pair<kListSelectKeys, D>(sp, pair, scratch, rank == 0, [&](int place, int32_t id) {
            s_list[place] = id;
            if (rank == 0) out[place] = id;
        });
        fence_proxy_async();                     // the scratch was written here, the stages are filled by the copy engine
        __syncthreads();
    } else {
        grid_dependency_wait();
        grid_launch_dependents();
    }
    if (tiles == 0) {                            // unusable: the same for the whole cluster
        if (rank == 0) {
            for (int i = threadIdx.x; i < G * D / 8; i += W * 32) ((uint4 *)out_rows)[i] = make_uint4(0u, 0u, 0u, 0u);
            if (!kSelect && threadIdx.x == 0) atomicOr(p.status, kStatusBadLength);
        }
        return;
    }

    const int32_t *list = p.pages + (size_t)pair * p.budget;
    const uint64_t policy = l2_evict_first_policy();
    auto tokens_of = [&](int tile) { return min(kTileTokens, L - tile * kTileTokens); };
    auto issue = [&](int tile) {
        const int np = (tokens_of(tile) + kPageSize - 1) / kPageSize;
        if (lane == 0) mbar_arrive_expect_tx(bar, np * Lay::kPageBytes);
        __syncwarp();
        if (lane < np * Lay::kHalves) {
            const int pg = lane / Lay::kHalves, hf = lane % Lay::kHalves;
            int page = kSelect ? s_list[tile * kPagesPerTile + pg] : __ldg(list + tile * kPagesPerTile + pg);
            if (page < 0 || page >= p.num_pages) {
                atomicOr(p.status, kStatusBadPage);
                page = 0;
            }
            const int y = ((p.layer_page_base + page) * p.num_kv_heads + h) * 32;
            tma_load_2d(stage + pg * Lay::kPageBytes + hf * Lay::kHalfBytes, &tmap, hf * 64, y, bar, policy);
        }
    };
    const int step = ctas * W;
    int tile = rank * W + warp;
    if (tile < tiles) issue(tile);

    const int g0 = (lane & 3) * 2;               // first of the two columns this lane accumulates
    uint32_t k_off[4], v_off[4];                 // ldmatrix lane offsets inside one page block
    {
        const int krow = (lane & 7) + ((lane >> 3) & 1) * 8, ksel = lane >> 4;
        const int vrow = 16 + (lane & 7) + (lane >> 4) * 8, vsel = (lane >> 3) & 1;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            k_off[j] = krow * 128 + (((j * 2 + ksel) ^ (lane & 7)) << 4);
            v_off[j] = vrow * 128 + (((j * 2 + vsel) ^ (lane & 7)) << 4);
        }
    }
    float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
    float o[kDTiles][4];
#pragma unroll
    for (int dt = 0; dt < kDTiles; ++dt) o[dt][0] = o[dt][1] = o[dt][2] = o[dt][3] = 0.f;
    bool alive = true;
    uint32_t phase = 0;
#pragma unroll 1
    for (; tile < tiles && alive; tile += step, phase ^= 1u) {
        alive = __all_sync(0xffffffffu, mbar_wait_bounded(bar, phase, p.status));
        if (!alive) break;
        const int ntok = tokens_of(tile), np = (ntok + kPageSize - 1) / kPageSize;
        if (ntok & (kPageSize - 1)) {
            // value rows past the context's end may hold anything; their weights are zero, 0 * NaN is not
            const int row0 = ntok - (np - 1) * kPageSize, pieces = (kPageSize - row0) * 8 * Lay::kHalves;
            for (int i = lane; i < pieces; i += 32) {
                const int hf = i / ((kPageSize - row0) * 8), rem = i % ((kPageSize - row0) * 8);
                const uint32_t at = stage + (np - 1) * Lay::kPageBytes + hf * Lay::kHalfBytes + (16 + row0 + rem / 8) * 128 + (rem % 8) * 16;
                asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" ::"r"(at), "r"(0u) : "memory");
            }
            fence_proxy_async();                  // these writes precede the stage's next fill
            __syncwarp();
        }
        float s[kPagesPerTile][4];
#pragma unroll
        for (int mt = 0; mt < kPagesPerTile; ++mt) s[mt][0] = s[mt][1] = s[mt][2] = s[mt][3] = 0.f;
#pragma unroll
        for (int ks = 0; ks < kKSteps; ++ks) {
#pragma unroll
            for (int mt = 0; mt < kPagesPerTile; ++mt) {
                if (mt < np) {
                    uint32_t a[4];
                    ldmatrix_x4(a, stage + mt * Lay::kPageBytes + (ks / 4) * Lay::kHalfBytes + k_off[ks % 4]);
                    mma_bf16_16816(s[mt], a, qf[ks][0], qf[ks][1]);
                }
            }
        }
        float mx0 = -INFINITY, mx1 = -INFINITY;
#pragma unroll
        for (int mt = 0; mt < kPagesPerTile; ++mt) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (mt * kPageSize + (lane >> 2) + (i >= 2 ? 8 : 0) >= ntok) s[mt][i] = -INFINITY;      // selected, never multiplied
            mx0 = fmaxf(mx0, fmaxf(s[mt][0], s[mt][2]));
            mx1 = fmaxf(mx1, fmaxf(s[mt][1], s[mt][3]));
        }
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) {
            mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, x));
            mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, x));
        }
        const float mn0 = fmaxf(m0, mx0 * p.scale_log2), mn1 = fmaxf(m1, mx1 * p.scale_log2);
        // so far only scores of -inf (infinite keys): exponentials are taken against 0 and come out 0
        const float ref0 = mn0 == -INFINITY ? 0.f : mn0, ref1 = mn1 == -INFINITY ? 0.f : mn1;
        const float al0 = fast_exp2(m0 - ref0), al1 = fast_exp2(m1 - ref1);
        m0 = mn0; m1 = mn1;
        l0 *= al0; l1 *= al1;
#pragma unroll
        for (int dt = 0; dt < kDTiles; ++dt) { o[dt][0] *= al0; o[dt][2] *= al0; o[dt][1] *= al1; o[dt][3] *= al1; }
        uint32_t pb[kPagesPerTile][2];
#pragma unroll
        for (int mt = 0; mt < kPagesPerTile; ++mt) {
            const float p0 = fast_exp2(fmaf(s[mt][0], p.scale_log2, -ref0)), p1 = fast_exp2(fmaf(s[mt][1], p.scale_log2, -ref1));
            const float p2 = fast_exp2(fmaf(s[mt][2], p.scale_log2, -ref0)), p3 = fast_exp2(fmaf(s[mt][3], p.scale_log2, -ref1));
            l0 += p0 + p2;
            l1 += p1 + p3;
            pb[mt][0] = movmatrix_trans(pack_bf16x2(p0, p1));
            pb[mt][1] = movmatrix_trans(pack_bf16x2(p2, p3));
        }
#pragma unroll
        for (int dt = 0; dt < kDTiles; ++dt) {
#pragma unroll
            for (int mt = 0; mt < kPagesPerTile; ++mt) {
                if (mt < np) {
                    uint32_t a[4];
                    ldmatrix_x4_trans(a, stage + mt * Lay::kPageBytes + (dt / 4) * Lay::kHalfBytes + v_off[dt % 4]);
                    mma_bf16_16816(o[dt], a, pb[mt][0], pb[mt][1]);
                }
            }
        }
        if (tile + step < tiles) issue(tile + step);              // the stage's reads have been consumed
    }

    // Do not go on while a copy into this warp's stage may still be in flight (only after a wait gave up).
    if (!alive) mbar_wait_bounded(bar, phase, p.status);

    __syncwarp();
    // ---- this warp's partial (m = -inf, l = 0 if it had no tile)
#pragma unroll
    for (int x = 4; x < 32; x <<= 1) {
        l0 += __shfl_xor_sync(0xffffffffu, l0, x);
        l1 += __shfl_xor_sync(0xffffffffu, l1, x);
    }
#pragma unroll
    for (int dt = 0; dt < kDTiles; ++dt) {
        const int d = dt * 16 + (lane >> 2);
        part[g0 * Lay::kPitch + d] = o[dt][0];
        part[(g0 + 1) * Lay::kPitch + d] = o[dt][1];
        part[g0 * Lay::kPitch + d + 8] = o[dt][2];
        part[(g0 + 1) * Lay::kPitch + d + 8] = o[dt][3];
    }
    if (lane < 4) {
        float *ml = part + kMaxGroup * Lay::kPitch;
        ml[g0] = m0; ml[g0 + 1] = m1;
        ml[kMaxGroup + g0] = l0; ml[kMaxGroup + g0 + 1] = l1;
    }
    __syncthreads();

    // ---- the CTA's fold: warp g takes column g, its lanes four elements of the row each
    constexpr int kPartStride = Lay::kStageBytes / 4;
    const float *parts = (const float *)smem;
    float *mine = (float *)(smem + Lay::kCtaPartOff);
    auto store = [&](int g, float4 acc, float l) {
        const float inv = 1.f / l;
        uint2 packed;
        packed.x = pack_bf16x2(acc.x * inv, acc.y * inv);
        packed.y = pack_bf16x2(acc.z * inv, acc.w * inv);
        *(uint2 *)(out_rows + g * D + lane * 4) = packed;
    };
    for (int g = warp; g < G; g += W) {
        float M = -INFINITY, l = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < W; ++w) M = fmaxf(M, parts[w * kPartStride + kMaxGroup * Lay::kPitch + g]);
        const float ref = M == -INFINITY ? 0.f : M;              // no warp of this CTA had a tile, or only scores of -inf
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float *src = parts + w * kPartStride;
            const float f = fast_exp2(src[kMaxGroup * Lay::kPitch + g] - ref);
            l += f * src[kMaxGroup * Lay::kPitch + kMaxGroup + g];
            if (lane * 4 < D) {
                const float4 a = *(const float4 *)(src + g * Lay::kPitch + lane * 4);
                acc.x += f * a.x; acc.y += f * a.y; acc.z += f * a.z; acc.w += f * a.w;
            }
        }
        if (ctas == 1) {
            if (lane * 4 < D && alive) store(g, acc, l);
        } else {
            if (lane * 4 < D) *(float4 *)(mine + g * Lay::kPitch + lane * 4) = acc;
            if (lane == 0) { mine[kMaxGroup * Lay::kPitch + g] = M; mine[kMaxGroup * Lay::kPitch + kMaxGroup + g] = l; }
        }
    }
    if (ctas == 1) return;
    cluster_barrier();
    // ---- the cluster's fold: CTA c takes columns c, c + ctas, ...
    for (int g = rank + warp * ctas; g < G; g += W * ctas) {
        const uint32_t row = smem_u32(mine) + (g * Lay::kPitch + lane * 4) * 4, ml = smem_u32(mine) + (kMaxGroup * Lay::kPitch + g) * 4;
        float M = -INFINITY, l = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int c = 0; c < ctas; ++c) M = fmaxf(M, ld_cluster_f32(cluster_map(ml, c)));
        const float ref = M == -INFINITY ? 0.f : M;              // only scores of -inf (0 / 0 below), or a wait gave up everywhere
        for (int c = 0; c < ctas; ++c) {
            const float f = fast_exp2(ld_cluster_f32(cluster_map(ml, c)) - ref);
            l += f * ld_cluster_f32(cluster_map(ml + 4 * kMaxGroup, c));
            if (lane * 4 < D) {
                const float4 a = ld_cluster_f32x4(cluster_map(row, c));
                acc.x += f * a.x; acc.y += f * a.y; acc.z += f * a.z; acc.w += f * a.w;
            }
        }
        if (lane * 4 < D) store(g, acc, l);
    }
    cluster_barrier();                            // nobody leaves while others read its partial
}

}  // namespace ckv
