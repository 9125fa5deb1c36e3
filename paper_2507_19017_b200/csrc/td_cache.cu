// Host side of the paged key-value cache (include/td.h): argument checks and launches.
// Nothing is allocated and nothing synchronises.
#include <algorithm>
#include <atomic>
#include <cmath>

#include "td_attend.cuh"
#include "td_cache.cuh"
#include "td_host.cuh"
#include "td_range.h"

using namespace td;

namespace {

constexpr uint32_t kMaxSeqs = 1u << 24, kMaxRows = 1u << 24, kMaxDim = 256;

bool cache_sizes_ok(uint32_t n_pages, uint32_t max_seqs) { return n_pages < kIndexLimit && max_seqs < kMaxSeqs; }

struct CacheLayout {
    size_t tile_pages, tile_need, tile_add, need_before, add_before, first, tokens, given, from, to, rank, moves, total;
};
CacheLayout cache_layout(uint32_t n_pages, uint32_t max_seqs) {
    CacheLayout L{};
    size_t p = 0;
    auto take = [&](size_t bytes) { const size_t at = p; p = round_up(p + bytes, 256); return at; };
    L.tile_pages = take(kMaxTiles * 4);
    L.tile_need = take(kMaxTiles * 8);
    L.tile_add = take(kMaxTiles * 8);
    L.moves = take(8);
    L.need_before = take((size_t)max_seqs * 8);
    L.add_before = take((size_t)max_seqs * 4);
    L.first = take((size_t)max_seqs * 4);
    L.tokens = take((size_t)max_seqs * 4);
    L.given = take((size_t)max_seqs * 4);
    L.from = take((size_t)n_pages * 4);
    L.to = take((size_t)n_pages * 4);
    L.rank = take((size_t)n_pages * 4);
    L.total = p;
    return L;
}
CacheScratch scratch_of(const td_cache *c) {
    const CacheLayout L = cache_layout(c->n_pages, c->max_seqs);
    uint8_t *ws = static_cast<uint8_t *>(c->workspace);
    auto u32 = [&](size_t at) { return reinterpret_cast<uint32_t *>(ws + at); };
    auto u64 = [&](size_t at) { return reinterpret_cast<unsigned long long *>(ws + at); };
    CacheScratch w{};
    w.tile_pages = u32(L.tile_pages);
    w.tile_need = u64(L.tile_need);
    w.tile_add = u64(L.tile_add);
    w.moves = u32(L.moves);
    w.need_before = u64(L.need_before);
    w.add_before = u32(L.add_before);
    w.first = u32(L.first);
    w.tokens = reinterpret_cast<int32_t *>(ws + L.tokens);
    w.given = reinterpret_cast<int32_t *>(ws + L.given);
    w.from = u32(L.from);
    w.to = u32(L.to);
    w.rank = u32(L.rank);
    const uint32_t page_units = (c->n_pages + kPageStep - 1) / kPageStep, seq_units = (c->max_seqs + kSeqStep - 1) / kSeqStep;
    w.page_steps = std::max(1u, (page_units + kMaxTiles - 1) / kMaxTiles);
    w.seq_steps = std::max(1u, (seq_units + kMaxTiles - 1) / kMaxTiles);
    w.page_tiles = (page_units + w.page_steps - 1) / w.page_steps;
    w.seq_tiles = (seq_units + w.seq_steps - 1) / w.seq_steps;
    return w;
}

// Everything but the workspace.  need_pool: the call reads or writes keys and values.
int check_cache(const td_cache *c, bool need_pool) {
    if (!c || !float_type(c->dtype) || c->page_size == 0 || c->page_size >= (1u << 16)) return TD_EINVAL;
    if (!cache_sizes_ok(c->n_pages, c->max_seqs) || (uint64_t)c->n_pages * c->page_size >= (1ull << 40)) return TD_EINVAL;
    if ((uint64_t)c->max_pages * c->page_size >= kIndexLimit) return TD_EINVAL;
    if (!aligned(c->table, 4) || !aligned(c->length, 4) || !aligned(c->holders, 4) || !aligned(c->status, 4)) return TD_EINVAL;
    if ((c->max_seqs && !c->length) || (c->max_seqs && c->max_pages && !c->table) || (c->n_pages && !c->holders)) return TD_EINVAL;
    if ((c->keys == nullptr) != (c->values == nullptr)) return TD_EINVAL;
    if (!c->keys) return need_pool && c->n_pages ? TD_EINVAL : TD_OK;
    if (c->n_layers == 0 || c->n_layers >= (1u << 16) || c->n_heads == 0 || c->n_heads >= (1u << 16) || c->dim == 0 || c->dim >= (1u << 16)) return TD_EINVAL;
    if ((uint64_t)c->page_size * c->n_heads * c->dim >= kIndexLimit) return TD_EINVAL;
    if (c->layer_stride < 0 || c->page_stride < 0 || c->token_stride < 0 || c->head_stride < 0) return TD_EINVAL;
    const uint32_t es = size_of(c->dtype);
    if (!aligned(c->keys, es) || !aligned(c->values, es)) return TD_EINVAL;
    return TD_OK;
}
int check_workspace(const td_cache *c) {
    if (!c->workspace || !aligned(c->workspace, 256) || c->workspace_bytes < cache_layout(c->n_pages, c->max_seqs).total) return TD_EWORKSPACE;
    return TD_OK;
}
CacheView cache_view(const td_cache *c) {
    return CacheView{c->table, c->length, c->holders, c->status, c->n_pages, c->page_size, c->max_seqs, c->max_pages, make_fastdiv(c->page_size)};
}

// Bytes of the widest vector (16, 4 or 2) that every row of dim elements is made of whole ones of.
uint32_t vector_bytes(const td_cache *c, const void *a, const void *b, int64_t stride_a, int64_t stride_b) {
    const int64_t es = size_of(c->dtype);
    for (uint32_t v : {16u, 4u}) {
        bool ok = aligned(c->keys, v) && aligned(c->values, v) && aligned(a, v) && aligned(b, v);
        for (int64_t n : {(int64_t)c->dim, c->layer_stride, c->page_stride, c->token_stride, c->head_stride, stride_a, stride_b}) ok = ok && n * es % v == 0;
        if (ok) return v;
    }
    return 2;
}
PoolView pool_view(const td_cache *c, uint32_t vec) {
    const int64_t es = size_of(c->dtype);
    PoolView p{};
    p.keys = static_cast<uint8_t *>(c->keys);
    p.values = static_cast<uint8_t *>(c->values);
    p.layer = c->layer_stride * es;
    p.page = c->page_stride * es;
    p.token = c->token_stride * es;
    p.head = c->head_stride * es;
    p.layers = c->n_layers;
    p.heads = c->n_heads;
    p.vecs = (uint32_t)(c->dim * es / vec);
    p.heads_first = c->head_stride <= c->token_stride;
    p.by_vecs = make_fastdiv(p.vecs);
    p.by_heads = make_fastdiv(p.heads);
    return p;
}

// Runs of `dim` elements, outer x inner of them at these strides, none of which overlap.
bool apart(uint32_t rows, int64_t row, uint32_t heads, int64_t head, int64_t dim) {
    if (row < 0 || head < 0) return false;
    const bool rows_apart = rows == 1 || row >= (heads - 1) * head + dim, heads_inside = heads == 1 || head >= dim;
    const bool heads_apart = heads == 1 || head >= (rows - 1) * row + dim, rows_inside = rows == 1 || row >= dim;
    return (rows_apart && heads_inside) || (heads_apart && rows_inside);
}

constexpr uint32_t kWarps = kCacheThreads / 32;
uint32_t warp_blocks(uint32_t n) { return (n + kWarps - 1) / kWarps; }

int result(cudaError_t rc) { return rc == cudaSuccess ? TD_OK : rc == cudaErrorInvalidValue ? TD_EINVAL : TD_ECUDA; }

template <Give kGive>
cudaError_t run_give(const CacheView &v, const CacheScratch &w, const int32_t *ask, int32_t *cu, uint32_t sharing, cudaStream_t st) {
    const uint32_t tiles = w.page_tiles + w.seq_tiles;
    const cudaError_t rc = launch(cache_count_kernel<kGive>, tiles, kCacheThreads, st, 1u, v, w, ask);
    return rc != cudaSuccess ? rc : launch(cache_assign_kernel<kGive>, (uint64_t)tiles + sharing, kCacheThreads, st, 1u, v, w, ask, cu);
}
template <typename V>
cudaError_t run_fork_copy(const CacheView &v, const CacheScratch &w, const PoolView &p, const int32_t *parent, cudaStream_t st) {
    const unsigned long long units = (unsigned long long)v.max_seqs * 2 * p.layers;
    return launch(cache_fork_copy_kernel<V>, std::min<unsigned long long>(units, 148 * 64), kCacheThreads, st, 1u, v, w, p, parent, units);
}
template <typename V>
cudaError_t run_move(const CacheView &v, const CacheScratch &w, const PoolView &p, int32_t *moved, cudaStream_t st) {
    const uint32_t seq_blocks = warp_blocks(v.max_seqs), page_blocks = std::min((v.n_pages / 2 + kCacheThreads - 1) / kCacheThreads + 1, 148u);
    const unsigned long long units = (unsigned long long)(v.n_pages / 2) * 2 * p.layers;
    const uint32_t blocks = (uint32_t)std::max(1ull, std::min<unsigned long long>(units, 148 * 8));
    return launch(cache_move_kernel<V>, (uint64_t)seq_blocks + page_blocks + blocks, kCacheThreads, st, 1u, v, w, p, moved, seq_blocks, page_blocks);
}
template <typename V>
cudaError_t run_write(const CacheView &v, const PoolView &p, WriteArgs k, cudaStream_t st) {
    uint32_t rows = kMaxWriteRows;
    while (rows > 1 && (k.n_rows + rows - 1) / rows < 296) rows /= 2;
    k.rows_per_block = rows;
    return launch(cache_write_kernel<V>, (k.n_rows + rows - 1) / rows, kCacheThreads, st, 1u, v, p, k);
}

// ---- attention ----
std::atomic<uint32_t> g_lost_block{~0u}, g_lost_tile{~0u};    // td_debug_cache_wait
constexpr uint32_t kBlocks = 148;                             // one per SM
template <int kChunks>
constexpr size_t part_bytes() {
    return std::max((size_t)(2 * AttendShape<kChunks, 1>::kWarps + 2) * kBlocks * AttendShape<kChunks, 1>::kPartFloats * 4,
                    (size_t)(2 * AttendShape<kChunks, 2>::kWarps + 2) * kBlocks * AttendShape<kChunks, 2>::kPartFloats * 4);
}
template <int kChunks>
constexpr size_t share_bytes() { return (size_t)2 * kBlocks * ShareShape<kChunks, 2>::kPartFloats * 4; }
struct AttendLayout {
    size_t arrived, share_arrived, shared, common, parts, share_parts, total;
};
AttendLayout attend_layout(uint32_t n_rows, uint32_t n_heads, uint32_t dim) {          // no area shrinks as an argument grows
    size_t parts = part_bytes<4>(), share = share_bytes<4>(), padded = 64;
    auto at_least = [&](uint32_t d, size_t p, size_t s) { if (dim > padded) { parts = std::max(parts, p); share = std::max(share, s); padded = d; } };
    at_least(96, part_bytes<6>(), share_bytes<6>());
    at_least(128, part_bytes<8>(), share_bytes<8>());
    at_least(192, part_bytes<12>(), share_bytes<12>());
    at_least(256, part_bytes<16>(), share_bytes<16>());
    AttendLayout L{};
    size_t p = 0;
    auto take = [&](size_t bytes) { const size_t at = p; p = round_up(p + bytes, 256); return at; };
    L.arrived = take(kBlocks * 4);
    L.share_arrived = take(kBlocks * 4);
    L.shared = take((size_t)n_rows * 8);
    L.parts = take(parts);
    L.share_parts = take(share);
    L.common = take((size_t)n_rows * n_heads * (padded + 2) * 4);
    L.total = p;
    return L;
}
// The common tokens on the tensor memory (128 heads at a time, most of them empty where there are few) or by warps of 16 heads.  In us,
// 256 groups with prompts of 2000 tokens, 4 key heads of 128, the whole call: 16 heads to a key head 419 and 423, 20 heads 445 and 477,
// 32 heads 452 and 491; 64 groups of 8 heads to 8 key heads 249 and 244.  The shapes above 128 elements do not fit in shared memory.
constexpr uint32_t kWideHeads = 16;
template <typename T, int kChunks>
cudaError_t run_share(const CacheView &v, const AttendArgs &k, cudaStream_t st) {
    if constexpr (kChunks <= 8) {
        if (k.m_rows >= kWideHeads) {
            using W = WideShape<kChunks>;
            const cudaError_t rc = cudaFuncSetAttribute(share_wide_kernel<T, kChunks>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)W::kBytes);
            return rc != cudaSuccess ? rc : launch_smem(share_wide_kernel<T, kChunks>, kBlocks, kShareThreads, W::kBytes, st, 1u, v, k);
        }
    }
    using H = ShareShape<kChunks, 2>;
    const cudaError_t rc = cudaFuncSetAttribute(share_kernel<T, kChunks, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)H::kBytes);
    return rc != cudaSuccess ? rc : launch_smem(share_kernel<T, kChunks, 2>, kBlocks, kShareThreads, H::kBytes, st, 1u, v, k);
}
template <typename T, int kChunks, int kN>
cudaError_t run_attend(const CacheView &v, AttendArgs k, cudaStream_t st) {
    using S = AttendShape<kChunks, kN>;
    k.per_kv = (k.ratio + S::kHeads - 1) / S::kHeads;
    k.units = k.kv_heads * k.per_kv;
    k.by_per_kv = make_fastdiv(k.per_kv);
    cudaError_t rc = cudaFuncSetAttribute(attend_kernel<T, kChunks, kN>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::kBytes);
    if (rc == cudaSuccess && k.group > 1) {
        rc = launch(share_plan_kernel, k.n_groups, kShareThreads, st, 1u, v, k);
        if (rc == cudaSuccess) rc = run_share<T, kChunks>(v, k, st);
    }
    if (rc == cudaSuccess) rc = launch_smem(attend_kernel<T, kChunks, kN>, kBlocks, S::kThreads, S::kBytes, st, 1u, v, k);
    return rc;
}
template <typename T, int kChunks>
cudaError_t run_attend(const CacheView &v, const AttendArgs &k, cudaStream_t st) {
    return k.ratio <= 8 ? run_attend<T, kChunks, 1>(v, k, st) : run_attend<T, kChunks, 2>(v, k, st);
}
template <typename T>
cudaError_t run_attend(const CacheView &v, const AttendArgs &k, cudaStream_t st) {
    if (k.dim <= 64) return run_attend<T, 4>(v, k, st);
    if (k.dim <= 96) return run_attend<T, 6>(v, k, st);
    if (k.dim <= 128) return run_attend<T, 8>(v, k, st);
    if (k.dim <= 192) return run_attend<T, 12>(v, k, st);
    return run_attend<T, 16>(v, k, st);
}
cudaError_t run_attend_float(const CacheView &v, AttendArgs k, cudaStream_t st) {
    k.per_kv = (k.ratio + kFloatHeads - 1) / kFloatHeads;
    k.units = k.kv_heads * k.per_kv;
    k.by_per_kv = make_fastdiv(k.per_kv);
    const uint64_t blocks = (uint64_t)k.n_rows * k.units;
    return blocks > kMaxGrid ? cudaErrorInvalidValue : launch(attend_float_kernel, blocks, kFloatThreads, st, 1u, v, k);
}

}  // namespace

extern "C" {

size_t td_cache_workspace_bytes(uint32_t n_pages, uint32_t max_seqs) {
    return cache_sizes_ok(n_pages, max_seqs) ? cache_layout(n_pages, max_seqs).total : 0;
}

int td_cache_extend(const td_cache *c, const int32_t *add, int32_t *cu, void *stream) {
    TD_RANGE("td_cache_extend");
    int chk = check_cache(c, false);
    if (chk == TD_OK && (!aligned(add, 4) || !aligned(cu, 4))) chk = TD_EINVAL;
    if (chk == TD_OK) chk = check_workspace(c);
    if (chk != TD_OK) return chk;
    if (c->max_seqs == 0 && !cu) return TD_OK;
    DeviceGuard dev(c->device);
    if (!dev.ok()) return TD_ECUDA;
    cudaStream_t st = (cudaStream_t)stream;
    if (c->max_seqs == 0) return result(cudaMemsetAsync(cu, 0, 4, st));
    const CacheView v = cache_view(c);
    const CacheScratch w = scratch_of(c);
    return result(run_give<Give::kExtend>(v, w, add, cu, 0u, st));
}

int td_cache_fork(const td_cache *c, const int32_t *parent, void *stream) {
    TD_RANGE("td_cache_fork");
    int chk = check_cache(c, true);
    if (chk == TD_OK && (!aligned(parent, 4) || (c->max_seqs && !parent))) chk = TD_EINVAL;
    if (chk == TD_OK) chk = check_workspace(c);
    if (chk != TD_OK) return chk;
    if (c->max_seqs == 0 || c->n_pages == 0) return TD_OK;
    DeviceGuard dev(c->device);
    if (!dev.ok()) return TD_ECUDA;
    cudaStream_t st = (cudaStream_t)stream;
    const CacheView v = cache_view(c);
    const CacheScratch w = scratch_of(c);
    if (run_give<Give::kFork>(v, w, parent, nullptr, warp_blocks(c->max_seqs), st) != cudaSuccess) return TD_ECUDA;
    const uint32_t vec = vector_bytes(c, nullptr, nullptr, 0, 0);
    const PoolView p = pool_view(c, vec);
    return result(vec == 16 ? run_fork_copy<uint4>(v, w, p, parent, st) : vec == 4 ? run_fork_copy<uint32_t>(v, w, p, parent, st)
                                                                                     : run_fork_copy<uint16_t>(v, w, p, parent, st));
}

int td_cache_free(const td_cache *c, const uint8_t *release, void *stream) {
    TD_RANGE("td_cache_free");
    const int chk = check_cache(c, false);
    if (chk != TD_OK) return chk;
    if (c->max_seqs == 0) return TD_OK;
    DeviceGuard dev(c->device);
    if (!dev.ok()) return TD_ECUDA;
    return result(launch(cache_free_kernel, warp_blocks(c->max_seqs), kCacheThreads, (cudaStream_t)stream, 1u, cache_view(c), release));
}

int td_cache_compact(const td_cache *c, uint32_t *used, int32_t *moved, void *stream) {
    TD_RANGE("td_cache_compact");
    int chk = check_cache(c, true);
    if (chk == TD_OK && (!aligned(used, 4) || !aligned(moved, 4))) chk = TD_EINVAL;
    if (chk == TD_OK) chk = check_workspace(c);
    if (chk != TD_OK) return chk;
    if (c->n_pages == 0 && !used) return TD_OK;
    DeviceGuard dev(c->device);
    if (!dev.ok()) return TD_ECUDA;
    cudaStream_t st = (cudaStream_t)stream;
    if (c->n_pages == 0) return result(cudaMemsetAsync(used, 0, 4, st));
    const CacheView v = cache_view(c);
    const CacheScratch w = scratch_of(c);
    // Few pages: both steps in one launch, by the blocks of a cluster with its barrier between them.  On the device that is as long as two
    // launches (a pool of 104 pages 9.4 us both ways), but the host has one less to make (17.9 us a call from Python, 19.6).
    cudaError_t rc;
    if (w.page_tiles <= kClusterBlocks) {
        rc = launch(cache_held_rank_kernel, kClusterBlocks, kCacheThreads, st, kClusterBlocks, v, w, used, moved);
    } else {
        rc = launch(cache_held_kernel, w.page_tiles, kCacheThreads, st, 1u, v, w);
        if (rc == cudaSuccess) rc = launch(cache_rank_kernel, w.page_tiles, kCacheThreads, st, 1u, v, w, used, moved);
    }
    if (rc != cudaSuccess) return TD_ECUDA;
    const uint32_t vec = vector_bytes(c, nullptr, nullptr, 0, 0);
    const PoolView p = pool_view(c, vec);
    return result(vec == 16 ? run_move<uint4>(v, w, p, moved, st) : vec == 4 ? run_move<uint32_t>(v, w, p, moved, st)
                                                                               : run_move<uint16_t>(v, w, p, moved, st));
}

int td_cache_write(const td_cache_write_args *a, void *stream) {
    TD_RANGE("td_cache_write");
    if (!a) return TD_EINVAL;
    const td_cache *c = a->cache;
    const int chk = check_cache(c, true);
    if (chk != TD_OK) return chk;
    if (a->n_rows >= kIndexLimit || a->row_stride < 0 || a->head_stride < 0 || !aligned(a->cu, 4) || (c->keys && a->layer >= c->n_layers)) return TD_EINVAL;
    if (a->n_rows == 0 || c->max_seqs == 0 || c->n_pages == 0) return TD_OK;
    const uint32_t es = size_of(c->dtype);
    if (!a->keys || !a->values || !a->cu || !aligned(a->keys, es) || !aligned(a->values, es)) return TD_EINVAL;
    DeviceGuard dev(c->device);
    if (!dev.ok()) return TD_ECUDA;
    const uint32_t vec = vector_bytes(c, a->keys, a->values, a->row_stride, a->head_stride);
    WriteArgs k{static_cast<const uint8_t *>(a->keys), static_cast<const uint8_t *>(a->values), a->row_stride * es, a->head_stride * es, a->cu,
                a->layer, a->n_rows, 0u};
    cudaStream_t st = (cudaStream_t)stream;
    const CacheView v = cache_view(c);
    const PoolView p = pool_view(c, vec);
    return result(vec == 16 ? run_write<uint4>(v, p, k, st) : vec == 4 ? run_write<uint32_t>(v, p, k, st) : run_write<uint16_t>(v, p, k, st));
}

size_t td_cache_attention_workspace_bytes(uint32_t n_rows, uint32_t n_heads, uint32_t dim) {
    if (n_rows >= kMaxRows || n_heads >= (1u << 16) || dim > kMaxDim) return 0;
    return attend_layout(n_rows, n_heads, dim).total;
}

int td_cache_attention(const td_cache_attention_args *a, void *stream) {
    TD_RANGE("td_cache_attention");
    if (!a) return TD_EINVAL;
    const td_cache *c = a->cache;
    const int chk = check_cache(c, true);
    if (chk != TD_OK) return chk;
    const float scale2 = (float)(1.4426950408889634 * (double)a->scale);
    if (a->n_rows >= kMaxRows || a->n_heads >= (1u << 16) || a->group == 0 || !std::isfinite(scale2)) return TD_EINVAL;
    if (a->q_row_stride < 0 || a->q_head_stride < 0) return TD_EINVAL;
    if (!c->keys || a->layer >= c->n_layers || c->dim > kMaxDim || c->dim % 8 || a->n_heads == 0 || a->n_heads % c->n_heads) return TD_EINVAL;
    if (a->n_rows == 0) return TD_OK;
    if (!apart(a->n_rows, a->out_row_stride, a->n_heads, a->out_head_stride, c->dim)) return TD_EINVAL;
    const uint32_t es = size_of(c->dtype);
    for (int64_t n : {c->layer_stride, c->page_stride, c->token_stride, c->head_stride, a->q_row_stride, a->q_head_stride, a->out_row_stride, a->out_head_stride})
        if (n * es % 16) return TD_EINVAL;
    if (!a->q || !a->out || !aligned(c->keys, 16) || !aligned(c->values, 16) || !aligned(a->q, 16) || !aligned(a->out, 16) || !aligned(a->lse, 4) ||
        !aligned(a->seqs, 4)) return TD_EINVAL;
    if (!a->workspace || !aligned(a->workspace, 256) || a->workspace_bytes < td_cache_attention_workspace_bytes(a->n_rows, a->n_heads, c->dim))
        return TD_EWORKSPACE;
    DeviceGuard dev(c->device);
    if (!dev.ok()) return TD_ECUDA;
    AttendArgs k{};
    k.seqs = a->seqs;
    k.q = a->q;
    k.out = a->out;
    k.lse = a->lse;
    k.keys = static_cast<const uint8_t *>(c->keys) + a->layer * c->layer_stride * es;
    k.values = static_cast<const uint8_t *>(c->values) + a->layer * c->layer_stride * es;
    k.page = c->page_stride;
    k.token = c->token_stride;
    k.head = c->head_stride;
    k.q_row = a->q_row_stride;
    k.q_head = a->q_head_stride;
    k.out_row = a->out_row_stride;
    k.out_head = a->out_head_stride;
    k.n_rows = a->n_rows;
    k.n_heads = a->n_heads;
    k.kv_heads = c->n_heads;
    k.ratio = a->n_heads / c->n_heads;
    k.dim = c->dim;
    k.window = a->window;
    k.scale2 = scale2;
    // rows that share, and their heads over one key head in blocks of like size
    k.whole = std::min(a->group, a->n_rows);
    k.pieces = (k.whole + kMaxGroup - 1) / kMaxGroup;
    k.group = (k.whole + k.pieces - 1) / k.pieces;
    k.n_groups = (a->n_rows + k.whole - 1) / k.whole * k.pieces;
    k.m_blocks = (k.group * k.ratio + kShareHeads - 1) / kShareHeads;
    k.m_rows = (k.group * k.ratio + k.m_blocks - 1) / k.m_blocks;
    k.by_group = make_fastdiv(k.group);
    k.by_whole = make_fastdiv(k.whole);
    k.by_ratio = make_fastdiv(k.ratio);
    const AttendLayout L = attend_layout(a->n_rows, a->n_heads, c->dim);
    uint8_t *ws = static_cast<uint8_t *>(a->workspace);
    k.arrived = reinterpret_cast<uint32_t *>(ws + L.arrived);
    k.share_arrived = reinterpret_cast<uint32_t *>(ws + L.share_arrived);
    k.shared = reinterpret_cast<int2 *>(ws + L.shared);
    k.parts = reinterpret_cast<float *>(ws + L.parts);
    k.share_parts = reinterpret_cast<float *>(ws + L.share_parts);
    k.common = reinterpret_cast<float *>(ws + L.common);
    k.lost_block = g_lost_block.load(std::memory_order_relaxed);
    k.lost_tile = g_lost_tile.load(std::memory_order_relaxed);
    cudaStream_t st = (cudaStream_t)stream;
    const CacheView v = cache_view(c);
    return result(c->dtype == TD_F32 ? run_attend_float(v, k, st) : c->dtype == TD_BF16 ? run_attend<__nv_bfloat16>(v, k, st)
                                                                                          : run_attend<__half>(v, k, st));
}

int td_debug_cache_wait(uint32_t block, uint32_t tile) {
    g_lost_block.store(block, std::memory_order_relaxed);
    g_lost_tile.store(tile, std::memory_order_relaxed);
    return TD_OK;
}

}  // extern "C"
