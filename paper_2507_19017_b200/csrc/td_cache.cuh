// Paged key-value cache: the calls that hand out, share, give back and move pages, and the writing of new
// tokens' keys and values.
//
// Pages are handed out lowest free number first in order of the sequences that need them: the r-th page needed is
// the r-th page without a holder.  So a call is two prefix sums (free pages by number, pages needed by
// sequence) and one meeting of the two.  cache_count_kernel takes the sums of tiles, cache_assign_kernel
// adds up the tiles before its own (at most kMaxTiles of them) and hands out; nothing waits inside a
// kernel.  Integer sums and one writer per word: the same call gives the same tables.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "td_ops.cuh"

namespace td {

constexpr uint32_t kCacheThreads = 256;
constexpr uint32_t kPagesPerThread = 8;                       // consecutive pages of a thread
constexpr uint32_t kPageStep = kCacheThreads * kPagesPerThread;
constexpr uint32_t kSeqsPerThread = 4;
constexpr uint32_t kSeqStep = kCacheThreads * kSeqsPerThread;
constexpr uint32_t kMaxTiles = 1024;                          // tiles of pages, and of sequences

// What is handed out: room for new tokens, or the pages of forked sequences' last tokens.
enum class Give { kExtend, kFork };

struct CacheView {
    int32_t *table, *length, *holders;
    uint32_t *status;
    uint32_t n_pages, page_size, max_seqs, max_pages;
    FastDiv by_page;
};

// The workspace of one call.
struct CacheScratch {
    uint32_t *tile_pages;                                     // [page tiles] free (or held) pages
    unsigned long long *tile_need, *tile_add;                 // [sequence tiles] pages needed, tokens added
    unsigned long long *need_before;                          // [sequences] pages needed ahead of it in its tile
    uint32_t *add_before;                                     // [sequences] tokens added ahead of it in its tile
    uint32_t *first;                                          // [sequences] place of the first page it is given
    int32_t *tokens;                                          // [sequences] its length after the call, -1: left as it is
    int32_t *given;                                           // [sequences] the page a fork is given, -1: none
    uint32_t *from, *to;                                      // [pages] compaction: source by rank, free number by rank
    uint32_t *rank;                                           // [pages] rank of a source among the held pages
    uint32_t *moves;                                          // how many pages move, how many are held
    uint32_t page_steps, seq_steps;                           // steps of kPageStep pages (kSeqStep sequences) per tile
    uint32_t page_tiles, seq_tiles;
};

__device__ __forceinline__ void cache_flag(const CacheView &c, uint32_t bit) {
    if (c.status) atomicOr(c.status, bit);
}
__device__ __forceinline__ uint32_t pages_for(const CacheView &c, uint32_t tokens) {
    return tokens ? fast_div(tokens - 1, c.by_page) + 1 : 0u;
}
__device__ __forceinline__ bool length_ok(const CacheView &c, int32_t n) {
    return n >= 0 && (unsigned long long)n <= (unsigned long long)c.max_pages * c.page_size;
}

// Sum over the block of a value per thread, and what the threads before have.  `room`: one word per warp.
template <typename T>
__device__ __forceinline__ T block_before(T x, T *room, T &total) {
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    T incl = x;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const T y = __shfl_up_sync(kFullMask, incl, d);
        if (lane >= (uint32_t)d) incl += y;
    }
    __syncthreads();                                          // the room's last use is over
    if (lane == 31) room[warp] = incl;
    __syncthreads();
    T before = 0;
    total = 0;
#pragma unroll
    for (uint32_t w = 0; w < kCacheThreads / 32; ++w) {
        const T v = room[w];
        before += w < warp ? v : 0;
        total += v;
    }
    return before + incl - x;
}

// Which of a thread's kPagesPerThread pages from `page` on are free (kHeld: held), as bits.
template <bool kHeld>
__device__ __forceinline__ uint32_t page_bits(const CacheView &c, uint32_t page) {
    uint32_t bits = 0;
    if (page + kPagesPerThread <= c.n_pages && (reinterpret_cast<uintptr_t>(c.holders) & 15u) == 0) {
        const int4 a = *reinterpret_cast<const int4 *>(c.holders + page), b = *reinterpret_cast<const int4 *>(c.holders + page + 4);
        bits = (a.x == 0) | (a.y == 0) << 1 | (a.z == 0) << 2 | (a.w == 0) << 3 | (b.x == 0) << 4 | (b.y == 0) << 5 |
               (b.z == 0) << 6 | (b.w == 0) << 7;
        return kHeld ? bits ^ 0xffu : bits;
    }
#pragma unroll
    for (uint32_t k = 0; k < kPagesPerThread; ++k)
        if (page < c.n_pages && k < c.n_pages - page) bits |= (uint32_t)((c.holders[page + k] == 0) != kHeld) << k;
    return bits;
}

// What sequence s asks for: pages, and in `tokens` its new length (-1: nothing happens to it), in `first` the place of its
// first new page, in `add` the tokens it is given.
template <Give kGive>
__device__ __forceinline__ uint32_t pages_needed(const CacheView &c, const int32_t *ask, uint32_t s, int32_t &tokens, uint32_t &first,
                                                 uint32_t &add) {
    tokens = -1;
    first = add = 0;
    const int32_t n = c.length[s];
    if constexpr (kGive == Give::kExtend) {
        const int32_t want = ask ? ask[s] : (n != 0 ? 1 : 0);          // a negative length is looked at, and noted
        if (want == 0) return 0;
        if (want < 0 || !length_ok(c, n) || (unsigned long long)n + want > (unsigned long long)c.max_pages * c.page_size) {
            cache_flag(c, TD_ERR_BAD_LENGTH);
            return 0;
        }
        tokens = n + want;
        add = (uint32_t)want;
        first = pages_for(c, (uint32_t)n);
        return pages_for(c, (uint32_t)tokens) - first;
    } else {
        const int32_t p = ask[s];
        if (p < 0) return 0;
        if ((uint32_t)p >= c.max_seqs) { cache_flag(c, TD_ERR_OOB_INDEX); return 0; }
        if (n != 0) { cache_flag(c, TD_ERR_DUP_PUT); return 0; }
        const int32_t m = c.length[p];
        if (!length_ok(c, m)) { cache_flag(c, TD_ERR_BAD_LENGTH); return 0; }
        tokens = m;
        first = fast_div((uint32_t)m, c.by_page);
        return (uint32_t)m != first * c.page_size ? 1u : 0u;
    }
}

// Sums of tiles: blocks 0 .. page_tiles - 1 count pages, the others what sequences need.
template <Give kGive>
__global__ void __launch_bounds__(kCacheThreads) cache_count_kernel(CacheView c, CacheScratch w, const int32_t *ask) {
    __shared__ unsigned long long room[2][kCacheThreads / 32];
    griddep_launch_dependents();
    griddep_wait();
    const uint32_t tile = blockIdx.x;
    if (tile < w.page_tiles) {
        unsigned long long count = 0, total;
        for (uint32_t k = 0; k < w.page_steps; ++k) {
            const unsigned long long page = ((unsigned long long)tile * w.page_steps + k) * kPageStep + threadIdx.x * kPagesPerThread;
            if (page < c.n_pages) count += __popc(page_bits<false>(c, (uint32_t)page));
        }
        block_before(count, room[0], total);
        if (threadIdx.x == 0) w.tile_pages[tile] = (uint32_t)total;
        return;
    }
    const uint32_t st = tile - w.page_tiles;
    unsigned long long need_base = 0, add_base = 0;
    for (uint32_t k = 0; k < w.seq_steps; ++k) {
        const uint32_t s0 = (st * w.seq_steps + k) * kSeqStep + threadIdx.x * kSeqsPerThread;
        uint32_t need[kSeqsPerThread], add[kSeqsPerThread], first[kSeqsPerThread];
        int32_t tokens[kSeqsPerThread];
        unsigned long long needs = 0, adds = 0, need_total, add_total;
#pragma unroll
        for (uint32_t i = 0; i < kSeqsPerThread; ++i) {
            need[i] = add[i] = 0;
            if (s0 + i < c.max_seqs) need[i] = pages_needed<kGive>(c, ask, s0 + i, tokens[i], first[i], add[i]);
            needs += need[i];
            adds += add[i];
        }
        unsigned long long nb = need_base + block_before(needs, room[0], need_total), ab = add_base + block_before(adds, room[1], add_total);
#pragma unroll
        for (uint32_t i = 0; i < kSeqsPerThread; ++i) {
            if (s0 + i < c.max_seqs) {
                w.need_before[s0 + i] = nb;
                w.add_before[s0 + i] = (uint32_t)ab;
                w.first[s0 + i] = first[i];
                w.tokens[s0 + i] = tokens[i];
                if (kGive == Give::kFork) w.given[s0 + i] = -1;
            }
            nb += need[i];
            ab += add[i];
        }
        need_base += need_total;
        add_base += add_total;
    }
    if (threadIdx.x == 0) {
        w.tile_need[st] = need_base;
        w.tile_add[st] = add_base;
    }
}

// The sums of the tiles before `mine` and of all.
struct TileSum {
    unsigned long long before, all;
};
template <typename T>
__device__ __forceinline__ TileSum tile_part(const T *sums, uint32_t n, uint32_t mine) {          // a thread's share
    TileSum t{0, 0};
    for (uint32_t i = threadIdx.x; i < n; i += kCacheThreads) {
        const unsigned long long v = sums[i];
        t.all += v;
        t.before += i < mine ? v : 0;
    }
    return t;
}
template <int kSums>
__device__ __forceinline__ void tile_sums(TileSum (&t)[kSums], unsigned long long (*room)[2 * kSums]) {          // the block's, one row of room per warp
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
#pragma unroll
    for (int k = 0; k < kSums; ++k) {
#pragma unroll
        for (int d = 16; d; d /= 2) {
            t[k].before += __shfl_xor_sync(kFullMask, t[k].before, d);
            t[k].all += __shfl_xor_sync(kFullMask, t[k].all, d);
        }
        if (lane == 0) {
            room[warp][2 * k] = t[k].before;
            room[warp][2 * k + 1] = t[k].all;
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kSums; ++k) {
        t[k] = TileSum{0, 0};
#pragma unroll
        for (uint32_t w = 0; w < kCacheThreads / 32; ++w) {
            t[k].before += room[w][2 * k];
            t[k].all += room[w][2 * k + 1];
        }
    }
}

// Blocks of page tiles hand out their free pages; blocks of sequence tiles set lengths and cu; fork: further blocks, a warp per
// sequence, share the full pages.
template <Give kGive>
__global__ void __launch_bounds__(kCacheThreads) cache_assign_kernel(CacheView c, CacheScratch w, const int32_t *ask, int32_t *cu) {
    __shared__ unsigned long long room[kCacheThreads / 32], sums[kCacheThreads / 32][6];
    __shared__ unsigned long long tile_need[kMaxTiles];       // pages needed ahead of each sequence tile
    __shared__ uint32_t given[kPageStep];                     // free pages of a step, in order
    griddep_launch_dependents();
    griddep_wait();
    const uint32_t seq_block = blockIdx.x - w.page_tiles;     // for blocks behind the page tiles
    const bool page_block = blockIdx.x < w.page_tiles;
    TileSum t[3] = {tile_part(w.tile_need, w.seq_tiles, 0u), tile_part(w.tile_add, w.seq_tiles, page_block ? 0u : seq_block),
                    tile_part(w.tile_pages, w.page_tiles, page_block ? blockIdx.x : 0u)};
    tile_sums<3>(t, sums);
    const unsigned long long need_total = t[0].all, add_total = t[1].all, add_base = t[1].before, page_total = t[2].all;
    const bool enough = need_total <= page_total && (!cu || add_total < (1ull << 31));          // cu's words are 32 bits wide
    if (page_block) {
        unsigned long long base = t[2].before;
        if (!enough || base >= need_total) return;
        unsigned long long before = 0;
        for (uint32_t t0 = 0; t0 < w.seq_tiles; t0 += kCacheThreads) {
            const uint32_t i = t0 + threadIdx.x;
            unsigned long long step;
            const unsigned long long b = block_before(i < w.seq_tiles ? w.tile_need[i] : 0ull, room, step);
            if (i < w.seq_tiles) tile_need[i] = before + b;
            before += step;
        }
        for (uint32_t k = 0; k < w.page_steps && base < need_total; ++k) {
            const unsigned long long page = ((unsigned long long)blockIdx.x * w.page_steps + k) * kPageStep + threadIdx.x * kPagesPerThread;
            uint32_t bits = page < c.n_pages ? page_bits<false>(c, (uint32_t)page) : 0u;
            uint32_t step;
            uint32_t at = block_before((uint32_t)__popc(bits), reinterpret_cast<uint32_t *>(room), step);
            for (; bits; bits &= bits - 1) given[at++] = (uint32_t)page + (uint32_t)__ffs(bits) - 1;
            __syncthreads();
            // a thread per page that is handed out: whose it is takes a search, so they go side by side
            const uint32_t some = (uint32_t)min((unsigned long long)step, need_total - base);
            for (uint32_t i = threadIdx.x; i < some; i += kCacheThreads) {
                const unsigned long long r = base + i;
                uint32_t lo = 0, hi = w.seq_tiles;            // the last tile with no more than r ahead of it
                while (hi - lo > 1) {
                    const uint32_t mid = (lo + hi) / 2;
                    if (tile_need[mid] <= r) lo = mid; else hi = mid;
                }
                const unsigned long long local = r - tile_need[lo];
                const uint32_t per_tile = w.seq_steps * kSeqStep, p = given[i];
                uint32_t s = lo * per_tile, end = min(c.max_seqs - s, per_tile) + s;
                while (end - s > 1) {                         // and the last sequence of it
                    const uint32_t mid = s + (end - s) / 2;
                    if (w.need_before[mid] <= local) s = mid; else end = mid;
                }
                const uint32_t place = w.first[s] + (uint32_t)(local - w.need_before[s]);
                c.table[(size_t)s * c.max_pages + place] = (int32_t)p;
                c.holders[p] = 1;
                if (kGive == Give::kFork) w.given[s] = (int32_t)p;
            }
            base += step;
        }
        return;
    }
    if (seq_block < w.seq_tiles) {
        for (uint32_t k = 0; k < w.seq_steps * kSeqsPerThread; ++k) {
            const uint32_t s = seq_block * w.seq_steps * kSeqStep + k * kCacheThreads + threadIdx.x;
            if (s >= c.max_seqs) break;
            const int32_t n = w.tokens[s];
            if (enough && n >= 0) c.length[s] = n;
            if (kGive == Give::kExtend && cu) cu[s] = enough ? (int32_t)(add_base + w.add_before[s]) : 0;
        }
        if (seq_block == 0 && threadIdx.x == 0) {
            if (kGive == Give::kExtend && cu) cu[c.max_seqs] = enough ? (int32_t)add_total : 0;
            if (need_total > page_total) cache_flag(c, TD_ERR_ARENA_FULL);
            else if (!enough) cache_flag(c, TD_ERR_BAD_LENGTH);
        }
        return;
    }
    if constexpr (kGive == Give::kFork) {
        const uint32_t s = (seq_block - w.seq_tiles) * (kCacheThreads / 32) + threadIdx.x / 32;
        if (!enough || s >= c.max_seqs || w.tokens[s] < 0) return;
        const uint32_t full = w.first[s];
        const int32_t *from = c.table + (size_t)(uint32_t)ask[s] * c.max_pages;
        int32_t *to = c.table + (size_t)s * c.max_pages;
        for (uint32_t j = threadIdx.x & 31u; j < full; j += 32) {
            const int32_t p = from[j];
            to[j] = p;
            if ((uint32_t)p < c.n_pages) atomicAdd(c.holders + p, 1);
            else cache_flag(c, TD_ERR_OOB_INDEX);
        }
    }
}

constexpr uint32_t kClusterBlocks = 8;                        // of a compaction of few pages
__device__ __forceinline__ void cluster_sync() {              // what the blocks wrote before it they all see behind it
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// A warp per sequence.
__global__ void __launch_bounds__(kCacheThreads) cache_free_kernel(CacheView c, const uint8_t *release) {
    griddep_launch_dependents();
    griddep_wait();
    const uint32_t s = blockIdx.x * (kCacheThreads / 32) + threadIdx.x / 32, lane = threadIdx.x & 31u;
    if (s >= c.max_seqs || (release && !release[s])) return;
    const int32_t n = c.length[s];
    __syncwarp();
    if (!length_ok(c, n)) {
        if (lane == 0) cache_flag(c, TD_ERR_BAD_LENGTH);
        return;
    }
    const int32_t *row = c.table + (size_t)s * c.max_pages;
    for (uint32_t j = lane, pages = pages_for(c, (uint32_t)n); j < pages; j += 32) {
        const int32_t p = row[j];
        if ((uint32_t)p >= c.n_pages) { cache_flag(c, TD_ERR_OOB_INDEX); continue; }
        if (atomicSub(c.holders + p, 1) <= 0) {
            atomicAdd(c.holders + p, 1);
            cache_flag(c, TD_ERR_DUP_PUT);
        }
    }
    if (lane == 0) c.length[s] = 0;
}

// ---- compaction ----
__device__ __forceinline__ void held_block(const CacheView &c, const CacheScratch &w, uint32_t block) {
    __shared__ unsigned long long room[kCacheThreads / 32];
    unsigned long long count = 0, total;
    for (uint32_t k = 0; k < w.page_steps; ++k) {
        const unsigned long long page = ((unsigned long long)block * w.page_steps + k) * kPageStep + threadIdx.x * kPagesPerThread;
        if (page < c.n_pages) count += __popc(page_bits<true>(c, (uint32_t)page));
    }
    block_before(count, room, total);
    if (threadIdx.x == 0) w.tile_pages[block] = (uint32_t)total;
}

// With U pages held and b(p) of them before page p: the held pages from U on are those of ranks U - M .. U - 1 among the held, where
// M = U - b(U) is how many free numbers lie below U; free number f has rank f - b(f) among the free.
__device__ __forceinline__ void rank_block(const CacheView &c, const CacheScratch &w, uint32_t *used, int32_t *moved, uint32_t block) {
    __shared__ unsigned long long room[kCacheThreads / 32];
    __shared__ unsigned long long sums[kCacheThreads / 32][2];
    TileSum t[1] = {tile_part(w.tile_pages, w.page_tiles, block)};
    tile_sums<1>(t, sums);
    unsigned long long base = t[0].before;
    const uint32_t U = (uint32_t)t[0].all;
    if (block == 0 && threadIdx.x == 0) {
        if (used) *used = U;
        w.moves[1] = U;
        if (U == c.n_pages) w.moves[0] = 0;
    }
    for (uint32_t k = 0; k < w.page_steps; ++k) {
        const unsigned long long page = ((unsigned long long)block * w.page_steps + k) * kPageStep + threadIdx.x * kPagesPerThread;
        const uint32_t bits = page < c.n_pages ? page_bits<true>(c, (uint32_t)page) : 0u;
        unsigned long long step;
        uint32_t b = (uint32_t)(base + block_before((unsigned long long)__popc(bits), room, step));
        base += step;
        for (uint32_t i = 0; i < kPagesPerThread && page + i < c.n_pages; ++i) {
            const uint32_t p = (uint32_t)page + i;
            if (p == U) w.moves[0] = U - b;
            if (bits >> i & 1u) {
                if (p >= U) {
                    w.from[b] = p;
                    w.rank[p] = b;
                } else if (moved) {
                    moved[p] = (int32_t)p;
                }
                ++b;
            } else {
                if (p < U) w.to[p - b] = p;
                if (moved) moved[p] = -1;
            }
        }
    }
}

__global__ void __launch_bounds__(kCacheThreads) cache_held_kernel(CacheView c, CacheScratch w) {
    griddep_launch_dependents();
    griddep_wait();
    held_block(c, w, blockIdx.x);
}
__global__ void __launch_bounds__(kCacheThreads) cache_rank_kernel(CacheView c, CacheScratch w, uint32_t *used, int32_t *moved) {
    griddep_launch_dependents();
    griddep_wait();
    rank_block(c, w, used, moved, blockIdx.x);
}
__global__ void __launch_bounds__(kCacheThreads) cache_held_rank_kernel(CacheView c, CacheScratch w, uint32_t *used, int32_t *moved) {          // one cluster
    griddep_launch_dependents();
    griddep_wait();
    for (uint32_t b = blockIdx.x; b < w.page_tiles; b += gridDim.x, __syncthreads()) held_block(c, w, b);
    cluster_sync();
    for (uint32_t b = blockIdx.x; b < w.page_tiles; b += gridDim.x, __syncthreads()) rank_block(c, w, used, moved, b);
}

// ---- contents ----
// Rows of dim elements, (token, head) by (token, head), as vectors of V; byte strides.
struct PoolView {
    uint8_t *keys, *values;
    int64_t layer, page, token, head;
    uint32_t layers, heads;
    uint32_t vecs;                                            // vectors in a row
    uint32_t heads_first;                                     // a token's heads lie closer together than a head's tokens
    FastDiv by_vecs, by_heads;
};

// The first `tokens` tokens of a page to another, by a block.
template <typename V>
__device__ __forceinline__ void copy_page(const PoolView &p, uint8_t *pool, uint32_t layer, uint32_t from, uint32_t to, uint32_t tokens) {
    const uint8_t *src = pool + layer * p.layer + from * p.page;
    uint8_t *dst = pool + layer * p.layer + to * p.page;
    const uint32_t n = tokens * p.heads * p.vecs;             // below 2^31: checked on the host
    const FastDiv by_tokens = make_fastdiv_dev(tokens);
    constexpr uint32_t kUnroll = 4;
    for (uint32_t i0 = threadIdx.x; i0 < n; i0 += kCacheThreads * kUnroll) {
        V v[kUnroll];
        int64_t at[kUnroll];
#pragma unroll
        for (uint32_t k = 0; k < kUnroll; ++k) {
            const uint32_t i = i0 + k * kCacheThreads;
            if (i >= n) break;
            const uint32_t row = fast_div(i, p.by_vecs), vec = i - row * p.vecs;
            uint32_t token, head;
            if (p.heads_first) { token = fast_div(row, p.by_heads); head = row - token * p.heads; }
            else { head = fast_div(row, by_tokens); token = row - head * tokens; }
            at[k] = token * p.token + head * p.head + vec * (int64_t)sizeof(V);
            v[k] = *reinterpret_cast<const V *>(src + at[k]);
        }
#pragma unroll
        for (uint32_t k = 0; k < kUnroll; ++k)
            if (i0 + k * kCacheThreads < n) *reinterpret_cast<V *>(dst + at[k]) = v[k];
    }
}

// Forked sequences' last pages; units (layer and side, sequence), siblings side by side so that their common source comes
// from L2 after the first.
template <typename V>
__global__ void __launch_bounds__(kCacheThreads) cache_fork_copy_kernel(CacheView c, CacheScratch w, PoolView p, const int32_t *parent,
                                                                        unsigned long long units) {
    griddep_launch_dependents();
    griddep_wait();
    for (unsigned long long u = blockIdx.x; u < units; u += gridDim.x) {
        const uint32_t side = (uint32_t)(u / c.max_seqs), s = (uint32_t)(u - (unsigned long long)side * c.max_seqs);
        const int32_t to = w.given[s];
        if (to < 0) continue;
        const uint32_t full = w.first[s];
        const int32_t from = c.table[(size_t)(uint32_t)parent[s] * c.max_pages + full];
        if ((uint32_t)from >= c.n_pages) {
            if (threadIdx.x == 0) cache_flag(c, TD_ERR_OOB_INDEX);
            continue;
        }
        copy_page<V>(p, side & 1u ? p.values : p.keys, side >> 1, (uint32_t)from, (uint32_t)to, (uint32_t)w.tokens[s] - full * c.page_size);
    }
}

// The first blocks bring the tables, a warp per sequence, and the holders up to date; the others move pages, units (page, layer and side).
template <typename V>
__global__ void __launch_bounds__(kCacheThreads) cache_move_kernel(CacheView c, CacheScratch w, PoolView p, int32_t *moved, uint32_t seq_blocks,
                                                                   uint32_t page_blocks) {
    griddep_launch_dependents();
    griddep_wait();
    const uint32_t M = w.moves[0];
    if (M == 0) return;
    const uint32_t U = w.moves[1], kept = U - M;
    if (blockIdx.x < seq_blocks) {
        const uint32_t s = blockIdx.x * (kCacheThreads / 32) + threadIdx.x / 32, lane = threadIdx.x & 31u;
        if (s >= c.max_seqs) return;
        const int32_t n = c.length[s];
        if (!length_ok(c, n)) {
            if (lane == 0) cache_flag(c, TD_ERR_BAD_LENGTH);
            return;
        }
        int32_t *row = c.table + (size_t)s * c.max_pages;
        for (uint32_t j = lane, pages = pages_for(c, (uint32_t)n); j < pages; j += 32) {
            const uint32_t q = (uint32_t)row[j];
            if (q < U) continue;
            // a page in the table without a holder has no rank: the tables are not sound
            if (q >= c.n_pages) { cache_flag(c, TD_ERR_OOB_INDEX); continue; }
            const uint32_t r = w.rank[q];
            if (r < kept || r >= U || w.from[r] != q) { cache_flag(c, TD_ERR_DUP_PUT); continue; }
            row[j] = (int32_t)w.to[r - kept];
        }
        return;
    }
    if (blockIdx.x < seq_blocks + page_blocks) {
        for (uint32_t r = (blockIdx.x - seq_blocks) * kCacheThreads + threadIdx.x; r < M; r += page_blocks * kCacheThreads) {
            const uint32_t from = w.from[kept + r], to = w.to[r];
            c.holders[to] = c.holders[from];
            c.holders[from] = 0;
            if (moved) moved[from] = (int32_t)to;
        }
        return;
    }
    const uint32_t sides = 2 * p.layers, blocks = gridDim.x - seq_blocks - page_blocks;
    for (unsigned long long u = blockIdx.x - seq_blocks - page_blocks; u < (unsigned long long)M * sides; u += blocks) {
        const uint32_t r = (uint32_t)(u / sides), side = (uint32_t)(u - (unsigned long long)r * sides);
        copy_page<V>(p, side & 1u ? p.values : p.keys, side >> 1, w.from[kept + r], w.to[r], c.page_size);
    }
}

// ---- new tokens ----
struct WriteArgs {
    const uint8_t *keys, *values;
    int64_t row_stride, head_stride;                          // bytes
    const int32_t *cu;
    uint32_t layer, n_rows, rows_per_block;
};
constexpr uint32_t kMaxWriteRows = 32;                        // rows of a block

template <typename V>
__global__ void __launch_bounds__(kCacheThreads) cache_write_kernel(CacheView c, PoolView p, WriteArgs a) {
    __shared__ int64_t place[kMaxWriteRows];                  // byte offset of a row's token in the layer, -1: none
    griddep_launch_dependents();
    griddep_wait();
    const uint32_t first = blockIdx.x * a.rows_per_block;     // below n_rows
    const uint32_t rows = min(a.rows_per_block, a.n_rows - first);
    if (threadIdx.x < rows) {
        const long long t = first + threadIdx.x;
        int64_t at = -1;
        if (c.max_seqs && t < a.cu[c.max_seqs]) {
            const uint32_t s = sample_of(a.cu, 0u, c.max_seqs, t);
            const int32_t n = c.length[s];
            const long long end = a.cu[s + 1], pos = (long long)n - (end - t);
            if (a.cu[s] > t || end <= t || !length_ok(c, n) || pos < 0) {
                cache_flag(c, TD_ERR_BAD_LENGTH);
            } else {
                const uint32_t page = fast_div((uint32_t)pos, c.by_page);
                const int32_t id = c.table[(size_t)s * c.max_pages + page];
                if ((uint32_t)id < c.n_pages) at = id * p.page + (pos - (long long)page * c.page_size) * p.token;
                else cache_flag(c, TD_ERR_OOB_INDEX);
            }
        }
        place[threadIdx.x] = at;
    }
    __syncthreads();
    const uint32_t per_row = p.heads * p.vecs, n = rows * per_row;
    uint8_t *keys = p.keys + a.layer * p.layer, *values = p.values + a.layer * p.layer;
    constexpr uint32_t kUnroll = 4;
    for (uint32_t i0 = threadIdx.x; i0 < n; i0 += kCacheThreads * kUnroll) {
        V k[kUnroll], v[kUnroll];
        int64_t to[kUnroll];
#pragma unroll
        for (uint32_t u = 0; u < kUnroll; ++u) {
            const uint32_t i = i0 + u * kCacheThreads;
            to[u] = -1;
            if (i >= n) continue;
            const uint32_t rh = fast_div(i, p.by_vecs), vec = i - rh * p.vecs, row = fast_div(rh, p.by_heads), head = rh - row * p.heads;
            if (place[row] < 0) continue;
            to[u] = place[row] + head * p.head + vec * (int64_t)sizeof(V);
            const int64_t from = (int64_t)(first + row) * a.row_stride + head * a.head_stride + vec * (int64_t)sizeof(V);
            k[u] = *reinterpret_cast<const V *>(a.keys + from);
            v[u] = *reinterpret_cast<const V *>(a.values + from);
        }
#pragma unroll
        for (uint32_t u = 0; u < kUnroll; ++u)
            if (to[u] >= 0) {
                *reinterpret_cast<V *>(keys + to[u]) = k[u];
                *reinterpret_cast<V *>(values + to[u]) = v[u];
            }
    }
}

}  // namespace td
