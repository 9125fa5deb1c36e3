// Embedding rows of token ids, and the gradient with respect to the table by sorted tokens.
#pragma once

#include "td_ops.cuh"

namespace td {

struct EmbedArgs {
    const int32_t *ids;
    uint32_t n_tokens, vocab, dim, tokens;
    float scale;
    BatchView batch;
    uint32_t *status;
    const void *table;                   // forward
    void *out;
    long long table_stride, out_stride;
    // gradient
    const void *grad_out;
    void *grad_table;
    uint32_t accumulate;
    uint32_t rows_per_chunk;             // sorted positions per chunk of the segment sums
    uint32_t n_chunks;
    uint32_t *keys;                      // [n_tokens] sorted ids; vocab: no token
    uint32_t *pos;                       // [n_tokens] their positions
    uint32_t *present;                   // [ceil(vocab / 32)] a bit per id that occurs, or nullptr
    float *partial;                      // [2][n_chunks][partial_stride]: sums of a run cut by the chunk's start / by its end
    size_t partial_stride;               // dim rounded up to a warp's columns
};

// Positions that hold a token of the batch.
__device__ __forceinline__ uint32_t tokens_in(const EmbedArgs &a) {
    if (!a.batch.max_samples && !a.batch.cu_prompt && !a.batch.cu_response) return a.n_tokens;
    const uint32_t n = batch_samples(a.batch);
    if (n == 0) return 0;
    long long t = 0;
    if (a.tokens & TD_TOKENS_PROMPT) t += a.batch.cu_prompt[n];
    if (a.tokens & TD_TOKENS_RESPONSE) t += a.batch.cu_response[n];
    return (uint32_t)max(0ll, min(t, (long long)a.n_tokens));
}

// Id at position t, or vocab when there is no token.
__device__ __forceinline__ uint32_t id_at(const EmbedArgs &a, uint32_t t, uint32_t n) {
    if (t >= n) return a.vocab;
    const int32_t id = __ldg(a.ids + t);
    if (id < 0) return a.vocab;
    if ((uint32_t)id >= a.vocab) {
        if (a.status) atomicOr(a.status, TD_ERR_OOB_INDEX);
        return a.vocab;
    }
    return (uint32_t)id;
}

constexpr int kEmbedThreads = 256, kEmbedUnroll = 4;
constexpr uint32_t kEmbedVectors = 32 * kEmbedUnroll;        // 16-byte vectors of a row that one warp moves

// A warp per (position, piece of the row).
template <typename T, bool kWide>
__global__ void __launch_bounds__(kEmbedThreads) embed_kernel(const EmbedArgs a, uint32_t pieces) {
    griddep_launch_dependents();
    griddep_wait();
    const unsigned long long item = (unsigned long long)blockIdx.x * (kEmbedThreads / 32) + (threadIdx.x >> 5);
    const unsigned long long t64 = item / pieces;
    const uint32_t piece = (uint32_t)(item % pieces), lane = threadIdx.x & 31u;
    if (t64 >= a.n_tokens) return;
    const uint32_t t = (uint32_t)t64;
    const uint32_t id = id_at(a, t, tokens_in(a));
    const bool none = id >= a.vocab;
    constexpr int E = Elem<T>::kVec;
    const T *row = static_cast<const T *>(a.table) + (long long)(none ? 0 : id) * a.table_stride;
    T *out = static_cast<T *>(a.out) + (long long)t * a.out_stride;
    if constexpr (kWide) {
        const uint32_t nvec = a.dim / E, lo = piece * kEmbedVectors;
        const uint4 *rv = reinterpret_cast<const uint4 *>(row);
        uint4 *ov = reinterpret_cast<uint4 *>(out);
        uint4 v[kEmbedUnroll];
#pragma unroll
        for (int u = 0; u < kEmbedUnroll; ++u) {
            const uint32_t j = lo + u * 32 + lane;
            v[u] = make_uint4(0u, 0u, 0u, 0u);
            if (j < nvec && !none) v[u] = __ldg(rv + j);
        }
        const f32x2 sc = pack2(a.scale, a.scale);
#pragma unroll
        for (int u = 0; u < kEmbedUnroll; ++u) {
            const uint32_t j = lo + u * 32 + lane;
            if (j >= nvec) break;
            if (!none) {
#pragma unroll
                for (int k = 0; k < E / 2; ++k) {
                    float p, q;
                    unpack2(mul2(Elem<T>::pair(v[u], k), sc), p, q);
                    Elem<T>::put_pair(v[u], k, p, q);
                }
            }
            st_stream(ov + j, v[u]);
        }
        if (piece == pieces - 1 && lane < a.dim - nvec * E) {        // what does not fill a vector
            const uint32_t j = nvec * E + lane;
            out[j] = Elem<T>::from(none ? 0.0f : Elem<T>::load(row + j) * a.scale);
        }
    } else {
        const uint32_t lo = piece * kEmbedVectors * E, hi = min(a.dim, lo + kEmbedVectors * E);
        for (uint32_t j = lo + lane; j < hi; j += 32) out[j] = Elem<T>::from(none ? 0.0f : Elem<T>::load(row + j) * a.scale);
    }
}

// ---- sorting positions by id: least significant digit first, stable, so that the positions of one
// id stay in ascending order ----
constexpr int kSortBits = 9, kSortBins = 1 << kSortBits;

// Ranks of a block's entries among those of the same digit.  Entries are in registers, warp by warp, turn by turn,
// lane by lane; warp_bins[w][d] ends up as the number of entries with digit d in the warp.
template <int kItems, int kWarps, typename Count>
__device__ __forceinline__ void rank_digits(const uint32_t (&key)[kItems], uint32_t (&rank)[kItems], uint32_t in_mask, uint32_t shift,
                                            Count (*warp_bins)[kSortBins], uint32_t items) {
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    for (int b = lane; b < kSortBins; b += 32) warp_bins[warp][b] = 0;
    __syncwarp();
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        if ((uint32_t)k >= items) break;
        const bool in = (in_mask >> k) & 1u;
        const uint32_t d = in ? (key[k] >> shift) & (kSortBins - 1) : kSortBins;        // absent entries match only each other
        const uint32_t peers = __match_any_sync(kFullMask, d);
        const uint32_t before = in ? warp_bins[warp][d] : 0u;
        rank[k] = before + __popc(peers & ((1u << lane) - 1u));
        __syncwarp();
        if (in && lane == (uint32_t)__ffs(peers) - 1u) warp_bins[warp][d] = (Count)(before + __popc(peers));
        __syncwarp();
    }
}

// Exclusive sum over a block's first kSortBins threads; every thread of the block calls it.
__device__ __forceinline__ uint32_t scan_bins(uint32_t x, uint32_t *warp_sum) {
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    uint32_t scan = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t v = __shfl_up_sync(kFullMask, scan, o);
        if (lane >= (uint32_t)o) scan += v;
    }
    if (lane == 31 && warp < kSortBins / 32) warp_sum[warp] = scan;
    __syncthreads();
    uint32_t before = scan - x;
    for (uint32_t w = 0; w < min(warp, (uint32_t)(kSortBins / 32)); ++w) before += warp_sum[w];
    return before;
}

// Zeros at [p, p + bytes) by n threads, of which this is number i; p and bytes are multiples of 2.
__device__ __forceinline__ void fill_zero(uint8_t *p, size_t bytes, size_t i, size_t n) {
    const size_t head = min(bytes, (size_t)((16u - (reinterpret_cast<uintptr_t>(p) & 15u)) & 15u)), nvec = (bytes - head) / 16;
    for (size_t j = i; j < nvec; j += n) st_stream(p + head + j * 16, make_uint4(0u, 0u, 0u, 0u));
    const size_t tail = head + nvec * 16;
    if (i < head / 2) reinterpret_cast<uint16_t *>(p)[i] = 0;
    if (i < (bytes - tail) / 2) reinterpret_cast<uint16_t *>(p + tail)[i] = 0;
}

// One block sorts everything: up to 8192 positions, in shared memory.  Blocks beyond the first clear the gradient
// table meanwhile, where the launch has such blocks.
constexpr int kSmallThreads = 1024, kSmallItems = 8, kSmallWarps = kSmallThreads / 32;
constexpr uint32_t kSmallMax = kSmallThreads * kSmallItems;
constexpr size_t kSmallSmem = (size_t)kSmallWarps * kSortBins * 2 + kSmallMax * (4 + 2) + 64;

__global__ void __launch_bounds__(kSmallThreads) sort_small_kernel(const EmbedArgs a, uint32_t passes, uint32_t grad_size) {
    griddep_launch_dependents();
    griddep_wait();
    if (blockIdx.x > 0) {
        const size_t i = (size_t)(blockIdx.x - 1) * kSmallThreads + threadIdx.x, n = (size_t)(gridDim.x - 1) * kSmallThreads;
        uint8_t *t = static_cast<uint8_t *>(a.grad_table);
        const size_t row = (size_t)a.dim * grad_size, stride = (size_t)a.table_stride * grad_size;
        if (row == stride) return fill_zero(t, row * a.vocab, i, n);
        const size_t warp = i / 32, warps = n / 32, lane = threadIdx.x & 31u;
        for (size_t v = warp; v < a.vocab; v += warps) fill_zero(t + v * stride, row, lane, 32);
        return;
    }
    extern __shared__ __align__(16) uint8_t sort_smem[];
    uint16_t(*warp_bins)[kSortBins] = reinterpret_cast<uint16_t(*)[kSortBins]>(sort_smem);
    uint32_t *keys = reinterpret_cast<uint32_t *>(sort_smem + (size_t)kSmallWarps * kSortBins * 2);
    uint16_t *pos = reinterpret_cast<uint16_t *>(keys + kSmallMax);
    uint32_t *warp_sum = reinterpret_cast<uint32_t *>(pos + kSmallMax);
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    const uint32_t n = tokens_in(a), items = (a.n_tokens + kSmallThreads - 1) / kSmallThreads, base = warp * items * 32 + lane;
    if (a.present) {
        for (uint32_t w = threadIdx.x; w < (a.vocab + 31) / 32; w += kSmallThreads) a.present[w] = 0u;
        __syncthreads();
    }
    uint32_t key[kSmallItems], at[kSmallItems], rank[kSmallItems], in_mask = 0;
#pragma unroll
    for (int k = 0; k < kSmallItems; ++k) {
        if ((uint32_t)k >= items) break;
        at[k] = base + k * 32;
        if (at[k] < a.n_tokens) {
            in_mask |= 1u << k;
            key[k] = id_at(a, at[k], n);
            if (a.present && key[k] < a.vocab) atomicOr(a.present + (key[k] >> 5), 1u << (key[k] & 31u));
        }
    }
    for (uint32_t p = 0; p < passes; ++p) {
        if (p) {
#pragma unroll
            for (int k = 0; k < kSmallItems; ++k) {
                if ((uint32_t)k >= items) break;
                if ((in_mask >> k) & 1u) {
                    key[k] = keys[base + k * 32];
                    at[k] = pos[base + k * 32];
                }
            }
        }
        const uint32_t shift = p * kSortBits;
        rank_digits<kSmallItems, kSmallWarps>(key, rank, in_mask, shift, warp_bins, items);
        __syncthreads();
        uint32_t total = 0;
        if (threadIdx.x < kSortBins)
            for (int w = 0; w < kSmallWarps; ++w) {          // entries of the bin in earlier warps
                const uint32_t c = warp_bins[w][threadIdx.x];
                warp_bins[w][threadIdx.x] = (uint16_t)total;
                total += c;
            }
        const uint32_t start = scan_bins(total, warp_sum);
        if (threadIdx.x < kSortBins)
            for (int w = 0; w < kSmallWarps; ++w) warp_bins[w][threadIdx.x] = (uint16_t)(warp_bins[w][threadIdx.x] + start);
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kSmallItems; ++k) {
            if ((uint32_t)k >= items) break;
            if (!((in_mask >> k) & 1u)) continue;
            const uint32_t to = warp_bins[warp][(key[k] >> shift) & (kSortBins - 1)] + rank[k];
            if (p + 1 < passes) {
                keys[to] = key[k];
                pos[to] = (uint16_t)at[k];
            } else {
                a.keys[to] = key[k];
                a.pos[to] = at[k];
            }
        }
        __syncthreads();
    }
}

// More positions: tiles of kSortThreads * kItems entries.  A counting kernel for the first digit, then one
// placing kernel per digit, which counts the next digit where its entries go.
constexpr int kSortThreads = 512, kSortWarps = kSortThreads / 32;
static_assert(kSortBins == kSortThreads, "one thread per bin");

struct SortPass {
    uint32_t shift, first, last;         // first: keys come from the ids, positions are implicit
    uint32_t n_tiles, passes;
    uint32_t *counts;                    // [passes][n_tiles][kSortBins]
    const uint32_t *keys_in, *pos_in;
    uint32_t *keys_out, *pos_out;
};

template <int kItems>
__global__ void __launch_bounds__(kSortThreads) sort_count_kernel(const EmbedArgs a, const SortPass s) {
    griddep_launch_dependents();
    griddep_wait();
    __shared__ uint32_t bins[kSortBins];
    bins[threadIdx.x] = 0;
    __syncthreads();
    const uint32_t n = tokens_in(a), base = blockIdx.x * (kSortThreads * kItems);
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        const uint32_t i = base + k * kSortThreads + threadIdx.x;
        if (i < a.n_tokens) atomicAdd(&bins[id_at(a, i, n) & (kSortBins - 1)], 1u);
    }
    __syncthreads();
    s.counts[(size_t)blockIdx.x * kSortBins + threadIdx.x] = bins[threadIdx.x];
    // what the placing kernels add to
    for (uint32_t p = 1; p < s.passes; ++p) s.counts[((size_t)p * s.n_tiles + blockIdx.x) * kSortBins + threadIdx.x] = 0u;
    if (a.present)
        for (uint32_t w = blockIdx.x * kSortThreads + threadIdx.x; w < (a.vocab + 31) / 32; w += gridDim.x * kSortThreads) a.present[w] = 0u;
}

template <int kItems>
__global__ void __launch_bounds__(kSortThreads) sort_place_kernel(const EmbedArgs a, const SortPass s) {
    griddep_launch_dependents();
    griddep_wait();
    __shared__ uint32_t warp_bins[kSortWarps][kSortBins];
    __shared__ uint32_t warp_sum[kSortBins / 32];
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    const uint32_t pass = s.shift / kSortBits;
    // a warp owns kItems * 32 consecutive entries of the tile
    const uint32_t n = tokens_in(a), base = blockIdx.x * (kSortThreads * kItems) + warp * (kItems * 32) + lane;
    uint32_t key[kItems], at[kItems], rank[kItems], in_mask = 0;
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        at[k] = base + k * 32;
        key[k] = 0;
        if (at[k] < a.n_tokens) {
            in_mask |= 1u << k;
            key[k] = s.first ? id_at(a, at[k], n) : s.keys_in[at[k]];
            if (!s.first) at[k] = s.pos_in[at[k]];
        }
    }
    // thread b: entries of bin b in all tiles, and in the tiles before this one
    uint32_t total = 0, ahead = 0;
    const uint32_t *counts = s.counts + (size_t)pass * s.n_tiles * kSortBins + threadIdx.x;
#pragma unroll 8
    for (uint32_t tile = 0; tile < s.n_tiles; ++tile) {
        const uint32_t c = __ldcg(counts + (size_t)tile * kSortBins);
        if (tile < blockIdx.x) ahead += c;
        total += c;
    }
    rank_digits<kItems, kSortWarps>(key, rank, in_mask, s.shift, warp_bins, kItems);
    uint32_t start = scan_bins(total, warp_sum) + ahead;     // its barrier also ends the ranking
    for (int w = 0; w < kSortWarps; ++w) {
        const uint32_t c = warp_bins[w][threadIdx.x];
        warp_bins[w][threadIdx.x] = start;
        start += c;
    }
    __syncthreads();
    uint32_t *next = s.last ? nullptr : s.counts + (size_t)(pass + 1) * s.n_tiles * kSortBins;
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        if (!((in_mask >> k) & 1u)) continue;
        const uint32_t to = warp_bins[warp][(key[k] >> s.shift) & (kSortBins - 1)] + rank[k];
        s.keys_out[to] = key[k];
        s.pos_out[to] = at[k];
        if (next) atomicAdd(next + (size_t)(to / (kSortThreads * kItems)) * kSortBins + ((key[k] >> (s.shift + kSortBits)) & (kSortBins - 1)), 1u);
        if (s.first && a.present && key[k] < a.vocab) atomicOr(a.present + (key[k] >> 5), 1u << (key[k] & 31u));
    }
}

// ---- sums over the runs of equal ids ----
// kSumCols columns of a row per lane, kSumWarpCols per warp.  Wide: a lane's columns are consecutive, moved
// 16 bytes at a time; else the warp's lanes take turns, element by element.
constexpr int kSumThreads = 256, kSumCols = 8;
constexpr uint32_t kSumWarpCols = 32 * kSumCols;

template <typename T, bool kWide>
struct Columns {
    static constexpr int kVecs = kWide ? kSumCols / Elem<T>::kVec : 0;
    uint4 v[kWide ? kVecs : 1];
    float x[kWide ? 1 : kSumCols];
    // row: the warp's first column; n: columns of the row from there on
    __device__ __forceinline__ void load(const T *row, uint32_t lane, uint32_t n, bool on) {
        if constexpr (kWide) {
#pragma unroll
            for (int q = 0; q < kVecs; ++q) {
                v[q] = make_uint4(0u, 0u, 0u, 0u);
                if (on && lane * kSumCols < n) v[q] = *reinterpret_cast<const uint4 *>(row + lane * kSumCols + q * Elem<T>::kVec);
            }
        } else {
#pragma unroll
            for (int j = 0; j < kSumCols; ++j) x[j] = on && j * 32 + lane < n ? Elem<T>::load(row + j * 32 + lane) : 0.0f;
        }
    }
    __device__ __forceinline__ void add_to(f32x2 (&sum)[kSumCols / 2]) const {
        if constexpr (kWide) {
#pragma unroll
            for (int q = 0; q < kVecs; ++q)
#pragma unroll
                for (int k = 0; k < Elem<T>::kVec / 2; ++k) sum[q * Elem<T>::kVec / 2 + k] = add2(sum[q * Elem<T>::kVec / 2 + k], Elem<T>::pair(v[q], k));
        } else {
#pragma unroll
            for (int k = 0; k < kSumCols / 2; ++k) sum[k] = add2(sum[k], pack2(x[2 * k], x[2 * k + 1]));
        }
    }
    static __device__ __forceinline__ void store(T *row, const f32x2 (&sum)[kSumCols / 2], uint32_t lane, uint32_t n) {
        if constexpr (kWide) {
            if (lane * kSumCols >= n) return;
#pragma unroll
            for (int q = 0; q < kVecs; ++q) {
                uint4 o;
#pragma unroll
                for (int k = 0; k < Elem<T>::kVec / 2; ++k) {
                    float a, b;
                    unpack2(sum[q * Elem<T>::kVec / 2 + k], a, b);
                    Elem<T>::put_pair(o, k, a, b);
                }
                st_stream(row + lane * kSumCols + q * Elem<T>::kVec, o);
            }
        } else {
#pragma unroll
            for (int k = 0; k < kSumCols / 2; ++k) {
                float a, b;
                unpack2(sum[k], a, b);
                if (2 * k * 32 + lane < n) row[2 * k * 32 + lane] = Elem<T>::from(a);
                if ((2 * k + 1) * 32 + lane < n) row[(2 * k + 1) * 32 + lane] = Elem<T>::from(b);
            }
        }
    }
};

// scale * sum to row v of the gradient table, or added to what is there
template <typename G, bool kWide>
__device__ __forceinline__ void write_row(const EmbedArgs &a, uint32_t v, const f32x2 (&sum)[kSumCols / 2], uint32_t c0, uint32_t lane) {
    G *row = static_cast<G *>(a.grad_table) + (long long)v * a.table_stride + c0;
    f32x2 x[kSumCols / 2];
    const f32x2 sc = pack2(a.scale, a.scale);
#pragma unroll
    for (int k = 0; k < kSumCols / 2; ++k) x[k] = mul2(sum[k], sc);
    if (a.accumulate) {
        Columns<G, kWide> old;
        old.load(row, lane, a.dim - c0, true);
        old.add_to(x);
    }
    Columns<G, kWide>::store(row, x, lane, a.dim - c0);
}

__device__ __forceinline__ float *partial_row(const EmbedArgs &a, uint32_t which, uint32_t chunk) {
    return a.partial + ((size_t)which * a.n_chunks + chunk) * a.partial_stride;
}

// Rows of the gradient table whose bit in a.present is not set, 32 per block.
template <typename G>
__device__ __forceinline__ void zero_rows(const EmbedArgs &a, uint32_t word) {
    const uint32_t bits = a.present[word], lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    for (uint32_t k = warp; k < 32 && word * 32 + k < a.vocab; k += kSumThreads / 32)
        if (!((bits >> k) & 1u))
            fill_zero(reinterpret_cast<uint8_t *>(static_cast<G *>(a.grad_table) + (long long)(word * 32 + k) * a.table_stride), (size_t)a.dim * sizeof(G), lane, 32);
}

// A warp per (chunk of sorted positions, 256 columns).  A run that lies inside the chunk is written out; the part of
// a run that began in an earlier chunk goes to partial 0, the part of one that began here and goes on to
// partial 1.  Spread among the blocks that do this, as many as a.present has words clear rows without a token.
template <typename T, typename G, bool kWide>
__global__ void __launch_bounds__(kSumThreads) embed_sum_kernel(const EmbedArgs a, uint32_t slices, uint32_t sum_blocks) {
    griddep_launch_dependents();
    griddep_wait();
    const uint32_t sums_before = (uint32_t)((unsigned long long)blockIdx.x * sum_blocks / gridDim.x);
    if ((uint32_t)((unsigned long long)(blockIdx.x + 1ull) * sum_blocks / gridDim.x) == sums_before)
        return zero_rows<G>(a, blockIdx.x - sums_before);
    const unsigned long long item = (unsigned long long)sums_before * (kSumThreads / 32) + (threadIdx.x >> 5);
    const unsigned long long chunk64 = item / slices;
    if (chunk64 >= a.n_chunks) return;
    const uint32_t chunk = (uint32_t)chunk64, lane = threadIdx.x & 31u;
    const uint32_t c0 = (uint32_t)(item % slices) * kSumWarpCols, cols = a.dim - c0;
    const uint32_t lo = chunk * a.rows_per_chunk, hi = min(a.n_tokens, lo + a.rows_per_chunk);
    const uint32_t first = a.keys[lo];
    if (first >= a.vocab) return;                            // sorted behind all ids
    bool cont = lo > 0 && a.keys[lo - 1] == first;
    f32x2 sum[kSumCols / 2];
    auto clear = [&]() {
#pragma unroll
        for (int k = 0; k < kSumCols / 2; ++k) sum[k] = pack2(0.0f, 0.0f);
    };
    clear();
    uint32_t v = first;
    const T *in = static_cast<const T *>(a.grad_out) + c0;
    constexpr int kRows = kWide && sizeof(T) == 2 ? 8 : 4;   // rows on their way at a time
    for (uint32_t e0 = lo; e0 < hi; e0 += 32) {
        const uint32_t left = min(hi - e0, 32u);
        const uint32_t my_key = lane < left ? a.keys[e0 + lane] : a.vocab, my_pos = lane < left ? a.pos[e0 + lane] : 0u;
        for (uint32_t k0 = 0; k0 < left; k0 += kRows) {
            Columns<T, kWide> x[kRows];
#pragma unroll
            for (int u = 0; u < kRows; ++u) {
                const uint32_t key = __shfl_sync(kFullMask, my_key, k0 + u), p = __shfl_sync(kFullMask, my_pos, k0 + u);
                x[u].load(in + (long long)p * a.out_stride, lane, cols, key < a.vocab);
            }
#pragma unroll
            for (int u = 0; u < kRows; ++u) {
                const uint32_t key = __shfl_sync(kFullMask, my_key, k0 + u);
                if (k0 + u >= left) break;
                if (key != v) {                              // the run of v ends here
                    if (v < a.vocab) {
                        if (cont) Columns<float, kWide>::store(partial_row(a, 0, chunk) + c0, sum, lane, cols);
                        else write_row<G, kWide>(a, v, sum, c0, lane);
                    }
                    cont = false;
                    v = key;
                    clear();
                }
                x[u].add_to(sum);
            }
        }
    }
    if (v >= a.vocab) return;
    const bool goes_on = hi < a.n_tokens && a.keys[hi] == v;
    if (cont) Columns<float, kWide>::store(partial_row(a, 0, chunk) + c0, sum, lane, cols);
    else if (goes_on) Columns<float, kWide>::store(partial_row(a, 1, chunk) + c0, sum, lane, cols);
    else write_row<G, kWide>(a, v, sum, c0, lane);
}

// Runs that chunk borders cut: the block of the chunk a run begins in adds the parts up.  Up to kJoinAlone parts one
// warp adds in order, a slice of columns each; more are cut into one piece per warp, and the pieces' sums added
// in order.
constexpr uint32_t kJoinAlone = 8;
template <typename G, bool kWide>
__global__ void __launch_bounds__(kSumThreads) embed_join_kernel(const EmbedArgs a, uint32_t slices) {
    griddep_launch_dependents();
    griddep_wait();
    constexpr uint32_t kWarps = kSumThreads / 32;
    __shared__ f32x2 piece[kWarps][kSumCols / 2][32];
    const uint32_t chunk = blockIdx.x, lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    const uint32_t lo = chunk * a.rows_per_chunk;
    const unsigned long long hi = (unsigned long long)lo + a.rows_per_chunk;
    if (hi >= a.n_tokens) return;
    const uint32_t v = a.keys[hi - 1];
    if (v >= a.vocab || a.keys[hi] != v || (lo > 0 && a.keys[lo - 1] == v)) return;      // ends here, or began earlier
    // chunks behind this one that begin with v
    uint32_t parts = 0;
    for (;;) {
        const unsigned long long c = (unsigned long long)chunk + 1 + parts + lane;
        const uint32_t same = __ballot_sync(kFullMask, c < a.n_chunks && a.keys[c * a.rows_per_chunk] == v);
        if (same == kFullMask) { parts += 32; continue; }
        parts += __ffs(~same) - 1;
        break;
    }
    auto add_parts = [&](f32x2 (&sum)[kSumCols / 2], uint32_t from, uint32_t to, uint32_t c0) {
        for (uint32_t p = from; p < to; p += 4) {
            Columns<float, kWide> x[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) x[u].load(partial_row(a, 0, chunk + 1 + min(p + u, to - 1)) + c0, lane, a.dim - c0, p + u < to);
#pragma unroll
            for (int u = 0; u < 4; ++u) x[u].add_to(sum);
        }
    };
    const bool alone = parts <= kJoinAlone;
    for (uint32_t s = alone ? warp : 0; s < slices; s += alone ? kWarps : 1) {
        const uint32_t c0 = s * kSumWarpCols;
        f32x2 sum[kSumCols / 2];
#pragma unroll
        for (int k = 0; k < kSumCols / 2; ++k) sum[k] = pack2(0.0f, 0.0f);
        if (alone || warp == 0) {
            Columns<float, kWide> x;
            x.load(partial_row(a, 1, chunk) + c0, lane, a.dim - c0, true);
            x.add_to(sum);
        }
        if (alone) {
            add_parts(sum, 0, parts, c0);
            write_row<G, kWide>(a, v, sum, c0, lane);
            continue;
        }
        add_parts(sum, (uint32_t)((unsigned long long)parts * warp / kWarps), (uint32_t)((unsigned long long)parts * (warp + 1) / kWarps), c0);
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kSumCols / 2; ++k) piece[warp][k][lane] = sum[k];
        __syncthreads();
        if (warp == 0) {
            for (uint32_t w = 1; w < kWarps; ++w)
#pragma unroll
                for (int k = 0; k < kSumCols / 2; ++k) sum[k] = add2(sum[k], piece[w][k][lane]);
            write_row<G, kWide>(a, v, sum, c0, lane);
        }
    }
}

}  // namespace td
