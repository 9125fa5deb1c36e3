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
    float *partial;                      // [2][n_chunks][dim]: sums of a run cut by the chunk's start / by its end
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
constexpr int kSortThreads = 512, kSortItems = 8;
constexpr uint32_t kSortTile = kSortThreads * kSortItems;
constexpr int kSortBits = 9, kSortBins = 1 << kSortBits;
constexpr int kSortWarps = kSortThreads / 32;

struct SortPass {
    uint32_t shift, first;               // first pass: keys come from the ids, positions are implicit
    uint32_t n_tiles;
    uint32_t *counts;                    // [n_tiles][kSortBins]
    const uint32_t *keys_in, *pos_in;
    uint32_t *keys_out, *pos_out;
};

__device__ __forceinline__ uint32_t sort_key(const EmbedArgs &a, const SortPass &s, uint32_t i, uint32_t n) {
    return s.first ? id_at(a, i, n) : s.keys_in[i];
}

__global__ void __launch_bounds__(kSortThreads) sort_count_kernel(const EmbedArgs a, const SortPass s) {
    griddep_launch_dependents();
    griddep_wait();
    __shared__ uint32_t bins[kSortBins];
    for (int b = threadIdx.x; b < kSortBins; b += kSortThreads) bins[b] = 0;
    __syncthreads();
    const uint32_t n = tokens_in(a), base = blockIdx.x * kSortTile;
#pragma unroll
    for (int k = 0; k < kSortItems; ++k) {
        const uint32_t i = base + k * kSortThreads + threadIdx.x;
        if (i < a.n_tokens) atomicAdd(&bins[(sort_key(a, s, i, n) >> s.shift) & (kSortBins - 1)], 1u);
    }
    __syncthreads();
    for (int b = threadIdx.x; b < kSortBins; b += kSortThreads) s.counts[(size_t)blockIdx.x * kSortBins + b] = bins[b];
}

__global__ void __launch_bounds__(kSortThreads) sort_place_kernel(const EmbedArgs a, const SortPass s) {
    griddep_launch_dependents();
    griddep_wait();
    static_assert(kSortBins == kSortThreads, "one thread per bin");
    __shared__ uint32_t warp_bins[kSortWarps][kSortBins];
    __shared__ uint32_t warp_sum[kSortWarps];
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    for (int b = lane; b < kSortBins; b += 32) warp_bins[warp][b] = 0;
    __syncwarp();
    // a warp owns kSortItems * 32 consecutive entries of the tile
    const uint32_t n = tokens_in(a), base = blockIdx.x * kSortTile + warp * (kSortItems * 32);
    uint32_t key[kSortItems], at[kSortItems], rank[kSortItems];
#pragma unroll
    for (int k = 0; k < kSortItems; ++k) {
        const uint32_t i = base + k * 32 + lane;
        key[k] = i < a.n_tokens ? sort_key(a, s, i, n) : 0u;
        at[k] = s.first || i >= a.n_tokens ? i : s.pos_in[i];
    }
#pragma unroll
    for (int k = 0; k < kSortItems; ++k) {
        const bool in = base + k * 32 + lane < a.n_tokens;
        const uint32_t d = in ? (key[k] >> s.shift) & (kSortBins - 1) : kSortBins;      // absent entries match only each other
        const uint32_t peers = __match_any_sync(kFullMask, d);
        const uint32_t before = in ? warp_bins[warp][d] : 0u;
        rank[k] = before + __popc(peers & ((1u << lane) - 1u));
        __syncwarp();
        if (in && lane == (uint32_t)__ffs(peers) - 1u) warp_bins[warp][d] = before + __popc(peers);
        __syncwarp();
    }
    __syncthreads();
    // thread b: where bin b of this tile starts in the output
    const uint32_t b = threadIdx.x;
    uint32_t total = 0, ahead = 0;
    for (uint32_t tile = 0; tile < s.n_tiles; ++tile) {
        const uint32_t c = __ldcg(s.counts + (size_t)tile * kSortBins + b);
        if (tile < blockIdx.x) ahead += c;
        total += c;
    }
    uint32_t scan = total;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t v = __shfl_up_sync(kFullMask, scan, o);
        if (lane >= (uint32_t)o) scan += v;
    }
    if (lane == 31) warp_sum[warp] = scan;
    __syncthreads();
    uint32_t start = scan - total + ahead;
    for (uint32_t w = 0; w < warp; ++w) start += warp_sum[w];
    for (int w = 0; w < kSortWarps; ++w) {
        const uint32_t c = warp_bins[w][b];
        warp_bins[w][b] = start;
        start += c;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kSortItems; ++k) {
        const uint32_t i = base + k * 32 + lane;
        if (i >= a.n_tokens) continue;
        const uint32_t to = warp_bins[warp][(key[k] >> s.shift) & (kSortBins - 1)] + rank[k];
        s.keys_out[to] = key[k];
        s.pos_out[to] = at[k];
    }
}

// ---- sums over the runs of equal ids ----
// Row v of the gradient table, columns [c0, c0 + kCols) of this lane.
template <typename T, int kCols>
struct Columns {
    static __device__ __forceinline__ void load(float (&x)[kCols], const T *row, uint32_t c0, uint32_t dim, bool wide) {
        if (wide) {
            constexpr int E = Elem<T>::kVec;
#pragma unroll
            for (int q = 0; q < kCols / E; ++q) {
                const uint4 v = *reinterpret_cast<const uint4 *>(row + c0 + q * E);
#pragma unroll
                for (int k = 0; k < E / 2; ++k) unpack2(Elem<T>::pair(v, k), x[q * E + 2 * k], x[q * E + 2 * k + 1]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < kCols; ++j) x[j] = c0 + j < dim ? Elem<T>::load(row + c0 + j) : 0.0f;
        }
    }
    static __device__ __forceinline__ void store(T *row, const float (&x)[kCols], uint32_t c0, uint32_t dim, bool wide) {
        if (wide) {
            constexpr int E = Elem<T>::kVec;
#pragma unroll
            for (int q = 0; q < kCols / E; ++q) {
                uint4 v;
#pragma unroll
                for (int k = 0; k < E / 2; ++k) Elem<T>::put_pair(v, k, x[q * E + 2 * k], x[q * E + 2 * k + 1]);
                st_stream(row + c0 + q * E, v);
            }
        } else {
#pragma unroll
            for (int j = 0; j < kCols; ++j)
                if (c0 + j < dim) row[c0 + j] = Elem<T>::from(x[j]);
        }
    }
};

constexpr int kSumThreads = 256, kSumCols = 8;               // columns per lane: a warp covers 256
constexpr uint32_t kSumWarpCols = 32 * kSumCols;

template <typename G>
__device__ __forceinline__ void write_row(const EmbedArgs &a, uint32_t v, const float (&sum)[kSumCols], uint32_t c0, bool wide) {
    G *row = static_cast<G *>(a.grad_table) + (long long)v * a.table_stride;
    float x[kSumCols];
#pragma unroll
    for (int j = 0; j < kSumCols; ++j) x[j] = sum[j] * a.scale;
    if (a.accumulate) {
        float old[kSumCols];
        Columns<G, kSumCols>::load(old, row, c0, a.dim, wide);
#pragma unroll
        for (int j = 0; j < kSumCols; ++j) x[j] += old[j];
    }
    Columns<G, kSumCols>::store(row, x, c0, a.dim, wide);
}

__device__ __forceinline__ float *partial_row(const EmbedArgs &a, uint32_t which, uint32_t chunk) {
    return a.partial + ((size_t)which * a.n_chunks + chunk) * a.dim;
}

// A warp per (chunk of sorted positions, 256 columns).  A run that lies inside the chunk is written
// out; the part of a run that began in an earlier chunk goes to partial 0, the part of one that
// began here and goes on to partial 1.
template <typename T, typename G>
__global__ void __launch_bounds__(kSumThreads) embed_sum_kernel(const EmbedArgs a, uint32_t slices, bool wide_in, bool wide_out) {
    griddep_launch_dependents();
    griddep_wait();
    const unsigned long long item = (unsigned long long)blockIdx.x * (kSumThreads / 32) + (threadIdx.x >> 5);
    const unsigned long long chunk64 = item / slices;
    if (chunk64 >= a.n_chunks) return;
    const uint32_t chunk = (uint32_t)chunk64, lane = threadIdx.x & 31u;
    const uint32_t c0 = (uint32_t)(item % slices) * kSumWarpCols + lane * kSumCols;
    const bool full = c0 + kSumCols <= a.dim;                // this lane's columns all exist
    const uint32_t lo = chunk * a.rows_per_chunk, hi = min(a.n_tokens, lo + a.rows_per_chunk);
    const uint32_t first = a.keys[lo];
    if (first >= a.vocab) return;                            // sorted behind all ids
    bool cont = lo > 0 && a.keys[lo - 1] == first;
    float sum[kSumCols];
#pragma unroll
    for (int j = 0; j < kSumCols; ++j) sum[j] = 0.0f;
    uint32_t v = first;
    for (uint32_t e0 = lo; e0 < hi; e0 += 32) {
        const uint32_t left = min(hi - e0, 32u);
        const uint32_t my_key = lane < left ? a.keys[e0 + lane] : a.vocab, my_pos = lane < left ? a.pos[e0 + lane] : 0u;
        for (uint32_t k0 = 0; k0 < left; k0 += 4) {
            float x[4][kSumCols];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const uint32_t key = __shfl_sync(kFullMask, my_key, (k0 + u) & 31u), p = __shfl_sync(kFullMask, my_pos, (k0 + u) & 31u);
#pragma unroll
                for (int j = 0; j < kSumCols; ++j) x[u][j] = 0.0f;
                if (k0 + u < left && key < a.vocab && c0 < a.dim)
                    Columns<T, kSumCols>::load(x[u], static_cast<const T *>(a.grad_out) + (long long)p * a.out_stride, c0, a.dim, wide_in && full);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (k0 + u >= left) break;
                const uint32_t key = __shfl_sync(kFullMask, my_key, (k0 + u) & 31u);
                if (key != v) {                              // the run of v ends here
                    if (c0 < a.dim && v < a.vocab) {
                        if (cont) Columns<float, kSumCols>::store(partial_row(a, 0, chunk), sum, c0, a.dim, full && (a.dim & 3u) == 0);
                        else write_row<G>(a, v, sum, c0, wide_out && full);
                    }
                    cont = false;
                    v = key;
#pragma unroll
                    for (int j = 0; j < kSumCols; ++j) sum[j] = 0.0f;
                }
#pragma unroll
                for (int j = 0; j < kSumCols; ++j) sum[j] += x[u][j];
            }
        }
    }
    if (v >= a.vocab || c0 >= a.dim) return;
    const bool goes_on = hi < a.n_tokens && a.keys[hi] == v;
    if (cont) Columns<float, kSumCols>::store(partial_row(a, 0, chunk), sum, c0, a.dim, full && (a.dim & 3u) == 0);
    else if (goes_on) Columns<float, kSumCols>::store(partial_row(a, 1, chunk), sum, c0, a.dim, full && (a.dim & 3u) == 0);
    else write_row<G>(a, v, sum, c0, wide_out && full);
}

// Runs that chunk borders cut: the chunk a run begins in adds the parts up in order.
template <typename G>
__global__ void __launch_bounds__(kSumThreads) embed_join_kernel(const EmbedArgs a, uint32_t slices, bool wide_out) {
    griddep_launch_dependents();
    griddep_wait();
    const unsigned long long item = (unsigned long long)blockIdx.x * (kSumThreads / 32) + (threadIdx.x >> 5);
    const unsigned long long chunk64 = item / slices;
    if (chunk64 >= a.n_chunks) return;
    const uint32_t chunk = (uint32_t)chunk64, lane = threadIdx.x & 31u;
    const uint32_t c0 = (uint32_t)(item % slices) * kSumWarpCols + lane * kSumCols;
    const uint32_t lo = chunk * a.rows_per_chunk;
    const unsigned long long hi = (unsigned long long)lo + a.rows_per_chunk;
    if (hi >= a.n_tokens) return;
    const uint32_t v = a.keys[hi - 1];
    if (v >= a.vocab || a.keys[hi] != v || (lo > 0 && a.keys[lo - 1] == v)) return;      // ends here, or began earlier
    if (c0 >= a.dim) return;
    const bool full = c0 + kSumCols <= a.dim, wide = full && (a.dim & 3u) == 0;
    float sum[kSumCols], x[kSumCols];
    Columns<float, kSumCols>::load(sum, partial_row(a, 1, chunk), c0, a.dim, wide);
    for (uint32_t c = chunk + 1; c < a.n_chunks && a.keys[(size_t)c * a.rows_per_chunk] == v; ++c) {
        Columns<float, kSumCols>::load(x, partial_row(a, 0, c), c0, a.dim, wide);
#pragma unroll
        for (int j = 0; j < kSumCols; ++j) sum[j] += x[j];
    }
    write_row<G>(a, v, sum, c0, wide_out && full);
}

// Rows of the gradient table that no token has.
template <typename G>
__global__ void __launch_bounds__(kSumThreads) embed_zero_kernel(const EmbedArgs a, bool wide_out) {
    griddep_launch_dependents();
    griddep_wait();
    constexpr uint32_t kRows = 32;
    __shared__ uint32_t present;
    const uint32_t v0 = blockIdx.x * kRows;
    if (threadIdx.x < 32) {
        const uint32_t v = v0 + threadIdx.x;
        uint32_t lo = 0, hi = a.n_tokens;                    // first entry with key >= v
        while (lo < hi) {
            const uint32_t mid = lo + (hi - lo) / 2;
            if (a.keys[mid] < v) lo = mid + 1; else hi = mid;
        }
        const uint32_t bits = __ballot_sync(kFullMask, lo < a.n_tokens && a.keys[lo] == v);
        if (threadIdx.x == 0) present = bits;
    }
    __syncthreads();
    const uint32_t bits = present;
    constexpr int E = Elem<G>::kVec;
    for (uint32_t k = 0; k < kRows && v0 + k < a.vocab; ++k) {
        if ((bits >> k) & 1u) continue;
        G *row = static_cast<G *>(a.grad_table) + (long long)(v0 + k) * a.table_stride;
        uint32_t done = 0;
        if (wide_out) {
            const uint32_t nvec = a.dim / E;
            for (uint32_t j = threadIdx.x; j < nvec; j += kSumThreads) st_stream(reinterpret_cast<uint4 *>(row) + j, make_uint4(0u, 0u, 0u, 0u));
            done = nvec * E;
        }
        for (uint32_t j = done + threadIdx.x; j < a.dim; j += kSumThreads) row[j] = Elem<G>::from(0.0f);
    }
}

}  // namespace td
