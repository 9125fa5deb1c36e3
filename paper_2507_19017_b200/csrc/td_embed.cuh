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
    uint32_t accumulate, grad_size;      // bytes of a gradient element
    uint32_t rows_per_chunk;             // sorted positions per chunk of the segment sums
    uint32_t n_chunks;
    uint32_t *keys;                      // [n_tokens] sorted ids; vocab: no token
    uint32_t *pos;                       // [n_tokens] their positions
    uint32_t *present;                   // [ceil(vocab / 32)] a bit per id that occurs, or nullptr: found in the keys
    float *partial;                      // [2][n_chunks][partial_stride]: sums of a run cut by the chunk's start / by its end
    size_t partial_stride;               // dim rounded up to a warp's columns
    uint32_t *arrived;                   // [3][n_chunks][slices] parts, and groups of parts, stored of cut runs
    uint32_t n_arrived, zero_from;       // blocks of zero_rows that ran before the sums
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
    const int32_t id = a.ids[t];
    if (id < 0) return a.vocab;
    if ((uint32_t)id >= a.vocab) {
        if (a.status) atomicOr(a.status, TD_ERR_OOB_INDEX);
        return a.vocab;
    }
    return (uint32_t)id;
}

// Bound by writing the rows: 65536 rows of 4096 bfloat16 in 120 us, 5.9 TB/s; of 4095, where every vector is shifted, 171 us;
// 64 rows 1.8 us.  A team of 2^team lanes (4 to 32) per piece of a position's row; a lane moves kEmbedUnroll vectors of 16 bytes, the
// team's lanes taking turns.  Aligned: rows of both sides start on 16-byte boundaries.  Else the vectors are
// aligned on the output row and put together from two loads each, and the first piece's lanes move the elements
// before the first and behind the last vector.
constexpr int kEmbedThreads = 256, kEmbedUnroll = 4;

template <typename T, bool kAligned>
__global__ void __launch_bounds__(kEmbedThreads) embed_kernel(const EmbedArgs a, uint32_t team, uint32_t pieces) {
    griddep_launch_dependents();
    griddep_wait();
    constexpr int E = Elem<T>::kVec;
    const uint32_t lanes = 1u << team, lane = threadIdx.x & (lanes - 1u);
    unsigned long long t64 = (unsigned long long)blockIdx.x * (kEmbedThreads >> team) + (threadIdx.x >> team);
    uint32_t piece = 0;
    if (pieces > 1) {
        piece = (uint32_t)(t64 % pieces);
        t64 /= pieces;
    }
    if (t64 >= a.n_tokens) return;
    const uint32_t t = (uint32_t)t64;
    const uint32_t id = id_at(a, t, tokens_in(a));
    const bool none = id >= a.vocab;
    const T *table = static_cast<const T *>(a.table), *row = table + (long long)(none ? 0u : id) * a.table_stride;
    T *out = static_cast<T *>(a.out) + (long long)t * a.out_stride;
    const uint32_t head = kAligned ? 0u : min((16u - (uint32_t)(reinterpret_cast<uintptr_t>(out) & 15u)) % 16u / (uint32_t)sizeof(T), a.dim);
    const uint32_t nvec = (a.dim - head) / E, lo = piece * (kEmbedUnroll << team);
    uint4 v[kEmbedUnroll];
    if constexpr (kAligned) {
#pragma unroll
        for (int u = 0; u < kEmbedUnroll; ++u) {
            const uint32_t j = lo + (u << team) + lane;
            v[u] = make_uint4(0u, 0u, 0u, 0u);
            if (j < nvec && !none) v[u] = reinterpret_cast<const uint4 *>(row)[j];
        }
    } else {
        const T *end = table + (long long)(a.vocab - 1) * a.table_stride + a.dim;
        const bool edge = id == 0 || id == a.vocab - 1;
        Window<T> w[kEmbedUnroll];
#pragma unroll
        for (int u = 0; u < kEmbedUnroll; ++u) {
            const uint32_t j = lo + (u << team) + lane;
            if (j < nvec && !none) w[u].open(row + head + j * E, table, end, edge);
        }
#pragma unroll
        for (int u = 0; u < kEmbedUnroll; ++u) {
            const uint32_t j = lo + (u << team) + lane;
            v[u] = make_uint4(0u, 0u, 0u, 0u);
            if (j < nvec && !none) v[u] = w[u].close(row + head + j * E);
        }
    }
    const f32x2 sc = pack2(a.scale, a.scale);
#pragma unroll
    for (int u = 0; u < kEmbedUnroll; ++u) {
        const uint32_t j = lo + (u << team) + lane;
        if (j >= nvec) break;
        if (!none)                       // zeros stay zeros, whatever the scale's sign or value
#pragma unroll
            for (int k = 0; k < E / 2; ++k) {
                float p, q;
                unpack2(mul2(Elem<T>::pair(v[u], k), sc), p, q);
                Elem<T>::put_pair(v[u], k, p, q);
            }
        st_stream(out + head + j * E, v[u]);
    }
    if (piece == 0) {
        const uint32_t tail = head + nvec * E, loose = head + (a.dim - tail);
        for (uint32_t i = lane; i < loose; i += lanes) {
            const uint32_t j = i < head ? i : tail + i - head;
            out[j] = Elem<T>::from(none ? 0.0f : Elem<T>::load(row + j) * a.scale);
        }
    }
}

// ---- sorting positions by id: least significant digit first, stable, so that the positions of one
// id stay in ascending order ----
constexpr int kSortBits = 9, kSortBins = 1 << kSortBits;

// Ranks of a block's entries among those of the same digit.  Entries are in registers, warp by warp, turn by turn,
// lane by lane; warp_bins[w][d] ends up as the number of entries with digit d in the warp.
template <int kItems>
__device__ __forceinline__ void rank_digits(const uint32_t (&key)[kItems], uint32_t (&rank)[kItems], uint32_t in_mask, uint32_t shift,
                                            uint32_t (*warp_bins)[kSortBins]) {
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    for (int b = lane; b < kSortBins; b += 32) warp_bins[warp][b] = 0;
    __syncwarp();
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        const bool in = (in_mask >> k) & 1u;
        const uint32_t d = (key[k] >> shift) & (kSortBins - 1);
        // lanes with the same digit, one vote per bit (a match instruction took 300 to 400 cycles here)
        uint32_t peers = __ballot_sync(kFullMask, in);
#pragma unroll
        for (int b = 0; b < kSortBits; ++b) {
            const bool set = (d >> b) & 1u;
            const uint32_t v = __ballot_sync(kFullMask, set);
            peers &= set ? v : ~v;
        }
        const uint32_t before = in ? warp_bins[warp][d] : 0u;
        rank[k] = before + __popc(peers & ((1u << lane) - 1u));
        __syncwarp();
        if (in && lane == (uint32_t)__ffs(peers) - 1u) warp_bins[warp][d] = before + __popc(peers);
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

constexpr uint32_t kZeroWords = 8;       // words of a.present per block, where rows are short

// Zeros at [p, p + bytes) by n threads, of which this is number i; p and bytes are multiples of 2.
__device__ __forceinline__ void fill_zero(uint8_t *p, size_t bytes, size_t i, size_t n) {
    const size_t head = min(bytes, (size_t)((16u - (reinterpret_cast<uintptr_t>(p) & 15u)) & 15u)), nvec = (bytes - head) / 16;
    for (size_t j = i; j < nvec; j += n) st_stream(p + head + j * 16, make_uint4(0u, 0u, 0u, 0u));
    const size_t tail = head + nvec * 16;
    if (i < head / 2) reinterpret_cast<uint16_t *>(p)[i] = 0;
    if (i < (bytes - tail) / 2) reinterpret_cast<uint16_t *>(p + tail)[i] = 0;
}

// Clears the rows of the gradient table whose bit in a.present is not set.  Long rows: the block takes 32 rows,
// a warp at a time one of them.  Short ones: every warp takes 32, neighbours without a gap between them at once.
constexpr uint32_t kLongRow = 1024;      // bytes
__device__ __forceinline__ bool long_rows(const EmbedArgs &a) { return a.dim * (unsigned long long)a.grad_size >= kLongRow; }
__device__ __forceinline__ void zero_rows(const EmbedArgs &a, uint32_t block, const uint32_t *present) {       // the block's words
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    const size_t row = (size_t)a.dim * a.grad_size, stride = (size_t)a.table_stride * a.grad_size;
    uint8_t *table = static_cast<uint8_t *>(a.grad_table);
    if (long_rows(a)) {
        const uint32_t bits = present[0];
        for (uint32_t k = warp; k < 32 && block * 32 + k < a.vocab; k += blockDim.x >> 5)
            if (!((bits >> k) & 1u)) fill_zero(table + (size_t)(block * 32 + k) * stride, row, lane, 32);
        return;
    }
    const uint32_t word = block * kZeroWords + warp;
    if (warp >= kZeroWords || word >= (a.vocab + 31) / 32) return;
    const uint32_t rows = min(32u, a.vocab - word * 32);
    uint32_t absent = ~present[warp] & (rows == 32 ? kFullMask : (1u << rows) - 1u);
    while (absent) {
        const uint32_t from = __ffs(absent) - 1, free = ~(absent >> from), n = row == stride ? (free ? __ffs(free) - 1 : 32) : 1;
        fill_zero(table + (size_t)(word * 32 + from) * stride, row * n, lane, 32);
        absent &= from + n >= 32 ? 0u : kFullMask << (from + n);
    }
}
__device__ __forceinline__ uint32_t zero_words(const EmbedArgs &a) { return long_rows(a) ? 1u : kZeroWords; }       // per block

// The bits of the block's rows, from the sorted keys; for all threads of a block of kSumThreads.
constexpr int kSumThreads = 256, kSumWarps = kSumThreads / 32;
__device__ __forceinline__ void present_in_keys(const EmbedArgs &a, uint32_t block, uint32_t *bits) {
    const uint32_t v0 = block * zero_words(a) * 32, v1 = v0 + zero_words(a) * 32;
    if (threadIdx.x < kZeroWords) bits[threadIdx.x] = 0u;
    uint32_t lo = 0, hi = a.n_tokens;                        // the first entry that is not below v0 lies in [lo, hi]
    while (lo < hi) {
        const uint32_t step = (hi - lo + kSumThreads - 1) / kSumThreads, at = lo + threadIdx.x * step;
        const uint32_t below = __syncthreads_count(at < hi && a.keys[at] < v0);
        if (below == 0) break;
        hi = min(hi, lo + below * step);
        lo += (below - 1) * step + 1;
    }
    for (uint32_t e = lo + threadIdx.x;; e += kSumThreads) {
        const uint32_t id = e < a.n_tokens ? a.keys[e] : a.vocab;
        const bool in = id < min(v1, a.vocab);
        if (in) atomicOr(bits + (id - v0) / 32, 1u << ((id - v0) & 31u));
        if (__syncthreads_count(in) < kSumThreads) break;
    }
}

// Up to kRankMax positions: a position's place among the sorted ones is the number of smaller ids, and of equal ids at
// earlier positions.  A block counts it for 32 positions, one per lane, its warps going through a share of all ids
// each.  positions^2 comparisons: 4000 positions 6 us, 8192 15 us, where sorting by digits takes 17 for any number.
constexpr int kRankThreads = 1024, kRankWarps = kRankThreads / 32;
constexpr uint32_t kRankMax = 8192;

__global__ void __launch_bounds__(kRankThreads) embed_rank_kernel(const EmbedArgs a) {
    griddep_launch_dependents();
    griddep_wait();
    __shared__ __align__(16) uint32_t ids[kRankMax];
    __shared__ uint32_t place[32];
    const uint32_t n = tokens_in(a), lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    for (uint32_t w = blockIdx.x * kRankThreads + threadIdx.x; w < a.n_arrived; w += gridDim.x * kRankThreads) a.arrived[w] = 0u;
    const uint32_t padded = (a.n_tokens + 3) & ~3u;
    for (uint32_t t = threadIdx.x; t < padded; t += kRankThreads) ids[t] = t < a.n_tokens ? id_at(a, t, n) : 0xffffffffu;
    if (threadIdx.x < 32) place[threadIdx.x] = 0u;
    __syncthreads();
    const uint32_t t0 = blockIdx.x * 32, t = t0 + lane, mine = t < a.n_tokens ? ids[t] : 0u;
    const uint32_t share = (padded / 4 + kRankWarps - 1) / kRankWarps * 4, lo = min(padded, warp * share), hi = min(padded, lo + share);
    uint32_t count = 0;
    const uint4 *v = reinterpret_cast<const uint4 *>(ids);
#pragma unroll 4
    for (uint32_t s = lo; s < min(hi, t0); s += 4) {         // before the block's positions: equal ids come first
        const uint4 x = v[s / 4];
        count += (uint32_t)(x.x <= mine) + (uint32_t)(x.y <= mine) + (uint32_t)(x.z <= mine) + (uint32_t)(x.w <= mine);
    }
#pragma unroll 4
    for (uint32_t s = max(lo, t0 + 32); s < hi; s += 4) {
        const uint4 x = v[s / 4];
        count += (uint32_t)(x.x < mine) + (uint32_t)(x.y < mine) + (uint32_t)(x.z < mine) + (uint32_t)(x.w < mine);
    }
    if (warp == 0)
        for (uint32_t s = t0; s < min(t0 + 32, a.n_tokens); ++s) count += ids[s] < mine || (ids[s] == mine && s < t);
    atomicAdd(place + lane, count);
    __syncthreads();
    if (warp == 0 && t < a.n_tokens) {
        a.keys[place[lane]] = mine;
        a.pos[place[lane]] = t;
    }
}

// More positions: tiles of kSortThreads * kItems entries.  A counting kernel for the first digit, then one
// placing kernel per digit, which counts the next digit where its entries go.  Blocks beyond the tiles clear the
// first rows without a token, where the last of several placing kernels has such blocks.
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
    for (uint32_t w = blockIdx.x * kSortThreads + threadIdx.x; w < a.n_arrived; w += gridDim.x * kSortThreads) a.arrived[w] = 0u;
}

template <int kItems>
__global__ void __launch_bounds__(kSortThreads) sort_place_kernel(const EmbedArgs a, const SortPass s) {
    griddep_launch_dependents();
    griddep_wait();
    __shared__ uint32_t warp_bins[kSortWarps][kSortBins];
    __shared__ uint32_t warp_sum[kSortBins / 32];
    if (blockIdx.x >= s.n_tiles) return zero_rows(a, blockIdx.x - s.n_tiles, a.present + (size_t)(blockIdx.x - s.n_tiles) * zero_words(a));
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
#pragma unroll 16
    for (uint32_t tile = 0; tile < s.n_tiles; ++tile) {
        const uint32_t c = __ldcg(counts + (size_t)tile * kSortBins);
        if (tile < blockIdx.x) ahead += c;
        total += c;
    }
    rank_digits<kItems>(key, rank, in_mask, s.shift, warp_bins);
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
// A warp adds up kSumWarpCols columns of rows, kSumCols per lane.
//   kWide: rows start on 16-byte boundaries and are whole lanes' columns; a lane loads its own consecutive columns
//     of kRows rows at a time into registers.
//   else: the aligned 16-byte pieces that cover the warp's columns of a row are copied to shared memory, two groups of
//     kRows rows in turn, and a lane reads pairs of columns, 64 apart, from wherever in them the row begins;
//     written rows go through shared memory too, to leave in vectors aligned on the row.
constexpr int kSumCols = 8, kSumPairs = kSumCols / 2;
constexpr uint32_t kSumWarpCols = 32 * kSumCols;

template <typename T, bool kWide>
struct SumLayout {
    static constexpr int kRows = kWide && sizeof(T) == 2 ? 8 : 4;
    static constexpr uint32_t kSlot = kSumWarpCols * sizeof(T) + 16;
    static constexpr uint32_t kStage = (kSumWarpCols + kSumWarpCols / 32) * 4;     // a word of padding per 32: lanes 8 apart in different banks
    static constexpr uint32_t kWarpBytes = kWide ? 0 : 2 * kRows * kSlot + kStage;
};
// column of a lane's pair k, from the warp's first
template <bool kWide>
__device__ __forceinline__ uint32_t pair_column(int k) {
    const uint32_t lane = threadIdx.x & 31u;
    return kWide ? lane * kSumCols + 2 * k : 64 * k + 2 * lane;
}

// A row's columns [c0, c0 + cols) on their way into a slot; the row lies in [begin, end).
template <typename T>
__device__ __forceinline__ void fetch_row(uint8_t *slot, const T *row, uint32_t c0, uint32_t cols, const T *begin, const T *end) {
    constexpr uint32_t E = Elem<T>::kVec;
    const T *from = row + c0;
    const uint32_t skew = (uint32_t)(reinterpret_cast<uintptr_t>(from) & 15u) / (uint32_t)sizeof(T), pieces = (skew + cols + E - 1) / E;
    for (uint32_t i = threadIdx.x & 31u; i < pieces; i += 32) {
        const T *at = from - skew + i * E;
        if (at >= begin && at + E <= end) copy_async<16>(slot + i * 16, at);
        else                                                 // a piece that reaches over an end of the array
            for (uint32_t k = 0; k < E; ++k)
                if (at + k >= begin && at + k < end) reinterpret_cast<T *>(slot + i * 16)[k] = at[k];
    }
}
// skew: bytes from the slot's start to the row's first column
template <typename T>
__device__ __forceinline__ void add_slot(f32x2 (&sum)[kSumPairs], const uint8_t *slot, uint32_t skew) {
    const uint32_t lane = threadIdx.x & 31u, *w = reinterpret_cast<const uint32_t *>(slot + (skew & ~3u));
#pragma unroll
    for (int k = 0; k < kSumPairs; ++k) {
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if constexpr (sizeof(T) == 4) {
            v.x = w[64 * k + 2 * lane];
            v.y = w[64 * k + 2 * lane + 1];
        } else v.x = __funnelshift_r(w[32 * k + lane], w[32 * k + lane + 1], (skew & 2u) * 8u);
        sum[k] = add2(sum[k], Elem<T>::pair(v, 0));
    }
}

// Four floats added to those at p (16-byte aligned).
__device__ __forceinline__ void add_vector(void *p, const uint4 &v) {
    asm volatile("red.relaxed.gpu.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(p), "f"(__uint_as_float(v.x)), "f"(__uint_as_float(v.y)),
                 "f"(__uint_as_float(v.z)), "f"(__uint_as_float(v.w)) : "memory");
}

// scale * sum to columns [c0, c0 + cols) of row v of the gradient table, or added to what is there.
template <typename G, bool kWide>
__device__ __forceinline__ void write_row(const EmbedArgs &a, uint32_t v, const f32x2 (&sum)[kSumPairs], uint32_t c0, uint32_t cols, float *stage) {
    G *out = static_cast<G *>(a.grad_table) + (long long)v * a.table_stride + c0;
    const uint32_t lane = threadIdx.x & 31u;
    constexpr uint32_t E = Elem<G>::kVec;
    float x[kSumCols];
#pragma unroll
    for (int k = 0; k < kSumPairs; ++k) {
        const uint32_t c = pair_column<kWide>(k);
        unpack2(mul2(sum[k], pack2(a.scale, a.scale)), x[2 * k], x[2 * k + 1]);
        if (sizeof(G) == 2 && a.accumulate) {
            if (c < cols) x[2 * k] += Elem<G>::load(out + c);
            if (c + 1 < cols) x[2 * k + 1] += Elem<G>::load(out + c + 1);
        }
    }
    // a float row is added to where it lies: one addition per element, so the order of the warps is nothing to it
    const bool add = sizeof(G) == 4 && a.accumulate;
    if constexpr (kWide) {
        if (lane * kSumCols >= cols) return;
#pragma unroll
        for (uint32_t q = 0; q < kSumCols / E; ++q) {
            uint4 o;
#pragma unroll
            for (uint32_t k = 0; k < E / 2; ++k) Elem<G>::put_pair(o, k, x[q * E + 2 * k], x[q * E + 2 * k + 1]);
            if (add) add_vector(out + lane * kSumCols + q * E, o); else st_stream(out + lane * kSumCols + q * E, o);
        }
    } else {
        auto at = [](uint32_t c) { return c + c / 32; };
        __syncwarp();
#pragma unroll
        for (int k = 0; k < kSumPairs; ++k) {
            stage[at(pair_column<false>(k))] = x[2 * k];
            stage[at(pair_column<false>(k) + 1)] = x[2 * k + 1];
        }
        __syncwarp();
        const uint32_t head = min((16u - (uint32_t)(reinterpret_cast<uintptr_t>(out) & 15u)) % 16u / (uint32_t)sizeof(G), cols), nvec = (cols - head) / E;
        for (uint32_t j = lane; j < nvec; j += 32) {
            uint4 o;
#pragma unroll
            for (uint32_t k = 0; k < E / 2; ++k) Elem<G>::put_pair(o, k, stage[at(head + j * E + 2 * k)], stage[at(head + j * E + 2 * k + 1)]);
            if (add) add_vector(out + head + j * E, o); else st_stream(out + head + j * E, o);
        }
        const uint32_t tail = head + nvec * E;
        auto loose = [&](uint32_t c) {
            if (add) atomicAdd(reinterpret_cast<float *>(out) + c, stage[at(c)]); else out[c] = Elem<G>::from(stage[at(c)]);
        };
        if (lane < head) loose(lane);
        if (lane < cols - tail) loose(tail + lane);
    }
}

// Sums of a run's part: which = 0 cut by the chunk's start, 1 by its end.  A row has room for whole warps' columns.
__device__ __forceinline__ float *partial_row(const EmbedArgs &a, uint32_t which, uint32_t chunk) {
    return a.partial + ((size_t)which * a.n_chunks + chunk) * a.partial_stride;
}

template <bool kWide>
__device__ __forceinline__ void store_partial(const EmbedArgs &a, uint32_t which, uint32_t chunk, uint32_t c0, const f32x2 (&sum)[kSumPairs]) {
    float *to = partial_row(a, which, chunk) + c0, x[kSumCols];
#pragma unroll
    for (int k = 0; k < kSumPairs; ++k) unpack2(sum[k], x[2 * k], x[2 * k + 1]);
    if constexpr (kWide) {
        float4 *p = reinterpret_cast<float4 *>(to + pair_column<true>(0));
        __stcg(p, make_float4(x[0], x[1], x[2], x[3]));
        __stcg(p + 1, make_float4(x[4], x[5], x[6], x[7]));
    } else {
#pragma unroll
        for (int k = 0; k < kSumPairs; ++k) __stcg(reinterpret_cast<float2 *>(to + pair_column<false>(k)), make_float2(x[2 * k], x[2 * k + 1]));
    }
}

// The parts of a run that chunk borders cut, of which this warp has just stored one (run v; cont: it began before
// `chunk`): whichever warp stores the last one adds them up, in the order of the chunks.  True for that warp.
constexpr uint32_t kJoinGroup = 16;
template <bool kWide>
__device__ __forceinline__ bool join_run(const EmbedArgs &a, uint32_t v, uint32_t chunk, bool cont, uint32_t slice, uint32_t slices, f32x2 (&sum)[kSumPairs]) {
    const uint32_t lane = threadIdx.x & 31u, c0 = slice * kSumWarpCols;
    // chunks that continue the run: behind this one (those that begin with v), and before it back to the one
    // it begins in (the last whose predecessor does not end with v)
    uint32_t behind = 0, back = 0;
    for (;;) {
        const unsigned long long c = (unsigned long long)chunk + 1 + behind + lane;
        const uint32_t same = __ballot_sync(kFullMask, c < a.n_chunks && a.keys[c * a.rows_per_chunk] == v);
        if (same != kFullMask) { behind += __ffs(~same) - 1; break; }
        behind += 32;
    }
    if (cont)
        for (;;) {
            const long long c = (long long)chunk - 1 - back - lane;
            const uint32_t same = __ballot_sync(kFullMask, c > 0 && a.keys[(size_t)c * a.rows_per_chunk - 1] == v);
            if (same != kFullMask) { back += __ffs(~same); break; }
            back += 32;
        }
    const uint32_t owner = chunk - back, parts = back + behind;      // `parts` partial 0, and the owner's partial 1
    const size_t counters = (size_t)a.n_chunks * slices;
    // part q: the owner's partial 1, then the following chunks' partial 0.  Groups of kJoinGroup parts are added up
    // first, each by the last to arrive, then the groups' sums, which take the place of their first part.
    uint32_t group = back / kJoinGroup;
#pragma unroll 1
    for (uint32_t level = 0;; ++level) {
        const uint32_t from = level == 0 ? group * kJoinGroup : 0u, step = level == 0 ? 1u : kJoinGroup;
        const uint32_t terms = level == 0 ? min(kJoinGroup, parts + 1 - from) : parts / kJoinGroup + 1;
        // a chunk may begin one run and start a group of another: three sets of counters
        uint32_t *counter = a.arrived + (level ? 2 * counters : group ? counters : 0u) + (size_t)(owner + from) * slices + slice;
        __threadfence();
        __syncwarp();
        uint32_t before = 0;
        if (lane == 0) before = atomicAdd(counter, 1u);
        if (__shfl_sync(kFullMask, before, 0) != terms - 1) return false;
        __threadfence();
        constexpr uint32_t kAhead = 8;
        for (uint32_t t = 0; t < terms; t += kAhead) {
            float2 x[kAhead][kSumPairs];
#pragma unroll
            for (uint32_t u = 0; u < kAhead; ++u) {
                const uint32_t q = from + min(t + u, terms - 1) * step;
                const float *p = (q ? partial_row(a, 0, owner + q) : partial_row(a, 1, owner)) + c0;
#pragma unroll
                for (int k = 0; k < kSumPairs; ++k) x[u][k] = __ldcg(reinterpret_cast<const float2 *>(p + pair_column<kWide>(k)));
            }
#pragma unroll
            for (uint32_t u = 0; u < kAhead; ++u) {
                if (t + u >= terms) break;
#pragma unroll
                for (int k = 0; k < kSumPairs; ++k) {
                    const f32x2 y = pack2(x[u][k].x, x[u][k].y);
                    sum[k] = t + u ? add2(sum[k], y) : y;
                }
            }
        }
        if (level == 1 || parts < kJoinGroup) return true;
        store_partial<kWide>(a, from ? 0u : 1u, owner + from, c0, sum);
    }
}

// Bound by memory: 65536 rows of 2048 bfloat16 into a table of 129280 float rows (268 MB read, 1059 MB written) 207 us of
// the call's 239, the rest being the sort (one counting kernel of 3 us and two placing kernels of 8); rows of 2047, which go
// through shared memory, 281 us a call.
// A warp per (chunk of sorted positions, 256 columns).  A run that lies inside the chunk is written out; the part of
// a run that began in an earlier chunk goes to partial 0, the part of one that began here and goes on to
// partial 1, and the last part to arrive writes the run out.  The blocks behind the sum_blocks that do this clear
// rows without a token (before them or spread among them they cost 65536 x 2048 into float 5 to 10 % more).
template <typename T, typename G, bool kWide>
__global__ void __launch_bounds__(kSumThreads, kWide ? 3 : 4) embed_sum_kernel(const __grid_constant__ EmbedArgs a, uint32_t slices, uint32_t sum_blocks) {
    griddep_launch_dependents();
    griddep_wait();
    if (blockIdx.x >= sum_blocks) {
        const uint32_t block = blockIdx.x - sum_blocks + a.zero_from;
        if (a.present) return zero_rows(a, block, a.present + (size_t)block * zero_words(a));
        __shared__ uint32_t bits[kZeroWords];
        present_in_keys(a, block, bits);
        return zero_rows(a, block, bits);
    }
    using Layout = SumLayout<T, kWide>;
    constexpr int kRows = Layout::kRows, E = Elem<T>::kVec;
    extern __shared__ __align__(16) uint8_t sum_smem[];
    uint8_t *ring = sum_smem + (threadIdx.x >> 5) * Layout::kWarpBytes;
    float *stage = kWide ? nullptr : reinterpret_cast<float *>(ring + 2 * kRows * Layout::kSlot);
    const unsigned long long item = (unsigned long long)blockIdx.x * kSumWarps + (threadIdx.x >> 5);
    const unsigned long long chunk64 = item / slices;
    if (chunk64 >= a.n_chunks) return;
    const uint32_t chunk = (uint32_t)chunk64, slice = (uint32_t)(item % slices), lane = threadIdx.x & 31u;
    const uint32_t c0 = slice * kSumWarpCols, cols = min(a.dim - c0, kSumWarpCols);
    const uint32_t lo = chunk * a.rows_per_chunk, n = min(a.n_tokens - lo, a.rows_per_chunk);
    const T *in = static_cast<const T *>(a.grad_out), *in_end = in + (long long)(a.n_tokens - 1) * a.out_stride + a.dim;

    // keys and positions, 32 entries at a time; the rows of the next group are on their way while one is added
    const uint32_t *keys = a.keys + lo, *pos = a.pos + lo;
    auto batch = [&](const uint32_t *p, uint32_t b, uint32_t none) { return b + lane < n ? p[b + lane] : none; };
    uint32_t my_key = batch(keys, 0, a.vocab), my_pos = batch(pos, 0, 0u);
    const uint32_t before = lo > 0 ? a.keys[lo - 1] : a.vocab, after = lo + n < a.n_tokens ? keys[n] : a.vocab;
    uint32_t v = __shfl_sync(kFullMask, my_key, 0);
    if (v >= a.vocab) return;                                // sorted behind all ids
    const uint32_t first = v;
    const bool began_before = before == first;
    bool cont = began_before;                                // still in that run
    f32x2 sum[kSumPairs];
    auto clear = [&]() {
#pragma unroll
        for (int k = 0; k < kSumPairs; ++k) sum[k] = pack2(0.0f, 0.0f);
    };
    clear();
    auto next_run = [&](uint32_t key) {  // ends the run of v, unless key is v
        if (key == v) return;
        if (v < a.vocab) {
            if (cont) store_partial<kWide>(a, 0u, chunk, c0, sum);
            else write_row<G, kWide>(a, v, sum, c0, cols, stage);
        }
        cont = false;
        v = key;
        clear();
    };

    if constexpr (kWide) {
        constexpr int kVecs = kSumCols / E;
        const T *mine = in + c0 + lane * kSumCols;
        const bool on = lane * kSumCols < cols;
        for (uint32_t e0 = 0; e0 < n; e0 += 32) {
            if (e0) { my_key = batch(keys, e0, a.vocab); my_pos = batch(pos, e0, 0u); }
            const uint32_t left = min(n - e0, 32u);
            for (uint32_t k0 = 0; k0 < left; k0 += kRows) {
                uint4 x[kRows][kVecs];
#pragma unroll
                for (int u = 0; u < kRows; ++u) {
                    const uint32_t key = __shfl_sync(kFullMask, my_key, k0 + u), p = __shfl_sync(kFullMask, my_pos, k0 + u);
                    const bool some = on && key < a.vocab;
                    const T *row = mine + (long long)p * a.out_stride;
#pragma unroll
                    for (int q = 0; q < kVecs; ++q) {
                        x[u][q] = make_uint4(0u, 0u, 0u, 0u);
                        if (some) x[u][q] = ld_stream(row + q * E);
                    }
                }
#pragma unroll
                for (int u = 0; u < kRows; ++u) {
                    if (k0 + u >= left) break;
                    next_run(__shfl_sync(kFullMask, my_key, k0 + u));
#pragma unroll
                    for (int q = 0; q < kVecs; ++q)
#pragma unroll
                        for (int k = 0; k < E / 2; ++k) sum[q * E / 2 + k] = add2(sum[q * E / 2 + k], Elem<T>::pair(x[u][q], k));
                }
            }
        }
    } else {
        const uint32_t in_skew = (uint32_t)reinterpret_cast<uintptr_t>(in + c0), stride_skew = (uint32_t)a.out_stride * (uint32_t)sizeof(T);
        uint32_t far_key = my_key, far_pos = my_pos;         // the batch that rows are fetched from
        auto issue = [&](uint32_t f) {   // the group of kRows rows from entry f on
            if (f < n) {
                if (f && (f & 31u) == 0) { far_key = batch(keys, f, a.vocab); far_pos = batch(pos, f, 0u); }
#pragma unroll
                for (int u = 0; u < kRows; ++u) {
                    const uint32_t key = __shfl_sync(kFullMask, far_key, (f + u) & 31u), p = __shfl_sync(kFullMask, far_pos, (f + u) & 31u);
                    if (key < a.vocab) fetch_row(ring + ((f / kRows) % 2 * kRows + u) * Layout::kSlot, in + (long long)p * a.out_stride, c0, cols, in, in_end);
                }
            }
            copy_commit();
        };
        issue(0);
        issue(kRows);
        for (uint32_t e = 0; e < n; e += kRows) {
            if (e && (e & 31u) == 0) { my_key = batch(keys, e, a.vocab); my_pos = batch(pos, e, 0u); }
            copy_wait<1>();
            __syncwarp();
#pragma unroll 1
            for (int u = 0; u < kRows; ++u) {
                const uint32_t key = __shfl_sync(kFullMask, my_key, (e + u) & 31u), p = __shfl_sync(kFullMask, my_pos, (e + u) & 31u);
                if (e + u >= n) break;
                next_run(key);
                if (key < a.vocab) add_slot<T>(sum, ring + ((e / kRows) % 2 * kRows + u) * Layout::kSlot, (in_skew + p * stride_skew) & 15u);
            }
            __syncwarp();
            issue(e + 2 * kRows);
        }
        copy_wait<0>();                                      // nothing of this warp's is still on its way
    }
    const bool goes_on = v < a.vocab && after == v;
    if (v < a.vocab) {
        if (cont || goes_on) store_partial<kWide>(a, cont ? 0u : 1u, chunk, c0, sum);
        else write_row<G, kWide>(a, v, sum, c0, cols, stage);
    }
    // the runs of which this chunk had a part: the one it began in, and the one it ended in
#pragma unroll 1
    for (int side = 0; side < 2; ++side) {
        const bool part = side == 0 ? began_before : goes_on && !cont;
        const uint32_t run = side == 0 ? first : v;
        if (part && join_run<kWide>(a, run, chunk, side == 0, slice, slices, sum)) write_row<G, kWide>(a, run, sum, c0, cols, stage);
    }
}

// ---- few positions: no sort, one launch ----
// A block per (position, 256 columns) looks its id up among all positions, a share of them per warp, and stops unless
// the position is the id's first.  Each warp adds up the id's rows in its share, and the shares' sums are added in
// order.  Blocks behind the sum_blocks clear rows without a token; they look through the ids for their own rows.
// The looking costs positions^2 comparisons: nothing for hundreds of positions, too much for many thousands.
template <typename T, typename G, bool kWide>
__global__ void __launch_bounds__(kSumThreads) embed_few_kernel(const EmbedArgs a, uint32_t slices, uint32_t sum_blocks) {
    griddep_launch_dependents();
    griddep_wait();
    __shared__ f32x2 piece[kSumWarps][kSumPairs][32];
    __shared__ bool found[kSumWarps];
    __shared__ float stage[SumLayout<T, false>::kStage / 4];
    __shared__ uint32_t bits[kZeroWords];
    const uint32_t n = tokens_in(a), lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    if (blockIdx.x >= sum_blocks) {
        const uint32_t block = blockIdx.x - sum_blocks, words = zero_words(a);
        const uint32_t v0 = block * words * 32;
        if (threadIdx.x < kZeroWords) bits[threadIdx.x] = 0u;
        __syncthreads();
        for (uint32_t t = threadIdx.x; t < a.n_tokens; t += kSumThreads) {
            const uint32_t id = id_at(a, t, n);
            if (id < a.vocab && id >= v0 && id - v0 < words * 32) atomicOr(bits + (id - v0) / 32, 1u << ((id - v0) & 31u));
        }
        __syncthreads();
        return zero_rows(a, block, bits);
    }
    const uint32_t t = blockIdx.x / slices, c0 = blockIdx.x % slices * kSumWarpCols, cols = min(a.dim - c0, kSumWarpCols);
    const uint32_t v = id_at(a, t, n);
    if (v >= a.vocab) return;
    const uint32_t share = (a.n_tokens + kSumThreads - 1) / kSumThreads * 32, lo = warp * share, hi = min(a.n_tokens, lo + share);
    auto matches = [&](uint32_t g) { return __ballot_sync(kFullMask, g + lane < hi && id_at(a, g + lane, n) == v); };
    bool earlier = false;
    for (uint32_t g = lo; g < hi && g < t; g += 32) earlier |= (matches(g) & (t - g < 32 ? (1u << (t - g)) - 1u : kFullMask)) != 0;
    if (__syncthreads_or(earlier)) return;

    constexpr int E = Elem<T>::kVec, kRows = 4;
    const T *in = static_cast<const T *>(a.grad_out) + c0;
    f32x2 sum[kSumPairs];
#pragma unroll
    for (int k = 0; k < kSumPairs; ++k) sum[k] = pack2(0.0f, 0.0f);
    bool any = false;
    for (uint32_t g = lo; g < hi; g += 32) {
        uint32_t mask = matches(g);
        any |= mask != 0;
        while (mask) {                   // kRows rows at a time, in ascending order of position
            f32x2 x[kRows][kSumPairs];
            uint32_t taken = 0;
#pragma unroll
            for (int u = 0; u < kRows; ++u) {
                if (!mask) break;
                const T *row = in + (long long)(g + __ffs(mask) - 1) * a.out_stride;
                mask &= mask - 1;
                ++taken;
                if constexpr (kWide) {
#pragma unroll
                    for (int q = 0; q < kSumCols / E; ++q) {
                        uint4 w = make_uint4(0u, 0u, 0u, 0u);
                        if (lane * kSumCols < cols) w = *reinterpret_cast<const uint4 *>(row + lane * kSumCols + q * E);
#pragma unroll
                        for (int k = 0; k < E / 2; ++k) x[u][q * E / 2 + k] = Elem<T>::pair(w, k);
                    }
                } else {
#pragma unroll
                    for (int k = 0; k < kSumPairs; ++k) {
                        const uint32_t c = pair_column<false>(k);
                        x[u][k] = pack2(c < cols ? Elem<T>::load(row + c) : 0.0f, c + 1 < cols ? Elem<T>::load(row + c + 1) : 0.0f);
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < kRows; ++u) {
                if ((uint32_t)u >= taken) break;
#pragma unroll
                for (int k = 0; k < kSumPairs; ++k) sum[k] = add2(sum[k], x[u][k]);
            }
        }
    }
    if (lane == 0) found[warp] = any;
    if (any && warp)
#pragma unroll
        for (int k = 0; k < kSumPairs; ++k) piece[warp][k][lane] = sum[k];
    __syncthreads();
    if (warp) return;
    for (int w = 1; w < kSumWarps; ++w)
        if (found[w])
#pragma unroll
            for (int k = 0; k < kSumPairs; ++k) sum[k] = add2(sum[k], piece[w][k][lane]);
    write_row<G, kWide>(a, v, sum, c0, cols, stage);
}

}  // namespace td
