// Attention of one new token per row over a paged cache.
//
// The work is one pass over the keys and values with a running maximum and sum per row and head.  A unit is a row's
// heads over one key head (16 at most: the rows of a matrix instruction), its tokens come in tiles of kTile.  All
// units' tiles, one unit after the other, are a line that is cut into equal pieces, a piece per warp, wherever the cuts
// fall: so one long sequence and a thousand short ones load the machine alike.  A warp has its tiles brought by its own ring of
// asynchronous copies, several tiles ahead and across units; no warp waits for another.  Units that a cut
// went through leave parts (maximum, sum, weighted values), joined in the order of the tokens: within a block after its
// warps are done, between blocks by the last block to arrive.  The same call gives the same bits.
#pragma once

#include "td_cache.cuh"
#include "td_mma.cuh"

namespace td {

struct AttendArgs {
    const int32_t *seqs;
    const void *q;
    void *out;
    float *lse;
    const void *keys, *values;                                // of the layer
    int64_t page, token, head;                                // element strides of the cache
    int64_t q_row, q_head, out_row, out_head;
    uint32_t n_rows, n_heads, kv_heads, ratio, dim, window;
    uint32_t units;                                           // of a row: key heads times sixteens of heads of each
    float scale, scale2;                                      // scale2 = scale * log2(e)
    float *parts;                                             // [2 per warp, then 2 per block][part_floats]
    uint32_t *arrived;                                        // [blocks], zero between calls
};

constexpr uint32_t kTile = 16;                                // tokens of a tile
constexpr uint32_t kHeadRows = 16;                            // heads of a unit
constexpr uint32_t kLeastTiles = 4;                           // of a warp, before another block is used

// Shapes of a kernel for heads of up to 16 * kChunks elements.
template <int kChunks>
struct AttendShape {
    static constexpr uint32_t kDim = 16 * kChunks;
    static constexpr uint32_t kWarps = kChunks <= 8 ? 8 : 4;
    static constexpr uint32_t kThreads = 32 * kWarps;
    static constexpr uint32_t kPitch = kDim * 2 + 16;         // bytes of a row in shared memory: an odd number of 16s, so that 8 rows lie in different banks
    static constexpr uint32_t kSide = kTile * kPitch;         // keys, or values, of a tile
    static constexpr uint32_t kStage = 2 * kSide;
    static constexpr bool kQueryInRegisters = kChunks <= 8;
    static constexpr uint32_t kQuery = kQueryInRegisters ? 0 : kHeadRows * kPitch;
    static constexpr uint32_t kRoom = 216 * 1024 / kWarps;    // bytes a warp may have
    static constexpr uint32_t kFits = (kRoom - kQuery) / (kStage + 16);
    static constexpr uint32_t kStages = kFits < 6 ? kFits : 6;
    static constexpr uint32_t kWarpBytes = kStages * (kStage + 16) + kQuery;
    static constexpr uint32_t kBytes = kWarps * kWarpBytes;
    static constexpr uint32_t kPartFloats = kHeadRows * (kDim + 2);      // weighted values [16][kDim], then {maximum, sum} [16]
};

struct Span {                                                 // the tokens [lo, n) of sequence s
    int32_t s, lo, n;
    __device__ __forceinline__ uint32_t tiles() const { return (uint32_t)(n - lo + (int32_t)kTile - 1) / kTile; }
};
__device__ __forceinline__ Span span_of(const CacheView &c, const AttendArgs &a, uint32_t row, bool flag) {
    Span p{a.seqs ? a.seqs[row] : (int32_t)row, 0, 0};
    if (p.s < 0) return p;
    if ((uint32_t)p.s >= c.max_seqs) {
        if (flag) cache_flag(c, TD_ERR_OOB_INDEX);
        return p;
    }
    const int32_t n = c.length[p.s];
    if (!length_ok(c, n)) {
        if (flag) cache_flag(c, TD_ERR_BAD_LENGTH);
        return p;
    }
    p.n = n;
    p.lo = a.window && (uint32_t)n > a.window ? n - (int32_t)a.window : 0;
    return p;
}

// The line of all units' tiles; a unit has one place ahead of its tiles (what it costs to begin one), so that of a row with T
// tiles each unit has T + 1 places.  Warp w of `warps` has places [total w / warps, total (w + 1) / warps).
struct Line {
    unsigned long long total;
    uint32_t warps;
    __device__ __forceinline__ unsigned long long begin(uint32_t w) const { return total * w / warps; }
    __device__ __forceinline__ uint32_t warp_of(unsigned long long place) const {          // the last w with begin(w) <= place
        return (uint32_t)(((place + 1) * warps + total - 1) / total) - 1;
    }
};

// A unit that a cut went through: its first place and tiles.
struct Cut {
    unsigned long long place;
    uint32_t row, unit, tiles, valid;
};

__device__ __forceinline__ uint32_t heads_of(const AttendArgs &a, uint32_t unit, uint32_t &first) {          // heads of a unit, from `first` on
    const uint32_t per_kv = a.units / a.kv_heads, kv = unit / per_kv, at = (unit - kv * per_kv) * kHeadRows;
    first = kv * a.ratio + at;
    return min(kHeadRows, a.ratio - at);
}

// Joins the parts k = 0 .. count - 1 of a unit (slot(k) of `parts`) into out and lse, or into another part; `me` of `all` threads.
// A maximum of -inf means that a part has nothing; NaN stays.
template <typename T, uint32_t kDim, typename Slot>
__device__ __forceinline__ void join_parts(const AttendArgs &a, uint32_t row, uint32_t unit, const float *parts, uint32_t count, Slot slot,
                                           float *to, uint32_t me, uint32_t all) {
    constexpr uint32_t kFloats = kHeadRows * (kDim + 2);
    uint32_t first;
    const uint32_t heads = heads_of(a, unit, first), pairs = kDim / 2;
    for (uint32_t i = me; i < heads * pairs; i += all) {
        const uint32_t h = i / pairs, d = (i - h * pairs) * 2;
        if (d >= a.dim) continue;
        float top = -CUDART_INF_F;
        for (uint32_t k = 0; k < count; ++k) top = max_nan(__ldcg(parts + (size_t)slot(k) * kFloats + kHeadRows * kDim + 2 * h), top);
        const float ref = top == -CUDART_INF_F ? 0.0f : top;
        float sum = 0.0f, x = 0.0f, y = 0.0f;
#pragma unroll 4
        for (uint32_t k = 0; k < count; ++k) {
            const float *p = parts + (size_t)slot(k) * kFloats;
            const float2 ml = __ldcg(reinterpret_cast<const float2 *>(p + kHeadRows * kDim + 2 * h)), v = __ldcg(reinterpret_cast<const float2 *>(p + h * kDim + d));
            const float e = exp2_approx(ml.x - ref);
            sum = fmaf(ml.y, e, sum);
            x = fmaf(v.x, e, x);
            y = fmaf(v.y, e, y);
        }
        if (to) {
            *reinterpret_cast<float2 *>(to + h * kDim + d) = make_float2(x, y);
            if (d == 0) *reinterpret_cast<float2 *>(to + kHeadRows * kDim + 2 * h) = make_float2(top, sum);
            continue;
        }
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        *reinterpret_cast<uint32_t *>(static_cast<T *>(a.out) + row * a.out_row + (first + h) * a.out_head + d) = pair_of<T>(x * inv, y * inv);
        if (a.lse && d == 0) a.lse[(size_t)row * a.n_heads + first + h] = sum == 0.0f ? -CUDART_INF_F : (top + log2f(sum)) * 0.69314718055994531f;
    }
}

template <typename T, int kChunks>
__global__ void __launch_bounds__(AttendShape<kChunks>::kThreads, 1) attend_kernel(CacheView c, AttendArgs a) {
    using S = AttendShape<kChunks>;
    extern __shared__ __align__(16) uint8_t memory[];
    __shared__ unsigned long long sums[S::kThreads];          // places of all rows up to and with those of each thread
    __shared__ Cut cut_in, cut_out[S::kWarps];                // the unit that warp 0 began in the middle of; those a warp began and left
    __shared__ uint32_t last;
    griddep_launch_dependents();
    griddep_wait();
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;

    // ---- this warp's share ----
    const uint32_t per_thread = (a.n_rows + S::kThreads - 1) / S::kThreads;
    {
        unsigned long long mine = 0;
        for (uint32_t r = threadIdx.x * per_thread; r < min(a.n_rows, (threadIdx.x + 1) * per_thread); ++r)
            mine += (unsigned long long)a.units * (span_of(c, a, r, blockIdx.x == 0).tiles() + 1);
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const unsigned long long y = __shfl_up_sync(kFullMask, mine, d);
            if (lane >= (uint32_t)d) mine += y;
        }
        sums[threadIdx.x] = mine;
        __syncthreads();
        unsigned long long before = 0;
        for (uint32_t w = 0; w < warp; ++w) before += sums[w * 32 + 31];
        __syncthreads();
        sums[threadIdx.x] = mine + before;
        if (lane == 0) cut_in.valid = cut_out[warp].valid = 0;
        __syncthreads();
    }
    Line line;
    line.total = sums[S::kThreads - 1];
    const uint32_t blocks = (uint32_t)min((unsigned long long)gridDim.x, line.total / (S::kWarps * kLeastTiles) + 1);
    if (blockIdx.x >= blocks) return;
    line.warps = (uint32_t)min((unsigned long long)blocks * S::kWarps, line.total);          // each has a place at least
    const uint32_t w_global = blockIdx.x * S::kWarps + warp;
    const unsigned long long begin = line.begin(min(w_global, line.warps)), end = line.begin(min(w_global + 1, line.warps));

    uint8_t *const mem = memory + warp * S::kWarpBytes;
    const uint32_t ring = shared_address(mem), query = ring + S::kStages * S::kStage;
    uint4 *const notes = reinterpret_cast<uint4 *>(mem + S::kStages * S::kStage + S::kQuery);          // per stage: row, unit, tokens that count and flags and heads, first head
    if (a.dim != S::kDim)                                     // columns that no copy writes
        for (uint32_t i = lane; i < S::kStages * S::kStage / 16; i += 32) reinterpret_cast<uint4 *>(mem)[i] = make_uint4(0u, 0u, 0u, 0u);
    __syncwarp();

    if (begin < end) {
        // where `begin` lies: the thread whose rows it is among, then the row
        uint32_t lo = 0, hi = S::kThreads - 1;                // the first thread with sums > begin
        while (lo < hi) {
            const uint32_t mid = (lo + hi) / 2;
            if (sums[mid] > begin) hi = mid; else lo = mid + 1;
        }
        unsigned long long row_place = lo ? sums[lo - 1] : 0;
        uint32_t row = lo * per_thread;
        Span span;
        for (;; ++row) {
            span = span_of(c, a, row, false);
            const unsigned long long places = (unsigned long long)a.units * (span.tiles() + 1);
            if (row_place + places > begin) break;
            row_place += places;
        }
        uint32_t tiles = span.tiles();
        uint32_t unit = (uint32_t)((begin - row_place) / (tiles + 1));
        int32_t tile = (int32_t)(begin - row_place - (unsigned long long)unit * (tiles + 1)) - 1;          // -1: the place ahead
        unsigned long long place = begin;                     // of the next tile to bring
        Span next = row + 1 < a.n_rows ? span_of(c, a, row + 1, false) : Span{-1, 0, 0};

        uint32_t kv, first, heads;
        auto enter = [&]() {                                  // a unit's key head and its heads
            heads = heads_of(a, unit, first);
            kv = first / a.ratio;
        };
        auto leave = [&]() {                                  // to the unit behind
            tile = -1;
            if (++unit == a.units) {
                unit = 0;
                ++row;
                span = next;
                tiles = span.tiles();
                next = row + 1 < a.n_rows ? span_of(c, a, row + 1, false) : Span{-1, 0, 0};
            }
            enter();
        };
        enter();
        // Brings the next tile into stage `to`; false: there is none.  An empty unit's result is written on the way.
        auto bring = [&](uint32_t to) -> bool {
            for (;;) {
                if (place >= end) return false;
                if (tile >= 0) break;
                ++place;
                if (tiles == 0) {
                    const uint32_t pairs = a.dim / 2;
                    for (uint32_t i = lane; i < heads * pairs; i += 32) {
                        const uint32_t h = i / pairs, d = (i - h * pairs) * 2;
                        *reinterpret_cast<uint32_t *>(static_cast<T *>(a.out) + row * a.out_row + (first + h) * a.out_head + d) = 0u;
                    }
                    if (a.lse && lane < heads) a.lse[(size_t)row * a.n_heads + first + lane] = -CUDART_INF_F;
                    leave();
                } else {
                    tile = 0;
                }
            }
            // lanes 0 .. 15: where each token lies
            const int32_t j = span.lo + tile * (int32_t)kTile + (int32_t)(lane & 15u);
            int64_t at = -1;
            if (j < span.n) {
                const uint32_t page = fast_div((uint32_t)j, c.by_page);
                const int32_t id = c.table[(size_t)span.s * c.max_pages + page];
                if ((uint32_t)id < c.n_pages) at = id * a.page + (j - (int64_t)page * c.page_size) * a.token;
                else if (unit == 0 && lane < 16) cache_flag(c, TD_ERR_OOB_INDEX);
            }
            const uint32_t counts = __ballot_sync(kFullMask, at >= 0) & 0xffffu;
            const T *keys = static_cast<const T *>(a.keys) + kv * a.head, *values = static_cast<const T *>(a.values) + kv * a.head;
            const uint32_t stage = ring + to * S::kStage;
            constexpr uint32_t kPer = S::kDim / 8;            // 16-byte vectors of a row
#pragma unroll
            for (uint32_t i0 = 0; i0 < kTile * kPer; i0 += 32) {
                const uint32_t i = i0 + lane, r = i / kPer, v = i - r * kPer;
                const int64_t from = __shfl_sync(kFullMask, at, r);
                if (v * 8 < a.dim) {
                    const int64_t o = from < 0 ? 0 : from + v * 8;
                    copy_async_or_zero(stage + r * S::kPitch + v * 16, keys + o, from < 0 ? 0u : 16u);
                    copy_async_or_zero(stage + S::kSide + r * S::kPitch + v * 16, values + o, from < 0 ? 0u : 16u);
                }
            }
            const bool fresh = tile == 0 || place == begin, final = tile + 1 == (int32_t)tiles, over = final || place + 1 == end;
            if (lane == 0) notes[to] = make_uint4(row, unit, counts | (fresh ? 1u << 16 : 0u) | (over ? 1u << 17 : 0u) | (tile == 0 ? 1u << 18 : 0u) |
                                                  (final ? 1u << 19 : 0u) | heads << 20, first);
            // a cut unit, for the join: the note is complete before the block's barrier
            if (lane == 0 && over) {
                const bool whole_head = place - tile >= begin, whole_tail = final;
                const Cut cut{place - (uint32_t)tile - 1, row, unit, tiles, 1u};
                if (!whole_head) { if (warp == 0) cut_in = cut; }
                else if (!whole_tail) cut_out[warp] = cut;
            }
            ++place;
            if (++tile == (int32_t)tiles) leave();
            return true;
        };

        uint32_t brought = 0;                                 // tiles on their way or here
        bool more = true;
#pragma unroll 1
        for (uint32_t i = 0; i + 1 < S::kStages; ++i) {
            if (more) more = bring(i);
            if (more) ++brought;
            copy_commit();
        }
        uint32_t qf[S::kQueryInRegisters ? kChunks : 1][4];
        float o[2 * kChunks][4], m[2], l[2];
        bool head_whole = false;
        uint32_t stage = 0, put = S::kStages - 1;
#pragma unroll 1
        for (uint32_t done = 0; done < brought; ++done) {
            copy_wait<S::kStages - 2>();
            __syncwarp();
            if (more) more = bring(put);                      // into the stage that the last turn was done with
            if (more) ++brought;
            copy_commit();
            put = put + 1 == S::kStages ? 0 : put + 1;
            const uint4 note = notes[stage];
            const uint32_t at = ring + stage * S::kStage;
            stage = stage + 1 == S::kStages ? 0 : stage + 1;
            const uint32_t first = note.w, heads = note.z >> 20, g = lane >> 2, t = lane & 3u;
            if (note.z >> 16 & 1u) {                          // a unit begins here
                head_whole = note.z >> 18 & 1u;
                const T *q = static_cast<const T *>(a.q) + note.x * a.q_row + first * a.q_head;
                if constexpr (S::kQueryInRegisters) {
#pragma unroll
                    for (int k = 0; k < kChunks; ++k)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t h = g + (i & 1) * 8, d = k * 16 + t * 2 + (i >> 1) * 8;
                            qf[k][i] = h < heads && d < a.dim ? *reinterpret_cast<const uint32_t *>(q + h * a.q_head + d) : 0u;
                        }
                } else {
                    for (uint32_t i = lane; i < kHeadRows * S::kDim / 8; i += 32) {
                        const uint32_t h = i / (S::kDim / 8), v = i - h * (S::kDim / 8);
                        uint4 x = make_uint4(0u, 0u, 0u, 0u);
                        if (h < heads && v * 8 < a.dim) x = *reinterpret_cast<const uint4 *>(q + h * a.q_head + v * 8);
                        *reinterpret_cast<uint4 *>(mem + S::kStages * S::kStage + h * S::kPitch + v * 16) = x;
                    }
                    __syncwarp();
                }
#pragma unroll
                for (int k = 0; k < 2 * kChunks; ++k) o[k][0] = o[k][1] = o[k][2] = o[k][3] = 0.0f;
                m[0] = m[1] = -CUDART_INF_F;
                l[0] = l[1] = 0.0f;
            }
            // scores of 16 heads and 16 tokens, two products of 8 tokens
            float s[2][4] = {};
#pragma unroll
            for (int k = 0; k < kChunks; ++k) {
                uint32_t b[4], qa[4];
                load_matrices(b, at + ((lane & 7u) + (lane >> 4) * 8) * S::kPitch + k * 32 + (lane >> 3 & 1u) * 16);
                if constexpr (S::kQueryInRegisters) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) qa[i] = qf[k][i];
                } else {
                    load_matrices(qa, query + (lane & 15u) * S::kPitch + k * 32 + (lane >> 4) * 16);
                }
                multiply_add<T>(s[0], qa, b[0], b[1]);
                multiply_add<T>(s[1], qa, b[2], b[3]);
            }
            float top[2] = {m[0], m[1]};
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const bool counts = note.z >> (i * 8 + t * 2 + (k & 1)) & 1u;
                    s[i][k] = counts ? s[i][k] * a.scale2 : -CUDART_INF_F;
                    top[k >> 1] = max_nan(top[k >> 1], s[i][k]);
                }
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                top[r] = max_nan(top[r], __shfl_xor_sync(kFullMask, top[r], 1));
                top[r] = max_nan(top[r], __shfl_xor_sync(kFullMask, top[r], 2));
            }
            // the sums so far are brought to the new maximum where it has moved (or is NaN), which is seldom
            if (__any_sync(kFullMask, !(top[0] == m[0]) || !(top[1] == m[1]))) {
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const float keep = m[r] == -CUDART_INF_F ? 0.0f : exp2_approx(m[r] - top[r]);
                    l[r] *= keep;
#pragma unroll
                    for (int k = 0; k < 2 * kChunks; ++k) {
                        o[k][2 * r] *= keep;
                        o[k][2 * r + 1] *= keep;
                    }
                    m[r] = top[r];
                }
            }
            uint32_t p[4];
            {
                const float ref[2] = {m[0] == -CUDART_INF_F ? 0.0f : m[0], m[1] == -CUDART_INF_F ? 0.0f : m[1]};
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        s[i][k] = exp2_approx(s[i][k] - ref[k >> 1]);
                        l[k >> 1] += s[i][k];
                    }
                // Weights are rounded to the type of the values, as the matrix instruction takes them; their sum is not.
                p[0] = pair_of<T>(s[0][0], s[0][1]);
                p[1] = pair_of<T>(s[0][2], s[0][3]);
                p[2] = pair_of<T>(s[1][0], s[1][1]);
                p[3] = pair_of<T>(s[1][2], s[1][3]);
            }
#pragma unroll
            for (int k = 0; k < kChunks; ++k) {
                uint32_t b[4];
                load_matrices_transposed(b, at + S::kSide + ((lane & 7u) + (lane >> 3 & 1u) * 8) * S::kPitch + k * 32 + (lane >> 4) * 16);
                multiply_add<T>(o[2 * k], p, b[0], b[1]);
                multiply_add<T>(o[2 * k + 1], p, b[2], b[3]);
            }
            if (note.z >> 17 & 1u) {                          // the unit, or this warp's part of it, ends here
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    l[r] += __shfl_xor_sync(kFullMask, l[r], 1);
                    l[r] += __shfl_xor_sync(kFullMask, l[r], 2);
                }
                const bool whole = head_whole && (note.z >> 19 & 1u);
                float *part = a.parts + ((size_t)2 * w_global + (head_whole ? 1 : 0)) * S::kPartFloats;
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const uint32_t h = g + r * 8;
                    if (h >= heads) continue;
                    if (whole) {
                        const float inv = l[r] == 0.0f ? 0.0f : 1.0f / l[r];
                        T *out = static_cast<T *>(a.out) + note.x * a.out_row + (first + h) * a.out_head;
#pragma unroll
                        for (int k = 0; k < 2 * kChunks; ++k)
                            if (k * 8 + t * 2 < a.dim) *reinterpret_cast<uint32_t *>(out + k * 8 + t * 2) = pair_of<T>(o[k][2 * r] * inv, o[k][2 * r + 1] * inv);
                        if (a.lse && t == 0)
                            a.lse[(size_t)note.x * a.n_heads + first + h] = l[r] == 0.0f ? -CUDART_INF_F : (m[r] + log2f(l[r])) * 0.69314718055994531f;
                    } else {
#pragma unroll
                        for (int k = 0; k < 2 * kChunks; ++k)
                            *reinterpret_cast<float2 *>(part + h * S::kDim + k * 8 + t * 2) = make_float2(o[k][2 * r], o[k][2 * r + 1]);
                        if (t == 0) *reinterpret_cast<float2 *>(part + kHeadRows * S::kDim + 2 * h) = make_float2(m[r], l[r]);
                    }
                }
            }
        }
    }
    copy_wait<0>();
    __syncthreads();

    // ---- units that cuts went through ----
    const uint32_t w_first = blockIdx.x * S::kWarps, w_last = w_first + S::kWarps - 1;
    if (cut_out[warp].valid) {                                // begun by this warp and ended within the block
        const Cut u = cut_out[warp];
        const uint32_t w0 = w_global, w1 = line.warp_of(u.place + u.tiles);
        if (w1 <= w_last)
            join_parts<T, S::kDim>(a, u.row, u.unit, a.parts, w1 - w0 + 1, [=](uint32_t k) { return 2 * (w0 + k) + (k == 0); }, nullptr, lane, 32);
    }
    float *const block_parts = a.parts + (size_t)2 * gridDim.x * S::kWarps * S::kPartFloats;
    // a unit that came in from the block before, and one that goes on into the next: at most one each, and they may be the same
#pragma unroll 1
    for (uint32_t side = 0; side < 2; ++side) {
        Cut u{};
        if (side == 0) {
            u = cut_in;
        } else {
#pragma unroll 1
            for (uint32_t w = 0; w < S::kWarps; ++w)
                if (cut_out[w].valid && line.warp_of(cut_out[w].place + cut_out[w].tiles) > w_last) u = cut_out[w];
        }
        if (!u.valid) continue;
        const uint32_t w0 = line.warp_of(u.place + 1), w1 = line.warp_of(u.place + u.tiles), from = max(w0, w_first), to = min(w1, w_last);
        const uint32_t b0 = w0 / S::kWarps, b1 = w1 / S::kWarps;
        join_parts<T, S::kDim>(a, u.row, u.unit, a.parts, to - from + 1, [=](uint32_t k) { return 2 * (from + k) + (from + k == w0); },
                               block_parts + ((size_t)2 * blockIdx.x + (blockIdx.x == b0)) * S::kPartFloats, threadIdx.x, S::kThreads);
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) {
            last = atomicAdd(a.arrived + b0, 1u) == b1 - b0;
            if (last) a.arrived[b0] = 0;
            __threadfence();
        }
        __syncthreads();
        if (last)
            join_parts<T, S::kDim>(a, u.row, u.unit, block_parts, b1 - b0 + 1, [=](uint32_t k) { return 2 * (b0 + k) + (k == 0); }, nullptr,
                                   threadIdx.x, S::kThreads);
        __syncthreads();
    }
}

constexpr uint32_t kFloatThreads = 256;

// A warp per row and head; a token at a time.
template <typename T>
__global__ void __launch_bounds__(kFloatThreads) attend_float_kernel(CacheView c, AttendArgs a) {
    griddep_launch_dependents();
    griddep_wait();
    const uint32_t lane = threadIdx.x & 31u;
    const unsigned long long unit = (unsigned long long)blockIdx.x * (kFloatThreads / 32) + threadIdx.x / 32;
    if (unit >= (unsigned long long)a.n_rows * a.n_heads) return;
    const uint32_t row = (uint32_t)(unit / a.n_heads), h = (uint32_t)(unit - (unsigned long long)row * a.n_heads), kv = h / a.ratio;
    const int32_t s = a.seqs ? a.seqs[row] : (int32_t)row;
    int32_t n = 0;
    if (s >= 0) {
        if ((uint32_t)s < c.max_seqs) {
            n = c.length[s];
            if (!length_ok(c, n)) { n = 0; if (lane == 0) cache_flag(c, TD_ERR_BAD_LENGTH); }
        } else if (lane == 0) {
            cache_flag(c, TD_ERR_OOB_INDEX);
        }
    }
    const T *q = static_cast<const T *>(a.q) + row * a.q_row + h * a.q_head;
    float qv[8], o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t d = lane + 32 * i;
        qv[i] = d < a.dim ? Elem<T>::load(q + d) * a.scale : 0.0f;
        o[i] = 0.0f;
    }
    float m = -CUDART_INF_F, sum = 0.0f;
    for (int32_t j = a.window && (uint32_t)n > a.window ? n - (int32_t)a.window : 0; j < n; ++j) {
        const uint32_t page = fast_div((uint32_t)j, c.by_page);
        const int32_t id = c.table[(size_t)s * c.max_pages + page];
        if ((uint32_t)id >= c.n_pages) { if (lane == 0) cache_flag(c, TD_ERR_OOB_INDEX); continue; }
        const int64_t at = id * a.page + (j - (int64_t)page * c.page_size) * a.token + kv * a.head;
        const T *k = static_cast<const T *>(a.keys) + at, *v = static_cast<const T *>(a.values) + at;
        float x = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (lane + 32 * i < a.dim) x = fmaf(qv[i], Elem<T>::load(k + lane + 32 * i), x);
#pragma unroll
        for (int d = 16; d; d /= 2) x += __shfl_xor_sync(kFullMask, x, d);
        if (x == -CUDART_INF_F) continue;
        const float top = max_nan(x, m), keep = expf(m - top), p = expf(x - top);
        sum = sum * keep + p;
        m = top;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (lane + 32 * i < a.dim) o[i] = fmaf(p, Elem<T>::load(v + lane + 32 * i), o[i] * keep);
    }
    T *out = static_cast<T *>(a.out) + row * a.out_row + h * a.out_head;
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (lane + 32 * i < a.dim) out[lane + 32 * i] = Elem<T>::from(o[i] * inv);
    if (a.lse && lane == 0) a.lse[(size_t)row * a.n_heads + h] = sum == 0.0f ? -CUDART_INF_F : m + logf(sum);
}

}  // namespace td
