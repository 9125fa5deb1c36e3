// Attention of one new token per row over a paged cache.
//
// The work is one pass over the keys and values with a running reference and sum per row and head.  A unit is a row's
// heads over one key head, 8 or 16 at most; its tokens come in tiles of kTile.  Both products have the cache on the matrix
// instructions' long side: scores are (16 tokens) x (8 heads), results (16 columns of values) x (8 heads), so that few heads
// waste nothing; a transposition of 8 x 8 matrices turns the one's output into the other's input.  All units'
// tiles, one unit after the other, are a line that is cut into equal pieces, a piece per warp, wherever the cuts
// fall: so one long sequence and a thousand short ones load the machine alike.  A warp has its tiles brought by its own ring of
// asynchronous copies, several tiles ahead and across units; no warp waits for another.  Units that a cut
// went through leave parts (reference, sum, weighted values), joined in the order of the tokens: within a block after its
// warps are done, between blocks by the last block to arrive.  The same call gives the same bits.
#pragma once

#include "td_cache.cuh"
#include "td_mma.cuh"
#include "td_tensor.cuh"

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
    uint32_t units, per_kv;                                   // of a row: per_kv for each key head
    FastDiv by_per_kv;
    float scale2;                                             // scale * log2(e)
    float *parts;                                             // [2 per warp, then 2 per block][part floats]
    uint32_t *arrived;                                        // [blocks], zero between calls
    // groups of rows with common pages; group == 1: none.  Those of more than kMaxGroup rows are taken as `pieces` groups of like size each.
    uint32_t group, n_groups, m_blocks, m_rows;               // a group's heads over one key head in m_blocks blocks of m_rows (128 at most)
    uint32_t whole, pieces;                                   // rows of a group as the caller has them
    FastDiv by_group, by_whole, by_ratio;
    int2 *shared;                                             // [n_groups] common tokens, and a sequence that has them
    float *common;                                            // [rows * heads][dim, then maximum, sum] what the common tokens give
    float *share_parts;                                       // [2 per block]
    uint32_t *share_arrived;                                  // [blocks], zero between calls
    uint32_t lost_block, lost_tile;                           // a wait of share_wide_kernel that is taken as run out, for tests; ~0: none
};

constexpr uint32_t kTile = 16;                                // tokens of a tile
constexpr float kSlack = 8.0f;                                // how far (log2) a score may pass the reference's place before that moves
// The reference is set this far (log2) below the maximum.  Weights are rounded to T, and half has no normal numbers below 2^-14 and none below
// 2^-24: from weights of up to 2^(7 + 8) on, it keeps what lies 2^32 below the largest, so that a long row of small weights behind a large one counts.
template <typename T> constexpr float kLift = 0.0f;
template <> constexpr float kLift<__half> = 7.0f;
// A result lies among the values, but weights are rounded and their sum is not: near half's largest value, which an ordinary value may well be,
// the quotient can be a half step too large and would round to infinity.
template <typename T> __device__ __forceinline__ float fitted(float x) { return x; }
template <> __device__ __forceinline__ float fitted<__half>(float x) {
    return fabsf(x) < CUDART_INF_F ? fminf(fmaxf(x, -65504.0f), 65504.0f) : x;
}
constexpr uint32_t kLeastTiles = 2;                           // of a warp, before another block is used

// Shapes of a kernel for heads of up to 16 * kChunks elements, 8 * kN of them side by side.
template <int kChunks, int kN>
struct AttendShape {
    static constexpr uint32_t kDim = 16 * kChunks, kHeads = 8 * kN;
    static constexpr uint32_t kWarps = kChunks <= 8 ? (kN == 1 ? 12 : 8) : 4;
    static constexpr uint32_t kThreads = 32 * kWarps;
    static constexpr uint32_t kPitch = kDim * 2 + 16;         // bytes of a row in shared memory: an odd number of 16s, so that 8 rows lie in different banks
    static constexpr uint32_t kSide = kTile * kPitch;         // keys, or values, of a tile
    static constexpr uint32_t kStage = 2 * kSide;
    static constexpr bool kQueryInRegisters = kChunks * kN <= 16;
    static constexpr uint32_t kQuery = kQueryInRegisters ? 0 : kHeads * kPitch;
    static constexpr uint32_t kRoom = 216 * 1024 / kWarps;    // bytes a warp may have
    static constexpr uint32_t kFits = (kRoom - kQuery) / (kStage + 16);
    static constexpr uint32_t kStages = kFits < 6 ? kFits : 6;
    static constexpr uint32_t kWarpBytes = kStages * (kStage + 16) + kQuery;
    static constexpr uint32_t kBytes = kWarps * kWarpBytes;
    static constexpr uint32_t kPartFloats = kHeads * (kDim + 2);         // weighted values [kHeads][kDim], then {reference, sum} [kHeads]
};

// Lengths reach 2^31 - 1, so positions, which run to a tile's end, are unsigned.
struct Span {                                                 // the tokens [lo, n) of sequence s
    int32_t s, lo, n;
    __device__ __forceinline__ uint32_t tiles() const { return ((uint32_t)(n - lo) + kTile - 1) / kTile; }
    __device__ __forceinline__ uint32_t at(int32_t tile, uint32_t i) const { return (uint32_t)lo + (uint32_t)tile * kTile + i; }          // position of token i of a tile
};
// The group of a row; the rows of a group.
__device__ __forceinline__ uint32_t group_of(const AttendArgs &a, uint32_t row) {
    const uint32_t g = fast_div(row, a.by_whole);
    return a.pieces == 1 ? g : g * a.pieces + fast_div(row - g * a.whole, a.by_group);
}
__device__ __forceinline__ uint32_t rows_of(const AttendArgs &a, uint32_t group, uint32_t &first) {
    const uint32_t g = a.pieces == 1 ? group : group / a.pieces, at = (group - g * a.pieces) * a.group;
    first = g * a.whole + at;
    return first < a.n_rows ? min(min(a.group, a.whole - at), a.n_rows - first) : 0u;
}
// kOwn: without the tokens that the row's group has in common.
template <bool kOwn>
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
    if (kOwn && a.group > 1 && n > 0) p.lo = max(p.lo, a.shared[group_of(a, row)].x);          // never both: see share_plan_kernel
    return p;
}

// n / d; a 64-bit division takes some hundred instructions, and the numbers here hardly ever need one.
__device__ __forceinline__ unsigned long long quotient(unsigned long long n, unsigned long long d) {
    return ((n | d) >> 32) == 0 ? (uint32_t)n / (uint32_t)d : n / d;
}
// The line of all units' tiles; a unit has one place ahead of its tiles (what it costs to begin one), so that of a row with T
// tiles each unit has T + 1 places.  The first `more` of `warps` warps have base + 1 places each, the others base (>= 1).
struct Line {
    unsigned long long total, base;
    uint32_t warps, more;
    __device__ __forceinline__ Line(unsigned long long places, uint32_t most) : total(places) {
        warps = places < most ? (uint32_t)places : most;
        base = quotient(places, warps);
        more = (uint32_t)(places - base * warps);
    }
    __device__ __forceinline__ unsigned long long begin(uint32_t w) const {
        return w >= warps ? total : base * w + min(w, more);
    }
    __device__ __forceinline__ uint32_t warp_of(unsigned long long place) const {          // the last w with begin(w) <= place
        const unsigned long long wide = (base + 1) * more;
        return (uint32_t)(place < wide ? quotient(place, base + 1) : more + quotient(place - wide, base));
    }
};

// Places of n items, per_thread consecutive ones to a thread: sums[i] those up to and with thread i's.
template <uint32_t kThreads, typename Places>
__device__ __forceinline__ void sum_places(unsigned long long *sums, uint32_t n, uint32_t per_thread, Places places) {
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    unsigned long long mine = 0;
    for (uint32_t i = threadIdx.x * per_thread; i < min(n, (threadIdx.x + 1) * per_thread); ++i) mine += places(i);
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
    __syncthreads();
}
// The thread whose items `place` is among.
template <uint32_t kThreads>
__device__ __forceinline__ uint32_t thread_of(const unsigned long long *sums, unsigned long long place) {
    uint32_t lo = 0, hi = kThreads - 1;
    while (lo < hi) {
        const uint32_t mid = (lo + hi) / 2;
        if (sums[mid] > place) hi = mid; else lo = mid + 1;
    }
    return lo;
}

// A unit that a cut went through, and the warps that have its first and its last tile.
struct Cut {
    uint32_t row, unit, first, last, valid;
};

template <uint32_t kHeads>
__device__ __forceinline__ uint32_t heads_of(const AttendArgs &a, uint32_t unit, uint32_t &kv, uint32_t &first) {          // heads of a unit, from `first` on
    kv = fast_div(unit, a.by_per_kv);
    const uint32_t at = (unit - kv * a.per_kv) * kHeads;
    first = kv * a.ratio + at;
    return min(kHeads, a.ratio - at);
}

// What a row's head has from the tokens its group has in common; nullptr: there are none.
template <uint32_t kDim>
__device__ __forceinline__ const float *common_of(const AttendArgs &a, uint32_t row, uint32_t head) {
    if (a.group <= 1 || a.shared[group_of(a, row)].x == 0) return nullptr;
    return a.common + ((size_t)row * a.n_heads + head) * (kDim + 2);
}

// A head's result from its weighted values (pair i of a lane: columns 2 (lane + 32 i) and one more), reference and sum; `also`:
// with what its group has in common.
template <typename T, uint32_t kDim>
__device__ __forceinline__ void write_result(const AttendArgs &a, uint32_t row, uint32_t head, bool also, float2 (&v)[(kDim / 2 + 31) / 32],
                                             float top, float sum) {
    const uint32_t lane = threadIdx.x & 31u;
    const float *w = also ? common_of<kDim>(a, row, head) : nullptr;
    if (w) {
        const float2 ml = *reinterpret_cast<const float2 *>(w + kDim);
        const float most = max_nan(top, ml.x), ref = most == -CUDART_INF_F ? 0.0f : most, e = exp2_approx(top - ref), f = exp2_approx(ml.x - ref);
#pragma unroll
        for (uint32_t i = 0; i < (kDim / 2 + 31) / 32; ++i) {
            if (lane + 32 * i >= kDim / 2) continue;
            const float2 x = *reinterpret_cast<const float2 *>(w + 2 * (lane + 32 * i));
            v[i] = make_float2(fmaf(x.x, f, v[i].x * e), fmaf(x.y, f, v[i].y * e));
        }
        sum = fmaf(ml.y, f, sum * e);
        top = most;
    }
    const float inv = 1.0f / sum;
    T *out = static_cast<T *>(a.out) + row * a.out_row + head * a.out_head;
#pragma unroll
    for (uint32_t i = 0; i < (kDim / 2 + 31) / 32; ++i)
        if (2 * (lane + 32 * i) < a.dim)
            *reinterpret_cast<uint32_t *>(out + 2 * (lane + 32 * i)) = sum == 0.0f ? 0u : pair_of<T>(fitted<T>(v[i].x * inv), fitted<T>(v[i].y * inv));          // 0, also where the values are not finite
    if (a.lse && lane == 0) a.lse[(size_t)row * a.n_heads + head] = sum == 0.0f ? -CUDART_INF_F : (top + log2f(sum)) * 0.69314718055994531f;
}

// Joins the parts k = 0 .. count - 1 (part k at slot(k) of `parts`: weighted values [kRows][kDim], then {reference, sum} [kRows])
// of rows 0 .. rows - 1, by warps; emit(row, values, reference, sum) gets a row's in the layout of write_result.  It is a chain of loads
// with next to nothing between, so a warp has kRowsAtOnce rows and kPartsAtOnce parts of each on their way together: the joins
// of one sequence of 2000 tokens took 10 us value by value.  A reference of -inf means that a part has nothing; NaN stays.
template <uint32_t kDim, uint32_t kRows, int kRowsAtOnce, int kPartsAtOnce, typename Slot, typename Emit>
__device__ __forceinline__ void join_parts(const float *parts, uint32_t count, Slot slot, uint32_t rows, uint32_t worker, uint32_t workers, Emit emit) {
    constexpr uint32_t kFloats = kRows * (kDim + 2), kPairs = (kDim / 2 + 31) / 32;
    const uint32_t lane = threadIdx.x & 31u;
#pragma unroll 1
    for (uint32_t h0 = worker * kRowsAtOnce; h0 < rows; h0 += workers * kRowsAtOnce) {
        float top[kRowsAtOnce], sum[kRowsAtOnce];
        float2 v[kRowsAtOnce][kPairs];
#pragma unroll
        for (int b = 0; b < kRowsAtOnce; ++b) {
            top[b] = -CUDART_INF_F;
            sum[b] = 0.0f;
#pragma unroll
            for (uint32_t i = 0; i < kPairs; ++i) v[b][i] = make_float2(0.0f, 0.0f);
        }
        auto head = [&](int b) { return min(h0 + b, rows - 1); };
        for (uint32_t k = lane; k < count; k += 32) {
            const float *p = parts + (size_t)slot(k) * kFloats + kRows * kDim;
#pragma unroll
            for (int b = 0; b < kRowsAtOnce; ++b) top[b] = max_nan(top[b], __ldcg(p + 2 * head(b)));
        }
#pragma unroll
        for (int b = 0; b < kRowsAtOnce; ++b)
#pragma unroll
            for (int d = 1; d < 32; d *= 2) top[b] = max_nan(top[b], __shfl_xor_sync(kFullMask, top[b], d));
        for (uint32_t k0 = 0; k0 < count; k0 += 32) {
            const uint32_t some = min(32u, count - k0);
            float e[kRowsAtOnce];
#pragma unroll
            for (int b = 0; b < kRowsAtOnce; ++b) {
                e[b] = 0.0f;
                if (lane >= some) continue;
                const float2 ml = __ldcg(reinterpret_cast<const float2 *>(parts + (size_t)slot(k0 + lane) * kFloats + kRows * kDim + 2 * head(b)));
                e[b] = exp2_approx(ml.x - (top[b] == -CUDART_INF_F ? 0.0f : top[b]));
                sum[b] = fmaf(ml.y, e[b], sum[b]);
            }
            for (uint32_t j0 = 0; j0 < some; j0 += kPartsAtOnce) {
                float2 x[kPartsAtOnce][kRowsAtOnce][kPairs];
#pragma unroll
                for (int j = 0; j < kPartsAtOnce; ++j) {
                    const float *p = parts + (size_t)slot(k0 + min(j0 + j, some - 1)) * kFloats;
#pragma unroll
                    for (int b = 0; b < kRowsAtOnce; ++b)
#pragma unroll
                        for (uint32_t i = 0; i < kPairs; ++i)
                            x[j][b][i] = lane + 32 * i < kDim / 2 ? __ldcg(reinterpret_cast<const float2 *>(p + head(b) * kDim + 2 * (lane + 32 * i))) : make_float2(0.0f, 0.0f);
                }
#pragma unroll
                for (int j = 0; j < kPartsAtOnce; ++j) {
                    if (j0 + j >= some) break;
#pragma unroll
                    for (int b = 0; b < kRowsAtOnce; ++b) {
                        const float f = __shfl_sync(kFullMask, e[b], j0 + j);
#pragma unroll
                        for (uint32_t i = 0; i < kPairs; ++i) v[b][i] = make_float2(fmaf(x[j][b][i].x, f, v[b][i].x), fmaf(x[j][b][i].y, f, v[b][i].y));
                    }
                }
            }
        }
#pragma unroll
        for (int b = 0; b < kRowsAtOnce; ++b) {
#pragma unroll
            for (int d = 1; d < 32; d *= 2) sum[b] += __shfl_xor_sync(kFullMask, sum[b], d);
            if (h0 + b < rows) emit(h0 + b, v[b], top[b], sum[b]);
        }
    }
}
// A row's values, reference and sum as a part.
template <uint32_t kDim>
__device__ __forceinline__ void write_part(float *to, float *ml, const float2 (&v)[(kDim / 2 + 31) / 32], float top, float sum) {
    const uint32_t lane = threadIdx.x & 31u;
#pragma unroll
    for (uint32_t i = 0; i < (kDim / 2 + 31) / 32; ++i)
        if (lane + 32 * i < kDim / 2) *reinterpret_cast<float2 *>(to + 2 * (lane + 32 * i)) = v[i];
    if (lane == 0) *reinterpret_cast<float2 *>(ml) = make_float2(top, sum);
}

// The running reference (in units of log2), sum and weighted values of 8 * kN heads, in the layout of the matrix instructions: lane
// 4 g + t has heads 8 n + 2 t and 8 n + 2 t + 1, of every 16 columns of values those g and g + 8 places in, and of every 16
// tokens the same.  The reference follows the scores' maximum (kLift below it) only when one passes it by kSlack more: weights stay
// below 2^(kSlack + kLift), and results hardly ever have to be brought to a new reference.
template <typename T, int kChunks, int kN>
struct Fold {
    using S = AttendShape<kChunks, kN>;
    uint32_t qf[S::kQueryInRegisters ? kChunks : 1][kN][2];
    float o[kChunks][kN][4], m[kN][2], l[kN][2];

    __device__ __forceinline__ void begin() {
#pragma unroll
        for (int n = 0; n < kN; ++n) {
#pragma unroll
            for (int c = 0; c < kChunks; ++c) o[c][n][0] = o[c][n][1] = o[c][n][2] = o[c][n][3] = 0.0f;
            m[n][0] = m[n][1] = -CUDART_INF_F;
            l[n][0] = l[n][1] = 0.0f;
        }
    }
    // The heads' queries, from q + offset(head) on (negative: zeros), into registers or, for many long ones, into the warp's shared memory.
    template <typename Offset>
    __device__ __forceinline__ void query(const T *q, uint32_t shared, uint32_t dim, Offset offset) {
        const uint32_t lane = threadIdx.x & 31u, g = lane >> 2, t = lane & 3u;
        if constexpr (S::kQueryInRegisters) {
#pragma unroll
            for (int n = 0; n < kN; ++n) {
                const int64_t at = offset(n * 8 + g);
#pragma unroll
                for (int c = 0; c < kChunks; ++c)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint32_t d = c * 16 + i * 8 + t * 2;
                        qf[c][n][i] = at >= 0 && d < dim ? *reinterpret_cast<const uint32_t *>(q + at + d) : 0u;
                    }
            }
        } else {
            __syncwarp();
            for (uint32_t i = lane; i < S::kHeads * S::kDim / 8; i += 32) {
                const uint32_t h = i / (S::kDim / 8), v = i - h * (S::kDim / 8);
                const int64_t at = offset(h);
                uint4 x = make_uint4(0u, 0u, 0u, 0u);
                if (at >= 0 && v * 8 < dim) x = *reinterpret_cast<const uint4 *>(q + at + v * 8);
                store_shared(shared + h * S::kPitch + v * 16, x);
            }
            __syncwarp();
        }
    }
    // Sixteen more tokens: keys and values in shared memory, bit i of the 16 in `counts`: token i counts.
    __device__ __forceinline__ void add(uint32_t keys, uint32_t values, uint32_t shared, uint32_t counts, float scale2) {
        const uint32_t lane = threadIdx.x & 31u, g = lane >> 2, row = lane & 7u, upper = lane >> 3 & 1u, right = lane >> 4;
        constexpr int kChains = kN == 1 ? 2 : 1;              // sums that do not wait for one another
        float s[kN][4], part[kChains][kN][4] = {};
        const uint32_t key = keys + (row + upper * 8) * S::kPitch + right * 16;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            uint32_t a[4];
            load_matrices(a, key + c * 32);
            if constexpr (S::kQueryInRegisters) {
#pragma unroll
                for (int n = 0; n < kN; ++n) multiply_add<T>(part[c % kChains][n], a, qf[c][n][0], qf[c][n][1]);
            } else {
                static_assert(S::kQueryInRegisters || kN == 2, "two columns of matrices, loaded together");
                uint32_t b[4];
                load_matrices(b, shared + (row + right * 8) * S::kPitch + c * 32 + upper * 16);
                multiply_add<T>(part[0][0], a, b[0], b[1]);
                multiply_add<T>(part[0][kN - 1], a, b[2], b[3]);
            }
        }
#pragma unroll
        for (int n = 0; n < kN; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[n][i] = kChains == 2 ? part[0][n][i] + part[kChains - 1][n][i] : part[0][n][i];
        bool past = false;
#pragma unroll
        for (int n = 0; n < kN; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[n][i] = counts >> (g + (i >> 1) * 8) & 1u ? s[n][i] * scale2 : -CUDART_INF_F;
                past |= !(s[n][i] - m[n][i & 1] <= kSlack + kLift<T>);          // the difference: from 2^27 on the sum would round up by as much again
            }
        if (__any_sync(kFullMask, past)) {                    // a new reference (also where a score is NaN, which stays)
#pragma unroll
            for (int n = 0; n < kN; ++n) {
                float top[2], keep[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    top[i] = max_nan(max_nan(s[n][i], s[n][i + 2]) - kLift<T>, m[n][i]);
#pragma unroll
                    for (int d = 4; d < 32; d *= 2) top[i] = max_nan(top[i], __shfl_xor_sync(kFullMask, top[i], d));
                    keep[i] = m[n][i] == -CUDART_INF_F ? 0.0f : exp2_approx(m[n][i] - top[i]);
                    l[n][i] *= keep[i];
                    m[n][i] = top[i];
                }
#pragma unroll
                for (int c = 0; c < kChunks; ++c)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[c][n][i] *= keep[i & 1];
            }
        }
        uint32_t p[kN][2];
#pragma unroll
        for (int n = 0; n < kN; ++n) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[n][i] = exp2_approx(s[n][i] - (m[n][i & 1] == -CUDART_INF_F ? 0.0f : m[n][i & 1]));
                l[n][i & 1] += s[n][i];
            }
            // Weights are rounded to the type of the values, as the matrix instruction takes them; their sum is not.
            p[n][0] = transposed(pair_of<T>(s[n][0], s[n][1]));
            p[n][1] = transposed(pair_of<T>(s[n][2], s[n][3]));
        }
        const uint32_t value = values + (row + right * 8) * S::kPitch + upper * 16;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            uint32_t a[4];
            load_matrices_transposed(a, value + c * 32);
#pragma unroll
            for (int n = 0; n < kN; ++n) multiply_add<T>(o[c][n], a, p[n][0], p[n][1]);
        }
    }
    // The sums over all tokens, in every lane.
    __device__ __forceinline__ void end() {
#pragma unroll
        for (int n = 0; n < kN; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int d = 4; d < 32; d *= 2) l[n][i] += __shfl_xor_sync(kFullMask, l[n][i], d);
    }
    // Head 8 n + 2 t + i joined with a part of it, and as a part: values and {reference, sum}.
    __device__ __forceinline__ void join(const float *from, const float *ml, int n, int i) {
        const uint32_t g = (threadIdx.x & 31u) >> 2;
        const float2 other = *reinterpret_cast<const float2 *>(ml);
        const float top = max_nan(m[n][i], other.x), ref = top == -CUDART_INF_F ? 0.0f : top, e = exp2_approx(m[n][i] - ref), f = exp2_approx(other.x - ref);
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
#pragma unroll
            for (int k = 0; k < 2; ++k) o[c][n][i + 2 * k] = fmaf(from[c * 16 + k * 8 + g], f, o[c][n][i + 2 * k] * e);
        l[n][i] = fmaf(other.y, f, l[n][i] * e);
        m[n][i] = top;
    }
    __device__ __forceinline__ void store(float *to, float *ml, int n, int i) const {
        const uint32_t g = (threadIdx.x & 31u) >> 2;
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
#pragma unroll
            for (int k = 0; k < 2; ++k) to[c * 16 + k * 8 + g] = o[c][n][i + 2 * k];
        if (g == 0) *reinterpret_cast<float2 *>(ml) = make_float2(m[n][i], l[n][i]);
    }
    // The head's result.
    __device__ __forceinline__ void finish(T *out, float *lse, uint32_t dim, int n, int i) const {
        const uint32_t g = (threadIdx.x & 31u) >> 2;
        const float inv = 1.0f / l[n][i];
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
#pragma unroll
            for (int k = 0; k < 2; ++k)
                if (c * 16 + k * 8 < dim) out[c * 16 + k * 8 + g] = Elem<T>::from(l[n][i] == 0.0f ? 0.0f : fitted<T>(o[c][n][i + 2 * k] * inv));
        if (lse && g == 0) *lse = l[n][i] == 0.0f ? -CUDART_INF_F : (m[n][i] + log2f(l[n][i])) * 0.69314718055994531f;
    }
};

template <typename T, int kChunks, int kN>
__global__ void __launch_bounds__(AttendShape<kChunks, kN>::kThreads, 1) attend_kernel(CacheView c, AttendArgs a) {
    using S = AttendShape<kChunks, kN>;
    extern __shared__ __align__(16) uint8_t memory[];
    __shared__ unsigned long long sums[S::kThreads];          // places of all rows up to and with those of each thread
    // units that cuts went through: cut[0] came in from the block before, cut[1] goes on into the next, cut_out[w] were begun by warp w
    // and ended within the block
    __shared__ Cut cut[2], cut_out[S::kWarps];
    __shared__ uint32_t last[2];
    griddep_launch_dependents();
    griddep_wait();
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;

    // ---- this warp's share ----
    const uint32_t per_thread = (a.n_rows + S::kThreads - 1) / S::kThreads;
    if (lane == 0) cut_out[warp].valid = 0;
    if (threadIdx.x < 2) cut[threadIdx.x].valid = last[threadIdx.x] = 0;
    sum_places<S::kThreads>(sums, a.n_rows, per_thread, [&](uint32_t r) {
        return (unsigned long long)a.units * (span_of<true>(c, a, r, blockIdx.x == 0).tiles() + 1);
    });
    const unsigned long long total = sums[S::kThreads - 1];
    const uint32_t blocks = (uint32_t)min((unsigned long long)gridDim.x, quotient(total, S::kWarps * kLeastTiles) + 1);
    if (blockIdx.x >= blocks) return;
    const Line line(total, blocks * S::kWarps);
    const uint32_t w_first = blockIdx.x * S::kWarps, w_last = w_first + S::kWarps - 1, w_global = w_first + warp;
    const unsigned long long begin = line.begin(w_global), end = line.begin(w_global + 1);

    uint8_t *const mem = memory + warp * S::kWarpBytes;
    const uint32_t ring = shared_address(mem), query = ring + S::kStages * S::kStage;
    uint4 *const notes = reinterpret_cast<uint4 *>(mem + S::kStages * S::kStage + S::kQuery);          // per stage: row, unit, tokens that count and flags and heads, first head
    if (a.dim != S::kDim)                                     // columns that no copy writes
        for (uint32_t i = lane; i < S::kStages * S::kStage / 16; i += 32) reinterpret_cast<uint4 *>(mem)[i] = make_uint4(0u, 0u, 0u, 0u);
    __syncwarp();

    if (begin < end) {
        // where `begin` lies: the thread whose rows it is among, then the row
        const uint32_t lo = thread_of<S::kThreads>(sums, begin);
        unsigned long long row_place = lo ? sums[lo - 1] : 0;
        uint32_t row = lo * per_thread;
        Span span;
        for (;; ++row) {
            span = span_of<true>(c, a, row, false);
            const unsigned long long places = (unsigned long long)a.units * (span.tiles() + 1);
            if (row_place + places > begin) break;
            row_place += places;
        }
        uint32_t tiles = span.tiles();
        uint32_t unit = (uint32_t)quotient(begin - row_place, tiles + 1);
        int32_t tile = (int32_t)(begin - row_place - (unsigned long long)unit * (tiles + 1)) - 1;          // -1: the place ahead
        unsigned long long place = begin;                     // of the next tile to bring
        Span next = row + 1 < a.n_rows ? span_of<true>(c, a, row + 1, false) : Span{-1, 0, 0};

        uint32_t kv, first, heads;
        auto enter = [&]() {                                  // a unit's key head and its heads
            heads = heads_of<S::kHeads>(a, unit, kv, first);
        };
        auto leave = [&]() {                                  // to the unit behind
            tile = -1;
            if (++unit == a.units) {
                unit = 0;
                ++row;
                span = next;
                tiles = span.tiles();
                next = row + 1 < a.n_rows ? span_of<true>(c, a, row + 1, false) : Span{-1, 0, 0};
            }
            enter();
        };
        enter();
        // To the next tile; an empty unit's result is written on the way.  Then lanes 0 .. 15 fetch the numbers of its
        // tokens' pages (16 .. 31 the same), which the next call of bring() needs.
        bool more = true;
        int32_t id = -1;
        auto look = [&]() {
            while (place < end && tile < 0) {
                ++place;
                if (tiles) {
                    tile = 0;
                } else {
                    for (uint32_t h = 0; h < heads; ++h) {     // nothing, or what its group has in common
                        float2 none[(S::kDim / 2 + 31) / 32] = {};
                        write_result<T, S::kDim>(a, row, first + h, span.n > 0, none, -CUDART_INF_F, 0.0f);
                    }
                    leave();
                }
            }
            more = place < end;
            const uint32_t j = span.at(tile, lane & 15u);
            id = more && j < (uint32_t)span.n ? c.table[(size_t)span.s * c.max_pages + fast_div(j, c.by_page)] : -1;
        };
        // Brings the tile into stage `to`.
        const int64_t apart = static_cast<const T *>(a.values) - static_cast<const T *>(a.keys);
        auto bring = [&](uint32_t to) {
            const uint32_t j = span.at(tile, lane & 15u);
            const bool on = (uint32_t)id < c.n_pages;
            const uint32_t counts = __ballot_sync(kFullMask, on) & 0xffffu;
            const int64_t from = on ? id * a.page + (int64_t)(j - fast_div(j, c.by_page) * c.page_size) * a.token : 0;
            const T *keys = static_cast<const T *>(a.keys) + kv * a.head;
            const uint32_t at = ring + to * S::kStage;
            constexpr uint32_t kPer = S::kDim / 8;            // vectors of a row
#pragma unroll
            for (uint32_t i0 = 0; i0 < kTile * kPer; i0 += 32) {
                const uint32_t i = i0 + lane, r = i / kPer, v = i - r * kPer, o = r * S::kPitch + v * 16;
                const T *k = keys + __shfl_sync(kFullMask, from, r) + v * 8;
                if (kPer * 8 != a.dim && v * 8 >= a.dim) continue;
                if (counts == 0xffffu) {
                    copy_vector(at + o, k);
                    copy_vector(at + S::kSide + o, k + apart);
                } else {                                      // behind the end, or not a page: zeros, so that nothing there is used
                    const uint32_t bytes = counts >> r & 1u ? 16u : 0u;
                    copy_vector_or_zero(at + o, k, bytes);
                    copy_vector_or_zero(at + S::kSide + o, k + apart, bytes);
                }
            }
            if (!on && j < (uint32_t)span.n && unit == 0 && lane < 16) cache_flag(c, TD_ERR_OOB_INDEX);
            const bool fresh = tile == 0 || place == begin, final = tile + 1 == (int32_t)tiles, over = final || place + 1 == end;
            if (lane == 0) {
                notes[to] = make_uint4(row, unit, counts | (fresh ? 1u << 16 : 0u) | (over ? 1u << 17 : 0u) | (tile == 0 ? 1u << 18 : 0u) |
                                       (final ? 1u << 19 : 0u) | heads << 20, first);
                if (over) {                                   // a cut unit, for the joins: noted before the block's barrier
                    const bool in = place - (uint32_t)tile < begin;
                    if (in ? warp == 0 : !final) {
                        const unsigned long long tile0 = place - (uint32_t)tile;
                        const Cut u{row, unit, line.warp_of(tile0), line.warp_of(tile0 + tiles - 1), 1u};
                        if (in) cut[0] = u; else if (u.last > w_last) cut[1] = u; else cut_out[warp] = u;
                    }
                }
            }
            ++place;
            if (++tile == (int32_t)tiles) leave();
            look();
        };

        uint32_t brought = 0, used = 0, put = 0, stage = 0;   // tiles; stages of the next to bring and to use
        Fold<T, kChunks, kN> f;
        bool head_whole = false, asked = false;               // asked: the first unit's queries are on their way already
        look();
        auto ask = [&](uint32_t of_row, uint32_t of_first, uint32_t of_heads) {
            f.begin();
            f.query(static_cast<const T *>(a.q) + of_row * a.q_row + of_first * a.q_head, query, a.dim,
                    [&](uint32_t h) { return h < of_heads ? (int64_t)h * a.q_head : (int64_t)-1; });
        };
        if (more) {
            ask(row, first, heads);
            asked = true;
        }
#pragma unroll 1
        for (uint32_t turn = 0;; ++turn) {
            if (turn + 1 >= S::kStages) {                     // the ring has been filled
                if (used == brought) break;
                copy_wait<S::kStages - 2>();
                __syncwarp();
            }
            if (more) {                                       // into the stage that the last turn was done with
                bring(put);
                ++brought;
            }
            copy_commit();
            put = put + 1 == S::kStages ? 0 : put + 1;
            if (turn + 1 < S::kStages) continue;
            ++used;
            const uint4 note = notes[stage];
            const uint32_t at = ring + stage * S::kStage;
            stage = stage + 1 == S::kStages ? 0 : stage + 1;
            const uint32_t first = note.w, heads = note.z >> 20, t = lane & 3u;
            if (note.z >> 16 & 1u) {                          // a unit begins here
                head_whole = note.z >> 18 & 1u;
                if (!asked) ask(note.x, first, heads);
                asked = false;
            }
            f.add(at, at + S::kSide, query, note.z, a.scale2);
            if (note.z >> 17 & 1u) {                          // the unit, or this warp's part of it, ends here
                f.end();
                const bool whole = head_whole && (note.z >> 19 & 1u);
                float *part = a.parts + ((size_t)2 * w_global + (head_whole ? 1 : 0)) * S::kPartFloats;
#pragma unroll
                for (int n = 0; n < kN; ++n)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint32_t h = n * 8 + t * 2 + i;
                        if (h >= heads) continue;
                        if (whole) {
                            if (const float *w = common_of<S::kDim>(a, note.x, first + h)) f.join(w, w + S::kDim, n, i);
                            f.finish(static_cast<T *>(a.out) + note.x * a.out_row + (first + h) * a.out_head,
                                     a.lse ? a.lse + (size_t)note.x * a.n_heads + first + h : nullptr, a.dim, n, i);
                        } else {
                            f.store(part + h * S::kDim, part + S::kHeads * S::kDim + 2 * h, n, i);
                        }
                    }
            }
        }
    }
    copy_wait<0>();
    __syncthreads();

    // ---- units that cuts went through ----
    if (cut_out[warp].valid) {
        const Cut u = cut_out[warp];
        uint32_t kv, first;
        const uint32_t heads = heads_of<S::kHeads>(a, u.unit, kv, first);
        join_parts<S::kDim, S::kHeads, 4, 2>(a.parts, u.last - u.first + 1, [=](uint32_t k) { return 2 * (u.first + k) + (k == 0); }, heads, 0u, 1u,
                                             [&](uint32_t h, auto &v, float top, float sum) { write_result<T, S::kDim>(a, u.row, first + h, true, v, top, sum); });
    }
    if (!cut[0].valid && !cut[1].valid) return;
    // This block's share of the one and of the other, half of the warps each where there are both; then the last block of
    // a unit joins the blocks' shares.
    const bool both = cut[0].valid && cut[1].valid;
    const uint32_t half = S::kWarps / 2, side = both ? warp / half : cut[1].valid, worker = both ? warp % half : warp, workers = both ? half : S::kWarps;
    const Cut u = cut[side];
    const uint32_t from = max(u.first, w_first), to = min(u.last, w_last), b0 = u.first / S::kWarps, b1 = u.last / S::kWarps;
    float *const block_parts = a.parts + (size_t)2 * gridDim.x * S::kWarps * S::kPartFloats;
    float *const mine = block_parts + ((size_t)2 * blockIdx.x + (blockIdx.x == b0)) * S::kPartFloats;
    uint32_t kv, first;
    const uint32_t heads = heads_of<S::kHeads>(a, u.unit, kv, first);
    join_parts<S::kDim, S::kHeads, 2, 4>(a.parts, to - from + 1, [=](uint32_t k) { return 2 * (from + k) + (from + k == u.first); }, heads, worker, workers,
                                         [&](uint32_t h, auto &v, float top, float sum) {
                                             write_part<S::kDim>(mine + h * S::kDim, mine + S::kHeads * S::kDim + 2 * h, v, top, sum);
                                         });
    __threadfence();
    __syncthreads();
    if (worker == 0 && lane == 0) {
        const uint32_t before = atomicAdd(a.arrived + b0, 1u);
        last[side] = before == b1 - b0;
        if (before == b1 - b0) a.arrived[b0] = 0;
        __threadfence();
    }
    __syncthreads();
    if (last[side])
        join_parts<S::kDim, S::kHeads, 2, 4>(block_parts, b1 - b0 + 1, [=](uint32_t k) { return 2 * (b0 + k) + (k == 0); }, heads, worker, workers,
                                             [&](uint32_t h, auto &v, float top, float sum) { write_result<T, S::kDim>(a, u.row, first + h, true, v, top, sum); });
}

// ---- tokens that a group's rows have in common ----
// The responses of a GRPO group begin with the same pages.  share_plan_kernel finds how many, share_kernel takes those tokens
// once for all the group's heads over a key head (blocks of up to 128 of them), and attend_kernel takes the rest of
// each row and adds what the common tokens gave.
constexpr uint32_t kMaxGroup = 512;                           // rows
constexpr uint32_t kShareHeads = 128;                         // heads of a block: 8 warps of 16
constexpr uint32_t kShareThreads = 256;
constexpr uint32_t kLeastShared = 64;                         // common tokens
// Common tokens times the rows that need not read them: below it two more kernels cost more than they spare.  256 groups of 8, 28 heads over 4
// of 128, prompts of 150 and 300 tokens on average: 213 us without and 254 with, 288 and 289.  Above it they do not always pay: they win
// with many rows and tokens (us without and with, prompts of 2000, 32 heads over 4 of 128: 128 groups of 8 603 and 303, 256 of 4
// 692 and 455, 170 of 3 349 and 319) and lose with few (256 groups of 2 364 and 412, 24 of 4 64 and 95; prompts of 600, 170 of 3 121 and 164).  The
// caller says whether rows are to share at all.
constexpr uint32_t kLeastSpared = 2000;

// A block per group.
__global__ void __launch_bounds__(kShareThreads) share_plan_kernel(CacheView c, AttendArgs a) {
    __shared__ int32_t seqs[kMaxGroup];
    __shared__ int32_t least, lead, whole, active;
    __shared__ uint32_t equal;
    griddep_launch_dependents();
    griddep_wait();
    uint32_t first;
    const uint32_t rows = rows_of(a, blockIdx.x, first);
    if (threadIdx.x == 0) {
        least = 0x7fffffff;
        lead = kMaxGroup;
        whole = 1;
        active = 0;
    }
    __syncthreads();
    for (uint32_t r = threadIdx.x; r < rows; r += kShareThreads) {
        const Span p = span_of<false>(c, a, first + r, false);
        seqs[r] = p.n > 0 ? p.s : -1;
        if (p.n > 0) {
            atomicMin(&least, p.n);
            atomicMin(&lead, (int32_t)r);
            atomicAdd(&active, 1);
            if (p.lo > 0) whole = 0;                          // a window that has left the first tokens: nothing is shared
        }
    }
    __syncthreads();
    uint32_t pages = 0;
    if (active > 1 && whole) pages = fast_div((uint32_t)least, c.by_page);
    if (threadIdx.x == 0) equal = pages;
    __syncthreads();
    if (pages) {
        // every row's pages against the leader's, some pages at a time, all rows side by side
        const int32_t *first_row = c.table + (size_t)seqs[lead] * c.max_pages;
        constexpr uint32_t kSome = 256;
        for (uint32_t j0 = 0; j0 < pages; j0 += kSome) {
            const uint32_t some = min(kSome, pages - j0), rest = rows - lead - 1;
            const FastDiv by_some = make_fastdiv_dev(some);
#pragma unroll 4
            for (uint32_t i = threadIdx.x; i < rest * some; i += kShareThreads) {
                const uint32_t r = fast_div(i, by_some), j = j0 + i - r * some;
                const int32_t s = seqs[lead + 1 + r];
                if (s >= 0 && c.table[(size_t)s * c.max_pages + j] != first_row[j]) atomicMin(&equal, j);
            }
            __syncthreads();
            const bool over = equal < j0 + some;
            __syncthreads();
            if (over) break;
        }
    }
    if (threadIdx.x == 0) {
        const uint32_t tokens = equal * c.page_size;
        const bool worth = tokens >= kLeastShared && (unsigned long long)tokens * (uint32_t)(active - 1) >= kLeastSpared;
        a.shared[blockIdx.x] = make_int2(worth ? (int32_t)tokens : 0, pages ? seqs[lead] : 0);
    }
}

template <int kChunks, int kN>
struct ShareShape {
    using S = AttendShape<kChunks, kN>;
    static constexpr uint32_t kTokens = kChunks <= 8 ? 64 : 32;          // of a tile
    static constexpr uint32_t kSide = kTokens * S::kPitch;
    static constexpr uint32_t kStage = 2 * kSide + 16;                   // keys, values, which tokens count (a bit each)
    // Few heads leave warps idle: those take a share of a tile's tokens, and a unit's results are joined through `merge`.
    static constexpr uint32_t kSplits = kChunks <= 8 ? 4 : 1;
    static constexpr uint32_t kMerge = kChunks <= 8 ? 6 * S::kHeads * (S::kDim + 2) * 4 : 0;          // 2 x 3 or 4 x 1 or 1 x 3 warps' heads
    static constexpr uint32_t kQuery = S::kQueryInRegisters ? 0 : kShareHeads * S::kPitch;
    static constexpr uint32_t kFits = (220 * 1024 - kMerge - kQuery) / kStage;
    static constexpr uint32_t kStages = kFits < 6 ? kFits : 6;
    static constexpr uint32_t kBytes = kStages * kStage + kMerge + kQuery;
    static constexpr uint32_t kPartFloats = kShareHeads * (S::kDim + 2);
};

// A place in the line of all groups' units (blocks of heads of a key head), as attend_kernel's, a block of threads to a piece.
struct Walk {
    unsigned long long place;
    uint32_t group, unit, tiles;
    int32_t tile, tokens, seq;
    __device__ __forceinline__ void enter(const AttendArgs &a, uint32_t per_tile) {
        while (group < a.n_groups && a.shared[group].x == 0) ++group;
        const int2 p = group < a.n_groups ? a.shared[group] : make_int2(0, 0);
        tokens = p.x;
        seq = p.y;
        tiles = ((uint32_t)tokens + per_tile - 1) / per_tile;
    }
    __device__ __forceinline__ bool here(unsigned long long end) {          // to a tile, if there is one
        if (place < end && tile < 0) {
            ++place;
            tile = 0;
        }
        return place < end;
    }
    __device__ __forceinline__ void step(const AttendArgs &a, uint32_t units, uint32_t per_tile) {
        ++place;
        if (++tile < (int32_t)tiles) return;
        tile = -1;
        if (++unit < units) return;
        unit = 0;
        ++group;
        enter(a, per_tile);
    }
};
struct ShareCut {
    unsigned long long place;
    uint32_t group, unit, tiles, valid;
};

// Units that were cut: the last of their blocks to come joins the parts.
template <uint32_t kDim>
__device__ __forceinline__ void join_shares(const AttendArgs &a, const Line &line, const ShareCut &cut_in, const ShareCut &cut_out, uint32_t *last) {
    const uint32_t warp = threadIdx.x >> 5;
#pragma unroll 1
    for (uint32_t side = 0; side < 2; ++side) {
        const ShareCut u = side == 0 ? cut_in : cut_out;
        if (!u.valid) continue;
        const uint32_t b0 = line.warp_of(u.place + 1), b1 = line.warp_of(u.place + u.tiles);
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) {
            *last = atomicAdd(a.share_arrived + b0, 1u) == b1 - b0;
            if (*last) a.share_arrived[b0] = 0;
            __threadfence();
        }
        __syncthreads();
        const bool joins = *last;
        __syncthreads();
        if (!joins) continue;
        const uint32_t m_block = u.unit / a.kv_heads, kv = u.unit - m_block * a.kv_heads, first = m_block * a.m_rows, count = min(a.m_rows, a.group * a.ratio - first);
        uint32_t first_row;
        const uint32_t rows = rows_of(a, u.group, first_row);
        join_parts<kDim, kShareHeads, 4, 2>(a.share_parts, b1 - b0 + 1, [=](uint32_t k) { return 2 * (b0 + k) + (k == 0); }, count, warp, kShareThreads / 32,
                                               [&](uint32_t r, auto &v, float top, float sum) {
                                                   const uint32_t rr = fast_div(first + r, a.by_ratio);
                                                   if (rr >= rows) return;
                                                   float *to = a.common + ((size_t)(first_row + rr) * a.n_heads + kv * a.ratio + first + r - rr * a.ratio) * (kDim + 2);
                                                   write_part<kDim>(to, to + kDim, v, top, sum);
                                               });
    }
}

template <typename T, int kChunks, int kN>
__global__ void __launch_bounds__(kShareThreads, 1) share_kernel(CacheView c, AttendArgs a) {
    using S = AttendShape<kChunks, kN>;
    using H = ShareShape<kChunks, kN>;
    extern __shared__ __align__(16) uint8_t memory[];
    __shared__ unsigned long long sums[kShareThreads];
    __shared__ uint32_t last;
    griddep_launch_dependents();
    griddep_wait();
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, units = a.kv_heads * a.m_blocks;
    const uint32_t per_thread = (a.n_groups + kShareThreads - 1) / kShareThreads;
    auto places_of = [&](uint32_t g) {
        const uint32_t tokens = (uint32_t)a.shared[g].x;
        return tokens ? (unsigned long long)units * ((tokens + H::kTokens - 1) / H::kTokens + 1) : 0ull;
    };
    sum_places<kShareThreads>(sums, a.n_groups, per_thread, places_of);
    const unsigned long long total = sums[kShareThreads - 1];
    if (total == 0) return;
    const Line line(total, gridDim.x);                        // a block to a piece
    if (blockIdx.x >= line.warps) return;
    const unsigned long long begin = line.begin(blockIdx.x), end = line.begin(blockIdx.x + 1);

    // stages (keys and values), then the tokens that count of each
    const uint32_t ring = shared_address(memory);
    uint32_t *const counts = reinterpret_cast<uint32_t *>(memory + H::kStages * 2 * H::kSide);
    float *const merge = reinterpret_cast<float *>(memory + H::kStages * H::kStage);
    const uint32_t query = ring + H::kStages * H::kStage + H::kMerge + warp * (H::kQuery / 8);
    if (a.dim != S::kDim)                                     // columns that no copy writes
        for (uint32_t i = threadIdx.x; i < H::kStages * 2 * H::kSide / 16; i += kShareThreads) reinterpret_cast<uint4 *>(memory)[i] = make_uint4(0u, 0u, 0u, 0u);
    __syncthreads();

    Walk load;
    {
        const uint32_t lo = thread_of<kShareThreads>(sums, begin);
        unsigned long long before = lo ? sums[lo - 1] : 0;
        load.group = lo * per_thread;
        for (;; ++load.group) {
            const unsigned long long places = places_of(load.group);
            if (before + places > begin) break;
            before += places;
        }
        load.enter(a, H::kTokens);
        load.place = begin;
        load.unit = (uint32_t)quotient(begin - before, load.tiles + 1);
        load.tile = (int32_t)(begin - before - (unsigned long long)load.unit * (load.tiles + 1)) - 1;
    }
    Walk use = load;
    constexpr uint32_t kPer = S::kDim / 8, kCopies = H::kTokens * kPer / kShareThreads;          // vectors of a row, and of a thread
    static_assert(H::kTokens * kPer % kShareThreads == 0, "a tile is the same work for all threads");
    bool more = true;
    int32_t ids[kCopies];                                     // pages of the tokens this thread copies next
    int32_t id = -1;                                          // page of token `threadIdx.x`
    const int64_t apart = static_cast<const T *>(a.values) - static_cast<const T *>(a.keys);
    auto look = [&]() {
        more = load.here(end);
        if (!more) return;
        const int32_t *row = c.table + (size_t)load.seq * c.max_pages;
        const uint32_t j0 = (uint32_t)load.tile * H::kTokens, j = j0 + threadIdx.x, tokens = (uint32_t)load.tokens;
        id = threadIdx.x < H::kTokens && j < tokens ? row[fast_div(j, c.by_page)] : -1;
#pragma unroll
        for (uint32_t k = 0; k < kCopies; ++k) {
            const uint32_t jk = j0 + (threadIdx.x + k * kShareThreads) / kPer;
            ids[k] = jk < tokens ? row[fast_div(jk, c.by_page)] : -1;
        }
    };
    auto bring = [&](uint32_t to) {
        const uint32_t j0 = (uint32_t)load.tile * H::kTokens;
        const T *keys = static_cast<const T *>(a.keys) + (load.unit % a.kv_heads) * a.head;
        const uint32_t at = ring + to * 2 * H::kSide;
#pragma unroll
        for (uint32_t k = 0; k < kCopies; ++k) {
            const uint32_t i = threadIdx.x + k * kShareThreads, r = i / kPer, v = i - r * kPer, o = r * S::kPitch + v * 16;
            const uint32_t j = j0 + r, bytes = (uint32_t)ids[k] < c.n_pages ? 16u : 0u;
            const int64_t from = bytes ? ids[k] * a.page + (int64_t)(j - fast_div(j, c.by_page) * c.page_size) * a.token + v * 8 : 0;
            if (kPer * 8 != a.dim && v * 8 >= a.dim) continue;
            copy_vector_or_zero(at + o, keys + from, bytes);
            copy_vector_or_zero(at + H::kSide + o, keys + from + apart, bytes);
        }
        if (threadIdx.x < H::kTokens) {
            const uint32_t which = __ballot_sync(kFullMask, (uint32_t)id < c.n_pages);
            if (lane == 0) counts[to * 4 + warp] = which;
            if ((uint32_t)id >= c.n_pages && j0 + threadIdx.x < (uint32_t)load.tokens && load.unit == 0) cache_flag(c, TD_ERR_OOB_INDEX);
        }
        load.step(a, units, H::kTokens);
        look();
    };
    uint32_t stage = 0, put = H::kStages - 1, m_count = 0, m_tile = 0, split = 0, splits = 1, wide = 1;
    look();
    for (uint32_t i = 0; i + 1 < H::kStages; ++i) {
        if (more) bring(i);
        copy_commit();
    }
    Fold<T, kChunks, kN> f;
    ShareCut cut_in{}, cut_out{};
    bool active = false, head_whole = false;
#pragma unroll 1
    while (use.here(end)) {
        copy_wait<H::kStages - 2>();
        __syncthreads();                                      // the tile is here, and the stage of the last turn is free
        if (more) bring(put);
        copy_commit();
        put = put + 1 == H::kStages ? 0 : put + 1;
        const uint32_t m_block = use.unit / a.kv_heads, kv = use.unit - m_block * a.kv_heads, m_first = m_block * a.m_rows;
        // The row and head of the block's row i (ratio rows of heads per row of the group), or false.
        auto at_row = [&](uint32_t i, uint32_t &row, uint32_t &head) {
            const uint32_t rr = fast_div(m_first + i, a.by_ratio);
            const bool there = rr < rows_of(a, use.group, row);
            row += rr;
            head = kv * a.ratio + m_first + i - rr * a.ratio;
            return i < m_count && there;
        };
        if (use.tile == 0 || use.place == begin) {            // a unit begins here
            head_whole = use.tile == 0;
            m_count = min(a.m_rows, a.group * a.ratio - m_first);
            const uint32_t m_tiles = (m_count + S::kHeads - 1) / S::kHeads;
            wide = m_tiles <= 1 ? 1 : m_tiles <= 2 ? 2 : m_tiles <= 4 ? 4 : 8;
            splits = min(H::kSplits, 8 / wide);
            m_tile = warp & (wide - 1);
            split = warp / wide;
            active = m_tile < m_tiles && split < splits;
            if (active) {
                f.begin();
                f.query(static_cast<const T *>(a.q), query, a.dim, [&](uint32_t h) {
                    uint32_t row, head;
                    return at_row(m_tile * S::kHeads + h, row, head) ? row * a.q_row + head * a.q_head : (int64_t)-1;
                });
            }
        }
        if (active) {
            const uint32_t at = ring + stage * 2 * H::kSide;
#pragma unroll 1
            for (uint32_t sub = split; sub < H::kTokens / 16; sub += splits) {
                const uint32_t which = counts[stage * 4 + sub / 2] >> (sub & 1u) * 16 & 0xffffu;
                if (which) f.add(at + sub * 16 * S::kPitch, at + H::kSide + sub * 16 * S::kPitch, query, which, a.scale2);
            }
        }
        stage = stage + 1 == H::kStages ? 0 : stage + 1;
        const bool final = use.tile + 1 == (int32_t)use.tiles;
        if (final || use.place + 1 == end) {                  // the unit, or this block's part of it, ends here
            const uint32_t t = lane & 3u;
            if (active) f.end();
            auto merged = [&](uint32_t k, int n, int i) { return merge + (size_t)(((k - 1) * wide + m_tile) * S::kHeads + n * 8 + t * 2 + i) * (S::kDim + 2); };
            if (splits > 1) {
                if (active && split > 0) {
#pragma unroll
                    for (int n = 0; n < kN; ++n)
#pragma unroll
                        for (int i = 0; i < 2; ++i) f.store(merged(split, n, i), merged(split, n, i) + S::kDim, n, i);
                }
                __syncthreads();
                if (active && split == 0) {
#pragma unroll 1
                    for (uint32_t k = 1; k < splits; ++k) {
#pragma unroll
                        for (int n = 0; n < kN; ++n)
#pragma unroll
                            for (int i = 0; i < 2; ++i) f.join(merged(k, n, i), merged(k, n, i) + S::kDim, n, i);
                    }
                }
            }
            const bool whole = head_whole && final;
            if (active && split == 0) {
#pragma unroll
                for (int n = 0; n < kN; ++n)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint32_t r = m_tile * S::kHeads + n * 8 + t * 2 + i;
                        uint32_t row, head;
                        if (!at_row(r, row, head)) continue;
                        if (whole) {
                            float *to = a.common + ((size_t)row * a.n_heads + head) * (S::kDim + 2);
                            f.store(to, to + S::kDim, n, i);
                        } else {
                            float *to = a.share_parts + ((size_t)2 * blockIdx.x + (head_whole ? 1 : 0)) * H::kPartFloats;
                            f.store(to + r * S::kDim, to + kShareHeads * S::kDim + 2 * r, n, i);
                        }
                    }
            }
            if (!whole) {
                const ShareCut cut{use.place - (uint32_t)use.tile - 1, use.group, use.unit, use.tiles, 1u};
                if (head_whole) cut_out = cut; else cut_in = cut;
            }
        }
        use.step(a, units, H::kTokens);
    }
    copy_wait<0>();
    join_shares<S::kDim>(a, line, cut_in, cut_out, &last);
}

// The same for heads of up to 128 elements, the products on the tensor memory: 128 heads by 128 tokens at a time, scores and weights
// never in shared memory.  Two threads have a head's 64 scores each.  While the threads turn a tile's scores into weights, the
// tensor cores take the last tile's values and the next tile's scores: per tile of 128 tokens there are
//   scores i + 1 = queries keys   ->   (threads: weights i from scores i)   ->   results += weights i values i.
// Keys come three tiles and values one tile ahead through 16-byte copies that put each vector where the products expect it, so any
// pages and strides will do.  The reference is moved as in Fold: the weights are first taken against the one there is, and
// only where a score passed it is the tile taken again.
template <int kChunks>
struct WideShape {
    static constexpr uint32_t kDim = 16 * kChunks, kHalves = (kChunks + 3) / 4, kColumns = 64 * kHalves;
    static constexpr uint32_t kTokens = 128, kHalf = kTokens * 128, kSide = kHalves * kHalf;
    static constexpr uint32_t kKeys = 3, kValues = 2;         // tiles of each in shared memory
    static constexpr uint32_t kBytes = (kKeys + kValues + 1) * kSide + 1024;
    static constexpr uint32_t kPartFloats = kShareHeads * (kDim + 2);
    static constexpr uint32_t kScores = 0, kResults = 256, kWeights = 384, kTensor = 512;          // columns of tensor memory: 2 x 128, 128, 2 x 64
};

template <typename T, int kChunks>
__global__ void __launch_bounds__(kShareThreads, 1) share_wide_kernel(CacheView c, AttendArgs a) {
    using W = WideShape<kChunks>;
    extern __shared__ __align__(16) uint8_t memory[];
    __shared__ unsigned long long sums[kShareThreads];
    __shared__ int64_t offsets[4][W::kTokens];                // of a tile's tokens; -1: does not count
    __shared__ uint32_t counts[8][W::kTokens / 32];
    __shared__ float exchange[2][kShareHeads];
    __shared__ __align__(8) unsigned long long bars[4];       // scores of even and odd tiles, results, all products where a wait ran out
    __shared__ uint32_t tensor_at, failed, last;
    griddep_launch_dependents();
    griddep_wait();
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, units = a.kv_heads * a.m_blocks;
    const uint32_t per_thread = (a.n_groups + kShareThreads - 1) / kShareThreads;
    auto places_of = [&](uint32_t g) {
        const uint32_t tokens = (uint32_t)a.shared[g].x;
        return tokens ? (unsigned long long)units * ((tokens + W::kTokens - 1) / W::kTokens + 1) : 0ull;
    };
    sum_places<kShareThreads>(sums, a.n_groups, per_thread, places_of);
    const unsigned long long total = sums[kShareThreads - 1];
    if (total == 0) return;
    const Line line(total, gridDim.x);                        // a block to a piece
    if (blockIdx.x >= line.warps) return;
    const unsigned long long begin = line.begin(blockIdx.x), end = line.begin(blockIdx.x + 1);

    const uint32_t memory_at = shared_address(memory), pad = (1024u - memory_at % 1024u) % 1024u;
    const uint32_t queries = memory_at + pad, keys = queries + W::kSide, values = keys + W::kKeys * W::kSide;
    const uint32_t bar = shared_address(bars);
    if (a.dim != W::kColumns)                                 // columns that no copy writes
        for (uint32_t i = threadIdx.x; i < (W::kKeys + W::kValues + 1) * W::kSide / 16; i += kShareThreads)
            reinterpret_cast<uint4 *>(memory + pad)[i] = make_uint4(0u, 0u, 0u, 0u);
    if (threadIdx.x == 0) {
        failed = 0;
        for (uint32_t i = 0; i < 4; ++i) product_bar_init(bar + 8 * i);
    }
    __syncwarp();
    if (warp == 0) tensor_alloc(shared_address(&tensor_at), W::kTensor);

    Walk ahead;
    {
        const uint32_t lo = thread_of<kShareThreads>(sums, begin);
        unsigned long long before = lo ? sums[lo - 1] : 0;
        ahead.group = lo * per_thread;
        for (;; ++ahead.group) {
            const unsigned long long places = places_of(ahead.group);
            if (before + places > begin) break;
            before += places;
        }
        ahead.enter(a, W::kTokens);
        ahead.place = begin;
        ahead.unit = (uint32_t)quotient(begin - before, ahead.tiles + 1);
        ahead.tile = (int32_t)(begin - before - (unsigned long long)ahead.unit * (ahead.tiles + 1)) - 1;
    }
    Walk use = ahead;
    // Where the tokens of the tile that `ahead` is at lie: looked up by 128 threads, noted later as those of tile `number`.
    int32_t id = -1;
    uint32_t token = 0, ahead_unit = 0;
    bool there = false, counted = false;
    auto look = [&]() {
        there = ahead.here(end);
        id = -1;
        counted = false;
        if (!there) return;
        ahead_unit = ahead.unit;
        token = (uint32_t)ahead.tile * W::kTokens + threadIdx.x;
        counted = threadIdx.x < W::kTokens && token < (uint32_t)ahead.tokens;
        if (counted) id = c.table[(size_t)ahead.seq * c.max_pages + fast_div(token, c.by_page)];
        ahead.step(a, units, W::kTokens);
    };
    auto note = [&](uint32_t number) {
        if (threadIdx.x >= W::kTokens) return;
        const bool on = (uint32_t)id < c.n_pages;
        offsets[number & 3u][threadIdx.x] =
            on ? id * a.page + (int64_t)(token - fast_div(token, c.by_page) * c.page_size) * a.token + (ahead_unit % a.kv_heads) * a.head : -1;
        if (counted && !on && ahead_unit == 0) cache_flag(c, TD_ERR_OOB_INDEX);
        const uint32_t which = __ballot_sync(kFullMask, on);
        if (lane == 0) counts[number & 7u][warp] = which;
    };
    // Vectors of tile `number` from `from` to `to`.
    auto bring = [&](const void *from, uint32_t to, uint32_t number) {
        constexpr uint32_t kPer = 8 * W::kHalves;
#pragma unroll
        for (uint32_t k = 0; k < W::kTokens * kPer / kShareThreads; ++k) {
            const uint32_t i = threadIdx.x + k * kShareThreads, r = i / kPer, v = i - r * kPer;
            const int64_t at = offsets[number & 3u][r];
            if (v * 8 >= a.dim) continue;
            copy_vector_or_zero(to + (v >> 3) * W::kHalf + r * 128 + ((v ^ r) & 7u) * 16, static_cast<const T *>(from) + (at < 0 ? 0 : at + v * 8), at < 0 ? 0u : 16u);
        }
    };
    uint32_t tiles_noted = 0;
    for (; tiles_noted < 4; ++tiles_noted) {
        look();
        note(tiles_noted);
    }
    tensor_before_sync();
    __syncthreads();
    tensor_after_sync();
    const uint32_t tensor = tensor_at, mine = tensor + ((warp & 3u) * 32 << 16), half = warp >> 2, my_row = (warp & 3u) * 32 + lane;
    // copies in groups: {keys 0}, {keys 1}, {keys 2, values 0}, then {keys i + 3, values i + 1} in turn i; tiles behind the last are zeros
    bring(a.keys, keys, 0);
    copy_commit();
    bring(a.keys, keys + W::kSide, 1);
    copy_commit();
    bring(a.keys, keys + 2 * W::kSide, 2);
    bring(a.values, values, 0);
    copy_commit();

    auto heads_in = [&](const Walk &w, uint32_t &kv, uint32_t &first) {
        const uint32_t m_block = w.unit / a.kv_heads;
        kv = w.unit - m_block * a.kv_heads;
        first = m_block * a.m_rows;
        return min(a.m_rows, a.group * a.ratio - first);
    };
    // The queries of a unit into shared memory, zeros behind them.
    auto ask = [&](const Walk &w) {
        uint32_t kv, first, first_row;
        const uint32_t n = heads_in(w, kv, first), rows = rows_of(a, w.group, first_row);
        constexpr uint32_t kPer = 8 * W::kHalves;
#pragma unroll 4
        for (uint32_t k = 0; k < kShareHeads * kPer / kShareThreads; ++k) {
            const uint32_t i = threadIdx.x + k * kShareThreads, r = i / kPer, v = i - r * kPer, rr = fast_div(first + r, a.by_ratio);
            uint4 x = make_uint4(0u, 0u, 0u, 0u);
            if (r < n && rr < rows && v * 8 < a.dim)
                x = *reinterpret_cast<const uint4 *>(static_cast<const T *>(a.q) + (first_row + rr) * a.q_row + (kv * a.ratio + first + r - rr * a.ratio) * a.q_head + v * 8);
            store_shared(queries + (v >> 3) * W::kHalf + r * 128 + ((v ^ r) & 7u) * 16, x);
        }
    };
    auto score = [&](uint32_t number) {                       // scores of tile `number`, by one thread
        const uint32_t at = keys + number % W::kKeys * W::kSide;
#pragma unroll
        for (uint32_t k = 0; k < 4 * W::kHalves; ++k)
            product(tensor + W::kScores + (number & 1u) * 128, shared_matrix(queries + (k >> 2) * W::kHalf + (k & 3u) * 32, 1024, 16),
                    shared_matrix(at + (k >> 2) * W::kHalf + (k & 3u) * 32, 1024, 16), product_kind<T>(128, false), k > 0);
        product_commit(bar + 8 * (number & 1u));
    };
    bool fine = true;
    uint32_t i = 0;                                           // the tile of this turn
    ShareCut cut_in{}, cut_out{};
    bool head_whole = false;
    float m = -CUDART_INF_F, l = 0.0f;
    // Where what a unit gives this thread's row goes: its values, and its reference and sum.  False: nowhere.
    auto place_of = [&](const Walk &w, bool whole, float *&to, float *&ml) {
        uint32_t kv, first, row;
        const uint32_t n = heads_in(w, kv, first), rr = fast_div(first + my_row, a.by_ratio), head = kv * a.ratio + first + my_row - rr * a.ratio;
        const bool there = rr < rows_of(a, w.group, row);
        row += rr;
        float *const part = a.share_parts + ((size_t)2 * blockIdx.x + (head_whole ? 1 : 0)) * W::kPartFloats;
        to = whole ? a.common + ((size_t)row * a.n_heads + head) * (W::kDim + 2) : part + my_row * W::kDim;
        ml = whole ? to + W::kDim : part + kShareHeads * W::kDim + 2 * my_row;
        return my_row < n && there;
    };
    auto cut_of = [&](const Walk &w) {
        const ShareCut cut{w.place - (uint32_t)w.tile - 1, w.group, w.unit, w.tiles, 1u};
        if (head_whole) cut_out = cut; else cut_in = cut;
    };
    use.here(end);
    if (use.place < end) {
        ask(use);
        copy_wait<2>();
        shared_for_products();
        __syncthreads();
        if (threadIdx.x == 0) {
            tensor_after_sync();
            score(0);
        }
    }
#pragma unroll 1
    for (; use.here(end); ++i) {
        Walk next = use;
        next.step(a, units, W::kTokens);
        const bool more = next.here(end), other = more && next.tile == 0;
        copy_wait<1>();                                       // keys i + 1
        if (other) {                                          // the next tile is another unit's: its queries, once the scores of this one are done
            fine &= product_wait(bar + 8 * (i & 1u), i >> 1 & 1u);
            ask(next);
        }
        shared_for_products();
        __syncthreads();
        if (more && threadIdx.x == 0) {
            tensor_after_sync();
            score(i + 1);
        }
        __syncwarp();
        const bool fresh = use.tile == 0 || use.place == begin;
        if (fresh) {
            head_whole = use.tile == 0;
            m = -CUDART_INF_F;
            l = 0.0f;
        }
        look();
        // Half of the warps copy before they weigh and half behind it, so that the one's copies go with the other's arithmetic.
        if (i > 0) fine &= product_wait(bar + 16, (i - 1) & 1u);          // results of the last tile: its values' place is free
        fine &= product_wait(bar + 8 * (i & 1u), i >> 1 & 1u);            // scores of this tile: its keys' place is free
        fine &= blockIdx.x != a.lost_block || i != a.lost_tile;
        auto copies = [&]() {
            bring(a.keys, keys + i % W::kKeys * W::kSide, i + 3);
            bring(a.values, values + (i + 1) % W::kValues * W::kSide, i + 1);
        };
        if (half == 0) copies();
        // scores to weights
        __syncwarp();
        tensor_after_sync();
        float x[64];
        {
            uint32_t r[4][16];
#pragma unroll
            for (int k = 0; k < 4; ++k) tensor_load16(r[k], mine + W::kScores + (i & 1u) * 128 + half * 64 + 16 * k);
            tensor_wait_loads();
#pragma unroll
            for (int k = 0; k < 64; ++k) x[k] = __uint_as_float(r[k >> 4][k & 15]);
        }
        const uint32_t which[2] = {counts[i & 7u][half * 2], counts[i & 7u][half * 2 + 1]};
        if ((which[0] & which[1]) != ~0u) {
#pragma unroll
            for (int k = 0; k < 64; ++k) x[k] = which[k >> 5] >> (k & 31) & 1u ? x[k] * a.scale2 : -CUDART_INF_F;
        } else {
#pragma unroll
            for (int k = 0; k < 64; ++k) x[k] *= a.scale2;
        }
        auto weigh = [&](float ref, float &sum) {             // the largest of the weights, which go to tensor memory
            float most = 0.0f;
            float part[4] = {};
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                uint32_t p[16];
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const float u = exp2_approx(x[32 * k + 2 * j] - ref), w = exp2_approx(x[32 * k + 2 * j + 1] - ref);
                    part[j & 3] += u + w;
                    most = max_nan(most, max_nan(u, w));
                    p[j] = pair_of<T>(u, w);                  // rounded as in Fold
                }
                tensor_store16(mine + W::kWeights + (i & 1u) * 64 + half * 32 + 16 * k, p);
            }
            sum = (part[0] + part[1]) + (part[2] + part[3]);
            return most;
        };
        float sum = 0.0f;
        bool past = fresh;                                    // a unit's first tile sets the reference
        if (!fresh) {
            past = !(weigh(m == -CUDART_INF_F ? 0.0f : m, sum) <= (kLift<T> == 7.0f ? 32768.0f : 256.0f));          // 2^(kSlack + kLift)
            if (m == -CUDART_INF_F) {                         // nothing counted so far
#pragma unroll
                for (int k = 0; k < 64; ++k) past |= !(x[k] == -CUDART_INF_F);
            }
        }
        if (half == 1) copies();
        copy_commit();
        copy_wait<1>();                                       // values i
        shared_for_products();
        if (!fine) failed = 1;
        __syncwarp();
        tensor_wait_stores();
        tensor_before_sync();
        const bool again = __syncthreads_or(past || !fine);
        if (again && failed) break;                           // a wait ran out: never seen
        note(i + 4);
        if (again) {
            float top = x[0];
#pragma unroll
            for (int k = 1; k < 64; ++k) top = max_nan(top, x[k]);
            exchange[half][my_row] = top;
            __syncthreads();
            top = max_nan(max_nan(exchange[0][my_row], exchange[1][my_row]) - kLift<T>, m);
            const float keep = m == -CUDART_INF_F ? 0.0f : exp2_approx(m - top);
            if (!fresh) {
                tensor_after_sync();
#pragma unroll
                for (uint32_t k = 0; k < W::kColumns / 32; ++k) {
                    uint32_t r[16];
                    const uint32_t at = mine + W::kResults + half * (W::kColumns / 2) + 16 * k;
                    tensor_load16(r, at);
                    tensor_wait_loads();
#pragma unroll
                    for (int j = 0; j < 16; ++j) r[j] = __float_as_uint(__uint_as_float(r[j]) * keep);
                    tensor_store16(at, r);
                }
            }
            m = top;
            l *= keep;
            weigh(m == -CUDART_INF_F ? 0.0f : m, sum);
            tensor_wait_stores();
            tensor_before_sync();
            __syncthreads();
        }
        l += sum;
        if (threadIdx.x == 0) {
            tensor_after_sync();
            const uint32_t at = values + i % W::kValues * W::kSide;
#pragma unroll
            for (uint32_t k = 0; k < 8; ++k)
                product_from_tensor(tensor + W::kResults, tensor + W::kWeights + (i & 1u) * 64 + 8 * k, shared_matrix(at + k * 2048, 1024, W::kHalf),
                                    product_kind<T>(W::kColumns, true), !fresh || k > 0);
            product_commit(bar + 16);
        }
        __syncwarp();
        const bool final = use.tile + 1 == (int32_t)use.tiles;
        if (final || use.place + 1 == end) {                  // the unit, or this block's part of it, ends here
            exchange[half][my_row] = l;
            fine &= product_wait(bar + 16, i & 1u);
            if (!fine) failed = 1;
            __syncthreads();
            tensor_after_sync();
            const bool whole = head_whole && final;
            float *to, *ml;
            const bool writes = place_of(use, whole, to, ml);
#pragma unroll
            for (uint32_t k = 0; k < W::kColumns / 32; ++k) {
                uint32_t r[16];
                const uint32_t column = half * (W::kColumns / 2) + 16 * k;
                tensor_load16(r, mine + W::kResults + column);
                tensor_wait_loads();
                if (writes && column < W::kDim)
#pragma unroll
                    for (int j = 0; j < 16; j += 2) *reinterpret_cast<float2 *>(to + column + j) = make_float2(__uint_as_float(r[j]), __uint_as_float(r[j + 1]));
            }
            if (writes && half == 0) *reinterpret_cast<float2 *>(ml) = failed ? make_float2(CUDART_NAN_F, CUDART_NAN_F) : make_float2(m, exchange[0][my_row] + exchange[1][my_row]);
            tensor_before_sync();                             // read before the next unit's results are begun
            if (!whole) cut_of(use);
        }
        use.step(a, units, W::kTokens);
    }
    copy_wait<0>();
    // A wait ran out (never seen): the block's units that are not done get NaN, so that their heads' results are NaN and nothing of an
    // earlier call is taken for theirs, and the block arrives where it is counted on.  What is still being computed is waited for, again with
    // a limit, before the tensor memory is given back.
    if (failed) {
        if (threadIdx.x == 0) {
            cache_flag(c, TD_ERR_COPY_TIMEOUT);
            product_commit(bar + 24);
            product_wait(bar + 24, 0u);
        }
        for (; use.here(end); use.step(a, units, W::kTokens)) {
            if (use.tile == 0 || use.place == begin) head_whole = use.tile == 0;
            const bool final = use.tile + 1 == (int32_t)use.tiles, whole = head_whole && final;
            if (!final && use.place + 1 != end) continue;
            float *to, *ml;
            if (place_of(use, whole, to, ml) && half == 0) *reinterpret_cast<float2 *>(ml) = make_float2(CUDART_NAN_F, CUDART_NAN_F);
            if (!whole) cut_of(use);
        }
    }
    tensor_before_sync();
    __syncthreads();
    if (warp == 0) tensor_free(tensor, W::kTensor);
    join_shares<W::kDim>(a, line, cut_in, cut_out, &last);
}

// ---- a cache of float ----
// Float keys and values would lose 13 bits to the matrix instructions, so they are multiplied as they are: a block per row and 8 heads
// of a key head, a token at a time per warp (a lane has every 32nd column), the warps' results joined at the end.
constexpr uint32_t kFloatThreads = 256, kFloatHeads = 8, kFloatColumns = 8;          // columns of a lane: dim <= 256
__global__ void __launch_bounds__(kFloatThreads) attend_float_kernel(CacheView c, AttendArgs a) {
    constexpr uint32_t kWarps = kFloatThreads / 32;
    __shared__ float values[kWarps][32 * kFloatColumns], ml[kWarps][2];
    griddep_launch_dependents();
    griddep_wait();
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    const uint32_t row = (uint32_t)(blockIdx.x / a.units), unit = blockIdx.x - row * a.units;
    uint32_t kv, first;
    const uint32_t heads = heads_of<kFloatHeads>(a, unit, kv, first);
    const Span span = span_of<false>(c, a, row, unit == 0 && threadIdx.x == 0);
    const float *q = static_cast<const float *>(a.q) + row * a.q_row + first * a.q_head;
    float qv[kFloatHeads][kFloatColumns], o[kFloatHeads][kFloatColumns], m[kFloatHeads], l[kFloatHeads];
#pragma unroll
    for (uint32_t h = 0; h < kFloatHeads; ++h) {
        m[h] = -CUDART_INF_F;
        l[h] = 0.0f;
#pragma unroll
        for (uint32_t i = 0; i < kFloatColumns; ++i) {
            o[h][i] = 0.0f;
            qv[h][i] = h < heads && lane + 32 * i < a.dim ? q[h * a.q_head + lane + 32 * i] * a.scale2 : 0.0f;
        }
    }
    for (uint32_t j = span.at(0, warp); j < (uint32_t)span.n; j += kWarps) {
        const uint32_t page = fast_div(j, c.by_page);
        const int32_t id = c.table[(size_t)span.s * c.max_pages + page];
        if ((uint32_t)id >= c.n_pages) {
            if (unit == 0 && lane == 0) cache_flag(c, TD_ERR_OOB_INDEX);
            continue;
        }
        const int64_t at = id * a.page + ((int64_t)j - (int64_t)page * c.page_size) * a.token + kv * a.head;
        float k[kFloatColumns], v[kFloatColumns], x[kFloatHeads];
#pragma unroll
        for (uint32_t i = 0; i < kFloatColumns; ++i) {
            const bool on = lane + 32 * i < a.dim;
            k[i] = on ? static_cast<const float *>(a.keys)[at + lane + 32 * i] : 0.0f;
            v[i] = on ? static_cast<const float *>(a.values)[at + lane + 32 * i] : 0.0f;
        }
#pragma unroll
        for (uint32_t h = 0; h < kFloatHeads; ++h) {
            x[h] = 0.0f;
#pragma unroll
            for (uint32_t i = 0; i < kFloatColumns; ++i) x[h] = fmaf(qv[h][i], k[i], x[h]);
        }
#pragma unroll
        for (int d = 16; d; d /= 2)
#pragma unroll
            for (uint32_t h = 0; h < kFloatHeads; ++h) x[h] += __shfl_xor_sync(kFullMask, x[h], d);
#pragma unroll
        for (uint32_t h = 0; h < kFloatHeads; ++h) {
            if (!(x[h] <= m[h])) {                            // a new maximum, or NaN, which stays
                const float top = max_nan(x[h], m[h]), keep = exp2f(m[h] - top);
                l[h] *= keep;
                m[h] = top;
#pragma unroll
                for (uint32_t i = 0; i < kFloatColumns; ++i) o[h][i] *= keep;
            }
            const float p = m[h] == -CUDART_INF_F ? 0.0f : exp2f(x[h] - m[h]);
            l[h] += p;
#pragma unroll
            for (uint32_t i = 0; i < kFloatColumns; ++i) o[h][i] = fmaf(p, v[i], o[h][i]);
        }
    }
#pragma unroll
    for (uint32_t h = 0; h < kFloatHeads; ++h) {
        if (h >= heads) break;
#pragma unroll
        for (uint32_t i = 0; i < kFloatColumns; ++i) values[warp][lane + 32 * i] = o[h][i];
        if (lane == 0) {
            ml[warp][0] = m[h];
            ml[warp][1] = l[h];
        }
        __syncthreads();
        float top = -CUDART_INF_F, sum = 0.0f, x = 0.0f;
        for (uint32_t w = 0; w < kWarps; ++w) top = max_nan(top, ml[w][0]);
        for (uint32_t w = 0; w < kWarps; ++w) {
            const float e = exp2f(ml[w][0] - (top == -CUDART_INF_F ? 0.0f : top));
            sum = fmaf(ml[w][1], e, sum);
            x = fmaf(values[w][threadIdx.x], e, x);
        }
        if (threadIdx.x < a.dim) static_cast<float *>(a.out)[row * a.out_row + (first + h) * a.out_head + threadIdx.x] = sum == 0.0f ? 0.0f : x / sum;
        if (a.lse && threadIdx.x == 0)
            a.lse[(size_t)row * a.n_heads + first + h] = sum == 0.0f ? -CUDART_INF_F : (top + log2f(sum)) * 0.69314718055994531f;
        __syncthreads();
    }
}

}  // namespace td
