// Clipped policy loss with a KL term over the response tokens of a batch, and its gradient.
#pragma once

#include "td_ops.cuh"

namespace td {

constexpr float kLogRatioLimit = 30.0f;
constexpr int kPolicyThreads = 256, kPolicyBlocksPerSm = 4;
constexpr uint32_t kPolicyMaxBlocks = 148 * kPolicyBlocksPerSm;
constexpr int kPolicySums = 7;           // pg, kl, entropy (weighted); clipped, old kl, ratio, tokens

struct PolicyArgs {
    BatchView batch;
    unsigned long long n_tokens, row_width;      // row_width 0: packed
    uint32_t bf16_columns;
    float kl_c1, kl_c2;                          // kKlPoly: kl = c1 k + c2 k^2
    uint32_t mean_samples;
    float lo, hi;                                // 1 - clip_low, 1 + clip_high
    float dual_clip, kl_coef, entropy_coef, norm, grad_scale;
    const float *logprob;
    const void *old_logprob, *ref_logprob;
    const float *entropy;
    const uint8_t *mask;
    const float *advantages;
    float *grad_logprob, *grad_entropy, *stats;
    double *partials;                            // [kPolicyMaxBlocks][kPolicySums]
    uint32_t *ticket;                            // 0 between calls
    int32_t *counts;                             // [max_samples] counted tokens per sample
    uint32_t need_counts;
};

// Positions of sample s: [first, first + room), of which the first `len` hold response tokens.
struct Span {
    long long first, valid_end, end;
};
__device__ __forceinline__ Span span_of(const PolicyArgs &a, uint32_t s) {
    const long long c0 = a.batch.cu_response[s], c1 = a.batch.cu_response[s + 1];
    Span p;
    if (a.row_width) {
        p.first = (long long)s * (long long)a.row_width;
        p.end = p.first + (long long)a.row_width;
        p.valid_end = p.first + min(max(c1 - c0, 0ll), (long long)a.row_width);
    } else {
        p.first = c0;
        p.end = c1;
        p.valid_end = c1;
    }
    p.valid_end = min(p.valid_end, (long long)a.n_tokens);
    return p;
}

// Counted tokens of every sample, a warp per sample.
__global__ void __launch_bounds__(kPolicyThreads) policy_count_kernel(const PolicyArgs a) {
    // the loss kernel is let in once everything ahead of this kernel is done: it may then read the
    // call's inputs before it waits for the counts
    griddep_wait();
    griddep_launch_dependents();
    const uint32_t s = blockIdx.x * (kPolicyThreads / 32) + (threadIdx.x >> 5), lane = threadIdx.x & 31u;
    if (s >= a.batch.max_samples) return;
    int32_t c = 0;
    if (s < batch_samples(a.batch)) {
        const Span p = span_of(a, s);
        const long long len = max(p.valid_end - max(p.first, 0ll), 0ll);
        if (!a.mask) c = (int32_t)len;
        else {
            const uint8_t *m = a.mask + max(p.first, 0ll);
            const long long head = min(len, (long long)((16u - (reinterpret_cast<uintptr_t>(m) & 15u)) & 15u));
            const long long nvec = (len - head) / 16;
            if (lane < head) c += m[lane] != 0;
            const uint4 *mv = reinterpret_cast<const uint4 *>(m + head);
#pragma unroll 4
            for (long long i = lane; i < nvec; i += 32) {
                const uint4 v = mv[i];
                c += (__popc(__vcmpne4(v.x, 0u)) + __popc(__vcmpne4(v.y, 0u)) + __popc(__vcmpne4(v.z, 0u)) + __popc(__vcmpne4(v.w, 0u))) >> 3;
            }
            const long long tail = head + nvec * 16;
            if (lane < len - tail) c += m[tail + lane] != 0;
            c = __reduce_add_sync(kFullMask, c);
        }
    }
    if (lane == 0) a.counts[s] = c;
}

constexpr float kLog2e = 1.44269504088896341f;

__device__ __forceinline__ f32x2 both(float x) { return pack2(x, x); }

// e^x - 1 and e^x - 1 - x of a pair.  Near 0 both come from the series (its terms beyond x^9 are below 2^-28 of the
// sum for |x| <= 1/2), so neither loses digits to the subtraction; further out from the exponential.
__device__ __forceinline__ void exp_minus_one(f32x2 x, f32x2 &e1, f32x2 &e2) {
    f32x2 q = both(1.0f / 362880.0f);
    q = fma2(q, x, both(1.0f / 40320.0f));
    q = fma2(q, x, both(1.0f / 5040.0f));
    q = fma2(q, x, both(1.0f / 720.0f));
    q = fma2(q, x, both(1.0f / 120.0f));
    q = fma2(q, x, both(1.0f / 24.0f));
    q = fma2(q, x, both(1.0f / 6.0f));
    q = fma2(q, x, both(0.5f));
    const f32x2 near2 = mul2(mul2(q, x), x), near1 = add2(x, near2);
    float t0, t1, x0, x1, n0, n1, m0, m1, f0, f1, g0, g1;
    unpack2(mul2(x, both(kLog2e)), t0, t1);
    const f32x2 far1 = add2(pack2(exp2_approx(t0), exp2_approx(t1)), both(-1.0f)), far2 = fma2(x, both(-1.0f), far1);
    unpack2(x, x0, x1);
    unpack2(near1, n0, n1);
    unpack2(near2, m0, m1);
    unpack2(far1, f0, f1);
    unpack2(far2, g0, g1);
    const bool a = fabsf(x0) <= 0.5f, b = fabsf(x1) <= 0.5f;
    e1 = pack2(a ? n0 : f0, b ? n1 : f1);
    e2 = pack2(a ? m0 : g0, b ? m1 : g1);
}

// How the KL term is computed: not at all, K3, or K1 and K2 as polynomials of the log ratio.
enum { kNoKl = 0, kKlExp = 1, kKlPoly = 2 };

// The sample a thread is in: where its response tokens are, and what they share.
struct Seat {
    int first, end, next;                // positions counted from the share's start; next: of the next sample
    float neg_adv, most, w;              // -A, the most that pg may be, the weight of a token
};

// What a thread adds up; pairs are added together at the end.
struct PolicySums {
    f32x2 pg, kl, raw, ratio;
    float ent;
    uint32_t clipped, counted;
};

// Two tokens with raw = logprob - old_logprob and gap = ref_logprob - logprob: adds their terms to the
// sums and returns d(loss) / d(logprob) without the weight.  kSelect: a token that is not `on` counts for
// nothing, whatever the inputs hold there.  min and max keep a NaN, so that one shows in the loss and the gradient.
template <int kKl, bool kSelect>
__device__ __forceinline__ f32x2 policy_pair(const PolicyArgs &a, const Seat &seat, bool on0, bool on1, f32x2 raw, f32x2 gap, PolicySums &sums) {
    auto limited = [](f32x2 x) {
        float p, q;
        unpack2(x, p, q);
        return pack2(min_nan(max_nan(p, -kLogRatioLimit), kLogRatioLimit), min_nan(max_nan(q, -kLogRatioLimit), kLogRatioLimit));
    };
    auto beyond = [](float x) { return fabsf(x) > kLogRatioLimit; };
    float r0, r1, t0, t1, f0, f1, h0, h1, d0, d1;
    unpack2(raw, r0, r1);
    unpack2(mul2(limited(raw), both(kLog2e)), t0, t1);
    const float q0 = exp2_approx(t0), q1 = exp2_approx(t1);
    f32x2 ratio = pack2(q0, q1);
    const f32x2 neg_adv = both(seat.neg_adv);
    unpack2(mul2(neg_adv, ratio), f0, f1);
    unpack2(mul2(neg_adv, pack2(min_nan(max_nan(q0, a.lo), a.hi), min_nan(max_nan(q1, a.lo), a.hi))), h0, h1);
    const float p0 = max_nan(f0, h0), p1 = max_nan(f1, h1);
    bool c0 = f0 < h0 || p0 > seat.most, c1 = f1 < h1 || p1 > seat.most;
    f32x2 pg = pack2(min_nan(p0, seat.most), min_nan(p1, seat.most));
    d0 = c0 || beyond(r0) ? 0.0f : f0;
    d1 = c1 || beyond(r1) ? 0.0f : f1;
    f32x2 kl = both(0.0f), d = pack2(d0, d1);
    if (kKl != kNoKl) {
        const f32x2 k = limited(gap);
        f32x2 dk;
        float g0, g1, v0, v1;
        if (kKl == kKlExp) exp_minus_one(k, dk, kl);
        else {
            kl = mul2(k, fma2(both(a.kl_c2), k, both(a.kl_c1)));
            dk = fma2(both(2.0f * a.kl_c2), k, both(a.kl_c1));
        }
        unpack2(gap, g0, g1);
        unpack2(fma2(both(-a.kl_coef), dk, d), v0, v1);      // gap falls as logprob rises
        d = pack2(beyond(g0) ? d0 : v0, beyond(g1) ? d1 : v1);
    }
    if (kSelect) {
        auto keep = [&](f32x2 x) {
            float p, q;
            unpack2(x, p, q);
            return pack2(on0 ? p : 0.0f, on1 ? q : 0.0f);
        };
        pg = keep(pg);
        if (kKl != kNoKl) kl = keep(kl);
        raw = keep(raw);
        ratio = keep(ratio);
        d = keep(d);
        c0 = c0 && on0;
        c1 = c1 && on1;
        sums.counted += (uint32_t)on0 + (uint32_t)on1;
    }
    const f32x2 w = both(seat.w);
    sums.pg = fma2(w, pg, sums.pg);
    if (kKl != kNoKl) sums.kl = fma2(w, kl, sums.kl);
    sums.raw = add2(sums.raw, raw);
    sums.ratio = add2(sums.ratio, ratio);
    sums.clipped += (uint32_t)c0 + (uint32_t)c1;
    return d;
}

// Positions rel .. rel + kVec of a per-token array that ends at `limit`; `whole`: all of them exist, and the
// array is aligned for one access of kVec.  A slot is the kVec elements' place in shared memory.
template <int kVec>
__device__ __forceinline__ void fetch_floats(float *slot, const float *c, int rel, int limit, bool whole) {
    if (whole) copy_async<4 * kVec>(slot, c + rel);
    else {
#pragma unroll
        for (int j = 0; j < kVec; ++j) slot[j] = rel + j < limit ? c[rel + j] : 0.0f;
    }
}
template <int kVec>
__device__ __forceinline__ void fetch_column(float *slot, const void *c, bool bf16, int rel, int limit, bool whole) {
    if (!bf16) return fetch_floats<kVec>(slot, static_cast<const float *>(c), rel, limit, whole);
    const uint16_t *h = static_cast<const uint16_t *>(c);
    uint16_t *to = reinterpret_cast<uint16_t *>(slot);
    if (kVec == 4 && whole) copy_async<8>(to, h + rel);
    else {
#pragma unroll
        for (int j = 0; j < kVec; ++j) to[j] = rel + j < limit ? h[rel + j] : (uint16_t)0;
    }
}
template <int kVec>
__device__ __forceinline__ void read_floats(float (&o)[kVec], const float *slot) {
    if constexpr (kVec == 4) {
        const float4 f = *reinterpret_cast<const float4 *>(slot);
        o[0] = f.x; o[1] = f.y; o[2] = f.z; o[3] = f.w;
    } else o[0] = *slot;
}
template <int kVec>
__device__ __forceinline__ void read_column(float (&o)[kVec], const float *slot, bool bf16) {
    if (!bf16) return read_floats<kVec>(o, slot);
    if constexpr (kVec == 4) {
        const uint2 u = *reinterpret_cast<const uint2 *>(slot);
        o[0] = __uint_as_float(u.x << 16); o[1] = __uint_as_float(u.x & 0xffff0000u);
        o[2] = __uint_as_float(u.y << 16); o[3] = __uint_as_float(u.y & 0xffff0000u);
    } else o[0] = __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t *>(slot) << 16);
}
template <int kVec>
__device__ __forceinline__ void store_floats(float *c, const float *x, int rel, int limit, bool whole) {
    if (kVec == 4 && whole)
        __stcs(reinterpret_cast<float4 *>(c + rel), make_float4(x[0], x[kVec > 1], x[kVec > 1 ? 2 : 0], x[kVec > 1 ? 3 : 0]));
    else {
#pragma unroll
        for (int j = 0; j < kVec; ++j)
            if (rel + j < limit) __stcs(c + rel + j, x[j]);
    }
}

// The per-token arrays from the share's start on, and what a thread has loaded of them.
struct PolicyArrays {
    const float *logprob, *entropy;
    const void *old_logprob, *ref_logprob;
    const uint8_t *mask;
    float *grad_logprob, *grad_entropy;
    int limit;                           // positions up to the arrays' end, or more than the share has
};
// What is on its way for a block: kStages turns of every array in use, each thread's elements in a slot of its own.
// Three, or two where three would leave no room for four blocks on an SM (the whole grid is resident at once).
template <int kVec, int kKl, bool kMask, bool kEnt>
struct PolicyStage {
    static constexpr int kArrays = 2 + (kKl != kNoKl) + kEnt;
    static constexpr size_t kBytes = (size_t)kPolicyThreads * (kArrays * kVec * 4 + (kMask ? 4 : 0));      // of one turn
    static constexpr int kStages = 3 * kBytes > 48 * 1024 ? 2 : 3;
    float *at;
    __device__ __forceinline__ PolicyStage(uint8_t *smem, int stage) : at(reinterpret_cast<float *>(smem + stage * kBytes)) {}
    __device__ __forceinline__ float *slot(int array) const { return at + ((size_t)array * kPolicyThreads + threadIdx.x) * kVec; }
    __device__ __forceinline__ uint8_t *mask_slot() const {
        return reinterpret_cast<uint8_t *>(at + (size_t)kArrays * kPolicyThreads * kVec) + 4 * threadIdx.x;
    }
    __device__ __forceinline__ void fetch(const PolicyArrays &p, bool bf16, int rel) const {
        const bool whole = rel + kVec <= p.limit;            // else the arrays end among the positions
        fetch_floats<kVec>(slot(0), p.logprob, rel, p.limit, whole);
        if (p.old_logprob) fetch_column<kVec>(slot(1), p.old_logprob, bf16, rel, p.limit, whole);
        if (kKl != kNoKl) fetch_column<kVec>(slot(2), p.ref_logprob, bf16, rel, p.limit, whole);
        if (kEnt) fetch_floats<kVec>(slot(kArrays - 1), p.entropy, rel, p.limit, whole);
        if (kMask) {
            if (kVec == 4 && whole) copy_async<4>(mask_slot(), p.mask + rel);
            else {
#pragma unroll
                for (int j = 0; j < kVec; ++j) mask_slot()[j] = rel + j < p.limit ? p.mask[rel + j] : (uint8_t)0;
            }
        }
    }
};

// Samples that a block keeps in shared memory, counted from the one its first position is in.
constexpr int kPolicyWindow = 256;
static_assert(kPolicyWindow == kPolicyThreads, "one thread fills one entry");

// 12 to 25 bytes and some 80 instructions per token.  75 million tokens of the R1-shaped batch: 246 us, 5.0 TB/s (0.77 of
// a plain copy's rate) at 73 % of the instruction issue slots; a separate path for small log ratios, more or fewer resident
// blocks and deeper staging measured the same or worse.  Small batches are latency: 8 samples 6.1 us, 64 masked ones
// 10.1 us with the counting kernel.
// A block's consecutive share of the positions, kVec (4 or 1) per thread and turn.  Positions are
// counted from the share's start; the next turn's loads are under way while a turn is worked on.
template <int kVec, int kKl, bool kMask, bool kEnt>
__global__ void __launch_bounds__(kPolicyThreads, kPolicyBlocksPerSm) policy_loss_kernel(const PolicyArgs a) {
    griddep_launch_dependents();
    if (!a.need_counts) griddep_wait();
    extern __shared__ __align__(16) uint8_t policy_smem[];
    __shared__ int win_first[kPolicyWindow], win_end[kPolicyWindow];        // of the sample's response tokens
    __shared__ float win_adv[kPolicyWindow], win_w[kPolicyWindow];
    __shared__ double warp_sums[kPolicyThreads / 32][kPolicySums];
    __shared__ long long warp_counts[kPolicyThreads / 32];
    __shared__ bool last;
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    const unsigned long long groups = (a.n_tokens + kVec - 1) / kVec;
    const unsigned long long share = (groups + gridDim.x - 1) / gridDim.x;
    const unsigned long long g0 = min(groups, blockIdx.x * share), g1 = min(groups, g0 + share);
    const long long base = (long long)(g0 * kVec);
    const int size = (int)((g1 - g0) * kVec);

    const size_t column_bytes = a.bf16_columns ? 2 : 4;
    auto column_at = [&](const void *c) { return c ? static_cast<const uint8_t *>(c) + (size_t)base * column_bytes : nullptr; };
    const PolicyArrays arr{a.logprob + base, kEnt ? a.entropy + base : nullptr, column_at(a.old_logprob), column_at(a.ref_logprob),
                           kMask ? a.mask + base : nullptr, a.grad_logprob + base, a.grad_entropy ? a.grad_entropy + base : nullptr,
                           (int)min((long long)a.n_tokens - base, (long long)size)};

    using Stage = PolicyStage<kVec, kKl, kMask, kEnt>;
    constexpr int kTurn = kPolicyThreads * kVec;
    int rel = (int)threadIdx.x * kVec;
#pragma unroll
    for (int k = 0; k < Stage::kStages; ++k) {
        if (rel + k * kTurn < size) Stage(policy_smem, k).fetch(arr, a.bf16_columns, rel + k * kTurn);
        copy_commit();
    }

    const uint32_t n = batch_samples(a.batch);
    // the sample of the share's first position: all threads look at once, in rounds of 256 entries
    // (a batch that fits the window needs no search)
    uint32_t s0 = 0;
    if (n > kPolicyWindow && a.row_width) s0 = (uint32_t)min(base / (long long)a.row_width, (long long)n - 1);
    else if (n > kPolicyWindow) {
        uint32_t lo = 0, hi = n;                             // cu[lo] <= base, and cu[hi] > base or hi = n
        while (hi - lo > 1) {
            const uint32_t step = (hi - lo + kPolicyThreads - 1) / kPolicyThreads;
            const uint64_t at = lo + (uint64_t)(threadIdx.x + 1) * step;
            const int below = __syncthreads_count(at < hi && (long long)a.batch.cu_response[at] <= base);
            lo += (uint32_t)below * step;
            hi = min(hi, lo + step);
        }
        s0 = lo;
    }
    if (a.need_counts) griddep_wait();
    // weight of a counted token, or its factor common to all samples
    float common;
    if (a.mean_samples) common = a.norm > 0.0f ? 1.0f / a.norm : n ? 1.0f / (float)n : 0.0f;
    else if (a.norm > 0.0f) common = 1.0f / a.norm;
    else {
        long long c = 0;
        if (a.need_counts) {
            for (uint32_t s = threadIdx.x; s < n; s += kPolicyThreads) c += a.counts[s];
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) c += __shfl_xor_sync(kFullMask, c, o);
            if (lane == 0) warp_counts[warp] = c;
            __syncthreads();
            c = 0;
            for (int w = 0; w < kPolicyThreads / 32; ++w) c += warp_counts[w];
        } else if (n) {
            c = min((long long)a.batch.cu_response[n], (long long)a.n_tokens) - max(a.batch.cu_response[0], 0);
        }
        common = c > 0 ? 1.0f / (float)c : 0.0f;
    }
    auto weight = [&](uint32_t s, const Span &p) {
        if (!a.mean_samples) return common;
        // (with a load that passes by L1, ld.global.cg, the kernel took 8 us more whether or not it has counts)
        const int32_t c = a.need_counts ? a.counts[s] : (int32_t)(p.valid_end - p.first);
        return c > 0 ? common / (float)c : 0.0f;
    };
    auto from_base = [&](long long p) { return (int)max(-1ll, min(p - base, (long long)size)); };
    if (s0 + threadIdx.x < n) {
        const uint32_t s = s0 + threadIdx.x;
        const Span p = span_of(a, s);
        win_first[threadIdx.x] = from_base(p.first);
        win_end[threadIdx.x] = from_base(p.valid_end);
        win_adv[threadIdx.x] = a.advantages[s];
        win_w[threadIdx.x] = weight(s, p);
    }
    __syncthreads();

    PolicySums sum{both(0.0f), both(0.0f), both(0.0f), both(0.0f), 0.0f, 0u, 0u};
    const uint32_t in_window = min(n - s0, (uint32_t)kPolicyWindow);       // n = 0: none
    uint32_t at = 0;                     // the sample this thread is in, counted from s0
    Seat seat{0, 0, n ? -1 : size, 0.0f, 0.0f, 0.0f};
    auto move = [&](int q) {             // to the sample that holds position q
        const uint32_t left = n - s0;
        auto starts = [&](uint32_t i) {
            if (i < in_window) return win_first[i];
            return a.row_width ? from_base((long long)(s0 + i) * (long long)a.row_width) : from_base(a.batch.cu_response[s0 + i]);
        };
        uint32_t lo = at, step = 1;      // gallop: the next sample is usually near
        while (lo + step < left && starts(lo + step) <= q) { lo += step; step <<= 1; }
        uint32_t hi = min(left, lo + step);
        while (hi - lo > 1) {
            const uint32_t mid = lo + (hi - lo) / 2;
            if (starts(mid) <= q) lo = mid; else hi = mid;
        }
        at = lo;
        seat.next = lo + 1 < left ? starts(lo + 1) : size;
        float adv;
        if (lo < in_window) {
            seat.first = win_first[lo];
            seat.end = win_end[lo];
            adv = win_adv[lo];
            seat.w = win_w[lo];
        } else {
            const Span p = span_of(a, s0 + lo);
            seat.first = from_base(p.first);
            seat.end = from_base(p.valid_end);
            adv = a.advantages[s0 + lo];
            seat.w = weight(s0 + lo, p);
        }
        seat.neg_adv = -adv;
        seat.most = adv < 0.0f ? -adv * a.dual_clip : CUDART_INF_F;         // dual_clip = inf: no limit
    };

    for (int k = 0; rel < size; k = k + 1 == Stage::kStages ? 0 : k + 1) {
        // kPairs pairs of positions; a single position goes as a pair whose second is off
        constexpr int kPairs = (kVec + 1) / 2;
        f32x2 raw[kPairs], gap[kPairs];
        float en[kVec], gl[2 * kPairs], ge[2 * kPairs];
        uint32_t on = 0xffffffffu;
        copy_wait<Stage::kStages - 1>();
        {
            const Stage stage(policy_smem, k);
            float lp[kVec], old[kVec], ref[kVec];
            read_floats<kVec>(lp, stage.slot(0));
            if (arr.old_logprob) read_column<kVec>(old, stage.slot(1), a.bf16_columns);
            if (kKl != kNoKl) read_column<kVec>(ref, stage.slot(2), a.bf16_columns);
            if (kEnt) read_floats<kVec>(en, stage.slot(Stage::kArrays - 1));
            if (kMask) on = kVec == 4 ? *reinterpret_cast<const uint32_t *>(stage.mask_slot()) : *stage.mask_slot();
#pragma unroll
            for (int j = 0; j < kPairs; ++j) {
                const int x = 2 * j, y = kVec > 1 ? 2 * j + 1 : 0;
                raw[j] = arr.old_logprob ? pack2(lp[x] - old[x], lp[y] - old[y]) : both(0.0f);
                gap[j] = kKl != kNoKl ? pack2(ref[x] - lp[x], ref[y] - lp[y]) : both(0.0f);
            }
            const int ahead = rel + Stage::kStages * kTurn;
            if (ahead < size) stage.fetch(arr, a.bf16_columns, ahead);
            copy_commit();
        }
        if (rel >= seat.next) move(rel);
        if (kVec > 1 && rel >= seat.first && rel + kVec <= seat.end) {      // one sample's tokens, as nearly always
            const float scale = seat.w * a.grad_scale, e = -a.entropy_coef * scale;
            if (!kMask) sum.counted += kVec;
#pragma unroll
            for (int j = 0; j < kPairs; ++j) {
                const bool on0 = (on & (255u << (16 * j))) != 0, on1 = (on & (65280u << (16 * j))) != 0;
                const f32x2 d = mul2(both(scale), policy_pair<kKl, kMask>(a, seat, on0, on1, raw[j], gap[j], sum));
                unpack2(d, gl[2 * j], gl[2 * j + 1]);
                ge[2 * j] = kEnt && (!kMask || on0) ? e : 0.0f;
                ge[2 * j + 1] = kEnt && (!kMask || on1) ? e : 0.0f;
                if (kEnt && (!kMask || on0)) sum.ent = fmaf(seat.w, en[2 * j], sum.ent);
                if (kEnt && (!kMask || on1)) sum.ent = fmaf(seat.w, en[2 * j + (kVec > 1)], sum.ent);
            }
        } else {
            // a sample begins or ends here: one position after the other
#pragma unroll 1
            for (int j = 0; j < kVec; ++j) {
                const int q = rel + j;
                if (q >= seat.next && q < size) move(q);
                // positions 2i and 2i + 1 share a pair: the one at j is on
                f32x2 pr = raw[0], pk = gap[0];
                float pe = en[0];
#pragma unroll
                for (int i = 1; i < kPairs; ++i)
                    if (j >> 1 == i) { pr = raw[i]; pk = gap[i]; }
#pragma unroll
                for (int i = 1; i < kVec; ++i)
                    if (j == i) pe = en[i];
                const bool in = q >= seat.first && q < seat.end && (!kMask || ((on >> (8 * j)) & 255u) != 0);
                const float scale = seat.w * a.grad_scale;
                float x, y;
                unpack2(mul2(both(scale), policy_pair<kKl, true>(a, seat, in && !(j & 1), in && (j & 1), pr, pk, sum)), x, y);
                const float g = in ? ((j & 1) ? y : x) : 0.0f, e = kEnt && in ? -a.entropy_coef * scale : 0.0f;
                if (kEnt && in) sum.ent = fmaf(seat.w, pe, sum.ent);
#pragma unroll
                for (int i = 0; i < kVec; ++i)
                    if (j == i) { gl[i] = g; ge[i] = e; }
            }
        }
        const bool whole = rel + kVec <= arr.limit;
        store_floats<kVec>(arr.grad_logprob, gl, rel, arr.limit, whole);
        if (a.grad_entropy) store_floats<kVec>(arr.grad_entropy, ge, rel, arr.limit, whole);
        rel += kTurn;
    }

    // sums of the threads, the warps and the blocks, each in a fixed order
    {
        auto total = [](f32x2 x) {
            float p, q;
            unpack2(x, p, q);
            return (double)p + (double)q;
        };
        double sums[kPolicySums] = {total(sum.pg), total(sum.kl), sum.ent, (double)sum.clipped, -total(sum.raw), total(sum.ratio), (double)sum.counted};
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
#pragma unroll
            for (int k = 0; k < kPolicySums; ++k) sums[k] += __shfl_xor_sync(kFullMask, sums[k], o);
        if (lane == 0)
#pragma unroll
            for (int k = 0; k < kPolicySums; ++k) warp_sums[warp][k] = sums[k];
    }
    __syncthreads();
    if (threadIdx.x < kPolicySums) {
        double x = 0.0;
        for (int v = 0; v < kPolicyThreads / 32; ++v) x += warp_sums[v][threadIdx.x];
        if (gridDim.x > 1) {
            a.partials[(size_t)threadIdx.x * kPolicyMaxBlocks + blockIdx.x] = x;
            __threadfence();
        }
        warp_sums[0][threadIdx.x] = x;
    }
    __syncthreads();
    if (gridDim.x > 1) {
        // the block that finishes last adds the blocks' sums
        if (threadIdx.x == 0) last = atomicAdd(a.ticket, 1u) == gridDim.x - 1;
        __syncthreads();
        if (!last) return;
        __threadfence();
        if (warp < kPolicySums) {
            double x = 0.0;
            for (uint32_t b = lane; b < gridDim.x; b += 32) x += __ldcg(a.partials + (size_t)warp * kPolicyMaxBlocks + b);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(kFullMask, x, o);
            if (lane == 0) warp_sums[0][warp] = x;
        }
        __syncthreads();
        if (threadIdx.x == 0) *a.ticket = 0u;
    }
    if (threadIdx.x == 0) {
        const double *sums = warp_sums[0];
        const double each = sums[6] > 0.0 ? 1.0 / sums[6] : 0.0;
        a.stats[TD_POLICY_LOSS] = (float)(sums[0] + (double)a.kl_coef * sums[1] - (double)a.entropy_coef * sums[2]);
        a.stats[TD_POLICY_PG] = (float)sums[0];
        a.stats[TD_POLICY_KL] = (float)sums[1];
        a.stats[TD_POLICY_ENTROPY] = (float)sums[2];
        a.stats[TD_POLICY_CLIPPED] = (float)(sums[3] * each);
        a.stats[TD_POLICY_OLD_KL] = (float)(sums[4] * each);
        a.stats[TD_POLICY_RATIO] = (float)(sums[5] * each);
        a.stats[TD_POLICY_TOKENS] = (float)sums[6];
    }
}

}  // namespace td
