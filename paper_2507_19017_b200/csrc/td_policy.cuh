// Clipped policy loss with a KL term over the response tokens of a batch, and its gradient.
#pragma once

#include "td_ops.cuh"

namespace td {

constexpr float kLogRatioLimit = 30.0f;
constexpr int kPolicyThreads = 256;
constexpr uint32_t kPolicyMaxBlocks = 148 * 8;
constexpr int kPolicySums = 7;           // pg, kl, entropy (weighted); clipped, old kl, ratio, tokens

struct PolicyArgs {
    BatchView batch;
    unsigned long long n_tokens, row_width;      // row_width 0: packed
    uint32_t bf16_columns;
    int32_t kl_kind;
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
    griddep_launch_dependents();
    griddep_wait();
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
                const uint4 v = __ldg(mv + i);
                c += (__popc(__vcmpne4(v.x, 0u)) + __popc(__vcmpne4(v.y, 0u)) + __popc(__vcmpne4(v.z, 0u)) + __popc(__vcmpne4(v.w, 0u))) >> 3;
            }
            const long long tail = head + nvec * 16;
            if (lane < len - tail) c += m[tail + lane] != 0;
            c = __reduce_add_sync(kFullMask, c);
        }
    }
    if (lane == 0) a.counts[s] = c;
}

// a sum over the block's threads, in a fixed order, for thread 0
template <typename V>
__device__ __forceinline__ V block_sum(V x, V *scratch) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(kFullMask, x, o);
    __syncthreads();
    if ((threadIdx.x & 31u) == 0) scratch[threadIdx.x >> 5] = x;
    __syncthreads();
    V total = 0;
    if (threadIdx.x == 0)
        for (int w = 0; w < kPolicyThreads / 32; ++w) total += scratch[w];
    return total;
}

struct PolicyTerms {
    float pg, kl, d, ratio, raw;
    bool clipped;
};
__device__ __forceinline__ float limited(float x) {          // keeps a NaN
    return x < -kLogRatioLimit ? -kLogRatioLimit : x > kLogRatioLimit ? kLogRatioLimit : x;
}
__device__ __forceinline__ PolicyTerms policy_terms(const PolicyArgs &a, float lp, float old, float ref, float adv) {
    PolicyTerms r;
    r.raw = lp - old;
    const float lr = limited(r.raw);
    r.ratio = expf(lr);
    const float held_ratio = r.ratio < a.lo ? a.lo : r.ratio > a.hi ? a.hi : r.ratio;
    const float free = -adv * r.ratio, held = -adv * held_ratio;
    r.clipped = free < held;
    r.pg = r.clipped ? held : free;
    r.d = r.clipped || (lr != r.raw && r.raw == r.raw) ? 0.0f : free;      // a NaN reaches the gradient
    if (a.dual_clip > 0.0f && adv < 0.0f) {
        const float most = -adv * a.dual_clip;
        if (r.pg > most) { r.pg = most; r.d = 0.0f; r.clipped = true; }
    }
    r.kl = 0.0f;
    if (a.ref_logprob) {
        const float gap = ref - lp, k = limited(gap);
        float dk;
        if (a.kl_kind == TD_KL_K1) { r.kl = -k; dk = 1.0f; }
        else if (a.kl_kind == TD_KL_K2) { r.kl = 0.5f * k * k; dk = -k; }
        else { const float e = expm1f(k); r.kl = e - k; dk = -e; }
        if (k == gap || gap != gap) r.d = fmaf(a.kl_coef, dk, r.d);
    }
    return r;
}

// Positions p0 .. p0 + kVec of a per-token array; `whole`: all of them exist, and for kVec = 4 the
// array is aligned for one access.
template <int kVec>
__device__ __forceinline__ void load_floats(float (&o)[kVec], const float *c, long long p0, unsigned long long n, bool whole) {
    if (kVec == 4 && whole) {
        const float4 f = __ldcs(reinterpret_cast<const float4 *>(c + p0));
        o[0] = f.x; o[kVec > 1] = f.y; o[kVec > 1 ? 2 : 0] = f.z; o[kVec > 1 ? 3 : 0] = f.w;
    } else {
#pragma unroll
        for (int j = 0; j < kVec; ++j) o[j] = whole || p0 + j < (long long)n ? __ldcs(c + p0 + j) : 0.0f;
    }
}
template <int kVec>
__device__ __forceinline__ void load_column(float (&o)[kVec], const void *c, bool bf16, long long p0, unsigned long long n, bool whole) {
    if (!bf16) return load_floats<kVec>(o, static_cast<const float *>(c), p0, n, whole);
    const uint16_t *h = static_cast<const uint16_t *>(c);
    if (kVec == 4 && whole) {
        const uint2 u = __ldcs(reinterpret_cast<const uint2 *>(h + p0));
        o[0] = __uint_as_float(u.x << 16); o[kVec > 1] = __uint_as_float(u.x & 0xffff0000u);
        o[kVec > 1 ? 2 : 0] = __uint_as_float(u.y << 16); o[kVec > 1 ? 3 : 0] = __uint_as_float(u.y & 0xffff0000u);
    } else {
#pragma unroll
        for (int j = 0; j < kVec; ++j) o[j] = whole || p0 + j < (long long)n ? __uint_as_float((uint32_t)h[p0 + j] << 16) : 0.0f;
    }
}
template <int kVec>
__device__ __forceinline__ void load_mask(bool (&o)[kVec], const uint8_t *c, long long p0, unsigned long long n, bool whole) {
    if (kVec == 4 && whole) {
        const uint32_t m = __ldcs(reinterpret_cast<const uint32_t *>(c + p0));
#pragma unroll
        for (int j = 0; j < kVec; ++j) o[j] = ((m >> (8 * j)) & 255u) != 0;
    } else {
#pragma unroll
        for (int j = 0; j < kVec; ++j) o[j] = (whole || p0 + j < (long long)n) && c[p0 + j] != 0;
    }
}
template <int kVec>
__device__ __forceinline__ void store_floats(float *c, const float (&x)[kVec], long long p0, unsigned long long n, bool whole) {
    if (kVec == 4 && whole)
        __stcs(reinterpret_cast<float4 *>(c + p0), make_float4(x[0], x[kVec > 1], x[kVec > 1 ? 2 : 0], x[kVec > 1 ? 3 : 0]));
    else {
#pragma unroll
        for (int j = 0; j < kVec; ++j)
            if (whole || p0 + j < (long long)n) __stcs(c + p0 + j, x[j]);
    }
}

// kVec positions (4 or 1) per thread and turn, turn after turn over the block's share of the
// positions; the thread carries the sample it is in.
template <int kVec>
__global__ void __launch_bounds__(kPolicyThreads) policy_loss_kernel(const PolicyArgs a) {
    griddep_launch_dependents();
    griddep_wait();
    __shared__ double scratch[kPolicyThreads / 32];
    __shared__ long long whole_scratch[kPolicyThreads / 32];
    __shared__ long long total_s;
    __shared__ bool last;
    const uint32_t n = batch_samples(a.batch);

    // weight of a counted token, or its factor common to all samples
    float common;
    {
        if (a.mean_samples) common = a.norm > 0.0f ? 1.0f / a.norm : n ? 1.0f / (float)n : 0.0f;
        else if (a.norm > 0.0f) common = 1.0f / a.norm;
        else {
            long long c = 0;
            if (a.need_counts) {
                for (uint32_t s = threadIdx.x; s < n; s += kPolicyThreads) c += __ldg(a.counts + s);
                c = block_sum(c, whole_scratch);
                if (threadIdx.x == 0) total_s = c;
                __syncthreads();
                c = total_s;
                __syncthreads();
            } else {
                if (n) c = min((long long)a.batch.cu_response[n], (long long)a.n_tokens) - max(a.batch.cu_response[0], 0);
            }
            common = c > 0 ? 1.0f / (float)c : 0.0f;
        }
    }

    float pg = 0.0f, kl = 0.0f, ent = 0.0f, old_kl = 0.0f, ratio = 0.0f;
    uint32_t clipped = 0, counted = 0;
    const unsigned long long groups = (a.n_tokens + kVec - 1) / kVec;
    const unsigned long long share = (groups + gridDim.x - 1) / gridDim.x;
    const unsigned long long g0 = blockIdx.x * share, g1 = min(groups, g0 + share);
    uint32_t s = 0;
    Span span{0, 0, 0};
    float adv = 0.0f, w = 0.0f;
    bool seated = false;

    for (unsigned long long gi = g0 + threadIdx.x; gi < g1; gi += kPolicyThreads) {
        const long long p0 = (long long)(gi * kVec);
        float lp[kVec], old[kVec], ref[kVec], en[kVec], gl[kVec], ge[kVec];
        bool on[kVec];
        // all kVec positions with one access, unless the array ends among them
        const bool whole = kVec == 1 || p0 + kVec <= (long long)a.n_tokens;
        load_floats<kVec>(lp, a.logprob, p0, a.n_tokens, whole);
        if (a.old_logprob) load_column<kVec>(old, a.old_logprob, a.bf16_columns, p0, a.n_tokens, whole);
        if (a.ref_logprob) load_column<kVec>(ref, a.ref_logprob, a.bf16_columns, p0, a.n_tokens, whole);
        if (a.entropy) load_floats<kVec>(en, a.entropy, p0, a.n_tokens, whole);
        if (a.mask) load_mask<kVec>(on, a.mask, p0, a.n_tokens, whole);
#pragma unroll
        for (int j = 0; j < kVec; ++j) {
            const long long p = p0 + j;
            gl[j] = ge[j] = 0.0f;
            if (n && (!seated || p >= span.end)) {
                if (a.row_width) s = (uint32_t)min((long long)(p / (long long)a.row_width), (long long)n - 1);
                else {
                    // gallop from where the thread is: the next sample is usually near
                    uint32_t step = 1, lo = s;
                    while (lo + step < n && (long long)__ldg(a.batch.cu_response + lo + step) <= p) { lo += step; step <<= 1; }
                    s = sample_of(a.batch.cu_response, lo, min(n, lo + step), p);
                }
                seated = true;
                span = span_of(a, s);
                adv = __ldg(a.advantages + s);
                w = common;
                if (a.mean_samples) {
                    const int32_t c = a.need_counts ? __ldg(a.counts + s) : (int32_t)(span.valid_end - span.first);
                    w = c > 0 ? common / (float)c : 0.0f;
                }
            }
            if (!n || p < span.first || p >= span.valid_end || (a.mask && !on[j])) continue;
            const PolicyTerms r = policy_terms(a, lp[j], a.old_logprob ? old[j] : lp[j], a.ref_logprob ? ref[j] : 0.0f, adv);
            pg = fmaf(w, r.pg, pg);
            kl = fmaf(w, r.kl, kl);
            old_kl -= r.raw;
            ratio += r.ratio;
            clipped += r.clipped;
            ++counted;
            gl[j] = w * r.d * a.grad_scale;
            if (a.entropy) {
                ent = fmaf(w, en[j], ent);
                ge[j] = -a.entropy_coef * w * a.grad_scale;
            }
        }
        store_floats<kVec>(a.grad_logprob, gl, p0, a.n_tokens, whole);
        if (a.grad_entropy) store_floats<kVec>(a.grad_entropy, ge, p0, a.n_tokens, whole);
    }

    double sums[kPolicySums] = {pg, kl, ent, (double)clipped, old_kl, ratio, (double)counted};
#pragma unroll
    for (int k = 0; k < kPolicySums; ++k) sums[k] = block_sum(sums[k], scratch);
    if (threadIdx.x == 0) {
        for (int k = 0; k < kPolicySums; ++k) a.partials[(size_t)blockIdx.x * kPolicySums + k] = sums[k];
        __threadfence();
        last = atomicAdd(a.ticket, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    // the block that finishes last adds the partial sums in the order of the blocks
    for (int k = 0; k < kPolicySums; ++k) {
        double x = 0.0;
        for (uint32_t b = threadIdx.x; b < gridDim.x; b += kPolicyThreads) x += __ldcg(a.partials + (size_t)b * kPolicySums + k);
        sums[k] = block_sum(x, scratch);
    }
    if (threadIdx.x == 0) {
        const double each = sums[6] > 0.0 ? 1.0 / sums[6] : 0.0;
        a.stats[TD_POLICY_LOSS] = (float)(sums[0] + (double)a.kl_coef * sums[1] - (double)a.entropy_coef * sums[2]);
        a.stats[TD_POLICY_PG] = (float)sums[0];
        a.stats[TD_POLICY_KL] = (float)sums[1];
        a.stats[TD_POLICY_ENTROPY] = (float)sums[2];
        a.stats[TD_POLICY_CLIPPED] = (float)(sums[3] * each);
        a.stats[TD_POLICY_OLD_KL] = (float)(sums[4] * each);
        a.stats[TD_POLICY_RATIO] = (float)(sums[5] * each);
        a.stats[TD_POLICY_TOKENS] = (float)sums[6];
        *a.ticket = 0u;
    }
}

}  // namespace td
