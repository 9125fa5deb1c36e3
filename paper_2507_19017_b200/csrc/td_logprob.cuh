// Log-probability and entropy of tokens under rows of logits, and the gradient with respect to the
// logits.
#pragma once

#include <cooperative_groups.h>

#include "td_ops.cuh"

namespace td {

struct LogprobArgs {
    const void *logits;
    long long stride;                    // elements
    uint32_t vocab, n_rows, n_tokens;
    uint32_t stream_rows;                // rows are laid out as the fused stream
    float inv_tau, scale2;               // 1 / tau, log2(e) / tau
    BatchView batch;
    const int32_t *targets;
    uint32_t *status;
    // forward
    float *logprob, *norm, *entropy;
    __nv_bfloat16 *entropy_bf16;
    // gradient
    const float *norm_in, *entropy_in, *grad_logprob, *grad_entropy;
    void *grad;
    long long grad_stride;
    uint32_t chunks;                     // blocks per row
};

constexpr float kLn2 = 0.693147180559945309f;
constexpr float kFarBelow = -1000.0f;    // 2^-1000 is 0 in float: scores below it contribute nothing, and stay finite

// Target of token t, or -1; a target past the vocabulary is reported.
__device__ __forceinline__ int32_t target_of(const LogprobArgs &a, uint32_t t) {
    const int32_t y = __ldg(a.targets + t);
    if (y >= 0 && (uint32_t)y >= a.vocab) {
        if (a.status && threadIdx.x == 0) atomicOr(a.status, TD_ERR_OOB_INDEX);
        return -1;
    }
    return y;
}

// Running maximum m, S = sum 2^t and W = sum 2^t t with t = (x - m) * scale2, over the scores seen
// so far.  m starts at the lowest finite float, so that -inf scores give 2^-inf = 0 without a test.
struct Running {
    float m, s, w;
};

// Moves the reference from r.m up to m.
__device__ __forceinline__ void lift(Running &r, float m, float scale2) {
    const float d = fmaxf((r.m - m) * scale2, kFarBelow);
    const float f = exp2_approx(d);
    r.w = f * fmaf(d, r.s, r.w);
    r.s *= f;
    r.m = m;
}

__device__ __forceinline__ void join(Running &r, Running o, float scale2) {
    const float m = fmaxf(r.m, o.m);
    lift(r, m, scale2);
    lift(o, m, scale2);
    r.s += o.s;
    r.w += o.w;
}

template <typename T, int U, bool kEntropy>
__device__ __forceinline__ void take(Running &r, f32x2 &s2, f32x2 &w2, const uint4 (&v)[U], float scale2) {
    const float cm = Elem<T>::vmax(v);
    if (cm > r.m) {                                          // the pairs' sums hang on the old reference
        float a, b, c, d;
        unpack2(s2, a, b);
        unpack2(w2, c, d);
        r.s = a + b;
        r.w = c + d;
        lift(r, cm, scale2);
        s2 = pack2(r.s, 0.0f);
        w2 = pack2(r.w, 0.0f);
    }
    const f32x2 neg = pack2(-r.m, -r.m), sc = pack2(scale2, scale2);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int k = 0; k < Elem<T>::kVec / 2; ++k) {
            f32x2 t = mul2(add2(Elem<T>::pair(v[u], k), neg), sc);
            float a, b;
            unpack2(t, a, b);
            if (kEntropy) {
                a = max_nan(a, kFarBelow);
                b = max_nan(b, kFarBelow);
                t = pack2(a, b);
            }
            const f32x2 e = pack2(exp2_approx(a), exp2_approx(b));
            s2 = add2(s2, e);
            if (kEntropy) w2 = fma2(e, t, w2);
        }
}

constexpr int kLogprobThreads = 512, kLogprobUnroll = 4;

// One row per cluster of gridDim.x / n_tokens blocks (1 to 8).  A single pass: every thread keeps a
// running maximum and sums over its share of the row, and the shares are joined in a fixed order
// over the warp, the block and (through distributed shared memory) the cluster.
template <typename T, bool kEntropy>
__global__ void __launch_bounds__(kLogprobThreads, 2) token_logprob_kernel(const LogprobArgs a) {
    griddep_launch_dependents();
    griddep_wait();
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    const uint32_t parts = cluster.num_blocks(), part = cluster.block_rank();
    const uint32_t t = blockIdx.x / parts;
    __shared__ Running warp_part[kLogprobThreads / 32];
    __shared__ Running block_part;

    long long row = t;
    bool have_row = true;
    if (a.batch.cu_response) {
        const uint32_t n = batch_samples(a.batch);
        if (n == 0 || (long long)t >= (long long)a.batch.cu_response[n]) return;          // the whole cluster
        if (a.stream_rows) {
            const uint32_t i = sample_of(a.batch.cu_response, 0, n, t);
            const long long end_prompt = a.batch.cu_prompt[i + 1];
            row = end_prompt + t - 1;
            have_row = row >= (long long)a.batch.cu_prompt[i] + a.batch.cu_response[i] && row < (long long)a.n_rows;
        }
    }
    const int32_t y = target_of(a, t);
    if (!have_row || y < 0) {
        if (part == 0 && threadIdx.x == 0) {
            a.logprob[t] = 0.0f;
            if (a.norm) { a.norm[2ull * t] = 0.0f; a.norm[2ull * t + 1] = 0.0f; }
            if (a.entropy) a.entropy[t] = 0.0f;
            if (a.entropy_bf16) a.entropy_bf16[t] = Elem<__nv_bfloat16>::from(0.0f);
        }
        return;
    }

    const T *x = static_cast<const T *>(a.logits) + row * a.stride;
    constexpr int E = Elem<T>::kVec, U = kLogprobUnroll;
    const uint32_t head = min((uint32_t)((16u - (reinterpret_cast<uintptr_t>(x) & 15u)) & 15u) / (uint32_t)sizeof(T), a.vocab);
    const uint32_t nvec = (a.vocab - head) / E;
    const uint4 *xv = reinterpret_cast<const uint4 *>(x + head);
    const uint32_t lo = (uint32_t)((unsigned long long)nvec * part / parts);
    const uint32_t hi = (uint32_t)((unsigned long long)nvec * (part + 1) / parts);
    Running r{-FLT_MAX, 0.0f, 0.0f};
    f32x2 s2 = pack2(0.0f, 0.0f), w2 = pack2(0.0f, 0.0f);
    uint4 fill;
    fill.x = fill.y = fill.z = fill.w = Elem<T>::kFill;

    auto fetch = [&](uint4 (&v)[U], uint32_t i) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t j = i + u * kLogprobThreads;
            v[u] = j < hi ? ld_stream(xv + j) : fill;
        }
    };
    uint4 cur[U], nxt[U];
    uint32_t i = lo + threadIdx.x;
    fetch(cur, i);
    // the ends of the row that do not fill a vector: at most 2 * (E - 1) elements
    if (part == 0) {
        const uint32_t tail = head + nvec * E, n_loose = head + (a.vocab - tail);
        if (threadIdx.x < n_loose) {
            const float z = Elem<T>::load(x + (threadIdx.x < head ? threadIdx.x : tail + threadIdx.x - head));
            r.m = fmaxf(z, -FLT_MAX);
            const float d = max_nan((z - r.m) * a.scale2, kFarBelow);
            const float e = exp2_approx(d);
            s2 = pack2(e, 0.0f);
            w2 = pack2(e * d, 0.0f);
        }
    }
    while (i < hi) {
        const uint32_t ahead = i + U * kLogprobThreads;
        fetch(nxt, ahead);
        take<T, U, kEntropy>(r, s2, w2, cur, a.scale2);
#pragma unroll
        for (int u = 0; u < U; ++u) cur[u] = nxt[u];
        i = ahead;
    }
    {
        float p, q;
        unpack2(s2, p, q);
        r.s = p + q;
        unpack2(w2, p, q);
        r.w = p + q;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        Running other{__shfl_xor_sync(kFullMask, r.m, o), __shfl_xor_sync(kFullMask, r.s, o), __shfl_xor_sync(kFullMask, r.w, o)};
        join(r, other, a.scale2);
    }
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    if (lane == 0) warp_part[warp] = r;
    __syncthreads();
    if (warp == 0) {
        r = lane < kLogprobThreads / 32 ? warp_part[lane] : Running{-FLT_MAX, 0.0f, 0.0f};
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            Running other{__shfl_xor_sync(kFullMask, r.m, o), __shfl_xor_sync(kFullMask, r.s, o), __shfl_xor_sync(kFullMask, r.w, o)};
            join(r, other, a.scale2);
        }
        if (lane == 0) block_part = r;
    }
    if (parts > 1) {
        cluster.sync();
        if (part == 0 && threadIdx.x == 0)
            for (uint32_t p = 1; p < parts; ++p) join(r, *cluster.map_shared_rank(&block_part, p), a.scale2);
        cluster.sync();                                      // a block's shared memory stays until it has been read
    }
    if (part == 0 && threadIdx.x == 0) {
        const bool none = r.s == 0.0f;                       // every logit -inf
        const float ln_s = none ? 0.0f : logf(r.s);
        const float lp = none ? -CUDART_INF_F : fmaf(Elem<T>::load(x + y) - r.m, a.inv_tau, -ln_s);
        a.logprob[t] = lp;
        if (a.norm) {
            a.norm[2ull * t] = none ? -CUDART_INF_F : r.m;
            a.norm[2ull * t + 1] = ln_s;
        }
        if (kEntropy) {
            const float h = none ? 0.0f : ln_s - kLn2 * (r.w / r.s);
            if (a.entropy) a.entropy[t] = h;
            if (a.entropy_bf16) a.entropy_bf16[t] = Elem<__nv_bfloat16>::from(h);
        }
    }
}

constexpr int kGradThreads = 256, kGradUnroll = 4;
constexpr uint32_t kGradVectors = kGradThreads * kGradUnroll * 4;        // vectors of a row per block

// One block per (row, chunk of the row).
template <typename T>
__global__ void __launch_bounds__(kGradThreads, 4) token_logprob_grad_kernel(const LogprobArgs a) {
    griddep_launch_dependents();
    griddep_wait();
    const uint32_t chunk = blockIdx.x % a.chunks;
    const long long row = blockIdx.x / a.chunks;
    const T *x = static_cast<const T *>(a.logits) + row * a.stride;
    T *out = static_cast<T *>(a.grad) + row * a.grad_stride;
    constexpr int E = Elem<T>::kVec, U = kGradUnroll;

    // the row's token
    long long t = row < (long long)a.n_tokens ? row : -1;
    if (a.batch.cu_response) {
        const uint32_t n = batch_samples(a.batch);
        if (n == 0) t = -1;
        else if (!a.stream_rows) { if (row >= (long long)a.batch.cu_response[n]) t = -1; }
        else {
            // the sample whose stream row [cu_prompt + cu_response)[i] .. [i + 1] holds this row
            uint32_t lo = 0, hi = n;
            while (hi - lo > 1) {
                const uint32_t mid = lo + (hi - lo) / 2;
                if ((long long)a.batch.cu_prompt[mid] + a.batch.cu_response[mid] <= row) lo = mid; else hi = mid;
            }
            t = row + 1 - (long long)a.batch.cu_prompt[lo + 1];
            if (t < (long long)a.batch.cu_response[lo] || t >= (long long)a.batch.cu_response[lo + 1] || t >= (long long)a.n_tokens) t = -1;
        }
    }
    float ca = 0.0f, cb = 0.0f, g = 0.0f, m = 0.0f, log2_s = 0.0f;
    int32_t y = -1;
    if (t >= 0) {
        y = target_of(a, (uint32_t)t);
        g = a.grad_logprob ? a.grad_logprob[t] : 0.0f;
        const float h = a.grad_entropy ? a.grad_entropy[t] : 0.0f;
        m = a.norm_in[2 * t];
        log2_s = a.norm_in[2 * t + 1] * (1.0f / kLn2);
        ca = -(g + (a.grad_entropy ? h * a.entropy_in[t] : 0.0f)) * a.inv_tau;
        cb = -h * kLn2 * a.inv_tau;
        if ((g == 0.0f && h == 0.0f) || m == -CUDART_INF_F) y = -1;
    }
    const uint32_t phase_x = (uint32_t)(reinterpret_cast<uintptr_t>(x) & 15u), phase_o = (uint32_t)(reinterpret_cast<uintptr_t>(out) & 15u);
    const bool zero = y < 0;
    const bool wide = zero || phase_x == phase_o;
    // where the row's vectors start, by the place it is written to
    const uint32_t head = wide ? min(((16u - phase_o) & 15u) / (uint32_t)sizeof(T), a.vocab) : 0u;
    const uint32_t nvec = (a.vocab - head) / E;
    const uint32_t lo = chunk * kGradVectors, hi = min(nvec, lo + kGradVectors);
    const float gy = g * a.inv_tau;
    auto value = [&](float z, uint32_t v) {
        const float d = max_nan(fmaf(z - m, a.scale2, -log2_s), kFarBelow);
        return exp2_approx(d) * fmaf(cb, d, ca) + (v == (uint32_t)y ? gy : 0.0f);
    };
    if (chunk == 0) {                                        // the ends that do not fill a vector
        const uint32_t tail = head + nvec * E, n_loose = head + (a.vocab - tail);
        if (threadIdx.x < n_loose) {
            const uint32_t v = threadIdx.x < head ? threadIdx.x : tail + threadIdx.x - head;
            out[v] = Elem<T>::from(zero ? 0.0f : value(Elem<T>::load(x + v), v));
        }
    }
    uint4 *ov = reinterpret_cast<uint4 *>(out + head);
    if (zero) {
        const uint4 z = make_uint4(0u, 0u, 0u, 0u);
        for (uint32_t i = lo + threadIdx.x; i < hi; i += kGradThreads) st_stream(ov + i, z);
        return;
    }
    if (!wide) {                                             // logits and gradient rows at different phases: element by element
        const uint32_t end = min(nvec * E, hi * E);
        for (uint32_t v = lo * E + threadIdx.x; v < end; v += kGradThreads) out[v] = Elem<T>::from(value(Elem<T>::load(x + v), v));
        return;
    }
    const uint4 *xv = reinterpret_cast<const uint4 *>(x + head);
    const uint32_t y_vec = (uint32_t)y >= head ? ((uint32_t)y - head) / E : 0xffffffffu, y_in = ((uint32_t)y - head) % E;
    const f32x2 neg = pack2(-m, -m), sc = pack2(a.scale2, a.scale2), off = pack2(-log2_s, -log2_s), c0 = pack2(ca, ca), c1 = pack2(cb, cb);
    for (uint32_t i = lo + threadIdx.x; i < hi; i += kGradThreads * U) {
        uint4 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i + u * kGradThreads < hi) v[u] = ld_stream(xv + i + u * kGradThreads);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t j = i + u * kGradThreads;
            if (j >= hi) break;
            uint4 o;
#pragma unroll
            for (int k = 0; k < E / 2; ++k) {
                f32x2 d = fma2(add2(Elem<T>::pair(v[u], k), neg), sc, off);
                float p, q;
                unpack2(d, p, q);
                p = max_nan(p, kFarBelow);
                q = max_nan(q, kFarBelow);
                d = mul2(pack2(exp2_approx(p), exp2_approx(q)), fma2(c1, pack2(p, q), c0));
                unpack2(d, p, q);
                if (j == y_vec) {
                    if (y_in == 2u * k) p += gy;
                    if (y_in == 2u * k + 1u) q += gy;
                }
                Elem<T>::put_pair(o, k, p, q);
            }
            st_stream(ov + j, o);
        }
    }
}

}  // namespace td
