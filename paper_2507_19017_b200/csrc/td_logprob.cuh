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
__device__ __forceinline__ int32_t target_of(const LogprobArgs &a, uint32_t t, bool report) {
    const int32_t y = a.targets[t];
    if (y >= 0 && (uint32_t)y >= a.vocab) {
        if (a.status && report) atomicOr(a.status, TD_ERR_OOB_INDEX);
        return -1;
    }
    return y;
}

// Sums over the scores seen so far, relative to a reference: S = sum 2^t and W = sum 2^t t.  How t comes from a
// score x (c = scale2) and when the reference moves depends on the pass:
//   quick: t = x c - ref, one packed multiply-add per two scores; ref is the rounded product of a score
//          and c, moved up when a score passes it by more than 2^kSlack, so that it seldom moves.  -inf is
//          raised to the type's kLow first (entropy only), which keeps 0 * t finite; the reference begins half
//          way down to it.
//   safe:  t = (x - ref) c, not below kFarBelow; ref is the running maximum, from the lowest finite float up.
// The quick pass is right unless the row's maximum times c is beyond 1e30, or within 1000 of kLow / 2 times c: rows
// masked by the lowest finite value, of infinities, at extreme temperatures.  Those go
// through the safe pass.
struct Running {
    float ref, s, w;
};
constexpr float kSlack = 4.0f;

// Moves the reference up; unit: what a difference of references is worth in t (1 quick, c safe).
__device__ __forceinline__ void lift(Running &r, float ref, float unit) {
    const float d = fmaxf((r.ref - ref) * unit, kFarBelow);
    const float f = exp2_approx(d);
    r.w = f * fmaf(d, r.s, r.w);
    r.s *= f;
    r.ref = ref;
}
__device__ __forceinline__ void join(Running &r, Running o, float unit) {
    const float ref = fmaxf(r.ref, o.ref);
    lift(r, ref, unit);
    lift(o, ref, unit);
    r.s += o.s;
    r.w += o.w;
}

// A thread's share of a pass: the reference, the sums as pairs, the maximum.
struct Share {
    float ref, top;
    f32x2 s, w;
    __device__ __forceinline__ Running total() const {
        float a, b, c, d;
        unpack2(s, a, b);
        unpack2(w, c, d);
        return Running{ref, a + b, c + d};
    }
    __device__ __forceinline__ void lift_to(float to, float unit) {
        Running r = total();
        lift(r, to, unit);
        ref = to;
        s = pack2(r.s, 0.0f);
        w = pack2(r.w, 0.0f);
    }
};

template <typename T, int U, bool kEntropy, bool kSafe>
__device__ __forceinline__ void take(Share &r, uint4 (&v)[U], float scale2) {
    if (kEntropy && !kSafe)
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = Elem<T>::raise(v[u]);
    const float cm = Elem<T>::vmax(v);
    r.top = fmaxf(r.top, cm);
    if (kSafe ? cm > r.ref : cm * scale2 > r.ref + kSlack) r.lift_to(kSafe ? cm : cm * scale2, kSafe ? scale2 : 1.0f);
    const f32x2 neg = pack2(-r.ref, -r.ref), sc = pack2(scale2, scale2);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int k = 0; k < Elem<T>::kVec / 2; ++k) {
            f32x2 t = kSafe ? mul2(add2(Elem<T>::pair(v[u], k), neg), sc) : fma2(Elem<T>::pair(v[u], k), sc, neg);
            float a, b;
            unpack2(t, a, b);
            if (kSafe) {
                a = max_nan(a, kFarBelow);
                b = max_nan(b, kFarBelow);
                t = pack2(a, b);
            }
            const f32x2 e = pack2(exp2_approx(a), exp2_approx(b));
            r.s = add2(r.s, e);
            if (kEntropy) r.w = fma2(e, t, r.w);
        }
}

constexpr int kLogprobUnroll = 4;

// One pass over the vectors [lo, hi) of a row, and for the row's first part over the ends that do not fill a
// vector (at most 2 (kVec - 1) elements).
template <typename T, bool kEntropy, bool kSafe, int kThreads>
__device__ __forceinline__ Share pass_over(const T *x, uint32_t vocab, uint32_t head, uint32_t nvec, uint32_t lo, uint32_t hi, bool ends, float scale2, uint32_t tid) {
    constexpr int E = Elem<T>::kVec, U = kLogprobUnroll;
    constexpr uint32_t kChunk = U * kThreads;
    const uint4 *xv = reinterpret_cast<const uint4 *>(x + head) + lo + tid;
    const uint32_t n = hi - lo, full = n / kChunk;
    Share r{kSafe ? -FLT_MAX : fmaxf(0.5f * Elem<T>::kLow * scale2, -FLT_MAX), -CUDART_INF_F, pack2(0.0f, 0.0f), pack2(0.0f, 0.0f)};
    uint4 p[U], q[U];
    auto fetch = [&](uint4 (&v)[U], uint32_t chunk) {
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = ld_stream(xv + (size_t)chunk * kChunk + u * kThreads);
    };
    // what is left behind the full chunks, filled up with -inf
    auto rest = [&](uint4 (&v)[U]) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            v[u].x = v[u].y = v[u].z = v[u].w = Elem<T>::kFill;
            if (full * kChunk + u * kThreads + tid < n) v[u] = ld_stream(xv + (size_t)full * kChunk + u * kThreads);
        }
    };
    if (full) fetch(p, 0); else rest(p);
    if (ends) {
        const uint32_t tail = head + nvec * E, n_loose = head + (vocab - tail);
        if (tid < n_loose) {
            float z = Elem<T>::load(x + (tid < head ? tid : tail + tid - head));
            if (!kSafe) z = max_nan(z, Elem<T>::kLow);
            r.top = z;
            r.ref = kSafe ? fmaxf(z, -FLT_MAX) : fmaxf(z * scale2, r.ref);
            const float t = max_nan(kSafe ? (z - r.ref) * scale2 : fmaf(z, scale2, -r.ref), kFarBelow), e = exp2_approx(t);
            r.s = pack2(e, 0.0f);
            r.w = pack2(e * t, 0.0f);
        }
    }
    uint32_t k = 0;
    while (k + 2 <= full) {              // two chunks a turn, each loaded while the other is added up
        fetch(q, k + 1);
        take<T, U, kEntropy, kSafe>(r, p, scale2);
        if (k + 2 < full) fetch(p, k + 2); else rest(p);
        take<T, U, kEntropy, kSafe>(r, q, scale2);
        k += 2;
    }
    if (k < full) {
        rest(q);
        take<T, U, kEntropy, kSafe>(r, p, scale2);
        if (n > full * kChunk) take<T, U, kEntropy, kSafe>(r, q, scale2);
    } else if (n > full * kChunk) take<T, U, kEntropy, kSafe>(r, p, scale2);
    return r;
}

// Bound by reading the logits once: 8192 rows of 152064 bfloat16 in 400 to 431 us, 5.8 to 6.2 TB/s (0.89 to 0.96 of
// a plain copy's rate), the spread being the clock under power limit, because next to the memory the exponential unit is
// 78 % busy (one exponential per score) at 5.7 instructions per score.
// One row per cluster of `parts` blocks (1 to 8); or, kThreads = 32, per warp, kWarpRows rows a block.  A single pass over the row: every thread keeps a reference and
// sums over its share, and the shares are joined in a fixed order over the warp, the block and (through
// distributed shared memory) the cluster.
constexpr int kWarpRows = 4;
template <typename T, bool kEntropy, int kThreads>
__global__ void __launch_bounds__(kThreads == 32 ? 32 * kWarpRows : kThreads, kThreads == 32 ? 32 / kWarpRows : 1024 / kThreads)
token_logprob_kernel(const LogprobArgs a) {
    griddep_launch_dependents();
    griddep_wait();
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    constexpr bool kWarpRow = kThreads == 32;
    const uint32_t parts = kWarpRow ? 1u : cluster.num_blocks(), part = kWarpRow ? 0u : cluster.block_rank();
    const uint32_t t = kWarpRow ? blockIdx.x * kWarpRows + threadIdx.x / 32 : blockIdx.x / parts, tid = kWarpRow ? threadIdx.x & 31u : threadIdx.x;
    if (kWarpRow && t >= a.n_tokens) return;
    struct Part { Running sums; float top; };
    __shared__ Part warp_part[kThreads / 32], block_part;
    __shared__ bool quick_holds;

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
    const int32_t y = target_of(a, t, tid == 0);
    if (!have_row || y < 0) {
        if (part == 0 && tid == 0) {
            a.logprob[t] = 0.0f;
            if (a.norm) { a.norm[2ull * t] = 0.0f; a.norm[2ull * t + 1] = 0.0f; }
            if (a.entropy) a.entropy[t] = 0.0f;
            if (a.entropy_bf16) a.entropy_bf16[t] = Elem<__nv_bfloat16>::from(0.0f);
        }
        return;
    }

    const T *x = static_cast<const T *>(a.logits) + row * a.stride;
    constexpr int E = Elem<T>::kVec;
    const uint32_t head = min((uint32_t)((16u - (reinterpret_cast<uintptr_t>(x) & 15u)) & 15u) / (uint32_t)sizeof(T), a.vocab);
    const uint32_t nvec = (a.vocab - head) / E;
    const uint32_t lo = (uint32_t)((unsigned long long)nvec * part / parts);
    const uint32_t hi = (uint32_t)((unsigned long long)nvec * (part + 1) / parts);
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    const float x_y = Elem<T>::load(x + y);

    // Joins the threads' shares; the first block's first thread has the row's sums and maximum.
    auto join_all = [&](const Share &mine, float unit) {
        Running r = mine.total();
        float top = mine.top;
        auto over_lanes = [&]() {
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                const Running other{__shfl_xor_sync(kFullMask, r.ref, o), __shfl_xor_sync(kFullMask, r.s, o), __shfl_xor_sync(kFullMask, r.w, o)};
                join(r, other, unit);
                top = fmaxf(top, __shfl_xor_sync(kFullMask, top, o));
            }
        };
        over_lanes();
        if constexpr (kWarpRow) return Part{r, top};         // the same in all lanes
        if (lane == 0) warp_part[warp] = Part{r, top};
        __syncthreads();
        if (warp == 0) {
            const Part p = warp_part[lane < kThreads / 32 ? lane : 0];
            r = p.sums;
            top = p.top;
            if (lane >= kThreads / 32) r.s = r.w = 0.0f;
            over_lanes();
            if (lane == 0) block_part = Part{r, top};
        }
        if (parts > 1) {
            cluster.sync();
            if (part == 0 && threadIdx.x == 0)
                for (uint32_t p = 1; p < parts; ++p) {
                    const Part o = *cluster.map_shared_rank(&block_part, p);
                    join(r, o.sums, unit);
                    top = fmaxf(top, o.top);
                }
        }
        return Part{r, top};
    };

    Part all = join_all(pass_over<T, kEntropy, false, kThreads>(x, a.vocab, head, nvec, lo, hi, part == 0, a.scale2, tid), 1.0f);
    bool quick = a.scale2 < 1e8f && fabsf(all.top) * a.scale2 < 1e30f && (all.top - 0.5f * Elem<T>::kLow) * a.scale2 > -kFarBelow;
    if constexpr (!kWarpRow) {           // the first block's first thread has the maximum and says; the others look
        if (part == 0 && threadIdx.x == 0) quick_holds = quick;
        if (parts > 1) {
            cluster.sync();
            quick = *cluster.map_shared_rank(&quick_holds, 0);
            cluster.sync();                                  // a block's shared memory stays until it has been read
        } else {
            __syncthreads();
            quick = quick_holds;
        }
    }
    if (!quick) {
        all = join_all(pass_over<T, kEntropy, true, kThreads>(x, a.vocab, head, nvec, lo, hi, part == 0, a.scale2, tid), a.scale2);
        if (parts > 1) cluster.sync();
    }
    if (part == 0 && tid == 0) {
        const Running r = all.sums;
        const bool none = r.s == 0.0f;                       // every logit -inf
        const float ln_s = none ? 0.0f : logf(r.s);
        const float h = none ? 0.0f : ln_s - kLn2 * (r.w / r.s);
        const float top = quick ? all.top : r.ref;
        const float ln_top = quick ? ln_s - fmaf(top, a.scale2, -r.ref) * kLn2 : ln_s;      // relative to the maximum
        a.logprob[t] = none ? -CUDART_INF_F : fmaf(x_y - top, a.inv_tau, -ln_top);
        if (a.norm) {
            a.norm[2ull * t] = none ? -CUDART_INF_F : top;
            a.norm[2ull * t + 1] = ln_top;
        }
        if (kEntropy) {
            if (a.entropy) a.entropy[t] = h;
            if (a.entropy_bf16) a.entropy_bf16[t] = Elem<__nv_bfloat16>::from(h);
        }
    }
}

constexpr int kGradThreads = 256, kGradUnroll = 4;
constexpr uint32_t kGradVectors = kGradThreads * kGradUnroll * 4;        // vectors of a row per block

// Elementwise over the rows: p = 2^d with d = (x - max) c - log2 S, gradient p (ca + cb d), and g / tau more at the target.
// Bound by memory: the stream of four 7B-shaped samples, 7774 rows of 152064 bfloat16 of which 5057 have a gradient and the
// others are only cleared (3.9 GB), in 605 us, 6.45 TB/s.  One block per (row, chunk of the row).  kSame: a row of
// logits and its gradient's start at the same offset from a 16-byte boundary; else the logits' vectors are put together from two loads each.  kTeam = 32: a row
// per warp.
template <typename T, bool kSame, int kTeam>
__global__ void __launch_bounds__(kGradThreads, kSame ? 4 : 3) token_logprob_grad_kernel(const LogprobArgs a) {
    griddep_launch_dependents();
    griddep_wait();
    constexpr bool kWarpRow = kTeam == 32;
    const uint32_t tid = kWarpRow ? threadIdx.x & 31u : threadIdx.x;
    const uint32_t chunk = kWarpRow ? 0u : blockIdx.x % a.chunks;
    const long long row = kWarpRow ? (long long)blockIdx.x * (kGradThreads / 32) + threadIdx.x / 32 : blockIdx.x / a.chunks;
    if (kWarpRow && row >= (long long)a.n_rows) return;
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
        y = target_of(a, (uint32_t)t, tid == 0 && chunk == 0);
        g = a.grad_logprob ? a.grad_logprob[t] : 0.0f;
        const float h = a.grad_entropy ? a.grad_entropy[t] : 0.0f;
        m = a.norm_in[2 * t];
        log2_s = a.norm_in[2 * t + 1] * (1.0f / kLn2);
        ca = -(g + (a.grad_entropy ? h * a.entropy_in[t] : 0.0f)) * a.inv_tau;
        cb = -h * kLn2 * a.inv_tau;
        if ((g == 0.0f && h == 0.0f) || m == -CUDART_INF_F) y = -1;
    }
    const bool zero = y < 0;
    // the row's vectors are aligned on the place it is written to
    const uint32_t head = min((16u - (uint32_t)(reinterpret_cast<uintptr_t>(out) & 15u)) % 16u / (uint32_t)sizeof(T), a.vocab);
    const uint32_t nvec = (a.vocab - head) / E;
    const uint32_t lo = chunk * kGradVectors, hi = kWarpRow ? nvec : min(nvec, lo + kGradVectors);
    const float gy = g * a.inv_tau;
    auto value = [&](float z, uint32_t v) {
        const float d = max_nan(fmaf(z - m, a.scale2, -log2_s), kFarBelow);
        return exp2_approx(d) * fmaf(cb, d, ca) + (v == (uint32_t)y ? gy : 0.0f);
    };
    if (chunk == 0) {                                        // the ends that do not fill a vector
        const uint32_t tail = head + nvec * E, n_loose = head + (a.vocab - tail);
        if (tid < n_loose) {
            const uint32_t v = tid < head ? tid : tail + tid - head;
            out[v] = Elem<T>::from(zero ? 0.0f : value(Elem<T>::load(x + v), v));
        }
    }
    uint4 *ov = reinterpret_cast<uint4 *>(out + head);
    if (zero) {
        const uint4 z = make_uint4(0u, 0u, 0u, 0u);
        for (uint32_t i = lo + tid; i < hi; i += kTeam) st_stream(ov + i, z);
        return;
    }
    const bool edge = row == 0 || row == (long long)a.n_rows - 1 || a.stride < (long long)a.vocab;      // rows may overlap
    const T *xh = x + head, *begin = static_cast<const T *>(a.logits), *end = begin + (long long)(a.n_rows - 1) * a.stride + a.vocab;
    const uint32_t y_vec = (uint32_t)y >= head ? ((uint32_t)y - head) / E : 0xffffffffu, y_in = ((uint32_t)y - head) % E;
    const f32x2 neg = pack2(-m, -m), sc = pack2(a.scale2, a.scale2), off = pack2(-log2_s, -log2_s), c0 = pack2(ca, ca), c1 = pack2(cb, cb);
    for (uint32_t i = lo + tid; i < hi; i += kTeam * U) {
        uint4 v[U];
        if constexpr (kSame) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u * kTeam < hi) v[u] = ld_stream(xh + (size_t)(i + u * kTeam) * E);
        } else {
            Window<T> w[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u * kTeam < hi) w[u].open(xh + (size_t)(i + u * kTeam) * E, begin, end, edge);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u * kTeam < hi) v[u] = w[u].close(xh + (size_t)(i + u * kTeam) * E);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t j = i + u * kTeam;
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
