// Attention of one new token per row over a paged cache.
#pragma once

#include "td_cache.cuh"

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
    float scale;
};

constexpr uint32_t kAttendThreads = 256;

// A warp per row and head; a token at a time.
template <typename T>
__global__ void __launch_bounds__(kAttendThreads) attend_kernel(CacheView c, AttendArgs a) {
    griddep_launch_dependents();
    griddep_wait();
    const uint32_t lane = threadIdx.x & 31u;
    const unsigned long long unit = (unsigned long long)blockIdx.x * (kAttendThreads / 32) + threadIdx.x / 32;
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
