// What the operators on a served batch share: the batch's row structure as kernels see it, element
// types, 16-byte vector access and packed float arithmetic.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <float.h>
#include <math_constants.h>
#include <stdint.h>

#include "../../include/td.h"
#include "td_common.cuh"

namespace td {

// A td_batch by value; cu_response == nullptr: no batch.
struct BatchView {
    const int32_t *cu_prompt, *cu_response;
    const td_result *result;
    uint32_t max_samples;
};

__device__ __forceinline__ uint32_t batch_samples(const BatchView &b) {
    return b.result ? min(b.result->n_samples, b.max_samples) : b.max_samples;
}

// Operands are read with ordinary loads, never through the read-only path (__ldg, ld.global.nc): that path is
// defined only for memory that nothing writes while the kernel runs, and a kernel here is let in while the one
// ahead of it, which may be what writes an operand, is still running.  Behind griddep_wait() an ordinary load
// has that kernel's results.

// The sample whose row [cu[s], cu[s + 1]) holds position t: the last s in [lo, n) with cu[s] <= t.
// Rows of length zero are passed over; for a cu array that is not non-decreasing the answer is some
// index of [lo, n).
__device__ __forceinline__ uint32_t sample_of(const int32_t *cu, uint32_t lo, uint32_t n, long long t) {
    uint32_t hi = n;
    while (hi - lo > 1) {
        const uint32_t mid = lo + (hi - lo) / 2;
        if ((long long)cu[mid] <= t) lo = mid; else hi = mid;
    }
    return lo;
}

// ---- packed pairs of floats (one instruction for two operations) ----
struct f32x2 { unsigned long long v; };
__device__ __forceinline__ f32x2 pack2(float a, float b) {
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpack2(f32x2 x, float &a, float &b) {
    asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x.v));
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}
__device__ __forceinline__ float exp2_approx(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// max(x, lo) and min(x, hi) that keep a NaN
__device__ __forceinline__ float min_nan(float x, float hi) {
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(hi));
    return r;
}
__device__ __forceinline__ float max_nan(float x, float lo) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(lo));
    return r;
}

// ---- element types ----
// Elem<T>::kVec elements make 16 bytes; pair k of a vector is elements 2k and 2k + 1.
template <typename T> struct Elem;

template <> struct Elem<float> {
    static constexpr int kVec = 4;
    static constexpr uint32_t kFill = 0xff800000u;           // -inf
    static __device__ __forceinline__ f32x2 pair(const uint4 &v, int k) {
        return k == 0 ? pack2(__uint_as_float(v.x), __uint_as_float(v.y)) : pack2(__uint_as_float(v.z), __uint_as_float(v.w));
    }
    static __device__ __forceinline__ float vmax(const uint4 &v) {
        return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
    }
    template <int U> static __device__ __forceinline__ float vmax(const uint4 (&v)[U]) {
        float m = vmax(v[0]);
#pragma unroll
        for (int u = 1; u < U; ++u) m = fmaxf(m, vmax(v[u]));
        return m;
    }
    // lowest score that is told from -inf where the two must not be confused, and the vector raised to it (a NaN stays)
    static constexpr float kLow = -1e30f;
    static __device__ __forceinline__ uint4 raise(const uint4 &v) {
        return make_uint4(__float_as_uint(max_nan(__uint_as_float(v.x), kLow)), __float_as_uint(max_nan(__uint_as_float(v.y), kLow)),
                          __float_as_uint(max_nan(__uint_as_float(v.z), kLow)), __float_as_uint(max_nan(__uint_as_float(v.w), kLow)));
    }
    static __device__ __forceinline__ void put_pair(uint4 &v, int k, float a, float b) {
        if (k == 0) { v.x = __float_as_uint(a); v.y = __float_as_uint(b); }
        else { v.z = __float_as_uint(a); v.w = __float_as_uint(b); }
    }
    static __device__ __forceinline__ float load(const float *p) { return *p; }
    static __device__ __forceinline__ float from(float x) { return x; }
};

__device__ __forceinline__ uint32_t word_of(const uint4 &v, int k) { return k == 0 ? v.x : k == 1 ? v.y : k == 2 ? v.z : v.w; }
__device__ __forceinline__ void set_word(uint4 &v, int k, uint32_t w) {
    if (k == 0) v.x = w; else if (k == 1) v.y = w; else if (k == 2) v.z = w; else v.w = w;
}

template <> struct Elem<__nv_bfloat16> {
    static constexpr int kVec = 8;
    static constexpr uint32_t kFill = 0xff80ff80u;
    static __device__ __forceinline__ __nv_bfloat162 h2(uint32_t w) { return *reinterpret_cast<const __nv_bfloat162 *>(&w); }
    static __device__ __forceinline__ f32x2 pair(const uint4 &v, int k) {
        const uint32_t w = word_of(v, k);                    // a bf16 is the upper half of a float
        return pack2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    }
    template <int U> static __device__ __forceinline__ float vmax(const uint4 (&v)[U]) {
        __nv_bfloat162 m = h2(v[0].x);
#pragma unroll
        for (int u = 0; u < U; ++u)
            m = __hmax2(__hmax2(m, __hmax2(h2(v[u].x), h2(v[u].y))), __hmax2(h2(v[u].z), h2(v[u].w)));
        return fmaxf(__low2float(m), __high2float(m));
    }
    static constexpr float kLow = -1e30f;
    static __device__ __forceinline__ uint32_t raise(uint32_t w) {
        const __nv_bfloat162 m = __hmax2_nan(h2(w), __float2bfloat162_rn(kLow));
        return *reinterpret_cast<const uint32_t *>(&m);
    }
    static __device__ __forceinline__ uint4 raise(const uint4 &v) { return make_uint4(raise(v.x), raise(v.y), raise(v.z), raise(v.w)); }
    static __device__ __forceinline__ void put_pair(uint4 &v, int k, float a, float b) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        set_word(v, k, *reinterpret_cast<const uint32_t *>(&h));
    }
    static __device__ __forceinline__ float load(const __nv_bfloat16 *p) { return __bfloat162float(*p); }
    static __device__ __forceinline__ __nv_bfloat16 from(float x) { return __float2bfloat16_rn(x); }
};

template <> struct Elem<__half> {
    static constexpr int kVec = 8;
    static constexpr uint32_t kFill = 0xfc00fc00u;
    static __device__ __forceinline__ __half2 h2(uint32_t w) { return *reinterpret_cast<const __half2 *>(&w); }
    static __device__ __forceinline__ f32x2 pair(const uint4 &v, int k) {
        const float2 f = __half22float2(h2(word_of(v, k)));
        return pack2(f.x, f.y);
    }
    template <int U> static __device__ __forceinline__ float vmax(const uint4 (&v)[U]) {
        __half2 m = h2(v[0].x);
#pragma unroll
        for (int u = 0; u < U; ++u)
            m = __hmax2(__hmax2(m, __hmax2(h2(v[u].x), h2(v[u].y))), __hmax2(h2(v[u].z), h2(v[u].w)));
        return fmaxf(__low2float(m), __high2float(m));
    }
    static constexpr float kLow = -65504.0f;
    static __device__ __forceinline__ uint32_t raise(uint32_t w) {
        const __half2 m = __hmax2_nan(h2(w), __float2half2_rn(kLow));
        return *reinterpret_cast<const uint32_t *>(&m);
    }
    static __device__ __forceinline__ uint4 raise(const uint4 &v) { return make_uint4(raise(v.x), raise(v.y), raise(v.z), raise(v.w)); }
    static __device__ __forceinline__ void put_pair(uint4 &v, int k, float a, float b) {
        const __half2 h = __floats2half2_rn(a, b);
        set_word(v, k, *reinterpret_cast<const uint32_t *>(&h));
    }
    static __device__ __forceinline__ float load(const __half *p) { return __half2float(*p); }
    static __device__ __forceinline__ __half from(float x) { return __float2half_rn(x); }
};

// 16 bytes that start `phase` bytes (even, below 16) into a and end in b.  A warp works on one row at a time and its lanes'
// places are 16 bytes apart, so phase is the same in all of them.
__device__ __forceinline__ uint4 shifted(const uint4 &a, const uint4 &b, uint32_t phase) {
    const uint32_t half = (phase & 2u) * 8u;
    uint32_t w0 = a.x, w1 = a.y, w2 = a.z, w3 = a.w, w4 = b.x;
    switch (phase >> 2) {
        case 1: w0 = a.y; w1 = a.z; w2 = a.w; w3 = b.x; w4 = b.y; break;
        case 2: w0 = a.z; w1 = a.w; w2 = b.x; w3 = b.y; w4 = b.z; break;
        case 3: w0 = a.w; w1 = b.x; w2 = b.y; w3 = b.z; w4 = b.w; break;
        default: break;
    }
    return make_uint4(__funnelshift_r(w0, w1, half), __funnelshift_r(w1, w2, half), __funnelshift_r(w2, w3, half), __funnelshift_r(w3, w4, half));
}
// kVec elements at p, whatever its alignment, put together from two aligned loads.  Those may reach up to 14 bytes over
// the ends of the elements' row, into the rows before and behind; `edge`: there may be none, so they are made only where
// they stay within [begin, end), the buffer, and elsewhere the elements are loaded one by one.  open() issues the loads
// and close() takes what they brought, so that several can be on their way.
template <typename T>
struct Window {
    uint4 a, b;
    bool whole;
    __device__ __forceinline__ void open(const T *p, const T *begin, const T *end, bool edge) {
        const uint32_t phase = (uint32_t)(reinterpret_cast<uintptr_t>(p) & 15u);
        const uint4 *at = reinterpret_cast<const uint4 *>(p - phase / sizeof(T));
        whole = true;
        if (edge) whole = p - phase / sizeof(T) >= begin && (phase == 0 || p - phase / sizeof(T) + 2 * Elem<T>::kVec <= end);
        a = b = make_uint4(0u, 0u, 0u, 0u);
        if (whole) a = at[0];
        if (whole && phase != 0) b = at[1];
    }
    __device__ __forceinline__ uint4 close(const T *p) const {
        if (whole) return shifted(a, b, (uint32_t)(reinterpret_cast<uintptr_t>(p) & 15u));
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int k = 0; k < Elem<T>::kVec / 2; ++k) Elem<T>::put_pair(v, k, Elem<T>::load(p + 2 * k), Elem<T>::load(p + 2 * k + 1));
        return v;
    }
};

// 16-byte accesses that data used once goes through: read past L1, written without being kept.
__device__ __forceinline__ uint4 ld_stream(const void *p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ void st_stream(void *p, const uint4 &v) {
    asm volatile("st.global.L1::no_allocate.v4.u32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// Asynchronous copy of kBytes (4, 8 or 16) from global to shared memory.  What a thread has copied it may read after
// copy_wait; others also need a barrier.
template <int kBytes>
__device__ __forceinline__ void copy_async(void *shared, const void *global) {
    const uint32_t to = (uint32_t)__cvta_generic_to_shared(shared);
    if constexpr (kBytes == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(global) : "memory");
    else
        asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(global), "n"(kBytes) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kPending>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kPending) : "memory"); }

}  // namespace td
