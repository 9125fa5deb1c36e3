// What every kernel of the library uses.
#pragma once

#include <stdint.h>

namespace td {

constexpr uint32_t kFullMask = 0xffffffffu;

// Division by a run-time constant d through a multiply and a shift, exact for n < 2^31:
// n / d = (umulhi(n, mul) + n) >> shr with shr = ceil(log2 d), mul = floor(2^32 (2^shr - d) / d) + 1
// (mul = 0 when d is a power of two).
struct FastDiv {
    uint32_t mul, shr;
};
static inline FastDiv make_fastdiv(uint32_t d) {
    uint32_t l = 0;
    while ((1ull << l) < d) ++l;
    const uint64_t m = (1ull << l) == d ? 0 : ((1ull << 32) * ((1ull << l) - d)) / d + 1;
    return FastDiv{(uint32_t)m, l};
}
__device__ __forceinline__ FastDiv make_fastdiv_dev(uint32_t d) {          // the same constants, computed on the device
    const uint32_t l = d > 1u ? 32u - (uint32_t)__clz(d - 1u) : 0u;
    const unsigned long long m = (1ull << l) == d ? 0ull : ((1ull << 32) * ((1ull << l) - d)) / d + 1ull;
    return FastDiv{(uint32_t)m, l};
}
__device__ __forceinline__ uint32_t fast_div(uint32_t n, FastDiv f) {
    return (__umulhi(n, f.mul) + n) >> f.shr;
}

// Programmatic dependent launch: the kernels of one call are chained so that the next one is
// launched, and runs its prologue, while the previous one is still finishing.  A kernel calls
// griddep_wait() before it touches anything the kernel before it in the stream wrote (the wait
// returns when that kernel has completed and its writes are visible; without the launch
// attribute it returns at once), and griddep_launch_dependents() as soon as the next kernel
// may be brought on.
__device__ __forceinline__ void griddep_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void griddep_launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

}  // namespace td
