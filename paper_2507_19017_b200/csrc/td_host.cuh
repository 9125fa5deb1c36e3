// What the host sides of the operators share: argument checks, the device a call belongs to, launches.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>
#include <utility>

#include "../../include/td.h"

namespace {

constexpr uint64_t kMaxGrid = 0x7fffffffull;
constexpr uint32_t kIndexLimit = 1u << 31;

inline size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
inline uint32_t size_of(int32_t dtype) { return dtype == TD_F32 ? 4u : 2u; }
inline bool float_type(int32_t dtype) { return dtype == TD_F32 || dtype == TD_BF16 || dtype == TD_F16; }
inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// The call's device made current, and the caller's put back.
class DeviceGuard {
public:
    explicit DeviceGuard(int device) {
        ok_ = cudaGetDevice(&before_) == cudaSuccess;
        if (ok_ && before_ != device) {
            ok_ = cudaSetDevice(device) == cudaSuccess;
            changed_ = ok_;
        }
    }
    ~DeviceGuard() { if (changed_) cudaSetDevice(before_); }
    DeviceGuard(const DeviceGuard &) = delete;
    DeviceGuard &operator=(const DeviceGuard &) = delete;
    bool ok() const { return ok_; }
private:
    int before_ = 0;
    bool ok_ = false, changed_ = false;
};

// Launch that may be brought on while the kernel ahead of it in the stream drains; every kernel here
// waits for that one before it touches memory.  cluster: blocks per cluster.
template <typename... KArgs, typename... Args>
cudaError_t launch_smem(void (*kernel)(KArgs...), uint64_t grid, uint32_t block, size_t smem, cudaStream_t st, uint32_t cluster,
                        Args &&...args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((uint32_t)grid);
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    cfg.attrs = attr;
#ifndef TD_NO_PDL
    attr[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[cfg.numAttrs++].val.programmaticStreamSerializationAllowed = 1;
#endif
    if (cluster > 1) {
        attr[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
        attr[cfg.numAttrs].val.clusterDim.x = cluster;
        attr[cfg.numAttrs].val.clusterDim.y = attr[cfg.numAttrs].val.clusterDim.z = 1;
        ++cfg.numAttrs;
    }
    return cudaLaunchKernelEx(&cfg, kernel, KArgs(std::forward<Args>(args))...);
}

template <typename... KArgs, typename... Args>
cudaError_t launch(void (*kernel)(KArgs...), uint64_t grid, uint32_t block, cudaStream_t st, uint32_t cluster, Args &&...args) {
    return launch_smem(kernel, grid, block, 0, st, cluster, std::forward<Args>(args)...);
}

}  // namespace
