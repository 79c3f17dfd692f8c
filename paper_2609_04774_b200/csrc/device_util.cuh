// Small device and host helpers of the serving operators (decode attention, rotary append, page care).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "internal.h"

namespace cpattn {

// Makes `device` current for the lifetime of the object and the caller's device current again afterwards.
class DeviceGuard {
public:
    explicit DeviceGuard(int device) {
        rc_ = check_cuda(cudaGetDevice(&before_), "cudaGetDevice");
        if (rc_ == CP_OK && before_ != device) {
            rc_ = check_cuda(cudaSetDevice(device), "cudaSetDevice");
            restore_ = rc_ == CP_OK;
        }
    }
    ~DeviceGuard() {
        if (restore_) cudaSetDevice(before_);
    }
    DeviceGuard(const DeviceGuard&) = delete;
    DeviceGuard& operator=(const DeviceGuard&) = delete;
    int rc() const { return rc_; }

private:
    int before_ = 0, rc_ = CP_OK;
    bool restore_ = false;
};

// True when [a, a + na) and [b, b + nb) share a byte.
inline bool ranges_overlap(const void* a, size_t na, const void* b, size_t nb) {
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return x < y + nb && y < x + na;
}

inline int log2_exact(int v) {      // v is a power of two
    int s = 0;
    while ((1 << s) < v) ++s;
    return s;
}

#ifdef __CUDACC__
// Two launches of one call, the second reading what the first writes: the first lets the second be set up while it runs
// (let_next_launch_begin), the second waits for the first one's end (wait_for_launch_before) before it reads anything.
__device__ __forceinline__ void let_next_launch_begin() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_launch_before() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
template <typename... Params, typename... Args>
int launch_behind(void (*kernel)(Params...), dim3 grid, int threads, cudaStream_t s, const char* who, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return check_cuda(cudaLaunchKernelEx(&cfg, kernel, args...), who);
}

// The first error of a launch sequence lands in the context's status words {code, index, block, value}.
__device__ __forceinline__ void report_status(int32_t* status, int32_t code, int64_t index, int64_t value) {
    if (atomicCAS(status, 0, code) == 0) {
        status[1] = (int32_t)index;
        status[2] = (int32_t)blockIdx.x;
        status[3] = (int32_t)value;
    }
}
#endif

}  // namespace cpattn
