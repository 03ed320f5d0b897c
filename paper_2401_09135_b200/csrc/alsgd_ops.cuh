// Shared by the worker-side training operators (gradient clipping, attention): device selection for one call,
// dependent launches, element conversions.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>

namespace alsgd_ops {

constexpr int kSMs = 148;          // B200
constexpr int kMaxDevices = 64;

// Makes `device` current for the duration of one call.
struct UseDevice {
    int prev = -1;
    bool ok = false;
    explicit UseDevice(int device) : target(device) {
        if (cudaGetDevice(&prev) != cudaSuccess) return;
        ok = prev == device || cudaSetDevice(device) == cudaSuccess;
    }
    ~UseDevice() {
        if (ok && prev != target) cudaSetDevice(prev);
    }
    UseDevice(const UseDevice&) = delete;
    UseDevice& operator=(const UseDevice&) = delete;

private:
    int target;
};

// kernel<<<grid, block, smem, stream>>>(args...) whose blocks may be placed while the stream's previous kernel
// drains; the kernel itself waits (grid_dependency_sync) before its first access to memory that kernel may write.
template <typename... P, typename... A>
inline cudaError_t launch_dependent(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t s, const A&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// Raises a kernel's dynamic shared memory limit to what a block may have, once per device (the call costs more than a launch's
// other host work).  One table per kernel.  Threads that race on it set the same value: the runtime keeps the last one, so
// that a limit of each call's own size could end below what another has been told.
struct SmemLimit {
    static constexpr int kMost = 227 * 1024;
    std::atomic<bool> set[kMaxDevices] = {};
    template <typename K>
    bool raise(K kernel, int device, size_t bytes) {
        if (bytes > kMost) return false;
        if (set[device].load(std::memory_order_relaxed)) return true;
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost) != cudaSuccess) return false;
        set[device].store(true, std::memory_order_relaxed);
        return true;
    }
};

// Lets the next launch of the stream place its blocks, then waits until the previous one has completed and its
// writes are visible.  Does nothing in a launch without the attribute.
__device__ __forceinline__ void grid_dependency_sync() {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
}

// Division of 0 <= n < 2^31 by a divisor known at the launch: n * ceil(2^shift / d) >> shift with 2^(shift - 31) >= d, which
// is exact for those n.  A kernel's walk over its items divides in every warp.
struct Divide {
    uint32_t factor, shift;
    __device__ __forceinline__ int operator()(int n) const { return (int)((uint64_t)(uint32_t)n * factor >> shift); }
};

inline Divide divide_by(int d) {
    uint32_t shift = 31;
    while ((1ull << (shift - 31)) < (uint64_t)d) ++shift;
    return {(uint32_t)(((1ull << shift) + d - 1) / d), shift};
}

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// Two floats rounded to nearest even; `lo` lands in the low half.
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t w;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
    return w;
}

}  // namespace alsgd_ops
