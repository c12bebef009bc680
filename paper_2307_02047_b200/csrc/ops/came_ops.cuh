// Shared by the operators that stand around the optimizer step (gradient norm and clipping,
// embedding lookup and its gradient): error reporting, wide loads and stores, small reductions.
#pragma once
#include "../../../include/came_b200.h"

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>
#include <cfloat>
#include <cmath>

namespace came_ops {

// Text for came_last_error(NULL) on the calling thread; returns `s`.  Defined with the step's API.
came_status report(came_status s, const char* msg);
came_status report_cuda(cudaError_t e, const char* what);
// CAME_OK when `device` is the calling thread's current device.
came_status require_current_device(int32_t device);

inline bool aligned_to(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
inline size_t dtype_bytes(int32_t dt) { return dt == CAME_BF16 ? 2 : 4; }
// A factor that kernels take as fp32: neither infinite there nor, unless it is zero, zero.  (No NaN passes.)
inline bool holds_in_fp32(double x) { return x == 0.0 || (std::fabs(x) <= FLT_MAX && std::fabs(x) >= FLT_TRUE_MIN); }
inline bool known_dtype(int32_t dt) { return dt == CAME_F32 || dt == CAME_BF16; }

// Lets `kernel` use `bytes` of dynamic shared memory; the runtime is asked once per device.
template <typename K>
inline cudaError_t allow_smem(K kernel, size_t bytes, int32_t device, std::atomic<uint64_t>& done)
{
    const uint64_t bit = device < 64 ? 1ull << device : 0ull;
    if (done.load(std::memory_order_relaxed) & bit) return cudaSuccess;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes));
    if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x)
{
    return __float2bfloat16_rn(x);
}

__device__ __forceinline__ double warp_sum(double v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Orders this thread's writes before, and its reads after, a counter that other blocks see (the
// acquire-release fence; __threadfence is the sequentially consistent one, which takes longer).
__device__ __forceinline__ void publish() { asm volatile("fence.acq_rel.gpu;" ::: "memory"); }

// Programmatic dependent launch: let the next grid of the stream be scheduled / wait until the
// grids before this one have finished and their memory is visible.
__device__ __forceinline__ void release_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous_grid() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

}  // namespace came_ops
