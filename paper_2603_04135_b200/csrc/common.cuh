// Shared host/device helpers of libdppo (not part of the ABI).
#pragma once
#include <cuda_runtime.h>
#include <cuda_bf16.h>
#include <stdint.h>
#include <stdarg.h>
#include <stdio.h>

#include <nvtx3/nvToolsExt.h>

#include "dppo.h"

namespace dppo {

// ---- host: thread-local error message ------------------------------------------------------------
int fail(int code, const char* fmt, ...);          // records the message, returns code
int cuda_fail(cudaError_t e, const char* what);    // DPPO_ERR_CUDA with the CUDA error string
int sm_count();                                    // SMs of the current device (cached per device)

#define DPPO_CHECK_LAUNCH(what)                                        \
    do {                                                               \
        cudaError_t e__ = cudaGetLastError();                          \
        if (e__ != cudaSuccess) return ::dppo::cuda_fail(e__, what);   \
    } while (0)

// ---- host: a named NVTX range around each entry point's host work (its launches show under it in a timeline
// tool; a few nanoseconds when no tool is attached)
struct NvtxRange {
    explicit NvtxRange(const char* name) { nvtxRangePushA(name); }
    ~NvtxRange() { nvtxRangePop(); }
    NvtxRange(const NvtxRange&) = delete;
    NvtxRange& operator=(const NvtxRange&) = delete;
};

// ---- kernels that overlap their start with the end of the kernel before them -----------------------
// A kernel launched by launch_after may be set up while the kernel before it in the stream still runs, once every CTA of that
// one has called let_next_start() or has ended (a kernel that never calls it is followed as usual, after its end).
// wait_for_previous() comes before every access to global memory, in every thread: it waits until everything before this
// kernel has completed and its writes can be seen.  Back to back, a call of a few microseconds otherwise loses about two
// of them to its launch.  let_next_start() belongs at the start of a kernel, except where the next one's CTAs would then take
// up places unevenly beside a grid that fills the SMs once (a row per cluster: 300 rows 42 us instead of 31): at its end.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void enter_kernel() {
    let_next_start();
    wait_for_previous();
}
// cluster: CTAs per cluster (1: none).
template <class... P, class... A>
inline int launch_after(const char* what, void (*kernel)(P...), long long grid, int block, size_t smem, cudaStream_t s, int cluster,
                        const A&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid, 1, 1);
    cfg.blockDim = dim3((unsigned)block, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = cluster > 1 ? 2 : 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, args...);
    if (e != cudaSuccess) { cudaGetLastError(); return cuda_fail(e, what); }
    return DPPO_OK;
}

// ---- device: status word ---------------------------------------------------------------------------
__device__ __forceinline__ void set_status(int32_t* status, int32_t code) {
    if (status != nullptr) atomicCAS(status, 0, code);   // first error wins
}

// ---- device: warp / block reductions -----------------------------------------------------------
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
// The same, no NaN among them, in one reduction: by integers in the order of the floats.  The f32 form of that instruction is not used: under
// a condition, even one that all lanes share (the vote's `bad ? 0 : max`), it returned another register's value for some rows of one
// kernel; the same kernel with the reduction moved out of the condition was right.
__device__ __forceinline__ int order_of(float v) {
    const int i = __float_as_int(v);
    return i ^ (i >> 31 & 0x7fffffff);
}
__device__ __forceinline__ float float_of(int order) { return __int_as_float(order ^ (order >> 31 & 0x7fffffff)); }
__device__ __forceinline__ float warp_max_f32(float v) { return float_of(__reduce_max_sync(0xffffffffu, order_of(v))); }
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

}  // namespace dppo
