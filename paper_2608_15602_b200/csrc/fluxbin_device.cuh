// Small device and launch helpers shared by the attention-side kernels (rotary, cache, attention, block tables).
#ifndef FLUXBIN_DEVICE_CUH
#define FLUXBIN_DEVICE_CUH

#include "fluxbin_internal.h"

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#define FBD_CUDA(call) do { cudaError_t e_ = (call); if (e_ != cudaSuccess) return fb::record_cuda_error((int)e_); } while (0)

namespace fbd {

// ---- element types -------------------------------------------------------------------------------------

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

inline int type_size(int dtype) { return dtype == FLUXBIN_TYPE_FP32 ? 4 : 2; }
inline bool type_known(int dtype) { return dtype == FLUXBIN_TYPE_FP16 || dtype == FLUXBIN_TYPE_FP32 || dtype == FLUXBIN_TYPE_BF16; }
inline bool aligned_to(const void *p, size_t n) { return ((uintptr_t)p % n) == 0; }

// whether the heads of an output lie apart: the larger stride covers what the smaller one spans
inline bool heads_apart(int64_t tokens, int64_t heads, int64_t token, int64_t head, int64_t dim)
{
    token = token < 0 ? -token : token;
    head = head < 0 ? -head : head;
    if (tokens < 2 || heads < 2) return tokens > 1 ? token >= dim : heads < 2 || head >= dim;
    return token < head ? token >= dim && head >= token * (tokens - 1) + dim : head >= dim && token >= head * (heads - 1) + dim;
}

// ---- launches ------------------------------------------------------------------------------------------

// Programmatic stream serialization, as for the layer kernels: the kernel may be set up while its predecessor drains;
// wait_for_predecessor() comes before its first access to memory that an earlier kernel may write.
template <typename... Params, typename... Args>
inline cudaError_t launch(void (*kernel)(Params...), dim3 grid, int threads, size_t smem, cudaStream_t s, Args... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, Params(args)...);
}

__device__ __forceinline__ void let_successor_start() { asm volatile("griddepcontrol.launch_dependents;"); }
__device__ __forceinline__ void wait_for_predecessor() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

} // namespace fbd

#endif
