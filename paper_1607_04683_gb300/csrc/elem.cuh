// elem.cuh — values of the types that pass between layers (qnn_dtype): to and from fp32, each rounded once.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "../../include/qnn.h"

namespace qnn {

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }

template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

}  // namespace qnn

// Calls f with a value of the C++ type of a qnn_dtype.
template <typename F>
inline auto with_type(int dtype, F f) {
    switch (dtype) {
        case QNN_BF16: return f(__nv_bfloat16());
        case QNN_F16: return f(__half());
        default: return f(float());
    }
}
