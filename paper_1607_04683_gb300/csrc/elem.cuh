// elem.cuh — values of the types that pass between layers (qnn_dtype): runs of them as 32-bit words, to and from fp32 (each
// value rounded once), and the layer functions of the hardware's exponential and reciprocal.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <type_traits>

#include "../../include/qnn.h"
#include "qnn_device.cuh"

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

// V consecutive values as they lie in memory, a pair of 16-bit ones to a word, the first in its low half.
template <typename T, int V>
struct Run {
    static constexpr int kWords = (V * (int)sizeof(T) + 3) / 4;
    uint32_t w[kWords];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0;
    }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (sizeof(T) == 4)
            return __uint_as_float(w[i]);
        else if constexpr (std::is_same<T, __nv_bfloat16>::value)
            return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
        else
            return __half2float(__ushort_as_half((unsigned short)(i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu)));
    }
    __device__ __forceinline__ void set(const float *v) {
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            if constexpr (sizeof(T) == 4)
                w[i] = __float_as_uint(v[i]);
            else if constexpr (V == 1)
                w[i] = bits(from_f32<T>(v[0]));
            else if constexpr (std::is_same<T, __nv_bfloat16>::value) {
                const __nv_bfloat162 p = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t *>(&p);
            } else {
                const __half2 p = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
                w[i] = *reinterpret_cast<const uint32_t *>(&p);
            }
        }
    }
    static __device__ __forceinline__ uint32_t bits(float v) { return __float_as_uint(v); }
    static __device__ __forceinline__ uint32_t bits(__nv_bfloat16 v) { return __bfloat16_as_ushort(v); }
    static __device__ __forceinline__ uint32_t bits(__half v) { return __half_as_ushort(v); }
    // All V values at an address that is a multiple of their bytes (16 at most).
    __device__ __forceinline__ void load(const T *p) {
        if constexpr (V * sizeof(T) == 32) {
            const uint4 a = *reinterpret_cast<const uint4 *>(p), b = *(reinterpret_cast<const uint4 *>(p) + 1);
            w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w, w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
        } else if constexpr (V * sizeof(T) == 16) {
            const uint4 a = *reinterpret_cast<const uint4 *>(p);
            w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
        } else if constexpr (V * sizeof(T) == 8) {
            const uint2 a = *reinterpret_cast<const uint2 *>(p);
            w[0] = a.x, w[1] = a.y;
        } else if constexpr (V * sizeof(T) == 4) {
            w[0] = *reinterpret_cast<const uint32_t *>(p);
        } else {
            w[0] = *reinterpret_cast<const unsigned short *>(p);
        }
    }
    __device__ __forceinline__ void store(T *p) const {
        if constexpr (V * sizeof(T) == 32) {
            *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
            *(reinterpret_cast<uint4 *>(p) + 1) = make_uint4(w[4], w[5], w[6], w[7]);
        } else if constexpr (V * sizeof(T) == 16) {
            *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        } else if constexpr (V * sizeof(T) == 8) {
            *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
        } else if constexpr (V * sizeof(T) == 4) {
            *reinterpret_cast<uint32_t *>(p) = w[0];
        } else {
            *reinterpret_cast<unsigned short *>(p) = (unsigned short)w[0];
        }
    }
    // The first `count` values one by one, the others 0 (left out of a store).
    __device__ __forceinline__ void load_some(const T *p, int count) {
        clear();
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < count) {
                if constexpr (sizeof(T) == 4)
                    w[i] = *reinterpret_cast<const uint32_t *>(p + i);
                else
                    w[i / 2] |= (uint32_t) * reinterpret_cast<const unsigned short *>(p + i) << (16 * (i & 1));
            }
    }
    __device__ __forceinline__ void store_some(T *p, int count) const {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < count) {
                if constexpr (sizeof(T) == 4)
                    *reinterpret_cast<uint32_t *>(p + i) = w[i];
                else
                    *reinterpret_cast<unsigned short *>(p + i) = (unsigned short)(w[i / 2] >> (16 * (i & 1)));
            }
    }
};

// 2^x and 1/x by the hardware: 2 ulp and 1 ulp off at most; results below 2^-126 are 0.
__device__ __forceinline__ float exp2_hw(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float rcp_hw(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
constexpr float kLog2e = 1.44269504088896341f;

// v / (1 + exp(-v)).
__device__ __forceinline__ float silu(float v) { return __fmul_rn(v, rcp_hw(__fadd_rn(1.0f, exp2_hw(__fmul_rn(v, -kLog2e))))); }

// log(1 + exp(x)) = max(x, 0) + log(1 + e), e = exp(-|x|) in (0, 1], to a few ulp of the result also where e is small:
// log(1 + e) = 2 atanh(q), q = e / (2 + e) <= 1/3, and atanh(q) / q as a polynomial in q^2 on [0, 1/9], fitted to
// the series 2 (1 + q^2/3 + q^4/5 + ...) at five Chebyshev points (relative error 8e-9). A NaN stays one.
constexpr float kAtanh0 = 2.0f, kAtanh1 = 0.6666632294654846f, kAtanh2 = 0.4002459645271301f, kAtanh3 = 0.27965158224105835f,
                kAtanh4 = 0.28157779574394226f;
__device__ __forceinline__ float softplus(float x) {
    const float e = exp2_hw(__fmul_rn(fabsf(x), -kLog2e));
    const float q = __fmul_rn(e, rcp_hw(__fadd_rn(2.0f, e))), s = __fmul_rn(q, q);
    float p = __fmaf_rn(s, kAtanh4, kAtanh3);
    p = __fmaf_rn(p, s, kAtanh2);
    p = __fmaf_rn(p, s, kAtanh1);
    p = __fmaf_rn(p, s, kAtanh0);
    return __fmaf_rn(p, q, fmaxf(x, 0.0f));
}

// silu and softplus of two values, in paired instructions (one issue slot for two results).
__device__ __forceinline__ float2 silu2(float2 v) {
    const float2 x = fmul2_rn(v, f2(-kLog2e)), d = fadd2_rn(make_float2(exp2_hw(x.x), exp2_hw(x.y)), f2(1.0f));
    return fmul2_rn(v, make_float2(rcp_hw(d.x), rcp_hw(d.y)));
}
__device__ __forceinline__ float2 softplus2(float2 x) {
    const float2 y = fmul2_rn(make_float2(fabsf(x.x), fabsf(x.y)), f2(-kLog2e));
    const float2 e = make_float2(exp2_hw(y.x), exp2_hw(y.y)), d = fadd2_rn(e, f2(2.0f));
    const float2 q = fmul2_rn(e, make_float2(rcp_hw(d.x), rcp_hw(d.y))), s = fmul2_rn(q, q);
    float2 p = ffma2_rn(s, f2(kAtanh4), f2(kAtanh3));
    p = ffma2_rn(p, s, f2(kAtanh2));
    p = ffma2_rn(p, s, f2(kAtanh1));
    p = ffma2_rn(p, s, f2(kAtanh0));
    return ffma2_rn(p, q, make_float2(fmaxf(x.x, 0.0f), fmaxf(x.y, 0.0f)));
}

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
