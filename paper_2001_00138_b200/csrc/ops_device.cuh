// Device helpers of the operators: vector access for the three storage types, and the activations.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "../../include/patdnn.h"

namespace patdnn {
namespace {

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// V consecutive elements, loaded and stored as one access of V * sizeof(T) bytes (a power of two, at most 16).
template <typename T, int V>
struct alignas(sizeof(T) * V) Vec {
    T v[V];
};

// 1 / (1 + exp(-z)): exp(-z) overflows to infinity for z < -88, where the quotient is 0, its limit in fp32.
__device__ __forceinline__ float sigmoid(float z) { return __fdividef(1.f, 1.f + __expf(-z)); }
__device__ __forceinline__ float activate(float z, int act) {
    if (act == PATDNN_ACT_RELU) return z < 0.f ? 0.f : z;          // NaN stays NaN
    if (act == PATDNN_ACT_SILU) return z * sigmoid(z);
    return z;
}
// d act / d z; ReLU has slope 0 at z = 0
__device__ __forceinline__ float activate_slope(float z, int act) {
    if (act == PATDNN_ACT_RELU) return z > 0.f ? 1.f : (z <= 0.f ? 0.f : z);
    if (act == PATDNN_ACT_SILU) {
        const float s = sigmoid(z);
        return s * fmaf(z, 1.f - s, 1.f);
    }
    return 1.f;
}

}  // namespace
}  // namespace patdnn
