// Values of the three floating types the layer operators take, and the warp reductions they share.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math_constants.h>

#include "route_index.cuh"
#include "vp_internal.h"

namespace {

constexpr unsigned kAll = 0xffffffffu;

__device__ __forceinline__ float value_of(float x) { return x; }
__device__ __forceinline__ float value_of(__half x) { return __half2float(x); }
__device__ __forceinline__ float value_of(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T rounded(float x);
template <> __device__ __forceinline__ float rounded<float>(float x) { return x; }
template <> __device__ __forceinline__ __half rounded<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 rounded<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// V values that travel as one load or store.
template <typename T, int V>
struct alignas(sizeof(T) * V) Pack { T v[V]; };

__device__ __forceinline__ float warp_max(float x) {
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
    return r;
}
template <typename T>
__device__ __forceinline__ T warp_sum(T x) {          // the same tree for every lane: the order of the additions is fixed
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(kAll, x, o);
    return x;
}

// Calls fn with a null pointer of the element type that `dtype` names; false if there is none.
template <typename F>
bool with_type(int dtype, F fn) {
    if (dtype == VP_BF16) fn((__nv_bfloat16*)nullptr);
    else if (dtype == VP_F16) fn((__half*)nullptr);
    else if (dtype == VP_F32) fn((float*)nullptr);
    else return false;
    return true;
}
inline int size_of_type(int dtype) { return dtype == VP_F32 ? 4 : 2; }
inline bool is_type(int dtype) { return dtype == VP_BF16 || dtype == VP_F16 || dtype == VP_F32; }

}  // namespace
