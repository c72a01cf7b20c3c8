// Elements of three types as float: V of them with one access.
#pragma once
#include "hf_common.cuh"
#include <cuda_fp16.h>

// (WIDE false: aligned as one element only)
template <typename T, int V, bool WIDE = true> struct alignas(!WIDE ? sizeof(T) : (sizeof(T) * V < 16 ? sizeof(T) * V : 16)) Vec { T v[V]; };

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(bf16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ bf16 from_float<bf16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }
