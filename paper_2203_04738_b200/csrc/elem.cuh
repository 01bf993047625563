// Element types of the operators over given arrays (fp32, bf16, fp16): loads to fp32, stores rounded once to nearest.
#pragma once
#include <cuda_fp16.h>

#include "common.cuh"

namespace mg {

template <class T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }
template <class T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

inline size_t elem_size(int dtype) { return dtype == MGRIT_F32 ? 4 : 2; }
inline bool elem_known(int dtype) { return dtype == MGRIT_F32 || dtype == MGRIT_BF16 || dtype == MGRIT_F16; }
inline bool elem_aligned(const void* p, int dtype) { return ((uintptr_t)p & (elem_size(dtype) - 1)) == 0; }
inline bool aligned4(const void* p) { return ((uintptr_t)p & 3u) == 0; }

// f(tag) with a value of the C++ type of `dtype`
template <class F> inline void with_elem(int dtype, F&& f) {
  if (dtype == MGRIT_F32) f(float{});
  else if (dtype == MGRIT_BF16) f(__nv_bfloat16{});
  else f(__half{});
}

}  // namespace mg
