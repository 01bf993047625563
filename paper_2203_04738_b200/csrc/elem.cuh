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

// two values rounded and packed by one instruction
__device__ __forceinline__ unsigned pack2(float a, float b, __nv_bfloat16) { const __nv_bfloat162 v = __floats2bfloat162_rn(a, b); return *reinterpret_cast<const unsigned*>(&v); }
__device__ __forceinline__ unsigned pack2(float a, float b, __half) { const __half2 v = __floats2half2_rn(a, b); return *reinterpret_cast<const unsigned*>(&v); }
__device__ __forceinline__ float2 unpack2(unsigned v, __nv_bfloat16) { return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)); }
__device__ __forceinline__ float2 unpack2(unsigned v, __half) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }

__device__ __forceinline__ float ex2(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

// VC values side by side.  Two of them use the packed fp32 instructions, which take one issue slot for both: streams of 16-bit types are
// bound by instructions rather than bytes otherwise (scan: 55 an element of 6 bytes without them and with 4-byte loads, 170 us where
// the bytes take 61).
template <int VC> struct F {
  float x[VC];
  __device__ __forceinline__ static F all(float v) {
    F f;
#pragma unroll
    for (int i = 0; i < VC; ++i) f.x[i] = v;
    return f;
  }
  __device__ __forceinline__ float& at(int i) { return x[i]; }
  __device__ __forceinline__ float at(int i) const { return x[i]; }
};
template <int VC> __device__ __forceinline__ F<VC> operator*(const F<VC>& a, const F<VC>& b) {
  F<VC> r;
  if (VC == 1) { r.x[0] = a.x[0] * b.x[0]; return r; }
#pragma unroll
  for (int i = 0; i + 1 < VC; i += 2)
    asm("{.reg .b64 p, q, r; mov.b64 p, {%2, %3}; mov.b64 q, {%4, %5}; mul.rn.f32x2 r, p, q; mov.b64 {%0, %1}, r;}"
        : "=f"(r.x[i]), "=f"(r.x[i + 1]) : "f"(a.x[i]), "f"(a.x[i + 1]), "f"(b.x[i]), "f"(b.x[i + 1]));
  return r;
}
template <int VC> __device__ __forceinline__ F<VC> operator+(const F<VC>& a, const F<VC>& b) {
  F<VC> r;
  if (VC == 1) { r.x[0] = a.x[0] + b.x[0]; return r; }
#pragma unroll
  for (int i = 0; i + 1 < VC; i += 2)
    asm("{.reg .b64 p, q, r; mov.b64 p, {%2, %3}; mov.b64 q, {%4, %5}; add.rn.f32x2 r, p, q; mov.b64 {%0, %1}, r;}"
        : "=f"(r.x[i]), "=f"(r.x[i + 1]) : "f"(a.x[i]), "f"(a.x[i + 1]), "f"(b.x[i]), "f"(b.x[i + 1]));
  return r;
}
template <int VC> __device__ __forceinline__ F<VC> fma_(const F<VC>& a, const F<VC>& b, const F<VC>& c) {
  F<VC> r;
  if (VC == 1) { r.x[0] = fmaf(a.x[0], b.x[0], c.x[0]); return r; }
#pragma unroll
  for (int i = 0; i + 1 < VC; i += 2)
    asm("{.reg .b64 p, q, r, s; mov.b64 p, {%2, %3}; mov.b64 q, {%4, %5}; mov.b64 r, {%6, %7}; fma.rn.f32x2 s, p, q, r; mov.b64 {%0, %1}, s;}"
        : "=f"(r.x[i]), "=f"(r.x[i + 1])
        : "f"(a.x[i]), "f"(a.x[i + 1]), "f"(b.x[i]), "f"(b.x[i + 1]), "f"(c.x[i]), "f"(c.x[i + 1]));
  return r;
}
template <int VC, class Fn> __device__ __forceinline__ F<VC> each(F<VC> a, Fn&& fn) {
  F<VC> r;
#pragma unroll
  for (int i = 0; i < VC; ++i) r.at(i) = fn(a.at(i), i);
  return r;
}

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
