// Shared pieces of the operators around the layer: 16- and 32-bit element types, the SiLU of a convolution and the code of its
// value (correctly rounded from the exact quotient), and the reading of slots.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"

namespace ssdi8 {

// Four consecutive elements as floats (exact), and back (rounded to nearest even).
template <typename T> struct Elem;
template <> struct Elem<float> {
  typedef float4 raw4;
  static __device__ __forceinline__ float get(float v) { return v; }
  static __device__ __forceinline__ float put(float v) { return v; }
  static __device__ __forceinline__ float4 cvt(const raw4& v) { return v; }
  static __device__ __forceinline__ raw4 pack(const float4& v) { return v; }
};
template <> struct Elem<__half> {
  typedef uint2 raw4;
  static __device__ __forceinline__ float get(__half v) { return __half2float(v); }
  static __device__ __forceinline__ __half put(float v) { return __float2half_rn(v); }
  static __device__ __forceinline__ float4 cvt(const raw4& v) {
    const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&v.x));
    const float2 b = __half22float2(*reinterpret_cast<const __half2*>(&v.y));
    return make_float4(a.x, a.y, b.x, b.y);
  }
  static __device__ __forceinline__ raw4 pack(const float4& v) {
    const __half2 a = __floats2half2_rn(v.x, v.y), b = __floats2half2_rn(v.z, v.w);
    return make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
  }
};
template <> struct Elem<__nv_bfloat16> {
  typedef uint2 raw4;
  static __device__ __forceinline__ float get(__nv_bfloat16 v) { return __bfloat162float(v); }
  static __device__ __forceinline__ __nv_bfloat16 put(float v) { return __float2bfloat16_rn(v); }
  static __device__ __forceinline__ float4 cvt(const raw4& v) {
    return make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16),
                       __uint_as_float(v.y & 0xffff0000u));
  }
  static __device__ __forceinline__ raw4 pack(const float4& v) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
    return make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
  }
};
// four elements at p: one load where p is aligned to four elements, else one by one
template <typename T, bool ALIGNED>
__device__ __forceinline__ typename Elem<T>::raw4 load4(const T* p) {
  typename Elem<T>::raw4 r;
  if (ALIGNED) {
    r = __ldcs(reinterpret_cast<const typename Elem<T>::raw4*>(p));
  } else {
    T* e = reinterpret_cast<T*>(&r);
#pragma unroll
    for (int i = 0; i < 4; ++i) e[i] = p[i];
  }
  return r;
}

__device__ __forceinline__ float ex2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// The code of SiLU(v) is decided in binary32 wherever that is safe.  With M = |bias| + sum |w_k x_k| and eps = 2^-24:
//   v, a chain of W <= 4 fused multiply-adds, is off by at most 4 eps M, and SiLU's slope is below 1.1;
//   exp2(-v log2e): the product is off by 1.5 eps |v log2e|, ex2.approx by 4 eps; 1 + e, rcp.approx, the product with v, the
//   reciprocal of the step size and the product with it add 1, 2, 1, 2 and 1 eps
// so the quotient q is off by at most delta = 4.4 eps M / step + (11 + 1.5 |v|) eps |q|.  A quotient that lies nearer than that to the
// middle of two integers is formed again in binary64.  What each kernel allows for stands beside it (conv.cu: M and |q| of several
// tokens at once, a step size that is multiplied into 1 + e; token_step.cu: 5 eps M / step + (14 + 2 |v|) eps |q|).  Step sizes outside
// [1e-30, 1e30] always go that way.
constexpr float kEps = 5.9604645e-8f;   // 2^-24

// A slot or position that no call may have: the status word becomes SSDI8_ERR_SHAPE.  A time-out stays one (then there is more amiss
// than a row), whichever of the two a call meets first.
__device__ __forceinline__ void bad_row(int32_t* status) {
  constexpr int32_t timeout = (int32_t)SSDI8_ERR_DEVICE_TIMEOUT;
  if (status && atomicExch(status, (int32_t)SSDI8_ERR_SHAPE) == timeout) atomicExch(status, timeout);
}

// The slot of sequence b, or -1 (padding) with *bad set where the call names one that it may not: out of range, a negative
// position, or the slot of an earlier sequence.  All threads of the block call it.
__device__ __forceinline__ int slot_of(const int32_t* slots, const int32_t* pos, int nslots, int b, bool* bad) {
  const int s = slots ? slots[b] : b;
  const int p = pos ? pos[b] : 0;
  int twice = 0;
  if (slots)
    for (int i = threadIdx.x; i < b; i += blockDim.x) twice |= slots[i] == s;
  twice = __syncthreads_or(twice);
  *bad = s >= nslots || (s >= 0 && (p < 0 || twice));
  return *bad ? -1 : s;
}

}  // namespace ssdi8
