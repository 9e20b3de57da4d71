// 16-byte vectors of the floating types that the loss and dropout kernels take
// (GMC_F32, GMC_BF16, GMC_F16), as 32-bit floats and back.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "gmc.h"
#include "gmc_device.cuh"

namespace gmc {

// 2^x, 2 ulp (ex2.approx): every exponential of a logit is formed with it, in 32 bits.
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// 16 bytes of a row, as floats and back (one rounding, to nearest even).
template <typename T>
struct Vec;
template <>
struct Vec<float> {
  static constexpr int N = 4;
  __device__ static void get(const uint4& q, float* f) {
    f[0] = __uint_as_float(q.x), f[1] = __uint_as_float(q.y);
    f[2] = __uint_as_float(q.z), f[3] = __uint_as_float(q.w);
  }
  __device__ static uint4 put(const float* f) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
  __device__ static float one(float v) { return v; }
  __device__ static float round(float v) { return v; }
};
template <>
struct Vec<__nv_bfloat16> {
  static constexpr int N = 8;
  __device__ static void get(const uint4& q, float* f) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) f[2 * i] = __uint_as_float(w[i] << 16), f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
  __device__ static uint4 put(const float* f) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  __device__ static float one(__nv_bfloat16 v) { return __bfloat162float(v); }
  __device__ static __nv_bfloat16 round(float v) { return __float2bfloat16_rn(v); }
};
template <>
struct Vec<__half> {
  static constexpr int N = 8;
  __device__ static void get(const uint4& q, float* f) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
      f[2 * i] = h.x, f[2 * i + 1] = h.y;
    }
  }
  __device__ static uint4 put(const float* f) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __half2 h = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  __device__ static float one(__half v) { return __half2float(v); }
  __device__ static __half round(float v) { return __float2half_rn(v); }
};

// The elements of a row that lie before its first 16-byte boundary.
template <typename T>
__device__ __forceinline__ int head_of(const T* p, int64_t V) {
  const int h = (int)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / (int)sizeof(T);
  return V < h ? (int)V : h;
}

template <typename F>
inline cudaError_t by_type(int32_t dtype, F&& f) {
  if (dtype == GMC_F32) return f(float());
  if (dtype == GMC_BF16) return f(__nv_bfloat16());
  return f(__half());
}

}  // namespace gmc
