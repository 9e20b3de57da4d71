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

// Two floats in a register pair: one instruction for both (each rounded as alone).
using Pair = unsigned long long;
__device__ __forceinline__ Pair pair_of(float a, float b) {
  Pair p;
  asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "f"(a), "f"(b));
  return p;
}
__device__ __forceinline__ void split(Pair p, float* a, float* b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(*a), "=f"(*b) : "l"(p));
}
__device__ __forceinline__ Pair fma_pair(Pair a, Pair b, Pair c) {
  Pair d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ Pair add_pair(Pair a, Pair b) {
  Pair d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ Pair mul_pair(Pair a, Pair b) {
  Pair d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ Pair exp2_pair(Pair x) {
  float a, b;
  split(x, &a, &b);
  return pair_of(exp2_fast(a), exp2_fast(b));
}

// 16 bytes of a row, as floats and back (one rounding, to nearest even). top: the larger
// of two words' values, place by place; kLow: a word of -inf.
template <typename T>
struct Vec;
template <>
struct Vec<float> {
  static constexpr int N = 4;
  static constexpr uint32_t kLow = 0xff800000u;
  __device__ static uint32_t top(uint32_t a, uint32_t b) {
    return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
  }
  __device__ static float top_of(uint32_t w) { return __uint_as_float(w); }
  __device__ static void pairs(const uint4& q, Pair* p) {
    p[0] = pair_of(__uint_as_float(q.x), __uint_as_float(q.y));
    p[1] = pair_of(__uint_as_float(q.z), __uint_as_float(q.w));
  }
  __device__ static uint4 put_pairs(const Pair* p) {
    float f[4];
    split(p[0], f, f + 1);
    split(p[1], f + 2, f + 3);
    return put(f);
  }
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
  static constexpr uint32_t kLow = 0xff80ff80u;
  __device__ static uint32_t top(uint32_t a, uint32_t b) {
    const __nv_bfloat162 h = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  __device__ static float top_of(uint32_t w) {
    return fmaxf(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  }
  __device__ static void pairs(const uint4& q, Pair* p) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = pair_of(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
  }
  __device__ static uint4 put_pairs(const Pair* p) {
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) split(p[i], f + 2 * i, f + 2 * i + 1);
    return put(f);
  }
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
  static constexpr uint32_t kLow = 0xfc00fc00u;
  __device__ static uint32_t top(uint32_t a, uint32_t b) {
    const __half2 h = __hmax2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  __device__ static float top_of(uint32_t w) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    return fmaxf(f.x, f.y);
  }
  __device__ static void pairs(const uint4& q, Pair* p) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
      p[i] = pair_of(f.x, f.y);
    }
  }
  __device__ static uint4 put_pairs(const Pair* p) {
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) split(p[i], f + 2 * i, f + 2 * i + 1);
    return put(f);
  }
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

// 32 bytes of a row: the widest load and store there is. N elements.
template <typename T>
struct Wide {
  static constexpr int N = 2 * Vec<T>::N;
  uint4 a, b;
};
__device__ __forceinline__ bool on32(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 31) == 0; }
template <typename T>
__device__ __forceinline__ Wide<T> load_wide(const T* p, bool aligned) {
  Wide<T> v;
  if (aligned) {
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(v.a.x), "=r"(v.a.y), "=r"(v.a.z), "=r"(v.a.w), "=r"(v.b.x), "=r"(v.b.y), "=r"(v.b.z), "=r"(v.b.w)
                 : "l"(p));
    return v;
  }
  alignas(16) T e[Wide<T>::N];
#pragma unroll
  for (int i = 0; i < Wide<T>::N; ++i) e[i] = p[i];
  v.a = *reinterpret_cast<const uint4*>(e);
  v.b = *reinterpret_cast<const uint4*>(e + Vec<T>::N);
  return v;
}
template <typename T>
__device__ __forceinline__ void store_wide(T* p, const Wide<T>& v, bool aligned) {
  if (aligned) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v.a.x), "r"(v.a.y), "r"(v.a.z),
                 "r"(v.a.w), "r"(v.b.x), "r"(v.b.y), "r"(v.b.z), "r"(v.b.w)
                 : "memory");
    return;
  }
  alignas(16) T e[Wide<T>::N];
  *reinterpret_cast<uint4*>(e) = v.a;
  *reinterpret_cast<uint4*>(e + Vec<T>::N) = v.b;
#pragma unroll
  for (int i = 0; i < Wide<T>::N; ++i) p[i] = e[i];
}
// The elements of a row that lie before its first 32-byte boundary.
template <typename T>
__device__ __forceinline__ int wide_head(const T* p, int64_t n) {
  const int h = (int)((32 - (reinterpret_cast<uintptr_t>(p) & 31)) & 31) / (int)sizeof(T);
  return n < h ? (int)n : h;
}

template <typename F>
inline cudaError_t by_type(int32_t dtype, F&& f) {
  if (dtype == GMC_F32) return f(float());
  if (dtype == GMC_BF16) return f(__nv_bfloat16());
  return f(__half());
}

}  // namespace gmc
