// Dropout whose mask is a function of (seed, t, worker, site, index) and is never
// stored: the library's SplitMix64 counter stream gives element i of worker k 16
// bits, those of draw i/4 of the stream keyed by (seed, t, worker, site), from bit
// 16 (i mod 4) on. The element is kept iff they are at least q = round(65536 p),
// and divided by the share kept, (65536 - q) / 65536. The backward pass is the
// same call on the output's gradient.
#include <cmath>

#include "gmc.h"
#include "gmc_internal.h"
#include "gmc_vec.cuh"

using namespace gmc;

namespace {

constexpr int kDropThreads = 256;
// Sets the dropout streams apart from those of the block choice and the sample
// of the same (seed, t).
constexpr uint64_t kDropTag = 0x44524F504F555421ull;

template <typename T>
struct DropArgs {
  const T *x, *res;  // res may be NULL
  T* out;
  int64_t ldx, ldr, ldo;
  int64_t n;
  int64_t k0;
  uint32_t q;
  float gain;
  uint64_t seed;
  int64_t t, site;
};

__device__ __forceinline__ uint64_t drop_key(uint64_t seed, int64_t t, int64_t worker, int64_t site) {
  return sm64_mix(stream_key(seed ^ kDropTag, t, (uint64_t)(worker + 1)) + kGamma * (uint64_t)(site + 1));
}

// A thread a group of 4 elements (one draw).
template <typename T>
__global__ void __launch_bounds__(kDropThreads) k_dropout(DropArgs<T> A, int64_t blocks_per_row) {
  const int64_t k = blockIdx.x / blocks_per_row;
  const int64_t g = (blockIdx.x - k * blocks_per_row) * kDropThreads + threadIdx.x;
  const int64_t i0 = g * 4;
  if (i0 >= A.n) return;
  const uint64_t z = draw(drop_key(A.seed, A.t, A.k0 + k, A.site), (uint64_t)g);
  const T* x = A.x + k * A.ldx;
  const T* res = A.res ? A.res + k * A.ldr : nullptr;
  T* out = A.out + k * A.ldo;
  for (int e = 0; e < 4; ++e) {
    const int64_t i = i0 + e;
    if (i >= A.n) break;
    const bool keep = ((uint32_t)(z >> (16 * e)) & 0xffffu) >= A.q;
    float v = keep ? Vec<T>::one(x[i]) * A.gain : 0.f;
    if (res) v += Vec<T>::one(res[i]);
    out[i] = Vec<T>::round(v);
  }
}

template <typename T>
cudaError_t run(const DropArgs<T>& A, int64_t K, cudaStream_t s) {
  const int64_t per = (A.n + 4 * kDropThreads - 1) / (4 * kDropThreads);
  k_dropout<T><<<(unsigned)(per * K), kDropThreads, 0, s>>>(A, per);
  return cudaGetLastError();
}

}  // namespace

extern "C" int gmc_dropout(const void* x_dev, int64_t ldx, const void* residual_dev, int64_t ldr, void* out_dev,
                           int64_t ldo, int32_t dtype, int64_t worker0, int64_t K, int64_t n, double p,
                           uint64_t seed, int64_t t, int64_t site, void* stream) {
  if (dtype != GMC_F32 && dtype != GMC_BF16 && dtype != GMC_F16) return GMC_EINVAL;
  const uintptr_t size = dtype == GMC_F32 ? 4 : 2;
  constexpr int64_t kMost = int64_t(1) << 40;
  if (K < 0 || n < 0 || worker0 < 0 || t < 0 || site < 0 || !(p >= 0.0 && p <= 1.0)) return GMC_EINVAL;
  if (K > (int64_t(1) << 20) || n > kMost || worker0 > (int64_t(1) << 40)) return GMC_EINVAL;
  if (K > 1 && (ldx < n || ldo < n || ldx > kMost || ldo > kMost)) return GMC_EINVAL;
  if (K > 1 && residual_dev && (ldr < n || ldr > kMost)) return GMC_EINVAL;
  const int64_t per = (n + 4 * kDropThreads - 1) / (4 * kDropThreads);
  if (K * per >= (int64_t(1) << 31)) return GMC_EINVAL;
  if (K == 0 || n == 0) return GMC_OK;
  if (!x_dev || !out_dev) return GMC_EINVAL;
  for (const void* q : {x_dev, residual_dev, (const void*)out_dev})
    if (reinterpret_cast<uintptr_t>(q) % size) return GMC_EINVAL;
  const uint32_t q = (uint32_t)std::lrint(p * 65536.0);
  const float gain = q < 65536u ? 65536.f / (float)(65536u - q) : 0.f;
  const cudaError_t err = by_type(dtype, [&](auto z) {
    using T = decltype(z);
    const DropArgs<T> A{static_cast<const T*>(x_dev), static_cast<const T*>(residual_dev), static_cast<T*>(out_dev),
                        ldx, ldr, ldo, n, worker0, q, gain, seed, t, site};
    return run(A, K, static_cast<cudaStream_t>(stream));
  });
  return err == cudaSuccess ? GMC_OK : GMC_ECUDA;
}
