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
constexpr int kDropVecs = 2;  // 32-byte vectors of a tensor that a thread loads together
// Sets the dropout streams apart from those of the block choice and the sample
// of the same (seed, t).
constexpr uint64_t kDropTag = 0x44524F504F555421ull;

template <typename T>
struct DropArgs {
  const T *x, *res;  // res may be NULL
  T* out;
  int64_t ldx, ldr, ldo;
  int64_t n;
  uint64_t key;       // of (seed, t)
  uint64_t worker0, site;
  uint32_t q;
  float gain;
};

// The stream's 16-bit numbers of N elements from element i on, two to a word. r =
// i mod 4 is the same for the whole row: 0 where its vectors begin with a draw.
template <int N>
__device__ __forceinline__ void bits_of(uint64_t key, int64_t i, int r, uint32_t* w) {
  uint64_t z[N / 4];
  uint64_t at = key + kGamma * (uint64_t)(i / 4 + 1);
#pragma unroll
  for (int d = 0; d < N / 4; ++d, at += kGamma) z[d] = sm64_mix(at);
  if (r) {  // each word pair spans two draws
    const uint64_t last = sm64_mix(at);
#pragma unroll
    for (int d = 0; d < N / 4; ++d) z[d] = (z[d] >> (16 * r)) | ((d + 1 < N / 4 ? z[d + 1] : last) << (64 - 16 * r));
  }
#pragma unroll
  for (int d = 0; d < N / 4; ++d) w[2 * d] = (uint32_t)z[d], w[2 * d + 1] = (uint32_t)(z[d] >> 32);
}

// One vector's elements: x kept and divided, or 0, plus res.
template <typename T, bool RES>
__device__ __forceinline__ uint4 drop_vec(const uint4& x, const uint4& res, const uint32_t* w, uint32_t q, bool none,
                                          float gain) {
  constexpr int N = Vec<T>::N;
  float f[N], g[N];
  Vec<T>::get(x, f);
  if (RES) Vec<T>::get(res, g);
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const uint32_t bits = e & 1 ? w[e / 2] : w[e / 2] << 16;  // the number in the upper half
    f[e] = bits >= q && !none ? f[e] * gain : 0.f;
    if (RES) f[e] += g[e];
  }
  return Vec<T>::put(f);
}

// A block takes kDropThreads * kDropVecs vectors of 32 bytes of a worker's row: those
// between x's 32-byte boundaries; the row's first elements (before its first boundary) and
// its last are left to a few threads of the row's first block.
//
// Bound by memory, nearly: a draw (two 64-bit products) gives four elements their 16 bits, so
// about 6 of a dozen instructions an element are the generator's.
template <typename T, bool RES>
__global__ void __launch_bounds__(kDropThreads) k_dropout(DropArgs<T> A, int64_t blocks_per_row) {
  constexpr int N = Wide<T>::N, H = Vec<T>::N, U = kDropVecs;
  griddep_wait();
  const int64_t k = blockIdx.x / blocks_per_row;
  const int64_t b = blockIdx.x - k * blocks_per_row;
  const T* x = A.x + k * A.ldx;
  const T* res = RES ? A.res + k * A.ldr : nullptr;
  T* out = A.out + k * A.ldo;
  const uint64_t key = sm64_mix(sm64_mix(A.key + kGamma * (A.worker0 + (uint64_t)k + 2)) + kGamma * (A.site + 1));
  const int head = wide_head(x, A.n);
  const int64_t nv = (A.n - head) / N;
  const int r = head & 3;
  const bool res_on = RES && on32(res + head), out_on = on32(out + head);
  const uint32_t q = A.q << 16;
  const bool none = A.q > 0xffffu;  // p = 1
  const int64_t v0 = b * (kDropThreads * U) + threadIdx.x;
  Wide<T> xv[U], rv[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t v = v0 + u * kDropThreads;
    if (v >= nv) continue;
    const int64_t i = head + v * N;
    xv[u] = load_wide(x + i, true);
    if (RES) rv[u] = load_wide(res + i, res_on);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t v = v0 + u * kDropThreads;
    if (v >= nv) continue;
    const int64_t i = head + v * N;
    uint32_t w[N / 2];
    bits_of<N>(key, i, r, w);
    Wide<T> y;
    y.a = drop_vec<T, RES>(xv[u].a, rv[u].a, w, q, none, A.gain);
    y.b = drop_vec<T, RES>(xv[u].b, rv[u].b, w + H / 2, q, none, A.gain);
    store_wide(out + i, y, out_on);
  }
  const int tail = (int)(A.n - head - nv * N);
  if (b == 0 && (int)threadIdx.x < head + tail) {
    const int t = (int)threadIdx.x;
    const int64_t i = t < head ? (int64_t)t : A.n - tail + (t - head);
    const uint32_t bits = (uint32_t)(draw(key, (uint64_t)(i / 4)) >> (16 * (i & 3))) & 0xffffu;
    float f = bits >= A.q ? Vec<T>::one(x[i]) * A.gain : 0.f;
    if (RES) f += Vec<T>::one(res[i]);
    out[i] = Vec<T>::round(f);
  }
}

// Blocks of a row: its vectors, and at least one for its edges.
int64_t blocks_of(int64_t n, int64_t per_vec) {
  const int64_t per = kDropThreads * kDropVecs * per_vec;
  return n / per + 1;
}

template <typename T>
cudaError_t run(const DropArgs<T>& A, int64_t K, cudaStream_t s) {
  const int64_t per = blocks_of(A.n, Wide<T>::N);
  const dim3 grid((unsigned)(per * K)), block(kDropThreads);
  return A.res ? launch_pdl(k_dropout<T, true>, grid, block, 0, s, A, per)
               : launch_pdl(k_dropout<T, false>, grid, block, 0, s, A, per);
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
  if (K * blocks_of(n, 32 / (int64_t)size) >= (int64_t(1) << 31)) return GMC_EINVAL;
  if (K == 0 || n == 0) return GMC_OK;
  if (!x_dev || !out_dev) return GMC_EINVAL;
  for (const void* q : {x_dev, residual_dev, (const void*)out_dev})
    if (reinterpret_cast<uintptr_t>(q) % size) return GMC_EINVAL;
  // in place: the same rows
  if (K > 1 && ((out_dev == x_dev && ldo != ldx) || (out_dev == residual_dev && ldo != ldr))) return GMC_EINVAL;
  const uint32_t q = (uint32_t)std::lrint(p * 65536.0);
  const float gain = q < 65536u ? 65536.f / (float)(65536u - q) : 0.f;
  const cudaError_t err = by_type(dtype, [&](auto z) {
    using T = decltype(z);
    const DropArgs<T> A{static_cast<const T*>(x_dev), static_cast<const T*>(residual_dev), static_cast<T*>(out_dev),
                        ldx, ldr, ldo, n, sm64_mix((seed ^ kDropTag) + kGamma * (uint64_t)(t + 1)),
                        (uint64_t)worker0, (uint64_t)site, q, gain};
    return run(A, K, static_cast<cudaStream_t>(stream));
  });
  return err == cudaSuccess ? GMC_OK : GMC_ECUDA;
}
