// Orthogonalised matrices by Newton-Schulz products: X = G / |G|, then `steps` times
//   A = X X',  B = b A + c A^2,  X <- a X + B X
// with the shorter side of G as X's rows (X is G' where G is taller than wide).
#include <cmath>

#include "gmc.h"
#include "gmc_device.cuh"
#include "gmc_internal.h"
#include "gmc_vec.cuh"

using namespace gmc;

namespace {

constexpr int kMostSteps = 16;

// One matrix of K, element (i, j) of X's orientation at x + i * si + j * sj.
template <typename T>
struct Side {
  T* x;
  int64_t sk, si, sj;
};
struct Shape {
  int64_t m, n;  // m <= n
};

// sum of squares of each matrix, 64 bits
template <typename T>
__global__ void __launch_bounds__(256) k_size(Side<const T> G, Shape S, double* size) {
  __shared__ double ws[8];
  double s = 0.;
  for (int64_t i = threadIdx.x; i < S.m * S.n; i += 256) {
    const double v = Vec<T>::one(G.x[blockIdx.x * G.sk + i / S.n * G.si + i % S.n * G.sj]);
    s += v * v;
  }
  s = warp_sum(s);
  if (threadIdx.x % 32 == 0) ws[threadIdx.x / 32] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < 8; ++i) s += ws[i];
    size[blockIdx.x] = sqrt(s);
  }
}
template <typename T>
__global__ void __launch_bounds__(256) k_first(Side<const T> G, Shape S, const double* size, float* x) {
  const int64_t i = blockIdx.x * 256ll + threadIdx.x, k = blockIdx.y;
  if (i >= S.m * S.n) return;
  const double v = Vec<T>::one(G.x[k * G.sk + i / S.n * G.si + i % S.n * G.sj]);
  x[k * S.m * S.n + i] = size[k] == 0. ? 0.f : (float)(v / size[k]);
}
template <typename T>
__global__ void __launch_bounds__(256) k_last(Side<T> O, Shape S, const float* x, float scale) {
  const int64_t i = blockIdx.x * 256ll + threadIdx.x, k = blockIdx.y;
  if (i < S.m * S.n) O.x[k * O.sk + i / S.n * O.si + i % S.n * O.sj] = Vec<T>::round(scale * x[k * S.m * S.n + i]);
}
// D = alpha C + beta P Q (or P Q' with kT), row-major, 32 x 32 a block.
template <bool kT>
__global__ void __launch_bounds__(256) k_product(const float* P, const float* Q, const float* C, float* D, int64_t m,
                                                 int64_t n, int64_t l, float alpha, float beta) {
  __shared__ float p[32][33], q[32][33];
  const int64_t k = blockIdx.z, i0 = blockIdx.y * 32ll, j0 = blockIdx.x * 32ll;
  const int tx = threadIdx.x % 32, ty = threadIdx.x / 32;
  P += k * m * l;
  Q += k * l * n;
  float s[4] = {0.f, 0.f, 0.f, 0.f};
  for (int64_t l0 = 0; l0 < l; l0 += 32) {
    for (int r = ty; r < 32; r += 8) {
      p[r][tx] = i0 + r < m && l0 + tx < l ? P[(i0 + r) * l + l0 + tx] : 0.f;
      if (kT) q[tx][r] = j0 + r < n && l0 + tx < l ? Q[(j0 + r) * l + l0 + tx] : 0.f;
      else q[r][tx] = l0 + r < l && j0 + tx < n ? Q[(l0 + r) * n + j0 + tx] : 0.f;
    }
    __syncthreads();
    // (sums of sums: 5,000 terms one after the other were off by 2.7e-6 of the result after five steps)
    for (int u = 0; u < 4; ++u) {
      float t = 0.f;
      for (int c = 0; c < 32; ++c) t = __fmaf_rn(p[ty + 8 * u][c], q[c][tx], t);
      s[u] += t;
    }
    __syncthreads();
  }
  for (int u = 0; u < 4; ++u) {
    const int64_t i = i0 + ty + 8 * u, j = j0 + tx, at = k * m * n + i * n + j;
    if (i < m && j < n) D[at] = C ? __fmaf_rn(beta, s[u], alpha * C[at]) : s[u];
  }
}

struct Work {
  double* size;
  float *x, *y, *a, *b;
};
int64_t up(int64_t v) { return (v + 63) / 64 * 64; }
int64_t work_of(int64_t K, Shape S, char* at, Work* w) {
  const int64_t size = up(8 * K), x = up(4 * K * S.m * S.n), a = up(4 * K * S.m * S.m);
  if (w) {
    w->size = reinterpret_cast<double*>(at);
    w->x = reinterpret_cast<float*>(at + size);
    w->y = reinterpret_cast<float*>(at + size + x);
    w->a = reinterpret_cast<float*>(at + size + 2 * x);
    w->b = reinterpret_cast<float*>(at + size + 2 * x + a);
  }
  return size + 2 * x + 2 * a;
}
Shape shape_of(int64_t m, int64_t n) { return m <= n ? Shape{m, n} : Shape{n, m}; }

bool sizes_ok(int32_t dtype, int64_t K, int64_t m, int64_t n) {
  if (dtype != GMC_F32 && dtype != GMC_BF16 && dtype != GMC_F16) return false;
  if (K < 0 || m < 0 || n < 0 || K > 65535 || m > (1 << 20) || n > (1 << 20)) return false;
  return K == 0 || m == 0 || n <= (int64_t(1) << 36) / K / m;
}
bool strides_ok(const void* p, int32_t dtype, int64_t K, int64_t m, int64_t n, int64_t sk, int64_t ld) {
  const uintptr_t size = dtype == GMC_F32 ? 4 : 2;
  if (!p || reinterpret_cast<uintptr_t>(p) % size) return false;
  if (m > 1 && (ld < n || ld > (int64_t(1) << 40))) return false;
  return K <= 1 || (sk >= (m - 1) * (m > 1 ? ld : 0) + n && sk <= (int64_t(1) << 40));
}

}  // namespace

extern "C" {

int64_t gmc_orthogonalize_workspace(int32_t dtype, int64_t K, int64_t m, int64_t n) {
  if (!sizes_ok(dtype, K, m, n)) return -1;
  return work_of(K, shape_of(m, n), nullptr, nullptr);
}

int gmc_orthogonalize(const void* x_dev, int64_t ldk, int64_t ld, void* out_dev, int64_t out_ldk, int64_t out_ld,
                      int32_t dtype, int64_t K, int64_t m, int64_t n, int32_t steps, const float* coefficients_host,
                      float scale, void* workspace_dev, int64_t workspace_bytes, void* stream) {
  if (!sizes_ok(dtype, K, m, n) || steps < 1 || steps > kMostSteps || !coefficients_host || !std::isfinite(scale))
    return GMC_EINVAL;
  for (int i = 0; i < 3 * steps; ++i)
    if (!std::isfinite(coefficients_host[i])) return GMC_EINVAL;
  if (K == 0 || m == 0 || n == 0) return GMC_OK;
  if (!strides_ok(x_dev, dtype, K, m, n, ldk, ld) || !strides_ok(out_dev, dtype, K, m, n, out_ldk, out_ld))
    return GMC_EINVAL;
  const Shape S = shape_of(m, n);
  Work w;
  if (!workspace_dev || reinterpret_cast<uintptr_t>(workspace_dev) % 256 ||
      workspace_bytes < work_of(K, S, static_cast<char*>(workspace_dev), &w))
    return GMC_EINVAL;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool turned = m > n;
  const cudaError_t err = by_type(dtype, [&](auto t) {
    using T = decltype(t);
    const Side<const T> G{static_cast<const T*>(x_dev), ldk, turned ? 1 : ld, turned ? ld : 1};
    const Side<T> O{static_cast<T*>(out_dev), out_ldk, turned ? 1 : out_ld, turned ? out_ld : 1};
    const dim3 each((unsigned)((S.m * S.n + 255) / 256), (unsigned)K);
    const unsigned tm = (unsigned)((S.m + 31) / 32), tn = (unsigned)((S.n + 31) / 32);
    k_size<T><<<(unsigned)K, 256, 0, s>>>(G, S, w.size);
    k_first<T><<<each, 256, 0, s>>>(G, S, w.size, w.x);
    for (int i = 0; i < steps; ++i) {
      const float* c = coefficients_host + 3 * i;
      k_product<true><<<dim3(tm, tm, (unsigned)K), 256, 0, s>>>(w.x, w.x, nullptr, w.a, S.m, S.m, S.n, 0.f, 1.f);
      k_product<false><<<dim3(tm, tm, (unsigned)K), 256, 0, s>>>(w.a, w.a, w.a, w.b, S.m, S.m, S.m, c[1], c[2]);
      k_product<false><<<dim3(tn, tm, (unsigned)K), 256, 0, s>>>(w.b, w.x, w.x, w.y, S.m, S.n, S.m, c[0], 1.f);
      float* was = w.x;
      w.x = w.y;
      w.y = was;
    }
    k_last<T><<<each, 256, 0, s>>>(O, S, w.x, scale);
    return cudaGetLastError();
  });
  return err == cudaSuccess ? GMC_OK : GMC_ECUDA;
}

}  // extern "C"
