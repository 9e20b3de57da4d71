// The losses a post-training step starts its backward pass from, with the
// gradient of the logits: log-probabilities of given tokens, the preference loss on
// paired log ratios, and the host side of these and of the policy loss
// (gmc_policy.cu). gmc_loss.cuh states the mathematics.
#include <cfloat>
#include <cmath>
#include <new>

#include "gmc.h"
#include "gmc_loss.cuh"

using namespace gmc;

namespace {

// logp and (m, log S) of each row: a cluster of blocks a row. S is written as +inf for an
// empty row, which no sum reaches.
template <typename T>
__global__ void __launch_bounds__(kLossThreads) k_stats(Rows<T> R, float* logp, float2* stats, int parts) {
  __shared__ MaxSum ws[32], cs[kMaxParts];
  const int64_t row = blockIdx.x / parts;
  const int part = (int)(blockIdx.x - row * parts);
  const int64_t y = R.y[row];
  if (y < 0) {  // not scored
    if (part == 0 && threadIdx.x == 0) {
      logp[row] = 0.f;
      if (stats) stats[row] = make_float2(0.f, 0.f);
    }
    return;
  }
  if (parts > 1) cluster_arrive();
  const T* x = R.x + row * R.ld;
  const float xy = target_logit(x, R.V, y);
  MaxSum a = block_merge(sweep(x, R.V, R.b, part, parts), R.b, ws);
  if (parts > 1) cluster_wait();  // every block has begun
  a = cluster_merge(a, parts, R.b, cs);
  if (part == 0 && threadIdx.x == 0) {
    const RowStats r = finish(a, xy, R.b);
    logp[row] = r.logp;
    if (stats) stats[row] = make_float2(r.h.h, r.empty ? INFINITY : r.ls);
  }
}

// dx = g s ([v = y] - p) of each row from its saved (m, log S); slope: g of a
// row is that of its pair, read through the sequences' offsets, instead of g[row].
template <typename T>
__global__ void __launch_bounds__(kLossThreads) k_grad(Rows<T> R, const float2* stats, const float* g,
                                                       const int64_t* offsets, const float* slope, int64_t pairs,
                                                       T* dx, int64_t dld, int parts) {
  const int64_t row = blockIdx.x / parts;
  const int part = (int)(blockIdx.x - row * parts);
  const int64_t y = R.y[row];
  float coef = 0.f;
  if (y >= 0) {
    if (offsets) {  // the last sequence that starts at or before the row
      int64_t lo = 0, hi = 2 * pairs;
      while (lo < hi) {
        const int64_t mid = (lo + hi) >> 1;
        if (offsets[mid] <= row) lo = mid + 1;
        else hi = mid;
      }
      const int64_t s = lo - 1;
      if (s >= 0 && row < offsets[s + 1]) coef = (s & 1) ? -slope[s >> 1] : slope[s >> 1];
    } else {
      coef = g[row];
    }
    if (y >= R.V) coef = __uint_as_float(kNan);
  }
  const float2 st = coef != 0.f ? stats[row] : make_float2(0.f, 0.f);
  write_gradient(R.x + row * R.ld, dx + row * dld, R.V, grad_of(shift_of(st.x, R.b), st.y, coef, y, R.b), R.b,
                 coef == 0.f || st.y == INFINITY, part, parts);
}

// Sum of n doubles in a fixed order, one block.
__global__ void __launch_bounds__(1024) k_sum(const double* v, int64_t n, float* out) {
  __shared__ double ws[32];
  double s = 0.;
  for (int64_t i = threadIdx.x; i < n; i += blockDim.x) s += v[i];
  s = warp_sum(s);
  if ((threadIdx.x & 31) == 0) ws[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x < 32) {
    s = warp_sum(ws[threadIdx.x]);
    if (threadIdx.x == 0) *out = (float)s;
  }
}

struct PairArgs {
  const int64_t* offsets;
  int64_t n, pairs;
  const int64_t* y;
  const float* logp;
  const float2* stats;
  const float *ref_logp, *weights;
  float weight, beta, smoothing;
  float *pair_loss, *seq_ratio, *slope;
  double* wloss;
};
__device__ __forceinline__ float softplus(float x) { return fmaxf(x, 0.f) + log1pf(expf(-fabsf(x))); }

// One block a pair: the log ratios of its two sequences, its loss and the slope
// beta w dl/dmargin of the chosen sequence's log-probabilities.
__global__ void __launch_bounds__(256) k_pair(PairArgs P) {
  __shared__ double ws[8];
  const int64_t p = blockIdx.x;
  double sums[2];
  for (int side = 0; side < 2; ++side) {
    int64_t lo = P.offsets[2 * p + side], hi = P.offsets[2 * p + side + 1];
    lo = lo < 0 ? 0 : lo;
    hi = hi > P.n ? P.n : hi;
    double s = 0.;
    for (int64_t i = lo + threadIdx.x; i < hi; i += blockDim.x)
      if (P.y[i] >= 0 && P.stats[i].y != INFINITY) s += (double)P.logp[i] - (P.ref_logp ? (double)P.ref_logp[i] : 0.);
    s = warp_sum(s);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) ws[threadIdx.x >> 5] = s;
    __syncthreads();
    s = 0.;
    for (int i = 0; i < 8; ++i) s += ws[i];
    sums[side] = s;
  }
  if (threadIdx.x) return;
  const float margin = (float)((double)P.beta * (sums[0] - sums[1]));
  const float w = P.weights ? P.weights[p] : P.weight;
  const float up = softplus(-margin), down = softplus(margin);  // -log sigmoid(margin), -log sigmoid(-margin)
  const float loss = (1.f - P.smoothing) * up + P.smoothing * down;
  const float sig_up = 1.f / (1.f + expf(-margin)), sig_down = 1.f / (1.f + expf(margin));
  P.slope[p] = w == 0.f ? 0.f : w * P.beta * (P.smoothing * sig_up - (1.f - P.smoothing) * sig_down);
  P.wloss[p] = w == 0.f ? 0. : (double)w * (double)loss;
  if (P.pair_loss) P.pair_loss[p] = loss;
  if (P.seq_ratio) P.seq_ratio[2 * p] = (float)sums[0], P.seq_ratio[2 * p + 1] = (float)sums[1];
}

}  // namespace

struct gmc_loss_ctx {
  int device = 0;
  int64_t max_rows = 0, max_pairs = 0;
  void* mem = nullptr;
  float2* stats = nullptr;   // max_rows
  double* wloss = nullptr;   // max_pairs
  double* partial = nullptr; // kMostClusters
  uint32_t* ticket = nullptr;
  float* logp = nullptr;     // max_rows
  float* slope = nullptr;    // max_pairs
};

namespace {

// Checks shared by the calls that read logits.
bool rows_ok(const void* x, int32_t dtype, int64_t n, int64_t V, int64_t ld, float scale, const int64_t* y) {
  if (dtype != GMC_F32 && dtype != GMC_BF16 && dtype != GMC_F16) return false;
  const uintptr_t size = dtype == GMC_F32 ? 4 : 2;
  if (n < 0 || V < 1 || V >= (int64_t(1) << 31) || n > (int64_t(1) << 27)) return false;
  if (ld < V || ld > (int64_t(1) << 40)) return false;
  if (!std::isfinite(scale) || !(scale > 0.f)) return false;
  if (n == 0) return true;
  return x && y && reinterpret_cast<uintptr_t>(x) % size == 0 && reinterpret_cast<uintptr_t>(y) % 8 == 0;
}
// A pointer to T (or NULL).
template <typename T>
bool at_own_size(const T* p) {
  return reinterpret_cast<uintptr_t>(p) % sizeof(T) == 0;
}
template <typename... T>
bool aligned(const T*... p) {
  return (at_own_size(p) && ...);
}
bool out_ok(const void* x, int64_t ld, const void* dx, int64_t dld, int32_t dtype, int64_t V) {
  const uintptr_t size = dtype == GMC_F32 ? 4 : 2;
  if (dld < V || dld > (int64_t(1) << 40) || reinterpret_cast<uintptr_t>(dx) % size != 0) return false;
  return dx != x || dld == ld;  // in place: the same rows
}

template <typename T>
Rows<T> rows_of(const void* x, int64_t n, int64_t V, int64_t ld, float scale, const int64_t* y) {
  return Rows<T>{static_cast<const T*>(x), n, V, ld, base_of(scale), y};
}

int done(cudaError_t err) { return err == cudaSuccess ? GMC_OK : GMC_ECUDA; }

}  // namespace

extern "C" {

int gmc_token_logp(const void* logits_dev, int32_t dtype, int64_t n, int64_t vocab, int64_t ld, float scale,
                   const int64_t* targets_dev, float* logp_dev, float* stats_dev, void* stream) {
  if (!rows_ok(logits_dev, dtype, n, vocab, ld, scale, targets_dev)) return GMC_EINVAL;
  if (!aligned(logp_dev) || (reinterpret_cast<uintptr_t>(stats_dev) & 7)) return GMC_EINVAL;
  if (n == 0) return GMC_OK;
  if (!logp_dev) return GMC_EINVAL;
  return done(by_type(dtype, [&](auto t) {
    using T = decltype(t);
    const int parts = parts_for(n, vocab * (int64_t)sizeof(T));
    return launch(k_stats<T>, n * parts, kLossThreads, parts, static_cast<cudaStream_t>(stream),
                  rows_of<T>(logits_dev, n, vocab, ld, scale, targets_dev), logp_dev,
                  reinterpret_cast<float2*>(stats_dev), parts);
  }));
}

int gmc_token_logp_backward(const void* logits_dev, int32_t dtype, int64_t n, int64_t vocab, int64_t ld, float scale,
                            const int64_t* targets_dev, const float* stats_dev, const float* dlogp_dev,
                            void* dlogits_dev, int64_t dld, void* stream) {
  if (!rows_ok(logits_dev, dtype, n, vocab, ld, scale, targets_dev)) return GMC_EINVAL;
  if (!out_ok(logits_dev, ld, dlogits_dev, dld, dtype, vocab)) return GMC_EINVAL;
  if (!aligned(dlogp_dev) || (reinterpret_cast<uintptr_t>(stats_dev) & 7)) return GMC_EINVAL;
  if (n == 0) return GMC_OK;
  if (!stats_dev || !dlogp_dev || !dlogits_dev) return GMC_EINVAL;
  return done(by_type(dtype, [&](auto t) {
    using T = decltype(t);
    const int parts = parts_for(n, vocab * (int64_t)sizeof(T));
    return launch(k_grad<T>, n * parts, kLossThreads, 1, static_cast<cudaStream_t>(stream),
                  rows_of<T>(logits_dev, n, vocab, ld, scale, targets_dev),
                  reinterpret_cast<const float2*>(stats_dev), dlogp_dev, (const int64_t*)nullptr,
                  (const float*)nullptr, int64_t(0), static_cast<T*>(dlogits_dev), dld, parts);
  }));
}

int gmc_loss_create(gmc_loss_t* out, int64_t max_rows, int64_t max_pairs) {
  if (!out) return GMC_EINVAL;
  *out = nullptr;
  if (max_rows < 1 || max_rows > (int64_t(1) << 27) || max_pairs < 0 || max_pairs > (int64_t(1) << 26))
    return GMC_EINVAL;
  gmc_loss_ctx* h = new (std::nothrow) gmc_loss_ctx();
  if (!h) return GMC_ENOMEM;
  h->max_rows = max_rows;
  h->max_pairs = max_pairs;
  const size_t bytes = 8 * (size_t)(kMostClusters + 1 + max_pairs + max_rows) + 4 * (size_t)(max_rows + max_pairs);
  cudaError_t err = cudaGetDevice(&h->device);
  if (err == cudaSuccess) err = lib_malloc(&h->mem, bytes);
  // the memset runs on the default stream, with which a caller's need not be ordered
  if (err == cudaSuccess) err = cudaMemset(h->mem, 0, bytes);
  if (err == cudaSuccess) err = cudaStreamSynchronize(nullptr);
  if (err != cudaSuccess) {
    lib_free(h->mem);
    delete h;
    return err == cudaErrorMemoryAllocation ? GMC_ENOMEM : GMC_ECUDA;
  }
  h->partial = static_cast<double*>(h->mem);
  h->ticket = reinterpret_cast<uint32_t*>(h->partial + kMostClusters);
  h->wloss = h->partial + kMostClusters + 1;
  h->stats = reinterpret_cast<float2*>(h->wloss + max_pairs);
  h->logp = reinterpret_cast<float*>(h->stats + max_rows);
  h->slope = h->logp + max_rows;
  *out = h;
  return GMC_OK;
}

void gmc_loss_destroy(gmc_loss_t h) {
  if (!h) return;
  DeviceGuard g(h->device);
  cudaDeviceSynchronize();
  lib_free(h->mem);
  delete h;
}

int gmc_policy_loss(gmc_loss_t h, const void* logits_dev, int32_t dtype, int64_t n, int64_t vocab, int64_t ld,
                    float scale, const int64_t* targets_dev, const float* old_logp_dev, const float* ref_logp_dev,
                    const float* advantages_dev, const float* weights_dev, float clip_low, float clip_high, float kl,
                    float* loss_dev, float* token_loss_dev, float* logp_dev, void* dlogits_dev, int64_t dld,
                    void* stream) {
  if (!h || !rows_ok(logits_dev, dtype, n, vocab, ld, scale, targets_dev) || n > h->max_rows || !loss_dev)
    return GMC_EINVAL;
  if (!(clip_low >= 0.f && clip_low <= 1.f) || !(clip_high >= 0.f) || !std::isfinite(clip_high)) return GMC_EINVAL;
  if (!(kl >= 0.f) || !std::isfinite(kl) || (kl > 0.f && n > 0 && !ref_logp_dev)) return GMC_EINVAL;
  if (n > 0 && (!old_logp_dev || !advantages_dev)) return GMC_EINVAL;
  if (!aligned(old_logp_dev, ref_logp_dev, advantages_dev, weights_dev, loss_dev, token_loss_dev, logp_dev))
    return GMC_EINVAL;
  if (dlogits_dev && !out_ok(logits_dev, ld, dlogits_dev, dld, dtype, vocab)) return GMC_EINVAL;
  DeviceGuard g(h->device);
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t err = cudaSuccess;
  if (n > 0) {
    const PolicyArgs P{old_logp_dev, kl > 0.f ? ref_logp_dev : nullptr, advantages_dev, weights_dev, clip_low,
                       clip_high, kl, (float)(1.0 / (double)n), token_loss_dev, logp_dev, loss_dev, h->partial,
                       h->ticket, kWaitLimitNs};
    err = by_type(dtype, [&](auto t) {
      using T = decltype(t);
      return launch_policy<T>(rows_of<T>(logits_dev, n, vocab, ld, scale, targets_dev), P, static_cast<T*>(dlogits_dev),
                              dld, s);
    });
  } else {
    err = launch(k_sum, 1, 1024, 1, s, (const double*)h->wloss, n, loss_dev);
  }
  return done(err);
}

int gmc_preference_loss(gmc_loss_t h, const void* logits_dev, int32_t dtype, int64_t n, int64_t vocab, int64_t ld,
                        float scale, const int64_t* targets_dev, const int64_t* offsets_dev, int64_t pairs,
                        const float* ref_logp_dev, const float* weights_dev, float beta, float smoothing,
                        float* loss_dev, float* pair_loss_dev, float* seq_ratio_dev, float* logp_dev,
                        void* dlogits_dev, int64_t dld, void* stream) {
  if (!h || !rows_ok(logits_dev, dtype, n, vocab, ld, scale, targets_dev) || n > h->max_rows || !loss_dev)
    return GMC_EINVAL;
  if (pairs < 0 || pairs > h->max_pairs || (pairs > 0 && !offsets_dev)) return GMC_EINVAL;
  if (!aligned(offsets_dev, ref_logp_dev, weights_dev, loss_dev, pair_loss_dev, seq_ratio_dev, logp_dev))
    return GMC_EINVAL;
  if (!std::isfinite(beta) || !(beta > 0.f) || !(smoothing >= 0.f && smoothing <= 1.f)) return GMC_EINVAL;
  if (dlogits_dev && !out_ok(logits_dev, ld, dlogits_dev, dld, dtype, vocab)) return GMC_EINVAL;
  DeviceGuard g(h->device);
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  float* logp = logp_dev ? logp_dev : h->logp;
  const float weight = pairs ? (float)(1.0 / (double)pairs) : 0.f;
  cudaError_t err = by_type(dtype, [&](auto t) {
    using T = decltype(t);
    const Rows<T> R = rows_of<T>(logits_dev, n, vocab, ld, scale, targets_dev);
    const int parts = parts_for(n, vocab * (int64_t)sizeof(T));
    cudaError_t e = cudaSuccess;
    if (n > 0) e = launch(k_stats<T>, n * parts, kLossThreads, parts, s, R, logp, h->stats, parts);
    if (e == cudaSuccess && pairs > 0) {
      const PairArgs P{offsets_dev, n, pairs, targets_dev, logp, h->stats, ref_logp_dev, weights_dev, weight, beta, smoothing,
                       pair_loss_dev, seq_ratio_dev, h->slope, h->wloss};
      e = launch(k_pair, pairs, 256, 1, s, P);
    }
    if (e == cudaSuccess) e = launch(k_sum, 1, 1024, 1, s, (const double*)h->wloss, pairs, loss_dev);
    if (e == cudaSuccess && n > 0 && dlogits_dev)
      e = launch(k_grad<T>, n * parts, kLossThreads, 1, s, R, (const float2*)h->stats, (const float*)nullptr,
                 offsets_dev, (const float*)h->slope, pairs, static_cast<T*>(dlogits_dev), dld, parts);
    return e;
  });
  return done(err);
}

}  // extern "C"
