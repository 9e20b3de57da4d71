// The losses a post-training step starts its backward pass from, with the
// gradient of the logits: log-probabilities of given tokens, the clipped policy
// loss with a KL term, and the preference loss on paired log ratios.
//
// For a row x of V logits, a scale s (1 / temperature) and a target y:
//   m = max x,  S = sum_v exp(s (x_v - m)),  logp = s (x_y - m) - log S,
//   d logp / d x_v = s ([v = y] - p_v),  p_v = exp(s (x_v - m) - log S).
// A row whose logits are all -inf has no distribution: S = 0, logp = -inf, and
// it adds nothing to a loss or a gradient. Differences are taken before the
// scale is applied, so rows of the type's lowest value stay finite.
#include <cfloat>
#include <cmath>
#include <new>

#include "gmc.h"
#include "gmc_internal.h"
#include "gmc_vec.cuh"

using namespace gmc;

namespace {

constexpr int kLossThreads = 512;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kMaxParts = 8;  // blocks of a cluster that share a row (the portable limit)

// n rows of V logits, row r at x + r * ld, with the target of each.
template <typename T>
struct Rows {
  const T* x;
  int64_t n, V, ld;
  float scale, c;  // s and fl(s log2 e)
  const int64_t* y;
};

// A maximum and the sum of exp(s (x - m)) below it. m = -inf: nothing yet.
struct MaxSum {
  float m = -INFINITY, s = 0.f;
};
__device__ __forceinline__ float shift_of(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ MaxSum merge(const MaxSum& a, const MaxSum& b, float c) {
  MaxSum r;
  r.m = fmaxf(a.m, b.m);
  const float h = shift_of(r.m);
  r.s = a.s * exp2_fast((a.m - h) * c) + b.s * exp2_fast((b.m - h) * c);
  return r;
}
template <int N>
__device__ __forceinline__ void add(MaxSum* a, const float* f, float c) {
  float top = f[0];
#pragma unroll
  for (int i = 1; i < N; ++i) top = fmaxf(top, f[i]);
  const float m = fmaxf(a->m, top), h = shift_of(m);
  float s = a->s * exp2_fast((a->m - h) * c);
#pragma unroll
  for (int i = 0; i < N; ++i) s += exp2_fast((f[i] - h) * c);
  a->m = m;
  a->s = s;
}
// Over the block; every thread returns the result. ws: 32 entries of shared memory.
__device__ __forceinline__ MaxSum block_merge(MaxSum a, float c, MaxSum* ws) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    MaxSum b;
    b.m = __shfl_xor_sync(0xffffffffu, a.m, o);
    b.s = __shfl_xor_sync(0xffffffffu, a.s, o);
    a = merge(a, b, c);
  }
  if (lane == 0) ws[warp] = a;
  __syncthreads();
  a = lane < warps ? ws[lane] : MaxSum();
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    MaxSum b;
    b.m = __shfl_xor_sync(0xffffffffu, a.m, o);
    b.s = __shfl_xor_sync(0xffffffffu, a.s, o);
    a = merge(a, b, c);
  }
  return a;
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// Over the blocks of a cluster, in rank order: a is the block's, the same in all its
// threads. The blocks have arrived at the cluster's barrier once before, so that none
// writes into a block that has not begun.
__device__ __forceinline__ MaxSum cluster_merge(MaxSum a, int parts, float c, MaxSum* ws) {
  if (parts == 1) return a;
  cluster_wait();
  if (threadIdx.x < (unsigned)parts) {  // into slot `rank` of every block
    const uint32_t here = (uint32_t)__cvta_generic_to_shared(ws + cluster_rank());
    uint32_t there;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(here), "r"(threadIdx.x));
    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(there), "f"(a.m), "f"(a.s) : "memory");
  }
  cluster_arrive();
  cluster_wait();
  MaxSum r = ws[0];
  for (int i = 1; i < parts; ++i) r = merge(r, ws[i], c);
  return r;
}

// One block's share (`part` of `parts`) of a row's maximum and sum.
template <typename T>
__device__ __forceinline__ MaxSum sweep(const T* x, int64_t V, float c, int part, int parts) {
  constexpr int N = Vec<T>::N, U = 4;
  MaxSum a;
  const int head = head_of(x, V);
  const int64_t nv = (V - head) / N;
  const int tail = (int)(V - head - nv * N);
  const uint4* q = reinterpret_cast<const uint4*>(x + head);
  const int64_t per = (nv + parts - 1) / parts;
  const int64_t lo = per * part, hi = lo + per < nv ? lo + per : nv;
  int64_t i = lo + threadIdx.x;
  for (; i + (U - 1) * (int64_t)blockDim.x < hi; i += U * (int64_t)blockDim.x) {
    uint4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = q[i + u * (int64_t)blockDim.x];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float f[N];
      Vec<T>::get(v[u], f);
      add<N>(&a, f, c);
    }
  }
  for (; i < hi; i += blockDim.x) {
    float f[N];
    Vec<T>::get(q[i], f);
    add<N>(&a, f, c);
  }
  if (part == 0) {
    const int t = (int)threadIdx.x;
    if (t < head + tail) {
      const float f = Vec<T>::one(x[t < head ? (int64_t)t : V - tail + (t - head)]);
      add<1>(&a, &f, c);
    }
  }
  return a;
}

// log p of the target and log S from a row's maximum and sum.
struct RowStats {
  float m, ls, logp;  // shift, log of the sum (0 for an empty row), log-probability
  bool empty;
};
template <typename T>
__device__ __forceinline__ RowStats finish(const MaxSum& a, const T* x, int64_t V, int64_t y, float scale) {
  RowStats r;
  r.empty = a.m == -INFINITY && a.s == 0.f;
  r.m = shift_of(a.m);
  r.ls = r.empty ? 0.f : logf(a.s);
  r.logp = y >= V ? __int_as_float(0x7fffffff) : (Vec<T>::one(x[y]) - r.m) * scale - r.ls;
  return r;
}

// logp and (m, log S) of each row: a cluster of blocks a row.
template <typename T>
__global__ void __launch_bounds__(kLossThreads) k_stats(Rows<T> R, float* logp, float2* stats, int parts) {
  __shared__ MaxSum ws[32], cs[kMaxParts];
  const int64_t row = blockIdx.x / parts;
  const int part = (int)(blockIdx.x - row * parts);
  const int64_t y = R.y[row];
  if (y < 0) {  // not scored
    if (part == 0 && threadIdx.x == 0) {
      if (logp) logp[row] = 0.f;
      if (stats) stats[row] = make_float2(0.f, 0.f);
    }
    return;
  }
  if (parts > 1) cluster_arrive();
  const T* x = R.x + row * R.ld;
  MaxSum a = sweep(x, R.V, R.c, part, parts);
  a = cluster_merge(block_merge(a, R.c, ws), parts, R.c, cs);
  if (part == 0 && threadIdx.x == 0) {
    const RowStats r = finish(a, x, R.V, y, R.scale);
    if (logp) logp[row] = r.logp;
    if (stats) stats[row] = make_float2(r.m, r.empty ? INFINITY : r.ls);
  }
}

// Elements [lo, hi) of a row's gradient, coef s ([v = y] - p_v): 16-byte loads and,
// where the output row lies at the same offset from a 16-byte boundary, stores.
template <typename T>
__device__ __forceinline__ void write_gradient(const Rows<T>& R, const T* x, T* dx, int64_t y, float m, float ls,
                                               float coef, int64_t part, int64_t parts) {
  constexpr int N = Vec<T>::N;
  const int64_t V = R.V;
  const float k = coef * R.scale, ls2 = ls * kLog2e;
  const int head = head_of(x, V);
  const int64_t nv = (V - head) / N;
  const int tail = (int)(V - head - nv * N);
  const bool same = ((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(dx)) & 15) == 0;
  const bool skip = coef == 0.f || ls == INFINITY;  // no gradient: x is not read (it may hold anything)
  const int64_t per = (nv + parts - 1) / parts;
  const int64_t lo = per * part, hi = lo + per < nv ? lo + per : nv;
  auto at = [&](float v, int64_t j) {
    if (skip) return 0.f;
    if (j == y) return k * -expm1f((v - m) * R.scale - ls);
    return -k * exp2_fast((v - m) * R.c - ls2);
  };
  for (int64_t i = lo + threadIdx.x; i < hi; i += blockDim.x) {
    const int64_t j = head + i * N;
    float f[N];
    Vec<T>::get(skip ? make_uint4(0, 0, 0, 0) : *reinterpret_cast<const uint4*>(x + j), f);
#pragma unroll
    for (int e = 0; e < N; ++e) f[e] = at(f[e], j + e);
    if (same) {
      __stcs(reinterpret_cast<uint4*>(dx + j), Vec<T>::put(f));
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) dx[j + e] = Vec<T>::round(f[e]);
    }
  }
  if (part == 0 && (int)threadIdx.x < head + tail) {
    const int t = (int)threadIdx.x;
    const int64_t j = t < head ? (int64_t)t : V - tail + (t - head);
    dx[j] = Vec<T>::round(at(skip ? 0.f : Vec<T>::one(x[j]), j));
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
    if (y >= R.V) coef = __int_as_float(0x7fffffff);
  }
  const float2 st = y >= 0 ? stats[row] : make_float2(0.f, 0.f);
  write_gradient(R, R.x + row * R.ld, dx + row * dld, y, st.x, st.y, coef, part, parts);
}

struct PolicyArgs {
  const float *old_logp, *ref_logp, *adv, *weights;
  float clip_low, clip_high, kl, weight;  // weight: of every row, where weights is NULL
  float *token_loss, *logp;               // either may be NULL
  double* wloss;                          // weighted loss of each row
};

// The token's loss and its slope in logp.
__device__ __forceinline__ void policy_terms(const PolicyArgs& P, int64_t row, float logp, float* loss, float* slope) {
  const float adv = P.adv[row];
  const float ratio = expf(logp - P.old_logp[row]);
  const float plain = ratio * adv;
  const float lo = 1.f - P.clip_low, hi = 1.f + P.clip_high;
  const float clipped = (ratio < lo ? lo : ratio > hi ? hi : ratio) * adv;  // NaN stays NaN
  float l = plain <= clipped ? -plain : -clipped;
  float d = plain <= clipped ? -plain : 0.f;
  if (P.ref_logp) {
    const float far = P.ref_logp[row] - logp, ef = expf(far);
    l += P.kl * (ef - far - 1.f);
    d += P.kl * (1.f - ef);
  }
  if (l != l) d = l;
  *loss = l;
  *slope = d;
}

template <typename T>
__global__ void __launch_bounds__(kLossThreads) k_policy(Rows<T> R, PolicyArgs P, T* dx, int64_t dld, int parts) {
  __shared__ MaxSum ws[32], cs[kMaxParts];
  const int64_t row = blockIdx.x / parts;
  const int part = (int)(blockIdx.x - row * parts);
  const int64_t y = R.y[row];
  const float w = P.weights ? P.weights[row] : P.weight;
  const T* x = R.x + row * R.ld;
  RowStats r;
  float loss = 0.f, slope = 0.f;
  const bool counts = y >= 0 && w != 0.f;
  if (counts) {
    if (parts > 1) cluster_arrive();
    MaxSum a = sweep(x, R.V, R.c, part, parts);
    a = cluster_merge(block_merge(a, R.c, ws), parts, R.c, cs);
    r = finish(a, x, R.V, y, R.scale);
    if (!r.empty) policy_terms(P, row, r.logp, &loss, &slope);
  } else {
    r.m = r.ls = r.logp = 0.f;
  }
  if (part == 0 && threadIdx.x == 0) {
    if (P.token_loss) P.token_loss[row] = loss;
    if (P.logp) P.logp[row] = r.logp;
    P.wloss[row] = (double)w * (double)loss;
  }
  // x[y] was read by every thread before dx (which may be x itself) is written
  if (counts && parts > 1) {
    cluster_arrive();
    cluster_wait();
  } else {
    __syncthreads();
  }
  if (dx) write_gradient(R, x, dx + row * dld, y, r.m, r.ls, w * slope, part, parts);
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

// Launch a kernel of `blocks` blocks in clusters of `parts`.
template <typename... A, typename... B>
cudaError_t launch(void (*f)(A...), int64_t blocks, int threads, int parts, cudaStream_t s, B... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned)parts;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = parts > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, f, args...);
}

template <typename T>
int parts_for(int64_t n, int64_t V) {
  int parts = 1;
  while (parts < kMaxParts && n * parts < 304 && V * (int64_t)sizeof(T) / parts > 16384) parts *= 2;
  return parts;
}

}  // namespace

struct gmc_loss_ctx {
  int device = 0;
  int64_t max_rows = 0, max_pairs = 0;
  void* mem = nullptr;
  float2* stats = nullptr;   // max_rows
  double* wloss = nullptr;   // max(max_rows, max_pairs)
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
  return Rows<T>{static_cast<const T*>(x), n, V, ld, scale, scale * kLog2e, y};
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
    const int parts = parts_for<T>(n, vocab);
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
    const int parts = parts_for<T>(n, vocab);
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
  const int64_t most = max_rows > max_pairs ? max_rows : max_pairs;
  const size_t bytes = (size_t)max_rows * 12 + (size_t)most * 8 + (size_t)max_pairs * 4;
  cudaError_t err = cudaGetDevice(&h->device);
  if (err == cudaSuccess) err = lib_malloc(&h->mem, bytes);
  if (err != cudaSuccess) {
    delete h;
    return err == cudaErrorMemoryAllocation ? GMC_ENOMEM : GMC_ECUDA;
  }
  h->wloss = static_cast<double*>(h->mem);
  h->stats = reinterpret_cast<float2*>(h->wloss + most);
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
                       clip_high, kl, (float)(1.0 / (double)n), token_loss_dev, logp_dev, h->wloss};
    err = by_type(dtype, [&](auto t) {
      using T = decltype(t);
      const int parts = parts_for<T>(n, vocab);
      return launch(k_policy<T>, n * parts, kLossThreads, parts, s,
                    rows_of<T>(logits_dev, n, vocab, ld, scale, targets_dev), P, static_cast<T*>(dlogits_dev), dld,
                    parts);
    });
  }
  if (err == cudaSuccess) err = launch(k_sum, 1, 1024, 1, s, (const double*)h->wloss, n, loss_dev);
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
    const int parts = parts_for<T>(n, vocab);
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
