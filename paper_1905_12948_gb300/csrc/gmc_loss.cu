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

// The threads that work on a row: a block (G = kLossThreads), of which up to 8 share a row as
// a cluster, or a warp (G = 32).
struct Halves {
  double a, b;
};
template <int G>
struct Group {
  static_assert(G == 32 || G == kLossThreads, "a warp or a block");
  static constexpr int kRows = kLossThreads / G;  // rows of a block
  __device__ static int tid() { return G == 32 ? (int)threadIdx.x % 32 : (int)threadIdx.x; }
  __device__ static int of_block() { return G == 32 ? (int)threadIdx.x / 32 : 0; }  // of the block's rows
  // Over the group; every thread returns the result.
  __device__ static MaxSum merge(const MaxSum& a, const Base& b) {
    if constexpr (G == 32) {
      return warp_merge(a, b);
    } else {
      __shared__ MaxSum ws[32];
      return block_merge(a, b, ws);
    }
  }
  // Sums over the first and the second half of the group, in a fixed order.
  __device__ static Halves sums(double s) {
    Halves h{0., 0.};
    if constexpr (G == 32) {
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      h.a = __shfl_sync(0xffffffffu, s, 0);
      h.b = __shfl_sync(0xffffffffu, s, 16);
    } else {
      __shared__ double ws[kLossThreads / 32];
      s = warp_sum(s);
      __syncthreads();
      if ((threadIdx.x & 31) == 0) ws[threadIdx.x >> 5] = s;
      __syncthreads();
      for (int i = 0; i < kLossThreads / 64; ++i) h.a += ws[i], h.b += ws[kLossThreads / 64 + i];
    }
    return h;
  }
  // Thread 0 adds to a count that other groups add to; every thread returns whether it has
  // reached `all`. What the groups wrote before is then visible to this one.
  __device__ static bool last_of(uint32_t* count, uint32_t mine, int64_t all) {
    if constexpr (G == 32) {
      __syncwarp();
      int last = 0;
      if (tid() == 0) last = (int64_t)count_add(count, mine) + mine == all;
      last = __shfl_sync(0xffffffffu, last, 0);
      __syncwarp();  // what thread 0 acquired holds for all
      return last != 0;
    } else {
      __shared__ int last;
      __syncthreads();
      if (threadIdx.x == 0) last = (int64_t)count_add(count, mine) + mine == all;
      __syncthreads();
      return last != 0;
    }
  }
};

// logp and (m, log S) of a row, by a group or a cluster of blocks (thread 0 of part 0
// writes), and in ratio (NULL: not wanted) logp before its rounding, less ref's; 0 for a row
// that adds nothing. S is written as +inf for an empty row, which no sum reaches.
template <int G, typename T>
__device__ __forceinline__ void row_stats(const Rows<T>& R, int64_t row, int part, int parts, float* logp, float2* stats,
                                          const float* ref, double* ratio) {
  __shared__ MaxSum cs[kMaxParts];
  const bool writes = part == 0 && Group<G>::tid() == 0;
  const int64_t y = R.y[row];
  if (y < 0) {  // not scored
    if (writes) {
      logp[row] = 0.f;
      if (stats) stats[row] = make_float2(0.f, 0.f);
      if (ratio) ratio[row] = 0.;
    }
    return;
  }
  if (parts > 1) cluster_arrive();
  const T* x = R.x + row * R.ld;
  const float xy = target_logit(x, R.V, y);
  const double less = ref ? (double)ref[row] : 0.;
  MaxSum a = Group<G>::merge(sweep(x, R.V, R.b, part, parts, Group<G>::tid(), G), R.b);
  if (G != 32 && parts > 1) {
    cluster_wait();  // every block has begun
    a = cluster_merge(a, parts, R.b, cs);
  }
  if (writes) {
    const RowStats r = finish(a, xy, R.b);
    logp[row] = r.logp;
    if (stats) stats[row] = make_float2(r.h.h, r.empty ? INFINITY : r.ls);
    if (ratio) ratio[row] = r.empty ? 0. : (double)r.logp + (double)r.low - less;
  }
}

// Bound by memory: a block of 256 threads loads 16 KB at once, and six of them share an SM.
// 8,192 rows of 32,000 bf16 logits: 84 us, 6.2 TB/s; by warps, 8,000 rows of 4,096: 11.3 us,
// 5.8 TB/s, and 40,000 of 2,048: 39.6 us with 48 registers (five blocks an SM), 46 with 54.
template <typename T, int G>
__global__ void __launch_bounds__(kLossThreads, G == 32 ? 5 : 6) k_stats(Rows<T> R, float* logp, float2* stats,
                                                                         int parts) {
  griddep_wait();
  const int64_t at = blockIdx.x / parts, row = at * Group<G>::kRows + Group<G>::of_block();
  if (row < R.n)
    row_stats<G>(R, row, (int)(blockIdx.x - at * parts), parts, logp, stats, (const float*)nullptr, (double*)nullptr);
}

struct PairArgs {
  const int64_t* offsets;
  int64_t n, pairs;
  const float *ref_logp, *weights;
  double* ratio;                          // log ratio of each row
  float weight, beta, smoothing;          // weight: of every pair, where weights is NULL
  float *loss, *pair_loss, *seq_ratio;    // the last two may be NULL
  float* slope;                           // beta w dl/dmargin of each pair
  double* wloss;                          // weighted loss of each pair
  uint32_t* count;                        // rows done of each pair, then pairs done; 0 between calls
};
// The sequence that row is in (the last one that starts at or before it), -1: none.
__device__ __forceinline__ int64_t sequence_of(const PairArgs& P, int64_t row) {
  int64_t lo = 0, hi = 2 * P.pairs;
  while (lo < hi) {
    const int64_t mid = (lo + hi) >> 1;
    if (P.offsets[mid] <= row) lo = mid + 1;
    else hi = mid;
  }
  return lo > 0 && row < P.offsets[lo] ? lo - 1 : -1;
}

__device__ __forceinline__ float softplus(float x) { return fmaxf(x, 0.f) + log1pf(expf(-fabsf(x))); }
// A pair's loss and slope from its sequences' log ratios.
__device__ __forceinline__ void finish_pair(const PairArgs& P, int64_t p, float w, double chosen, double other) {
  const float margin = (float)((double)P.beta * (chosen - other));
  const float up = softplus(-margin), down = softplus(margin);  // -log sigmoid(margin), -log sigmoid(-margin)
  const float loss = (1.f - P.smoothing) * up + P.smoothing * down;
  const float sig_up = 1.f / (1.f + expf(-margin)), sig_down = 1.f / (1.f + expf(margin));
  P.slope[p] = w == 0.f ? 0.f : w * P.beta * (P.smoothing * sig_up - (1.f - P.smoothing) * sig_down);
  P.wloss[p] = w == 0.f ? 0. : (double)w * (double)loss;
  if (P.pair_loss) P.pair_loss[p] = loss;
  if (P.seq_ratio) P.seq_ratio[2 * p] = (float)chosen, P.seq_ratio[2 * p + 1] = (float)other;
}
__device__ __forceinline__ float weight_of(const PairArgs& P, int64_t p) { return P.weights ? P.weights[p] : P.weight; }
// By one group, half of it a sequence: the log ratios of a pair whose rows are all done.
template <int G>
__device__ __forceinline__ void pair_of_rows(const PairArgs& P, int64_t p) {
  constexpr int half = G / 2;
  const int tid = Group<G>::tid(), side = tid / half;
  const float w = weight_of(P, p);
  int64_t lo = P.offsets[2 * p + side], hi = P.offsets[2 * p + side + 1];
  lo = lo < 0 ? 0 : lo;
  hi = hi > P.n ? P.n : hi;
  double s = 0.;
  for (int64_t i = lo + tid % half; i < hi; i += half) s += __ldcg(P.ratio + i);
  const Halves h = Group<G>::sums(s);
  if (tid == 0) finish_pair(P, p, w, h.a, h.b);
}
// The pairs' weighted losses added up, by one group.
template <int G>
__device__ __forceinline__ void sum_pairs(const PairArgs& P) {
  double s = 0.;
  for (int64_t p = Group<G>::tid(); p < P.pairs; p += G) s += __ldcg(P.wloss + p);
  const Halves h = Group<G>::sums(s);
  if (Group<G>::tid() == 0) *P.loss = (float)(h.a + h.b);
}

// k_stats, and the pairs' losses and slopes: the group that does a pair's last row does the
// pair. The block (or cluster) past the last row does the pairs that have no rows. total:
// the group that does the last pair adds up the loss (k_grad does so where it follows).
// Six blocks an SM (40 registers): the pairs' part would take 58, and the sums' loads four
// blocks at once (16 pairs of 50,257: 391 us instead of 363).
template <typename T, int G>
__global__ void __launch_bounds__(kLossThreads, 6) k_pair_stats(Rows<T> R, PairArgs P, float* logp, float2* stats,
                                                                int parts, bool total) {
  griddep_wait();
  const int64_t at = blockIdx.x / parts, row = at * Group<G>::kRows + Group<G>::of_block();
  const int part = (int)(blockIdx.x - at * parts);
  uint32_t done = 1;
  if ((at + 1) * parts == gridDim.x) {
    if (part != 0 || Group<G>::of_block() != 0) return;
    uint32_t empty = 0;
    for (int64_t p = Group<G>::tid(); p < P.pairs; p += G)
      if (P.offsets[2 * p] >= P.offsets[2 * p + 2]) {
        finish_pair(P, p, weight_of(P, p), 0., 0.);
        ++empty;
      }
    const Halves h = Group<G>::sums((double)empty);
    done = (uint32_t)(h.a + h.b);
  } else {
    if (row >= R.n) return;
    int64_t p = -1, rows = 0;
    if (part == 0) {
      p = sequence_of(P, row);
      if (p >= 0) {
        p >>= 1;
        rows = P.offsets[2 * p + 2] - P.offsets[2 * p];
      }
    }
    row_stats<G>(R, row, part, parts, logp, stats, P.ref_logp, P.ratio);
    if (p < 0 || !Group<G>::last_of(P.count + p, 1, rows)) return;
    pair_of_rows<G>(P, p);
    if (Group<G>::tid() == 0) P.count[p] = 0;
  }
  if (!total || !Group<G>::last_of(P.count + P.pairs, done, P.pairs)) return;
  sum_pairs<G>(P);
  if (Group<G>::tid() == 0) P.count[P.pairs] = 0;
}

// dx = g s ([v = y] - p) of each row from its saved (m, log S). Without g, a row's is the
// slope of its pair (negated in the sequence not preferred).
template <typename T, int G>
__global__ void __launch_bounds__(kLossThreads, G == 32 ? 4 : 6) k_grad(Rows<T> R, const float2* stats, const float* g,
                                                                        PairArgs P, T* dx, int64_t dld, int parts) {
  griddep_wait();
  // from the last row to the first: the logits read last are still in the L2 cache
  const int64_t row = R.n - 1 - (blockIdx.x / parts * Group<G>::kRows + Group<G>::of_block());
  const int part = (int)(blockIdx.x % parts);
  if (row >= 0) {
    const int64_t y = R.y[row];
    float coef = 0.f;
    if (y >= 0) {
      if (!g) {
        const int64_t q = sequence_of(P, row);
        if (q >= 0) coef = q & 1 ? -P.slope[q >> 1] : P.slope[q >> 1];
      } else {
        coef = g[row];
      }
      if (y >= R.V) coef = __uint_as_float(kNan);
    }
    const float2 st = coef != 0.f ? stats[row] : make_float2(0.f, 0.f);
    write_gradient(R.x + row * R.ld, dx + row * dld, R.V, grad_of(shift_of(st.x, R.b), st.y, coef, y, R.b), R.b,
                   coef == 0.f || st.y == INFINITY, part, parts, Group<G>::tid(), G);
  }
  if (g || blockIdx.x != 0 || Group<G>::of_block() != 0) return;
  sum_pairs<G>(P);
  // whatever the offsets were, the next call finds the counts at 0
  for (int64_t i = Group<G>::tid(); i <= P.pairs; i += G) P.count[i] = 0;
}

}  // namespace

struct gmc_loss_ctx {
  int device = 0;
  Residency resident;
  int64_t hold_row = -1;     // test hook (gmc_test_withhold_row): of the next policy call,
  uint64_t hold_ns = 0;      // with this wait limit; 0: off
  int64_t max_rows = 0, max_pairs = 0;
  void* mem = nullptr;
  float2* stats = nullptr;   // max_rows
  double* wloss = nullptr;   // max_pairs
  double* partial = nullptr; // kMostClusters
  uint32_t* ticket = nullptr;
  float* logp = nullptr;     // max_rows
  double* ratio = nullptr;   // max_rows
  float* slope = nullptr;    // max_pairs
  uint32_t* count = nullptr; // max_pairs + 1, zero between calls
};

namespace {

// Checks shared by the calls that read logits.
bool rows_ok(const void* x, int32_t dtype, int64_t n, int64_t V, int64_t ld, float scale, const int64_t* y) {
  if (dtype != GMC_F32 && dtype != GMC_BF16 && dtype != GMC_F16) return false;
  const uintptr_t size = dtype == GMC_F32 ? 4 : 2;
  if (n < 0 || V < 1 || V >= (int64_t(1) << 31) || n > (int64_t(1) << 27)) return false;
  if (ld < V || ld > (int64_t(1) << 40)) return false;
  if (!(scale >= 0x1p-64f && scale <= 0x1p64f)) return false;
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

// Whether a warp does a row, or a block (or cluster) does. A block's barriers and merge cost
// as much as 10 KB of a row or more, a lone warp reads its row at 5 GB/s or so: warps where
// rows are short and there are enough of them for the last ones not to matter. The sums of
// bf16 rows, and the gradients, in us, by blocks and by warps:
//   rows   length     sums       gradients        rows   length     sums       gradients
//    620    2,048   3.7  3.3     3.7  3.4        2,000   8,192   9.1  7.4    12.1 11.1
//    620    8,192   4.3  6.0     5.3  6.9        2,000  16,384  12.7 11.7    21.0 29.4
//    900    4,096   4.8  4.3     5.5  4.7        8,000   4,096  29.1 11.5    38.9 22.4
//    900   12,000   6.6  7.7     7.0  9.2        8,192  16,384  53.4 49.1    75.2 86.2
bool by_warps(int64_t n, int64_t row_bytes) { return n >= 600 && row_bytes <= 24576 && row_bytes <= 12 * n; }
// Blocks of groups of G that do n rows.
template <int G>
int64_t blocks_for(int64_t n) {
  return (n + Group<G>::kRows - 1) / Group<G>::kRows;
}

template <typename T>
cudaError_t launch_grad(const Rows<T>& R, const float2* stats, const float* g, const PairArgs& P, T* dx, int64_t dld,
                        cudaStream_t s) {
  const int64_t bytes = R.V * (int64_t)sizeof(T);
  if (by_warps(R.n, bytes))
    return launch(k_grad<T, 32>, blocks_for<32>(R.n), kLossThreads, 1, s, R, stats, g, P, dx, dld, 1);
  const int parts = parts_for(R.n, bytes);
  return launch(k_grad<T, kLossThreads>, R.n * parts, kLossThreads, 1, s, R, stats, g, P, dx, dld, parts);
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
    const Rows<T> R = rows_of<T>(logits_dev, n, vocab, ld, scale, targets_dev);
    const int64_t bytes = vocab * (int64_t)sizeof(T);
    const cudaStream_t on = static_cast<cudaStream_t>(stream);
    float2* stats = reinterpret_cast<float2*>(stats_dev);
    if (by_warps(n, bytes))
      return launch(k_stats<T, 32>, blocks_for<32>(n), kLossThreads, 1, on, R, logp_dev, stats, 1);
    return with_parts(parts_for(n, bytes), [&](int parts) {
      return launch(k_stats<T, kLossThreads>, n * parts, kLossThreads, parts, on, R, logp_dev, stats, parts);
    });
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
    return launch_grad(rows_of<T>(logits_dev, n, vocab, ld, scale, targets_dev),
                       reinterpret_cast<const float2*>(stats_dev), dlogp_dev, PairArgs{}, static_cast<T*>(dlogits_dev), dld,
                       static_cast<cudaStream_t>(stream));
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
  const size_t bytes =
      8 * (size_t)(kMostClusters + 1 + max_pairs + 2 * max_rows) + 4 * (size_t)(max_rows + 2 * max_pairs + 1);
  cudaError_t err = cudaGetDevice(&h->device);
  if (err == cudaSuccess) err = cudaDeviceGetAttribute(&h->resident.sms, cudaDevAttrMultiProcessorCount, h->device);
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
  h->ratio = reinterpret_cast<double*>(h->stats + max_rows);
  h->logp = reinterpret_cast<float*>(h->ratio + max_rows);
  h->slope = h->logp + max_rows;
  h->count = reinterpret_cast<uint32_t*>(h->slope + max_pairs);
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

int gmc_test_withhold_row(gmc_loss_t h, int64_t row, uint64_t wait_limit_ns) {
  if (!h || row < 0 || row >= h->max_rows || wait_limit_ns < 1 || wait_limit_ns > 2000000000ull) return GMC_EINVAL;
  h->hold_row = row;
  h->hold_ns = wait_limit_ns;
  return GMC_OK;
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
                       h->ticket, h->hold_ns ? h->hold_ns : kWaitLimitNs, h->hold_ns ? h->hold_row : -1};
    h->hold_ns = 0;
    err = by_type(dtype, [&](auto t) {
      using T = decltype(t);
      return launch_policy<T>(rows_of<T>(logits_dev, n, vocab, ld, scale, targets_dev), P, static_cast<T*>(dlogits_dev),
                              dld, &h->resident, s);
    });
  } else {
    err = cudaMemsetAsync(loss_dev, 0, sizeof(float), s);
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
  const PairArgs P{offsets_dev, n, pairs, ref_logp_dev, weights_dev, h->ratio, weight, beta, smoothing,
                   loss_dev, pair_loss_dev, seq_ratio_dev, h->slope, h->wloss, h->count};
  const bool grad = n > 0 && dlogits_dev;
  cudaError_t err = by_type(dtype, [&](auto t) {
    using T = decltype(t);
    const Rows<T> R = rows_of<T>(logits_dev, n, vocab, ld, scale, targets_dev);
    const int64_t bytes = vocab * (int64_t)sizeof(T);
    cudaError_t e;
    if (by_warps(n, bytes))
      e = launch(k_pair_stats<T, 32>, blocks_for<32>(n) + 1, kLossThreads, 1, s, R, P, logp, h->stats, 1, !grad);
    else
      e = with_parts(parts_for(n, bytes), [&](int parts) {
        return launch(k_pair_stats<T, kLossThreads>, (n + 1) * parts, kLossThreads, parts, s, R, P, logp, h->stats, parts,
                      !grad);
      });
    if (e != cudaSuccess || !grad) return e;
    return launch_grad(R, (const float2*)h->stats, (const float*)nullptr, P, static_cast<T*>(dlogits_dev), dld, s);
  });
  if (err == cudaSuccess && !grad) err = cudaMemsetAsync(h->count, 0, sizeof(uint32_t) * (size_t)(pairs + 1), s);
  return done(err);
}

}  // extern "C"
