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
template <int G>
struct Group {
  static_assert(G == 32 || G == kLossThreads, "a warp or a block");
  static constexpr int kRows = kLossThreads / G;  // rows of a block
  __device__ static int tid() { return G == 32 ? (int)threadIdx.x % 32 : (int)threadIdx.x; }
  __device__ static int of_block() { return G == 32 ? (int)threadIdx.x / 32 : 0; }  // of the block's rows
  // Over the group; every thread returns the result.
  template <typename T>
  __device__ static MaxSum merge(const MaxSum& a, const Base& b) {
    if constexpr (G == 32) {
      return warp_merge<T>(a, b);
    } else {
      __shared__ MaxSum ws[32];
      return block_merge<T>(a, b, ws);
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
  MaxSum a = Group<G>::template merge<T>(sweep(x, R.V, R.b, part, parts, Group<G>::tid(), G), R.b);
  if (G != 32 && parts > 1) {
    cluster_wait();  // every block has begun
    a = cluster_merge<T>(a, parts, R.b, cs);
  }
  if (writes) {
    const RowStats r = finish(a, xy, R.b);
    logp[row] = r.logp;
    if (stats) stats[row] = make_float2(r.h.h, r.empty ? INFINITY : r.ls);
    if (ratio) ratio[row] = r.empty ? 0. : (double)r.logp + (double)r.low - less;
  }
}

// Bound by memory: a block of 256 threads loads 16 KB at once, and six of them share an SM.
// 8,192 rows of 32,000 bf16 logits: 83 us, 6.3 TB/s; by warps, 8,000 rows of 4,096: 11.3 us,
// 5.8 TB/s, and 40,000 of 2,048: 39.6 us with 48 registers (five blocks an SM), 46 with 54.
// kRatio: the log ratios are wanted (the code for them, where they are not, cost 10% of short
// rows' time).
template <typename T, int G, bool kRatio>
__global__ void __launch_bounds__(kLossThreads, G == 32 ? 5 : 6) k_stats(Rows<T> R, float* logp, float2* stats,
                                                                         const float* ref, double* ratio, int parts) {
  griddep_wait();
  const int64_t at = blockIdx.x / parts, row = at * Group<G>::kRows + Group<G>::of_block();
  if (row < R.n)
    row_stats<G>(R, row, (int)(blockIdx.x - at * parts), parts, logp, stats, kRatio ? ref : nullptr,
                 kRatio ? ratio : nullptr);
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
  uint32_t* ticket;                       // 0 between calls
};
// The sequence that row is in (the last one that starts at or before it), -1: none. By a
// warp, 32 offsets at a time: one read for 16 pairs, two for 500.
__device__ __forceinline__ int64_t sequence_of(const PairArgs& P, int64_t row) {
  const int lane = (int)threadIdx.x & 31;
  int64_t lo = 0, hi = 2 * P.pairs;  // the first offset past the row is in [lo, hi]
  while (lo < hi) {
    const int64_t step = (hi - lo + 31) >> 5, i = lo + (lane + 1) * step - 1;
    const uint32_t past = __ballot_sync(0xffffffffu, i >= hi || P.offsets[i] > row);
    const int64_t before = (past ? __ffs((int)past) - 1 : 32) * step;  // so many start at or before the row
    const int64_t end = lo + before + step - 1;
    lo = lo + before < hi ? lo + before : hi;
    hi = end < hi ? end : hi;
  }
  return lo > 0 && row < P.offsets[lo] ? lo - 1 : -1;
}

__device__ __forceinline__ float softplus(float x) { return fmaxf(x, 0.f) + log1pf(expf(-fabsf(x))); }
// A pair's loss and slope from its sequences' log ratios.
__device__ __forceinline__ void finish_pair(const PairArgs& P, int64_t p, float w, double chosen, double other) {
  const float margin = (float)((double)P.beta * (chosen - other));
  const float up = softplus(-margin), down = softplus(margin);  // -log sigmoid(margin), -log sigmoid(-margin)
  // a term with no weight is left out: the margin of a sequence with a masked token is infinite
  const float loss = (P.smoothing < 1.f ? (1.f - P.smoothing) * up : 0.f) + (P.smoothing > 0.f ? P.smoothing * down : 0.f);
  const float sig_up = 1.f / (1.f + expf(-margin)), sig_down = 1.f / (1.f + expf(margin));
  P.slope[p] = w == 0.f ? 0.f : w * P.beta * (P.smoothing * sig_up - (1.f - P.smoothing) * sig_down);
  P.wloss[p] = w == 0.f ? 0. : (double)w * (double)loss;
  if (P.pair_loss) P.pair_loss[p] = loss;
  if (P.seq_ratio) P.seq_ratio[2 * p] = (float)chosen, P.seq_ratio[2 * p + 1] = (float)other;
}
__device__ __forceinline__ float weight_of(const PairArgs& P, int64_t p) { return P.weights ? P.weights[p] : P.weight; }
// Sums over the first and the second half of the block, in a fixed order.
struct Halves {
  double a, b;
};
__device__ __forceinline__ Halves block_sums(double s) {
  __shared__ double ws[kLossThreads / 32];
  s = warp_sum(s);
  if ((threadIdx.x & 31) == 0) ws[threadIdx.x >> 5] = s;
  __syncthreads();
  Halves h{0., 0.};
  for (int i = 0; i < kLossThreads / 64; ++i) h.a += ws[i], h.b += ws[kLossThreads / 64 + i];
  return h;
}
// The pairs' weighted losses added up, by one block.
__device__ __forceinline__ void sum_pairs(const PairArgs& P) {
  double s = 0.;
  for (int64_t p = threadIdx.x; p < P.pairs; p += kLossThreads) s += __ldcg(P.wloss + p);
  const Halves h = block_sums(s);
  if (threadIdx.x == 0) *P.loss = (float)(h.a + h.b);
}

// The pairs' losses and slopes from their rows' log ratios: G threads a pair, half of them a
// sequence. total: the last block adds up the loss (k_grad does so where it follows).
// A chain of reads, 3 us; in the sums' kernel, by the block that counts the pair's last row,
// it took 5 to 7.
template <int G>
__global__ void __launch_bounds__(kLossThreads) k_pairs(PairArgs P, bool total) {
  constexpr int half = G / 2;
  griddep_wait();
  const int tid = Group<G>::tid();
  const int64_t p = blockIdx.x * (int64_t)Group<G>::kRows + Group<G>::of_block();
  if (p < P.pairs) {
    const int side = tid / half;
    const float w = weight_of(P, p);
    int64_t lo = P.offsets[2 * p + side], hi = P.offsets[2 * p + side + 1];
    lo = lo < 0 ? 0 : lo;
    hi = hi > P.n ? P.n : hi;
    double s = 0.;
#pragma unroll 4
    for (int64_t i = lo + tid % half; i < hi; i += half) s += P.ratio[i];
    Halves h;
    if constexpr (G == 32) {
#pragma unroll
      for (int o = half / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      h = Halves{s, __shfl_sync(0xffffffffu, s, half)};
    } else {
      h = block_sums(s);
    }
    if (tid == 0) finish_pair(P, p, w, h.a, h.b);
  }
  if (!total) return;
  __shared__ bool last;
  __syncthreads();
  if (threadIdx.x == 0) last = count_inc(P.ticket, gridDim.x - 1) == gridDim.x - 1;
  __syncthreads();
  if (last) sum_pairs(P);
}

// dx = g s ([v = y] - p) of each row from its saved (m, log S). Without g, a row's is the
// slope of its pair (negated in the sequence not preferred). Bound by memory, read and written:
// 4,096 rows of 50,257 fp32 239 us, 6.9 TB/s; by warps, 8,000 rows of 4,096 bf16 22 us, 5.9 TB/s.
template <typename T, int G>
__global__ void __launch_bounds__(kLossThreads, G == 32 ? 4 : 6) k_grad(Rows<T> R, const float2* stats, const float* g,
                                                                        PairArgs P, T* dx, int64_t dld, int parts) {
  griddep_wait();
  // from the last row to the first: the logits read last are still in the L2 cache
  const int64_t row = R.n - 1 - (blockIdx.x / parts * Group<G>::kRows + Group<G>::of_block());
  const int part = (int)(blockIdx.x % parts);
  if (row >= 0) {
    // all that the row needs to know, in as few reads behind each other as can be
    const int64_t y = R.y[row];
    const float2 st = stats[row];
    float coef = 0.f;
    if (g) {
      coef = g[row];
    } else {
      const int64_t q = sequence_of(P, row);
      if (q >= 0) coef = q & 1 ? -P.slope[q >> 1] : P.slope[q >> 1];
    }
    if (y >= R.V) coef = __uint_as_float(kNan);
    if (y < 0) coef = 0.f;
    write_gradient(R.x + row * R.ld, dx + row * dld, R.V, grad_of(shift_of(st.x, R.b), st.y, coef, y, R.b), R.b,
                   coef == 0.f || st.y == INFINITY, part, parts, Group<G>::tid(), G);
  }
  if (!g && blockIdx.x == 0) sum_pairs(P);
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
  double* partial = nullptr; // kMostBlocks
  uint32_t* ticket = nullptr;
  float* logp = nullptr;     // max_rows
  double* ratio = nullptr;   // max_rows
  float* slope = nullptr;    // max_pairs
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
//    900   12,000   6.6  7.7     7.0  9.2        4,000  12,000  23.4 16.9    33.4 35.9
//  1,300    8,192   6.7  7.3     8.2  8.4        8,192  16,384  53.4 49.1    75.2 86.2
constexpr int64_t kWarpStats = 32768, kWarpGrad = 18432;  // bytes of a row at most
bool by_warps(int64_t n, int64_t row_bytes, int64_t most) {
  return n >= 600 && row_bytes <= most && row_bytes <= 12 * n;
}
// Blocks of groups of G that do n rows.
template <int G>
int64_t blocks_for(int64_t n) {
  return (n + Group<G>::kRows - 1) / Group<G>::kRows;
}

template <bool kRatio, typename T>
cudaError_t launch_stats(const Rows<T>& R, float* logp, float2* stats, const float* ref, double* ratio, cudaStream_t s) {
  const int64_t bytes = R.V * (int64_t)sizeof(T);
  if (by_warps(R.n, bytes, kWarpStats))
    return launch(k_stats<T, 32, kRatio>, blocks_for<32>(R.n), kLossThreads, 1, s, R, logp, stats, ref, ratio, 1);
  return with_parts(parts_for(R.n, bytes), [&](int parts) {
    return launch(k_stats<T, kLossThreads, kRatio>, R.n * parts, kLossThreads, parts, s, R, logp, stats, ref, ratio, parts);
  });
}
// A warp a pair where that is two reads a thread or so: 10,000 pairs of single rows of 512
// logits 114 -> 53 us; one pair of 30,000 rows 160 us by a warp, 72 by a block.
cudaError_t launch_pairs(const PairArgs& P, bool total, cudaStream_t s) {
  if (P.pairs > 0 && P.n / P.pairs <= 64)
    return launch(k_pairs<32>, blocks_for<32>(P.pairs), kLossThreads, 1, s, P, total);
  return launch(k_pairs<kLossThreads>, P.pairs ? P.pairs : 1, kLossThreads, 1, s, P, total);
}
template <typename T>
cudaError_t launch_grad(const Rows<T>& R, const float2* stats, const float* g, const PairArgs& P, T* dx, int64_t dld,
                        cudaStream_t s) {
  const int64_t bytes = R.V * (int64_t)sizeof(T);
  if (by_warps(R.n, bytes, kWarpGrad))
    return launch(k_grad<T, 32>, blocks_for<32>(R.n), kLossThreads, 1, s, R, stats, g, P, dx, dld, 1);
  // pieces of up to 56 KB (they need no cluster): the last blocks end together. 4,096 rows of
  // 50,257 fp32 248 us whole, 239 in pieces of 50 KB, 269 of 13; 1,024 rows 73, 65 and 71; 300 of
  // 50,257 bf16 8.3 in pieces of 50 KB, 9.1 of 25.
  int parts = parts_for(R.n, bytes);
  while (bytes / parts > 57344) parts *= 2;
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
    return launch_stats<false>(rows_of<T>(logits_dev, n, vocab, ld, scale, targets_dev), logp_dev,
                               reinterpret_cast<float2*>(stats_dev), (const float*)nullptr, (double*)nullptr,
                               static_cast<cudaStream_t>(stream));
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
      8 * (size_t)(kMostBlocks + 1 + max_pairs + 2 * max_rows) + 4 * (size_t)(max_rows + max_pairs);
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
  h->ticket = reinterpret_cast<uint32_t*>(h->partial + kMostBlocks);
  h->wloss = h->partial + kMostBlocks + 1;
  h->stats = reinterpret_cast<float2*>(h->wloss + max_pairs);
  h->ratio = reinterpret_cast<double*>(h->stats + max_rows);
  h->logp = reinterpret_cast<float*>(h->ratio + max_rows);
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
                   loss_dev, pair_loss_dev, seq_ratio_dev, h->slope, h->wloss, h->ticket};
  const bool grad = n > 0 && dlogits_dev;
  cudaError_t err = by_type(dtype, [&](auto t) {
    using T = decltype(t);
    const Rows<T> R = rows_of<T>(logits_dev, n, vocab, ld, scale, targets_dev);
    cudaError_t e = n ? launch_stats<true>(R, logp, h->stats, ref_logp_dev, h->ratio, s) : cudaSuccess;
    if (e == cudaSuccess && (pairs || !grad)) e = launch_pairs(P, !grad, s);
    if (e != cudaSuccess || !grad) return e;
    return launch_grad(R, (const float2*)h->stats, (const float*)nullptr, P, static_cast<T*>(dlogits_dev), dld, s);
  });
  return done(err);
}

}  // extern "C"
