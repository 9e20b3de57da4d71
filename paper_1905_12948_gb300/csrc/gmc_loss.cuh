// Device-side definitions shared by the loss kernels: rows of logits, exponents,
// the running maximum and sum of a row, its log-probability, and its gradient.
//
// For a row x of V logits, a scale s (1 / temperature) and a target y:
//   m = max x,  S = sum_v exp(s (x_v - m)),  logp = s (x_y - m) - log S,
//   d logp / d x_v = s ([v = y] - p_v),  p_v = exp(s (x_v - m) - log S).
// A row whose logits are all -inf has no distribution: S = 0, logp = -inf, and
// it adds nothing to a loss or a gradient.
#pragma once

#include <cmath>

#include "gmc_internal.h"
#include "gmc_vec.cuh"

namespace gmc {

constexpr int kLossThreads = 256;
constexpr int kSweepVecs = 2;  // 32-byte vectors that a thread of a sweep loads together
constexpr double kLog2e = 1.4426950408889634;
constexpr double kLn2 = 0.6931471805599453;
// By how much of itself ex2.approx is too small on the mean (measured: 4.9e-8 to 5.1e-8 over each
// binade of results; at most 1.4e-7). It is put back into log S, lest the rows of a
// sequence add it up.
constexpr double kExp2Low = 5e-8;
constexpr int kMaxParts = 8;  // blocks of a cluster that share a row (the portable limit)

// Exponents are formed to base 2, by s log2 e in two words c + lo (c its lower
// neighbour, so that lo > 0 and -inf stays -inf): a log sum is then off by roundings of
// either sign alone, and a sum over a sequence's rows stays as good as its rows.
struct Base {
  float scale, c, lo;
};
inline Base base_of(float scale) {
  const double b = (double)scale * kLog2e;
  float c = (float)b;
  if ((double)c >= b) c = std::nextafter(c, 0.f);
  return Base{scale, c, (float)(b - (double)c)};
}

// n rows of V logits, row r at x + r * ld, with the target of each.
template <typename T>
struct Rows {
  const T* x;
  int64_t n, V, ld;
  Base b;
  const int64_t* y;
};

// What is subtracted from a row's exponents: that of its maximum m, rounded up to a whole
// number, so that sums change from one shift to another by exact powers of two (2^x is
// 5e-8 low on the mean, kExp2Low, which a second one would double). x c - m c is one fused
// operation as long as m c is not so large that its rounding matters (masks of the type's
// lowest value in a whole row); then the difference x - m is taken first.
constexpr float kFar = 1048576.f;  // 2^20
struct Shift {
  float h, hc;  // m (0 where nothing but -inf was seen), and m c rounded up
  bool far;
};
__device__ __forceinline__ Shift shift_of(float m, const Base& b) {
  Shift s;
  s.h = m == -INFINITY ? 0.f : m;
  s.hc = ceilf(s.h * b.c);
  s.far = !(fabsf(s.hc) < kFar);
  return s;
}
// Exponent of x (of x - h, with 0 for hc, where the shift is far).
__device__ __forceinline__ float exponent(float x, float hc, const Base& b) {
  return __fmaf_rn(x, b.lo, __fmaf_rn(x, b.c, -hc));
}
// By how much the shift of a sum kept under its maximum m lies below s, in exponents. Either may be
// far or not: a sum under a far maximum is 2^0 at m itself, any other at m c rounded up. For logits
// of 16 bits one rule does: two maxima on either side of 2^20 are 2^9 exponents apart, and
// the lower one's sum is nothing. (Policy loss, fp32, 1,024 x 128,256: 156 us, 151 by that rule; bf16,
// 8,192 x 131,072: 603, 608 by both.)
template <typename T>
__device__ __forceinline__ float between(float m, const Shift& s, const Base& b) {
  const float hc = ceilf(m * b.c);
  if constexpr (sizeof(T) == 4) {
    const bool far = !(fabsf(hc) < kFar);
    if (s.far) return far ? (m - s.h) * b.c : __fmaf_rn(-s.h, b.c, hc) - s.h * b.lo;
    return far ? exponent(m, s.hc, b) : hc - s.hc;
  } else {
    return s.far ? (m - s.h) * b.c : hc - s.hc;
  }
}

// A maximum and the sum of the exponentials below its shift. m = -inf: nothing yet.
struct alignas(8) MaxSum {  // one 8-byte message
  float m = -INFINITY, s = 0.f;
};
template <typename T>
__device__ __forceinline__ MaxSum merge(const MaxSum& a, const MaxSum& o, const Base& b) {
  MaxSum r;
  r.m = fmaxf(a.m, o.m);
  const Shift h = shift_of(r.m, b);
  r.s = a.s * exp2_fast(between<T>(a.m, h, b)) + o.s * exp2_fast(between<T>(o.m, h, b));
  return r;
}
// One value into a, and U vectors. Sums are kept four to a thread, and no NaN hides in a
// maximum's shadow: its exponential is NaN.
template <typename T>
__device__ __forceinline__ void add_one(MaxSum* a, float x, const Base& b) {
  const float m = fmaxf(a->m, x);
  const Shift h = shift_of(m, b);
  const float e = h.far ? exponent(x - h.h, 0.f, b) : exponent(x, h.hc, b);
  a->s = a->s * exp2_fast(between<T>(a->m, h, b)) + exp2_fast(e);
  a->m = m;
}
template <typename T, int U>
__device__ __forceinline__ void add(MaxSum* a, const uint4 (&v)[U], const Base& b) {
  constexpr int P = Vec<T>::N / 2;
  uint32_t top = Vec<T>::top(Vec<T>::top(v[0].x, v[0].y), Vec<T>::top(v[0].z, v[0].w));
#pragma unroll
  for (int u = 1; u < U; ++u)
    top = Vec<T>::top(top, Vec<T>::top(Vec<T>::top(v[u].x, v[u].y), Vec<T>::top(v[u].z, v[u].w)));
  const float m = fmaxf(a->m, Vec<T>::top_of(top));
  const Shift h = shift_of(m, b);
  const Pair c = pair_of(b.c, b.c), lo = pair_of(b.lo, b.lo), hc = pair_of(-h.hc, -h.hc);
  Pair s0 = pair_of(a->s * exp2_fast(between<T>(a->m, h, b)), 0.f), s1 = pair_of(0.f, 0.f);
  if (!h.far) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      Pair x[P];
      Vec<T>::pairs(v[u], x);
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const Pair e = exp2_pair(fma_pair(x[i], lo, fma_pair(x[i], c, hc)));
        if (i & 1) s1 = add_pair(s1, e);
        else s0 = add_pair(s0, e);
      }
    }
  } else {
    const Pair sh = pair_of(-h.h, -h.h), none = pair_of(0.f, 0.f);
#pragma unroll 1
    for (int u = 0; u < U; ++u) {
      Pair x[P];
      uint4 w = v[0];
#pragma unroll
      for (int i = 1; i < U; ++i)
        if (u == i) w = v[i];
      Vec<T>::pairs(w, x);
#pragma unroll
      for (int i = 0; i < P; ++i) {
        x[i] = add_pair(x[i], sh);
        s0 = add_pair(s0, exp2_pair(fma_pair(x[i], lo, fma_pair(x[i], c, none))));
      }
    }
  }
  float s[4];
  split(s0, s, s + 1);
  split(s1, s + 2, s + 3);
  a->s = (s[0] + s[1]) + (s[2] + s[3]);
  a->m = m;
}
// Over a warp; every lane returns the result.
template <typename T>
__device__ __forceinline__ MaxSum warp_merge(MaxSum a, const Base& b) {
  MaxSum r;
  r.m = a.m;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) r.m = fmaxf(r.m, __shfl_xor_sync(0xffffffffu, r.m, o));
  r.s = warp_sum(a.s * exp2_fast(between<T>(a.m, shift_of(r.m, b), b)));
  return r;
}
// Over the block; every thread returns the result. ws: 32 entries of shared memory.
template <typename T>
__device__ __forceinline__ MaxSum block_merge(MaxSum a, const Base& b, MaxSum* ws) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  a = warp_merge<T>(a, b);
  if (lane == 0) ws[warp] = a;
  __syncthreads();
  return warp_merge<T>(lane < warps ? ws[lane] : MaxSum(), b);
}
// Counts that tell the last of several blocks: what a block (or a warp) wrote before it
// counts is visible to the one that is told it is the last.
__device__ __forceinline__ uint32_t count_inc(uint32_t* p, uint32_t last) {  // back to 0 after `last`
  uint32_t before;
  asm volatile("atom.acq_rel.gpu.global.inc.u32 %0, [%1], %2;" : "=r"(before) : "l"(p), "r"(last) : "memory");
  return before;
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// Over the blocks of a cluster, in rank order: a is the block's, the same in all its
// threads. The caller has passed the cluster's barrier once before, so that none
// writes into a block that has not begun.
template <typename T>
__device__ __forceinline__ MaxSum cluster_merge(MaxSum a, int parts, const Base& b, MaxSum* ws) {
  if (parts == 1) return a;
  if (threadIdx.x < (unsigned)parts) {  // into slot `rank` of every block
    const uint32_t here = (uint32_t)__cvta_generic_to_shared(ws + cluster_rank());
    uint32_t there;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(here), "r"(threadIdx.x));
    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(there), "f"(a.m), "f"(a.s) : "memory");
  }
  cluster_arrive();
  cluster_wait();
  MaxSum r = ws[0];
  for (int i = 1; i < parts; ++i) r = merge<T>(r, ws[i], b);
  return r;
}

// One group's share (`part` of `parts`) of a row's maximum and sum, thread `tid` of
// `threads`: the row's 32-byte vectors, U at a time a thread, and its edges by a few threads of
// part 0.
template <typename T>
__device__ __forceinline__ MaxSum sweep(const T* x, int64_t V, const Base& b, int part, int parts, int tid, int threads) {
  constexpr int N = Wide<T>::N, U = kSweepVecs;
  MaxSum a;
  const int head = wide_head(x, V);
  const int64_t nv = (V - head) / N;
  const int tail = (int)(V - head - nv * N);
  const T* q = x + head;
  const int64_t per = (nv + parts - 1) / parts;
  const int64_t lo = per * part, hi = lo + per < nv ? lo + per : nv;
  for (int64_t i0 = lo + tid; i0 < hi; i0 += U * threads) {
    uint4 v[2 * U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t i = i0 + u * threads;
      v[2 * u] = v[2 * u + 1] = make_uint4(Vec<T>::kLow, Vec<T>::kLow, Vec<T>::kLow, Vec<T>::kLow);
      if (i < hi) {
        const Wide<T> w = load_wide(q + i * N, true);
        v[2 * u] = w.a;
        v[2 * u + 1] = w.b;
      }
    }
    add<T>(&a, v, b);
  }
  if (part == 0 && tid < head + tail)
    add_one<T>(&a, Vec<T>::one(x[tid < head ? (int64_t)tid : V - tail + (tid - head)]), b);
  return a;
}

// What follows from a row's maximum and sum.
struct RowStats {
  Shift h;
  float ls, logp;  // log of the sum (0 for an empty row), log-probability of the target
  float low;       // what logp's rounding took away
  bool empty;
};
// s x_y - (hc log 2 + log S): the shift counts, not the maximum.
__device__ __forceinline__ float logp_of(float xy, const Shift& h, float ls, const Base& b) {
  return h.far ? (xy - h.h) * b.scale - ls
               : (float)((double)xy * (double)b.scale - ((double)h.hc * kLn2 + ((double)ls + kExp2Low)));
}
// (A row's logp is formed from log S in two parts, the power of two and the rest: the sum
// is then rounded once, at logp's own last place, and to either side alike.)
__device__ __forceinline__ RowStats finish(const MaxSum& a, float xy, const Base& b) {
  RowStats r;
  r.h = shift_of(a.m, b);
  r.empty = a.m == -INFINITY && a.s == 0.f && xy == xy;  // a target outside the vocabulary marks this row too
  r.ls = r.empty ? 0.f : logf(a.s);
  r.low = 0.f;
  if (r.h.far || r.empty) {
    r.logp = logp_of(xy, r.h, r.ls, b);
  } else {
    const uint32_t bits = __float_as_uint(a.s);  // at least 1/2, the maximum's own term, or NaN (0: xy is NaN)
    const float power = (float)((int)(bits >> 23) - 127);
    const float rest = logf(__uint_as_float((bits & 0x007fffffu) | 0x3f800000u));
    const double full =
        (double)xy * (double)b.scale - ((double)(r.h.hc + power) * kLn2 + ((double)rest + kExp2Low));
    r.logp = a.s != a.s ? a.s : (float)full;
    if (fabsf(r.logp) < INFINITY) r.low = (float)(full - (double)r.logp);
  }
  return r;
}
constexpr uint32_t kNan = 0x7fffffffu;
// The target's logit; NaN for one outside the vocabulary.
template <typename T>
__device__ __forceinline__ float target_logit(const T* x, int64_t V, int64_t y) {
  return y < V ? Vec<T>::one(x[y]) : __uint_as_float(kNan);
}

// A row's gradient k ([v = y] - p_v), k = coef s, from its shift and log S.
struct RowGrad {
  Shift h;
  float k, f, ls;  // f = -k / S
  int64_t y;
};
__device__ __forceinline__ RowGrad grad_of(const Shift& h, float ls, float coef, int64_t y, const Base& b) {
  const float k = coef * b.scale;
  return RowGrad{h, k, -k * expf(-ls), ls, y};
}
// 1 - p_y without cancellation.
__device__ __forceinline__ float grad_at_target(float x, const RowGrad& g, const Base& b) {
  return g.k * -expm1f(logp_of(x, g.h, g.ls, b));
}
// A vector's logits to their gradients (the target's as any other's).
template <typename T>
__device__ __forceinline__ uint4 grad_vec(const uint4& v, const RowGrad& g, const Base& b) {
  constexpr int P = Vec<T>::N / 2;
  const float h = g.h.far ? -g.h.h : 0.f, hc = g.h.far ? 0.f : -g.h.hc;
  const Pair sh = pair_of(h, h), by = pair_of(g.f, g.f), c = pair_of(b.c, b.c), lo = pair_of(b.lo, b.lo),
             off = pair_of(hc, hc);
  Pair x[P];
  Vec<T>::pairs(v, x);
#pragma unroll
  for (int i = 0; i < P; ++i) {
    x[i] = add_pair(x[i], sh);
    x[i] = mul_pair(by, exp2_pair(fma_pair(x[i], lo, fma_pair(x[i], c, off))));
  }
  return Vec<T>::put_pairs(x);
}

// A share (`part` of `parts`) of a row's gradient, or of zeros (skip: x is not read, it may
// hold anything), by thread `tid` of `threads`: 32-byte loads, kSweepVecs at a time, and, where
// the output row lies at the same offset from a 32-byte boundary, stores.
template <typename T>
__device__ __forceinline__ void write_gradient(const T* x, T* dx, int64_t V, const RowGrad& g, const Base& b, bool skip,
                                               int64_t part, int64_t parts, int tid, int threads) {
  constexpr int N = Wide<T>::N, U = kSweepVecs;
  const int head = wide_head(x, V);
  const int64_t nv = (V - head) / N;
  const int tail = (int)(V - head - nv * N);
  const bool same = ((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(dx)) & 31) == 0;
  const int64_t per = (nv + parts - 1) / parts;
  const int64_t lo = per * part, hi = lo + per < nv ? lo + per : nv;
  const int64_t vy = g.y >= head ? (g.y - head) / N : -1;  // the target's vector (none of [lo, hi) where it is at an edge)
  for (int64_t i0 = lo + tid; i0 < hi; i0 += U * threads) {
    Wide<T> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t i = i0 + u * threads;
      v[u].a = v[u].b = make_uint4(0, 0, 0, 0);
      if (!skip && i < hi) v[u] = load_wide(x + head + i * N, true);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t i = i0 + u * threads;
      if (i >= hi) continue;
      T* to = dx + head + i * N;
      // (x may be dx: the target's logit is taken before its place is written)
      const float fy = !skip && i == vy ? grad_at_target(Vec<T>::one(x[g.y]), g, b) : 0.f;
      if (!skip) {
        v[u].a = grad_vec<T>(v[u].a, g, b);
        v[u].b = grad_vec<T>(v[u].b, g, b);
      }
      store_wide(to, v[u], same);
      if (!skip && i == vy) dx[g.y] = Vec<T>::round(fy);
    }
  }
  if (part == 0 && tid < head + tail) {
    const int64_t j = tid < head ? (int64_t)tid : V - tail + (tid - head);
    float f = 0.f;
    if (!skip) {
      const float v = Vec<T>::one(x[j]);
      f = j == g.y ? grad_at_target(v, g, b)
                   : g.f * exp2_fast(g.h.far ? exponent(v - g.h.h, 0.f, b) : exponent(v, g.h.hc, b));
    }
    dx[j] = Vec<T>::round(f);
  }
}

struct PolicyArgs {
  const float *old_logp, *ref_logp, *adv, *weights;  // ref_logp NULL: no KL term
  float clip_low, clip_high, kl, weight;  // weight: of every row, where weights is NULL
  float *token_loss, *logp;               // either may be NULL
  float* loss;
  double* partial;                        // the blocks' sums of weighted losses
  uint32_t* ticket;                       // counts the blocks that are done; 0 between calls
  uint64_t wait_ns;                       // bound of the waits on mbarriers
  int64_t hold_row;                       // test hook: no copy of this row is made; -1: none
};

// exp(d) - 1 - d, its slope expm1(d) given. Where d is small the difference cancels (at 1e-3 to 1e-4 of
// itself): below 1/2 it is d^2 sum_n d^n / (n + 2)!, whose terms from n = 8 on are below 2^-28 of the sum.
__device__ __forceinline__ float kl_term(float d, float slope) {
  if (!(fabsf(d) < 0.5f)) return slope - d;
  float s = 1.f / 362880.f;
  s = __fmaf_rn(s, d, 1.f / 40320.f);
  s = __fmaf_rn(s, d, 1.f / 5040.f);
  s = __fmaf_rn(s, d, 1.f / 720.f);
  s = __fmaf_rn(s, d, 1.f / 120.f);
  s = __fmaf_rn(s, d, 1.f / 24.f);
  s = __fmaf_rn(s, d, 1.f / 6.f);
  s = __fmaf_rn(s, d, 0.5f);
  return d * d * s;
}
// The token's loss and its slope in logp.
__device__ __forceinline__ void policy_terms(const PolicyArgs& P, float adv, float old_logp, float ref_logp, float logp,
                                             float* loss, float* slope) {
  const float ratio = expf(logp - old_logp);
  const float plain = ratio * adv;
  const float lo = 1.f - P.clip_low, hi = 1.f + P.clip_high;
  const float clipped = (ratio < lo ? lo : ratio > hi ? hi : ratio) * adv;  // NaN stays NaN
  float l = plain <= clipped ? -plain : -clipped;
  float d = plain <= clipped ? -plain : 0.f;
  if (P.ref_logp) {
    const float off = ref_logp - logp, up = expm1f(off);
    l += P.kl * kl_term(off, up);
    d -= P.kl * up;
  }
  if (l != l) d = l;
  *loss = l;
  *slope = d;
}

// Launch a kernel of `blocks` blocks in clusters of `parts`, with programmatic stream
// serialization (it begins with griddep_wait).
struct LaunchConfig {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute at[2];
  LaunchConfig(int64_t blocks, int threads, int parts, size_t smem, cudaStream_t s) {
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)parts;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = parts > 1 ? 2 : 1;
  }
};
template <typename... A, typename... B>
inline cudaError_t launch(void (*f)(A...), int64_t blocks, int threads, int parts, cudaStream_t s, B... args) {
  if (parts > 1 && refuse_cooperative()) return cudaErrorCooperativeLaunchTooLarge;
  LaunchConfig l(blocks, threads, parts, 0, s);
  return cudaLaunchKernelEx(&l.cfg, f, args...);
}
// f(parts), or f(1) where the context (an MPS share, a partitioned GPU) cannot hold clusters of
// that many blocks.
template <typename F>
inline cudaError_t with_parts(int parts, F&& f) {
  cudaError_t err = f(parts);
  if (parts > 1 && too_large_here(err)) {
    cudaGetLastError();  // this launch's
    err = f(1);
  }
  return err;
}

// Blocks that share a row: enough of them for two a SM, down to 16 KB of it each.
inline int parts_for(int64_t n, int64_t row_bytes) {
  int parts = 1;
  while (parts < kMaxParts && n * parts < 304 && row_bytes / parts > 16384) parts *= 2;
  return parts;
}

// Facts of a handle's device: its SMs, and the clusters of a launch configuration that can
// be resident, looked up once (with what the kernel needs set).
struct Residency {
  int sms = 1;
  struct {
    const void* f = nullptr;
    int threads = 0, parts = 0, clusters = 0;
    size_t smem = 0;
  } known[32];
  int next = 0;
  cudaError_t clusters(const void* f, const LaunchConfig& l, int parts, int64_t* out);
};

// The policy loss over n > 0 rows (gmc_policy.cu). A.partial has kMostBlocks slots.
constexpr int kMostBlocks = 8192;
template <typename T>
cudaError_t launch_policy(const Rows<T>& R, const PolicyArgs& A, T* dx, int64_t dld, Residency* device, cudaStream_t s);
}  // namespace gmc
