// Scores of token rows: log-probabilities of given tokens, the entropy and the top
// alternatives of each row, and the gradient of the first two in the logits.
//
// For a row x of V logits and a scale s, with the running maximum m and sum S of
// gmc_loss.cuh, exponents e_v = log2 exp(s x_v) less the row's shift, and T = sum_v e_v 2^e_v:
//   lp_v = e_v log 2 - log S,  p_v = 2^e_v / S,
//   H = -sum_v p_v lp_v = log S - log 2 T / S,
//   d/dx_v (sum_j g_j lp_{y_j} + h H) = s (sum_{j: y_j = v} g_j - p_v (G + h (lp_v + H))),  G = sum_j g_j.
// Where a sum moves to a shift that is d exponents higher, S becomes S 2^-d, T (T - d S) 2^-d:
// one pass over the row, whatever order its parts are merged in.
#include <cfloat>
#include <cmath>

#include "gmc.h"
#include "gmc_loss.cuh"

using namespace gmc;

namespace {

constexpr int kMostGiven = 64, kMostTop = 64;
constexpr int kHeld = kLossThreads;  // candidates of a block

// A maximum and the two sums under its shift. m = -inf: nothing yet.
struct alignas(16) Moments {
  float m = -INFINITY, s = 0.f, t = 0.f, none = 0.f;
};
// Where 2^e is 0 (a logit of -inf, a sum that is too low to matter) e may be -inf, and e 2^e is not
// a number; below 2^-126 the exponential is 0. (NaN passes through the exponential itself.)
__device__ __forceinline__ float low(float e) { return fmaxf(e, -256.f); }

template <typename T>
__device__ __forceinline__ void move(Moments* a, const Shift& to, const Base& b) {
  const float d = between<T>(a->m, to, b), f = exp2_fast(d);
  a->t = (a->t + low(d) * a->s) * f;
  a->s *= f;
}
template <typename T>
__device__ __forceinline__ Moments merge(Moments a, Moments o, const Base& b) {
  const float m = fmaxf(a.m, o.m);
  const Shift h = shift_of(m, b);
  move<T>(&a, h, b);
  move<T>(&o, h, b);
  Moments r;
  r.m = m;
  r.s = a.s + o.s;
  r.t = a.t + o.t;
  return r;
}
template <typename T>
__device__ __forceinline__ void add_one(Moments* a, float x, const Base& b) {
  const float m = fmaxf(a->m, x);
  const Shift h = shift_of(m, b);
  move<T>(a, h, b);
  const float e = h.far ? exponent(x - h.h, 0.f, b) : exponent(x, h.hc, b), p = exp2_fast(e);
  a->s += p;
  a->t = __fmaf_rn(low(e), p, a->t);
  a->m = m;
}
// U vectors whose largest value is `top`.
template <typename T, int U>
__device__ __forceinline__ void add(Moments* a, const uint4 (&v)[U], float top, const Base& b) {
  constexpr int P = Vec<T>::N / 2;
  const float m = fmaxf(a->m, top);
  const Shift h = shift_of(m, b);
  move<T>(a, h, b);
  a->m = m;
  const float sh = h.far ? -h.h : 0.f, off = h.far ? 0.f : -h.hc;
  const Pair by = pair_of(sh, sh), c = pair_of(b.c, b.c), lo = pair_of(b.lo, b.lo), hc = pair_of(off, off);
  Pair s = pair_of(a->s, 0.f), t = pair_of(a->t, 0.f);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    Pair x[P];
    Vec<T>::pairs(v[u], x);
#pragma unroll
    for (int i = 0; i < P; ++i) {
      if (h.far) x[i] = add_pair(x[i], by);
      const Pair e = fma_pair(x[i], lo, fma_pair(x[i], c, hc)), p = exp2_pair(e);
      float e0, e1;
      split(e, &e0, &e1);
      s = add_pair(s, p);
      t = fma_pair(pair_of(low(e0), low(e1)), p, t);
    }
  }
  float s0, s1;
  split(s, &s0, &s1);
  a->s = s0 + s1;
  split(t, &s0, &s1);
  a->t = s0 + s1;
}
template <typename T>
__device__ __forceinline__ float largest(const uint4& v) {
  return Vec<T>::top_of(Vec<T>::top(Vec<T>::top(v.x, v.y), Vec<T>::top(v.z, v.w)));
}
template <typename T>
__device__ __forceinline__ Moments warp_merge(Moments a, const Base& b) {
  float m = a.m;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  move<T>(&a, shift_of(m, b), b);
  Moments r;
  r.m = m;
  r.s = warp_sum(a.s);
  r.t = warp_sum(a.t);
  return r;
}
template <typename T>
__device__ __forceinline__ Moments block_merge(Moments a, const Base& b, Moments* ws) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  a = warp_merge<T>(a, b);
  if (lane == 0) ws[warp] = a;
  __syncthreads();
  return warp_merge<T>(lane < warps ? ws[lane] : Moments(), b);
}

// A logit and its place as one number: larger logits first, and lower places among equal ones
// (zeros of either sign are equal; any NaN is above all). No key is 0.
__device__ __forceinline__ uint64_t key_of(float x, int64_t at) {
  uint32_t u = __float_as_uint(x + 0.f);
  u = x != x ? 0xffffffffu : (u & 0x80000000u) ? ~u : u | 0x80000000u;
  return (uint64_t)u << 32 | (uint32_t)~(uint32_t)at;
}
__device__ __forceinline__ float value_of(uint64_t key) {
  const uint32_t u = (uint32_t)(key >> 32);
  return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ int64_t place_of(uint64_t key) { return (int64_t)(uint32_t)~(uint32_t)key; }

// The best `top` keys seen by a block: an unordered list that takes every key above the
// last bound, cut back to its best whenever it is half full.
struct Held {
  uint64_t key[kHeld];
  uint64_t bound;        // no key at or below it is among the best
  int n;
};
// All threads: the list's best `top`, in order, and the bound that follows.
__device__ __forceinline__ void cut(Held* H, int top) {
  __syncthreads();
  const int n = H->n < kHeld ? H->n : kHeld, tid = (int)threadIdx.x;
  const uint64_t mine = tid < n ? H->key[tid] : 0;
  int rank = 0;
  if (tid < n)
    for (int i = 0; i < n; ++i) rank += H->key[i] > mine;
  __syncthreads();
  if (tid < n && rank < top) H->key[rank] = mine;
  if (tid == 0) H->n = n < top ? n : top;
  if (tid < n && rank == top - 1) H->bound = mine;
  __syncthreads();
}
// Into the list; the place that the key got (kHeld or more: none, before the next cut).
__device__ __forceinline__ int offer(Held* H, uint64_t key) {
  const int at = atomicAdd(&H->n, 1);
  if (at < kHeld) H->key[at] = key;
  return at;
}

struct ScoreArgs {
  const int64_t* y;  // n x given
  int given, top;
  float *logp, *entropy, *top_logp;
  int64_t* top_index;
  float4* stats;     // shift, log S, H
};

// Whether a row counts: one of its given tokens is not negative, or none is asked for. By each warp.
__device__ __forceinline__ bool counts(const int64_t* y, int given) {
  if (given == 0) return true;
  const int lane = (int)threadIdx.x & 31;
  bool some = false;
  for (int j = lane; j < given; j += 32) some |= y[j] >= 0;
  return __any_sync(0xffffffffu, some);
}

// A row by a block. Bound by memory.
template <typename T, bool kTop>
__global__ void __launch_bounds__(kLossThreads) k_scores(Rows<T> R, ScoreArgs A) {
  constexpr int N = Wide<T>::N, U = kSweepVecs, M = Vec<T>::N;
  __shared__ Moments ws[32];
  __shared__ Held H;
  __shared__ float first[kLossThreads];
  griddep_wait();
  const int64_t row = blockIdx.x;
  const int tid = (int)threadIdx.x;
  const int64_t* y = A.y + row * A.given;
  if (!counts(y, A.given)) {
    if (tid < A.given && A.logp) A.logp[row * A.given + tid] = 0.f;
    if (tid < A.top) A.top_logp[row * A.top + tid] = 0.f, A.top_index[row * A.top + tid] = -1;
    if (tid == 0 && A.entropy) A.entropy[row] = 0.f;
    if (tid == 0 && A.stats) A.stats[row] = make_float4(0.f, 0.f, 0.f, 0.f);
    return;
  }
  const T* x = R.x + row * R.ld;
  const int64_t V = R.V;
  const int64_t yj = tid < A.given ? y[tid] : -1;
  const float xy = yj >= 0 ? target_logit(x, V, yj) : 0.f;

  const int head = wide_head(x, V);
  const int64_t nv = (V - head) / N;
  const int tail = (int)(V - head - nv * N);
  const T* q = x + head;
  Moments a;
  if (kTop && tid == 0) H.n = 0, H.bound = 0;
  uint64_t edge = 0;  // the row's ends, by a few threads
  if (tid < head + tail) {
    const int64_t i = tid < head ? (int64_t)tid : V - tail + (tid - head);
    const float v = Vec<T>::one(x[i]);
    add_one<T>(&a, v, R.b);
    edge = key_of(v, i);
  }
  for (int64_t i0 = tid, block0 = 0; block0 < nv || (kTop && block0 == 0); i0 += U * kLossThreads, block0 += U * kLossThreads) {
    float top = -INFINITY;
    {
      uint4 v[2 * U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t i = i0 + u * kLossThreads;
        v[2 * u] = v[2 * u + 1] = make_uint4(Vec<T>::kLow, Vec<T>::kLow, Vec<T>::kLow, Vec<T>::kLow);
        if (i < nv) {
          const Wide<T> w = load_wide(q + i * N, true);
          v[2 * u] = w.a;
          v[2 * u + 1] = w.b;
        }
      }
#pragma unroll
      for (int u = 0; u < 2 * U; ++u) top = fmaxf(top, largest<T>(v[u]));
      add<T>(&a, v, top, R.b);
    }
    if constexpr (kTop) {
      if (block0 == 0) {
        // Of the threads' largest values the top-th is a bound from below: so many are not less.
        first[tid] = top;
        __syncthreads();
        int above = 0;
        for (int i = 0; i < kLossThreads; ++i) above += first[i] > top || (first[i] == top && i < tid);
        if (above == A.top - 1 && top > -INFINITY) H.bound = (key_of(top, 0) >> 32 << 32) - 1;
        __syncthreads();
      }
      int done = 0;  // so many elements of this thread are in the list
      for (bool again = true; again;) {
        const uint64_t bound = H.bound;
        const float least = bound ? value_of(bound) : -INFINITY;
        bool full = false, left = false;
        if (edge > bound) {
          const int at = offer(&H, edge);
          full = at >= kHeld / 2;
          left = at >= kHeld;
          if (!left) edge = 0;
        }
        if (top >= least) {  // (rare: these vectors are read a second time)
#pragma unroll 1
          for (int u = 0; u < 2 * U; ++u) {
            const int64_t vec = i0 + u / 2 * kLossThreads;
            if (vec >= nv || done >= (u + 1) * M || left) continue;
            const int64_t at0 = head + vec * N + (u & 1) * M;
            const uint4 w = *reinterpret_cast<const uint4*>(x + at0);
            if (!(largest<T>(w) >= least)) continue;
            float f[M];
            Vec<T>::get(w, f);
#pragma unroll
            for (int i = 0; i < M; ++i)
              if (f[i] >= least && !left && done <= u * M + i) {
                const uint64_t key = key_of(f[i], at0 + i);
                if (key > bound) {
                  const int at = offer(&H, key);
                  full |= at >= kHeld / 2;
                  left = at >= kHeld;
                  if (!left) done = u * M + i + 1;
                }
              }
          }
        }
        again = __syncthreads_or(full);
        if (again) cut(&H, A.top);
      }
    }
  }
  a = block_merge<T>(a, R.b, ws);
  const MaxSum ms{a.m, a.s};
  if (tid < A.given && A.logp) A.logp[row * A.given + tid] = yj >= 0 ? finish(ms, xy, R.b).logp : 0.f;
  if (kTop) {
    cut(&H, A.top);
    if (tid < A.top) {
      const uint64_t key = H.key[tid];
      A.top_logp[row * A.top + tid] = finish(ms, value_of(key), R.b).logp;
      A.top_index[row * A.top + tid] = a.s != a.s ? -1 : place_of(key);
    }
  }
  if (tid == 0) {
    const RowStats r = finish(ms, 0.f, R.b);
    float h = r.empty ? 0.f : (float)((double)r.ls - kLn2 * ((double)a.t / (double)a.s));
    h = h < 0.f ? 0.f : h;  // (kExp2Low of S is left: a row of one token has no entropy)
    if (A.entropy) A.entropy[row] = h;
    if (A.stats) A.stats[row] = make_float4(r.h.h, r.empty ? INFINITY : r.ls, h, 0.f);
  }
}

// What a row's gradient is made of, in exponents: p_v (G + h (lp_v + H)) s = 2^e (c0 + c1 e).
struct ScoreGrad {
  Shift h;
  float c0, c1;
};
template <typename T>
__device__ __forceinline__ uint4 grad_vec(const uint4& v, const ScoreGrad& g, const Base& b) {
  constexpr int P = Vec<T>::N / 2;
  const float sh = g.h.far ? -g.h.h : 0.f, hc = g.h.far ? 0.f : -g.h.hc;
  const Pair by = pair_of(sh, sh), c = pair_of(b.c, b.c), lo = pair_of(b.lo, b.lo), off = pair_of(hc, hc),
             c0 = pair_of(g.c0, g.c0), c1 = pair_of(g.c1, g.c1);
  Pair x[P];
  Vec<T>::pairs(v, x);
#pragma unroll
  for (int i = 0; i < P; ++i) {
    x[i] = add_pair(x[i], by);
    const Pair e = fma_pair(x[i], lo, fma_pair(x[i], c, off));
    float e0, e1;
    split(e, &e0, &e1);
    x[i] = mul_pair(exp2_pair(e), fma_pair(pair_of(low(e0), low(e1)), c1, c0));
  }
  return Vec<T>::put_pairs(x);
}
template <typename T>
__device__ __forceinline__ float grad_one(float x, const ScoreGrad& g, const Base& b) {
  const float e = g.h.far ? exponent(x - g.h.h, 0.f, b) : exponent(x, g.h.hc, b);
  return exp2_fast(e) * __fmaf_rn(low(e), g.c1, g.c0);
}

// dx of a row, or a part of it, by a block. Bound by memory, read and written.
template <typename T>
__global__ void __launch_bounds__(kLossThreads, 6) k_scores_grad(Rows<T> R, int given, const float4* stats, const float* g,
                                                                 const float* dh, T* dx, int64_t dld, int parts) {
  constexpr int N = Wide<T>::N, U = kSweepVecs;
  __shared__ int64_t ys[kMostGiven];
  __shared__ float gs[kMostGiven];
  griddep_wait();
  // from the last row to the first: the logits read last are still in the L2 cache
  const int64_t row = R.n - 1 - blockIdx.x / parts;
  const int part = (int)(blockIdx.x % parts), tid = (int)threadIdx.x;
  const T* x = R.x + row * R.ld;
  T* out = dx + row * dld;
  const int64_t V = R.V;
  const int head = wide_head(x, V);
  const int64_t nv = (V - head) / N;
  const int tail = (int)(V - head - nv * N);
  const int64_t per = (nv + parts - 1) / parts;
  const int64_t lo = per * part < nv ? per * part : nv, hi = lo + per < nv ? lo + per : nv;

  const float4 st = stats[row];
  const bool counted = counts(R.y + row * given, given);
  bool wrong = false, any = false;
  if (tid < given) {
    const int64_t y = R.y[row * given + tid];
    ys[tid] = y;
    gs[tid] = y >= 0 && g ? g[row * given + tid] : 0.f;
    wrong = y >= V;
    any = y >= 0 && gs[tid] != 0.f;
  }
  wrong = __syncthreads_or(wrong);
  const float h = dh && counted ? dh[row] : 0.f;
  any = __syncthreads_or(any) || h != 0.f;
  const bool skip = !wrong && (!any || st.y == INFINITY);
  float G = 0.f;
  for (int j = 0; j < given; ++j) G += gs[j];
  if (wrong) G = __uint_as_float(kNan);
  const float k = -R.b.scale * expf(-st.y);
  const ScoreGrad q{shift_of(st.x, R.b), k * (G + h * (st.z - st.y)), k * h * (float)kLn2};

  // The given tokens in this part, taken before their places are written (out may be x):
  // g_y (1 - p_y) - p_y (G - g_y + h (lp_y + H)), the first without cancellation.
  float at_y = 0.f;
  bool mine = false;
  if (tid < given && !skip) {
    const int64_t y = ys[tid], v = y >= head ? (y - head) / N : -1;
    mine = y >= 0 && y < V && (y < head || v >= nv ? part == 0 : v >= lo && v < hi);
    float gy = 0.f;
    for (int j = 0; j < given; ++j) {
      if (ys[j] == y) gy += gs[j];
      if (j < tid && ys[j] == y) mine = false;
    }
    if (mine) {
      const float lp = logp_of(Vec<T>::one(x[y]), q.h, st.y, R.b);
      const float p = lp == -INFINITY ? 0.f : expf(lp), more = p == 0.f ? 0.f : p * (G - gy + h * (lp + st.z));
      at_y = R.b.scale * (gy * -expm1f(lp) - more);
      if (wrong) at_y = G;
    }
  }
  __syncthreads();
  const bool same = ((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(out)) & 31) == 0;
  for (int64_t i0 = lo + tid; i0 < hi; i0 += U * kLossThreads) {
    Wide<T> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t i = i0 + u * kLossThreads;
      v[u].a = v[u].b = make_uint4(0, 0, 0, 0);
      if (!skip && i < hi) v[u] = load_wide(x + head + i * N, true);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t i = i0 + u * kLossThreads;
      if (i >= hi) continue;
      if (!skip) {
        v[u].a = grad_vec<T>(v[u].a, q, R.b);
        v[u].b = grad_vec<T>(v[u].b, q, R.b);
      }
      store_wide(out + head + i * N, v[u], same);
    }
  }
  if (part == 0 && tid < head + tail) {
    const int64_t j = tid < head ? (int64_t)tid : V - tail + (tid - head);
    out[j] = Vec<T>::round(skip ? 0.f : grad_one<T>(Vec<T>::one(x[j]), q, R.b));
  }
  __syncthreads();
  if (mine) out[ys[tid]] = Vec<T>::round(at_y);
}

bool ok(const void* x, int32_t dtype, int64_t n, int64_t V, int64_t ld, float scale, const int64_t* y, int32_t given) {
  if (dtype != GMC_F32 && dtype != GMC_BF16 && dtype != GMC_F16) return false;
  const uintptr_t size = dtype == GMC_F32 ? 4 : 2;
  if (n < 0 || V < 1 || V >= (int64_t(1) << 31) || n > (int64_t(1) << 27)) return false;
  if (ld < V || ld > (int64_t(1) << 40) || given < 0 || given > kMostGiven) return false;
  if (!(scale >= 0x1p-64f && scale <= 0x1p64f)) return false;
  if (n == 0) return true;
  return x && (y || given == 0) && reinterpret_cast<uintptr_t>(x) % size == 0 && reinterpret_cast<uintptr_t>(y) % 8 == 0;
}
bool on_own(const void* p, uintptr_t size) { return reinterpret_cast<uintptr_t>(p) % size == 0; }

}  // namespace

extern "C" {

int gmc_token_scores(const void* logits_dev, int32_t dtype, int64_t n, int64_t vocab, int64_t ld, float scale,
                     const int64_t* targets_dev, int32_t given, int32_t top, float* logp_dev, float* entropy_dev,
                     float* top_logp_dev, int64_t* top_index_dev, float* stats_dev, void* stream) {
  if (!ok(logits_dev, dtype, n, vocab, ld, scale, targets_dev, given)) return GMC_EINVAL;
  if (top < 0 || top > kMostTop || top > vocab) return GMC_EINVAL;
  if (!on_own(logp_dev, 4) || !on_own(entropy_dev, 4) || !on_own(top_logp_dev, 4) || !on_own(top_index_dev, 8) || !on_own(stats_dev, 16))
    return GMC_EINVAL;
  if (n == 0) return GMC_OK;
  if (top > 0 && (!top_logp_dev || !top_index_dev)) return GMC_EINVAL;
  const cudaError_t err = by_type(dtype, [&](auto t) {
    using T = decltype(t);
    const Rows<T> R{static_cast<const T*>(logits_dev), n, vocab, ld, base_of(scale), targets_dev};
    const ScoreArgs A{targets_dev, given, top, logp_dev, entropy_dev, top_logp_dev, top_index_dev,
                      reinterpret_cast<float4*>(stats_dev)};
    return launch(top ? k_scores<T, true> : k_scores<T, false>, n, kLossThreads, 1, static_cast<cudaStream_t>(stream), R, A);
  });
  return err == cudaSuccess ? GMC_OK : GMC_ECUDA;
}

int gmc_token_scores_backward(const void* logits_dev, int32_t dtype, int64_t n, int64_t vocab, int64_t ld, float scale,
                              const int64_t* targets_dev, int32_t given, const float* stats_dev, const float* dlogp_dev,
                              const float* dentropy_dev, void* dlogits_dev, int64_t dld, void* stream) {
  if (!ok(logits_dev, dtype, n, vocab, ld, scale, targets_dev, given)) return GMC_EINVAL;
  if (dld < vocab || dld > (int64_t(1) << 40) || !on_own(dlogits_dev, dtype == GMC_F32 ? 4 : 2)) return GMC_EINVAL;
  if (dlogits_dev == logits_dev && dld != ld) return GMC_EINVAL;  // in place: the same rows
  if (!on_own(stats_dev, 16) || !on_own(dlogp_dev, 4) || !on_own(dentropy_dev, 4)) return GMC_EINVAL;
  if (n == 0) return GMC_OK;
  if (!stats_dev || !dlogits_dev) return GMC_EINVAL;
  const cudaError_t err = by_type(dtype, [&](auto t) {
    using T = decltype(t);
    const Rows<T> R{static_cast<const T*>(logits_dev), n, vocab, ld, base_of(scale), targets_dev};
    const int64_t bytes = vocab * (int64_t)sizeof(T);
    int parts = parts_for(n, bytes);
    while (bytes / parts > 57344) parts *= 2;
    return launch(k_scores_grad<T>, n * parts, kLossThreads, 1, static_cast<cudaStream_t>(stream), R, (int)given,
                  reinterpret_cast<const float4*>(stats_dev), dlogp_dev, dentropy_dev, static_cast<T*>(dlogits_dev), dld,
                  parts);
  });
  return err == cudaSuccess ? GMC_OK : GMC_ECUDA;
}

}  // extern "C"
