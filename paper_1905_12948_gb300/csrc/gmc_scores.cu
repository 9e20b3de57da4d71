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
constexpr int kBatches = 16;  // of a sweep, before its candidates are looked for

// Exponents to base 2 are x c less a shift, c the float next to scale log2 e: all of them, the given tokens' too, so that
// a log-probability is off by 2^-25 of itself, and no second word of c is wanted.
inline Base score_base(float scale) { return Base{scale, (float)((double)scale * kLog2e), 0.f}; }

// The threads that work on a row: a block of 256, of which up to 8 share a row as a cluster, a block of 128, or a
// warp, of which eight are a block.
template <int G>
struct Team {
  static_assert(G == 32 || G == 128 || G == kLossThreads, "a warp or a block");
  static constexpr int kThreads = G == 32 ? kLossThreads : G;  // of a block
  static constexpr int kRows = kThreads / G;                   // rows of a block
  __device__ static int tid() { return G == 32 ? (int)threadIdx.x % 32 : (int)threadIdx.x; }
  __device__ static int of_block() { return G == 32 ? (int)threadIdx.x / 32 : 0; }
  __device__ static void sync() {
    if constexpr (G == 32) __syncwarp();
    else __syncthreads();
  }
  // Also a barrier: what the team's threads wrote to shared memory before it is seen after it. (A warp's vote
  // alone orders no memory.)
  __device__ static bool any(bool p) {
    if constexpr (G == 32) {
      __syncwarp();
      return __any_sync(0xffffffffu, p);
    } else {
      return __syncthreads_or(p);
    }
  }
};

// What is summed below a shift: that of m, which is -inf where nothing has been seen, and at most
// kAbove exponents below the largest logit seen.
struct alignas(16) Moments {
  float m = -INFINITY, s = 0.f, t = 0.f, none = 0.f;
};
constexpr float kAbove = 8.f;
// Where 2^e is 0 (a logit of -inf, a sum that is too low to matter) e may be -inf, and e 2^e is not
// a number; below 2^-126 the exponential is 0. (NaN passes through the exponential itself.)
__device__ __forceinline__ float low(float e) { return fmaxf(e, -256.f); }

// By how much the shift of m lies below s, in exponents; as in gmc_loss.cuh, with one word of c.
template <typename T>
__device__ __forceinline__ float below(float m, const Shift& s, const Base& b) {
  if (m == -INFINITY) return m;
  const float hc = ceilf(m * b.c);
  const bool far = !(fabsf(hc) < kFar);
  if (sizeof(T) == 2 || far == s.far) return s.far ? (m - s.h) * b.c : hc - s.hc;
  return s.far ? __fmaf_rn(-s.h, b.c, hc) : __fmaf_rn(m, b.c, -s.hc);
}
template <typename T>
__device__ __forceinline__ void move(Moments* a, const Shift& to, const Base& b) {
  const float d = below<T>(a->m, to, b), f = exp2_fast(d);
  a->t = (a->t + low(d) * a->s) * f;
  a->s *= f;
}
template <typename T>
__device__ __forceinline__ uint32_t largest_word(const uint4& v) {
  return Vec<T>::top(Vec<T>::top(v.x, v.y), Vec<T>::top(v.z, v.w));
}
template <typename T>
__device__ __forceinline__ float largest(const uint4& v) {
  return Vec<T>::top_of(largest_word<T>(v));
}
// The word's two values, no less than those of `floor` (NaN stays NaN).
__device__ __forceinline__ uint32_t at_least(uint32_t w, uint32_t floor, __nv_bfloat16) {
  uint32_t r;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(w), "r"(floor));
  return r;
}
__device__ __forceinline__ uint32_t at_least(uint32_t w, uint32_t floor, __half) {
  uint32_t r;
  asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(w), "r"(floor));
  return r;
}

// A thread's running sums. The shift moves only when a logit lies kAbove exponents above it: hardly ever
// after the first batch, and sums are as exact at any shift.
template <typename T>
struct Running {
  Moments a;
  Pair s = 0, t = 0;                     // of a's shift
  Shift h{0.f, 0.f, false};
  float limit = -INFINITY;               // the largest logit that the shift is good for
  uint32_t floor = Vec<T>::kLow;         // 16-bit types: a logit, twice, whose exponential is 0
  bool clamp = true;                     // exponents are held above -256 one by one

  __device__ __forceinline__ void shift_to(float top, const Base& b) {
    split_sums();
    const float m = fmaxf(a.m, top);
    const Shift to = shift_of(m, b);
    if (a.m == -INFINITY) {
      // nothing but -inf and NaN so far: sums of 0 or NaN, at any shift
    } else if (!to.far && !h.far) {
      const float d = h.hc - to.hc, f = exp2_fast(d);
      a.t = (a.t + d * a.s) * f;
      a.s *= f;
    } else {
      move<T>(&a, to, b);
    }
    h = to;
    a.m = m;
    limit = h.far ? m : (h.hc + kAbove) / b.c;
    s = pair_of(a.s, 0.f);
    t = pair_of(a.t, 0.f);
    clamp = true;
    if constexpr (sizeof(T) == 2) {
      // its exponent is -200, give or take a rounding to the type: at most 9 where the shift is below 2^12, but
      // anything for a half that is not a normal number (scales from 2^21 on), which may be 0
      const float f = (h.hc - 200.f) / b.c;
      const T lowest = Vec<T>::round(f);
      clamp = h.far || fabsf(h.hc) > 4096.f || !(f > -60000.f) || !(Vec<T>::one(lowest) * b.c - h.hc < -150.f);
      const uint32_t half = *reinterpret_cast<const uint16_t*>(&lowest);
      floor = clamp ? Vec<T>::kLow : half << 16 | half;
    }
  }
  __device__ __forceinline__ void split_sums() {
    float x, y;
    split(s, &x, &y);
    a.s = x + y;
    split(t, &x, &y);
    a.t = x + y;
  }
  // U vectors whose largest value is `top`.
  template <int U>
  __device__ __forceinline__ void add(const uint4 (&v)[U], float top, const Base& b) {
    constexpr int P = Vec<T>::N / 2;
    if (top > limit) shift_to(top, b);
    const float off = h.far ? 0.f : -h.hc;
    const Pair c = pair_of(b.c, b.c), hc = pair_of(off, off);
    if (sizeof(T) == 2 && !clamp) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        uint4 w = v[u];
        if constexpr (sizeof(T) == 2)
          w = make_uint4(at_least(w.x, floor, T()), at_least(w.y, floor, T()), at_least(w.z, floor, T()), at_least(w.w, floor, T()));
        Pair x[P];
        Vec<T>::pairs(w, x);
#pragma unroll
        for (int i = 0; i < P; ++i) {
          const Pair e = fma_pair(x[i], c, hc), p = exp2_pair(e);
          s = add_pair(s, p);
          t = fma_pair(e, p, t);
        }
      }
    } else {
      const float sh = h.far ? -h.h : 0.f;
      const Pair by = pair_of(sh, sh);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        Pair x[P];
        Vec<T>::pairs(v[u], x);
#pragma unroll
        for (int i = 0; i < P; ++i) {
          if (h.far) x[i] = add_pair(x[i], by);
          const Pair e = fma_pair(x[i], c, hc), p = exp2_pair(e);
          float e0, e1;
          split(e, &e0, &e1);
          s = add_pair(s, p);
          t = fma_pair(pair_of(low(e0), low(e1)), p, t);
        }
      }
    }
  }
  __device__ __forceinline__ void add_one(float x, const Base& b) {
    if (x > limit) shift_to(x, b);
    const float e = h.far ? (x - h.h) * b.c : __fmaf_rn(x, b.c, -h.hc), p = exp2_fast(e);
    s = add_pair(s, pair_of(p, 0.f));
    t = fma_pair(pair_of(low(e), 0.f), pair_of(p, 0.f), t);
  }
  __device__ __forceinline__ Moments sums() {
    split_sums();
    return a;
  }
};
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
// (by the warps that need it: the others may go on)
template <typename T, int G>
__device__ __forceinline__ Moments team_merge(Moments a, const Base& b, bool needed) {
  a = warp_merge<T>(a, b);
  if constexpr (G != 32) {
    __shared__ Moments ws[G / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (lane == 0) ws[warp] = a;
    __syncthreads();
    if (needed) a = warp_merge<T>(lane < G / 32 ? ws[lane] : Moments(), b);
  }
  return a;
}
// The log-probability of a logit, from its row's sums.
__device__ __forceinline__ float score_of(const Moments& a, float x, const Base& b) {
  const Shift h = shift_of(a.m, b);
  if (h.far || (a.m == -INFINITY && a.s == 0.f)) {
    if (x != x) return x;
    return a.s == 0.f ? -INFINITY : (x - h.h) * b.scale - logf(a.s);
  }
  // log S in two parts, the power of two and the rest
  const uint32_t bits = __float_as_uint(a.s);
  const float power = (float)((int)(bits >> 23) - 127);
  const float rest = logf(__uint_as_float((bits & 0x007fffffu) | 0x3f800000u));
  const double full = ((double)x * (double)b.c - (double)(h.hc + power)) * kLn2 - ((double)rest + kExp2Low);
  return a.s != a.s ? a.s : (float)full;
}

// A logit as a number that is larger where it is (zeros of either sign are equal; any NaN is above
// all), never 0; with its place as one number: lower places first among equal ones.
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return x != x ? 0xffffffffu : (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t order) {
  return __uint_as_float(order & 0x80000000u ? order & 0x7fffffffu : ~order);
}
__device__ __forceinline__ uint64_t key_of(float x, int64_t at) { return (uint64_t)order_of(x) << 32 | (uint32_t)~(uint32_t)at; }
__device__ __forceinline__ int64_t place_of(uint64_t key) { return (int64_t)(uint32_t)~(uint32_t)key; }

// The best keys seen by a team: an unordered list that takes every key above the last
// bound, cut back to its best whenever it is full.
template <int G>
struct Held {
  static constexpr int N = G == 32 ? 128 : 256;
  uint64_t key[N];
  uint64_t bound;             // no key at or below it is among the best
  int n;
  uint32_t least[G / 32];     // of a sweep, by warps
  uint16_t list[G / 32][kBatches * 32];
  uint32_t most[kBatches][G]; // the threads' marks, by batches
};
// The whole team: the list's best `top`, in order, and the bound that follows.
template <int G>
__device__ __forceinline__ void cut(Held<G>* H, int top) {
  constexpr int N = Held<G>::N, per = N / G;  // keys of a thread
  Team<G>::sync();
  const int n = H->n < N ? H->n : N, tid = Team<G>::tid();
  if (G == 32 && n <= G) {
    // a key's place is counted by as many lanes as there are for it (16,000 x 1,000 fp32, 20 best: 53 -> 50 us; in blocks it costs
    // their sweeps registers, 8,192 x 131,072 bf16, 5 best: 363 -> 385)
    int lanes = 1;
    while (lanes < 8 && n * lanes * 2 <= G) lanes *= 2;
    const int own = tid / lanes;
    const uint64_t key = own < n ? H->key[own] : 0;
    int place = 0;
    if (own < n)
#pragma unroll 4
      for (int i = tid % lanes; i < n; i += lanes) place += H->key[i] > key;
    for (int o = 1; o < lanes; o *= 2) place += __shfl_xor_sync(0xffffffffu, place, o);
    Team<G>::sync();
    if (own < n && place < top) {
      H->key[place] = key;
      if (place == top - 1) H->bound = key;
    }
    if (tid == 0) H->n = n < top ? n : top;
    Team<G>::sync();
    return;
  }
  uint64_t mine[per];
  int rank[per];
#pragma unroll
  for (int u = 0; u < per; ++u) {
    mine[u] = tid + u * G < n ? H->key[tid + u * G] : 0;
    rank[u] = 0;
  }
  if (tid < n)
#pragma unroll 4
    for (int i = 0; i < n; ++i) {
      const uint64_t other = H->key[i];
#pragma unroll
      for (int u = 0; u < per; ++u) rank[u] += other > mine[u];
    }
  Team<G>::sync();
#pragma unroll
  for (int u = 0; u < per; ++u) {
    const bool in = tid + u * G < n;
    if (in && rank[u] < top) H->key[rank[u]] = mine[u];
    if (in && rank[u] == top - 1) H->bound = mine[u];
  }
  if (tid == 0) H->n = n < top ? n : top;
  Team<G>::sync();
}
// Into the list; false: there is no room before the next cut.
template <int G>
__device__ __forceinline__ bool offer(Held<G>* H, uint64_t key) {
  const int at = atomicAdd(&H->n, 1);
  if (at < Held<G>::N) H->key[at] = key;
  return at < Held<G>::N;
}
// What a batch leaves behind of a thread's two vectors: of 16-bit types both vectors' largest logits, of float
// the larger one.
template <typename T>
struct Mark {
  static constexpr uint32_t kNone = Vec<T>::kLow;
  // of two words of pairwise largest logits
  __device__ static uint32_t of(uint32_t t0, uint32_t t1) {
    return Vec<T>::top(__byte_perm(t0, t1, 0x5410), __byte_perm(t0, t1, 0x7632));
  }
  __device__ static bool reaches(uint32_t w, uint32_t from) { return mask(w, from) != 0; }
  __device__ static int count(uint32_t w, uint32_t from) { return __popc(mask(w, from) & 0x00010001u); }
  __device__ static uint32_t mask(uint32_t w, uint32_t from);
  // upper halves of the orders of its logits, and back
  __device__ static uint32_t ordered(uint32_t w) {
    const uint32_t sign = (w >> 15 & 0x00010001u) * 0x7fffu;  // 0x7fff where negative
    return w ^ (sign | 0x80008000u);
  }
  __device__ static uint32_t raw(uint32_t w) {
    const uint32_t sign = (~w >> 15 & 0x00010001u) * 0x7fffu;
    return w ^ (sign | 0x80008000u);
  }
  __device__ static int reach(uint32_t ordered, uint32_t half) {
    return (int)(ordered >> 16 >= half) + (int)((ordered & 0xffff) >= half);
  }
  // the order of the logit whose order's upper half that is
  __device__ static uint32_t order(uint32_t half) {
    const uint16_t bits = (uint16_t)raw(half);
    return order_of(Vec<T>::one(*reinterpret_cast<const T*>(&bits)));
  }
  __device__ static uint32_t word(float from) {
    const T t = Vec<T>::round(from);
    const uint32_t b = *reinterpret_cast<const uint16_t*>(&t);
    return b << 16 | b;
  }
};
template <>
__device__ __forceinline__ uint32_t Mark<__nv_bfloat16>::mask(uint32_t w, uint32_t from) {
  return __hge2_mask(*reinterpret_cast<__nv_bfloat162*>(&w), *reinterpret_cast<__nv_bfloat162*>(&from));
}
template <>
__device__ __forceinline__ uint32_t Mark<__half>::mask(uint32_t w, uint32_t from) {
  return __hge2_mask(*reinterpret_cast<__half2*>(&w), *reinterpret_cast<__half2*>(&from));
}
template <>
struct Mark<float> {
  static constexpr uint32_t kNone = Vec<float>::kLow;
  __device__ static uint32_t of(uint32_t t0, uint32_t t1) { return Vec<float>::top(t0, t1); }
  __device__ static bool reaches(uint32_t w, uint32_t from) { return __uint_as_float(w) >= __uint_as_float(from); }
  __device__ static int count(uint32_t w, uint32_t from) { return reaches(w, from); }
  __device__ static uint32_t ordered(uint32_t w) { return order_of(__uint_as_float(w)); }
  __device__ static uint32_t raw(uint32_t w) { return __float_as_uint(value_of(w)); }
  __device__ static int reach(uint32_t ordered, uint32_t half) { return ordered >> 16 >= half; }
  __device__ static uint32_t order(uint32_t half) { return half << 16; }
  __device__ static uint32_t word(float from) { return __float_as_uint(from); }
};
// The j-th largest of a warp's numbers.
__device__ __forceinline__ uint32_t jth_largest(uint32_t u, int j) {
  for (int i = 1; i < j; ++i) {
    const uint32_t most = __reduce_max_sync(0xffffffffu, u);
    const uint32_t who = __ballot_sync(0xffffffffu, u == most);
    if (((int)threadIdx.x & 31) == __ffs((int)who) - 1) u = 0;
  }
  return __reduce_max_sync(0xffffffffu, u);
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

// A team's share (`part` of `parts`) of a row. Its best `top` logits are found by bounds: of the
// largest logits of some groups of its elements the top-th is a bound from below. A sweep of kBatches
// batches leaves the threads' largest ones behind; the few batches that reach the bound are then read
// again, and what is above it goes into the list.
template <typename T, int G, bool kTop>
__device__ __forceinline__ Moments score_sweep(const T* x, int64_t V, const Base& b, int part, int parts, int top, Held<G>* H) {
  constexpr int N = Wide<T>::N, U = kSweepVecs, M = Vec<T>::N;
  [[maybe_unused]] constexpr int kFew = sizeof(T) / 2;  // batches of a warp that leave 64 marks behind
  const int tid = Team<G>::tid();
  const int head = wide_head(x, V);
  const int64_t nv = (V - head) / N;
  const int tail = (int)(V - head - nv * N);
  const T* q = x + head;
  const int64_t per = (nv + parts - 1) / parts;
  const int64_t lo = per * part < nv ? per * part : nv, hi = lo + per < nv ? lo + per : nv;
  Running<T> a;
  uint64_t edge = 0;  // the row's ends, by a few threads of the first part
  if (part == 0 && tid < head + tail) {
    const int64_t i = tid < head ? (int64_t)tid : V - tail + (tid - head);
    const float v = Vec<T>::one(x[i]);
    a.add_one(v, b);
    edge = key_of(v, i);
  }
  if (kTop) {
    if (tid == 0) H->n = 0, H->bound = 0;
    Team<G>::sync();
  }
  int64_t begin = lo;
  do {
    uint32_t best = Mark<T>::kNone;
    int batches = 0;
    for (; batches < kBatches && begin + batches * (U * G) < hi; ++batches) {
      const int64_t i0 = begin + batches * (U * G) + tid;
      uint4 v[2 * U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t i = i0 + u * G;
        v[2 * u] = v[2 * u + 1] = make_uint4(Vec<T>::kLow, Vec<T>::kLow, Vec<T>::kLow, Vec<T>::kLow);
        if (i < hi) {
          const Wide<T> w = load_wide(q + i * N, true);
          v[2 * u] = w.a;
          v[2 * u + 1] = w.b;
        }
      }
      static_assert(U == 2, "two vectors a thread");
      const uint32_t mark = Mark<T>::of(Vec<T>::top(largest_word<T>(v[0]), largest_word<T>(v[1])),
                                        Vec<T>::top(largest_word<T>(v[2]), largest_word<T>(v[3])));
      a.add(v, Vec<T>::top_of(mark), b);
      if constexpr (kTop) {
        H->most[batches][tid] = mark;
        best = Vec<T>::top(best, mark);
      }
    }
    if constexpr (kTop) {
      uint32_t least;
      if constexpr (G == 32) {
        if (top <= 8) {
          least = jth_largest(order_of(Vec<T>::top_of(best)), top);
        } else if (batches <= kFew && top > 32) {
          // (64 marks bound 64 alternatives badly: 16,000 rows of 1,000 bf16 230 us, so 90.) The largest upper
          // half of an order that `top` of the elements reach.
          uint4 v[2 * U * kFew];
#pragma unroll
          for (int u = 0; u < 2 * U * kFew; ++u) {
            const int64_t vec = begin + u / (2 * U) * (U * G) + tid + u / 2 % U * G;
            v[u] = make_uint4(Vec<T>::kLow, Vec<T>::kLow, Vec<T>::kLow, Vec<T>::kLow);
            if (vec < hi) v[u] = *reinterpret_cast<const uint4*>(q + vec * N + (u & 1) * M);
          }
          uint32_t half = 0;
          for (uint32_t bit = 0x8000; bit; bit >>= 1) {
            const uint32_t word = Mark<T>::word(value_of(Mark<T>::order(half | bit)));
            int reach = 0;
#pragma unroll
            for (int u = 0; u < 2 * U * kFew; ++u)
              reach += Mark<T>::count(v[u].x, word) + Mark<T>::count(v[u].y, word) + Mark<T>::count(v[u].z, word) + Mark<T>::count(v[u].w, word);
            if (__reduce_add_sync(0xffffffffu, reach) >= top) half |= bit;
          }
          least = half ? Mark<T>::order(half) : 0;
        } else {
          // the largest upper half of an order that `top` of the vectors reach
          for (int i = 0; i < batches; ++i) H->most[i][tid] = Mark<T>::ordered(H->most[i][tid]);
          uint32_t half = 0;
          for (uint32_t bit = 0x8000; bit; bit >>= 1) {
            int reach = 0;
            for (int i = 0; i < batches; ++i) reach += Mark<T>::reach(H->most[i][tid], half | bit);
            if (__reduce_add_sync(0xffffffffu, reach) >= top) half |= bit;
          }
          for (int i = 0; i < batches; ++i) H->most[i][tid] = Mark<T>::raw(H->most[i][tid]);
          least = half ? Mark<T>::order(half) : 0;
        }
      } else {
        // (of each warp's so many that the warps have `top` together)
        const uint32_t of_warp = jth_largest(order_of(Vec<T>::top_of(best)), (top + G / 32 - 1) / (G / 32));
        if (tid % 32 == 0) H->least[tid / 32] = of_warp;
        __syncthreads();
        least = H->least[0];
#pragma unroll
        for (int i = 1; i < G / 32; ++i) least = H->least[i] < least ? H->least[i] : least;
      }
      const uint32_t none = order_of(-INFINITY);
      // The batches of this warp's lanes that reach the bound: four lanes read one of them again, a
      // vector each, eight batches at a time, the next eight already under way.
      uint64_t bound = H->bound;
      if (least > none && bound < ((uint64_t)least << 32) - 1) bound = ((uint64_t)least << 32) - 1;
      float from = bound ? value_of((uint32_t)((bound + 1) >> 32)) : -INFINITY;
      const uint32_t from_word = Mark<T>::word(from);
      uint16_t* list = H->list[tid / 32];
      int found = 0;
      for (int i = 0; i < batches; ++i) {
        const bool hit = Mark<T>::reaches(H->most[i][tid], from_word);
        const uint32_t who = __ballot_sync(0xffffffffu, hit);
        if (hit) list[found + __popc(who & lanemask_lt())] = (uint16_t)(i * G + tid);
        found += __popc(who);
      }
      __syncwarp();
      auto vector_at = [&](int i) {  // this lane's one of batch i of the list: its first place, -1: none
        if (i >= found) return (int64_t)-1;
        const int entry = list[i], u = tid & 3;
        const int64_t vec = begin + (int64_t)(entry / G) * (U * G) + entry % G + u / 2 * G;
        return vec < hi ? head + vec * N + (u & 1) * M : (int64_t)-1;
      };
      int i = tid % 32 / 4, done = 0;  // elements of this vector before `done` have been offered
      int64_t at0 = vector_at(i), at1 = vector_at(i + 8);
      uint4 w = make_uint4(0, 0, 0, 0), next = w;
      if (at0 >= 0) w = *reinterpret_cast<const uint4*>(x + at0);
      for (int rest = found;;) {
        bool left = false;
        if (edge > bound) left = !offer(H, edge);
        if (!left) edge = 0;
        while (rest > 0) {
          if (at1 >= 0) next = *reinterpret_cast<const uint4*>(x + at1);
          if (at0 >= 0 && largest<T>(w) >= from) {
            float f[M];
            Vec<T>::get(w, f);
#pragma unroll
            for (int j = 0; j < M; ++j)
              if (f[j] >= from && !left && done <= j) {
                const uint64_t key = key_of(f[j], at0 + j);
                if (key > bound) left = !offer(H, key);
                if (!left) done = j + 1;
              }
          }
          if (__any_sync(0xffffffffu, left)) break;
          rest -= 8;
          i += 8;
          done = 0;
          at0 = at1;
          w = next;
          at1 = vector_at(i + 8);
        }
        if (!Team<G>::any(left)) break;
        cut(H, top);
        bound = H->bound > bound ? H->bound : bound;
        from = value_of((uint32_t)((bound + 1) >> 32));
      }
    }
    begin += kBatches * (U * G);
  } while (begin < hi);
  return a.sums();
}

// What a row that does not count gets.
__device__ __forceinline__ void no_score(const ScoreArgs& A, int64_t row, int tid, int threads) {
  for (int j = tid; j < A.given; j += threads)
    if (A.logp) A.logp[row * A.given + j] = 0.f;
  for (int j = tid; j < A.top; j += threads) A.top_logp[row * A.top + j] = 0.f, A.top_index[row * A.top + j] = -1;
  if (tid == 0 && A.entropy) A.entropy[row] = 0.f;
  if (tid == 0 && A.stats) A.stats[row] = make_float4(0.f, 0.f, 0.f, 0.f);
}
__device__ __forceinline__ void write_scores(const ScoreArgs& A, const Moments& a, int64_t row, const Base& b) {
  const bool empty = a.m == -INFINITY && a.s == 0.f;
  const Shift h = shift_of(a.m, b);
  const float ls = empty ? 0.f : logf(a.s);
  float e = empty ? 0.f : __fmaf_rn(-(float)kLn2, a.t / a.s, ls);
  e = e < 0.f ? 0.f : e;  // (kExp2Low of S is left: a row of one token has no entropy)
  if (A.entropy) A.entropy[row] = e;
  if (A.stats) A.stats[row] = make_float4(h.h, empty ? INFINITY : ls, e, 0.f);
}

// Rows by blocks, by clusters of `parts` blocks where there are few, by warps where there are many
// short ones. Bound by memory where rows are long (8,192 x 131,072 bf16: 305 us, 7.0 TB/s, with 8 alternatives 363), else by
// the chain of reads, sums and candidates of each row (4,096 x 50,257 bf16: 72 us, 5.7 TB/s, with 8 alternatives 92).
template <typename T, int G, bool kTop>
__global__ void __launch_bounds__(Team<G>::kThreads, G == 128 ? 10 : G == 32 && kTop ? 4 : 5) k_scores(Rows<T> R, ScoreArgs A, int parts) {
  using Te = Team<G>;
  __shared__ Held<G> held[kTop ? Te::kRows : 1];
  __shared__ Moments cs[kMaxParts];
  __shared__ uint64_t ck[kTop && G != 32 ? kMaxParts : 1][kMostTop];
  griddep_wait();
  const int64_t at = blockIdx.x / parts, row = at * Te::kRows + Te::of_block();
  const int part = (int)(blockIdx.x - at * parts), tid = Te::tid();
  if (G == 32 && row >= R.n) return;
  const int64_t* y = A.y + row * A.given;
  if (!counts(y, A.given)) {  // (all blocks of a cluster)
    if (part == 0) no_score(A, row, tid, G);
    return;
  }
  if (G != 32 && parts > 1) cluster_arrive();
  const T* x = R.x + row * R.ld;
  // the given tokens' logits, read while there is time; by threads that have no alternative to finish
  constexpr int kOwn = G == 32 ? kMostGiven / 32 : 1;
  const int mine = G == 32 ? tid : tid - kMostTop;
  float xy[kOwn];
  bool scored[kOwn];
#pragma unroll
  for (int o = 0; o < kOwn; ++o) {
    const int j = mine + o * G;
    const int64_t t = j >= 0 && j < A.given ? y[j] : -1;
    scored[o] = t >= 0;
    xy[o] = t >= 0 ? target_logit(x, R.V, t) : 0.f;
  }
  Held<G>* H = &held[kTop ? Te::of_block() : 0];
  Moments a = score_sweep<T, G, kTop>(x, R.V, R.b, part, parts, A.top, H);
  // alternatives are finished by the first two warps, given tokens by the next two, the row by the last
  const int warp = (int)threadIdx.x / 32;
  a = team_merge<T, G>(a, R.b, warp == G / 32 - 1 || (warp < 4 && warp * 32 < (warp < 2 ? A.top : A.given + kMostTop)) || warp == 0);
  const uint64_t* best = H->key;
  if (kTop) cut(H, A.top);
  if (G != 32 && parts > 1) {
    cluster_wait();  // every block has begun
    // into slot `part` of the first block: the sums, and the best keys (0: none)
    const uint32_t here = smem_addr(cs + part), keys = smem_addr(ck[kTop ? part : 0]);
    uint32_t there;
    if (tid == 0) {
      asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(there) : "r"(here));
      asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(there), "f"(a.m), "f"(a.s), "f"(a.t), "f"(0.f) : "memory");
    }
    if (kTop && tid < A.top) {
      const uint64_t key = tid < H->n ? H->key[tid] : 0;
      asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(there) : "r"(keys + tid * 8));
      asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(there), "l"(key) : "memory");
    }
    cluster_arrive();
    cluster_wait();
    if (part != 0) return;
    a = warp_merge<T>((int)threadIdx.x % 32 < parts ? cs[threadIdx.x % 32] : Moments(), R.b);
    if (kTop) {
      // each key's place: its own in its list, and how many of the others' are above it
      for (int i = tid; i < parts * A.top; i += G) {
        const int list = i / A.top, own = i % A.top;
        const uint64_t key = ck[list][own];
        int above[kMaxParts] = {}, rank = 0;  // the lists are in order: so many of each, by halving, all at once
        for (int bit = kMostTop; bit; bit >>= 1)
#pragma unroll
          for (int l = 0; l < kMaxParts; ++l) {
            const int to = above[l] + bit;
            if (l < parts && to <= A.top && ck[l][to - 1] > key) above[l] = to;
          }
#pragma unroll
        for (int l = 0; l < kMaxParts; ++l) rank += above[l];
        if (key && rank < A.top) H->key[rank] = key;
      }
      __syncthreads();
    }
  }
#pragma unroll
  for (int o = 0; o < kOwn; ++o) {
    const int j = mine + o * G;
    if (j >= 0 && j < A.given && A.logp) A.logp[row * A.given + j] = scored[o] ? score_of(a, xy[o], R.b) : 0.f;
  }
  if (kTop)
    for (int j = tid; j < A.top; j += G) {
      const uint64_t key = best[j];
      A.top_logp[row * A.top + j] = score_of(a, value_of((uint32_t)(key >> 32)), R.b);
      A.top_index[row * A.top + j] = a.s != a.s ? -1 : place_of(key);
    }
  if (tid == G - 1) write_scores(A, a, row, R.b);
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
  const Pair by = pair_of(sh, sh), c = pair_of(b.c, b.c), off = pair_of(hc, hc),
             c0 = pair_of(g.c0, g.c0), c1 = pair_of(g.c1, g.c1);
  Pair x[P];
  Vec<T>::pairs(v, x);
#pragma unroll
  for (int i = 0; i < P; ++i) {
    x[i] = add_pair(x[i], by);
    const Pair e = fma_pair(x[i], c, off);
    float e0, e1;
    split(e, &e0, &e1);
    x[i] = mul_pair(exp2_pair(e), fma_pair(pair_of(low(e0), low(e1)), c1, c0));
  }
  return Vec<T>::put_pairs(x);
}
template <typename T>
__device__ __forceinline__ float grad_one(float x, const ScoreGrad& g, const Base& b) {
  const float e = g.h.far ? (x - g.h.h) * b.c : __fmaf_rn(x, b.c, -g.h.hc);
  return exp2_fast(e) * __fmaf_rn(low(e), g.c1, g.c0);
}

// dx of a row, or a part of it, by a block or a warp. Bound by memory, read and written: 8,192 x 131,072 bf16 642 us,
// 6.7 TB/s, 4,096 x 50,257 130 us, 6.4; 16,384 x 4,096 53 us, 5.1, where a row's own slopes and sums come first.
template <typename T, int G>
__global__ void __launch_bounds__(kLossThreads, G == 32 ? 4 : 5) k_scores_grad(Rows<T> R, int given, const float4* stats,
                                                                               const float* g, const float* dh, T* dx,
                                                                               int64_t dld, int parts) {
  using Te = Team<G>;
  constexpr int N = Wide<T>::N, U = kSweepVecs, kOwn = G == 32 ? kMostGiven / 32 : 1;
  __shared__ int64_t all_ys[Te::kRows][kMostGiven];
  __shared__ float all_gs[Te::kRows][kMostGiven];
  griddep_wait();
  // from the last row to the first: the logits read last are still in the L2 cache
  const int64_t row = R.n - 1 - (blockIdx.x / parts * Te::kRows + Te::of_block());
  if (G == 32 && row < 0) return;
  const int part = (int)(blockIdx.x % parts), tid = Te::tid();
  int64_t* ys = all_ys[Te::of_block()];
  float* gs = all_gs[Te::of_block()];
  const T* x = R.x + row * R.ld;
  T* out = dx + row * dld;
  const int64_t V = R.V;
  const int head = wide_head(x, V);
  const int64_t nv = (V - head) / N;
  const int tail = (int)(V - head - nv * N);
  const int64_t per = (nv + parts - 1) / parts;
  const int64_t lo = per * part < nv ? per * part : nv, hi = lo + per < nv ? lo + per : nv;

  const float4 st = stats[row];
  float h = dh ? dh[row] : 0.f;
  bool wrong = false, some = given == 0, any = false;
  for (int j = tid; j < given; j += G) {
    const int64_t y = R.y[row * given + j];
    const float gy = y >= 0 && g ? g[row * given + j] : 0.f;
    ys[j] = y;
    gs[j] = gy;
    wrong |= y >= V;
    some |= y >= 0;
    any |= gy != 0.f;
  }
  wrong = Te::any(wrong);
  if (!Te::any(some)) {
    if (st.y != st.y) {  // it counted, and its alternatives (-1: NaN has none) are the tokens: all of its slopes are looked at
      bool slope = h != 0.f;
      for (int j = tid; g && j < given; j += G) slope |= g[row * given + j] != 0.f;
      wrong |= Te::any(slope);
    }
    h = 0.f;  // the row does not count
  }
  any = Te::any(any) || h != 0.f;
  const bool skip = !wrong && (!any || st.y == INFINITY);
  float sum = 0.f;
  for (int j = 0; j < given; ++j) sum += gs[j];
  if (wrong) sum = __uint_as_float(kNan);
  const float k = -R.b.scale * expf(-st.y);
  const ScoreGrad q{shift_of(st.x, R.b), k * (sum + h * (st.z - st.y)), k * h * (float)kLn2};

  // The given tokens in this part, taken before their places are written (out may be x):
  // g_y (1 - p_y) - p_y (G - g_y + h (lp_y + H)), the first without cancellation.
  float at_y[kOwn];
  bool mine[kOwn];
#pragma unroll
  for (int o = 0; o < kOwn; ++o) {
    const int own = tid + o * G;
    mine[o] = false;
    if (own >= given || skip) continue;
    const int64_t y = ys[own], v = y >= head ? (y - head) / N : -1;
    mine[o] = y >= 0 && y < V && (y < head || v >= nv ? part == 0 : v >= lo && v < hi);
    if (!mine[o]) continue;
    float gy = 0.f;
    for (int j = 0; j < given; ++j) {
      if (ys[j] != y) continue;
      gy += gs[j];
      if (j < own) mine[o] = false;  // (the first of equal ones writes)
    }
    const float xy = Vec<T>::one(x[y]);
    const float lp = q.h.far ? (xy - q.h.h) * R.b.scale - st.y
                             : (float)(((double)xy * (double)R.b.c - (double)q.h.hc) * kLn2 - ((double)st.y + kExp2Low));
    const float p = lp == -INFINITY ? 0.f : expf(lp), more = p == 0.f ? 0.f : p * (sum - gy + h * (lp + st.z));
    at_y[o] = wrong ? sum : R.b.scale * (gy * -expm1f(lp) - more);
  }
  if (given) Te::sync();
  const bool same = ((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(out)) & 31) == 0;
  for (int64_t i0 = lo + tid; i0 < hi; i0 += U * G) {
    Wide<T> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t i = i0 + u * G;
      v[u].a = v[u].b = make_uint4(0, 0, 0, 0);
      if (!skip && i < hi) v[u] = load_wide(x + head + i * N, true);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t i = i0 + u * G;
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
  if (given) Te::sync();
#pragma unroll
  for (int o = 0; o < kOwn; ++o)
    if (mine[o]) out[ys[tid + o * G]] = Vec<T>::round(at_y[o]);
}

// The team of a row. A row begins and ends with some microseconds of reads that wait for one another: a smaller
// team streams longer in between, and more of them share an SM. The scores of bf16 rows, with 8
// alternatives, in us, by blocks of 256, of 128 and by warps:
//   rows   length     256    128  warps
//    700    4,096    10.5    8.2    9.0
//  2,000    2,000      -    14.9    9.4
// 16,000    4,096      -    90.3   51.5
//  4,000   12,000      -    35.9   29.9
//  2,000   16,384    29.6   24.8
//  4,096   50,257   102.5   92.3
//  1,000   60,000    36.9   31.8
// Gradients by warps as in gmc_loss.cu.
constexpr int64_t kWarpScores = 32768, kWarpGrad = 18432, kHalfScores = 131072;  // bytes of a row at most
bool by_warps(int64_t n, int64_t rows, int64_t row_bytes, int64_t most) {
  return n >= rows && row_bytes <= most && row_bytes <= 12 * n;
}

template <typename T, bool kTop>
cudaError_t launch_scores(const Rows<T>& R, const ScoreArgs& A, cudaStream_t s) {
  const int64_t bytes = R.V * (int64_t)sizeof(T);
  if (by_warps(R.n, 1400, bytes, kWarpScores))
    return launch(k_scores<T, 32, kTop>, (R.n + 7) / 8, kLossThreads, 1, s, R, A, 1);
  const int most = parts_for(R.n, bytes);
  if (most == 1 && bytes <= kHalfScores) return launch(k_scores<T, 128, kTop>, R.n, 128, 1, s, R, A, 1);
  return with_parts(most, [&](int parts) {
    return launch(k_scores<T, kLossThreads, kTop>, R.n * parts, kLossThreads, parts, s, R, A, parts);
  });
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
    const Rows<T> R{static_cast<const T*>(logits_dev), n, vocab, ld, score_base(scale), targets_dev};
    const ScoreArgs A{targets_dev, given, top, logp_dev, entropy_dev, top_logp_dev, top_index_dev,
                      reinterpret_cast<float4*>(stats_dev)};
    const cudaStream_t q = static_cast<cudaStream_t>(stream);
    return top ? launch_scores<T, true>(R, A, q) : launch_scores<T, false>(R, A, q);
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
    const Rows<T> R{static_cast<const T*>(logits_dev), n, vocab, ld, score_base(scale), targets_dev};
    const int64_t bytes = vocab * (int64_t)sizeof(T);
    const float4* st = reinterpret_cast<const float4*>(stats_dev);
    const cudaStream_t q = static_cast<cudaStream_t>(stream);
    if (by_warps(n, 600, bytes, kWarpGrad))
      return launch(k_scores_grad<T, 32>, (n + 7) / 8, kLossThreads, 1, q, R, (int)given, st, dlogp_dev, dentropy_dev,
                    static_cast<T*>(dlogits_dev), dld, 1);
    int parts = parts_for(n, bytes);
    while (bytes / parts > 57344) parts *= 2;
    return launch(k_scores_grad<T, kLossThreads>, n * parts, kLossThreads, 1, q, R, (int)given, st, dlogp_dev, dentropy_dev,
                  static_cast<T*>(dlogits_dev), dld, parts);
  });
  return err == cudaSuccess ? GMC_OK : GMC_ECUDA;
}

}  // extern "C"
