// The clipped policy loss with its gradient in one pass over the logits. A row's slope
// depends on its own log-probability alone, so a row is read from HBM once, kept on
// the chip until its sum is known, and its gradient written.
//
// k_policy_rows: persistent clusters of 1 to 8 blocks, a block per SM taking its share of each
// of its cluster's rows. The block's warps have one task each and meet at mbarriers only:
//   load    one warp copies the share into a ring of 32 KB chunks in shared memory by
//           bulk copies (the vectors at the row's two ends element by element, with
//           -inf beside the row)
//   stats   eight warps read the chunks as they land, keeping a maximum and a sum a thread
//   finish  two warps, a row each in turn, merge the threads' sums, exchange them with the
//           cluster's other blocks by messages, and form the token's loss and slope
//   grad    eight warps read the chunks again, write k ([v = y] - p_v) and free them
// so that nothing in a row's long chain of small steps (3 to 4 us) holds up another row's
// traffic: 192 KB of ring cover about 40 KB in flight from HBM, the chain, and a row's
// share of up to 64 KB (128 KB for the longest rows). Bound by HBM at shares of 64 KB (8,192 x
// 131,072 bf16: 603 us, 6.7 TB/s read and written), by the gradient warps at smaller ones (12,160
// x 50,257, shares of 49 KB: 401 us, 6.1 TB/s), and by the first and last row's chains where
// there are few rows (64 x 32,000: 7.9 us).
// k_policy_short: many short rows, one a warp. k_policy: rows over 1 MB, swept twice from global
// memory.
#include <new>

#include "gmc.h"
#include "gmc_loss.cuh"

namespace gmc {
namespace {

constexpr int kChunkVecs = 2048;       // 16-byte vectors of a chunk
constexpr int kMostChunks = 6;         // of the ring
constexpr int kRowSlots = 8;           // rows between the load of their first chunk and their end
constexpr int kFinishers = 2;
constexpr int kStatsWarps = 8, kGradWarps = 8;
constexpr int kStatsBatch = 8;         // vectors of a chunk that a thread takes at once
constexpr int kGradBatch = 4;
constexpr int kWorkWarps = kStatsWarps + kGradWarps;
constexpr int kRowsThreads = (kWorkWarps + kFinishers + 1) * 32;
constexpr int64_t kMostShare = 4 * kChunkVecs;  // vectors of a row that a block takes at most
static_assert(kChunkVecs % (kStatsWarps * 32 * kStatsBatch) == 0, "whole batches");
static_assert(kChunkVecs % (kGradWarps * 32 * kGradBatch) == 0, "whole batches");
static_assert(kRowSlots % kFinishers == 0, "a slot's rows have one finisher");

// The weighted losses' sum in block order, by the last of `blocks` to be done (lane 0 of a
// warp of each calls with its sum, NaN where a wait gave up; the lanes of the last warp add).
__device__ __forceinline__ void reduce_loss(const PolicyArgs& P, double mine, uint32_t block, uint32_t blocks) {
  const int lane = threadIdx.x & 31;
  uint32_t last = 0;
  if (lane == 0) {
    P.partial[block] = mine;
    last = count_inc(P.ticket, blocks - 1) == blocks - 1;
  }
  if (!__shfl_sync(0xffffffffu, last, 0)) return;
  __syncwarp();  // what lane 0's count acquired is there for the other lanes too: a shuffle orders no memory
  double s = 0.;
  for (uint32_t i = lane; i < blocks; i += 32) s += __ldcg(P.partial + i);
  s = warp_sum(s);
  if (lane == 0) *P.loss = (float)s;
}

// What the gradient of a row needs.
struct RowResult {
  float h, hc;   // subtracted from a logit, and from its exponent
  float f, at_y; // -k / S, and k (1 - p_y)
  int64_t y;
  int go, far;   // go: a gradient (else zeros); far: h is subtracted
};
struct alignas(128) RowsShared {
  uint64_t full[kMostChunks], empty[kMostChunks];
  uint64_t summed[kRowSlots];            // the stats warps' sums are there
  uint64_t heard[kFinishers][2];         // the cluster's sums have come, for a finisher's rows in turn
  uint64_t ready[kRowSlots];             // the result is there
  uint64_t free[kRowSlots];              // the row is done
  uint64_t from[kFinishers][2][kMaxParts];  // (m, S) of each block of the cluster
  MaxSum ws[kRowSlots][kStatsWarps * 32];  // of each stats thread
  RowResult res[kRowSlots];
  double total[kFinishers];
  int dead;                              // a wait gave up
};

__device__ __forceinline__ void mbar_expect_tx(uint64_t* bar, uint32_t bytes) {
  asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(smem_addr(bar)), "r"(bytes) : "memory");
}
// Eight bytes into block `rank`'s copy of dst, counted by its barrier.
__device__ __forceinline__ void send(uint64_t* dst, uint64_t* bar, uint32_t rank, uint64_t v) {
  uint32_t d, b;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(d) : "r"(smem_addr(dst)), "r"(rank));
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(b) : "r"(smem_addr(bar)), "r"(rank));
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.b64 [%0], %1, [%2];" ::"r"(d), "l"(v), "r"(b)
               : "memory");
}
__device__ __forceinline__ bool try_wait_cluster(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(smem_addr(bar)), "r"(parity)
      : "memory");
  return ok != 0;
}
// What a block that gave up leaves to copies and messages under way before its shared memory may be
// another's: they land within microseconds.
constexpr uint64_t kLandNs = 1000000;
__device__ __forceinline__ uint64_t landing(uint64_t limit_ns) { return limit_ns > kLandNs ? limit_ns : kLandNs; }
// A warp's waits: bounded, with one answer for all its lanes.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, uint64_t limit_ns) {
  return __all_sync(0xffffffffu, wait_bounded(bar, parity, limit_ns));
}
__device__ __forceinline__ bool warp_wait_cluster(uint64_t* bar, uint32_t parity, uint64_t limit_ns) {
  bool ok = try_wait_cluster(bar, parity);
  const uint64_t t0 = global_ns();
  while (!ok && global_ns() - t0 <= limit_ns) ok = try_wait_cluster(bar, parity);
  return __all_sync(0xffffffffu, ok);
}

// A row cut into the 16-byte vectors that cover it: vector i begins `ph` elements
// before element i N.
template <typename T>
struct Cover {
  int ph;
  int64_t nv;        // vectors, the first and last perhaps in part
  bool first, last;  // whether those are in part
  __device__ Cover(const T* x, int64_t V) {
    constexpr int N = Vec<T>::N;
    ph = (int)((reinterpret_cast<uintptr_t>(x) & 15) / sizeof(T));
    nv = (ph + V + N - 1) / N;
    first = ph != 0;
    last = (ph + V) % N != 0;
  }
};

constexpr int kStatsThreads = kStatsWarps * 32;
// U of a chunk's vectors into a: those at q, q + kStatsThreads, ... that lie before `left`.
template <typename T, int U>
__device__ __forceinline__ void add_some(MaxSum* a, const uint4* q, int left, const Base& b) {
  uint4 v[U];
#pragma unroll
  for (int u = 0; u < U; ++u)
    v[u] = u * kStatsThreads < left ? q[u * kStatsThreads]
                                    : make_uint4(Vec<T>::kLow, Vec<T>::kLow, Vec<T>::kLow, Vec<T>::kLow);
  add<T>(a, v, b);
}
// A warp's merge of all stats threads' maxima and sums.
template <typename T>
__device__ __forceinline__ MaxSum block_of(const MaxSum* ws, int lane, const Base& b) {
  MaxSum t[kStatsWarps], r;
#pragma unroll
  for (int i = 0; i < kStatsWarps; ++i) {
    t[i] = ws[i * 32 + lane];
    r.m = fmaxf(r.m, t[i].m);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) r.m = fmaxf(r.m, __shfl_xor_sync(0xffffffffu, r.m, o));
  const Shift h = shift_of(r.m, b);
#pragma unroll
  for (int i = 0; i < kStatsWarps; ++i) r.s += t[i].s * exp2_fast(between<T>(t[i].m, h, b));
  r.s = warp_sum(r.s);
  return r;
}

// What tells whether a row counts: loaded a row ahead of its use, and looked at only then,
// so that nothing waits for it.
struct Facts {
  int64_t y;
  float w;
  __device__ __forceinline__ bool count() const { return y >= 0 && w != 0.f; }
};
template <typename T>
__device__ __forceinline__ Facts facts_of(const Rows<T>& R, const PolicyArgs& P, int64_t row) {
  if (row >= R.n) row = R.n - 1;
  return Facts{R.y[row], P.weights ? P.weights[row] : P.weight};
}

// A place in the ring, and how often it was used before.
struct RingAt {
  int i = 0;
  uint32_t turn = 0;
  __device__ __forceinline__ void next(int size) {
    if (++i == size) i = 0, ++turn;
  }
};

// The loss and its gradient (dx may be NULL). per: vectors of a block's share of a row;
// chunks: of the ring.
template <typename T>
__global__ void __launch_bounds__(kRowsThreads, 1)
    k_policy_rows(Rows<T> R, PolicyArgs P, T* dx, int64_t dld, int parts, int per, int chunks) {
  constexpr int N = Vec<T>::N;
  extern __shared__ __align__(128) unsigned char smem[];
  RowsShared& S = *reinterpret_cast<RowsShared*>(smem);
  uint4* ring = reinterpret_cast<uint4*>(smem + sizeof(RowsShared));
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int rank = parts > 1 ? (int)cluster_rank() : 0;
  const int64_t cluster = blockIdx.x / parts, clusters = gridDim.x / parts;
  const int64_t lo = (int64_t)per * rank;  // this block's first vector of a row
  const uint64_t limit = P.wait_ns;

  if (threadIdx.x == 0) {
    for (int i = 0; i < chunks; ++i) {
      mbar_init(&S.full[i], 1);
      mbar_init(&S.empty[i], kGradWarps);
    }
    for (int i = 0; i < kRowSlots; ++i) {
      mbar_init(&S.summed[i], kStatsWarps);
      mbar_init(&S.ready[i], 1);
      mbar_init(&S.free[i], kGradWarps);
    }
    for (int i = 0; i < 2 * kFinishers; ++i) mbar_init(&S.heard[i / 2][i & 1], 1);
    S.dead = 0;
    fence_mbar_init();
  }
  __syncthreads();
  if (parts > 1) {  // no message before every block's barriers are there
    cluster_arrive();
    cluster_wait();
  }
  griddep_wait();

  auto facts_at = [&](int64_t row) { return facts_of(R, P, row); };
  // this block's vectors of a row
  auto share_of = [&](const Cover<T>& c) { return (int)max((int64_t)0, (lo + per < c.nv ? lo + per : c.nv) - lo); };

  if (warp < kStatsWarps) {
    const int tid = (int)threadIdx.x;
    RingAt at;
    uint32_t r = 0;  // rows taken before this one
    Facts next = facts_at(cluster);
    for (int64_t row = cluster; row < R.n; row += clusters, ++r) {
      const bool now = next.count();
      next = facts_at(row + clusters);
      const int slot = r % kRowSlots;
      const uint32_t turn = r / kRowSlots;
      // every row passes every barrier of its slot, also one that does not count: a
      // parity told in advance is then never two phases old
      bool ok = !turn || warp_wait(&S.free[slot], (turn - 1) & 1, limit);
      const Cover<T> c(R.x + row * R.ld, R.V);
      const int cnt = now ? share_of(c) : 0;
      MaxSum a;
      for (int q = 0; q < cnt; q += kChunkVecs, at.next(chunks)) {
        if (!(ok = ok && warp_wait(&S.full[at.i], at.turn & 1, limit))) break;
        const uint4* chunk = ring + at.i * kChunkVecs;
        const int here = min(kChunkVecs, cnt - q);
        const int here_warp = here - (int)threadIdx.x + lane;  // from this warp's first vector on
#pragma unroll 1
        for (int v0 = 0; v0 < here_warp; v0 += kStatsThreads * kStatsBatch) {
          // as many vectors at once as the warp has, or the next power of two
          const int left = here_warp - v0;
          const uint4* from = chunk + tid + v0;
          if (left > 4 * kStatsThreads) add_some<T, 8>(&a, from, left - lane, R.b);
          else if (left > 2 * kStatsThreads) add_some<T, 4>(&a, from, left - lane, R.b);
          else if (left > kStatsThreads) add_some<T, 2>(&a, from, left - lane, R.b);
          else add_some<T, 1>(&a, from, left - lane, R.b);
        }
      }
      if (!ok) {
        S.dead = 1;
        break;
      }
      S.ws[slot][tid] = a;
      __syncwarp();
      if (lane == 0) mbar_arrive(&S.summed[slot]);
    }
  } else if (warp < kWorkWarps) {
    constexpr int kGradThreads = kGradWarps * 32;
    const int tid = (int)threadIdx.x - kStatsWarps * 32;
    RingAt at;
    uint32_t r = 0;
    Facts next = facts_at(cluster);
    for (int64_t row = cluster; row < R.n; row += clusters, ++r) {
      const bool now = next.count();
      next = facts_at(row + clusters);
      const int slot = r % kRowSlots;
      // The result comes after the sums, and these after the row's chunks. It comes, or a wait that
      // it depends on gives up, here or in the finisher, and S.dead says so: a block whose gradient is
      // not complete is one whose finishers know of it. (A finisher waits three times at most for a row.)
      bool ok = warp_wait(&S.ready[slot], (r / kRowSlots) & 1, limit);
      for (const uint64_t t0 = global_ns(); !ok;) {
        const bool over = *(volatile int*)&S.dead || global_ns() - t0 > 4 * kWaitLimitNs;
        if (__any_sync(0xffffffffu, over)) break;
        ok = warp_wait(&S.ready[slot], (r / kRowSlots) & 1, limit);
      }
      if (!ok) {
        S.dead = 1;
        break;
      }
      const T* x = R.x + row * R.ld;
      const Cover<T> c(x, R.V);
      const int cnt = share_of(c);
      const RowResult g = S.res[slot];
      T* out = dx + row * dld;
      // whether vectors can be written whole; the few far rows are left to the slow path too
      const bool same = !g.far && (reinterpret_cast<uintptr_t>(out) & 15) / sizeof(T) == (unsigned)c.ph;
      const int64_t vy = g.y < R.V ? (g.y + c.ph) / N - lo : -1;  // the target's vector
      for (int q = 0; q < cnt; q += kChunkVecs) {
        const int place = at.i;
        if (now) at.next(chunks);  // a row that does not count holds no chunks
        const uint4* chunk = ring + place * kChunkVecs;
        const int here = min(kChunkVecs, cnt - q);
        const Pair cc = pair_of(R.b.c, R.b.c), cl = pair_of(R.b.lo, R.b.lo), hc = pair_of(-g.hc, -g.hc),
                   by = pair_of(g.f, g.f);
        auto slope = [&](Pair v) { return mul_pair(by, exp2_pair(fma_pair(v, cl, fma_pair(v, cc, hc)))); };
        const int64_t j0 = (lo + q) * N - c.ph;  // the chunk's first element
        // the whole vectors among them
        const int vb = !same ? here : j0 < 0 ? 1 : 0;
        const int ve = !same ? here : j0 + (int64_t)here * N > R.V ? here - 1 : here;
        uint4* dst = reinterpret_cast<uint4*>(out + j0);
        if (!dx) {
        } else if (g.go) {
#pragma unroll 1
          for (int v0 = tid; v0 < ve; v0 += kGradThreads * kGradBatch) {
            uint4 w[kGradBatch];  // (past the end: what the chunk last held, not stored)
#pragma unroll
            for (int u = 0; u < kGradBatch; ++u) w[u] = chunk[v0 + u * kGradThreads];
#pragma unroll
            for (int u = 0; u < kGradBatch; ++u) {
              const int v = v0 + u * kGradThreads;
              Pair f[N / 2];
              Vec<T>::pairs(w[u], f);
#pragma unroll
              for (int e = 0; e < N / 2; ++e) f[e] = slope(f[e]);
              w[u] = Vec<T>::put_pairs(f);
              if (v >= vb && v < ve) dst[v] = w[u];
            }
          }
        } else {
          for (int v = tid; v < ve; v += kGradThreads)
            if (v >= vb) dst[v] = make_uint4(0, 0, 0, 0);
        }
        // the rest element by element: the row's ends, or all of a row that lies otherwise
        if (dx && (vb > 0 || ve < here)) {
          auto single = [&](int i) {
            const int64_t j = j0 + i;
            if (j < 0 || j >= R.V) return;
            float one = 0.f, none = 0.f;
            if (g.go)
              split(slope(pair_of(Vec<T>::one(reinterpret_cast<const T*>(chunk)[i]) - (g.far ? g.h : 0.f), 0.f)), &one,
                    &none);
            out[j] = Vec<T>::round(one);
          };
          for (int i = tid; i < vb * N; i += kGradThreads) single(i);
          for (int i = max(ve, vb) * N + tid; i < here * N; i += kGradThreads) single(i);
        }
        // the target's own, by the thread that wrote its place
        const int64_t v = vy - q;
        if (dx && g.go && v >= 0 && v < here) {
          const int i = (int)(g.y - j0);
          const int by_tid = (v >= vb && v < ve ? (int)v : v < vb ? i : i - max(ve, vb) * N) & (kGradThreads - 1);
          if (tid == by_tid) out[g.y] = Vec<T>::round(g.at_y);
        }
        if (now) {
          __syncwarp();
          if (lane == 0) mbar_arrive(&S.empty[place]);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&S.free[slot]);
    }
  } else if (warp < kWorkWarps + kFinishers) {
    const int me = warp - kWorkWarps;
    double total = 0.;
    uint32_t r = (uint32_t)me;
    uint32_t trades = 0;  // rows whose sums this finisher exchanged
    Facts next = facts_at(cluster + me * clusters);
    bool alive = true;
    for (int64_t row = cluster + me * clusters; row < R.n; row += kFinishers * clusters, r += kFinishers) {
      const int slot = r % kRowSlots;
      const uint32_t turn = r / kRowSlots;
      const Facts facts = next;
      const int64_t y = facts.y;
      const float w = facts.w;
      const bool counts = facts.count();
      next = facts_at(row + kFinishers * clusters);
      float xy = 0.f, adv = 0.f, old_logp = 0.f, ref_logp = 0.f;
      if (counts) {
        xy = target_logit(R.x + row * R.ld, R.V, y);
        adv = P.adv[row];
        old_logp = P.old_logp[row];
        ref_logp = P.ref_logp ? P.ref_logp[row] : 0.f;
      }
      RowResult g = {};
      RowStats st = {};
      float loss = 0.f;
      alive = (!turn || warp_wait(&S.free[slot], (turn - 1) & 1, limit)) && warp_wait(&S.summed[slot], turn & 1, limit);
      if (alive && counts) {
        MaxSum a = block_of<T>(S.ws[slot], lane, R.b);
        if (parts > 1) {
          // Where dx is x, the block that holds x[y] writes its gradient there as soon as it has
          // heard from all. So the sums that it waits for are made of xy: a target that is NaN
          // makes them NaN (as it does the row), and no block sends before it has xy.
          if (__any_sync(0xffffffffu, xy != xy)) a.s = __uint_as_float(kNan);
          // two sets of slots in turn: a block sends its next but one row's sums only after
          // it has heard this one's next, which this one sends after it has read these
          const int set = trades & 1;
          uint64_t* bar = &S.heard[me][set];
          if (lane == 0) mbar_arrive_expect_tx(bar, 8u * (uint32_t)parts);
          __syncwarp();
          if (lane < parts)
            send(&S.from[me][set][rank], bar, (uint32_t)lane,
                 ((uint64_t)__float_as_uint(a.s) << 32) | __float_as_uint(a.m));
          alive = warp_wait_cluster(bar, (trades >> 1) & 1, limit);
          ++trades;
          a = MaxSum();
          if (lane < parts) {
            const uint64_t v = *reinterpret_cast<volatile uint64_t*>(&S.from[me][set][lane]);
            a.m = __uint_as_float((uint32_t)v);
            a.s = __uint_as_float((uint32_t)(v >> 32));
          }
          a = warp_merge<T>(a, R.b);
        }
        st = finish(a, xy, R.b);
        float slope = 0.f;
        if (!st.empty) policy_terms(P, adv, old_logp, ref_logp, st.logp, &loss, &slope);
        const float k = w * slope * R.b.scale;
        g.h = st.h.h;
        g.far = st.h.far;
        g.hc = st.h.far ? 0.f : st.h.hc;
        g.f = -k / a.s;
        g.at_y = k * -expm1f(st.logp);
        g.y = y;
        g.go = slope != 0.f && !st.empty;
        if (!st.empty) total += (double)w * (double)loss;
      }
      if (!alive) {
        S.dead = 1;
        break;
      }
      if (lane == 0) {
        S.res[slot] = g;
        mbar_arrive(&S.ready[slot]);
        if (rank == 0) {
          if (P.token_loss) P.token_loss[row] = loss;
          if (P.logp) P.logp[row] = st.logp;
        }
      }
    }
    // The loss, before the last gradients are out. A wait that gave up anywhere in the block
    // ends, or has ended, a finisher's too; and every block counts, since only its own finishers
    // may know of it.
    if (lane == 0) S.total[me] = total;
    __syncwarp();
    asm volatile("bar.sync 1, %0;" ::"n"(kFinishers * 32) : "memory");
    if (me == 0) {
      total = 0.;
      for (int i = 0; i < kFinishers; ++i) total += S.total[i];
      if (rank > 0) total = 0.;  // its cluster's first block has them
      if (*(volatile int*)&S.dead) total = (double)__uint_as_float(kNan);
      reduce_loss(P, total, blockIdx.x, gridDim.x);
    }
  } else {
    RingAt at;
    bool alive = true;
    Facts next = facts_at(cluster);
    for (int64_t row = cluster; row < R.n && alive; row += clusters) {
      const bool now = next.count();
      next = facts_at(row + clusters);
      if (!now) continue;
      const T* x = R.x + row * R.ld;
      const Cover<T> c(x, R.V);
      const int cnt = share_of(c);
      for (int q = 0; q < cnt; q += kChunkVecs) {
        if (at.turn && !warp_wait(&S.empty[at.i], (at.turn - 1) & 1, limit)) {
          S.dead = 1;
          alive = false;
          break;
        }
        uint4* chunk = ring + at.i * kChunkVecs;
        const int64_t v0 = lo + q, v1 = v0 + min(kChunkVecs, cnt - q);
        const int64_t a = c.first && v0 == 0 ? 1 : v0, b = c.last && v1 == c.nv ? v1 - 1 : v1;
        if (row == P.hold_row) {
          at.next(chunks);
          continue;
        }
        if (lane == 0 && b > a) {
          const uint32_t bytes = (uint32_t)(b - a) * 16u;
          mbar_expect_tx(&S.full[at.i], bytes);
          bulk_load(chunk + (a - v0), x - c.ph + a * N, bytes, &S.full[at.i]);
        }
        // the vectors that the row covers in part
        if (a > v0 && lane < N) {
          const int64_t j = (int64_t)lane - c.ph;
          reinterpret_cast<T*>(chunk)[lane] = j >= 0 && j < R.V ? x[j] : Vec<T>::round(-INFINITY);
        }
        if (b < v1 && b >= a && lane < N) {
          const int64_t j = b * N - c.ph + lane;
          reinterpret_cast<T*>(chunk + (b - v0))[lane] = j < R.V ? x[j] : Vec<T>::round(-INFINITY);
        }
        fence_proxy_async();  // these come before a later bulk copy into the same bytes
        __syncwarp();
        if (lane == 0) mbar_arrive(&S.full[at.i]);
        at.next(chunks);
      }
    }
    // no copy is under way when the block ends, whatever became of its readers
    for (int i = 0; i < chunks; ++i) {
      const uint32_t uses = i < at.i ? at.turn + 1 : at.turn;
      if (uses) wait_bounded(&S.full[i], (uses - 1) & 1, landing(limit));
    }
  }
  if (parts > 1) {  // no block ends while another may still send to it
    __syncthreads();
    cluster_arrive();
    cluster_wait();
    if (S.dead) {  // all is sent, but nobody waits for it here
      const uint64_t t0 = global_ns();
      while (global_ns() - t0 < kLandNs) __nanosleep(1000);
    }
  }
}

// ---------------------------------------------------------------------------
// Short rows, one a warp
// ---------------------------------------------------------------------------
// Each warp has a buffer of a row and takes rows by itself: the other warps work while it
// waits for its bulk copy. (Two buffers a warp, and half as many warps: 13,463 bf16 rows of
// 4,999 72 us instead of 62.) Nothing is shared with another warp but the sum of the losses at
// the end. cap: vectors of a buffer.
constexpr int kShortWarps = 28;  // of a block at most
constexpr int kShortBatch = 4;   // vectors that a lane takes at once
constexpr int64_t kShortVecs = 1440;         // vectors of a row at most (22.5 KB)
constexpr int64_t kShortBytes = 220 * 1024;  // of all buffers of a block

template <typename T>
__global__ void __launch_bounds__(kShortWarps * 32, 1)
    k_policy_short(Rows<T> R, PolicyArgs P, T* dx, int64_t dld, int cap) {
  constexpr int N = Vec<T>::N;
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ uint64_t full[kShortWarps];
  __shared__ double totals[kShortWarps];
  __shared__ int dead;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  uint4* mine = reinterpret_cast<uint4*>(smem) + (int64_t)warp * cap;
  if (threadIdx.x == 0) dead = 0;
  if (lane == 0) {
    mbar_init(&full[warp], 1);
    fence_mbar_init();
  }
  __syncthreads();
  griddep_wait();
  const int64_t first = (int64_t)warp * gridDim.x + blockIdx.x, step = (int64_t)warps * gridDim.x;
  double total = 0.;
  uint32_t loaded = 0;
  // begin the copy of a row that counts
  auto load = [&](int64_t row, const Facts& f) {
    if (row >= R.n || !f.count()) return;
    ++loaded;
    if (row == P.hold_row) return;
    const T* x = R.x + row * R.ld;
    const Cover<T> c(x, R.V);
    const int64_t v0 = c.first ? 1 : 0, v1 = c.last ? c.nv - 1 : c.nv;
    if (lane == 0 && v1 > v0) {
      const uint32_t bytes = (uint32_t)(v1 - v0) * 16u;
      mbar_expect_tx(&full[warp], bytes);
      bulk_load(mine + v0, x - c.ph + v0 * N, bytes, &full[warp]);
    }
    if (c.first && lane < N) {
      const int64_t j = (int64_t)lane - c.ph;
      reinterpret_cast<T*>(mine)[lane] = j >= 0 && j < R.V ? x[j] : Vec<T>::round(-INFINITY);
    }
    if (c.last && v1 >= v0 && lane < N) {
      const int64_t j = v1 * N - c.ph + lane;
      reinterpret_cast<T*>(mine + v1)[lane] = j < R.V ? x[j] : Vec<T>::round(-INFINITY);
    }
    fence_proxy_async();  // these come before a later bulk copy into the same bytes
    __syncwarp();
    if (lane == 0) mbar_arrive(&full[warp]);
  };
  Facts now = facts_of(R, P, first);
  load(first, now);
  for (int64_t row = first; row < R.n; row += step) {
    const Facts next = facts_of(R, P, row + step);
    const int64_t y = now.y;
    const float w = now.w;
    const bool counts = now.count();
    const T* x = R.x + row * R.ld;
    T* out = dx + row * dld;
    const Cover<T> c(x, R.V);
    const int nv = (int)c.nv;
    const uint4* v = mine;
    RowStats st = {};
    float loss = 0.f, slope = 0.f;
    if (counts) {
      const float xy = target_logit(x, R.V, y);
      const float adv = P.adv[row], old_logp = P.old_logp[row], ref_logp = P.ref_logp ? P.ref_logp[row] : 0.f;
      if (!warp_wait(&full[warp], (loaded - 1) & 1, P.wait_ns)) {
        dead = 1;
        break;
      }
      MaxSum a;
#pragma unroll 1
      for (int k0 = lane; k0 < nv; k0 += 32 * kShortBatch) {
        uint4 q[kShortBatch];
#pragma unroll
        for (int u = 0; u < kShortBatch; ++u)
          q[u] = k0 + 32 * u < nv ? v[k0 + 32 * u] : make_uint4(Vec<T>::kLow, Vec<T>::kLow, Vec<T>::kLow, Vec<T>::kLow);
        add<T>(&a, q, R.b);
      }
      st = finish(warp_merge<T>(a, R.b), xy, R.b);
      if (!st.empty) policy_terms(P, adv, old_logp, ref_logp, st.logp, &loss, &slope);
    }
    if (lane == 0) {
      if (counts && !st.empty) total += (double)w * (double)loss;  // (w may be inf or NaN where nothing counts)
      if (P.token_loss) P.token_loss[row] = loss;
      if (P.logp) P.logp[row] = st.logp;
    }
    if (dx) {
      const bool skip = slope == 0.f || st.empty;  // (0 also where the row does not count)
      const bool same = (reinterpret_cast<uintptr_t>(out) & 15) / sizeof(T) == (unsigned)c.ph;
      const RowGrad g = grad_of(st.h, st.ls, w * slope, y, R.b);
      const int vb = !same ? nv : c.first ? 1 : 0, ve = !same ? nv : c.last ? nv - 1 : nv;
      uint4* dst = reinterpret_cast<uint4*>(out - c.ph);
#pragma unroll 1
      for (int k0 = lane; k0 < ve; k0 += 32 * kShortBatch) {
        uint4 q[kShortBatch];
#pragma unroll
        for (int u = 0; u < kShortBatch; ++u) q[u] = skip ? make_uint4(0, 0, 0, 0) : v[min(k0 + 32 * u, nv - 1)];
#pragma unroll
        for (int u = 0; u < kShortBatch; ++u) {
          const int k = k0 + 32 * u;
          if (!skip) q[u] = grad_vec<T>(q[u], g, R.b);
          if (k >= vb && k < ve) dst[k] = q[u];
        }
      }
      // the rest element by element: the row's ends, or all of a row that lies otherwise
      auto single = [&](int i) {
        const int64_t j = i - c.ph;
        if (j < 0 || j >= R.V) return;
        float f = 0.f;
        if (!skip) {
          const float l = Vec<T>::one(reinterpret_cast<const T*>(v)[i]);
          f = g.f * exp2_fast(g.h.far ? exponent(l - g.h.h, 0.f, R.b) : exponent(l, g.h.hc, R.b));
        }
        out[j] = Vec<T>::round(f);
      };
      if (vb > 0 || ve < nv) {
        for (int i = lane; i < vb * N; i += 32) single(i);
        for (int i = max(ve, vb) * N + lane; i < nv * N; i += 32) single(i);
      }
      __syncwarp();  // the target's own, after what is in its place
      if (lane == 0 && !skip && y < R.V) out[y] = Vec<T>::round(g.k * -expm1f(st.logp));
    }
    __syncwarp();  // every lane has read the buffer
    load(row + step, next);
    now = next;
  }
  // no copy is under way when the block ends
  if (loaded) warp_wait(&full[warp], (loaded - 1) & 1, landing(P.wait_ns));
  if (lane == 0) totals[warp] = total;
  __syncthreads();
  if (warp == 0) {
    total = 0.;
    for (int i = 0; i < warps; ++i) total += totals[i];
    reduce_loss(P, dead ? (double)__uint_as_float(kNan) : total, blockIdx.x, gridDim.x);
  }
}

// ---------------------------------------------------------------------------
// Rows swept twice
// ---------------------------------------------------------------------------
template <typename T>
__global__ void __launch_bounds__(kLossThreads) k_policy(Rows<T> R, PolicyArgs P, T* dx, int64_t dld, int parts) {
  __shared__ MaxSum ws[32], cs[kMaxParts];
  const int64_t cluster = blockIdx.x / parts, clusters = gridDim.x / parts;
  const int part = (int)(blockIdx.x - cluster * parts);
  double total = 0.;
  griddep_wait();
  if (parts > 1) {  // no message before every block has begun
    cluster_arrive();
    cluster_wait();
  }
  for (int64_t row = cluster; row < R.n; row += clusters) {
    const int64_t y = R.y[row];
    const float w = P.weights ? P.weights[row] : P.weight;
    const T* x = R.x + row * R.ld;
    RowStats r = {};
    float loss = 0.f, slope = 0.f;
    const bool counts = y >= 0 && w != 0.f;
    if (counts) {
      const float xy = target_logit(x, R.V, y);
      MaxSum a = block_merge<T>(sweep(x, R.V, R.b, part, parts, (int)threadIdx.x, kLossThreads), R.b, ws);
      a = cluster_merge<T>(a, parts, R.b, cs);
      r = finish(a, xy, R.b);
      if (!r.empty)
        policy_terms(P, P.adv[row], P.old_logp[row], P.ref_logp ? P.ref_logp[row] : 0.f, r.logp, &loss, &slope);
    }
    if (part == 0 && threadIdx.x == 0) {
      if (counts && !r.empty) total += (double)w * (double)loss;
      if (P.token_loss) P.token_loss[row] = loss;
      if (P.logp) P.logp[row] = r.logp;
    }
    // every block has read its x[y] and the shared maxima before dx (perhaps x itself) is
    // written and the next row begins
    if (counts && parts > 1) {
      cluster_arrive();
      cluster_wait();
    } else {
      __syncthreads();
    }
    if (dx)
      write_gradient(x, dx + row * dld, R.V, grad_of(r.h, r.ls, w * slope, y, R.b), R.b,
                     !counts || slope == 0.f || r.empty, part, parts, (int)threadIdx.x, kLossThreads);
  }
  if (part == 0 && threadIdx.x < 32) reduce_loss(P, total, (uint32_t)cluster, (uint32_t)clusters);
}

// The vectors that cover a row at most, whatever its alignment (all rows alike: at theirs).
template <typename T>
int64_t most_vecs(const Rows<T>& R) {
  const int64_t bytes = R.V * (int64_t)sizeof(T);
  const bool alike = (reinterpret_cast<uintptr_t>(R.x) & 15) == 0 && (R.ld * (int64_t)sizeof(T) & 15) == 0;
  return alike ? (bytes + 15) / 16 : (bytes + 15) / 16 + 1;
}

template <typename T>
cudaError_t launch_rows(const Rows<T>& R, const PolicyArgs& A, T* dx, int64_t dld, int64_t nv, Residency* device,
                        cudaStream_t s) {
  const int sms = device->sms;
  // shares of 64 KB at most where 8 blocks a row allow it, and smaller ones while there
  // are blocks without a row
  int parts = 1;
  while (parts < kMaxParts && (nv > (int64_t)parts * 2 * kChunkVecs || (R.n * parts * 2 <= sms && nv > parts * 512)))
    parts *= 2;
  const int per = (int)((nv + parts - 1) / parts);
  const int64_t mine = (R.n * parts + sms - 1) / sms * ((per + kChunkVecs - 1) / kChunkVecs);  // chunks of a block's rows
  int chunks = kMostChunks;
  if (mine < chunks) chunks = (int)mine;
  const int least = (per + kChunkVecs - 1) / kChunkVecs;
  if (chunks < least) chunks = least;
  LaunchConfig l(parts, kRowsThreads, parts, sizeof(RowsShared) + (size_t)chunks * kChunkVecs * 16, s);
  if (parts > 1 && refuse_cooperative()) return cudaErrorCooperativeLaunchTooLarge;
  int64_t clusters = 1;
  const cudaError_t err = device->clusters((const void*)k_policy_rows<T>, l, parts, &clusters);
  if (err != cudaSuccess) return err;
  if (clusters > R.n) clusters = R.n;
  if (clusters > kMostBlocks / parts) clusters = kMostBlocks / parts;
  l.cfg.gridDim.x = (unsigned)(clusters * parts);
  return cudaLaunchKernelEx(&l.cfg, k_policy_rows<T>, R, A, dx, dld, parts, per, chunks);
}

}  // namespace

cudaError_t Residency::clusters(const void* f, const LaunchConfig& l, int parts, int64_t* out) {
  const int threads = (int)l.cfg.blockDim.x;
  const size_t smem = l.cfg.dynamicSmemBytes;
  for (const auto& k : known)
    if (k.f == f && k.threads == threads && k.parts == parts && k.smem == smem) {
      *out = k.clusters;
      return cudaSuccess;
    }
  cudaError_t err = cudaSuccess;
  if (smem > 32 * 1024)  // 48 KB, with the static shared memory, are had without; of 227 KB this leaves that room too
    err = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, 224 * 1024);
  int n = 0;
  if (err == cudaSuccess)
    err = parts > 1 ? cudaOccupancyMaxActiveClusters(&n, f, &l.cfg)
                    : cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, f, threads, smem);
  if (err != cudaSuccess) {
    cudaGetLastError();  // this call's
    return err;
  }
  if (parts == 1) n *= sms;
  if (n < 1) return cudaErrorLaunchOutOfResources;
  known[next] = {f, threads, parts, n, smem};
  next = (next + 1) % 32;
  *out = n;
  return cudaSuccess;
}

template <typename T>
cudaError_t launch_policy(const Rows<T>& R, const PolicyArgs& A, T* dx, int64_t dld, Residency* device, cudaStream_t s) {
  const int64_t nv = most_vecs(R);
  const int sms = device->sms;
  // Short rows, and so many that a lone warp's 10 us for 20 KB do not matter: a warp a row.
  // bf16, in us, by a warp and by the ring: 30,000 x 2,000 52 201, 16,384 x 2,221 44 140, 30,000 x 10,000
  // 200 290, 8,000 x 11,000 74 83, 4,000 x 12,001 51 50, 1,000 x 2,500 9.1 12.0, 1,000 x 10,000 12.7 14.8,
  // 600 x 7,000 9.7 9.2, 310 x 2,500 8.1 8.0, 310 x 7,000 9.5 8.2.
  if (nv <= kShortVecs && R.n > 2 * sms && nv * 16 <= 20 * R.n) {
    const int cap = (int)(nv + 7) / 8 * 8;
    int warps = (int)(kShortBytes / (cap * 16));
    if (warps > kShortWarps) warps = kShortWarps;
    LaunchConfig l(1, warps * 32, 1, (size_t)warps * cap * 16, s);
    int64_t blocks = 1;
    const cudaError_t err = device->clusters((const void*)k_policy_short<T>, l, 1, &blocks);
    if (err != cudaSuccess) return err;
    if (blocks > R.n) blocks = R.n;
    l.cfg.gridDim.x = (unsigned)blocks;
    return cudaLaunchKernelEx(&l.cfg, k_policy_short<T>, R, A, dx, dld, cap);
  }
  if (nv <= kMaxParts * kMostShare) {
    const cudaError_t err = launch_rows<T>(R, A, dx, dld, nv, device, s);
    if (!too_large_here(err)) return err;
    cudaGetLastError();  // this launch's: no room for its clusters in this context
  }
  return with_parts(nv > kMaxParts * kMostShare ? kMaxParts : 1, [&](int parts) {
    int64_t clusters = 2 * sms / parts;
    if (clusters > R.n) clusters = R.n;
    return launch(k_policy<T>, clusters * parts, kLossThreads, parts, s, R, A, dx, dld, parts);
  });
}
template cudaError_t launch_policy<float>(const Rows<float>&, const PolicyArgs&, float*, int64_t, Residency*,
                                                 cudaStream_t);
template cudaError_t launch_policy<__nv_bfloat16>(const Rows<__nv_bfloat16>&, const PolicyArgs&, __nv_bfloat16*, int64_t, Residency*,
                                                 cudaStream_t);
template cudaError_t launch_policy<__half>(const Rows<__half>&, const PolicyArgs&, __half*, int64_t, Residency*,
                                                 cudaStream_t);

}  // namespace gmc
