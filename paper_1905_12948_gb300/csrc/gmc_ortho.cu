// Orthogonalised matrices by Newton-Schulz products: X = G / |G|, then `steps` times
//   A = X X',  B = b A + c A^2,  X <- a X + B X
// with the shorter side of G as X's rows (X is G' where G is taller than wide).
//
// The products run on the tensor cores, from halves, with sums in 32 bits. What is rounded to
// them is chosen so that a result is as good as its type:
//   - A and B are near multiples of the identity once X's rows are orthogonal, and a rounding of
//     their diagonals would act on all of X. They are kept as a diagonal in 32 bits and the rest,
//       A = D + O,  B = E + R:  A^2 = O^2 + D O + O D + D^2,  X <- (a + E_i) X + R X,
//     where the matrix products take O, R and X alone.
//   - X is two halves, 22 bits, the second one what the first one left. The first steps multiply small
//     singular values by `a` each, and a rounding of X to 11 bits with them: 3.4^5 of 2^-12
//     would be left of it. Products take the first half (bfloat16 matrices: the result is off by 2 to 8e-4,
//     its own rounding by 1.7e-3), or the terms hi hi + hi lo + lo hi (float: 0.6 to 1.5e-6, where 32-bit arithmetic
//     is off by 2.3 to 5e-6).
// X is kept 2^14 times, O and R 2^11 times what they are: the second halves then stay normal
// numbers, and a singular value of X may come to 4, one of A or B (less their diagonals) to 32.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>

#include <cuda.h>

#include "gmc.h"
#include "gmc_device.cuh"
#include "gmc_internal.h"
#include "gmc_loss.cuh"
#include "gmc_vec.cuh"

using namespace gmc;

namespace {

constexpr int kMostSteps = 16;
constexpr int64_t kMostWork = int64_t(1) << 38;  // bytes: 2^31 rows of 128
constexpr float kX = 16384.f, kO = 2048.f;  // the scales of X, and of O and R

// m <= n: X's sides; padded to whole blocks. Halves lie in blocks of 128 rows x 64 columns, 16 KB
// each, as shared memory holds them for the tensor cores: rows of 128 bytes, whose 16-byte
// pieces are permuted by the row's last three bits. A block is one copy, whatever it is used as.
struct Shape {
  int64_t m, n, mp, np;
  __host__ __device__ int64_t x() const { return mp * np; }
  __host__ __device__ int64_t o() const { return mp * mp; }
};
constexpr int kBlock = 128 * 64;  // halves of a block
__device__ __forceinline__ uint32_t piece_at(uint32_t row, uint32_t piece) { return row * 128 + ((piece ^ (row & 7)) << 4); }

// Whether factors are the sum of two halves: where the result keeps more bits than one has.
template <typename T>
constexpr bool kOfTwo = !std::is_same<T, __nv_bfloat16>::value;

struct Halves2 {
  __half *hi, *lo;
};
// What this thread wrote is seen by copies that follow (another launch's).
__device__ __forceinline__ void fence_proxy_async_all() { asm volatile("fence.proxy.async;" ::: "memory"); }
// Two numbers as sums of two halves each.
__device__ __forceinline__ void two_halves(float x, float y, __half2* hi, __half2* lo) {
  *hi = __floats2half2_rn(x, y);
  const float2 back = __half22float2(*hi);
  float a, b;
  split(add_pair(pair_of(x, y), pair_of(-back.x, -back.y)), &a, &b);
  *lo = __floats2half2_rn(a, b);
}

// What makes v of a matrix X: a power of two that puts the norm near 1 is taken out, in two steps (either
// may be large), then the rest, 1 / [1, 2), in two words: an error of the norm is one of all singular values,
// which five steps may multiply by tens.
struct Scaled {
  float p1, p2, q, low;
  __device__ __forceinline__ float operator()(float v) const {
    v = v * p1 * p2;
    return __fmaf_rn(v, q, v * low);
  }
};
__device__ __forceinline__ float power2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }  // -126 <= e <= 127
__device__ __forceinline__ Scaled scaled_by(double squares) {
  const uint64_t bits = (uint64_t)__double_as_longlong(squares);
  const int biased = (int)(bits >> 52);  // (no sum of squares of floats is below 2^-298 but 0)
  if (biased >= 0x7ff) return Scaled{1.f, 1.f, __uint_as_float(kNan), 0.f};
  if (biased == 0) return Scaled{1.f, 1.f, 0.f, 0.f};
  const int e = (biased - 1023) >> 1;  // squares = 4^e r, r in [1, 4)
  const double r = __longlong_as_double((long long)((bits & 0xfffffffffffffull) | (uint64_t)(biased - 2 * e) << 52));
  // r^(-1/2): that of 32 bits, off by some 2^-23, and a step of Newton's
  const double y = (double)rsqrtf((float)r), q = (double)kX * __fma_rn(0.5 * y, __fma_rn(-(r * y), y, 1.), y);
  return Scaled{power2(-(e / 2)), power2(-(e - e / 2)), (float)q, (float)(q - (double)(float)q)};
}

// The squares of N numbers added up: in 32 bits, with a power of two taken out where they would
// not fit, so that the sum is the same at any magnitude.
template <int N>
__device__ __forceinline__ double squares(const float* f) {
  float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < N; ++i) s[i % 4] = __fmaf_rn(f[i], f[i], s[i % 4]);
  float sum = (s[0] + s[1]) + (s[2] + s[3]);
  if (sum > 0x1p-90f && sum < 0x1p100f) return (double)sum;
  float most = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) most = fmaxf(most, fabsf(f[i]));
  if (sum != sum || most == INFINITY) return (double)sum;
  if (most == 0.f) return 0.;
  int e;
  frexpf(most, &e);
  const float p1 = power2(-(e / 2)), p2 = power2(-(e - e / 2));
#pragma unroll
  for (int i = 0; i < 4; ++i) s[i] = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float x = f[i] * p1 * p2;
    s[i % 4] = __fmaf_rn(x, x, s[i % 4]);
  }
  sum = (s[0] + s[1]) + (s[2] + s[3]);
  return ldexp((double)sum, 2 * e);
}
// Sums of squares of parts of each matrix G (as it is given: m rows of n), in a fixed order: warps
// take rows, or pieces of 4,096 elements of them. Bound by memory (2 x 4,096 x 25,088 bf16: 67 us, 6.1 TB/s; 8 x
// 1,000 x 4,096, as many blocks as are resident: 15.7 us, twice as many 16.6).
constexpr int kMostSizeParts = 256, kSizePiece = 4096;
template <typename T>
__global__ void __launch_bounds__(256, 4) k_size(const T* g, int64_t sk, int64_t ld, int64_t m, int64_t n, double* part,
                                              uint32_t* counts, int64_t counters) {
  constexpr int N = Vec<T>::N;
  __shared__ double ws[8];
  griddep_wait();
  for (int64_t i = (blockIdx.y * (int64_t)gridDim.x + blockIdx.x) * 256 + threadIdx.x; i < counters;
       i += (int64_t)gridDim.x * gridDim.y * 256)
    counts[i] = 0;
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int64_t pieces = (n + kSizePiece - 1) / kSizePiece;
  double s = 0.;
  for (int64_t w = blockIdx.x * 8 + warp; w < m * pieces; w += gridDim.x * 8) {
    const int64_t at = w % pieces * kSizePiece;
    const T* x = g + blockIdx.y * sk + w / pieces * ld + at;
    const int len = (int)(n - at < kSizePiece ? n - at : kSizePiece);
    int head = (int)((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / (int)sizeof(T);
    if (head > len) head = len;
    const int nv = (len - head) / N, tail = len - head - nv * N;
    if (lane < head + tail) {
      float v = Vec<T>::one(x[lane < head ? lane : len - tail + (lane - head)]);
      s += squares<1>(&v);
    }
    for (int i = lane; i < nv; i += 4 * 32) {
      uint4 v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        v[u] = i + u * 32 < nv ? *reinterpret_cast<const uint4*>(x + head + (i + u * 32) * N) : make_uint4(0, 0, 0, 0);
      float f[4 * N];
#pragma unroll
      for (int u = 0; u < 4; ++u) Vec<T>::get(v[u], f + u * N);
      s += squares<4 * N>(f);
    }
  }
  s = warp_sum(s);
  if (lane == 0) ws[warp] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < 8; ++i) s += ws[i];
    part[blockIdx.y * kMostSizeParts + blockIdx.x] = s;
  }
}
// The parts of a matrix added up, by a warp, in a fixed order.
__device__ __forceinline__ double squares_of(const double* part, int parts) {
  double s = 0.;
  for (int i = (int)threadIdx.x % 32; i < parts; i += 32) s += part[i];
  return warp_sum(s);
}
// The four pieces (8 columns of a row) of a block of halves that are a thread's: neighbours along a row
// of G, whichever way X lies.
template <bool kTurned>
__device__ __forceinline__ void piece_of(int u, int* row, int* piece) {
  const int t = (int)threadIdx.x;
  *row = kTurned ? t % 128 : t / 8 + 32 * u;
  *piece = kTurned ? t / 128 + 2 * u : t % 8;
}
// X = G / |G| as two halves, a block of them by a block. Bound by memory, G (from the L2 cache where it fits) and four
// bytes an element written: 8 x 1,000 x 4,096 bf16 43 us, 4.6 TB/s, 2 x 4,096 x 25,088 231 us, 5.3 TB/s. (Half a block
// at a time with the next one's loads before: the same.) Turned, by loads of single elements: 72 us.
template <typename T, bool kTurned>
__global__ void __launch_bounds__(256) k_first(const T* g, int64_t sk, int64_t ld, Shape S, const double* part, int parts,
                                               Halves2 X) {
  griddep_wait();
  const int64_t k = blockIdx.y, xc = S.np / 64, blocks = S.x() / kBlock;
  const Scaled by = scaled_by(squares_of(part + k * kMostSizeParts, parts));
  const bool vectors = !kTurned && ((reinterpret_cast<uintptr_t>(g) | (uintptr_t)(ld * sizeof(T)) | (uintptr_t)(sk * sizeof(T))) & 15) == 0;
  for (int64_t block = blockIdx.x; block < blocks; block += gridDim.x) {
    const int64_t rb = block / xc, cb = block % xc, to = k * S.x() + block * kBlock;
    float f[4][8];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      int row, piece;
      piece_of<kTurned>(u, &row, &piece);
      const int64_t i = rb * 128 + row, j0 = cb * 64 + piece * 8;
      const T* x = g + k * sk + (kTurned ? j0 * ld + i : i * ld + j0);
      if (vectors && i < S.m && j0 + 8 <= S.n) {
#pragma unroll
        for (int v = 0; v < 8; v += Vec<T>::N) Vec<T>::get(*reinterpret_cast<const uint4*>(x + v), f[u] + v);
      } else {
#pragma unroll
        for (int v = 0; v < 8; ++v) f[u][v] = i < S.m && j0 + v < S.n ? Vec<T>::one(x[v * (kTurned ? ld : 1)]) : 0.f;
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      int row, piece;
      piece_of<kTurned>(u, &row, &piece);
      const int64_t i = rb * 128 + row, j0 = cb * 64 + piece * 8;
      alignas(16) __half2 hi[4], lo[4];
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        float x[2];
#pragma unroll
        for (int o = 0; o < 2; ++o)  // (what pads a matrix that is NaN stays 0)
          x[o] = i < S.m && j0 + 2 * v + o < S.n ? by(f[u][2 * v + o]) : 0.f;
        two_halves(x[0], x[1], hi + v, lo + v);
      }
      const uint32_t in = piece_at((uint32_t)row, (uint32_t)piece);
      *reinterpret_cast<uint4*>(reinterpret_cast<char*>(X.hi + to) + in) = *reinterpret_cast<uint4*>(hi);
      *reinterpret_cast<uint4*>(reinterpret_cast<char*>(X.lo + to) + in) = *reinterpret_cast<uint4*>(lo);
    }
  }
  fence_proxy_async_all();
}
// NaN for all of the result where a wait has given up. (The products write the result themselves. 1.8 us.)
template <typename T>
__global__ void __launch_bounds__(256) k_gave_up(T* out, int64_t sk, int64_t ld, int64_t m, int64_t n, const uint32_t* gave_up) {
  griddep_wait();
  if (!*gave_up) return;
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < m * n; i += gridDim.x * 256ll)
    out[blockIdx.y * sk + i / n * ld + i % n] = Vec<T>::round(__uint_as_float(kNan));
}

// -- products on the tensor cores ------------------------------------------------

__device__ __forceinline__ uint32_t remote(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
// Says that an accumulator was read, to the block that issues the products. Across blocks without a release: what comes
// before it are reads of tensor memory, which have ended, and a release would wait for all of the thread's stores
// (1,000 cycles).
template <int CG>
__device__ __forceinline__ void arrive_first(uint64_t* bar) {
  if constexpr (CG == 1) mbar_arrive(bar);
  else asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(remote(smem_addr(bar), 0)) : "memory");
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
// What a block's waits have in common: whether one of its threads has given up, and after how long they do.
struct Patience {
  volatile uint32_t* dead;
  uint64_t ns;
};
// As wait_bounded, ordered after arrivals from the other block of the cluster; gives up at once where
// a thread of this block has given up. (The timer takes longer to read than most waits last: it is
// looked at every 256th time.)
__device__ __forceinline__ bool wait_for(uint64_t* bar, uint32_t parity, const Patience& p) {
  uint64_t t0 = 0;
  for (uint32_t n = 1; !try_wait_cluster(bar, parity); ++n) {
    if (n % 256) continue;
    if (*p.dead) return false;
    const uint64_t now = global_ns();
    if (t0 == 0) t0 = now;
    if (now - t0 > p.ns) {
      *p.dead = 1;
      return false;
    }
  }
  return true;
}

// Until a count that others raise has come to `to`.
__device__ __forceinline__ bool wait_count(const uint32_t* count, uint32_t to, const Patience& p) {
  uint64_t t0 = 0;
  for (uint32_t n = 1;; ++n) {
    uint32_t v;
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(count) : "memory");
    if (v >= to) return true;
    if (n % 64) continue;
    if (*p.dead) return false;
    const uint64_t now = global_ns();
    if (t0 == 0) t0 = now;
    if (now - t0 > p.ns) {
      *p.dead = 1;
      return false;
    }
  }
}

template <int CG>
__device__ __forceinline__ void tmem_alloc(uint32_t* to, uint32_t columns) {
  if constexpr (CG == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(to)), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  } else {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(to)), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
  }
}
template <int CG>
__device__ __forceinline__ void tmem_free(uint32_t at, uint32_t columns) {
  if constexpr (CG == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns));
  else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns));
}
// d += a b (d = a b without `add`), K = 16.
template <int CG>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t what, bool add) {
  if constexpr (CG == 1)
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(what), "r"((uint32_t)add)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(what), "r"((uint32_t)add)
        : "memory");
}
// Arrives at `bar` (in both blocks of a pair) once all products issued so far are done.
template <int CG>
__device__ __forceinline__ void commit(uint64_t* bar) {
  if constexpr (CG == 1)
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
  else
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
                     smem_addr(bar)),
                 "h"((uint16_t)3)
                 : "memory");
}
// kStep columns of a warp's 32 rows of tensor memory, and back.
constexpr int kStep = 16;
__device__ __forceinline__ void tmem_load(uint32_t at, float (&f)[kStep]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=f"(f[0]), "=f"(f[1]), "=f"(f[2]), "=f"(f[3]), "=f"(f[4]), "=f"(f[5]), "=f"(f[6]), "=f"(f[7]), "=f"(f[8]),
        "=f"(f[9]), "=f"(f[10]), "=f"(f[11]), "=f"(f[12]), "=f"(f[13]), "=f"(f[14]), "=f"(f[15])
      : "r"(at));
}
__device__ __forceinline__ void tmem_store(uint32_t at, const float* f) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(at),
      "f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]), "f"(f[4]), "f"(f[5]), "f"(f[6]), "f"(f[7]), "f"(f[8]), "f"(f[9]),
      "f"(f[10]), "f"(f[11]), "f"(f[12]), "f"(f[13]), "f"(f[14]), "f"(f[15])
      : "memory");
}
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// (The registers are named: nothing may look at them before.)
__device__ __forceinline__ void tmem_loaded(float (&f)[kStep]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+f"(f[0]), "+f"(f[1]), "+f"(f[2]), "+f"(f[3]), "+f"(f[4]), "+f"(f[5]), "+f"(f[6]), "+f"(f[7]),
                 "+f"(f[8]), "+f"(f[9]), "+f"(f[10]), "+f"(f[11]), "+f"(f[12]), "+f"(f[13]), "+f"(f[14]), "+f"(f[15])
               :
               : "memory");
}
// Shared memory of a factor: rows of 128 bytes, eight of them (1 KB) a group; `stride` bytes
// from one 64-column block to the next where the factor's rows are the sum's index.
__device__ __forceinline__ uint64_t factor(uint32_t addr, uint32_t stride) {
  return (uint64_t)((addr & 0x3ffff) >> 4) | (uint64_t)(stride >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 |
         (uint64_t)2 << 61;
}
__device__ __forceinline__ void bulk_store(void* to, const void* from, uint32_t bytes) {
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(to), "r"(smem_addr(from)), "r"(bytes)
               : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
// Until all stores have read what they store.
__device__ __forceinline__ void bulk_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void bulk_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

// A copy of 64 rows of 128 bytes; row `at` of the workspace. With pairs of blocks the bytes are counted by the barrier of the
// block that issues the products.
template <int CG>
__device__ __forceinline__ void tile_load(void* to, const CUtensorMap* map, int64_t at, uint32_t bar) {
  if constexpr (CG == 1)
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
            smem_addr(to)),
        "l"(map), "r"(0), "r"((int)at), "r"(bar)
        : "memory");
  else
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], "
        "[%4];" ::"r"(smem_addr(to)),
        "l"(map), "r"(0), "r"((int)at), "r"(bar)
        : "memory");
}

enum Phase { kGram, kSquare, kUpdate };  // A = X X';  B = b A + c A^2;  X <- a X + B X

struct ProductArgs {
  Shape S;
  int64_t K;
  const __half* base;   // of the workspace, which the map is of
  Halves2 x[2], o, r;   // X before and after each step, in turn; O, R
  float *d, *e;         // diagonals of A and B, mp each
  int begin, end;       // phases of this launch, three a step
  int last;             // the phase that writes the result: element (i, j) of X at out + k * sk + i * si + j * sj, by
  void* out;            // `scale`
  int64_t sk, si, sj;
  float scale;
  bool triangle[2];     // of A, of B: tiles on and below the diagonal
  int64_t whole;        // tiles of A that one block (or pair) sums alone,
  int splits;           // and in how many shares the others are summed
  float* shares;        // their sums,
  uint32_t* shared;     // and how many of them are there, by warps
  uint32_t* phases;     // counts the blocks that are done with each
  uint64_t wait_ns;     // bound of every wait
  bool hold;            // test hook: the first block does not say that it is done
  uint32_t* gave_up;
  float coef[3 * kMostSteps];
};
template <int P>
struct PhaseOf {
  static constexpr int value = P;
};

constexpr int kFactorBytes = 16384;  // of a stage: 128 rows, or columns, by 64
constexpr int kHeldBytes = 4096;     // a warp's part of a block of halves
template <int CG, typename T>
struct Plan {
  static constexpr bool kFine = kOfTwo<T>;
  // Warps that read the sums back, 32 rows each; 64 columns at a time, with as many parts of a block (two
  // halves) on their way to it.
  static constexpr int kWarps = CG == 2 && !kFine ? 4 : 8;
  static constexpr int kBuffers = kFine ? 1 : 2;
  // Of pairs' factors that are two halves, the second halves are a stage and the first ones the next: the second ones
  // are free again before the last third of the products, and their next ones under way (4 x 2,417 x 4,507 fp32: 4,510 -> 4,310
  // us, half 4,300 -> 4,010; single blocks wait for their port to the L2 cache: 4 x 700 x 900 277 us so, 287 in parts).
  static constexpr int kHalves = kFine ? 2 : 1, kParts = CG == 2 ? kHalves : 1;
  static constexpr int kStages = kFine ? 2 * kParts : CG == 1 ? 3 : 5;
  static constexpr int kStageBytes = 2 * kHalves / kParts * kFactorBytes;
  static constexpr int kItems = 8 * CG / kWarps;  // of a warp, 64 columns each
  static constexpr int kThreads = 64 + 32 * kWarps;
  static constexpr int kHeld = kWarps * kBuffers * 2 * kHeldBytes;
  // Sums in the tensor cores are cut off, not rounded: by a quarter of a last place an addition where
  // all terms have one sign, as on A's diagonal (4,608 columns of fp32 matrices: 2.8e-5 off the result, by three
  // additions for 16 columns). They are added up in registers after so many stages. float: A after 128 columns, the
  // others, whose terms have either sign, after 256 (8 x 512 x 4,608: 9e-7 off, 626 us; after 128 8e-7, 655; after 512
  // 1.2e-6, 610, but 2.5e-6 for 1,024 x 1,024, where 32-bit arithmetic is 3e-6 off). half: A after 2,048 columns (its
  // own rounding is 2e-4; 4 x 2,417 x 4,507 4,630 -> 4,230 us).
  __host__ __device__ static constexpr int chunk(int phase) {
    return std::is_same<T, float>::value ? (phase == kGram ? 2 : 4) : kFine && phase == kGram ? 32 : 1 << 30;
  }
};
struct alignas(8) ProductBars {
  uint64_t full[5], empty[5];
  uint64_t sums[2], taken[2];  // accumulators: written, read back
  uint64_t held[8][2];
  uint64_t phase;              // the phases before the next one are done
  uint32_t tmem, dead;
};
template <int CG, typename T>
constexpr int product_smem() {
  using Pl = Plan<CG, T>;
  return Pl::kStages * Pl::kStageBytes + Pl::kHeld + 1024 + (int)sizeof(ProductBars);
}

// Tiles of all K matrices. A and B are symmetric: the tiles on and below the diagonal do, where that
// saves more than writing each of them twice takes.
struct Tiles {
  int rows, cols;  // of a matrix; cols = 0: a triangle
  int64_t each, all;
  __device__ Tiles(const Shape& S, int64_t K, int unit, bool symmetric, bool triangle) {
    rows = (int)(S.mp / unit);
    cols = !symmetric ? (int)(S.np / unit) : triangle ? 0 : rows;
    each = cols ? (int64_t)rows * cols : (int64_t)rows * (rows + 1) / 2;
    all = each * K;
  }
  // (a workspace of kMostWork holds less than 2^24 of them)
  __device__ void at(int64_t t, int64_t* k, int* row, int* col) const {
    const uint32_t n = (uint32_t)t / (uint32_t)each;
    *k = n;
    const int i = (int)((uint32_t)t - n * (uint32_t)each);
    if (cols) {
      *row = i % rows;
      *col = i / rows;
    } else {
      int r = (int)((sqrtf(8.f * (float)i + 1.f) - 1.f) * 0.5f);
      while ((int64_t)r * (r + 1) / 2 > i) --r;
      while ((int64_t)(r + 1) * (r + 2) / 2 <= i) ++r;
      *row = r;
      *col = i - r * (r + 1) / 2;
    }
  }
};

// The units of work of a phase: tiles, then, of A, shares of tiles, a part of X's columns each. (Tiles that are too
// few for another round of all blocks are shared.)
struct Parts {
  int splits, kblocks, per;
  int64_t whole, all;
  __device__ Parts(const ProductArgs& P, const Tiles& tiles, int phase) {
    splits = phase == kGram ? P.splits : 1;
    kblocks = (int)(((phase == kGram ? P.S.n : P.S.m) + 63) / 64);
    per = (kblocks + splits - 1) / splits;
    whole = splits > 1 ? P.whole : tiles.all;
    all = whole + (tiles.all - whole) * splits;
  }
  // its tile, and blocks of 64 of the sum
  __device__ void at(int64_t unit, int64_t* t, int* begin, int* end) const {
    *t = unit < whole ? unit : whole + (uint32_t)(unit - whole) / (uint32_t)splits;
    *begin = unit < whole ? 0 : split_of(unit) * per;
    *end = unit < whole || *begin + per > kblocks ? kblocks : *begin + per;
  }
  __device__ int split_of(int64_t unit) const { return (int)((uint32_t)(unit - whole) % (uint32_t)splits); }
};

// The phases of all steps, with a barrier over the grid between two of them (the blocks are resident together);
// or one of them. A block holds 128 rows of the left factor and 128 rows (columns
// in kUpdate) of the right one, 64 of the sum at a time; a pair of blocks (CG = 2) shares them, and its tile
// is 256 x 256, 128 x 256 of it in each block's tensor memory; CG = 1: 128 x 128.
// Warp 0 issues the copies, warp 1 the products; the others read the sums back (the tensor memory
// holds two tiles) and put the new halves where the next product takes them from, or the result into its place.
// What bounds it: with deep sums the tensor cores under the power limit (2 x 4,096 x 25,088 bf16: 1.36 to 1.48 PFLOP/s, by card; cuBLAS
// 1.89 in a burst, 1.72 sustained); with short ones a block's port to the L2 cache, 53 to 60 bytes a cycle for the
// factors and X, which is read and written whole (8 x 1,000 x 4,096: 16,500 cycles for a tile of 256 x 256, of which
// the products take 8,200); with few tiles the barriers and the first copies after them (8 x 256 x 256: 6.5 us a
// phase). Pairs of blocks, with tiles of 256 x 256, halve the factors' bytes; see course_of().
template <int CG, typename T>
__global__ void __launch_bounds__(Plan<CG, T>::kThreads, 1) k_products(const __grid_constant__ CUtensorMap map,
                                                                            const __grid_constant__ ProductArgs P) {
  constexpr bool kFine = kOfTwo<T>;
  using Pl = Plan<CG, T>;
  extern __shared__ char raw[];
  char* smem = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  char* held = smem + Pl::kStages * Pl::kStageBytes;
  ProductBars& bars = *reinterpret_cast<ProductBars*>(held + Pl::kHeld);
  const int warp = (int)threadIdx.x / 32, lane = (int)threadIdx.x % 32;
  const uint32_t rank = CG == 2 ? cluster_rank() : 0;
  constexpr uint32_t kColumns = CG * 128;  // of an accumulator

  const Shape S = P.S;
  const int64_t xc = S.np / 64, oc = S.mp / 64;  // blocks in a row of blocks
  const int64_t first = blockIdx.x / CG, step = gridDim.x / CG;

  if (threadIdx.x == 0) {
    for (int i = 0; i < Pl::kStages; ++i) {
      mbar_init(&bars.full[i], 1);
      mbar_init(&bars.empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars.sums[i], 1);
      mbar_init(&bars.taken[i], Pl::kWarps * CG);
    }
    for (int w = 0; w < Pl::kWarps; ++w) mbar_init(&bars.held[w][0], 1), mbar_init(&bars.held[w][1], 1);
    mbar_init(&bars.phase, 1);
    bars.dead = 0;
    fence_mbar_init();
  }
  if (warp == 1) tmem_alloc<CG>(&bars.tmem, 2 * kColumns);
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (CG == 2) {
    cluster_arrive();
    cluster_wait();
  }
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = *(volatile uint32_t*)&bars.tmem;
  const Patience patience{&bars.dead, P.wait_ns};
  griddep_wait();

  // Until every block is done with the phases before this one. The thread that issues the copies looks at the count
  // and tells the others of its block.
  auto wait_phase = [&](int index, bool first_of_block) {
    if (index == P.begin) return true;
    bool there;
    if (first_of_block) {
      there = wait_count(P.phases, (uint32_t)(index - P.begin) * gridDim.x, patience);
      if (there) mbar_arrive(&bars.phase);
    } else {
      there = wait_for(&bars.phase, (index - P.begin - 1) & 1, patience);
    }
    fence_proxy_async_all();
    return there;
  };
  auto each_phase = [&](auto&& f) {
    for (int i = P.begin; i < P.end; ++i) {
      const Halves2& x = P.x[i / 3 & 1];
      if (i % 3 == kGram) f(PhaseOf<kGram>(), i, x);
      else if (i % 3 == kSquare) f(PhaseOf<kSquare>(), i, x);
      else f(PhaseOf<kUpdate>(), i, x);
    }
  };

  if (warp == 0) {
    if (lane == 0) {
      uint32_t n = 0;  // stages filled
      bool going = true;
      each_phase([&](auto phase, int index, const Halves2& x) {
        constexpr int kPhase = decltype(phase)::value;
        const Tiles tiles(S, P.K, 128 * CG, kPhase != kUpdate, kPhase != kUpdate && P.triangle[kPhase % kUpdate]);
        const Parts parts(P, tiles, kPhase);
        going = going && wait_phase(index, true);
        const Halves2 left = kPhase == kGram ? x : kPhase == kSquare ? P.o : P.r;
        const Halves2 right = kPhase == kSquare ? P.o : x;
        // rows of 64 halves from the workspace's beginning
        const int64_t lh = (left.hi - P.base) / 64, rh = (right.hi - P.base) / 64;
        const int64_t ll = kFine ? (left.lo - left.hi) / 64 : 0, rl = kFine ? (right.lo - right.hi) / 64 : 0;
        const int64_t lk = (kPhase == kGram ? S.x() : S.o()) / 64, rk = (kPhase == kSquare ? S.o() : S.x()) / 64;
        const int64_t lc = kPhase == kGram ? xc : oc, rc = kPhase == kSquare ? oc : xc;
        for (int64_t unit = first; unit < parts.all && going; unit += step) {
          int64_t t, k;
          int begin, end, row, col;
          parts.at(unit, &t, &begin, &end);
          tiles.at(t, &k, &row, &col);
          const int64_t ra = (int64_t)row * CG + rank, rb = (int64_t)col * CG + rank;
          for (int kb = begin; kb < end && going; ++kb) {
#pragma unroll
            for (int part = Pl::kParts - 1; part >= 0; --part, ++n) {
              const int s = (int)(n % Pl::kStages);
              if (n >= Pl::kStages && !wait_for(&bars.empty[s], (n / Pl::kStages - 1) & 1, patience)) {
                going = false;
                break;
              }
              char* to = smem + s * Pl::kStageBytes;
              const uint32_t bar = CG == 1 ? smem_addr(&bars.full[s]) : remote(smem_addr(&bars.full[s]), 0);
              if (rank == 0) mbar_arrive_expect_tx(&bars.full[s], CG * Pl::kStageBytes);
#pragma unroll
              for (int h = 0; h < 2; ++h) {  // 64 rows each
                char* at = to + h * (kFactorBytes / 2);
                const int64_t l = lh + lk * k + (ra * lc + kb) * 128 + h * 64;
                const int64_t r = rh + rk * k + (kPhase == kUpdate ? ((kb / 2) * rc + rb * 2 + h) * 128 + (kb & 1) * 64
                                                                   : (rb * rc + kb) * 128 + h * 64);
                tile_load<CG>(at, &map, l + part * ll, bar);
                tile_load<CG>(at + kFactorBytes, &map, r + part * rl, bar);
                if (Pl::kHalves > Pl::kParts) {
                  tile_load<CG>(at + 2 * kFactorBytes, &map, l + ll, bar);
                  tile_load<CG>(at + 3 * kFactorBytes, &map, r + rl, bar);
                }
              }
            }
          }
        }
      });
      // what is under way has landed before the block ends
      if (rank == 0)
        for (uint32_t i = n > Pl::kStages ? n - Pl::kStages : 0; i < n; ++i)
          wait_bounded(&bars.full[i % Pl::kStages], (i / Pl::kStages) & 1, kWaitLimitNs);
      if (!going)  // (the other block's barrier may not count all of it)
        for (const uint64_t t0 = global_ns(); global_ns() - t0 < 2000000;) {}
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      uint32_t n = 0, it = 0;
      bool going = true;
      each_phase([&](auto phase, int, const Halves2&) {
        constexpr int kPhase = decltype(phase)::value;
        const Tiles tiles(S, P.K, 128 * CG, kPhase != kUpdate, kPhase != kUpdate && P.triangle[kPhase % kUpdate]);
        const Parts parts(P, tiles, kPhase);
        // 32-bit sums of halves; the right factor's rows are the sum's index in kUpdate
        constexpr int kChunk = Pl::chunk(kPhase);
        constexpr uint32_t what = 1u << 4 | (kPhase == kUpdate ? 1u << 16 : 0) | (CG * 128 / 8) << 17 | (CG * 128 / 16) << 24;
        for (int64_t unit = first; unit < parts.all && going; unit += step) {
          int64_t t;
          int kb, last;
          parts.at(unit, &t, &kb, &last);
          while (kb < last && going) {
            const uint32_t acc = tmem + (it & 1) * kColumns;
            going = it < 2 || wait_for(&bars.taken[it & 1], (it / 2 - 1) & 1, patience);
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const int begin = kb, end = last - kb > kChunk ? kb + kChunk : last;
            for (; kb < end && going; ++kb, n += Pl::kParts) {
              // the stage of the first halves, and before it that of the second ones (the same where they are not apart)
              const uint32_t first_n = n + Pl::kParts - 1;
              const int s = (int)(first_n % Pl::kStages), t = (int)(n % Pl::kStages);
              going = wait_for(&bars.full[t], (n / Pl::kStages) & 1, patience);
              if (Pl::kParts == 2) going = going && wait_for(&bars.full[s], (first_n / Pl::kStages) & 1, patience);
              if (!going) break;
              asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
              const uint32_t at = smem_addr(smem + s * Pl::kStageBytes);
              constexpr uint32_t apart = kPhase == kUpdate ? kFactorBytes / 2 : 0;
              const uint64_t l = factor(at, 0), r = factor(at + kFactorBytes, apart);
              // 16 of the sum at a time: 32 bytes of each row, or 16 rows
              auto left = [](int q) { return (uint64_t)(q * 32 >> 4); };
              auto right = [](int q) { return (uint64_t)((kPhase == kUpdate ? q * 2048 : q * 32) >> 4); };
              if (kFine) {  // the small terms first, while there is less to cut off
                const uint32_t low = Pl::kParts == 2 ? smem_addr(smem + t * Pl::kStageBytes) : at + 2 * kFactorBytes;
                const uint64_t ll = factor(low, 0), rl = factor(low + kFactorBytes, apart);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                  mma<CG>(acc, l + left(q), rl + right(q), what, kb > begin || q > 0);
                  mma<CG>(acc, ll + left(q), r + right(q), what, true);
                }
                if (Pl::kParts == 2) commit<CG>(&bars.empty[t]);
              }
#pragma unroll
              for (int q = 0; q < 4; ++q) mma<CG>(acc, l + left(q), r + right(q), what, kFine || kb > begin || q > 0);
              commit<CG>(&bars.empty[s]);
            }
            if (going) commit<CG>(&bars.sums[it & 1]);
            ++it;
          }
        }
      });
      // the last products are done before the tensor memory is given back
      for (uint32_t i = n > Pl::kStages ? n - Pl::kStages : 0; i < n; ++i)
        wait_bounded(&bars.empty[i % Pl::kStages], (i / Pl::kStages) & 1, kWaitLimitNs);
    }
  } else {
    const int w = warp & 3, e = (warp - 2) / 4;  // rows 32 w of the block's part of the tile, columns 64 kItems e
    char* own = held + (warp - 2) * Pl::kBuffers * 2 * kHeldBytes;
    uint64_t* in = bars.held[warp - 2];
    uint32_t fetched = 0, q = 0, it = 0;  // parts of blocks on their way or read, read; accumulators read
    bool going = true;
    each_phase([&](auto phase, int index, const Halves2& x) {
      constexpr int kPhase = decltype(phase)::value;
      const Tiles tiles(S, P.K, 128 * CG, kPhase != kUpdate, kPhase != kUpdate && P.triangle[kPhase % kUpdate]);
      const Parts parts(P, tiles, kPhase);
      const float c1 = P.coef[index / 3 * 3], c3 = P.coef[index / 3 * 3 + 1], c5 = P.coef[index / 3 * 3 + 2];
      going = __all_sync(0xffffffffu, going && (lane != 0 || wait_phase(index, false)));
      __syncwarp();  // (a vote orders no memory: the diagonals that all lanes read are those that lane 0 waited for)
      constexpr bool kLow = kPhase == kUpdate || kFine;  // two halves are kept
      const Halves2 from = kPhase == kUpdate ? x : P.o;
      const Halves2 to = kPhase == kGram ? P.o : kPhase == kSquare ? P.r : P.x[(index / 3 + 1) & 1];
      const int64_t bc = kPhase == kUpdate ? xc : oc, plane = kPhase == kUpdate ? S.x() : S.o();
      // where this warp's part of a tile's first block of halves lies (the next blocks follow it)
      auto part_of = [&](int64_t t) {
        int64_t k;
        int row, col;
        tiles.at(t, &k, &row, &col);
        const int64_t rb = (int64_t)row * CG + rank, cb = ((int64_t)col * (Pl::kWarps / 4) + e) * Pl::kItems;
        return k * plane + (rb * bc + cb) * kBlock + w * (kHeldBytes / 2);
      };
      auto fetch = [&](int64_t at) {  // the next one
        if (kPhase == kGram) return;
        char* to = own + fetched % Pl::kBuffers * 2 * kHeldBytes;
        uint64_t* bar = in + fetched % Pl::kBuffers;
        mbar_arrive_expect_tx(bar, (kLow ? 2 : 1) * kHeldBytes);
        bulk_load(to, from.hi + at, kHeldBytes, bar);
        if (kLow) bulk_load(to + kHeldBytes, from.lo + at, kHeldBytes, bar);
        ++fetched;
      };
      // this warp's sums of one share of tile t, 64 kItems columns of 32 rows
      auto share_of = [&](int64_t t, int split) {
        return P.shares + (((((t - parts.whole) * parts.splits + split) * CG + rank) * Pl::kWarps + warp - 2) * (64 * Pl::kItems)) * 32 + lane;
      };
      // and the count of them
      auto shared = [&](int64_t t) {
        return P.shared + ((t - parts.whole) * CG + rank) * Pl::kWarps + warp - 2;
      };
      if (lane == 0 && going && first < parts.whole) fetch(part_of(first));

      // Items [item, items) of a tile, and `then` the next one (-1: none): `sums(at, acc)` gives kStep columns of its sums, in the order of the columns, `done()` says that all were given.
      auto finish = [&](int64_t t, int64_t then, int item, int items, auto&& sums, auto&& done) {
        int64_t k;
        int tr, tc;
        tiles.at(t, &k, &tr, &tc);
        const int64_t row = ((int64_t)tr * CG + rank) * 128 + w * 32 + lane;
        const int64_t part = part_of(t), next_part = then >= 0 ? part_of(then) : -1;
        // the item after c
        auto fetch_after = [&](int c) {
          if (c + 1 < items) fetch(part + (c + 1) * kBlock);
          else if (next_part >= 0) fetch(next_part);
        };
        // D and E of the row, D of the warp's columns: 32 at a time, a lane each
        const float* D = P.d + k * S.mp;
        [[maybe_unused]] const float dr = kPhase == kSquare ? D[row] : 0.f, di = c3 + c5 * dr;
        [[maybe_unused]] const float ei = kPhase == kUpdate ? c1 + P.e[k * S.mp + row] : 0.f;
        const int64_t cols = ((int64_t)tc * (Pl::kWarps / 4) + e) * (64 * Pl::kItems);  // the warp's first column
        [[maybe_unused]] const float by_out = P.scale * (1.f / kX);
        // (Loops that are not unrolled: each tile goes through this code once, and instructions have to be
        // fetched. 64 columns took 4,500 to 9,000 cycles unrolled.)
#pragma unroll 1
        for (int c = item; c < items; ++c) {
          char* b = own + (kPhase == kGram ? 0 : q % Pl::kBuffers) * 2 * kHeldBytes;
          if (kPhase == kGram || Pl::kBuffers == 2) {
            __syncwarp();                // (the last tile's mirror has been read)
            if (lane == 0) bulk_read();  // the last store
            if (lane == 0 && Pl::kBuffers == 2) fetch_after(c);
            __syncwarp();
          }
          if (kPhase != kGram) {
            going = __all_sync(0xffffffffu, wait_for(in + q % Pl::kBuffers, (q / Pl::kBuffers) & 1, patience));
            ++q;
          }
          if (!going) return;
          // this lane's halves of kStep columns, two pieces of each plane; read a step ahead where there are registers for it
          uint4 halves[2 * kStep / 8];
          auto read = [&](int h) {
#pragma unroll
            for (int p = 0; p < kStep / 8; ++p) {
              const char* at = b + piece_at((uint32_t)lane, (uint32_t)(h / 8 + p));
              halves[2 * p] = *reinterpret_cast<const uint4*>(at);
              if (kLow) halves[2 * p + 1] = *reinterpret_cast<const uint4*>(at + kHeldBytes);
            }
          };
          if (kPhase != kGram && !kFine) read(0);
#pragma unroll 1
          for (int h = 0; h < 64; h += kStep) {  // so many columns, eight a piece
            float was[kStep];
            if (kPhase != kGram) {
              if (kFine) read(h);
#pragma unroll
              for (int p = 0; p < kStep / 8; ++p) {
                Vec<__half>::get(halves[2 * p], was + p * 8);
                if (kLow) {
                  float low[8];
                  Vec<__half>::get(halves[2 * p + 1], low);
#pragma unroll
                  for (int u = 0; u < 8; u += 2) {
                    float* x = was + p * 8 + u;
                    split(add_pair(pair_of(x[0], x[1]), pair_of(low[u], low[u + 1])), x, x + 1);
                  }
                }
              }
              if (!kFine && h + kStep < 64) read(h + kStep);
            }
            // D of the columns, the same for all lanes
            [[maybe_unused]] float dc[kStep];
            if (kPhase == kSquare)
#pragma unroll
              for (int u = 0; u < kStep; u += 4)
                Vec<float>::get(*reinterpret_cast<const uint4*>(D + cols + c * 64 + h + u), dc + u);
            float acc[kStep];
            sums(c * 64 + h, acc);
            // (acc: X X' 2^28 times, O^2 2^22 times, R X 2^25 times)
            const int on = (int)(row - (cols + c * 64 + h));  // the column that is on the diagonal
            if (kPhase != kUpdate && tr == tc && on >= 0 && on < kStep) {
              float mid = 0.f;
#pragma unroll
              for (int u = 0; u < kStep; ++u) mid = u == on ? acc[u] : mid;
              if (kPhase == kGram) P.d[k * S.mp + row] = mid * (1.f / (kX * kX));
              else P.e[k * S.mp + row] = c3 * dr + c5 * __fmaf_rn(dr, dr, mid * (1.f / (kO * kO)));
            }
#pragma unroll
            for (int p = 0; p < kStep / 8; ++p) {
              alignas(16) __half2 nh[4], nl[4];
#pragma unroll
              for (int u = 0; u < 8; u += 2) {
                float v[2];
                const int j = p * 8 + u;
                const Pair sum = pair_of(acc[j], acc[j + 1]);
                auto two = [](float x) { return pair_of(x, x); };
                if constexpr (kPhase == kGram) {
                  split(mul_pair(sum, two(kO / (kX * kX))), v, v + 1);
                } else if constexpr (kPhase == kSquare) {  // b O + c (O^2 + (D_i + D_j) O)
                  split(fma_pair(fma_pair(two(c5), pair_of(dc[j], dc[j + 1]), two(di)), pair_of(was[j], was[j + 1]), mul_pair(sum, two(c5 / kO))), v, v + 1);
                } else {
                  split(fma_pair(two(ei), pair_of(was[j], was[j + 1]), mul_pair(sum, two(1.f / kO))), v, v + 1);
                }
                if (kPhase == kUpdate && index == P.last) {  // what they stand for, in the place of the halves
                  const T r0 = Vec<T>::round(v[0] * by_out), r1 = Vec<T>::round(v[1] * by_out);
                  if (P.sj != 1) {  // (neighbours are the lanes' rows)
                    const int64_t col = cols + c * 64 + h + p * 8 + u;
                    T* o = static_cast<T*>(P.out) + k * P.sk + row * P.si + col * P.sj;
                    if (row < S.m && col < S.n) o[0] = r0;
                    if (row < S.m && col + 1 < S.n) o[P.sj] = r1;
                  } else if constexpr (sizeof(T) == 2) {
                    memcpy(&nh[u / 2], &r0, 2);
                    memcpy(reinterpret_cast<char*>(&nh[u / 2]) + 2, &r1, 2);
                  } else {
                    __half2* four = (u < 4 ? nh : nl) + u % 4;
                    memcpy(four, &r0, 4);
                    memcpy(four + 1, &r1, 4);
                  }
                } else {
                  two_halves(v[0], v[1], nh + u / 2, nl + u / 2);
                }
              }
              char* at = b + piece_at((uint32_t)lane, (uint32_t)(h / 8 + p));
              *reinterpret_cast<uint4*>(at) = *reinterpret_cast<const uint4*>(nh);
              if (kLow) *reinterpret_cast<uint4*>(at + kHeldBytes) = *reinterpret_cast<const uint4*>(nl);
            }
            if (kPhase != kUpdate && tr == tc && on >= 0 && on < kStep) {  // (O and R have none)
              char* place = b + piece_at((uint32_t)lane, (uint32_t)((h + on) / 8)) + on % 8 * 2;
              *reinterpret_cast<uint16_t*>(place) = 0;
              if (kLow) *reinterpret_cast<uint16_t*>(place + kHeldBytes) = 0;
            }
          }
          if (c == items - 1) done();
          if (kPhase == kUpdate && index == P.last) {
            __syncwarp();
            if (P.sj == 1) {
              // the result's rows from where they lie, eight lanes a row's 64 columns
              const int64_t row0 = ((int64_t)tr * CG + rank) * 128 + w * 32, col = cols + c * 64 + lane % 8 * 8;
              T* o = static_cast<T*>(P.out) + k * P.sk + col;
              const bool vectors = ((reinterpret_cast<uintptr_t>(P.out) | (uintptr_t)(P.sk * sizeof(T)) | (uintptr_t)(P.si * sizeof(T))) & 15) == 0;
#pragma unroll 1
              for (int r = lane / 8; r < 32 && row0 + r < S.m; r += 4) {
                alignas(16) T e8[8];
                const char* from_smem = b + piece_at((uint32_t)r, (uint32_t)(lane % 8));
                memcpy(e8, from_smem, 16);
                if (sizeof(T) == 4) memcpy(reinterpret_cast<char*>(e8) + 16 * (sizeof(T) / 4), from_smem + kHeldBytes, 16);
                T* to_row = o + (row0 + r) * P.si;
                if (vectors && col + 8 <= S.n) {
#pragma unroll
                  for (int u = 0; u < 8; u += Vec<T>::N) memcpy(__builtin_assume_aligned(to_row + u, 16), e8 + u, 16);
                } else {
#pragma unroll
                  for (int u = 0; u < 8; ++u)
                    if (col + u < S.n) to_row[u] = e8[u];
                }
              }
            }
            fence_proxy_async();  // (read and written before the next copy into it)
            __syncwarp();
            if (lane == 0 && Pl::kBuffers == 1) fetch_after(c);
            continue;
          }
          fence_proxy_async();
          __syncwarp();
          if (lane == 0) {
            const int64_t at = part + c * kBlock;
            bulk_store(to.hi + at, b, kHeldBytes);
            if (kLow) bulk_store(to.lo + at, b + kHeldBytes, kHeldBytes);
            bulk_commit();
          }
          if (kPhase != kUpdate && P.triangle[kPhase % kUpdate] && tr != tc) {
            // the same above the diagonal: this warp's 64 columns are rows there, two of them a lane, its rows
            // 32 columns, four pieces
            const int64_t first_row = cols + c * 64;
            const int64_t cb = ((int64_t)tr * CG + rank) * 2 + w / 2;
            const int64_t block = k * plane + (first_row / 128 * bc + cb) * kBlock;
#pragma unroll 1
            for (int i = 0; i < (kLow ? 16 : 8); ++i) {
              const int low = i / 8, h = i / 4 % 2, p = i % 4;
              const char* plane_at = b + low * kHeldBytes;
              char* out = reinterpret_cast<char*>((low ? to.lo : to.hi) + block);
              const uint32_t j = h * 32 + lane, r = (uint32_t)(first_row % 128) + j;  // column here, row there
              alignas(16) uint16_t v[8];
#pragma unroll
              for (int u = 0; u < 8; ++u)
                v[u] = *reinterpret_cast<const uint16_t*>(plane_at + piece_at((uint32_t)(p * 8 + u), j / 8) + j % 8 * 2);
              *reinterpret_cast<uint4*>(out + piece_at(r, (uint32_t)(w % 2 * 4 + p))) = *reinterpret_cast<const uint4*>(v);
            }
          }
          __syncwarp();
          if (lane == 0 && kPhase != kGram && Pl::kBuffers == 1) {
            bulk_read();
            fetch_after(c);
          }
        }
      };

      for (int64_t unit = first; unit < parts.all && going; unit += step) {
        const uint32_t acc_at = tmem + e * (64 * Pl::kItems) + ((uint32_t)w << 21);  // this warp's part of the first accumulator
        int64_t t;
        int begin, end;
        parts.at(unit, &t, &begin, &end);
        constexpr int kChunk = Pl::chunk(kPhase);
        bool added_up = false;
        if constexpr (kFine && kChunk < 1 << 30) added_up = end - begin > kChunk;
        if (added_up) {
          float sum[64 * Pl::kItems];
#pragma unroll
          for (int i = 0; i < 64 * Pl::kItems; ++i) sum[i] = 0.f;
          for (int kb = begin; kb < end; kb += kChunk) {
            going = __all_sync(0xffffffffu, wait_for(&bars.sums[it & 1], (it / 2) & 1, patience));
            if (!going) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
            for (int i = 0; i < 64 * Pl::kItems; i += 2 * kStep) {
              float one[kStep], two[kStep];
              tmem_load(acc_at + (it & 1) * kColumns + i, one);
              tmem_load(acc_at + (it & 1) * kColumns + i + kStep, two);
              tmem_loaded(one);
              tmem_loaded(two);
#pragma unroll
              for (int u = 0; u < kStep; ++u) sum[i + u] += one[u], sum[i + kStep + u] += two[u];
            }
            if (kb + kChunk < end) {
              asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
              __syncwarp();
              if (lane == 0) arrive_first<CG>(&bars.taken[it & 1]);
              ++it;
            }
          }
          // back into the last accumulator: what follows takes them from there in a loop
#pragma unroll
          for (int i = 0; i < 64 * Pl::kItems; i += kStep) tmem_store(acc_at + (it & 1) * kColumns + i, sum + i);
          tmem_stored();
        } else {
          going = __all_sync(0xffffffffu, wait_for(&bars.sums[it & 1], (it / 2) & 1, patience));
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        }
        if (!going) break;
        float next[kStep];
        tmem_load(acc_at + (it & 1) * kColumns, next);
        auto sums = [&](int at, float (&acc)[kStep]) {
          tmem_loaded(next);
#pragma unroll
          for (int u = 0; u < kStep; ++u) acc[u] = next[u];
          if (at + kStep < 64 * Pl::kItems) tmem_load(acc_at + (it & 1) * kColumns + at + kStep, next);
        };
        auto done = [&] {
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          __syncwarp();
          if (lane == 0) arrive_first<CG>(&bars.taken[it & 1]);
        };
        if (kPhase == kGram && unit >= parts.whole) {
          float* share = share_of(t, parts.split_of(unit));
#pragma unroll 1
          for (int i = 0; i < 64 * Pl::kItems; i += kStep) {
            float acc[kStep];
            sums(i, acc);
#pragma unroll
            for (int u = 0; u < kStep; ++u) share[(i + u) * 32] = acc[u];
          }
          done();  // (a barrier of the warp)
          if (lane == 0) asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(shared(t)) : "memory");
        } else {
          finish(t, unit + step < parts.whole ? unit + step : -1, 0, Pl::kItems, sums, done);
        }
        tmem_loaded(next);  // (nothing is on its way, but where a wait gave up)
        ++it;
      }
      if constexpr (kPhase == kGram) {
        // Shares of tiles are added up, in their order, by the warps that have the same place in the tile:
        // each share's block takes some items of them. (None waits before all its own shares are out.)
        if (parts.all > parts.whole)
          for (int64_t unit = first; unit < parts.all && going; unit += step) {
            if (unit < parts.whole) continue;
            const int64_t t = parts.whole + (unit - parts.whole) / parts.splits;
            const uint32_t to = (uint32_t)parts.splits * (index / 3 + 1);
            going = __all_sync(0xffffffffu, lane != 0 || wait_count(shared(t), to, patience));
            __syncwarp();  // (as above: the shares)
            auto sums = [&](int at, float (&acc)[kStep]) {
#pragma unroll
              for (int u = 0; u < kStep; ++u) acc[u] = 0.f;
#pragma unroll 1
              for (int split = 0; split < parts.splits; split += 4) {
                float of[4][kStep];
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                  const float* share = share_of(t, split + v) + at * 32;
#pragma unroll
                  for (int u = 0; u < kStep; ++u) of[v][u] = split + v < parts.splits ? __ldcg(share + u * 32) : 0.f;
                }
#pragma unroll
                for (int v = 0; v < 4; ++v)
#pragma unroll
                  for (int u = 0; u < kStep; ++u) acc[u] += of[v][u];
              }
            };
            for (int c = 0; c < Pl::kItems && going; ++c) {
              if (((warp - 2) * Pl::kItems + c) % parts.splits != parts.split_of(unit)) continue;
              finish(t, -1, c, c + 1, sums, [] {});
            }
          }
      }
      // what this block wrote is there for the next phase (which orders its copies after it)
      if (lane == 0) bulk_done();
      if (index + 1 == P.end) {
        fence_proxy_async_all();
      } else {
        asm volatile("bar.sync 1, %0;" ::"n"(32 * Pl::kWarps) : "memory");
        if (warp == 2 && lane == 0 && !(P.hold && blockIdx.x == 0)) asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(P.phases) : "memory");
      }
    });
    if (lane == 0)
      for (uint32_t i = fetched > Pl::kBuffers ? fetched - Pl::kBuffers : 0; i < fetched; ++i)
        wait_bounded(in + i % Pl::kBuffers, (i / Pl::kBuffers) & 1, kWaitLimitNs);
  }
  __syncwarp();
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (CG == 2) {
    cluster_arrive();
    cluster_wait();
  }
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  if (warp == 1) tmem_free<CG>(tmem, 2 * kColumns);
  if (threadIdx.x == 0 && bars.dead) atomicExch(P.gave_up, 1u);
}

// The phases [P.begin, P.end) in one launch: more than one need all blocks resident at once.
template <int CG, typename T>
cudaError_t launch_phases(const CUtensorMap& map, const ProductArgs& P, int device, int sms, cudaStream_t s) {
  using Pl = Plan<CG, T>;
  constexpr int smem = product_smem<CG, T>();
  static_assert(smem <= 232448, "shared memory of a block");
  auto* f = k_products<CG, T>;
  static std::atomic<uint64_t> known{0};  // devices whose limit is raised
  if (device >= 64 || !(known.load(std::memory_order_relaxed) >> device & 1)) {
    const cudaError_t e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    if (device < 64) known.fetch_or(uint64_t(1) << device, std::memory_order_relaxed);
  }
  const bool together = P.end - P.begin > 1;
  if ((CG > 1 || together) && refuse_cooperative()) return cudaErrorCooperativeLaunchTooLarge;
  const int64_t rows = P.S.mp / (128 * CG), cols = P.S.np / (128 * CG), most = sms / CG;
  int64_t tiles = P.K * rows * cols;
  for (int i = 0; i < 2; ++i) {
    const int64_t all = P.K * (P.triangle[i] ? rows * (rows + 1) / 2 : rows * rows);
    tiles = std::max(tiles, i == 0 && P.splits > 1 ? P.whole + (all - P.whole) * P.splits : all);
  }
  LaunchConfig l((tiles < most ? tiles : most) * CG, Pl::kThreads, CG, smem, s);
  if (together) {  // in the place of programmatic serialization
    l.at[0].id = cudaLaunchAttributeCooperative;
    l.at[0].val.cooperative = 1;
  }
  return cudaLaunchKernelEx(&l.cfg, f, map, P);
}
// All steps: in one launch, or, where the context has no room for all blocks, phase by phase.
template <int CG, typename T>
cudaError_t all_steps(const CUtensorMap& map, ProductArgs P, int device, int sms, cudaStream_t s) {
  cudaError_t e = launch_phases<CG, T>(map, P, device, sms, s);
  if (!too_large_here(e)) return e;
  cudaGetLastError();  // this launch's
  const int end = P.end;
  P.splits = 1;  // (shares wait for each other)
  for (e = cudaSuccess; P.begin < end && e == cudaSuccess; ++P.begin) {
    P.end = P.begin + 1;
    e = launch_phases<CG, T>(map, P, device, sms, s);
  }
  return e;
}

// The workspace as rows of 128 bytes, for copies of 64 of them.
cudaError_t map_of(void* base, int64_t bytes, CUtensorMap* map) {
  using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                              const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  static std::atomic<void*> found{nullptr};
  void* f = found.load(std::memory_order_relaxed);
  if (!f) {
    cudaDriverEntryPointQueryResult how;
    const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &how);
    if (e != cudaSuccess) return e;
    if (how != cudaDriverEntryPointSuccess || !f) return cudaErrorNotSupported;
    found.store(f, std::memory_order_relaxed);
  }
  const cuuint64_t size[2] = {64, (cuuint64_t)(bytes / 128)}, stride[1] = {128};
  const cuuint32_t box[2] = {64, 64}, one[2] = {1, 1};
  const CUresult r = reinterpret_cast<Encode>(f)(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, base, size, stride, box, one,
                                                 CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
                                                 CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

// -- small matrices -----------------------------------------------------------------

// X of up to 128 rows and 128 columns a block, in shared memory from the first step to the last: one launch
// for everything. The blocks of a cluster have 128 columns each; of A = X X' each adds up the shares of all
// for its own columns, and gives them to all. A^2 and B are each block's own. What bounds it is the chain of
// products (0.3 us each, 1.1 of fp32) and of what is made of their sums by 16 warps (by 8: 128 x 128 bf16 26 us, so
// 24); with clusters also the exchange of A, 64 KB into each block and 32 out of it (2 us). 16 x 16 bf16 12.8 us, by way of
// the workspace 31; 128 x 128 fp32 41; 4 x 1,000 x 64 fp32 43, so 108; 8 x 128 x 1,024 bf16 48.
constexpr int kSmallSide = 128, kMostSmallParts = 8, kSmallThreads = 512;
struct SmallArgs {
  int64_t m, n;  // of X
  int steps, parts;
  float scale;
  uint64_t wait_ns;  // bound of every wait
  int hold_block, hold_product;  // test hook: the product that this block does not issue; -1: none
  float coef[3 * kMostSteps];
};
template <bool kFine>
struct alignas(1024) SmallSmem {
  __half xh[2][kBlock], xl[2][kBlock];  // X, blocks of 64 columns
  __half oh[2][kBlock];                 // O, then R
  __half ol[kFine ? 2 : 1][kFine ? kBlock : 8];
  float share[kSmallSide * kSmallSide]; // of A's columns that are this block's, by the blocks they come from, by columns
  float d[kSmallSide], e[kSmallSide];   // diagonals of A and B
  double squares[kMostSmallParts], ws[kSmallThreads / 32];
  Scaled by;
  uint64_t done, ended;                 // products; all of them, where a wait gave up
  uint32_t tmem, dead;
};
__device__ __forceinline__ void store_at(uint32_t addr, uint32_t rank, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(remote(addr, rank)), "r"(v) : "memory");
}
__device__ __forceinline__ void store_at(uint32_t addr, uint32_t rank, const uint4& v) {
  asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(remote(addr, rank)), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w)
               : "memory");
}
__device__ __forceinline__ void store_at(uint32_t addr, uint32_t rank, float v) {
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(remote(addr, rank)), "f"(v) : "memory");
}
__device__ __forceinline__ void store_at(uint32_t addr, uint32_t rank, double v) {
  asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(remote(addr, rank)), "d"(v) : "memory");
}

__device__ __forceinline__ int64_t up16(int64_t v) { return (v + 15) / 16 * 16; }

template <typename T, bool kTurned>
__global__ void __launch_bounds__(kSmallThreads, 1) k_small(const T* g, int64_t sk, int64_t ld, T* out, int64_t osk, int64_t old,
                                                  const __grid_constant__ SmallArgs A) {
  constexpr bool kFine = kOfTwo<T>;
  extern __shared__ char raw[];
  auto& sm = *reinterpret_cast<SmallSmem<kFine>*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  const int tid = (int)threadIdx.x, warp = tid / 32, lane = tid % 32;
  const uint32_t parts = (uint32_t)A.parts, rank = parts > 1 ? cluster_rank() : 0;
  const int64_t k = blockIdx.x / parts, j0 = (int64_t)rank * kSmallSide;
  if (parts > 1) cluster_arrive();  // (it has begun)
  if (tid == 0) {
    mbar_init(&sm.done, 1);
    mbar_init(&sm.ended, 1);
    sm.dead = 0;
    fence_mbar_init();
  }
  if (warp == 0) tmem_alloc<1>(&sm.tmem, kSmallSide);
  griddep_wait();

  // this block's columns of G: some pieces of eight columns a thread, neighbours along a row of G
  g += k * sk;
  constexpr int kPieces = kSmallSide * kSmallSide / 8 / kSmallThreads, kGroups = kSmallThreads / 128;
  float f[kPieces][8];
  double s = 0.;
  const bool vectors = !kTurned && ((reinterpret_cast<uintptr_t>(g) | (uintptr_t)(ld * sizeof(T))) & 15) == 0;
  auto piece_of = [&](int u, int* row, int* piece) {
    *row = kTurned ? tid % 128 : tid / 16 + kSmallThreads / 16 * u;
    *piece = kTurned ? tid / 128 + kGroups * u : tid % 16;
  };
#pragma unroll
  for (int u = 0; u < kPieces; ++u) {
    int row, piece;
    piece_of(u, &row, &piece);
    const int64_t j = j0 + piece * 8;
    const T* x = g + (kTurned ? j * ld + row : row * ld + j);
    if (vectors && row < A.m && j + 8 <= A.n) {
#pragma unroll
      for (int v = 0; v < 8; v += Vec<T>::N) Vec<T>::get(*reinterpret_cast<const uint4*>(x + v), f[u] + v);
    } else {
#pragma unroll
      for (int v = 0; v < 8; ++v) f[u][v] = row < A.m && j + v < A.n ? Vec<T>::one(x[v * (kTurned ? ld : 1)]) : 0.f;
    }
  }
  s = warp_sum(squares<8 * kPieces>(&f[0][0]));
  if (lane == 0) sm.ws[warp] = s;
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = *(volatile uint32_t*)&sm.tmem;
  // (64-bit arithmetic is slow: by one warp)
  if (warp == 0) s = warp_sum(lane < kSmallThreads / 32 ? sm.ws[lane] : 0.);
  if (parts > 1) {
    cluster_wait();  // all have begun
    if (tid < (int)parts) store_at(smem_addr(&sm.squares[rank]), (uint32_t)tid, s);
    cluster_arrive();
    cluster_wait();
    if (warp == 0) s = warp_sum(lane < (int)parts ? sm.squares[lane] : 0.);
  }
  if (warp == 0) {
    const Scaled by = scaled_by(s);
    if (lane == 0) sm.by = by;
  }
  __syncthreads();
  const Scaled by = sm.by;
#pragma unroll
  for (int u = 0; u < kPieces; ++u) {
    int row, piece;
    piece_of(u, &row, &piece);
    alignas(16) __half2 hi[4], lo[4];
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      float x[2];
#pragma unroll
      for (int o = 0; o < 2; ++o)  // (what pads a matrix that is NaN stays 0)
        x[o] = row < A.m && j0 + piece * 8 + 2 * v + o < A.n ? by(f[u][2 * v + o]) : 0.f;
      two_halves(x[0], x[1], hi + v, lo + v);
    }
    const uint32_t in = piece_at((uint32_t)row, (uint32_t)(piece % 8));
    *reinterpret_cast<uint4*>(reinterpret_cast<char*>(sm.xh[piece / 8]) + in) = *reinterpret_cast<uint4*>(hi);
    *reinterpret_cast<uint4*>(reinterpret_cast<char*>(sm.xl[piece / 8]) + in) = *reinterpret_cast<uint4*>(lo);
  }

  // Sums of this thread: its row, every fourth kStep columns. Of A and B, what lies beyond X's rows is neither
  // computed nor looked at.
  const int row = warp % 4 * 32 + lane, half = warp / 4 * kStep, side = (int)up16(A.m);
  const bool in_rows = warp % 4 * 32 < side;  // (the same for a warp)
  const int columns = A.n - j0 > kSmallSide ? kSmallSide : A.n > j0 ? (int)up16(A.n - j0) : 16;  // of X that are not padding
  const uint32_t acc_at = tmem + ((uint32_t)(warp % 4) << 21);
  uint32_t products = 0;
  bool waited = true;  // no wait gave up
  // All threads: what they wrote is there for the products, which `issue` issues; they are done.
  auto product = [&](auto&& issue) {
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    fence_proxy_async();
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (tid == 0 && !((int)products == A.hold_product && (int)blockIdx.x == A.hold_block)) {
      issue();
      commit<1>(&sm.done);
    }
    waited = wait_for(&sm.done, products & 1, Patience{&sm.dead, A.wait_ns}) && waited;
    ++products;
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  };
  const uint32_t xh = smem_addr(sm.xh), xl = smem_addr(sm.xl), oh = smem_addr(sm.oh), ol = smem_addr(sm.ol);
  constexpr uint32_t kBlockBytes = 2 * kBlock;
  // `columns` columns of L R' (or L R: the right factor's rows are the sum's index) over `terms`, the small terms first
  auto issue = [&](uint32_t lh, uint32_t ll, uint32_t rh, uint32_t rl, bool rows, int columns, int terms) {
    const uint32_t what = 1u << 4 | (rows ? 1u << 16 : 0) | (uint32_t)(columns / 8) << 17 | (128 / 16) << 24;
    for (int t = kFine ? 0 : 2; t < 3; ++t) {
      const uint32_t l = t == 1 ? ll : lh, r = t == 0 ? rl : rh;
      for (int q = 0; q < terms / 16; ++q) {
        const uint64_t dl = factor(l + q / 4 * kBlockBytes, 0) + (q % 4 * 32 >> 4);
        const uint64_t dr = rows ? factor(r, kBlockBytes) + (q * 2048 >> 4) : factor(r + q / 4 * kBlockBytes, 0) + (q % 4 * 32 >> 4);
        mma<1>(tmem, dl, dr, what, q > 0 || t > (kFine ? 0 : 2));
      }
    }
  };
  // eight columns of a plane of this thread's row
  auto place = [&](void* plane, int column) {
    return reinterpret_cast<uint4*>(static_cast<char*>(plane) + column / 64 * kBlockBytes + piece_at((uint32_t)row, (uint32_t)(column % 64 / 8)));
  };
  auto both = [&](void* hi, void* lo, bool two, int column, float* v) {  // as numbers
    Vec<__half>::get(*place(hi, column), v);
    if (!two) return;
    float low[8];
    Vec<__half>::get(*place(lo, column), low);
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] += low[u];
  };
  auto halves = [&](const float* v, uint4* hi, uint4* lo) {
    alignas(16) __half2 h[4], l[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) two_halves(v[2 * u], v[2 * u + 1], h + u, l + u);
    *hi = *reinterpret_cast<uint4*>(h);
    *lo = *reinterpret_cast<uint4*>(l);
  };

  // After the last product, and in a cluster's blocks an arrival: whether a wait gave up is known in all of them.
  auto all_told = [&] {
    if (parts > 1) cluster_wait();
    __syncthreads();
  };
  auto gave_up = [&] { return *(volatile uint32_t*)&sm.dead != 0; };

  // the sum on the diagonal, of eight columns that have it; O and R have none
  auto taken_out = [&](const float* sums, int column) {
    const int on = row - column;
    reinterpret_cast<uint16_t*>(place(sm.oh, column))[on] = 0;
    if (kFine) reinterpret_cast<uint16_t*>(place(sm.ol, column))[on] = 0;
    float mid = 0.f;
#pragma unroll
    for (int u = 0; u < 8; ++u) mid = u == on ? sums[u] : mid;
    return mid;
  };

#pragma unroll 1
  for (int step = 0; step < A.steps; ++step) {
    const float c1 = A.coef[3 * step], c3 = A.coef[3 * step + 1], c5 = A.coef[3 * step + 2];
    product([&] { issue(xh, xl, xh, xl, false, side, columns); });
    if (parts == 1) {
#pragma unroll 1
      for (int at = half; at < side && in_rows; at += kGroups * kStep) {
        float acc[kStep];
        tmem_load(acc_at + at, acc);
        tmem_loaded(acc);
#pragma unroll
        for (int p = 0; p < kStep; p += 8) {
          const int column = at + p;
          float v[8];
#pragma unroll
          for (int u = 0; u < 8; ++u) v[u] = acc[p + u] * (kO / (kX * kX));
          uint4 hi, lo;
          halves(v, &hi, &lo);
          *place(sm.oh, column) = hi;
          if (kFine) *place(sm.ol, column) = lo;
          if ((uint32_t)(row - column) < 8) sm.d[row] = taken_out(acc + p, column) * (1.f / (kX * kX));
        }
      }
    } else {
      // this block's shares to the blocks that add them up, `wide` columns each
      const int wide = (side / 8 + (int)parts - 1) / (int)parts * 8;
#pragma unroll 1
      for (int at = half; at < side && in_rows; at += kGroups * kStep) {
        float acc[kStep];
        tmem_load(acc_at + at, acc);
        tmem_loaded(acc);
#pragma unroll
        for (int p = 0; p < kStep; p += 8) {
          const int column = at + p;
          const uint32_t to = remote(smem_addr(sm.share + ((int)rank * wide + column % wide) * side + row), (uint32_t)(column / wide));
          if (row < side)
#pragma unroll
            for (int u = 0; u < 8; ++u)
              asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to + u * side * 4), "f"(acc[p + u]) : "memory");
        }
      }
      cluster_arrive();
      cluster_wait();
      // (A is symmetric: its columns are rows. Pieces of eight columns of a row: all of a piece's shares, then its
      // halves to all blocks, neighbours along a row)
#pragma unroll 1
      for (int i = tid; i < side * wide / 8; i += kSmallThreads) {
        const int c = i / (side / 8), column = i % (side / 8) * 8, r = (int)rank * wide + c;
        if (r >= side) break;
        float v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = 0.f;
#pragma unroll 1
        for (uint32_t p = 0; p < parts; ++p) {
          const float4* share = reinterpret_cast<const float4*>(sm.share + ((int)p * wide + c) * side + column);
          const float4 x = share[0], y = share[1];
          v[0] += x.x, v[1] += x.y, v[2] += x.z, v[3] += x.w;
          v[4] += y.x, v[5] += y.y, v[6] += y.z, v[7] += y.w;
        }
        float mid = 0.f;
        const int on = r - column;  // the column that is on the diagonal
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          if (u == on) mid = v[u] * (1.f / (kX * kX));
          v[u] = u == on ? 0.f : v[u] * (kO / (kX * kX));
        }
        uint4 hi, lo;
        halves(v, &hi, &lo);
        const uint32_t at = (uint32_t)(column / 64) * kBlockBytes + piece_at((uint32_t)r, (uint32_t)(column % 64 / 8));
        for (uint32_t p = 0; p < parts; ++p) {
          store_at(oh + at, p, hi);
          if (kFine) store_at(ol + at, p, lo);
          if (on >= 0 && on < 8) store_at(smem_addr(sm.d + r), p, mid);
        }
      }
      asm volatile("fence.proxy.async.shared::cluster;" ::: "memory");
      cluster_arrive();
      cluster_wait();
    }
    product([&] { issue(oh, ol, oh, ol, false, side, side); });
    const float dr = sm.d[row], di = c3 + c5 * dr;
#pragma unroll 1
    for (int at = half; at < side && in_rows; at += kGroups * kStep) {
      float acc[kStep];
      tmem_load(acc_at + at, acc);
      tmem_loaded(acc);
#pragma unroll
      for (int p = 0; p < kStep; p += 8) {
        const int column = at + p;
        float v[8], dc[8];
        both(sm.oh, sm.ol, kFine, column, v);
        Vec<float>::get(*reinterpret_cast<const uint4*>(sm.d + column), dc);
        Vec<float>::get(*reinterpret_cast<const uint4*>(sm.d + column + 4), dc + 4);
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = __fmaf_rn(__fmaf_rn(c5, dc[u], di), v[u], acc[p + u] * (c5 / kO));
        uint4 hi, lo;
        halves(v, &hi, &lo);
        *place(sm.oh, column) = hi;
        if (kFine) *place(sm.ol, column) = lo;
        if ((uint32_t)(row - column) < 8) sm.e[row] = c3 * dr + c5 * __fmaf_rn(dr, dr, taken_out(acc + p, column) * (1.f / (kO * kO)));
      }
    }
    product([&] { issue(oh, ol, xh, xl, true, columns, side); });
    const float ei = c1 + sm.e[row];
    const bool last = step + 1 == A.steps;
    if (last) {  // a wait that gave up is one of the whole matrix
      if (parts > 1) {
        for (uint32_t p = 0; p < parts && !waited; ++p) store_at(smem_addr(&sm.dead), p, 1u);
        cluster_arrive();
      }
      if (kTurned) all_told();
    }
    const float by_out = kTurned && last && gave_up() ? __uint_as_float(kNan) : A.scale * (1.f / kX);
#pragma unroll 1
    for (int at = half; at < columns && in_rows; at += kGroups * kStep) {
      float acc[kStep];
      tmem_load(acc_at + at, acc);
      tmem_loaded(acc);
#pragma unroll
      for (int p = 0; p < kStep; p += 8) {
        const int column = at + p;
        float v[8];
        both(sm.xh, sm.xl, true, column, v);
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = __fmaf_rn(ei, v[u], acc[p + u] * (1.f / kO));
        if (!last) {
          uint4 hi, lo;
          halves(v, &hi, &lo);
          *place(sm.xh, column) = hi;
          *place(sm.xl, column) = lo;
        } else if (kTurned) {  // (neighbours are the lanes' rows)
          const int64_t j = j0 + column;
          T* o = out + k * osk + j * old + row;
#pragma unroll
          for (int u = 0; u < 8; ++u)
            if (row < A.m && j + u < A.n) o[u * old] = Vec<T>::round(v[u] * by_out);
        } else {  // in the place of the halves
          alignas(16) T e8[8];
#pragma unroll
          for (int u = 0; u < 8; ++u) e8[u] = Vec<T>::round(v[u] * by_out);
          memcpy(__builtin_assume_aligned(place(sm.xh, column), 16), e8, 16);
          if (sizeof(T) == 4) memcpy(__builtin_assume_aligned(place(sm.xl, column), 16), reinterpret_cast<const char*>(e8) + sizeof(e8) - 16, 16);
        }
      }
    }
  }
  if (!kTurned) {
    // the result's rows from where they lie, sixteen lanes a row
    all_told();
    const bool nothing = gave_up();
    out += k * osk;
    const bool rows16 = ((reinterpret_cast<uintptr_t>(out) | (uintptr_t)(old * sizeof(T))) & 15) == 0;
#pragma unroll 1
    for (int r = tid / 16; r < A.m; r += kSmallThreads / 16) {
      const int piece = tid % 16;
      const int64_t j = j0 + piece * 8;
      const uint32_t in = (uint32_t)(piece / 8) * kBlockBytes + piece_at((uint32_t)r, (uint32_t)(piece % 8));
      alignas(16) T e8[8];
      memcpy(e8, __builtin_assume_aligned(reinterpret_cast<const char*>(sm.xh) + in, 16), 16);
      if (sizeof(T) == 4) memcpy(reinterpret_cast<char*>(e8) + sizeof(e8) - 16, __builtin_assume_aligned(reinterpret_cast<const char*>(sm.xl) + in, 16), 16);
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (nothing) e8[u] = Vec<T>::round(__uint_as_float(kNan));
      T* o = out + r * old + j;
      if (rows16 && j + 8 <= A.n) {
#pragma unroll
        for (int u = 0; u < 8; u += Vec<T>::N) memcpy(__builtin_assume_aligned(o + u, 16), e8 + u, 16);
      } else {
#pragma unroll
        for (int u = 0; u < 8; ++u)
          if (j + u < A.n) o[u] = e8[u];
      }
    }
  }
  if (tid == 0 && gave_up()) {  // products that are late end before their memory is given back
    commit<1>(&sm.ended);
    wait_bounded(&sm.ended, 0, kWaitLimitNs);
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  if (warp == 0) tmem_free<1>(tmem, kSmallSide);
}

bool in_shared_memory(int64_t m, int64_t n) {
  return std::min(m, n) <= kSmallSide && std::max(m, n) <= kSmallSide * kMostSmallParts;
}
template <typename T>
cudaError_t launch_small(const T* g, int64_t sk, int64_t ld, T* out, int64_t osk, int64_t old, bool turned, int64_t K,
                         const SmallArgs& A, int device, cudaStream_t s) {
  constexpr int smem = (int)sizeof(SmallSmem<kOfTwo<T>>) + 1024;
  static_assert(smem <= 232448, "shared memory of a block");
  auto* f = turned ? k_small<T, true> : k_small<T, false>;
  static std::atomic<uint64_t> known[2];  // devices whose limit is raised
  if (device >= 64 || !(known[turned].load(std::memory_order_relaxed) >> device & 1)) {
    const cudaError_t e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    if (device < 64) known[turned].fetch_or(uint64_t(1) << device, std::memory_order_relaxed);
  }
  if (A.parts > 1 && refuse_cooperative()) return cudaErrorCooperativeLaunchTooLarge;
  LaunchConfig l(K * A.parts, kSmallThreads, A.parts, smem, s);
  return cudaLaunchKernelEx(&l.cfg, f, g, sk, ld, out, osk, old, A);
}

int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// How a call is carried out: tiles of one block or of a pair, triangles or whole squares of them, and the shares
// that X's columns are taken in. By what the phases take, in cycles. Measured both ways, us (bf16, then float):
//                          single tiles   pairs      whole squares  triangles   unshared  shared
//    32 x    256 x  1,024   182   262    229   319    182   260     196   289
//     1 x  1,024 x  1,024   153   249    213   327    154   248     172   264    153   252  152   246
//     8 x    512 x  4,608   417   690    397   625    404   664     411   644    416   734  397   622
//     8 x  1,000 x  4,096   906 1,693    709 1,540    722 1,774     727 1,594    725 1,729  707 1,545
//     2 x  3,000 x  3,000 1,413 2,985    951 2,563  1,086 3,058     940 2,685    963 2,768  975 2,575
//     7 x    136 x 13,517   404   545    442   572                               655 1,187  405   541
struct Course {
  Shape S;
  bool pairs;
  struct Symmetric {  // A, B
    bool triangle;
    int64_t tiles;
  } of[2];
  int64_t whole;  // of A, those that are not shared,
  int splits;     // and the shares of the others
};
constexpr int kSms = 152, kMostSplits = 16;
// What a tile takes: its products of 64 columns, and what becomes of its sums meanwhile (fine: afterwards,
// since the same warps take the sums of the next tile out); and what the last tile leaves behind.
struct Cost {
  int64_t kblock, use, tail;
  bool fine;
  int64_t tile(int64_t kblocks) const { return fine ? kblocks * kblock + use : std::max(kblocks * kblock, use); }
};
int64_t phase_cycles(int64_t tiles, int slots, int64_t kblocks, const Cost& c) {
  return (tiles + slots - 1) / slots * c.tile(kblocks) + c.tail;
}
// The same with the tiles of the last round in shares, the best number of them.
int64_t shared_cycles(int64_t tiles, int slots, int64_t kblocks, const Cost& c, int cg, int* splits) {
  int64_t least = phase_cycles(tiles, slots, kblocks, c);
  *splits = 1;
  const int64_t rest = tiles % slots, whole = tiles - rest;
  for (int64_t s = 2; rest && s <= kMostSplits && s <= kblocks; ++s) {
    const int64_t each = (kblocks + s - 1) / s;
    if ((s - 1) * each >= kblocks) continue;  // a share of nothing
    const int64_t rounds = (rest * s + slots - 1) / slots;
    // written, and added up: of the 8 cg parts of a tile, some by each share's warps
    const int64_t sum = 3000 + ((8 * cg + s - 1) / s + 7) / 8 * (1500 + 4000 * ((s + 3) / 4));
    const int64_t t = phase_cycles(whole, slots, kblocks, c) + rounds * (each * c.kblock + sum);
    if (t < least) least = t, *splits = (int)s;
  }
  return least;
}
Course course_of(int64_t K, int64_t m, int64_t n, bool fine) {
  if (m > n) std::swap(m, n);
  Course best{};
  int64_t least = INT64_MAX;
  for (int cg = 1; cg <= 2; ++cg) {
    const int unit = 128 * cg, slots = kSms / cg;
    const Cost cost = cg == 1 ? (fine ? Cost{1800, 3000, 5000, true} : Cost{900, 5000, 3500, false})
                              : (fine ? Cost{2200, 10000, 10000, true} : Cost{640, 12000, 9000, false});
    const Shape S{m, n, up(m, unit), up(n, unit)};
    const int64_t R = S.mp / unit, C = S.np / unit;
    Course c{S, cg == 2, {}, 0, 1};
    int64_t all = phase_cycles(K * R * C, slots, (m + 63) / 64, cost);
    for (int phase = 0; phase < 2; ++phase) {
      int64_t cycles = INT64_MAX;
      for (int triangle = 0; triangle < 2; ++triangle) {
        const Course::Symmetric of{triangle == 1, K * (triangle ? R * (R + 1) / 2 : R * R)};
        Cost two = cost;
        if (triangle && R > 1) two.tail += 3000 * cg;  // written above the diagonal too
        int splits = 1;
        const int64_t t = phase ? phase_cycles(of.tiles, slots, (m + 63) / 64, two)
                                : shared_cycles(of.tiles, slots, (n + 63) / 64, two, cg, &splits);
        if (t >= cycles) continue;
        cycles = t;
        c.of[phase] = of;
        if (phase == 0) c.whole = of.tiles - of.tiles % slots, c.splits = splits;
      }
      all += cycles;
    }
    if (all < least) least = all, best = c;
  }
  return best;
}

struct Work {
  double* part;
  uint32_t* counts;  // gave up, phases
  uint32_t* shared;
  int64_t counters;  // of all these
  float *shares, *d, *e;
  Halves2 x, y, o, r;
};
int64_t work_of(bool fine, int64_t K, const Course& c, char* at, Work* w) {
  int64_t bytes = 0;
  auto take = [&](int64_t n) {
    char* p = at + bytes;
    bytes += up(n, 1024);
    return p;
  };
  const Shape& S = c.S;
  const int cg = c.pairs ? 2 : 1;
  const int64_t shared = c.splits > 1 ? c.of[0].tiles - c.whole : 0;  // tiles in shares
  Work v;
  v.part = reinterpret_cast<double*>(take(8 * K * kMostSizeParts));
  v.counters = 2 + shared * cg * 8;  // (at most 8 warps of a block read sums back)
  v.counts = reinterpret_cast<uint32_t*>(take(4 * v.counters));
  v.shared = v.counts + 2;
  v.shares = reinterpret_cast<float*>(take(4 * shared * c.splits * (128 * cg) * (128 * cg)));
  v.d = reinterpret_cast<float*>(take(4 * K * S.mp));
  v.e = reinterpret_cast<float*>(take(4 * K * S.mp));
  for (Halves2* h : {&v.x, &v.y, &v.o, &v.r}) {
    const bool is_x = h == &v.x || h == &v.y;
    const int64_t n = 2 * K * (is_x ? S.x() : S.o());
    h->hi = reinterpret_cast<__half*>(take(n));
    h->lo = is_x || fine ? reinterpret_cast<__half*>(take(n)) : nullptr;
  }
  if (w) *w = v;
  return bytes;
}

// The matrices of a call that are worked on together, and the workspace of so many. Its sides are padded to 128 or 256, so that
// many thin matrices would take far more than their own size: K goes in slices of at most kSliceBytes (or one
// matrix): 5,000 of 129 x 131 bf16 6.0 ms, 65,535 in slices 79. Matrices that stay in shared memory want a workspace
// where a context has no room for their clusters alone: slices of kSmallSliceBytes; those of one block none (its token size).
constexpr int64_t kSliceBytes = int64_t(4) << 30, kSmallSliceBytes = int64_t(64) << 20, kNoWorkspace = 256;
struct Slices {
  int64_t each;
  Course course;  // of `each` matrices
  int64_t bytes;
};
Slices slices_of(bool fine, int64_t K, int64_t m, int64_t n) {
  if (std::max(m, n) <= kSmallSide) return {K, Course{}, kNoWorkspace};
  const int64_t most = in_shared_memory(m, n) ? kSmallSliceBytes : kSliceBytes;
  for (int64_t parts = 1;; parts *= 2) {
    Slices s;
    s.each = (K + parts - 1) / parts;
    s.course = course_of(s.each, m, n, fine);
    s.bytes = work_of(fine, s.each, s.course, nullptr, nullptr);
    const int64_t last = s.each ? K % s.each : 0;
    if (last) s.bytes = std::max(s.bytes, work_of(fine, last, course_of(last, m, n, fine), nullptr, nullptr));
    if (s.bytes <= most || s.each <= 1) return s;
  }
}

// Test hooks (gmc_test_withhold_phase, gmc_test_withhold_product): the next call's wait limit, 0 = off, and what is withheld.
std::atomic<uint64_t> g_hold_ns{0};
std::atomic<int> g_hold_block{0}, g_hold_product{0};

bool sizes_ok(int32_t dtype, int64_t K, int64_t m, int64_t n) {
  if (dtype != GMC_F32 && dtype != GMC_BF16 && dtype != GMC_F16) return false;
  if (K < 0 || m < 0 || n < 0 || K > 65535 || m > (1 << 20) || n > (1 << 20)) return false;
  return K == 0 || m == 0 || n <= (int64_t(1) << 36) / K / m;
}
bool strides_ok(const void* p, int32_t dtype, int64_t K, int64_t m, int64_t n, int64_t sk, int64_t ld) {
  const uintptr_t size = dtype == GMC_F32 ? 4 : 2;
  if (!p || reinterpret_cast<uintptr_t>(p) % size) return false;
  if (m > 1 && (ld < n || ld > (int64_t(1) << 40))) return false;
  if (K <= 1) return true;
  if (sk < n || sk > (int64_t(1) << 40)) return false;
  // a matrix after the other, or a row of each in turn
  return m <= 1 || sk >= (m - 1) * ld + n || ld >= (K - 1) * sk + n;
}

// K matrices by way of the workspace.
template <typename T>
cudaError_t orthogonalize_slice(const T* g, int64_t sk, int64_t ld, T* o, int64_t osk, int64_t old, int64_t K, int64_t m, int64_t n, int steps,
                                const float* coefficients, float scale, const Course& course, void* workspace,
                                const CUtensorMap& map, uint64_t wait_ns, bool hold, int device, int sms, cudaStream_t s) {
  const Shape S = course.S;
  const bool turned = m > n;
  Work w;
  work_of(kOfTwo<T>, K, course, static_cast<char*>(workspace), &w);
  // parts of |G|^2: as many blocks as are resident at once, of eight rows or pieces each
  const int64_t rows8 = (m * ((n + kSizePiece - 1) / kSizePiece) + 7) / 8;
  const int parts = (int)std::min({rows8, (sms * 4 + K - 1) / K, (int64_t)kMostSizeParts});
  const dim3 some((unsigned)std::min(S.x() / kBlock, (sms * 8 + K - 1) / K), (unsigned)K);
  cudaError_t e = launch_pdl(k_size<T>, dim3((unsigned)parts, (unsigned)K), dim3(256), 0, s, g, sk, ld, m, n, w.part, w.counts,
                             w.counters);
  if (e != cudaSuccess) return e;
  e = launch_pdl(turned ? k_first<T, true> : k_first<T, false>, some, dim3(256), 0, s, g, sk, ld, S, (const double*)w.part,
                 parts, w.x);
  if (e != cudaSuccess) return e;
  ProductArgs P{S, K, static_cast<const __half*>(workspace), {w.x, w.y}, w.o, w.r, w.d, w.e, 0, 3 * steps,
                3 * steps - 1, o, osk, turned ? 1 : old, turned ? old : 1, scale,
                {course.of[0].triangle, course.of[1].triangle}, course.whole, course.splits, w.shares, w.shared,
                w.counts + 1, wait_ns, hold, w.counts, {}};
  std::copy(coefficients, coefficients + 3 * steps, P.coef);
  bool pairs = course.pairs;
  if (pairs) e = all_steps<2, T>(map, P, device, sms, s);
  if (pairs && too_large_here(e)) {  // a context without room for clusters
    cudaGetLastError();
    pairs = false;
    P.splits = 1;
  }
  if (!pairs) e = all_steps<1, T>(map, P, device, sms, s);
  if (e != cudaSuccess) return e;
  return launch_pdl(k_gave_up<T>, dim3((unsigned)std::min<int64_t>(4, (m * n + 255) / 256), (unsigned)K), dim3(256), 0, s, o, osk,
                    old, m, n, (const uint32_t*)w.counts);
}

}  // namespace

extern "C" {

int64_t gmc_orthogonalize_workspace(int32_t dtype, int64_t K, int64_t m, int64_t n) {
  if (!sizes_ok(dtype, K, m, n)) return -1;
  const int64_t bytes = slices_of(dtype != GMC_BF16, K, m, n).bytes;
  return bytes <= kMostWork ? bytes : -1;
}

int gmc_test_orthogonalize_course(int32_t dtype, int64_t K, int64_t m, int64_t n) {
  if (!sizes_ok(dtype, K, m, n)) return -1;
  if (in_shared_memory(m, n)) return 0;
  const Course c = slices_of(dtype != GMC_BF16, K, m, n).course;
  return 1 | c.pairs << 1 | c.of[0].triangle << 2 | c.of[1].triangle << 3 | c.splits << 4 | (c.whole > 0) << 12;
}

int gmc_test_withhold_phase(uint64_t wait_limit_ns) {
  return gmc_test_withhold_product(wait_limit_ns, 0, 0);
}

int gmc_test_withhold_product(uint64_t wait_limit_ns, int32_t block, int32_t product) {
  if (wait_limit_ns > 2000000000ull || block < 0 || product < 0) return GMC_EINVAL;
  g_hold_block.store(block, std::memory_order_relaxed);
  g_hold_product.store(product, std::memory_order_relaxed);
  g_hold_ns.store(wait_limit_ns, std::memory_order_relaxed);
  return GMC_OK;
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
  if (out_dev == x_dev && ((m > 1 && out_ld != ld) || (K > 1 && out_ldk != ldk))) return GMC_EINVAL;  // in place: the same rows
  const bool of_two = dtype != GMC_BF16, turned = m > n, small = in_shared_memory(m, n);
  const Slices slices = slices_of(of_two, K, m, n);
  if (!workspace_dev || reinterpret_cast<uintptr_t>(workspace_dev) % 256 || slices.bytes > kMostWork || workspace_bytes < slices.bytes)
    return GMC_EINVAL;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const uint64_t hold_ns = g_hold_ns.exchange(0, std::memory_order_relaxed), wait_ns = hold_ns ? hold_ns : kWaitLimitNs;
  int device = 0, sms = 0;
  cudaError_t err = cudaGetDevice(&device);
  if (err == cudaSuccess) err = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
  if (err != cudaSuccess) return GMC_ECUDA;
  err = by_type(dtype, [&](auto t) {
    using T = decltype(t);
    const T* g = static_cast<const T*>(x_dev);
    T* o = static_cast<T*>(out_dev);
    if (small) {
      SmallArgs A{std::min(m, n), std::max(m, n), steps, 1, scale, wait_ns, hold_ns ? g_hold_block.load() : -1,
                  hold_ns ? g_hold_product.load() : -1, {}};
      while (A.parts * kSmallSide < A.n) A.parts *= 2;
      std::copy(coefficients_host, coefficients_host + 3 * steps, A.coef);
      const cudaError_t e = launch_small<T>(g, ldk, ld, o, out_ldk, out_ld, turned, K, A, device, s);
      if (A.parts == 1 || !too_large_here(e)) return e;
      cudaGetLastError();  // a context without room for clusters
    }
    CUtensorMap map;
    cudaError_t e = map_of(workspace_dev, slices.bytes, &map);
    for (int64_t k = 0; k < K && e == cudaSuccess; k += slices.each) {
      const int64_t some = std::min(slices.each, K - k);  // (the last slice may be smaller)
      const Course course = some == slices.each ? slices.course : course_of(some, m, n, of_two);
      e = orthogonalize_slice<T>(g + k * ldk, ldk, ld, o + k * out_ldk, out_ldk, out_ld, some, m, n, steps, coefficients_host, scale,
                                 course, workspace_dev, map, wait_ns, hold_ns != 0, device, sms, s);
    }
    return e;
  });
  return err == cudaSuccess ? GMC_OK : GMC_ECUDA;
}

}  // extern "C"
