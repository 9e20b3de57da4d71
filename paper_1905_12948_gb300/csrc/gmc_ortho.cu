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
//     its own rounding by 1.7e-3), or the terms hi hi + hi lo + lo hi (float and half: 1e-7 to 8e-6).
// X is kept 2^14 times, O and R 2^11 times what they are: the second halves then stay normal
// numbers, and a singular value may come to 4.
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

struct Halves2 {
  __half *hi, *lo;
};
// What this thread wrote is seen by copies that follow (another launch's).
__device__ __forceinline__ void fence_proxy_async_all() { asm volatile("fence.proxy.async;" ::: "memory"); }
__device__ __forceinline__ void two_halves(float x, __half* hi, __half* lo) {
  *hi = __float2half_rn(x);
  *lo = __float2half_rn(x - __half2float(*hi));
}

// v with a power of two that puts its norm near 1 taken out, in two steps (either may be large).
struct Scaled {
  float p1, p2, q;  // x = ((v p1) p2) q
};
__device__ __forceinline__ float power2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }  // -126 <= e <= 127
__device__ __forceinline__ Scaled scaled_by(double size) {
  if (!(size < (double)INFINITY)) return Scaled{1.f, 1.f, __uint_as_float(kNan)};
  if (size == 0.) return Scaled{1.f, 1.f, 0.f};
  int e;
  const double f = frexp(size, &e);
  return Scaled{power2(-(e / 2)), power2(-(e - e / 2)), (float)((double)kX / f)};
}

// The squares of N numbers added up: in 32 bits, with a power of two taken out where they would
// not fit, so that the sum is the same at any magnitude.
template <int N>
__device__ __forceinline__ double squares(const float* f) {
  float s = 0.f, most = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    s = __fmaf_rn(f[i], f[i], s);
    most = fmaxf(most, fabsf(f[i]));
  }
  if (s > 0x1p-90f && s < 0x1p100f) return (double)s;
  if (s != s || most == INFINITY) return (double)s;
  if (most == 0.f) return 0.;
  int e;
  frexpf(most, &e);
  const float p1 = power2(-(e / 2)), p2 = power2(-(e - e / 2));
  s = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float v = f[i] * p1 * p2;
    s = __fmaf_rn(v, v, s);
  }
  return ldexp((double)s, 2 * e);
}
// Sums of squares of parts of each matrix G (as it is given: m rows of n), in a fixed order: warps
// take rows, or pieces of 4,096 elements of them.
constexpr int kMostSizeParts = 256, kSizePiece = 4096;
template <typename T>
__global__ void __launch_bounds__(256) k_size(const T* g, int64_t sk, int64_t ld, int64_t m, int64_t n, double* part,
                                              uint32_t* gave_up) {
  constexpr int N = Vec<T>::N;
  __shared__ double ws[8];
  griddep_wait();
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *gave_up = 0;
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
      const float v = Vec<T>::one(x[lane < head ? lane : len - tail + (lane - head)]);
      s += squares<1>(&v);
    }
#pragma unroll 4
    for (int i = lane; i < nv; i += 32) {
      float f[N];
      Vec<T>::get(*reinterpret_cast<const uint4*>(x + head + i * N), f);
      s += squares<N>(f);
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
__device__ __forceinline__ double size_of(const double* part, int parts) {  // by a block of 256
  __shared__ double ws[8];
  const double s = warp_sum((int)threadIdx.x < parts ? part[threadIdx.x] : 0.);
  if (threadIdx.x % 32 == 0) ws[threadIdx.x / 32] = s;
  __syncthreads();
  double t = 0.;
  for (int i = 0; i < 8; ++i) t += ws[i];
  return sqrt(t);
}
// The four pieces (8 columns of a row) of a block of halves that are a thread's: neighbours along a row
// of G, whichever way X lies.
template <bool kTurned>
__device__ __forceinline__ void piece_of(int u, int* row, int* piece) {
  const int t = (int)threadIdx.x;
  *row = kTurned ? t % 128 : t / 8 + 32 * u;
  *piece = kTurned ? t / 128 + 2 * u : t % 8;
}
// X = G / |G| as two halves, a block of them by a block.
template <typename T, bool kTurned>
__global__ void __launch_bounds__(256) k_first(const T* g, int64_t sk, int64_t ld, Shape S, const double* part, int parts,
                                               Halves2 X) {
  griddep_wait();
  const int64_t k = blockIdx.y, xc = S.np / 64, rb = blockIdx.x / xc, cb = blockIdx.x % xc;
  const Scaled by = scaled_by(size_of(part + k * kMostSizeParts, parts));
  const int64_t to = k * S.x() + blockIdx.x * (int64_t)kBlock;
  const bool vectors = !kTurned && ((reinterpret_cast<uintptr_t>(g) | (uintptr_t)(ld * sizeof(T)) | (uintptr_t)(sk * sizeof(T))) & 15) == 0;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    int row, piece;
    piece_of<kTurned>(u, &row, &piece);
    const int64_t i = rb * 128 + row, j0 = cb * 64 + piece * 8;
    float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (i < S.m) {
      const T* x = g + k * sk + (kTurned ? j0 * ld + i : i * ld + j0);
      if (vectors && j0 + 8 <= S.n) {
#pragma unroll
        for (int v = 0; v < 8; v += Vec<T>::N) Vec<T>::get(*reinterpret_cast<const uint4*>(x + v), f + v);
      } else {
#pragma unroll
        for (int v = 0; v < 8; ++v)
          if (j0 + v < S.n) f[v] = Vec<T>::one(x[v * (kTurned ? ld : 1)]);
      }
#pragma unroll
      for (int v = 0; v < 8; ++v)
        if (j0 + v < S.n) f[v] = f[v] * by.p1 * by.p2 * by.q;
    }
    alignas(16) __half hi[8], lo[8];
#pragma unroll
    for (int v = 0; v < 8; ++v) two_halves(f[v], hi + v, lo + v);
    const uint32_t in = piece_at((uint32_t)row, (uint32_t)piece);
    *reinterpret_cast<uint4*>(reinterpret_cast<char*>(X.hi + to) + in) = *reinterpret_cast<uint4*>(hi);
    *reinterpret_cast<uint4*>(reinterpret_cast<char*>(X.lo + to) + in) = *reinterpret_cast<uint4*>(lo);
  }
  fence_proxy_async_all();
}
template <typename T, bool kTurned>
__global__ void __launch_bounds__(256) k_last(T* out, int64_t sk, int64_t ld, Shape S, Halves2 X, float scale,
                                              const uint32_t* gave_up) {
  griddep_wait();
  const int64_t k = blockIdx.y, xc = S.np / 64, rb = blockIdx.x / xc, cb = blockIdx.x % xc;
  const int64_t from = k * S.x() + blockIdx.x * (int64_t)kBlock;
  const float by = *gave_up ? __uint_as_float(kNan) : scale * (1.f / kX);
  const bool vectors = !kTurned && ((reinterpret_cast<uintptr_t>(out) | (uintptr_t)(ld * sizeof(T)) | (uintptr_t)(sk * sizeof(T))) & 15) == 0;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    int row, piece;
    piece_of<kTurned>(u, &row, &piece);
    const int64_t i = rb * 128 + row, j0 = cb * 64 + piece * 8;
    if (i >= S.m || j0 >= S.n) continue;
    const uint32_t in = piece_at((uint32_t)row, (uint32_t)piece);
    float hi[8], lo[8];
    Vec<__half>::get(*reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(X.hi + from) + in), hi);
    Vec<__half>::get(*reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(X.lo + from) + in), lo);
#pragma unroll
    for (int v = 0; v < 8; ++v) hi[v] = (hi[v] + lo[v]) * by;
    T* x = out + k * sk + (kTurned ? j0 * ld + i : i * ld + j0);
    if (vectors && j0 + 8 <= S.n) {
#pragma unroll
      for (int v = 0; v < 8; v += Vec<T>::N) *reinterpret_cast<uint4*>(x + v) = Vec<T>::put(hi + v);
    } else {
#pragma unroll
      for (int v = 0; v < 8; ++v)
        if (j0 + v < S.n) x[v * (kTurned ? ld : 1)] = Vec<T>::round(hi[v]);
    }
  }
}

// -- products on the tensor cores ------------------------------------------------

__device__ __forceinline__ uint32_t remote(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ void arrive_at(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
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
// As wait_bounded, ordered after arrivals from the other block of the cluster; gives up at once where
// a thread of this block has given up. (The timer takes longer to read than most waits last: it is
// looked at every 256th time.)
__device__ __forceinline__ bool wait_for(uint64_t* bar, uint32_t parity, volatile uint32_t* dead) {
  uint64_t t0 = 0;
  for (uint32_t n = 1; !try_wait_cluster(bar, parity); ++n) {
    if (n % 256) continue;
    if (*dead) return false;
    const uint64_t now = global_ns();
    if (t0 == 0) t0 = now;
    if (now - t0 > kWaitLimitNs) {
      *dead = 1;
      return false;
    }
  }
  return true;
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
__device__ __forceinline__ void tmem_load32(uint32_t at, float* f) {
  uint32_t* r = reinterpret_cast<uint32_t*>(f);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
        "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
        "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(at));
}
__device__ __forceinline__ void tmem_loaded() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
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
  const __half* base;  // of the workspace, which the map is of
  Halves2 x, o, r, y;  // X, O, R; the new X
  float *d, *e;        // diagonals of A and B, mp each
  float a, b, c;
  uint32_t* gave_up;
};

constexpr int kFactorBytes = 16384;  // of a stage: 128 rows, or columns, by 64
constexpr int kHeldBytes = 4096;     // a warp's part of a block of halves
template <int CG, bool kFine>
struct Plan {
  static constexpr int kStages = kFine ? 2 : 5;
  static constexpr int kStageBytes = (kFine ? 4 : 2) * kFactorBytes;
  static constexpr int kWarps = 4 * CG;                // that read the sums back
  static constexpr int kThreads = 64 + 32 * kWarps;
  static constexpr int kBuffers = CG == 1 ? 2 : 1;     // of such a warp, two parts of a block each
  static constexpr int kHeld = kWarps * kBuffers * 2 * kHeldBytes;
  // Sums in the tensor cores are cut off, not rounded: by a quarter of a last place an addition where
  // all terms have one sign (4,608 columns of fp32 matrices: 2.8e-5 off the result, by three additions for
  // 16 columns). They are added up in registers after 128.
  static constexpr int kChunk = kFine ? 2 : 1 << 30;   // stages
};
struct alignas(8) ProductBars {
  uint64_t full[5], empty[5];
  uint64_t sums[2], taken[2];  // accumulators: written, read back
  uint64_t held[8][2];
  uint32_t tmem, dead;
};
template <int CG, bool kFine>
constexpr int product_smem() {
  using Pl = Plan<CG, kFine>;
  return Pl::kStages * Pl::kStageBytes + Pl::kHeld + 1024 + (int)sizeof(ProductBars);
}

// Tiles of all K matrices. A and B are symmetric: the tiles on and below the diagonal.
struct Tiles {
  int rows, cols;  // of a matrix; cols = 0: a triangle
  int64_t each, all;
  __device__ Tiles(const Shape& S, int64_t K, int unit, bool triangle) {
    rows = (int)(S.mp / unit);
    cols = triangle ? 0 : (int)(S.np / unit);
    each = triangle ? (int64_t)rows * (rows + 1) / 2 : (int64_t)rows * cols;
    all = each * K;
  }
  __device__ void at(int64_t t, int64_t* k, int* row, int* col) const {
    *k = t / each;
    const int i = (int)(t - *k * each);
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

// One product of all K matrices. A block holds 128 rows of the left factor and 128 rows (columns
// in kUpdate) of the right one, 64 of the sum at a time; a pair of blocks (CG = 2) shares them, and its tile
// is 256 x 256, 128 x 256 of it in each block's tensor memory; CG = 1: 128 x 128.
// Warp 0 issues the copies, warp 1 the products; the others read the sums back (the tensor memory
// holds two tiles) and put the new halves where the next product takes them from.
template <int CG, bool kFine, int kPhase>
__global__ void __launch_bounds__(Plan<CG, kFine>::kThreads, 1) k_product(const __grid_constant__ CUtensorMap map, ProductArgs P) {
  using Pl = Plan<CG, kFine>;
  extern __shared__ char raw[];
  char* smem = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  char* held = smem + Pl::kStages * Pl::kStageBytes;
  ProductBars& bars = *reinterpret_cast<ProductBars*>(held + Pl::kHeld);
  const int warp = (int)threadIdx.x / 32, lane = (int)threadIdx.x % 32;
  const uint32_t rank = CG == 2 ? cluster_rank() : 0;
  constexpr uint32_t kColumns = CG * 128;  // of an accumulator

  const Shape S = P.S;
  const int64_t xc = S.np / 64, oc = S.mp / 64;  // blocks in a row of blocks
  const Tiles tiles(S, P.K, 128 * CG, kPhase != kUpdate);
  const int64_t first = blockIdx.x / CG, step = gridDim.x / CG;
  const int kblocks = (int)(((kPhase == kGram ? S.n : S.m) + 63) / 64);

  if (threadIdx.x == 0) {
    for (int i = 0; i < Pl::kStages; ++i) {
      mbar_init(&bars.full[i], 1);
      mbar_init(&bars.empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars.sums[i], 1);
      mbar_init(&bars.taken[i], Pl::kWarps * CG);
      for (int w = 0; w < Pl::kWarps; ++w) mbar_init(&bars.held[w][i], 1);
    }
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
  volatile uint32_t* dead = &bars.dead;
  griddep_wait();

  if (warp == 0) {
    if (lane == 0) {
      const Halves2 left = kPhase == kGram ? P.x : kPhase == kSquare ? P.o : P.r;
      const Halves2 right = kPhase == kSquare ? P.o : P.x;
      // rows of 64 halves from the workspace's beginning
      const int64_t lh = (left.hi - P.base) / 64, rh = (right.hi - P.base) / 64;
      const int64_t ll = kFine ? (left.lo - left.hi) / 64 : 0, rl = kFine ? (right.lo - right.hi) / 64 : 0;
      const int64_t lk = (kPhase == kGram ? S.x() : S.o()) / 64, rk = (kPhase == kSquare ? S.o() : S.x()) / 64;
      const int64_t lc = kPhase == kGram ? xc : oc, rc = kPhase == kSquare ? oc : xc;
      uint32_t n = 0;  // stages filled
      bool going = true;
      for (int64_t t = first; t < tiles.all && going; t += step) {
        int64_t k;
        int row, col;
        tiles.at(t, &k, &row, &col);
        const int64_t ra = (int64_t)row * CG + rank, rb = (int64_t)col * CG + rank;
        for (int kb = 0; kb < kblocks; ++kb, ++n) {
          const int s = (int)(n % Pl::kStages);
          if (n >= Pl::kStages && !wait_for(&bars.empty[s], (n / Pl::kStages - 1) & 1, dead)) {
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
            tile_load<CG>(at, &map, l, bar);
            tile_load<CG>(at + kFactorBytes, &map, r, bar);
            if (kFine) {
              tile_load<CG>(at + 2 * kFactorBytes, &map, l + ll, bar);
              tile_load<CG>(at + 3 * kFactorBytes, &map, r + rl, bar);
            }
          }
        }
      }
      // what is under way has landed before the block ends
      if (rank == 0)
        for (uint32_t i = n > Pl::kStages ? n - Pl::kStages : 0; i < n; ++i)
          wait_bounded(&bars.full[i % Pl::kStages], (i / Pl::kStages) & 1, kWaitLimitNs);
      if (!going)  // (the other block's barrier may not count all of it)
        for (const uint64_t t0 = global_ns(); global_ns() - t0 < 2000000;) {}
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      // 32-bit sums of halves; the right factor's rows are the sum's index in kUpdate
      constexpr uint32_t what = 1u << 4 | (kPhase == kUpdate ? 1u << 16 : 0) | (CG * 128 / 8) << 17 | (CG * 128 / 16) << 24;
      uint32_t n = 0, it = 0;
      bool going = true;
      for (int64_t t = first; t < tiles.all && going; t += step) {
        for (int kb = 0; kb < kblocks && going; ++it) {
          const uint32_t acc = tmem + (it & 1) * kColumns;
          going = it < 2 || wait_for(&bars.taken[it & 1], (it / 2 - 1) & 1, dead);
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const int begin = kb, end = kblocks - kb > Pl::kChunk ? kb + Pl::kChunk : kblocks;
          for (; kb < end && going; ++kb, ++n) {
            const int s = (int)(n % Pl::kStages);
            going = wait_for(&bars.full[s], (n / Pl::kStages) & 1, dead);
            if (!going) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t at = smem_addr(smem + s * Pl::kStageBytes);
            constexpr uint32_t apart = kPhase == kUpdate ? kFactorBytes / 2 : 0;
            const uint64_t l = factor(at, 0), r = factor(at + kFactorBytes, apart);
            constexpr uint64_t lo = (2 * kFactorBytes) >> 4;
#pragma unroll
            for (int q = 0; q < 4; ++q) {  // 16 of the sum: 32 bytes of each row, or 16 rows
              const uint64_t dl = q * 32 >> 4, dr = (kPhase == kUpdate ? q * 2048 : q * 32) >> 4;
              if (kFine) {  // the small terms first, while there is less to cut off
                mma<CG>(acc, l + dl, r + dr + lo, what, kb > begin || q > 0);
                mma<CG>(acc, l + dl + lo, r + dr, what, true);
              }
              mma<CG>(acc, l + dl, r + dr, what, kFine || kb > begin || q > 0);
            }
            commit<CG>(&bars.empty[s]);
          }
          if (going) commit<CG>(&bars.sums[it & 1]);
        }
      }
      // the last products are done before the tensor memory is given back
      for (uint32_t i = n > Pl::kStages ? n - Pl::kStages : 0; i < n; ++i)
        wait_bounded(&bars.empty[i % Pl::kStages], (i / Pl::kStages) & 1, kWaitLimitNs);
    }
  } else {
    const int w = warp & 3, e = warp - 2;   // 32 rows of the block's part of the tile, and 128 columns
    char* mine = held + e * Pl::kBuffers * 2 * kHeldBytes;
    uint64_t* in = bars.held[e];
    constexpr bool kLow = kPhase == kUpdate || kFine;  // two halves are kept
    const Halves2 from = kPhase == kUpdate ? P.x : P.o, to = kPhase == kGram ? P.o : kPhase == kSquare ? P.r : P.y;
    const int64_t bc = kPhase == kUpdate ? xc : oc, plane = kPhase == kUpdate ? S.x() : S.o();
    // where this warp's part of a block of halves lies
    auto part_of = [&](int64_t k, int row, int col, int c) {
      const int64_t rb = (int64_t)row * CG + rank, cb = (int64_t)col * (2 * CG) + e / 4 * 2 + c;
      return k * plane + (rb * bc + cb) * kBlock + w * (kHeldBytes / 2);
    };
    uint32_t fetched = 0;
    auto fetch = [&](int64_t t, int c) {  // the next one
      if (kPhase == kGram || t >= tiles.all) return;
      int64_t k;
      int row, col;
      tiles.at(t, &k, &row, &col);
      const int64_t at = part_of(k, row, col, c);
      char* b = mine + fetched % Pl::kBuffers * 2 * kHeldBytes;
      uint64_t* bar = &in[fetched % Pl::kBuffers];
      mbar_arrive_expect_tx(bar, (kLow ? 2 : 1) * kHeldBytes);
      bulk_load(b, from.hi + at, kHeldBytes, bar);
      if (kLow) bulk_load(b + kHeldBytes, from.lo + at, kHeldBytes, bar);
      ++fetched;
    };
    uint32_t q = 0, it = 0;
    bool going = true;
    if (lane == 0) fetch(first, 0);
    for (int64_t t = first; t < tiles.all && going; t += step) {
      int64_t k;
      int tr, tc;
      tiles.at(t, &k, &tr, &tc);
      const int64_t row = ((int64_t)tr * CG + rank) * 128 + w * 32 + lane;
      const float* D = P.d + k * S.mp;
      const float di = kPhase == kSquare ? D[row] : 0.f, ei = kPhase == kUpdate ? P.a + P.e[k * S.mp + row] : 0.f;
      float sum[kFine ? 128 : 1];
      if constexpr (kFine) {
#pragma unroll
        for (int i = 0; i < 128; ++i) sum[i] = 0.f;
        for (int kb = 0; kb < kblocks && going; kb += Pl::kChunk, ++it) {
          going = __all_sync(0xffffffffu, wait_for(&bars.sums[it & 1], (it / 2) & 1, dead));
          if (!going) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float acc[32];
            tmem_load32(tmem + (it & 1) * kColumns + e / 4 * 128 + i * 32 + ((uint32_t)w << 21), acc);
            tmem_loaded();
#pragma unroll
            for (int u = 0; u < 32; ++u) sum[i * 32 + u] += acc[u];
          }
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          __syncwarp();
          if (lane == 0) arrive_at(remote(smem_addr(&bars.taken[it & 1]), 0));
        }
      } else {
        going = __all_sync(0xffffffffu, wait_for(&bars.sums[it & 1], (it / 2) & 1, dead));
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      }
      if (!going) break;
#pragma unroll
      for (int c = 0; c < 2; ++c, ++q) {
        char* b = mine + q % Pl::kBuffers * 2 * kHeldBytes;
        if (lane == 0) {
          bulk_read();  // earlier stores: what they were read from may be written again
          if (Pl::kBuffers == 2) fetch(c == 0 ? t : t + step, c ^ 1);
        }
        __syncwarp();
        if (kPhase != kGram)
          going = __all_sync(0xffffffffu, wait_for(&in[q % Pl::kBuffers], (q / Pl::kBuffers) & 1, dead));
        if (!going) break;
        const int64_t col0 = ((int64_t)tc * (2 * CG) + e / 4 * 2 + c) * 64;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          float acc[32];
          if constexpr (kFine) {
#pragma unroll
            for (int u = 0; u < 32; ++u) acc[u] = sum[c * 64 + half * 32 + u];
          } else {
            tmem_load32(tmem + (it & 1) * kColumns + e / 4 * 128 + c * 64 + half * 32 + ((uint32_t)w << 21), acc);
            tmem_loaded();
          }
#pragma unroll
          for (int p = 0; p < 4; ++p) {
            char* at = b + piece_at((uint32_t)lane, (uint32_t)(half * 4 + p));
            float was[8];
            if (kPhase != kGram) {
              Vec<__half>::get(*reinterpret_cast<const uint4*>(at), was);
              if (kLow) {
                float low[8];
                Vec<__half>::get(*reinterpret_cast<const uint4*>(at + kHeldBytes), low);
#pragma unroll
                for (int u = 0; u < 8; ++u) was[u] += low[u];
              }
            }
            alignas(16) __half nh[8], nl[8];
            const int64_t col = col0 + half * 32 + p * 8;
#pragma unroll
            for (int u = 0; u < 8; ++u) {
              float v = acc[p * 8 + u];
              if constexpr (kPhase == kGram) {
                v *= kO / (kX * kX);
                if (col + u == row) P.d[k * S.mp + row] = v * (1.f / kO), v = 0.f;
              } else if constexpr (kPhase == kSquare) {
                v *= 1.f / kO;  // O^2, 2^11 times
                if (col + u == row) {
                  P.e[k * S.mp + row] = P.b * di + P.c * __fmaf_rn(di, di, v * (1.f / kO));
                  v = 0.f;
                } else {
                  v = P.b * was[u] + P.c * __fmaf_rn(di + D[col + u], was[u], v);
                }
              } else {
                v = __fmaf_rn(ei, was[u], v * (1.f / kO));
              }
              two_halves(v, nh + u, nl + u);
            }
            *reinterpret_cast<uint4*>(at) = *reinterpret_cast<const uint4*>(nh);
            if (kLow) *reinterpret_cast<uint4*>(at + kHeldBytes) = *reinterpret_cast<const uint4*>(nl);
          }
        }
        if (!kFine && c == 1) {  // the sums are read
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          __syncwarp();
          if (lane == 0) arrive_at(remote(smem_addr(&bars.taken[it & 1]), 0));
        }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) {
          const int64_t at = part_of(k, tr, tc, c);
          bulk_store(to.hi + at, b, kHeldBytes);
          if (kLow) bulk_store(to.lo + at, b + kHeldBytes, kHeldBytes);
          bulk_commit();
        }
        if (kPhase != kUpdate && tr != tc) {
          // the same above the diagonal: this warp's 64 columns are rows there, two of them a lane, its rows
          // 32 columns, four pieces
          const int64_t rb = ((int64_t)tc * (2 * CG) + e / 4 * 2 + c) / 2;  // (64 columns: half a block's rows)
          const int64_t cb = ((int64_t)tr * CG + rank) * 2 + w / 2;
          const int64_t block = k * plane + (rb * bc + cb) * kBlock;
#pragma unroll
          for (int low = 0; low < (kLow ? 2 : 1); ++low) {
            const char* plane_at = b + low * kHeldBytes;
            char* out = reinterpret_cast<char*>((low ? to.lo : to.hi) + block);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint32_t j = h * 32 + lane, r = c * 64 + j;  // column here, row there
#pragma unroll
              for (int p = 0; p < 4; ++p) {
                alignas(16) uint16_t v[8];
#pragma unroll
                for (int u = 0; u < 8; ++u)
                  v[u] = *reinterpret_cast<const uint16_t*>(plane_at + piece_at((uint32_t)(p * 8 + u), j / 8) + j % 8 * 2);
                *reinterpret_cast<uint4*>(out + piece_at(r, (uint32_t)(w % 2 * 4 + p))) = *reinterpret_cast<const uint4*>(v);
              }
            }
          }
        }
        if (Pl::kBuffers == 1) {
          __syncwarp();
          if (lane == 0) {
            bulk_read();
            fetch(c == 0 ? t : t + step, c ^ 1);
          }
        }
      }
      if (!kFine) ++it;
    }
    if (kPhase != kUpdate) fence_proxy_async_all();
    if (lane == 0) {
      bulk_done();
      for (uint32_t i = fetched > Pl::kBuffers ? fetched - Pl::kBuffers : 0; i < fetched; ++i)
        wait_bounded(&in[i % Pl::kBuffers], (i / Pl::kBuffers) & 1, kWaitLimitNs);
    }
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

template <int CG, bool kFine, int kPhase>
cudaError_t launch_product(const CUtensorMap& map, const ProductArgs& P, int device, int sms, cudaStream_t s) {
  using Pl = Plan<CG, kFine>;
  constexpr int smem = product_smem<CG, kFine>();
  static_assert(smem <= 232448, "shared memory of a block");
  auto* f = k_product<CG, kFine, kPhase>;
  static std::atomic<uint64_t> known{0};  // devices whose limit is raised
  if (device >= 64 || !(known.load(std::memory_order_relaxed) >> device & 1)) {
    const cudaError_t e = cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    if (device < 64) known.fetch_or(uint64_t(1) << device, std::memory_order_relaxed);
  }
  const int64_t rows = P.S.mp / (128 * CG), cols = P.S.np / (128 * CG);
  const int64_t most = sms / CG, tiles = P.K * (kPhase == kUpdate ? rows * cols : rows * (rows + 1) / 2);
  if (CG > 1 && refuse_cooperative()) return cudaErrorCooperativeLaunchTooLarge;
  LaunchConfig l((tiles < most ? tiles : most) * CG, Pl::kThreads, CG, smem, s);
  return cudaLaunchKernelEx(&l.cfg, f, map, P);
}
template <int CG, bool kFine>
cudaError_t one_step(const CUtensorMap& map, const ProductArgs& P, int device, int sms, cudaStream_t s) {
  cudaError_t e = launch_product<CG, kFine, kGram>(map, P, device, sms, s);
  if (e == cudaSuccess) e = launch_product<CG, kFine, kSquare>(map, P, device, sms, s);
  if (e == cudaSuccess) e = launch_product<CG, kFine, kUpdate>(map, P, device, sms, s);
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

struct Work {
  double* part;
  uint32_t* gave_up;
  float *d, *e;
  Halves2 x, y, o, r;
};
int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
// Whether pairs of blocks take tiles of 256 x 256.
bool by_pairs(int64_t m, int64_t n) { return (m < n ? m : n) >= 512; }
Shape shape_of(int64_t m, int64_t n) {
  const int64_t whole = by_pairs(m, n) ? 256 : 128;
  if (m > n) {
    const int64_t t = m;
    m = n;
    n = t;
  }
  return Shape{m, n, up(m, whole), up(n, whole)};
}
int64_t work_of(int32_t dtype, int64_t K, const Shape& S, char* at, Work* w) {
  int64_t bytes = 0;
  auto take = [&](int64_t n) {
    char* p = at + bytes;
    bytes += up(n, 1024);
    return p;
  };
  Work v;
  v.part = reinterpret_cast<double*>(take(8 * K * kMostSizeParts));
  v.gave_up = reinterpret_cast<uint32_t*>(take(4));
  v.d = reinterpret_cast<float*>(take(4 * K * S.mp));
  v.e = reinterpret_cast<float*>(take(4 * K * S.mp));
  const bool fine = dtype != GMC_BF16;
  for (Halves2* h : {&v.x, &v.y, &v.o, &v.r}) {
    const bool is_x = h == &v.x || h == &v.y;
    const int64_t n = 2 * K * (is_x ? S.x() : S.o());
    h->hi = reinterpret_cast<__half*>(take(n));
    h->lo = is_x || fine ? reinterpret_cast<__half*>(take(n)) : nullptr;
  }
  if (w) *w = v;
  return bytes;
}

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
  const int64_t bytes = work_of(dtype, K, shape_of(m, n), nullptr, nullptr);
  return bytes <= kMostWork ? bytes : -1;
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
  const int64_t need = work_of(dtype, K, S, static_cast<char*>(workspace_dev), &w);
  if (!workspace_dev || reinterpret_cast<uintptr_t>(workspace_dev) % 256 || need > kMostWork || workspace_bytes < need)
    return GMC_EINVAL;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool turned = m > n;
  bool pairs = by_pairs(m, n);
  int device = 0, sms = 0;
  cudaError_t err = cudaGetDevice(&device);
  if (err == cudaSuccess) err = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
  if (err != cudaSuccess) return GMC_ECUDA;
  CUtensorMap map;
  err = map_of(workspace_dev, need, &map);
  if (err != cudaSuccess) return GMC_ECUDA;
  // parts of |G|^2: as many blocks as are resident at once, of eight rows or pieces each
  const int64_t rows8 = (m * ((n + kSizePiece - 1) / kSizePiece) + 7) / 8, share = (sms * 8 + K - 1) / K;
  const int parts = (int)std::min({rows8, share, (int64_t)kMostSizeParts});
  const dim3 blocks((unsigned)(S.x() / kBlock), (unsigned)K);
  err = by_type(dtype, [&](auto t) {
    using T = decltype(t);
    constexpr bool fine = !std::is_same<T, __nv_bfloat16>::value;
    const T* g = static_cast<const T*>(x_dev);
    T* o = static_cast<T*>(out_dev);
    cudaError_t e = launch_pdl(k_size<T>, dim3((unsigned)parts, (unsigned)K), dim3(256), 0, s, g, ldk, ld, m, n, w.part, w.gave_up);
    if (e != cudaSuccess) return e;
    e = launch_pdl(turned ? k_first<T, true> : k_first<T, false>, blocks, dim3(256), 0, s, g, ldk, ld, S, (const double*)w.part,
                   parts, w.x);
    for (int i = 0; i < steps && e == cudaSuccess; ++i) {
      const float* c = coefficients_host + 3 * i;
      const ProductArgs P{S, K, static_cast<const __half*>(workspace_dev), w.x, w.o, w.r, w.y, w.d, w.e, c[0], c[1], c[2], w.gave_up};
      if (pairs) e = one_step<2, fine>(map, P, device, sms, s);
      if (pairs && too_large_here(e)) {  // a context without room for clusters
        cudaGetLastError();              // this launch's
        pairs = false;
      }
      if (!pairs) e = one_step<1, fine>(map, P, device, sms, s);
      const Halves2 was = w.x;
      w.x = w.y;
      w.y = was;
    }
    if (e != cudaSuccess) return e;
    return launch_pdl(turned ? k_last<T, true> : k_last<T, false>, blocks, dim3(256), 0, s, o, out_ldk, out_ld, S, w.x, scale,
                      (const uint32_t*)w.gave_up);
  });
  return err == cudaSuccess ? GMC_OK : GMC_ECUDA;
}

}  // extern "C"
