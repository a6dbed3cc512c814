// The orthogonalised update direction of G workers' weight matrices: momentum, then `steps` products that bring the
// singular values of the (Frobenius-normalised) momentum near one.
//
//   u = m u + g,  x = g + m u (Nesterov) or u,  X = x / ||x||_F,
//   steps times:  A = X X^T,  P = b A + c A A,  X = a X + P X      (a, b, c) = (3.4445, -4.7750, 2.0315),
//   o = X in bf16.
//
// With n the smaller and m the larger of the two sizes, A and P are n x n and symmetric; where the rows are the more,
// A = X^T X and X = a X + X P.  Work: n^2 m + n^3 + 2 n^2 m ... of which the two symmetric products need a triangle.
//
// Number formats.  The products run on the tensor cores with fp16 operands and fp32 sums.  A step multiplies small
// singular values by a = 3.4445, five steps by 485, and so the rounding errors of X where X itself has nothing: rank-
// deficient momenta (a gradient's rank is at most its mini-batch) would come out of bf16 operands 10 to 100 % off, of fp16
// ones 1 to 15 %.  So X is carried as a pair of fp16 values, X = h + l (22 bits).  h is the products' operand: P h, with P's
// rounding, adds nothing outside the space that X spans.  The diagonals of A and P stay in fp32 vectors dA and d (the
// operands have zeros there), which leaves fewer and smaller roundings, and the last product's epilogue forms
//   X' = (a + d_i) h + (a + t) l + (P - diag d) h.
// t stands in for the part of P l that is a multiple of l: 0, but in the last two steps the largest d_i.  (A t that is not
// an eigenvalue of P puts (P - t) l where X has nothing, which later steps would amplify.)  fp16 rather than bf16: the
// same rate, 3 more bits; its range is enough because every value is stored times 2^12 and bounded: singular values of X
// are at most 1.21, so |A| < 1.47 and |P| < 2.9 at all steps.  Measured and modelled: 6e-4 to 1.3e-3 off (relative 2-norm,
// before the bf16 rounding of 1.7e-3) for random, rank-deficient and ill-conditioned matrices, up to 1.9e-3 for a handful of
// values or a smaller side of at most 64.
#include <cuda_fp16.h>
#include <cudaTypedefs.h>

#include <algorithm>
#include <atomic>
#include <mutex>
#include <string>
#include <type_traits>

#include "../../include/lsgd.h"
#include "common.cuh"
#include "lsgd_internal.h"
#include "tc_ptx.cuh"

namespace lsgd {

__device__ int g_direction_timeout = 0;
static std::atomic<bool> g_direction_used{false};  // the flag is read only once a call has been made

namespace {

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr float kUnscale = 1.f / 4096.f, kUnscale2 = kUnscale * kUnscale;  // values are stored times 2^12
constexpr long long kWaitCycles = 4000000000LL;  // ~2 s at 2 GHz

// ------------------------------------------------------------------------------------------------
// Momentum and the norm

// Sums of squares in three ranges, so that neither overflow nor underflow of a square loses the norm (as in Blue's
// 1978 algorithm, with fixed scalings).
struct NormSums {
  float mid, big, small;
};
constexpr float kBig = 0x1p-80f, kSmall = 0x1p84f;

__device__ __forceinline__ void norm_add(NormSums& s, float x) {
  s.mid = fmaf(x, x, s.mid);
  const float b = x * kBig, t = x * kSmall;
  s.big = fmaf(b, b, s.big);
  s.small = fmaf(t, t, s.small);
}

// 2^12 / ||x|| as two factors, applied one after the other without leaving the range of fp32, from the sums over the
// matrix.  ||x|| = 0 gives 0: the direction of a zero matrix is zero.  (fp32 sums of at most 256 in a row: an error of the norm
// scales X, by 1 + 2e-6 for equal squares of the worst of 40 sizes and less for others.)
__device__ __forceinline__ float2 norm_factors(float mid, float big, float small) {
  if (mid > 0x1p-60f && mid < 0x1p120f) return make_float2(__frsqrt_rn(mid), 4096.f);
  if (!(mid < 0x1p120f)) return make_float2(__frsqrt_rn(big), 0x1p-68f);  // also infinite and NaN values: 0 or NaN times them
  return small == 0.f ? make_float2(0.f, 0.f) : make_float2(__frsqrt_rn(small), 0x1p96f);
}

struct DirArgs {
  float* u;
  const void* g;
  uint16_t* o;
  int64_t u_gs, g_gs, o_gs;
  int g_bf16, nesterov;
  float mom;
  int G, rows, cols;
  int64_t ld;        // of h and l (a multiple of 16)
  __half *h, *l;     // [G][rows][ld]
  float* part;       // [G][chunks][3]
  int chunks, per;   // ranges of a matrix (elements per range)
  uint32_t* done;    // [3][G] (done and top of the products), set to zero for them
};

constexpr int kMomThreads = 256;

// Two passes before the products, because all of a matrix's squares come before its first quotient: u and the norm's partial
// sums, then h and l.  Bound by memory, 12 bytes a value each (the second finds part of u and g in L2): 27 and 31 us for 16 x
// 1024 x 1024 in fp32, 7.4 and 6.5 TB/s.  Vectors of 8 or 4 values where every matrix's rows are aligned to them, single
// values otherwise (the whole call 401, 403 and 438 us).

// V gradient or momentum values from element i of a matrix.
template <int V>
__device__ __forceinline__ void load_f32(const float* p, float (&v)[V]) {
  if constexpr (V == 1) {
    v[0] = *p;
  } else {
#pragma unroll
    for (int j = 0; j < V / 4; ++j) {
      const float4 t = reinterpret_cast<const float4*>(p)[j];
      v[4 * j] = t.x, v[4 * j + 1] = t.y, v[4 * j + 2] = t.z, v[4 * j + 3] = t.w;
    }
  }
}
// One gradient value whose type is known.
template <bool BF16>
__device__ __forceinline__ float grad_value(const void* g, int64_t i) {
  return BF16 ? bf2f(static_cast<const uint16_t*>(g)[i]) : static_cast<const float*>(g)[i];
}
template <int V>
__device__ __forceinline__ void load_grad(const DirArgs& a, int64_t i, float (&v)[V]) {
  if (!a.g_bf16) {
    load_f32<V>(static_cast<const float*>(a.g) + i, v);
    return;
  }
  const uint16_t* p = static_cast<const uint16_t*>(a.g) + i;
  if constexpr (V == 1) {
    v[0] = bf2f(*p);
  } else {
#pragma unroll
    for (int j = 0; j < V / 4; ++j) {
      const uint2 t = reinterpret_cast<const uint2*>(p)[j];
      v[4 * j] = __uint_as_float(t.x << 16), v[4 * j + 1] = __uint_as_float(t.x & 0xffff0000u);
      v[4 * j + 2] = __uint_as_float(t.y << 16), v[4 * j + 3] = __uint_as_float(t.y & 0xffff0000u);
    }
  }
}

template <int V>
__global__ void __launch_bounds__(kMomThreads) direction_momentum_kernel(const DirArgs a) {
  pdl_begin();
  const int n = a.rows * a.cols, i0 = blockIdx.x * a.per, i1 = min(n, i0 + a.per);
  const int64_t k = blockIdx.y;
  if (blockIdx.x == 0 && threadIdx.x < 3) a.done[threadIdx.x * a.G + k] = 0;
  // a thread's squares 64 at a time, at most 256 times: of 16384 equal ones in a row the sum would be 1.6e-4 off
  constexpr int kStep = kMomThreads * V, kSegment = 64 * kMomThreads;
  NormSums s{0.f, 0.f, 0.f};
  for (int from = i0 + threadIdx.x * V; from < i1; from += kSegment) {
    const int end = min(i1, from + kSegment);
    NormSums some{0.f, 0.f, 0.f};
#pragma unroll 2
    for (int i = from; i < end; i += kStep) {
      float x[V];
      load_grad<V>(a, k * a.g_gs + i, x);
      if (a.mom != 0.f) {
        float u[V];
        float* up = a.u + k * a.u_gs + i;
        load_f32<V>(up, u);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          u[j] = fmaf(a.mom, u[j], x[j]);
          x[j] = a.nesterov ? fmaf(a.mom, u[j], x[j]) : u[j];
        }
        if constexpr (V == 1) {
          *up = u[0];
        } else {
#pragma unroll
          for (int j = 0; j < V / 4; ++j)
            reinterpret_cast<float4*>(up)[j] = make_float4(u[4 * j], u[4 * j + 1], u[4 * j + 2], u[4 * j + 3]);
        }
      }
#pragma unroll
      for (int j = 0; j < V; ++j) norm_add(some, x[j]);
    }
    s.mid += some.mid, s.big += some.big, s.small += some.small;
  }
  __shared__ float red[3][kMomThreads / 32];
  float v[3] = {s.mid, s.big, s.small};
#pragma unroll
  for (int j = 0; j < 3; ++j) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v[j] += __shfl_xor_sync(~0u, v[j], o);
    if ((threadIdx.x & 31) == 0) red[j][threadIdx.x >> 5] = v[j];
  }
  __syncthreads();
  if (threadIdx.x < 3) {
    float t = 0.f;
    for (int w = 0; w < kMomThreads / 32; ++w) t += red[threadIdx.x][w];
    a.part[(k * a.chunks + blockIdx.x) * 3 + threadIdx.x] = t;
  }
}

__device__ __forceinline__ void split_pair(float x, __half& h, __half& l) {
  h = __float2half_rn(x);
  l = __float2half_rn(x - __half2float(h));
}

template <int V>
__global__ void __launch_bounds__(kMomThreads) direction_normalise_kernel(const DirArgs a) {
  pdl_begin();
  const int64_t k = blockIdx.y;
  __shared__ float2 factors;
  if (threadIdx.x < 32) {
    float t[3] = {0.f, 0.f, 0.f};
    for (int c = threadIdx.x; c < a.chunks; c += 32)
      for (int j = 0; j < 3; ++j) t[j] += a.part[(k * a.chunks + c) * 3 + j];
    for (int j = 0; j < 3; ++j)
      for (int o = 16; o; o >>= 1) t[j] += __shfl_xor_sync(~0u, t[j], o);
    if (threadIdx.x == 0) factors = norm_factors(t[0], t[1], t[2]);
  }
  __syncthreads();
  const float2 f = factors;
  const int n = a.rows * a.cols, i0 = blockIdx.x * a.per, i1 = min(n, i0 + a.per);
#pragma unroll 2
  for (int i = i0 + threadIdx.x * V; i < i1; i += kMomThreads * V) {
    float x[V];
    if (a.mom == 0.f) {
      load_grad<V>(a, k * a.g_gs + i, x);
    } else {
      load_f32<V>(a.u + k * a.u_gs + i, x);
      if (a.nesterov) {
        float g[V];
        load_grad<V>(a, k * a.g_gs + i, g);
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] = fmaf(a.mom, x[j], g[j]);
      }
    }
    __align__(16) __half h[V], l[V];
#pragma unroll
    for (int j = 0; j < V; ++j) split_pair(x[j] * f.x * f.y, h[j], l[j]);
    const int r = (uint32_t)i / (uint32_t)a.cols;
    const int64_t at = (k * a.rows + r) * a.ld + (i - r * a.cols);
    if constexpr (V == 1) {
      a.h[at] = h[0];
      a.l[at] = l[0];
    } else if constexpr (V == 4) {
      *reinterpret_cast<uint2*>(a.h + at) = *reinterpret_cast<const uint2*>(h);
      *reinterpret_cast<uint2*>(a.l + at) = *reinterpret_cast<const uint2*>(l);
    } else {
      *reinterpret_cast<uint4*>(a.h + at) = *reinterpret_cast<const uint4*>(h);
      *reinterpret_cast<uint4*>(a.l + at) = *reinterpret_cast<const uint4*>(l);
    }
  }
}

// ------------------------------------------------------------------------------------------------
// The products: pairs of CTAs on 256 x 256 tiles (tcgen05 cta_group::2), all steps in one launch
//
// A cluster of two CTAs computes a 256 x 256 fp32 tile; CTA r holds rows 128 r .. of it in its tensor memory, loads rows
// 128 r .. of the left operand and 128 r .. of the right operand's 256, and the leader (r = 0) issues the products, which
// read both CTAs' shared memory.  Per k-block of 64 a CTA moves 32 KB for 128 x 256 x 64 products, two thirds of what
// a 128 x 256 tile by one CTA would.
//   warp 0      TMA producer of both operands into a ring of kStages stages (both CTAs' bytes counted on the leader's
//               barrier)
//   warp 1      MMA issuer (leader only)
//   warp 2      tensor memory allocation (two accumulators of a tile's columns); TMA stores of the epilogue's buffers, and the
//               count of finished tiles
//   warp 3      TMA loads of what the epilogue reads (h and l, or A), 64 columns at a time into a ring of kEpi buffers,
//               ahead of the accumulator
//   warps 4-19  epilogue: a warp per 32 rows and 16 columns of a buffer, in place, each at its own pace (8 warps took 13,000
//               cycles a tile, mostly latencies, against the products' 8,200 at k = 1024)
//
// Where the tiles are few (PAIR false) each CTA works for itself on 128 x 128 tiles: half the products and half the epilogue
// between a tile's start and its count, for twice the operand bytes per product (direction_pairs chooses).
//
// The tiles of all steps form one list: per step the tiles of A = X X^T of every matrix, then those of P, then those of
// X.  Pair p takes tiles p, p + pairs, ...; `done[g]` counts the CTAs' finished tiles of matrix g, whose phases follow one
// another, and a tile starts when its matrix's earlier phases are complete.  The launch is cooperative (all pairs are
// resident) and every tile's predecessors stand before it in the list, so that every wait ends; matrices fill each
// other's phase ends, and nothing is launched between phases.
//
// Measured, five steps: 16 x 1024 x 1024 in 329 us (1.04 PFLOP/s of the products that symmetry leaves; the tensor pipe is active
// 50 % of the time and L2 at 46 % of its peak: neither is the bound.  Tiles wait for their matrix at the phases' ends; the rest is
// latency that has not been told apart), 4 x 4096 x 4096 in 4.1 ms (1.34 PFLOP/s; the SM clock falls to 1.4 GHz under the power
// limit, where a library product runs at 1.70).

constexpr int kHalf = 128, kBK = 64, kStages = 4, kEpi = 3, kEpiWarps = 16, kThreads = 128 + 32 * kEpiWarps, kChunk = 64;
constexpr uint32_t kOpBytes = kHalf * kBK * 2;  // one operand's share of a stage in a CTA; half an epilogue buffer

enum Role { GRAM = 0, POLY = 1, NEXT = 2, LAST = 3 };

struct MmArgs {
  // K-major operands and epilogue tiles: box {64, 128}; MN-major operands and mirrored tiles: box {64, 64}
  CUtensorMap xk[2], xm[2], lk[2], ak, am, pk, pm, om;
  int G, n, rows, cols, steps, tall, o_tma;
  float *diag_a, *diag;  // [G][n]: the diagonals of A and P
  uint32_t* done;        // [G]
  uint32_t* top;         // [2][G]: the largest of P's diagonal in each of the last two steps, as an ordered integer
  uint16_t* o;
  int64_t o_gs;
};

struct MmSmem {
  uint8_t a[kStages][kOpBytes];  // 1024-aligned
  uint8_t b[kStages][kOpBytes];
  uint8_t e[kEpi][2][kOpBytes];  // h or A and the tile stored; l or the mirrored tile
  uint64_t full[kStages], empty[kStages];
  uint64_t acc_full[2], acc_empty[2];
  uint64_t epi_full[kEpi], epi_ready[kEpi], epi_empty[kEpi];
  uint32_t tmem_base;
};

__device__ __forceinline__ bool wait_bar(uint64_t* bar, uint32_t parity) {
  const uint32_t at = smem_u32(bar);
  auto poll = [&]() -> bool {
    uint32_t ok;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n"
        " selp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(ok)
        : "r"(at), "r"(parity)
        : "memory");
    return ok != 0;
  };
  if (poll()) return true;
  const long long t0 = clock64();
  while (!poll()) {
    if (clock64() - t0 > kWaitCycles) {
      atomicExch(&g_direction_timeout, 1);
      return false;
    }
  }
  return true;
}
__device__ __forceinline__ bool wait_bar_warp(uint64_t* bar, uint32_t parity) {
  return __all_sync(0xffffffffu, wait_bar(bar, parity) ? 1 : 0) != 0;
}
// Until *count, counted up by other CTAs, has reached `need` (by the whole warp).  What they wrote before is then visible
// to this warp's loads and, behind the proxy fence, to its TMA copies.
__device__ __forceinline__ bool wait_count_warp(const uint32_t* count, uint32_t need) {
  int ok = 1;
  if ((threadIdx.x & 31) == 0) {
    auto reached = [&]() -> bool {
      uint32_t v;
      asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(count) : "memory");
      return v >= need;
    };
    if (!reached()) {
      const long long t0 = clock64();
      while (!reached()) {
        if (clock64() - t0 > kWaitCycles) {
          atomicExch(&g_direction_timeout, 1);
          ok = 0;
          break;
        }
        __nanosleep(64);
      }
    }
  }
  ok = __shfl_sync(0xffffffffu, ok, 0);
  asm volatile("fence.proxy.async.global;" ::: "memory");
  return ok != 0;
}

// An order-preserving map of floats to integers above 0, and back.
__device__ __forceinline__ uint32_t to_ordered(float f) {
  const uint32_t b = __float_as_uint(f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float from_ordered(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

__device__ __forceinline__ uint32_t cta_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t in_cta(const void* p, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(p)), "r"(rank));
  return r;
}
__device__ __forceinline__ void pair_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// A box into this CTA's shared memory, its bytes counted on the barrier at cluster address `bar`.
__device__ __forceinline__ void tma_load_pair(void* dst, const CUtensorMap* map, uint32_t bar, int x, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(y), "r"(z)
      : "memory");
}
__device__ __forceinline__ void tma_store(const CUtensorMap* map, const void* src, int x, int y, int z) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(
                   reinterpret_cast<uint64_t>(map)),
               "r"(smem_u32(src)), "r"(x), "r"(y), "r"(z)
               : "memory");
}
__device__ __forceinline__ void mma_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
// One arrival on the barrier at this offset of both CTAs once the products issued so far are done.
__device__ __forceinline__ void commit_pair(uint64_t* bar) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
          smem_u32(bar)),
      "h"((uint16_t)3)
      : "memory");
}
__device__ __forceinline__ void mma_one(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void commit_one(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
template <bool PAIR>
__device__ __forceinline__ void mma_of(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  if constexpr (PAIR) mma_pair(d, a, b, idesc, accumulate);
  else mma_one(d, a, b, idesc, accumulate);
}
template <bool PAIR>
__device__ __forceinline__ void commit_of(uint64_t* bar) {
  if constexpr (PAIR) commit_pair(bar);
  else commit_one(bar);
}
__device__ __forceinline__ void arrive_at(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// 16 accumulator columns of this warp's 32 rows, one row per lane.
__device__ __forceinline__ void tmem_ld16(uint32_t at, float (&v)[16]) {
  uint32_t r[16];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(at)
      : "memory");
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}

// Shared memory by its 32-bit address.
__device__ __forceinline__ uint4 lds16(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ void sts16(uint32_t at, const uint4 v) {
  asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ void sts2(uint32_t at, uint32_t low_half) {
  asm volatile("{\n .reg .b16 h, x;\n mov.b32 {h, x}, %1;\n st.shared.b16 [%0], h;\n}\n" ::"r"(at), "r"(low_half) : "memory");
}

// Eight fp16 (or bf16) values in 16 bytes.
__device__ __forceinline__ void unpack8(const uint4 w, float (&f)[8]) {
  const uint32_t r[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 t = __half22float2(*reinterpret_cast<const __half2*>(&r[i]));
    f[2 * i] = t.x, f[2 * i + 1] = t.y;
  }
}
__device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
  uint32_t r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half2 t = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
    r[i] = *reinterpret_cast<const uint32_t*>(&t);
  }
  return make_uint4(r[0], r[1], r[2], r[3]);
}
__device__ __forceinline__ uint4 pack8_bf16(const float (&f)[8]) {
  uint32_t r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 t = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
    r[i] = *reinterpret_cast<const uint32_t*>(&t);
  }
  return make_uint4(r[0], r[1], r[2], r[3]);
}

// One tile of the list.
struct Item {
  int role, step, g, m0, n0, M, N, K;
  uint32_t need;  // of done[g], before it starts
};
template <bool PAIR>
struct Plan {
  static constexpr int kTile = PAIR ? 256 : 128;
  static constexpr uint32_t kCtas = PAIR ? 2 : 1;  // counts of a finished tile
  int ts, tm, tn, per_sym, per_x;  // tiles a side of A; of X; tiles of a symmetric product and of X
  int per_step, total;  // the host has checked that the list has fewer than 2^31 tiles
  __device__ __forceinline__ explicit Plan(const MmArgs& a) {
    ts = (a.n + kTile - 1) / kTile;
    tm = (a.rows + kTile - 1) / kTile, tn = (a.cols + kTile - 1) / kTile;
    per_sym = ts * (ts + 1) / 2, per_x = tm * tn;
    per_step = a.G * (2 * per_sym + per_x);
    total = per_step * a.steps;
  }
  __device__ __noinline__ Item at(const MmArgs& a, int t) const {
    Item it;
    it.step = t / per_step;
    int r = t - it.step * per_step;
    const int syms = a.G * per_sym;
    it.need = kCtas * (uint32_t)it.step * (uint32_t)(2 * per_sym + per_x);
    if (r < 2 * syms) {
      it.role = r < syms ? GRAM : POLY;
      if (it.role == POLY) r -= syms, it.need += kCtas * per_sym;
      it.g = r / per_sym;
      const int q = r - it.g * per_sym;
      // tiles on and below the diagonal, row by row
      int i = (int)((sqrtf(8.f * (float)q + 1.f) - 1.f) * 0.5f);
      while (i * (i + 1) / 2 > q) --i;
      while ((i + 1) * (i + 2) / 2 <= q) ++i;
      it.m0 = i * kTile, it.n0 = (q - i * (i + 1) / 2) * kTile;
      it.M = it.N = a.n;
      it.K = it.role == GRAM ? max(a.rows, a.cols) : a.n;
    } else {
      r -= 2 * syms;
      it.role = it.step + 1 < a.steps ? NEXT : LAST;
      it.need += 2u * kCtas * per_sym;
      it.g = r / per_x;
      const int q = r - it.g * per_x;
      it.m0 = q % tm * kTile, it.n0 = q / tm * kTile;
      it.M = a.rows, it.N = a.cols, it.K = a.n;
    }
    return it;
  }
};

template <bool PAIR>
__global__ void __launch_bounds__(kThreads, 1) __cluster_dims__(PAIR ? 2 : 1, 1, 1)
    direction_product_kernel(const __grid_constant__ MmArgs args) {
  constexpr int kTile = Plan<PAIR>::kTile;
  constexpr uint32_t kCols = 2 * kTile;  // of tensor memory
  extern __shared__ uint8_t smem_raw[];
  MmSmem& sm = *reinterpret_cast<MmSmem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const int warp = uniform_warp(), lane = threadIdx.x & 31;
  const uint32_t rank = PAIR ? cta_rank() : 0;
  const int pair = PAIR ? blockIdx.x >> 1 : blockIdx.x, pairs = PAIR ? gridDim.x >> 1 : gridDim.x;
  const Plan<PAIR> plan(args);

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&sm.full[s], 1);
      mbar_init(&sm.empty[s], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sm.acc_full[i], 1);
      mbar_init(&sm.acc_empty[i], (PAIR ? 2 : 1) * kEpiWarps);  // the epilogue warps of all its CTAs
    }
    for (int i = 0; i < kEpi; ++i) {
      mbar_init(&sm.epi_full[i], 1);
      mbar_init(&sm.epi_ready[i], kEpiWarps);
      mbar_init(&sm.epi_empty[i], 1);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 2) {
    if constexpr (PAIR) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sm.tmem_base)), "r"(kCols)
                   : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sm.tmem_base)), "r"(kCols)
                   : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if constexpr (PAIR) pair_sync();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = sm.tmem_base;

  if (warp == 0) {
    const bool el = elect_one();
    int s = 0, of = -1;
    int64_t it = 0;
    uint32_t ph = 1, seen = 0;
    bool ok = true;
    for (int t = pair; t < plan.total && ok; t += pairs) {
      const Item q = plan.at(args, t);
      if (seen != q.need || of != q.g) {  // (the last tile's wait covers this one where it is of the same phase)
        if (!(ok = wait_count_warp(args.done + q.g, q.need))) break;
        seen = q.need, of = q.g;
      }
      const int in = q.step & 1, m0 = q.m0 + rank * kHalf, n0 = q.n0 + rank * kHalf, nk = (q.K + kBK - 1) / kBK;
      const CUtensorMap* ma = q.role == GRAM ? (args.tall ? &args.xm[in] : &args.xk[in])
                              : q.role == POLY ? &args.ak : (args.tall ? &args.xk[in] : &args.pk);
      const CUtensorMap* mb = q.role <= POLY ? ma : (args.tall ? &args.pk : &args.xm[in]);
      const bool a_mn = q.role == GRAM && args.tall, b_mn = q.role <= POLY ? a_mn : !args.tall;
      for (int kb = 0; kb < nk; ++kb, ++it) {
        if (!wait_bar_warp(&sm.empty[s], ph)) {
          ok = false;
          break;
        }
        if (el) {
          const uint32_t bar = PAIR ? in_cta(&sm.full[s], 0) : 0;
          if (rank == 0) mbar_expect_tx(&sm.full[s], (PAIR ? 4 : 2) * kOpBytes);  // two operands of every CTA
          const int k0 = kb * kBK;
          auto load = [&](void* to, const CUtensorMap* map, int x, int y) {
            if constexpr (PAIR) tma_load_pair(to, map, bar, x, y, q.g);
            else tma_load_3d(to, map, &sm.full[s], x, y, q.g);
          };
          if (!a_mn) {
            load(sm.a[s], ma, k0, m0);
          } else {
            load(sm.a[s], ma, m0, k0);
            load(sm.a[s] + kOpBytes / 2, ma, m0 + 64, k0);
          }
          if (!b_mn) {
            load(sm.b[s], mb, k0, n0);
          } else {
            load(sm.b[s], mb, n0, k0);
            load(sm.b[s] + kOpBytes / 2, mb, n0 + 64, k0);
          }
        }
        if (++s == kStages) s = 0, ph ^= 1;
      }
    }
    // after a wait that ran out, the copies in flight (the leader's barriers count both CTAs') are waited for
    if (!ok && rank == 0)
      for (int64_t j = it > kStages ? it - kStages : 0; j < it; ++j) wait_bar(&sm.full[j % kStages], (j / kStages) & 1);
  } else if (warp == 1 && rank == 0) {
    const bool el = elect_one();
    int i = 0, s = 0;
    uint32_t ph = 0;
    bool ok = true;
    for (int t = pair; t < plan.total && ok; t += pairs, ++i) {
      const Item q = plan.at(args, t);
      const int nk = (q.K + kBK - 1) / kBK, ab = i & 1;
      const bool a_mn = q.role == GRAM && args.tall, b_mn = q.role <= POLY ? a_mn : !args.tall;
      // fp32 accumulators, fp16 operands, M = N = kTile
      const uint32_t idesc = (1u << 4) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) |
                             ((uint32_t)(kTile >> 3) << 17) | ((uint32_t)(kTile >> 4) << 24);
      const uint64_t a0 = smem_desc(smem_u32(sm.a[0]), a_mn ? kOpBytes / 2 : 16, 1024);
      const uint64_t b0 = smem_desc(smem_u32(sm.b[0]), b_mn ? kOpBytes / 2 : 16, 1024);
      const uint32_t a_step = a_mn ? 2048 >> 4 : 32 >> 4, b_step = b_mn ? 2048 >> 4 : 32 >> 4;
      if (!wait_bar_warp(&sm.acc_empty[ab], ((i >> 1) & 1) ^ 1)) break;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const uint32_t acc = tmem + (uint32_t)(ab * kTile);
      for (int kb = 0; kb < nk; ++kb) {
        if (!wait_bar_warp(&sm.full[s], ph)) {
          ok = false;
          break;
        }
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint64_t ad = a0 + (uint32_t)s * (kOpBytes >> 4), bd = b0 + (uint32_t)s * (kOpBytes >> 4);
#pragma unroll
        for (int kk = 0; kk < kBK / 16; ++kk)
          if (el) mma_of<PAIR>(acc, ad + kk * a_step, bd + kk * b_step, idesc, (kb > 0 || kk > 0) ? 1u : 0u);
        if (el) commit_of<PAIR>(&sm.empty[s]);
        if (++s == kStages) s = 0, ph ^= 1;
      }
      if (ok && el) commit_of<PAIR>(&sm.acc_full[ab]);
    }
  } else if (warp == 3) {
    const bool el = elect_one();
    int e = 0, of = -1;
    int64_t it = 0;
    uint32_t ph = 1, seen = 0;
    bool ok = true;
    for (int t = pair; t < plan.total && ok; t += pairs) {
      const Item q = plan.at(args, t);
      if (seen != q.need || of != q.g) {
        if (!(ok = wait_count_warp(args.done + q.g, q.need))) break;
        seen = q.need, of = q.g;
      }
      const int in = q.step & 1, m0 = q.m0 + rank * kHalf;
      for (int c = 0; c < kTile && q.n0 + c < q.N; c += kChunk, ++it) {
        if (!wait_bar_warp(&sm.epi_empty[e], ph)) {
          ok = false;
          break;
        }
        if (el) {
          if (q.role == GRAM) {
            mbar_arrive(&sm.epi_full[e]);
          } else if (q.role == POLY) {
            mbar_expect_tx(&sm.epi_full[e], kOpBytes);
            tma_load_3d(sm.e[e][0], &args.ak, &sm.epi_full[e], q.n0 + c, m0, q.g);
          } else {
            mbar_expect_tx(&sm.epi_full[e], 2 * kOpBytes);
            tma_load_3d(sm.e[e][0], &args.xk[in], &sm.epi_full[e], q.n0 + c, m0, q.g);
            tma_load_3d(sm.e[e][1], &args.lk[in], &sm.epi_full[e], q.n0 + c, m0, q.g);
          }
        }
        if (++e == kEpi) e = 0, ph ^= 1;
      }
    }
    if (!ok)
      for (int64_t j = it > kEpi ? it - kEpi : 0; j < it; ++j) wait_bar(&sm.epi_full[j % kEpi], (j / kEpi) & 1);
  } else if (warp == 2) {
    const bool el = elect_one();
    int e = 0;
    uint32_t ph = 0;
    bool ok = true;
    for (int t = pair; t < plan.total && ok; t += pairs) {
      const Item q = plan.at(args, t);
      const int m0 = q.m0 + rank * kHalf, in = q.step & 1;
      const bool mirror = q.role <= POLY && q.m0 != q.n0, by_tma = q.role != LAST || args.o_tma;
      for (int c = 0; c < kTile && q.n0 + c < q.N; c += kChunk) {
        if (!(ok = wait_bar_warp(&sm.epi_ready[e], ph))) break;
        const bool end = c + kChunk >= kTile || q.n0 + c + kChunk >= q.N;
        if (el) {
          const int x = q.n0 + c;
          if (m0 < q.M && by_tma) {
            const CUtensorMap* to = q.role == GRAM   ? &args.ak
                                    : q.role == POLY ? &args.pk
                                    : q.role == NEXT ? &args.xk[in ^ 1]
                                                     : &args.om;
            tma_store(to, sm.e[e][0], x, m0, q.g);
            if (q.role == NEXT) tma_store(&args.lk[in ^ 1], sm.e[e][1], x, m0, q.g);
            if (mirror) {
              to = q.role == GRAM ? &args.am : &args.pm;
              tma_store(to, sm.e[e][1], m0, x, q.g);
              if (m0 + 64 < q.M) tma_store(to, sm.e[e][1] + kOpBytes / 2, m0 + 64, x, q.g);
            }
          }
          asm volatile("cp.async.bulk.commit_group;" ::: "memory");
          // the buffer before this one has been read by its stores (kEpi > 2: the ring goes on meanwhile)
          if (c > 0) {
            asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
            mbar_arrive(&sm.epi_empty[e == 0 ? kEpi - 1 : e - 1]);
          }
          if (end) {
            asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
            mbar_arrive(&sm.epi_empty[e]);
            asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
            // the tile's writes, and the diagonal's by the epilogue warps, before the count
            asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(args.done + q.g) : "memory");
          }
        }
        __syncwarp();
        if (++e == kEpi) e = 0, ph ^= 1;
      }
    }
    if (el) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    __syncwarp();
  } else if (warp >= 4) {
    const int quarter = warp & 3, cc = ((warp - 4) >> 2) * 16;  // 32 rows; columns cc .. cc + 15 of each chunk
    const int r = quarter * 32 + lane;  // the row of this CTA's half tile
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    // within a buffer: this row's two 16-byte pieces (piece p of a row stands at p ^ (r & 7)), and the place of value r in
    // row cc of the transpose, whose 16-byte piece k of the row's number is still to be flipped by
    const uint32_t epi_base = smem_u32(sm.e[0][0]);
    const uint32_t piece0 = r * 128 + ((cc / 8) ^ (r & 7)) * 16, piece1 = r * 128 + ((cc / 8 + 1) ^ (r & 7)) * 16;
    const uint32_t flip = (uint32_t)((r >> 6) * (kOpBytes / 2) + cc * 128 + ((r & 63) >> 3) * 16 + (r & 7) * 2);
    int i = 0, e = 0;
    uint32_t ph = 0;
    bool ok = true;
    for (int t = pair; t < plan.total && ok; t += pairs, ++i) {
      const Item q = plan.at(args, t);
      const int role = q.role, ab = i & 1, m0 = q.m0 + rank * kHalf, row = m0 + r;
      const bool sym = role <= POLY, on_diag = sym && q.m0 == q.n0;
      // The first chunk's loads were issued behind the wait for this matrix's earlier phases, so that what those wrote
      // is visible once they are here: the diagonal's value of this row and, by lane, of the chunk's columns.
      if (!(ok = wait_bar_warp(&sm.epi_full[e], ph))) break;
      float* da = args.diag_a + (int64_t)q.g * args.n;
      float* dg = args.diag + (int64_t)q.g * args.n;
      const bool by_row = role == POLY || (!sym && !args.tall), by_col = role == POLY || (!sym && args.tall);
      const float* dsrc = role == POLY ? da : dg;
      const float dr = by_row && row < q.M ? __ldcg(dsrc + row) : 0.f;
      const float drow = role == POLY ? fmaf(kC, dr, kB) : kA + dr;
      int col = q.n0 + cc + (lane & 15);
      float dnext = by_col && col < q.N ? __ldcg(dsrc + col) : 0.f;
      const int late = q.step + 2 - args.steps;  // 0 and 1 in the last two steps
      uint32_t* top = args.top + (late > 0 ? args.G : 0) + q.g;
      const float tl = !sym && late >= 0 ? kA + from_ordered(__ldcg(top)) : kA;
      if (!(ok = wait_bar_warp(&sm.acc_full[ab], (i >> 1) & 1))) break;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll 1
      for (int c = 0; c < kTile && q.n0 + c < q.N; c += kChunk) {
        const float dcol = role == POLY ? kC * dnext : dnext;
        col += kChunk;
        dnext = by_col && c + kChunk < kTile && col < q.N ? __ldcg(dsrc + col) : 0.f;
        if (c > 0 && !(ok = wait_bar_warp(&sm.epi_full[e], ph))) break;
        const uint32_t mine = epi_base + (uint32_t)e * (2 * kOpBytes), other = mine + kOpBytes;
        float v[16];
        tmem_ld16(tmem + (uint32_t)(ab * kTile + c + cc) + lanes, v);
        const int dd = row - (q.n0 + c + cc);  // the diagonal's place among the columns
        auto eight = [&](auto J, uint32_t piece) {  // columns 8 J .. 8 J + 7 of the 16
          constexpr int j = decltype(J)::value;
          float f[8];
          if (sym) {
            if (role == GRAM) {
#pragma unroll
              for (int k = 0; k < 8; ++k) f[k] = v[8 * j + k] * kUnscale;
            } else {  // with D = diag dA and O the rest of A: A A = O O + D O + O D + D D
              unpack8(lds16(mine + piece), f);
#pragma unroll
              for (int k = 0; k < 8; ++k)
                f[k] = fmaf(drow + __shfl_sync(~0u, dcol, 8 * j + k), f[k], kC * kUnscale * v[8 * j + k]);
            }
            if (on_diag && __any_sync(~0u, (dd >> 3) == j)) {
              float acc = 0.f;
#pragma unroll
              for (int k = 0; k < 8; ++k) {  // (sums and selects: an index into the registers would put them in memory)
                acc += dd == 8 * j + k ? v[8 * j + k] : 0.f;
                f[k] = dd == 8 * j + k ? 0.f : f[k];
              }
              if ((dd >> 3) == j && row < q.M) {
                const float d = role == GRAM ? acc * kUnscale2 : fmaf(kB, dr, kC * fmaf(dr, dr, acc * kUnscale2));
                (role == GRAM ? da : dg)[row] = d;
                if (role == POLY && late >= 0) atomicMax(top, to_ordered(d));
              }
            }
          } else {
            float lo[8];
            unpack8(lds16(mine + piece), f);
            unpack8(lds16(other + piece), lo);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const float d = by_col ? kA + __shfl_sync(~0u, dcol, 8 * j + k) : drow;
              f[k] = fmaf(d, f[k], fmaf(tl, lo[k], kUnscale * v[8 * j + k]));
            }
          }
          if (role == LAST) {
#pragma unroll
            for (int k = 0; k < 8; ++k) f[k] *= kUnscale;
            sts16(mine + piece, pack8_bf16(f));
          } else {
            const uint4 w = pack8(f);
            sts16(mine + piece, w);
            if (role == NEXT) {
              float hi[8];
              unpack8(w, hi);
#pragma unroll
              for (int k = 0; k < 8; ++k) hi[k] = f[k] - hi[k];
              sts16(other + piece, pack8(hi));
            } else if (!on_diag) {
              // the transpose: rows cc + .. of a box of 64 values of r; the low bits of a row's number are k
              const uint32_t words[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
              for (int k = 0; k < 8; ++k)
                sts2(other + ((flip ^ (k << 4)) + (8 * j + k) * 128), k & 1 ? words[k / 2] >> 16 : words[k / 2]);
            }
          }
        };
        eight(std::integral_constant<int, 0>{}, piece0);
        eight(std::integral_constant<int, 1>{}, piece1);
        if (role == LAST && !args.o_tma) {
          // o's rows are not on 16-byte boundaries: this warp's 32 rows of 16 columns, two rows at a time
          __syncwarp();
          const int oc = cc + (lane & 15), x = q.n0 + c + oc;
          uint16_t* o = args.o + (int64_t)q.g * args.o_gs + x;
          if (x < q.N)
#pragma unroll 4
            for (int k = lane >> 4; k < 32; k += 2) {
              const int rr = quarter * 32 + k;
              if (m0 + rr < q.M)
                o[(int64_t)(m0 + rr) * args.cols] =
                    *reinterpret_cast<const uint16_t*>(sm.e[e][0] + rr * 128 + (((oc >> 3) ^ (rr & 7)) * 16) + (oc & 7) * 2);
            }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.epi_ready[e]);
        if (++e == kEpi) e = 0, ph ^= 1;
      }
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) {
        if constexpr (PAIR) arrive_at(in_cta(&sm.acc_empty[ab], 0));
        else mbar_arrive(&sm.acc_empty[ab]);
      }
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if constexpr (PAIR) pair_sync();  // no CTA leaves while the other may still signal its barriers or read its operands
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  if (warp == 2) {
    if constexpr (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kCols) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kCols) : "memory");
  }
}

// ------------------------------------------------------------------------------------------------
// Resident form: a matrix of a smaller side n <= 128 in the shared memory of one CTA or several, all of it in one launch
//
// X is held with its longer side down, [m][n], a CTA having up to 512 of the m rows and a thread one row.  The CTAs of a
// matrix are a cluster; or (GLOBAL) any CTAs of a cooperative launch, in groups that take one matrix after another and exchange
// through global memory, where a cluster would be too small or leave SMs idle.
// A row is 128 fp16 values, two swizzled pieces of 64: up to n = 64 h and l, above it h alone (l in tensor memory, 64 columns
// beside the two accumulators).  A step:
//   1. tcgen05: [h l]^T [h l] over the CTA's rows into tensor memory, 128 x 128; above 64 that is A, up to 64 A is the sum
//      of its parts h h, h l and l h;
//   2. the CTAs' sums are added up in rank order (each CTA a slice of A, through distributed shared memory) and the
//      slices given to all;  (GLOBAL: the same through L2, two counted barriers)
//   3. tcgen05: A A, then P in A's place;
//   4. tcgen05: X P, 128 rows to a tile (above n = 64 two tiles at a time); each thread updates its row from its tile.
// Up to n = 64 both h and l are multiplied, so that small matrices, whose roundings do not average out, are off by less
// than 2.5e-3 too.  What bounds it is each step's chain of latencies (products, their sums' exchange, products, products, the
// rows' update), which the work in it hardly lengthens: 16 matrices of 16 x 144 take 15 us (launch included; their bytes
// 0.1), 16 of 100 x 4096 take 119 (bytes 13.5).  The 128 columns that a tile of products has are its limit; there it is still the
// faster: 16 x 128 x 1024 in 83 us (110 by the tiles of the form above), 16 x 128 x 128 in 70 (90), 16 x 100 x 4096 in 119 (198).

constexpr int kRows = 512;       // rows of a CTA
constexpr int kResSide = 128;
constexpr int kPiece = 128;      // bytes of a piece's row

struct ResArgs {
  DirArgs d;
  int n, m, cl, per, steps;  // per: rows of a CTA
  // GLOBAL: groups of cl CTAs, and per group the CTAs' sums [cl][n16][n16], A [n16][n16] without its diagonal, the diagonal
  // [n16], the CTAs' norm sums [cl][3] and the count of barrier arrivals
  int groups;
  float* part;
  uint2* full;
  float *diag, *norms;
  uint32_t* count;
};

// Shared memory, from a 1024-byte boundary: X's two pieces [2][rows][64], A and P [NP / 64][128][64], the sums [128][128] in
// fp32, then ResTail.
struct __align__(16) ResTail {
  float da[kResSide], d[kResSide];
  float norm[3];
  float red[3][kRows / 32];
  uint64_t bar[5];  // the symmetric products, and each tile of X P
  uint32_t tmem;
};
template <int NP>
constexpr size_t res_smem(int rows) {
  return 1024 + (size_t)rows * 2 * kPiece + (NP / 64) * 128 * kPiece + 128 * 128 * 4 + sizeof(ResTail);
}

__device__ __forceinline__ uint4 lds16_at(uint32_t cluster_addr) {
  uint4 v;
  asm volatile("ld.shared::cluster.v4.b32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "r"(cluster_addr)
               : "memory");
  return v;
}
__device__ __forceinline__ uint32_t at_rank(uint32_t addr, int rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}

__device__ __forceinline__ void vec8(uint32_t at, float (&f)[8]) {
  const uint4 a = lds16(at), b = lds16(at + 16);
  f[0] = __uint_as_float(a.x), f[1] = __uint_as_float(a.y), f[2] = __uint_as_float(a.z), f[3] = __uint_as_float(a.w);
  f[4] = __uint_as_float(b.x), f[5] = __uint_as_float(b.y), f[6] = __uint_as_float(b.z), f[7] = __uint_as_float(b.w);
}

// Eight accumulator columns of this warp's 32 rows, and the same stored.
__device__ __forceinline__ void tmem_ld16_8(uint32_t at16, float (&v)[16], uint32_t at8, uint32_t (&w)[8]) {
  uint32_t r[16];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%24];\n"
      "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%16,%17,%18,%19,%20,%21,%22,%23}, [%25];\n"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(w[0]), "=r"(w[1]),
        "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
      : "r"(at16), "r"(at8)
      : "memory");
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_st8(uint32_t at, const uint32_t (&w)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]),
               "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}

template <int NP, bool GLOBAL>
__global__ void __launch_bounds__(kRows, 1) direction_resident_kernel(const ResArgs a) {
  constexpr bool kBoth = NP == 64;  // l is in shared memory and multiplied too
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023) & ~1023u;
  const int rows = blockDim.x, warps = rows >> 5;
  const uint32_t xs = base, xpiece = (uint32_t)rows * kPiece;                  // X: piece p at xs + p xpiece
  const uint32_t as = xs + 2 * xpiece;                                         // A, P: piece p at as + p 128 kPiece
  const uint32_t sums = as + (NP / 64) * 128 * kPiece;
  const uint32_t tail_at = sums + 128 * 128 * 4;
  ResTail& tail = *reinterpret_cast<ResTail*>(smem_raw + (tail_at - smem_u32(smem_raw)));
  const int warp = uniform_warp(), lane = threadIdx.x & 31, tid = threadIdx.x;
  const int rank = GLOBAL ? blockIdx.x % a.cl : a.cl > 1 ? (int)cta_rank() : 0, group = blockIdx.x / a.cl;
  const int n = a.n, m0 = rank * a.per, have = max(0, min(a.per, a.m - m0));  // this CTA's rows
  const bool tall = a.d.rows > a.d.cols;
  const int tiles = rows / 128;
  // tensor memory: the symmetric products' 128 columns and the tiles' NP each, in the same place; above n = 64 two tiles'
  // accumulators at a time and 64 columns of l for every tile behind them
  const uint32_t low = kBoth || tiles > 1 ? 256 : 128;  // l's first column
  const uint32_t cols = kBoth ? (tiles > 2 ? 256 : 128) : 2 * low;

  if (tid == 0) {
    for (int i = 0; i < 5; ++i) mbar_init(&tail.bar[i], 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tail.tmem)), "r"(cols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  pdl_begin();

  // a barrier of the CTAs of this matrix; what they wrote before is visible behind it
  uint32_t epoch = 0;
  bool dead = false;
  auto sync = [&]() {
    if constexpr (GLOBAL) {
      __syncthreads();
      if (tid == 0) asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(a.count + group) : "memory");
      epoch += a.cl;
      // (after a wait that ran out the flag is set and the results do not count: no more waits)
      dead = __syncthreads_or(dead || (warp == 0 && !wait_count_warp(a.count + group, epoch)));
    } else if (a.cl > 1) {
      pair_sync();
    } else {
      __syncthreads();
    }
  };
  uint32_t ph = 0, ph2 = 0;
  for (int64_t k = group; k < a.d.G; k += GLOBAL ? a.groups : a.d.G) {
    // rows and columns past the matrix are zero
    for (uint32_t i = tid * 16; i < 2 * xpiece; i += rows * 16) sts16(xs + i, make_uint4(0, 0, 0, 0));
    __syncthreads();
    // momentum and the norm: this CTA's values, neighbouring ones by neighbouring threads
    const DirArgs& d = a.d;
    const int64_t gk = k * d.g_gs, uk = k * d.u_gs;
    // the place of value (j, i), row j of this CTA's and column i of X
    auto place = [&](int j, int i) -> int { return tall ? (m0 + j) * n + i : i * a.m + m0 + j; };
    const uint32_t row_at = xs + tid * kPiece, turn = (tid & 7) << 4;  // 16-byte piece p of a row stands at p ^ (row & 7)
    {
      NormSums s{0.f, 0.f, 0.f};
      // value (j, i) of up to n = 64 waits for the norm in row j, 64 fp32 values to a row's two pieces
      auto keep = [&](int j, int i, float x) {
        if constexpr (kBoth) {
          const uint32_t at = xs + (i >> 5) * xpiece + j * kPiece + ((((i & 31) >> 2) ^ (j & 7)) << 4) + (i & 3) * 4;
          asm volatile("st.shared.f32 [%0], %1;" ::"r"(at), "f"(x) : "memory");
        }
      };
      // 16 values at a time, their loads before the first store
      constexpr int kAt = 16;
      auto some = [&](auto bf16, int64_t at, int64_t stride, int from, int step, int end, auto where) {
        constexpr bool kBf16 = decltype(bf16)::value;
        for (int b = from; b < end; b += kAt * step, at += kAt * stride) {
          float g[kAt], u[kAt];
          const float* up = d.u + uk + at;
#pragma unroll
          for (int q = 0; q < kAt; ++q) {
            const bool in = b + q * step < end;
            g[q] = in ? grad_value<kBf16>(d.g, gk + at + q * stride) : 0.f;
            u[q] = in && d.mom != 0.f ? up[q * stride] : 0.f;
          }
#pragma unroll
          for (int q = 0; q < kAt; ++q)
            if (b + q * step < end) {
              float x = g[q];
              if (d.mom != 0.f) {
                const float t = fmaf(d.mom, u[q], x);
                d.u[uk + at + q * stride] = t;
                x = d.nesterov ? fmaf(d.mom, t, x) : t;
              }
              norm_add(s, x);
              where(b + q * step, x);
            }
        }
      };
      auto all = [&](auto bf16) {
        if (tall) some(bf16, (int64_t)m0 * n + tid, rows, tid, rows, have * n, [&](int e, float x) { keep(e / n, e % n, x); });
        else if (tid < have) some(bf16, m0 + tid, a.m, 0, 1, n, [&](int i, float x) { keep(tid, i, x); });
      };
      if (d.g_bf16) all(std::true_type{});
      else all(std::false_type{});
      float v[3] = {s.mid, s.big, s.small};
#pragma unroll
      for (int j = 0; j < 3; ++j) {
#pragma unroll
        for (int o = 16; o; o >>= 1) v[j] += __shfl_xor_sync(~0u, v[j], o);
        if (lane == 0) tail.red[j][warp] = v[j];
      }
      __syncthreads();
      if (tid < 3) {
        float t = 0.f;
        for (int w = 0; w < warps; ++w) t += tail.red[tid][w];
        if constexpr (GLOBAL) __stcg(a.norms + (group * a.cl + rank) * 3 + tid, t);
        else tail.norm[tid] = t;
      }
      sync();
    }
    const uint32_t tmem = tail.tmem;
    const uint32_t stage = sums + warp * 4096;  // 32 x 32 fp32 values of a warp, where the sums are not in use
    {
      float t[3] = {0.f, 0.f, 0.f};
      for (int c = 0; c < a.cl; ++c)
#pragma unroll
        for (int j = 0; j < 3; ++j) {
          float v;
          if constexpr (GLOBAL) v = __ldcg(a.norms + (group * a.cl + c) * 3 + j);
          else asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at_rank(smem_u32(&tail.norm[j]), c)) : "memory");
          t[j] += v;
        }
      const float2 f = norm_factors(t[0], t[1], t[2]);
      if constexpr (kBoth) {
        uint4 raw[16];
#pragma unroll
        for (int q = 0; q < 16; ++q) raw[q] = lds16(row_at + (q >> 3) * xpiece + (((q & 7) << 4) ^ turn));
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const uint4 r0 = raw[2 * q], r1 = raw[2 * q + 1];
          const uint32_t w[8] = {r0.x, r0.y, r0.z, r0.w, r1.x, r1.y, r1.z, r1.w};
          float x[8], hi[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(w[i]) * f.x * f.y;
          const uint4 h = pack8(x);
          unpack8(h, hi);
#pragma unroll
          for (int i = 0; i < 8; ++i) hi[i] = x[i] - hi[i];
          sts16(row_at + ((q << 4) ^ turn), h);
          sts16(row_at + xpiece + ((q << 4) ^ turn), pack8(hi));
        }
      } else {  // once more from L2, a row's values 16 at a time (rolled: code that runs once is fetched at its size)
        const uint32_t ltile = tmem + low + (warp >> 2) * 64 + ((uint32_t)(warp & 3) << 21);
        // 16 values' loads before they are used: value q at at + q stride where in(q)
        auto batch = [&](auto bf16, int64_t at, int64_t stride, auto in, auto use) {
          constexpr bool kBf16 = decltype(bf16)::value;
          const bool want_g = d.mom == 0.f || d.nesterov, want_u = d.mom != 0.f;
          const float* up = d.u + uk + at;
          float g[16], u[16];
#pragma unroll
          for (int q = 0; q < 16; ++q) {
            g[q] = want_g && in(q) ? grad_value<kBf16>(d.g, gk + at + q * stride) : 0.f;
            u[q] = want_u && in(q) ? up[q * stride] : 0.f;
          }
          const float mg = want_g ? 1.f : 0.f, mu = !want_u ? 0.f : d.nesterov ? d.mom : 1.f;
#pragma unroll
          for (int q = 0; q < 16; ++q) use(q, fmaf(mu, u[q], mg * g[q]) * f.x * f.y);
        };
#pragma unroll 1
        for (int b = 0; b < n; b += 16) {
          float x[16];
          auto all = [&](auto bf16) {
            if (!tall) {
              batch(bf16, (int64_t)b * a.m + m0 + tid, a.m, [&](int q) { return tid < have && b + q < n; },
                    [&](int q, float v) { x[q] = v; });
            } else {  // neighbouring lanes read neighbouring values; the warp's 32 x 16 values change places
              const int row = lane >> 4, col = lane & 15;
              batch(bf16, (int64_t)(m0 + warp * 32 + row) * n + b + col, 2 * n,
                    [&](int q) { return warp * 32 + 2 * q + row < have && b + col < n; },
                    [&](int q, float v) {
                      asm volatile("st.shared.f32 [%0], %1;" ::"r"(stage + (2 * q + row) * 64 + ((col ^ (q & 15)) << 2)), "f"(v)
                                   : "memory");
                    });
              __syncwarp();
#pragma unroll
              for (int q = 0; q < 16; ++q)
                asm volatile("ld.shared.f32 %0, [%1];"
                             : "=f"(x[q])
                             : "r"(stage + lane * 64 + ((q ^ (lane >> 1 & 15)) << 2))
                             : "memory");
              __syncwarp();
            }
          };
          if (d.g_bf16) all(std::true_type{});
          else all(std::false_type{});
          uint32_t low8[8];
#pragma unroll
          for (int p = 0; p < 2; ++p) {
            const int q = b / 8 + p;
            float v[8], hi[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = x[8 * p + i];
            const uint4 w = pack8(v);
            unpack8(w, hi);
#pragma unroll
            for (int i = 0; i < 8; ++i) hi[i] = v[i] - hi[i];
            const uint4 lo = pack8(hi);
            sts16(row_at + (q >> 3) * xpiece + (((q & 7) << 4) ^ turn), w);
            low8[4 * p] = lo.x, low8[4 * p + 1] = lo.y, low8[4 * p + 2] = lo.z, low8[4 * p + 3] = lo.w;
          }
          tmem_st8(ltile + b / 2, low8);
        }
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
      }
    }

    const uint32_t quarter = (uint32_t)(warp & 3) * 32, lanes = quarter << 16;
    const int r128 = (int)quarter + lane, groups = warps / 4;  // this thread's row of the symmetric products
    const int ks = (have + 15) / 16, kn = (n + 15) / 16, n16 = kn * 16;  // rows and columns from n16 on are not computed
    for (int step = 0; step < a.steps; ++step) {
      // 1. [h l]^T [h l]
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncthreads();
      if (warp == 0) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const bool el = elect_one();
        // M = N = 128, both operands with the sum running down the rows
        constexpr uint32_t idesc = (1u << 4) | (1u << 15) | (1u << 16) | ((128u >> 3) << 17) | ((128u >> 4) << 24);
        const uint64_t x0 = smem_desc(xs, xpiece, 1024);
        for (int i = 0; i < max(ks, 1); ++i)
          if (el) mma_one(tmem, x0 + i * (2048 >> 4), x0 + i * (2048 >> 4), idesc, i > 0);
        if (el) commit_one(&tail.bar[0]);
      }
      wait_bar_warp(&tail.bar[0], ph);
      ph ^= 1;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      // row r128 of the sums; 16-byte piece p of a row stands at p ^ (row & 31)
      for (int c = (warp >> 2) * 16; c < 128 && ((int)quarter & (NP - 1)) < n16; c += groups * 16) {
        if ((c & (NP - 1)) >= n16) continue;
        float v[16];
        tmem_ld16(tmem + c + lanes, v);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          sts16(sums + r128 * 512 + (((c / 4 + j) ^ lane) << 4),
                make_uint4(__float_as_uint(v[4 * j]), __float_as_uint(v[4 * j + 1]), __float_as_uint(v[4 * j + 2]),
                           __float_as_uint(v[4 * j + 3])));
      }
      if constexpr (GLOBAL) __syncthreads();
      else sync();
      // 2. this CTA's slice of A: rows rank, rank + cl, ...; four columns to a thread
      {
        auto slice = [&](auto ctas) {
          constexpr int kCtas = decltype(ctas)::value;
          constexpr bool kOne = kCtas == 1;
          const int per_row = n16 / 4, mine = (n16 - rank + kCtas - 1) / kCtas;
          for (int e = tid; e < mine * per_row; e += rows) {
            const int i = rank + e / per_row * kCtas, j = e % per_row;
            float f[4] = {0.f, 0.f, 0.f, 0.f};
            constexpr int kParts = kBoth ? 3 : 1;
            uint4 w[kCtas][kParts];  // every CTA's parts, loaded before the first is used
#pragma unroll
            for (int c = 0; c < kCtas; ++c) {
              const uint32_t from = kOne ? sums : at_rank(sums, c);
              auto part = [&](int row, int piece) {
                const uint32_t at = from + row * 512 + ((piece ^ (row & 31)) << 4);
                return kOne ? lds16(at) : lds16_at(at);
              };
              w[c][0] = part(i, j);
              if constexpr (kBoth) w[c][1] = part(i, 16 + j), w[c][2] = part(64 + i, j);
            }
#pragma unroll
            for (int c = 0; c < kCtas; ++c) {
#pragma unroll
              for (int q = 0; q < kParts; ++q) {
                f[0] += __uint_as_float(w[c][q].x), f[1] += __uint_as_float(w[c][q].y);
                f[2] += __uint_as_float(w[c][q].z), f[3] += __uint_as_float(w[c][q].w);
              }
            }
            float diag = 0.f;
            const bool on = j == i >> 2;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              diag += 4 * j + q == i ? f[q] * kUnscale2 : 0.f;
              f[q] = 4 * j + q == i ? 0.f : f[q] * kUnscale;
            }
            const __half2 w0 = __floats2half2_rn(f[0], f[1]), w1 = __floats2half2_rn(f[2], f[3]);
            const uint32_t b0 = *reinterpret_cast<const uint32_t*>(&w0), b1 = *reinterpret_cast<const uint32_t*>(&w1);
            const uint32_t to = as + (j >> 4) * (128 * kPiece) + i * kPiece +
                                ((((j & 15) >> 1) << 4) ^ ((i & 7) << 4)) + (j & 1) * 8;
            const uint32_t da = smem_u32(&tail.da[i]);
            if constexpr (kOne) {
              asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(to), "r"(b0), "r"(b1) : "memory");
              if (on) tail.da[i] = diag;
            } else {
#pragma unroll
              for (int c = 0; c < kCtas; ++c) {
                asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(at_rank(to, c)), "r"(b0), "r"(b1) : "memory");
                if (on) asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at_rank(da, c)), "f"(diag) : "memory");
              }
            }
          }
        };
        if constexpr (GLOBAL) {
          const int per_row = n16 / 4, all = n16 * per_row;
          float4* part = reinterpret_cast<float4*>(a.part) + (int64_t)group * a.cl * all;
          uint2* full = a.full + (int64_t)group * all;
          float* diag = a.diag + group * n16;
          auto word = [](float x, float y) {
            const __half2 w = __floats2half2_rn(x, y);
            return *reinterpret_cast<const uint32_t*>(&w);
          };
          for (int e = tid; e < all; e += rows) {
            const int i = e / per_row, j = e % per_row;
            float f[4] = {0.f, 0.f, 0.f, 0.f};
            auto add = [&](int row, int piece) {
              const uint4 w = lds16(sums + row * 512 + ((piece ^ (row & 31)) << 4));
              f[0] += __uint_as_float(w.x), f[1] += __uint_as_float(w.y);
              f[2] += __uint_as_float(w.z), f[3] += __uint_as_float(w.w);
            };
            add(i, j);
            if constexpr (kBoth) add(i, 16 + j), add(64 + i, j);
            __stcg(part + (int64_t)rank * all + e, make_float4(f[0], f[1], f[2], f[3]));
          }
          sync();
          const int mine = (n16 - rank + a.cl - 1) / a.cl;
          for (int e = tid; e < mine * per_row; e += rows) {
            const int i = rank + e / per_row * a.cl, j = e % per_row;
            float f[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
            for (int c = 0; c < a.cl; ++c) {
              const float4 w = __ldcg(part + (int64_t)c * all + i * per_row + j);
              f[0] += w.x, f[1] += w.y, f[2] += w.z, f[3] += w.w;
            }
            float on_diag = 0.f;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              on_diag += 4 * j + q == i ? f[q] * kUnscale2 : 0.f;
              f[q] = 4 * j + q == i ? 0.f : f[q] * kUnscale;
            }
            __stcg(full + i * per_row + j, make_uint2(word(f[0], f[1]), word(f[2], f[3])));
            if (j == i >> 2) __stcg(diag + i, on_diag);
          }
          sync();
          for (int e = tid; e < all; e += rows) {
            const int i = e / per_row, j = e % per_row;
            const uint2 w = __ldcg(full + e);
            const uint32_t to = as + (j >> 4) * (128 * kPiece) + i * kPiece +
                                ((((j & 15) >> 1) << 4) ^ ((i & 7) << 4)) + (j & 1) * 8;
            asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(to), "r"(w.x), "r"(w.y) : "memory");
          }
          for (int i = tid; i < n16; i += rows) tail.da[i] = __ldcg(diag + i);
        } else if (a.cl == 1) slice(std::integral_constant<int, 1>{});
        else if (a.cl == 2) slice(std::integral_constant<int, 2>{});
        else if (a.cl == 4) slice(std::integral_constant<int, 4>{});
        else slice(std::integral_constant<int, 8>{});
      }
      if (!GLOBAL && a.cl > 1) pair_sync();
      // 3. A A, and P in A's place
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncthreads();
      if (warp == 0) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const bool el = elect_one();
        constexpr uint32_t idesc = (1u << 4) | ((uint32_t)(NP >> 3) << 17) | ((128u >> 4) << 24);
        const uint64_t a0 = smem_desc(as, 16, 1024);
        for (int i = 0; i < kn; ++i) {
          const uint64_t at = a0 + (i >> 2) * (128 * kPiece >> 4) + (i & 3) * 2;
          if (el) mma_one(tmem, at, at, idesc, i > 0);
        }
        if (el) commit_one(&tail.bar[0]);
      }
      wait_bar_warp(&tail.bar[0], ph);
      ph ^= 1;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      if ((int)quarter < n16) {
        const float di = r128 < n16 ? tail.da[r128] : 0.f;
        for (int c = (warp >> 2) * 16; c < n16; c += groups * 16) {
          float v[16], mine = 0.f;
          tmem_ld16(tmem + c + lanes, v);
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const uint32_t at = as + (c >> 6) * (128 * kPiece) + r128 * kPiece + ((((c & 63) / 8 + j) << 4) ^ ((r128 & 7) << 4));
            float f[8], dj[8];
            unpack8(lds16(at), f);
            vec8(smem_u32(tail.da) + (c + 8 * j) * 4, dj);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              f[i] = fmaf(fmaf(kC, di + dj[i], kB), f[i], kC * kUnscale * v[8 * j + i]);
              mine += c + 8 * j + i == r128 ? v[8 * j + i] : 0.f;
              f[i] = c + 8 * j + i == r128 ? 0.f : f[i];
            }
            sts16(at, pack8(f));
          }
          if (c == (r128 & ~15)) tail.d[r128] = fmaf(kB, di, kC * fmaf(di, di, mine * kUnscale2));
        }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncthreads();
      // 4. X P
      float top = 0.f;  // t of the number formats above
      if (!kBoth && step + 2 >= a.steps) {
        top = -INFINITY;
        for (int i = lane; i < n; i += 32) top = fmaxf(top, tail.d[i]);
#pragma unroll
        for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
      }
      const bool last = step + 1 == a.steps;
      const int tile = warp >> 2, at_once = kBoth ? tiles : 2;
#pragma unroll 1
      for (int t0 = 0; t0 < tiles; t0 += at_once) {
        if (t0 > 0) {  // the accumulators have been read
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          __syncthreads();
        }
        if (warp == 0) {
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const bool el = elect_one();
          constexpr uint32_t idesc = (1u << 4) | ((uint32_t)(NP >> 3) << 17) | ((128u >> 4) << 24);
          const uint64_t x0 = smem_desc(xs, 16, 1024), p0 = smem_desc(as, 16, 1024);
          for (int t = t0; t < min(tiles, t0 + at_once); ++t) {
            const uint64_t xt = x0 + (uint32_t)(t * 128 * kPiece >> 4);
#pragma unroll
            for (int i = 0; i < 8; ++i) {  // up to n = 64 the h, then the l of four slices of 16 columns; else eight of h
              const int slice = kBoth ? i & 3 : i;
              const uint64_t xa = xt + (i >> 2) * (xpiece >> 4) + (i & 3) * 2;
              const uint64_t pb = p0 + (kBoth ? 0 : (i >> 2) * (128 * kPiece >> 4)) + (i & 3) * 2;
              if (el && slice < kn) mma_one(tmem + (t - t0) * NP, xa, pb, idesc, i > 0);
            }
            if (el) commit_one(&tail.bar[1 + t]);
          }
          __syncwarp();
        }
        if (tile < t0 || tile >= t0 + at_once) continue;
        wait_bar_warp(&tail.bar[1 + tile], ph2);
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint32_t dtile = tmem + (tile - t0) * NP + lanes, ltile = tmem + low + tile * 64 + lanes;
#pragma unroll 1
        for (int c = 0; c < n; c += 16) {  // (rolled: the instruction cache holds a step then)
          float v[16];
          uint32_t low8[8];
          if constexpr (kBoth) tmem_ld16(dtile + c, v);
          else tmem_ld16_8(dtile + c, v, ltile + c / 2, low8);
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int q = c / 8 + j;
            const uint32_t at = row_at + (kBoth ? 0 : (q >> 3) * xpiece) + (((q & 7) << 4) ^ turn);
            float f[8], lo[8], dj[8];
            unpack8(lds16(at), f);
            vec8(smem_u32(tail.d) + 32 * q, dj);
            if constexpr (kBoth) unpack8(lds16(at + xpiece), lo);
            else unpack8(make_uint4(low8[4 * j], low8[4 * j + 1], low8[4 * j + 2], low8[4 * j + 3]), lo);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float t = kA + dj[i];
              f[i] = kBoth ? fmaf(t, f[i] + lo[i], kUnscale * v[8 * j + i])
                           : fmaf(t, f[i], fmaf(kA + top, lo[i], kUnscale * v[8 * j + i]));
            }
            if (!last) {
              const uint4 w = pack8(f);
              sts16(at, w);
              float hi[8];
              unpack8(w, hi);
#pragma unroll
              for (int i = 0; i < 8; ++i) hi[i] = f[i] - hi[i];
              const uint4 l = pack8(hi);
              if constexpr (kBoth) sts16(at + xpiece, l);
              else low8[4 * j] = l.x, low8[4 * j + 1] = l.y, low8[4 * j + 2] = l.z, low8[4 * j + 3] = l.w;
            } else if (!tall) {
              uint16_t* o = d.o + k * d.o_gs;
              if (tid < have)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                  if (8 * q + i < n) o[place(tid, 8 * q + i)] = f2bf(f[i] * kUnscale);
            } else {  // 16 columns of the warp's rows, to be written row by row
#pragma unroll
              for (int i = 0; i < 8; ++i) f[i] *= kUnscale;
              sts16(stage + lane * 32 + ((j ^ (lane >> 2 & 1)) << 4), pack8_bf16(f));
            }
          }
          if (!kBoth && !last) tmem_st8(ltile + c / 2, low8);
          if (last && tall) {
            __syncwarp();
            uint16_t* o = d.o + k * d.o_gs + (int64_t)(m0 + warp * 32) * n + c + (lane & 15);
            const int i = lane & 15;
            if (c + i < n)
#pragma unroll 4
              for (int rr = lane >> 4; rr < 32; rr += 2)
                if (warp * 32 + rr < have) {
                  uint16_t v;
                  const uint32_t from = stage + rr * 32 + (((i >> 3) ^ (rr >> 2 & 1)) << 4) + (i & 7) * 2;
                  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(from) : "memory");
                  o[rr * n] = v;
                }
            __syncwarp();
          }
        }
        if constexpr (!kBoth) asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
      }
      ph2 ^= 1;
    }
    __syncthreads();  // the next matrix is written where this one was read
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (!GLOBAL && a.cl > 1) pair_sync();  // no CTA leaves while another may read its sums
  if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tail.tmem), "r"(cols) : "memory");
}

// ------------------------------------------------------------------------------------------------
// w = (1 - lr wd) w - lr scale o, and its bf16 copy: one pass bound by memory, 12 bytes a value.  16 x 4096 x 4096 in 526 us,
// 6.1 TB/s.  Eight values to a thread's access where addresses and strides allow, else one (746 us).  Workers' values that
// follow one another are one long vector, whatever n is.

constexpr int kUpdThreads = 256;

template <int V>  // values per access: 8 (16 bytes of o, 32 of w) or 1
__global__ void __launch_bounds__(kUpdThreads) direction_update_kernel(float* w, const uint16_t* o, uint16_t* wb,
                                                                       int64_t n, int64_t w_gs, int64_t o_gs,
                                                                       float keep, float step) {
  pdl_begin();
  const int64_t k = blockIdx.y;
  w += k * w_gs, o += k * o_gs;
  if (wb) wb += k * w_gs;
  auto one = [&](int64_t i) {
    const float v = fmaf(-step, bf2f(o[i]), keep * w[i]);
    w[i] = v;
    if (wb) wb[i] = f2bf(v);
  };
  const int64_t stride = (int64_t)gridDim.x * kUpdThreads * V;
  for (int64_t i = ((int64_t)blockIdx.x * kUpdThreads + threadIdx.x) * V; i + V <= n; i += stride) {
    if constexpr (V == 1) {
      one(i);
    } else {
      const uint4 ov = *reinterpret_cast<const uint4*>(o + i);
      float4 a = *reinterpret_cast<const float4*>(w + i), b = *reinterpret_cast<const float4*>(w + i + 4);
      const uint32_t r[4] = {ov.x, ov.y, ov.z, ov.w};
      float* f[2] = {&a.x, &b.x};
      uint32_t bw[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float& x = f[j / 2][2 * (j & 1)];
        float& y = f[j / 2][2 * (j & 1) + 1];
        x = fmaf(-step, __uint_as_float(r[j] << 16), keep * x);
        y = fmaf(-step, __uint_as_float(r[j] & 0xffff0000u), keep * y);
        const __nv_bfloat162 t = __floats2bfloat162_rn(x, y);
        bw[j] = *reinterpret_cast<const uint32_t*>(&t);
      }
      *reinterpret_cast<float4*>(w + i) = a;
      *reinterpret_cast<float4*>(w + i + 4) = b;
      if (wb) *reinterpret_cast<uint4*>(wb + i) = make_uint4(bw[0], bw[1], bw[2], bw[3]);
    }
  }
  if (blockIdx.x == 0 && threadIdx.x < n % V) one(n - n % V + threadIdx.x);
}

// ------------------------------------------------------------------------------------------------
// Host side

PFN_cuTensorMapEncodeTiled_v12000 g_encode = nullptr;
std::once_flag g_encode_once;
void load_encode() {
  void* f = nullptr;
  cudaDriverEntryPointQueryResult q;
  if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) == cudaSuccess &&
      q == cudaDriverEntryPointSuccess)
    g_encode = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(f);
  else
    cudaGetLastError();
}

int64_t pad16(int64_t v) { return (v + 15) / 16 * 16; }

// The workspace: two pairs of X, A and P, P's diagonals, the norms' partial sums; each part 1024-byte aligned.
struct DirLayout {
  int64_t ldx, lda, n;
  int chunks, per;
  size_t h[2], l[2], A, P, diag_a, diag, part, done, bytes;
};
size_t resident_bytes(int G, int64_t rows, int64_t cols);
DirLayout direction_layout(int G, int64_t rows, int64_t cols) {
  DirLayout d{};
  if (std::min(rows, cols) <= kResSide) {
    d.bytes = resident_bytes(G, rows, cols);
    return d;
  }
  d.n = std::min(rows, cols);
  d.ldx = pad16(cols), d.lda = pad16(d.n);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t was = at;
    at += (bytes + 1023) / 1024 * 1024;
    return was;
  };
  const size_t x = 2 * (size_t)G * rows * d.ldx, a = 2 * (size_t)G * d.n * d.lda;
  for (int i = 0; i < 2; ++i) d.h[i] = take(x), d.l[i] = take(x);
  d.A = take(a), d.P = take(a);
  d.diag_a = take(4 * (size_t)G * d.n);
  d.diag = take(4 * (size_t)G * d.n);
  const int64_t elems = rows * cols;
  d.per = (int)(std::max<int64_t>(4096, (elems + 255) / 256) + 7) / 8 * 8;
  d.chunks = (int)((elems + d.per - 1) / d.per);
  d.part = take(12 * (size_t)G * d.chunks);
  d.done = take(12 * (size_t)G);
  d.bytes = at;
  return d;
}

constexpr int kMaxSide = 32768;

const char* direction_shape_error(int G, int64_t rows, int64_t cols) {
  if (G < 1 || rows < 1 || cols < 1) return "G, rows and cols must be at least 1";
  if (G > 65535 || rows > kMaxSide || cols > kMaxSide) return "at most 65535 matrices of 32768 rows and columns";
  return nullptr;
}

lsgd_status dir_error(lsgd_status s, const char* fn, const char* what) {
  set_last_error(std::string(fn) + ": " + what);
  return s;
}

bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a && b && x < y + nb && y < x + na;
}

bool off_align(const void* p, int z) { return reinterpret_cast<uintptr_t>(p) % z != 0; }

// A rank-3 map over [G][rows][ld] 16-bit values (cols of them in use), 128-byte swizzle, box {64, box_rows}.
bool half_map(CUtensorMap* map, CUtensorMapDataType type, const void* base, int64_t cols, int64_t rows, int64_t ld, int64_t gs,
              int G, int box_rows) {
  cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)G};
  cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)gs * 2};
  cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1}, estr[3] = {1, 1, 1};
  return g_encode(map, type, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The CTAs (PAIR: in pairs) that are resident at once on device `dev` (0: an error), and the kernel's shared-memory limit raised.
template <bool PAIR>
int resident_product_ctas(int dev, size_t smem, cudaError_t* err) {
  static std::atomic<int> known{0};  // (device + 1) << 16 | CTAs
  const int k = known;
  if (k >> 16 == dev + 1) return k & 0xffff;
  *err = cudaFuncSetAttribute(direction_product_kernel<PAIR>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (*err != cudaSuccess) return 0;
  int sms = 0, n = 0;
  *err = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (*err != cudaSuccess) return 0;
  if (PAIR) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(sms / 2 * 2);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2, attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr, cfg.numAttrs = 1;
    *err = cudaOccupancyMaxActiveClusters(&n, direction_product_kernel<PAIR>, &cfg);
    n = 2 * std::min(n, sms / 2);
  } else {
    *err = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, direction_product_kernel<PAIR>, kThreads, smem);
    n = std::min(n, 1) * sms;
  }
  if (*err != cudaSuccess || n < 1) return 0;
  known = (dev + 1) << 16 | n;
  return n;
}

// Whether pairs of CTAs on 256 x 256 tiles are the faster, by a model of a step's three phases: rounds of tiles, each the longer
// of the products' time per k-block of 64 (600 cycles for a pair; 450 for a CTA alone, whose tile a quarter the size needs
// half the operand bytes) and what a tile costs beside them (from the wait for its matrix's last phase to its count: 11,000
// and 7,000 cycles).  Measured, pairs against single CTAs, in us: 16 x 1024 x 1024 399 and 504, 4096 x 4096 1065 and 1430, but
// 2048 x 2048 263 and 248, 5 x 1031 x 777 222 and 188, 16 x 512 x 512 162 and 138, 512 x 512 135 and 103.
bool direction_pairs(int G, int64_t rows, int64_t cols) {
  const int64_t n = std::min(rows, cols), m = std::max(rows, cols);
  auto cost = [&](int tile, int workers, int per_block, int beside) {
    const int64_t ts = (n + tile - 1) / tile, sym = ts * (ts + 1) / 2 * G;
    const int64_t x = ((rows + tile - 1) / tile) * ((cols + tile - 1) / tile) * G;
    auto phase = [&](int64_t tiles, int64_t k) {
      return (tiles + workers - 1) / workers * ((k + kBK - 1) / kBK) * per_block + beside;
    };
    return phase(sym, m) + phase(sym, n) + phase(x, n);
  };
  return cost(256, kNumSMs / 2, 600, 11000) <= cost(128, kNumSMs, 450, 7000);
}

template <bool PAIR>
cudaError_t launch_products(const MmArgs& a, cudaStream_t st) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const size_t smem = sizeof(MmSmem) + 1024;
  const int ctas = resident_product_ctas<PAIR>(dev, smem, &e);
  if (ctas < 1) return e == cudaSuccess ? cudaErrorInvalidConfiguration : e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(ctas);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeCooperative;
  attr[0].val.cooperative = 1;
  cfg.attrs = attr, cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, direction_product_kernel<PAIR>, a);
}

// The resident form's CTAs per matrix: a cluster (a power of two up to 8, the portable size), or `groups` groups of `cl` that
// exchange through global memory where the m rows are too many for a cluster, or where clusters of 8, of which the SMs hold 15 at
// once, take more rounds than the groups, of which they hold 152 / cl.  (16 x 100 x 4096: 195 us in two rounds of clusters, 119 in
// one of groups; of as many rounds the clusters' are the shorter: 8 x 100 x 4096 91 and 113.)  CTAs of at most 256 rows where
// that takes no second round: 16 x 100 x 512 78 us in single CTAs, 61 in clusters of two; 32 x 2048 36 and 28; in groups only above
// n = 64: 100 x 5000 115 and 99, but 2 x 40 x 9000 71 and 73.  Below 256 rows another CTA costs more than it takes over (4 x 16 x
// 256: 16 and 18).  cl = 0: the smaller side is too large.
struct ResPlan {
  int cl, groups;  // groups = 0: clusters
};
ResPlan resident_plan(int G, int64_t rows, int64_t cols) {
  const int64_t n = std::min(rows, cols), m = std::max(rows, cols);
  if (n > kResSide) return ResPlan{0, 0};
  int cl = 1;
  while (cl < 8 && (m + cl - 1) / cl > kRows) cl *= 2;
  const int need = (int)((m + kRows - 1) / kRows), at_once = kNumSMs / need;
  // (all matrices in one round of the larger clusters, of which 76, 36 and 15 fit)
  while (cl < 8 && (m + cl - 1) / cl > kRows / 2 && G <= (cl == 1 ? 76 : cl == 2 ? 36 : 15)) cl *= 2;
  const bool fits = (m + cl - 1) / cl <= kRows;
  if (fits && (cl < 8 || (G + 14) / 15 <= (G + at_once - 1) / at_once)) return ResPlan{cl, 0};
  const int half = (int)((m + kRows / 2 - 1) / (kRows / 2));
  if (n > 64 && (int64_t)G * half <= kNumSMs) return ResPlan{half, G};
  return ResPlan{need, std::min(G, at_once)};
}

// The workspace of the groups: their sums, A, diagonals, norms and counts.
struct ResLayout {
  size_t full, diag, norms, count, bytes;
};
ResLayout resident_layout(const ResPlan& p, int64_t n) {
  ResLayout l{};
  if (!p.groups) return l;
  const size_t n16 = pad16(n), a = n16 * n16;
  l.full = (size_t)p.groups * p.cl * a * 4;
  l.diag = l.full + (size_t)p.groups * a * 2;
  l.norms = l.diag + (size_t)p.groups * n16 * 4;
  l.count = l.norms + (size_t)p.groups * p.cl * 12;
  l.bytes = l.count + (size_t)p.groups * 4;
  return l;
}

size_t resident_bytes(int G, int64_t rows, int64_t cols) {
  return resident_layout(resident_plan(G, rows, cols), std::min(rows, cols)).bytes;
}

template <int NP, bool GLOBAL>
cudaError_t launch_resident(const ResArgs& a, cudaStream_t st) {
  static std::atomic<int> raised{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (raised != dev + 1) {
    e = cudaFuncSetAttribute(direction_resident_kernel<NP, GLOBAL>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             (int)res_smem<NP>(kRows));
    if (e != cudaSuccess) return e;
    raised = dev + 1;
  }
  const int threads = (a.per + 127) / 128 * 128;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)((GLOBAL ? a.groups : a.d.G) * a.cl));
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = res_smem<NP>(threads);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  if (GLOBAL) {  // all CTAs are resident, so that every barrier ends
    attr[0].id = cudaLaunchAttributeCooperative;
    attr[0].val.cooperative = 1;
  } else {
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
  }
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = a.cl, attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr, cfg.numAttrs = !GLOBAL && a.cl > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, direction_resident_kernel<NP, GLOBAL>, a);
}

cudaError_t run_resident(const DirArgs& d, const ResPlan& p, uint8_t* ws, int steps, cudaStream_t st) {
  ResArgs a{};
  a.d = d, a.cl = p.cl, a.groups = p.groups, a.steps = steps;
  a.n = std::min(d.rows, d.cols), a.m = std::max(d.rows, d.cols);
  a.per = (a.m + p.cl - 1) / p.cl;
  if (!p.groups) return a.n <= 64 ? launch_resident<64, false>(a, st) : launch_resident<128, false>(a, st);
  const ResLayout l = resident_layout(p, a.n);
  a.part = reinterpret_cast<float*>(ws), a.full = reinterpret_cast<uint2*>(ws + l.full);
  a.diag = reinterpret_cast<float*>(ws + l.diag), a.norms = reinterpret_cast<float*>(ws + l.norms);
  a.count = reinterpret_cast<uint32_t*>(ws + l.count);
  const cudaError_t e = cudaMemsetAsync(a.count, 0, (size_t)p.groups * 4, st);
  if (e != cudaSuccess) return e;
  return a.n <= 64 ? launch_resident<64, true>(a, st) : launch_resident<128, true>(a, st);
}

cudaError_t run_direction(DirArgs d, const DirLayout& ly, uint8_t* ws, int steps, cudaStream_t st) {
  std::call_once(g_encode_once, load_encode);
  if (!g_encode) return cudaErrorNotSupported;
  __half *h[2], *l[2], *A = reinterpret_cast<__half*>(ws + ly.A), *P = reinterpret_cast<__half*>(ws + ly.P);
  for (int i = 0; i < 2; ++i) h[i] = reinterpret_cast<__half*>(ws + ly.h[i]), l[i] = reinterpret_cast<__half*>(ws + ly.l[i]);
  d.h = h[0], d.l = l[0], d.ld = ly.ldx, d.chunks = ly.chunks, d.per = ly.per;
  d.part = reinterpret_cast<float*>(ws + ly.part);
  d.done = reinterpret_cast<uint32_t*>(ws + ly.done);
  MmArgs a{};
  const int n = (int)ly.n;
  const int64_t x_gs = (int64_t)d.rows * ly.ldx, a_gs = (int64_t)n * ly.lda;
  a.G = d.G, a.n = n, a.rows = d.rows, a.cols = d.cols, a.steps = steps, a.tall = d.rows > d.cols;
  a.diag_a = reinterpret_cast<float*>(ws + ly.diag_a), a.diag = reinterpret_cast<float*>(ws + ly.diag);
  a.done = d.done, a.top = d.done + d.G, a.o = d.o, a.o_gs = d.o_gs;
  a.o_tma = !off_align(d.o, 16) && d.cols % 8 == 0 && d.o_gs % 8 == 0;
  const CUtensorMapDataType f16 = CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
  bool ok = true;
  for (int i = 0; i < 2; ++i)
    ok = ok && half_map(&a.xk[i], f16, h[i], d.cols, d.rows, ly.ldx, x_gs, d.G, kHalf) &&
         half_map(&a.xm[i], f16, h[i], d.cols, d.rows, ly.ldx, x_gs, d.G, 64) &&
         half_map(&a.lk[i], f16, l[i], d.cols, d.rows, ly.ldx, x_gs, d.G, kHalf);
  ok = ok && half_map(&a.ak, f16, A, n, n, ly.lda, a_gs, d.G, kHalf) && half_map(&a.am, f16, A, n, n, ly.lda, a_gs, d.G, 64) &&
       half_map(&a.pk, f16, P, n, n, ly.lda, a_gs, d.G, kHalf) && half_map(&a.pm, f16, P, n, n, ly.lda, a_gs, d.G, 64);
  if (a.o_tma)
    ok = ok && half_map(&a.om, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, d.o, d.cols, d.rows, d.cols, d.o_gs, d.G, kHalf);
  if (!ok) return cudaErrorInvalidValue;
  const dim3 grid(ly.chunks, d.G);
  // values per access: a row of h and l is 32-byte aligned, so a vector that divides the columns stays within a row
  auto aligned = [&](int v) {
    const bool u = d.mom == 0.f || (!off_align(d.u, 16) && (d.G == 1 || d.u_gs % 4 == 0));
    return d.cols % v == 0 && u && !off_align(d.g, d.g_bf16 ? 8 : 16) && (d.G == 1 || d.g_gs % 4 == 0);
  };
  auto prepare = [&](auto momentum, auto normalise) {
    const cudaError_t r = launch_pdl(momentum, grid, dim3(kMomThreads), 0, st, d);
    return r == cudaSuccess ? launch_pdl(normalise, grid, dim3(kMomThreads), 0, st, d) : r;
  };
  cudaError_t e = aligned(8) ? prepare(direction_momentum_kernel<8>, direction_normalise_kernel<8>)
                  : aligned(4) ? prepare(direction_momentum_kernel<4>, direction_normalise_kernel<4>)
                               : prepare(direction_momentum_kernel<1>, direction_normalise_kernel<1>);
  if (e != cudaSuccess) return e;
  return direction_pairs(d.G, d.rows, d.cols) ? launch_products<true>(a, st) : launch_products<false>(a, st);
}

}  // namespace

int direction_take_timeout_flag() {
  int h = 0;
  if (!g_direction_used) return 0;
  if (cudaMemcpyFromSymbol(&h, g_direction_timeout, sizeof(int)) != cudaSuccess) {
    cudaGetLastError();
    return 0;
  }
  if (h) {
    const int zero = 0;
    cudaMemcpyToSymbol(g_direction_timeout, &zero, sizeof(int));
  }
  return h;
}

}  // namespace lsgd

extern "C" {

lsgd_status lsgd_orthogonal_workspace(int G, int64_t rows, int64_t cols, size_t* bytes) {
  using namespace lsgd;
  const char* bad = direction_shape_error(G, rows, cols);
  if (!bad && !bytes) bad = "bytes is NULL";
  if (bad) return dir_error(LSGD_EINVAL, "lsgd_orthogonal_workspace", bad);
  *bytes = direction_layout(G, rows, cols).bytes;
  return LSGD_OK;
}

lsgd_status lsgd_orthogonal_direction(float* u, int64_t u_gs, const void* g, int g_type, int64_t g_gs, uint16_t* o,
                                      int64_t o_gs, int G, int64_t rows, int64_t cols, float momentum, int nesterov,
                                      int steps, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace lsgd;
  const char* fn = "lsgd_orthogonal_direction";
  const char* bad = direction_shape_error(G, rows, cols);
  if (bad) return dir_error(LSGD_EINVAL, fn, bad);
  const DirLayout ly = direction_layout(G, rows, cols);
  const int64_t n = rows * cols;
  if (G == 1) u_gs = g_gs = o_gs = n;  // a single matrix's strides do not matter
  const bool gb = g_type == LSGD_BF16;
  const size_t span_u = 4 * ((size_t)(G - 1) * std::max<int64_t>(u_gs, 0) + n);
  const size_t span_g = (gb ? 2 : 4) * ((size_t)(G - 1) * std::max<int64_t>(g_gs, 0) + n);
  const size_t span_o = 2 * ((size_t)(G - 1) * std::max<int64_t>(o_gs, 0) + n);
  if (!g || !o || (!u && momentum != 0.f)) bad = "a pointer is NULL (u may be only without momentum)";
  else if (!gb && g_type != LSGD_FP32) bad = "g_type is LSGD_FP32 or LSGD_BF16";
  else if (!(momentum >= 0.f) || !(momentum < 1e30f)) bad = "momentum must be non-negative and finite";
  else if (steps < 1 || steps > 100) bad = "steps must be 1 to 100";
  else if (G > 1 && (g_gs < n || o_gs < n || (momentum != 0.f && u_gs < n))) bad = "a matrix stride is below rows * cols";
  else if (off_align(u, 4) || off_align(g, gb ? 2 : 4) || off_align(o, 2)) bad = "a pointer is not aligned to its element";
  else if (ly.bytes && (!workspace || workspace_bytes < ly.bytes || off_align(workspace, 256)))
    bad = "workspace NULL, not 256-byte aligned or smaller than lsgd_orthogonal_workspace says";
  else if (overlap(g, span_g, o, span_o) || overlap(workspace, ly.bytes, g, span_g) || overlap(workspace, ly.bytes, o, span_o) ||
           (momentum != 0.f && (overlap(u, span_u, g, span_g) || overlap(u, span_u, o, span_o) ||
                                overlap(workspace, ly.bytes, u, span_u))))
    bad = "tensors overlap";
  const int64_t ts = (ly.n + 127) / 128, tx = ((rows + 127) / 128) * ((cols + 127) / 128);
  if (!bad && ly.n && G * (ts * (ts + 1) + tx) * steps > 0x3fffffff) bad = "too many matrices of this size in one call";
  if (bad) return dir_error(LSGD_EINVAL, fn, bad);
  if (!g_direction_used) g_direction_used = true;
  DirArgs d{};
  d.u = u, d.g = g, d.o = o, d.u_gs = u_gs, d.g_gs = g_gs, d.o_gs = o_gs;
  d.g_bf16 = gb, d.nesterov = nesterov != 0, d.mom = momentum;
  d.G = G, d.rows = (int)rows, d.cols = (int)cols;
  const ResPlan plan = resident_plan(G, rows, cols);
  const cudaError_t e = plan.cl ? run_resident(d, plan, static_cast<uint8_t*>(workspace), steps, (cudaStream_t)stream)
                                : run_direction(d, ly, static_cast<uint8_t*>(workspace), steps, (cudaStream_t)stream);
  if (e == cudaErrorNotSupported) return dir_error(LSGD_EUNSUPPORTED, fn, "no tensor maps (cuTensorMapEncodeTiled)");
  return e == cudaSuccess ? LSGD_OK : dir_error(LSGD_ECUDA, fn, cudaGetErrorString(e));
}

lsgd_status lsgd_direction_update(float* w, int64_t w_gs, const uint16_t* o, int64_t o_gs, uint16_t* Wb, int G,
                                  int64_t n, float lr, float scale, float weight_decay, void* stream) {
  using namespace lsgd;
  const char* fn = "lsgd_direction_update";
  const char* bad = nullptr;
  if (G < 1 || G > 65535 || n < 1 || n > (int64_t)kMaxSide * kMaxSide) bad = "G is 1 to 65535 and n 1 to 2^30";
  else if (!w || !o) bad = "a pointer is NULL";
  else if (G > 1 && (w_gs < n || o_gs < n)) bad = "a matrix stride is below n";
  else if (off_align(w, 4) || off_align(o, 2) || off_align(Wb, 2)) bad = "a pointer is not aligned to its element";
  else {
    const size_t spw = 4 * ((size_t)(G - 1) * w_gs + n), spo = 2 * ((size_t)(G - 1) * o_gs + n);
    const size_t spb = 2 * ((size_t)(G - 1) * w_gs + n);
    if (overlap(w, spw, o, spo) || overlap(w, spw, Wb, spb) || overlap(o, spo, Wb, spb)) bad = "tensors overlap";
  }
  if (bad) return dir_error(LSGD_EINVAL, fn, bad);
  if (w_gs == n && o_gs == n) n *= G, G = 1;
  const bool vec = n >= 8 && !off_align(w, 16) && !off_align(o, 16) && !off_align(Wb, 16) &&
                   (G == 1 || (w_gs % 8 == 0 && o_gs % 8 == 0));
  const int64_t per = (int64_t)kUpdThreads * (vec ? 8 : 1);
  const int64_t most = std::max<int64_t>(1, 8LL * kNumSMs / G);
  const dim3 grid((unsigned)std::min<int64_t>((n + per - 1) / per, most), G);
  const float keep = (float)(1.0 - (double)lr * weight_decay), step = (float)((double)lr * scale);
  const cudaStream_t st = (cudaStream_t)stream;
  const cudaError_t e = launch_pdl(vec ? direction_update_kernel<8> : direction_update_kernel<1>, grid, dim3(kUpdThreads), 0, st, w,
                                   o, Wb, n, w_gs, o_gs, keep, step);
  return e == cudaSuccess ? LSGD_OK : dir_error(LSGD_ECUDA, fn, cudaGetErrorString(e));
}

}  // extern "C"
