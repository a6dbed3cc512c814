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
// are at most 1.21, so |A| < 1.47 and |P| < 2.9 at all steps.  Measured and modelled: 6e-4 to 1e-3 off (relative 2-norm,
// before the bf16 rounding of 1.7e-3) for random, rank-deficient and ill-conditioned matrices.
#include <cuda_fp16.h>
#include <cudaTypedefs.h>

#include <algorithm>
#include <atomic>
#include <mutex>
#include <string>

#include "../../include/lsgd.h"
#include "common.cuh"
#include "lsgd_internal.h"
#include "tc_ptx.cuh"

namespace lsgd {

__device__ int g_direction_timeout = 0;

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

// kScale / ||x|| as two factors (each in range; applied one after the other), from the sums over the matrix.
// ||x|| = 0 gives 0: the direction of a zero matrix is zero.
__device__ __forceinline__ float2 norm_factors(double mid, double big, double small) {
  double sq;
  int e2 = 0;  // ||x||^2 = sq 2^e2
  if (mid > 0x1p-60 && mid < 1e37) {
    sq = mid;
  } else if (mid >= 1e37 || mid != mid) {
    sq = big, e2 = 160;
  } else {
    sq = small, e2 = -168;
  }
  if (sq == 0.0) return make_float2(0.f, 0.f);
  const double norm = sqrt(sq);  // times 2^(e2 / 2)
  int e = 0;
  double f = 1.0 / norm;  // 0 or NaN where a value is infinite or NaN
  if (f > 0.0) f = frexp(f, &e);
  e += 12 - e2 / 2;
  return make_float2((float)ldexp(f, e / 2), (float)ldexp(1.0, e - e / 2));
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
};

constexpr int kMomThreads = 256;

__device__ __forceinline__ float grad_at(const DirArgs& a, int64_t i) {
  return a.g_bf16 ? bf2f(static_cast<const uint16_t*>(a.g)[i]) : static_cast<const float*>(a.g)[i];
}

__global__ void __launch_bounds__(kMomThreads) direction_momentum_kernel(const DirArgs a) {
  pdl_begin();
  const int64_t n = (int64_t)a.rows * a.cols, i0 = (int64_t)blockIdx.x * a.per, i1 = min(n, i0 + a.per);
  const int64_t k = blockIdx.y;
  NormSums s{0.f, 0.f, 0.f};
#pragma unroll 4
  for (int64_t i = i0 + threadIdx.x; i < i1; i += kMomThreads) {
    const float g = grad_at(a, k * a.g_gs + i);
    float x = g;
    if (a.mom != 0.f) {
      const float u = fmaf(a.mom, a.u[k * a.u_gs + i], g);
      a.u[k * a.u_gs + i] = u;
      x = a.nesterov ? fmaf(a.mom, u, g) : u;
    }
    norm_add(s, x);
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

__global__ void __launch_bounds__(kMomThreads) direction_normalise_kernel(const DirArgs a) {
  pdl_begin();
  const int64_t k = blockIdx.y;
  __shared__ float2 factors;
  if (threadIdx.x < 32) {
    double t[3] = {0, 0, 0};
    for (int c = threadIdx.x; c < a.chunks; c += 32)
      for (int j = 0; j < 3; ++j) t[j] += a.part[(k * a.chunks + c) * 3 + j];
    for (int j = 0; j < 3; ++j)
      for (int o = 16; o; o >>= 1) t[j] += __shfl_xor_sync(~0u, t[j], o);
    if (threadIdx.x == 0) factors = norm_factors(t[0], t[1], t[2]);
  }
  __syncthreads();
  const float2 f = factors;
  const int64_t n = (int64_t)a.rows * a.cols, i0 = (int64_t)blockIdx.x * a.per, i1 = min(n, i0 + a.per);
#pragma unroll 4
  for (int64_t i = i0 + threadIdx.x; i < i1; i += kMomThreads) {
    float x;
    if (a.mom == 0.f) {
      x = grad_at(a, k * a.g_gs + i);
    } else {
      x = a.u[k * a.u_gs + i];
      if (a.nesterov) x = fmaf(a.mom, x, grad_at(a, k * a.g_gs + i));
    }
    __half h, l;
    split_pair(x * f.x * f.y, h, l);
    const int64_t r = i / a.cols, at = (k * a.rows + r) * a.ld + (i - r * a.cols);
    a.h[at] = h;
    a.l[at] = l;
  }
}

// ------------------------------------------------------------------------------------------------
// The products: pairs of CTAs on 256 x 256 tiles (tcgen05 cta_group::2)
//
// A cluster of two CTAs computes a 256 x 256 fp32 tile; CTA r holds rows 128 r .. of it in its tensor memory, loads rows
// 128 r .. of the left operand and 128 r .. of the right operand's 256, and the leader (r = 0) issues the products, which
// read both CTAs' shared memory.  Per k-block of 64 a CTA moves 32 KB for 128 x 256 x 64 products, two thirds of what
// a 128 x 256 tile by one CTA would.
//   warp 0    TMA producer of both operands into a ring of kStages stages (both CTAs' bytes counted on the leader's
//             barrier)
//   warp 1    MMA issuer (leader only)
//   warp 2    tensor memory allocation (two accumulators of 256 columns)
//   warps 4-7 epilogue, a warp per 32 rows

constexpr int kTile = 256, kHalf = 128, kBK = 64, kStages = 6, kThreads = 256;
constexpr uint32_t kOpBytes = kHalf * kBK * 2;  // one operand's share of a stage in a CTA

enum Role { GRAM = 0, POLY = 1, NEXT = 2, LAST = 3 };

struct MmArgs {
  CUtensorMap a, b;   // K-major: box {64 k, 128 rows}; MN-major: box {64 rows, 64 k}
  int a_mn, b_mn;
  int M, N, K, G, role;
  int tall;           // NEXT and LAST: the diagonal goes by column
  int late;           // NEXT and LAST: t is the largest of the diagonal
  const __half* A;    // [G][n][lda], POLY's input
  __half* out;        // GRAM: A, POLY: P (both [G][n][lda], mirrored); NEXT: h
  __half* out_l;      // NEXT
  const __half *h, *l;
  float *diag_a, *diag;  // [G][n]: the diagonals of A and P
  uint16_t* o;
  int64_t lda, ldx, x_gs, o_gs;  // x_gs: elements per matrix of h and l
  int n, ldo, o_vec;  // o_vec: rows of o are 32-byte aligned
};

struct MmSmem {
  uint8_t a[kStages][kOpBytes];  // 1024-aligned
  uint8_t b[kStages][kOpBytes];
  uint64_t full[kStages], empty[kStages];
  uint64_t acc_full[2], acc_empty[2];
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
__device__ __forceinline__ void arrive_at(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// 32 accumulator columns of this warp's 32 rows, one row per lane.
__device__ __forceinline__ void tmem_ld32(uint32_t at, float (&v)[32]) {
  uint32_t r[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,"
      "%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(at)
      : "memory");
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}

// fp16 rows of the workspace: 32 values from or to a 32-byte aligned place (row strides are multiples of 16 values,
// tiles start at multiples of 32); what lies past the row's last value is padding or, past the stride, not touched.
__device__ __forceinline__ void load_half32(const __half* p, int have, float (&v)[32]) {
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    if (16 * q < have) {
      uint32_t w[8];
      asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                   : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                   : "l"(p + 16 * q)
                   : "memory");
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
        v[16 * q + 2 * i] = f.x;
        v[16 * q + 2 * i + 1] = f.y;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) v[16 * q + i] = 0.f;
    }
  }
}
__device__ __forceinline__ void store_words16(void* p, const uint32_t* w) {
  asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]),
               "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}
__device__ __forceinline__ void store_half32(__half* p, int have, const float (&v)[32]) {
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    if (16 * q >= have) break;
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const __half2 t = __floats2half2_rn(v[16 * q + 2 * i], v[16 * q + 2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&t);
    }
    store_words16(p + 16 * q, w);
  }
}

// The epilogue of 32 columns of one row: acc holds columns c0 .. c0 + 31 of row `row` of matrix g.  Rows at or past M
// have been skipped by the caller; `mirror`: the tile's transpose is written too.
__device__ __forceinline__ void mm_epilogue(const MmArgs& a, int g, int row, int c0, float (&v)[32], bool mirror, float t) {
  const int have = a.N - c0;  // > 0
  if (a.role <= POLY) {
    const int64_t base = (int64_t)g * a.n * a.lda;
    float* da = a.diag_a + (int64_t)g * a.n;
    if (a.role == GRAM) {
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        if (c0 + i == row) da[row] = v[i] * kUnscale2, v[i] = 0.f;
        v[i] *= kUnscale;
      }
    } else {  // with D = diag dA and O the rest of A: A A = O O + D O + O D + D D
      float in[32];
      load_half32(a.A + base + (int64_t)row * a.lda + c0, have, in);
      const float dr = da[row];
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const float dc = i < have ? da[c0 + i] : 0.f;
        if (c0 + i == row) {
          a.diag[(int64_t)g * a.n + row] = fmaf(kB, dr, kC * fmaf(dr, dr, v[i] * kUnscale2));
          v[i] = 0.f;
        } else {
          v[i] = fmaf(kB, in[i], kC * fmaf(dr + dc, in[i], kUnscale * v[i]));
        }
      }
    }
    store_half32(a.out + base + (int64_t)row * a.lda + c0, have, v);
    if (mirror) {
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (i < have) a.out[base + (int64_t)(c0 + i) * a.lda + row] = __float2half_rn(v[i]);
    }
    return;
  }
  const int64_t at = (int64_t)g * a.x_gs + (int64_t)row * a.ldx + c0;
  float x[32], lo[32];
  load_half32(a.h + at, have, x);
  load_half32(a.l + at, have, lo);
  const float* dg = a.diag + (int64_t)g * a.n;
  const float dr = a.tall ? 0.f : dg[row];
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    const float d = kA + (a.tall ? (i < have ? dg[c0 + i] : 0.f) : dr);
    x[i] = fmaf(d, x[i], fmaf(kA + t, lo[i], kUnscale * v[i]));
  }
  if (a.role == NEXT) {
#pragma unroll
    for (int i = 0; i < 32; ++i) lo[i] = x[i] - __half2float(__float2half_rn(x[i]));
    store_half32(a.out + at, have, x);
    store_half32(a.out_l + at, have, lo);
    return;
  }
  uint16_t* o = a.o + (int64_t)g * a.o_gs + (int64_t)row * a.ldo + c0;
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    if (a.o_vec && 16 * q + 16 <= have) {
      uint32_t w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const __nv_bfloat162 t = __floats2bfloat162_rn(x[16 * q + 2 * i] * kUnscale, x[16 * q + 2 * i + 1] * kUnscale);
        w[i] = *reinterpret_cast<const uint32_t*>(&t);
      }
      store_words16(o + 16 * q, w);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (16 * q + i < have) o[16 * q + i] = f2bf(x[16 * q + i] * kUnscale);
    }
  }
}

__global__ void __launch_bounds__(kThreads, 1) __cluster_dims__(2, 1, 1)
    direction_product_kernel(const __grid_constant__ MmArgs args) {
  extern __shared__ uint8_t smem_raw[];
  MmSmem& sm = *reinterpret_cast<MmSmem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const int warp = uniform_warp(), lane = threadIdx.x & 31;
  const uint32_t rank = cta_rank();
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  const bool sym = args.role <= POLY;
  const int tm = (args.M + kTile - 1) / kTile, tn = (args.N + kTile - 1) / kTile;
  const int per_matrix = sym ? tm * (tm + 1) / 2 : tm * tn;
  const int tiles = per_matrix * args.G;
  const int nk = (args.K + kBK - 1) / kBK;
  // tile t: matrix by matrix; of a symmetric product the tiles on and below the diagonal, row by row
  auto coords = [&](int t, int& g, int& m0, int& n0) {
    g = t / per_matrix;
    int r = t - g * per_matrix, i, j;
    if (sym) {
      i = (int)((sqrtf(8.f * (float)r + 1.f) - 1.f) * 0.5f);
      while (i * (i + 1) / 2 > r) --i;
      while ((i + 1) * (i + 2) / 2 <= r) ++i;
      j = r - i * (i + 1) / 2;
    } else {
      i = r % tm, j = r / tm;
    }
    m0 = i * kTile, n0 = j * kTile;
  };

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&sm.full[s], 1);
      mbar_init(&sm.empty[s], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sm.acc_full[i], 1);
      mbar_init(&sm.acc_empty[i], 8);  // the epilogue warps of both CTAs
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sm.tmem_base)),
                 "r"(512u)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  pair_sync();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = sm.tmem_base;
  pdl_begin();

  if (warp == 0) {
    const bool el = elect_one();
    int it = 0, s = 0;
    uint32_t ph = 1;
    bool ok = true;
    for (int t = pair; t < tiles && ok; t += pairs) {
      int g, m0, n0;
      coords(t, g, m0, n0);
      m0 += rank * kHalf, n0 += rank * kHalf;
      for (int kb = 0; kb < nk; ++kb, ++it) {
        if (!wait_bar_warp(&sm.empty[s], ph)) {
          ok = false;
          break;
        }
        if (el) {
          const uint32_t bar = in_cta(&sm.full[s], 0);
          if (rank == 0) mbar_expect_tx(&sm.full[s], 4 * kOpBytes);  // two operands, two CTAs
          const int k0 = kb * kBK;
          if (!args.a_mn) {
            tma_load_pair(sm.a[s], &args.a, bar, k0, m0, g);
          } else {
            tma_load_pair(sm.a[s], &args.a, bar, m0, k0, g);
            tma_load_pair(sm.a[s] + kOpBytes / 2, &args.a, bar, m0 + 64, k0, g);
          }
          if (!args.b_mn) {
            tma_load_pair(sm.b[s], &args.b, bar, k0, n0, g);
          } else {
            tma_load_pair(sm.b[s], &args.b, bar, n0, k0, g);
            tma_load_pair(sm.b[s] + kOpBytes / 2, &args.b, bar, n0 + 64, k0, g);
          }
        }
        if (++s == kStages) s = 0, ph ^= 1;
      }
    }
    // after a wait that ran out, the copies in flight (the leader's barriers count both CTAs') are waited for
    if (!ok && rank == 0)
      for (int j = it > kStages ? it - kStages : 0; j < it; ++j) wait_bar(&sm.full[j % kStages], (j / kStages) & 1);
  } else if (warp == 1 && rank == 0) {
    const bool el = elect_one();
    // fp32 accumulators, fp16 operands, N = 256, M = 256
    const uint32_t idesc = (1u << 4) | ((uint32_t)args.a_mn << 15) | ((uint32_t)args.b_mn << 16) |
                           ((uint32_t)(kTile >> 3) << 17) | ((uint32_t)(kTile >> 4) << 24);
    const uint64_t a0 = args.a_mn ? smem_desc(smem_u32(sm.a[0]), kOpBytes / 2, 1024) : smem_desc(smem_u32(sm.a[0]), 16, 1024);
    const uint64_t b0 = args.b_mn ? smem_desc(smem_u32(sm.b[0]), kOpBytes / 2, 1024) : smem_desc(smem_u32(sm.b[0]), 16, 1024);
    const uint32_t a_step = args.a_mn ? 2048 >> 4 : 32 >> 4, b_step = args.b_mn ? 2048 >> 4 : 32 >> 4;
    int i = 0, s = 0;
    uint32_t ph = 0;
    bool ok = true;
    for (int t = pair; t < tiles && ok; t += pairs, ++i) {
      const int ab = i & 1;
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
          if (el) mma_pair(acc, ad + kk * a_step, bd + kk * b_step, idesc, (kb > 0 || kk > 0) ? 1u : 0u);
        if (el) commit_pair(&sm.empty[s]);
        if (++s == kStages) s = 0, ph ^= 1;
      }
      if (ok && el) commit_pair(&sm.acc_full[ab]);
    }
  } else if (warp >= 4) {
    const int quarter = warp & 3;
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    int i = 0, of = -1;
    float top = 0.f;
    for (int t = pair; t < tiles; t += pairs, ++i) {
      int g, m0, n0;
      coords(t, g, m0, n0);
      const int ab = i & 1;
      if (args.late && g != of) {
        const float* d = args.diag + (int64_t)g * args.n;
        top = -INFINITY;
        for (int k = lane; k < args.n; k += 32) top = fmaxf(top, d[k]);
#pragma unroll
        for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
        of = g;
      }
      if (!wait_bar_warp(&sm.acc_full[ab], (i >> 1) & 1)) break;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const int row = m0 + (int)rank * kHalf + quarter * 32 + lane;
      const bool mirror = sym && m0 != n0;
      for (int c = 0; c < kTile && n0 + c < args.N; c += 32) {
        float v[32];
        tmem_ld32(tmem + (uint32_t)(ab * kTile + c) + lanes, v);
        if (row < args.M) mm_epilogue(args, g, row, n0 + c, v, mirror, top);
      }
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) arrive_at(in_cta(&sm.acc_empty[ab], 0));
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  pair_sync();  // no CTA leaves while the other may still signal its barriers or read its operands
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  if (warp == 2)
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
}

// ------------------------------------------------------------------------------------------------
// w = (1 - lr wd) w - lr scale o, and its bf16 copy

constexpr int kUpdThreads = 256;

template <int V>  // values per access: 8 (16 bytes of o, 32 of w) or 1
__global__ void __launch_bounds__(kUpdThreads) direction_update_kernel(float* w, const uint16_t* o, uint16_t* wb,
                                                                       int64_t n, int64_t w_gs, int64_t o_gs,
                                                                       float keep, float step) {
  pdl_begin();
  const int64_t k = blockIdx.y;
  w += k * w_gs, o += k * o_gs;
  if (wb) wb += k * w_gs;
  const int64_t stride = (int64_t)gridDim.x * kUpdThreads * V;
  for (int64_t i = ((int64_t)blockIdx.x * kUpdThreads + threadIdx.x) * V; i < n; i += stride) {
    if constexpr (V == 1) {
      const float v = fmaf(-step, bf2f(o[i]), keep * w[i]);
      w[i] = v;
      if (wb) wb[i] = f2bf(v);
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

// A rank-3 map over [G][rows][ld] fp16 (cols of them in use), 128-byte swizzle, box {64, box_rows}.
bool half_map(CUtensorMap* map, const __half* base, int64_t cols, int64_t rows, int64_t ld, int64_t gs, int G, int box_rows) {
  cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)G};
  cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)gs * 2};
  cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1}, estr[3] = {1, 1, 1};
  return g_encode(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<__half*>(base), dims, strides, box, estr,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int64_t pad16(int64_t v) { return (v + 15) / 16 * 16; }

// The workspace: two pairs of X, A and P, P's diagonals, the norms' partial sums; each part 1024-byte aligned.
struct DirLayout {
  int64_t ldx, lda, n;
  int chunks, per;
  size_t h[2], l[2], A, P, diag_a, diag, part, bytes;
};
DirLayout direction_layout(int G, int64_t rows, int64_t cols) {
  DirLayout d{};
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
  d.per = (int)std::max<int64_t>(4096, (elems + 255) / 256);
  d.chunks = (int)((elems + d.per - 1) / d.per);
  d.part = take(12 * (size_t)G * d.chunks);
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

cudaError_t launch_product(const MmArgs& a, cudaStream_t st) {
  static std::atomic<int> raised{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const size_t smem = sizeof(MmSmem) + 1024;
  if (raised != dev + 1) {
    e = cudaFuncSetAttribute(direction_product_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    raised = dev + 1;
  }
  const int64_t tm = (a.M + kTile - 1) / kTile, tn = (a.N + kTile - 1) / kTile;
  const int64_t tiles = (a.role <= POLY ? tm * (tm + 1) / 2 : tm * tn) * a.G;
  if (tiles > 0x7fffffff) return cudaErrorInvalidValue;
  return launch_pdl(direction_product_kernel, dim3(2 * (unsigned)std::min<int64_t>(tiles, kNumSMs / 2)), dim3(kThreads),
                    smem, st, a);
}

cudaError_t run_direction(DirArgs d, const DirLayout& ly, uint8_t* ws, int steps, cudaStream_t st) {
  std::call_once(g_encode_once, load_encode);
  if (!g_encode) return cudaErrorNotSupported;
  __half *h[2], *l[2], *A = reinterpret_cast<__half*>(ws + ly.A), *P = reinterpret_cast<__half*>(ws + ly.P);
  for (int i = 0; i < 2; ++i) h[i] = reinterpret_cast<__half*>(ws + ly.h[i]), l[i] = reinterpret_cast<__half*>(ws + ly.l[i]);
  d.h = h[0], d.l = l[0], d.ld = ly.ldx, d.chunks = ly.chunks, d.per = ly.per;
  d.part = reinterpret_cast<float*>(ws + ly.part);
  const dim3 grid(ly.chunks, d.G);
  cudaError_t e = launch_pdl(direction_momentum_kernel, grid, dim3(kMomThreads), 0, st, d);
  if (e != cudaSuccess) return e;
  e = launch_pdl(direction_normalise_kernel, grid, dim3(kMomThreads), 0, st, d);
  if (e != cudaSuccess) return e;
  const int n = (int)ly.n, tall = d.rows > d.cols;
  const int64_t x_gs = (int64_t)d.rows * ly.ldx, a_gs = (int64_t)n * ly.lda;
  MmArgs a{};
  a.G = d.G, a.tall = tall, a.n = n, a.lda = ly.lda, a.ldx = ly.ldx, a.x_gs = x_gs;
  a.diag_a = reinterpret_cast<float*>(ws + ly.diag_a), a.diag = reinterpret_cast<float*>(ws + ly.diag);
  a.o = d.o, a.o_gs = d.o_gs, a.ldo = d.cols;
  a.o_vec = !off_align(d.o, 32) && d.cols % 16 == 0 && d.o_gs % 16 == 0;
  CUtensorMap xk[2], xm[2], ak, pk;
  for (int i = 0; i < 2; ++i)
    if (!half_map(&xk[i], h[i], d.cols, d.rows, ly.ldx, x_gs, d.G, kHalf) ||
        !half_map(&xm[i], h[i], d.cols, d.rows, ly.ldx, x_gs, d.G, 64))
      return cudaErrorInvalidValue;
  if (!half_map(&ak, A, n, n, ly.lda, a_gs, d.G, kHalf) || !half_map(&pk, P, n, n, ly.lda, a_gs, d.G, kHalf))
    return cudaErrorInvalidValue;
  for (int s = 0; s < steps; ++s) {
    const int in = s & 1;
    MmArgs q = a;
    q.role = GRAM, q.M = q.N = n, q.K = tall ? d.rows : d.cols;
    q.a = q.b = tall ? xm[in] : xk[in];
    q.a_mn = q.b_mn = tall;
    q.out = A;
    if ((e = launch_product(q, st)) != cudaSuccess) return e;
    q = a;
    q.role = POLY, q.M = q.N = q.K = n, q.a = q.b = ak, q.A = A, q.out = P;
    if ((e = launch_product(q, st)) != cudaSuccess) return e;
    q = a;
    q.role = s + 1 < steps ? NEXT : LAST, q.late = s + 2 >= steps, q.M = d.rows, q.N = d.cols, q.K = n;
    if (tall) q.a = xk[in], q.b = pk;
    else q.a = pk, q.b = xm[in], q.b_mn = 1;
    q.h = h[in], q.l = l[in], q.out = h[in ^ 1], q.out_l = l[in ^ 1];
    if ((e = launch_product(q, st)) != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace

int direction_take_timeout_flag() {
  int h = 0;
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
  else if (!workspace || workspace_bytes < ly.bytes || off_align(workspace, 256))
    bad = "workspace NULL, not 256-byte aligned or smaller than lsgd_orthogonal_workspace says";
  else if (overlap(g, span_g, o, span_o) || overlap(workspace, ly.bytes, g, span_g) || overlap(workspace, ly.bytes, o, span_o) ||
           (momentum != 0.f && (overlap(u, span_u, g, span_g) || overlap(u, span_u, o, span_o) ||
                                overlap(workspace, ly.bytes, u, span_u))))
    bad = "tensors overlap";
  if (bad) return dir_error(LSGD_EINVAL, fn, bad);
  DirArgs d{};
  d.u = u, d.g = g, d.o = o, d.u_gs = u_gs, d.g_gs = g_gs, d.o_gs = o_gs;
  d.g_bf16 = gb, d.nesterov = nesterov != 0, d.mom = momentum;
  d.G = G, d.rows = (int)rows, d.cols = (int)cols;
  const cudaError_t e = run_direction(d, ly, static_cast<uint8_t*>(workspace), steps, (cudaStream_t)stream);
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
  const bool vec = n % 8 == 0 && !off_align(w, 16) && !off_align(o, 16) && !off_align(Wb, 16) &&
                   (G == 1 || (w_gs % 8 == 0 && o_gs % 8 == 0));
  const int64_t per = (int64_t)kUpdThreads * (vec ? 8 : 1);
  const int64_t most = std::max<int64_t>(1, 8LL * kNumSMs / G);
  const dim3 grid((unsigned)std::min<int64_t>((n + per - 1) / per, most), G);
  const float keep = (float)(1.0 - (double)lr * weight_decay), step = (float)((double)lr * scale);
  const cudaStream_t st = (cudaStream_t)stream;
  const cudaError_t e = vec ? launch_pdl(direction_update_kernel<8>, grid, dim3(kUpdThreads), 0, st, w, o, Wb, n, w_gs, o_gs, keep, step)
                            : launch_pdl(direction_update_kernel<1>, grid, dim3(kUpdThreads), 0, st, w, o, Wb, n, w_gs, o_gs, keep, step);
  return e == cudaSuccess ? LSGD_OK : dir_error(LSGD_ECUDA, fn, cudaGetErrorString(e));
}

}  // extern "C"
