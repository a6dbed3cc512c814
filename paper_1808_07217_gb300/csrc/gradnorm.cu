// The norm of each worker's whole gradient, which stands in many tensors, the gradients clipped by it, and the local update with
// the clipped gradient.
//
// For worker k:  norm = sqrt(sum over its tensors' values g^2),  f = min(1, max_norm / norm),  out = f g,
// and in the update  g' = f g + wd w, then the momentum step of lsgd_sgd_update.
//
// All are bound by memory.  The tensors are cut into pieces of one size in bytes, and every warp takes every n-th piece of one
// worker: where the tensors begin is found in a table that comes with the launch, so that hundreds of small tensors cost one
// launch and keep every SM busy.  A warp has a whole piece's loads under way at once.
//
// Sums.  A warp's squares of a piece (at most 66 to a lane, then pairs of lanes) are added in fp32, the pieces' sums in 64 bits, all in
// a fixed order.  Where a piece's fp32 sum is too large or too small for fp32's range its values are squared and added in 64
// bits, whose range holds the square of any fp32 value: no finite gradient overflows, none vanishes.  An SM does two 64-bit
// operations a cycle, a warp's one in 16: they are kept to one lane of a warp and one warp of a CTA (with every thread of 32 warps
// adding their sums up and taking the root, ResNet-20's 16 norms took 34 us).
#include <algorithm>
#include <new>
#include <string>
#include <type_traits>
#include <vector>

#include "../../include/lsgd.h"
#include "common.cuh"
#include "lsgd_internal.h"
#include "operands.h"

struct lsgd_tensors {
  std::vector<lsgd_tensor> list;     // without the empty ones, those of the same types together
  std::vector<uint32_t> first;       // first piece of each, and their number
  struct Launch {
    size_t from, to;                 // tensors, all of the same types
    bool bf16, out_bf16;
    std::vector<uint64_t> table;     // what their kernels find them in
  };
  std::vector<Launch> launches;
  int G = 0, piece = 0;              // workers; bytes of a piece
  bool places = false;               // every tensor has an `out`
  bool overlap = false;              // what a clipping would write overlaps something
  int blocks = 0;                    // CTAs of a worker in the passes
  int cluster = 0;                   // CTAs of a worker where one launch takes the norm (0: two)
  bool clip_once = false;            // and clips
  uintptr_t lo = UINTPTR_MAX, hi = 0;  // all that is read or written lies between
};

namespace lsgd {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxPiece = 4096, kMinPiece = 512;
constexpr int64_t kShare = 160 << 10, kMinShare = 16 << 10;  // bytes of a worker's gradient to a CTA of a cluster
// Bytes that a worker's clipping reads and writes in one launch.  Its CTAs have a pass over all of them behind the norm's; two launches
// give that to all SMs, for 3 us more of the host's time (one worker of 0.47 MB in fp32: 5.9 us, 4.5 on the host; 1.28 MB: 9.4 and
// 4.4 us, 5.2 and 7.7 in two launches; 1.28 MB of bf16 to fp32: 18.1 and 6.3).
constexpr int64_t kClipOnce = 1 << 20;

struct Entry {
  const void* in;
  void* out;
  int64_t n, gs, out_gs;
};
// The tensors of a launch, all of one type and clipped to one type.  A launch's parameters hold up to 32,764 bytes: longer lists take
// several launches.  They are read through the constant caches, where a miss costs as much as one of memory: what is searched
// stands close together, and a piece's tensor is sought from a hint on (40 workers of 200 tensors of about 300 values, clusters of 8:
// 17.5 us, 21 with a search by halves).
constexpr int kHints = 128;
template <int MAX>
struct Table {
  int count, shift;         // tensors; log2 of a piece's bytes
  uint32_t begin, end;      // the launch's pieces
  int hint_shift;           // log2 of the pieces from one hint to the next
  uint16_t hint[kHints];    // the tensor of every 2^hint_shift-th piece
  uint32_t first[MAX + 1];  // first piece of each tensor, and the launch's end
  Entry e[MAX];
};
constexpr int kFew = 64, kSome = 256, kMany = 640;  // sizes of table (a smaller one is a shorter launch)
static_assert(sizeof(Table<kMany>) <= 32000, "a launch's parameters");

// A piece's tensor: the last whose first piece is at most p.
template <int MAX>
__device__ __forceinline__ int find(const Table<MAX>& tab, uint32_t p) {
  int t = tab.hint[(p - tab.begin) >> tab.hint_shift];
  while (tab.first[t + 1] <= p) ++t;
  return t;
}

template <bool BF16>
struct Range {  // a piece's values
  const uint8_t* p;
  int len, head, nv;  // values; those before the first 16-byte boundary; whole vectors behind them
  __device__ __forceinline__ Range(const Entry& e, int shift, int64_t worker, uint32_t piece) {  // piece: of the tensor's
    constexpr int zs = BF16 ? 1 : 2;  // log2 of a value's bytes
    const int64_t at = (int64_t)piece << (shift - zs);
    p = static_cast<const uint8_t*>(e.in) + ((worker * e.gs + at) << zs);
    len = (int)min((int64_t)1 << (shift - zs), e.n - at);
    head = min(len, (int)((0u - (uint32_t)reinterpret_cast<uintptr_t>(p)) & 15u) >> zs);
    nv = (len - head) >> (4 - zs);
  }
};

__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// f(value) for every value of a vector.
template <bool BF16, typename F>
__device__ __forceinline__ void each(const uint4& r, F f) {
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
  if constexpr (BF16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f(bf_lo(w[i])), f(bf_hi(w[i]));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) f(__uint_as_float(w[i]));
  }
}

constexpr int kVecs = kMaxPiece / 16 / 32;  // vectors of a lane

__device__ __forceinline__ double warp_sum(double v) {
  for (int d = 16; d; d /= 2) v += __shfl_xor_sync(0xffffffffu, v, d);
  return v;
}

// The sum of squares of a piece, in lane 0.
template <bool BF16>
__device__ __forceinline__ double piece_squares(const Range<BF16>& r, int lane) {
  const uint4* v = reinterpret_cast<const uint4*>(r.p + r.head * (BF16 ? 2 : 4));
  uint4 raw[kVecs];
#pragma unroll
  for (int i = 0; i < kVecs; ++i)
    raw[i] = lane + 32 * i < r.nv ? __ldg(v + lane + 32 * i) : make_uint4(0, 0, 0, 0);
  // the values before and behind the vectors: at most 7 each
  const int tail = r.head + r.nv * (BF16 ? 8 : 4) + lane;
  uint32_t h = 0, t = 0;
  if constexpr (BF16) {
    if (lane < r.head) h = (uint32_t)__ldg(reinterpret_cast<const uint16_t*>(r.p) + lane) << 16;
    if (tail < r.len) t = (uint32_t)__ldg(reinterpret_cast<const uint16_t*>(r.p) + tail) << 16;
  } else {
    if (lane < r.head) h = __ldg(reinterpret_cast<const uint32_t*>(r.p) + lane);
    if (tail < r.len) t = __ldg(reinterpret_cast<const uint32_t*>(r.p) + tail);
  }
  const float hf = __uint_as_float(h), tf = __uint_as_float(t);
  float s = fmaf(hf, hf, tf * tf);
#pragma unroll
  for (int i = 0; i < kVecs; ++i) each<BF16>(raw[i], [&](float x) { s = fmaf(x, x, s); });
#pragma unroll
  for (int d = 16; d; d /= 2) s += __shfl_xor_sync(0xffffffffu, s, d);
  // (the same sum in every lane: a + b is b + a.  A value whose square lost bits below 2^-149 is at most 2^-49 of a sum of 2^-100.)
  if (s >= 0x1p-100f && s < 0x1p126f) return s;
  uint32_t any = (h | t) & 0x7fffffffu;
#pragma unroll
  for (int i = 0; i < kVecs; ++i) any |= (raw[i].x | raw[i].y | raw[i].z | raw[i].w) & (BF16 ? 0x7fff7fffu : 0x7fffffffu);
  if (!__any_sync(0xffffffffu, any)) return 0.0;
  double d = (double)hf * hf + (double)tf * tf;
#pragma unroll 1
  for (int i = 0; i < kVecs; ++i) {
    uint4 w = raw[0];
#pragma unroll
    for (int j = 1; j < kVecs; ++j)
      if (j == i) w = raw[j];
    each<BF16>(w, [&](float x) {
      if (x != 0.f) d += (double)x * x;
    });
  }
  return warp_sum(d);
}

// The warps' sums (in lane 0 of each), added by the first warp: in thread 0.
template <int THREADS>
__device__ __forceinline__ double block_sum(double v) {
  __shared__ double part[THREADS / 32];
  if ((threadIdx.x & 31) == 0) part[threadIdx.x / 32] = v;
  __syncthreads();
  if (threadIdx.x >= 32) return 0.0;
  return warp_sum(threadIdx.x < THREADS / 32 ? part[threadIdx.x] : 0.0);
}
// The root of a sum of squares, to fp32: by the fp32 root where the sum is in its range.
__device__ __forceinline__ float root(double s) {
  if (s >= 0x1p-100 && s < 0x1p120) return __fsqrt_rn((float)s);
  return (float)sqrt(s);
}

// The sum of squares of every `stride`-th piece of a worker from p on, in lane 0.
template <bool BF16, int MAX>
__device__ __forceinline__ double squares_of(const Table<MAX>& tab, int64_t worker, uint64_t p, uint32_t stride) {
  double s = 0.0;
  int t = p < tab.end ? find(tab, (uint32_t)p) : 0;  // (the table does not depend on other kernels: it is there before they are done)
  pdl_begin();
  for (; p < tab.end; p += stride) {
    t = find(tab, (uint32_t)p);
    const double q = piece_squares(Range<BF16>(tab.e[t], tab.shift, worker, (uint32_t)p - tab.first[t]), threadIdx.x & 31);
    if ((threadIdx.x & 31) == 0) s += q;
  }
  return s;
}

// One sum for each CTA into part [G][slots] from slot `slot` on, or, with `norm`, the norm of its worker.
template <int MAX, bool BF16>
__global__ void __launch_bounds__(kThreads, 4) grad_squares_kernel(const __grid_constant__ Table<MAX> tab, double* part, int slot,
                                                                   int slots, float* norm) {
  const double s = block_sum<kThreads>(squares_of<BF16>(tab, blockIdx.y, tab.begin + blockIdx.x * kWarps + threadIdx.x / 32,
                                                  gridDim.x * kWarps));
  if (threadIdx.x) return;
  if (norm) norm[blockIdx.y] = root(s);
  else part[(int64_t)blockIdx.y * slots + slot + blockIdx.x] = s;
}

// A worker's sum of squares from its CTAs' sums, in thread 0.
__device__ __forceinline__ double sum_of_parts(const double* part, int slots, int worker) {
  double s = 0.0;
  for (int i = threadIdx.x; i < slots; i += kThreads) s += part[(int64_t)worker * slots + i];
  return block_sum<kThreads>(warp_sum(s));
}
__global__ void __launch_bounds__(kThreads) grad_norm_kernel(const double* part, int slots, float* norm) {
  pdl_begin();
  const double s = sum_of_parts(part, slots, blockIdx.x);
  if (threadIdx.x == 0) norm[blockIdx.x] = root(s);
}

// min(1, max_norm / norm): NaN for a NaN norm, 0 for an infinite one.
__device__ __forceinline__ float clip_factor(float norm, float max_norm) { return norm <= max_norm ? 1.f : __fdiv_rn(max_norm, norm); }
// A factor below 2^-100, which below 2^-126 fp32 holds with few bits or not at all though f g may be an ordinary number: to be multiplied
// by as p, a power of two, and then as q, of full precision (from f = 2^-252 on; below, no product reaches 2^-124, and q is off by
// 2^-150).  A value that p takes below fp32's normal range has a product below 2^-149.
constexpr float kSmallFactor = 0x1p-100f;
struct Factor {
  float p, q;
  __device__ __forceinline__ float operator()(float x) const { return x * p * q; }
};
// max_norm / (norm 2^64).
__device__ __forceinline__ Factor small_factor(float norm, float max_norm) {
  const float q = __fdiv_rn(max_norm, norm);
  if (q >= 0x1p-36f) return {1.f, q * 0x1p-64f};
  if (q >= 0x1p-126f) return {0x1p-64f, q};
  return {0x1p-126f, __fdiv_rn(max_norm * 0x1p62f, norm)};
}
// Any factor, of a norm that is all that is known.
__device__ __forceinline__ Factor any_factor(float norm, float max_norm) {
  const float f = clip_factor(norm, max_norm);
  return f < kSmallFactor && norm < INFINITY ? small_factor(norm, max_norm * 0x1p64f) : Factor{1.f, f};
}

// The 16 bytes that begin `shift` (an even number, below 16) bytes behind a's first, of a and what follows it, b.
__device__ __forceinline__ uint4 funnel(const uint4& a, const uint4& b, int shift) {
  uint32_t w[5];
  const int words = shift >> 2;
  if (words == 0) w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w, w[4] = b.x;
  else if (words == 1) w[0] = a.y, w[1] = a.z, w[2] = a.w, w[3] = b.x, w[4] = b.y;
  else if (words == 2) w[0] = a.z, w[1] = a.w, w[2] = b.x, w[3] = b.y, w[4] = b.z;
  else w[0] = a.w, w[1] = b.x, w[2] = b.y, w[3] = b.z, w[4] = b.w;
  if (shift & 2) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __byte_perm(w[i], w[i + 1], 0x5432);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// 16 bytes of values times f to `to`, in 8, 16 or 32 bytes.
template <bool BF16, bool OB>
__device__ __forceinline__ void scale_vector(const uint4& r, void* to, float f) {
  float x[8];
  int k = 0;
  each<BF16>(r, [&](float q) { x[k++] = q * f; });
  const auto pair = [&](int q) { return (uint32_t)f2bf(x[q]) | (uint32_t)f2bf(x[q + 1]) << 16; };
  if constexpr (OB && BF16) {
    __stcs(static_cast<uint4*>(to), make_uint4(pair(0), pair(2), pair(4), pair(6)));
  } else if constexpr (OB) {
    __stcs(static_cast<uint2*>(to), make_uint2(pair(0), pair(2)));
  } else {
    __stcs(static_cast<float4*>(to), make_float4(x[0], x[1], x[2], x[3]));
    if (BF16) __stcs(static_cast<float4*>(to) + 1, make_float4(x[4], x[5], x[6], x[7]));
  }
}

// A piece's values times f to its place, by a warp.  (Stores that leave L2 to the gradients that are still to be read.)
template <bool BF16, bool OB>
__device__ __forceinline__ void scale_piece(const Range<BF16>& r, uint8_t* out, float f) {
  const int lane = threadIdx.x & 31;
  constexpr int z = BF16 ? 2 : 4, oz = OB ? 2 : 4, width = 16 / z;  // bytes of a value; values of 16 bytes
  const auto one = [&](int i) {
    const float v = BF16 ? bf2f(reinterpret_cast<const uint16_t*>(r.p)[i]) : reinterpret_cast<const float*>(r.p)[i];
    if constexpr (OB) reinterpret_cast<uint16_t*>(out)[i] = f2bf(v * f);
    else reinterpret_cast<float*>(out)[i] = v * f;
  };
  constexpr int align = width * oz < 16 ? width * oz : 16;  // of a store
  if ((reinterpret_cast<uintptr_t>(out) + r.head * oz) % align == 0) {
    const uint4* v = reinterpret_cast<const uint4*>(r.p + r.head * z);
    const int tail = r.head + r.nv * width + lane;
#pragma unroll 1
    for (int i = lane; i < r.nv; i += 128) {
      uint4 raw[4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (i + 32 * j < r.nv) raw[j] = v[i + 32 * j];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (i + 32 * j < r.nv) scale_vector<BF16, OB>(raw[j], out + (r.head + (i + 32 * j) * width) * oz, f);
    }
    if (lane < r.head) one(lane);
    if (tail < r.len) one(tail);
    return;
  }
  // What is read and what is written are not aligned together: every store's values from two aligned loads, as far as these lie within
  // the piece; the values before and behind them (at most 15 each) one by one.
  int first = (int)((0u - (uint32_t)reinterpret_cast<uintptr_t>(out)) & (align - 1)) / oz;
  const uintptr_t p = reinterpret_cast<uintptr_t>(r.p);
  if (((p + first * z) & ~(uintptr_t)15) < p) first += width;
  const uintptr_t base = (p + first * z) & ~(uintptr_t)15, end = p + r.len * z;
  const int by = (int)(p + first * z - base), nv = end >= base + 16 ? (int)((end - base - 16) / 16) : 0;
  first = min(first, r.len);
  const int rest = nv ? first + nv * width : first;
  const uint4* v = reinterpret_cast<const uint4*>(base);
#pragma unroll 1
  for (int i = lane; i < nv; i += 64) {
    uint4 a[2], b[2];
#pragma unroll
    for (int j = 0; j < 2; ++j)
      if (i + 32 * j < nv) a[j] = v[i + 32 * j], b[j] = v[i + 32 * j + 1];
#pragma unroll
    for (int j = 0; j < 2; ++j)
      if (i + 32 * j < nv) scale_vector<BF16, OB>(funnel(a[j], b[j], by), out + (first + (i + 32 * j) * width) * oz, f);
  }
  if (lane < first) one(lane);
  for (int i = rest + lane; i < r.len; i += 32) one(i);
}
// Every `stride`-th piece of a worker, times f, from the last to the first: L2 still holds what was read last.
template <bool BF16, bool OB, int MAX>
__device__ __forceinline__ void scale_pieces(const Table<MAX>& tab, int64_t worker, uint32_t p, uint32_t stride, float f) {
  if (p >= tab.end) return;
  for (p += (tab.end - 1 - p) / stride * stride;; p -= stride) {
    const int t = find(tab, p);
    const Entry& e = tab.e[t];
    // (left as it is only where this worker's place is the one that was read: the first worker's may be, and no other's)
    if (f != 1.f || e.out != e.in || (worker && e.out_gs != e.gs)) {
      const uint32_t piece = p - tab.first[t];
      const int64_t at = worker * e.out_gs + ((int64_t)piece << (tab.shift - (BF16 ? 1 : 2)));
      scale_piece<BF16, OB>(Range<BF16>(e, tab.shift, worker, piece), static_cast<uint8_t*>(e.out) + at * (OB ? 2 : 4), f);
    }
    if (p < tab.begin + stride) return;
  }
}

// Every `stride`-th piece of a worker from p on, times its small factor; false, and nothing done, where there is none: the norm is
// that of an infinite value.  `squares`: the norm's square, which holds what the norm does not where this passes fp32's range (and its root
// does not times 2^-64); NULL: to be summed, by a CTA that has all of the worker's pieces.  Rare: value by value, and apart from the
// kernels' own code (with factors of two parts for every value there, 300 ragged bf16 tensors of 26 MB took 19.5 to 19.8 us, and take 19.3).
template <int THREADS, bool BF16, bool OB, int MAX>
__device__ __noinline__ bool scale_by_small(const Table<MAX>& tab, int64_t worker, uint32_t p, uint32_t stride, float norm,
                                            const double* squares, float max_norm) {
  Factor f;
  if (norm < INFINITY) {
    f = small_factor(norm, max_norm * 0x1p64f);
  } else {
    __shared__ double sum;
    if (!squares) {
      const double s = block_sum<THREADS>(squares_of<BF16>(tab, worker, p, stride));
      if (threadIdx.x == 0) sum = s;
      __syncthreads();
      squares = &sum;
    }
    if (!(*squares < INFINITY)) return false;
    f = small_factor(root(*squares * 0x1p-128), max_norm);
  }
  for (uint64_t at_piece = p; at_piece < tab.end; at_piece += stride) {
    const int t = find(tab, (uint32_t)at_piece);
    const Entry& e = tab.e[t];
    const uint32_t piece = (uint32_t)at_piece - tab.first[t];
    const Range<BF16> r(e, tab.shift, worker, piece);
    const int64_t at = worker * e.out_gs + ((int64_t)piece << (tab.shift - (BF16 ? 1 : 2)));
    for (int i = threadIdx.x & 31; i < r.len; i += 32) {
      const float v = f(BF16 ? bf2f(reinterpret_cast<const uint16_t*>(r.p)[i]) : reinterpret_cast<const float*>(r.p)[i]);
      if constexpr (OB) static_cast<uint16_t*>(e.out)[at + i] = f2bf(v);
      else static_cast<float*>(e.out)[at + i] = v;
    }
  }
  return true;
}
// What a worker's norm makes of its gradients.
template <int THREADS, bool BF16, bool OB, int MAX>
__device__ __forceinline__ void clip_pieces(const Table<MAX>& tab, int64_t worker, uint32_t p, uint32_t stride, float norm,
                                            const double* squares, float max_norm) {
  const float f = clip_factor(norm, max_norm);
  if (f < kSmallFactor && scale_by_small<THREADS, BF16, OB>(tab, worker, p, stride, norm, squares, max_norm)) return;
  scale_pieces<BF16, OB>(tab, worker, p, stride, f);
}

// The second of two launches: every CTA adds its worker's sums up by itself.
template <int MAX, bool BF16, bool OB>
__global__ void __launch_bounds__(kThreads, 4) grad_scale_kernel(const __grid_constant__ Table<MAX> tab, const double* part, int slots,
                                                                 float* norm, float max_norm) {
  pdl_begin();
  __shared__ float shared;
  __shared__ double squares;
  const uint32_t p = tab.begin + blockIdx.x * kWarps + threadIdx.x / 32, stride = gridDim.x * kWarps;
  float n;
  if (slots > 1) {
    const double s = sum_of_parts(part, slots, blockIdx.y);
    if (threadIdx.x == 0) {
      shared = root(s), squares = s;
      if (blockIdx.x == 0) norm[blockIdx.y] = shared;
    }
    __syncthreads();
    n = shared;
  } else {
    n = norm[blockIdx.y];  // (a worker's only CTA has written it in the first launch, but not the sum that it is the root of)
  }
  clip_pieces<kThreads, BF16, OB>(tab, blockIdx.y, p, stride, n, slots > 1 ? &squares : nullptr, max_norm);
}

// Both in one launch, a worker to a cluster: the CTAs' sums meet in shared memory.
constexpr int kClusterThreads = 512, kMaxCluster = 8;

template <int MAX, bool BF16, bool CLIP, bool OB>
__global__ void __launch_bounds__(kClusterThreads) grad_cluster_kernel(const __grid_constant__ Table<MAX> tab, float* norm,
                                                                          float max_norm) {
  __shared__ double sums[kMaxCluster];
  const uint32_t cl = gridDim.x;  // a cluster is a row of the grid
  if (cl > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  const uint32_t p = tab.begin + blockIdx.x * (kClusterThreads / 32) + threadIdx.x / 32, stride = cl * (kClusterThreads / 32);
  double s = block_sum<kClusterThreads>(squares_of<BF16>(tab, blockIdx.y, p, stride));
  if (cl > 1) {
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");  // every CTA's shared memory is there
    if (threadIdx.x == 0)
      for (uint32_t i = 0; i < cl; ++i) {
        uint32_t to;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"((uint32_t)__cvta_generic_to_shared(&sums[blockIdx.x])), "r"(i));
        asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(to), "d"(s) : "memory");
      }
    if (threadIdx.x < 32) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");  // (only its stores count)
    else asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
  __shared__ float shared;
  __shared__ double squares;
  if (threadIdx.x == 0) {
    if (cl > 1) {
      s = 0.0;
      for (uint32_t i = 0; i < cl; ++i) s += sums[i];
    }
    shared = root(s);
    if (CLIP) squares = s;
    if (blockIdx.x == 0) norm[blockIdx.y] = shared;
  }
  if constexpr (!CLIP) return;
  __syncthreads();
  const float n = shared;
  if constexpr (CLIP) clip_pieces<kClusterThreads, BF16, OB>(tab, blockIdx.y, p, stride, n, &squares, max_norm);
}

// ---- the local update with the clipped gradient ----
struct UpdateArgs {
  float *w, *u;
  const void* g;
  uint16_t* wb;
  int64_t w_gs, g_gs, n, decay_end;
  const float* norm;
  float max_norm, lr, m, wd;
};

template <bool GB, bool MOM, bool NEST, bool SHADOW, bool WIDE>
__global__ void __launch_bounds__(256) clipped_update_kernel(const UpdateArgs a) {
  pdl_begin();
  const int64_t k = blockIdx.y, stride = (int64_t)gridDim.x * blockDim.x, first = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  const Factor f = any_factor(a.norm[k], a.max_norm);
  float *w = a.w + k * a.w_gs, *u = a.u + (MOM ? k * a.w_gs : 0);
  uint16_t* wb = a.wb + (SHADOW ? k * a.w_gs : 0);
  const float* gf = static_cast<const float*>(a.g) + (GB ? 0 : k * a.g_gs);
  const uint16_t* gb = static_cast<const uint16_t*>(a.g) + (GB ? k * a.g_gs : 0);
  const auto one = [&](int64_t i) {
    float wv = w[i], uv = MOM ? u[i] : 0.f;
    sgd_elem<MOM, NEST>(wv, uv, f(GB ? bf2f(gb[i]) : gf[i]), a.lr, a.m, i < a.decay_end ? a.wd : 0.f);
    w[i] = wv;
    if (MOM) u[i] = uv;
    if (SHADOW) wb[i] = f2bf(wv);
  };
  int64_t done = 0;
  if constexpr (WIDE) {
    const int64_t n4 = a.n / 4;
    for (int64_t j = first; j < n4; j += stride) {
      const int64_t i = n4 - 1 - j;  // from the end on: L2 still holds what the norm read last
      float gv[4], wv[4], uv[4];
      if constexpr (GB) {
        const uint2 r = __ldcs(reinterpret_cast<const uint2*>(gb) + i);
        gv[0] = bf_lo(r.x), gv[1] = bf_hi(r.x), gv[2] = bf_lo(r.y), gv[3] = bf_hi(r.y);
      } else {
        *reinterpret_cast<float4*>(gv) = __ldcs(reinterpret_cast<const float4*>(gf) + i);
      }
      *reinterpret_cast<float4*>(wv) = __ldcs(reinterpret_cast<const float4*>(w) + i);
      if (MOM) *reinterpret_cast<float4*>(uv) = __ldcs(reinterpret_cast<const float4*>(u) + i);
#pragma unroll
      for (int k = 0; k < 4; ++k)
        sgd_elem<MOM, NEST>(wv[k], uv[k], f(gv[k]), a.lr, a.m, 4 * i + k < a.decay_end ? a.wd : 0.f);
      if (MOM) __stcs(reinterpret_cast<float4*>(u) + i, *reinterpret_cast<float4*>(uv));
      __stcs(reinterpret_cast<float4*>(w) + i, *reinterpret_cast<float4*>(wv));
      if (SHADOW)
        __stcs(reinterpret_cast<uint2*>(wb) + i, make_uint2((uint32_t)f2bf(wv[0]) | (uint32_t)f2bf(wv[1]) << 16,
                                                            (uint32_t)f2bf(wv[2]) | (uint32_t)f2bf(wv[3]) << 16));
    }
    done = n4 * 4;
  }
  for (int64_t i = done + first; i < a.n; i += stride) one(i);
}

template <bool GB, bool MOM, bool NEST, bool SHADOW>
cudaError_t launch_clipped(const UpdateArgs& a, int G, bool wide, cudaStream_t st) {
  const int64_t items = wide ? std::max<int64_t>(a.n / 4, 1) : a.n;
  const int64_t most = std::max<int64_t>(1, (int64_t)kNumSMs * 8 / G);
  const dim3 grid((unsigned)std::min<int64_t>(most, (items + 255) / 256), G);
  return wide ? launch_pdl(clipped_update_kernel<GB, MOM, NEST, SHADOW, true>, grid, dim3(256), 0, st, a)
              : launch_pdl(clipped_update_kernel<GB, MOM, NEST, SHADOW, false>, grid, dim3(256), 0, st, a);
}
template <bool GB, bool MOM, bool NEST>
cudaError_t clipped_shadow(const UpdateArgs& a, int G, bool wide, cudaStream_t st) {
  return a.wb ? launch_clipped<GB, MOM, NEST, true>(a, G, wide, st) : launch_clipped<GB, MOM, NEST, false>(a, G, wide, st);
}
template <bool GB>
cudaError_t clipped_rule(const UpdateArgs& a, int G, bool nesterov, bool wide, cudaStream_t st) {
  if (a.m == 0.f) return clipped_shadow<GB, false, false>(a, G, wide, st);
  return nesterov ? clipped_shadow<GB, true, true>(a, G, wide, st) : clipped_shadow<GB, true, false>(a, G, wide, st);
}

lsgd_status gr_error(lsgd_status s, const char* fn, const char* what) {
  set_last_error(std::string(fn) + ": " + what);
  return s;
}
int size_of(int type) { return type == LSGD_BF16 ? 2 : 4; }

int slots_of(const lsgd_tensors& l) { return l.blocks * (int)l.launches.size(); }
int out_type(const lsgd_tensor& t, bool places) { return places ? t.out_type : t.g_type; }

template <int MAX>
void fill(lsgd_tensors::Launch& launch, const lsgd_tensors& l) {
  launch.table.resize((sizeof(Table<MAX>) + 7) / 8);
  Table<MAX>& tab = *reinterpret_cast<Table<MAX>*>(launch.table.data());
  tab.count = (int)(launch.to - launch.from);
  tab.shift = __builtin_ctz(l.piece);
  tab.begin = l.first[launch.from], tab.end = l.first[launch.to];
  while ((tab.end - tab.begin - 1) >> tab.hint_shift >= kHints) ++tab.hint_shift;
  for (uint32_t i = 0, t = 0; i < kHints && (i << tab.hint_shift) < tab.end - tab.begin; ++i) {
    while (l.first[launch.from + t + 1] <= tab.begin + (i << tab.hint_shift)) ++t;
    tab.hint[i] = (uint16_t)t;
  }
  tab.first[tab.count] = tab.end;
  for (size_t i = launch.from; i < launch.to; ++i) {
    const lsgd_tensor& t = l.list[i];
    Entry& e = tab.e[i - launch.from];
    e.in = t.g, e.out = l.places ? t.out : const_cast<void*>(t.g);
    e.n = t.n, e.gs = t.g_gs, e.out_gs = l.places ? t.out_gs : t.g_gs;
    tab.first[i - launch.from] = l.first[i];
  }
}
template <typename F>
auto with_size(size_t count, F f) {
  if (count <= kFew) return f(std::integral_constant<int, kFew>{});
  if (count <= kSome) return f(std::integral_constant<int, kSome>{});
  return f(std::integral_constant<int, kMany>{});
}
// f(the table's size, BF16, OB) of a launch.
template <typename F>
cudaError_t with_kind(const lsgd_tensors::Launch& l, F f) {
  return with_size(l.to - l.from, [&](auto max) {
    if (l.bf16) return l.out_bf16 ? f(max, std::true_type{}, std::true_type{}) : f(max, std::true_type{}, std::false_type{});
    return l.out_bf16 ? f(max, std::false_type{}, std::true_type{}) : f(max, std::false_type{}, std::false_type{});
  });
}

// The launch of a kernel on its table (which is copied once, by the launch itself); cluster: CTAs of one.
template <typename TAB, typename... T, typename... A>
cudaError_t launch_table(void (*kernel)(TAB, T...), const lsgd_tensors::Launch& l, dim3 grid, int threads, int cluster,
                         cudaStream_t st, A... given) {
  return [&](T... args) {
    void* p[] = {const_cast<uint64_t*>(l.table.data()), &args...};
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelExC(&cfg, reinterpret_cast<const void*>(kernel), p);
  }(given...);
}

// The norms and, with max_norm > 0, the clipped gradients.
cudaError_t norm_and_clip(const lsgd_tensors& l, float* norm, float max_norm, double* part, cudaStream_t st) {
  const size_t n = l.launches.size();
  const bool clip = max_norm > 0.f;
  if (n == 0) return cudaMemsetAsync(norm, 0, sizeof(float) * l.G, st);
  if (clip ? l.clip_once : l.cluster > 0)
    return with_kind(l.launches[0], [&](auto max, auto bf16, auto ob) {
      constexpr bool B = decltype(bf16)::value, O = decltype(ob)::value;
      constexpr int MAX = decltype(max)::value;
      return launch_table(clip ? grad_cluster_kernel<MAX, B, true, O> : grad_cluster_kernel<MAX, B, false, false>, l.launches[0],
                          dim3(l.cluster, l.G), kClusterThreads, l.cluster, st, norm, max_norm);
    });
  const int slots = slots_of(l);
  const dim3 grid(l.blocks, l.G);
  cudaError_t e = cudaSuccess;
  for (size_t i = 0; i < n && e == cudaSuccess; ++i)
    e = with_kind(l.launches[i], [&](auto max, auto bf16, auto) {
      return launch_table(grad_squares_kernel<decltype(max)::value, decltype(bf16)::value>, l.launches[i], grid, kThreads, 1, st, part,
                          (int)i * l.blocks, slots, slots == 1 ? norm : nullptr);
    });
  if (!clip) {
    if (e != cudaSuccess || slots == 1) return e;
    return launch_pdl(grad_norm_kernel, dim3(l.G), dim3(kThreads), 0, st, (const double*)part, slots, norm);
  }
  for (size_t i = 0; i < n && e == cudaSuccess; ++i)
    e = with_kind(l.launches[i], [&](auto max, auto bf16, auto ob) {
      return launch_table(grad_scale_kernel<decltype(max)::value, decltype(bf16)::value, decltype(ob)::value>, l.launches[i], grid,
                          kThreads, 1, st, part, slots, norm, max_norm);
    });
  return e;
}

size_t gr_workspace(const lsgd_tensors& l) { return !l.clip_once && slots_of(l) > 1 ? (size_t)l.G * slots_of(l) * sizeof(double) : 0; }

// The first or the last address of a tensor's blocks (gs may be any number where there is one worker).
uintptr_t end_of(const void* p, int64_t n, int64_t gs, int type, int G) {
  return reinterpret_cast<uintptr_t>(p) + (uintptr_t)((G - 1) * gs + n) * size_of(type);
}

// Whether what a clipping writes meets anything: every worker's every tensor, in order of address.  A tensor may be clipped in
// place (what is written there is what is read), but not twice.
bool clip_overlaps(const lsgd_tensors& l) {
  struct Block {
    uintptr_t at, end;
    bool written;
  };
  std::vector<Block> b;
  b.reserve(l.list.size() * l.G * 2);
  for (const lsgd_tensor& t : l.list)
    for (int k = 0; k < l.G; ++k) {
      const uintptr_t in = reinterpret_cast<uintptr_t>(t.g) + (uintptr_t)(k * t.g_gs) * size_of(t.g_type);
      const uintptr_t in_end = in + (uintptr_t)t.n * size_of(t.g_type);
      const uintptr_t out = l.places ? reinterpret_cast<uintptr_t>(t.out) + (uintptr_t)(k * t.out_gs) * size_of(t.out_type) : in;
      const uintptr_t out_end = out + (uintptr_t)t.n * size_of(l.places ? t.out_type : t.g_type);
      b.push_back({out, out_end, true});
      if (in != out || in_end != out_end) b.push_back({in, in_end, false});
    }
  std::sort(b.begin(), b.end(), [](const Block& x, const Block& y) { return x.at < y.at; });
  uintptr_t end = 0, written_end = 0;  // of all blocks so far, of the written ones
  for (const Block& x : b) {
    if (x.at < (x.written ? end : written_end)) return true;
    end = std::max(end, x.end);
    if (x.written) written_end = std::max(written_end, x.end);
  }
  return false;
}

// Whether [p, p + bytes) meets a tensor of the list.
bool meets(const lsgd_tensors& l, const void* p, size_t bytes) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(p);
  if (!bytes || at >= l.hi || at + bytes <= l.lo) return false;
  const Blocks mine(p, bytes);
  for (const lsgd_tensor& t : l.list)
    if (blocks_meet(mine, Blocks(t.g, (size_t)t.n * size_of(t.g_type), t.g_gs, l.G, size_of(t.g_type))) ||
        (l.places && blocks_meet(mine, Blocks(t.out, (size_t)t.n * size_of(t.out_type), t.out_gs, l.G, size_of(t.out_type)))))
      return true;
  return false;
}

const char* norm_error(const lsgd_tensors* l, const float* norm, const void* workspace, size_t bytes) {
  if (!l) return "the list is NULL";
  const size_t need = gr_workspace(*l);
  if (!norm || misaligned(norm, 4)) return "norm is NULL or not aligned";
  if (need && (!workspace || bytes < need || misaligned(workspace, 16)))
    return "workspace NULL, not 16-byte aligned or smaller than lsgd_gradient_workspace says";
  if (meets(*l, norm, 4 * (size_t)l->G) || meets(*l, workspace, need) ||
      (need && blocks_meet(Blocks(norm, 4 * (size_t)l->G), Blocks(workspace, need))))
    return "tensors overlap";
  return nullptr;
}

}  // namespace
}  // namespace lsgd

extern "C" {

lsgd_status lsgd_tensors_create(const lsgd_tensor* tensors, int count, int G, lsgd_tensors** out) {
  using namespace lsgd;
  const char* fn = "lsgd_tensors_create";
  if (!tensors || !out || count < 1) return gr_error(LSGD_EINVAL, fn, "tensors or out is NULL, or count below 1");
  if (G < 1 || G > 65535 || (int64_t)count * G > (1 << 22))
    return gr_error(LSGD_EINVAL, fn, "at least 1 and at most 65535 workers, at most 2^22 tensors of all workers");
  int places = 0;
  int64_t bytes = 0, out_bytes = 0;  // of a worker
  for (int i = 0; i < count; ++i) {
    const lsgd_tensor& t = tensors[i];
    const auto bad_type = [](int type) { return type != LSGD_FP32 && type != LSGD_BF16; };
    const auto bad_place = [&](const void* p, int64_t gs, int type) {
      return (t.n && !p) || misaligned(p, size_of(type)) ||
             (G > 1 && (gs < t.n || gs > ((int64_t)1 << 50) / G));
    };
    if (t.n < 0 || t.n > ((int64_t)1 << 40)) return gr_error(LSGD_EINVAL, fn, "a tensor has 0 to 2^40 values of a worker");
    if (bad_type(t.g_type) || (t.out && bad_type(t.out_type))) return gr_error(LSGD_EINVAL, fn, "types are LSGD_FP32 or LSGD_BF16");
    if (bad_place(t.g, t.g_gs, t.g_type) || (t.out && bad_place(t.out, t.out_gs, t.out_type)))
      return gr_error(LSGD_EINVAL, fn, "a tensor is NULL, not aligned to its element, or its workers' strides below n or above 2^50");
    if (t.n) places |= t.out ? 1 : 2;
    bytes += t.n * size_of(t.g_type);
    out_bytes += t.n * size_of(t.out ? t.out_type : t.g_type);
    if (bytes > ((int64_t)1 << 42)) return gr_error(LSGD_EINVAL, fn, "at most 2^42 bytes of a worker");
  }
  if (places == 3) return gr_error(LSGD_EINVAL, fn, "either every tensor has an out or none has");
  try {
    auto* l = new lsgd_tensors;
    try {
      l->G = G, l->places = places == 1;
      for (int i = 0; i < count; ++i)
        if (tensors[i].n) l->list.push_back(tensors[i]);
      const auto types = [&](const lsgd_tensor& t) { return 2 * (t.g_type == LSGD_BF16) + (out_type(t, l->places) == LSGD_BF16); };
      std::stable_sort(l->list.begin(), l->list.end(), [&](const lsgd_tensor& x, const lsgd_tensor& y) { return types(x) < types(y); });
      for (size_t i = 0, from = 0; i < l->list.size(); ++i)
        if (i == 0 || i - from == kMany || types(l->list[i]) != types(l->list[i - 1])) {
          l->launches.push_back({from = i, i, types(l->list[i]) >= 2, (types(l->list[i]) & 1) != 0, {}});
        }
      for (size_t i = 0; i < l->launches.size(); ++i)
        l->launches[i].to = i + 1 < l->launches.size() ? l->launches[i + 1].from : l->list.size();
      // One launch, a worker to a cluster, where it takes one and the CTAs have little to read each: as many as get 16 KB or two
      // tensors to a warp; not where that makes more than two to an SM (64 workers of 70 KB, 320 CTAs: norm 7.2 us, 5.1 in two
      // launches; 300 of 16 KB, 300 CTAs: 4.3 and 8.6).
      if (l->launches.size() == 1 && bytes <= kShare * kMaxCluster) {
        const int64_t want = std::max<int64_t>(bytes / kMinShare, (int64_t)l->list.size() / (kClusterThreads / 16)) + 1;
        l->cluster = (int)std::max<int64_t>(1, std::min<int64_t>(kMaxCluster, want));
        if ((int64_t)l->cluster * G > 2 * kNumSMs) l->cluster = 0;
        l->clip_once = l->cluster && bytes + out_bytes <= kClipOnce;
      }
      // Pieces small enough for every warp to have one, up to 4096 bytes (8 vectors a lane).
      const int64_t warps = l->cluster ? l->cluster * (kClusterThreads / 32) : std::max<int64_t>(1, (int64_t)kNumSMs * 4 * kWarps / G);
      l->piece = kMaxPiece;
      while (l->piece > kMinPiece && bytes / l->piece < warps) l->piece /= 2;
      uint32_t at = 0;
      for (const lsgd_tensor& t : l->list) {
        l->first.push_back(at);
        at += (uint32_t)((t.n * size_of(t.g_type) + l->piece - 1) / l->piece);
        l->lo = std::min(l->lo, reinterpret_cast<uintptr_t>(t.g));
        l->hi = std::max(l->hi, end_of(t.g, t.n, t.g_gs, t.g_type, G));
        if (l->places) {
          l->lo = std::min(l->lo, reinterpret_cast<uintptr_t>(t.out));
          l->hi = std::max(l->hi, end_of(t.out, t.n, t.out_gs, t.out_type, G));
        }
      }
      l->first.push_back(at);
      const int64_t most = std::max<int64_t>(1, (int64_t)kNumSMs * 4 / G);
      l->blocks = (int)std::min<int64_t>(most, ((int64_t)at + kWarps - 1) / kWarps);
      for (auto& launch : l->launches)
        with_size(launch.to - launch.from, [&](auto max) {
          fill<decltype(max)::value>(launch, *l);
          return 0;
        });
      l->overlap = clip_overlaps(*l);
    } catch (...) {
      delete l;
      throw;
    }
    *out = l;
  } catch (...) {  // (what the containers throw)
    return gr_error(LSGD_ENOMEM, fn, "out of host memory");
  }
  return LSGD_OK;
}

void lsgd_tensors_destroy(lsgd_tensors* list) { delete list; }

lsgd_status lsgd_gradient_workspace(const lsgd_tensors* list, size_t* bytes) {
  using namespace lsgd;
  if (!list || !bytes) return gr_error(LSGD_EINVAL, "lsgd_gradient_workspace", "a pointer is NULL");
  *bytes = gr_workspace(*list);
  return LSGD_OK;
}

lsgd_status lsgd_gradient_norm(const lsgd_tensors* list, float* norm, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace lsgd;
  const char* fn = "lsgd_gradient_norm";
  const char* bad = norm_error(list, norm, workspace, workspace_bytes);
  if (bad) return gr_error(LSGD_EINVAL, fn, bad);
  const cudaError_t e = norm_and_clip(*list, norm, 0.f, static_cast<double*>(workspace), (cudaStream_t)stream);
  return e == cudaSuccess ? LSGD_OK : gr_error(LSGD_ECUDA, fn, cudaGetErrorString(e));
}

lsgd_status lsgd_gradient_clip(const lsgd_tensors* list, float* norm, float max_norm, void* workspace, size_t workspace_bytes,
                               void* stream) {
  using namespace lsgd;
  const char* fn = "lsgd_gradient_clip";
  const char* bad = norm_error(list, norm, workspace, workspace_bytes);
  if (!bad && !(max_norm > 0.f && max_norm < INFINITY)) bad = "max_norm must be positive and finite";
  if (!bad && list->overlap) bad = "what would be written overlaps another tensor of the list";
  if (bad) return gr_error(LSGD_EINVAL, fn, bad);
  const cudaError_t e = norm_and_clip(*list, norm, max_norm, static_cast<double*>(workspace), (cudaStream_t)stream);
  return e == cudaSuccess ? LSGD_OK : gr_error(LSGD_ECUDA, fn, cudaGetErrorString(e));
}

lsgd_status lsgd_clipped_update(float* w, float* u, int64_t w_gs, const void* g, int g_type, int64_t g_gs, uint16_t* Wb, int G,
                                int64_t n, const float* norm, float max_norm, float lr, float momentum, int nesterov,
                                float weight_decay, int64_t decay_end, void* stream) {
  using namespace lsgd;
  const char* fn = "lsgd_clipped_update";
  const char* bad = nullptr;
  const int gz = size_of(g_type);
  if (G < 1 || G > 65535 || n < 0 || n > ((int64_t)1 << 40)) bad = "at least 1 and at most 65535 workers, 0 to 2^40 values";
  else if (g_type != LSGD_FP32 && g_type != LSGD_BF16) bad = "types are LSGD_FP32 or LSGD_BF16";
  else if (n && (!w || !g || !norm || (momentum != 0.f && !u))) bad = "a pointer is NULL (u may be only without momentum)";
  else if (G > 1 && (w_gs < n || g_gs < n || w_gs > ((int64_t)1 << 50) / G || g_gs > ((int64_t)1 << 50) / G))
    bad = "w_gs and g_gs must be at least n (and addresses fit 64 bits)";
  else if (misaligned(w, 4) || misaligned(u, 4) || misaligned(g, gz) || misaligned(Wb, 2) || misaligned(norm, 4))
    bad = "a pointer is not aligned to its element";
  else if (!(max_norm > 0.f && max_norm < INFINITY)) bad = "max_norm must be positive and finite";
  else if (decay_end < 0) bad = "decay_end must not be negative";
  if (bad) return gr_error(LSGD_EINVAL, fn, bad);
  if (n == 0) return LSGD_OK;
  const float* mom = momentum != 0.f ? u : nullptr;
  const auto values = [&](const void* p, int64_t gs, int z) { return Blocks(p, (size_t)n * z, gs, G, z); };
  // (blocks_meet takes one block or equal strides: tensors of other strides or sizes of values count as wholes)
  const auto whole = [&](const void* p, int64_t gs, int z) { return Blocks(p, (size_t)((G - 1) * gs + n) * z); };
  const Blocks W = values(w, w_gs, 4), U = values(mom, w_gs, 4), S = values(Wb, w_gs, 2), N(norm, 4 * (size_t)G);
  const bool same = g_type != LSGD_BF16 && g_gs == w_gs;
  const Blocks mine = same ? values(g, g_gs, 4) : whole(g, g_gs, gz);
  const auto g_meets = [&](const Blocks& exact, const Blocks& all) { return blocks_meet(same ? exact : all, mine); };
  if (blocks_meet(W, U) || blocks_meet(N, W) || blocks_meet(N, U) || blocks_meet(N, S) || g_meets(W, whole(w, w_gs, 4)) ||
      g_meets(U, whole(mom, w_gs, 4)) ||
      any_overlap({whole(Wb, w_gs, 2)}, {whole(w, w_gs, 4), whole(mom, w_gs, 4), whole(g, g_gs, gz)}))
    return gr_error(LSGD_EINVAL, fn, "tensors overlap");
  UpdateArgs a{w, u, g, Wb, w_gs, g_gs, n, decay_end, norm, max_norm, lr, momentum, weight_decay};
  const bool wide = !misaligned(w, 16) && !(momentum != 0.f && misaligned(u, 16)) && !misaligned(g, 4 * gz) && !misaligned(Wb, 8) &&
                    (G == 1 || (w_gs % 4 == 0 && g_gs % 4 == 0));
  const cudaStream_t st = (cudaStream_t)stream;
  const cudaError_t e = g_type == LSGD_BF16 ? clipped_rule<true>(a, G, nesterov, wide, st) : clipped_rule<false>(a, G, nesterov, wide, st);
  return e == cudaSuccess ? LSGD_OK : gr_error(LSGD_ECUDA, fn, cudaGetErrorString(e));
}

}  // extern "C"
