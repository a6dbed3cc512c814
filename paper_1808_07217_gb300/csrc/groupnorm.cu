// Group normalisation with an activation over channels-last tensors, forward and backward, for G workers of B
// images each.  Unlike the per-worker BatchNorm of Sec. A.4 it keeps no statistics that differ from worker to worker.
//
// For image n, group q (D = C / groups channels) and its P x D values x:
//   mean = sum x / (P D),  rstd = 1 / sqrt(sum (x - mean)^2 / (P D) + eps),  xh = (x - mean) rstd,
//   y = act(gamma xh + beta).
// Backward, with dz = dy act'(.), m1 and m2 the group's means of gamma dz and gamma dz xh:
//   dgamma = sum dz xh,  dbeta = sum dz (over the worker's images and positions),
//   dx = rstd (gamma dz - m1 - xh m2).
//
// Both are bound by memory: x read and y written once, and x, dy (for ReLU y) read and dx written once, where an image stays
// on chip (the resident form below), one more read of the inputs where it does not (the split form).  A thread owns V
// neighbouring channels (a vector of up to 16 bytes) and walks down the positions, so that its parameters and channel sums
// stay in registers whatever the group width.
#include <algorithm>
#include <atomic>
#include <string>
#include <type_traits>

#include "../../include/lsgd.h"
#include "common.cuh"
#include "lsgd_internal.h"
#include "operands.h"
#include "tc_ptx.cuh"
#include "vectors.cuh"

namespace lsgd {

__device__ int g_norm_timeout = 0;
static std::atomic<bool> g_norm_used{false};  // the flag is read only once a call has been made

namespace {

struct GnArgs {
  const void *x, *y, *dy;
  void* out;  // y (forward), dx (backward)
  const float *gamma, *beta;
  int64_t par_gs;
  float *mean, *rstd;
  float* part;    // split form: per (image, split, channel) pairs; backward's channel sums
  float* sums;    // split backward: per (image, channel) pairs
  float* m12;     // split backward: per (image, group) pairs (m1, m2)
  float *dgamma, *dbeta;
  int B, P, C, groups, D, act;
  int S;          // position ranges of an image
  int rows;       // positions of a range
  int64_t N;
  float eps;
  int cl, sub;    // resident form: CTAs per image; channels summed in a thread
  int stages, slab, slab_y;  // its pipeline: images ahead; bytes of an image of x and of dy (or y)
};

constexpr long long kWaitCycles = 4000000000LL;  // ~2 s at 2 GHz

__device__ __forceinline__ bool wait_full(uint64_t* bar, uint32_t parity) {
  if (mbar_try_wait(bar, parity)) return true;
  const long long t0 = clock64();
  while (!mbar_try_wait(bar, parity))
    if (clock64() - t0 > kWaitCycles) {
      atomicExch(&g_norm_timeout, 1);
      return false;
    }
  return true;
}
__device__ __forceinline__ void bulk_load(void* dst, const void* src, int bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
               "l"(src), "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}

// ---- split form: any size, three launches ----
//
// The sums over ranges of an image's positions, their merge, and a second pass from the statistics.  Forward of 8 images of 127 x
// 129 x 320 in bf16 with SiLU: 55 us (about 20, 5 and 28; 168 MB at least, 3.1 TB/s): the merge's latency, the second read of x,
// most of which L2 no longer holds, and SiLU's two special functions a value.  One cooperative launch that keeps a third of x
// in shared memory between the passes took 57.6: its two ends and the wait between them cost what the kept third saves.

constexpr int kSplitThreads = 256;

// (count, mean, M2) <- merged with (nb, mb, qb)
__device__ __forceinline__ void chan(float& n, float& m, float& q, float nb, float mb, float qb) {
  if (nb == 0.f) return;
  const float t = n + nb, w = __fdividef(nb, t), d = mb - m;  // (the weight's last bits scale d only)
  m = fmaf(d, w, m);
  q += fmaf(d * d, n * w, qb);
  n = t;
}

// Per range and channel: forward (mean, sum of squared deviations), backward (sum dz, sum dz xh).
template <typename XT, typename YT, int V, bool BWD>
__global__ void __launch_bounds__(kSplitThreads) gn_partial_kernel(const GnArgs a, int tx_n, int ty_n) {
  pdl_begin();
  const int tx = threadIdx.x % tx_n, ty = threadIdx.x / tx_n;
  const int c0 = (blockIdx.y * tx_n + tx) * V;
  const bool on = ty < ty_n && c0 < a.C;
  const int n = blockIdx.x / a.S, s = blockIdx.x % a.S;
  const int p0 = s * a.rows, p1 = min(a.P, p0 + a.rows);
  __shared__ float red[kSplitThreads * V * 2];
  __shared__ float rc[kSplitThreads];
  float s0[V], s1[V];
  float cnt = 0.f;
#pragma unroll
  for (int j = 0; j < V; ++j) s0[j] = s1[j] = 0.f;
  if (on) {
    const int64_t base = (int64_t)n * a.P * a.C + c0;
    const XT* x = static_cast<const XT*>(a.x) + base;
    const int64_t step = (int64_t)ty_n * a.C;
    if constexpr (!BWD) {
      // Segments: sums of the deviations from the first U values' mean, and of their squares, merged into the running
      // moments by Chan et al.'s formula.  The pivot is far from the segment's mean only if one of its U values
      // is, and then that value's square in the sums bounds what the difference loses.
      constexpr int U = 8;
      int p = p0 + ty;
      const int most = segment((p1 - p + ty_n - 1) / ty_n);
      const XT* at = x + (int64_t)p * a.C;
      while (p < p1) {
        const int k = min(most, (p1 - p + ty_n - 1) / ty_n);  // positions of the segment
        float pivot[V], d0[V], d1[V];
#pragma unroll
        for (int j = 0; j < V; ++j) d0[j] = d1[j] = 0.f;
        for (int b = 0; b < k; b += U) {
          Vec<XT, V> r[U];
#pragma unroll
          for (int i = 0; i < U; ++i)
            if (b + i < k) r[i].load(at + i * step);
          if (b == 0) {
#pragma unroll
            for (int j = 0; j < V; ++j) pivot[j] = 0.f;
#pragma unroll
            for (int i = 0; i < U; ++i)
              if (i < k) {
                float v[V];
                r[i].floats(v);
#pragma unroll
                for (int j = 0; j < V; ++j) pivot[j] += v[j];
              }
            const float inv = 1.f / min(k, U);
#pragma unroll
            for (int j = 0; j < V; ++j) pivot[j] *= inv;
          }
#pragma unroll
          for (int i = 0; i < U; ++i)
            if (b + i < k) {
              float v[V];
              r[i].floats(v);
#pragma unroll
              for (int j = 0; j < V; ++j) {
                const float d = v[j] - pivot[j];
                d0[j] += d;
                d1[j] = fmaf(d, d, d1[j]);
              }
            }
          at += U * step;
        }
        p += k * ty_n;
        at = x + (int64_t)p * a.C;
        const float kf = (float)k, inv = 1.f / kf, w = kf / (cnt + kf), cw = cnt * w;
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float e = d0[j] * inv, d = pivot[j] + e - s0[j];
          s0[j] = fmaf(d, w, s0[j]);
          s1[j] += fmaf(d * d, cw, fmaxf(fmaf(-e, d0[j], d1[j]), 0.f) + (d1[j] != d1[j] ? d1[j] : 0.f));
        }
        cnt += kf;
      }
    } else {
      const YT* dy = static_cast<const YT*>(a.dy) + base;
      const YT* y = static_cast<const YT*>(a.y) + base;
      const bool relu = a.act == LSGD_ACT_RELU, silu = a.act == LSGD_ACT_SILU;
      float ga[V], be[V], mu[V], rs[V];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int64_t pc = (int64_t)(n / a.B) * a.par_gs + c0 + j;
        const int64_t pg = (int64_t)n * a.groups + (c0 + j) / a.D;
        ga[j] = a.gamma[pc];
        be[j] = a.beta[pc];
        mu[j] = a.mean[pg];
        rs[j] = a.rstd[pg];
      }
      constexpr int U = V >= 8 ? 2 : 4;
      int p = p0 + ty;
      const int span = segment((p1 - p + ty_n - 1) / ty_n) * ty_n;  // (a multiple of U positions)
      bool more = false;  // earlier segments' sums stand in this thread's place of red
      while (p < p1) {
        if (more) {
#pragma unroll
          for (int j = 0; j < V; ++j) s0[j] = s1[j] = 0.f;
        }
        for (const int end = min(p1, p + span); p < end; p += U * ty_n) {
          Vec<XT, V> rx[U];
          Vec<YT, V> rd[U], ry[U];
#pragma unroll
          for (int i = 0; i < U; ++i)
            if (p + i * ty_n < p1) {
              const int64_t at = (int64_t)(p + i * ty_n) * a.C;
              rx[i].load(x + at);
              rd[i].load(dy + at);
              if (relu) ry[i].load(y + at);
            }
#pragma unroll
          for (int i = 0; i < U; ++i)
            if (p + i * ty_n < p1) {
              float xv[V], dv[V], yv[V];
              rx[i].floats(xv);
              rd[i].floats(dv);
              if (relu) ry[i].floats(yv);
#pragma unroll
              for (int j = 0; j < V; ++j) {
                const float xh = (xv[j] - mu[j]) * rs[j];
                float dz = dv[j];
                if (relu) dz = yv[j] > 0.f ? dz : 0.f;
                if (silu) {
                  const float z = fmaf(xh, ga[j], be[j]), sg = sigmoid<sizeof(XT) == 4 ? kExact : kSums>(z);
                  dz *= sg * fmaf(z, 1.f - sg, 1.f);
                }
                s0[j] += dz;
                s1[j] = fmaf(dz, xh, s1[j]);
              }
            }
        }
        if (more || p < p1) {
#pragma unroll
          for (int j = 0; j < V; ++j) {
            float &t0 = red[2 * j * kSplitThreads + threadIdx.x], &t1 = red[(2 * j + 1) * kSplitThreads + threadIdx.x];
            if (more) s0[j] += t0, s1[j] += t1;
            t0 = s0[j], t1 = s1[j];
          }
          more = true;
        }
      }
    }
  }
  // the rows of threads, one after another in thread 0's row
#pragma unroll
  for (int j = 0; j < V; ++j) {
    red[2 * j * kSplitThreads + threadIdx.x] = s0[j];
    red[(2 * j + 1) * kSplitThreads + threadIdx.x] = s1[j];
  }
  rc[threadIdx.x] = cnt;
  __syncthreads();
  // halves of the rows are merged until one is left
  for (int half = 1; half < ty_n; half *= 2) {
    const int other = ty + half;
    if (on && ty % (2 * half) == 0 && other < ty_n) {
      const int o = threadIdx.x + half * tx_n;
      const float oc = rc[o];
      const float w = BWD || oc == 0.f ? 0.f : oc / (cnt + oc), cw = cnt * w;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float b0 = red[2 * j * kSplitThreads + o], b1 = red[(2 * j + 1) * kSplitThreads + o];
        if constexpr (BWD) {
          s0[j] += b0;
          s1[j] += b1;
        } else if (oc > 0.f) {
          const float d = b0 - s0[j];
          s0[j] = fmaf(d, w, s0[j]);
          s1[j] += fmaf(d * d, cw, b1);
        }
        red[2 * j * kSplitThreads + threadIdx.x] = s0[j];
        red[(2 * j + 1) * kSplitThreads + threadIdx.x] = s1[j];
      }
      cnt += oc;
      rc[threadIdx.x] = cnt;
    }
    __syncthreads();
  }
  if (on && ty == 0) {
    float* out = a.part + (((int64_t)n * a.S + s) * a.C + c0) * 2;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      out[2 * j] = s0[j];
      out[2 * j + 1] = s1[j];
    }
  }
}

// The forward's first pass where the vectors are of 16 bytes: a range's positions lie one behind another in memory, and bulk
// copies bring kRingRows of them to every row of threads at a time, two to four such chunks ahead, so that the loads do not wait
// for the sums.  (84 MB of 8 images: 20 us, 26 with the kernel above, whose loads stop while a batch is added up; the whole call
// 57 and 62.5.)  Other vectors take that kernel: bulk copies need 16-byte rows.
constexpr int kRingRows = 4;
constexpr size_t kRingSmem = 112 * 1024;  // two CTAs to an SM

template <typename XT, int V>
__global__ void __launch_bounds__(512, 2) gn_ring_partial_kernel(const GnArgs a) {
  constexpr int U = kRingRows;
  extern __shared__ __align__(16) uint8_t raw[];
  const int tx = threadIdx.x, ty = threadIdx.y, c0 = tx * V, tid = ty * blockDim.x + tx;
  const int tx_n = blockDim.x, ty_n = blockDim.y, chunk = ty_n * U, chunk_bytes = chunk * a.C * (int)sizeof(XT);
  uint64_t* full = reinterpret_cast<uint64_t*>(raw);
  uint8_t* ring = raw + 64;
  const int threads = tx_n * ty_n;
  float* red = reinterpret_cast<float*>(ring + a.stages * chunk_bytes);  // [2 V][threads]: the running moments
  float* rc = red + threads * V * 2;                                     // [threads]: their counts
  const int n = blockIdx.x / a.S, s = blockIdx.x % a.S;
  const int p0 = s * a.rows, cnt = min(a.P, p0 + a.rows) - p0, chunks = (cnt + chunk - 1) / chunk;
  const XT* x = static_cast<const XT*>(a.x) + ((int64_t)n * a.P + p0) * a.C;
  auto fetch = [&](int k, int b) {
    const int bytes = min(chunk, cnt - k * chunk) * a.C * (int)sizeof(XT);
    mbar_expect_tx(&full[b], bytes);
    bulk_load(ring + b * chunk_bytes, x + (int64_t)k * chunk * a.C, bytes, &full[b]);
  };
  if (tid == 0) {
    for (int b = 0; b < a.stages; ++b) mbar_init(&full[b], 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  __syncthreads();
  pdl_begin();
  if (tid == 0)
    for (int b = 0; b < min(a.stages, chunks); ++b) fetch(b, b);
  float* run = red + tid;
#pragma unroll
  for (int j = 0; j < 2 * V; ++j) run[j * threads] = 0.f;
  float total = 0.f, pivot[V], d0[V], d1[V];
  const int most = segment(chunks * U) / U;  // the chunks of a segment
  // a segment ends: its sums, of deviations from the pivot, into the running moments
  auto merge = [&](int k) {
    if (k == 0) return;
    const float kf = (float)k, inv = 1.f / kf, w = kf / (total + kf), cw = total * w;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      float& mean = run[2 * j * threads];
      const float m = mean, e = d0[j] * inv, d = pivot[j] + e - m;
      mean = fmaf(d, w, m);
      run[(2 * j + 1) * threads] += fmaf(d * d, cw, fmaxf(fmaf(-e, d0[j], d1[j]), 0.f) + (d1[j] != d1[j] ? d1[j] : 0.f));
    }
    total += kf;
  };
  int b = 0, k_seg = 0, next = 0;
  uint32_t ph = 0;
  for (int k = 0; k < chunks; ++k) {
    const bool ok = wait_full(&full[b], ph);
    const int have = max(0, min(U, (cnt - k * chunk - ty + ty_n - 1) / ty_n));  // of this thread's U positions
    Vec<XT, V> r[U];
    const uint8_t* from = ring + b * chunk_bytes + (ty * a.C + c0) * (int)sizeof(XT);
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (i < have) r[i].load_shared(from + i * ty_n * a.C * (int)sizeof(XT));
    if (__syncthreads_or(!ok)) {  // a wait ran out: the copies under way first
      if (tid == 0)
        for (int c = 0; c < a.stages; ++c) wait_full(&full[c], ph ^ (c < b ? 1 : 0));
      return;
    }
    if (tid == 0 && k + a.stages < chunks) fetch(k + a.stages, b);
    if (++b == a.stages) b = 0, ph ^= 1;
    if (k == next) {
      merge(k_seg);
      k_seg = 0;
      next += most;
      const float first = 1.f / max(have, 1);
#pragma unroll
      for (int j = 0; j < V; ++j) pivot[j] = d0[j] = d1[j] = 0.f;
#pragma unroll
      for (int i = 0; i < U; ++i)
        if (i < have) {
          float v[V];
          r[i].floats(v);
#pragma unroll
          for (int j = 0; j < V; ++j) pivot[j] = fmaf(v[j], first, pivot[j]);
        }
    }
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (i < have) {
        float v[V];
        r[i].floats(v);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float d = v[j] - pivot[j];
          d0[j] += d;
          d1[j] = fmaf(d, d, d1[j]);
        }
      }
    k_seg += have;
  }
  merge(k_seg);
  rc[tid] = total;
  __syncthreads();
  // halves of the rows are merged until one is left
  for (int half = 1; half < ty_n; half *= 2) {
    if (ty % (2 * half) == 0 && ty + half < ty_n) {
      const float* o = run + half * tx_n;
      const float oc = rc[tid + half * tx_n];
      if (oc > 0.f) {
        const float w = oc / (total + oc), cw = total * w;
#pragma unroll
        for (int j = 0; j < V; ++j) {
          float& mean = run[2 * j * threads];
          const float d = o[2 * j * threads] - mean;
          mean = fmaf(d, w, mean);
          run[(2 * j + 1) * threads] += fmaf(d * d, cw, o[(2 * j + 1) * threads]);
        }
        total += oc;
        rc[tid] = total;
      }
    }
    __syncthreads();
  }
  if (ty == 0) {
    float* out = a.part + (((int64_t)n * a.S + s) * a.C + c0) * 2;
#pragma unroll
    for (int j = 0; j < 2 * V; ++j) out[j] = run[j * threads];
  }
}

// Forward: a block per (image, group) merges its ranges' channels into mean and rstd, about eight to a thread where 1024 threads
// are enough, one after another, 64 of them at a time.  A chain of latencies: 4.7 us for 256 blocks of 38 x 10 values, 20.5 for 4
// of 152 x 512.
__global__ void __launch_bounds__(1024) gn_stats_merge_kernel(const GnArgs a) {
  pdl_begin();
  const int n = blockIdx.x / a.groups, q = blockIdx.x % a.groups, threads = blockDim.x;
  const float2* part = reinterpret_cast<const float2*>(a.part) + (int64_t)n * a.S * a.C + q * a.D;
  float cn = 0.f, cm = 0.f, cq = 0.f;
  // range by range where a group has many channels, else threads / D ranges at a time
  const int dw = min(a.D, threads), lanes = threads / dw;
  const int d0 = threadIdx.x % dw, s0 = threadIdx.x / dw;
  if (s0 < lanes) {
    constexpr int U = 8;  // loads before the first merge
    float sn = 0.f, sm = 0.f, sq = 0.f;  // earlier segments' moments
    const int batches = 64 / min(U, (a.S + lanes - 1) / lanes);  // of a segment
    int left = batches;
    for (int d = d0; d < a.D; d += dw)
      for (int s = s0; s < a.S; s += U * lanes) {
        float2 v[U];
#pragma unroll
        for (int i = 0; i < U; ++i)
          if (s + i * lanes < a.S) v[i] = part[(int64_t)(s + i * lanes) * a.C + d];
        if (--left < 0) {
          chan(sn, sm, sq, cn, cm, cq);
          cn = cm = cq = 0.f;
          left = batches - 1;
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
          const int r = s + i * lanes;
          if (r < a.S) chan(cn, cm, cq, (float)(min(a.P, (r + 1) * a.rows) - r * a.rows), v[i].x, v[i].y);
        }
      }
    if (sn > 0.f) chan(cn, cm, cq, sn, sm, sq);
  }
  auto warp_merge = [&]() {
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      const float nb = __shfl_xor_sync(~0u, cn, o), mb = __shfl_xor_sync(~0u, cm, o), qb = __shfl_xor_sync(~0u, cq, o);
      chan(cn, cm, cq, nb, mb, qb);
    }
  };
  __shared__ float red[3][32];
  warp_merge();
  const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (lane == 0) red[0][w] = cn, red[1][w] = cm, red[2][w] = cq;
  __syncthreads();
  if (w == 0) {
    const bool have = lane < threads / 32;
    cn = have ? red[0][lane] : 0.f, cm = have ? red[1][lane] : 0.f, cq = have ? red[2][lane] : 0.f;
    warp_merge();
    if (lane == 0) {
      a.mean[blockIdx.x] = cm;
      a.rstd[blockIdx.x] = __frsqrt_rn(cq / cn + a.eps);
    }
  }
}

// Backward: per image and `per` groups of it, the ranges' channel sums added up (several threads to a channel where the
// channels are fewer than the threads), and the groups' m1 and m2.  4 blocks of 152 x 512 values: 13 us, 46 with 256 threads.
__global__ void __launch_bounds__(1024) gn_sums_merge_kernel(const GnArgs a, int per) {
  pdl_begin();
  __shared__ float2 red[1024];
  const int n = blockIdx.x, q0 = blockIdx.y * per, q1 = min(a.groups, q0 + per), threads = blockDim.x;
  float2* sums = reinterpret_cast<float2*>(a.sums) + (int64_t)n * a.C;
  const float2* part = reinterpret_cast<const float2*>(a.part) + (int64_t)n * a.S * a.C + q0 * a.D;
  const int width = (q1 - q0) * a.D, dw = min(width, threads), lanes = threads / dw;
  const int d0 = threadIdx.x % dw, s0 = threadIdx.x / dw;
  auto sum = [&](int d, int from, int step) {
    float2 t = make_float2(0.f, 0.f);
#pragma unroll 8
    for (int s = from; s < a.S; s += step) {
      const float2 v = part[(int64_t)s * a.C + d];
      t.x += v.x;
      t.y += v.y;
    }
    return t;
  };
  if (lanes == 1) {
    for (int d = threadIdx.x; d < width; d += threads) sums[q0 * a.D + d] = sum(d, 0, 1);
  } else {
    if (s0 < lanes) red[threadIdx.x] = sum(d0, s0, lanes);
    __syncthreads();
    if (s0 == 0) {
      float2 t = red[d0];
      for (int k = 1; k < lanes; ++k) t.x += red[k * dw + d0].x, t.y += red[k * dw + d0].y;
      sums[q0 * a.D + d0] = t;
    }
  }
  __syncthreads();
  const int lane = threadIdx.x & 31;
  const float inv = 1.f / ((float)a.P * (float)a.D);
  const float* gamma = a.gamma + (int64_t)(n / a.B) * a.par_gs;
  for (int q = q0 + (threadIdx.x >> 5); q < q1; q += threads / 32) {
    float2 t = make_float2(0.f, 0.f);
    for (int from = lane; from < a.D; from += 32 * 64) {  // 64 channels of a lane at a time
      float2 some = make_float2(0.f, 0.f);
      const int end = min(a.D, from + 32 * 64);
#pragma unroll 4
      for (int d = from; d < end; d += 32) {
        const float ga = gamma[q * a.D + d];
        const float2 v = sums[q * a.D + d];
        some.x = fmaf(ga, v.x, some.x);
        some.y = fmaf(ga, v.y, some.y);
      }
      t.x += some.x;
      t.y += some.y;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      t.x += __shfl_xor_sync(~0u, t.x, o);
      t.y += __shfl_xor_sync(~0u, t.y, o);
    }
    if (lane == 0) reinterpret_cast<float2*>(a.m12)[(int64_t)n * a.groups + q] = make_float2(t.x * inv, t.y * inv);
  }
}

// The second pass: y or dx from the statistics.  The ranges in the opposite order: the last that the first pass read are
// still in L2.
template <typename XT, typename YT, int V, bool BWD>
__global__ void __launch_bounds__(kSplitThreads, BWD ? 2 : 4) gn_apply_kernel(const GnArgs a, int tx_n, int ty_n) {
  pdl_begin();
  const int tx = threadIdx.x % tx_n, ty = threadIdx.x / tx_n;
  const int c0 = (blockIdx.y * tx_n + tx) * V;
  if (ty >= ty_n || c0 >= a.C) return;
  const int block = gridDim.x - 1 - blockIdx.x, n = block / a.S;
  const int p0 = (block % a.S) * a.rows, p1 = min(a.P, p0 + a.rows);
  const int64_t base = (int64_t)n * a.P * a.C + c0;
  const XT* x = static_cast<const XT*>(a.x) + base;
  const bool relu = a.act == LSGD_ACT_RELU, silu = a.act == LSGD_ACT_SILU;
  float ga[V], be[V], mu[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int64_t pc = (int64_t)(n / a.B) * a.par_gs + c0 + j, pg = (int64_t)n * a.groups + (c0 + j) / a.D;
    ga[j] = a.gamma[pc];
    be[j] = a.beta[pc];
    mu[j] = a.mean[pg];
  }
  if constexpr (!BWD) {
    YT* out = static_cast<YT*>(a.out) + base;
#pragma unroll
    for (int j = 0; j < V; ++j) ga[j] *= a.rstd[(int64_t)n * a.groups + (c0 + j) / a.D];
    constexpr int U = 4, kKind = sizeof(YT) == 4 ? kExact : kFast;
    with_act(a.act, [&](auto act) {
      for (int p = p0 + ty; p < p1; p += U * ty_n) {
        Vec<XT, V> r[U];
#pragma unroll
        for (int i = 0; i < U; ++i)
          if (p + i * ty_n < p1) r[i].load(x + (int64_t)(p + i * ty_n) * a.C);
#pragma unroll
        for (int i = 0; i < U; ++i)
          if (p + i * ty_n < p1) {
            float v[V];
            r[i].floats(v);
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = activate<kKind, decltype(act)::value>(fmaf(v[j] - mu[j], ga[j], be[j]));
            Vec<YT, V> o;
            o.set(v);
            o.stream(out + (int64_t)(p + i * ty_n) * a.C);
          }
      }
    });
  } else {
    const YT* dy = static_cast<const YT*>(a.dy) + base;
    const YT* y = static_cast<const YT*>(a.y) + base;
    XT* out = static_cast<XT*>(a.out) + base;
    float rs[V], m1[V], m2[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int64_t pg = (int64_t)n * a.groups + (c0 + j) / a.D;
      rs[j] = a.rstd[pg];
      m1[j] = a.m12[2 * pg] * rs[j];
      m2[j] = a.m12[2 * pg + 1] * rs[j];
    }
    constexpr int U = V >= 8 ? 2 : 4;
    for (int p = p0 + ty; p < p1; p += U * ty_n) {
      Vec<XT, V> rx[U];
      Vec<YT, V> rd[U], ry[U];
#pragma unroll
      for (int i = 0; i < U; ++i)
        if (p + i * ty_n < p1) {
          const int64_t at = (int64_t)(p + i * ty_n) * a.C;
          rx[i].load(x + at);
          rd[i].load(dy + at);
          if (relu) ry[i].load(y + at);
        }
#pragma unroll
      for (int i = 0; i < U; ++i)
        if (p + i * ty_n < p1) {
          float xv[V], dv[V], yv[V];
          rx[i].floats(xv);
          rd[i].floats(dv);
          if (relu) ry[i].floats(yv);
#pragma unroll
          for (int j = 0; j < V; ++j) {
            const float xh = (xv[j] - mu[j]) * rs[j];
            float dz = dv[j];
            if (relu) dz = yv[j] > 0.f ? dz : 0.f;
            if (silu) {
              const float z = fmaf(xh, ga[j], be[j]), sg = sigmoid<sizeof(XT) == 4 ? kExact : kFast>(z);
              dz *= sg * fmaf(z, 1.f - sg, 1.f);
            }
            xv[j] = fmaf(ga[j] * rs[j], dz, -m1[j]) - xh * m2[j];
          }
          Vec<XT, V> o;
          o.set(xv);
          o.stream(out + (int64_t)(p + i * ty_n) * a.C);
        }
    }
  }
}

// dgamma and dbeta of worker g: the sums of its `rows` rows of channel pairs (sum dz, sum dz xh), a fixed order.
__global__ void __launch_bounds__(1024, 2) gn_param_grad_kernel(const float2* sums, int64_t rows, int C, int64_t par_gs,
                                                             float* dgamma, float* dbeta) {
  pdl_begin();
  const int cx = threadIdx.x & 15, ry = threadIdx.x >> 4;
  const int c = blockIdx.x * 16 + cx;
  const int64_t g = blockIdx.y;
  float2 t = make_float2(0.f, 0.f);
  if (c < C) {
    const int span = 64 * segment((int)((rows + 63) / 64));  // the rows of a segment of this thread's additions
    for (int64_t from = ry; from < rows; from += span) {
      float2 some = make_float2(0.f, 0.f);
      const int n = (int)min((int64_t)span, rows - from);
      const float2* at = sums + (g * rows + from) * C + c;
#pragma unroll 8
      for (int r = 0; r < n; r += 64) {
        const float2 v = at[(int64_t)r * C];
        some.x += v.x;
        some.y += v.y;
      }
      t.x += some.x;
      t.y += some.y;
    }
  }
  // two rows of 16 channels to a warp
  t.x += __shfl_xor_sync(~0u, t.x, 16);
  t.y += __shfl_xor_sync(~0u, t.y, 16);
  __shared__ float2 red[32][17];
  if ((threadIdx.x & 16) == 0) red[threadIdx.x >> 5][cx] = t;
  __syncthreads();
  if (threadIdx.x < 512) {  // a warp per channel
    const int ch = threadIdx.x >> 5, lane = threadIdx.x & 31;
    float2 v = red[lane][ch];
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      v.x += __shfl_xor_sync(~0u, v.x, o);
      v.y += __shfl_xor_sync(~0u, v.y, o);
    }
    const int cc = blockIdx.x * 16 + ch;
    if (lane == 0 && cc < C) dbeta[g * par_gs + cc] = v.x, dgamma[g * par_gs + cc] = v.y;
  }
}

bool gn_aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// Ranges per image of the split form: enough for four CTAs per SM, of 2048 values at least.
int gn_ranges(int64_t N, int P, int C) {
  const int64_t by_size = ((int64_t)P * C + 2047) / 2048, by_sms = (4LL * kNumSMs + N - 1) / N;
  const int64_t s = std::max<int64_t>(1, std::min<int64_t>({by_size, by_sms, (int64_t)P, 256}));
  const int64_t rows = (P + s - 1) / s;
  return (int)((P + rows - 1) / rows);
}

// The first pass through the ring; false: not for these sizes and addresses.  Sets a.S and a.rows, its ranges.
template <typename XT, int V>
bool gn_ring_partial(GnArgs& a, cudaStream_t st, cudaError_t* e) {
  if constexpr (V * sizeof(XT) == 16) {
    static std::atomic<int> raised{0};
    const int tx = a.C / V, ty = std::min(512 / std::max(tx, 1), 512);
    if (tx > 512 || !gn_aligned16(a.x)) return false;
    const size_t chunk = (size_t)ty * kRingRows * a.C * sizeof(XT), rest = 64 + (size_t)tx * ty * (2 * V + 1) * 4;
    const int stages = (int)std::min<size_t>(4, (kRingSmem - rest) / chunk);
    const size_t smem = rest + stages * chunk;
    // ranges for two CTAs to an SM in one wave (never more than the workspace has), of eight chunks at least
    const int64_t fill = (2LL * kNumSMs + a.N - 1) / a.N, chunks = (a.P + ty * kRingRows - 1) / (ty * kRingRows);
    const int S = (int)std::min<int64_t>({(int64_t)a.S, fill, chunks / 8});
    if (S < 1 || a.N * S < kNumSMs || stages < 2) return false;
    a.stages = stages;
    a.rows = (a.P + S - 1) / S;
    a.S = (a.P + a.rows - 1) / a.rows;
    int dev = 0;
    *e = cudaGetDevice(&dev);
    if (*e == cudaSuccess && raised != dev + 1) {
      *e = cudaFuncSetAttribute(gn_ring_partial_kernel<XT, V>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kRingSmem);
      if (*e == cudaSuccess) raised = dev + 1;
    }
    if (*e == cudaSuccess) *e = launch_pdl(gn_ring_partial_kernel<XT, V>, dim3((unsigned)(a.N * a.S)), dim3(tx, ty), smem, st, a);
    return true;
  }
  return false;
}

template <typename XT, typename YT, int V, bool BWD>
cudaError_t gn_split(GnArgs a, cudaStream_t st) {
  a.S = gn_ranges(a.N, a.P, a.C);
  a.rows = (a.P + a.S - 1) / a.S;
  const int cols = a.C / V, tx = std::min(cols, kSplitThreads), ty = kSplitThreads / tx;
  const GnArgs ranges = a;  // the second pass's
  const dim3 grid((unsigned)(a.N * a.S), (cols + tx - 1) / tx);
  cudaError_t e = cudaSuccess;
  if (BWD || !gn_ring_partial<XT, V>(a, st, &e))
    e = launch_pdl(gn_partial_kernel<XT, YT, V, BWD>, grid, dim3(kSplitThreads), 0, st, a, tx, ty);
  if (e != cudaSuccess) return e;
  if constexpr (BWD) {
    // about 256 channels to a block
    const int per = std::max(1, std::min(a.groups, 256 / a.D));
    int threads = 256;
    while (threads < 1024 && (int64_t)per * a.D * a.S > 8 * threads) threads *= 2;
    e = launch_pdl(gn_sums_merge_kernel, dim3((unsigned)a.N, (a.groups + per - 1) / per), dim3(threads), 0, st, a, per);
  } else {
    int threads = 128;
    while (threads < 1024 && (int64_t)a.D * a.S > 8 * threads) threads *= 2;
    e = launch_pdl(gn_stats_merge_kernel, dim3((unsigned)(a.N * a.groups)), dim3(threads), 0, st, a);
  }
  if (e != cudaSuccess) return e;
  e = launch_pdl(gn_apply_kernel<XT, YT, V, BWD>, grid, dim3(kSplitThreads), 0, st, ranges, tx, ty);
  if (e != cudaSuccess || !BWD) return e;
  return launch_pdl(gn_param_grad_kernel, dim3((a.C + 15) / 16, (unsigned)(a.N / a.B)), dim3(1024), 0, st,
                    (const float2*)a.sums, (int64_t)a.B, a.C, a.par_gs, a.dgamma, a.dbeta);
}

// ---- resident form: an image (or, in a cluster, a CTA's range of its positions) stays in registers ----
//
// One read of x, one write: the values that a thread loads are summed, their squared deviations from the CTA's own
// mean are summed, and they are normalised, all out of registers.  A cluster's CTAs exchange (count, mean, squared
// deviations) through distributed shared memory and merge them in rank order (Chan et al.).  A thread holds kHold
// values, so that 1024 threads per SM fit the register file (64 each) and keep 64 to 128 KB of loads in flight.

constexpr int kFwdHold = 32, kBwdHold = 16;  // the backward also holds dz

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// An arrival that only says that reading is over: nothing written has to be seen.
__device__ __forceinline__ void cluster_read() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
// The float at `p` of this CTA's shared memory, in CTA `rank` of the cluster.
__device__ __forceinline__ float peer_float(const float* p, int rank) {
  uint32_t at;
  float v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
  return v;
}

// Adds up every thread's values v[0 .. NV) over the block's rows of threads: afterwards red[r][c] for r < the number of
// rows (a warp's, or every thread row) holds partial sums of column c = tx NV + j.  Where the threads across are a power of
// two below a warp, the rows of a warp are added first: at each step a lane gives half of its values away and adds up the
// other half, so that NV values cost about NV exchanges and not NV for every step.
template <int NV>
__device__ __forceinline__ void column_sums(float* v, float* red, int tx, int ty, int tx_n, bool shuffled) {
  const int cols = tx_n * NV;
  if (!shuffled) {
#pragma unroll
    for (int j = 0; j < NV; ++j) red[ty * cols + tx * NV + j] = v[j];
    return;
  }
  const int lane = (ty * tx_n + tx) & 31;
  int first = 0, have = NV;  // this lane's values: first .. first + have - 1
  bool mine = true;          // of the lanes with the same values one writes
#pragma unroll
  for (int k = 0; k < 5; ++k) {
    const int o = 16 >> k;
    if (o >= tx_n) {
      const bool up = lane & o;
      constexpr int kW[5] = {NV / 2, NV / 4, NV / 8, 0, 0};
      const int w = kW[k];
      if (w > 0) {
#pragma unroll
        for (int j = 0; j < w; ++j) {
          const float give = up ? v[j] : v[j + w], keep = up ? v[j + w] : v[j];
          v[j] = keep + __shfl_xor_sync(~0u, give, o);
        }
        first += up ? w : 0;
        have = w;
      } else {
        v[0] += __shfl_xor_sync(~0u, v[0], o);
        mine = mine && !up;
      }
    }
  }
  if (mine) {
    float* to = red + ((ty * tx_n + tx) >> 5) * cols + tx * NV + first;
#pragma unroll
    for (int j = 0; j < NV; ++j)
      if (j < have) to[j] = v[j];
  }
}

// The same for V channels of which `sub` neighbours are always of one group: those are added first.
template <int V>
__device__ __forceinline__ void channel_sums(float (&v)[V], float* red, int tx, int ty, int tx_n, bool shuffled, int sub) {
  if (V >= 2 && sub >= 2) {
#pragma unroll
    for (int j = 0; j < V / 2; ++j) v[j] = v[2 * j] + v[2 * j + 1];
  }
  if (V >= 4 && sub >= 4) {
#pragma unroll
    for (int j = 0; j < V / 4; ++j) v[j] = v[2 * j] + v[2 * j + 1];
  }
  if (V >= 8 && sub >= 8) {
#pragma unroll
    for (int j = 0; j < V / 8; ++j) v[j] = v[2 * j] + v[2 * j + 1];
  }
  const int nv = V / sub;
  if (nv == 1) column_sums<1>(v, red, tx, ty, tx_n, shuffled);
  if constexpr (V >= 2)
    if (nv == 2) column_sums<2>(v, red, tx, ty, tx_n, shuffled);
  if constexpr (V >= 4)
    if (nv == 4) column_sums<4>(v, red, tx, ty, tx_n, shuffled);
  if constexpr (V >= 8)
    if (nv == 8) column_sums<8>(v, red, tx, ty, tx_n, shuffled);
}

// out[q] = the sum over red's rows and the columns of group q (dn columns each), a warp per group, the block's full warps.
__device__ __forceinline__ void group_sums(const float* red, int rows, int groups, int dn, float* out, int tid, int nw) {
  if (tid >= min(nw, groups) * 32) return;
  const int lane = tid & 31, cols = groups * dn;
  const int wide = min(dn, 32), r0 = lane / wide, d0 = lane - r0 * wide, down = 32 / wide;
  for (int q = tid >> 5; q < groups; q += nw) {
    float t = 0.f;
    if (r0 < down)
      for (int r = r0; r < rows; r += down)
        for (int d = d0; d < dn; d += wide) t += red[r * cols + q * dn + d];
#pragma unroll
    for (int o = 16; o; o >>= 1) t += __shfl_xor_sync(~0u, t, o);
    if (lane == 0) out[q] = t;
  }
}

// The groups of a thread's V channels, from the group and the place in it of the first.
template <int V, typename F>
__device__ __forceinline__ void each_group(int c0, int D, F f) {
  int q = c0 / D, r = c0 - q * D;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    f(j, q);
    if (++r == D) r = 0, ++q;
  }
}

// Pipelined (PIPE): where there are more images than CTAs on the SMs at once, a CTA takes images blockIdx.x, blockIdx.x +
// gridDim.x, ... and bulk copies bring the next `stages` of them to shared memory while one is worked on in registers, so
// that the loads never stop for the sums' barriers.  One CTA to an image then, and 16-byte vectors.  2048 images of 1024 x 16, fp32
// to bf16 with ReLU: forward 37 us (5.4 TB/s), 55 without; backward 78 us (5.2 TB/s), 102 without; what is left is the
// sums' latency at the start and the end, and the copies' and stores' turns on the memory.  With fewer than two rounds of
// CTAs there is nothing to bring ahead.
constexpr int kMaxStages = 4, kPipeHead = 64;  // bytes before the first buffer: the barriers

template <typename XT, typename YT, int V, bool PIPE>
__global__ void __launch_bounds__(1024, 1) gn_fwd_resident_kernel(const GnArgs a) {
  constexpr int R = kFwdHold / V;
  extern __shared__ __align__(16) uint8_t raw[];
  float* sm = reinterpret_cast<float*>(raw + (PIPE ? kPipeHead + a.stages * a.slab : 0));
  uint64_t* full = reinterpret_cast<uint64_t*>(raw);
  float* gmean = sm;                // [groups]: the CTA's, then the image's mean
  float* gsq = gmean + a.groups;    // [groups]: squared deviations, then rstd
  float* own = gsq + a.groups;      // [2 groups]: what the other CTAs of the cluster read
  float* par = own + 2 * a.groups;  // [2][C]: gamma and beta
  float* red = par + 2 * a.C;
  const int tx = threadIdx.x, ty = threadIdx.y, c0 = tx * V;
  const int tx_n = blockDim.x, ty_n = blockDim.y, threads = tx_n * ty_n, tid = ty * tx_n + tx, nw = threads >> 5;
  const int rank = PIPE ? 0 : blockIdx.x % a.cl;
  const bool shuffled = tx_n < 32 && (tx_n & (tx_n - 1)) == 0;
  const int p0 = rank * a.rows, p1 = min(a.P, p0 + a.rows), cnt = max(0, p1 - p0);
  const int first = p0 + ty, last = p1;
  const int dn = a.D / a.sub, rows = shuffled ? nw : ty_n, step = ty_n * a.C;
  const float inv = cnt ? 1.f / ((float)cnt * (float)a.D) : 0.f;
  auto fetch = [&](int m, int s) {  // image m to buffer s
    mbar_expect_tx(&full[s], a.slab);
    bulk_load(raw + kPipeHead + s * a.slab, static_cast<const uint8_t*>(a.x) + (int64_t)m * a.slab, a.slab, &full[s]);
  };
  int n = PIPE ? blockIdx.x : blockIdx.x / a.cl, stage = 0;
  uint32_t ph = 0;
  if constexpr (PIPE) {
    if (tid == 0) {
      for (int s = 0; s < a.stages; ++s) mbar_init(&full[s], 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncthreads();
  }
  pdl_begin();
  if constexpr (PIPE) {
    if (tid == 0)
      for (int s = 0; s < a.stages; ++s)
        if (n + s * (int)gridDim.x < a.N) fetch(n + s * gridDim.x, s);
  }
  do {
    const int64_t base = (int64_t)n * a.P * a.C + (int64_t)first * a.C + c0;
    const int64_t pc = (int64_t)(n / a.B) * a.par_gs;
    float ga0 = 0.f, be0 = 0.f;  // the parameters of channel tid, on their way while the image is waited for
    if (tid < a.C) ga0 = a.gamma[pc + tid], be0 = a.beta[pc + tid];
    Vec<XT, V> r[R];
    if constexpr (PIPE) {
      const bool ok = wait_full(&full[stage], ph);
      const uint8_t* from = raw + kPipeHead + stage * a.slab + (first * a.C + c0) * (int)sizeof(XT);
#pragma unroll
      for (int i = 0; i < R; ++i)
        if (first + i * ty_n < last) r[i].load_shared(from + i * step * (int)sizeof(XT));
      if (__syncthreads_or(!ok)) {  // a wait ran out: the copies under way first
        if (tid == 0)
          for (int s = 0; s < a.stages; ++s) wait_full(&full[s], ph ^ (s < stage ? 1 : 0));
        break;
      }
      if (tid == 0 && n + a.stages * (int)gridDim.x < a.N) fetch(n + a.stages * gridDim.x, stage);
      if (++stage == a.stages) stage = 0, ph ^= 1;
    } else {
      const XT* x = static_cast<const XT*>(a.x) + base;
#pragma unroll
      for (int i = 0; i < R; ++i)
        if (first + i * ty_n < last) r[i].load(x + i * step);
    }
    if (tid < a.C) par[tid] = ga0, par[a.C + tid] = be0;
    for (int c = tid + threads; c < a.C; c += threads) par[c] = a.gamma[pc + c], par[a.C + c] = a.beta[pc + c];
    float t[V];
#pragma unroll
    for (int j = 0; j < V; ++j) t[j] = 0.f;
#pragma unroll
    for (int i = 0; i < R; ++i)
      if (first + i * ty_n < last) {
        float v[V];
        r[i].floats(v);
#pragma unroll
        for (int j = 0; j < V; ++j) t[j] += v[j];
      }
    channel_sums<V>(t, red, tx, ty, tx_n, shuffled, a.sub);
    __syncthreads();
    group_sums(red, rows, a.groups, dn, gmean, tid, nw);
    __syncthreads();
    float mu[V];
    each_group<V>(c0, a.D, [&](int j, int q) { mu[j] = gmean[q] * inv; });
#pragma unroll
    for (int j = 0; j < V; ++j) t[j] = 0.f;
#pragma unroll
    for (int i = 0; i < R; ++i)
      if (first + i * ty_n < last) {
        float v[V];
        r[i].floats(v);
#pragma unroll
        for (int j = 0; j < V; ++j) t[j] = fmaf(v[j] - mu[j], v[j] - mu[j], t[j]);
      }
    channel_sums<V>(t, red, tx, ty, tx_n, shuffled, a.sub);
    __syncthreads();
    group_sums(red, rows, a.groups, dn, gsq, tid, nw);
    __syncthreads();
    if (!PIPE && a.cl > 1) {
      for (int q = tid; q < a.groups; q += threads) own[2 * q] = gmean[q] * inv, own[2 * q + 1] = gsq[q];
      cluster_arrive();
      cluster_wait();
    }
    for (int q = tid; q < a.groups; q += threads) {
      float m = gmean[q] * inv, sq = gsq[q], k = (float)cnt * a.D;
      if (!PIPE && a.cl > 1) {
        k = m = sq = 0.f;
        for (int c = 0; c < a.cl; ++c)
          chan(k, m, sq, (float)max(0, min(a.P, (c + 1) * a.rows) - c * a.rows) * a.D, peer_float(own + 2 * q, c),
               peer_float(own + 2 * q + 1, c));
      }
      const float rs = __frsqrt_rn(sq / k + a.eps);
      gmean[q] = m;
      gsq[q] = rs;
      if (rank == 0) a.mean[(int64_t)n * a.groups + q] = m, a.rstd[(int64_t)n * a.groups + q] = rs;
    }
    __syncthreads();
    if (!PIPE && a.cl > 1) cluster_read();  // this CTA has read the others' sums; the wait is at the end
    {
      float ga[V], be[V];
      each_group<V>(c0, a.D, [&](int j, int q) {
        mu[j] = gmean[q], ga[j] = par[c0 + j] * gsq[q], be[j] = par[a.C + c0 + j];
      });
      YT* out = static_cast<YT*>(a.out) + base;
      constexpr int kKind = sizeof(YT) == 4 ? kExact : kFast;
      with_act(a.act, [&](auto act) {
#pragma unroll
        for (int i = 0; i < R; ++i)
          if (first + i * ty_n < last) {
            float v[V];
            r[i].floats(v);
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = activate<kKind, decltype(act)::value>(fmaf(v[j] - mu[j], ga[j], be[j]));
            Vec<YT, V> o;
            o.set(v);
            o.store(out + i * step);
          }
      });
    }
    if (!PIPE && a.cl > 1) cluster_wait();
    n += gridDim.x;
  } while (PIPE && n < a.N);
}

template <typename XT, typename YT, int V, bool PIPE>
__global__ void __launch_bounds__(1024, 1) gn_bwd_resident_kernel(const GnArgs a) {
  constexpr int R = kBwdHold / V;
  extern __shared__ __align__(16) uint8_t raw[];
  const bool relu = a.act == LSGD_ACT_RELU, silu = a.act == LSGD_ACT_SILU;
  const int slabs = a.slab + (relu ? 2 : 1) * a.slab_y;  // x, dy and, for ReLU, y
  float* sm = reinterpret_cast<float*>(raw + (PIPE ? kPipeHead + a.stages * slabs : 0));
  uint64_t* full = reinterpret_cast<uint64_t*>(raw);
  float* gm = sm;                     // [2 groups]: m1 and m2
  float* own = gm + 2 * a.groups;     // [2 groups]
  float* stat = own + 2 * a.groups;   // [2 groups]: mean and rstd
  float* par = stat + 2 * a.groups;   // [2][C]: gamma and beta
  float* chans = par + 2 * a.C;       // [2][C]: sum dz, sum dz xh
  float* red = chans + 2 * a.C;       // [rows][C], twice
  const int tx = threadIdx.x, ty = threadIdx.y, c0 = tx * V;
  const int tx_n = blockDim.x, ty_n = blockDim.y, threads = tx_n * ty_n, tid = ty * tx_n + tx, nw = threads >> 5;
  const int rank = PIPE ? 0 : blockIdx.x % a.cl;
  const bool shuffled = tx_n < 32 && (tx_n & (tx_n - 1)) == 0;
  const int p0 = rank * a.rows, p1 = min(a.P, p0 + a.rows);
  const int first = p0 + ty, last = p1, step = ty_n * a.C, lane = tid & 31;
  const int rows = shuffled ? nw : ty_n;
  float* red1 = red + rows * a.C;
  const float inv = 1.f / ((float)a.P * (float)a.D);
  auto fetch = [&](int m, int s) {  // image m to buffer s
    uint8_t* to = raw + kPipeHead + s * slabs;
    mbar_expect_tx(&full[s], slabs);
    bulk_load(to, static_cast<const uint8_t*>(a.x) + (int64_t)m * a.slab, a.slab, &full[s]);
    bulk_load(to + a.slab, static_cast<const uint8_t*>(a.dy) + (int64_t)m * a.slab_y, a.slab_y, &full[s]);
    if (relu) bulk_load(to + a.slab + a.slab_y, static_cast<const uint8_t*>(a.y) + (int64_t)m * a.slab_y, a.slab_y, &full[s]);
  };
  int n = PIPE ? blockIdx.x : blockIdx.x / a.cl, stage = 0;
  uint32_t ph = 0;
  if constexpr (PIPE) {
    if (tid == 0) {
      for (int s = 0; s < a.stages; ++s) mbar_init(&full[s], 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncthreads();
  }
  pdl_begin();
  if constexpr (PIPE) {
    if (tid == 0)
      for (int s = 0; s < a.stages; ++s)
        if (n + s * (int)gridDim.x < a.N) fetch(n + s * gridDim.x, s);
  }
  do {
    const int64_t base = (int64_t)n * a.P * a.C + (int64_t)first * a.C + c0;
    const int64_t pc = (int64_t)(n / a.B) * a.par_gs, pg = (int64_t)n * a.groups;
    float ga0 = 0.f, be0 = 0.f, mu0 = 0.f, rs0 = 0.f;  // channel tid's and group tid's, while the image is waited for
    if (tid < a.C) ga0 = a.gamma[pc + tid], be0 = a.beta[pc + tid];
    if (tid < a.groups) mu0 = a.mean[pg + tid], rs0 = a.rstd[pg + tid];
    Vec<XT, V> r[R];
    float dz[R][V];
    auto masked = [&](const Vec<YT, V>& rd, const Vec<YT, V>& ry, float (&d)[V]) {
      rd.floats(d);
      if (relu) {
        float yv[V];
        ry.floats(yv);
#pragma unroll
        for (int j = 0; j < V; ++j) d[j] = yv[j] > 0.f ? d[j] : 0.f;
      }
    };
    if constexpr (PIPE) {
      const bool ok = wait_full(&full[stage], ph);
      const uint8_t* fx = raw + kPipeHead + stage * slabs + (first * a.C + c0) * (int)sizeof(XT);
      const uint8_t* fd = raw + kPipeHead + stage * slabs + a.slab + (first * a.C + c0) * (int)sizeof(YT);
#pragma unroll
      for (int i = 0; i < R; ++i) {
#pragma unroll
        for (int j = 0; j < V; ++j) dz[i][j] = 0.f;
        if (first + i * ty_n < last) {
          Vec<YT, V> rd, ry;
          r[i].load_shared(fx + i * step * (int)sizeof(XT));
          rd.load_shared(fd + i * step * (int)sizeof(YT));
          if (relu) ry.load_shared(fd + a.slab_y + i * step * (int)sizeof(YT));
          masked(rd, ry, dz[i]);
        }
      }
      if (__syncthreads_or(!ok)) {  // a wait ran out: the copies under way first
        if (tid == 0)
          for (int s = 0; s < a.stages; ++s) wait_full(&full[s], ph ^ (s < stage ? 1 : 0));
        break;
      }
      if (tid == 0 && n + a.stages * (int)gridDim.x < a.N) fetch(n + a.stages * gridDim.x, stage);
      if (++stage == a.stages) stage = 0, ph ^= 1;
    } else {
      const XT* x = static_cast<const XT*>(a.x) + base;
      const YT* dy = static_cast<const YT*>(a.dy) + base;
      const YT* y = static_cast<const YT*>(a.y) + base;
      Vec<YT, V> rd[R], ry[R];
#pragma unroll
      for (int i = 0; i < R; ++i)
        if (first + i * ty_n < last) {
          const int at = i * step;
          r[i].load(x + at);
          rd[i].load(dy + at);
          if (relu) ry[i].load(y + at);
        }
#pragma unroll
      for (int i = 0; i < R; ++i) {
#pragma unroll
        for (int j = 0; j < V; ++j) dz[i][j] = 0.f;
        if (first + i * ty_n < last) masked(rd[i], ry[i], dz[i]);
      }
    }
    if (tid < a.C) par[tid] = ga0, par[a.C + tid] = be0;
    for (int c = tid + threads; c < a.C; c += threads) par[c] = a.gamma[pc + c], par[a.C + c] = a.beta[pc + c];
    if (tid < a.groups) stat[2 * tid] = mu0, stat[2 * tid + 1] = rs0;
    for (int q = tid + threads; q < a.groups; q += threads) stat[2 * q] = a.mean[pg + q], stat[2 * q + 1] = a.rstd[pg + q];
    __syncthreads();
    float s0[V], s1[V];
#pragma unroll
    for (int j = 0; j < V; ++j) s0[j] = s1[j] = 0.f;
    // channel by channel, so that one channel's parameters are in registers at a time
    each_group<V>(c0, a.D, [&](int j, int q) {
      const float mu = stat[2 * q], rs = stat[2 * q + 1];
      if (silu) {
        const float ga = par[c0 + j], be = par[a.C + c0 + j];
#pragma unroll
        for (int i = 0; i < R; ++i)
          if (first + i * ty_n < last) {
            const float z = fmaf((r[i].at(j) - mu) * rs, ga, be), sg = sigmoid<sizeof(XT) == 4 ? kExact : kSums>(z);
            dz[i][j] *= sg * fmaf(z, 1.f - sg, 1.f);
          }
      }
#pragma unroll
      for (int i = 0; i < R; ++i)
        if (first + i * ty_n < last) {
          s0[j] += dz[i][j];
          s1[j] = fmaf(dz[i][j], (r[i].at(j) - mu) * rs, s1[j]);
        }
    });
    column_sums<V>(s0, red, tx, ty, tx_n, shuffled);
    column_sums<V>(s1, red1, tx, ty, tx_n, shuffled);
    __syncthreads();
    if (rows <= 32) {
      for (int c = tid; c < 2 * a.C; c += threads) {  // first the sums of dz, then those of dz xh
        const float* from = c < a.C ? red + c : red1 + (c - a.C);
        float t = 0.f;
        for (int i = 0; i < rows; ++i) t += from[i * a.C];
        chans[c] = t;
      }
    } else {  // many rows over few channels: a warp per channel
      for (int c = tid < nw * 32 ? tid >> 5 : 2 * a.C; c < 2 * a.C; c += nw) {
        const float* from = c < a.C ? red + c : red1 + (c - a.C);
        float t = 0.f;
        for (int i = lane; i < rows; i += 32) t += from[i * a.C];
#pragma unroll
        for (int o = 16; o; o >>= 1) t += __shfl_xor_sync(~0u, t, o);
        if (lane == 0) chans[c] = t;
      }
    }
    __syncthreads();
    for (int q = tid < nw * 32 ? tid >> 5 : a.groups; q < a.groups; q += nw) {
      float t0 = 0.f, t1 = 0.f;
      for (int d = lane; d < a.D; d += 32) {
        const float g = par[q * a.D + d];
        t0 = fmaf(g, chans[q * a.D + d], t0);
        t1 = fmaf(g, chans[a.C + q * a.D + d], t1);
      }
#pragma unroll
      for (int o = 16; o; o >>= 1) t0 += __shfl_xor_sync(~0u, t0, o), t1 += __shfl_xor_sync(~0u, t1, o);
      if (lane == 0) {
        float* to = !PIPE && a.cl > 1 ? own : gm;
        to[2 * q] = t0 * inv, to[2 * q + 1] = t1 * inv;
      }
    }
    if (!PIPE && a.cl > 1) {
      cluster_arrive();
      cluster_wait();
      for (int q = tid; q < 2 * a.groups; q += threads) {
        float t = 0.f;
        for (int c = 0; c < a.cl; ++c) t += peer_float(own + q, c);
        gm[q] = t;
      }
    }
    __syncthreads();
    if (!PIPE && a.cl > 1) cluster_read();
    float2* out = reinterpret_cast<float2*>(a.sums) + ((int64_t)n * a.cl + rank) * a.C;
    for (int c = tid; c < a.C; c += threads) out[c] = make_float2(chans[c], chans[a.C + c]);
    each_group<V>(c0, a.D, [&](int j, int q) {
      const float mu = stat[2 * q], rs = stat[2 * q + 1], k = rs * par[c0 + j], b = rs * gm[2 * q];
      const float m = rs * rs * gm[2 * q + 1];
#pragma unroll
      for (int i = 0; i < R; ++i) dz[i][j] = fmaf(k, dz[i][j], -b) - (r[i].at(j) - mu) * m;
    });
    XT* dx = static_cast<XT*>(a.out) + base;
#pragma unroll
    for (int i = 0; i < R; ++i)
      if (first + i * ty_n < last) {
        Vec<XT, V> o;
        o.set(dz[i]);
        o.store(dx + i * step);
      }
    if (!PIPE && a.cl > 1) cluster_wait();
    n += gridDim.x;
  } while (PIPE && n < a.N);
}

// The resident form's CTAs per image (up to 16, the largest cluster), or 0: the split form.  A
// CTA of T threads takes `rows` positions if rows C / hold + C <= T, whatever the vector width (a row of threads is
// C / V wide, and hold / V positions fall to each).  A power of two: CTAs of about 512 threads or fewer where they do; then,
// where the images are few, more CTAs to an image down to 4096 values each.  (One row of threads more than needed covers every
// V; with rows rounded up to full warps a CTA has at most T + 31 threads.)  A cluster lies in one GPC: of 9 CTAs, 15 run at
// once, of 10, 13, but of 16, 7.  Images that these fewer CTAs hold, and that would take another round in clusters of 16,
// take one (backward of 15 images of 1517 x 90 in fp32: 31 us in clusters of 16, 19 in clusters of 9).
bool gn_fits(int P, int C, int cl, int hold, int threads) {
  return (int64_t)((P + cl - 1) / cl) * C / hold + 1 + C <= threads;
}
// The threads across and down of a CTA of `rows` positions with vectors of V values: full warps where the rows of a warp are
// added by shuffles, one at least otherwise.
dim3 gn_block(int rows, int C, int V, int hold, bool* shuffled) {
  const int tx = C / V;
  *shuffled = tx < 32 && (tx & (tx - 1)) == 0;
  int ty = std::max((rows + hold / V - 1) / (hold / V), (32 + tx - 1) / tx);
  if (*shuffled) ty = (ty + 32 / tx - 1) / (32 / tx) * (32 / tx);
  return dim3(tx, ty);
}
// The most threads that a CTA of a cluster of cl has, over the vectors that may be used.
int64_t gn_threads(int P, int C, int cl, int hold) {
  int64_t most = 0;
  bool shuffled;
  for (int V = 1; V <= 8 && C % V == 0; V *= 2) {
    const dim3 b = gn_block((P + cl - 1) / cl, C, V, hold, &shuffled);
    most = std::max(most, (int64_t)b.x * b.y);
  }
  return most;
}
constexpr int kMaxCluster = 16;
int gn_cluster(int64_t N, int P, int C, int hold) {
  int cl = 0;
  for (int T : {608, 992})
    for (int c = 1; c <= kMaxCluster && !cl; c *= 2)
      if (gn_fits(P, C, c, hold, T)) cl = c;
  while (cl && cl < 8 && N * cl < kNumSMs && (int64_t)P * C / (2 * cl) >= 4096) cl *= 2;
  if (cl == kMaxCluster && N > 7) {
    if (N <= 13 && gn_threads(P, C, 10, hold) <= 1024) return 10;
    if (N <= 15 && gn_threads(P, C, 9, hold) <= 1024) return 9;
  }
  return cl;
}

// Whether the split form, which reads its inputs twice but fills all SMs, takes less time than many rounds of clusters, whose
// CTAs load, wait for one another and store in turn.  A model in us, fitted to 120 pairs of measurements (4 to 512 images of
// 32,000 to 400,000 values): a round costs 6 us of bf16 images, 9 of fp32 ones, more in clusters of 16 and with one CTA to
// an SM; the split form its launches and 6 TB/s.  (Of another 100 pairs it takes the slower form, by 3 us or more, in 17.)
// Forward of 128 images of 3100 x 64 in bf16: 66 us in clusters, 35 split, of 32 images: 18.4 and 17.7; backward of 128 images of
// 1550 x 64: 66 and 43, of 32: 18.4 and 21.1.
bool gn_split_faster(int cl, int64_t N, int P, int C, bool bwd, int xz, int yz, bool relu) {
  if (cl < 4) return false;  // such images mostly fit one CTA, whose pipelined form overlaps its rounds
  const int per_sm = (int64_t)((P + cl - 1) / cl) * C / (bwd ? kBwdHold : kFwdHold) + C / 8 <= 512 ? 2 : 1;
  const int at_once = (cl == 4 ? 36 : cl <= 9 ? 15 : cl == 10 ? 13 : 7) * per_sm;
  const double round = (3 + 0.75 * (xz + yz)) * (per_sm == 2 ? 1.0 : 1.2) * (cl > 10 ? 1.15 : 1.0);
  const int bytes = bwd ? 3 * xz + (relu ? 4 : 2) * yz : 2 * xz + yz;
  return (bwd ? 20 : 18) + (double)N * P * C * bytes / 6e6 < 5 + round * ((N + at_once - 1) / at_once);
}
// The form of a call: CTAs per image, or 0.
int gn_plan(int64_t N, int P, int C, bool bwd, int xz, int yz, bool relu) {
  const int cl = gn_cluster(N, P, C, bwd ? kBwdHold : kFwdHold);
  return gn_split_faster(cl, N, P, C, bwd, xz, yz, relu) ? 0 : cl;
}

// The shape of a resident launch with vectors of V values, and its bytes of shared memory.
void gn_resident_shape(GnArgs& a, int V, int hold, bool bwd, dim3* block, size_t* smem) {
  a.rows = (a.P + a.cl - 1) / a.cl;
  bool shuffled;
  *block = gn_block(a.rows, a.C, V, hold, &shuffled);
  a.sub = std::min(V, a.D & -a.D);
  const int rows = shuffled ? block->x * block->y / 32 : block->y;
  *smem = 4 * (bwd ? 6 * (size_t)a.groups + 4 * (size_t)a.C + 2 * (size_t)rows * a.C
                   : 4 * (size_t)a.groups + 2 * (size_t)a.C + (size_t)rows * (a.C / a.sub));
}

constexpr size_t kGnMaxSmem = 224 * 1024;
template <typename K>
cudaError_t gn_launch_resident(K kernel, std::atomic<int>& raised, const GnArgs& a, int grid, dim3 block, size_t smem,
                               cudaStream_t st) {
  if (block.x * block.y > 1024 || smem > kGnMaxSmem) return cudaErrorInvalidValue;
  if (smem > 48 * 1024 || a.cl > 8) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (raised != dev + 1) {
      e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kGnMaxSmem);
      if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
      if (e != cudaSuccess) return e;
      raised = dev + 1;
    }
  }
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = a.cl;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = a.cl > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, a);
}

template <typename XT, typename YT, int V, bool BWD>
cudaError_t gn_resident(GnArgs a, cudaStream_t st) {
  static std::atomic<int> raised{0}, raised_pipe{0};  // device + 1 whose limits this kernel's have been raised to
  constexpr int hold = BWD ? kBwdHold : kFwdHold;
  dim3 block;
  size_t smem = 0;
  cudaError_t e = cudaErrorInvalidValue;
  bool piped = false;
  if constexpr (V * sizeof(XT) == 16 || V * sizeof(YT) == 16) {
    // the pipelined form: one CTA to an image, images of whole 16-byte pieces, at least two rounds of CTAs
    GnArgs b = a;
    b.cl = 1;
    const int64_t values = (int64_t)a.P * a.C;
    if (values <= 1024 * hold && values * sizeof(XT) % 16 == 0 && values * sizeof(YT) % 16 == 0 &&
        gn_aligned16(a.x) && gn_aligned16(BWD ? a.dy : a.x) && gn_aligned16(BWD && a.act == LSGD_ACT_RELU ? a.y : a.x)) {
      gn_resident_shape(b, V, hold, BWD, &block, &smem);
      const int threads = block.x * block.y;
      b.slab = (int)(values * sizeof(XT)), b.slab_y = (int)(values * sizeof(YT));
      const int bytes = BWD ? b.slab + (a.act == LSGD_ACT_RELU ? 2 : 1) * b.slab_y : b.slab;
      // as many CTAs to an SM as the registers take, and the images ahead that the shared memory then holds
      int per_sm = threads <= 1024 ? std::min(1024 / threads, 8) : 0;
      const int64_t room = per_sm ? 222 * 1024 / per_sm - 1024 - (int64_t)smem - kPipeHead : 0;
      b.stages = (int)std::min<int64_t>(kMaxStages, room / bytes);
      if (per_sm && b.stages >= 1 && a.N >= 2LL * per_sm * kNumSMs) {
        piped = true;
        const int grid = per_sm * kNumSMs;
        smem += kPipeHead + (size_t)b.stages * bytes;
        if constexpr (BWD) e = gn_launch_resident(gn_bwd_resident_kernel<XT, YT, V, true>, raised_pipe, b, grid, block, smem, st);
        else e = gn_launch_resident(gn_fwd_resident_kernel<XT, YT, V, true>, raised_pipe, b, grid, block, smem, st);
        a.cl = 1;
      }
    }
  }
  if (!piped) {
    gn_resident_shape(a, V, hold, BWD, &block, &smem);
    const int grid = (int)(a.N * a.cl);
    if constexpr (BWD) e = gn_launch_resident(gn_bwd_resident_kernel<XT, YT, V, false>, raised, a, grid, block, smem, st);
    else e = gn_launch_resident(gn_fwd_resident_kernel<XT, YT, V, false>, raised, a, grid, block, smem, st);
  }
  if (e != cudaSuccess || !BWD) return e;
  return launch_pdl(gn_param_grad_kernel, dim3((a.C + 15) / 16, (unsigned)(a.N / a.B)), dim3(1024), 0, st,
                    (const float2*)a.sums, (int64_t)a.B * a.cl, a.C, a.par_gs, a.dgamma, a.dbeta);
}

template <typename XT, typename YT, int V, bool BWD>
cudaError_t gn_form(const GnArgs& a, cudaStream_t st) {
  return a.cl ? gn_resident<XT, YT, V, BWD>(a, st) : gn_split<XT, YT, V, BWD>(a, st);
}

template <typename XT, typename YT, bool BWD>
cudaError_t gn_run(const GnArgs& a, int vmax, cudaStream_t st) {
  if constexpr (sizeof(XT) == 2) {
    if (vmax >= 8) return gn_form<XT, YT, 8, BWD>(a, st);
  }
  if (vmax >= 4) return gn_form<XT, YT, 4, BWD>(a, st);
  if (vmax >= 2) return gn_form<XT, YT, 2, BWD>(a, st);
  return gn_form<XT, YT, 1, BWD>(a, st);
}

template <bool BWD>
cudaError_t gn_typed(const GnArgs& a, bool xb, bool yb, int vmax, cudaStream_t st) {
  if (xb) return yb ? gn_run<uint16_t, uint16_t, BWD>(a, vmax, st) : gn_run<uint16_t, float, BWD>(a, vmax, st);
  return yb ? gn_run<float, uint16_t, BWD>(a, vmax, st) : gn_run<float, float, BWD>(a, vmax, st);
}

// The widest vector (a power of two of values) that divides C and whose accesses to p (size z each) are aligned.
int gn_vec(int v, int C, const void* p, int z) {
  while (v > 1 && (C % v || reinterpret_cast<uintptr_t>(p) % std::min(16, v * z))) v >>= 1;
  return v;
}

// Enough for the form that any types and activation take.
size_t gn_workspace(int64_t N, int P, int C, int groups, bool backward) {
  const int cl = gn_cluster(N, P, C, backward ? kBwdHold : kFwdHold);
  bool split = cl == 0;
  for (int t = 0; t < 8 && !split; ++t) split = gn_split_faster(cl, N, P, C, backward, t & 1 ? 4 : 2, t & 2 ? 4 : 2, t & 4);
  const size_t resident = backward ? (size_t)N * cl * C * 2 : 0;
  const size_t ranges = (size_t)N * gn_ranges(N, P, C) * C * 2 + (backward ? (size_t)N * C * 2 + (size_t)N * groups * 2 : 0);
  return 4 * (split ? std::max(resident, ranges) : resident);
}

lsgd_status gn_error(lsgd_status s, const char* fn, const char* what) {
  set_last_error(std::string(fn) + ": " + what);
  return s;
}

const char* gn_shape_error(int G, int B, int64_t P, int C, int groups) {
  if (G < 1 || B < 1 || P < 1 || C < 1 || groups < 1) return "G, B, P, C and groups must be at least 1";
  if (C % groups) return "C must be a multiple of groups";
  if (G > 65535 || (int64_t)G * B > (1 << 24) || C > 65536 || P > (1 << 24) || (int64_t)G * B * groups > 0x7fffffff)
    return "at most 65535 workers, 2^24 images (G B), 2^31 - 1 groups in all, 65536 channels and 2^24 positions";
  return nullptr;
}


}  // namespace

int norm_take_timeout_flag() {
  int h = 0;
  if (!g_norm_used) return 0;
  if (cudaMemcpyFromSymbol(&h, g_norm_timeout, sizeof(int)) != cudaSuccess) {
    cudaGetLastError();
    return 0;
  }
  if (h) {
    const int zero = 0;
    cudaMemcpyToSymbol(g_norm_timeout, &zero, sizeof(int));
  }
  return h;
}

}  // namespace lsgd

extern "C" {

lsgd_status lsgd_groupnorm_workspace(int G, int B, int64_t P, int C, int groups, int backward, size_t* bytes) {
  using namespace lsgd;
  const char* bad = gn_shape_error(G, B, P, C, groups);
  if (!bad && !bytes) bad = "bytes is NULL";
  if (bad) return gn_error(LSGD_EINVAL, "lsgd_groupnorm_workspace", bad);
  *bytes = gn_workspace((int64_t)G * B, (int)P, C, groups, backward != 0);
  return LSGD_OK;
}

lsgd_status lsgd_groupnorm_forward(const void* x, int x_type, const float* gamma, const float* beta,
                                   int64_t par_gs, void* y, int y_type, float* mean, float* rstd, int G, int B,
                                   int64_t P, int C, int groups, float eps, int act, void* workspace,
                                   size_t workspace_bytes, void* stream) {
  using namespace lsgd;
  const char* fn = "lsgd_groupnorm_forward";
  const char* bad = gn_shape_error(G, B, P, C, groups);
  const bool xb = x_type == LSGD_BF16, yb = y_type == LSGD_BF16;
  const int xz = xb ? 2 : 4, yz = yb ? 2 : 4;
  if (bad) return gn_error(LSGD_EINVAL, fn, bad);
  const int64_t N = (int64_t)G * B;
  const size_t n = (size_t)N * P * C, ns = (size_t)N * groups * 4, need = gn_workspace(N, (int)P, C, groups, false);
  const auto params = [&](const float* p) { return Blocks(p, 4 * (size_t)C, par_gs, G); };
  if (!x || !gamma || !beta || !y || !mean || !rstd) bad = "a pointer is NULL";
  else if ((!xb && x_type != LSGD_FP32) || (!yb && y_type != LSGD_FP32)) bad = "types are LSGD_FP32 or LSGD_BF16";
  else if (act != LSGD_ACT_NONE && act != LSGD_ACT_RELU && act != LSGD_ACT_SILU) bad = "unknown activation";
  else if (!(eps > 0.f) || !(eps < 1e30f)) bad = "eps must be positive and finite";
  else if (par_gs < C) bad = "par_gs must be at least C";
  else if (misaligned(x, xz) || misaligned(y, yz) || misaligned(gamma, 4) || misaligned(beta, 4) ||
           misaligned(mean, 4) || misaligned(rstd, 4))
    bad = "a pointer is not aligned to its element";
  else if (need && (!workspace || workspace_bytes < need || misaligned(workspace, 16)))
    bad = "workspace NULL, not 16-byte aligned or smaller than lsgd_groupnorm_workspace says";
  else if (any_overlap({Blocks(y, n * yz), Blocks(mean, ns), Blocks(rstd, ns), Blocks(workspace, need)},
                      {Blocks(x, n * xz), params(gamma), params(beta)}))
    bad = "tensors overlap";
  if (bad) return gn_error(LSGD_EINVAL, fn, bad);
  if (!g_norm_used) g_norm_used = true;
  GnArgs a{};
  a.x = x, a.out = y, a.gamma = gamma, a.beta = beta, a.par_gs = par_gs, a.mean = mean, a.rstd = rstd;
  a.part = static_cast<float*>(workspace);
  a.B = B, a.P = (int)P, a.C = C, a.groups = groups, a.D = C / groups, a.act = act, a.N = N, a.eps = eps;
  a.cl = gn_plan(N, a.P, C, false, xz, yz, false);
  const int v = gn_vec(gn_vec(xb ? 8 : 4, C, x, xz), C, y, yz);
  const cudaError_t e = gn_typed<false>(a, xb, yb, v, (cudaStream_t)stream);
  return e == cudaSuccess ? LSGD_OK : gn_error(LSGD_ECUDA, fn, cudaGetErrorString(e));
}

lsgd_status lsgd_groupnorm_backward(const void* x, int x_type, const void* y, const void* dy, int y_type,
                                    const float* gamma, const float* beta, int64_t par_gs, const float* mean,
                                    const float* rstd, void* dx, float* dgamma, float* dbeta, int G, int B,
                                    int64_t P, int C, int groups, int act, void* workspace,
                                    size_t workspace_bytes, void* stream) {
  using namespace lsgd;
  const char* fn = "lsgd_groupnorm_backward";
  const char* bad = gn_shape_error(G, B, P, C, groups);
  const bool xb = x_type == LSGD_BF16, yb = y_type == LSGD_BF16;
  const int xz = xb ? 2 : 4, yz = yb ? 2 : 4;
  if (bad) return gn_error(LSGD_EINVAL, fn, bad);
  const int64_t N = (int64_t)G * B;
  const size_t n = (size_t)N * P * C, ns = (size_t)N * groups * 4, need = gn_workspace(N, (int)P, C, groups, true);
  const auto params = [&](const float* p) { return Blocks(p, 4 * (size_t)C, par_gs, G); };
  const bool relu = act == LSGD_ACT_RELU;
  if (!x || !dy || !gamma || !beta || !mean || !rstd || !dx || !dgamma || !dbeta || (relu && !y))
    bad = "a pointer is NULL (y may be only where the activation is not ReLU)";
  else if ((!xb && x_type != LSGD_FP32) || (!yb && y_type != LSGD_FP32)) bad = "types are LSGD_FP32 or LSGD_BF16";
  else if (act != LSGD_ACT_NONE && !relu && act != LSGD_ACT_SILU) bad = "unknown activation";
  else if (par_gs < C) bad = "par_gs must be at least C";
  else if (misaligned(x, xz) || misaligned(dx, xz) || misaligned(dy, yz) || (relu && misaligned(y, yz)) ||
           misaligned(gamma, 4) || misaligned(beta, 4) || misaligned(mean, 4) || misaligned(rstd, 4) ||
           misaligned(dgamma, 4) || misaligned(dbeta, 4))
    bad = "a pointer is not aligned to its element";
  else if (!workspace || workspace_bytes < need || misaligned(workspace, 16))
    bad = "workspace NULL, not 16-byte aligned or smaller than lsgd_groupnorm_workspace says";
  else if (any_overlap({Blocks(dx, n * xz), params(dgamma), params(dbeta), Blocks(workspace, need)},
                      {Blocks(x, n * xz), Blocks(dy, n * yz), Blocks(relu ? y : nullptr, n * yz), params(gamma),
                       params(beta), Blocks(mean, ns), Blocks(rstd, ns)}))
    bad = "tensors overlap";
  if (bad) return gn_error(LSGD_EINVAL, fn, bad);
  if (!g_norm_used) g_norm_used = true;
  GnArgs a{};
  a.x = x, a.y = y, a.dy = dy, a.out = dx, a.gamma = gamma, a.beta = beta, a.par_gs = par_gs;
  a.mean = const_cast<float*>(mean), a.rstd = const_cast<float*>(rstd), a.dgamma = dgamma, a.dbeta = dbeta;
  a.B = B, a.P = (int)P, a.C = C, a.groups = groups, a.D = C / groups, a.act = act, a.N = N;
  a.part = static_cast<float*>(workspace);
  a.cl = gn_plan(N, a.P, C, true, xz, yz, relu);
  a.sums = a.cl ? a.part : a.part + (size_t)N * gn_ranges(N, a.P, C) * C * 2;
  a.m12 = a.sums + (size_t)N * C * 2;
  int v = gn_vec(gn_vec(gn_vec(xb ? 8 : 4, C, x, xz), C, dx, xz), C, dy, yz);
  if (relu) v = gn_vec(v, C, y, yz);
  const cudaError_t e = gn_typed<true>(a, xb, yb, v, (cudaStream_t)stream);
  return e == cudaSuccess ? LSGD_OK : gn_error(LSGD_ECUDA, fn, cudaGetErrorString(e));
}

}  // extern "C"
