// Layer normalisation of rows with an activation, and with the addition of a residual before it, forward and backward, for G
// workers of R rows of C values each.
//
// For a row x (and r, where there is a residual):
//   s = x + r (rounded to x's type),  mean = sum s / C,  rstd = 1 / sqrt(sum (s - mean)^2 / C + eps),
//   xh = (s - mean) rstd,  y = act(gamma xh + beta).
// Backward, with dz = dy act'(.), t = gamma dz, m1 and m2 the row's means of t and t xh:
//   dx = rstd (t - m1 - xh m2) + ds,  dgamma = sum dz xh,  dbeta = sum dz (over the worker's rows).
//
// Both are bound by memory.  A team of threads holds a row, kHold neighbouring or vector-strided values to a thread, so that
// every input is read once; a thread's columns stay the same from row to row, so that its parameters and the sums for dgamma and
// dbeta stay in registers.  A team is a part of a warp, a warp, several warps of a CTA, or the CTAs of a cluster, by the
// row's length; a CTA holds several teams where they are small.  The next row's loads are under way while one is reduced.
#include <algorithm>
#include <string>
#include <type_traits>

#include "../../include/lsgd.h"
#include "common.cuh"
#include "lsgd_internal.h"
#include "operands.h"
#include "tc_ptx.cuh"
#include "vectors.cuh"

namespace lsgd {
namespace {

constexpr int kHold = 8;            // values of a row in a thread
constexpr int kMaxThreads = 512;    // of a CTA
constexpr int kMaxCluster = 16;
constexpr int kMaxC = kHold * kMaxThreads * kMaxCluster;  // 65536

struct LnArgs {
  const void *x, *r, *y, *dy, *ds;
  void *s, *out;  // the stored sum; y (forward), dx (backward)
  const float *gamma, *beta;
  int64_t par_gs;
  float *mean, *rstd;
  float *part, *dgamma, *dbeta;  // backward; part [G][ranges][2][C]
  int64_t R, x_ld, y_ld;
  int C, act;
  float eps;
  int T, teams;   // threads of a team in a CTA, teams of a CTA
  int cl, slice;  // CTAs of a row, columns of each
  int seg;        // rows that are added up at a time
};

// How the rows are dealt out, whatever the types.
struct LnPlan {
  int T, teams, cl, slice;
  int64_t ranges;  // CTAs (clusters) of a worker
  int64_t rows;    // rows of a team at most
};

LnPlan ln_plan(int G, int64_t R, int C, int threads_per_sm) {
  LnPlan p;
  p.cl = (C + kHold * kMaxThreads - 1) / (kHold * kMaxThreads);
  p.slice = ((C + p.cl - 1) / p.cl + kHold - 1) / kHold * kHold;
  p.cl = (C + p.slice - 1) / p.slice;
  const int need = (std::min(C, p.slice) + kHold - 1) / kHold;
  p.T = 1;
  while (p.T < need && p.T < 32) p.T *= 2;
  if (need > 32) p.T = (need + 31) / 32 * 32;
  p.teams = std::max(1, 256 / (p.T < 32 ? p.T : (p.T + 31) / 32 * 32));
  const int threads = p.T * p.teams;
  const int64_t slots = (int64_t)kNumSMs * std::max(1, threads_per_sm / threads);
  const int64_t most = std::max<int64_t>(1, slots / ((int64_t)G * p.cl));
  const int64_t turns = (R + p.teams - 1) / p.teams;  // of a CTA's teams, if there were one CTA
  p.rows = std::max<int64_t>(1, (turns + most - 1) / most);
  p.ranges = (turns + p.rows - 1) / p.rows;
  return p;
}

__device__ __forceinline__ void team_barrier(int id, int threads) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void store_peer(const float4* at, int rank, float4 v) {
  uint32_t p;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(p) : "r"(smem_u32(at)), "r"(rank));
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(p), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}

// A thread's place, and what its team shares.
struct Team {
  int T, t, team, lane, warps, warp, cl, rank, slots;
  int col0, Cs;  // the CTA's columns
  int n;         // the warp's (or smaller team's) columns
  __device__ __forceinline__ Team(const LnArgs& a, int vec) {
    T = a.T, team = threadIdx.x / T, t = threadIdx.x - team * T, lane = threadIdx.x & 31;
    warps = T < 32 ? 1 : T / 32, warp = T < 32 ? 0 : t / 32;
    cl = a.cl;
    rank = 0;
    if (cl > 1) asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    slots = warps * cl;
    col0 = rank * a.slice, Cs = min(a.slice, a.C - col0);
    n = Cs;
    if (T > 32) {
      n = 0;
      for (int j = 0; j < kHold / vec; ++j) n += min(32 * vec, max(0, Cs - (j * T + warp * 32) * vec));
    }
  }
  __device__ __forceinline__ float sum(float v) const {  // over the warp, or over the team within it
    for (int d = min(T, 32) / 2; d; d /= 2) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
  }
  // Every warp's v to every warp of the row, in `stat` [slots] (the team's, one of two that take turns).
  __device__ __forceinline__ void share(float4* stat, float4 v) const {
    if (cl == 1) {
      if (lane == 0) stat[warp] = v;
      team_barrier(team + 1, T);
    } else {
      if (lane < cl) store_peer(stat + rank * warps + warp, lane, v);
      cluster_arrive();
      cluster_wait();
    }
  }
  // f(slot) over the slots, summed in an order of its own that is the same in every thread.
  template <typename F>
  __device__ __forceinline__ float over(F f) const {
    float v = 0.f;
    if (slots <= 8) {
      for (int i = 0; i < slots; ++i) v += f(i);
      return v;
    }
    for (int i = lane; i < slots; i += 32) v += f(i);
    for (int d = 16; d; d /= 2) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
  }
};

// ---- forward ----
template <typename XT, typename YT, int V, bool RES>
__global__ void __launch_bounds__(kMaxThreads) ln_forward_kernel(const LnArgs a) {
  constexpr int N = kHold / V;
  __shared__ float4 stats[2][kMaxThreads / 32 * kMaxCluster];
  const Team m(a, V);
  if (m.cl > 1) {  // every CTA's shared memory is there from here on
    cluster_arrive();
    cluster_wait();
  }
  pdl_begin();
  const int g = blockIdx.y;
  const int64_t step = (int64_t)(gridDim.x / m.cl) * a.teams, first = (int64_t)(blockIdx.x / m.cl) * a.teams;
  int left[N];
  float ga[N][V], be[N][V];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int c = (j * m.T + m.t) * V;
    left[j] = m.Cs - c;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const bool in = i < left[j];
      ga[j][i] = in ? __ldg(a.gamma + g * a.par_gs + m.col0 + c + i) : 0.f;
      be[j][i] = in ? __ldg(a.beta + g * a.par_gs + m.col0 + c + i) : 0.f;
    }
  }
  const int64_t at0 = m.col0 + m.t * V, hop = m.T * V;
  const XT* x = static_cast<const XT*>(a.x) + (int64_t)g * a.R * a.x_ld + at0;
  const XT* res = static_cast<const XT*>(a.r) + (int64_t)g * a.R * a.x_ld + at0;
  Vec<XT, V> rx[N], rr[N];
  const auto fetch = [&](int64_t row) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int l = row < a.R ? left[j] : 0;
      rx[j].zero();
      if (l > 0) rx[j].load_first(x + row * a.x_ld + j * hop, l);
      if constexpr (RES) {
        rr[j].zero();
        if (l > 0) rr[j].load_first(res + row * a.x_ld + j * hop, l);
      }
    }
  };
  // (the rows of a warp's teams lie next to one another: its first one tells whether any is left)
  const int lead = m.T < 32 ? (threadIdx.x & ~31) / m.T : m.team;
  int64_t row = first + m.team;
  fetch(row);
  for (int64_t base = first + lead, k = 0; base < a.R; base += step, row += step, ++k) {
    const bool on = row < a.R;
    float v[N][V];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      rx[j].floats(v[j]);
      if constexpr (RES) {
        float q[V];
        rr[j].floats(q);
#pragma unroll
        for (int i = 0; i < V; ++i) v[j][i] += q[i];
        Vec<XT, V> o;
        o.set(v[j]);
        o.floats(v[j]);
        if (on && left[j] > 0) o.store_first(static_cast<XT*>(a.s) + ((int64_t)g * a.R + row) * a.x_ld + at0 + j * hop, left[j]);
      }
    }
    fetch(row + step);
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) s += v[j][i];
    s = m.sum(s);
    float mean = m.n ? s / m.n : 0.f, q = 0.f;
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float d = i < left[j] ? v[j][i] - mean : 0.f;
        q = fmaf(d, d, q);
      }
    q = m.sum(q);
    if (m.slots > 1) {
      float4* stat = stats[k & 1] + m.team * m.warps;
      m.share(stat, make_float4(s, mean, q, (float)m.n));
      mean = m.over([&](int i) { return stat[i].x; }) / a.C;
      q = m.over([&](int i) {
        const float4 f = stat[i];
        const float d = f.y - mean;
        return fmaf(f.w * d, d, f.z);
      });
    }
    const float rstd = rsqrtf(q / a.C + a.eps);
    if (!on) continue;
    if (m.t == 0 && m.rank == 0) {
      a.mean[(int64_t)g * a.R + row] = mean;
      a.rstd[(int64_t)g * a.R + row] = rstd;
    }
    YT* y = static_cast<YT*>(a.out) + ((int64_t)g * a.R + row) * a.y_ld + at0;
    with_act(a.act, [&](auto act) {
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (left[j] > 0) {
          float z[V];
#pragma unroll
          for (int i = 0; i < V; ++i)
            z[i] = activate<sizeof(YT) == 2 ? kFast : kExact, decltype(act)::value>(fmaf((v[j][i] - mean) * rstd, ga[j][i], be[j][i]));
          Vec<YT, V> o;
          o.set(z);
          o.store_first(y + j * hop, left[j]);
        }
    });
  }
}

// ---- backward ----
template <typename XT, typename YT, int V, bool RES>
__global__ void __launch_bounds__(kMaxThreads) ln_backward_kernel(const LnArgs a) {
  constexpr int N = kHold / V;
  __shared__ float4 stats[2][kMaxThreads / 32 * kMaxCluster];
  extern __shared__ float sums[];  // [2 kHold][threads]
  const Team m(a, V);
  if (m.cl > 1) {
    cluster_arrive();
    cluster_wait();
  }
  pdl_begin();
  const int g = blockIdx.y, tid = threadIdx.x, threads = blockDim.x;
  const int64_t ranges = gridDim.x / m.cl, range = blockIdx.x / m.cl;
  const int64_t step = ranges * a.teams, first = range * a.teams;
  const bool relu = a.act == LSGD_ACT_RELU, silu = a.act == LSGD_ACT_SILU;
  int left[N];
  float ga[N][V], be[N][V], dga[N][V], dbe[N][V];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int c = (j * m.T + m.t) * V;
    left[j] = m.Cs - c;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const bool in = i < left[j];
      ga[j][i] = in ? __ldg(a.gamma + g * a.par_gs + m.col0 + c + i) : 0.f;
      be[j][i] = in ? __ldg(a.beta + g * a.par_gs + m.col0 + c + i) : 0.f;
      dga[j][i] = dbe[j][i] = 0.f;
    }
  }
  const int64_t at0 = m.col0 + m.t * V, hop = m.T * V, xw = (int64_t)g * a.R * a.x_ld + at0, yw = (int64_t)g * a.R * a.y_ld + at0;
  Vec<XT, V> rx[N], rs[N];
  Vec<YT, V> rd[N], ry[N];
  float mean = 0.f, rstd = 0.f;
  const auto fetch = [&](int64_t row) {
    if (row < a.R) {
      mean = __ldg(a.mean + (int64_t)g * a.R + row);
      rstd = __ldg(a.rstd + (int64_t)g * a.R + row);
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int l = row < a.R ? left[j] : 0;
      const int64_t xo = xw + row * a.x_ld + j * hop, yo = yw + row * a.y_ld + j * hop;
      rx[j].zero();
      rd[j].zero();
      if (l > 0) {
        rx[j].load_first(static_cast<const XT*>(a.x) + xo, l);
        rd[j].load_first(static_cast<const YT*>(a.dy) + yo, l);
        if (relu) ry[j].load_first(static_cast<const YT*>(a.y) + yo, l);
        if constexpr (RES) rs[j].load_first(static_cast<const XT*>(a.ds) + xo, l);
      }
    }
  };
  const int lead = m.T < 32 ? (tid & ~31) / m.T : m.team;
  int64_t row = first + m.team;
  fetch(row);
  int run = 0;        // rows in the registers' sums
  bool more = false;  // earlier segments' sums stand in this thread's places of `sums`
  const auto flush = [&] {
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float &p = sums[(j * V + i) * threads + tid], &q = sums[(kHold + j * V + i) * threads + tid];
        if (more) dga[j][i] += p, dbe[j][i] += q;
        p = dga[j][i], q = dbe[j][i];
        dga[j][i] = dbe[j][i] = 0.f;
      }
    more = true;
    run = 0;
  };
  for (int64_t base = first + lead, k = 0; base < a.R; base += step, row += step, ++k) {
    const bool on = row < a.R;
    const float rs_row = rstd;
    float xh[N][V], t[N][V], e[N][V];  // t: gamma dz; e: ds
    float m1 = 0.f, m2 = 0.f;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      float d[V];
      rx[j].floats(xh[j]);
      rd[j].floats(d);
      if constexpr (RES) rs[j].floats(e[j]);
#pragma unroll
      for (int i = 0; i < V; ++i) xh[j][i] = i < left[j] && on ? (xh[j][i] - mean) * rstd : 0.f;
      if (relu) {
        float y[V];
        ry[j].floats(y);
#pragma unroll
        for (int i = 0; i < V; ++i) d[i] = y[i] > 0.f ? d[i] : 0.f;
      } else if (silu) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float z = fmaf(xh[j][i], ga[j][i], be[j][i]), sg = sigmoid<sizeof(XT) == 4 ? kExact : kSums>(z);
          d[i] *= sg * fmaf(z, 1.f - sg, 1.f);
        }
      }
#pragma unroll
      for (int i = 0; i < V; ++i) {
        dbe[j][i] += d[i];
        dga[j][i] = fmaf(d[i], xh[j][i], dga[j][i]);
        t[j][i] = ga[j][i] * d[i];
        m1 += t[j][i];
        m2 = fmaf(t[j][i], xh[j][i], m2);
      }
    }
    fetch(row + step);
    m1 = m.sum(m1);
    m2 = m.sum(m2);
    if (m.slots > 1) {
      float4* stat = stats[k & 1] + m.team * m.warps;
      m.share(stat, make_float4(m1, m2, 0.f, 0.f));
      m1 = m.over([&](int i) { return stat[i].x; });
      m2 = m.over([&](int i) { return stat[i].y; });
    }
    m1 /= a.C;
    m2 /= a.C;
    if (on) {
      XT* dx = static_cast<XT*>(a.out) + xw + row * a.x_ld;
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (left[j] > 0) {
          float o[V];
#pragma unroll
          for (int i = 0; i < V; ++i) {
            o[i] = rs_row * (t[j][i] - m1 - xh[j][i] * m2);
            if constexpr (RES) o[i] += e[j][i];
          }
          Vec<XT, V> q;
          q.set(o);
          q.store_first(dx + j * hop, left[j]);
        }
    }
    if (++run == a.seg) flush();
  }
  if (more || a.teams > 1) flush();
  // halves of the teams are merged until one is left
  if (a.teams > 1) {
    for (int half = 1; half < a.teams; half *= 2) {
      __syncthreads();
      const int o = tid + half * m.T;
      if (m.team % (2 * half) == 0 && m.team + half < a.teams) {
#pragma unroll
        for (int i = 0; i < 2 * kHold; ++i) sums[i * threads + tid] += sums[i * threads + o];
      }
    }
    if (m.team) return;
  }
  float *pg = a.dgamma + g * a.par_gs, *pb = a.dbeta + g * a.par_gs;
  if (ranges > 1) {
    pg = a.part + ((int64_t)g * ranges + range) * 2 * a.C;
    pb = pg + a.C;
  }
  const bool kept = more || a.teams > 1;
#pragma unroll
  for (int j = 0; j < N; ++j)
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < left[j]) {
        const int c = m.col0 + (j * m.T + m.t) * V + i;
        pg[c] = kept ? sums[(j * V + i) * threads + tid] : dga[j][i];
        pb[c] = kept ? sums[(kHold + j * V + i) * threads + tid] : dbe[j][i];
      }
}

// dgamma and dbeta from the ranges' sums part [G][ranges][2][C] (none: zeros).  32 columns of a worker to a block; each of 32 rows of
// threads adds every 32nd range, and these are added in pairs.
__global__ void __launch_bounds__(1024) ln_param_grad_kernel(const float* part, int ranges, int C, int64_t par_gs, float* dgamma,
                                                              float* dbeta) {
  pdl_begin();
  __shared__ float red[32][33];
  const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5, c = blockIdx.x * 32 + tx, g = blockIdx.y, which = blockIdx.z;
  const float* p = part + ((int64_t)g * ranges * 2 + which) * C + c;
  float v = 0.f;
  if (c < C) {
#pragma unroll 4
    for (int i = ty; i < ranges; i += 32) v += __ldg(p + (int64_t)i * 2 * C);
  }
  red[tx][ty] = v;
  __syncthreads();
  v = red[ty][tx];
  for (int d = 16; d; d /= 2) v += __shfl_xor_sync(0xffffffffu, v, d);
  const int col = blockIdx.x * 32 + ty;
  if (tx == 0 && col < C) (which ? dbeta : dgamma)[g * par_gs + col] = v;
}

constexpr int kFwdThreadsPerSm = 1536, kBwdThreadsPerSm = 768;

template <typename K>
cudaError_t ln_launch(K kernel, const LnArgs& a, dim3 grid, size_t smem, cudaStream_t st) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(a.T * a.teams);
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
  if (a.cl > 8) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
  }
  return cudaLaunchKernelEx(&cfg, kernel, a);
}

template <typename XT, typename YT, int V, bool BWD>
cudaError_t ln_form(LnArgs a, int G, cudaStream_t st) {
  const LnPlan p = ln_plan(G, a.R, a.C, BWD ? kBwdThreadsPerSm : kFwdThreadsPerSm);
  a.T = p.T, a.teams = p.teams, a.cl = p.cl, a.slice = p.slice;
  a.seg = 64;
  const dim3 grid((unsigned)(p.ranges * p.cl), G);
  cudaError_t e = cudaSuccess;
  if constexpr (!BWD) {
    if (a.R == 0) return e;
    return a.r ? ln_launch(ln_forward_kernel<XT, YT, V, true>, a, grid, 0, st)
               : ln_launch(ln_forward_kernel<XT, YT, V, false>, a, grid, 0, st);
  } else {
    const size_t smem = p.teams > 1 || p.rows >= a.seg ? 2 * kHold * 4 * (size_t)(p.T * p.teams) : 0;
    if (a.R)
      e = a.ds ? ln_launch(ln_backward_kernel<XT, YT, V, true>, a, grid, smem, st)
               : ln_launch(ln_backward_kernel<XT, YT, V, false>, a, grid, smem, st);
    if (e != cudaSuccess || p.ranges == 1) return e;
    return launch_pdl(ln_param_grad_kernel, dim3((a.C + 31) / 32, G, 2), dim3(1024), 0, st, (const float*)a.part, (int)p.ranges, a.C,
                      a.par_gs, a.dgamma, a.dbeta);
  }
}

template <typename XT, typename YT, bool BWD>
cudaError_t ln_vector(const LnArgs& a, int G, int vmax, cudaStream_t st) {
  if constexpr (sizeof(XT) == 2 && sizeof(YT) == 2) {
    if (vmax >= 8) return ln_form<XT, YT, 8, BWD>(a, G, st);
  }
  if (vmax >= 4) return ln_form<XT, YT, 4, BWD>(a, G, st);
  if (vmax >= 2) return ln_form<XT, YT, 2, BWD>(a, G, st);
  return ln_form<XT, YT, 1, BWD>(a, G, st);
}
template <bool BWD>
cudaError_t ln_typed(const LnArgs& a, int G, bool xb, bool yb, int vmax, cudaStream_t st) {
  if (xb) return yb ? ln_vector<uint16_t, uint16_t, BWD>(a, G, vmax, st) : ln_vector<uint16_t, float, BWD>(a, G, vmax, st);
  return yb ? ln_vector<float, uint16_t, BWD>(a, G, vmax, st) : ln_vector<float, float, BWD>(a, G, vmax, st);
}

// The widest vector (a power of two of values, at most v) with which rows of stride ld from p on (values of z bytes) are aligned.
int ln_vec(int v, int64_t rows, int64_t ld, const void* p, int z) {
  while (v > 1 && ((rows > 1 && ld % v) || reinterpret_cast<uintptr_t>(p) % std::min(16, v * z))) v >>= 1;
  return v;
}

size_t ln_workspace(int G, int64_t R, int C) {
  const LnPlan p = ln_plan(G, R, C, kBwdThreadsPerSm);
  return p.ranges > 1 ? (size_t)G * p.ranges * C * 8 : 0;
}

const char* ln_shape_error(int G, int64_t R, int64_t C) {
  if (G < 1 || C < 1 || R < 0) return "G and C must be at least 1, R at least 0";
  if (G > 65535 || C > kMaxC || R > ((int64_t)1 << 40) / G) return "at most 65535 workers, 2^40 rows (G R) and 65536 values a row";
  return nullptr;
}
// Rows of stride ld whose values' addresses are whole numbers.
bool ln_bad_ld(int G, int64_t R, int64_t C, int64_t ld) {
  const int64_t rows = (int64_t)G * R;
  return ld < C || (rows > 1 && ld > ((int64_t)1 << 60) / rows);
}
lsgd_status ln_error(lsgd_status s, const char* fn, const char* what) {
  set_last_error(std::string(fn) + ": " + what);
  return s;
}

}  // namespace
}  // namespace lsgd

extern "C" {

lsgd_status lsgd_layernorm_workspace(int G, int64_t R, int64_t C, size_t* bytes) {
  using namespace lsgd;
  const char* bad = ln_shape_error(G, R, C);
  if (!bad && !bytes) bad = "bytes is NULL";
  if (bad) return ln_error(LSGD_EINVAL, "lsgd_layernorm_workspace", bad);
  *bytes = ln_workspace(G, R, (int)C);
  return LSGD_OK;
}

lsgd_status lsgd_layernorm_forward(const void* x, const void* r, int x_type, int64_t x_ld, const float* gamma, const float* beta,
                                   int64_t par_gs, void* s, void* y, int y_type, int64_t y_ld, float* mean, float* rstd, int G,
                                   int64_t R, int64_t C, float eps, int act, void* stream) {
  using namespace lsgd;
  const char* fn = "lsgd_layernorm_forward";
  const char* bad = ln_shape_error(G, R, C);
  if (bad) return ln_error(LSGD_EINVAL, fn, bad);
  const bool xb = x_type == LSGD_BF16, yb = y_type == LSGD_BF16;
  const int xz = xb ? 2 : 4, yz = yb ? 2 : 4;
  const int64_t N = (int64_t)G * R;
  if (ln_bad_ld(G, R, C, x_ld) || ln_bad_ld(G, R, C, y_ld)) bad = "x_ld and y_ld must be at least C (and addresses fit 64 bits)";
  else if (N && (!x || !gamma || !beta || !y || !mean || !rstd)) bad = "a pointer is NULL";
  else if (!r != !s) bad = "r and s come together";
  else if ((!xb && x_type != LSGD_FP32) || (!yb && y_type != LSGD_FP32)) bad = "types are LSGD_FP32 or LSGD_BF16";
  else if (act != LSGD_ACT_NONE && act != LSGD_ACT_RELU && act != LSGD_ACT_SILU) bad = "unknown activation";
  else if (!(eps > 0.f) || !(eps < 1e30f)) bad = "eps must be positive and finite";
  else if (par_gs < C) bad = "par_gs must be at least C";
  else if (misaligned(x, xz) || misaligned(r, xz) || misaligned(s, xz) || misaligned(y, yz) || misaligned(gamma, 4) ||
           misaligned(beta, 4) || misaligned(mean, 4) || misaligned(rstd, 4))
    bad = "a pointer is not aligned to its element";
  if (bad) return ln_error(LSGD_EINVAL, fn, bad);
  if (N == 0) return LSGD_OK;
  const size_t nx = (size_t)((N - 1) * x_ld + C) * xz, ny = (size_t)((N - 1) * y_ld + C) * yz, ns = (size_t)N * 4;
  const auto params = [&](const float* p) { return Blocks(p, 4 * (size_t)C, par_gs, G); };
  if (any_overlap({Blocks(y, ny), Blocks(s, nx), Blocks(mean, ns), Blocks(rstd, ns)},
                  {Blocks(x, nx), Blocks(r, nx), params(gamma), params(beta)}))
    return ln_error(LSGD_EINVAL, fn, "tensors overlap");
  LnArgs a{};
  a.x = x, a.r = r, a.s = s, a.out = y, a.gamma = gamma, a.beta = beta, a.par_gs = par_gs, a.mean = mean, a.rstd = rstd;
  a.R = R, a.x_ld = x_ld, a.y_ld = y_ld, a.C = (int)C, a.act = act, a.eps = eps;
  int v = ln_vec(ln_vec(xb && yb ? 8 : 4, N, x_ld, x, xz), N, y_ld, y, yz);
  if (r) v = ln_vec(ln_vec(v, N, x_ld, r, xz), N, x_ld, s, xz);
  const cudaError_t e = ln_typed<false>(a, G, xb, yb, v, (cudaStream_t)stream);
  return e == cudaSuccess ? LSGD_OK : ln_error(LSGD_ECUDA, fn, cudaGetErrorString(e));
}

lsgd_status lsgd_layernorm_backward(const void* x, int x_type, int64_t x_ld, const void* y, const void* dy, int y_type, int64_t y_ld,
                                    const void* ds, const float* gamma, const float* beta, int64_t par_gs, const float* mean,
                                    const float* rstd, void* dx, float* dgamma, float* dbeta, int G, int64_t R, int64_t C, int act,
                                    void* workspace, size_t workspace_bytes, void* stream) {
  using namespace lsgd;
  const char* fn = "lsgd_layernorm_backward";
  const char* bad = ln_shape_error(G, R, C);
  if (bad) return ln_error(LSGD_EINVAL, fn, bad);
  const bool xb = x_type == LSGD_BF16, yb = y_type == LSGD_BF16, relu = act == LSGD_ACT_RELU;
  const int xz = xb ? 2 : 4, yz = yb ? 2 : 4;
  const int64_t N = (int64_t)G * R;
  const size_t need = ln_workspace(G, R, (int)C);
  if (ln_bad_ld(G, R, C, x_ld) || ln_bad_ld(G, R, C, y_ld)) bad = "x_ld and y_ld must be at least C (and addresses fit 64 bits)";
  else if (!gamma || !beta || !dgamma || !dbeta) bad = "a pointer is NULL";
  else if (N && (!x || !dy || !mean || !rstd || !dx || (relu && !y)))
    bad = "a pointer is NULL (y may be only where the activation is not ReLU)";
  else if ((!xb && x_type != LSGD_FP32) || (!yb && y_type != LSGD_FP32)) bad = "types are LSGD_FP32 or LSGD_BF16";
  else if (act != LSGD_ACT_NONE && !relu && act != LSGD_ACT_SILU) bad = "unknown activation";
  else if (par_gs < C) bad = "par_gs must be at least C";
  else if (misaligned(x, xz) || misaligned(dx, xz) || misaligned(ds, xz) || misaligned(dy, yz) || (relu && misaligned(y, yz)) ||
           misaligned(gamma, 4) || misaligned(beta, 4) || misaligned(mean, 4) || misaligned(rstd, 4) || misaligned(dgamma, 4) ||
           misaligned(dbeta, 4))
    bad = "a pointer is not aligned to its element";
  else if (need && (!workspace || workspace_bytes < need || misaligned(workspace, 16)))
    bad = "workspace NULL, not 16-byte aligned or smaller than lsgd_layernorm_workspace says";
  if (bad) return ln_error(LSGD_EINVAL, fn, bad);
  const size_t nx = N ? (size_t)((N - 1) * x_ld + C) * xz : 0, ny = N ? (size_t)((N - 1) * y_ld + C) * yz : 0, ns = (size_t)N * 4;
  const auto rows = [&](const void* p, size_t n) { return Blocks(N ? p : nullptr, n); };
  const auto params = [&](const float* p) { return Blocks(p, 4 * (size_t)C, par_gs, G); };
  if (any_overlap({rows(dx, nx), params(dgamma), params(dbeta), Blocks(need ? workspace : nullptr, need)},
                  {rows(x, nx), rows(dy, ny), rows(ds, nx), rows(relu ? y : nullptr, ny), params(gamma), params(beta),
                   rows(mean, ns), rows(rstd, ns)}))
    return ln_error(LSGD_EINVAL, fn, "tensors overlap");
  LnArgs a{};
  a.x = x, a.y = y, a.dy = dy, a.ds = ds, a.out = dx, a.gamma = gamma, a.beta = beta, a.par_gs = par_gs;
  a.mean = const_cast<float*>(mean), a.rstd = const_cast<float*>(rstd), a.dgamma = dgamma, a.dbeta = dbeta;
  a.part = static_cast<float*>(workspace);
  a.R = R, a.x_ld = x_ld, a.y_ld = y_ld, a.C = (int)C, a.act = act;
  int v = ln_vec(ln_vec(ln_vec(xb && yb ? 8 : 4, N, x_ld, x, xz), N, x_ld, dx, xz), N, y_ld, dy, yz);
  if (relu) v = ln_vec(v, N, y_ld, y, yz);
  if (ds) v = ln_vec(v, N, x_ld, ds, xz);
  const cudaError_t e = ln_typed<true>(a, G, xb, yb, v, (cudaStream_t)stream);
  return e == cudaSuccess ? LSGD_OK : ln_error(LSGD_ECUDA, fn, cudaGetErrorString(e));
}

}  // extern "C"
