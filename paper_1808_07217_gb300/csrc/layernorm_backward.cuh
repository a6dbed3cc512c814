// Layer norm's backward pass (layernorm.cu has the formulas).  A thread keeps its columns' parts of dgamma and dbeta over all rows of
// its team; a CTA's teams are added at the end, and the CTAs of a worker by a second kernel, in a fixed order.
#pragma once
#include "layernorm.cuh"

namespace lsgd {
namespace {

// Where a slot's inputs and what follows the slots stand in shared memory.  E: values of a row in a thread.
template <typename XT, typename YT, int V, bool RES, int ACT, int E, bool CLUSTER>
struct BwdShape {
  static constexpr int N = E / V;
  using X = Feed<XT, V, N, CLUSTER>;
  using Y = Feed<YT, V, N, CLUSTER>;
  static constexpr int kDy = X::kSlot, kY = kDy + Y::kSlot, kDs = kY + (ACT == LSGD_ACT_RELU ? Y::kSlot : 0),
                       kSlot = kDs + (RES ? X::kSlot : 0);
  static constexpr int kBetas = ACT == LSGD_ACT_SILU ? 4 * E * kThreads : 0, kSums = 8 * E * kThreads;
};

// CLUSTER: as in the forward, the sums of row k + 1 are sent before those of row k are waited for; row k is read once more.
template <typename XT, typename YT, int V, bool RES, int ACT, int E, bool CLUSTER>
__global__ void __launch_bounds__(kThreads, 2) ln_backward_kernel(const LnArgs a) {
  using M = Team<CLUSTER>;
  using S = BwdShape<XT, YT, V, RES, ACT, E, CLUSTER>;
  constexpr int N = S::N, H = E / 2;
  constexpr bool RELU = ACT == LSGD_ACT_RELU, SILU = ACT == LSGD_ACT_SILU;
  __shared__ float2 stats[M::kPlaces];
  extern __shared__ __align__(16) uint8_t ring[];
  __shared__ uint64_t bars[M::kTurns];
  M m(a, V, N, bars);
  m.begin();
  pdl_begin();
  const int64_t ranges = gridDim.x / m.cl, range = blockIdx.x / m.cl;
  const Rows rows(a, m, ranges, range);
  const int hop = m.T * V, left = m.Cs - m.t * V;  // from a vector to the thread's next one; columns from its first one on
  const bool whole = __all_sync(0xffffffffu, left >= (N - 1) * hop + V);
  const int at0 = m.col0 + m.t * V;
  const int64_t x_step = rows.step * a.x_ld, y_step = rows.step * a.y_ld;
  const int64_t x0 = rows.row * a.x_ld + at0, y0 = rows.row * a.y_ld + at0;
  const uint32_t base = smem_u32(ring);
  typename S::X fx, fs;
  typename S::Y fd, fy;
  fx.init(a.x, x0, base);
  fd.init(a.dy, y0, base + S::kDy);
  if (RELU) fy.init(a.y, y0, base + S::kY);
  if (RES) fs.init(a.ds, x0, base + S::kDs);
  const auto fetch = [&](int k, uint32_t slot) {
    const bool on = k < rows.mine, w = whole && on;
    const int l = on ? left : 0;
    fx.fetch(w, l, hop, slot, a.x, x_step);
    fd.fetch(w, l, hop, slot, a.dy, y_step);
    if (RELU) fy.fetch(w, l, hop, slot, a.dy, y_step);
    if (RES) fs.fetch(w, l, hop, slot, a.x, x_step);
    copies_issued();
  };
  const auto land = [&](uint32_t slot) {
    fx.land(slot);
    fd.land(slot);
    if (RELU) fy.land(slot);
    if (RES) fs.land(slot);
  };
  int64_t row = rows.row;
  float next_mean, next_rstd;
  const auto fetch_stats = [&](int k) {
    next_mean = next_rstd = 0.f;
    if (k < rows.mine) {  // (volatile: issued here, not where they are used)
      asm volatile("ld.global.nc.f32 %0, [%1];" : "=f"(next_mean) : "l"(a.mean + row) : "memory");
      asm volatile("ld.global.nc.f32 %0, [%1];" : "=f"(next_rstd) : "l"(a.rstd + row) : "memory");
    }
    row += rows.step;
  };
  uint32_t slot = 0, next = 0;
  const int early = a.ahead + (CLUSTER ? 1 : 0);
  for (int d = 0; d < early; ++d, next += S::kSlot) {
    fetch(d, next);
    land(next);
  }
  const uint32_t last = next;
  const auto advance = [&](uint32_t& s) { s = s == last ? 0 : s + S::kSlot; };
  fetch_stats(0);
  u64 ga[H], dga[H], dbe[H];
  load_params<V, N>(a.gamma + blockIdx.y * a.par_gs + m.col0, m, ga);
  u64* betas = reinterpret_cast<u64*>(ring + last + S::kSlot) + threadIdx.x;  // [H][kThreads], for SiLU
  if (SILU) {
    u64 be[H];
    load_params<V, N>(a.beta + blockIdx.y * a.par_gs + m.col0, m, be);
#pragma unroll
    for (int i = 0; i < H; ++i) betas[i * kThreads] = be[i];
  }
#pragma unroll
  for (int i = 0; i < H; ++i) dga[i] = dbe[i] = 0;
  float* sums = reinterpret_cast<float*>(ring + a.sums) + threadIdx.x;  // [2 E][kThreads]
  int run = 0;        // rows in the registers' sums
  bool more = false;  // earlier segments' sums stand in this thread's places of `sums`
  const auto flush = [&] {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      float &p = sums[e * kThreads], &q = sums[(E + e) * kThreads];
      const float2 dg = unpack2(dga[e / 2]), db = unpack2(dbe[e / 2]);
      p = (more ? p : 0.f) + (e & 1 ? dg.y : dg.x);
      q = (more ? q : 0.f) + (e & 1 ? db.y : db.x);
    }
#pragma unroll
    for (int i = 0; i < H; ++i) dga[i] = dbe[i] = 0;
    more = true;
    run = 0;
  };
  const float inv = -1.f / a.C;
  XT* out = static_cast<XT*>(a.out) + x0;
  // A row's xh and dz; what lies behind its end has dz = 0.
  const auto values = [&](uint32_t slot, float mean, float rstd, u64 (&xh)[H], u64 (&t)[H], u64 (&y)[H]) {
    fx.read(slot, xh);
    fd.read(slot, t);
    if constexpr (RELU) {
      fy.read(slot, y);
#pragma unroll
      for (int i = 0; i < H; ++i) {
        const float2 f = unpack2(y[i]), d = unpack2(t[i]);
        t[i] = pack2(f.x > 0.f ? d.x : 0.f, f.y > 0.f ? d.y : 0.f);
      }
    }
#pragma unroll
    for (int i = 0; i < H; ++i) {
      xh[i] = mul2(sum2(xh[i], both(-mean)), both(rstd));
      if constexpr (SILU) {
        constexpr int kind = sizeof(XT) == 4 ? kClose : kSums;
        const float2 z = unpack2(mad2(xh[i], ga[i], betas[i * kThreads])), d = unpack2(t[i]);
        const float p = sigmoid<kind>(z.x), q = sigmoid<kind>(z.y);
        t[i] = pack2(d.x * p * fmaf(z.x, 1.f - p, 1.f), d.y * q * fmaf(z.y, 1.f - q, 1.f));
      }
    }
  };
  // Adds a row to dgamma and dbeta; t = gamma dz and its sums s1 and, with xh, s2.
  const auto add = [&](u64 (&xh)[H], u64 (&t)[H], float& m1, float& m2) {
    u64 s1 = 0, s2 = 0;
#pragma unroll
    for (int i = 0; i < H; ++i) {
      add2(dbe[i], t[i]);
      dga[i] = mad2(t[i], xh[i], dga[i]);
      t[i] = mul2(t[i], ga[i]);
      add2(s1, t[i]);
      s2 = mad2(t[i], xh[i], s2);
    }
    m1 = added(s1), m2 = added(s2);
  };
  const auto finish = [&](bool on, uint32_t slot, u64 (&xh)[H], u64 (&t)[H], u64 (&e)[H], float m1, float m2, float rstd) {
    m1 *= inv, m2 *= inv;
    if constexpr (RES) fs.read(slot, e);
#pragma unroll
    for (int i = 0; i < H; ++i) {
      t[i] = mad2(xh[i], both(m2), sum2(t[i], both(m1)));
      t[i] = RES ? mad2(t[i], both(rstd), e[i]) : mul2(t[i], both(rstd));
    }
    if (on) store_row<XT, V, N>(t, out, whole, left, hop);
    out += x_step;
  };
  if constexpr (!CLUSTER) {
    for (int k = 0; k < rows.turns; ++k, advance(slot), advance(next)) {
      const float mean = next_mean, rstd = next_rstd;
      u64 xh[H], t[H], y[H], e[H];
      fx.take(xh);
      fd.take(t);
      if (RELU) fy.take(y);
      if (RES) fs.take(e);
      fetch(k + a.ahead, next);
      fetch_stats(k + 1);
      copies_wait(a.ahead);
      float m1, m2;
      values(slot, mean, rstd, xh, t, y);
      add(xh, t, m1, m2);
      if (m.slots > 1) {
        m.post_both(m1, m2, stats, k);
        m.collect_both(m1, m2, stats, k);
      } else {
        m.sum_both(m1, m2);
      }
      finish(k < rows.mine, slot, xh, t, e, m1, m2, rstd);
      if (++run == a.seg) flush();
    }
  } else {
    uint32_t before = 0, coming = 0;  // the places of row k - 1, and of the row that was fetched last
    float mean = 0.f, rstd = 0.f;     // of row k - 1
    for (int k = 0; k <= rows.turns; ++k) {
      u64 xh[H], t[H], y[H], e[H];
      float m1, m2;
      const float old_mean = mean, old_rstd = rstd;
      if (k < rows.turns) {
        mean = next_mean, rstd = next_rstd;
        fetch_stats(k + 1);
        copies_wait(a.ahead);
        values(slot, mean, rstd, xh, t, y);
        add(xh, t, m1, m2);
        m.post_both(m1, m2, stats, k);
        if (++run == a.seg) flush();
      }
      if (k) {
        land(coming);
        values(before, old_mean, old_rstd, xh, t, y);
#pragma unroll
        for (int i = 0; i < H; ++i) t[i] = mul2(t[i], ga[i]);
        m.collect_both(m1, m2, stats, k - 1);
        finish(true, before, xh, t, e, m1, m2, old_rstd);
      }
      fetch(k + early, next);
      before = slot, coming = next;
      advance(slot);
      advance(next);
    }
    m.end();
  }
  // (the sums may stand where the rows did: every thread's copies are there, and read, before any is overwritten)
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();
  const bool kept = more || a.teams > 1;
  if (kept) flush();
  // halves of the teams are merged until one is left
  if (a.teams > 1) {
    for (int half = 1; half < a.teams; half *= 2) {
      __syncthreads();
      if (m.team % (2 * half) == 0 && m.team + half < a.teams) {
#pragma unroll
        for (int i = 0; i < 2 * E; ++i) sums[i * kThreads] += sums[i * kThreads + half * m.T];
      }
    }
    if (m.team) return;
  }
  float *pg = a.dgamma + blockIdx.y * a.par_gs, *pb = a.dbeta + blockIdx.y * a.par_gs;
  if (ranges > 1) {
    pg = a.part + (blockIdx.y * ranges + range) * 2 * a.C;
    pb = pg + a.C;
  }
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int c = (e / V * m.T + m.t) * V + e % V;
    if (c < m.Cs) {
      const float2 dg = unpack2(dga[e / 2]), db = unpack2(dbe[e / 2]);
      pg[m.col0 + c] = kept ? sums[e * kThreads] : e & 1 ? dg.y : dg.x;
      pb[m.col0 + c] = kept ? sums[(E + e) * kThreads] : e & 1 ? db.y : db.x;
    }
  }
}

// dgamma and dbeta from the ranges' sums part [G][ranges][2][C] (none: zeros).  TX columns of a worker to a block; each of its TY rows of
// threads adds every TY-th range, and these are added in pairs.
template <int TX, int TY>
__global__ void __launch_bounds__(TX * TY) ln_param_grad_kernel(const float* part, int ranges, int C, int64_t par_gs, float* dgamma,
                                                                 float* dbeta) {
  pdl_begin();
  const int tx = threadIdx.x % TX, ty = threadIdx.x / TX, c = blockIdx.x * TX + tx;
  const float* p = part + (int64_t)blockIdx.y * ranges * 2 * C + c;
  float2 v = make_float2(0.f, 0.f);
  if (c < C) {
#pragma unroll 8
    for (int i = ty; i < ranges; i += TY) {
      v.x += __ldg(p + (int64_t)i * 2 * C);
      v.y += __ldg(p + (int64_t)i * 2 * C + C);
    }
  }
  if constexpr (TY > 1) {
    __shared__ float2 red[TY][TX];
    for (int half = TY / 2; half; half /= 2) {
      red[ty][tx] = v;
      __syncthreads();
      if (ty < half) {
        v.x += red[ty + half][tx].x;
        v.y += red[ty + half][tx].y;
      }
      __syncthreads();
    }
  }
  if (ty == 0 && c < C) {
    dgamma[blockIdx.y * par_gs + c] = v.x;
    dbeta[blockIdx.y * par_gs + c] = v.y;
  }
}
// As few rows of threads as keep the SMs busy and no thread's chain above 64 ranges: with 32 for any number, 19 ranges of 16 x 4096
// columns took 20 us of idle threads, with 4, 3 ranges of 30 x 11,000 took 12 us.
inline cudaError_t launch_param_grads(const LnArgs& a, int G, int ranges, cudaStream_t st) {
  const auto run = [&](auto kernel, int tx, int ty) {
    return launch_pdl(kernel, dim3((a.C + tx - 1) / tx, G), dim3(tx * ty), 0, st, (const float*)a.part, ranges, a.C, a.par_gs, a.dgamma,
                      a.dbeta);
  };
  const int64_t columns = (int64_t)G * a.C;
  const auto enough = [&](int ty) { return ranges <= 4 * ty || (ranges <= 64 * ty && columns * ty >= kNumSMs * 512); };
  if (enough(1)) return run(ln_param_grad_kernel<128, 1>, 128, 1);
  if (enough(4)) return run(ln_param_grad_kernel<64, 4>, 64, 4);
  if (enough(16)) return run(ln_param_grad_kernel<32, 16>, 32, 16);
  return run(ln_param_grad_kernel<32, 32>, 32, 32);
}

template <typename XT, typename YT, int V, bool RES, int ACT, int E, bool CLUSTER>
cudaError_t ln_backward_as(LnArgs a, int G, cudaStream_t st) {
  static std::atomic<int> raised{0};  // device + 1 whose limits this kernel's have been raised to
  using S = BwdShape<XT, YT, V, RES, ACT, E, CLUSTER>;
  constexpr int more = CLUSTER ? 2 : 1, own = kStaticSmem<CLUSTER>;
  // as many CTAs to an SM as the shared memory takes with a row ahead
  const auto used = [](int ahead, bool apart) {
    const int rows = (ahead + more) * S::kSlot + S::kBetas;
    return own + (apart ? rows + S::kSums : std::max(rows, S::kSums));
  };
  static_assert(own + (1 + more) * S::kSlot + S::kBetas + S::kSums <= kSmemPerSm, "one CTA with a row ahead fits");
  const auto kernel = ln_backward_kernel<XT, YT, V, RES, ACT, E, CLUSTER>;
  const auto plan = [&](bool apart) {
    const int fit = std::max(1, kSmemPerSm / used(1, apart));
    LnPlan p = ln_plan(G, a.R, a.C, E, kFewRows, fit);
    if constexpr (CLUSTER) {
      static ClusterCounts counts;
      // A sixteenth fewer of more than two CTAs: behind the parameters' kernel they are not placed as densely as they could be
      // (2,000 x 17,000: 104 us with 58, 84 with 55; 3,000 x 9,000: 99 with 97, 72 with 92).
      const int n = ln_clusters(kernel, raised, counts, p.T * p.teams, used(1, apart) - own, p.cl);
      p = ln_plan(G, a.R, a.C, E, kFewRows, fit, p.cl > 2 ? n - n / 16 : n);
    }
    return p;
  };
  LnPlan p = plan(false);
  const bool apart = p.rows >= 64;  // sums that are added to while rows are under way
  if (apart) p = plan(true);
  a.seg = std::max(64, (int)std::ceil(std::sqrt((double)p.rows)));  // no chain of additions is longer than this
  const int threads = p.T * p.teams;
  const int per_sm = std::max(1, std::min(kThreadsPerSm / threads, kSmemPerSm / used(1, apart)));
  a.T = p.T, a.teams = p.teams, a.cl = p.cl, a.slice = p.slice, a.rows = (int)p.rows;
  a.ahead = S::X::kAsync && S::Y::kAsync && per_sm * used(2, apart) <= kSmemPerSm
                ? ln_ahead(p.rows, per_sm * threads, S::kSlot / kThreads) : 1;
  a.sums = apart ? (a.ahead + more) * S::kSlot + S::kBetas : 0;
  cudaError_t e = cudaSuccess;
  if (a.R)
    e = ln_launch(kernel, raised, a, dim3((unsigned)(p.ranges * p.cl), G), used(a.ahead, apart) - own, st);
  if (e != cudaSuccess || p.ranges == 1) return e;
  return launch_param_grads(a, G, (int)p.ranges, st);
}
// 16 values to a thread; 8 where all is fp32 and a CTA holds a row so or CTAs of 16 do not (as many bytes in shared memory), and where
// single bf16 values come through registers, but not where these are two at most and a cluster would be needed for a row that one CTA
// of 16 holds (8,000 x 3001, fp32 to bf16 with SiLU: 102 us, 127 in clusters; of four, 4,000 x 3333 took 134 us, 69 in clusters).
template <typename XT, typename YT, int V, bool RES, int ACT>
cudaError_t ln_backward(const LnArgs& a, int G, cudaStream_t st) {
  constexpr int single = (V * sizeof(XT) < 4 ? 1 + RES : 0) + (V * sizeof(YT) < 4 ? 1 + (ACT == LSGD_ACT_RELU) : 0);
  constexpr bool fp32 = sizeof(XT) + sizeof(YT) == 8, small = single || fp32;
  if constexpr (small) {
    if (a.C <= 8 * kThreads) return ln_backward_as<XT, YT, V, RES, ACT, 8, false>(a, G, st);
  }
  if constexpr (single <= 2) {
    if (a.C <= 16 * kThreads) return ln_backward_as<XT, YT, V, RES, ACT, 16, false>(a, G, st);
  }
  return ln_backward_as<XT, YT, V, RES, ACT, small ? 8 : 16, true>(a, G, st);
}

template <int ACT>
cudaError_t ln_backward_any(const LnArgs& a, int G, bool xb, bool yb, int vmax, cudaStream_t st) {
  return ln_dispatch(xb, yb, vmax, [&](auto xv, auto yv, auto vec) {
    using XT = decltype(xv);
    using YT = decltype(yv);
    constexpr int V = decltype(vec)::value;
    return a.ds ? ln_backward<XT, YT, V, true, ACT>(a, G, st) : ln_backward<XT, YT, V, false, ACT>(a, G, st);
  });
}

}  // namespace
}  // namespace lsgd
