// Layer normalisation of rows with an activation, and with the addition of a residual before it, forward and backward, for G
// workers of R rows of C values each.
//
// For a row x (and r, where there is a residual):
//   s = x + r (rounded to x's type),  mean = sum s / C,  rstd = 1 / sqrt(sum (s - mean)^2 / C + eps),
//   xh = (s - mean) rstd,  y = act(gamma xh + beta).
// Backward, with dz = dy act'(.), t = gamma dz, m1 and m2 the row's means of t and t xh:
//   dx = rstd (t - m1 - xh m2) + ds,  dgamma = sum dz xh,  dbeta = sum dz (over the worker's rows).
//
// Both are bound by memory.  A team of threads holds a row, E values to a thread (as vectors that lie next to one another across
// the team), so that every input is read once; a thread's columns stay the same from row to row, so that its parameters and
// the sums for dgamma and dbeta stay in registers.  A team is a part of a warp, a warp, several warps of a CTA, or the CTAs of a
// cluster, by the row's length; a CTA holds several teams where they are small.  Every thread copies its values of the next rows to
// shared memory while a row is reduced (cp.async, each thread its own, so that nothing but its own copies is waited for):
// as many bytes are under way as the memory's latency takes, at 16 warps to an SM.  What is the same for all values of a row (the
// exchanges, the barrier, the addresses) costs as many instructions as 16 values do, and the arithmetic is done on pairs
// (fma.rn.f32x2): with 8 values to a thread, single operations and the next row in registers the instructions bounded both
// (32,768 x 2048 in bf16 with a residual: 171 us forward, 200 us backward).
#include <string>

#include "layernorm.cuh"
#include "operands.h"

namespace lsgd {

int rows_take_timeout_flag() {
  return take_rows_late() | take_ln_backward_late_none() | take_ln_backward_late_relu() | take_ln_backward_late_silu();
}

namespace {

// ---- forward ----
// E: values of a row in a thread.  CLUSTER: a row's CTAs exchange their sums over the cluster's network, which takes about as long as a row:
// the sums of row k + 1 are formed and sent before those of row k are waited for, and row k is read from shared memory once more.
// (4 x 2,000 x 6,000 in bf16 with a residual: 110 us with the cluster's barrier in every row, 92 with the exchange alone, 86 so.)
template <typename XT, typename YT, int V, bool RES, int E, bool CLUSTER>
__global__ void __launch_bounds__(kThreads, 2) ln_forward_kernel(const LnArgs a) {
  constexpr int N = E / V, H = E / 2;
  using In = Feed<XT, V, N, CLUSTER>;
  using M = Team<CLUSTER>;
  constexpr uint32_t kSlotBytes = In::kSlot * (RES ? 2 : 1);
  __shared__ float4 stats[M::kPlaces];
  extern __shared__ __align__(16) uint8_t ring[];
  __shared__ uint64_t bars[M::kTurns];
  M m(a, V, N, bars);
  m.begin();
  pdl_begin();
  const Rows rows(a, m, gridDim.x / m.cl, blockIdx.x / m.cl);
  const int hop = m.T * V, left = m.Cs - m.t * V;  // from a vector to the thread's next one; columns from its first one on
  const bool whole = __all_sync(0xffffffffu, left >= (N - 1) * hop + V);
  const int at0 = m.col0 + m.t * V;
  const int64_t x_step = rows.step * a.x_ld, y_step = rows.step * a.y_ld, x0 = rows.row * a.x_ld + at0;
  In fx, fr;
  fx.init(a.x, x0, smem_u32(ring));
  if (RES) fr.init(a.r, x0, smem_u32(ring) + In::kSlot);
  const auto fetch = [&](int k, uint32_t slot) {
    const bool on = k < rows.mine;
    fx.fetch(whole && on, on ? left : 0, hop, slot, a.x, x_step);
    if (RES) fr.fetch(whole && on, on ? left : 0, hop, slot, a.x, x_step);
    copies_issued();
  };
  const auto land = [&](uint32_t slot) {
    fx.land(slot);
    if (RES) fr.land(slot);
  };
  uint32_t slot = 0, next = 0;
  const int early = a.ahead + (CLUSTER ? 1 : 0);
  for (int d = 0; d < early; ++d, next += kSlotBytes) {
    fetch(d, next);
    land(next);
  }
  const uint32_t last = next;
  const auto advance = [&](uint32_t& s) { s = s == last ? 0 : s + kSlotBytes; };
  u64 ga[H], be[H];
  load_params<V, N>(a.gamma + blockIdx.y * a.par_gs + m.col0, m, ga);
  load_params<V, N>(a.beta + blockIdx.y * a.par_gs + m.col0, m, be);
  XT* s_out = static_cast<XT*>(a.s) + x0;
  YT* y_out = static_cast<YT*>(a.out) + rows.row * a.y_ld + at0;
  int64_t row = rows.row;
  const float inv_n = m.n ? 1.f / m.n : 0.f, inv_C = 1.f / a.C;

  // A row's values v (p: the residual's), their sum s, the mean of the thread's warp (or smaller team) and the squared deviations from
  // it.
  const auto sums = [&](bool on, u64 (&v)[H], u64 (&p)[H], float& s, float& mean, float& q) {
    fx.read(slot, v);
    if constexpr (RES) {
      fr.read(slot, p);
#pragma unroll
      for (int i = 0; i < H; ++i) add2(v[i], p[i]);
      if constexpr (sizeof(XT) == 2) {
#pragma unroll
        for (int i = 0; i < H; ++i) {
          const float2 f = unpack2(v[i]);
          const __nv_bfloat162 b = __floats2bfloat162_rn(f.x, f.y);
          const uint32_t w = *reinterpret_cast<const uint32_t*>(&b);
          v[i] = pack2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
        }
      }
      if (on) store_row<XT, V, N>(v, s_out, whole, left, hop);
      s_out += x_step;
    }
    u64 acc = v[0];
#pragma unroll
    for (int i = 1; i < H; ++i) add2(acc, v[i]);
    s = m.sum(added(acc));
    mean = s * inv_n;
    acc = 0;
    if (whole) {
#pragma unroll
      for (int i = 0; i < H; ++i) {
        const u64 d = sum2(v[i], both(-mean));
        acc = mad2(d, d, acc);
      }
    } else {
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        const float2 d = unpack2(sum2(v[e / 2], both(-mean)));
        const u64 w = pack2(e / V * hop + e % V < left ? d.x : 0.f, (e + 1) / V * hop + (e + 1) % V < left ? d.y : 0.f);
        acc = mad2(w, w, acc);
      }
    }
    q = m.sum(added(acc));
  };
  const auto finish = [&](bool on, u64 (&v)[H], float mean, float q) {
    const float rstd = rsqrtf(fmaf(q, inv_C, a.eps));
    if (on) {
      if (m.t == 0 && m.rank == 0) {
        a.mean[row] = mean;
        a.rstd[row] = rstd;
      }
#pragma unroll
      for (int i = 0; i < H; ++i) v[i] = mad2(mul2(sum2(v[i], both(-mean)), both(rstd)), ga[i], be[i]);
      if (a.act != LSGD_ACT_NONE)
        with_act(a.act, [&](auto act) {
#pragma unroll
          for (int i = 0; i < H; ++i) {
            const float2 z = unpack2(v[i]);
            constexpr int kind = sizeof(YT) == 2 ? kFast : kClose;
            v[i] = pack2(activate<kind, decltype(act)::value>(z.x), activate<kind, decltype(act)::value>(z.y));
          }
        });
      store_row<YT, V, N>(v, y_out, whole, left, hop);
    }
    y_out += y_step;
    row += rows.step;
  };

  if constexpr (!CLUSTER) {
    for (int k = 0; k < rows.turns; ++k, advance(slot), advance(next)) {
      const bool on = k < rows.mine;
      u64 v[H], p[H];
      fx.take(v);
      if (RES) fr.take(p);
      fetch(k + a.ahead, next);
      copies_wait(a.ahead);
      float s, mean, q;
      sums(on, v, p, s, mean, q);
      if (m.slots > 1) {
        m.post_moments(s, mean, q, stats, k);
        m.collect_moments(mean, q, inv_C, stats, k);
      }
      finish(on, v, mean, q);
    }
  } else {
    uint32_t before = 0, coming = 0;  // the places of row k - 1, and of the row that was fetched last
    for (int k = 0; k <= rows.turns; ++k) {
      u64 v[H], p[H];
      float s, mean, q;
      if (k < rows.turns) {
        copies_wait(a.ahead);
        sums(true, v, p, s, mean, q);
        if constexpr (RES) fx.write(slot, v);
        m.post_moments(s, mean, q, stats, k);
      }
      if (k) {
        land(coming);
        m.collect_moments(mean, q, inv_C, stats, k - 1);
        fx.read(before, v);
        finish(true, v, mean, q);
      }
      fetch(k + early, next);
      before = slot, coming = next;
      advance(slot);
      advance(next);
    }
    m.end();
  }
}

template <typename XT, typename YT, int V, bool RES, int E, bool CLUSTER>
cudaError_t ln_forward_as(LnArgs a, int G, cudaStream_t st) {
  static std::atomic<int> raised{0};  // device + 1 whose limits this kernel's have been raised to
  using In = Feed<XT, V, E / V, CLUSTER>;
  constexpr int slot = In::kSlot * (RES ? 2 : 1), more = CLUSTER ? 2 : 1, own = kStaticSmem<CLUSTER>;
  constexpr int fit = kSmemPerSm / ((1 + more) * slot + own);
  const auto kernel = ln_forward_kernel<XT, YT, V, RES, E, CLUSTER>;
  LnPlan p = ln_plan(G, a.R, a.C, E, 0, fit);
  if constexpr (CLUSTER) {
    static ClusterCounts counts;
    p = ln_plan(G, a.R, a.C, E, 0, fit, ln_clusters(kernel, raised, counts, p.T * p.teams, (1 + more) * slot, p.cl));
  }
  const int threads = p.T * p.teams, per_sm = std::min(std::max(1, kThreadsPerSm / threads), fit);
  a.T = p.T, a.teams = p.teams, a.cl = p.cl, a.slice = p.slice;
  a.ahead = In::kAsync && per_sm * ((2 + more) * slot + own) <= kSmemPerSm ? ln_ahead(p.rows, per_sm * threads, slot / kThreads) : 1;
  return ln_launch(kernel, raised, a, dim3((unsigned)(p.ranges * p.cl), G), (a.ahead + more) * slot, st);
}
// 16 values to a thread; 8 where single bf16 values come through registers, 32 of which they would take with a residual (32,768 x 1531:
// 214 and 122 us), but not where a cluster would then be needed for a row that one CTA of 16 holds (8,000 x 3001: 35 us, 97 in clusters).
template <typename XT, typename YT, int V, bool RES>
cudaError_t ln_forward(const LnArgs& a, int G, cudaStream_t st) {
  constexpr int E = V * sizeof(XT) >= 4 ? 16 : 8;
  if (a.C <= E * kThreads) return ln_forward_as<XT, YT, V, RES, E, false>(a, G, st);
  if constexpr (E == 8) {
    if (a.C <= 16 * kThreads) return ln_forward_as<XT, YT, V, RES, 16, false>(a, G, st);
  }
  return ln_forward_as<XT, YT, V, RES, E, true>(a, G, st);
}

// The widest vector (a power of two of values, at most v) with which rows of stride ld from p on (values of z bytes) are aligned.
int ln_vec(int v, int64_t rows, int64_t ld, const void* p, int z) {
  while (v > 1 && ((rows > 1 && ld % v) || reinterpret_cast<uintptr_t>(p) % std::min(16, v * z))) v >>= 1;
  return v;
}

// Enough for the backward of any types and vectors.
size_t ln_workspace(int G, int64_t R, int C) {
  int64_t most = 1;
  for (int E : {8, 16}) most = std::max(most, ln_plan(G, R, C, E, kFewRows).ranges);
  return most > 1 ? (size_t)G * most * C * 8 : 0;
}

const char* ln_shape_error(int G, int64_t R, int64_t C) {
  if (G < 1 || C < 1 || R < 0) return "G and C must be at least 1, R at least 0";
  if (G > 65535 || C > kMaxC || R > ((int64_t)1 << 36) / G) return "at most 65535 workers, 2^36 rows (G R) and 32768 values a row";
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
  const cudaError_t e = ln_dispatch(xb, yb, v, [&](auto xv, auto yv, auto vec) {
    using XT = decltype(xv);
    using YT = decltype(yv);
    constexpr int V = decltype(vec)::value;
    return r ? ln_forward<XT, YT, V, true>(a, G, (cudaStream_t)stream) : ln_forward<XT, YT, V, false>(a, G, (cudaStream_t)stream);
  });
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
  const auto launch = relu ? launch_ln_backward_relu : act == LSGD_ACT_SILU ? launch_ln_backward_silu : launch_ln_backward_none;
  const cudaError_t e = launch(a, G, xb, yb, v, (cudaStream_t)stream);
  return e == cudaSuccess ? LSGD_OK : ln_error(LSGD_ECUDA, fn, cudaGetErrorString(e));
}

}  // extern "C"
