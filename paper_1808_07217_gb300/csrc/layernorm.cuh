// What layer norm's kernels share: how rows are dealt out to teams of threads, a team's sums, and the rows' way through shared
// memory (layernorm.cu describes the operator).
#pragma once
#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>

#include "../../include/lsgd.h"
#include "common.cuh"
#include "lsgd_internal.h"
#include "tc_ptx.cuh"
#include "vectors.cuh"

namespace lsgd {

constexpr int kThreads = 256;     // of a CTA at most
constexpr int kMaxCluster = 16;
constexpr int kMaxC = 8 * kThreads * kMaxCluster;  // with 8 values to a thread
constexpr int kThreadsPerSm = 512;            // at 128 registers
constexpr int kSmemPerSm = 222 * 1024;
template <bool CLUSTER>
constexpr int kSlotsOf = kThreads / 32 * (CLUSTER ? kMaxCluster : 1);  // of an exchange
constexpr int kExchange = 8;                  // slots that are read together
template <bool CLUSTER>  // of a CTA: the exchanges' at most (of 16 bytes), barriers, and the system's
constexpr int kStaticSmem = 16 * ((CLUSTER ? 4 : 2) * kSlotsOf<CLUSTER> + kExchange) + 64 + 1024;

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
  int ahead;      // rows whose copies are under way while one is reduced: 1 or 2
  int rows;       // neighbouring rows of a team (0: it takes every n-th)
  int seg;        // rows that are added up at a time
  int sums;       // backward: where in shared memory their sums stand, in bytes
};

// Each source file that includes this has a flag of its own, which a wait that runs out sets (and which is read only once a cluster,
// whose CTAs alone wait so, has been launched).
namespace {
__device__ int g_rows_late = 0;
std::atomic<bool> g_rows_clustered{false};
int take_rows_late() {
  int h = 0;
  if (!g_rows_clustered) return 0;
  if (cudaMemcpyFromSymbol(&h, g_rows_late, sizeof(int)) != cudaSuccess) {
    cudaGetLastError();
    return 0;
  }
  if (h) {
    const int zero = 0;
    cudaMemcpyToSymbol(g_rows_late, &zero, sizeof(int));
  }
  return h;
}

// How the rows are dealt out, whatever the types.
struct LnPlan {
  int T, teams, cl, slice;
  int64_t ranges;  // CTAs (clusters) of a worker
  int64_t rows;    // rows of a team at most
};

// few: as many rows of a team stay with one CTA; per_sm: CTAs that an SM holds at once (0: as many as its threads allow); clusters: of
// those that the GPU holds at once (0: as many as the SMs' CTAs make).
inline LnPlan ln_plan(int G, int64_t R, int C, int E, int few, int per_sm = 0, int clusters = 0) {
  LnPlan p;
  p.cl = (C + E * kThreads - 1) / (E * kThreads);
  p.slice = ((C + p.cl - 1) / p.cl + E - 1) / E * E;
  p.cl = (C + p.slice - 1) / p.slice;
  const int need = (std::min(C, p.slice) + E - 1) / E;
  p.T = 1;
  while (p.T < need && p.T < 32) p.T *= 2;
  if (need > 32) p.T = (need + 31) / 32 * 32;
  p.teams = std::max(1, kThreads / p.T);
  const int by_threads = std::max(1, kThreadsPerSm / (p.T * p.teams));
  const int64_t slots = (int64_t)kNumSMs * (per_sm ? std::min(per_sm, by_threads) : by_threads);
  const int64_t at_once = clusters ? std::min<int64_t>(clusters, slots / p.cl) : slots / p.cl;
  const int64_t most = std::max<int64_t>(1, at_once / G);
  const int64_t turns = (R + p.teams - 1) / p.teams;  // of a CTA's teams, if there were one CTA
  p.rows = std::max<int64_t>(1, (turns + most - 1) / most);
  if (turns <= few) p.rows = std::max<int64_t>(1, turns);
  p.ranges = (turns + p.rows - 1) / p.rows;
  return p;
}

__device__ __forceinline__ void team_barrier(int id, int threads) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}
// Every CTA of the cluster is here (and its shared memory there before the first time).
__device__ __forceinline__ void cluster_meet() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// v to the place `at` of the cluster's CTA `rank`, whose barrier `bar` counts the bytes.  (No barrier of the whole cluster in every row: its
// release would wait for the rows' stores.)
__device__ __forceinline__ uint32_t peer_address(const void* p, int rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(p)), "r"(rank));
  return r;
}
__device__ __forceinline__ void send(const float* at, const uint64_t* bar, int rank, float v) {
  asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.f32 [%0], %1, [%2];" ::"r"(peer_address(at, rank)), "f"(v),
               "r"(peer_address(bar, rank))
               : "memory");
}
__device__ __forceinline__ void send(const float4* at, const uint64_t* bar, int rank, float4 v) {
  asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(
                   peer_address(at, rank)),
               "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w), "r"(peer_address(bar, rank))
               : "memory");
}
// Whether the bytes of the phase came; not within about 2 s: the flag is set.
__device__ __forceinline__ bool wait_bytes(uint64_t* bar, uint32_t parity) {
  const auto there = [&] {
    uint32_t ok;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n"
        " selp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
    return ok != 0;
  };
  if (there()) return true;
  const long long t0 = clock64();
  while (!there())
    if (clock64() - t0 > 4000000000LL) {
      atomicExch(&g_rows_late, 1);
      return false;
    }
  return true;
}

// A thread's place, and what its team shares.  The row's warps exchange their sums in two halves, post and collect, through one of kTurns
// places in turn.  In a CTA a barrier lies between; whoever posts row k + 2 has passed that of row k + 1, which every warp
// reaches when it has collected row k.  A cluster's CTAs post row k + 1 before they collect row k (below), so that whoever posts
// row k + 4 has collected row k + 2, which every warp posted when it had collected row k: four places.
template <bool CLUSTER>
struct Team {
  static constexpr int kTurns = CLUSTER ? 4 : 2, kSlots = kSlotsOf<CLUSTER>, kPlaces = kTurns * kSlots + kExchange;
  int T, t, team, lane, warps, warp, cl, rank, slots;
  int col0, Cs;    // the CTA's columns
  int n;           // the warp's (or smaller team's) columns
  uint64_t* bars;  // a cluster's: [kTurns]
  bool lost = false;  // a wait ran out: what follows is wrong, and waits no more
  __device__ __forceinline__ Team(const LnArgs& a, int vec, int vecs, uint64_t* cluster_bars) {
    T = a.T, team = threadIdx.x / T, t = threadIdx.x - team * T, lane = threadIdx.x & 31;
    warps = T < 32 ? 1 : T / 32, warp = T < 32 ? 0 : t / 32;
    bars = cluster_bars;
    if constexpr (CLUSTER) {
      cl = a.cl;
      asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    } else {
      cl = 1, rank = 0;
    }
    slots = warps * cl;
    col0 = rank * a.slice, Cs = min(a.slice, a.C - col0);
    n = Cs;
    if (T > 32) {
      n = 0;
      for (int j = 0; j < vecs; ++j) n += min(32 * vec, max(0, Cs - (j * T + warp * 32) * vec));
    }
  }
  __device__ __forceinline__ float sum(float v) const {  // over the warp, or over the team within it
    if (T >= 32) return warp_sum(v);
    for (int d = T / 2; d; d /= 2) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
  }
  static __device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int d = 16; d; d /= 2) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
  }
  // Before a cluster's first exchange, and before its CTAs leave.
  __device__ __forceinline__ void begin() const {
    if constexpr (CLUSTER) {
      if (threadIdx.x == 0) {
#pragma unroll
        for (int i = 0; i < kTurns; ++i) mbar_init(bars + i, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
      }
      cluster_meet();
    }
  }
  __device__ __forceinline__ void end() const {
    if constexpr (CLUSTER) cluster_meet();
  }
  // What the row's warps posted (`bytes` each) is there; k counts the rows.
  __device__ __forceinline__ void meet(int k, int bytes) {
    if constexpr (CLUSTER) {
      if (threadIdx.x == 0) mbar_expect_tx(bars + k % kTurns, slots * bytes);
      if (!lost) lost = !wait_bytes(bars + k % kTurns, (k / kTurns) & 1);
    } else {
      team_barrier(team + 1, T);
    }
  }
  // The row's mean and sum of squared deviations q from a warp's sum s, mean and sum q.  (Alone: the warp is the team.)
  __device__ __forceinline__ void post_moments(float s, float mean, float q, float4* stats, int k) const {
    float4* stat = stats + k % kTurns * kSlots + team * warps;
    const float4 mine = make_float4(s, mean, q, (float)n);
    if constexpr (CLUSTER) {
      if (lane < cl) send(stat + rank * warps + warp, bars + k % kTurns, lane, mine);
    } else {
      if (lane == 0) stat[warp] = mine;
    }
  }
  __device__ __forceinline__ void collect_moments(float& mean, float& q, float inv_C, const float4* stats, int k) {
    const float4* stat = stats + k % kTurns * kSlots + team * warps;
    meet(k, 16);
    float s = 0.f;
    q = 0.f;
    if (slots <= kExchange) {  // (what stands behind the slots is read, and not used: `stats` has room for it)
#pragma unroll
      for (int i = 0; i < kExchange; ++i) {
        const float f = stat[i].x;
        s += i < slots ? f : 0.f;
      }
      mean = s * inv_C;
#pragma unroll
      for (int i = 0; i < kExchange; ++i) {
        const float f = deviation(stat[i], mean);
        q += i < slots ? f : 0.f;
      }
    } else {
      for (int i = lane; i < slots; i += 32) s += stat[i].x;
      mean = warp_sum(s) * inv_C;
      for (int i = lane; i < slots; i += 32) q += deviation(stat[i], mean);
      q = warp_sum(q);
    }
  }
  static __device__ __forceinline__ float deviation(const float4& f, float mean) {
    const float d = f.y - mean;
    return fmaf(f.w * d, d, f.z);
  }
  // p and q summed over the row.  In a warp the halves sum one each: 5 exchanges instead of 10.
  __device__ __forceinline__ void post_both(float p, float q, float2* stats, int k) const {
    const float v = halves(p, q);
    float2* stat = stats + k % kTurns * kSlots + team * warps;
    if constexpr (CLUSTER) {
      if ((lane & 15) < cl)
        send(reinterpret_cast<float*>(stat + rank * warps + warp) + (lane >> 4), bars + k % kTurns, lane & 15, v);
    } else {
      if ((lane & 15) == 0) (lane ? stat[warp].y : stat[warp].x) = v;
    }
  }
  __device__ __forceinline__ void collect_both(float& p, float& q, const float2* stats, int k) {
    const float2* stat = stats + k % kTurns * kSlots + team * warps;
    meet(k, 8);
    p = q = 0.f;
    if (slots <= kExchange) {
#pragma unroll
      for (int i = 0; i < kExchange; ++i) {
        const float2 f = stat[i];
        p += i < slots ? f.x : 0.f;
        q += i < slots ? f.y : 0.f;
      }
    } else {
      for (int i = lane; i < slots; i += 32) {
        const float2 f = stat[i];
        p += f.x;
        q += f.y;
      }
      spread(halves(p, q), p, q);
    }
  }
  __device__ __forceinline__ void sum_both(float& p, float& q) const {  // of a team that is a warp or less
    if (T == 32) {
      spread(halves(p, q), p, q);
      return;
    }
    for (int d = T / 2; d; d /= 2) {
      p += __shfl_xor_sync(0xffffffffu, p, d);
      q += __shfl_xor_sync(0xffffffffu, q, d);
    }
  }
  // The warp's sum of p in lanes 0 to 15, of q in the others.
  __device__ __forceinline__ float halves(float p, float q) const {
    const bool high = lane & 16;
    float v = (high ? q : p) + __shfl_xor_sync(0xffffffffu, high ? p : q, 16);
#pragma unroll
    for (int d = 8; d; d /= 2) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
  }
  static __device__ __forceinline__ void spread(float v, float& p, float& q) {
    p = __shfl_sync(0xffffffffu, v, 0);
    q = __shfl_sync(0xffffffffu, v, 16);
  }
};

// N vectors as E / 2 pairs of floats.
template <typename T, int V, int N>
__device__ __forceinline__ void to_pairs(const Vec<T, V> (&r)[N], u64 (&p)[N * V / 2]) {
#pragma unroll
  for (int k = 0; k < N * V / 2; ++k) p[k] = pack2(r[2 * k / V].at(2 * k % V), r[(2 * k + 1) / V].at((2 * k + 1) % V));
}
template <typename T, int V, int N>
__device__ __forceinline__ void from_pairs(const u64 (&p)[N * V / 2], Vec<T, V> (&r)[N]) {
  float v[N][V];
#pragma unroll
  for (int k = 0; k < N * V / 2; ++k) {
    const float2 f = unpack2(p[k]);
    v[2 * k / V][2 * k % V] = f.x;
    v[(2 * k + 1) / V][(2 * k + 1) % V] = f.y;
  }
#pragma unroll
  for (int j = 0; j < N; ++j) r[j].set(v[j]);
}
__device__ __forceinline__ u64 both(float v) { return pack2(v, v); }
__device__ __forceinline__ float added(u64 p) {
  const float2 f = unpack2(p);
  return f.x + f.y;
}

// A thread's values of the parameter at p (worker's, CTA's first column), zeros behind the row's end.
template <int V, int N, typename M>
__device__ __forceinline__ void load_params(const float* p, const M& m, u64 (&out)[N * V / 2]) {
  float v[N * V];
#pragma unroll
  for (int e = 0; e < N * V; ++e) {
    const int c = (e / V * m.T + m.t) * V + e % V;
    v[e] = c < m.Cs ? __ldg(p + c) : 0.f;
  }
#pragma unroll
  for (int k = 0; k < N * V / 2; ++k) out[k] = pack2(v[2 * k], v[2 * k + 1]);
}

// One input's rows on their way through shared memory: every thread's own N vectors of the next rows, in slots of one row each.
// Vectors of 4 bytes and more are copied by cp.async, which writes zeros where there is nothing to read (behind the row's end, and
// rows behind the last); single bf16 values, which it does not take, come through registers, one row ahead, and only where a row is
// read twice (in a cluster) go on to shared memory.  The vectors of a slot lie kThreads vectors from one another whatever the block's
// size, so that they cost no address arithmetic.
template <typename T, int V, int N, bool CLUSTER>
struct Feed {
  static constexpr int kBytes = V * (int)sizeof(T);  // of a vector
  static constexpr bool kAsync = kBytes >= 4, kShared = kAsync || CLUSTER;
  static constexpr int kSlot = kShared ? N * kThreads * kBytes : 0;
  const T* row;   // the thread's first value of the next row to fetch
  uint32_t at;    // the thread's first vector in slot 0
  uint16_t held[kAsync ? 1 : N];
  __device__ __forceinline__ void init(const void* p, int64_t first, uint32_t base) {
    row = static_cast<const T*>(p) + first;
    at = base + threadIdx.x * kBytes;
  }
  // whole: all of the warp's vectors are there; otherwise left: columns from the thread's first on (none: zeros).  hop: columns
  // between its vectors; some: an address that may be read; step: to the next row.
  __device__ __forceinline__ void fetch(bool whole, int left, int hop, uint32_t slot, const void* some, int64_t step) {
    if constexpr (kAsync) {
      if (whole) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const uint32_t dst = at + slot + j * kThreads * kBytes;
          if constexpr (kBytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(row + j * hop) : "memory");
          else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(row + j * hop), "n"(kBytes) : "memory");
        }
      } else {
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const uint32_t dst = at + slot + j * kThreads * kBytes;
          const int n = min(V, max(0, left - j * hop)) * (int)sizeof(T);
          const void* src = n ? row + j * hop : some;
          if constexpr (kBytes == 16)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
          else
            asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(kBytes), "r"(n) : "memory");
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) {  // (volatile: issued here, not where they land)
        held[j] = 0;
        if (left > j * hop) asm volatile("ld.global.nc.u16 %0, [%1];" : "=h"(held[j]) : "l"(row + j * hop) : "memory");
      }
    }
    row += step;
  }
  // The row that came through registers (before the next is fetched).
  __device__ __forceinline__ void take(u64 (&out)[N * V / 2]) const {
    if constexpr (!kShared) {
#pragma unroll
      for (int i = 0; i < N * V / 2; ++i) out[i] = pack2(bf2f(held[2 * i]), bf2f(held[2 * i + 1]));
    }
  }
  __device__ __forceinline__ void land(uint32_t slot) const {
    if constexpr (!kAsync && kShared) {
#pragma unroll
      for (int j = 0; j < N; ++j)
        asm volatile("st.shared.u16 [%0], %1;" ::"r"(at + slot + j * kThreads * kBytes), "h"(held[j]) : "memory");
    }
  }
  // A row from shared memory (nothing to do where it has been taken).
  __device__ __forceinline__ void read(uint32_t slot, u64 (&out)[N * V / 2]) const {
    if constexpr (!kShared) return;
    Vec<T, V> r[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const uint32_t p = at + slot + j * kThreads * kBytes;
      if constexpr (kBytes == 16)
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r[j].r[0].x), "=r"(r[j].r[0].y), "=r"(r[j].r[0].z),
                     "=r"(r[j].r[0].w) : "r"(p) : "memory");
      else if constexpr (kBytes == 8)
        asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(r[j].r[0].x), "=r"(r[j].r[0].y) : "r"(p) : "memory");
      else if constexpr (kBytes == 4)
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(r[j].r[0]) : "r"(p) : "memory");
      else
        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(r[j].r[0]) : "r"(p) : "memory");
    }
    to_pairs(r, out);
  }
  __device__ __forceinline__ void write(uint32_t slot, const u64 (&in)[N * V / 2]) const {  // back to a row's place
    Vec<T, V> r[N];
    from_pairs(in, r);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const uint32_t p = at + slot + j * kThreads * kBytes;
      if constexpr (kBytes == 16)
        asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(p), "r"(r[j].r[0].x), "r"(r[j].r[0].y), "r"(r[j].r[0].z),
                     "r"(r[j].r[0].w) : "memory");
      else if constexpr (kBytes == 8)
        asm volatile("st.shared.v2.u32 [%0], {%1, %2};" ::"r"(p), "r"(r[j].r[0].x), "r"(r[j].r[0].y) : "memory");
      else if constexpr (kBytes == 4)
        asm volatile("st.shared.u32 [%0], %1;" ::"r"(p), "r"(__builtin_bit_cast(uint32_t, r[j].r[0])) : "memory");
      else
        asm volatile("st.shared.u16 [%0], %1;" ::"r"(p), "h"(r[j].r[0]) : "memory");
    }
  }
};
__device__ __forceinline__ void copies_issued() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copies_wait(int newer) {  // until all but the `newer` (1 or 2) last groups are there
  if (newer == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
  else asm volatile("cp.async.wait_group 2;" ::: "memory");
}

// A row's values to p: all, or those before the row's end.
template <typename T, int V, int N>
__device__ __forceinline__ void store_row(const u64 (&v)[N * V / 2], T* p, bool whole, int left, int hop) {
  Vec<T, V> o[N];
  from_pairs(v, o);
  if (whole) {
#pragma unroll
    for (int j = 0; j < N; ++j) o[j].store(p + j * hop);
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (left > j * hop) o[j].store_first(p + j * hop, left - j * hop);
  }
}
// Rows of a team that one CTA of the backward takes by itself: more CTAs need the second kernel, whose launch costs as much of the host's
// time as it saves of the GPU's (3 x 20 x 600, five rows: 17.5 us a call, 8.9 of them the GPU's; 20.1 and 6.7 with it).
constexpr int kFewRows = 6;

// The rows that fall to a team.  Forward: every step-th of the worker's, so that all CTAs together walk through memory; backward: one of
// the CTA's `rows` x teams neighbouring ones (32,768 x 2048 in bf16: 92 us, with every step-th 105; the forward 84 and 82).
struct Rows {
  int mine, turns;     // the team's rows; the turns of its warp's loop, in which teams that lie in one warp go together
  int64_t step, row;   // row: of the first one, of all workers'
  template <typename M>
  __device__ __forceinline__ Rows(const LnArgs& a, const M& m, int64_t ranges, int64_t range) {
    int64_t from = range * a.teams, end = a.R;
    step = ranges * a.teams;
    if (a.rows) {
      from *= a.rows;
      end = min(a.R, from + (int64_t)a.rows * a.teams);
      step = a.teams;
    }
    const int64_t first = from + m.team, lead = from + (m.T < 32 ? (int)(threadIdx.x & ~31) / m.T : m.team);
    mine = first < end ? (int)((end - first + step - 1) / step) : 0;
    turns = lead < end ? (int)((end - lead + step - 1) / step) : 0;
    row = blockIdx.y * a.R + first;
  }
};

// Rows ahead: two, unless the copies under way then pass 28 KB an SM (threads of all its CTAs x bytes of a row).  More of them slow the
// memory: 32,768 x 2048 in bf16 with a residual take 96 us with two or three rows of 32 KB ahead, 82 with one; 32,768 x
// 1534 in fp32, of 24 KB, 71 with two and 74 with one.
inline int ln_ahead(int rows, int threads, int bytes) { return rows > 1 && threads * bytes <= 28 * 1024 ? 2 : 1; }

cudaLaunchConfig_t ln_config(cudaLaunchAttribute (&attr)[2], dim3 grid, int threads, size_t smem, int cl, cudaStream_t st) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cl;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cl > 1 ? 2 : 1;
  return cfg;
}

// A kernel's limits raised to what the largest call needs.
template <typename K>
cudaError_t ln_raise(K kernel, std::atomic<int>& raised) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess || raised == dev + 1) return e;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemPerSm - kStaticSmem<true>);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e == cudaSuccess) raised = dev + 1;
  return e;
}

// The clusters that the GPU holds at once (a cluster lies in one GPC, whose SMs are mostly no multiple of it: 2,000 x 17,000 in bf16,
// clusters of 5 with two CTAs to an SM, took 107 us with the 60 that the SMs' CTAs make and takes 72 with as many as are held at
// once).  0 if unknown.  The answers are kept by the launch's shape.
struct ClusterCounts {
  std::atomic<uint64_t> known[16] = {};
};
template <typename K>
int ln_clusters(K kernel, std::atomic<int>& raised, ClusterCounts& counts, int threads, size_t smem, int cl) {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || ln_raise(kernel, raised) != cudaSuccess) return 0;
  const uint64_t key = ((((uint64_t)dev * 32 + cl) * 2048 + threads) * (1 << 18) + smem) + 1;
  std::atomic<uint64_t>& at = counts.known[(key ^ (key >> 18) ^ (key >> 29)) % 16];
  const uint64_t known = at;
  if (known >> 12 == key) return (int)(known & 4095);
  cudaLaunchAttribute attr[2];
  const cudaLaunchConfig_t cfg = ln_config(attr, dim3(cl), threads, smem, cl, nullptr);
  if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) {
    cudaGetLastError();
    return 0;
  }
  n = std::min(n, 4095);
  at = key << 12 | (uint64_t)n;
  return n;
}

template <typename K>
cudaError_t ln_launch(K kernel, std::atomic<int>& raised, const LnArgs& a, dim3 grid, size_t smem, cudaStream_t st) {
  if (a.cl > 1 && !g_rows_clustered) g_rows_clustered = true;
  if (smem > 40 * 1024 || a.cl > 8) {
    const cudaError_t e = ln_raise(kernel, raised);
    if (e != cudaSuccess) return e;
  }
  cudaLaunchAttribute attr[2];
  const cudaLaunchConfig_t cfg = ln_config(attr, grid, a.T * a.teams, smem, a.cl, st);
  return cudaLaunchKernelEx(&cfg, kernel, a);
}

// The kernel for the types and the widest vectors (vmax values) of a call: form(XT, YT, V).
template <typename F>
cudaError_t ln_dispatch(bool xb, bool yb, int vmax, F form) {
  const auto vec = [&](auto x, auto y) {
    if constexpr (sizeof(x) == 2 && sizeof(y) == 2) {
      if (vmax >= 8) return form(x, y, std::integral_constant<int, 8>{});
    }
    if (vmax >= 4) return form(x, y, std::integral_constant<int, 4>{});
    if (vmax >= 2) return form(x, y, std::integral_constant<int, 2>{});
    return form(x, y, std::integral_constant<int, 1>{});
  };
  const float f = 0.f;
  const uint16_t h = 0;
  if (xb) return yb ? vec(h, h) : vec(h, f);
  return yb ? vec(f, h) : vec(f, f);
}

}  // namespace

// layernorm_backward_*.cu: the backward with one activation each.
cudaError_t launch_ln_backward_none(const LnArgs& a, int G, bool xb, bool yb, int vmax, cudaStream_t st);
cudaError_t launch_ln_backward_relu(const LnArgs& a, int G, bool xb, bool yb, int vmax, cudaStream_t st);
cudaError_t launch_ln_backward_silu(const LnArgs& a, int G, bool xb, bool yb, int vmax, cudaStream_t st);
int take_ln_backward_late_none();
int take_ln_backward_late_relu();
int take_ln_backward_late_silu();

}  // namespace lsgd
