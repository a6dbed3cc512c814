// Vectors of up to 16 bytes, activations and the length of a sum's segments: what the normalisations share.
#pragma once
#include <type_traits>

#include "../../include/lsgd.h"
#include "common.cuh"

namespace lsgd {

template <int BYTES>
struct RawOf;
template <>
struct RawOf<16> {
  using type = uint4;
};
template <>
struct RawOf<8> {
  using type = uint2;
};
template <>
struct RawOf<4> {
  using type = uint32_t;
};
template <>
struct RawOf<2> {
  using type = uint16_t;
};

// V values of T as loaded, and as floats.
template <typename T, int V>
struct Vec {
  using Raw = typename RawOf<V * (int)sizeof(T) <= 16 ? V * (int)sizeof(T) : 16>::type;
  static constexpr int kN = V * (int)sizeof(T) <= 16 ? 1 : V * (int)sizeof(T) / 16;
  Raw r[kN];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < kN; ++i) r[i] = __ldg(reinterpret_cast<const Raw*>(p) + i);
  }
  __device__ __forceinline__ void load_shared(const void* p) {
#pragma unroll
    for (int i = 0; i < kN; ++i) r[i] = static_cast<const Raw*>(p)[i];
  }
  __device__ __forceinline__ void floats(float (&v)[V]) const {
    if constexpr (sizeof(T) == 4) {
      const float* f = reinterpret_cast<const float*>(r);
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] = f[j];
    } else if constexpr (V == 1) {
      v[0] = bf2f((uint16_t)r[0]);
    } else {
      const uint32_t* w = reinterpret_cast<const uint32_t*>(r);
#pragma unroll
      for (int j = 0; j < V / 2; ++j) {
        v[2 * j] = __uint_as_float(w[j] << 16);
        v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
      }
    }
  }
  __device__ __forceinline__ float at(int j) const {
    if constexpr (sizeof(T) == 4) return reinterpret_cast<const float*>(r)[j];
    else if constexpr (V == 1) return bf2f((uint16_t)r[0]);
    else {
      const uint32_t w = reinterpret_cast<const uint32_t*>(r)[j / 2];
      return __uint_as_float(j & 1 ? w & 0xffff0000u : w << 16);
    }
  }
  __device__ __forceinline__ void set(const float (&v)[V]) {
    if constexpr (sizeof(T) == 4) {
      float* f = reinterpret_cast<float*>(r);
#pragma unroll
      for (int j = 0; j < V; ++j) f[j] = v[j];
    } else if constexpr (V == 1) {
      r[0] = f2bf(v[0]);
    } else {
      uint32_t* w = reinterpret_cast<uint32_t*>(r);
#pragma unroll
      for (int j = 0; j < V / 2; ++j) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
        w[j] = *reinterpret_cast<const uint32_t*>(&b);
      }
    }
  }
  __device__ __forceinline__ void store(T* p) const {
#pragma unroll
    for (int i = 0; i < kN; ++i) reinterpret_cast<Raw*>(p)[i] = r[i];
  }
  // The first `left` values alone (what lies behind them is not touched).
  __device__ __forceinline__ void store_first(T* p, int left) const {
    if (left >= V) {
      store(p);
      return;
    }
#pragma unroll
    for (int j = 0; j < V - 1; ++j)
      if (j < left) {
        if constexpr (sizeof(T) == 4) p[j] = reinterpret_cast<const float*>(r)[j];
        else p[j] = (T)(reinterpret_cast<const uint32_t*>(r)[j / 2] >> 16 * (j & 1));
      }
  }
  __device__ __forceinline__ void stream(T* p) const {  // leaves L2 to what will be read again
#pragma unroll
    for (int i = 0; i < kN; ++i) __stcs(reinterpret_cast<Raw*>(p) + i, r[i]);
  }
};

// 1 / (1 + exp(-z)): the exponential's overflow gives 0.  kExact (fp32 tensors): the accurate exponential and division.  kSums
// (the sums over bf16 tensors, dgamma and dbeta among them, which are fp32 results): the accurate exponential and the fast
// reciprocal, 2^-23 off.  kFast: the fast exponential too, 2^-21 and |z| 2^-23 off, which a bf16 result's rounding of 2^-8 hides: y
// (54.9 against 56.9 us for 8 images of 127 x 129 x 320, whose second pass the special function unit bounds) and the split form's
// dx.  The fast reciprocal flushes what is below 2^-126: y is 0 from z = -87.3 on, where it is 1e-36 at most.
// kClose (layer norm's fp32 results): the accurate exponential, and the fast reciprocal with a step of Newton's iteration, which leaves
// half a unit in the last place (a quotient takes a dozen instructions more).
enum { kFast, kSums, kExact, kClose };
template <int KIND>
__device__ __forceinline__ float sigmoid(float z) {
  if constexpr (KIND == kExact) return 1.f / (1.f + expf(-z));
  float e, r;
  if constexpr (KIND == kClose) {
    const float d = 1.f + expf(-z);
    asm("rcp.approx.f32 %0, %1;" : "=f"(r) : "f"(d));
    return d < 1e30f ? fmaf(r, fmaf(-d, r, 1.f), r) : r;  // (infinity: 0)
  }
  if constexpr (KIND == kSums) e = expf(-z);
  else asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(z * -1.44269504f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
  return r;
}

// act(z).
template <int KIND, int ACT>
__device__ __forceinline__ float activate(float z) {
  if constexpr (ACT == LSGD_ACT_RELU) {
    float r;
    asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(r) : "f"(z));
    return r;
  }
  if constexpr (ACT == LSGD_ACT_SILU) return z * sigmoid<KIND>(z);
  return z;
}
// f with the activation as a constant.
template <typename F>
__device__ __forceinline__ void with_act(int act, F f) {
  if (act == LSGD_ACT_RELU) f(std::integral_constant<int, LSGD_ACT_RELU>{});
  else if (act == LSGD_ACT_SILU) f(std::integral_constant<int, LSGD_ACT_SILU>{});
  else f(std::integral_constant<int, LSGD_ACT_NONE>{});
}

// How many of a thread's k values are added up at a time: the sums of these segments are added in turn, so that no chain of
// additions is longer than the root of k or 64.  (fp32 sums of 2048 equal values in a row are up to 1.7e-5 off, of 16384 1.6e-4.)
__device__ __forceinline__ int segment(int k) { return max(64, ((int)sqrtf((float)k) + 7) / 8 * 8); }

}  // namespace lsgd
