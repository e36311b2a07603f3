// Element types and small cross-lane helpers of the expert-layer kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ll_device.hpp"

namespace llc {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Elements as they lie in memory.  Arithmetic is binary32; a store rounds once.
template <typename T>
struct Num;
template <>
struct Num<float> {
  static constexpr int kPer16 = 4;
  static __device__ __forceinline__ float get(float v) { return v; }
  static __device__ __forceinline__ float put(float v) { return v; }
};
template <>
struct Num<__bf16> {
  static constexpr int kPer16 = 8;
  static __device__ __forceinline__ float get(__bf16 v) { return (float)v; }
  static __device__ __forceinline__ __bf16 put(float v) { return (__bf16)v; }
};

// N consecutive elements held as binary32.  VEC: the address is aligned to
// min(16, N * sizeof(T)) bytes.
template <typename T, int N, bool VEC>
struct Pack {
  float v[N];
  __device__ __forceinline__ void load(const T *p) {
    if constexpr (VEC) {
      constexpr int kBytes = N * (int)sizeof(T) < 16 ? N * (int)sizeof(T) : 16;
      constexpr int kEach = kBytes / (int)sizeof(T);
      typedef T vec __attribute__((ext_vector_type(kEach)));
#pragma unroll
      for (int i = 0; i < N / kEach; ++i) {
        const vec r = *reinterpret_cast<const vec *>(p + i * kEach);
#pragma unroll
        for (int j = 0; j < kEach; ++j) v[i * kEach + j] = Num<T>::get(r[j]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = Num<T>::get(p[i]);
    }
  }
  __device__ __forceinline__ void store(T *p) const {
    if constexpr (VEC) {
      constexpr int kBytes = N * (int)sizeof(T) < 16 ? N * (int)sizeof(T) : 16;
      constexpr int kEach = kBytes / (int)sizeof(T);
      typedef T vec __attribute__((ext_vector_type(kEach)));
#pragma unroll
      for (int i = 0; i < N / kEach; ++i) {
        vec r;
#pragma unroll
        for (int j = 0; j < kEach; ++j) r[j] = Num<T>::put(v[i * kEach + j]);
        *reinterpret_cast<vec *>(p + i * kEach) = r;
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) p[i] = Num<T>::put(v[i]);
    }
  }
  // The first n of the N elements (n may be 0 or less); the others read as `fill`.
  __device__ __forceinline__ void load_some(const T *p, int n, float fill) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = i < n ? Num<T>::get(p[i]) : fill;
  }
  __device__ __forceinline__ void store_some(T *p, int n) const {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < n) p[i] = Num<T>::put(v[i]);
  }
};

// e^x to about two units in the last place: 2^t with t = x log2(e) rounded,
// times 1 + the first-order correction for that rounding.  Results below
// 2^-126 are 0; NaN stays NaN.
__device__ __forceinline__ float exp_f32(float x) {
  x = x < -150.f ? -150.f : x;  // keeps the correction finite at the infinities
  x = x > 150.f ? 150.f : x;
  const float t = x * 1.44269502162933349609375f;
  float r = __builtin_fmaf(x, 1.44269502162933349609375f, -t);
  r = __builtin_fmaf(x, 1.92596299112661746887e-8f, r);
  return __builtin_amdgcn_exp2f(t) * __builtin_fmaf(r, 0.693147180559945309417f, 1.f);
}

template <int kCtrl>
__device__ __forceinline__ float dpp_f32(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), kCtrl, 0xF, 0xF, true));
}

// The partner's value for the steps over 16 and 32 lanes: the two results of a
// lane swap with itself are the value of the even and of the odd half.
typedef uint32_t u32pair __attribute__((ext_vector_type(2)));
template <int kDist>
__device__ __forceinline__ u32pair lane_halves(uint32_t v) {
  if constexpr (kDist == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return u32pair{r[0], r[1]};
  } else {
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return u32pair{r[0], r[1]};
  }
}
template <int kDist>
__device__ __forceinline__ float add_halves(float v) {
  const u32pair r = lane_halves<kDist>((uint32_t)__float_as_int(v));
  return __int_as_float((int)r[0]) + __int_as_float((int)r[1]);
}
template <int kDist>
__device__ __forceinline__ float max_halves(float v) {
  const u32pair r = lane_halves<kDist>((uint32_t)__float_as_int(v));
  return fmaxf(__int_as_float((int)r[0]), __int_as_float((int)r[1]));
}
template <int kDist>
__device__ __forceinline__ int max_halves(int v) {
  const u32pair r = lane_halves<kDist>((uint32_t)v);
  return max((int)r[0], (int)r[1]);
}

// Sum / maximum over each aligned group of W lanes (16 or 64); every lane gets
// the same bits, since each step adds the same two partial results in both
// lanes.  Within 16 lanes the partners come from the DPP controls xor 1, xor
// 2, mirrored halves of 8, mirrored 16.
template <int W>
__device__ __forceinline__ float group_sum(float v) {
  v += dpp_f32<0xB1>(v);
  v += dpp_f32<0x4E>(v);
  v += dpp_f32<0x141>(v);
  v += dpp_f32<0x140>(v);
  if constexpr (W == 64) {
    v = add_halves<16>(v);
    v = add_halves<32>(v);
  }
  return v;
}
template <int W>
__device__ __forceinline__ float group_max(float v) {
  v = fmaxf(v, dpp_f32<0xB1>(v));
  v = fmaxf(v, dpp_f32<0x4E>(v));
  v = fmaxf(v, dpp_f32<0x141>(v));
  v = fmaxf(v, dpp_f32<0x140>(v));
  if constexpr (W == 64) {
    v = max_halves<16>(v);
    v = max_halves<32>(v);
  }
  return v;
}

}  // namespace llc
