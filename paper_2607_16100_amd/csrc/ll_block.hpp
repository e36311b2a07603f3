// Rows and weights in 8 bits, the norms around a block, and the weight update
// (include/llblock.h).  All of them are bound by memory where they are large
// and by latency where they are small.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/llblock.h"
#include "ll_e4m3.hpp"
#include "ll_linear.hpp"
#include "ll_num.hpp"

namespace llc {
namespace blk {

constexpr int kW = 8;  // consecutive values of a lane

// kW values of a row as they lie in memory.  All of them are loaded and stored 16
// bytes at a time whatever the address is aligned to, which the vector memory unit
// takes (8 of 6896 x 809 bfloat16 weights by single elements: 111 us).
template <typename T>
struct Chunk {
  static constexpr int kPer = 16 / (int)sizeof(T), kParts = kW / kPer;
  typedef T vec __attribute__((ext_vector_type(kPer)));
  vec r[kParts];
  // the first `left` (any number) of the kW; the others are 0
  __device__ __forceinline__ void load(const T *p, int left) {
    if (left >= kW) {
#pragma unroll
      for (int i = 0; i < kParts; ++i) __builtin_memcpy(&r[i], p + i * kPer, 16);
    } else {
#pragma unroll
      for (int i = 0; i < kW; ++i) r[i / kPer][i % kPer] = i < left ? p[i] : (T)0.f;
    }
  }
  __device__ __forceinline__ void store(T *p, int left) const {
    if (left >= kW) {
#pragma unroll
      for (int i = 0; i < kParts; ++i) __builtin_memcpy(p + i * kPer, &r[i], 16);
    } else {
#pragma unroll
      for (int i = 0; i < kW; ++i)
        if (i < left) p[i] = r[i / kPer][i % kPer];
    }
  }
  __device__ __forceinline__ lin::Vals vals() const {
    lin::Vals v;
#pragma unroll
    for (int i = 0; i < kW; ++i) v.v[i] = Num<T>::get(r[i / kPer][i % kPer]);
    return v;
  }
  __device__ __forceinline__ void set(const lin::Vals &v) {
#pragma unroll
    for (int i = 0; i < kW; ++i) r[i / kPer][i % kPer] = Num<T>::put(v.v[i]);
  }
};
template <typename T>
__device__ __forceinline__ lin::Vals get(const T *p, int left) {
  Chunk<T> c;
  c.load(p, left);
  return c.vals();
}
template <typename T>
__device__ __forceinline__ void put(T *p, const lin::Vals &v, int left) {
  Chunk<T> c;
  c.set(v);
  c.store(p, left);
}
__device__ __forceinline__ void put_codes(uint8_t *p, const uint32_t *w, int left) {
  if (left >= kW) {
    __builtin_memcpy(p, w, 8);
  } else {
#pragma unroll
    for (int i = 0; i < kW; ++i)
      if (i < left) p[i] = (uint8_t)(w[i / 4] >> (i % 4 * 8));
  }
}

// The largest magnitude's bits; at least those of Infinity where a value is not finite.
__device__ __forceinline__ uint32_t top_bits(const lin::Vals &v) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < kW; ++i) top = max(top, (uint32_t)__float_as_int(v.v[i]) & 0x7FFFFFFFu);
  return top;
}
constexpr uint32_t kInfBits = 0x7F800000u;

// kW values of a block of 16 lanes to codes; returns the block's scale.  Every
// value is looked at one by one only in a wave that has one that is not finite.
__device__ __forceinline__ uint32_t quantise8(const lin::Vals &v, uint32_t *w) {
  uint32_t top = top_bits(v);
  if (__any(top >= kInfBits)) {
    top = 0;
#pragma unroll
    for (int i = 0; i < kW; ++i) top = max(top, finite_bits(v.v[i]));
    const uint32_t s = scale_of<8>(max16(top));
    const float inv = scale_inverse(s);
#pragma unroll
    for (int i = 0; i < 2; ++i)
      w[i] = to_e4m3(v.v[4 * i] * inv, v.v[4 * i + 1] * inv) | to_e4m3(v.v[4 * i + 2] * inv, v.v[4 * i + 3] * inv) << 16;
    return s;
  }
  const uint32_t s = scale_of<8>(max16(top));
  const float inv = scale_inverse(s);
#pragma unroll
  for (int i = 0; i < 2; ++i) w[i] = pack_e4m3(v.v[4 * i] * inv, v.v[4 * i + 1] * inv, v.v[4 * i + 2] * inv, v.v[4 * i + 3] * inv);
  return s;
}

// Activations in front of the rounding to 8 bits.  SiLU is x / (1 + 2^(-x log2
// e)) by the exponential and the reciprocal of the vector unit: relatively off by
// |x| 2^-24 and a few units in the last place, where a code's half step is 2^-4.
// Below about -87.3 the reciprocal is that of a number above 2^126 and may be 0: so
// then is the result, less than 2^-119 in magnitude (a code only in a block that has
// no value above 2^-110).
// With the library's exponential and division they were most of the kernel's time
// (16384 x 2 x 2048 through SwiGLU 57 us, with an exponential corrected for the
// product's rounding 39.3, so 36.7; with 16 bytes at any alignment 33.9).
__device__ __forceinline__ void act_rows(lin::Vals &v, int act) {
  if (act == LL_ACT_SILU || act == LL_ACT_SWIGLU) {
#pragma unroll
    for (int i = 0; i < kW; ++i)
      v.v[i] *= __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(v.v[i] * -1.44269502162933349609375f));
  } else {
    lin::act8(v, act);
  }
}

// ---------------------------------------------------------------- rows
//
// 16 lanes a block of 128 features, U blocks of a lane under way at a time.  Bound
// by memory: 16384 x 2 x 2048 bfloat16 through SwiGLU 33.9 us, 5.0 TB/s of what is
// read and written; 16 x 7168 2.6 us, a load's latency.
struct QuantArgs {
  const void *x;
  uint8_t *q, *scales;
  const int32_t *end;
  uint64_t ldx, ldq, lds;
  uint32_t rows, features, blocks;  // blocks a row
  int act;
};

template <typename T, int U>
__global__ __launch_bounds__(256) void k_quantise(QuantArgs a) {
  uint32_t rows = a.rows;
  if (a.end != nullptr) rows = (uint32_t)min(max(*a.end, 0), (int)a.rows);
  const uint32_t items = rows * a.blocks;  // (fewer than 2^30, by the launch's limit)
  const uint32_t first = blockIdx.x * (16 * U) + threadIdx.x / 16;
  if (blockIdx.x * (16 * U) >= items) return;
  const bool gate = lin::gated(a.act);
  lin::Vals v[U], u[U];
  uint32_t row[U], col[U];
#pragma unroll
  for (int n = 0; n < U; ++n) {
    const uint32_t item = first + n * 16;
    row[n] = item < items ? item / a.blocks : 0u;
    col[n] = item < items ? item % a.blocks * kBlock + threadIdx.x % 16 * kW : 0xFFFFFFFFu;
    const int left = col[n] < a.features ? (int)(a.features - col[n]) : 0;
    const T *p = (const T *)a.x + (uint64_t)row[n] * a.ldx + (left > 0 ? col[n] : 0);
    v[n] = get<T>(p, left);
    if (gate) u[n] = get<T>(p + a.features, left);
  }
#pragma unroll
  for (int n = 0; n < U; ++n) {
    act_rows(v[n], a.act);
    if (gate) {
#pragma unroll
      for (int i = 0; i < kW; ++i) v[n].v[i] *= u[n].v[i];
    }
    uint32_t w[2];
    const int left = col[n] < a.features ? (int)(a.features - col[n]) : 0;
#pragma unroll
    for (int i = 0; i < kW; ++i) v[n].v[i] = i < left ? v[n].v[i] : 0.f;
    const uint32_t s = quantise8(v[n], w);
    if (left > 0) {
      put_codes(a.q + (uint64_t)row[n] * a.ldq + col[n], w, left);
      if (threadIdx.x % 16 == 0) a.scales[(uint64_t)row[n] * a.lds + col[n] / kBlock] = (uint8_t)s;
    }
  }
}

// ---------------------------------------------------------------- weights
//
// Bound by memory: 8 of 7168 x 2048 binary32, transposed, 108 us, 5.4 TB/s.  A
// workgroup has one block of 128 x 128: a thread 8 rows of 8 columns, 16 threads a
// row.  Transposed, two codes of a column are rounded into one word
// at a time, so the 8 of a column lie together without a permutation; they go
// through LDS to leave in whole lines.
struct WeightArgs {
  const void *w;
  uint8_t *q, *scales;
  uint64_t ldw, wstride, ldq, qstride, lds, sstride;
  uint32_t out, in;
};

template <typename T, bool TRANSPOSE>
__global__ __launch_bounds__(256) void k_quantise_weight(WeightArgs a) {
  constexpr int kPitch = 128 + 16;  // rows of the transposed block start 16 bytes on in the banks
  __shared__ __attribute__((aligned(16))) uint8_t tile[TRANSPOSE ? 128 * kPitch : 16];
  __shared__ uint32_t tops[4];
  const uint32_t bi = blockIdx.x, bo = blockIdx.y, g = blockIdx.z;
  const uint32_t tr = threadIdx.x / 16, tc = threadIdx.x % 16;
  const uint32_t row0 = bo * kBlock + tr * 8, col0 = bi * kBlock + tc * 8;
  const int left = col0 < a.in ? (int)(a.in - col0) : 0;
  const T *p = (const T *)a.w + g * a.wstride + (uint64_t)row0 * a.ldw + col0;
  lin::Vals v[8];
  uint32_t top = 0;
#pragma unroll
  for (int r = 0; r < 8; ++r) v[r] = get<T>(p + r * a.ldw, row0 + r < a.out ? left : 0);
#pragma unroll
  for (int r = 0; r < 8; ++r)
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, finite_bits(v[r].v[i]));
  top = max16(top);
  top = max(top, max(lane_halves<16>(top)[0], lane_halves<16>(top)[1]));
  top = max(top, max(lane_halves<32>(top)[0], lane_halves<32>(top)[1]));
  if (threadIdx.x % 64 == 0) tops[threadIdx.x / 64] = top;
  __syncthreads();
  top = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
  const uint32_t s = scale_of<8>(top);
  const float inv = scale_inverse(s);
  uint8_t *q = a.q + g * a.qstride;
  if (threadIdx.x == 0) a.scales[g * a.sstride + (TRANSPOSE ? (uint64_t)bi * a.lds + bo : (uint64_t)bo * a.lds + bi)] = (uint8_t)s;
  if constexpr (!TRANSPOSE) {
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      uint32_t w[2];
#pragma unroll
      for (int i = 0; i < 2; ++i)
        w[i] = to_e4m3(v[r].v[4 * i] * inv, v[r].v[4 * i + 1] * inv) |
               to_e4m3(v[r].v[4 * i + 2] * inv, v[r].v[4 * i + 3] * inv) << 16;
      if (row0 + r >= a.out) continue;
      put_codes(q + (uint64_t)(row0 + r) * a.ldq + col0, w, left);
    }
  } else {
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      uint32_t w[2];
#pragma unroll
      for (int i = 0; i < 2; ++i)
        w[i] = to_e4m3(v[4 * i].v[c] * inv, v[4 * i + 1].v[c] * inv) |
               to_e4m3(v[4 * i + 2].v[c] * inv, v[4 * i + 3].v[c] * inv) << 16;
      *reinterpret_cast<uint2 *>(tile + (tc * 8 + c) * kPitch + tr * 8) = uint2{w[0], w[1]};
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const uint32_t at = n * 256 + threadIdx.x, r = at / 8, c = at % 8 * 16;
      const uint32_t orow = bi * kBlock + r, ocol = bo * kBlock + c;
      if (orow >= a.in || ocol >= a.out) continue;
      const u32x4 w = *reinterpret_cast<const u32x4 *>(tile + r * kPitch + c);
      uint8_t *to = q + (uint64_t)orow * a.ldq + ocol;
      if (ocol + 16 <= a.out) {
        __builtin_memcpy(to, &w, 16);
      } else {
#pragma unroll
        for (uint32_t i = 0; i < 16; ++i)
          if (ocol + i < a.out) to[i] = (uint8_t)(w[i / 4] >> (i % 4 * 8));
      }
    }
  }
}

// ---------------------------------------------------------------- norms
struct NormArgs {
  const void *y, *x, *post, *weight;
  const float *gate;
  void *r, *h;
  uint8_t *q, *scales;
  // gradients
  const void *dh, *dr;
  void *dr_out, *dy;
  float *dgate, *parts;  // parts: [2][gridDim.x][features], of dweight and dpost
  uint64_t ldy, ldx, ldr, ldh, ldq, lds, ldd, ldo, lddy;
  uint32_t rows, features;
  float eps, scale;
  bool w32;  // post and weight are binary32
};

// Sums of N values over the TPR threads of a row; every thread gets the same
// bits.  `red`: [N][TPR / 64] of this row and of this sum alone.
template <int TPR, int N>
__device__ __forceinline__ void row_sums(float *v, float *red) {
#pragma unroll
  for (int n = 0; n < N; ++n) v[n] = group_sum<64>(v[n]);
  if constexpr (TPR > 64) {
    constexpr int kWaves = TPR / 64;
    if (threadIdx.x % 64 == 0) {
#pragma unroll
      for (int n = 0; n < N; ++n) red[n * kWaves + threadIdx.x / 64] = v[n];
    }
    __syncthreads();
    // (lane i takes wave i's part, and each aligned kWaves lanes add them up)
#pragma unroll
    for (int n = 0; n < N; ++n) {
      float s = red[n * kWaves + threadIdx.x % kWaves];
      s += dpp_f32<0xB1>(s);
      if constexpr (kWaves > 2) s += dpp_f32<0x4E>(s);
      if constexpr (kWaves > 4) s += dpp_f32<0x141>(s);
      if constexpr (kWaves > 8) s += dpp_f32<0x140>(s);
      v[n] = s;
    }
  }
}

// A norm's weights, of the rows' type or binary32.
template <typename T>
__device__ __forceinline__ lin::Vals get_weight(const void *w, bool w32, uint32_t at, int left) {
  if (left <= 0) return get<float>((const float *)nullptr, 0);
  return w32 ? get<float>((const float *)w + at, left) : get<T>((const T *)w + at, left);
}

// Threads of a row's workgroup; a wave a row: four of them.
constexpr int norm_threads(int tpr) { return tpr == 64 ? 256 : tpr; }

// A thread's only chunk: everything the row needs is asked for at once, weights
// too.  Two (more than 8192 features): the weights are read when they are used,
// from L2.  8192 x 7168 bfloat16, residual and norm: 86 us, 5.4 TB/s (256 threads
// of four chunks: 103); with post, gate and the codes 104 us.
template <typename T, int TPR, int C>
__global__ __launch_bounds__(norm_threads(TPR)) void k_norm(NormArgs a) {
  constexpr bool kEarly = C == 1;
  constexpr int kRows = norm_threads(TPR) / TPR;
  __shared__ float red[2][TPR / 64];
  const uint32_t t = threadIdx.x % TPR;
  const uint32_t row = blockIdx.x * kRows + threadIdx.x / TPR;
  if (kRows > 1 && row >= a.rows) return;  // (a wave has a row then, and no barrier comes)
  lin::Vals v[C], x[C], post[kEarly ? C : 1], weight[kEarly ? C : 1];
  const float n = (float)a.features;
  auto left = [&](int c) { return (int)a.features - (int)((c * TPR + t) * kW); };
#pragma unroll
  for (int c = 0; c < C; ++c) v[c] = get<T>((const T *)a.y + row * a.ldy + (c * TPR + t) * kW, left(c));
  if (a.x != nullptr) {
#pragma unroll
    for (int c = 0; c < C; ++c) x[c] = get<T>((const T *)a.x + row * a.ldx + (c * TPR + t) * kW, left(c));
  }
  if (kEarly && a.post != nullptr) post[0] = get_weight<T>(a.post, a.w32, t * kW, left(0));
  if (kEarly && a.weight != nullptr) weight[0] = get_weight<T>(a.weight, a.w32, t * kW, left(0));
  const float by = a.gate != nullptr ? a.gate[row] * a.scale : a.scale;
  auto squares = [&](float *s) {
    *s = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < kW; ++i) *s = __builtin_fmaf(v[c].v[i], v[c].v[i], *s);
  };
  float s;
  if (a.post != nullptr) {
    squares(&s);
    row_sums<TPR, 1>(&s, red[0]);
    const float rstd = 1.f / sqrtf(s / n + a.eps);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if constexpr (!kEarly) post[0] = get_weight<T>(a.post, a.w32, (c * TPR + t) * kW, left(c));
#pragma unroll
      for (int i = 0; i < kW; ++i) v[c].v[i] = v[c].v[i] * rstd * post[0].v[i];
    }
  }
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int i = 0; i < kW; ++i) v[c].v[i] *= by;
  if (a.x != nullptr) {
#pragma unroll
    for (int c = 0; c < C; ++c) lin::add8(v[c], x[c]);
  }
  if (a.r != nullptr) {
#pragma unroll
    for (int c = 0; c < C; ++c) put<T>((T *)a.r + row * a.ldr + (c * TPR + t) * kW, v[c], left(c));
  }
  if (a.weight == nullptr) return;
  squares(&s);
  row_sums<TPR, 1>(&s, red[1]);
  const float rstd = 1.f / sqrtf(s / n + a.eps);
#pragma unroll
  for (int c = 0; c < C; ++c) {
    if constexpr (!kEarly) weight[0] = get_weight<T>(a.weight, a.w32, (c * TPR + t) * kW, left(c));
#pragma unroll
    for (int i = 0; i < kW; ++i) v[c].v[i] = v[c].v[i] * rstd * weight[0].v[i];
    if (a.h != nullptr) put<T>((T *)a.h + row * a.ldh + (c * TPR + t) * kW, v[c], left(c));
    if (a.q != nullptr) {  // 16 lanes have a block, whole or to the row's end
      uint32_t w[2];
      const uint32_t at = (c * TPR + t) * kW;
      const uint32_t sc = quantise8(v[c], w);
      if (left(c) > 0) {
        put_codes(a.q + row * a.ldq + at, w, left(c));
        if (t % 16 == 0) a.scales[row * a.lds + at / kBlock] = (uint8_t)sc;
      }
    }
  }
}

// The gradients: a workgroup takes rows blockIdx.x, + gridDim.x, ... and keeps
// its share of dweight and dpost in registers; k_norm_join adds the shares up.
//
// With u = r / d, d = sqrt(mean(r^2) + eps): dr_out = dr + (weight dh - u
// mean(u weight dh)) / d, and the same once more from dr_out to y.  Two rounds
// of sums a row: r^2, weight dh r and y^2; then dr_out post y, which gives both
// dgate and what dy needs.
//
// A thread has one chunk of a row (two of more than 8192 features), and with one
// the next row is loaded while one is worked on (with four chunks a thread, all
// read when their row came: 8192 x 7168 bfloat16 with post and gate 460 us, so
// 149).  Values are held as they lie in memory.
template <typename T, int TPR, int C>
__global__ __launch_bounds__(norm_threads(TPR)) void k_norm_grad(NormArgs a) {
  constexpr int kRows = norm_threads(TPR) / TPR;
  constexpr bool kHold = C == 1;  // the weights stay in registers, and the next row comes there
  __shared__ float red[2][2][3 * (TPR / 64)];
  const uint32_t t = threadIdx.x % TPR;
  const float rn = 1.f / (float)a.features;
  const uint32_t lane_row = threadIdx.x / TPR, step = gridDim.x * kRows;
  auto left = [&](int c) { return (int)a.features - (int)((c * TPR + t) * kW); };
  auto at = [&](int c) { return left(c) > 0 ? (c * TPR + t) * kW : 0u; };
  const bool with_y = a.post != nullptr || a.dgate != nullptr;
  lin::Vals dw[C], dp[C], weight, post;
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int i = 0; i < kW; ++i) dw[c].v[i] = dp[c].v[i] = 0.f;
  if constexpr (kHold) {
    if (a.weight != nullptr) weight = get_weight<T>(a.weight, a.w32, at(0), left(0));
    if (a.post != nullptr) post = get_weight<T>(a.post, a.w32, at(0), left(0));
  }
  typedef Chunk<T> Row[C];
  auto load = [&](uint32_t row, Row &r, Row &g, Row &y, Row &d) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (a.weight != nullptr) {
        r[c].load((const T *)a.r + row * a.ldr + at(c), left(c));
        g[c].load((const T *)a.dh + row * a.ldh + at(c), left(c));
      }
      if (a.dr != nullptr) d[c].load((const T *)a.dr + row * a.ldd + at(c), left(c));
      if (with_y) y[c].load((const T *)a.y + row * a.ldy + at(c), left(c));
    }
  };
  Row r, g, y, e, nr, ng, ny, ne;
  uint32_t row = blockIdx.x * kRows + lane_row;
  if (kHold && row < a.rows) load(row, nr, ng, ny, ne);
  uint32_t turn = 0;
  for (; row < a.rows; row += step, ++turn) {
    float(*sums)[3 * (TPR / 64)] = red[turn & 1];
    if constexpr (kHold) {
#pragma unroll
      for (int c = 0; c < C; ++c) r[c] = nr[c], g[c] = ng[c], y[c] = ny[c], e[c] = ne[c];
      if (row + step < a.rows) load(row + step, nr, ng, ny, ne);
    } else {
      load(row, r, g, y, e);
    }
    float s[3] = {0.f, 0.f, 0.f};
    if (a.weight != nullptr) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        if constexpr (!kHold) weight = get_weight<T>(a.weight, a.w32, at(c), left(c));
        const lin::Vals rv = r[c].vals(), gv = g[c].vals();
#pragma unroll
        for (int i = 0; i < kW; ++i) {
          s[0] = __builtin_fmaf(rv.v[i], rv.v[i], s[0]);
          s[1] = __builtin_fmaf(weight.v[i] * gv.v[i], rv.v[i], s[1]);
        }
      }
    }
    if (a.post != nullptr) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const lin::Vals yv = y[c].vals();
#pragma unroll
        for (int i = 0; i < kW; ++i) s[2] = __builtin_fmaf(yv.v[i], yv.v[i], s[2]);
      }
    }
    row_sums<TPR, 3>(s, sums[0]);
    lin::Vals d[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (a.dr != nullptr) {
        d[c] = e[c].vals();
      } else {
#pragma unroll
        for (int i = 0; i < kW; ++i) d[c].v[i] = 0.f;
      }
    }
    if (a.weight != nullptr) {
      const float rstd = 1.f / sqrtf(s[0] * rn + a.eps);
      const float mean = s[1] * rstd * rn;  // of u weight dh
#pragma unroll
      for (int c = 0; c < C; ++c) {
        if constexpr (!kHold) weight = get_weight<T>(a.weight, a.w32, at(c), left(c));
        const lin::Vals rv = r[c].vals(), gv = g[c].vals();
#pragma unroll
        for (int i = 0; i < kW; ++i) {
          const float u = rv.v[i] * rstd;
          dw[c].v[i] = __builtin_fmaf(gv.v[i], u, dw[c].v[i]);
          d[c].v[i] = __builtin_fmaf(rstd, weight.v[i] * gv.v[i] - u * mean, d[c].v[i]);
        }
      }
    }
    if (a.dr_out != nullptr) {
#pragma unroll
      for (int c = 0; c < C; ++c) put<T>((T *)a.dr_out + row * a.ldo + at(c), d[c], left(c));
    }
    if (!with_y && a.dy == nullptr) continue;
    const float by = (a.gate != nullptr ? a.gate[row] : 1.f) * a.scale;
    if (with_y) {
      float dot = 0.f;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const lin::Vals yv = y[c].vals();
        if (a.post != nullptr) {
          if constexpr (!kHold) post = get_weight<T>(a.post, a.w32, at(c), left(c));
#pragma unroll
          for (int i = 0; i < kW; ++i) dot = __builtin_fmaf(d[c].v[i] * post.v[i], yv.v[i], dot);
        } else {
#pragma unroll
          for (int i = 0; i < kW; ++i) dot = __builtin_fmaf(d[c].v[i], yv.v[i], dot);
        }
      }
      row_sums<TPR, 1>(&dot, sums[1]);
      const float rstd = a.post != nullptr ? 1.f / sqrtf(s[2] * rn + a.eps) : 1.f;
      if (a.dgate != nullptr && t == 0) a.dgate[row] = a.scale * dot * rstd;
      if (a.post != nullptr) {
        const float mean = by * dot * rstd * rn;
#pragma unroll
        for (int c = 0; c < C; ++c) {
          if constexpr (!kHold) post = get_weight<T>(a.post, a.w32, at(c), left(c));
          const lin::Vals yv = y[c].vals();
#pragma unroll
          for (int i = 0; i < kW; ++i) {
            const float f = by * d[c].v[i], u = yv.v[i] * rstd;
            dp[c].v[i] = __builtin_fmaf(f, u, dp[c].v[i]);
            d[c].v[i] = rstd * (f * post.v[i] - u * mean);
          }
        }
      }
    }
    if (a.dy != nullptr) {
      if (a.post == nullptr) {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int i = 0; i < kW; ++i) d[c].v[i] *= by;
      }
#pragma unroll
      for (int c = 0; c < C; ++c) put<T>((T *)a.dy + row * a.lddy + at(c), d[c], left(c));
    }
  }
  if (a.parts == nullptr) return;
  if constexpr (kRows > 1) {  // the waves' shares in their order
    __shared__ lin::Vals others[2][kRows - 1][TPR];
    if (lane_row != 0) {
      others[0][lane_row - 1][t] = dw[0];
      others[1][lane_row - 1][t] = dp[0];
    }
    __syncthreads();
    if (lane_row != 0) return;
#pragma unroll
    for (int i = 0; i < kRows - 1; ++i) {
      lin::add8(dw[0], others[0][i][t]);
      lin::add8(dp[0], others[1][i][t]);
    }
  }
#pragma unroll
  for (int c = 0; c < C; ++c) {
    put<float>(a.parts + (uint64_t)blockIdx.x * a.features + at(c), dw[c], left(c));
    if (a.post != nullptr)
      put<float>(a.parts + ((uint64_t)gridDim.x + blockIdx.x) * a.features + at(c), dp[c], left(c));
  }
}

// dweight and dpost from the workgroups' shares, in their order: 64 columns a
// workgroup, kJoin threads a column, whose sums are added in order.
constexpr int kJoin = 16;
struct NormJoin {
  const float *parts;
  float *out[2];
  uint32_t count, features;
  bool add;
};
__global__ __launch_bounds__(64 * kJoin) void k_norm_join(NormJoin a) {
  __shared__ float part[kJoin][64];
  const uint32_t col = blockIdx.x * 64 + threadIdx.x % 64, lane = threadIdx.x / 64;
  const float *from = a.parts + (uint64_t)blockIdx.y * a.count * a.features + col;
  float s = 0.f;
  if (col < a.features) {
#pragma unroll 8
    for (uint32_t i = lane; i < a.count; i += kJoin) s += from[(uint64_t)i * a.features];
  }
  part[lane][threadIdx.x % 64] = s;
  __syncthreads();
  float *out = blockIdx.y == 0 ? a.out[0] : a.out[1];
  if (lane != 0 || col >= a.features || out == nullptr) return;
#pragma unroll
  for (int i = 1; i < kJoin; ++i) s += part[i][threadIdx.x % 64];
  out[col] = a.add ? out[col] + s : s;
}

// ---------------------------------------------------------------- weight update
//
// Bound by memory: 352 M bfloat16 parameters with binary32 masters and gradients
// and 8-bit states 1.17-1.2 ms, 5.4 TB/s; 9 M binary32 in 40 tensors with binary32
// states 50-52 us, 5.5 TB/s, and 2.4 for the step before it.  A thread has two runs
// of eight values, all of whose loads are under way together.
//
// The tensors' addresses travel with the launch, kTensors at a time, so that a
// captured launch keeps them and nothing is copied first.  Coefficients that
// depend on the step come from k_adamw_begin, which counts it: a replayed step
// is the next one.
struct AdamwCoef {
  float step, rden, decay, grad_scale;  // lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t), 1 - lr decay
  uint32_t key;
};
struct AdamwBegin {
  int32_t *step;
  const float *lr_ptr, *grad_scale;
  AdamwCoef *coef;
  double lr, log_beta1, log_beta2, decay;  // logarithms to base 2
  uint32_t seed;
};

// A bijection of 32-bit numbers whose every output bit depends on every input bit:
// multiplications by odd numbers and xors with the upper half.  Its constants are those
// of the 32-bit hash that Chris Wellons published as "lowbias32" (Prospecting for Hash
// Functions, 2018), found there by a search for the least bias.
__device__ __forceinline__ uint32_t mix32(uint32_t x) {
  x = (x ^ (x >> 16)) * 0x7FEB352Du;
  x = (x ^ (x >> 15)) * 0x846CA68Bu;
  return x ^ (x >> 16);
}

__global__ void k_adamw_begin(AdamwBegin a) {
  if (threadIdx.x != 0) return;
  const int32_t t = *a.step + 1;
  *a.step = t;
  const double lr = a.lr_ptr != nullptr ? (double)*a.lr_ptr : a.lr;
  AdamwCoef c;
  c.step = (float)(lr / (1. - exp2(a.log_beta1 * t)));
  c.rden = (float)(1. / sqrt(1. - exp2(a.log_beta2 * t)));
  c.decay = (float)(1. - lr * a.decay);
  c.grad_scale = a.grad_scale != nullptr ? *a.grad_scale : 1.f;
  c.key = mix32(a.seed + (uint32_t)t * 0x9E3779B9u);
  *a.coef = c;
}

struct AdamwTensor {
  void *param;
  const void *grad;
  float *master;
  void *m, *v;
  uint8_t *m_scales, *v_scales;
  uint64_t n, at;
  uint32_t chunk;  // the first of its chunks
  uint32_t kind;   // kBf16 | kGradBf16
};
constexpr uint32_t kBf16 = 1, kGradBf16 = 2;
constexpr int kTensors = 40;
constexpr uint32_t kChunk = 4096;  // values a workgroup
struct AdamwArgs {
  const AdamwCoef *coef;
  float beta1, rest1, beta2, rest2, eps;  // rest: 1 - beta
  uint32_t count;
  AdamwTensor t[kTensors];
};
static_assert(sizeof(AdamwArgs) <= 4000, "a launch's arguments");

// Up or down to MANT bits of mantissa, of which a value has `r` / 2^(23 - MANT)
// as its chance: the random bits are added below the last one kept.  Below the
// least normal number 2^EMIN the steps are those of 2^EMIN, in whole numbers.
// The value is at most the format's largest, so the code cannot pass it.
template <int MANT, int EMIN, int BIAS>
__device__ __forceinline__ uint32_t to_code(float y, uint32_t r) {
  constexpr int kCut = 23 - MANT;
  const uint32_t b = (uint32_t)__float_as_int(y) & 0x7FFFFFFFu;
  if (b >= 0x7F800000u) return 0x7Fu;
  const float mag = __int_as_float((int)b);
  constexpr float kUp = (float)(1ull << (MANT - EMIN + kCut));
  constexpr uint32_t kMin = (uint32_t)(EMIN + 127) << 23;
  const uint32_t fine = ((b + r) >> kCut) - ((127u - BIAS) << MANT);
  const uint32_t low = ((uint32_t)fminf(mag * kUp, 8388608.f) + r) >> kCut;
  return (b < kMin ? low : fine) | ((uint32_t)__float_as_int(y) >> 31) << 7;
}

// FLOOR: a v above 0 has its least code at least.  Rounded to 0, as its mean asks for,
// it leaves m alone in front of next to nothing (blocks of one gradient of 1 and the
// others of 2^-16, 400 steps: single steps of 1367 lr, so 1.22).
template <bool EIGHT, bool FLOOR>
__global__ __launch_bounds__(256) void k_adamw(AdamwArgs a) {
  uint32_t lo = 0, hi = a.count;
  while (hi - lo > 1) {
    const uint32_t mid = (lo + hi) / 2;
    if (a.t[mid].chunk <= blockIdx.x)
      lo = mid;
    else
      hi = mid;
  }
  const AdamwTensor &t = a.t[lo];
  const AdamwCoef c = *a.coef;
  const uint64_t n = t.n, base = (uint64_t)(blockIdx.x - t.chunk) * kChunk;
  const bool bf16 = t.kind & kBf16, gbf16 = t.kind & kGradBf16;
  constexpr int U = kChunk / (256 * kW);
  lin::Vals p[U], g[U], m[U], v[U];
  uint2 m8[U], v8[U];
  uint32_t ms[U], vs[U];
  auto at = [&](int u) { return base + (uint64_t)(u * 256 + threadIdx.x) * kW; };
  auto left = [&](int u) { return at(u) < n ? (int)min(n - at(u), (uint64_t)kW) : 0; };
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint64_t i = at(u);
    const int l = left(u);
    const uint64_t j = l > 0 ? i : 0;
    p[u] = get<float>((bf16 ? t.master : (const float *)t.param) + j, l);
    g[u] = gbf16 ? get<__bf16>((const __bf16 *)t.grad + j, l) : get<float>((const float *)t.grad + j, l);
    if constexpr (EIGHT) {
      // the states' last block is whole in memory only as far as the tensor goes
      m8[u] = v8[u] = uint2{0, 0};
      ms[u] = vs[u] = 1;
      if (l > 0) {
        ms[u] = t.m_scales[i / kBlock];
        vs[u] = t.v_scales[i / kBlock];
        if (l == kW) {
          __builtin_memcpy(&m8[u], (const uint8_t *)t.m + i, 8);
          __builtin_memcpy(&v8[u], (const uint8_t *)t.v + i, 8);
        } else {
          uint32_t mw[2] = {0, 0}, vw[2] = {0, 0};
#pragma unroll
          for (int e = 0; e < kW; ++e)
            if (e < l) {
              mw[e / 4] |= (uint32_t)((const uint8_t *)t.m)[i + e] << (e % 4 * 8);
              vw[e / 4] |= (uint32_t)((const uint8_t *)t.v)[i + e] << (e % 4 * 8);
            }
          m8[u] = uint2{mw[0], mw[1]};
          v8[u] = uint2{vw[0], vw[1]};
        }
      }
    } else {
      m[u] = get<float>((const float *)t.m + j, l);
      v[u] = get<float>((const float *)t.v + j, l);
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint64_t i = at(u);
    const int l = left(u);
    if constexpr (EIGHT) {
      const float fm = scale_value(ms[u]), fv = scale_value(vs[u]);
#pragma unroll
      for (int e = 0; e < kW; ++e) {
        const uint32_t wm = e < 4 ? m8[u].x : m8[u].y, wv = e < 4 ? v8[u].x : v8[u].y;
        switch (e % 4) {
          case 0: m[u].v[e] = __builtin_amdgcn_cvt_f32_fp8((int)wm, 0); v[u].v[e] = __builtin_amdgcn_cvt_f32_bf8((int)wv, 0); break;
          case 1: m[u].v[e] = __builtin_amdgcn_cvt_f32_fp8((int)wm, 1); v[u].v[e] = __builtin_amdgcn_cvt_f32_bf8((int)wv, 1); break;
          case 2: m[u].v[e] = __builtin_amdgcn_cvt_f32_fp8((int)wm, 2); v[u].v[e] = __builtin_amdgcn_cvt_f32_bf8((int)wv, 2); break;
          default: m[u].v[e] = __builtin_amdgcn_cvt_f32_fp8((int)wm, 3); v[u].v[e] = __builtin_amdgcn_cvt_f32_bf8((int)wv, 3); break;
        }
        m[u].v[e] *= fm;
        v[u].v[e] *= fv;
      }
    }
#pragma unroll
    for (int e = 0; e < kW; ++e) {
      const float gr = g[u].v[e] * c.grad_scale;
      m[u].v[e] = m[u].v[e] * a.beta1 + gr * a.rest1;
      v[u].v[e] = v[u].v[e] * a.beta2 + gr * gr * a.rest2;
      p[u].v[e] = p[u].v[e] * c.decay - c.step * m[u].v[e] / (sqrtf(v[u].v[e]) * c.rden + a.eps);
    }
    if constexpr (EIGHT) {
      uint32_t tm = 0, tv = 0;
#pragma unroll
      for (int e = 0; e < kW; ++e) {
        tm = max(tm, e < l ? finite_bits(m[u].v[e]) : 0u);
        tv = max(tv, e < l ? finite_bits(v[u].v[e]) : 0u);
      }
      const uint32_t sm = scale_of<8>(max16(tm)), sv = scale_of<15>(max16(tv));
      if (l > 0) {
        const float im = scale_inverse(sm), iv = scale_inverse(sv);
        const uint64_t no = t.at + i;
        uint32_t mw[2] = {0, 0}, vw[2] = {0, 0};
#pragma unroll
        for (int e = 0; e < kW; ++e) {
          const uint64_t k = no + e;
          const uint32_t r = mix32((uint32_t)k ^ ((uint32_t)(k >> 32) * 0x9E3779B9u) ^ c.key);
          mw[e / 4] |= to_code<3, -6, 7>(m[u].v[e] * im, r >> 16 << 4) << (e % 4 * 8);
          uint32_t vc = to_code<2, -14, 15>(v[u].v[e] * iv, (r & 0xFFFFu) << 5);
          if (FLOOR && v[u].v[e] > 0.f) vc = max(vc, 1u);  // (the product may underflow)
          vw[e / 4] |= vc << (e % 4 * 8);
        }
        put_codes((uint8_t *)t.m + i, mw, l);
        put_codes((uint8_t *)t.v + i, vw, l);
        if (threadIdx.x % 16 == 0) {
          t.m_scales[i / kBlock] = (uint8_t)sm;
          t.v_scales[i / kBlock] = (uint8_t)sv;
        }
      }
    }
    if (l <= 0) continue;
    if constexpr (!EIGHT) {
      put<float>((float *)t.m + i, m[u], l);
      put<float>((float *)t.v + i, v[u], l);
    }
    if (bf16) {
      put<float>(t.master + i, p[u], l);
      put<__bf16>((__bf16 *)t.param + i, p[u], l);
    } else {
      put<float>((float *)t.param + i, p[u], l);
    }
  }
}

}  // namespace blk
}  // namespace llc
