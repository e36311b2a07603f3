// Routing, dispatch and combine kernels (include/llmoe.h).
//
// All of them are bound by memory, or at small sizes by the launch: each
// reads its rows once and writes its rows once.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/llmoe.h"
#include "ll_num.hpp"

namespace llc {
namespace moe {

constexpr int kThreads = 256;
constexpr float kNegInf = -__builtin_inff();

// ---------------------------------------------------------------- routing
//
// W lanes hold one token's logits, NPL consecutive ones each, so that among
// equal keys the lowest lane holds the lowest index.  k rounds: every lane's
// best key, the maximum over the lanes, the lowest lane that has it.
//
// Bound by vector instructions, not by memory: 32301 tokens x 160 bfloat16
// logits, 6 choices, take 8.5 us (1.2 TB/s), and their gradient, which computes
// the exponentials again and nothing else, 6.5 us (3.2 TB/s).  One token takes
// 3.5 us, a chain of 8 rounds behind two loads.
struct RouteArgs {
  const void *logits;
  uint64_t ld;
  uint32_t tokens;
  int experts, k;
  const float *bias;
  int score, normalise;
  float scale;
  int32_t *ids;
  float *weights;
  const float *dweights;
  void *dlogits;
  uint64_t ldd;
};

// The logits of one lane; past the last expert, and for NaN, -Infinity.
// VEC: rows start at multiples of 4 bytes, and NPL elements are whole dwords.
template <typename T, int NPL, bool VEC>
__device__ __forceinline__ void load_logits(const T *row, int e0, int experts, float (&l)[NPL]) {
  if (VEC && e0 + NPL <= experts) {
    T v[NPL];
    __builtin_memcpy(v, __builtin_assume_aligned(row + e0, 4), sizeof v);
#pragma unroll
    for (int i = 0; i < NPL; ++i) l[i] = Num<T>::get(v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < NPL; ++i) l[i] = e0 + i < experts ? Num<T>::get(row[e0 + i]) : kNegInf;
  }
#pragma unroll
  for (int i = 0; i < NPL; ++i) l[i] = l[i] == l[i] ? l[i] : kNegInf;
}

// Softmax statistics of a token over its W lanes: e <- the exponentials of l
// less the maximum, inv <- the reciprocal of their sum (0 where every logit is
// -Infinity).  Returns the maximum.
template <int W, int NPL>
__device__ __forceinline__ float softmax_stats(const float (&l)[NPL], float (&e)[NPL], float *inv) {
  float mx = l[0];
#pragma unroll
  for (int i = 1; i < NPL; ++i) mx = fmaxf(mx, l[i]);
  mx = group_max<W>(mx);
  if (mx == kNegInf) mx = 0.f;
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < NPL; ++i) {
    e[i] = exp_f32(l[i] - mx);
    s += e[i];
  }
  s = group_sum<W>(s);
  *inv = s > 0.f || s != s ? 1.f / s : 0.f;
  return mx;
}

__device__ __forceinline__ float sigmoid(float x) { return 1.f / (1.f + exp_f32(-x)); }

// The score of a choice with logit x (-Infinity: none), before any division by
// the chosen ones' sum.  m, inv: softmax statistics, where they are needed.
// A normalised softmax is one over the chosen logits alone, whatever m is, so
// the other experts' exponentials are never computed for it.  A normalised
// sigmoid is e^x / (1 + e^x) times e^-m, m the row's largest chosen logit but at
// most 0: the factor leaves the shares as they are and keeps the scores of a row
// of small logits inside binary32.  m ends at -700, where binary64 ends too, so
// that masks of the type's lowest value have no share.  Only a wave that has
// such a logit takes m (all of them: 32768 x 64, 6 choices 7.1 -> 7.4 us).
template <int W>
__device__ __forceinline__ float choice_score(const RouteArgs &a, float x, float m, float inv) {
  if (a.score != 0) {
    if (!a.normalise || __ballot(x < -64.f && x > kNegInf) == 0) return x == kNegInf ? 0.f : sigmoid(x);
    m = fminf(fmaxf(group_max<W>(x), -700.f), 0.f);
    return x == kNegInf ? 0.f : (x > 0.f ? 1.f : exp_f32(x - m)) / (1.f + exp_f32(-fabsf(x)));
  }
  if (!a.normalise) return exp_f32(x - m) * inv;
  m = group_max<W>(x);
  return x == kNegInf ? 0.f : exp_f32(x - m);
}

// Keys as integers of the same order (-0 made +0 first, as they compare equal),
// which compare and reduce without the care NaN takes.
__device__ __forceinline__ int sort_key(float x) {
  const int i = __float_as_int(x + 0.f);
  return i ^ ((i >> 31) & 0x7fffffff);
}
__device__ __forceinline__ float key_value(int k) { return __int_as_float(k ^ ((k >> 31) & 0x7fffffff)); }
constexpr int kNoKey = (int)0x807fffff;  // of -Infinity

template <int W>
__device__ __forceinline__ int group_max_key(int v) {
  v = max(v, __builtin_amdgcn_update_dpp(v, v, 0xB1, 0xF, 0xF, false));
  v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x4E, 0xF, 0xF, false));
  v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x141, 0xF, 0xF, false));
  v = max(v, __builtin_amdgcn_update_dpp(v, v, 0x140, 0xF, 0xF, false));
  if constexpr (W == 64) {
    v = max_halves<16>(v);
    v = max_halves<32>(v);
  }
  return v;
}

template <typename T, int W, int NPL, bool VEC>
__global__ __launch_bounds__(kThreads) void k_route(RouteArgs a) {
  const int sub = threadIdx.x % W, lane = threadIdx.x % 64;
  const uint32_t t = blockIdx.x * (kThreads / W) + threadIdx.x / W;
  const bool live = t < a.tokens;  // no early exit: the lanes of a wave work on several tokens together
  const T *row = (const T *)a.logits + (uint64_t)(live ? t : 0) * a.ld;
  const int e0 = sub * NPL;
  float l[NPL], bias[NPL];
  if (a.bias != nullptr) {  // under way together with the logits
#pragma unroll
    for (int i = 0; i < NPL; ++i) bias[i] = e0 + i < a.experts ? a.bias[e0 + i] : 0.f;
  }
  load_logits<T, NPL, VEC>(row, e0, a.experts, l);
  float m = 0.f, inv = 0.f;
  if (a.score == 0 && !a.normalise) {
    float e[NPL];
    m = softmax_stats<W, NPL>(l, e, &inv);
  }
  if (a.bias != nullptr) {
#pragma unroll
    for (int i = 0; i < NPL; ++i) {
      const float x = l[i] + bias[i];
      l[i] = x == x ? x : kNegInf;
    }
  }
  int key[NPL];
#pragma unroll
  for (int i = 0; i < NPL; ++i) key[i] = sort_key(l[i]);
  int mine = -1;  // lane j keeps the j-th choice and its key
  float x = kNegInf;
  auto lane_best = [&]() __attribute__((always_inline)) {
    int best = key[0];
#pragma unroll
    for (int i = 1; i + 1 < NPL; i += 2) best = max(max(best, key[i]), key[i + 1]);
    return NPL % 2 == 0 ? max(best, key[NPL - 1]) : best;
  };
  if (sizeof(T) == 2 && a.bias == nullptr) {
    // bfloat16 logits leave room for the index below the key's 16 bits, high
    // for low indices: keys are unique and say which expert they are
#pragma unroll
    for (int i = 0; i < NPL; ++i) key[i] = (key[i] & (int)0xffff0000) | (0xffff - (e0 + i));
    for (int j = 0; j < a.k; ++j) {
      const int top = group_max_key<W>(lane_best());
#pragma unroll
      for (int i = 0; i < NPL; ++i) key[i] = key[i] == top ? kNoKey : key[i];
      if (sub == j && top > (kNoKey | 0xffff)) {
        mine = 0xffff - (top & 0xffff);
        x = key_value((top & (int)0xffff0000) | (top < 0 ? 0xffff : 0));
      }
    }
  } else {
    for (int j = 0; j < a.k; ++j) {
      const int best = lane_best(), top = group_max_key<W>(best);
      uint64_t have = __ballot(best == top && top > kNoKey);
      if constexpr (W == 16) have = (have >> (lane & 48)) & 0xFFFFull;
      const int who = have == 0 ? -1 : __ffsll((unsigned long long)have) - 1;
      // the winner's lowest key that is the maximum: found and taken out
      bool open = sub == who;
      int at = 0;
#pragma unroll
      for (int i = 0; i < NPL; ++i) {
        const bool hit = open && key[i] == top;
        key[i] = hit ? kNoKey : key[i];
        at = hit ? i : at;
        open = open && !hit;
      }
      const int won = __shfl(at, who < 0 ? 0 : who, W);
      if (sub == j) {
        mine = who < 0 ? -1 : who * NPL + won;
        x = who < 0 ? kNegInf : key_value(top);
      }
    }
  }
  if (a.bias != nullptr && mine >= 0) {  // the key is not the logit
    x = Num<T>::get(row[mine]);
    if (x != x) x = kNegInf;
  }
  float u = choice_score<W>(a, x, m, inv);
  if (a.normalise) {
    const float tot = group_sum<W>(u);
    u = tot > 0.f || tot != tot ? u / tot : 0.f;
  }
  if (live && sub < a.k) {
    a.ids[(uint64_t)t * a.k + sub] = mine;
    a.weights[(uint64_t)t * a.k + sub] = a.scale * u;
  }
}

// The gradient recomputes the scores from the logits.  With u the chosen
// scores, divided by their sum where normalised, and g = scale * dweights:
//   softmax             dl_i = p_i (g_i - sum u g)        (g_i = 0 if not chosen)
//   softmax, normalised dl_i = u_i (g_i - sum u g)        (chosen only)
//   sigmoid             dl_i = g_i s_i (1 - s_i)          (chosen only)
//   sigmoid, normalised dl_i = u_i (g_i - sum u g)(1 - s_i)
// 1 - s is the sigmoid of -l: the difference would be a rounding error where s
// is near 1.  Only the first needs the row; the others read the chosen logits.
template <typename T, int W, int NPL, bool VEC>
__global__ __launch_bounds__(kThreads) void k_route_grad(RouteArgs a) {
  __shared__ float coef[kThreads * NPL];
  const int sub = threadIdx.x % W;
  const uint32_t t = blockIdx.x * (kThreads / W) + threadIdx.x / W;
  const bool live = t < a.tokens;
  const T *row = (const T *)a.logits + (uint64_t)(live ? t : 0) * a.ld;
  const int e0 = sub * NPL;
  const bool all = a.score == 0 && !a.normalise;  // every expert's logit moves the softmax
  float *mine = coef + (threadIdx.x / W) * (W * NPL);
#pragma unroll
  for (int i = 0; i < NPL; ++i) mine[e0 + i] = 0.f;
  int id = -1;
  float g = 0.f, x = kNegInf;
  if (live && sub < a.k) {
    id = a.ids[(uint64_t)t * a.k + sub];
    if (id < 0 || id >= a.experts) id = -1;
    if (id >= 0) {
      g = a.scale * a.dweights[(uint64_t)t * a.k + sub];
      x = Num<T>::get(row[id]);
      if (x != x) x = kNegInf;
    }
  }
  float e[NPL];
  float m = 0.f, inv = 0.f;
  if (all) {
    float l[NPL];
    load_logits<T, NPL, VEC>(row, e0, a.experts, l);
    m = softmax_stats<W, NPL>(l, e, &inv);
  }
  const float p = choice_score<W>(a, x, m, inv);
  float u = p;
  if (a.normalise) {
    const float tot = group_sum<W>(p);
    u = tot > 0.f || tot != tot ? p / tot : 0.f;
  }
  const float mean = group_sum<W>(u * g);
  __syncthreads();
  if (id >= 0) {
    float c;
    if (a.score == 0)
      c = a.normalise ? u * (g - mean) : p * g;
    else
      c = (a.normalise ? u * (g - mean) : g * p) * sigmoid(-x);
    mine[id] = c;
  }
  __syncthreads();
  if (!live) return;
  float d[NPL];
#pragma unroll
  for (int i = 0; i < NPL; ++i) {
    d[i] = mine[e0 + i];
    if (all) d[i] -= e[i] * inv * mean;
  }
  T *drow = (T *)a.dlogits + (uint64_t)t * a.ldd;
  if (VEC && e0 + NPL <= a.experts) {
    T v[NPL];
#pragma unroll
    for (int i = 0; i < NPL; ++i) v[i] = Num<T>::put(d[i]);
    __builtin_memcpy(__builtin_assume_aligned(drow + e0, 4), v, sizeof v);
  } else {
#pragma unroll
    for (int i = 0; i < NPL; ++i)
      if (e0 + i < a.experts) drow[e0 + i] = Num<T>::put(d[i]);
  }
}

// ---------------------------------------------------------------- sorting by expert
//
// A stable counting sort.  Each block takes `chunk` consecutive (token,
// choice) pairs, each of its waves a consecutive quarter of them, and a wave
// 64 at a time, so a pair's place is: the rows of smaller experts, the
// expert's rows in earlier blocks, in earlier waves of this block, in earlier
// batches of this wave, and among the lower lanes.  Two launches, 4.8 + 6.4 us
// for 49152 pairs, almost all of it latency; up to 1024 pairs every block that
// copies rows sorts them for itself instead, which saves a launch or two (128
// pairs over 32 experts with their rows of 14 KiB: 6 us in all).
struct SortArgs {
  const int32_t *ids;
  uint32_t pairs, chunk, blocks;
  int first, experts, bits;
  int32_t *offsets, *slots, *rows;
  int32_t *hist;  // [blocks][experts]
};

__device__ __forceinline__ int local_expert(const SortArgs &a, uint32_t i) {
  const int64_t e = (int64_t)a.ids[i] - a.first;
  return e >= 0 && e < a.experts ? (int)e : -1;
}

constexpr int kAheadIds = 4;  // ids of a lane under way

// f(i, local expert or -1) for a wave's pairs [lo, hi), 64 at a time (every
// lane takes part in each batch; past hi the expert is -1).
template <typename F>
__device__ __forceinline__ void wave_pairs(const SortArgs &a, uint32_t lo, uint32_t hi, F f) {
  for (uint32_t base = lo + threadIdx.x % 64; base - threadIdx.x % 64 < hi; base += 64 * kAheadIds) {
    int e[kAheadIds];
#pragma unroll
    for (int n = 0; n < kAheadIds; ++n) e[n] = base + 64 * n < hi ? local_expert(a, base + 64 * n) : -1;
#pragma unroll
    for (int n = 0; n < kAheadIds; ++n) f(base + 64 * n, e[n]);
  }
}

// Counts of a wave's pairs [lo, hi) into cnt[experts] (zeroed, LDS).
__device__ __forceinline__ void wave_count(const SortArgs &a, uint32_t lo, uint32_t hi, int *cnt) {
  wave_pairs(a, lo, hi, [&](uint32_t, int e) {
    if (e >= 0) atomicAdd(&cnt[e], 1);  // integers: the order does not matter
  });
}

// Places of a wave's pairs [lo, hi), cnt[e] = the first place of expert e for
// this wave (advanced).  put(i, place) is called for every pair, -1 where it
// is not local.
template <typename F>
__device__ __forceinline__ void wave_place(const SortArgs &a, uint32_t lo, uint32_t hi, int *cnt, F put) {
  const int lane = threadIdx.x % 64;
  wave_pairs(a, lo, hi, [&](uint32_t i, int e) {
    uint64_t same = __ballot(e >= 0);  // lanes with this lane's expert
    for (int b = 0; b < a.bits; ++b) {
      const uint64_t m = __ballot(e >= 0 && ((e >> b) & 1));
      same &= ((e >> b) & 1) ? m : ~m;
    }
    const int before = __popcll(same & ((1ull << lane) - 1ull));
    int place = -1;
    if (e >= 0) place = cnt[e] + before;
    __builtin_amdgcn_wave_barrier();
    if (e >= 0 && before == 0) cnt[e] += __popcll(same);
    __builtin_amdgcn_wave_barrier();
    if (i < hi) put(i, place);
  });
}

// base[e] <- sum of total[e'] for e' < e, by the block's first wave; returns
// the sum of all through *sum (LDS).
__device__ __forceinline__ void scan_experts(const int *total, int *base, int experts, int *sum) {
  if (threadIdx.x < 64) {
    int carry = 0;
    for (int e0 = 0; e0 < experts; e0 += 64) {
      const int e = e0 + threadIdx.x;
      const int v = e < experts ? total[e] : 0;
      int s = v;
      for (int d = 1; d < 64; d <<= 1) {
        const int up = __shfl_up(s, d);
        if ((int)threadIdx.x >= d) s += up;
      }
      if (e < experts) base[e] = carry + s - v;
      carry += __shfl(s, 63);
    }
    if (threadIdx.x == 0) *sum = carry;
  }
}

constexpr int kWaves = kThreads / 64;

// First launch of a large sort: each block's counts.
static __global__ __launch_bounds__(kThreads) void k_sort_count(SortArgs a) {
  extern __shared__ int cnt[];
  for (int e = threadIdx.x; e < a.experts; e += kThreads) cnt[e] = 0;
  __syncthreads();
  const uint32_t lo = blockIdx.x * a.chunk, hi = min(a.pairs, lo + a.chunk);
  for (uint32_t i = lo + threadIdx.x; i < hi; i += kThreads) {
    const int e = local_expert(a, i);
    if (e >= 0) atomicAdd(&cnt[e], 1);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < a.experts; e += kThreads) a.hist[(uint64_t)blockIdx.x * a.experts + e] = cnt[e];
}

// Places of this block's pairs.  LDS: total[experts], base[experts],
// before[experts], cnt[kWaves][experts].  hist NULL: the block has every pair
// (blocks == 1).
constexpr int kSortInts = 3 + kWaves;  // LDS integers an expert

template <typename F>
__device__ __forceinline__ void block_sort(const SortArgs &a, uint32_t block, int *lds, int *sum, F put) {
  int *total = lds, *base = lds + a.experts, *before = lds + 2 * a.experts, *cnt = lds + 3 * a.experts;
  for (int i = threadIdx.x; i < kSortInts * a.experts; i += kThreads) lds[i] = 0;
  __syncthreads();
  const int wave = threadIdx.x / 64;
  const uint32_t part = a.chunk / kWaves;
  const uint32_t lo = min(a.pairs, block * a.chunk + wave * part);
  const uint32_t hi = min(a.pairs, lo + part);
  wave_count(a, lo, hi, cnt + wave * a.experts);
  // per expert: rows of all blocks, and of the blocks before this one
  if (a.hist != nullptr) {
    const uint32_t n = a.blocks * a.experts;
    for (uint32_t i = threadIdx.x; i < n; i += kThreads) {
      const int v = a.hist[i], e = i % a.experts;
      if (v == 0) continue;
      atomicAdd(&total[e], v);
      if (i < block * a.experts) atomicAdd(&before[e], v);
    }
  }
  __syncthreads();
  if (a.hist == nullptr) {
    for (int e = threadIdx.x; e < a.experts; e += kThreads) {
      int all = 0;
      for (int w = 0; w < kWaves; ++w) all += cnt[w * a.experts + e];
      total[e] = all;
    }
    __syncthreads();
  }
  scan_experts(total, base, a.experts, sum);
  __syncthreads();
  for (int e = threadIdx.x; e < a.experts; e += kThreads) {
    int at = base[e] + before[e];
    for (int w = 0; w < kWaves; ++w) {
      const int c = cnt[w * a.experts + e];
      cnt[w * a.experts + e] = at;
      at += c;
    }
  }
  __syncthreads();
  wave_place(a, lo, hi, cnt + wave * a.experts, put);
}

__device__ __forceinline__ void write_offsets(const SortArgs &a, const int *base, int sum) {
  for (int e = threadIdx.x; e < a.experts; e += kThreads) a.offsets[e] = base[e];
  if (threadIdx.x == 0) a.offsets[a.experts] = sum;
}

// Second launch: places, the sorted order and the offsets.
static __global__ __launch_bounds__(kThreads) void k_sort_place(SortArgs a) {
  extern __shared__ int lds[];
  __shared__ int sum;
  block_sort(a, blockIdx.x, lds, &sum, [&](uint32_t i, int place) {
    a.rows[i] = place;
    if (place >= 0) a.slots[place] = (int32_t)i;
  });
  if (blockIdx.x == 0) write_offsets(a, lds + a.experts, sum);
  const uint32_t lo = blockIdx.x * a.chunk, hi = min(a.pairs, lo + a.chunk);
  for (uint32_t i = lo + threadIdx.x; i < hi; i += kThreads)
    if (i >= (uint32_t)sum) a.slots[i] = -1;
}

// ---------------------------------------------------------------- rows
struct RowArgs {
  const void *x;  // dispatch: token rows; combine: expert rows
  uint64_t ldx;
  const void *extra;  // combine: residual; combine_grad: dout
  uint64_t lde;
  void *out;
  uint64_t ldo;
  const int32_t *rows;
  const float *weights;
  float *dweights;
  uint32_t tokens, nrows;
  int k;
  uint32_t features;
};

// A row is cut into chunks of 16 bytes (VEC) or single elements; TPR threads
// (64 or 256) work on one token's row.
template <typename T, bool VEC>
constexpr int chunk_elems() {
  return VEC ? Num<T>::kPer16 : 1;
}

// A chunk as it lies in memory: converted where it is used, so that a load
// does not wait for the one before it.
template <typename T, int C>
struct Raw {
  typedef T vec __attribute__((ext_vector_type(C)));
  vec r;
  __device__ __forceinline__ void load(const T *p) { r = *reinterpret_cast<const vec *>(p); }
  __device__ __forceinline__ float get(int i) const { return Num<T>::get(r[i]); }
};

// One token's row to each of its local sorted rows; read once, written up to
// k times, so a token's row comes from memory once however many experts it
// has here.  Bound by memory: the whole dispatch of 8192 tokens of 14 KiB to
// 12288 rows takes 58-73 us (3.8-4.7 TB/s).
template <typename T, bool VEC, int TPR>
__device__ __forceinline__ void push_row(const RowArgs &a, uint32_t t, const int32_t *rows_of) {
  constexpr int C = chunk_elems<T, VEC>();
  typedef T vec __attribute__((ext_vector_type(C)));
  bool any = false;
  for (int j = 0; j < a.k; ++j) any = any || rows_of[j] >= 0;
  if (!any) return;
  const uint32_t chunks = a.features / C;
  const vec *src = (const vec *)((const T *)a.x + (uint64_t)t * a.ldx);
  constexpr int kAhead = 4;  // loads of a thread under way
  for (uint32_t c0 = threadIdx.x % TPR; c0 < chunks; c0 += TPR * kAhead) {
    vec v[kAhead];
#pragma unroll
    for (int n = 0; n < kAhead; ++n)
      if (c0 + n * TPR < chunks) v[n] = src[c0 + n * TPR];
    for (int j = 0; j < a.k; ++j) {
      const int r = rows_of[j];
      if (r < 0) continue;
      vec *to = (vec *)((T *)a.out + (uint64_t)(uint32_t)r * a.ldo);
#pragma unroll
      for (int n = 0; n < kAhead; ++n)
        if (c0 + n * TPR < chunks) to[c0 + n * TPR] = v[n];
    }
  }
}

template <typename T, bool VEC, int TPR>
__global__ __launch_bounds__(kThreads) void k_push(RowArgs a) {
  const uint32_t t = blockIdx.x * (kThreads / TPR) + threadIdx.x / TPR;
  if (t >= a.tokens) return;
  push_row<T, VEC, TPR>(a, t, a.rows + (uint64_t)t * a.k);
}

// Few pairs: every block sorts all of them for itself and pushes its own
// tokens, in one launch instead of two.
template <typename T, bool VEC>
__global__ __launch_bounds__(kThreads) void k_dispatch_small(SortArgs s, RowArgs a) {
  extern __shared__ int lds[];
  __shared__ int sum;
  int *mine = lds + kSortInts * s.experts;  // rows of this block's token
  const uint32_t t = blockIdx.x;
  const uint32_t lo = t * (uint32_t)a.k, hi = lo + (uint32_t)a.k;
  const bool lead = blockIdx.x == 0;
  block_sort(s, 0, lds, &sum, [&](uint32_t i, int place) {
    if (i >= lo && i < hi) mine[i - lo] = place;
    if (lead) {
      s.rows[i] = place;
      if (place >= 0) s.slots[place] = (int32_t)i;
    }
  });
  __syncthreads();
  if (lead) {
    write_offsets(s, lds + s.experts, sum);
    for (uint32_t i = threadIdx.x; i < s.pairs; i += kThreads)
      if (i >= (uint32_t)sum) s.slots[i] = -1;
  }
  if (a.x != nullptr && t < a.tokens) push_row<T, VEC, kThreads>(a, t, mine);
}

// out[t] = sum_j w[t,j] y[rows[t,j]] (+ residual).  The loads of up to
// kBatch expert rows are issued before the first of them is used (converting
// each as it is loaded made them wait for each other: 174 -> 98 us).  Bound by
// memory: 8192 tokens of 14 KiB from 12288 rows in 91-106 us (3.9-4.6 TB/s).
// Few tokens by the chain of four such batches a thread: 1, 16 and 64 tokens of
// 8 rows of 14 KiB take 10.5, 11.0 and 11.6 us.
constexpr int kBatch = 8;

template <typename T, bool VEC, int TPR>
__global__ __launch_bounds__(kThreads) void k_combine(RowArgs a) {
  constexpr int C = chunk_elems<T, VEC>();
  const uint32_t t = blockIdx.x * (kThreads / TPR) + threadIdx.x / TPR;
  if (t >= a.tokens) return;
  const int32_t *rows = a.rows + (uint64_t)t * a.k;
  const float *w = a.weights == nullptr ? nullptr : a.weights + (uint64_t)t * a.k;
  const uint32_t chunks = a.features / C;
  for (uint32_t c = threadIdx.x % TPR; c < chunks; c += TPR) {
    Pack<T, C, VEC> acc;
    Raw<T, C> res;
#pragma unroll
    for (int i = 0; i < C; ++i) acc.v[i] = 0.f;
    if (a.extra != nullptr) res.load((const T *)a.extra + (uint64_t)t * a.lde + c * C);
    for (int j0 = 0; j0 < a.k; j0 += kBatch) {
      Raw<T, C> y[kBatch];
      bool ok[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int r = j0 + j < a.k ? rows[j0 + j] : -1;
        ok[j] = r >= 0 && (uint32_t)r < a.nrows;
        if (ok[j]) y[j].load((const T *)a.x + (uint64_t)(uint32_t)r * a.ldx + c * C);
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        if (!ok[j]) continue;
        const float wj = w == nullptr ? 1.f : w[j0 + j];
#pragma unroll
        for (int i = 0; i < C; ++i) acc.v[i] = __builtin_fmaf(wj, y[j].get(i), acc.v[i]);
      }
    }
    if (a.extra != nullptr) {
#pragma unroll
      for (int i = 0; i < C; ++i) acc.v[i] += res.get(i);
    }
    acc.store((T *)a.out + (uint64_t)t * a.ldo + c * C);
  }
}

// dy[rows[t,j]] = w[t,j] dout[t], dw[t,j] = <dout[t], y[rows[t,j]]>.  A
// thread's partial products of up to kBatch choices stay in registers; the
// row's threads join them once a batch.  Bound by memory: 4397 tokens of 4104
// binary32, 2 choices, in 82 us (4.4 TB/s).
template <typename T, bool VEC, int TPR>
__global__ __launch_bounds__(kThreads) void k_combine_grad(RowArgs a) {
  constexpr int C = chunk_elems<T, VEC>();
  __shared__ float part[kWaves][kBatch];
  const uint32_t t = blockIdx.x * (kThreads / TPR) + threadIdx.x / TPR;
  const bool live = t < a.tokens;
  const uint64_t t0 = live ? t : 0;
  const int32_t *rows = a.rows + t0 * a.k;
  const float *w = a.weights == nullptr ? nullptr : a.weights + t0 * a.k;
  const uint32_t chunks = live ? a.features / C : 0;
  const int wave = threadIdx.x / 64;
  for (int j0 = 0; j0 < a.k; j0 += kBatch) {
    float dot[kBatch], wj[kBatch];
    int r[kBatch];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      dot[j] = 0.f;
      r[j] = j0 + j < a.k ? rows[j0 + j] : -1;
      if (r[j] >= 0 && (uint32_t)r[j] >= a.nrows) r[j] = -1;
      wj[j] = w == nullptr || r[j] < 0 ? 1.f : w[j0 + j];
    }
    for (uint32_t c = threadIdx.x % TPR; c < chunks; c += TPR) {
      Pack<T, C, VEC> d, o;
      Raw<T, C> y[kBatch];
      d.load((const T *)a.extra + t0 * a.lde + c * C);
      if (a.dweights != nullptr) {
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
          if (r[j] >= 0) y[j].load((const T *)a.x + (uint64_t)r[j] * a.ldx + c * C);
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        if (r[j] < 0) continue;
#pragma unroll
        for (int i = 0; i < C; ++i) o.v[i] = wj[j] * d.v[i];
        o.store((T *)a.out + (uint64_t)r[j] * a.ldo + c * C);
        if (a.dweights != nullptr) {
#pragma unroll
          for (int i = 0; i < C; ++i) dot[j] = __builtin_fmaf(d.v[i], y[j].get(i), dot[j]);
        }
      }
    }
    if (a.dweights == nullptr) continue;
#pragma unroll
    for (int j = 0; j < kBatch; ++j) dot[j] = group_sum<64>(dot[j]);
    if constexpr (TPR == 64) {
      const int lane = threadIdx.x % 64;
#pragma unroll
      for (int j = 0; j < kBatch; ++j)
        if (live && lane == j && j0 + j < a.k) a.dweights[t0 * a.k + j0 + j] = r[j] < 0 ? 0.f : dot[j];
    } else {
      __syncthreads();
      if (threadIdx.x % 64 == 0) {
#pragma unroll
        for (int j = 0; j < kBatch; ++j) part[wave][j] = dot[j];
      }
      __syncthreads();
      const int j = threadIdx.x;
      if (live && j < kBatch && j0 + j < a.k) {
        float s = 0.f;
#pragma unroll
        for (int v = 0; v < kWaves; ++v) s += part[v][j];
        a.dweights[t0 * a.k + j0 + j] = s;
      }
    }
  }
}

}  // namespace moe
}  // namespace llc
