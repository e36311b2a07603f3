// Grouped matrix products with their epilogues (include/llmoe.h, ll_linear*).
//
// One kernel computes C[m, n] = sum_k P(m, k) Q(n, k) for the three products:
//   forward  C = y,  P = x  (rows),        Q = w (rows: out),   k = in
//   grad_x   C = dx, P = dz (rows),        Q = w (columns: in), k = out
//   grad_w   C = dw, P = dz (columns: out), Q = x (columns: in), k = rows
// An operand lies in memory either along k ("KM": a row is one m or n) or
// along m or n ("RM": a row is one k).
//
// A workgroup owns a BM x BN tile of C, in registers.  Both operands pass
// through LDS in stages of 64 (bf16) or 32 (binary32) k, loaded straight from
// memory into LDS.  The matrix instruction takes Q as its first operand, so a
// lane ends up with four consecutive n of one m.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/llmoe.h"
#include "ll_num.hpp"

namespace llc {
namespace lin {

enum Pass { kForward = 0, kGradX = 1, kGradW = 2 };

struct Args {
  const void *p, *q;
  uint64_t ldp, ldq;
  uint64_t qstride, cstride;  // between groups: weights (forward, grad_x), dw (grad_w)
  const int32_t *offsets;
  int groups;
  uint32_t rows;     // of x / dz
  uint32_t m, n, k;  // extents of C and of the sum; rows stand for m (forward, grad_x) or k (grad_w)
  uint32_t tiles_m, tiles_n;
  const void *bias, *res, *z;
  uint64_t ldr, ldz, ldc;
  void *c, *zout, *dbias;
  int act;
  uint32_t flags;  // LL_GRAD_*
  bool vec_c;      // dx: every epilogue row starts at a 16-byte address
  float *parts;      // sums of the splits of k, [splits][rows of C][part_row], or NULL
  uint32_t splits, rows_c;
  bool sum_bias;  // grad_w: the tile kernel computes dbias too
  uint32_t tail;  // 1: leaves a short last round of tiles out; 2: runs that round, in quarters
  uint32_t part_half, part_row;  // columns of a (gated: half a) row of parts, multiples of kEw
};

// ---------------------------------------------------------------- activations
//
// GELU is x Phi(x), Phi the normal distribution function.  As (1 + erf) / 2 it
// cancels below zero (x = -5: 4 % of the result, x = -5.6: all of it), so it is
// Phi(-z) = e^(-z^2 / 2) M(z) for z >= 0, and 1 less that above.  M, Mills'
// ratio over sqrt(2 pi), falls like 1 / z and is smooth in u = 1 / (1 + .34 z):
// u times a polynomial of degree 8 in u, fitted to erfcx by least squares
// weighted towards the largest relative error (3e-8; 3.1e-7 as computed here,
// z up to 13).  The slope shares the exponential.  Gradient of 8192 x 4096
// bfloat16 through GELU: 36.9 us, 5.4 TB/s; with erf 41.5, with erfc 54.0.
__device__ __forceinline__ float normal_cdf(float x, float *bell) {
  const float z = fabsf(x), u = __builtin_amdgcn_rcpf(__builtin_fmaf(0.34f, z, 1.f));
  float m = -0.02612048014998436f;
  m = __builtin_fmaf(m, u, 0.1394995152950287f);
  m = __builtin_fmaf(m, u, -0.2731328010559082f);
  m = __builtin_fmaf(m, u, 0.20218272507190704f);
  m = __builtin_fmaf(m, u, -0.044718485325574875f);
  m = __builtin_fmaf(m, u, 0.11535917222499847f);
  m = __builtin_fmaf(m, u, 0.11519765853881836f);
  m = __builtin_fmaf(m, u, 0.13611219823360443f);
  m = __builtin_fmaf(m, u, 0.13562050461769104f);
  *bell = exp_f32(-0.5f * x * x);
  const float tail = *bell * (m * u);
  return x < 0.f ? tail : 1.f - tail;
}
__device__ __forceinline__ float gelu(float x) {
  float bell;
  return x * normal_cdf(x, &bell);
}
__device__ __forceinline__ float silu(float x) { return x / (1.f + expf(-x)); }
__device__ __forceinline__ float gelu_slope(float x) {
  float bell;
  const float phi = normal_cdf(x, &bell);
  return phi + x * bell * 0.39894228040143268f;
}
__device__ __forceinline__ float silu_slope(float x) {
  const float s = 1.f / (1.f + expf(-x));
  return s * (1.f + x * (1.f - s));
}
// The ungated activation, or a gated one's activation of its first half.
__device__ __forceinline__ float act1(float x, int act) {
  switch (act) {
    case LL_ACT_RELU: return x > 0.f || x != x ? x : 0.f;
    case LL_ACT_GELU:
    case LL_ACT_GEGLU: return gelu(x);
    case LL_ACT_SILU:
    case LL_ACT_SWIGLU: return silu(x);
    default: return x;
  }
}
__device__ __forceinline__ float slope1(float x, int act) {
  switch (act) {
    case LL_ACT_RELU: return x > 0.f ? 1.f : 0.f;
    case LL_ACT_GELU:
    case LL_ACT_GEGLU: return gelu_slope(x);
    case LL_ACT_SILU:
    case LL_ACT_SWIGLU: return silu_slope(x);
    default: return 1.f;
  }
}
__host__ __device__ constexpr bool gated(int act) { return act == LL_ACT_SWIGLU || act == LL_ACT_GEGLU; }

// ---------------------------------------------------------------- which tile
//
// Workgroups go to the 8 XCDs in turn, each with an L2 of its own.  Tiles are
// numbered in bands of kBand row tiles, column by column, and XCD x takes runs
// x, x + 8, ... of kRun consecutive tiles, what its 32 CUs work on at a time:
// those share a few panels of each operand, and tiles of less work (a group's
// last) fall to every XCD alike.
constexpr uint32_t kBand = 4, kRun = 32;

// Tile number t, in bands.
__device__ __forceinline__ void number_of(uint32_t t, uint32_t tiles_m, uint32_t tiles_n, uint32_t *tm, uint32_t *tn) {
  const uint32_t band = t / (kBand * tiles_n), in_band = t % (kBand * tiles_n);
  const uint32_t high = min(kBand, tiles_m - band * kBand);
  *tm = band * kBand + in_band % high;
  *tn = in_band / high;
}

// Workgroup `id`'s tile among the first `total` of tiles_m x tiles_n.
__device__ __forceinline__ bool tile_of(uint32_t id, uint32_t total, uint32_t tiles_m, uint32_t tiles_n, uint32_t *tm,
                                        uint32_t *tn) {
  if (id >= total) return false;
  const uint32_t whole = total / (8 * kRun) * (8 * kRun);
  uint32_t t;
  if (id < whole) {
    const uint32_t x = id % 8, i = id / 8;
    t = (i / kRun * 8 + x) * kRun + i % kRun;
  } else {  // the last, shorter runs
    const uint32_t left = total - whole, i = id - whole, x = i % 8, each = left / 8, more = left % 8;
    t = whole + x * each + min(x, more) + i / 8;
  }
  number_of(t, tiles_m, tiles_n, tm, tn);
  return true;
}

// Rows [lo, hi) of group g; clamped to the rows there are.
__device__ __forceinline__ void group_rows(const Args &a, int g, uint32_t *lo, uint32_t *hi) {
  *lo = 0;
  *hi = a.rows;
  if (a.offsets == nullptr) return;
  *lo = (uint32_t)min(max(a.offsets[g], 0), (int)a.rows);
  *hi = (uint32_t)min(max(a.offsets[g + 1], (int)*lo), (int)a.rows);
}

// Inclusive sums of the row tiles of groups g0 .. g0 + 63, one a lane.
__device__ __forceinline__ uint32_t scan_tiles(const Args &a, int g0, uint32_t bm, uint32_t *lo, uint32_t *hi,
                                               uint32_t *tiles) {
  const int lane = threadIdx.x % 64;
  *lo = *hi = 0;
  if (g0 + lane < a.groups) group_rows(a, g0 + lane, lo, hi);
  *tiles = (*hi - *lo + bm - 1) / bm;
  uint32_t incl = *tiles;
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t up = __shfl_up(incl, d);
    if (lane >= d) incl += up;
  }
  return incl;
}

// A round is what the chip's 256 CUs work on at a time, one 256-wide tile each.
// A last round of at most kMaxTail tiles takes as long as a whole one, so the
// launch leaves it out and another runs it in 128-wide quarters (grad_x of 8
// groups of about 1024 rows, 7168 -> 2048, 288 tiles: 400 -> 300-315 us).
constexpr uint32_t kRound = 256, kMaxTail = 128;

__device__ __forceinline__ uint32_t tail_tiles(uint32_t total) {
  const uint32_t rest = total % kRound;
  return total > kRound && rest <= kMaxTail ? rest : 0;
}

// Workgroup `id`'s tile among tiles_m x tiles_n of edge bm.  Quarters (tail 2):
// the tiles are twice as wide as the workgroup's, whose edge is bm / 2, and
// *quarter is which of the four.
__device__ __forceinline__ bool pick_tile(const Args &a, uint32_t id, uint32_t tiles_m, uint32_t *tm, uint32_t *tn,
                                          uint32_t *quarter) {
  const uint32_t total = tiles_m * a.tiles_n;
  *quarter = 0;
  if (a.tail == 0) return tile_of(id, total, tiles_m, a.tiles_n, tm, tn);
  const uint32_t rest = tail_tiles(total);
  if (a.tail == 1) return tile_of(id, total - rest, tiles_m, a.tiles_n, tm, tn);
  if (id >= 4 * rest) return false;
  *quarter = id / rest;
  number_of(total - rest + id % rest, tiles_m, a.tiles_n, tm, tn);
  return true;
}

// The tile of workgroup `id` among the grouped rows: its group, first row, end
// of the group's rows, and column tile.  false: there is none.  Every lane of
// the calling wave takes part.
__device__ __forceinline__ bool find_rows(const Args &a, uint32_t id, uint32_t edge, int *group, uint32_t *row0,
                                          uint32_t *row1, uint32_t *tn) {
  const uint32_t bm = a.tail == 2 ? 2 * edge : edge;
  uint32_t tm, quarter;
  auto place = [&]() {
    if (a.tail == 2) {
      *row0 += quarter / 2 * edge;
      *tn = *tn * 2 + quarter % 2;
    }
    return *row0 < *row1;
  };
  if (a.offsets == nullptr) {
    if (!pick_tile(a, id, (a.rows + bm - 1) / bm, &tm, tn, &quarter)) return false;
    *group = 0;
    *row0 = tm * bm;
    *row1 = a.rows;
    return place();
  }
  uint32_t lo, hi, tiles, incl = 0, total = 0;
  for (int g0 = 0; g0 < a.groups; g0 += 64) {
    incl = scan_tiles(a, g0, bm, &lo, &hi, &tiles);
    total += (uint32_t)__builtin_amdgcn_readlane((int)incl, 63);
  }
  if (!pick_tile(a, id, total, &tm, tn, &quarter)) return false;
  uint32_t before = 0;
  for (int g0 = 0; g0 < a.groups; g0 += 64) {
    if (a.groups > 64) incl = scan_tiles(a, g0, bm, &lo, &hi, &tiles);
    const uint64_t past = __ballot(before + incl > tm);
    if (past != 0) {
      const int who = __ffsll((unsigned long long)past) - 1;
      const uint32_t first = before + __builtin_amdgcn_readlane((int)(incl - tiles), who);
      *group = g0 + who;
      *row0 = __builtin_amdgcn_readlane((int)lo, who) + (tm - first) * bm;
      *row1 = __builtin_amdgcn_readlane((int)hi, who);
      return place();
    }
    before += (uint32_t)__builtin_amdgcn_readlane((int)incl, 63);
  }
  return false;
}

// ---------------------------------------------------------------- operand stages in LDS
//
// A stage holds R entries of m or n by 128 bytes of k in R * 128 bytes, as
// 16-byte chunks.  KM: entry r's 8 chunks at r * 128, chunk c at position c ^
// (r & 7), so that 8 lanes that read one chunk of 8 entries touch 8 different
// 16-byte columns.  128 bytes of k at a time, because a load of half a cache
// line costs L2 as much as a whole one: with stages of 64 bytes the forward
// product of 8192^3 took 892 us against 768 for grad_x, one of whose operands
// is loaded in longer rows.  RM: k row r's chunks at r * R * sizeof(T), chunk c
// at position c ^ swz(r), which keeps pairs (bf16) or fours (binary32) of
// chunks together, as one fragment reads them, and spreads the k rows of a
// read over the banks.
template <typename T>
struct Step;
template <>
struct Step<__bf16> {
  static constexpr int kBK = 64, kMma = 32;  // a 16x16x32 instruction per half of a stage
  typedef bf16x8 frag;
};
template <>
struct Step<float> {
  static constexpr int kBK = 32, kMma = 16;  // four 16x16x4 instructions
  typedef f32x4 frag;
};

template <typename T, int R>
__device__ __forceinline__ uint32_t rm_swz(uint32_t krow) {
  constexpr uint32_t kMask = R * sizeof(T) / 16 - 1;
  if constexpr (sizeof(T) == 2)
    return (((krow & 3) | (((krow >> 3) & 1) << 2)) << 1) & kMask;
  else
    return (((krow >> 2) & 3) << 2) & kMask;
}

// A fragment of half ks of a stage: lane (i, q) = (lane % 16, lane / 16) holds
// entry dim0 + i at k = ks * kMma + q * kMma / 4 + 0 .. kMma / 4 - 1.  frag_off
// is where a lane's part of it starts in an operand's stage; RM: the second
// half lies kMma k rows further on, with the same swizzle.
template <typename T, int R, bool KM>
__device__ __forceinline__ uint32_t frag_off(uint32_t dim0, int ks) {
  const uint32_t lane = threadIdx.x % 64, i = lane % 16, q = lane / 16;
  if constexpr (KM) {
    const uint32_t r = dim0 + i, chunk = ks * 4 + q;
    return r * 128 + ((chunk ^ (r & 7)) << 4);
  } else if constexpr (sizeof(T) == 2) {
    const uint32_t krow = q * 8 + i / 4, chunk = dim0 / 8 + (i % 4) / 2;
    return (ks * 32 + krow) * (R * 2) + ((chunk ^ rm_swz<T, R>(krow)) << 4) + (i % 2) * 8;
  } else {
    const uint32_t krow = q * 4, col = dim0 + i;
    return (ks * 16 + krow) * (R * 4) + (((col / 4) ^ rm_swz<T, R>(krow)) << 4) + (col % 4) * 4;
  }
}
template <typename T, int R, bool KM>
__device__ __forceinline__ typename Step<T>::frag read_frag(const char *at) {
  if constexpr (KM) {
    return *reinterpret_cast<const typename Step<T>::frag *>(at);
  } else if constexpr (sizeof(T) == 2) {
    // the transposing read: 16 lanes take 4 k rows of 16 columns, and lane i
    // receives column i of the 4 rows; 4 rows on, the swizzle is the same
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    union {
      s16x4 half[2];
      bf16x8 all;
    } u;
    u.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)at);
    u.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(at + 4 * R * 2));
    return u.all;
  } else {
    f32x4 v;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = *reinterpret_cast<const float *>(at + j * R * 4);
    return v;
  }
}

__device__ __forceinline__ f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(f32x4 a, f32x4 b, f32x4 c) {
#pragma unroll
  for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
  return c;
}

// Which row of the weight entry j of a tile is.  Gated: a wave's first half of
// columns are activations, its second half the same columns of the other half
// of the weight, so both halves of a column end up in one lane.
template <int WTN, bool GATED>
__device__ __forceinline__ uint32_t q_row(uint32_t tile_n, uint32_t bn, uint32_t j, uint32_t n, bool *ok) {
  if constexpr (!GATED) {
    const uint32_t r = tile_n * bn + j;
    *ok = r < n;
    return r;
  } else {
    const uint32_t w = j / WTN, i = j % WTN, half = n / 2;
    const uint32_t col = tile_n * (bn / 2) + w * (WTN / 2) + i % (WTN / 2);
    *ok = col < half;
    return i < WTN / 2 ? col : half + col;
  }
}

constexpr uint32_t kOutside = 0xFFFFFFF0u;  // a buffer offset past the resource: reads as zero

// How an operand's rows lie in memory.
enum Rows {
  kAnyRows = 0,    // 2-byte aligned (bf16): through registers
  kDwordRows = 1,  // every row at a multiple of 4 bytes
  kChunkRows = 2   // every row at a multiple of 16 bytes and whole 16-byte chunks long
};

// Loads one operand's stages, one after the other, kChunks chunks a thread.
//   kChunkRows, kDwordRows: chunks go straight into LDS through a buffer
//   resource; issue() leaves them in flight until the caller waits.  A chunk
//   of kChunkRows lies in the matrix or outside it.  One of kDwordRows may
//   reach past the end of its row: along m or n that touches columns nobody
//   stores, along k clear_tail() writes zeros over it once it has arrived.
//   kAnyRows: fetch() brings them to registers, 16 bytes at any alignment where
//   they lie inside the matrix and single elements at its end, and commit()
//   writes them to LDS.
// KM: SHIFT 1 puts chunk c of entry r at c ^ (r / 2 & 7) instead of c ^ (r & 7).
template <typename T, int R, int NW, bool KM, Rows ROWS, int SHIFT = 0>
struct Loader {
  static constexpr int kEpc = 16 / (int)sizeof(T);
  static constexpr int kBK = Step<T>::kBK;
  static constexpr int kChunks = R * 8 / (NW * 64);
  static constexpr int kRowChunks = KM ? 8 : R / kEpc;
  static_assert(kChunks * NW * 64 == R * 8, "every thread loads the same number of chunks");
  uint64_t base;  // of the stage to load next
  uint64_t left;  // not kChunkRows: bytes from base to the end of the matrix
  uint64_t step;  // bytes from one stage to the next
  uint32_t off[kChunks];  // of the chunk, from base; kOutside: not in the matrix
  uint32_t kk0;
  u32x4 raw[ROWS == kAnyRows ? kChunks : 1];

  // KM: matrix [mat_rows][k], the tile's entry j is row row_of(j) >= first.
  // RM: matrix [k][cols], the tile's first column is `first`.
  template <typename F>
  __device__ __forceinline__ void init(const T *mat, uint64_t ld, uint32_t k, uint32_t mat_rows, uint32_t cols,
                                       uint32_t first, F row_of) {
    constexpr uint64_t kEs = sizeof(T);
    if constexpr (KM) {
      base = (uint64_t)(mat + (uint64_t)first * ld);
      left = mat_rows > first ? ((uint64_t)(mat_rows - 1 - first) * ld + k) * kEs : 0;
      step = kBK * kEs;
    } else {
      base = (uint64_t)(mat + first);
      left = k > 0 && cols > first ? ((uint64_t)(k - 1) * ld + cols - first) * kEs : 0;
      step = kBK * ld * kEs;
    }
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
      const uint32_t pos = (uint32_t)(threadIdx.x / 64 * kChunks + c) * 64 + threadIdx.x % 64;
      if constexpr (KM) {
        static_assert(SHIFT == 0 || kChunks % 2 == 0, "chunk c's place depends on c % 2");
        const uint32_t r = pos / 8, chunk = (pos % 8) ^ (r >> SHIFT & 7);
        bool ok;
        const uint32_t mr = row_of(r, &ok);
        if (SHIFT == 0 || c == 0) kk0 = chunk * kEpc;  // SHIFT 0: the same for every c, rows are 8 apart
        off[c] = ok ? (uint32_t)((uint64_t)(mr - first) * ld * kEs) + chunk * 16 : kOutside;
      } else {
        const uint32_t krow = pos / kRowChunks, chunk = (pos % kRowChunks) ^ rm_swz<T, R>(krow);
        if (c == 0) kk0 = krow;
        off[c] = first + chunk * kEpc < cols ? (uint32_t)(krow * ld * kEs) + chunk * 16 : kOutside;
      }
    }
  }

  // chunk c's first k (KM) or its k row (RM) within a stage
  __device__ __forceinline__ uint32_t kk(int c) const {
    if constexpr (KM && SHIFT == 1) return kk0 ^ (c % 2 * 4 * kEpc);
    return KM ? kk0 : kk0 + c * (64 / kRowChunks);
  }

  __device__ __forceinline__ void advance() {
    base += step;
    if constexpr (ROWS != kChunkRows) left = left > step ? left - step : 0;
  }

  __device__ __forceinline__ void skip(uint32_t stages) {
    base += stages * step;
    if constexpr (ROWS != kChunkRows) left = left > stages * step ? left - stages * step : 0;
  }

  // Issues chunk c of a stage to LDS byte `at` (this wave's part of the
  // operand's stage); whole: the stage has kBK k left, else `have` of them.
  // In assembly so that the compiler does not wait for the load before the
  // next LDS read, as it must where it sees a write to LDS; it has no result
  // register, and the caller waits for it.  The compiler does not know that
  // this reads scalar registers from the vector memory unit either, which
  // must come five wait states after a vector instruction (v_readfirstlane)
  // wrote them: they are inside the block.
  template <bool WHOLE>
  __device__ __forceinline__ void issue(uint32_t at, int c, uint32_t have) {
    // the base and the LDS address are the same in every lane
    // (the last dword of a matrix of bfloat16 may be half outside it)
    const uint32_t records = ROWS == kChunkRows || left > kOutside - 4 ? kOutside : ((uint32_t)left + 3) & ~3u;
    const u32x4 rs = {uniform_u32((uint32_t)base), uniform_u32((uint32_t)(base >> 32)), uniform_u32(records),
                      (uint32_t)kRsrcWord3};
    const uint32_t o = WHOLE || kk(c) < have ? off[c] : kOutside;
    asm volatile(
        "s_mov_b32 m0, %0\n\t"
        "s_nop 3\n\t"
        "buffer_load_dwordx4 %1, %2, 0 offen lds"
        :
        : "s"(uniform_u32(at + c * 1024)), "v"(o), "s"(rs)
        : "memory");
  }

  // kDwordRows along k: zeros over what this thread's chunks of a stage with
  // `have` k hold past them.  After the thread's loads have arrived.
  __device__ __forceinline__ void clear_tail(char *tile, int have) const {
    if constexpr (KM && ROWS == kDwordRows) {
      const uint32_t chunk0 = threadIdx.x / 64 * kChunks;
#pragma unroll
      for (int c = 0; c < kChunks; ++c) {
        const int from = have - (int)kk(c);
        if (from <= 0 || from >= kEpc) continue;
        T *e = reinterpret_cast<T *>(tile + (chunk0 + c) * 1024 + threadIdx.x % 64 * 16);
        for (int i = from; i < kEpc; ++i) e[i] = (T)0.f;
      }
    }
  }

  // kAnyRows: the stage's chunks to registers; have: k left from the stage's
  // first (may be 0 or less).
  __device__ __forceinline__ void fetch(int have) {
    if constexpr (ROWS == kAnyRows) {
#pragma unroll
      for (int c = 0; c < kChunks; ++c) {
        union {
          T e[kEpc];
          u32x4 raw;
        } v;
        v.raw = u32x4{0, 0, 0, 0};
        if (off[c] != kOutside && (int)kk(c) < have) {
          typedef const __attribute__((address_space(1))) T *global;
          const global p = (global)(base + off[c]);
          if ((uint64_t)off[c] + 16 <= left) {
            __builtin_memcpy(&v, p, 16);
          } else {
#pragma unroll
            for (int i = 0; i < kEpc; ++i)
              if ((uint64_t)off[c] + (i + 1) * sizeof(T) <= left) v.e[i] = p[i];
          }
          if constexpr (KM) {
            if ((int)kk(c) + kEpc > have) {  // the row ends inside the chunk
#pragma unroll
              for (int i = 0; i < kEpc; ++i)
                if ((int)kk(c) + i >= have) v.e[i] = (T)0.f;
            }
          }
        }
        raw[c] = v.raw;
      }
    }
  }
  __device__ __forceinline__ void commit(char *tile) {
    if constexpr (ROWS == kAnyRows) commit(tile, raw);
  }
  __device__ __forceinline__ void commit(char *tile, const u32x4 (&from)[kChunks]) {
    if constexpr (ROWS == kAnyRows) {
      const uint32_t chunk0 = threadIdx.x / 64 * kChunks;
#pragma unroll
      for (int c = 0; c < kChunks; ++c)
        *reinterpret_cast<u32x4 *>(tile + (chunk0 + c) * 1024 + threadIdx.x % 64 * 16) = from[c];
    }
  }
};

// ---------------------------------------------------------------- epilogues
//
// A wave's sums go through LDS, half of its rows at a time, so that each lane
// finishes kEw consecutive columns of a row and rows are written whole lines
// at a time.
constexpr int kEw = 8;
typedef Pack<float, kEw, true> Vals;

// kEw values at p, of which the row has n: 16 bytes at a time at any alignment,
// single ones at the row's end (8-bit 777 x 1001 -> 515, two results of binary32 rows
// of 515: 13.4 us with single ones everywhere, so 11.2).
template <typename T>
__device__ __forceinline__ void put8(T *p, const Vals &v, uint32_t n) {
  constexpr int kEach = 16 / (int)sizeof(T);
  if (n >= kEw) {
#pragma unroll
    for (int i = 0; i < kEw; i += kEach) {
      T r __attribute__((ext_vector_type(kEach)));
#pragma unroll
      for (int j = 0; j < kEach; ++j) r[j] = Num<T>::put(v.v[i + j]);
      __builtin_memcpy(p + i, &r, 16);
    }
  } else {
#pragma unroll
    for (int i = 0; i < kEw; ++i)
      if (i < (int)n) p[i] = Num<T>::put(v.v[i]);
  }
}
template <typename T>
__device__ __forceinline__ Vals get8(const T *p, uint32_t n) {
  constexpr int kEach = 16 / (int)sizeof(T);
  Vals v;
  if (n >= kEw) {
#pragma unroll
    for (int i = 0; i < kEw; i += kEach) {
      T r __attribute__((ext_vector_type(kEach)));
      __builtin_memcpy(&r, p + i, 16);
#pragma unroll
      for (int j = 0; j < kEach; ++j) v.v[i + j] = Num<T>::get(r[j]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < kEw; ++i) v.v[i] = i < (int)n ? Num<T>::get(p[i]) : 0.f;
  }
  return v;
}
// kEw elements as they lie in memory, converted where they are used.
template <typename T>
struct Held {
  typedef T vec __attribute__((ext_vector_type(16 / sizeof(T))));
  vec r[kEw * sizeof(T) / 16];
  __device__ __forceinline__ void load(const T *p) {
#pragma unroll
    for (int i = 0; i < (int)(kEw * sizeof(T) / 16); ++i) r[i] = reinterpret_cast<const vec *>(p)[i];
  }
  __device__ __forceinline__ Vals vals() const {
    Vals v;
#pragma unroll
    for (int i = 0; i < kEw; ++i) v.v[i] = Num<T>::get(r[i * sizeof(T) / 16][i % (16 / sizeof(T))]);
    return v;
  }
};
__device__ __forceinline__ void add8(Vals &v, const Vals &w) {
#pragma unroll
  for (int i = 0; i < kEw; ++i) v.v[i] += w.v[i];
}

// f(z) of all kEw values, f the (ungated or first half's) activation; the
// branch on it is taken once for all of them.
__device__ __forceinline__ void act8(Vals &v, int act) {
  switch (act) {
    case LL_ACT_NONE: break;
    case LL_ACT_RELU:
#pragma unroll
      for (int i = 0; i < kEw; ++i) v.v[i] = act1(v.v[i], LL_ACT_RELU);
      break;
    case LL_ACT_GELU:
    case LL_ACT_GEGLU:
#pragma unroll
      for (int i = 0; i < kEw; ++i) v.v[i] = gelu(v.v[i]);
      break;
    default:
#pragma unroll
      for (int i = 0; i < kEw; ++i) v.v[i] = silu(v.v[i]);
  }
}
__device__ __forceinline__ void slope8(Vals &v, int act) {
  switch (act) {
    case LL_ACT_RELU:
#pragma unroll
      for (int i = 0; i < kEw; ++i) v.v[i] = slope1(v.v[i], LL_ACT_RELU);
      break;
    case LL_ACT_GELU:
    case LL_ACT_GEGLU:
#pragma unroll
      for (int i = 0; i < kEw; ++i) v.v[i] = gelu_slope(v.v[i]);
      break;
    default:
#pragma unroll
      for (int i = 0; i < kEw; ++i) v.v[i] = silu_slope(v.v[i]);
  }
}

// Writes y (and z) for kEw columns n0.. of row r, v the sums; gated: u the
// sums of the second half's columns.
template <typename T, bool GATED>
__device__ __forceinline__ void put_forward(const Args &a, int g, uint64_t r, uint32_t n0, Vals v, Vals u) {
  const uint32_t width = GATED ? a.n / 2 : a.n;
  if (n0 >= width) return;
  const uint32_t left = width - n0;
  if (a.bias != nullptr) {
    const T *b = (const T *)a.bias + (uint64_t)g * a.n + n0;
    add8(v, get8(b, left));
    if constexpr (GATED) add8(u, get8(b + width, left));
  }
  if (a.zout != nullptr) {
    T *z = (T *)a.zout + r * a.ldz + n0;
    put8(z, v, left);
    if constexpr (GATED) put8(z + width, u, left);
  }
  act8(v, a.act);
  if constexpr (GATED) {
#pragma unroll
    for (int i = 0; i < kEw; ++i) v.v[i] *= u.v[i];
  }
  if (a.res != nullptr) add8(v, get8((const T *)a.res + r * a.ldr + n0, left));
  put8((T *)a.c + r * a.ldc + n0, v, left);
}

// The sums v through the activation of the layer below, whose pre-activations
// are z (gated: and u); gated: w <- the second half's.
__device__ __forceinline__ void through_act(const Args &a, Vals &v, const Vals &z, const Vals &u, Vals &w) {
  Vals s = z;
  slope8(s, a.act);
  if (gated(a.act)) {
    w = z;
    act8(w, a.act);
#pragma unroll
    for (int i = 0; i < kEw; ++i) {
      w.v[i] *= v.v[i];
      v.v[i] *= u.v[i];
    }
  }
#pragma unroll
  for (int i = 0; i < kEw; ++i) v.v[i] *= s.v[i];
}

// dx for kEw columns, through the activation of the layer below.
template <typename T>
__device__ __forceinline__ void put_grad_x(const Args &a, uint64_t r, uint32_t n0, Vals v) {
  if (n0 >= a.n) return;
  const uint32_t left = a.n - n0;
  T *out = (T *)a.c + r * a.ldc + n0;
  if (a.act != LL_ACT_NONE) {
    const T *zp = (const T *)a.z + r * a.ldz + n0;
    Vals u, w;
    const Vals z = get8(zp, left);
    if (gated(a.act)) u = get8(zp + a.n, left);
    through_act(a, v, z, u, w);
    if (gated(a.act)) put8(out + a.n, w, left);
  }
  put8(out, v, left);
}

template <typename G>
__device__ __forceinline__ void put_grad_w(const Args &a, int g, uint32_t m, uint32_t n0, Vals v) {
  if (n0 >= a.n) return;
  const uint32_t left = a.n - n0;
  G *out = (G *)a.c + (uint64_t)g * a.cstride + (uint64_t)m * a.ldc + n0;
  if (a.flags & LL_GRAD_ADD) add8(v, get8(out, left));
  put8(out, v, left);
}

template <typename T>
__device__ __forceinline__ void put_bias_grad(const Args &a, int g, uint32_t m, float b) {
  const uint64_t at = (uint64_t)g * a.m + m;
  if (a.flags & LL_GRAD_F32) {
    float *o = (float *)a.dbias + at;
    *o = (a.flags & LL_GRAD_ADD) ? *o + b : b;
  } else {
    T *o = (T *)a.dbias + at;
    *o = Num<T>::put((a.flags & LL_GRAD_ADD) ? Num<T>::get(*o) + b : b);
  }
}

// ---------------------------------------------------------------- the tile kernel
//
// ST stages of both operands lie in LDS.  A wave's rows are FM / 2 fragments
// in the tile's upper half and as many in its lower half, and a stage is four
// clusters of matrix instructions: upper and lower rows with the first half of
// the stage's k, then with the second.  The fragments of a cluster are read
// during the cluster before it, one LDS read between two matrix instructions.
// After the third cluster every fragment of the stage is in registers: a
// barrier there, the only one of a stage, frees its buffer, into which the
// loads of the stage ST further on go out during the fourth cluster, and says
// that the next stage has arrived (its loads went out ST - 1 stages earlier),
// whose first fragments are read meanwhile.  Large tiles have two stages;
// small ones four, since a stage of theirs is shorter than a load takes.
//
// Measured, bfloat16: 8192^3 in 760-840 us, 1310-1450 TFLOP/s, where the
// library's product takes 685-770 us.  The matrix cores are busy 72 % of the
// kernel's cycles (1.05 of 1.46 million a CU), and the chip runs at about 1.8
// GHz meanwhile, so power bounds it as much as anything; LDS reads take 28 %
// of the cycles, with no bank conflicts but the epilogue's.  Grouped, 32 groups
// of 128 to 512 rows, it is bound by reading each group's weight once for two
// or three row tiles (4.8 TB/s at 128 rows a group).
//
// Tiles of 64 have few matrix instructions between one LDS read and the next
// cluster that waits for it (0.5 us a stage with one wave a SIMD): they read
// the whole next stage's fragments at once, for which they have registers.
//
// A tile with no rows in its lower half (the last tile of a group, often)
// leaves that half's work out.
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// This wave's LDS reads and writes are done; then everyone's.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

template <typename T, Pass PASS, int BM, int BN, int WM, int WN, int ST, bool GATED, Rows ROWS>
__global__ __launch_bounds__(WM *WN * 64, ST *(BM + BN) > 640 && WM * WN == 4 ? 1 : 2) void k_tile(Args a) {
  constexpr bool kPkm = PASS != kGradW, kQkm = PASS == kForward;
  constexpr bool VEC = ROWS != kAnyRows;  // loads go straight into LDS
  constexpr bool kFlat = BM == 64;        // all fragments of a stage at once
  static_assert(VEC || ST == 2, "a stage in registers at a time");
  constexpr int NW = WM * WN, WTM = BM / WM, WTN = BN / WN, FM = WTM / 16, FN = WTN / 16, FH = FM / 2;
  constexpr int BK = Step<T>::kBK;
  constexpr int kStage = (BM + BN) * 128;
  constexpr int kPitch = WTN + 4;  // binary32 of an epilogue row: rows start in different banks
  constexpr int kEpi = NW * (WTM / 2) * kPitch * 4;
  constexpr int kLds = ST * kStage > kEpi ? ST * kStage : kEpi;
  typedef typename Step<T>::frag frag;
  __shared__ __attribute__((aligned(1024))) char lds[kLds];
  const int lane = threadIdx.x % 64;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int wm = wave / WN, wn = wave % WN;

  int g = 0;
  uint32_t tn = 0, m0 = 0, m_end = a.m, k = a.k;
  const T *p = (const T *)a.p, *q = (const T *)a.q;
  if constexpr (PASS == kGradW) {
    const uint32_t per = a.tiles_m * a.tiles_n;
    uint32_t tm, lo, hi;
    g = blockIdx.x / per;
    if (!tile_of(blockIdx.x % per, per, a.tiles_m, a.tiles_n, &tm, &tn)) return;
    m0 = tm * BM;
    group_rows(a, g, &lo, &hi);
    lo = uniform_u32(lo);
    k = uniform_u32(hi) - lo;
    p += (uint64_t)lo * a.ldp;
    q += (uint64_t)lo * a.ldq;
  } else {
    if (!find_rows(a, blockIdx.x, BM, &g, &m0, &m_end, &tn)) return;
    q += (uint64_t)g * a.qstride;
  }

  // this workgroup's share of k, whole stages
  const uint32_t share = a.splits == 1 ? k : ((k + BK - 1) / BK + a.splits - 1) / a.splits * BK;
  const uint32_t k_from = min(k, blockIdx.y * share);

  Loader<T, BM, NW, kPkm, ROWS> lp;
  Loader<T, BN, NW, kQkm, ROWS> lq;
  if constexpr (kPkm)
    lp.init(p, a.ldp, k, m_end, 0, m0, [&](uint32_t j, bool *ok) {
      *ok = m0 + j < m_end;
      return m0 + j;
    });
  else
    lp.init(p, a.ldp, k, 0, a.m, m0, [](uint32_t, bool *) { return 0u; });
  if constexpr (kQkm)
    lq.init(q, a.ldq, k, a.n, 0, GATED ? 0 : tn * BN,
            [&](uint32_t j, bool *ok) { return q_row<WTN, GATED>(tn, BN, j, a.n, ok); });
  else
    lq.init(q, a.ldq, k, 0, a.n, tn * BN, [](uint32_t, bool *) { return 0u; });

  if (a.splits > 1) {
    lp.skip(k_from / BK);
    lq.skip(k_from / BK);
    k = min(k - k_from, share);
  }

  f32x4 acc[FN][FM];
#pragma unroll
  for (int i = 0; i < FM; ++i) {
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[j][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  f32x4 accb[kFlat ? FM : 1];  // grad_w: the bias gradient's sums
  frag ones;
#pragma unroll
  for (auto &v : accb) v = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < (int)(sizeof(ones) / sizeof(T)); ++i) ones[i] = (T)1.f;

  const uint32_t steps = (k + BK - 1) / BK;
  constexpr int kLoads = lp.kChunks + lq.kChunks;  // of a thread, a stage
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
  const uint32_t at_p = lds0 + wave * lp.kChunks * 1024, at_q = lds0 + BM * 128 + wave * lq.kChunks * 1024;
  // load n (of kLoads) of the stage that goes to buffer `into`
  auto issue = [&](int into, int n, auto whole, uint32_t have) __attribute__((always_inline)) {
    if (n < lp.kChunks)
      lp.template issue<decltype(whole)::value>(at_p + into * kStage, n, have);
    else
      lq.template issue<decltype(whole)::value>(at_q + into * kStage, n - lp.kChunks, have);
  };
  // first entry of the wave's fragment i of P
  auto dim_p = [&](int i) __attribute__((always_inline)) {
    return (i < FH ? 0 : BM / 2) + wm * (WTM / 2) + (i % FH) * 16;
  };
  // Where the fragments lie in a stage, by half of its k (RM: a constant
  // apart).  Those of P's lower half lie a constant further on where the
  // swizzle does not reach that bit of the entry.
  constexpr bool kSame = kPkm || BM / 2 * sizeof(T) % 256 == 0;
  constexpr int kHalfOff = kPkm ? BM / 2 * 128 : BM / 2 * (int)sizeof(T);
  constexpr int kKsP = Step<T>::kMma * BM * (int)sizeof(T), kKsQ = Step<T>::kMma * BN * (int)sizeof(T);
  uint32_t off_q[2][FN], off_p[2][FM];
#pragma unroll
  for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
    for (int j = 0; j < FN; ++j)
      off_q[ks][j] = kQkm || ks == 0 ? BM * 128 + frag_off<T, BN, kQkm>(wn * WTN + j * 16, ks) : off_q[0][j] + kKsQ;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      if (i >= FH && kSame)
        off_p[ks][i] = off_p[ks][i - FH] + kHalfOff;
      else
        off_p[ks][i] = kPkm || ks == 0 ? frag_off<T, BM, kPkm>(dim_p(i), ks) : off_p[0][i] + kKsP;
    }
  }
  const bool lower = m_end - m0 > BM / 2;  // the tile has rows in its lower half

  if (steps > 0) {
#pragma unroll
    for (int s = 0; s < ST; ++s) {
      const int have = (int)k - s * BK;
      if constexpr (VEC) {
#pragma unroll
        for (int n = 0; n < kLoads; ++n) issue(s, n, std::false_type{}, have > 0 ? have : 0);
      } else {
        lp.fetch(have);
        lq.fetch(have);
        if (s == 0) {  // the second stage is committed during the first
          lp.commit(lds);
          lq.commit(lds + BM * 128);
        }
      }
      lp.advance();
      lq.advance();
    }
    wait_loads<VEC ? (ST - 1) * kLoads : 0>();
    lp.clear_tail(lds, (int)k);
    lq.clear_tail(lds + BM * 128, (int)k);
    lds_barrier();
    if constexpr (kFlat) {
      frag fq[2][2][FN], fp[2][2][FM];  // of two stages, by half of k
      const bool want_bias = PASS == kGradW && a.sum_bias && tn == 0 && wn == 0;
      auto read_all = [&](auto set_c, const char *from) __attribute__((always_inline)) {
        constexpr int set = decltype(set_c)::value;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
          for (int j = 0; j < FN; ++j) fq[set][ks][j] = read_frag<T, BN, kQkm>(from + off_q[ks][j]);
#pragma unroll
          for (int i = 0; i < FM; ++i) fp[set][ks][i] = read_frag<T, BM, kPkm>(from + off_p[ks][i]);
        }
      };
      read_all(std::integral_constant<int, 0>{}, lds);
      // One stage, its fragments in set `now`, from LDS buffer b.
      auto flat = [&](int b, auto now_c, int have, int next_has) __attribute__((always_inline)) {
        constexpr int now = decltype(now_c)::value;
        char *next = lds + (b + 1) % ST * kStage;
        lp.commit(next);
        lq.commit(next + BM * 128);
        wait_loads<VEC ? (ST - 2) * kLoads : 0>();
        if (ROWS == kDwordRows && next_has < BK) {
          lp.clear_tail(next, next_has);
          lq.clear_tail(next + BM * 128, next_has);
        }
        lds_barrier();
        if constexpr (VEC) {
#pragma unroll
          for (int n = 0; n < kLoads; ++n) issue(b, n, std::false_type{}, have > 0 ? have : 0);
        } else {
          lp.fetch(have);
          lq.fetch(have);
        }
        read_all(std::integral_constant<int, 1 - now>{}, next);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
          for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int i = 0; i < FM; ++i) acc[j][i] = mma(fq[now][ks][j], fp[now][ks][i], acc[j][i]);
        if constexpr (PASS == kGradW) {
          if (want_bias) {  // the product with a column of ones
#pragma unroll
            for (int ks = 0; ks < 2; ++ks)
#pragma unroll
              for (int i = 0; i < FM; ++i) accb[i] = mma(ones, fp[now][ks][i], accb[i]);
          }
        }
        lp.advance();
        lq.advance();
      };
      for (uint32_t s = 0;;) {
        flat(s % ST, std::integral_constant<int, 0>{}, (int)k - (int)(s + ST) * BK, (int)k - (int)(s + 1) * BK);
        if (++s >= steps) break;
        flat(s % ST, std::integral_constant<int, 1>{}, (int)k - (int)(s + ST) * BK, (int)k - (int)(s + 1) * BK);
        if (++s >= steps) break;
      }
    } else {
      frag fq[2][FN], fu[2][FH], fl[2][FH];  // by half of k: Q, P's upper rows, P's lower rows
#pragma unroll
      for (int j = 0; j < FN; ++j) fq[0][j] = read_frag<T, BN, kQkm>(lds + off_q[0][j]);
#pragma unroll
      for (int i = 0; i < FH; ++i) fu[0][i] = read_frag<T, BM, kPkm>(lds + off_p[0][i]);

      // The matrix instruction t of a cluster (none past the last).
      auto multiply = [&](int t, int ks, bool low) __attribute__((always_inline)) {
        if (t >= FN * FH) return;
        const int j = t / FH, i = t % FH;
        if (low)
          acc[j][FH + i] = mma(fq[ks][j], fl[ks][i], acc[j][FH + i]);
        else
          acc[j][i] = mma(fq[ks][j], fu[ks][i], acc[j][i]);
      };
      // One stage from LDS buffer b.  WHOLE: the stage loaded meanwhile has BK k,
      // else `have` of them (none: zeros are written).  next_has: k of the next one.
      auto stage = [&](int b, auto lower_c, auto whole, int have, int next_has) __attribute__((always_inline)) {
        constexpr bool kLower = decltype(lower_c)::value;
        constexpr int kMmas = FN * FH, kMmasL = kLower ? kMmas : 0;
        const char *here = lds + b * kStage, *next = lds + (b + 1) % ST * kStage;
#pragma unroll
        for (int t = 0; t < kMmas; ++t) {
          if (kLower && t < FH) fl[0][t < FH ? t : 0] = read_frag<T, BM, kPkm>(here + off_p[0][FH + (t < FH ? t : 0)]);
          multiply(t, 0, false);
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int t = 0; t < FN + FH || t < kMmasL; ++t) {
          if (t < FN)
            fq[1][t < FN ? t : 0] = read_frag<T, BN, kQkm>(here + off_q[1][t < FN ? t : 0]);
          else if (t < FN + FH)
            fu[1][t - FN] = read_frag<T, BM, kPkm>(here + off_p[1][t - FN]);
          if (kLower) multiply(t, 0, true);
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int t = 0; t < kMmas; ++t) {
          if (kLower && t < FH) fl[1][t < FH ? t : 0] = read_frag<T, BM, kPkm>(here + off_p[1][FH + (t < FH ? t : 0)]);
          multiply(t, 1, false);
          __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (!VEC) {
          // the next stage's chunks, fetched a stage ago
          lp.commit(const_cast<char *>(next));
          lq.commit(const_cast<char *>(next) + BM * 128);
        }
        wait_loads<VEC ? (ST - 2) * kLoads : 0>();
        if (ROWS == kDwordRows && next_has < BK) {
          lp.clear_tail(const_cast<char *>(next), next_has);
          lq.clear_tail(const_cast<char *>(next) + BM * 128, next_has);
        }
        lds_barrier();
        if constexpr (!VEC) {
          lp.fetch(have);
          lq.fetch(have);
        }
        constexpr int kReads = FN + FH, kAux = VEC && kLoads > kReads ? kLoads : kReads;
#pragma unroll
        for (int t = 0; t < kAux || t < kMmasL; ++t) {
          if (VEC && t < kLoads) issue(b, t, whole, have > 0 ? have : 0);
          if (t < FN)
            fq[0][t < FN ? t : 0] = read_frag<T, BN, kQkm>(next + off_q[0][t < FN ? t : 0]);
          else if (t < kReads)
            fu[0][t - FN] = read_frag<T, BM, kPkm>(next + off_p[0][t - FN]);
          if (kLower) multiply(t, 1, true);
          __builtin_amdgcn_sched_barrier(0);
        }
        lp.advance();
        lq.advance();
      };
      auto all = [&](auto lower_c) __attribute__((always_inline)) {
        uint32_t s = 0;
        if constexpr (VEC) {  // ST stages at a time: LDS addresses are constants
          for (; (s + 2 * ST) * BK <= k; s += ST) {
            stage(0, lower_c, std::true_type{}, BK, BK);
            stage(1, lower_c, std::true_type{}, BK, BK);
            if constexpr (ST > 2) {
              stage(2, lower_c, std::true_type{}, BK, BK);
              stage(3, lower_c, std::true_type{}, BK, BK);
            }
          }
        }
        for (; s < steps; ++s)
          stage(s % ST, lower_c, std::false_type{}, (int)k - (int)(s + ST) * BK, (int)k - (int)(s + 1) * BK);
      };
      if (PASS == kGradW || lower)
        all(std::true_type{});
      else
        all(std::false_type{});
    }
  }
  wait_loads<0>();
  lds_barrier();  // every wave is past its last stage, and no load is under way

  if constexpr (PASS == kGradW && kFlat) {
    if (a.sum_bias && tn == 0 && wn == 0 && lane < 16) {
#pragma unroll
      for (int i = 0; i < FM; ++i)
        if (m0 + dim_p(i) + lane < m_end) put_bias_grad<T>(a, g, m0 + dim_p(i) + lane, accb[i][0]);
    }
  }
  float *mine = reinterpret_cast<float *>(lds) + wave * (WTM / 2) * kPitch;
  auto finish = [&](auto half) __attribute__((always_inline)) {
    constexpr int h = decltype(half)::value;
#pragma unroll
    for (int i = 0; i < FH; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j)
        *reinterpret_cast<f32x4 *>(mine + (i * 16 + lane % 16) * kPitch + j * 16 + lane / 16 * 4) = acc[j][h * FH + i];
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_wave_barrier();
    constexpr int kWidth = GATED ? WTN / 2 : WTN;  // columns of C a wave has
    constexpr int kLanes = kWidth / kEw;           // lanes a row
    const int c = lane % kLanes * kEw;
    const uint32_t n0 = (GATED ? tn * (BN / 2) + wn * kWidth : tn * BN + wn * WTN) + c;
    constexpr int kRows = 64 / kLanes;  // rows of the wave's half at a time
    if constexpr (PASS == kGradX) {
      // Whole tiles through an activation: the pre-activations of kAhead rows
      // are read before the first of them is used (gradient of 8 experts' 2048
      // -> 7168 through SwiGLU, both gradients: 587 -> 578 us).
      constexpr int kAhead = WTM / 2 / kRows < 4 ? WTM / 2 / kRows : 4;
      if (a.parts == nullptr && a.act != LL_ACT_NONE && a.vec_c && a.n % kEw == 0 && (tn + 1) * BN <= a.n) {
        const uint32_t first = m0 + h * (BM / 2) + wm * (WTM / 2) + lane / kLanes;
#pragma unroll 1
        for (int r = 0; r < WTM / 2; r += kRows * kAhead) {
          Held<T> z[kAhead], u[kAhead];
#pragma unroll
          for (int i = 0; i < kAhead; ++i) {
            const T *zp = (const T *)a.z + (uint64_t)min(first + r + i * kRows, m_end - 1) * a.ldz + n0;
            z[i].load(zp);
            if (gated(a.act)) u[i].load(zp + a.n);
          }
#pragma unroll
          for (int i = 0; i < kAhead; ++i) {
            const uint32_t m = first + r + i * kRows;
            if (m >= m_end) continue;
            Vals v, w;
            Pack<float, kEw, true> sums;
            sums.load(mine + (lane / kLanes + r + i * kRows) * kPitch + c);
#pragma unroll
            for (int e = 0; e < kEw; ++e) v.v[e] = sums.v[e];
            through_act(a, v, z[i].vals(), u[i].vals(), w);
            T *out = (T *)a.c + (uint64_t)m * a.ldc + n0;
            if (gated(a.act)) put8(out + a.n, w, kEw);
            put8(out, v, kEw);
          }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_wave_barrier();
        return;
      }
    }
#pragma unroll 1
    for (int r = lane / kLanes; r < WTM / 2; r += 64 / kLanes) {
      const uint32_t m = m0 + h * (BM / 2) + wm * (WTM / 2) + r;
      if (m >= m_end) break;
      Pack<float, kEw, true> v, u;
      v.load(mine + r * kPitch + c);
      if (a.parts != nullptr) {
        const uint32_t rc = PASS == kGradW ? g * a.m + m : m;
        if (n0 < a.part_half) {
          float *to = a.parts + ((uint64_t)blockIdx.y * a.rows_c + rc) * a.part_row + n0;
          v.store(to);
          if constexpr (GATED) {
            u.load(mine + r * kPitch + kWidth + c);
            u.store(to + a.part_half);
          }
        }
      } else if constexpr (PASS == kForward) {
        if constexpr (GATED) u.load(mine + r * kPitch + kWidth + c);
        put_forward<T, GATED>(a, g, m, n0, v, u);
      } else if constexpr (PASS == kGradX) {
        put_grad_x<T>(a, m, n0, v);
      } else {
        if (a.flags & LL_GRAD_F32)
          put_grad_w<float>(a, g, m, n0, v);
        else
          put_grad_w<T>(a, g, m, n0, v);
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_wave_barrier();
  };
  finish(std::integral_constant<int, 0>{});
  if (PASS == kGradW || lower) finish(std::integral_constant<int, 1>{});
}

// ---------------------------------------------------------------- joining split sums
//
// Adds the splits of each element in order and finishes it as the product
// itself would have.  A lane has kEw columns of a row.  Bound by its launch
// and the chain of loads that finds a row's group before the first part is read
// (777 x 515 of 5 groups, 3 splits: 7.1-7.8 us).
template <typename T, Pass PASS, bool GATED>
__global__ __launch_bounds__(256) void k_join(Args a) {
  const uint32_t width = GATED ? a.n / 2 : a.n, cols = (width + kEw - 1) / kEw;
  const uint64_t id = blockIdx.x * 256ull + threadIdx.x;
  const uint32_t r = (uint32_t)(id / cols), n0 = (uint32_t)(id % cols) * kEw;
  if (r >= a.rows_c) return;
  int g = 0;
  if (PASS == kGradW) {
    g = r / a.m;
  } else if (a.offsets != nullptr) {
    // the last group that starts at or before r and has it
    int lo = 0, hi = a.groups;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (a.offsets[mid] <= (int)r)
        lo = mid;
      else
        hi = mid;
    }
    g = lo;
    if ((int)r < a.offsets[g] || (int)r >= a.offsets[g + 1]) return;
  }
  const uint64_t next = (uint64_t)a.rows_c * a.part_row;
  const float *from = a.parts + (uint64_t)r * a.part_row + n0;
  Vals v, u;
  v.load(from);
  if constexpr (GATED) u.load(from + a.part_half);
#pragma unroll 4
  for (uint32_t z = 1; z < a.splits; ++z) {
    from += next;
    Vals p;
    p.load(from);
    add8(v, p);
    if constexpr (GATED) {
      p.load(from + a.part_half);
      add8(u, p);
    }
  }
  if constexpr (PASS == kForward)
    put_forward<T, GATED>(a, g, r, n0, v, u);
  else if constexpr (PASS == kGradX)
    put_grad_x<T>(a, r, n0, v);
  else if (a.flags & LL_GRAD_F32)
    put_grad_w<float>(a, g, r % a.m, n0, v);
  else
    put_grad_w<T>(a, g, r % a.m, n0, v);
}

// ---------------------------------------------------------------- few rows a group
//
// The forward product of up to 16 * RB rows of a group, bound by reading the
// weight once: a workgroup owns 2 x 16 weight rows (gated: 16 of each half,
// else 32 in a row), its NW waves take 128 bytes of k of each in turn, straight
// from memory into registers, and the waves' sums are joined in LDS in order.
// The rows come from L2, as often as there are workgroups: two fragments of
// weight share one of them.  kAhead steps of loads are under way in each wave,
// in the registers that two workgroups a CU have (157 instead of 113: 16 rows
// over 32 groups 149 -> 158 us).
// 16 rows over 32 groups of 7168 -> 2 x 2048: 116-150 us, 5.0-6.5 TB/s of the
// weights that have rows (the tile kernel: 127); 1 and 16 rows of 7168 -> 8192:
// 21 and 24 us, 5.6 and 4.8 TB/s.
template <typename T, int RB, int NW, bool GATED>
__global__ __launch_bounds__(NW * 64, 4) void k_stream(Args a) {
  constexpr int kAhead = RB == 1 ? 4 : 2, kCols = GATED ? 16 : 32;  // columns of C
  constexpr int kStepK = 128 / (int)sizeof(T);
  constexpr int kPitch = 2 * 16 + 4;
  typedef typename Step<T>::frag frag;
  __shared__ float part[NW][RB * 16][kPitch];
  const int lane = threadIdx.x % 64, i = lane % 16, q = lane / 16;
  const uint32_t wave = uniform_u32(threadIdx.x / 64);
  int g = 0;
  uint32_t tn = 0, m0 = 0, m_end = 0;
  if (!find_rows(a, blockIdx.x, RB * 16, &g, &m0, &m_end, &tn)) return;
  const uint32_t width = GATED ? a.n / 2 : a.n;
  const uint64_t bw = (uint64_t)((const T *)a.q + (uint64_t)g * a.qstride + (uint64_t)(tn * kCols) * a.ldq);
  const uint64_t bx = (uint64_t)((const T *)a.p + (uint64_t)m0 * a.ldp);
  auto rsrc = [](uint64_t b) {
    return make_rsrc((const void *)(((uint64_t)uniform_u32((uint32_t)(b >> 32)) << 32) | uniform_u32((uint32_t)b)),
                     kOutside);
  };
  const rsrc_t rw = rsrc(bw), rx = rsrc(bx);
  uint32_t ow[2], ox[RB];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t row = i + h * (GATED ? width : 16);
    ow[h] = tn * kCols + (GATED ? i : row) < width ? (uint32_t)((uint64_t)row * a.ldq * sizeof(T)) + q * 16 : kOutside;
  }
#pragma unroll
  for (int b = 0; b < RB; ++b)
    ox[b] = m0 + b * 16 + i < m_end ? (uint32_t)((uint64_t)(b * 16 + i) * a.ldp * sizeof(T)) + q * 16 : kOutside;
  f32x4 acc[2][RB];
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int b = 0; b < RB; ++b) acc[h][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  const uint32_t steps = (a.k + kStepK - 1) / kStepK;
  const uint32_t row_bytes = a.k * (uint32_t)sizeof(T);
  union Raw {
    u32x4 u;
    frag f;
  };
  auto load = [](rsrc_t rs, uint32_t off, uint32_t o, bool in) __attribute__((always_inline)) {
    Raw r;
    r.u = __builtin_amdgcn_raw_buffer_load_b128(rs, (int)(in && off != kOutside ? off + o : kOutside), 0, 0);
    return r;
  };
  for (uint32_t s0 = wave; s0 < steps; s0 += NW * kAhead) {
    Raw fw[kAhead][2][2], fx[kAhead][2][RB];
#pragma unroll
    for (int n = 0; n < kAhead; ++n) {
      const uint32_t at = (s0 + n * NW) * 128;  // past the last step: outside
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const uint32_t o = at + c * 64;
        const bool in = o + q * 16 < row_bytes;
#pragma unroll
        for (int h = 0; h < 2; ++h) fw[n][c][h] = load(rw, ow[h], o, in);
#pragma unroll
        for (int b = 0; b < RB; ++b) fx[n][c][b] = load(rx, ox[b], o, in);
      }
    }
    __builtin_amdgcn_sched_barrier(0);  // every load is issued before the first result is used
#pragma unroll
    for (int n = 0; n < kAhead; ++n)
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int b = 0; b < RB; ++b) acc[h][b] = mma(fw[n][c][h].f, fx[n][c][b].f, acc[h][b]);
  }
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int b = 0; b < RB; ++b) *reinterpret_cast<f32x4 *>(&part[wave][b * 16 + i][h * 16 + q * 4]) = acc[h][b];
  __syncthreads();
  constexpr int kLanes = kCols / kEw;
  for (int t = threadIdx.x; t < RB * 16 * kLanes; t += NW * 64) {
    const int r = t / kLanes, c = t % kLanes * kEw;
    const uint32_t m = m0 + r;
    if (m >= m_end) continue;
    Vals v, u;
#pragma unroll
    for (int e = 0; e < kEw; ++e) {
      v.v[e] = part[0][r][c + e];
      if constexpr (GATED) u.v[e] = part[0][r][16 + c + e];
    }
    for (int o = 1; o < NW; ++o)
#pragma unroll
      for (int e = 0; e < kEw; ++e) {
        v.v[e] += part[o][r][c + e];
        if constexpr (GATED) u.v[e] += part[o][r][16 + c + e];
      }
    put_forward<T, GATED>(a, g, m, tn * kCols + c, v, u);
  }
}

// ---------------------------------------------------------------- bias gradient
//
// dbias[g] = the sum of dz over the group's rows.  The 64-wide tile kernel has
// the registers to sum it along.  With larger tiles or split sums it is a
// launch of its own: in the 256-wide kernel the sums sent its loop's addresses
// to memory (765 -> 1860 us for 8192^3).  kBiasChunks
// chunks of columns a workgroup (a cache line), the rows dealt to kBiasLanes
// threads a chunk, eight loads of a thread under way at a time; the threads'
// parts are added in order.
constexpr int kBiasChunks = 8, kBiasLanes = 128;

template <typename T, bool VEC>
__global__ __launch_bounds__(kBiasChunks *kBiasLanes) void k_bias_grad(Args a) {
  constexpr int C = VEC ? Num<T>::kPer16 : 1, kAhead = 8, kCols = kBiasChunks * C;
  __shared__ float part[kBiasLanes][kCols + 1];
  const int g = blockIdx.y, c = threadIdx.x % kBiasChunks, lane = threadIdx.x / kBiasChunks;
  const uint32_t col = (blockIdx.x * kBiasChunks + c) * C;
  uint32_t lo, hi;
  group_rows(a, g, &lo, &hi);
  float sum[C];
#pragma unroll
  for (int i = 0; i < C; ++i) sum[i] = 0.f;
  if (col < a.m) {
    const T *p = (const T *)a.p + col;
    uint32_t r = lo + lane;
    for (; r + kBiasLanes * (kAhead - 1) < hi; r += kBiasLanes * kAhead) {
      Pack<T, C, VEC> v[kAhead];
#pragma unroll
      for (int n = 0; n < kAhead; ++n) v[n].load(p + (uint64_t)(r + kBiasLanes * n) * a.ldp);
#pragma unroll
      for (int n = 0; n < kAhead; ++n)
#pragma unroll
        for (int i = 0; i < C; ++i) sum[i] += v[n].v[i];
    }
#pragma unroll 4
    for (; r < hi; r += kBiasLanes) {
      Pack<T, C, VEC> v;
      v.load(p + (uint64_t)r * a.ldp);
#pragma unroll
      for (int i = 0; i < C; ++i) sum[i] += v.v[i];
    }
  }
#pragma unroll
  for (int i = 0; i < C; ++i) part[lane][c * C + i] = sum[i];
  __syncthreads();
  const uint32_t m = blockIdx.x * kCols + threadIdx.x;
  if (threadIdx.x < kCols && m < a.m) {
    float b = 0.f;
#pragma unroll 8
    for (int r = 0; r < kBiasLanes; ++r) b += part[r][threadIdx.x];
    put_bias_grad<T>(a, g, m, b);
  }
}

// ---------------------------------------------------------------- dz = dy * act'(z)
// Bound by memory: one pass, 16 bytes a lane.  8192 x 4096 bfloat16 through
// GELU 37-39 us (5.1-5.4 TB/s), through SwiGLU 66 us (5.1 TB/s).
struct ActArgs {
  const void *dy, *z;
  void *dz;
  uint64_t lddy, ldz, lddz;
  uint32_t rows, features;
  int act;
};

template <typename T, bool VEC>
__global__ __launch_bounds__(256) void k_act_grad(ActArgs a) {
  constexpr int C = VEC ? Num<T>::kPer16 : 1;
  const uint32_t chunks = a.features / C;
  const uint64_t total = (uint64_t)a.rows * chunks;
  for (uint64_t i = blockIdx.x * 256ull + threadIdx.x; i < total; i += (uint64_t)gridDim.x * 256) {
    const uint64_t r = i / chunks;
    const uint32_t c = (uint32_t)(i % chunks) * C;
    Pack<T, C, VEC> g, z;
    g.load((const T *)a.dy + r * a.lddy + c);
    z.load((const T *)a.z + r * a.ldz + c);
    T *out = (T *)a.dz + r * a.lddz + c;
    if (gated(a.act)) {
      Pack<T, C, VEC> u, w;
      u.load((const T *)a.z + r * a.ldz + a.features + c);
#pragma unroll
      for (int e = 0; e < C; ++e) {
        w.v[e] = g.v[e] * act1(z.v[e], a.act);
        g.v[e] = g.v[e] * u.v[e] * slope1(z.v[e], a.act);
      }
      w.store(out + a.features);
    } else {
#pragma unroll
      for (int e = 0; e < C; ++e) g.v[e] *= slope1(z.v[e], a.act);
    }
    g.store(out);
  }
}

}  // namespace lin
}  // namespace llc
