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
// through LDS in steps of 128 bytes of k (KM) or of BK rows (RM), loaded
// straight from memory into LDS.  The matrix instruction takes Q as its first
// operand, so a lane ends up with four consecutive n of one m: rows of C are
// written 8 or 16 bytes at a time.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

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
  bool vec_c;      // four consecutive elements of every epilogue row are aligned
};

// ---------------------------------------------------------------- activations
__device__ __forceinline__ float gelu(float x) { return 0.5f * x * (1.f + erff(x * 0.70710678118654752f)); }
__device__ __forceinline__ float silu(float x) { return x / (1.f + expf(-x)); }
__device__ __forceinline__ float gelu_slope(float x) {
  return 0.5f * (1.f + erff(x * 0.70710678118654752f)) + x * expf(-0.5f * x * x) * 0.39894228040143268f;
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

// ---------------------------------------------------------------- groups
// Row tile `rt` of the grouped rows: its group, its first row and the end of
// the group's rows.  false: past the last tile.  Every lane of the calling
// wave takes part; the offsets are clamped to the rows there are.
__device__ __forceinline__ bool find_rows(const Args &a, uint32_t rt, uint32_t bm, int *group, uint32_t *row0,
                                          uint32_t *row1) {
  if (a.offsets == nullptr) {
    *group = 0;
    *row0 = rt * bm;
    *row1 = a.rows;
    return *row0 < a.rows;
  }
  const int lane = threadIdx.x % 64;
  uint32_t before = 0;
  for (int g0 = 0; g0 < a.groups; g0 += 64) {
    const int g = g0 + lane;
    uint32_t lo = 0, hi = 0;
    if (g < a.groups) {
      lo = (uint32_t)min(max(a.offsets[g], 0), (int)a.rows);
      hi = (uint32_t)min(max(a.offsets[g + 1], (int)lo), (int)a.rows);
    }
    const uint32_t tiles = (hi - lo + bm - 1) / bm;
    uint32_t incl = tiles;
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t up = __shfl_up(incl, d);
      if (lane >= d) incl += up;
    }
    const uint64_t past = __ballot(before + incl > rt);
    if (past != 0) {
      const int who = __ffsll((unsigned long long)past) - 1;
      const uint32_t first = __shfl(before + incl - tiles, who);
      *group = __builtin_amdgcn_readfirstlane(g0 + who);
      *row0 = __builtin_amdgcn_readfirstlane(__shfl(lo, who) + (rt - first) * bm);
      *row1 = __builtin_amdgcn_readfirstlane(__shfl(hi, who));
      return true;
    }
    before += __shfl(incl, 63);
  }
  return false;
}

// ---------------------------------------------------------------- operand tiles in LDS
//
// A tile holds R entries of m or n by BK of k in R * 128 bytes, as 16-byte
// chunks.  KM: entry r's 8 chunks at r * 128, chunk c at position c ^ (r & 7),
// so the 16 entries a fragment read touches spread over the banks.  RM: k row
// r's chunks at r * R * sizeof(T), chunk c at position c ^ swz(r), which keeps
// pairs (bf16) or fours (binary32) of chunks together, as one fragment reads
// them, and spreads the k rows of a read over the banks.
template <typename T>
struct Step;
template <>
struct Step<__bf16> {
  static constexpr int kBK = 64, kPerMma = 32;
  typedef bf16x8 frag;
};
template <>
struct Step<float> {
  static constexpr int kBK = 32, kPerMma = 16;  // four 16x16x4 instructions
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

typedef __attribute__((address_space(3))) char lds_char;

template <typename T, int R, bool KM>
__device__ __forceinline__ typename Step<T>::frag read_frag(const char *tile, int dim0, int ks) {
  const int lane = threadIdx.x % 64, i = lane % 16, q = lane / 16;
  if constexpr (KM) {
    const int r = dim0 + i, chunk = ks * 4 + q;
    return *reinterpret_cast<const typename Step<T>::frag *>(tile + r * 128 + ((chunk ^ (r & 7)) << 4));
  } else if constexpr (sizeof(T) == 2) {
    // the transposing read: 16 lanes take 4 k rows of 16 columns, and lane i
    // receives column i of the 4 rows
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    union {
      s16x4 half[2];
      bf16x8 all;
    } u;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t krow = ks * 32 + q * 8 + h * 4 + i / 4;
      const uint32_t chunk = dim0 / 8 + (i % 4) / 2;
      const char *at = tile + krow * (R * 2) + ((chunk ^ rm_swz<T, R>(krow)) << 4) + (i % 2) * 8;
      u.half[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)at);
    }
    return u.all;
  } else {
    f32x4 v;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t krow = ks * 16 + q * 4 + j, col = dim0 + i;
      v[j] = *reinterpret_cast<const float *>(tile + krow * (R * 4) + (((col / 4) ^ rm_swz<T, R>(krow)) << 4) +
                                              (col % 4) * 4);
    }
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

// Which row of an operand's matrix entry j of a tile is.  Gated: a wave's
// first half of columns are activations, its second half the same columns of
// the other half of the weight, so both halves of a column end up in one lane.
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

// Loads one operand's tiles.  VEC: 16-byte chunks straight into LDS through a
// buffer resource; a chunk outside the matrix gets an offset outside the
// resource, which reads as zero.  Otherwise single elements through registers.
template <typename T, int R, int NW, bool KM, bool VEC>
struct Loader {
  static constexpr int kEpc = 16 / (int)sizeof(T);
  static constexpr int kChunks = R * 8 / (NW * 64);  // per thread
  static constexpr int kRowChunks = KM ? 8 : R / kEpc;
  const T *base;       // VEC: of the tile's k position, advanced by load()
  uint64_t ld, left;   // left: bytes from base to the end of the matrix
  uint32_t off[kChunks];
  uint32_t kk[kChunks];  // the chunk's first k (KM) or its k row (RM), within a step
  uint32_t row[kChunks]; // !VEC: the chunk's matrix row (KM) or first column (RM)
  uint32_t lim;          // !VEC, RM: columns of the matrix

  // KM: matrix [rows..][k], entry j is row row_of(j).  RM: matrix [k][cols],
  // the tile's first column is col0.
  template <typename F>
  __device__ __forceinline__ void init(const T *mat, uint64_t ld_, uint32_t k, uint32_t mat_rows, uint32_t cols,
                                       uint32_t first, F row_of) {
    ld = ld_;
    lim = cols;
    const uint32_t tid = threadIdx.x;
    if constexpr (KM) {
      base = mat + (uint64_t)first * ld;
      left = mat_rows > first ? ((uint64_t)(mat_rows - 1 - first) * ld + k) * sizeof(T) : 0;
    } else {
      base = mat + first;
      left = k > 0 && cols > first ? ((uint64_t)(k - 1) * ld + cols - first) * sizeof(T) : 0;
    }
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
      const uint32_t pos = (uint32_t)(tid / 64 * kChunks + c) * 64 + tid % 64;
      if constexpr (KM) {
        const uint32_t r = pos / 8, chunk = (pos % 8) ^ (r & 7);
        bool ok;
        const uint32_t mr = row_of(r, &ok);
        kk[c] = chunk * kEpc;
        off[c] = ok ? (uint32_t)((uint64_t)(mr - first) * ld * sizeof(T)) + chunk * 16 : 0xFFFFFFF0u;
        row[c] = ok ? mr : 0xFFFFFFFFu;
      } else {
        const uint32_t krow = pos / kRowChunks, chunk = (pos % kRowChunks) ^ rm_swz<T, R>(krow);
        kk[c] = krow;
        off[c] = first + chunk * kEpc < cols ? (uint32_t)(krow * ld * sizeof(T)) + chunk * 16 : 0xFFFFFFF0u;
        row[c] = first + chunk * kEpc;
      }
    }
  }

  // Issues the loads of the k step that starts at k0 (consecutive steps).
  __device__ __forceinline__ void load(char *tile, uint32_t k0, uint32_t k) {
    const uint32_t lane_chunk0 = threadIdx.x / 64 * kChunks;
    if constexpr (VEC) {
      const uint32_t records = left > 0xFFFFFFF0ull ? 0xFFFFFFF0u : (uint32_t)left;
      const rsrc_t rs = make_rsrc(base, records);
#pragma unroll
      for (int c = 0; c < kChunks; ++c) {
        const uint32_t o = k0 + kk[c] < k ? off[c] : 0xFFFFFFF0u;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            rs, (__attribute__((address_space(3))) void *)(tile + (lane_chunk0 + c) * 1024), 16, (int)o, 0, 0, 0);
      }
      const uint64_t step = KM ? 128 : (uint64_t)Step<T>::kBK * ld * sizeof(T);
      base = reinterpret_cast<const T *>(reinterpret_cast<const char *>(base) + step);
      left = left > step ? left - step : 0;
    } else {
#pragma unroll
      for (int c = 0; c < kChunks; ++c) {
        union {
          T e[kEpc];
          u32x4 raw;
        } v;
        const uint32_t kc = k0 + kk[c];
#pragma unroll
        for (int i = 0; i < kEpc; ++i) {
          bool ok;
          uint64_t at;
          if constexpr (KM) {
            ok = row[c] != 0xFFFFFFFFu && kc + i < k;
            at = (uint64_t)row[c] * ld + kc + i;
          } else {
            ok = kc < k && row[c] + i < lim;
            at = (uint64_t)kc * ld + row[c] + i;
          }
          v.e[i] = ok ? base[at] : (T)0.f;
        }
        *reinterpret_cast<u32x4 *>(tile + (lane_chunk0 + c) * 1024 + threadIdx.x % 64 * 16) = v.raw;
      }
    }
  }
};

// ---------------------------------------------------------------- epilogues
template <typename T>
__device__ __forceinline__ void put4(T *p, f32x4 v, uint32_t n, bool vec) {
  Pack<T, 4, true> o;
#pragma unroll
  for (int i = 0; i < 4; ++i) o.v[i] = v[i];
  if (vec && n >= 4)
    o.store(p);
  else
    o.store_some(p, (int)n);
}
template <typename T>
__device__ __forceinline__ f32x4 get4(const T *p, uint32_t n, bool vec) {
  Pack<T, 4, true> o;
  if (vec && n >= 4)
    o.load(p);
  else
    o.load_some(p, (int)n, 0.f);
  f32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = o.v[i];
  return v;
}

// Writes y (and z) for four columns n0.. of row r, v the sums; gated: u the
// sums of the second half's columns.
template <typename T, bool GATED>
__device__ __forceinline__ void put_forward(const Args &a, int g, uint64_t r, uint32_t n0, f32x4 v, f32x4 u) {
  const uint32_t width = GATED ? a.n / 2 : a.n;
  if (n0 >= width) return;
  const uint32_t left = width - n0;
  if (a.bias != nullptr) {
    const T *b = (const T *)a.bias + (uint64_t)g * a.n + n0;
    v += get4(b, left, false);
    if constexpr (GATED) u += get4(b + width, left, false);
  }
  if (a.zout != nullptr) {
    T *z = (T *)a.zout + r * a.ldz + n0;
    put4(z, v, left, a.vec_c);
    if constexpr (GATED) put4(z + width, u, left, a.vec_c && width % 4 == 0);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = GATED ? act1(v[i], a.act) * u[i] : act1(v[i], a.act);
  if (a.res != nullptr) v += get4((const T *)a.res + r * a.ldr + n0, left, a.vec_c);
  put4((T *)a.c + r * a.ldc + n0, v, left, a.vec_c);
}

// dx for four columns, through the activation of the layer below.
template <typename T>
__device__ __forceinline__ void put_grad_x(const Args &a, uint64_t r, uint32_t n0, f32x4 v) {
  if (n0 >= a.n) return;
  const uint32_t left = a.n - n0;
  T *out = (T *)a.c + r * a.ldc + n0;
  if (a.act == LL_ACT_NONE) {
    put4(out, v, left, a.vec_c);
    return;
  }
  const T *zp = (const T *)a.z + r * a.ldz + n0;
  f32x4 z = get4(zp, left, a.vec_c), w;
  if (gated(a.act)) {
    const bool vec = a.vec_c && a.n % 4 == 0;
    const f32x4 u = get4(zp + a.n, left, vec);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[i] = v[i] * act1(z[i], a.act);
      v[i] = v[i] * u[i] * slope1(z[i], a.act);
    }
    put4(out + a.n, w, left, vec);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] *= slope1(z[i], a.act);
  }
  put4(out, v, left, a.vec_c);
}

template <typename G>
__device__ __forceinline__ void put_grad_w(const Args &a, int g, uint32_t m, uint32_t n0, f32x4 v) {
  if (n0 >= a.n) return;
  const uint32_t left = a.n - n0;
  G *out = (G *)a.c + (uint64_t)g * a.cstride + (uint64_t)m * a.ldc + n0;
  if (a.flags & LL_GRAD_ADD) v += get4(out, left, a.vec_c);
  put4(out, v, left, a.vec_c);
}

// ---------------------------------------------------------------- the tile kernel
template <typename T, Pass PASS, int BM, int BN, int WM, int WN, bool GATED, bool VEC>
__global__ __launch_bounds__(WM *WN * 64) void k_tile(Args a) {
  constexpr bool kPkm = PASS != kGradW, kQkm = PASS == kForward;
  constexpr int NW = WM * WN, WTM = BM / WM, WTN = BN / WN, FM = WTM / 16, FN = WTN / 16;
  constexpr int BK = Step<T>::kBK, KS = BK / Step<T>::kPerMma;
  constexpr int kTile = (BM + BN) * 128;
  __shared__ __attribute__((aligned(1024))) char lds[2 * kTile];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int wm = wave / WN, wn = wave % WN;

  const uint32_t tn = blockIdx.x % a.tiles_n, tm = blockIdx.x / a.tiles_n;
  int g = 0;
  uint32_t m0 = 0, m_end = a.m, k = a.k;
  const T *p = (const T *)a.p, *q = (const T *)a.q;
  if constexpr (PASS == kGradW) {
    g = tm / a.tiles_m;
    m0 = (tm % a.tiles_m) * BM;
    uint32_t lo = 0, hi = a.rows;
    if (a.offsets != nullptr) {
      lo = (uint32_t)min(max(a.offsets[g], 0), (int)a.rows);
      hi = (uint32_t)min(max(a.offsets[g + 1], (int)lo), (int)a.rows);
    }
    k = hi - lo;
    p += (uint64_t)lo * a.ldp;
    q += (uint64_t)lo * a.ldq;
  } else {
    if (!find_rows(a, tm, BM, &g, &m0, &m_end)) return;
    q += (uint64_t)g * a.qstride;
  }

  Loader<T, BM, NW, kPkm, VEC> lp;
  Loader<T, BN, NW, kQkm, VEC> lq;
  if constexpr (kPkm)
    lp.init(VEC ? p : p, a.ldp, k, m_end, 0, VEC ? m0 : 0, [&](uint32_t j, bool *ok) {
      *ok = m0 + j < m_end;
      return m0 + j;
    });
  else
    lp.init(p, a.ldp, k, 0, a.m, VEC ? m0 : 0, [](uint32_t, bool *) { return 0u; });
  if constexpr (kQkm)
    lq.init(q, a.ldq, k, a.n, 0, 0, [&](uint32_t j, bool *ok) { return q_row<WTN, GATED>(tn, BN, j, a.n, ok); });
  else
    lq.init(q, a.ldq, k, 0, a.n, VEC ? tn * BN : 0, [](uint32_t, bool *) { return 0u; });
  if constexpr (!VEC && !kPkm) {
    for (auto &c : lp.row) c += m0;
  }
  if constexpr (!VEC && !kQkm) {
    for (auto &c : lq.row) c += tn * BN;
  }

  f32x4 acc[FN][FM], accb[FM];
#pragma unroll
  for (int i = 0; i < FM; ++i) {
    accb[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[j][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const bool want_bias = PASS == kGradW && a.dbias != nullptr && tn == 0 && wn == 0;
  typename Step<T>::frag ones;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(ones) / sizeof(T)); ++i) ones[i] = (T)1.f;

  const uint32_t steps = (k + BK - 1) / BK;
  if (steps > 0) {
    lp.load(lds, 0, k);
    lq.load(lds + BM * 128, 0, k);
  }
  for (uint32_t s = 0; s < steps; ++s) {
    __syncthreads();  // step s has arrived, and step s-1's reads are done
    const char *tp = lds + (s & 1) * kTile, *tq = tp + BM * 128;
    if (s + 1 < steps) {
      char *next = lds + ((s + 1) & 1) * kTile;
      lp.load(next, (s + 1) * BK, k);
      lq.load(next + BM * 128, (s + 1) * BK, k);
    }
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      typename Step<T>::frag fp[FM], fq[FN];
#pragma unroll
      for (int i = 0; i < FM; ++i) fp[i] = read_frag<T, BM, kPkm>(tp, wm * WTM + i * 16, ks);
#pragma unroll
      for (int j = 0; j < FN; ++j) fq[j] = read_frag<T, BN, kQkm>(tq, wn * WTN + j * 16, ks);
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int i = 0; i < FM; ++i) acc[j][i] = mma(fq[j], fp[i], acc[j][i]);
      if constexpr (PASS == kGradW) {
        if (want_bias) {
#pragma unroll
          for (int i = 0; i < FM; ++i) accb[i] = mma(ones, fp[i], accb[i]);
        }
      }
    }
  }

#pragma unroll
  for (int i = 0; i < FM; ++i) {
    const uint32_t m = m0 + wm * WTM + i * 16 + lane % 16;
    if (m >= m_end) continue;
    if constexpr (PASS == kForward) {
#pragma unroll
      for (int j = 0; j < (GATED ? FN / 2 : FN); ++j) {
        const uint32_t n0 = GATED ? tn * (BN / 2) + wn * (WTN / 2) + j * 16 + lane / 16 * 4
                                  : tn * BN + wn * WTN + j * 16 + lane / 16 * 4;
        put_forward<T, GATED>(a, g, m, n0, acc[j][i], acc[GATED ? FN / 2 + j : j][i]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < FN; ++j) {
        const uint32_t n0 = tn * BN + wn * WTN + j * 16 + lane / 16 * 4;
        if constexpr (PASS == kGradX)
          put_grad_x<T>(a, m, n0, acc[j][i]);
        else if (a.flags & LL_GRAD_F32)
          put_grad_w<float>(a, g, m, n0, acc[j][i]);
        else
          put_grad_w<T>(a, g, m, n0, acc[j][i]);
      }
      if (want_bias && lane < 16) {
        const uint64_t at = (uint64_t)g * a.m + m;
        float b = accb[i][0];
        if (a.flags & LL_GRAD_F32) {
          float *o = (float *)a.dbias + at;
          *o = (a.flags & LL_GRAD_ADD) ? *o + b : b;
        } else {
          T *o = (T *)a.dbias + at;
          *o = Num<T>::put((a.flags & LL_GRAD_ADD) ? Num<T>::get(*o) + b : b);
        }
      }
    }
  }
}

// ---------------------------------------------------------------- dz = dy * act'(z)
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
