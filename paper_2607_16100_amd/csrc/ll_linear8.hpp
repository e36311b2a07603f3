// Grouped products of 8-bit rows and weights (include/llblock.h, ll_linear8).
//
// y[m, n] = sum over blocks b of 128 k of 2^(sx[m, b] + sw[n / 128, b]) times
// the sum over the block of x(m, k) w(n, k).  The matrix instruction takes a
// scale a row of each operand and 32 k, so the scales cost no instruction of
// their own: a block's scale is given to all four of its 32 k.
//
// Tiles, their order, the loads into LDS and the epilogue are those of the
// other products (ll_linear.hpp): a stage of 128 bytes of k is one block.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "ll_linear.hpp"

namespace llc {
namespace lin {

typedef uint8_t e4m3;
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

template <>
struct Step<e4m3> {
  static constexpr int kBK = 128;
};

struct Args8 : Args {
  const uint8_t *xs, *ws;
  uint64_t ldxs, ldws, wsstride;
  uint32_t first_part;  // k_wide8: workgroups from here on run the short last round's parts
};

constexpr int kScaleStages = 4;  // stages of which a row's scales lie in one word

// Which of a stage's 16-byte chunks a lane takes for half ks of its k does not
// matter as long as both operands' lanes agree; the scale is the same for all.
// An entry's chunks lie at chunk ^ (entry / 2 & 7): of 16 lanes that a read
// serves at a time, two entries 8 apart are in different banks then.
__device__ __forceinline__ uint32_t frag8_off(uint32_t dim0, int ks, int half) {
  const uint32_t lane = threadIdx.x % 64, r = dim0 + lane % 32, chunk = ks * 4 + lane / 32 * 2 + half;
  return r * 128 + ((chunk ^ (r / 2 & 7)) << 4);
}

union Frag8 {
  u32x4 half[2];
  i32x8 all;
};

// A lane's 32 codes of each operand, times their scales (low bytes), to the sums.
//
// For bfloat16 results by the 8-bit instruction.  It cuts each of eight
// consecutive k's products off 2^-13 below the largest one's power of two and
// adds the eights in binary32: about 2^-15 of a result of normal values, an
// eightieth of what its rounding to bfloat16 loses.  For binary32 results that
// would be most of the error, so the codes, which have four significant bits,
// become bfloat16 with their scale (which must lie in its range then) and take
// the bfloat16 instructions, whose products and sums are binary32 (777 x 1001 ->
// 515: 2.6e-5 off with the one, 6e-8 with the other).
__device__ __forceinline__ bf16x8 expand(uint32_t lo, uint32_t hi, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
template <typename O>
__device__ __forceinline__ f32x16 mma8(const Frag8 &a, int sa, const Frag8 &b, int sb, f32x16 c) {
  if constexpr (sizeof(O) == 2) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a.all, b.all, c, 0, 0, 0, sa, 0, sb);
  } else {
    const float fa = __int_as_float((sa & 0xFF) << 23), fb = __int_as_float((sb & 0xFF) << 23);
#pragma unroll
    for (int t = 0; t < 4; ++t)
      c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(expand(a.all[2 * t], a.all[2 * t + 1], fa),
                                                  expand(b.all[2 * t], b.all[2 * t + 1], fb), c, 0, 0, 0);
    return c;
  }
}
template <typename O>
__device__ __forceinline__ f32x4 mma8(const Frag8 &a, int sa, const Frag8 &b, int sb, f32x4 c) {
  if constexpr (sizeof(O) == 2) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a.all, b.all, c, 0, 0, 0, sa, 0, sb);
  } else {
    const float fa = __int_as_float((sa & 0xFF) << 23), fb = __int_as_float((sb & 0xFF) << 23);
#pragma unroll
    for (int t = 0; t < 4; ++t)
      c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(expand(a.all[2 * t], a.all[2 * t + 1], fa),
                                                  expand(b.all[2 * t], b.all[2 * t + 1], fb), c, 0, 0, 0);
    return c;
  }
}

// Bytes of LDS the epilogue takes.
constexpr int epilogue8(int bm, int bn) { return 4 * (bm > 64 ? bm / 4 : 32) * (bn / 2 + 4) * 4; }

// As the other products' epilogue: kEw consecutive columns of a row a lane, a
// wave's rows of one half of the tile at a time.  A lane's sums are of one row,
// four consecutive columns at a time.
template <typename O, int BM, int BN, bool GATED, int FM, int FN>
__device__ __forceinline__ void finish_tile8(const Args8 &a, int g, uint32_t tn, uint32_t m0, uint32_t m_end, bool lower,
                                             const f32x16 (&acc)[FN][FM], char *lds) {
  constexpr int WTN = BN / 2, FH = FM > 1 ? FM / 2 : 1, kPitch = WTN + 4, kRowsE = FH * 32;
  const int lane = threadIdx.x % 64;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int wm = wave / 2, wn = wave % 2;
  float *mine = reinterpret_cast<float *>(lds) + wave * kRowsE * kPitch;
  auto finish = [&](auto half) __attribute__((always_inline)) {
    constexpr int h = decltype(half)::value;
#pragma unroll
    for (int i = 0; i < FH; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const f32x16 &v = acc[j][h * FH + i];
          *reinterpret_cast<f32x4 *>(mine + (i * 32 + lane % 32) * kPitch + j * 32 + c * 8 + lane / 32 * 4) =
              f32x4{v[c * 4], v[c * 4 + 1], v[c * 4 + 2], v[c * 4 + 3]};
        }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_wave_barrier();
    constexpr int kWidth = GATED ? WTN / 2 : WTN;  // columns of y a wave has
    constexpr int kLanes = kWidth / kEw;           // lanes a row
    const int c = lane % kLanes * kEw;
    const uint32_t n0 = (GATED ? tn * (BN / 2) + wn * kWidth : tn * BN + wn * WTN) + c;
#pragma unroll 1
    for (int r = lane / kLanes; r < kRowsE; r += 64 / kLanes) {
      const uint32_t m = m0 + (FM > 1 ? h * (BM / 2) + wm * kRowsE : wm * 32) + r;
      if (m >= m_end) break;
      Pack<float, kEw, true> v, u;
      v.load(mine + r * kPitch + c);
      if constexpr (GATED) u.load(mine + r * kPitch + kWidth + c);
      if (a.parts != nullptr) {
        if (n0 < a.part_half) {
          float *to = a.parts + ((uint64_t)blockIdx.y * a.rows_c + m) * a.part_row + n0;
          v.store(to);
          if constexpr (GATED) u.store(to + a.part_half);
        }
      } else {
        put_forward<O, GATED>(a, g, m, n0, v, u);
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_wave_barrier();
  };
  finish(std::integral_constant<int, 0>{});
  if constexpr (FM > 1) {
    if (lower) finish(std::integral_constant<int, 1>{});
  }
}

// ---------------------------------------------------------------- the tile kernel
//
// Four waves of a quarter of the tile each, in fragments of 32 x 32 by the
// matrix instruction of 64 k: it reads half as many registers a product as that
// of 16 x 16, and a quarter needs fewer LDS reads than the halves of eight
// waves.  A stage is two halves of its k; the fragments of one are read while
// the other is multiplied.  In between, when all of a stage is in registers,
// the only barrier of a stage frees its buffer for the loads of the stage ST
// further on and says that the next stage has arrived.
//
// A row's scales come four stages to a word, through LDS like the operands; each
// stage reads its words from there and moves them down to its byte.

// LDS of a tile: its stages and scales, or its epilogue.
constexpr int tile8_lds(int bm, int bn, int st) {
  const int use = st * (bm + bn) * 128 + 2 * (bm + bn) * 4 + 1024, epi = epilogue8(bm, bn);
  return use > epi ? use : epi;
}

// Rows at any address go through registers, two stages ahead of the one that is
// written to LDS, with the same loads in every stage, so that the wait for a
// stage's loads leaves the next one's under way (777 x 1001 -> 515 to binary32, GELU:
// one stage ahead 16.6 us, two 13.3; 8000 x 4001 -> 4001: 573 us, 472-481).  16 bytes of
// a row that is not there come from the tile's first, those that would pass the
// matrix's end from in front of it; end8() puts those of the last stage in place.
template <typename L>
__device__ __forceinline__ void fetch8(const L &l, u32x4 (&to)[L::kChunks]) {
#pragma unroll
  for (int c = 0; c < L::kChunks; ++c) {
    const uint64_t o = l.off[c] != kOutside ? l.off[c] : 0;
    __builtin_memcpy(&to[c], (const __attribute__((address_space(1))) char *)(l.base + (o + 16 > l.left ? l.left - 16 : o)), 16);
  }
}
// The last stage, which has `have` k: bytes to their places, zeros behind the row.
template <typename L>
__device__ __forceinline__ void end8(const L &l, u32x4 (&v)[L::kChunks], int have) {
#pragma unroll
  for (int c = 0; c < L::kChunks; ++c) {
    const uint64_t past = (l.off[c] != kOutside ? l.off[c] : 0) + 16ull;
    const uint32_t by = past > l.left ? (uint32_t)(past - l.left) : 0u;  // (above 15 nothing of it is kept)
    const int n = (int)l.kk(c) < have ? have - (int)l.kk(c) : 0;
    uint64_t lo = (uint64_t)v[c][1] << 32 | v[c][0], hi = (uint64_t)v[c][3] << 32 | v[c][2];
    lo = by & 8 ? hi : lo;
    hi = by & 8 ? 0 : hi;
    const uint32_t bits = by % 8 * 8;
    lo = lo >> bits | hi << 1 << (63 - bits);
    hi >>= bits;
    const uint32_t keep_lo = (uint32_t)min(n, 8) * 8, keep_hi = (uint32_t)min(max(n - 8, 0), 8) * 8;
    lo &= keep_lo == 64 ? ~0ull : (1ull << keep_lo) - 1;
    hi &= keep_hi == 64 ? ~0ull : (1ull << keep_hi) - 1;
    v[c] = u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
  }
}
// An only stage of a matrix of fewer than 16 bytes.
template <typename L>
__device__ __forceinline__ void bytes8(const L &l, u32x4 (&to)[L::kChunks], int have) {
#pragma unroll
  for (int c = 0; c < L::kChunks; ++c) {
    const int n = l.off[c] != kOutside ? min(have - (int)l.kk(c), 16) : 0;
    const auto p = (const __attribute__((address_space(1))) uint8_t *)(l.base + l.off[c]);
    uint64_t lo = 0, hi = 0;
#pragma unroll 1
    for (int i = 0; i < n; ++i) {
      const uint64_t b = (uint64_t)p[i] << i % 8 * 8;
      lo |= i < 8 ? b : 0;
      hi |= i < 8 ? 0 : b;
    }
    to[c] = u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
  }
}

template <typename O, int BM, int BN, int ST, bool GATED, Rows ROWS>
__device__ __forceinline__ void tile8(const Args8 &a, int g, uint32_t tn, uint32_t m0, uint32_t m_end, char *lds) {
  constexpr bool VEC = ROWS != kAnyRows;  // loads go straight into LDS
  static_assert(VEC || ST == 2, "a stage in registers at a time");
  constexpr int NW = 4, WTM = BM / 2, WTN = BN / 2, FM = WTM / 32, FN = WTN / 32;
  constexpr int FH = FM > 1 ? FM / 2 : 1;  // fragments of a wave's rows in the tile's upper half
  constexpr int BK = 128, kStage = (BM + BN) * 128, kScales = (BM + BN) * 4;
  const int lane = threadIdx.x % 64;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int wm = wave / 2, wn = wave % 2;
  uint32_t k = a.k;
  const e4m3 *p = (const e4m3 *)a.p, *q = (const e4m3 *)a.q + (uint64_t)g * a.qstride;

  // this workgroup's share of k: whole words of scales
  constexpr uint32_t kWord = kScaleStages * BK;
  const uint32_t share = a.splits == 1 ? k : ((k + kWord - 1) / kWord + a.splits - 1) / a.splits * kWord;
  const uint32_t k_from = min(k, blockIdx.y * share);

  Loader<e4m3, BM, NW, true, ROWS, 1> lp;
  Loader<e4m3, BN, NW, true, ROWS, 1> lq;
  lp.init(p, a.ldp, k, m_end, 0, m0, [&](uint32_t j, bool *ok) {
    *ok = m0 + j < m_end;
    return m0 + j;
  });
  lq.init(q, a.ldq, k, a.n, 0, GATED ? 0 : tn * BN,
          [&](uint32_t j, bool *ok) { return q_row<WTN, GATED>(tn, BN, j, a.n, ok); });

  // Scales of the tile's rows (first BM) and of its weight rows: segments of 64,
  // dealt to the waves.
  constexpr int kSegs = (BM + BN) / 64, kMine = (kSegs + NW - 1) / NW;
  static_assert(VEC || NW % kSegs == 0, "a wave's only segment, which others have too");
  uint64_t sbase[kMine];
  uint32_t soff[kMine];
#pragma unroll
  for (int c = 0; c < kMine; ++c) {
    const uint32_t seg = VEC ? wave + c * NW : wave % kSegs, e = seg * 64 + lane;
    if (seg * 64 < BM) {
      sbase[c] = (uint64_t)(a.xs + (uint64_t)m0 * a.ldxs);
      soff[c] = m0 + e < m_end ? (uint32_t)(e * a.ldxs) : kOutside;
    } else {
      bool ok = false;
      const uint32_t r = seg < kSegs ? q_row<WTN, GATED>(tn, BN, e - BM, a.n, &ok) : 0u;
      sbase[c] = (uint64_t)(a.ws + (uint64_t)g * a.wsstride);
      soff[c] = ok ? (uint32_t)(r / 128 * a.ldws) : kOutside;
    }
  }
  const bool tiny = !VEC && (m0 * a.ldp + lp.left < 16 || (GATED ? 0 : (uint64_t)tn * BN * a.ldq) + lq.left < 16);
  if (a.splits > 1) {
    lp.skip(k_from / BK);
    lq.skip(k_from / BK);
#pragma unroll
    for (int c = 0; c < kMine; ++c) sbase[c] += k_from / BK;
    k = min(k - k_from, share);
  }

  f32x16 acc[FN][FM];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[j][i][e] = 0.f;

  const uint32_t steps = (k + BK - 1) / BK;
  constexpr int kLoads = lp.kChunks + lq.kChunks;  // of a thread, a stage
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
  const uint32_t at_p = lds0 + wave * lp.kChunks * 1024, at_q = lds0 + BM * 128 + wave * lq.kChunks * 1024;
  char *const scale_lds = lds + ST * kStage;
  auto issue = [&](int into, int n, auto whole, uint32_t have) __attribute__((always_inline)) {
    if (n < lp.kChunks)
      lp.template issue<decltype(whole)::value>(at_p + into * kStage, n, have);
    else
      lq.template issue<decltype(whole)::value>(at_q + into * kStage, n - lp.kChunks, have);
  };
  // The words of scales number `word` of the sum to their buffer (those past the
  // sum are zeros), or, unless `wanted`, zeros to a place nobody reads: a branch
  // here would let matrix instructions sink behind it.  As Loader's issue: in
  // assembly, without a result register, wait states inside.
  auto issue_scales = [&](uint32_t word, bool wanted) __attribute__((always_inline)) {
    const bool in = wanted && word * kScaleStages * BK < k;
#pragma unroll
    for (int c = 0; c < kMine; ++c) {
      const uint32_t seg = wave + c * NW;
      const uint64_t base = sbase[c] + (in ? word * 4 : 0);
      const uint32_t o = in ? soff[c] : kOutside;
      const uint32_t to = wanted && (kSegs % NW == 0 || seg < kSegs) ? (word & 1) * kScales + seg * 256 : 2 * kScales + wave * 256;
      const u32x4 rs = {uniform_u32((uint32_t)base), uniform_u32((uint32_t)(base >> 32)), kOutside, (uint32_t)kRsrcWord3};
      asm volatile(
          "s_mov_b32 m0, %0\n\t"
          "s_nop 3\n\t"
          "buffer_load_dword %1, %2, 0 offen lds"
          :
          : "s"(uniform_u32(lds0 + ST * kStage + to)), "v"(o), "s"(rs)
          : "memory");
    }
  };
  // Rows through registers: a stage's chunks and scales.
  struct Ahead {
    u32x4 p[decltype(lp)::kChunks], q[decltype(lq)::kChunks];
    uint32_t scales;
  };
  auto fetch = [&](Ahead &to, uint32_t s) __attribute__((always_inline)) {  // stage s, the next one, or the last again
    fetch8(lp, to.p);
    fetch8(lq, to.q);
    to.scales = *(const __attribute__((address_space(1))) uint32_t *)(sbase[0] + min(s, steps - 1) / kScaleStages * 4 +
                                                                     (soff[0] != kOutside ? soff[0] : 0));
    if (s + 1 < steps) {
      lp.advance();
      lq.advance();
    }
  };
  auto commit = [&](Ahead &from, uint32_t s, char *to) __attribute__((always_inline)) {
    if (s + 1 == steps) {
      end8(lp, from.p, (int)(k - s * BK));
      end8(lq, from.q, (int)(k - s * BK));
    }
    lp.commit(to, from.p);
    lq.commit(to + BM * 128, from.q);
    *reinterpret_cast<uint32_t *>(scale_lds + (s / kScaleStages & 1) * kScales + (wave % kSegs * 64 + lane) * 4) = from.scales;
  };
  // first entry of the wave's fragment i of the rows
  auto dim_p = [&](int i) __attribute__((always_inline)) {
    return FM > 1 ? (i < FH ? 0 : BM / 2) + wm * (WTM / 2) + (i % FH) * 32 : wm * 32;
  };
  uint32_t off_q[2][2], off_p[2][2];  // of the first fragment, by half of k and by 16 bytes; the others lie constants further
#pragma unroll
  for (int ks = 0; ks < 2; ++ks)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      off_q[ks][h] = BM * 128 + frag8_off(wn * WTN, ks, h);
      off_p[ks][h] = frag8_off(dim_p(0), ks, h);
    }
  auto read_q = [&](const char *from, int j, int ks, int h) __attribute__((always_inline)) {
    return *reinterpret_cast<const u32x4 *>(from + off_q[ks][h] + j * 32 * 128);
  };
  auto read_p = [&](const char *from, int i, int ks, int h) __attribute__((always_inline)) {
    return *reinterpret_cast<const u32x4 *>(from + off_p[ks][h] + (i < FH ? 0 : BM / 2 * 128) + (i % FH) * 32 * 128);
  };
  const bool lower = FM == 1 || m_end - m0 > BM / 2;  // the tile has rows in its lower half

  if (steps > 0) {
    Ahead ahead[2];  // !VEC: the two stages behind the next, by the lowest bit of the one that commits them
    if constexpr (VEC) {
      issue_scales(0, true);
#pragma unroll
      for (int s = 0; s < ST; ++s) {
        const int have = (int)k - s * BK;
#pragma unroll
        for (int n = 0; n < kLoads; ++n) issue(s, n, std::false_type{}, have > 0 ? have : 0);
        lp.advance();
        lq.advance();
      }
      wait_loads<(ST - 1) * kLoads>();
      lp.clear_tail(lds, (int)k);
      lq.clear_tail(lds + BM * 128, (int)k);
    } else {
      Ahead first;
      if (tiny) {
        bytes8(lp, first.p, (int)k);
        bytes8(lq, first.q, (int)k);
        first.scales = *(const __attribute__((address_space(1))) uint32_t *)(sbase[0] + (soff[0] != kOutside ? soff[0] : 0));
        asm volatile("" : "+v"(first.scales));  // (waited for here, not where the other branch's loads would be too)
        lp.left = lq.left = kOutside;           // nothing to move
        ahead[0] = ahead[1] = first;
      } else {
        fetch(first, 0);
        fetch(ahead[0], 1);
        fetch(ahead[1], 2);
      }
      commit(first, 0, lds);
    }
    lds_barrier();

    Frag8 fq[2][FN], fp[2][FM];  // by half of k
    int sq[FN], sp[FM];          // scales, in the low byte
    auto read_scales = [&](uint32_t s, int *sq, int *sp) __attribute__((always_inline)) {  // of stage s
      const uint32_t *from = reinterpret_cast<const uint32_t *>(scale_lds + (s / kScaleStages & 1) * kScales);
      const uint32_t down = s % kScaleStages * 8;
#pragma unroll
      for (int j = 0; j < FN; ++j) sq[j] = (int)(from[BM + wn * WTN + j * 32 + lane % 32] >> down);
#pragma unroll
      for (int i = 0; i < FM; ++i) sp[i] = (int)(from[dim_p(i) + lane % 32] >> down);
    };
    read_scales(0, sq, sp);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int j = 0; j < FN; ++j) fq[0][j].half[h] = read_q(lds, j, 0, h);
#pragma unroll
      for (int i = 0; i < FM; ++i) fp[0][i].half[h] = read_p(lds, i, 0, h);
    }

    // One stage, number s, from LDS buffer b.  `whole`: the stage loaded meanwhile
    // has BK k, else `have` of them (none: zeros are written).  next_has: k of the
    // next one.  !VEC: stage s + 3 is fetched meanwhile if `whole`.
    auto stage = [&](int b, uint32_t s, auto lower_c, auto whole, int have, int next_has) __attribute__((always_inline)) {
      constexpr int kRowsF = decltype(lower_c)::value ? FM : FH;  // fragments of rows that have rows
      constexpr int kMmas = FN * kRowsF, kReads = 2 * (FN + kRowsF);
      const char *here = lds + b * kStage, *next = lds + (b + 1) % ST * kStage;
      auto read = [&](const char *from, int n, int ks) __attribute__((always_inline)) {
        const int f = n / 2, h = n % 2;
        if (f < FN)
          fq[ks][f < FN ? f : 0].half[h] = read_q(from, f, ks, h);
        else
          fp[ks][f - FN].half[h] = read_p(from, f - FN, ks, h);
      };
      auto multiply = [&](int t, int ks) __attribute__((always_inline)) {
        const int j = t / kRowsF, i = t % kRowsF;
        acc[j][i] = mma8<O>(fq[ks][j], sq[j], fp[ks][i], sp[i], acc[j][i]);
      };
#pragma unroll
      for (int t = 0; t < kMmas; ++t) {
#pragma unroll
        for (int n = t * kReads / kMmas; n < (t + 1) * kReads / kMmas; ++n) read(here, n, 1);
        multiply(t, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (VEC)
        wait_loads<(ST - 2) * kLoads>();
      // The next stage's chunks, fetched two stages ago.  Behind the last stage the slot
      // holds an older one, whose word of scales may be the other of two words and would
      // go over the one that late waves still read for this stage.
      else if (decltype(whole)::value || s + 1 < steps)
        commit(ahead[b], s + 1, const_cast<char *>(next));
      if (ROWS == kDwordRows && next_has < BK) {
        lp.clear_tail(const_cast<char *>(next), next_has);
        lq.clear_tail(const_cast<char *>(next) + BM * 128, next_has);
      }
      lds_barrier();
      if constexpr (VEC)
        issue_scales(s / kScaleStages + 1, s % kScaleStages == 1);
      else if constexpr (decltype(whole)::value)
        fetch(ahead[b], s + 3);
      int nq[FN], np[FM];
      read_scales(s + 1, nq, np);
#pragma unroll
      for (int t = 0; t < kMmas; ++t) {
        if constexpr (VEC) {
#pragma unroll
          for (int n = t * kLoads / kMmas; n < (t + 1) * kLoads / kMmas; ++n) issue(b, n, whole, have > 0 ? have : 0);
        }
#pragma unroll
        for (int n = t * kReads / kMmas; n < (t + 1) * kReads / kMmas; ++n) read(next, n, 0);
        multiply(t, 1);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int j = 0; j < FN; ++j) sq[j] = nq[j];
#pragma unroll
      for (int i = 0; i < FM; ++i) sp[i] = np[i];
      if constexpr (VEC) {
        lp.advance();
        lq.advance();
      }
    };
    auto all = [&](auto lower_c) __attribute__((always_inline)) {
      uint32_t s = 0;
      if constexpr (VEC) {  // ST stages at a time: LDS addresses are constants
        for (; (s + 2 * ST) * BK <= k; s += ST) {
          stage(0, s, lower_c, std::true_type{}, BK, BK);
          stage(1, s + 1, lower_c, std::true_type{}, BK, BK);
          if constexpr (ST > 2) {
            stage(2, s + 2, lower_c, std::true_type{}, BK, BK);
            stage(3, s + 3, lower_c, std::true_type{}, BK, BK);
          }
        }
      }
      if constexpr (VEC) {
        for (; s < steps; ++s)
          stage(s % ST, s, lower_c, std::false_type{}, (int)k - (int)(s + ST) * BK, (int)k - (int)(s + 1) * BK);
      } else {
        for (; s + 4 < steps; s += 2) {
          stage(0, s, lower_c, std::true_type{}, 0, 0);
          stage(1, s + 1, lower_c, std::true_type{}, 0, 0);
        }
        if (s + 3 < steps) {
          stage(0, s, lower_c, std::true_type{}, 0, 0);
          stage(1, s + 1, lower_c, std::false_type{}, 0, 0);
          s += 2;
        }
        for (; s < steps; s += 2) {
          stage(0, s, lower_c, std::false_type{}, 0, 0);
          if (s + 1 < steps) stage(1, s + 1, lower_c, std::false_type{}, 0, 0);
        }
      }
    };
    if (FM == 1 || lower)
      all(std::true_type{});
    else
      all(std::false_type{});
  }
  wait_loads<0>();
  lds_barrier();  // every wave is past its last stage, and no load is under way

  finish_tile8<O, BM, BN, GATED>(a, g, tn, m0, m_end, lower, acc, lds);
}

template <typename O, int BM, int BN, int ST, bool GATED, Rows ROWS>
__global__ __launch_bounds__(256, ST *(BM + BN) > 640 ? 1 : ROWS == kAnyRows && sizeof(O) == 4 ? 3 : 2) void k_tile8(Args8 a) {
  __shared__ __attribute__((aligned(1024))) char lds[tile8_lds(BM, BN, ST)];
  int g = 0;
  uint32_t tn = 0, m0 = 0, m_end = a.m;
  if (!find_rows(a, blockIdx.x, BM, &g, &m0, &m_end, &tn)) return;
  tile8<O, BM, BN, ST, GATED, ROWS>(a, g, tn, m0, m_end, lds);
}

// The short last round of 256-wide tiles that their launch leaves out (tail_tiles):
// each tile in eighths of 128 x 64, quarters of 128 x 128 or halves of 128 x 256,
// the smallest that are no more than the CUs (32 tiles of 7168 k: eighths 31 us,
// quarters 39; 96 after a whole round: quarters 172, halves 163; 128: 183, 173,
// and as whole tiles 184).
constexpr uint32_t kEighths = 32, kQuarters = 64;

// Part `id`: as find_rows, and *cols, the columns of parts a tile has.
__device__ __forceinline__ bool find_part(const Args &a, uint32_t id, int *group, uint32_t *row0, uint32_t *row1,
                                          uint32_t *tn, uint32_t *cols) {
  constexpr uint32_t bm = 256;
  uint32_t lo, hi, tiles, incl = 0, rows = 0, tm;
  if (a.offsets == nullptr) {
    rows = (a.rows + bm - 1) / bm;
  } else {
    for (int g0 = 0; g0 < a.groups; g0 += 64) {
      incl = scan_tiles(a, g0, bm, &lo, &hi, &tiles);
      rows += (uint32_t)__builtin_amdgcn_readlane((int)incl, 63);
    }
  }
  const uint32_t total = rows * a.tiles_n, rest = tail_tiles(total);
  *cols = rest <= kEighths ? 4 : rest <= kQuarters ? 2 : 1;
  if (id >= 2 * *cols * rest) return false;
  const uint32_t part = id / rest;
  number_of(total - rest + id % rest, rows, a.tiles_n, &tm, tn);
  *tn = *tn * *cols + part % *cols;
  auto place = [&](int g, uint32_t first, uint32_t end) {
    *group = g;
    *row0 = first + part / *cols * (bm / 2);
    *row1 = end;
    return *row0 < *row1;
  };
  if (a.offsets == nullptr) return place(0, tm * bm, a.rows);
  uint32_t before = 0;
  for (int g0 = 0; g0 < a.groups; g0 += 64) {
    if (a.groups > 64) incl = scan_tiles(a, g0, bm, &lo, &hi, &tiles);
    const uint64_t past = __ballot(before + incl > tm);
    if (past != 0) {
      const int who = __ffsll((unsigned long long)past) - 1;
      const uint32_t skip = before + __builtin_amdgcn_readlane((int)(incl - tiles), who);
      return place(g0 + who, __builtin_amdgcn_readlane((int)lo, who) + (tm - skip) * bm,
                   __builtin_amdgcn_readlane((int)hi, who));
    }
    before += (uint32_t)__builtin_amdgcn_readlane((int)incl, 63);
  }
  return false;
}

template <typename O, bool GATED, Rows ROWS>
__device__ __forceinline__ void part8(const Args8 &a, uint32_t id, char *lds) {
  int g = 0;
  uint32_t tn = 0, m0 = 0, m_end = 0, cols = 0;
  if (!find_part(a, id, &g, &m0, &m_end, &tn, &cols)) return;
  if (cols == 4)
    tile8<O, 128, 64, 4, GATED, ROWS>(a, g, tn, m0, m_end, lds);
  else if (cols == 2)
    tile8<O, 128, 128, 4, GATED, ROWS>(a, g, tn, m0, m_end, lds);
  else
    tile8<O, 128, 256, 2, GATED, ROWS>(a, g, tn, m0, m_end, lds);
}

template <typename O, bool GATED, Rows ROWS>
__global__ __launch_bounds__(256, 1) void k_tail8(Args8 a) {
  __shared__ __attribute__((aligned(1024))) char lds[tile8_lds(128, 128, 4)];
  part8<O, GATED, ROWS>(a, blockIdx.x, lds);
}

// ---------------------------------------------------------------- the wide tile kernel
//
// Tiles of 256 x 256, the only ones with enough matrix instructions a stage to
// hide what a stage loads: 64 KB, for which the vector cache needs half of the
// stage's time.  In k_tile8's schedule those loads all go out in half of the stage, which
// makes the waves wait for the cache (dense 8192^3: 450 us, the matrix cores busy
// 61 % of the cycles).  Here a stage has four clusters of eight matrix
// instructions, one pair of quarters each, and everything is spread over them
// evenly:
//
//   cluster      U x Qf     U x Qs   |   L x Qs     L x Qf
//   reads        Qs         L        |   U of s+1   Qf of s+1
//   loads s+2    U          Qf       |   Qs         L
//
// U and L are the tile's upper and lower 128 rows, Q0 and Q1 the first and second
// half of each wave's columns; Qf is Q0 in even stages and Q1 in odd ones, so
// that the registers of one are free when the next stage's are read.  There is a
// barrier before the first cluster and one in the middle.  What a cluster loads
// was read by every wave before the barrier in front of it, and is waited for a
// stage or more later.  8192^3: 417-428 us, 2570-2640 TFLOP/s, the matrix cores
// busy 70 % of the cycles at 1.7 GHz; 16384 rows over 32 groups, 7168 -> 2 x 2048:
// 481-515 us.
//
// The short last round's parts are the last workgroups of the same launch and
// start where whole tiles, some of which have no lower half, leave a CU first.
// Rows are whole 16-byte chunks; others run k_tile8, and k_tail8 after it.
struct QuarterLoader {
  uint64_t base;  // of the stage to load next
  uint32_t off[8], kk0;

  // Which eight entries chunk c of this wave is: 0 .. 3 of the first quarter, 4 ..
  // 7 of the second.  `apart`: a quarter is the halves' halves (the weight).
  static __device__ __forceinline__ uint32_t block(uint32_t wave, int c, bool apart) {
    const uint32_t i = wave * 4 + c % 4;
    return apart ? i / 8 * 16 + i % 8 + c / 4 * 8 : i + c / 4 * 16;
  }
  template <typename F>
  __device__ __forceinline__ void init(const e4m3 *mat, uint64_t ld, uint32_t first, uint32_t wave, bool apart, F row_of) {
    const uint32_t lane = threadIdx.x % 64;
    base = (uint64_t)(mat + (uint64_t)first * ld);
    kk0 = ((lane % 8) ^ (lane / 16)) * 16;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      bool ok;
      const uint32_t r = row_of(block(wave, c, apart) * 8 + lane / 8, &ok);
      off[c] = ok ? (uint32_t)((uint64_t)(r - first) * ld) + kk(c) : kOutside;
    }
  }
  // chunk c's first k within a stage
  __device__ __forceinline__ uint32_t kk(int c) const { return kk0 ^ (c % 2 * 64); }
  __device__ __forceinline__ void advance() { base += 128; }
  // As Loader's issue, to LDS byte `at`.
  template <bool WHOLE>
  __device__ __forceinline__ void issue(uint32_t at, int c, uint32_t have) {
    const u32x4 rs = {uniform_u32((uint32_t)base), uniform_u32((uint32_t)(base >> 32)), kOutside, (uint32_t)kRsrcWord3};
    const uint32_t o = WHOLE || kk(c) < have ? off[c] : kOutside;
    asm volatile(
        "s_mov_b32 m0, %0\n\t"
        "s_nop 3\n\t"
        "buffer_load_dwordx4 %1, %2, 0 offen lds"
        :
        : "s"(uniform_u32(at)), "v"(o), "s"(rs)
        : "memory");
  }
};

template <typename O, bool GATED>
__global__ __launch_bounds__(256, 1) void k_wide8(Args8 a) {
  constexpr int BM = 256, BN = 256, WTN = 128, BK = 128, kStage = 65536, kScales = 2048;
  static_assert(tile8_lds(BM, BN, 2) >= tile8_lds(128, 128, 4), "the parts' LDS");
  __shared__ __attribute__((aligned(1024))) char lds[tile8_lds(BM, BN, 2)];
  if (blockIdx.x >= a.first_part) {
    part8<O, GATED, kChunkRows>(a, blockIdx.x - a.first_part, lds);
    return;
  }
  const int lane = threadIdx.x % 64;
  const uint32_t wave = uniform_u32(threadIdx.x / 64);
  const uint32_t wm = wave / 2, wn = wave % 2;

  int g = 0;
  uint32_t tn = 0, m0 = 0, m_end = a.m;
  const uint32_t k = a.k;
  if (!find_rows(a, blockIdx.x, BM, &g, &m0, &m_end, &tn)) return;
  QuarterLoader lp, lq;
  lp.init((const e4m3 *)a.p, a.ldp, m0, wave, false, [&](uint32_t j, bool *ok) {
    *ok = m0 + j < m_end;
    return m0 + j;
  });
  lq.init((const e4m3 *)a.q + (uint64_t)g * a.qstride, a.ldq, GATED ? 0 : tn * BN, wave, true,
          [&](uint32_t j, bool *ok) { return q_row<WTN, GATED>(tn, BN, j, a.n, ok); });
  // scales of the tile's rows, then of its weight rows: two segments of 64 each wave
  uint64_t sbase[2];
  uint32_t soff[2];
  {
    const uint32_t e = wave * 64 + lane;
    bool ok;
    const uint32_t r = q_row<WTN, GATED>(tn, BN, e, a.n, &ok);
    sbase[0] = (uint64_t)(a.xs + (uint64_t)m0 * a.ldxs);
    soff[0] = m0 + e < m_end ? (uint32_t)(e * a.ldxs) : kOutside;
    sbase[1] = (uint64_t)(a.ws + (uint64_t)g * a.wsstride);
    soff[1] = ok ? (uint32_t)(r / 128 * a.ldws) : kOutside;
  }

  f32x16 acc[4][4];
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[j][i][e] = 0.f;

  const uint32_t steps = (k + BK - 1) / BK;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
  char *const scale_lds = lds + 2 * kStage;
  auto issue_p = [&](int b, int c, auto whole, uint32_t have) __attribute__((always_inline)) {
    lp.template issue<decltype(whole)::value>(lds0 + b * kStage + lp.block(wave, c, false) * 1024, c, have);
  };
  auto issue_q = [&](int b, int c, auto whole, uint32_t have) __attribute__((always_inline)) {
    lq.template issue<decltype(whole)::value>(lds0 + b * kStage + BM * 128 + lq.block(wave, c, true) * 1024, c, have);
  };
  // as k_tile8's
  auto issue_scales = [&](uint32_t word, bool wanted) __attribute__((always_inline)) {
    const bool in = wanted && word * kScaleStages * BK < k;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const uint64_t base = sbase[c] + (in ? word * 4 : 0);
      const uint32_t o = in ? soff[c] : kOutside;
      const uint32_t to = wanted ? (word & 1) * kScales + (c * 4 + wave) * 256 : 2 * kScales + wave * 256;
      const u32x4 rs = {uniform_u32((uint32_t)base), uniform_u32((uint32_t)(base >> 32)), kOutside, (uint32_t)kRsrcWord3};
      asm volatile(
          "s_mov_b32 m0, %0\n\t"
          "s_nop 3\n\t"
          "buffer_load_dword %1, %2, 0 offen lds"
          :
          : "s"(uniform_u32(lds0 + 2 * kStage + to)), "v"(o), "s"(rs)
          : "memory");
    }
  };
  uint32_t off_q[2][2], off_p[2][2];  // by half of k and by 16 bytes
#pragma unroll
  for (int ks = 0; ks < 2; ++ks)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t chunk = ks * 4 + lane / 32 * 2 + h, at = lane % 32 * 128 + ((chunk ^ (lane % 32 / 2 & 7)) << 4);
      off_p[ks][h] = wm * 64 * 128 + at;
      off_q[ks][h] = BM * 128 + wn * 128 * 128 + at;
    }
  const bool lower = m_end - m0 > BM / 2;  // the tile has rows in its lower half

  if (steps > 0) {
    issue_scales(0, true);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int left_k = (int)k - s * BK;
      const uint32_t have = left_k > 0 ? left_k : 0;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
#pragma unroll
        for (int c = 0; c < 4; ++c) issue_p(s, half * 4 + c, std::false_type{}, have);
#pragma unroll
        for (int c = 0; c < 4; ++c) issue_q(s, (half ^ s) * 4 + c, std::false_type{}, have);
      }
      lp.advance();
      lq.advance();
    }
    wait_loads<16>();
    lds_barrier();

    Frag8 fq[2][2][2], fu[2][2], fl[2][2];  // halves of the columns; then fragment, half of k
    int sq[4], sp[4];                       // scales, in the low byte
    auto read_scales = [&](uint32_t s, int *sq, int *sp) __attribute__((always_inline)) {  // of stage s
      const uint32_t *from = reinterpret_cast<const uint32_t *>(scale_lds + (s / kScaleStages & 1) * kScales);
      const uint32_t down = s % kScaleStages * 8;
#pragma unroll
      for (int j = 0; j < 4; ++j) sq[j] = (int)(from[BM + wn * WTN + j * 32 + lane % 32] >> down);
#pragma unroll
      for (int i = 0; i < 4; ++i) sp[i] = (int)(from[i / 2 * 128 + wm * 64 + i % 2 * 32 + lane % 32] >> down);
    };
    // read n (of 8) of a quarter's fragments
    auto read_q = [&](const char *from, int half, int n) __attribute__((always_inline)) {
      const int ks = n / 4, f = n / 2 % 2, h = n % 2;
      fq[half][f][ks].half[h] = *reinterpret_cast<const u32x4 *>(from + off_q[ks][h] + (half * 2 + f) * 32 * 128);
    };
    auto read_p = [&](const char *from, int low, int n) __attribute__((always_inline)) {
      const int ks = n / 4, f = n / 2 % 2, h = n % 2;
      (low ? fl : fu)[f][ks].half[h] = *reinterpret_cast<const u32x4 *>(from + off_p[ks][h] + low * 128 * 128 + f * 32 * 128);
    };
    read_scales(0, sq, sp);
#pragma unroll
    for (int n = 0; n < 8; ++n) {
      read_p(lds, 0, n);
      read_q(lds, 0, n);
    }
    // matrix instruction t (of 8) of a cluster
    auto multiply = [&](int half, int low, int t) __attribute__((always_inline)) {
      const int ks = t / 4, j = t / 2 % 2, i = t % 2;
      acc[half * 2 + j][low * 2 + i] =
          mma8<O>(fq[half][j][ks], sq[half * 2 + j], (low ? fl : fu)[i][ks], sp[low * 2 + i], acc[half * 2 + j][low * 2 + i]);
    };
    // Stage s in buffer B (s % 2).  `whole`: the stage loaded meanwhile has BK k,
    // else `have_k` of them.  next_has: k of the next one.
    auto stage = [&](auto b_c, uint32_t s, auto lower_c, auto whole, int next_has, int have_k) __attribute__((always_inline)) {
      constexpr int B = decltype(b_c)::value, F = B, S = 1 - B;
      constexpr bool kLower = decltype(lower_c)::value;
      const char *here = lds + B * kStage, *next = lds + (1 - B) * kStage;
      const uint32_t have = have_k > 0 ? have_k : 0;
      wait_loads<16>();
      lds_barrier();
      issue_scales(s / kScaleStages + 1, s % kScaleStages == 1);
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        if (t % 2 == 0) issue_p(B, t / 2, whole, have);
        read_q(here, S, t);
        multiply(F, 0, t);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        if (t % 2 == 0) issue_q(B, F * 4 + t / 2, whole, have);
        if (kLower) read_p(here, 1, t);
        multiply(S, 0, t);
        __builtin_amdgcn_sched_barrier(0);
      }
      wait_loads<16>();
      lds_barrier();
      int nq[4], np[4];
      read_scales(s + 1, nq, np);
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        if (t % 2 == 0) issue_q(B, S * 4 + t / 2, whole, have);
        read_p(next, 0, t);
        if (kLower) multiply(S, 1, t);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        if (t % 2 == 0) issue_p(B, 4 + t / 2, whole, have);
        read_q(next, S, t);
        if (kLower) multiply(F, 1, t);
        __builtin_amdgcn_sched_barrier(0);
      }
      // a stage past the sum is zeros times what may be no number
      const bool none = !decltype(whole)::value && next_has <= 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) sq[j] = none ? 0 : nq[j];
#pragma unroll
      for (int i = 0; i < 4; ++i) sp[i] = none ? 0 : np[i];
      lp.advance();
      lq.advance();
    };
    auto all = [&](auto lower_c) __attribute__((always_inline)) {
      constexpr auto c0 = std::integral_constant<int, 0>{};
      constexpr auto c1 = std::integral_constant<int, 1>{};
      uint32_t s = 0;
      for (; (s + 4) * BK <= k; s += 2) {
        stage(c0, s, lower_c, std::true_type{}, BK, BK);
        stage(c1, s + 1, lower_c, std::true_type{}, BK, BK);
      }
      // an even number of stages, the last of zeros where there is none
      for (; s < steps; s += 2) {
        const int has = (int)(k - s * BK);
        stage(c0, s, lower_c, std::false_type{}, has - BK, has - 2 * BK);
        stage(c1, s + 1, lower_c, std::false_type{}, has - 2 * BK, has - 3 * BK);
      }
    };
    if (lower)
      all(std::true_type{});
    else
      all(std::false_type{});
  }
  wait_loads<0>();
  lds_barrier();  // every wave is past its last stage, and no load is under way
  finish_tile8<O, BM, BN, GATED>(a, g, tn, m0, m_end, lower, acc, lds);
}

// ---------------------------------------------------------------- few rows a group
//
// Up to 16 * RB rows of a group, bound by reading the weight once, as k_stream (16
// rows over 32 groups of 7168 -> 2 x 2048: 60-68 us, 5.9-6.2 TB/s of the weights
// that have rows): a workgroup owns 2 x 16 weight rows (gated: 16 of each half),
// each of its waves an equal run of the blocks of k, kAhead blocks' loads under way
// at a time.
// A lane has one weight row's (and one row's) scales of those blocks in a
// word, cut from the two words they lie in.
template <typename O, int RB, int NW, bool GATED>
__global__ __launch_bounds__(NW * 64, 4) void k_stream8(Args8 a) {
  constexpr int kAhead = RB == 1 ? 4 : 2, kCols = GATED ? 16 : 32;  // columns of y
  constexpr int kPitch = 2 * 16 + 4;
  __shared__ float part[NW][RB * 16][kPitch];
  const int lane = threadIdx.x % 64, i = lane % 16, q = lane / 16;
  const uint32_t wave = uniform_u32(threadIdx.x / 64);
  int g = 0;
  uint32_t tn = 0, m0 = 0, m_end = 0;
  if (!find_rows(a, blockIdx.x, RB * 16, &g, &m0, &m_end, &tn)) return;
  const uint32_t width = GATED ? a.n / 2 : a.n;
  auto rsrc = [](uint64_t b) {
    return make_rsrc((const void *)(((uint64_t)uniform_u32((uint32_t)(b >> 32)) << 32) | uniform_u32((uint32_t)b)),
                     kOutside);
  };
  const rsrc_t rw = rsrc((uint64_t)a.q + (uint64_t)g * a.qstride + (uint64_t)(tn * kCols) * a.ldq);
  const rsrc_t rx = rsrc((uint64_t)a.p + (uint64_t)m0 * a.ldp);
  const rsrc_t rws = rsrc((uint64_t)a.ws + (uint64_t)g * a.wsstride);
  const rsrc_t rxs = rsrc((uint64_t)a.xs + (uint64_t)m0 * a.ldxs);
  uint32_t ow[2], ox[RB], ows[2], oxs[RB];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t row = i + h * (GATED ? width : 16);
    const bool ok = tn * kCols + (GATED ? i : row) < width;
    ow[h] = ok ? (uint32_t)(row * a.ldq) + q * 16 : kOutside;
    ows[h] = ok ? (uint32_t)((tn * kCols + row) / 128 * a.ldws) : kOutside;
  }
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    const bool ok = m0 + b * 16 + i < m_end;
    ox[b] = ok ? (uint32_t)((b * 16 + i) * a.ldp) + q * 16 : kOutside;
    oxs[b] = ok ? (uint32_t)((b * 16 + i) * a.ldxs) : kOutside;
  }
  f32x4 acc[2][RB];
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int b = 0; b < RB; ++b) acc[h][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  const uint32_t steps = (a.k + 127) / 128, each = (steps + NW - 1) / NW;
  const uint32_t s_end = min(steps, (wave + 1) * each);
  auto load = [](rsrc_t rs, uint32_t off, uint32_t o, bool in) __attribute__((always_inline)) {
    return __builtin_amdgcn_raw_buffer_load_b128(rs, (int)(in && off != kOutside ? off + o : kOutside), 0, 0);
  };
  // four scales from block s0 on: words that hold blocks the sum has
  auto load_scales = [&](rsrc_t rs, uint32_t off, uint32_t s0) __attribute__((always_inline)) {
    const uint32_t at = s0 & ~3u;
    const uint32_t lo = __builtin_amdgcn_raw_buffer_load_b32(rs, (int)(off != kOutside ? off + at : kOutside), 0, 0);
    const uint32_t hi = __builtin_amdgcn_raw_buffer_load_b32(
        rs, (int)(off != kOutside && at + 4 < steps ? off + at + 4 : kOutside), 0, 0);
    return u32pair{lo, hi};
  };
  for (uint32_t s0 = wave * each; s0 < s_end; s0 += kAhead) {
    Frag8 fw[kAhead][2], fx[kAhead][RB];
    u32pair cw[2], cx[RB];
#pragma unroll
    for (int h = 0; h < 2; ++h) cw[h] = load_scales(rws, ows[h], s0);
#pragma unroll
    for (int b = 0; b < RB; ++b) cx[b] = load_scales(rxs, oxs[b], s0);
#pragma unroll
    for (int n = 0; n < kAhead; ++n) {
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const uint32_t o = (s0 + n) * 128 + c * 64;
        const bool in = s0 + n < s_end && o + q * 16 < a.k;
#pragma unroll
        for (int h = 0; h < 2; ++h) fw[n][h].half[c] = load(rw, ow[h], o, in);
#pragma unroll
        for (int b = 0; b < RB; ++b) fx[n][b].half[c] = load(rx, ox[b], o, in);
      }
    }
    __builtin_amdgcn_sched_barrier(0);  // every load is issued before the first result is used
    int sw[2], sx[RB];
#pragma unroll
    for (int h = 0; h < 2; ++h) sw[h] = (int)__builtin_amdgcn_alignbyte(cw[h][1], cw[h][0], s0 & 3);
#pragma unroll
    for (int b = 0; b < RB; ++b) sx[b] = (int)__builtin_amdgcn_alignbyte(cx[b][1], cx[b][0], s0 & 3);
#pragma unroll
    for (int n = 0; n < kAhead; ++n) {
      if (s0 + n >= s_end) break;  // another wave's block, or none: its scale may be no number
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int b = 0; b < RB; ++b)
          acc[h][b] = mma8<O>(fw[n][h], sw[h] >> (8 * n), fx[n][b], sx[b] >> (8 * n), acc[h][b]);
    }
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
    put_forward<O, GATED>(a, g, m, tn * kCols + c, v, u);
  }
}

}  // namespace lin
}  // namespace llc
