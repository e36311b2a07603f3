// Host helpers shared by the grouped products' entry points: checks of
// arguments, how rows lie in memory, how many tiles a product has.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/llmoe.h"
#include "ll_linear.hpp"

namespace llc {
namespace lin {

constexpr size_t kMaxExtent = 0x7fffffff;

inline int esize(ll_dtype dt) { return dt == LL_F32 ? 4 : 2; }
inline bool aligned(const void *p, size_t to) { return (uintptr_t)p % to == 0; }
inline bool overlap(const void *a, size_t an, const void *b, size_t bn) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return a != nullptr && b != nullptr && an != 0 && bn != 0 && x < y + bn && y < x + an;
}
inline size_t span(size_t rows, size_t ld, size_t len, int es) { return rows == 0 ? 0 : ((rows - 1) * ld + len) * es; }

inline int check_desc(const ll_linear_desc *d) {
  if (d == nullptr || d->size != sizeof(ll_linear_desc)) return LL_ERR_INVALID;
  if (d->dt != LL_F32 && d->dt != LL_BF16) return LL_ERR_UNSUPPORTED;
  if ((int)d->act < LL_ACT_NONE || (int)d->act > LL_ACT_GEGLU) return LL_ERR_INVALID;
  if (d->groups < 1 || (d->offsets == nullptr && d->groups != 1) || !aligned(d->offsets, 4)) return LL_ERR_INVALID;
  if (d->in < 1 || d->out < 1) return LL_ERR_INVALID;
  if (d->groups > LL_MOE_MAX_EXPERTS || d->rows > kMaxExtent) return LL_ERR_UNSUPPORTED;
  // a tile's rows lie within 32 bits of bytes
  constexpr size_t kMaxFeatures = 1u << 20;
  if (d->in > kMaxFeatures || d->out > kMaxFeatures) return LL_ERR_UNSUPPORTED;
  for (size_t ld : {d->ldx, d->ldw, d->ldy, d->ldz, d->ldr})
    if (ld > 2 * kMaxFeatures) return LL_ERR_UNSUPPORTED;
  if (d->ldw < d->in || (d->groups > 1 && d->wstride < (d->out - 1) * d->ldw + d->in)) return LL_ERR_INVALID;
  return LL_OK;
}

// Both halves of a gated weight are read from one base, so that a group's lies
// within 32 bits of bytes.
inline bool gate_fits(const ll_linear_desc *d) { return d->out * d->ldw <= 0xF0000000ull / esize(d->dt); }

// Every row starts at a 16-byte address.
inline bool rows16(const void *p, size_t ld, int es) { return p == nullptr || (aligned(p, 16) && ld * es % 16 == 0); }
inline Rows rows_of(const void *p, size_t ld, size_t len, int es) {
  if (aligned(p, 16) && ld * es % 16 == 0 && len * es % 16 == 0) return kChunkRows;
  return aligned(p, 4) && ld * es % 4 == 0 ? kDwordRows : kAnyRows;
}
inline bool chunked(const void *p, size_t ld, size_t len, int es) { return rows_of(p, ld, len, es) == kChunkRows; }

// The same of every group's weight.
inline Rows weight_rows(const ll_linear_desc *d, const void *w, int es) {
  const Rows r = rows_of(w, d->ldw, d->in, es);
  if (d->groups == 1) return r;
  return std::min(r, d->wstride * es % 16 == 0 ? kChunkRows : d->wstride * es % 4 == 0 ? kDwordRows : kAnyRows);
}

inline size_t weight_span(const ll_linear_desc *d, int es) {
  return ((size_t)(d->groups - 1) * d->wstride + (d->out - 1) * d->ldw + d->in) * es;
}

inline int check_rows(const void *p, size_t ld, size_t len, int es, bool any) {
  if ((any && p == nullptr) || !aligned(p, es) || ld < len) return LL_ERR_INVALID;
  return LL_OK;
}

// Tiles of b x b that a product has at most: every group with rows may add one
// partial row tile.
inline uint64_t count_tiles(Pass pass, const Args &a, uint32_t b) {
  const uint64_t n = (a.n + b - 1) / b;
  if (pass == kGradW) return (uint64_t)((a.m + b - 1) / b) * a.groups * n;
  return (a.offsets == nullptr ? (a.rows + b - 1) / b : a.rows / b + std::min<uint64_t>(a.groups, a.rows)) * n;
}

// Tiles it has, about: half of a row tile of each group with rows is lost, and
// some more, since a few tiles past a full round of the chip cost another.
inline uint64_t expect_tiles(Pass pass, const Args &a, uint32_t b) {
  if (pass == kGradW || a.groups == 1) return count_tiles(pass, a, b);
  const uint64_t eighths = 8 * (uint64_t)a.rows / b + 6 * (uint64_t)std::min<uint32_t>(a.groups, a.rows);
  return std::max<uint64_t>(1, eighths / 8) * ((a.n + b - 1) / b);
}

// How a product runs: the tile's edge, its stages in LDS, the splits of its sum.
struct Plan {
  uint32_t tile, stages, splits;
};

constexpr uint32_t kFill = 256;  // workgroups that fill the chip

// Sizes the rows of split sums; bytes of one split.
inline uint64_t size_parts(Args &a, bool gate) {
  const uint32_t width = gate ? a.n / 2 : a.n;
  a.part_half = (width + kEw - 1) / kEw * kEw;
  a.part_row = gate ? 2 * a.part_half : a.part_half;
  return (uint64_t)a.rows_c * a.part_row * 4;
}
constexpr uint64_t kMaxParts = 256 << 20;  // bytes of split sums

}  // namespace lin
}  // namespace llc
