// Grouped products of 8-bit rows and weights: entry points of
// include/llblock.h.  Arguments are checked before any HIP call.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/llblock.h"
#include "ll_host.hpp"
#include "ll_linear8.hpp"
#include "ll_linear_host.hpp"

using namespace llc;
using namespace llc::lin;

namespace {

// Both halves of a gated weight are read from one base, so that a group's lies
// within 32 bits of bytes.
bool gate_fits8(const ll_linear_desc *d) { return d->out * d->ldw <= 0xF0000000ull; }

constexpr size_t kMaxScaleRow = 1u << 18;  // a tile's scales lie within 32 bits of bytes

size_t blocks_of(size_t n) { return (n + LL_BLOCK - 1) / LL_BLOCK; }

int check_scales(const uint8_t *p, size_t ld, size_t blocks, bool any) {
  if ((any && p == nullptr) || !aligned(p, 4) || ld % 4 != 0 || ld < blocks) return LL_ERR_INVALID;
  return ld > kMaxScaleRow ? LL_ERR_UNSUPPORTED : LL_OK;
}

using tile8_fn = void (*)(Args8);
using join_fn = void (*)(Args);

// How a product runs.  A stage has the bytes of the bfloat16 products' stages and
// matrix instructions that take as long, so their rules hold (ll_linear.hip),
// with a stage of 128 k.  Measured with cold caches, us with tiles of 256 / 128
// with 2 and 4 stages / 64 with 2 and 4; in front what the rule's choice takes:
//   128 x 4096 -> 4096    11.5   34 / 25, 18.7 / 19.0, 11.1   128 of 64
//   512 x 8192 -> 2048    18.5   80 / 44, 30 / 34, 18.4       256 of 64
//   301 x 1024 -> 8192    11.8   23 / 11.5, 11.0 / 10.7, 12.0
//  1024 x 4096 -> 4096    21.8   48 / 27.5, 21.9 / 31, 31     256 of 128
//  2048 x 7168 -> 2048    32.7   74 / 45, 34 / 49, 50         256 of 128
//  4096 x 4096 -> 2048    36.1   51 / 35.6, 42 / 55, 57       512 of 128
//  8 x 100 x 4096 -> 4096  44.6  49 / 45, 42 / 46, 46
//    48 x 7168 -> 1024    14.2   - / -, 21.8 / 29, 15.6; 2 splits 14.8    16 of 64
//  1000 x 7008 -> 200     15.1   - / -, 36 / 29, 19.1; 4 splits 15.6      64 of 64
// binary32 4096 x 4096 -> 4096  122   - / 124, 145 / 161, 176
// Rows that pass through registers always take tiles of 64: three stages of 128
// do not fit a thread's registers (1995 x 159 -> 6254: 54 us, with one stage of 128
// ahead 74; 4000 x 1001 -> 2001 52, so 58).  One of their stages takes 0.5-0.6 us.
Plan plan_of8(const Args &a, ll_dtype dt, Rows rows, uint64_t room) {
  Plan p{64, 2, 1};
  const uint64_t steps = (a.k + 127) / 128;
  const uint64_t t128 = expect_tiles(kForward, a, 128), t64 = expect_tiles(kForward, a, 64);
  if (rows != kAnyRows && dt == LL_BF16 && expect_tiles(kForward, a, 256) >= kFill) {
    p.tile = 256;
  } else if (rows != kAnyRows && t128 >= kFill) {
    p.tile = 128;
    if (t128 <= kFill * 9 / 8 && steps >= 12) p.stages = 4;
  } else {
    if (rows != kAnyRows && t64 <= 2 * kFill) p.stages = 4;
    if (t64 < 200) {  // too few tiles: splits of whole words of scales
      const uint64_t words = (steps + kScaleStages - 1) / kScaleStages;
      const uint64_t one = (uint64_t)a.rows_c * a.part_row * 4;
      const uint64_t most = std::min<uint64_t>(std::min<uint64_t>(16, words), std::min(room, kMaxParts) / std::max<uint64_t>(one, 1));
      const double whole = .33 * (rows == kAnyRows ? 1.6 : 1.) * (double)steps;
      double best = whole;
      for (uint64_t s = 2; s <= most; ++s) {
        const double rounds = (double)((t64 * s + kFill - 1) / kFill);
        const double cost = whole * rounds / (double)s + 3. + .009 * (double)(t64 * s);
        if (cost < best) {
          best = cost;
          p.splits = (uint32_t)s;
        }
      }
    }
  }
  return p;
}

template <typename O, int B, int ST, Rows ROWS>
tile8_fn pick8(bool gate) {
  if constexpr (B == 256 && ROWS == kChunkRows) return gate ? k_wide8<O, true> : k_wide8<O, false>;
  else return gate ? k_tile8<O, B, B, ST, true, ROWS> : k_tile8<O, B, B, ST, false, ROWS>;
}

template <typename O, int B, int ST, Rows ROWS>
int launch_tiles8(Args8 &a, bool gate, void *stream) {
  const uint32_t width = gate ? a.n / 2 : a.n;
  const uint32_t per_n = gate ? B / 2 : B;
  a.tiles_n = (width + per_n - 1) / per_n;
  a.tiles_m = (a.m + B - 1) / B;
  const uint64_t grid = count_tiles(kForward, a, B) / ((a.n + B - 1) / B) * a.tiles_n;
  constexpr uint32_t kParts = 2 * kMaxTail;
  if ((grid + kParts) * 256 >= 1ull << 32) return LL_ERR_UNSUPPORTED;
  // a short last round of 256-wide tiles runs in parts
  const uint64_t rest = grid % kRound;
  const bool tail = B == 256 && grid > kRound && (a.offsets != nullptr || (rest != 0 && rest <= kMaxTail));
  static_assert(8 * kEighths <= kParts && 4 * kQuarters <= kParts, "a workgroup a part");
  constexpr bool kOne = B == 256 && ROWS == kChunkRows;  // tiles and parts in one launch
  if (tail) a.tail = 1;
  a.first_part = (uint32_t)grid;
  const uint32_t all = (uint32_t)grid + (kOne && tail ? kParts : 0);
  hipLaunchKernelGGL((pick8<O, B, ST, ROWS>(gate)), dim3(all, a.splits), dim3(256), 0, (hipStream_t)stream, a);
  if constexpr (B == 256 && !kOne) {
    if (tail) {
      const tile8_fn parts = gate ? k_tail8<O, true, ROWS> : k_tail8<O, false, ROWS>;
      hipLaunchKernelGGL(parts, dim3(kParts), dim3(256), 0, (hipStream_t)stream, a);
    }
  }
  if (a.parts != nullptr) {
    const uint64_t items = (uint64_t)a.rows_c * ((width + kEw - 1) / kEw);
    if ((items + 255) / 256 * 256 >= 1ull << 32) return LL_ERR_UNSUPPORTED;
    const join_fn join = gate ? k_join<O, kForward, true> : k_join<O, kForward, false>;
    hipLaunchKernelGGL(join, dim3((unsigned)((items + 255) / 256)), dim3(256), 0, (hipStream_t)stream, (const Args &)a);
  }
  return launch_status();
}

template <typename O, Rows ROWS>
int launch_plan8(Args8 &a, const Plan &p, bool gate, void *stream) {
  if constexpr (ROWS == kAnyRows) {
    return launch_tiles8<O, 64, 2, ROWS>(a, gate, stream);
  } else {
    if constexpr (sizeof(O) == 2) {
      if (p.tile == 256) return launch_tiles8<O, 256, 2, ROWS>(a, gate, stream);
    }
    if (p.tile == 128)
      return p.stages == 4 ? launch_tiles8<O, 128, 4, ROWS>(a, gate, stream) : launch_tiles8<O, 128, 2, ROWS>(a, gate, stream);
    return p.stages == 4 ? launch_tiles8<O, 64, 4, ROWS>(a, gate, stream) : launch_tiles8<O, 64, 2, ROWS>(a, gate, stream);
  }
}

// Row blocks of 16 a workgroup of the streaming kernel takes; 0: the product
// is not for it (as stream_blocks of the other products).
int stream_blocks8(const Args &a, Rows rows) {
  if (rows != kChunkRows) return 0;
  const uint32_t each = a.groups == 1 ? a.rows : 2 * ((a.rows + a.groups - 1) / a.groups);
  return each <= 16 ? 1 : each <= 32 ? 2 : 0;
}

template <typename O, int RB>
int launch_stream8(Args8 &a, bool gate, void *stream) {
  constexpr int kNW = 8;
  a.tiles_n = gate ? (a.n / 2 + 15) / 16 : (a.n + 31) / 32;
  const uint64_t rows = a.offsets == nullptr ? (a.rows + RB * 16 - 1) / (RB * 16)
                                             : a.rows / (RB * 16) + std::min<uint64_t>(a.groups, a.rows);
  const uint64_t grid = rows * a.tiles_n;
  if (grid * kNW * 64 >= 1ull << 32) return LL_ERR_UNSUPPORTED;
  const tile8_fn fn = gate ? k_stream8<O, RB, kNW, true> : k_stream8<O, RB, kNW, false>;
  hipLaunchKernelGGL(fn, dim3((unsigned)grid), dim3(kNW * 64), 0, (hipStream_t)stream, a);
  return launch_status();
}

template <typename O>
int launch8(Args8 &a, Rows rows, bool gate, void *workspace, size_t workspace_bytes, void *stream) {
  const int blocks = stream_blocks8(a, rows);
  if (blocks == 1) return launch_stream8<O, 1>(a, gate, stream);
  if (blocks == 2) return launch_stream8<O, 2>(a, gate, stream);
  const uint64_t one = size_parts(a, gate);
  if (workspace == nullptr) workspace_bytes = 0;
  const Plan p = plan_of8(a, sizeof(O) == 4 ? LL_F32 : LL_BF16, rows, workspace_bytes);
  a.splits = p.splits;
  if (a.splits * one > workspace_bytes) a.splits = one == 0 ? 1 : (uint32_t)std::max<uint64_t>(1, workspace_bytes / one);
  a.parts = a.splits > 1 ? (float *)workspace : nullptr;
  if (rows == kChunkRows) return launch_plan8<O, kChunkRows>(a, p, gate, stream);
  if (rows == kDwordRows) return launch_plan8<O, kDwordRows>(a, p, gate, stream);
  return launch_plan8<O, kAnyRows>(a, p, gate, stream);
}

}  // namespace

extern "C" {

int ll_linear8_bytes(const ll_linear_desc *d, size_t *bytes) {
  if (bytes == nullptr) return LL_ERR_INVALID;
  const int st = check_desc(d);
  if (st != LL_OK) return st;
  const bool gate = gated((int)d->act);
  if (gate && !gate_fits8(d)) return LL_ERR_UNSUPPORTED;
  Args a{};
  a.offsets = d->offsets;
  a.groups = d->groups;
  a.rows = a.m = a.rows_c = (uint32_t)d->rows;
  a.n = (uint32_t)d->out;
  a.k = (uint32_t)d->in;
  // the alignment that the leading dimensions allow; pointers that allow less
  // get no more splits than this
  const Rows rows = std::min(rows_of(nullptr, d->ldx, d->in, 1), weight_rows(d, nullptr, 1));
  *bytes = 0;
  if (stream_blocks8(a, rows) != 0) return LL_OK;
  const uint64_t one = size_parts(a, gate);
  const uint32_t splits = plan_of8(a, d->dt, rows, ~0ull).splits;
  *bytes = splits > 1 ? (size_t)splits * one : 0;
  return LL_OK;
}

int ll_linear8(const ll_linear_desc *d, const uint8_t *x, const uint8_t *xs, size_t ldxs, const uint8_t *w,
               const uint8_t *ws, size_t ldws, size_t wsstride, const void *bias, const void *residual, void *y,
               void *z, void *workspace, size_t workspace_bytes, void *stream) {
  int st = check_desc(d);
  if (st != LL_OK) return st;
  const int es = esize(d->dt);
  const bool gate = gated((int)d->act), any = d->rows != 0;
  if (gate && d->out % 2 != 0) return LL_ERR_INVALID;
  if (gate && !gate_fits8(d)) return LL_ERR_UNSUPPORTED;
  const size_t width = gate ? d->out / 2 : d->out, kb = blocks_of(d->in), ob = blocks_of(d->out);
  st = check_rows(x, d->ldx, d->in, 1, any);
  if (st == LL_OK) st = check_rows(w, d->ldw, d->in, 1, any);
  if (st == LL_OK) st = check_rows(y, d->ldy, width, es, any);
  if (st == LL_OK && z != nullptr) st = check_rows(z, d->ldz, d->out, es, any);
  if (st == LL_OK && residual != nullptr) st = check_rows(residual, d->ldr, width, es, any);
  if (st == LL_OK) st = check_scales(xs, ldxs, kb, any);
  if (st == LL_OK) st = check_scales(ws, ldws, kb, any);
  if (st != LL_OK) return st;
  if (d->groups > 1 && (wsstride % 4 != 0 || wsstride < (ob - 1) * ldws + kb)) return LL_ERR_INVALID;
  if (!aligned(bias, es) || !aligned(workspace, 16)) return LL_ERR_INVALID;
  const size_t yb = span(d->rows, d->ldy, width, es), zb = span(d->rows, d->ldz, d->out, es);
  const size_t rb = span(d->rows, d->ldr, width, es);
  const struct {
    const void *p;
    size_t n;
  } ins[] = {{x, span(d->rows, d->ldx, d->in, 1)},
             {w, weight_span(d, 1)},
             {xs, span(d->rows, ldxs, kb, 1)},
             {ws, (d->groups - 1) * wsstride + (ob - 1) * ldws + kb},
             {bias, d->groups * d->out * es}};
  for (const auto &i : ins)
    if (overlap(i.p, i.n, y, yb) || overlap(i.p, i.n, z, zb)) return LL_ERR_INVALID;
  if (overlap(y, yb, z, zb) || overlap(residual, rb, z, zb) ||
      (overlap(residual, rb, y, yb) && !(residual == y && d->ldr == d->ldy)))
    return LL_ERR_INVALID;
  if (!any) return LL_OK;
  Args8 a{};
  a.p = x;
  a.ldp = d->ldx;
  a.q = w;
  a.ldq = d->ldw;
  a.qstride = d->wstride;
  a.offsets = d->offsets;
  a.groups = d->groups;
  a.rows = a.m = a.rows_c = (uint32_t)d->rows;
  a.n = (uint32_t)d->out;
  a.k = (uint32_t)d->in;
  a.bias = bias;
  a.res = residual;
  a.ldr = d->ldr;
  a.zout = z;
  a.ldz = d->ldz;
  a.c = y;
  a.ldc = d->ldy;
  a.act = (int)d->act;
  a.xs = xs;
  a.ws = ws;
  a.ldxs = ldxs;
  a.ldws = ldws;
  a.wsstride = wsstride;
  const Rows rows = std::min(rows_of(x, d->ldx, d->in, 1), weight_rows(d, w, 1));
  return d->dt == LL_F32 ? launch8<float>(a, rows, gate, workspace, workspace_bytes, stream)
                         : launch8<__bf16>(a, rows, gate, workspace, workspace_bytes, stream);
}

}  // extern "C"
