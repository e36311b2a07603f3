// Grouped matrix products: entry points of include/llmoe.h.  Arguments are
// checked before any HIP call.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/llmoe.h"
#include "ll_host.hpp"
#include "ll_linear.hpp"
#include "ll_linear_host.hpp"

using namespace llc;
using namespace llc::lin;

namespace {

using tile_fn = void (*)(Args);

template <typename T, Pass PASS, int B, int WM, int WN, int ST, Rows ROWS>
tile_fn pick(bool gate) {
  if constexpr (PASS == kForward) {
    if (gate) return k_tile<T, PASS, B, B, WM, WN, ST, true, ROWS>;
  }
  return k_tile<T, PASS, B, B, WM, WN, ST, false, ROWS>;
}

// Larger tiles move fewer operand bytes but need many tiles to fill the chip.
// Measured with cold caches, bfloat16, us with tiles of 256 / 128 with 2 and 4
// stages / 64 with 2 and 4, and the number of tiles:
//   1024 x 4096 -> 4096   111 / 68, 54 / 70, 73      256 of 128
//   2048 x 2048 -> 2048    61 / 39, 32 / 40, 42      256 of 128
//    301 x 1024 -> 8192    38 / 23.7, 21.8 / 22.0, 23.2   192 of 128 (with bias and
//      residual, call after call: - / 19.6, 18.6 / 14.7, 16.9)
//   1024 x 1032 -> 2056    44 / 25.4, 24.4 / 22.8, 25.6   136 of 128, 528 of 64
//    512 x 2048 -> 2048    60 / 38, 32 / 29, 17.8    256 of 64
//    128 x 4096 -> 4096    98 / 69, 54 / 56, 31; 4 splits 26     128 of 64
//   1000 x 7000 -> 200    237 / 127, 94 / 82, 51; 4 splits 25     64 of 64
//     64 x 1024 -> 1024    30 / 22, 17 / 19, 14.8; 4 splits 11.9  16 of 64
//   weight gradient of 301 rows, 1024 x 8192  22 / 17.7, 24 / 23, 27  512 of 128
// 256 is for bfloat16 only: binary32 is bound by its matrix instructions, which
// are 16 times slower (1024^3: 68 us with 128, 28 us with 64).
//
// Up to 128 tiles of 128, and a long sum: s = 256 / tiles splits of them fill
// the chip in one round and read a quarter to a half of the operands that tiles
// of 64 do, for the cost of the joining.  us with 64-wide tiles / these:
//   bfloat16  640 x 2048 -> 2048  23.3 / 24.4   8192 -> 2048  67.8 / 45.6  3 splits
//             512 x 2048 -> 4096  26.7 / 28.8   8192 -> 4096  79.3 / 63.0  2 splits
//             weight gradient of 2300 rows, 1024 x 1024  18.7 / 24.9, of 8192 rows  51.5 / 39.5  4 splits
//             512 x 3584 -> 1024  20.8 / 23.1   8192 -> 1024  33.2 / 30.5  8 splits
//   binary32  640 x 1024 -> 2048  43.6 / 38.4   4096 -> 2048   148 / 99.7  3 splits
//             512 x 1024 -> 4096  44.3 / 49.3   4096 -> 4096   154 / 137   2 splits
// The lines through these times decide.  Returns the splits, or 0 where tiles of
// 64 are faster or `room` bytes do not hold the parts.  Groups of less
// than a tile of rows on average keep tiles of 64, since the larger ones are
// fewer than expected (8 groups of 100, 4096 -> 1024: 37 us, split 47), and so
// does a weight gradient with a bias, which tiles of 64 sum along (8192 rows,
// 1024 x 1024: 50 us, split and summed apart 72).
uint32_t wide_splits(const Args &a, ll_dtype dt, uint64_t steps, uint64_t t128, uint64_t t64, uint64_t room) {
  if (t128 < 32 || t128 > kFill / 2 || (dt == LL_F32 && t64 <= kFill)) return 0;
  const uint64_t s = kFill / t128;
  if (s * a.rows_c * a.part_row * 4 > std::min(room, kMaxParts)) return 0;
  const double n = (double)steps;
  double narrow, wide;
  if (dt == LL_F32) {
    narrow = 8. + 1.1 * n;
    wide = 18. + 1.87 * n / s;
  } else {
    narrow = t64 < 200 ? 12. + .0013 * t64 * n : 7. + (t64 <= kFill ? .34 : .51) * n;
    wide = 18. + .66 * n / s;
  }
  return wide < narrow ? (uint32_t)s : 0;
}

Plan plan_of(Pass pass, const Args &a, ll_dtype dt, Rows rows, uint64_t room) {
  Plan p{64, 2, 1};
  const uint32_t bk = 128 / esize(dt);
  const uint64_t k = pass == kGradW ? a.k / a.groups : a.k, steps = (k + bk - 1) / bk;
  const uint64_t t128 = expect_tiles(pass, a, 128), t64 = expect_tiles(pass, a, 64);
  // tiles of 128 are about a quarter of those of 64, and may replace them
  const bool full = rows != kAnyRows && (pass == kGradW ? a.dbias == nullptr : a.rows / a.groups >= 128);
  if (rows != kAnyRows && dt == LL_BF16 && expect_tiles(pass, a, 256) >= kFill) {
    p.tile = 256;
  } else if (t128 >= (dt == LL_BF16 ? kFill : 4 * kFill)) {
    p.tile = 128;
    // one workgroup a CU: four stages of it hide what two workgroups hide from each other
    if (t128 <= kFill * 9 / 8 && steps >= 12) p.stages = 4;
  } else if (const uint32_t s = full ? wide_splits(a, dt, steps, t128, t64, room) : 0) {
    p.tile = 128;
    p.stages = dt == LL_BF16 ? 4 : 2;
    p.splits = s;
  } else if (full && dt == LL_BF16 && t128 > 160 && steps >= 24) {
    // a round of 128 that is not quite full, and a sum long enough to pay for
    // its start (184 tiles: 1000 x 1024 -> 2944 19.4 us with 64, 19.8 with 128;
    // 2048 -> 2944 32.6 and 30.4; 8192 -> 2944 101 and 86)
    p.tile = 128;
    p.stages = 4;
  } else {
    if (t64 <= 2 * kFill) p.stages = 4;
    // Too few tiles: the sum is cut into shares of four stages or more.  s
    // splits cost the rounds of the chip they make, each 1 / s of a whole one
    // of .33 us a stage (binary32 .62), and the joining (bfloat16, us whole /
    // 2 / 3 / 4 splits: 16 tiles, 16 stages 11.2 / 11.6 / 11.4 / 11.2 and 64
    // stages 25.8 / 19.7 / 17.1 / 15.5; 64 tiles, 16 stages 11.6 / 12.8 / 13.2 /
    // 13.4 and 64 stages 26.2 / 21.2 / 18.6 / 17.7; 160 tiles, 16 stages 11.6 /
    // 16.9 / 17.5 / 20.5 and 64 stages 28.0 / 30.8 / 25.8 / 28.6).  A stage of
    // rows that are not whole chunks takes longer: of dwords 1.08-1.17 times as
    // long in binary32 and 1.2-1.7 in bfloat16, through registers 2.3-3.6 times.
    // Over 7 shapes of 16 to 176 tiles, 4 lengths and the three products the
    // splits chosen so are 0.6 %, 0.4 % and 9 % slower than the best of 1 to 6 and
    // 8 on average (caches warm 0.7 %, 0.4 %, 3.5 %); without the factors 0.8 %,
    // 0.9 % and 21 % (1.2 %, 0.6 %, 11 %).  Groups are taken at their average
    // (4 of 16 to 100 rows, 4096 -> 512 bfloat16: 18.2 us whole, 20.4 split).
    if (t64 < 200) {
      const uint64_t one = (uint64_t)a.rows_c * a.part_row * 4;
      const uint64_t most = std::min<uint64_t>(std::min<uint64_t>(16, steps / 4), kMaxParts / std::max<uint64_t>(one, 1));
      const double slower = rows == kChunkRows ? 1. : dt == LL_F32 ? 1.15 : rows == kDwordRows ? 1.4 : 2.4;
      const double whole = (dt == LL_BF16 ? .33 : .62) * slower * (double)steps;
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
  if (rows == kAnyRows) p.stages = 2;
  return p;
}

template <typename T, Pass PASS, int B, int WM, int WN, int ST, Rows ROWS>
int launch_tiles(Args &a, bool gate, void *stream) {
  const uint32_t width = gate ? a.n / 2 : a.n;
  const uint32_t per_n = gate ? B / 2 : B;
  a.tiles_n = (width + per_n - 1) / per_n;
  a.tiles_m = (a.m + B - 1) / B;
  const uint64_t grid = count_tiles(PASS, a, B) / ((a.n + B - 1) / B) * a.tiles_n;
  constexpr int kThreads = WM * WN * 64;
  if (grid * kThreads >= 1ull << 32) return LL_ERR_UNSUPPORTED;
  const tile_fn fn = pick<T, PASS, B, WM, WN, ST, ROWS>(gate);
  // more tiles than one round of the chip: a short last round is left to the
  // 128-wide kernel, four of whose tiles make one of these
  // (without offsets the number of tiles is known here)
  const uint64_t rest = grid % kRound;
  const bool tail = B == 256 && PASS != kGradW && grid > kRound &&
                    (a.offsets != nullptr || (rest != 0 && rest <= kMaxTail));
  if (tail) a.tail = 1;
  hipLaunchKernelGGL(fn, dim3((unsigned)grid, a.splits), dim3(kThreads), 0, (hipStream_t)stream, a);
  if constexpr (B == 256 && PASS != kGradW) {
    if (tail) {
      a.tail = 2;
      const tile_fn rest = pick<T, PASS, 128, 2, 2, 4, ROWS>(gate);
      hipLaunchKernelGGL(rest, dim3(4 * kMaxTail), dim3(256), 0, (hipStream_t)stream, a);
    }
  }
  if (a.parts != nullptr) {
    const uint64_t items = (uint64_t)a.rows_c * ((width + kEw - 1) / kEw);
    if ((items + 255) / 256 * 256 >= 1ull << 32) return LL_ERR_UNSUPPORTED;
    tile_fn join = k_join<T, PASS, false>;
    if constexpr (PASS == kForward) {
      if (gate) join = k_join<T, PASS, true>;
    }
    hipLaunchKernelGGL(join, dim3((unsigned)((items + 255) / 256)), dim3(256), 0, (hipStream_t)stream, a);
  }
  return launch_status();
}

template <typename T, Pass PASS, Rows ROWS>
int launch_plan(Args &a, const Plan &p, bool gate, void *stream) {
  if constexpr (sizeof(T) == 2 && ROWS != kAnyRows) {
    if (p.tile == 256) return launch_tiles<T, PASS, 256, 2, 4, 2, ROWS>(a, gate, stream);
  }
  if constexpr (ROWS == kAnyRows) {
    // eight waves: a stage of a thread's chunks lies in registers meanwhile
    if (p.tile == 128) return launch_tiles<T, PASS, 128, 2, 4, 2, ROWS>(a, gate, stream);
    return launch_tiles<T, PASS, 64, 2, 2, 2, ROWS>(a, gate, stream);
  } else {
    if (p.tile == 128)
      return p.stages == 4 ? launch_tiles<T, PASS, 128, 2, 2, 4, ROWS>(a, gate, stream)
                           : launch_tiles<T, PASS, 128, 2, 2, 2, ROWS>(a, gate, stream);
    return p.stages == 4 ? launch_tiles<T, PASS, 64, 2, 2, 4, ROWS>(a, gate, stream)
                         : launch_tiles<T, PASS, 64, 2, 2, 2, ROWS>(a, gate, stream);
  }
}

template <typename T, Pass PASS>
int launch_rows(Args &a, const Plan &p, Rows rows, bool gate, void *stream) {
  if (rows == kChunkRows) return launch_plan<T, PASS, kChunkRows>(a, p, gate, stream);
  if constexpr (sizeof(T) == 2) {  // binary32 rows are always whole dwords
    if (rows == kAnyRows) return launch_plan<T, PASS, kAnyRows>(a, p, gate, stream);
  }
  return launch_plan<T, PASS, kDwordRows>(a, p, gate, stream);
}

void launch_bias_grad(const Args &a, ll_dtype dt, void *stream) {
  const int es = esize(dt);
  const bool vec = chunked(a.p, a.ldp, a.m, es);
  const auto fn = dt == LL_F32 ? (vec ? k_bias_grad<float, true> : k_bias_grad<float, false>)
                               : (vec ? k_bias_grad<__bf16, true> : k_bias_grad<__bf16, false>);
  const unsigned cols = kBiasChunks * (vec ? 16 / es : 1);
  hipLaunchKernelGGL(fn, dim3((a.m + cols - 1) / cols, a.groups), dim3(kBiasChunks * kBiasLanes), 0,
                     (hipStream_t)stream, a);
}

template <Pass PASS>
int launch_product(Args &a, ll_dtype dt, bool gate, Rows rows, void *workspace, size_t workspace_bytes, void *stream) {
  const uint64_t one = size_parts(a, gate);
  if (workspace == nullptr) workspace_bytes = 0;
  Plan p = plan_of(PASS, a, dt, rows, workspace_bytes);
  if (p.splits * one > workspace_bytes) p.splits = one == 0 ? 1 : (uint32_t)std::max<uint64_t>(1, workspace_bytes / one);
  a.splits = p.splits;
  a.parts = p.splits > 1 ? (float *)workspace : nullptr;
  if (PASS == kGradW && a.dbias != nullptr) {
    a.sum_bias = p.tile == 64 && p.splits == 1;
    if (!a.sum_bias) launch_bias_grad(a, dt, stream);
  }
  return dt == LL_F32 ? launch_rows<float, PASS>(a, p, rows, gate, stream)
                      : launch_rows<__bf16, PASS>(a, p, rows, gate, stream);
}

// ---------------------------------------------------------------- few rows
// Row blocks of 16 a workgroup of the streaming kernel takes; 0: the product
// is not for it.
int stream_blocks(const Args &a, Rows rows) {
  if (rows != kChunkRows) return 0;
  // One group: its rows are known.  Several: their sizes are not, and one of
  // more than the workgroup's rows reads its weight twice (32 groups of 7168 ->
  // 2 x 2048, 32 rows each on average: 667 us here, 372 with tiles).
  const uint32_t each = a.groups == 1 ? a.rows : 2 * ((a.rows + a.groups - 1) / a.groups);
  return each <= 16 ? 1 : each <= 32 ? 2 : 0;
}

template <typename T, int RB>
int launch_stream(Args &a, bool gate, void *stream) {
  constexpr int kNW = 8;
  a.tiles_n = gate ? (a.n / 2 + 15) / 16 : (a.n + 31) / 32;
  const uint64_t rows = a.offsets == nullptr ? (a.rows + RB * 16 - 1) / (RB * 16)
                                             : a.rows / (RB * 16) + std::min<uint64_t>(a.groups, a.rows);
  const uint64_t grid = rows * a.tiles_n;
  if (grid * kNW * 64 >= 1ull << 32) return LL_ERR_UNSUPPORTED;
  const tile_fn fn = gate ? k_stream<T, RB, kNW, true> : k_stream<T, RB, kNW, false>;
  hipLaunchKernelGGL(fn, dim3((unsigned)grid), dim3(kNW * 64), 0, (hipStream_t)stream, a);
  return launch_status();
}

}  // namespace

extern "C" {

int ll_linear_desc_init(ll_linear_desc *d, ll_dtype dt, ll_act act, int groups, size_t rows, size_t in, size_t out) {
  if (d == nullptr) return LL_ERR_INVALID;
  *d = ll_linear_desc{};
  d->size = sizeof(ll_linear_desc);
  d->dt = dt;
  d->act = act;
  d->groups = groups;
  d->rows = rows;
  d->in = in;
  d->out = out;
  d->ldx = in;
  d->ldw = in;
  d->wstride = in * out;
  d->ldy = gated((int)act) ? out / 2 : out;
  d->ldz = out;
  d->ldr = d->ldy;
  return LL_OK;
}

int ll_linear_bytes(const ll_linear_desc *d, ll_linear_pass pass, size_t *bytes) {
  if (bytes == nullptr || (int)pass < LL_LINEAR_FORWARD || (int)pass > LL_LINEAR_GRAD_W) return LL_ERR_INVALID;
  const int st = check_desc(d);
  if (st != LL_OK) return st;
  if (pass == LL_LINEAR_FORWARD && gated((int)d->act) && !gate_fits(d)) return LL_ERR_UNSUPPORTED;
  Args a{};
  a.offsets = d->offsets;
  a.groups = d->groups;
  a.rows = (uint32_t)d->rows;
  const bool gw = pass == LL_LINEAR_GRAD_W;
  a.m = gw ? (uint32_t)d->out : a.rows;
  a.n = (uint32_t)(pass == LL_LINEAR_FORWARD ? d->out : d->in);
  a.k = gw ? a.rows : (uint32_t)(pass == LL_LINEAR_FORWARD ? d->in : d->out);
  a.rows_c = gw ? a.m * (uint32_t)a.groups : a.rows;
  const int es = esize(d->dt);
  // the alignment that the leading dimensions allow; pointers that allow less
  // get no more splits than this
  const Rows rx = rows_of(nullptr, d->ldx, d->in, es), rz = rows_of(nullptr, d->ldy, d->out, es);
  const Rows rw = weight_rows(d, nullptr, es);
  const Rows rows = gw ? std::min(rx, rz) : std::min(rw, pass == LL_LINEAR_FORWARD ? rx : rz);
  *bytes = 0;
  if (pass == LL_LINEAR_FORWARD && stream_blocks(a, rows) != 0) return LL_OK;
  const uint64_t one = size_parts(a, pass == LL_LINEAR_FORWARD && gated((int)d->act));
  uint32_t splits = plan_of((Pass)pass, a, d->dt, rows, ~0ull).splits;
  if (gw) {  // a bias gradient may change the plan
    a.dbias = &a;
    splits = std::max(splits, plan_of(kGradW, a, d->dt, rows, ~0ull).splits);
  }
  *bytes = splits > 1 ? (size_t)splits * one : 0;
  return LL_OK;
}

int ll_linear(const ll_linear_desc *d, const void *x, const void *w, const void *bias, const void *residual, void *y,
              void *z, void *workspace, size_t workspace_bytes, void *stream) {
  int st = check_desc(d);
  if (st != LL_OK) return st;
  const int es = esize(d->dt);
  const bool gate = gated((int)d->act), any = d->rows != 0;
  if (gate && d->out % 2 != 0) return LL_ERR_INVALID;
  if (gate && !gate_fits(d)) return LL_ERR_UNSUPPORTED;
  const size_t width = gate ? d->out / 2 : d->out;
  st = check_rows(x, d->ldx, d->in, es, any);
  if (st == LL_OK) st = check_rows(w, d->ldw, d->in, es, any);
  if (st == LL_OK) st = check_rows(y, d->ldy, width, es, any);
  if (st == LL_OK && z != nullptr) st = check_rows(z, d->ldz, d->out, es, any);
  if (st == LL_OK && residual != nullptr) st = check_rows(residual, d->ldr, width, es, any);
  if (st != LL_OK) return st;
  if (!aligned(bias, es) || !aligned(workspace, 16)) return LL_ERR_INVALID;
  const size_t yb = span(d->rows, d->ldy, width, es), zb = span(d->rows, d->ldz, d->out, es);
  const size_t xb = span(d->rows, d->ldx, d->in, es), rb = span(d->rows, d->ldr, width, es);
  if (overlap(x, xb, y, yb) || overlap(x, xb, z, zb) || overlap(y, yb, z, zb) || overlap(residual, rb, z, zb) ||
      overlap(w, weight_span(d, es), y, yb) || overlap(w, weight_span(d, es), z, zb) ||
      (overlap(residual, rb, y, yb) && !(residual == y && d->ldr == d->ldy)))
    return LL_ERR_INVALID;
  if (!any) return LL_OK;
  Args a{};
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
  Rows rows = std::min(rows_of(x, d->ldx, d->in, es), weight_rows(d, w, es));

  const int blocks = stream_blocks(a, rows);
  if (blocks == 1)
    return d->dt == LL_F32 ? launch_stream<float, 1>(a, gate, stream) : launch_stream<__bf16, 1>(a, gate, stream);
  if (blocks == 2)
    return d->dt == LL_F32 ? launch_stream<float, 2>(a, gate, stream) : launch_stream<__bf16, 2>(a, gate, stream);
  return launch_product<kForward>(a, d->dt, gate, rows, workspace, workspace_bytes, stream);
}

int ll_linear_grad_x(const ll_linear_desc *d, const void *dz, const void *w, const void *z, void *dx, void *workspace,
                     size_t workspace_bytes, void *stream) {
  int st = check_desc(d);
  if (st != LL_OK) return st;
  const int es = esize(d->dt);
  const bool any = d->rows != 0;
  const size_t width = gated((int)d->act) ? 2 * d->in : d->in;
  st = check_rows(dz, d->ldy, d->out, es, any);
  if (st == LL_OK) st = check_rows(w, d->ldw, d->in, es, any);
  if (st == LL_OK) st = check_rows(dx, d->ldx, width, es, any);
  if (st == LL_OK && d->act != LL_ACT_NONE) st = check_rows(z, d->ldz, width, es, any);
  if (st != LL_OK) return st;
  if (!aligned(workspace, 16)) return LL_ERR_INVALID;
  const size_t xb = span(d->rows, d->ldx, width, es);
  if (overlap(dz, span(d->rows, d->ldy, d->out, es), dx, xb) || overlap(w, weight_span(d, es), dx, xb) ||
      (d->act != LL_ACT_NONE && overlap(z, span(d->rows, d->ldz, width, es), dx, xb)))
    return LL_ERR_INVALID;
  if (!any) return LL_OK;
  Args a{};
  a.p = dz;
  a.ldp = d->ldy;
  a.q = w;
  a.ldq = d->ldw;
  a.qstride = d->wstride;
  a.offsets = d->offsets;
  a.groups = d->groups;
  a.rows = a.m = a.rows_c = (uint32_t)d->rows;
  a.n = (uint32_t)d->in;
  a.k = (uint32_t)d->out;
  a.z = z;
  a.ldz = d->ldz;
  a.c = dx;
  a.ldc = d->ldx;
  a.act = (int)d->act;
  a.vec_c = rows16(dx, d->ldx, es) && rows16(z, d->ldz, es);
  const Rows rows = std::min(rows_of(dz, d->ldy, d->out, es), weight_rows(d, w, es));
  return launch_product<kGradX>(a, d->dt, false, rows, workspace, workspace_bytes, stream);
}

int ll_linear_grad_w(const ll_linear_desc *d, const void *dz, const void *x, void *dw, void *dbias, uint32_t flags,
                     void *workspace, size_t workspace_bytes, void *stream) {
  int st = check_desc(d);
  if (st != LL_OK) return st;
  if ((flags & ~(LL_GRAD_F32 | LL_GRAD_ADD)) != 0) return LL_ERR_INVALID;
  const int es = esize(d->dt);
  const int gs = (flags & LL_GRAD_F32) ? 4 : es;
  const bool any = d->rows != 0;
  st = check_rows(dz, d->ldy, d->out, es, any);
  if (st == LL_OK) st = check_rows(x, d->ldx, d->in, es, any);
  if (st == LL_OK) st = check_rows(dw, d->ldw, d->in, gs, true);
  if (st != LL_OK) return st;
  if (!aligned(dbias, gs) || !aligned(workspace, 16)) return LL_ERR_INVALID;
  const size_t wb = weight_span(d, gs), bb = (size_t)d->groups * d->out * gs;
  const size_t yb = span(d->rows, d->ldy, d->out, es), xb = span(d->rows, d->ldx, d->in, es);
  if (overlap(dz, yb, dw, wb) || overlap(x, xb, dw, wb) || overlap(dz, yb, dbias, bb) || overlap(x, xb, dbias, bb) ||
      overlap(dw, wb, dbias, bb))
    return LL_ERR_INVALID;
  Args a{};
  a.p = dz;
  a.ldp = d->ldy;
  a.q = x;
  a.ldq = d->ldx;
  a.cstride = d->wstride;
  a.offsets = d->offsets;
  a.groups = d->groups;
  a.rows = (uint32_t)d->rows;
  a.m = (uint32_t)d->out;
  a.rows_c = a.m * (uint32_t)a.groups;
  a.n = (uint32_t)d->in;
  a.c = dw;
  a.ldc = d->ldw;
  a.dbias = dbias;
  a.flags = flags;
  const Rows rows = std::min(rows_of(dz, d->ldy, d->out, es), rows_of(x, d->ldx, d->in, es));
  a.k = a.rows;
  return launch_product<kGradW>(a, d->dt, false, rows, workspace, workspace_bytes, stream);
}

int ll_act_grad(const void *dy, size_t lddy, const void *z, size_t ldz, size_t rows, size_t features, ll_dtype dt,
                ll_act act, void *dz, size_t lddz, void *stream) {
  if (dt != LL_F32 && dt != LL_BF16) return LL_ERR_UNSUPPORTED;
  if ((int)act < LL_ACT_NONE || (int)act > LL_ACT_GEGLU) return LL_ERR_INVALID;
  if (rows > kMaxExtent || features > kMaxExtent / 2) return LL_ERR_UNSUPPORTED;
  const int es = esize(dt);
  const bool gate = gated((int)act);
  const size_t width = gate ? 2 * features : features;
  const bool any = rows != 0 && features != 0;
  int st = check_rows(dy, lddy, features, es, any);
  if (st == LL_OK) st = check_rows(z, ldz, width, es, any);
  if (st == LL_OK) st = check_rows(dz, lddz, width, es, any);
  if (st != LL_OK) return st;
  const size_t ob = span(rows, lddz, width, es);
  if (overlap(dy, span(rows, lddy, features, es), dz, ob) && !(!gate && dy == dz && lddy == lddz)) return LL_ERR_INVALID;
  if (overlap(z, span(rows, ldz, width, es), dz, ob) && !(z == dz && ldz == lddz)) return LL_ERR_INVALID;
  if (!any) return LL_OK;
  ActArgs a{dy, z, dz, lddy, ldz, lddz, (uint32_t)rows, (uint32_t)features, (int)act};
  const bool vec = chunked(dy, lddy, features, es) && chunked(z, ldz, features, es) && chunked(dz, lddz, features, es);
  int cus = 0;
  st = device_cus(&cus);
  if (st != LL_OK) return st;
  const uint64_t items = (uint64_t)rows * features / (vec ? 16 / es : 1);
  const unsigned grid = (unsigned)std::min<uint64_t>((items + 255) / 256, (uint64_t)cus * 16);
  const auto fn = dt == LL_F32 ? (vec ? k_act_grad<float, true> : k_act_grad<float, false>)
                               : (vec ? k_act_grad<__bf16, true> : k_act_grad<__bf16, false>);
  hipLaunchKernelGGL(fn, dim3(grid), dim3(256), 0, (hipStream_t)stream, a);
  return launch_status();
}

}  // extern "C"
