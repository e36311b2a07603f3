// Routing, dispatch and combine: entry points of include/llmoe.h.  Arguments
// are checked before any HIP call; a call is one to three launches.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/llmoe.h"
#include "ll_host.hpp"
#include "ll_moe.hpp"

using namespace llc;
using namespace llc::moe;

namespace {

constexpr size_t kMaxExtent = 0x7fffffff;
constexpr size_t kMaxTokens = (1u << 24) - 1;  // a workgroup of 256 threads each in one launch

int esize(ll_dtype dt) { return dt == LL_F32 ? 4 : 2; }

bool aligned(const void *p, size_t to) { return (uintptr_t)p % to == 0; }

// Vector path: the first row is 16-byte aligned and so is the distance of two rows.
bool vec16(const void *p, size_t ld, int es) { return p == nullptr || (aligned(p, 16) && ld * es % 16 == 0); }

// Bytes from the first to past the last element of `rows` rows.
bool overlap(const void *a, size_t an, const void *b, size_t bn) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return a != nullptr && b != nullptr && an != 0 && bn != 0 && x < y + bn && y < x + an;
}
size_t span(size_t rows, size_t ld, size_t len, int es) { return rows == 0 || len == 0 ? 0 : ((rows - 1) * ld + len) * es; }

// A matrix argument: not NULL, aligned to its element, rows no longer than ld.
int check_rows(const void *p, size_t ld, size_t len, int es) {
  if (p == nullptr || !aligned(p, es) || ld < len) return LL_ERR_INVALID;
  return ld > kMaxExtent ? LL_ERR_UNSUPPORTED : LL_OK;
}

int check_choice(size_t tokens, int experts, int k) {
  if (experts < 1 || k < 1 || k > LL_MOE_MAX_K) return LL_ERR_INVALID;
  if (experts > LL_MOE_MAX_EXPERTS || tokens > kMaxTokens || tokens * (size_t)k > kMaxExtent) return LL_ERR_UNSUPPORTED;
  return LL_OK;
}

// ---------------------------------------------------------------- routing
using route_fn = void (*)(RouteArgs);

template <typename T, int W, int NPL>
route_fn route_of(bool grad, bool vec) {
  if (grad) return vec ? k_route_grad<T, W, NPL, true> : k_route_grad<T, W, NPL, false>;
  return vec ? k_route<T, W, NPL, true> : k_route<T, W, NPL, false>;
}

// A lane's logits: the fewest of these that hold a row (fewer steps over them).
constexpr int kNpl[] = {1, 2, 4, 6, 8, 10, 12, 16};

template <typename T, int W>
route_fn route_fn_of(int npl, bool grad, bool vec) {
  switch (npl) {
    case 1: return route_of<T, W, 1>(grad, vec && sizeof(T) == 4);
    case 2: return route_of<T, W, 2>(grad, vec);
    case 4: return route_of<T, W, 4>(grad, vec);
    case 6: return route_of<T, W, 6>(grad, vec);
    case 8: return route_of<T, W, 8>(grad, vec);
    case 10: return route_of<T, W, 10>(grad, vec);
    case 12: return route_of<T, W, 12>(grad, vec);
    default: return route_of<T, W, 16>(grad, vec);
  }
}

int launch_route(const RouteArgs &a, ll_dtype dt, bool grad, void *stream) {
  // Many tokens: 16 lanes a token where its logits and choices fit them, so
  // that four tokens of a wave share the steps over the lanes (32301 x 160
  // bfloat16: 8.5 us, with 64 lanes 19.3).  Few: a wave a token, whose lanes
  // have fewer logits to go through one after the other (1 x 256: 3.5 us, with
  // 16 lanes 6.5; 2048 x 256: 4.4 and 7.0; at 8192 x 256 they meet).
  const int w = a.experts <= 256 && a.k <= 16 && a.tokens > 4096 ? 16 : 64;
  int npl = 16;
  for (int n : kNpl)
    if (n * w >= a.experts) {
      npl = n;
      break;
    }
  const int es = esize(dt);
  auto dwords = [&](const void *p, size_t ld) { return aligned(p, 4) && ld * es % 4 == 0; };
  const bool vec = dwords(a.logits, a.ld) && dwords(a.dlogits, a.ldd);
  route_fn fn;
  if (w == 16)
    fn = dt == LL_F32 ? route_fn_of<float, 16>(npl, grad, vec) : route_fn_of<__bf16, 16>(npl, grad, vec);
  else
    fn = dt == LL_F32 ? route_fn_of<float, 64>(npl, grad, vec) : route_fn_of<__bf16, 64>(npl, grad, vec);
  const unsigned per = kThreads / w;
  hipLaunchKernelGGL(fn, dim3((a.tokens + per - 1) / per), dim3(kThreads), 0, (hipStream_t)stream, a);
  return launch_status();
}

// ---------------------------------------------------------------- sorting
constexpr size_t kSmallPairs = 1024;

// Pairs per block of a sort of `pairs` pairs (a multiple of 256).
uint32_t sort_chunk(size_t pairs) {
  if (pairs <= kSmallPairs) return (uint32_t)((std::max<size_t>(pairs, 1) + 255) / 256 * 256);
  uint32_t c = 1024;
  while (c < (1u << 20) && (pairs + c - 1) / c > 128) c *= 2;  // every block reads all blocks' counts
  return c;
}

using row_fn = void (*)(RowArgs);

// TPR and VEC of a launch over token rows: a wave a row up to 4 KiB.
struct RowShape {
  bool vec, wide;
  unsigned grid(uint32_t tokens) const {
    const unsigned per = wide ? 1 : kThreads / 64;
    return (tokens + per - 1) / per;
  }
};

RowShape row_shape(const RowArgs &a, int es) {
  RowShape s;
  s.vec = a.features * (size_t)es % 16 == 0 && vec16(a.x, a.ldx, es) && vec16(a.extra, a.lde, es) &&
          vec16(a.out, a.ldo, es);
  s.wide = (size_t)a.features * es > 4096;
  return s;
}

#define LL_ROW_KERNEL(K, T, s) \
  ((s).vec ? ((s).wide ? (row_fn)K<T, true, 256> : (row_fn)K<T, true, 64>) \
           : ((s).wide ? (row_fn)K<T, false, 256> : (row_fn)K<T, false, 64>))

}  // namespace

extern "C" {

int ll_moe_route(const void *logits, size_t ld, size_t tokens, int experts, int k, ll_dtype dt, const float *bias,
                 ll_score score, int normalise, float scale, int32_t *ids, float *weights, void *stream) {
  if (dt != LL_F32 && dt != LL_BF16) return LL_ERR_UNSUPPORTED;
  if (score != LL_SCORE_SOFTMAX && score != LL_SCORE_SIGMOID) return LL_ERR_INVALID;
  int st = check_choice(tokens, experts, k);
  if (st != LL_OK) return st;
  if (k > experts) return LL_ERR_INVALID;
  if (tokens == 0) return LL_OK;
  st = check_rows(logits, ld, (size_t)experts, esize(dt));
  if (st != LL_OK) return st;
  if (ids == nullptr || weights == nullptr || !aligned(ids, 4) || !aligned(weights, 4) || !aligned(bias, 4))
    return LL_ERR_INVALID;
  RouteArgs a{};
  a.logits = logits;
  a.ld = ld;
  a.tokens = (uint32_t)tokens;
  a.experts = experts;
  a.k = k;
  a.bias = bias;
  a.score = score;
  a.normalise = normalise != 0;
  a.scale = scale;
  a.ids = ids;
  a.weights = weights;
  return launch_route(a, dt, false, stream);
}

int ll_moe_route_grad(const void *logits, size_t ld, size_t tokens, int experts, int k, ll_dtype dt, ll_score score,
                      int normalise, float scale, const int32_t *ids, const float *dweights, void *dlogits,
                      size_t ldd, void *stream) {
  if (dt != LL_F32 && dt != LL_BF16) return LL_ERR_UNSUPPORTED;
  if (score != LL_SCORE_SOFTMAX && score != LL_SCORE_SIGMOID) return LL_ERR_INVALID;
  int st = check_choice(tokens, experts, k);
  if (st != LL_OK) return st;
  if (k > experts) return LL_ERR_INVALID;
  if (tokens == 0) return LL_OK;
  const int es = esize(dt);
  st = check_rows(logits, ld, (size_t)experts, es);
  if (st == LL_OK) st = check_rows(dlogits, ldd, (size_t)experts, es);
  if (st != LL_OK) return st;
  if (ids == nullptr || dweights == nullptr || !aligned(ids, 4) || !aligned(dweights, 4)) return LL_ERR_INVALID;
  if (overlap(logits, span(tokens, ld, experts, es), dlogits, span(tokens, ldd, experts, es))) return LL_ERR_INVALID;
  RouteArgs a{};
  a.logits = logits;
  a.ld = ld;
  a.tokens = (uint32_t)tokens;
  a.experts = experts;
  a.k = k;
  a.score = score;
  a.normalise = normalise != 0;
  a.scale = scale;
  a.ids = const_cast<int32_t *>(ids);
  a.dweights = dweights;
  a.dlogits = dlogits;
  a.ldd = ldd;
  return launch_route(a, dt, true, stream);
}

int ll_moe_dispatch_bytes(size_t tokens, int k, int experts, size_t *bytes) {
  if (bytes == nullptr) return LL_ERR_INVALID;
  const int st = check_choice(tokens, experts, k);
  if (st != LL_OK) return st;
  const size_t pairs = tokens * (size_t)k;
  const size_t chunk = sort_chunk(pairs);
  *bytes = pairs <= kSmallPairs ? 0 : (pairs + chunk - 1) / chunk * (size_t)experts * 4;
  return LL_OK;
}

int ll_moe_dispatch(const int32_t *ids, size_t tokens, int k, int first, int experts, const void *x, size_t ldx,
                    size_t features, ll_dtype dt, int32_t *offsets, int32_t *slots, int32_t *rows, void *y, size_t ldy,
                    void *workspace, size_t workspace_bytes, void *stream) {
  if (dt != LL_F32 && dt != LL_BF16) return LL_ERR_UNSUPPORTED;
  if (first < 0) return LL_ERR_INVALID;
  size_t need = 0;
  int st = ll_moe_dispatch_bytes(tokens, k, experts, &need);
  if (st != LL_OK) return st;
  if (offsets == nullptr) return LL_ERR_INVALID;
  if (tokens != 0 && (ids == nullptr || slots == nullptr || rows == nullptr)) return LL_ERR_INVALID;
  if (!aligned(ids, 4) || !aligned(offsets, 4) || !aligned(slots, 4) || !aligned(rows, 4)) return LL_ERR_INVALID;
  const int es = esize(dt);
  const size_t pairs = tokens * (size_t)k;
  if (tokens == 0) x = y = nullptr;
  if ((x == nullptr) != (y == nullptr)) return LL_ERR_INVALID;
  if (x != nullptr) {
    if (features > kMaxExtent) return LL_ERR_UNSUPPORTED;
    st = check_rows(x, ldx, features, es);
    if (st == LL_OK) st = check_rows(y, ldy, features, es);
    if (st != LL_OK) return st;
  }
  if (need != 0) {
    if (workspace == nullptr || !aligned(workspace, 4)) return LL_ERR_INVALID;
    if (workspace_bytes < need) return LL_ERR_SCRATCH;
  }
  // Places come from ids that are read twice, and rows of y from places: an
  // array written over another could send rows anywhere.
  const struct {
    const void *p;
    size_t bytes;
  } arrays[] = {{ids, pairs * 4},
                {x, span(tokens, ldx, features, es)},  // the inputs first, then what is written
                {y, span(pairs, ldy, features, es)},
                {offsets, ((size_t)experts + 1) * 4},
                {slots, pairs * 4},
                {rows, pairs * 4},
                {workspace, need}};
  for (int i = 2; i < 7; ++i)
    for (int j = 0; j < i; ++j)
      if (overlap(arrays[i].p, arrays[i].bytes, arrays[j].p, arrays[j].bytes)) return LL_ERR_INVALID;
  SortArgs s{};
  s.ids = ids;
  s.pairs = (uint32_t)pairs;
  s.chunk = sort_chunk(pairs);
  s.blocks = (uint32_t)std::max<size_t>(1, (pairs + s.chunk - 1) / s.chunk);
  s.first = first;
  s.experts = experts;
  while ((1 << s.bits) < experts) ++s.bits;
  s.offsets = offsets;
  s.slots = slots;
  s.rows = rows;
  s.hist = need == 0 ? nullptr : (int32_t *)workspace;
  RowArgs a{};
  a.x = features == 0 ? nullptr : x;
  a.ldx = ldx;
  a.out = y;
  a.ldo = ldy;
  a.rows = rows;
  a.tokens = (uint32_t)tokens;
  a.k = k;
  a.features = (uint32_t)features;
  const RowShape shape = row_shape(a, es);
  const size_t lds = (size_t)kSortInts * experts * 4;
  if (pairs <= kSmallPairs) {
    const unsigned grid = a.x == nullptr ? 1 : std::max(1u, a.tokens);
    const auto fn = dt == LL_F32 ? (shape.vec ? k_dispatch_small<float, true> : k_dispatch_small<float, false>)
                                 : (shape.vec ? k_dispatch_small<__bf16, true> : k_dispatch_small<__bf16, false>);
    hipLaunchKernelGGL(fn, dim3(grid), dim3(kThreads), lds + (size_t)k * 4, (hipStream_t)stream, s, a);
    return launch_status();
  }
  hipLaunchKernelGGL(k_sort_count, dim3(s.blocks), dim3(kThreads), (size_t)experts * 4, (hipStream_t)stream, s);
  hipLaunchKernelGGL(k_sort_place, dim3(s.blocks), dim3(kThreads), lds, (hipStream_t)stream, s);
  if (a.x != nullptr) {
    const row_fn fn = dt == LL_F32 ? LL_ROW_KERNEL(k_push, float, shape) : LL_ROW_KERNEL(k_push, __bf16, shape);
    hipLaunchKernelGGL(fn, dim3(shape.grid(a.tokens)), dim3(kThreads), 0, (hipStream_t)stream, a);
  }
  return launch_status();
}

int ll_moe_combine(const void *y, size_t ldy, size_t nrows, const int32_t *rows, const float *weights,
                   const void *residual, size_t ldr, size_t tokens, int k, size_t features, ll_dtype dt, void *out,
                   size_t ldo, void *stream) {
  if (dt != LL_F32 && dt != LL_BF16) return LL_ERR_UNSUPPORTED;
  int st = check_choice(tokens, 1, k);
  if (st != LL_OK) return st;
  if (features > kMaxExtent || nrows > kMaxExtent) return LL_ERR_UNSUPPORTED;
  if (tokens == 0 || features == 0) return LL_OK;
  const int es = esize(dt);
  if (nrows != 0) st = check_rows(y, ldy, features, es);
  if (st == LL_OK) st = check_rows(out, ldo, features, es);
  if (st == LL_OK && residual != nullptr) st = check_rows(residual, ldr, features, es);
  if (st != LL_OK) return st;
  if (rows == nullptr || !aligned(rows, 4) || !aligned(weights, 4)) return LL_ERR_INVALID;
  const size_t out_bytes = span(tokens, ldo, features, es);
  if (overlap(y, span(nrows, ldy, features, es), out, out_bytes)) return LL_ERR_INVALID;
  if (overlap(residual, span(tokens, ldr, features, es), out, out_bytes) && !(residual == out && ldr == ldo))
    return LL_ERR_INVALID;
  RowArgs a{};
  a.x = y;
  a.ldx = ldy;
  a.extra = residual;
  a.lde = ldr;
  a.out = out;
  a.ldo = ldo;
  a.rows = rows;
  a.weights = weights;
  a.tokens = (uint32_t)tokens;
  a.nrows = (uint32_t)nrows;
  a.k = k;
  a.features = (uint32_t)features;
  const RowShape s = row_shape(a, es);
  const row_fn fn = dt == LL_F32 ? LL_ROW_KERNEL(k_combine, float, s) : LL_ROW_KERNEL(k_combine, __bf16, s);
  hipLaunchKernelGGL(fn, dim3(s.grid(a.tokens)), dim3(kThreads), 0, (hipStream_t)stream, a);
  return launch_status();
}

int ll_moe_combine_grad(const void *dout, size_t ldd, const void *y, size_t ldy, size_t nrows, const int32_t *rows,
                        const float *weights, size_t tokens, int k, size_t features, ll_dtype dt, void *dy,
                        size_t lddy, float *dweights, void *stream) {
  if (dt != LL_F32 && dt != LL_BF16) return LL_ERR_UNSUPPORTED;
  int st = check_choice(tokens, 1, k);
  if (st != LL_OK) return st;
  if (features > kMaxExtent || nrows > kMaxExtent) return LL_ERR_UNSUPPORTED;
  if (tokens == 0) return LL_OK;
  const int es = esize(dt);
  if (features != 0) {  // else the weights' gradient alone is left, zeros
    st = check_rows(dout, ldd, features, es);
    if (st == LL_OK && nrows != 0) st = check_rows(dy, lddy, features, es);
    if (st == LL_OK && nrows != 0 && dweights != nullptr) st = check_rows(y, ldy, features, es);
    if (st != LL_OK) return st;
    const size_t dy_bytes = span(nrows, lddy, features, es);
    if (overlap(dout, span(tokens, ldd, features, es), dy, dy_bytes) ||
        (dweights != nullptr && overlap(y, span(nrows, ldy, features, es), dy, dy_bytes)))
      return LL_ERR_INVALID;
  }
  if (rows == nullptr || !aligned(rows, 4) || !aligned(weights, 4) || !aligned(dweights, 4)) return LL_ERR_INVALID;
  if (features == 0 && dweights == nullptr) return LL_OK;
  RowArgs a{};
  a.x = dweights == nullptr ? nullptr : y;
  a.ldx = ldy;
  a.extra = dout;
  a.lde = ldd;
  a.out = dy;
  a.ldo = lddy;
  a.rows = rows;
  a.weights = weights;
  a.dweights = dweights;
  a.tokens = (uint32_t)tokens;
  a.nrows = (uint32_t)nrows;
  a.k = k;
  a.features = (uint32_t)features;
  const RowShape s = row_shape(a, es);
  const row_fn fn =
      dt == LL_F32 ? LL_ROW_KERNEL(k_combine_grad, float, s) : LL_ROW_KERNEL(k_combine_grad, __bf16, s);
  hipLaunchKernelGGL(fn, dim3(s.grid(a.tokens)), dim3(kThreads), 0, (hipStream_t)stream, a);
  return launch_status();
}

}  // extern "C"
