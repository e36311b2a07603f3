// 8-bit rows and weights, norms and the weight update: entry points of
// include/llblock.h.  Arguments are checked before any HIP call.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "../../include/llblock.h"
#include "ll_block.hpp"
#include "ll_host.hpp"

using namespace llc;
using namespace llc::blk;

namespace {

constexpr size_t kMaxExtent = 0x7fffffff;

int esize(ll_dtype dt) { return dt == LL_F32 ? 4 : 2; }
bool known(ll_dtype dt) { return dt == LL_F32 || dt == LL_BF16; }
bool aligned(const void *p, size_t to) { return (uintptr_t)p % to == 0; }
bool overlap(const void *a, size_t an, const void *b, size_t bn) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return a != nullptr && b != nullptr && an != 0 && bn != 0 && x < y + bn && y < x + an;
}
size_t span(size_t rows, size_t ld, size_t len, size_t es) {
  return rows == 0 || len == 0 ? 0 : ((rows - 1) * ld + len) * es;
}
size_t blocks_of(size_t n) { return (n + LL_BLOCK - 1) / LL_BLOCK; }

int check_scales(const uint8_t *p, size_t ld, size_t blocks) {
  if (p == nullptr || !aligned(p, 4) || ld % 4 != 0 || ld < blocks) return LL_ERR_INVALID;
  return ld > kMaxExtent ? LL_ERR_UNSUPPORTED : LL_OK;
}

template <typename T>
int launch_quantise(const QuantArgs &a, uint64_t items, void *stream) {
  // Many rows: two blocks of a lane's loads under way.  Few: as many waves as there are blocks.
  const bool many = items >= 65536;
  const uint64_t per = many ? 32 : 16;
  const uint64_t grid = (items + per - 1) / per;
  if (grid * 256 >= 1ull << 32) return LL_ERR_UNSUPPORTED;
  hipLaunchKernelGGL((many ? k_quantise<T, 2> : k_quantise<T, 1>), dim3((unsigned)grid), dim3(256), 0, (hipStream_t)stream, a);
  return launch_status();
}

template <typename T>
void launch_weight(const WeightArgs &a, bool transpose, dim3 grid, void *stream) {
  hipLaunchKernelGGL((transpose ? k_quantise_weight<T, true> : k_quantise_weight<T, false>), grid, dim3(256), 0, (hipStream_t)stream, a);
}

// ---------------------------------------------------------------- norms
using norm_fn = void (*)(NormArgs);

template <typename T, bool GRAD, int TPR, int C>
norm_fn norm_of() {
  if constexpr (GRAD)
    return k_norm_grad<T, TPR, C>;
  else
    return k_norm<T, TPR, C>;
}

// Threads a row, its chunks a thread, and rows a workgroup takes at a time.
struct NormShape {
  uint32_t tpr, chunks, rows;
};

NormShape norm_shape(size_t features) {
  if (features <= 512) return {64, 1, 4};
  if (features > 8192) return {1024, 2, 1};
  uint32_t tpr = 128;
  while (tpr * kW < features) tpr *= 2;
  return {tpr, 1, 1};
}

template <typename T, bool GRAD>
norm_fn pick_norm(const NormShape &s) {
  switch (s.tpr * s.chunks) {
    case 64: return norm_of<T, GRAD, 64, 1>();
    case 128: return norm_of<T, GRAD, 128, 1>();
    case 256: return norm_of<T, GRAD, 256, 1>();
    case 512: return norm_of<T, GRAD, 512, 1>();
    case 1024: return norm_of<T, GRAD, 1024, 1>();
    default: return norm_of<T, GRAD, 1024, 2>();
  }
}

// Workgroups of the gradient's launch, whose shares of dweight and dpost are
// added up afterwards: as many as the chip holds at a time, but 512 of 256 threads
// (16384 x 2048 bfloat16: 53.6 us, with 1024 59.1).
uint32_t grad_grid(const NormShape &s, size_t rows) {
  const size_t most = s.tpr == 1024 ? 256 : s.tpr == 128 ? 1024 : 512;
  return (uint32_t)std::min<size_t>((rows + s.rows - 1) / s.rows, most);
}

int check_norm(const ll_norm_desc *d) {
  if (d == nullptr || d->size != sizeof(ll_norm_desc)) return LL_ERR_INVALID;
  if (!known(d->dt) || !known(d->wdt)) return LL_ERR_UNSUPPORTED;
  if (d->wdt != d->dt && d->wdt != LL_F32) return LL_ERR_UNSUPPORTED;
  if (!(d->eps > 0.f)) return LL_ERR_INVALID;
  if (d->features < 1) return LL_ERR_INVALID;
  if (d->features > LL_NORM_MAX_FEATURES || d->rows > kMaxExtent) return LL_ERR_UNSUPPORTED;
  for (size_t ld : {d->ldy, d->ldx, d->ldr, d->ldh, d->ldq, d->lds, d->ldd, d->ldo, d->lddy})
    if (ld > kMaxExtent) return LL_ERR_UNSUPPORTED;
  return LL_OK;
}

// A matrix of rows that may be NULL.
bool good(const ll_norm_desc *d, const void *p, size_t ld) {
  return p == nullptr || (aligned(p, esize(d->dt)) && ld >= d->features);
}

struct Range {
  const void *p;
  size_t bytes, ld;
};
// Whether two arrays share memory otherwise than by being the same rows.
bool clash(const Range &a, const Range &b, bool same_allowed) {
  if (!overlap(a.p, a.bytes, b.p, b.bytes)) return false;
  return !(same_allowed && a.p == b.p && a.ld == b.ld);
}

}  // namespace

extern "C" {

int ll_quantise(const void *x, size_t ldx, size_t rows, const int32_t *end, size_t features, ll_dtype dt, ll_act act,
                uint8_t *q, size_t ldq, uint8_t *scales, size_t lds, void *stream) {
  if (!known(dt)) return LL_ERR_UNSUPPORTED;
  if ((int)act < LL_ACT_NONE || (int)act > LL_ACT_GEGLU || !aligned(end, 4)) return LL_ERR_INVALID;
  if (rows > kMaxExtent || features > kMaxExtent / 2 || ldx > kMaxExtent || ldq > kMaxExtent) return LL_ERR_UNSUPPORTED;
  if (rows == 0 || features == 0) return LL_OK;
  const size_t es = esize(dt), width = lin::gated((int)act) ? 2 * features : features;
  if (x == nullptr || !aligned(x, es) || ldx < width || q == nullptr || ldq < features) return LL_ERR_INVALID;
  const int st = check_scales(scales, lds, blocks_of(features));
  if (st != LL_OK) return st;
  const size_t xb = span(rows, ldx, width, es), qb = span(rows, ldq, features, 1), sb = span(rows, lds, blocks_of(features), 1);
  if (overlap(x, xb, q, qb) || overlap(x, xb, scales, sb) || overlap(q, qb, scales, sb) || overlap(end, 4, q, qb) ||
      overlap(end, 4, scales, sb))
    return LL_ERR_INVALID;
  QuantArgs a{x, q, scales, end, ldx, ldq, lds, (uint32_t)rows, (uint32_t)features, (uint32_t)blocks_of(features), (int)act};
  const uint64_t items = (uint64_t)rows * a.blocks;
  return dt == LL_F32 ? launch_quantise<float>(a, items, stream) : launch_quantise<__bf16>(a, items, stream);
}

int ll_quantise_weight(const void *w, size_t ldw, size_t wstride, int groups, size_t out, size_t in, ll_dtype dt,
                       int transpose, uint8_t *q, size_t ldq, size_t qstride, uint8_t *scales, size_t lds,
                       size_t sstride, void *stream) {
  if (!known(dt)) return LL_ERR_UNSUPPORTED;
  if (groups < 1 || out < 1 || in < 1) return LL_ERR_INVALID;
  constexpr size_t kMaxFeatures = 1u << 20;
  if (groups > LL_MOE_MAX_EXPERTS || out > kMaxFeatures || in > kMaxFeatures) return LL_ERR_UNSUPPORTED;
  if (ldw > kMaxExtent || ldq > kMaxExtent) return LL_ERR_UNSUPPORTED;
  const size_t es = esize(dt), qr = transpose ? in : out, qc = transpose ? out : in;
  const size_t sr = blocks_of(qr), sc = blocks_of(qc);
  if (w == nullptr || !aligned(w, es) || ldw < in || q == nullptr || ldq < qc) return LL_ERR_INVALID;
  const int st = check_scales(scales, lds, sc);
  if (st != LL_OK) return st;
  if (groups > 1 && (wstride < (out - 1) * ldw + in || qstride < (qr - 1) * ldq + qc || sstride < (sr - 1) * lds + sc ||
                     sstride % 4 != 0))
    return LL_ERR_INVALID;
  auto all = [&](size_t stride, size_t one) { return (groups - 1) * stride + one; };
  const size_t wb = all(wstride, (out - 1) * ldw + in) * es, qb = all(qstride, (qr - 1) * ldq + qc);
  const size_t sb = all(sstride, (sr - 1) * lds + sc);
  if (overlap(w, wb, q, qb) || overlap(w, wb, scales, sb) || overlap(q, qb, scales, sb)) return LL_ERR_INVALID;
  const WeightArgs a{w, q, scales, ldw, wstride, ldq, qstride, lds, sstride, (uint32_t)out, (uint32_t)in};
  const dim3 grid((unsigned)blocks_of(in), (unsigned)blocks_of(out), (unsigned)groups);
  if (dt == LL_F32)
    launch_weight<float>(a, transpose != 0, grid, stream);
  else
    launch_weight<__bf16>(a, transpose != 0, grid, stream);
  return launch_status();
}

int ll_norm_desc_init(ll_norm_desc *d, ll_dtype dt, ll_dtype wdt, size_t rows, size_t features, float eps,
                      float scale) {
  if (d == nullptr) return LL_ERR_INVALID;
  *d = ll_norm_desc{};
  d->size = sizeof(ll_norm_desc);
  d->dt = dt;
  d->wdt = wdt;
  d->eps = eps;
  d->scale = scale;
  d->rows = rows;
  d->features = features;
  d->ldy = d->ldx = d->ldr = d->ldh = d->ldq = d->ldd = d->ldo = d->lddy = features;
  d->lds = (blocks_of(features) + 3) / 4 * 4;
  return LL_OK;
}

int ll_norm(const ll_norm_desc *d, const void *y, const void *x, const float *gate, const void *post,
            const void *weight, void *r, void *h, uint8_t *q, uint8_t *scales, void *stream) {
  const int st = check_norm(d);
  if (st != LL_OK) return st;
  if ((h != nullptr || q != nullptr) && weight == nullptr) return LL_ERR_INVALID;
  if (!good(d, y, d->ldy) || !good(d, x, d->ldx) || !good(d, r, d->ldr) || !good(d, h, d->ldh)) return LL_ERR_INVALID;
  const size_t es = esize(d->dt), ws = esize(d->wdt), n = d->rows, f = d->features;
  if (!aligned(gate, 4) || !aligned(post, ws) || !aligned(weight, ws)) return LL_ERR_INVALID;
  if (q != nullptr) {
    if (d->ldq < f) return LL_ERR_INVALID;
    const int sst = check_scales(scales, d->lds, blocks_of(f));
    if (sst != LL_OK) return sst;
  }
  if (n == 0) return LL_OK;
  if (y == nullptr) return LL_ERR_INVALID;
  const Range outs[] = {{r, span(n, d->ldr, f, es), d->ldr},
                        {h, span(n, d->ldh, f, es), d->ldh},
                        {q, span(n, d->ldq, f, 1), d->ldq},
                        {q != nullptr ? scales : nullptr, span(n, d->lds, blocks_of(f), 1), d->lds}};
  const Range ins[] = {{y, span(n, d->ldy, f, es), d->ldy},
                       {x, span(n, d->ldx, f, es), d->ldx},
                       {gate, n * 4, 1},
                       {post, f * ws, 1},
                       {weight, f * ws, 1}};
  for (int o = 0; o < 4; ++o) {
    for (int p = o + 1; p < 4; ++p)
      if (clash(outs[o], outs[p], false)) return LL_ERR_INVALID;
    for (int i = 0; i < 5; ++i)
      if (clash(outs[o], ins[i], (o == 0 && i < 2) || (o == 1 && i == 0))) return LL_ERR_INVALID;
  }
  if (r == nullptr && h == nullptr && q == nullptr) return LL_OK;
  NormArgs a{};
  a.y = y;
  a.x = x;
  a.gate = gate;
  a.post = post;
  a.weight = h != nullptr || q != nullptr ? weight : nullptr;
  a.r = r;
  a.h = h;
  a.q = q;
  a.scales = scales;
  a.ldy = d->ldy;
  a.ldx = d->ldx;
  a.ldr = d->ldr;
  a.ldh = d->ldh;
  a.ldq = d->ldq;
  a.lds = d->lds;
  a.rows = (uint32_t)n;
  a.features = (uint32_t)f;
  a.eps = d->eps;
  a.scale = d->scale;
  a.w32 = d->wdt == LL_F32;
  const NormShape s = norm_shape(f);
  const norm_fn fn = d->dt == LL_F32 ? pick_norm<float, false>(s) : pick_norm<__bf16, false>(s);
  const uint32_t threads = norm_threads(s.tpr);
  const uint64_t grid = (n + s.rows - 1) / s.rows;
  if (grid * threads >= 1ull << 32) return LL_ERR_UNSUPPORTED;
  hipLaunchKernelGGL(fn, dim3((unsigned)grid), dim3(threads), 0, (hipStream_t)stream, a);
  return launch_status();
}

int ll_norm_bytes(const ll_norm_desc *d, size_t *bytes) {
  if (bytes == nullptr) return LL_ERR_INVALID;
  const int st = check_norm(d);
  if (st != LL_OK) return st;
  const NormShape s = norm_shape(d->features);
  *bytes = (size_t)2 * grad_grid(s, d->rows) * d->features * 4;
  return LL_OK;
}

int ll_norm_grad(const ll_norm_desc *d, const void *dh, const void *r, const void *dr, const void *y,
                 const float *gate, const void *post, const void *weight, void *dr_out, void *dy, float *dgate,
                 float *dweight, float *dpost, uint32_t flags, void *workspace, size_t workspace_bytes,
                 void *stream) {
  size_t need = 0;
  const int st = ll_norm_bytes(d, &need);
  if (st != LL_OK) return st;
  if ((flags & ~LL_GRAD_ADD) != 0) return LL_ERR_INVALID;
  const size_t es = esize(d->dt), ws = esize(d->wdt), n = d->rows, f = d->features;
  if (weight == nullptr ? dh != nullptr || dweight != nullptr : n != 0 && (dh == nullptr || r == nullptr)) return LL_ERR_INVALID;
  if (dpost != nullptr && post == nullptr) return LL_ERR_INVALID;
  if (n != 0 && y == nullptr && (dgate != nullptr || (post != nullptr && (dy != nullptr || dpost != nullptr)))) return LL_ERR_INVALID;
  if (!good(d, dh, d->ldh) || !good(d, r, d->ldr) || !good(d, dr, d->ldd) || !good(d, y, d->ldy) ||
      !good(d, dr_out, d->ldo) || !good(d, dy, d->lddy))
    return LL_ERR_INVALID;
  if (!aligned(gate, 4) || !aligned(post, ws) || !aligned(weight, ws) || !aligned(dgate, 4) || !aligned(dweight, 4) ||
      !aligned(dpost, 4) || !aligned(workspace, 16))
    return LL_ERR_INVALID;
  const bool sums = dweight != nullptr || dpost != nullptr;
  const Range outs[] = {{dr_out, span(n, d->ldo, f, es), d->ldo},
                        {dy, span(n, d->lddy, f, es), d->lddy},
                        {dgate, n * 4, 1},
                        {dweight, f * 4, 1},
                        {dpost, f * 4, 1},
                        {sums && n != 0 ? workspace : nullptr, need, 1}};
  const Range ins[] = {{dr, span(n, d->ldd, f, es), d->ldd}, {y, span(n, d->ldy, f, es), d->ldy},
                       {dh, span(n, d->ldh, f, es), d->ldh}, {r, span(n, d->ldr, f, es), d->ldr},
                       {gate, n * 4, 1},                     {post, f * ws, 1},
                       {weight, f * ws, 1}};
  for (int o = 0; o < 6; ++o) {
    for (int p = o + 1; p < 6; ++p)
      if (clash(outs[o], outs[p], false)) return LL_ERR_INVALID;
    for (int i = 0; i < 7; ++i)
      if (clash(outs[o], ins[i], o == i && o < 2)) return LL_ERR_INVALID;
  }
  if (sums && n != 0 && (workspace == nullptr || workspace_bytes < need)) return LL_ERR_SCRATCH;
  NormArgs a{};
  a.y = post != nullptr && dy == nullptr && dpost == nullptr && dgate == nullptr ? nullptr : y;
  a.gate = gate;
  a.post = dy != nullptr || dpost != nullptr || dgate != nullptr ? post : nullptr;
  a.weight = weight;
  a.r = const_cast<void *>(r);
  a.dh = dh;
  a.dr = dr;
  a.dr_out = dr_out;
  a.dy = dy;
  a.dgate = dgate;
  a.parts = sums ? (float *)workspace : nullptr;
  a.ldy = d->ldy;
  a.ldr = d->ldr;
  a.ldh = d->ldh;
  a.ldd = d->ldd;
  a.ldo = d->ldo;
  a.lddy = d->lddy;
  a.rows = (uint32_t)n;
  a.features = (uint32_t)f;
  a.eps = d->eps;
  a.scale = d->scale;
  a.w32 = d->wdt == LL_F32;
  const NormShape s = norm_shape(f);
  const uint32_t grid = grad_grid(s, n);
  if (n != 0 && (sums || dr_out != nullptr || dy != nullptr || dgate != nullptr)) {
    const norm_fn fn = d->dt == LL_F32 ? pick_norm<float, true>(s) : pick_norm<__bf16, true>(s);
    hipLaunchKernelGGL(fn, dim3(grid), dim3(norm_threads(s.tpr)), 0, (hipStream_t)stream, a);
    const int lst = launch_status();
    if (lst != LL_OK) return lst;
  }
  if (!sums) return LL_OK;
  const NormJoin j{(const float *)workspace, {dweight, dpost}, n == 0 ? 0 : grid, (uint32_t)f, (flags & LL_GRAD_ADD) != 0};
  hipLaunchKernelGGL(k_norm_join, dim3((unsigned)((f + 63) / 64), dpost != nullptr ? 2 : 1), dim3(64 * kJoin), 0,
                     (hipStream_t)stream, j);
  return launch_status();
}

int ll_adamw(const ll_adamw_desc *d, const ll_adamw_tensor *tensors, size_t count, int32_t *step, const float *lr_ptr,
             const float *grad_scale, void *workspace, size_t workspace_bytes, void *stream) {
  if (d == nullptr || d->size != sizeof(ll_adamw_desc)) return LL_ERR_INVALID;
  const bool floor = d->bits == (8 | LL_ADAMW_FLOOR), eight = floor || d->bits == 8;
  if (!eight && d->bits != 32) return LL_ERR_INVALID;
  // (written so that NaN is refused)
  if (!(d->beta1 >= 0. && d->beta1 < 1.) || !(d->beta2 >= 0. && d->beta2 < 1.) || !((float)d->eps > 0.f) || !(d->decay >= 0.) ||
      !(d->lr >= 0.))
    return LL_ERR_INVALID;
  if ((count != 0 && tensors == nullptr) || step == nullptr || !aligned(step, 4) || !aligned(lr_ptr, 4) ||
      !aligned(grad_scale, 4) || workspace == nullptr || !aligned(workspace, 16))
    return LL_ERR_INVALID;
  static_assert(sizeof(AdamwCoef) <= LL_ADAMW_WORKSPACE, "the coefficients");
  if (workspace_bytes < LL_ADAMW_WORKSPACE) return LL_ERR_SCRATCH;
  for (size_t i = 0; i < count; ++i) {
    const ll_adamw_tensor &t = tensors[i];
    if (!known(t.dt) || !known(t.gdt)) return LL_ERR_UNSUPPORTED;
    if (t.n == 0) continue;
    if (t.n > (size_t)1 << 40) return LL_ERR_UNSUPPORTED;
    if (t.param == nullptr || t.grad == nullptr || t.m == nullptr || t.v == nullptr) return LL_ERR_INVALID;
    if ((t.dt == LL_BF16) != (t.master != nullptr) || eight != (t.m_scales != nullptr) || eight != (t.v_scales != nullptr))
      return LL_ERR_INVALID;
    if (!aligned(t.param, esize(t.dt)) || !aligned(t.grad, esize(t.gdt)) || !aligned(t.master, 4)) return LL_ERR_INVALID;
    if (!eight && (!aligned(t.m, 4) || !aligned(t.v, 4))) return LL_ERR_INVALID;
  }
  AdamwBegin b{step, lr_ptr, grad_scale, (AdamwCoef *)workspace, d->lr, log2(d->beta1), log2(d->beta2), d->decay, d->seed};
  hipLaunchKernelGGL(k_adamw_begin, dim3(1), dim3(64), 0, (hipStream_t)stream, b);
  int st = launch_status();
  AdamwArgs a{};
  a.coef = (const AdamwCoef *)workspace;
  a.beta1 = (float)d->beta1;
  a.rest1 = (float)(1. - d->beta1);
  a.beta2 = (float)d->beta2;
  a.rest2 = (float)(1. - d->beta2);
  a.eps = (float)d->eps;
  uint32_t chunks = 0;
  auto launch = [&]() {
    hipLaunchKernelGGL((floor ? k_adamw<true, true> : eight ? k_adamw<true, false> : k_adamw<false, false>), dim3(chunks), dim3(256), 0, (hipStream_t)stream, a);
    a.count = chunks = 0;
    return launch_status();
  };
  constexpr uint32_t kMostChunks = 1u << 23;  // of a launch
  for (size_t i = 0; i < count && st == LL_OK; ++i) {
    ll_adamw_tensor t = tensors[i];
    while (t.n != 0 && st == LL_OK) {
      // (a tensor of more values than a launch has threads for goes in parts)
      const size_t most = (size_t)kMostChunks * kChunk, n = std::min(t.n, most);
      const uint32_t mine = (uint32_t)((n + kChunk - 1) / kChunk);
      if (a.count == kTensors || chunks + mine > kMostChunks) st = launch();
      if (st != LL_OK) break;
      AdamwTensor &k = a.t[a.count++];
      k = AdamwTensor{t.param, t.grad, t.master, t.m, t.v, t.m_scales, t.v_scales, n, t.at, chunks, 0};
      if (t.dt == LL_BF16) k.kind |= kBf16;
      if (t.gdt == LL_BF16) k.kind |= kGradBf16;
      chunks += mine;
      t.n -= n;
      t.at += n;
      t.param = (char *)t.param + n * esize(t.dt);
      t.grad = (const char *)t.grad + n * esize(t.gdt);
      if (t.master != nullptr) t.master += n;
      t.m = (char *)t.m + n * (eight ? 1 : 4);
      t.v = (char *)t.v + n * (eight ? 1 : 4);
      if (eight) {
        t.m_scales += n / LL_BLOCK;
        t.v_scales += n / LL_BLOCK;
      }
    }
  }
  if (st == LL_OK && a.count != 0) st = launch();
  return st;
}

}  // extern "C"
