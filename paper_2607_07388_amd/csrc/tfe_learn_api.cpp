// C ABI of the calls that learn the head from tokens and serve it in integers:
// cross entropy, gradient norm and clipping, the integer product.  Host checks
// only; no device memory is allocated and no state kept.
#include <hip/hip_runtime_api.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <memory>
#include <new>

#include "../../include/tfe.h"
#include "tfe_checks.h"
#include "tfe_internal.h"
#include "tfe_learn.h"
#include "tfe_logits.h"

namespace tfe {
namespace {

// ---- cross entropy ---------------------------------------------------------------

tfe_status xent_sizes(int64_t rows, int32_t vocab, int32_t dim) {
  NEED(rows >= 0 && rows <= kLogitsMaxRows, "rows outside [0, 2^20]");
  NEED(vocab >= 1 && vocab <= kLogitsMaxVocab, "vocab outside [1, 2^18]");
  NEED(dim >= 1 && dim <= kXentMaxDim, "dim outside [1, %d]", kXentMaxDim);
  return TFE_OK;
}

tfe_status xent_args(const void* hidden, int64_t ldh, const void* w, int64_t ldw,
                     const int32_t* targets, int64_t rows, int32_t vocab, int32_t dim,
                     void* workspace, int64_t bytes, XentArgs* a) {
  TRY(xent_sizes(rows, vocab, dim));
  TRY(matrix(hidden, TFE_BF16, ldh, rows, dim, "hidden"));
  TRY(matrix(w, TFE_BF16, ldw, vocab, dim, "w"));
  if (rows == 0) return TFE_OK;
  NEED(targets && aligned(targets, 4), "targets: null or not aligned");
  TRY(space(workspace, bytes, xent_space(rows, vocab, dim)));
  a->hidden = (const uint16_t*)hidden;
  a->ldh = ldh;
  a->w = (const uint16_t*)w;
  a->ldw = ldw;
  a->targets = targets;
  a->rows = (uint32_t)rows;
  a->vocab = (uint32_t)vocab;
  a->dim = (uint32_t)dim;
  a->space = (unsigned char*)workspace;
  return TFE_OK;
}

tfe_status xent_grads(int64_t rows, int32_t vocab, int32_t dim, const void* hidden, const void* w,
                      const float* weight, void* gx, int64_t ldgx, void* gw, int64_t ldgw,
                      int32_t dtype, int32_t accumulate, XentArgs* a) {
  TRY(matrix(gx, dtype, ldgx, rows, dim, "grad_hidden"));
  TRY(matrix(gw, dtype, ldgw, vocab, dim, "grad_w"));
  NEED(!accumulate || dtype == TFE_F32, "accumulate needs float32 gradients");
  NEED(gw != w && gw != hidden && gw != gx && gx != w && (gx != hidden || !gx),
       "a gradient in the place of another argument");
  NEED(aligned(weight, 4), "grad_loss: not aligned");
  a->weight = weight;
  a->gx = gx;
  a->ldgx = ldgx;
  a->gw = gw;
  a->ldgw = ldgw;
  a->gdtype = dtype;
  a->accumulate = accumulate != 0;
  a->vocab = (uint32_t)vocab;
  a->dim = (uint32_t)dim;
  return TFE_OK;
}

// ---- gradient norm ---------------------------------------------------------------

tfe_status grad_tensors(const tfe_grad_tensor* t, int64_t n, bool out) {
  NEED(n >= 0 && n <= 1 << 20, "tensors outside [0, 2^20]");
  NEED(t || n == 0, "null tensors");
  for (int64_t k = 0; k < n; ++k) {
    const tfe_grad_tensor& g = t[k];
    NEED(g.rows >= 0 && g.cols >= 0 && g.rows < (int64_t)1 << 31 && g.cols < (int64_t)1 << 40 &&
             (g.rows == 1 || g.cols < (int64_t)1 << 31),
         "tensor %lld: rows outside [0, 2^31) or cols outside [0, 2^31) (2^40 for one row)", (long long)k);
    NEED((double)g.rows * (double)g.cols <= (double)((int64_t)1 << 40), "tensor %lld: above 2^40 elements",
         (long long)k);
    const bool none = g.rows == 0 || g.cols == 0;
    // A single row has no pitch to keep.
    const int64_t rows = none ? 0 : g.rows;
    TRY(matrix(g.grad, g.dtype, g.rows == 1 ? 0 : g.ldg, rows, g.rows == 1 ? 0 : g.cols, "gradient"));
    if (!out) continue;
    TRY(matrix(g.out, g.dtype, g.rows == 1 ? 0 : g.ldo, rows, g.rows == 1 ? 0 : g.cols, "clipped gradient"));
    NEED(none || g.rows == 1 || g.grad != g.out || g.ldg == g.ldo, "tensor %lld: in place at another pitch",
         (long long)k);
  }
  return TFE_OK;
}

// The bytes of a clipped gradient or a gradient that surely are its own: of rows apart, between
// which other tensors may lie (columns of one matrix), the first.
struct Range {
  uintptr_t from, to;
  int64_t tensor;
};
Range range_of(const tfe_grad_tensor& g, const void* p, int64_t ld, int64_t k) {
  const bool whole = g.rows == 1 || ld == g.cols;
  return Range{(uintptr_t)p, (uintptr_t)p + (whole ? g.rows * g.cols : g.cols) * elem(g.dtype), k};
}

// Clipped gradients lie apart from each other and from every gradient but their own, which they
// are as a whole or not at all: blocks read and write them in no order.
tfe_status grad_places(const tfe_grad_tensor* t, int64_t n) {
  constexpr int64_t kNear = 512;
  Range near[kNear];
  std::unique_ptr<Range[]> many;
  if (n > kNear) {
    many.reset(alloc_fails() ? nullptr : new (std::nothrow) Range[n]);
    if (!many) return fail(TFE_ERR_OOM, "host memory for %lld tensors", (long long)n);
  }
  Range* const r = many ? many.get() : near;
  int64_t m = 0;
  bool sorted = true;
  for (int64_t k = 0; k < n; ++k) {
    if (t[k].rows == 0 || t[k].cols == 0) continue;
    r[m] = range_of(t[k], t[k].out, t[k].ldo, k);
    sorted = sorted && (m == 0 || r[m - 1].from <= r[m].from);
    ++m;
  }
  if (!sorted) std::sort(r, r + m, [](const Range& a, const Range& b) { return a.from < b.from; });
  for (int64_t k = 1; k < m; ++k)
    NEED(r[k - 1].to <= r[k].from, "tensors %lld and %lld: clipped into the same memory",
         (long long)r[k - 1].tensor, (long long)r[k].tensor);
  for (int64_t k = 0; k < n; ++k) {
    const tfe_grad_tensor& g = t[k];
    if (g.rows == 0 || g.cols == 0 || g.grad == g.out) continue;
    const Range x = range_of(g, g.grad, g.ldg, k);
    // The first that ends behind where this one begins.
    const Range* o = std::partition_point(r, r + m, [&](const Range& a) { return a.to <= x.from; });
    NEED(o == r + m || o->from >= x.to, "tensors %lld and %lld: a gradient under a clipped one",
         (long long)k, (long long)o->tensor);
  }
  return TFE_OK;
}

tfe_status max_norm_ok(float x) {
  NEED(x >= 0.f && isfinite(x), "max_norm negative or not finite");
  return TFE_OK;
}

// ---- integers ----------------------------------------------------------------------

tfe_status int8_sizes(int64_t rows, int32_t dim) {
  NEED(rows >= 0 && rows <= kLogitsMaxRows, "rows outside [0, 2^20]");
  NEED(dim >= 1 && dim <= kInt8MaxDim, "dim outside [1, %d]", kInt8MaxDim);
  return TFE_OK;
}
Int8QuantizeArgs int8_quantize_args(const void* x, int64_t ldx, int64_t rows, int32_t dim,
                                    int8_t* codes, float* scales) {
  return Int8QuantizeArgs{x, ldx, rows, (uint32_t)dim, int8_pitch(dim), codes, scales};
}
tfe_status int8_codes(const int8_t* codes, const float* scales) {
  NEED(codes && aligned(codes, 16), "codes: null or not 16-byte aligned");
  NEED(scales && aligned(scales, 4), "scales: null or not 4-byte aligned");
  return TFE_OK;
}
// Scales of the rows, then their codes.
int64_t int8_scales(int64_t rows) { return (rows * 4 + 15) / 16 * 16; }
int64_t int8_space(int64_t rows, int32_t dim) {
  return rows == 0 ? 0 : int8_scales(rows) + rows * (int64_t)int8_pitch(dim);
}
tfe_status int8_out(int64_t rows, int32_t n, int32_t dim, void* out, int32_t out_dtype, int64_t ldo) {
  TRY(int8_sizes(rows, dim));
  NEED(n >= 1 && n <= kInt8MaxOut, "out_dim outside [1, 2^20]");
  return matrix(out, out_dtype, ldo, rows, n, "out");
}

}  // namespace
}  // namespace tfe

extern "C" {

tfe_status tfe_cross_entropy_loss(const void* hidden, int64_t ldh, const void* w, int64_t ldw,
                                  const int32_t* targets, int64_t rows, int32_t vocab, int32_t dim,
                                  float* loss, float* lse, void* workspace,
                                  int64_t workspace_bytes, void* stream) {
  using namespace tfe;
  begin_call();
  XentArgs a{};
  TRY(xent_args(hidden, ldh, w, ldw, targets, rows, vocab, dim, workspace, workspace_bytes, &a));
  if (rows == 0) return TFE_OK;
  NEED(loss && lse && aligned(loss, 4) && aligned(lse, 4), "loss or lse: null or not aligned");
  a.loss = loss;
  a.lse = lse;
  return launched(launch_xent_loss(a, (hipStream_t)stream), "cross entropy launch");
}

tfe_status tfe_cross_entropy_grad(const void* hidden, int64_t ldh, const void* w, int64_t ldw,
                                  const int32_t* targets, int64_t rows, int32_t vocab, int32_t dim,
                                  const float* lse, const float* grad_loss, void* grad_hidden,
                                  int64_t ldgh, void* grad_w, int64_t ldgw, int32_t grad_dtype,
                                  int32_t accumulate, void* workspace, int64_t workspace_bytes,
                                  void* stream) {
  using namespace tfe;
  begin_call();
  XentArgs a{};
  TRY(xent_args(hidden, ldh, w, ldw, targets, rows, vocab, dim, workspace, workspace_bytes, &a));
  TRY(xent_grads(rows, vocab, dim, hidden, w, grad_loss, grad_hidden, ldgh, grad_w, ldgw, grad_dtype,
                 accumulate, &a));
  NEED(rows == 0 || (lse && aligned(lse, 4)), "lse: null or not aligned");
  a.lse = const_cast<float*>(lse);
  return launched(launch_xent_grad(a, false, (hipStream_t)stream), "cross entropy gradient launch");
}

tfe_status tfe_cross_entropy_loss_grad(const void* hidden, int64_t ldh, const void* w, int64_t ldw,
                                       const int32_t* targets, int64_t rows, int32_t vocab,
                                       int32_t dim, const float* grad_loss, float* loss, float* lse,
                                       void* grad_hidden, int64_t ldgh, void* grad_w, int64_t ldgw,
                                       int32_t grad_dtype, int32_t accumulate, void* workspace,
                                       int64_t workspace_bytes, void* stream) {
  using namespace tfe;
  begin_call();
  XentArgs a{};
  TRY(xent_args(hidden, ldh, w, ldw, targets, rows, vocab, dim, workspace, workspace_bytes, &a));
  TRY(xent_grads(rows, vocab, dim, hidden, w, grad_loss, grad_hidden, ldgh, grad_w, ldgw, grad_dtype,
                 accumulate, &a));
  NEED(rows == 0 || (loss && lse && aligned(loss, 4) && aligned(lse, 4)),
       "loss or lse: null or not aligned");
  a.loss = loss;
  a.lse = lse;
  if (rows) TRY(launched(launch_xent_loss(a, (hipStream_t)stream), "cross entropy launch"));
  return launched(launch_xent_grad(a, true, (hipStream_t)stream), "cross entropy gradient launch");
}

int64_t tfe_cross_entropy_workspace(int64_t rows, int32_t vocab, int32_t dim) {
  tfe::clear_error();
  return tfe::xent_sizes(rows, vocab, dim) == TFE_OK ? tfe::xent_space(rows, vocab, dim) : -1;
}

tfe_status tfe_grad_norm(const tfe_grad_tensor* tensors, int64_t n, float* norm, void* workspace,
                         int64_t workspace_bytes, void* stream) {
  using namespace tfe;
  begin_call();
  TRY(grad_tensors(tensors, n, false));
  NEED(norm && aligned(norm, 4), "norm: null or not aligned");
  TRY(space(workspace, workspace_bytes, grad_space(tensors, n)));
  return launched(launch_grad_norm(GradArgs{tensors, n, 0.f, norm, (unsigned char*)workspace},
                                   (hipStream_t)stream),
                  "gradient norm launch");
}

tfe_status tfe_grad_clip(const tfe_grad_tensor* tensors, int64_t n, float max_norm,
                         const float* norm, void* stream) {
  using namespace tfe;
  begin_call();
  TRY(grad_tensors(tensors, n, true));
  TRY(grad_places(tensors, n));
  TRY(max_norm_ok(max_norm));
  NEED(norm && aligned(norm, 4), "norm: null or not aligned");
  return launched(launch_grad_clip(GradArgs{tensors, n, max_norm, const_cast<float*>(norm), nullptr},
                                   (hipStream_t)stream),
                  "gradient clipping launch");
}

tfe_status tfe_grad_norm_clip(const tfe_grad_tensor* tensors, int64_t n, float max_norm,
                              float* norm, void* workspace, int64_t workspace_bytes, void* stream) {
  using namespace tfe;
  begin_call();
  TRY(grad_tensors(tensors, n, true));
  TRY(grad_places(tensors, n));
  TRY(max_norm_ok(max_norm));
  NEED(norm && aligned(norm, 4), "norm: null or not aligned");
  TRY(space(workspace, workspace_bytes, grad_space(tensors, n)));
  return launched(launch_grad_norm_clip(GradArgs{tensors, n, max_norm, norm, (unsigned char*)workspace},
                                        (hipStream_t)stream),
                  "gradient clipping launch");
}

int64_t tfe_grad_workspace(const tfe_grad_tensor* tensors, int64_t n) {
  tfe::clear_error();
  return tfe::grad_tensors(tensors, n, false) == TFE_OK ? tfe::grad_space(tensors, n) : -1;
}

tfe_status tfe_integer_quantize(const void* x, int32_t dtype, int64_t ldx, int64_t rows, int32_t dim,
                             int8_t* codes, float* scales, void* stream) {
  using namespace tfe;
  begin_call();
  TRY(int8_sizes(rows, dim));
  TRY(matrix(x, dtype, ldx, rows, dim, "x"));
  if (rows == 0) return TFE_OK;
  TRY(int8_codes(codes, scales));
  return launched(launch_int8_quantize(int8_quantize_args(x, ldx, rows, dim, codes, scales), dtype,
                                       (hipStream_t)stream),
                  "integer layout launch");
}

tfe_status tfe_integer_matmul(const int8_t* a, const float* a_scales, const int8_t* w,
                           const float* w_scales, int64_t rows, int32_t out_dim, int32_t dim,
                           void* out, int32_t out_dtype, int64_t ldo, void* stream) {
  using namespace tfe;
  begin_call();
  TRY(int8_out(rows, out_dim, dim, out, out_dtype, ldo));
  if (rows == 0) return TFE_OK;
  TRY(int8_codes(a, a_scales));
  TRY(int8_codes(w, w_scales));
  return launched(launch_int8_matmul(Int8MatmulArgs{a, a_scales, w, w_scales, out, ldo, (uint32_t)rows,
                                                    (uint32_t)out_dim, int8_pitch(dim)},
                                     out_dtype, (hipStream_t)stream),
                  "integer product launch");
}

tfe_status tfe_integer_linear(const void* x, int32_t dtype, int64_t ldx, const int8_t* w,
                           const float* w_scales, int64_t rows, int32_t out_dim, int32_t dim,
                           void* out, int32_t out_dtype, int64_t ldo, void* workspace,
                           int64_t workspace_bytes, void* stream) {
  using namespace tfe;
  begin_call();
  TRY(int8_out(rows, out_dim, dim, out, out_dtype, ldo));
  TRY(matrix(x, dtype, ldx, rows, dim, "x"));
  if (rows == 0) return TFE_OK;
  TRY(int8_codes(w, w_scales));
  TRY(space(workspace, workspace_bytes, int8_space(rows, dim)));
  float* scales = (float*)workspace;
  int8_t* codes = (int8_t*)workspace + int8_scales(rows);
  return launched(launch_int8_linear(int8_quantize_args(x, ldx, rows, dim, codes, scales),
                                     Int8MatmulArgs{codes, scales, w, w_scales, out, ldo, (uint32_t)rows,
                                                    (uint32_t)out_dim, int8_pitch(dim)},
                                     dtype, out_dtype, (hipStream_t)stream),
                  "integer product launch");
}

int64_t tfe_integer_workspace(int64_t rows, int32_t dim) {
  tfe::clear_error();
  return tfe::int8_sizes(rows, dim) == TFE_OK ? tfe::int8_space(rows, dim) : -1;
}

}  // extern "C"
