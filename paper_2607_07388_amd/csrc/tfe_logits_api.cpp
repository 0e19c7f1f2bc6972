// C ABI of the calls on the head's logits: the 8-bit product, sampling and
// distillation.  Host checks only; nothing is allocated and no state kept.
#include <hip/hip_runtime_api.h>
#include <math.h>
#include <stdint.h>
#include <stdlib.h>

#include <atomic>

#include "../../include/tfe.h"
#include "tfe_internal.h"
#include "tfe_logits.h"

namespace tfe {

int compute_units() {
  constexpr int kDevices = 64;
  static std::atomic<int> known[kDevices];
  int dev = 0, cus = 0;
  if (hipGetDevice(&dev) != hipSuccess) return 256;
  if (dev >= 0 && dev < kDevices && (cus = known[dev].load(std::memory_order_relaxed)) > 0) return cus;
  if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus < 1)
    return 256;
  if (dev >= 0 && dev < kDevices) known[dev].store(cus, std::memory_order_relaxed);
  return cus;
}

namespace {

bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
uintptr_t elem(int32_t dtype) { return dtype == TFE_BF16 ? 2 : 4; }

tfe_status launched(hipError_t e, const char* what) {
  if (e == hipSuccess) return TFE_OK;
  return fail(TFE_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

#define NEED(cond, ...)                                          \
  do {                                                           \
    if (!(cond)) return fail(TFE_ERR_INVALID_ARG, __VA_ARGS__);  \
  } while (0)
#define TRY(call)                      \
  do {                                 \
    const tfe_status st_ = (call);     \
    if (st_ != TFE_OK) return st_;     \
  } while (0)

// A matrix argument of `rows` rows of `cols` elements, `ld` apart.
tfe_status matrix(const void* p, int32_t dtype, int64_t ld, int64_t rows, int64_t cols,
                  const char* what) {
  NEED(dtype == TFE_F32 || dtype == TFE_BF16, "%s: unknown dtype %d", what, dtype);
  NEED(ld >= cols, "%s: pitch %lld below the row's %lld elements", what, (long long)ld,
       (long long)cols);
  NEED(ld < ((int64_t)1 << 31), "%s: pitch above 2^31", what);
  if (rows == 0) return TFE_OK;
  NEED(p, "%s: null", what);
  NEED(aligned(p, elem(dtype)), "%s: not aligned to its elements", what);
  return TFE_OK;
}

tfe_status space(const void* p, int64_t bytes, int64_t need) {
  if (need == 0) return TFE_OK;
  NEED(p, "null workspace");
  NEED(aligned(p, 16), "workspace not 16-byte aligned");
  NEED(bytes >= need, "workspace of %lld bytes, %lld needed", (long long)bytes, (long long)need);
  return TFE_OK;
}

tfe_status fp8_sizes(int64_t rows, int32_t dim) {
  NEED(rows >= 0 && rows <= kLogitsMaxRows, "rows outside [0, 2^20]");
  NEED(dim >= 1 && dim <= kFp8MaxDim, "dim outside [1, %d]", kFp8MaxDim);
  return TFE_OK;
}

QuantizeArgs quantize_args(const void* x, int64_t ldx, int64_t rows, int32_t dim, uint8_t* codes,
                           uint8_t* scales) {
  QuantizeArgs a{};
  a.x = x;
  a.ldx = ldx;
  a.rows = rows;
  a.dim = (uint32_t)dim;
  a.pitch = fp8_pitch(dim);
  a.spitch = fp8_scale_pitch(dim);
  a.codes = codes;
  a.scales = scales;
  return a;
}

MatmulArgs matmul_args(const uint8_t* x, const uint8_t* xs, const uint8_t* w, const uint8_t* ws,
                       int64_t rows, int32_t n, int32_t dim, void* out, int64_t ldo) {
  MatmulArgs a{};
  a.a = x;
  a.as = xs;
  a.w = w;
  a.ws = ws;
  a.out = out;
  a.ldo = ldo;
  a.rows = (uint32_t)rows;
  a.n = (uint32_t)n;
  a.pitch = fp8_pitch(dim);
  a.spitch = fp8_scale_pitch(dim);
  return a;
}

tfe_status quantize(const void* x, int32_t dtype, int64_t ldx, int64_t rows, int32_t dim,
                    int32_t block_rows, uint8_t* codes, uint8_t* scales, hipStream_t s) {
  TRY(fp8_sizes(rows, dim));
  NEED(block_rows == 1 || block_rows == kFp8Block, "block_rows is 1 or 128");
  TRY(matrix(x, dtype, ldx, rows, dim, "x"));
  if (rows == 0) return TFE_OK;
  NEED(codes && aligned(codes, 16), "codes: null or not 16-byte aligned");
  NEED(scales && aligned(scales, 4), "scales: null or not 4-byte aligned");
  return launched(launch_fp8_quantize(quantize_args(x, ldx, rows, dim, codes, scales), dtype,
                                      block_rows, s),
                  "quantize launch");
}

tfe_status matmul(const uint8_t* x, const uint8_t* xs, const uint8_t* w, const uint8_t* ws,
                  int64_t rows, int32_t n, int32_t dim, void* out, int32_t out_dtype, int64_t ldo,
                  hipStream_t s) {
  TRY(fp8_sizes(rows, dim));
  NEED(n >= 1 && n <= kFp8MaxOut, "out_dim outside [1, 2^20]");
  TRY(matrix(out, out_dtype, ldo, rows, n, "out"));
  if (rows == 0) return TFE_OK;
  NEED(x && aligned(x, 16) && w && aligned(w, 16), "codes: null or not 16-byte aligned");
  NEED(xs && aligned(xs, 4) && ws && aligned(ws, 4), "scales: null or not 4-byte aligned");
  return launched(launch_fp8_matmul(matmul_args(x, xs, w, ws, rows, n, dim, out, ldo), out_dtype, s),
                  "8-bit product launch");
}

// Codes of the rows, then their scales.
int64_t linear_codes(int64_t rows, int32_t dim) { return rows * (int64_t)fp8_pitch(dim); }
int64_t linear_space(int64_t rows, int32_t dim) {
  return linear_codes(rows, dim) + rows * (int64_t)fp8_scale_pitch(dim);
}

tfe_status linear(const void* x, int32_t dtype, int64_t ldx, const uint8_t* w, const uint8_t* ws,
                  int64_t rows, int32_t n, int32_t dim, void* out, int32_t out_dtype, int64_t ldo,
                  void* workspace, int64_t bytes, hipStream_t s) {
  TRY(fp8_sizes(rows, dim));
  NEED(n >= 1 && n <= kFp8MaxOut, "out_dim outside [1, 2^20]");
  TRY(matrix(x, dtype, ldx, rows, dim, "x"));
  TRY(matrix(out, out_dtype, ldo, rows, n, "out"));
  if (rows == 0) return TFE_OK;
  NEED(w && aligned(w, 16), "codes: null or not 16-byte aligned");
  NEED(ws && aligned(ws, 4), "scales: null or not 4-byte aligned");
  TRY(space(workspace, bytes, linear_space(rows, dim)));
  uint8_t* codes = (uint8_t*)workspace;
  uint8_t* scales = codes + linear_codes(rows, dim);
  return launched(launch_fp8_linear(quantize_args(x, ldx, rows, dim, codes, scales),
                                    matmul_args(codes, scales, w, ws, rows, n, dim, out, ldo), dtype,
                                    out_dtype, s),
                  "8-bit product launch");
}

tfe_status vocab_ok(int32_t vocab) {
  NEED(vocab >= 1 && vocab <= kLogitsMaxVocab, "vocab outside [1, 2^18]");
  return TFE_OK;
}

tfe_status sample_sizes(int64_t rows, int32_t vocab) {
  NEED(rows >= 0 && rows <= kLogitsMaxRows, "rows outside [0, 2^20]");
  return vocab_ok(vocab);
}

tfe_status sample(const void* logits, int32_t dtype, int64_t ld, int64_t rows, int32_t vocab,
                  const float* temperature, const int32_t* top_k, const float* top_p,
                  const float* min_p, const float* u, int32_t* token, float* prob,
                  void* workspace, int64_t bytes, hipStream_t s) {
  TRY(sample_sizes(rows, vocab));
  TRY(matrix(logits, dtype, ld, rows, vocab, "logits"));
  if (rows == 0) return TFE_OK;
  NEED(u && token, "null u or token");
  TRY(space(workspace, bytes, sample_space(rows, vocab)));
  SampleArgs a{};
  a.logits = logits;
  a.ld = ld;
  a.rows = (uint32_t)rows;
  a.vocab = (uint32_t)vocab;
  a.temperature = temperature;
  a.top_k = top_k;
  a.top_p = top_p;
  a.min_p = min_p;
  a.u = u;
  a.token = token;
  a.prob = prob;
  a.space = (unsigned char*)workspace;
  return launched(launch_sample(a, dtype, s), "sampling launch");
}

tfe_status distill_sizes(int64_t rows, int32_t vocab) {
  NEED(rows >= 0 && rows <= kLogitsMaxRows, "rows outside [0, 2^20]");
  return vocab_ok(vocab);
}

tfe_status distill_args(const void* logits, int32_t dtype, int64_t ld, int64_t rows, int32_t vocab,
                        const int32_t* ids, const void* teacher, int32_t tdtype, int32_t K,
                        float tau, DistillArgs* a) {
  TRY(distill_sizes(rows, vocab));
  NEED(K >= 1 && K <= kDistillMaxK, "K outside [1, %d]", kDistillMaxK);
  // The kernels multiply by log2(e) / tau.
  NEED(tau > 0.f && isfinite(tau) && isfinite(1.f / tau * 1.44269504f),
       "temperature not positive and finite, or below 4.3e-39");
  TRY(matrix(logits, dtype, ld, rows, vocab, "logits"));
  TRY(matrix(teacher, tdtype, K, rows, K, "teacher_logits"));
  if (rows == 0) return TFE_OK;
  NEED(ids, "null teacher_ids");
  a->logits = logits;
  a->ld = ld;
  a->rows = (uint32_t)rows;
  a->vocab = (uint32_t)vocab;
  a->ids = ids;
  a->teacher = teacher;
  a->K = (uint32_t)K;
  a->tau = tau;
  a->inv_tau = 1.f / tau;
  return TFE_OK;
}

tfe_status grad_args(const void* logits, int32_t dtype, int64_t ld, int64_t rows, int32_t vocab,
                     void* grad, int64_t ldg) {
  TRY(matrix(grad, dtype, ldg, rows, vocab, "grad"));
  NEED(grad != logits || ldg == ld || rows == 0, "gradient in place of the logits at another pitch");
  return TFE_OK;
}

}  // namespace
}  // namespace tfe

extern "C" {

tfe_status tfe_quantize(const void* x, int32_t dtype, int64_t ldx, int64_t rows, int32_t dim,
                        int32_t block_rows, uint8_t* codes, uint8_t* scales, void* stream) {
  tfe::begin_call();
  return tfe::quantize(x, dtype, ldx, rows, dim, block_rows, codes, scales, (hipStream_t)stream);
}

tfe_status tfe_quantized_matmul(const uint8_t* a, const uint8_t* a_scales, const uint8_t* w,
                                const uint8_t* w_scales, int64_t rows, int32_t out_dim,
                                int32_t dim, void* out, int32_t out_dtype, int64_t ldo,
                                void* stream) {
  tfe::begin_call();
  return tfe::matmul(a, a_scales, w, w_scales, rows, out_dim, dim, out, out_dtype, ldo,
                     (hipStream_t)stream);
}

tfe_status tfe_quantized_linear(const void* x, int32_t dtype, int64_t ldx, const uint8_t* w,
                                const uint8_t* w_scales, int64_t rows, int32_t out_dim,
                                int32_t dim, void* out, int32_t out_dtype, int64_t ldo,
                                void* workspace, int64_t workspace_bytes, void* stream) {
  tfe::begin_call();
  return tfe::linear(x, dtype, ldx, w, w_scales, rows, out_dim, dim, out, out_dtype, ldo,
                     workspace, workspace_bytes, (hipStream_t)stream);
}

int64_t tfe_quantized_workspace(int64_t rows, int32_t dim) {
  tfe::clear_error();
  return tfe::fp8_sizes(rows, dim) == TFE_OK ? tfe::linear_space(rows, dim) : -1;
}

tfe_status tfe_sample(const void* logits, int32_t dtype, int64_t ld, int64_t rows, int32_t vocab,
                      const float* temperature, const int32_t* top_k, const float* top_p,
                      const float* min_p, const float* u, int32_t* token, float* prob,
                      void* workspace, int64_t workspace_bytes, void* stream) {
  tfe::begin_call();
  return tfe::sample(logits, dtype, ld, rows, vocab, temperature, top_k, top_p, min_p, u, token,
                     prob, workspace, workspace_bytes, (hipStream_t)stream);
}

int64_t tfe_sample_workspace(int64_t rows, int32_t vocab) {
  tfe::clear_error();
  return tfe::sample_sizes(rows, vocab) == TFE_OK ? tfe::sample_space(rows, vocab) : -1;
}

tfe_status tfe_distill_loss(const void* logits, int32_t dtype, int64_t ld, int64_t rows,
                            int32_t vocab, const int32_t* teacher_ids, const void* teacher_logits,
                            int32_t teacher_dtype, int32_t K, float temperature, float* loss,
                            float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
  using namespace tfe;
  begin_call();
  DistillArgs a{};
  TRY(distill_args(logits, dtype, ld, rows, vocab, teacher_ids, teacher_logits, teacher_dtype, K,
                   temperature, &a));
  if (rows == 0) return TFE_OK;
  NEED(loss && lse, "null loss or lse");
  TRY(space(workspace, workspace_bytes, distill_space(rows, vocab)));
  a.loss = loss;
  a.lse = lse;
  a.space = (unsigned char*)workspace;
  return launched(launch_distill_loss(a, dtype, teacher_dtype, (hipStream_t)stream),
                  "distillation loss launch");
}

tfe_status tfe_distill_grad(const void* logits, int32_t dtype, int64_t ld, int64_t rows,
                            int32_t vocab, const int32_t* teacher_ids, const void* teacher_logits,
                            int32_t teacher_dtype, int32_t K, float temperature, const float* lse,
                            const float* grad_loss, void* grad, int64_t ldg, void* stream) {
  using namespace tfe;
  begin_call();
  DistillArgs a{};
  TRY(distill_args(logits, dtype, ld, rows, vocab, teacher_ids, teacher_logits, teacher_dtype, K,
                   temperature, &a));
  TRY(grad_args(logits, dtype, ld, rows, vocab, grad, ldg));
  if (rows == 0) return TFE_OK;
  NEED(lse, "null lse");
  a.lse = const_cast<float*>(lse);
  a.weight = grad_loss;
  a.grad = grad;
  a.ldg = ldg;
  return launched(launch_distill_grad(a, dtype, teacher_dtype, (hipStream_t)stream),
                  "distillation gradient launch");
}

tfe_status tfe_distill_loss_grad(const void* logits, int32_t dtype, int64_t ld, int64_t rows,
                                 int32_t vocab, const int32_t* teacher_ids,
                                 const void* teacher_logits, int32_t teacher_dtype, int32_t K,
                                 float temperature, const float* grad_loss, float* loss,
                                 float* lse, void* grad, int64_t ldg, void* workspace,
                                 int64_t workspace_bytes, void* stream) {
  using namespace tfe;
  begin_call();
  DistillArgs a{};
  TRY(distill_args(logits, dtype, ld, rows, vocab, teacher_ids, teacher_logits, teacher_dtype, K,
                   temperature, &a));
  TRY(grad_args(logits, dtype, ld, rows, vocab, grad, ldg));
  if (rows == 0) return TFE_OK;
  NEED(loss && lse, "null loss or lse");
  TRY(space(workspace, workspace_bytes, distill_space(rows, vocab)));
  a.loss = loss;
  a.lse = lse;
  a.weight = grad_loss;
  a.grad = grad;
  a.ldg = ldg;
  a.space = (unsigned char*)workspace;
  const char* wl = getenv("TFE_DISTILL_WAIT_LIMIT");
  a.wait_limit = wl ? (uint32_t)strtoul(wl, nullptr, 0) : kDistillWaitLimit;
  return launched(launch_distill_loss_grad(a, dtype, teacher_dtype, (hipStream_t)stream),
                  "distillation launch");
}

int64_t tfe_distill_workspace(int64_t rows, int32_t vocab) {
  tfe::clear_error();
  return tfe::distill_sizes(rows, vocab) == TFE_OK ? tfe::distill_space(rows, vocab) : -1;
}

}  // extern "C"
