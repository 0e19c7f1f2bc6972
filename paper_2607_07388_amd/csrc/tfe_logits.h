// Internal declarations of the calls on the head's logits: the 8-bit product,
// sampling and distillation (not part of the C ABI).
#pragma once
#include <stdint.h>

#include <hip/hip_runtime_api.h>

namespace tfe {

// Compute units of the current device.
int compute_units();

constexpr int kFp8Block = 128;
constexpr int kFp8MaxDim = 65536;
constexpr int kDistillMaxK = 256;
constexpr int kLogitsMaxVocab = 1 << 18;
constexpr int kLogitsMaxRows = 1 << 20;
constexpr int kFp8MaxOut = 1 << 20;

inline uint32_t fp8_pitch(int32_t dim) { return ((uint32_t)dim + 127) / 128 * 128; }
// Bytes of one row of scales.
inline uint32_t fp8_scale_pitch(int32_t dim) { return (fp8_pitch(dim) / 128 + 3) / 4 * 4; }

struct QuantizeArgs {
  const void* x;
  int64_t ldx, rows;
  uint32_t dim, pitch, spitch;
  uint8_t* codes;
  uint8_t* scales;
};
hipError_t launch_fp8_quantize(const QuantizeArgs& a, int dtype, int block_rows, hipStream_t s);

struct MatmulArgs {
  const uint8_t* a;   // [rows x pitch] codes
  const uint8_t* as;  // [rows x spitch]
  const uint8_t* w;   // [n x pitch]
  const uint8_t* ws;  // [ceil(n / 128) x spitch]
  void* out;
  int64_t ldo;
  uint32_t rows, n, pitch, spitch;
};
hipError_t launch_fp8_matmul(const MatmulArgs& a, int out_dtype, hipStream_t s);
// Both: x's codes and scales are a.a and a.as.
hipError_t launch_fp8_linear(const QuantizeArgs& x, const MatmulArgs& a, int dtype, int out_dtype,
                             hipStream_t s);

struct SampleArgs {
  const void* logits;
  int64_t ld;
  uint32_t rows, vocab;
  const float* temperature;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  const float* u;
  int32_t* token;
  float* prob;
  unsigned char* space;
};
int64_t sample_space(int64_t rows, int32_t vocab);
hipError_t launch_sample(const SampleArgs& a, int dtype, hipStream_t s);

struct DistillArgs {
  const void* logits;
  int64_t ld;
  uint32_t rows, vocab;
  const int32_t* ids;   // [rows x K]
  const void* teacher;  // [rows x K]
  uint32_t K;
  float tau, inv_tau;
  const float* weight;  // [rows] or null
  float* loss;
  float* lse;           // written by the loss, read by the gradient
  void* grad;
  int64_t ldg;
  unsigned char* space;
  uint32_t wait_limit;  // polls for the other parts' sums (kDistillWaitLimit)
};
// Polls before a block computes the sums that have not come itself (some
// milliseconds).  The environment variable TFE_DISTILL_WAIT_LIMIT overrides it
// per call, so that tests can force that from the host.
constexpr uint32_t kDistillWaitLimit = 1u << 12;
int64_t distill_space(int64_t rows, int32_t vocab);
hipError_t launch_distill_loss(const DistillArgs& a, int dtype, int tdtype, hipStream_t s);
hipError_t launch_distill_grad(const DistillArgs& a, int dtype, int tdtype, hipStream_t s);
hipError_t launch_distill_loss_grad(const DistillArgs& a, int dtype, int tdtype, hipStream_t s);

}  // namespace tfe
