// Internal declarations of the calls that learn the head from tokens and serve
// it in integers: cross entropy, the integer product, gradient norm and
// clipping (not part of the C ABI).
#pragma once
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#include "../../include/tfe.h"

namespace tfe {

// Compute units of the current device.
int compute_units();

constexpr int64_t kXentMaxPitch = 1 << 21;  // elements: 256 rows stay below 2^30 bytes
constexpr int kXentMaxDim = 16384;
constexpr int kInt8MaxDim = 65536;  // 65536 * 127^2 < 2^31
constexpr int kInt8MaxOut = 1 << 20;

struct XentArgs {
  const uint16_t* hidden;
  int64_t ldh;
  const uint16_t* w;
  int64_t ldw;
  const int32_t* targets;
  uint32_t rows, vocab, dim;
  float* loss;
  float* lse;           // written by the loss, read by the gradient
  const float* weight;  // [rows] or null
  void* gx;
  int64_t ldgx;
  void* gw;
  int64_t ldgw;
  int gdtype;
  bool accumulate;
  unsigned char* space;
};
int64_t xent_space(int64_t rows, int32_t vocab, int32_t dim);
hipError_t launch_xent_loss(const XentArgs& a, hipStream_t s);
// behind_loss: the loss of the same arguments was launched just before.
hipError_t launch_xent_grad(const XentArgs& a, bool behind_loss, hipStream_t s);

inline uint32_t int8_pitch(int32_t dim) { return ((uint32_t)dim + 127) / 128 * 128; }

struct Int8QuantizeArgs {
  const void* x;
  int64_t ldx, rows;
  uint32_t dim, pitch;
  int8_t* codes;
  float* scales;
};
hipError_t launch_int8_quantize(const Int8QuantizeArgs& a, int dtype, hipStream_t s);

struct Int8MatmulArgs {
  const int8_t* a;  // [rows x pitch]
  const float* as;  // [rows]
  const int8_t* w;  // [n x pitch]
  const float* ws;  // [n]
  void* out;
  int64_t ldo;
  uint32_t rows, n, pitch;
};
hipError_t launch_int8_matmul(const Int8MatmulArgs& a, int out_dtype, hipStream_t s);
// Both: x's codes and scales are a.a and a.as.
hipError_t launch_int8_linear(const Int8QuantizeArgs& x, const Int8MatmulArgs& a, int dtype,
                              int out_dtype, hipStream_t s);

struct GradArgs {
  const tfe_grad_tensor* tensors;  // host
  int64_t n;
  float max_norm;
  float* norm;
  unsigned char* space;
};
int64_t grad_space(const tfe_grad_tensor* tensors, int64_t n);
hipError_t launch_grad_norm(const GradArgs& a, hipStream_t s);
hipError_t launch_grad_clip(const GradArgs& a, hipStream_t s);
hipError_t launch_grad_norm_clip(const GradArgs& a, hipStream_t s);

}  // namespace tfe
