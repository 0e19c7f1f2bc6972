// Matrix product in 8-bit floating point (OCP e4m3) with a power-of-two scale
// for each block of 128: out[r, n] = sum_k A[r, k] W[n, k].
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "tfe_logits.h"
#include "tfe_rows.h"

namespace tfe {
namespace {

using namespace rows;

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// ---- layout ------------------------------------------------------------------

// Biased exponent of the least power of two 2^e, e >= -127, with
// amax <= 448 * 2^e (448 = 1.75 * 2^8); amax is finite.
__device__ __forceinline__ uint32_t block_exponent(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 8 + ((u & 0x7FFFFFu) > 0x600000u);
  return (uint32_t)max(e, 0);
}
// 2^-e of a biased exponent (at most 247: always a normal number).
__device__ __forceinline__ float unscale(uint32_t biased) {
  return __uint_as_float((254u - biased) << 23);
}
__device__ __forceinline__ float finite_abs(float x) {
  const float y = fabsf(x);
  return y < INFINITY ? y : 0.f;
}
// Nearest even; infinities saturate, NaN stays.
__device__ __forceinline__ float clamp448(float x) {
  return x != x ? x : fminf(fmaxf(x, -448.f), 448.f);
}
__device__ __forceinline__ uint32_t codes4(const float* x) {
  uint32_t r = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(clamp448(x[0]), clamp448(x[1]), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(clamp448(x[2]), clamp448(x[3]), (int)r, true);
}

// Eight columns from c of one row; those from dim on are zero.
template <int DT>
__device__ __forceinline__ void load8(const QuantizeArgs& a, int64_t row, uint32_t c, float* f) {
  const char* x = (const char*)a.x + (size_t)row * a.ldx * sizeof(typename Elem<DT>::T);
  if (c + 8 <= a.dim) {
    const char* p = x + (size_t)c * sizeof(typename Elem<DT>::T);
    unpack<DT>(load_vec<DT>(p, 0), f);
    if (DT == TFE_F32) unpack<DT>(load_vec<DT>(p, 1), f + 4);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = c + i < a.dim ? load1<DT>(x, c + i) : 0.f;
  }
}
__device__ __forceinline__ void store8(const QuantizeArgs& a, int64_t row, uint32_t c, float* f,
                                       uint32_t biased) {
  const float inv = unscale(biased);
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] *= inv;
  *(u32x2*)(a.codes + (size_t)row * a.pitch + c) = u32x2{codes4(f), codes4(f + 4)};
}

// Blocks of one row: 16 lanes hold a block of 128.  One thread per 8 columns;
// the threads behind a row's columns write its padding of the scales.
template <int DT> __global__ __launch_bounds__(256) void k_quantize_rows(QuantizeArgs a) {
  const uint32_t per_row = a.spitch * 16;  // threads
  const int64_t n = a.rows * per_row;
  // Whole groups of 16 lanes enter and leave together: per_row is a multiple of 16.
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / per_row;
    const uint32_t c = (uint32_t)(i - row * per_row) * 8;
    float f[8];
    uint32_t biased = 127;
    if (c < a.pitch) {
      load8<DT>(a, row, c, f);
      float amax = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) amax = fmaxf(amax, finite_abs(f[j]));
#pragma unroll
      for (int o = 8; o; o >>= 1) amax = fmaxf(amax, __shfl_xor(amax, o));
      biased = block_exponent(amax);
      store8(a, row, c, f, biased);
    }
    if ((threadIdx.x & 15) == 0)
      a.scales[(size_t)row * a.spitch + c / kFp8Block] = (uint8_t)biased;
  }
}

// Blocks of 128 x 128: one block of threads each; rows beyond the last are
// skipped.  blockIdx.y runs over the scales' whole pitch.
template <int DT> __global__ __launch_bounds__(256) void k_quantize_tiles(QuantizeArgs a) {
  __shared__ float red[4];
  const int64_t row0 = (int64_t)blockIdx.x * kFp8Block;
  const uint32_t cb = blockIdx.y, c = cb * kFp8Block + (threadIdx.x & 15) * 8;
  uint32_t biased = 127;
  if (cb * kFp8Block < a.pitch) {
    float f[8][8];
    float amax = 0.f;
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      const int64_t row = row0 + p * 16 + (threadIdx.x >> 4);
      if (row >= a.rows) continue;
      load8<DT>(a, row, c, f[p]);
#pragma unroll
      for (int j = 0; j < 8; ++j) amax = fmaxf(amax, finite_abs(f[p][j]));
    }
    biased = block_exponent(block_max<float, 256>(amax, red));
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      const int64_t row = row0 + p * 16 + (threadIdx.x >> 4);
      if (row < a.rows) store8(a, row, c, f[p], biased);
    }
  }
  if (threadIdx.x == 0) a.scales[(size_t)blockIdx.x * a.spitch + cb] = (uint8_t)biased;
}

// ---- product -----------------------------------------------------------------

// Eight codes times 2^(biased - 127) as bfloat16: exact.
__device__ __forceinline__ bf16x8 widen(uint32_t lo, uint32_t hi, float scale) {
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  const b2 x0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  const b2 x1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  const b2 x2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  const b2 x3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return bf16x8{x0[0], x0[1], x1[0], x1[1], x2[0], x2[1], x3[0], x3[1]};
}
__device__ __forceinline__ float scale_of(uint32_t biased) {
  return __uint_as_float(biased ? biased << 23 : 0x400000u);  // 2^-127 is subnormal
}

// One wave per 16 x 16 outputs.  The lane (g, i) of an operand holds columns
// 32 g .. 32 g + 31 of row i of a block of 128; the matrix instruction takes 8
// of them at a time, the same ones of both operands.
template <int DT> __global__ __launch_bounds__(256) void k_product(MatmulArgs a) {
  const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
  const uint32_t n0 = (blockIdx.x * 4 + wave) * 16;
  if (n0 >= a.n) return;
  const uint32_t n = min(n0 + i, a.n - 1);
  const uint8_t* wp = a.w + (size_t)n * a.pitch + g * 32;
  for (uint32_t r0 = blockIdx.y * 16; r0 < a.rows; r0 += gridDim.y * 16) {
    const uint32_t r = min(r0 + i, a.rows - 1);
    const uint8_t* xp = a.a + (size_t)r * a.pitch + g * 32;
    f32x4 acc{0.f, 0.f, 0.f, 0.f};
    for (uint32_t b = 0; b < a.pitch / kFp8Block; ++b) {
      const float sw = scale_of(a.ws[(size_t)(n0 / kFp8Block) * a.spitch + b]);
      const float sx = scale_of(a.as[(size_t)r * a.spitch + b]);
      u32x4 w[2], x[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        w[j] = *(const u32x4*)(wp + b * kFp8Block + 16 * j);
        x[j] = *(const u32x4*)(xp + b * kFp8Block + 16 * j);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            widen(w[j >> 1][2 * (j & 1)], w[j >> 1][2 * (j & 1) + 1], sw),
            widen(x[j >> 1][2 * (j & 1)], x[j >> 1][2 * (j & 1) + 1], sx), acc, 0, 0, 0);
    }
    if (r0 + i >= a.rows) continue;
    char* out = (char*)a.out + (size_t)(r0 + i) * a.ldo * sizeof(typename Elem<DT>::T);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (n0 + g * 4 + j < a.n) store1<DT>(out, n0 + g * 4 + j, acc[j]);
  }
}

}  // namespace

hipError_t launch_fp8_quantize(const QuantizeArgs& a, int dtype, int block_rows, hipStream_t s) {
  if (block_rows == 1) {
    const dim3 grid((uint32_t)std::min<int64_t>((a.rows * a.spitch * 16 + 255) / 256, 1 << 20));
    if (dtype == TFE_F32)
      k_quantize_rows<TFE_F32><<<grid, dim3(256), 0, s>>>(a);
    else
      k_quantize_rows<TFE_BF16><<<grid, dim3(256), 0, s>>>(a);
  } else {
    const dim3 grid((uint32_t)((a.rows + kFp8Block - 1) / kFp8Block), a.spitch);
    if (dtype == TFE_F32)
      k_quantize_tiles<TFE_F32><<<grid, dim3(256), 0, s>>>(a);
    else
      k_quantize_tiles<TFE_BF16><<<grid, dim3(256), 0, s>>>(a);
  }
  return hipGetLastError();
}

hipError_t launch_fp8_matmul(const MatmulArgs& a, int out_dtype, hipStream_t s) {
  const dim3 grid((a.n + 63) / 64, std::min((a.rows + 15) / 16, 32768u));
  if (out_dtype == TFE_F32)
    k_product<TFE_F32><<<grid, dim3(256), 0, s>>>(a);
  else
    k_product<TFE_BF16><<<grid, dim3(256), 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace tfe
