// Device building blocks of the calls on logits: rows of float32 or bfloat16
// at any element alignment, read 16 bytes a lane, and block reductions.
#pragma once
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "tfe_internal.h"

namespace tfe {
namespace rows {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// The same at the alignment of a bfloat16 (float32) element: a row need not
// start on a 16-byte boundary, and the hardware takes such loads.
typedef uint32_t u32x4_a2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

template <int DT> struct Elem;
template <> struct Elem<TFE_F32> {
  typedef float T;
  typedef u32x4_a4 V;
  static constexpr int N = 4;  // elements of a 16-byte vector
};
template <> struct Elem<TFE_BF16> {
  typedef uint16_t T;
  typedef u32x4_a2 V;
  static constexpr int N = 8;
};

template <int DT> __device__ __forceinline__ float load1(const void* row, size_t i) {
  if (DT == TFE_F32) return ((const float*)row)[i];
  return __uint_as_float((uint32_t)((const uint16_t*)row)[i] << 16);
}
// Nearest even, as every rounding to bfloat16 here.
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}
template <int DT> __device__ __forceinline__ void store1(void* row, size_t i, float v) {
  if (DT == TFE_F32)
    ((float*)row)[i] = v;
  else
    ((uint16_t*)row)[i] = (uint16_t)pack2(v, v);
}
// Vector v of a row (of less than 2^32 bytes: a scalar base and a 32-bit offset).
template <int DT> __device__ __forceinline__ u32x4 load_vec(const void* row, uint32_t v) {
  return *(const typename Elem<DT>::V*)((const char*)row + v * 16u);
}
template <int DT> __device__ __forceinline__ void store_vec(void* row, uint32_t v, u32x4 x) {
  *(typename Elem<DT>::V*)((char*)row + v * 16u) = x;
}
// The same for logits and results that pass by once.
template <int DT> __device__ __forceinline__ u32x4 load_stream(const void* row, uint32_t v) {
  return __builtin_nontemporal_load((const typename Elem<DT>::V*)((const char*)row + v * 16u));
}
template <int DT> __device__ __forceinline__ void store_stream(void* row, uint32_t v, u32x4 x) {
  __builtin_nontemporal_store(x, (typename Elem<DT>::V*)((char*)row + v * 16u));
}
template <int DT> __device__ __forceinline__ void unpack(u32x4 v, float* f) {
  if (DT == TFE_F32) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(v[i] << 16);
      f[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
    }
  }
}
template <int DT> __device__ __forceinline__ u32x4 pack(const float* f) {
  u32x4 v;
  if (DT == TFE_F32) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __float_as_uint(f[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = pack2(f[2 * i], f[2 * i + 1]);
  }
  return v;
}

template <class T> __device__ __forceinline__ T wave_max(T x) {
#pragma unroll
  for (int o = 32; o; o >>= 1) {
    const T y = __shfl_xor(x, o);
    x = x < y ? y : x;
  }
  return x;
}
template <class T> __device__ __forceinline__ T wave_add(T x) {
#pragma unroll
  for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
  return x;
}
// Block-wide, every thread gets the result; `lds` holds one T per wave and may
// be reused after the call's last barrier.  The order of the additions is fixed.
template <class T, int THREADS> __device__ __forceinline__ T block_max(T x, T* lds) {
  x = wave_max(x);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
  __syncthreads();
  T r = lds[0];
#pragma unroll
  for (int w = 1; w < THREADS / 64; ++w) r = r < lds[w] ? lds[w] : r;
  __syncthreads();
  return r;
}
template <class T, int THREADS> __device__ __forceinline__ T block_add(T x, T* lds) {
  x = wave_add(x);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
  __syncthreads();
  T r = lds[0];
#pragma unroll
  for (int w = 1; w < THREADS / 64; ++w) r += lds[w];
  __syncthreads();
  return r;
}

}  // namespace rows
}  // namespace tfe
