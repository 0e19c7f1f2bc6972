// Matrix product of 8-bit integers with a scale for each row of either operand:
// out[r, n] = (sum_k A[r, k] W[n, k]) as[r] ws[n], the sum exact.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>

#include "tfe_gemm.h"
#include "tfe_learn.h"
#include "tfe_rows.h"

namespace tfe {
namespace {

using namespace rows;
using gemm::Int8;
using gemm::Operand;
using gemm::Tile;
typedef gemm::i32x4 i32x4;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// ---- layout ------------------------------------------------------------------

constexpr float kInt8Least = 0x1p-100f;  // 127 (1 / m) stays finite above it

template <int DT>
__device__ __forceinline__ void load8(const void* x, uint32_t dim, uint32_t c, float* f) {
  if (c + 8 <= dim) {
    const char* p = (const char*)x + (size_t)c * sizeof(typename Elem<DT>::T);
    unpack<DT>(load_vec<DT>(p, 0), f);
    if (DT == TFE_F32) unpack<DT>(load_vec<DT>(p, 1), f + 4);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = c + i < dim ? load1<DT>(x, c + i) : 0.f;
  }
}
__device__ __forceinline__ void largest8(const float* f, float* top, bool* nan) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float y = fabsf(f[j]);
    *top = y < INFINITY ? fmaxf(*top, y) : *top;
    *nan |= y != y;
  }
}
__device__ __forceinline__ uint32_t code(float x, float inverse) {
  const float y = rintf(x * inverse);  // 0 x infinity is NaN, which both limits take to 0's place
  return (uint32_t)(int)(y != y ? 0.f : fminf(fmaxf(y, -127.f), 127.f)) & 255u;
}
__device__ __forceinline__ u32x2 codes8(const float* f, float inverse) {
  u32x2 r{0, 0};
#pragma unroll
  for (int j = 0; j < 8; ++j) r[j / 4] |= code(f[j], inverse) << (8 * (j & 3));
  return r;
}

// A wave a row: its largest magnitude, then the codes.
template <int DT> __global__ __launch_bounds__(256) void k_int8_quantize(Int8QuantizeArgs a) {
  const uint32_t lane = threadIdx.x & 63;
  const int64_t per = (int64_t)gridDim.x * 4;
  for (int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); row < a.rows; row += per) {
    const char* x = (const char*)a.x + (size_t)row * a.ldx * sizeof(typename Elem<DT>::T);
    float top = 0.f;
    bool nan = false;
    for (uint32_t c = lane * 8; c < a.dim; c += 512) {
      float f[8];
      load8<DT>(x, a.dim, c, f);
      largest8(f, &top, &nan);
    }
    top = wave_max(top);
    nan = __builtin_amdgcn_ballot_w64(nan) != 0;
    const bool some = top > kInt8Least;
    const float inverse = some ? 1.f / top * 127.f : 0.f;
    for (uint32_t c = lane * 8; c < a.pitch; c += 512) {
      float f[8];
      load8<DT>(x, a.dim, c, f);
      *(u32x2*)(a.codes + (size_t)row * a.pitch + c) = some ? codes8(f, inverse) : u32x2{0, 0};
    }
    if (lane == 0) a.scales[row] = nan ? NAN : some ? top / 127.f : 0.f;
  }
}

// ---- product -----------------------------------------------------------------

struct TileArgs {
  Int8MatmulArgs m;
  uint32_t tiles_q, total;
};

template <int TP, int TQ, int WP, int WQ, int DT>
__global__ __launch_bounds__(WP* WQ * 64) void k_int8_tiles(TileArgs b) {
  typedef typename Elem<DT>::T T;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const Int8MatmulArgs& a = b.m;
  Tile<Int8, TP, TQ, WP, WQ, false, false> t;
  const uint32_t place = (blockIdx.x & 7) * (b.total >> 3) + (blockIdx.x >> 3);
  const uint32_t p0 = place / b.tiles_q * TP, q0 = place % b.tiles_q * TQ;
  if (p0 >= a.n) return;
  t.clear();
  t.run(Operand{(const char*)a.w + (size_t)p0 * a.pitch, a.pitch, a.n - p0, a.pitch},
        Operand{(const char*)a.a + (size_t)q0 * a.pitch, a.pitch, a.rows - q0, a.pitch}, 0,
        a.pitch / gemm::kStep, lds);
  const uint32_t c0 = p0 + t.wp + t.g * 4;
#pragma unroll
  for (int n = 0; n < t.NT; ++n) {
    float ws[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) ws[j] = a.ws[min(c0 + n * 16 + j, a.n - 1)];
#pragma unroll
    for (int m = 0; m < t.MT; ++m) {
      const uint32_t r = q0 + t.wq + m * 16 + t.i;
      if (r >= a.rows) continue;
      const float as = a.as[r];
      T* out = (T*)a.out + (size_t)r * a.ldo + c0 + n * 16;
      f32x4 v;
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = (float)t.acc[n][m][j] * as * ws[j];
      typedef f32x4 f4 __attribute__((aligned(4)));
      typedef u32x2 u2 __attribute__((aligned(2)));
      if (c0 + n * 16 + 4 <= a.n) {
        if constexpr (DT == TFE_F32)
          *(f4*)out = v;
        else
          *(u2*)out = u2{pack2(v[0], v[1]), pack2(v[2], v[3])};
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (c0 + n * 16 + j < a.n) store1<DT>(out, j, v[j]);
      }
    }
  }
}

template <int TP, int TQ, int WP, int WQ, int DT>
hipError_t tiles(const Int8MatmulArgs& m, hipStream_t s) {
  typedef Tile<Int8, TP, TQ, WP, WQ, false, false> T;
  auto* k = k_int8_tiles<TP, TQ, WP, WQ, DT>;
  static std::atomic<uint64_t> told{0};
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (dev > 63 || !(told.load(std::memory_order_relaxed) & bit)) {
    e = hipFuncSetAttribute((const void*)k, hipFuncAttributeMaxDynamicSharedMemorySize, T::LDS);
    if (e != hipSuccess) return e;
    told.fetch_or(bit, std::memory_order_relaxed);
  }
  TileArgs a{m, (m.rows + TQ - 1) / TQ, 0};
  a.total = ((m.n + TP - 1) / TP * a.tiles_q + 7) / 8 * 8;
  k<<<dim3(a.total), dim3(T::THREADS), T::LDS, s>>>(a);
  return hipGetLastError();
}

template <int DT> hipError_t matmul(const Int8MatmulArgs& a, hipStream_t s) {
  if (a.rows <= 64) return tiles<256, 64, 2, 2, DT>(a, s);
  if (a.rows <= 256) return tiles<128, 128, 2, 2, DT>(a, s);
  return tiles<256, 256, 2, 4, DT>(a, s);
}

}  // namespace

hipError_t launch_int8_quantize(const Int8QuantizeArgs& a, int dtype, hipStream_t s) {
  const dim3 grid((uint32_t)std::min<int64_t>((a.rows + 3) / 4, 1 << 16));
  if (dtype == TFE_F32)
    k_int8_quantize<TFE_F32><<<grid, dim3(256), 0, s>>>(a);
  else
    k_int8_quantize<TFE_BF16><<<grid, dim3(256), 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_int8_matmul(const Int8MatmulArgs& a, int out_dtype, hipStream_t s) {
  return out_dtype == TFE_F32 ? matmul<TFE_F32>(a, s) : matmul<TFE_BF16>(a, s);
}

hipError_t launch_int8_linear(const Int8QuantizeArgs& x, const Int8MatmulArgs& a, int dtype,
                              int out_dtype, hipStream_t s) {
  const hipError_t e = launch_int8_quantize(x, dtype, s);
  return e == hipSuccess ? launch_int8_matmul(a, out_dtype, s) : e;
}

}  // namespace tfe
