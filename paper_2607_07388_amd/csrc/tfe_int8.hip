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

// Two tiles of 16 columns of a row, each lane's 4 + 4, as 16 bytes of bfloat16 at
// column piece_of(g): lanes of neighbouring rows of 16 exchange halves.
__device__ __forceinline__ u32x4 pair_of(const float* p, const float* q) {
#if defined(__HIP_DEVICE_COMPILE__)
  const auto lo = __builtin_amdgcn_permlane16_swap(pack2(p[0], p[1]), pack2(q[0], q[1]), false, false);
  const auto hi = __builtin_amdgcn_permlane16_swap(pack2(p[2], p[3]), pack2(q[2], q[3]), false, false);
  return u32x4{lo[0], hi[0], lo[1], hi[1]};
#else
  return u32x4{};
#endif
}
__device__ __forceinline__ uint32_t piece_of(uint32_t g) { return (g & 1) * 16 + (g >> 1) * 8; }

struct TileArgs {
  Int8MatmulArgs m;
  uint32_t tiles_q, total;
};

template <int TP, int TQ, int WP, int WQ, int DT>
__global__ __launch_bounds__(WP* WQ * 64) void k_int8_tiles(TileArgs b) {
  typedef typename Elem<DT>::T E;
  typedef Tile<Int8, TP, TQ, WP, WQ, false, false, false> T;
  typedef f32x4 V4;
  typedef f32x4 V4_a4 __attribute__((aligned(4)));
  typedef u32x2 u32x2_a2 __attribute__((aligned(2)));
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const Int8MatmulArgs& a = b.m;
  T t;
  auto find = [&](uint32_t at, uint32_t* p0, uint32_t* q0) {
    if (at >= b.total) return false;
    const uint32_t place = (at & 7) * (b.total >> 3) + (at >> 3);
    *p0 = place / b.tiles_q * TP;
    *q0 = place % b.tiles_q * TQ;
    return *p0 < a.n;
  };
  auto segment = [&](uint32_t p0, uint32_t q0) {
    return gemm::Segment{Operand{(const char*)a.w + (size_t)p0 * a.pitch, a.pitch, a.n - p0, a.pitch, 0, 0},
                         Operand{(const char*)a.a + (size_t)q0 * a.pitch, a.pitch, a.rows - q0, a.pitch, 0, 0}, 0,
                         a.pitch / gemm::kStep};
  };
  uint32_t at = blockIdx.x, p0, q0, np0 = 0, nq0 = 0;
  if (!find(at, &p0, &q0)) return;
  t.clear();
  // The rows' scales, then the columns'.
  constexpr int INFO = (TQ + TP) * 4;
  constexpr int STORES = DT == TFE_F32 ? T::NT * T::MT : T::NT * T::MT / 2;
  auto write = [&](const char* info) {
    const float* as = (const float*)info + t.wq + t.i;
    const f32x4* ws = (const f32x4*)(info + TQ * 4) + t.wp / 4 + t.g;
    const bool all = p0 + TP <= a.n && q0 + TQ <= a.rows;
    V4 w[T::NT];
#pragma unroll
    for (int n = 0; n < T::NT; ++n) w[n] = ws[n * 4];
#pragma unroll
    for (int m = 0; m < T::MT; ++m) {
      const uint32_t r = q0 + t.wq + m * 16 + t.i;
      const float x = as[m * 16];
#pragma unroll
      for (int n = 0; n < T::NT; n += 2) {
        V4 v[2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int j = 0; j < 4; ++j) v[h][j] = (float)t.acc[n + h][m][j] * x * w[n + h][j];
        if (DT == TFE_F32 || !all) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t c = p0 + t.wp + t.g * 4 + (n + h) * 16;
            E* out = (E*)a.out + (size_t)r * a.ldo + c;
            if (all || (r < a.rows && c + 4 <= a.n)) {
              if constexpr (DT == TFE_F32)
                *(V4_a4*)out = v[h];
              else
                *(u32x2_a2*)out = u32x2{pack2(v[h][0], v[h][1]), pack2(v[h][2], v[h][3])};
            } else if (r < a.rows) {
#pragma unroll
              for (int j = 0; j < 4; ++j)
                if (c + j < a.n) store1<DT>(out, j, v[h][j]);
            }
          }
        } else {
          E* out = (E*)a.out + (size_t)r * a.ldo + p0 + t.wp + n * 16 + piece_of(t.g);
          // Passed by, these stores took 373 us of 2048 rows of 151936 x 1024 to 334.
          __builtin_nontemporal_store(pair_of((const float*)&v[0], (const float*)&v[1]), (u32x4_a2*)out);
        }
      }
    }
    return all;
  };
  t.template run<STORES>(
      segment(p0, q0),
      [&](gemm::Segment* s) {
        at += gridDim.x;
        const bool more = find(at, &np0, &nq0);
        if (more) *s = segment(np0, nq0);
        return more;
      },
      [&](uint32_t odd) {
        char* to = lds + T::LDS + odd * INFO;
        static_assert(TP / 64 <= T::WAVES && TQ / 64 <= T::WAVES, "a wave for each 64 scales");
        if (t.wave < TQ / 64) gemm::load_numbers(a.as, q0, a.rows, t.wave, to);
        if (t.wave < TP / 64) gemm::load_numbers(a.ws, p0, a.n, t.wave, to + TQ * 4);
      },
      [&](uint32_t odd) {
        const bool stored = write(lds + T::LDS + odd * INFO);
        p0 = np0;
        q0 = nq0;
        t.clear();
        return stored;
      },
      lds);
}

template <int TP, int TQ, int WP, int WQ, int DT>
hipError_t tiles(const Int8MatmulArgs& m, hipStream_t s) {
  typedef Tile<Int8, TP, TQ, WP, WQ, false, false, false> T;
  auto* k = k_int8_tiles<TP, TQ, WP, WQ, DT>;
  constexpr int LDS = T::LDS + 2 * (TP + TQ) * 4;
  static std::atomic<uint64_t> told{0};
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (dev > 63 || !(told.load(std::memory_order_relaxed) & bit)) {
    e = hipFuncSetAttribute((const void*)k, hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
    if (e != hipSuccess) return e;
    told.fetch_or(bit, std::memory_order_relaxed);
  }
  TileArgs a{m, (m.rows + TQ - 1) / TQ, 0};
  a.total = ((m.n + TP - 1) / TP * a.tiles_q + 7) / 8 * 8;
  k<<<dim3(std::min<uint32_t>(a.total, (compute_units() * (163840 / LDS) + 7) / 8 * 8)), dim3(T::THREADS), LDS, s>>>(a);
  return hipGetLastError();
}

// Tiles of 256 x 256 where they fill the device and waste few rows, of 128 x 64 where those
// of 128 x 128 would not fill it.  us in tiles of 64 / 128 / 256 rows, dim 1024: 64 rows of 151936
// to float32 36 / 41 / 63; to bfloat16 100 rows of 20000 12 / 14 / 23, of 151936 45 / 41 / 59; 200 rows
// of 151936 69 / 67 / 71, 257 87 / 84 / 90, 400 120 / 109 / 99, 600 174 / 147 / 132; 700 rows of 3000
// 13 / 15 / 26, of 20000 30 / 31 / 32; 1024 rows of 151936 to float32 436 / 372 / 250.
template <int DT> hipError_t matmul(const Int8MatmulArgs& a, hipStream_t s) {
  const uint32_t cus = (uint32_t)compute_units(), r128 = (a.rows + 127) / 128, r256 = (a.rows + 255) / 256;
  if (a.rows > 256 && (uint64_t)((a.n + 255) / 256) * r256 >= cus * 2 && r256 * 200 <= r128 * 125)
    return tiles<256, 256, 2, 4, DT>(a, s);
  if (a.rows > 64 && (uint64_t)((a.n + 127) / 128) * r128 >= cus) return tiles<128, 128, 2, 2, DT>(a, s);
  return tiles<128, 64, 1, 4, DT>(a, s);
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
