// Matrix product in 8-bit floating point (OCP e4m3) with a power-of-two scale
// for each block of 128: out[r, n] = sum_k A[r, k] W[n, k].
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

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

__device__ __forceinline__ uint32_t pack4(const float* x) {
  const uint32_t r = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], (int)r, true);
}
// Maximum over the 16 lanes of a row of the wave.
template <int CTRL> __device__ __forceinline__ float dpp_max(float x) {
  return fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xF, 0xF, false)));
}
__device__ __forceinline__ float max16(float x) {
  x = dpp_max<0xB1>(x);   // quad_perm [1,0,3,2]
  x = dpp_max<0x4E>(x);   // quad_perm [2,3,0,1]
  x = dpp_max<0x141>(x);  // row_half_mirror
  return dpp_max<0x140>(x);  // row_mirror
}
// Eight columns of a block that 16 lanes hold: their codes (f is scaled in
// place) and the block's exponent.  Infinities and NaN, which the scale passes
// over and the codes must not, are looked for by one fma a number.
__device__ __forceinline__ u32x2 encode8(float* f, uint32_t* biased) {
  float amax = 0.f, odd = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    amax = fmaxf(amax, fabsf(f[j]));
    odd = fmaf(f[j], 0.f, odd);
  }
  const bool some = __builtin_amdgcn_ballot_w64(odd != 0.f) != 0;  // NaN compares unequal
  if (some) {
    amax = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) amax = fmaxf(amax, finite_abs(f[j]));
  }
  *biased = block_exponent(max16(amax));
  const float inv = unscale(*biased);
#pragma unroll
  for (int j = 0; j < 8; ++j) f[j] *= inv;
  return some ? u32x2{codes4(f), codes4(f + 4)} : u32x2{pack4(f), pack4(f + 4)};
}

// Blocks of one row: 16 lanes hold a block of 128.  One thread per 8 columns;
// 257 x 1000 float32 3.2 to 4.7 us: a launch (2 to 3 us where one does next to nothing)
// and a chain of a 64-bit division, a load and the codes' store.
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
      *(u32x2*)(a.codes + (size_t)row * a.pitch + c) = encode8(f, &biased);
    }
    if ((threadIdx.x & 15) == 0)
      a.scales[(size_t)row * a.spitch + c / kFp8Block] = (uint8_t)biased;
  }
}

// Blocks of 128 x 128: one block of threads each; rows beyond the last are
// skipped.  blockIdx.y runs over the scales' whole pitch.  151936 x 1024 bfloat16: 96 us,
// 4.9 TB/s read and written.
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

__device__ __forceinline__ uint32_t byte_of(uint32_t w, int i) { return (w >> (8 * i)) & 255u; }

// Lane (g, i) of a 16-row operand holds of row i's block of 128 columns two
// 16-byte pieces: g and 4 + g.  Both operands of a product use the same pieces,
// so the matrix instruction multiplies matching columns, whatever their order.

// Four results of a lane (columns n .. n + 3 of one row), stored together
// where the row has them.
template <int DT> __device__ __forceinline__ void store4_at(char* out, f32x4 v) {
  typedef uint32_t u2 __attribute__((ext_vector_type(2), aligned(2)));
  typedef f32x4 f4 __attribute__((aligned(4)));
  if (DT == TFE_F32)
    *(f4*)out = v;
  else
    *(u2*)out = u2{pack2(v[0], v[1]), pack2(v[2], v[3])};
}
template <int DT>
__device__ __forceinline__ void store4(const MatmulArgs& a, uint32_t r, uint32_t n, f32x4 v) {
  char* out = (char*)a.out + ((size_t)r * a.ldo + n) * sizeof(typename Elem<DT>::T);
  if (n + 4 <= a.n) {
    store4_at<DT>(out, v);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (n + j < a.n) store1<DT>(out, j, v[j]);
  }
}

// Few rows (at most 16 MT): bound by W's bytes, read once.  One block a
// compute unit (MT = 1: two); the rows lie in LDS as bfloat16, laid out there
// by the block itself when they come as hidden states (XDT a float type; one
// launch less), 16 bytes behind each row so that the 16 rows of an operand read
// fall on different banks.  A wave takes TPW 16-row tiles of W at a time and
// keeps PC blocks of 128 columns of each in flight ahead of those it
// multiplies.  151936 x 1024: 1 row 26 us (5.9 TB/s of W), 64 rows 46.  The exact
// bfloat16 instruction has time enough here.
constexpr int kCodes = 2;  // XDT of rows that are laid out already
constexpr int kSkinnyWaves = 8;
constexpr uint32_t kTurn = 2048;  // bytes of LDS a wave turns W's tiles in
constexpr uint32_t kSkinnyLds = 135168 + kSkinnyWaves * kTurn;

template <int XDT>
__device__ __forceinline__ void stage_rows(const MatmulArgs& a, const QuantizeArgs& x, uint32_t rows,
                                           char* xs, uint32_t xp) {
  constexpr int U = 4;  // pieces of 8 columns in flight a thread
  const uint32_t per_row = a.pitch / 8, n = rows * per_row;  // 16 of them a block
  for (uint32_t t0 = threadIdx.x; t0 < n; t0 += U * kSkinnyWaves * 64) {
    float f[U][8];
    u32x2 codes[U];
    uint32_t biased[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t t = t0 + u * kSkinnyWaves * 64, r = t / per_row, c = (t - r * per_row) * 8;
      codes[u] = u32x2{0, 0};
      biased[u] = 127;
#pragma unroll
      for (int j = 0; j < 8; ++j) f[u][j] = 0.f;
      if (t >= n || r >= a.rows) continue;
      if constexpr (XDT == kCodes) {
        codes[u] = *(const u32x2*)(a.a + (size_t)r * a.pitch + c);
        biased[u] = a.as[(size_t)r * a.spitch + c / kFp8Block];
      } else {
        load8<XDT>(x, r, c, f[u]);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t t = t0 + u * kSkinnyWaves * 64, r = t / per_row, c = (t - r * per_row) * 8;
      if constexpr (XDT != kCodes) codes[u] = encode8(f[u], &biased[u]);
      if (t < n)
        *(u32x4*)(xs + r * xp + c * 2) =
            __builtin_bit_cast(u32x4, widen(codes[u][0], codes[u][1], scale_of(biased[u])));
    }
  }
}

template <int MT, int TPW, int PC, int XDT, int DT>
__global__ __launch_bounds__(kSkinnyWaves * 64) void k_skinny(MatmulArgs a, QuantizeArgs x) {
  static_assert(PC == 4, "a chunk's scales are one word");
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
  const uint32_t xp = a.pitch * 2 + 16, kb = a.pitch / kFp8Block, chunks = (kb + PC - 1) / PC;
  const uint32_t groups = (a.n + 16 * TPW - 1) / (16 * TPW);
  const uint32_t lo = (uint32_t)((uint64_t)groups * blockIdx.x / gridDim.x);
  const uint32_t hi = (uint32_t)((uint64_t)groups * (blockIdx.x + 1) / gridDim.x);
  char* turn = lds + wave * kTurn;
  char* xs = lds + kSkinnyWaves * kTurn;
  u32x4 buf[2][TPW][PC][2];
  uint32_t sbuf[2];
  static_assert(kFp8Block % (16 * TPW) == 0, "a group's rows of W lie in one block of 128");
  // Loads of one chunk (columns past the last block read the last again): 8 rows
  // of 128 bytes an instruction.  Lane l has piece l % 8 of rows l / 8 and
  // 8 + l / 8 of a tile.
  auto load = [&](u32x4 (&v)[TPW][PC][2], uint32_t& sw, uint32_t grp, uint32_t ch) {
#pragma unroll
    for (int t = 0; t < TPW; ++t) {
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const uint32_t row = (grp * TPW + t) * 16 + q * 8 + (lane >> 3);
        const uint8_t* p = a.w + (size_t)min(row, a.n - 1) * a.pitch + (lane & 7) * 16;
#pragma unroll
        for (int c = 0; c < PC; ++c)
          v[t][c][q] = __builtin_nontemporal_load(
              (const u32x4*)(p + min(ch * PC + c, kb - 1) * kFp8Block));
      }
    }
    sw = *(const uint32_t*)(a.ws + (size_t)(grp * TPW * 16 / kFp8Block) * a.spitch + ch * PC);
  };
  // A block of a tile in the operand's layout, by way of the wave's own 2 KB of
  // LDS (pieces exchanged by row, so that neither side's lanes share banks).
  const uint32_t put = (lane >> 3) * 128 + ((lane & 7) ^ (lane >> 3)) * 16;
  const uint32_t get = i * 128 + (g ^ (i & 7)) * 16;
  auto operand = [&](const u32x4 (&v)[2], u32x4 (&w)[2]) {
    *(u32x4*)(turn + put) = v[0];
    *(u32x4*)(turn + 1024 + put) = v[1];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // lanes read what others wrote
    w[0] = *(const u32x4*)(turn + get);
    w[1] = *(const u32x4*)(turn + (get ^ 64));
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  };
  uint32_t grp = lo + wave;
  if (grp < hi) load(buf[0], sbuf[0], grp, 0);
  stage_rows<XDT>(a, x, MT * 16, xs, xp);
  __syncthreads();
  f32x4 acc[TPW][MT];
  auto multiply = [&](const u32x4 (&v)[TPW][PC][2], uint32_t sw, uint32_t grp, uint32_t ch) {
    if (ch == 0) {
#pragma unroll
      for (int t = 0; t < TPW; ++t)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[t][m] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll
    for (int c = 0; c < PC; ++c) {
      const uint32_t b = ch * PC + c;
      if (b >= kb) break;
      u32x4 w[TPW][2];
#pragma unroll
      for (int t = 0; t < TPW; ++t) operand(v[t][c], w[t]);
#pragma unroll
      for (int q = 0; q < 2; ++q) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          bf16x8 xv[MT];
#pragma unroll
          for (int m = 0; m < MT; ++m)
            xv[m] = *(const bf16x8*)(xs + (m * 16 + i) * xp +
                                     (b * kFp8Block + q * 64 + g * 16 + h * 8) * 2);
#pragma unroll
          for (int t = 0; t < TPW; ++t) {
            const bf16x8 wv = widen(w[t][q][2 * h], w[t][q][2 * h + 1], scale_of(byte_of(sw, c)));
#pragma unroll
            for (int m = 0; m < MT; ++m)
              acc[t][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv, xv[m], acc[t][m], 0, 0, 0);
          }
        }
      }
    }
    if (ch + 1 == chunks) {
#pragma unroll
      for (int t = 0; t < TPW; ++t)
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          const uint32_t r = m * 16 + i, n = (grp * TPW + t) * 16 + g * 4;
          if (r < a.rows && n < a.n) store4<DT>(a, r, n, acc[t][m]);
        }
    }
  };
  uint32_t ch = 0;
  // Two chunks a turn: the buffers stay in registers by name.
  while (grp < hi) {
    uint32_t ng = grp, nc = ch + 1;
    if (nc == chunks) nc = 0, ng += kSkinnyWaves;
    if (ng < hi) load(buf[1], sbuf[1], ng, nc);
    multiply(buf[0], sbuf[0], grp, ch);
    grp = ng, ch = nc;
    if (grp >= hi) break;
    nc = ch + 1;
    if (nc == chunks) nc = 0, ng += kSkinnyWaves;
    if (ng < hi) load(buf[0], sbuf[0], ng, nc);
    multiply(buf[1], sbuf[1], grp, ch);
    grp = ng, ch = nc;
  }
}

// Many rows: bound by the matrix instructions and the write of the results.
// A block computes TN columns (rows of W) x TM rows in accumulators of WN x WM
// waves; blocks of 128 columns of both operands go from memory straight into
// LDS, one ahead of the one that is multiplied, and a block takes one tile
// after another so that a tile's first loads are under way while the last
// one's results are written.
// In LDS a row's eight 16-byte pieces are exchanged by its number mod 8, so that
// the 8 lanes that an LDS cycle serves read different banks.
// Sums are float32 whatever the results' type: the bfloat16 instruction on codes
// widened in registers (exact products; on normal numbers 1.3e-8 of the result's
// size off), in k_skinny's order, so that a row's results do not depend on the
// rows it comes with and bfloat16 ones are the float32 ones rounded.  The scaled
// 8-bit instruction takes 412 us where this takes 636, but its sums are off by
// 1.4e-5 of a normal result and up to 2^-12 of the terms' magnitudes: a result
// small against its terms is lost.
// 2048 rows of 151936 x 1024 to bfloat16: 636 us, 1.0 PFLOP/s, 1024 rows to float32
// 376; the matrix cores are busy 41%.  A wave widens the codes it multiplies, 192
// conversions beside 128 products a step; LDS is read 8 bytes a lane, a third of the
// time, half of that conflicts.
#if defined(__HIP_DEVICE_COMPILE__)  // the host compiler has no buffer descriptors
// Loads go through buffer descriptors: 32-bit offsets, and rows past a matrix'
// last read as zeros (the whole offset is in the vector register, so that the
// descriptor's range covers it).
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_of(const uint8_t* p, uint32_t row, uint32_t rows,
                                                          uint32_t most, uint32_t pitch) {
  const uint32_t left = min(rows - row, most) * pitch;  // most * pitch < 2^25
  return __builtin_amdgcn_make_buffer_rsrc((void*)(p + (size_t)row * pitch), 0, (int)left, 0x00020000);
}
#endif

template <int TN, int TM, int WN, int WM, int DT>
__global__ __launch_bounds__(WN* WM * 64) void k_tiles(MatmulArgs a, uint32_t tiles_m,
                                                        uint32_t places) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int WAVES = WN * WM, NT = TN / WN / 16, MT = TM / WM / 16;
  constexpr int LW = TN / 8 / WAVES, LX = TM / 8 / WAVES, STAGE = (TN + TM) * kFp8Block;
  static_assert(TN % (8 * WAVES) == 0 && TM % (8 * WAVES) == 0, "whole loads of either operand");
  static_assert(kFp8Block % (TN / WN) == 0 || (TN / WN) % kFp8Block == 0, "one scale of W a wave");
  constexpr int PIECES = NT * 2;  // of 16 bytes, of a row of a wave's results in bfloat16
  __shared__ __attribute__((aligned(1024))) uint8_t lds[2 * STAGE];
  __shared__ __attribute__((aligned(1024))) uint8_t turn[DT == TFE_BF16 ? WAVES * 16 * PIECES * 16 : 16];
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
  const uint32_t wn = (wave % WN) * (TN / WN), wm = (wave / WN) * (TM / WM);
  const uint32_t kb = a.pitch / kFp8Block;

  // Place t: all row tiles of a column tile one after another on one XCD
  // (blocks go to the 8 XCDs in turn), so that its part of W is read into one
  // L2.  Places beyond the last column are empty.
  struct Tile {
    uint32_t t, n, m;
  };
  auto find = [&](uint32_t t) {
    Tile r{t, 0, 0};
    for (; r.t < places; r.t += gridDim.x) {
      const uint32_t l = r.t >> 3, q = l / tiles_m;
      r.n = (q * 8 + (r.t & 7)) * TN;
      r.m = (l - q * tiles_m) * TM;
      if (r.n < a.n) break;
    }
    r.t = __builtin_amdgcn_readfirstlane(r.t);
    r.n = __builtin_amdgcn_readfirstlane(r.n);
    r.m = __builtin_amdgcn_readfirstlane(r.m);
    return r;
  };
  // A load instruction fills 8 rows of a stage: lane l piece l % 8 ^ l / 8 of row l / 8.
  const uint32_t from = (lane >> 3) * a.pitch + ((lane & 7) ^ (lane >> 3)) * 16;
  auto stage = [&](uint32_t to, const Tile& t, uint32_t b) {
    const auto w = rows_of(a.w, t.n, a.n, TN, a.pitch), x = rows_of(a.a, t.m, a.rows, TM, a.pitch);
#pragma unroll
    for (int c = 0; c < LW + LX; ++c) {
      const uint32_t row = ((c < LW ? c : c - LW) * WAVES + wave) * 8;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          c < LW ? w : x,
          (__attribute__((address_space(3))) void*)(lds + to + ((c < LW ? 0 : TN) + row) * kFp8Block), 16,
          (int)(from + row * a.pitch + b * kFp8Block), 0, 0, 0);
    }
  };
  // Scales of four blocks from b: the wave's part of W lies in one block of 128 rows.
  auto scales = [&](const Tile& t, uint32_t b, uint32_t& sw, uint32_t (&sx)[MT]) {
    const uint32_t row = min(t.n + wn, a.n - 1) / kFp8Block;
    sw = *(const __attribute__((address_space(4))) uint32_t*)(a.ws + (size_t)row * a.spitch + b);
    const auto x = rows_of(a.as, t.m, a.rows, TM, a.spitch);
#pragma unroll
    for (int m = 0; m < MT; ++m)
      sx[m] = __builtin_amdgcn_raw_buffer_load_b32(x, (int)((wm + m * 16 + i) * a.spitch + b), 0, 0);
  };

  Tile cur = find(blockIdx.x);
  if (cur.t >= places) return;
  uint32_t at = 0, sw = 0, sx[MT], sw_next, sx_next[MT];
  bool stored = false;
  // Piece p of row 16 k + i lies at slot p ^ (i & 7); p = g and g + 4 differ in one bit.
  const uint32_t slot = (g ^ (i & 7)) * 16;
  const uint32_t own_w = (wn + i) * kFp8Block + slot, own_x = (TN + wm + i) * kFp8Block + slot;
  stage(at, cur, 0);
  scales(cur, 0, sw_next, sx_next);
  while (true) {
    f32x4 acc[NT][MT];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int m = 0; m < MT; ++m) acc[n][m] = f32x4{0.f, 0.f, 0.f, 0.f};
    const Tile next = find(cur.t + gridDim.x);
    for (uint32_t b = 0; b < kb; ++b) {
      // The stage has arrived, and everybody is done with the other one (its reads
      // have returned: the count of LDS operations).  A tile's first stage was
      // asked for before the last tile's results were stored (at least eight
      // stores a lane, and memory operations complete in order): those need not
      // have landed.
      if (stored)
        asm volatile("s_waitcnt vmcnt(8) lgkmcnt(0)" ::: "memory");
      else
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
      stored = false;
      __builtin_amdgcn_s_barrier();
      // The scales have come too; told here, or the compiler waits for them, and so
      // for the next stage, where they are used.
#pragma unroll
      for (int m = 0; m < MT; ++m) asm volatile("" : "+v"(sx_next[m]));
      asm volatile("" : "+s"(sw_next));
      __builtin_amdgcn_sched_barrier(0);
      const uint32_t to = STAGE - at;
      const uint8_t* lw = lds + at + own_w;
      const uint8_t* lx = lds + at + own_x;
      const uint8_t* lw2 = lds + at + (own_w ^ 64);
      const uint8_t* lx2 = lds + at + (own_x ^ 64);
      at = to;
      if ((b & 3) == 0) {
        sw = sw_next;
#pragma unroll
        for (int m = 0; m < MT; ++m) sx[m] = sx_next[m];
      }
      if (b + 1 < kb) {
        stage(to, cur, b + 1);
        if ((b & 3) == 3) scales(cur, b + 1, sw_next, sx_next);
      } else if (next.t < places) {
        stage(to, next, 0);
        scales(next, 0, sw_next, sx_next);
      }
      __builtin_amdgcn_sched_barrier(0);
      const float fw = scale_of(sw & 255u);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        auto operand = [&](const uint8_t* p, const uint8_t* p2, int k, float f) {
          const u32x2 v = *(const u32x2*)((q < 2 ? p : p2) + (q & 1) * 8 + k * 16 * kFp8Block);
          return widen(v[0], v[1], f);
        };
        bf16x8 xv[MT];
#pragma unroll
        for (int m = 0; m < MT; ++m) xv[m] = operand(lx, lx2, m, scale_of(sx[m] & 255u));
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const bf16x8 wv = operand(lw, lw2, n, fw);
#pragma unroll
          for (int m = 0; m < MT; ++m)
            acc[n][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv, xv[m], acc[n][m], 0, 0, 0);
        }
      }
      sw >>= 8;
#pragma unroll
      for (int m = 0; m < MT; ++m) sx[m] >>= 8;
    }
    const uint32_t r0 = cur.m + wm + i, c0 = cur.n + wn + g * 4;
    if (cur.n + TN <= a.n && cur.m + TM <= a.rows) {
      if constexpr (DT == TFE_F32) {
        static_assert(NT * MT >= 8, "the next step's wait counts on eight stores");
        float* out = (float*)a.out + (size_t)r0 * a.ldo + c0;
#pragma unroll
        for (int m = 0; m < MT; ++m) {
#pragma unroll
          for (int n = 0; n < NT; ++n) store4_at<DT>((char*)(out + n * 16), acc[n][m]);
          out += (size_t)a.ldo * 16;
        }
      } else {
        // Sixteen rows at a time turn in the wave's own LDS, so that an instruction
        // writes whole pieces of 128 or 256 bytes: the results of a lane's row and
        // its three neighbours' are 64, and at an odd pitch two parts of lines.  us,
        // so / at once: 257 x 40001 x 1000 42 / 48, 1024 x 151937 x 256 162 / 227,
        // 1024 x 151936 x 256 123 / 161, 2048 x 151936 x 1024 636 / 746, 256 rows of it
        // 99 / 101.  float32 gains nothing from it (512 x 151937 x 1024: 242 / 241).
        constexpr int ROWS = 64 / PIECES;  // of an instruction
        static_assert(NT % 2 == 0, "column tiles in pairs");
        static_assert(MT * 16 / ROWS >= 8, "the next step's wait counts on eight stores");
        uint8_t* mine = turn + wave * (16 * PIECES * 16);
        // Pieces of 16 bytes are exchanged by row, as the operands' are.
        auto place = [&](uint32_t row, uint32_t piece) {
          return (u32x4*)(mine + (row * PIECES + (piece ^ (row & (PIECES - 1)))) * 16);
        };
        uint32_t own = lane;
        asm volatile("" : "+v"(own));  // the addresses are worked out here, not kept over the steps
        const uint32_t row = own / PIECES, piece = own % PIECES, oi = own & 15, og = own >> 4;
        uint16_t* out = (uint16_t*)a.out + (size_t)(cur.m + wm + row) * a.ldo + cur.n + wn + piece * 8;
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          // Neighbouring lane rows exchange halves of two column tiles: 16 bytes a lane.
#pragma unroll
          for (int n = 0; n < NT; n += 2) {
            const f32x4 p = acc[n][m], q = acc[n + 1][m];
            const auto lo = __builtin_amdgcn_permlane16_swap(pack2(p[0], p[1]), pack2(q[0], q[1]), false, false);
            const auto hi = __builtin_amdgcn_permlane16_swap(pack2(p[2], p[3]), pack2(q[2], q[3]), false, false);
            *place(oi, n * 2 + (og & 1) * 2 + (og >> 1)) = u32x4{lo[0], hi[0], lo[1], hi[1]};
          }
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
          for (int k = 0; k < 16; k += ROWS) {
            *(u32x4_a2*)out = *place(row + k, piece);
            out += (size_t)a.ldo * ROWS;
          }
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
      }
      stored = true;
    } else {
      stored = false;
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n)
          if (r0 + m * 16 < a.rows && c0 + n * 16 < a.n)
            store4<DT>(a, r0 + m * 16, c0 + n * 16, acc[n][m]);
    }
    if (next.t >= places) break;
    cur = next;
  }
#endif
}

// ---- launches ------------------------------------------------------------------

uint32_t skinny_lds(const MatmulArgs& a) {
  const uint32_t mt = (a.rows + 15) / 16;
  return mt * 16 * (a.pitch * 2 + 16) + kSkinnyWaves * kTurn;
}

template <int MT, int TPW, int PC, int XDT, int DT>
hipError_t skinny(const MatmulArgs& a, const QuantizeArgs& x, hipStream_t s) {
  const uint32_t lds = skinny_lds(a), groups = (a.n + 16 * TPW - 1) / (16 * TPW);
  auto* k = k_skinny<MT, TPW, PC, XDT, DT>;
  // Once for each device: more LDS than a kernel may have by default.
  static std::atomic<uint64_t> told{0};
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (dev > 63 || !(told.load(std::memory_order_relaxed) & bit)) {
    e = hipFuncSetAttribute((const void*)k, hipFuncAttributeMaxDynamicSharedMemorySize, (int)kSkinnyLds);
    if (e != hipSuccess) return e;
    told.fetch_or(bit, std::memory_order_relaxed);
  }
  const uint32_t most = (uint32_t)compute_units() * (lds <= 81920 ? 2 : 1);
  const uint32_t want = (groups + kSkinnyWaves - 1) / kSkinnyWaves;
  k<<<dim3(std::min(most, want)), dim3(kSkinnyWaves * 64), lds, s>>>(a, x);
  return hipGetLastError();
}
template <int XDT, int DT>
hipError_t skinny_rows(const MatmulArgs& a, const QuantizeArgs& x, hipStream_t s) {
  switch ((a.rows + 15) / 16) {
    case 1: return skinny<1, 1, 4, XDT, DT>(a, x, s);
    case 2: return skinny<2, 2, 4, XDT, DT>(a, x, s);
    case 3: return skinny<3, 2, 4, XDT, DT>(a, x, s);
    default: return skinny<4, 2, 4, XDT, DT>(a, x, s);
  }
}

template <int TN, int TM, int WN, int WM>
hipError_t tiles(const MatmulArgs& a, int dt, int blocks_per_cu, hipStream_t s) {
  const uint32_t tn = (a.n + TN - 1) / TN, tm = (a.rows + TM - 1) / TM;
  const uint32_t places = (tn + 7) / 8 * 8 * tm;
  const uint32_t most = (uint32_t)(compute_units() * blocks_per_cu + 7) / 8 * 8;
  const dim3 grid(std::min(places, most)), block(WN * WM * 64);
  if (dt == TFE_F32)
    k_tiles<TN, TM, WN, WM, TFE_F32><<<grid, block, 0, s>>>(a, tm, places);
  else
    k_tiles<TN, TM, WN, WM, TFE_BF16><<<grid, block, 0, s>>>(a, tm, places);
  return hipGetLastError();
}

// us with the rows in LDS / in tiles, 151936 x 1024 to float32: 16 rows 33 / 48, 32 37 / 47,
// 48 41 / 48, 64 46 / 50 (x 256: 24 / 20); 16 rows of 151936 x 2048 57 / 99.  Rows that do
// not fit go to tiles: 64 of 151936 x 1152 55, 48 of x 1408 61.
bool is_skinny(const MatmulArgs& a) { return a.rows <= 64 && skinny_lds(a) <= kSkinnyLds; }

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
  if (is_skinny(a))
    return out_dtype == TFE_F32 ? skinny_rows<kCodes, TFE_F32>(a, QuantizeArgs{}, s)
                                : skinny_rows<kCodes, TFE_BF16>(a, QuantizeArgs{}, s);
  // Large tiles where they fill the device and waste few rows.  us at 151936 x 1024,
  // 256 x 256 / 128 x 128: bfloat16 256 rows 110 / 101, 512 176 / 182, 1024 339 / 355, 2048
  // 636 / 692; float32 256 rows 128 / 107, 512 199 / 196, 1024 376 / 379.  257 x 40001 x 1000
  // (two row tiles of 256 against three of 128): 63 / 37.
  const uint32_t r256 = (a.rows + 255) / 256, r128 = (a.rows + 127) / 128;
  const bool fills = (uint64_t)((a.n + 255) / 256) * r256 >= (uint64_t)compute_units() * 2;
  if (fills && a.rows > 256 && r256 * 2 * 92 <= r128 * 100)
    return tiles<256, 256, 2, 4>(a, out_dtype, 1, s);
  return tiles<128, 128, 2, 2>(a, out_dtype, 2, s);
}

hipError_t launch_fp8_linear(const QuantizeArgs& x, const MatmulArgs& a, int dtype, int out_dtype,
                             hipStream_t s) {
  if (is_skinny(a)) {
    if (dtype == TFE_F32)
      return out_dtype == TFE_F32 ? skinny_rows<TFE_F32, TFE_F32>(a, x, s)
                                  : skinny_rows<TFE_F32, TFE_BF16>(a, x, s);
    return out_dtype == TFE_F32 ? skinny_rows<TFE_BF16, TFE_F32>(a, x, s)
                                : skinny_rows<TFE_BF16, TFE_BF16>(a, x, s);
  }
  const hipError_t e = launch_fp8_quantize(x, dtype, 1, s);
  return e == hipSuccess ? launch_fp8_matmul(a, out_dtype, s) : e;
}

}  // namespace tfe
