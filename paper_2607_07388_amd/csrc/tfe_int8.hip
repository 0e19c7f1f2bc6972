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

// More rows: bound by the matrix cores, the results' conversion and their stores.  2048 rows of
// 151936 x 1024 to bfloat16 388 us, 1.6 POP/s (2.4 where the sums were left where they are, 2.0
// where the results were not stored); integers' sums are exact, so no widening stands beside them.
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
  bool more = true;
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
          // They pass by (2048 rows of 151936 x 1024 on one input over and over: 373 us, 334 so).
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
        more = find(at, &np0, &nq0);
        if (more) *s = segment(np0, nq0);
        return more;
      },
      [&](uint32_t odd) {
        char* to = lds + T::LDS + odd * INFO;
        static_assert(TP / 64 <= T::WAVES && TQ / 64 <= T::WAVES, "a wave for each 64 scales");
        if (t.wave < TQ / 64) gemm::load_numbers(a.as, q0, a.rows, t.wave, to);
        if (t.wave < TP / 64) gemm::load_numbers(a.ws, p0, a.n, t.wave, to + TQ * 4);
        // The next tile's part of W: its row tiles' blocks share it out.  A tile's steps are few,
        // and each waits for W's first reader: 2048 rows of 151936 x 1024 450 us without, 388 so.
        if (T::LARGE && more && np0 != p0)
          gemm::warm<T::THREADS>(segment(np0, nq0).p, TP, a.pitch, nq0 / TQ, b.tiles_q,
                                 lds + T::LDS + 2 * INFO + t.wave * 256);
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

// More LDS than a kernel may have by default: told once for each device.
template <class K> hipError_t allow(K* k, int bytes, std::atomic<uint64_t>* told) {
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (dev > 63 || !(told->load(std::memory_order_relaxed) & bit)) {
    e = hipFuncSetAttribute((const void*)k, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
    told->fetch_or(bit, std::memory_order_relaxed);
  }
  return hipSuccess;
}

template <int TP, int TQ, int WP, int WQ, int DT>
hipError_t tiles(const Int8MatmulArgs& m, hipStream_t s) {
  typedef Tile<Int8, TP, TQ, WP, WQ, false, false, false> T;
  auto* k = k_int8_tiles<TP, TQ, WP, WQ, DT>;
  constexpr int LDS = T::LDS + 2 * (TP + TQ) * 4 + (T::LARGE ? T::WAVES * 256 : 0);
  static std::atomic<uint64_t> told{0};
  const hipError_t e = allow(k, LDS, &told);
  if (e != hipSuccess) return e;
  TileArgs a{m, (m.rows + TQ - 1) / TQ, 0};
  a.total = ((m.n + TP - 1) / TP * a.tiles_q + 7) / 8 * 8;
  k<<<dim3(std::min<uint32_t>(a.total, (compute_units() * (163840 / LDS) + 7) / 8 * 8)), dim3(T::THREADS), LDS, s>>>(a);
  return hipGetLastError();
}

// Few rows (at most 16 MT): bound by W's bytes, read once, as the other 8-bit product of few
// rows.  The rows' codes lie in LDS, 16 bytes behind each so that the 16 rows of an operand
// read fall on different banks; a wave takes TPW 16-row tiles of W at a time, 8 rows of
// 128 bytes a load instruction, and keeps PC blocks of 128 columns of each in flight ahead of
// those it multiplies.  With XDT a float type the rows are hidden states, laid out by every block
// itself beside its first loads of W: one launch less.  151936 x 1024 to float32: 1 row 26 us
// (6.0 TB/s of W), 64 rows 39 and their layout 5.
constexpr int kCodes = 2;  // XDT of rows that are laid out already
constexpr int kSkinnyWaves = 8;
constexpr uint32_t kTurn = 2048;  // bytes of LDS a wave turns W's tiles in
constexpr uint32_t kSkinnyLds = 135168 + kSkinnyWaves * kTurn;
constexpr uint32_t kPrepared = 16;  // rows that every block lays out itself

struct SkinnyArgs {
  Int8MatmulArgs m;
  Int8QuantizeArgs x;
};

// A wave lays rows out: a lane has 8 columns of each 512, the row's first PER x 512 in registers.
template <int DT>
__device__ __forceinline__ void stage_row(const Int8QuantizeArgs& x, uint32_t row, uint32_t lane, char* to,
                                          float* scale) {
  constexpr int PER = 2;
  const char* in = (const char*)x.x + (size_t)row * x.ldx * sizeof(typename Elem<DT>::T);
  float f[PER][8], top = 0.f;
  bool nan = false;
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    load8<DT>(in, x.dim, k * 512 + lane * 8, f[k]);
    largest8(f[k], &top, &nan);
  }
  for (uint32_t c = PER * 512 + lane * 8; c < x.dim; c += 512) {
    float g[8];
    load8<DT>(in, x.dim, c, g);
    largest8(g, &top, &nan);
  }
  top = wave_max(top);
  nan = __builtin_amdgcn_ballot_w64(nan) != 0;
  const bool some = top > kInt8Least;
  const float inverse = some ? 1.f / top * 127.f : 0.f;
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const uint32_t c = k * 512 + lane * 8;
    if (c < x.pitch) *(u32x2*)(to + c) = some ? codes8(f[k], inverse) : u32x2{0, 0};
  }
  for (uint32_t c = PER * 512 + lane * 8; c < x.pitch; c += 512) {
    float g[8];
    load8<DT>(in, x.dim, c, g);
    *(u32x2*)(to + c) = some ? codes8(g, inverse) : u32x2{0, 0};
  }
  if (lane == 0) *scale = nan ? NAN : some ? top / 127.f : 0.f;
}

template <int MT, int TPW, int PC, int XDT, int DT>
__global__ __launch_bounds__(kSkinnyWaves * 64) void k_int8_skinny(SkinnyArgs b) {
  typedef typename Elem<DT>::T E;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  __shared__ float scales[MT * 16];
  const Int8MatmulArgs& a = b.m;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
  const uint32_t xp = a.pitch + 16, kb = a.pitch / 128, chunks = (kb + PC - 1) / PC;
  const uint32_t groups = (a.n + 16 * TPW - 1) / (16 * TPW);
  const uint32_t lo = (uint32_t)((uint64_t)groups * blockIdx.x / gridDim.x);
  const uint32_t hi = (uint32_t)((uint64_t)groups * (blockIdx.x + 1) / gridDim.x);
  char* turn = lds + wave * kTurn;
  char* xs = lds + kSkinnyWaves * kTurn;
  u32x4 buf[2][TPW][PC][2];
  f32x4 ws[2][TPW];
  // Loads of one chunk (columns past the last block read the last again): lane l has piece
  // l % 8 of rows l / 8 and 8 + l / 8 of a tile.
  auto load = [&](u32x4 (&v)[TPW][PC][2], f32x4 (&w)[TPW], uint32_t grp, uint32_t ch) {
#pragma unroll
    for (int t = 0; t < TPW; ++t) {
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const uint32_t row = (grp * TPW + t) * 16 + q * 8 + (lane >> 3);
        const char* p = (const char*)a.w + (size_t)min(row, a.n - 1) * a.pitch + (lane & 7) * 16;
#pragma unroll
        for (int c = 0; c < PC; ++c)
          v[t][c][q] = __builtin_nontemporal_load((const u32x4*)(p + min(ch * PC + c, kb - 1) * 128));
      }
      // The columns' scales, with their last chunk.
      if (ch + 1 == chunks) {
        const uint32_t n = (grp * TPW + t) * 16 + g * 4;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[t][j] = a.ws[min(n + j, a.n - 1)];
      }
    }
  };
  // A block of a tile in the operand's layout, by way of the wave's own 2 KB of LDS (pieces
  // exchanged by row, so that neither side's lanes share banks).
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
  if (grp < hi) load(buf[0], ws[0], grp, 0);
  if constexpr (XDT == kCodes) {
    const uint32_t per = a.pitch / 16;
    for (uint32_t t = threadIdx.x; t < MT * 16 * per; t += kSkinnyWaves * 64) {
      const uint32_t r = t / per, c = (t - r * per) * 16;
      *(u32x4*)(xs + r * xp + c) = r < a.rows ? *(const u32x4*)(a.a + (size_t)r * a.pitch + c) : u32x4{0, 0, 0, 0};
    }
    if (threadIdx.x < MT * 16) scales[threadIdx.x] = threadIdx.x < a.rows ? a.as[threadIdx.x] : 0.f;
  } else {
    for (uint32_t r = wave; r < a.rows; r += kSkinnyWaves) stage_row<XDT>(b.x, r, lane, xs + r * xp, scales + r);
    const uint32_t per = a.pitch / 16, from = a.rows * per;
    for (uint32_t t = from + threadIdx.x; t < MT * 16 * per; t += kSkinnyWaves * 64)
      *(u32x4*)(xs + t / per * xp + t % per * 16) = u32x4{0, 0, 0, 0};
  }
  __syncthreads();
  i32x4 acc[TPW][MT];
  auto multiply = [&](const u32x4 (&v)[TPW][PC][2], const f32x4 (&sw)[TPW], uint32_t grp, uint32_t ch) {
    if (ch == 0) {
#pragma unroll
      for (int t = 0; t < TPW; ++t)
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[t][m] = i32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int c = 0; c < PC; ++c) {
      const uint32_t blk = ch * PC + c;
      if (blk >= kb) break;
      u32x4 w[TPW][2];
#pragma unroll
      for (int t = 0; t < TPW; ++t) operand(v[t][c], w[t]);
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        u32x4 xv[MT];
#pragma unroll
        for (int m = 0; m < MT; ++m)
          xv[m] = *(const u32x4*)(xs + (m * 16 + i) * xp + blk * 128 + q * 64 + g * 16);
#pragma unroll
        for (int t = 0; t < TPW; ++t)
#pragma unroll
          for (int m = 0; m < MT; ++m) acc[t][m] = gemm::multiply<Int8>(w[t][q], xv[m], acc[t][m]);
      }
    }
    if (ch + 1 == chunks) {
#pragma unroll
      for (int t = 0; t < TPW; ++t)
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          const uint32_t r = m * 16 + i, n = (grp * TPW + t) * 16 + g * 4;
          if (r >= a.rows) continue;
          const float x = scales[r];
          f32x4 y;
#pragma unroll
          for (int j = 0; j < 4; ++j) y[j] = (float)acc[t][m][j] * x * sw[t][j];
          E* out = (E*)a.out + (size_t)r * a.ldo + n;
          typedef f32x4 f4 __attribute__((aligned(4)));
          typedef u32x2 u2 __attribute__((aligned(2)));
          if (n + 4 <= a.n) {
            if constexpr (DT == TFE_F32)
              *(f4*)out = y;
            else
              *(u2*)out = u2{pack2(y[0], y[1]), pack2(y[2], y[3])};
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (n + j < a.n) store1<DT>(out, j, y[j]);
          }
        }
    }
  };
  uint32_t ch = 0;
  // Two chunks a turn: the buffers stay in registers by name.
  while (grp < hi) {
    uint32_t ng = grp, nc = ch + 1;
    if (nc == chunks) nc = 0, ng += kSkinnyWaves;
    if (ng < hi) load(buf[1], ws[1], ng, nc);
    multiply(buf[0], ws[0], grp, ch);
    grp = ng, ch = nc;
    if (grp >= hi) break;
    nc = ch + 1;
    if (nc == chunks) nc = 0, ng += kSkinnyWaves;
    if (ng < hi) load(buf[0], ws[0], ng, nc);
    multiply(buf[1], ws[1], grp, ch);
    grp = ng, ch = nc;
  }
}

uint32_t skinny_lds(const Int8MatmulArgs& a) {
  return (a.rows + 15) / 16 * 16 * (a.pitch + 16) + kSkinnyWaves * kTurn;
}
bool is_skinny(const Int8MatmulArgs& a) { return a.rows <= 64 && skinny_lds(a) <= kSkinnyLds; }

template <int MT, int TPW, int PC, int XDT, int DT>
hipError_t skinny(const Int8MatmulArgs& a, const Int8QuantizeArgs& x, hipStream_t s) {
  const uint32_t lds = skinny_lds(a), groups = (a.n + 16 * TPW - 1) / (16 * TPW);
  auto* k = k_int8_skinny<MT, TPW, PC, XDT, DT>;
  static std::atomic<uint64_t> told{0};
  const hipError_t e = allow(k, (int)kSkinnyLds, &told);
  if (e != hipSuccess) return e;
  const uint32_t most = (uint32_t)compute_units() * (lds <= 81000 ? 2 : 1);
  const uint32_t want = (groups + kSkinnyWaves - 1) / kSkinnyWaves;
  k<<<dim3(std::min(most, want)), dim3(kSkinnyWaves * 64), lds, s>>>(SkinnyArgs{a, x});
  return hipGetLastError();
}
template <int DT> hipError_t skinny_rows(const Int8MatmulArgs& a, hipStream_t s) {
  switch ((a.rows + 15) / 16) {
    case 1: return skinny<1, 1, 4, kCodes, DT>(a, Int8QuantizeArgs{}, s);
    case 2: return skinny<2, 2, 4, kCodes, DT>(a, Int8QuantizeArgs{}, s);
    case 3: return skinny<3, 2, 4, kCodes, DT>(a, Int8QuantizeArgs{}, s);
    default: return skinny<4, 2, 4, kCodes, DT>(a, Int8QuantizeArgs{}, s);
  }
}

// Tiles of 256 x 256 where they fill the device and waste few rows, of 128 x 64 where those
// of 128 x 128 would not fill it.  us in tiles of 64 / 128 / 256 rows, dim 1024: 64 rows of 151936
// to float32 36 / 41 / 63; to bfloat16 100 rows of 20000 12 / 14 / 23, of 151936 45 / 41 / 59; 200 rows
// of 151936 69 / 67 / 71, 257 87 / 84 / 90, 400 120 / 109 / 99, 600 174 / 147 / 132; 700 rows of 3000
// 13 / 15 / 26, of 20000 30 / 31 / 32; 1024 rows of 151936 to float32 436 / 372 / 250.
template <int DT> hipError_t matmul(const Int8MatmulArgs& a, hipStream_t s) {
  if (is_skinny(a)) return skinny_rows<DT>(a, s);
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
  if (a.rows <= kPrepared && is_skinny(a)) {
    if (dtype == TFE_F32)
      return out_dtype == TFE_F32 ? skinny<1, 1, 4, TFE_F32, TFE_F32>(a, x, s)
                                  : skinny<1, 1, 4, TFE_F32, TFE_BF16>(a, x, s);
    return out_dtype == TFE_F32 ? skinny<1, 1, 4, TFE_BF16, TFE_F32>(a, x, s)
                                : skinny<1, 1, 4, TFE_BF16, TFE_BF16>(a, x, s);
  }
  const hipError_t e = launch_int8_quantize(x, dtype, s);
  return e == hipSuccess ? launch_int8_matmul(a, out_dtype, s) : e;
}

}  // namespace tfe
