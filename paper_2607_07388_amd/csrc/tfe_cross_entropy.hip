// Softmax cross entropy of the head's logits z = H W^T (H the hidden states
// [rows x dim], W the projection [vocab x dim], bfloat16), which are computed
// in tiles and not kept:
//   lse_r = log sum_v exp z_rv,  loss_r = lse_r - z_rt,
//   dz_rv = weight_r (exp(z_rv - lse_r) - [v = t]),  dH = dz W,  dW = dz^T H.
#include <float.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <atomic>

#include "tfe_gemm.h"
#include "tfe_learn.h"
#include "tfe_rows.h"

namespace tfe {
namespace {

using gemm::Bf16;
using gemm::Operand;
using gemm::Tile;
using rows::pack2;
using rows::u32x4;
typedef gemm::f32x4 f32x4;
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// A matrix in memory as the tiles read it.
struct Matrix {
  const uint16_t* at;
  uint32_t ld, rows, cols;
};
__device__ __forceinline__ Operand along(const Matrix& m, uint32_t row) {
  return Operand{(const char*)(m.at + (size_t)row * m.ld), m.ld * 2, m.rows > row ? m.rows - row : 0u, m.cols, 0, 0};
}
__device__ __forceinline__ Operand across(const Matrix& m, uint32_t col) {
  return Operand{(const char*)(m.at + col), m.ld * 2, m.rows, m.cols > col ? m.cols - col : 0u, 0, 0};
}

// dz of a piece of the vocabulary, in blocks of 2^log rows x 64 columns, `blocks` beside
// each other: 128 bytes of each of 4096 rows a long pitch apart took the products that
// read them 20 us longer of 235, and writing them 30 of 285.
struct Dz {
  uint16_t* at;
  uint64_t plane;  // elements to the next numbers of float32 gradients
  uint32_t log, blocks, rows, cols;  // rows and columns of whole blocks
  __device__ __forceinline__ size_t block(uint32_t row, uint32_t col) const {
    return ((size_t)(row >> log) * blocks + (col >> 6)) * (gemm::block_bytes(log) / 2);
  }
  // Steps [s0, s1) of `row`'s tile, k along the rows.
  __device__ __forceinline__ Operand along(uint32_t p, uint32_t row, uint32_t s1) const {
    return Operand{(const char*)(at + p * plane + block(row, 0)), 128, 1u << log, min(cols, s1 * 64), log, blocks};
  }
  __device__ __forceinline__ Operand across(uint32_t p, uint32_t col) const {
    return Operand{(const char*)(at + p * plane + block(0, col)), 128, rows, cols - col, log, blocks};
  }
};

// Blocks go to the 8 XCDs in turn; place t of them as if each XCD took a run of
// neighbouring places, so that those share its L2.  `total` is a multiple of 8.
__device__ __forceinline__ uint32_t place_of(uint32_t t, uint32_t total) {
  return (t & 7) * (total >> 3) + (t >> 3);
}

// ---- rows in aligned order -------------------------------------------------------

// Copies rows, with zeros behind their columns; rows whose target is none or
// whose weight is 0 (targets given) become zeros, so that whatever they hold
// takes no part in dW.
struct PackArgs {
  const uint16_t* x;
  int64_t ldx;
  uint32_t rows, cols, pitch;
  const int32_t* targets;
  const float* weight;
  uint32_t vocab;
  uint16_t* out;
};
template <int THREADS> __device__ __forceinline__ void packed(const PackArgs& a, uint32_t block, uint32_t blocks) {
  const uint32_t per = a.pitch / 8;
  const uint64_t n = (uint64_t)a.rows * per;
  for (uint64_t at = (uint64_t)block * THREADS + threadIdx.x; at < n; at += (uint64_t)blocks * THREADS) {
    const uint32_t r = (uint32_t)(at / per), c = (uint32_t)(at - (uint64_t)r * per) * 8;
    u32x4 v{0, 0, 0, 0};
    const bool none = a.targets && ((uint32_t)a.targets[r] >= a.vocab || (a.weight && a.weight[r] == 0.f));
    if (!none) {
      const uint16_t* x = a.x + (size_t)r * a.ldx + c;
      if (c + 8 <= a.cols) {
        v = *(const rows::u32x4_a2*)x;
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (c + j < a.cols) v[j / 2] |= (uint32_t)x[j] << (16 * (j & 1));
      }
    }
    *(u32x4*)(a.out + (size_t)r * a.pitch + c) = v;
  }
}
__global__ __launch_bounds__(256) void k_pack(PackArgs a) { packed<256>(a, blockIdx.x, gridDim.x); }

// ---- logits: their sums, or dz -----------------------------------------------------

// Bound by the matrix cores, which k_sums keeps 66% busy and the gradients' products 52 to 56%
// (a wave's registers hold 128 x 64 sums: a larger tile does not fit, and each step reads 192 KB
// of LDS), and by what
// follows a tile's products: exponentials (16 cycles a wave) beside maxima and sums, and dz's
// stores.  4096 rows of 151936 x 1024 on one input over and over: sums 1060 us (1.2 PFLOP/s; 840
// without what follows the products), dz of 32768 columns 265 (195).  Few rows: bound by W's
// bytes, 64 rows 53 to 61 us for 311 MB.

struct LogitsArgs {
  Matrix w, h;      // h: the rows of this launch
  uint32_t tiles_q, total;
  uint32_t vocab0;  // of w's first row
  const int32_t* targets;
  // sums
  f32x2* part;      // [slab][rows of the launch]
  uint32_t slab0;
  float* picked;    // the target's logit
  // dz
  const float* lse;
  const float* weight;
  uint32_t vocab;
  Dz dz;
  float* rest;      // what the rounding of a row's dz at its target leaves
};

// Tile t of a launch: its first column and row; false behind the last.
__device__ __forceinline__ bool logits_tile(const LogitsArgs& a, uint32_t t, uint32_t tp, uint32_t tq,
                                            uint32_t* p0, uint32_t* q0) {
  if (t >= a.total) return false;
  const uint32_t place = place_of(t, a.total);
  *p0 = place / a.tiles_q * tp;
  *q0 = place % a.tiles_q * tq;
  return *p0 < a.w.rows;
}
__device__ __forceinline__ gemm::Segment logits_segment(const LogitsArgs& a, uint32_t p0, uint32_t q0) {
  return gemm::Segment{along(a.w, p0), along(a.h, q0), 0, (a.w.cols * 2 + gemm::kStep - 1) / gemm::kStep};
}
// What a tile's rows have: targets, and for dz lse and weights, T::TQ numbers each.
template <int TQ> constexpr int kInfo = TQ * 12;

// A block's tiles: t, t + the grid and so on.  Places behind the last column
// are at the end of the last XCD's run, where a block's later tiles are too.
// done(p0, q0, info) has the rows' numbers in LDS.
template <class T, int TP, int TQ, int STORES, bool DZ, class Done>
__device__ __forceinline__ void logits_tiles(const LogitsArgs& a, T& tile, char* lds, Done done) {
  uint32_t t = blockIdx.x, p0, q0, np0 = 0, nq0 = 0;
  if (!logits_tile(a, t, TP, TQ, &p0, &q0)) return;
  tile.clear();
  tile.template run<STORES>(
      logits_segment(a, p0, q0),
      [&](gemm::Segment* s) {
        t += gridDim.x;
        const bool more = logits_tile(a, t, TP, TQ, &np0, &nq0);
        if (more) *s = logits_segment(a, np0, nq0);
        return more;
      },
      [&](uint32_t odd) {
        char* to = lds + T::LDS + odd * kInfo<TQ>;
        static_assert(T::WAVES * 64 >= TQ, "a wave for each 64 rows");
        if (tile.wave < TQ / 64) {
          gemm::load_numbers(a.targets, q0, a.h.rows, tile.wave, to);
          if (DZ) {
            gemm::load_numbers(a.lse, q0, a.h.rows, tile.wave, to + TQ * 4);
            if (a.weight) gemm::load_numbers(a.weight, q0, a.h.rows, tile.wave, to + TQ * 8);
          }
        }
      },
      [&](uint32_t odd) {
        const bool stored = done(p0, q0, lds + T::LDS + odd * kInfo<TQ>);
        p0 = np0;
        q0 = nq0;
        tile.clear();
        return stored;
      },
      lds);
}

// Columns of a slab: those of one wave.
constexpr int kSlab = 128;

template <int TP, int TQ, int WP, int WQ>
__global__ __launch_bounds__(WP* WQ * 64) void k_sums(LogitsArgs a) {
  typedef Tile<Bf16, TP, TQ, WP, WQ, false, false, false> T;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  T t;
  static_assert(TP / WP == kSlab, "a wave's columns are a slab");
  logits_tiles<T, TP, TQ, 0, false>(a, t, lds, [&](uint32_t p0, uint32_t q0, const char* info) {
    const uint32_t c0 = p0 + t.wp + t.g * 4, slab = a.slab0 + (p0 + t.wp) / kSlab;
    if (p0 + t.wp + kSlab > a.w.rows) {
#pragma unroll
      for (int n = 0; n < t.NT; ++n)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (c0 + n * 16 + j >= a.w.rows)
#pragma unroll
            for (int m = 0; m < t.MT; ++m) t.acc[n][m][j] = -INFINITY;
    }
#pragma unroll
    for (int m = 0; m < t.MT; ++m) {
      const uint32_t in = t.wq + m * 16 + t.i, r = q0 + in;
      float top = -FLT_MAX, sum = 0.f;
#pragma unroll
      for (int n = 0; n < t.NT; ++n)
#pragma unroll
        for (int j = 0; j < 4; ++j) top = fmaxf(top, t.acc[n][m][j]);
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
#pragma unroll
      for (int n = 0; n < t.NT; ++n)
#pragma unroll
        for (int j = 0; j < 4; ++j) sum += __expf(t.acc[n][m][j] - top);
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      if (r < a.h.rows) {
        if (t.g == 0 && p0 + t.wp < a.w.rows) a.part[(size_t)slab * a.h.rows + r] = f32x2{top, sum};
        const uint32_t at = ((const uint32_t*)info)[in] - a.vocab0 - c0;
        if (at < (uint32_t)kSlab && (at & 12) == 0) {
          float z = 0.f;
#pragma unroll
          for (int n = 0; n < t.NT; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j) z = at == (uint32_t)(n * 16 + j) ? t.acc[n][m][j] : z;
          if (c0 + at < a.w.rows) a.picked[r] = z;
        }
      }
    }
    return false;
  });
}

// A block joins the slabs of 16 rows.
struct JoinArgs {
  const f32x2* part;
  uint32_t slabs, rows, vocab;
  const int32_t* targets;
  const float* picked;
  float* loss;
  float* lse;
};
__device__ __forceinline__ f32x2 joined(f32x2 x, f32x2 y) {
  const float top = fmaxf(x[0], y[0]);
  return f32x2{top, x[1] * __expf(x[0] - top) + y[1] * __expf(y[0] - top)};
}
__global__ __launch_bounds__(1024) void k_join(JoinArgs a) {
  constexpr int LANES = 64, DEEP = 8;  // slabs of a row at a time, and of a thread under way
  __shared__ f32x2 red[LANES][17];
  const uint32_t i = threadIdx.x & 15, y = threadIdx.x >> 4, r = blockIdx.x * 16 + i;
  const f32x2 none{-FLT_MAX, 0.f};
  f32x2 sum = none;
  if (r < a.rows)
    for (uint32_t k = y; k < a.slabs; k += LANES * DEEP) {
      f32x2 v[DEEP];
#pragma unroll
      for (uint32_t j = 0; j < DEEP; ++j)
        v[j] = k + j * LANES < a.slabs ? a.part[(size_t)(k + j * LANES) * a.rows + r] : none;
#pragma unroll
      for (int j = 0; j < DEEP; ++j) sum = joined(sum, v[j]);
    }
  red[y][i] = sum;
  __syncthreads();
#pragma unroll 1
  for (uint32_t half = LANES / 2; half; half >>= 1) {
    if (y < half) red[y][i] = joined(red[y][i], red[y + half][i]);
    __syncthreads();
  }
  if (y != 0 || r >= a.rows) return;
  const float top = red[0][i][0], rest = logf(red[0][i][1]);
  a.lse[r] = top + rest;
  a.loss[r] = (uint32_t)a.targets[r] < a.vocab ? (top - a.picked[r]) + rest : 0.f;
}

// Numbers of bfloat16 that a number of dz is the sum of: float32 gradients take three, whose
// 24 bits are its own.  With two, dH and dW of few rows over 1000 tokens were off by up to 1.3e-6
// of their norm, where products of dz in float32 are by 4.6e-7; with three by up to 7e-7, the
// logits' own error.  257 rows of 40001 x 999 take 375 us, with two 330.
constexpr uint32_t planes_of(bool f32) { return f32 ? 3 : 1; }

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

template <int TP, int TQ, int WP, int WQ, int PLANES>
__global__ __launch_bounds__(WP* WQ * 64) void k_dz(LogitsArgs a) {
  typedef Tile<Bf16, TP, TQ, WP, WQ, false, false, false> T;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  T t;
  constexpr int STORES = T::MT * T::NT / 2 * PLANES;
  logits_tiles<T, TP, TQ, STORES, true>(a, t, lds, [&](uint32_t p0, uint32_t q0, const char* info) {
    const uint32_t c0 = p0 + t.wp + t.g * 4;
    // Whole blocks are written: zeros beyond the vocabulary and the rows.
    const bool ends = p0 + TP > a.w.rows;
    uint16_t* const tile = a.dz.at + a.dz.block(q0, p0 + t.wp) + piece_of(t.g);
#pragma unroll
    for (int m = 0; m < t.MT; ++m) {
      const uint32_t in = t.wq + m * 16 + t.i;
      const uint32_t target = ((const uint32_t*)info)[in];
      const float lse = ((const float*)info)[TQ + in];
      const float given = a.weight ? ((const float*)info)[2 * TQ + in] : 1.f;
      const float weight = target < a.vocab && q0 + in < a.h.rows ? given : 0.f;
      const uint32_t at = target - a.vocab0 - c0;
      const bool hit = at < (uint32_t)(TP / WP) && (at & 12) == 0;
#pragma unroll
      for (int n = 0; n < t.NT; ++n)
#pragma unroll
        for (int j = 0; j < 4; ++j) t.acc[n][m][j] = __expf(t.acc[n][m][j] - lse);
      if (__builtin_amdgcn_ballot_w64(hit)) {
#pragma unroll
        for (int n = 0; n < t.NT; ++n)
#pragma unroll
          for (int j = 0; j < 4; ++j) t.acc[n][m][j] -= at == (uint32_t)(n * 16 + j) ? 1.f : 0.f;
        if (PLANES == 1) {
          float d = 0.f;
#pragma unroll
          for (int n = 0; n < T::NT; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j) d = at == (uint32_t)(n * 16 + j) ? t.acc[n][m][j] * weight : d;
          if (hit && q0 + in < a.h.rows) a.rest[q0 + in] = weight == 0.f ? 0.f : d - (float)(__bf16)d;
        }
      }
      // Rows without a gradient are zeros, whatever their probabilities.
      if (__builtin_amdgcn_ballot_w64(weight == 0.f)) {
#pragma unroll
        for (int n = 0; n < t.NT; ++n)
#pragma unroll
          for (int j = 0; j < 4; ++j) t.acc[n][m][j] = weight == 0.f ? 0.f : t.acc[n][m][j];
      }
      uint16_t* const row = tile + in * 64;
#pragma unroll
      for (int n = 0; n < t.NT; n += 2) {
        float d[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          d[j] = t.acc[n + j / 4][m][j & 3] * weight;
          if (ends && c0 + (n + j / 4) * 16 + (j & 3) >= a.w.rows) d[j] = 0.f;
        }
        uint16_t* const out = row + (n / 4) * (gemm::block_bytes(__builtin_ctz(TQ)) / 2) + (n & 2) * 16;
#pragma unroll
        for (int p = 0; p < PLANES; ++p) {
          *(u32x4*)(out + p * a.dz.plane) = pair_of(d, d + 4);
#pragma unroll
          for (int j = 0; j < 8; ++j) d[j] -= (float)(__bf16)d[j];  // exact
        }
      }
    }
    return true;
  });
}

// ---- gradients -----------------------------------------------------------------------

// dz at a row's target is most of its dz (p - 1 beside small p), and its rounding most
// of bfloat16 gradients' error: up to 0.0027 of their norm, 0.0017 with what it leaves
// (`rest`) added in float32.  For dW the rows are listed by their target's 128 columns, in
// their order.  Up to kListed rows of a list are added one by one; of longer lists those of
// each token are summed by k_rests before: a row more of the product for each token.
constexpr uint32_t kBucket = 128, kListed = 64, kMostBuckets = (1 << 18) / kBucket;

struct ListArgs {
  const int32_t* targets;
  const float* weight;
  uint32_t rows, vocab;
  uint32_t* start;  // [buckets + 1]
  uint32_t* order;  // [rows]: row numbers, a bucket's in their order
  uint32_t* longer; // the buckets of more than kListed rows: how many, which
};
// Each wave lists a run of the rows, with counts of its own: [listers][buckets].
constexpr uint32_t kListers = 16;
constexpr uint32_t run_of(uint32_t rows) { return (rows + kListers * 64 - 1) / (kListers * 64) * 64; }
constexpr uint32_t listers_of(uint32_t rows) { return (rows + run_of(rows) - 1) / run_of(rows); }
__device__ __forceinline__ void list_rows(const ListArgs& a, uint32_t* count) {
  __shared__ uint32_t sums[kListers * 64], longer;
  const uint32_t buckets = (a.vocab + kBucket - 1) / kBucket, tid = threadIdx.x, lane = tid & 63;
  constexpr uint32_t EACH = kMostBuckets / (kListers * 64);
  uint32_t* const own = count + tid / 64 * buckets;
  const uint32_t run = run_of(a.rows), listers = listers_of(a.rows);
  const uint32_t r0 = min(tid / 64 * run, a.rows), r1 = min(r0 + run, a.rows);
  auto bucket_of = [&](uint32_t r) {
    const uint32_t t = (uint32_t)a.targets[r];
    return t < a.vocab && !(a.weight && a.weight[r] == 0.f) ? t / kBucket : kMostBuckets;
  };
  for (uint32_t k = tid; k < listers * buckets; k += kListers * 64) count[k] = 0;
  if (tid == 0) longer = 0;
  __syncthreads();
  for (uint32_t r = r0 + lane; r < r1; r += 64) {
    const uint32_t b = bucket_of(r);
    if (b < kMostBuckets) atomicAdd(&own[b], 1u);
  }
  __syncthreads();
  uint32_t mine = 0;
  for (uint32_t b = tid * EACH; b < min((tid + 1) * EACH, buckets); ++b)
    for (uint32_t w = 0; w < listers; ++w) mine += count[w * buckets + b];
  sums[tid] = mine;
  __syncthreads();
  for (uint32_t o = 1; o < kListers * 64; o <<= 1) {
    const uint32_t x = tid >= o ? sums[tid - o] : 0u;
    __syncthreads();
    sums[tid] += x;
    __syncthreads();
  }
  uint32_t at = sums[tid] - mine;
  for (uint32_t b = tid * EACH; b < min((tid + 1) * EACH, buckets); ++b) {
    const uint32_t here = at;
    a.start[b] = at;
    for (uint32_t w = 0; w < listers; ++w) {
      const uint32_t n = count[w * buckets + b];
      count[w * buckets + b] = at;
      at += n;
    }
    if (at - here > kListed) a.longer[1 + atomicAdd(&longer, 1u)] = b;
  }
  if (tid == kListers * 64 - 1) a.start[buckets] = at;
  __syncthreads();
  if (tid == 0) a.longer[0] = longer;
  for (uint32_t k = r0; k < r1; k += 64) {
    const uint32_t b = k + lane < r1 ? bucket_of(k + lane) : kMostBuckets;
    // The lanes with its bucket: those that agree in every bit.
    uint64_t same = ~0ull;
#pragma unroll
    for (uint32_t bit = 1; bit <= kMostBuckets; bit <<= 1) {
      const uint64_t set = __builtin_amdgcn_ballot_w64((b & bit) != 0);
      same &= b & bit ? set : ~set;
    }
    const uint32_t before = __builtin_popcountll(same & ((1ull << lane) - 1));
    if (b < kMostBuckets) {
      const uint32_t to = own[b] + before;
      a.order[to] = k + lane;
      if (same >> lane == 1) own[b] = to + 1;
    }
    // The next rows' lanes see what these wrote.
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

// The rows that take part packed, and listed by the last block.
__global__ __launch_bounds__(1024) void k_prepare(PackArgs a, ListArgs l) {
  extern __shared__ uint32_t counts[];
  if (blockIdx.x + 1 == gridDim.x)
    list_rows(l, counts);
  else
    packed<1024>(a, blockIdx.x, gridDim.x - 1);
}

// The sums of rest * hidden over the rows of a token, for the tokens of lists longer than
// kListed: a block has `tokens` of them and 512 columns, a wave every eighth 64 rows of the
// list.  Rounded to bfloat16: 2^-8 of what is itself 2^-8 of dW.
// Without them dW was off by 0.0024 of its norm where every list is long (4096 rows of
// 3001 x 256), with them by 0.0017.  Bound by the chain of
// loads of the commonest token: 4096 rows of 1000 x 1024 16 us (22 with four waves a block).
struct RestArgs {
  const int32_t* targets;
  const float* rest;
  const uint32_t* start;
  const uint32_t* order;
  const uint32_t* longer;
  const uint16_t* h;
  uint32_t pitch, tokens, bucket0, buckets;  // of this piece
  uint16_t* sums;   // [rows][pitch]: a token's at the place in `order` of its first row
  uint32_t* place;  // [128 a bucket]: that place, or kNoRow
};
constexpr uint32_t kRestWaves = 8, kNoRow = 0xFFFFFFFFu;
__global__ __launch_bounds__(kRestWaves * 64) void k_rests(RestArgs a) {
  if (blockIdx.x >= a.longer[0]) return;
  const uint32_t b = a.longer[1 + blockIdx.x];
  if (b - a.bucket0 >= a.buckets) return;
  const uint32_t from = a.start[b], n = a.start[b + 1] - from;
  __shared__ uint32_t first[kBucket];
  __shared__ float part[kRestWaves][512];
  const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid / 64;
  const uint32_t t0 = b * kBucket + blockIdx.z * a.tokens, c0 = blockIdx.y * 512;
  if (tid < a.tokens) first[tid] = n;
  __syncthreads();
  for (uint32_t k = tid; k < n; k += kRestWaves * 64) {
    const uint32_t t = (uint32_t)a.targets[a.order[from + k]] - t0;
    if (t < a.tokens) atomicMin(&first[t], k);
  }
  __syncthreads();
  const bool in = c0 + lane * 8 < a.pitch;
  for (uint32_t s = 0; s < a.tokens; ++s) {
    const uint32_t at = __builtin_amdgcn_readfirstlane(first[s]);
    if (tid == 0 && blockIdx.y == 0) a.place[t0 + s] = at < n ? from + at : kNoRow;
    if (at >= n) continue;
    float sum[8] = {};
    for (uint32_t k = wave * 64; k < n; k += kRestWaves * 64) {
      const bool there = k + lane < n;
      const uint32_t row = there ? a.order[from + k + lane] : 0u;
      const bool its = there && (uint32_t)a.targets[row] == t0 + s;
      const float rest = its ? a.rest[row] : 0.f;
      uint64_t left = __builtin_amdgcn_ballot_w64(its);
      while (left) {
        u32x4 x[8];
        float by[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int l = left ? __builtin_ctzll(left) : 0;
          const uint32_t r = __builtin_amdgcn_readlane(row, l);
          by[j] = left ? __int_as_float(__builtin_amdgcn_readlane(__float_as_int(rest), l)) : 0.f;
          x[j] = left && in ? *(const u32x4*)(a.h + (size_t)r * a.pitch + c0 + lane * 8) : u32x4{0, 0, 0, 0};
          left &= left - 1;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            sum[e] = fmaf(by[j], __uint_as_float(e & 1 ? x[j][e / 2] & 0xFFFF0000u : x[j][e / 2] << 16), sum[e]);
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) part[wave][lane * 8 + e] = sum[e];
    __syncthreads();
    for (uint32_t c = tid; c < min(512u, a.pitch - c0); c += kRestWaves * 64) {
      float v = 0.f;
      for (uint32_t w = 0; w < kRestWaves; ++w) v += part[w][c];
      // An infinite one would make NaN of the columns beside it, to which 0 of it is added.
      constexpr float MOST = 0x1.fep127f;
      v = v > MOST ? MOST : v < -MOST ? -MOST : v;
      rows::store1<TFE_BF16>(a.sums + (size_t)(from + at) * a.pitch, c0 + c, v);
    }
    __syncthreads();
  }
}

// dH = dz W over a piece of the vocabulary, cut along it where the tiles are few (the parts are
// joined by k_finish_h, in float32), and dW = dz^T H.  k runs across W, H, and for dW dz: such
// operands are turned by the LDS reads (ds_read_b64_tr_b16: four k of 16 columns a lane row).
// Bound by the matrix cores and the loads beside them; 4096 rows x 32768 columns x 1024: dH 235 us,
// dW 250 (1.1 PFLOP/s; 165 and 170 where nothing was loaded).  Few rows: dW by its stores.
struct GradHArgs {
  Matrix w;  // a piece of the vocabulary
  Dz dz;
  uint32_t planes;
  uint32_t tiles_p, tiles_q, splits, total, dim, rows;
  float* sums;  // [splits][rows][pitch]
  uint32_t pitch;
  bool add;
};
template <int TP, int TQ, int WP, int WQ>
__global__ __launch_bounds__(WP* WQ * 64) void k_grad_h(GradHArgs a) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  Tile<Bf16, TP, TQ, WP, WQ, true, false, true> t;
  const uint32_t place = place_of(blockIdx.x, a.total), tiles = a.tiles_p * a.tiles_q;
  const uint32_t split = place / tiles, in = place % tiles;
  if (split >= a.splits) return;
  const uint32_t p0 = in % a.tiles_p * TP, q0 = in / a.tiles_p * TQ;
  const uint32_t steps = (a.w.rows + 63) / 64;
  const uint32_t s0 = (uint32_t)((uint64_t)steps * split / a.splits);
  const uint32_t s1 = (uint32_t)((uint64_t)steps * (split + 1) / a.splits);
  t.clear();
  // The operands end with the split.
  Matrix w = a.w;
  w.rows = min(w.rows, s1 * 64);
  uint32_t plane = 0;
  t.template run<0>(
      gemm::Segment{across(w, p0), a.dz.along(0, q0, s1), s0, s1},
      [&](gemm::Segment* s) {
        if (++plane >= a.planes) return false;
        s->q = a.dz.along(plane, q0, s1);
        return true;
      },
      [](uint32_t) {}, [](uint32_t) { return false; }, lds);
  const uint32_t c0 = p0 + t.wp + t.g * 4;
#pragma unroll
  for (int m = 0; m < t.MT; ++m) {
    const uint32_t r = q0 + t.wq + m * 16 + t.i;
    if (r >= a.rows) continue;
    float* out = a.sums + ((size_t)split * a.rows + r) * a.pitch + c0;
#pragma unroll
    for (int n = 0; n < t.NT; ++n)
      if (c0 + n * 16 < a.pitch) {
        f32x4 v = t.acc[n][m];
        if (a.add) v += *(const f32x4*)(out + n * 16);
        *(f32x4*)(out + n * 16) = v;
      }
  }
}
struct FinishArgs {
  const float* sums;
  uint32_t splits, rows, pitch, dim;
  void* out;
  int64_t ldo;
  const int32_t* targets;
  const float* weight;
  uint32_t vocab;
  const float* rest;
  const uint16_t* w;
  int64_t ldw;
};
// 64 splits of 64 rows x 1024: 33 us where a thread waited for one after another.
template <int DT> __global__ __launch_bounds__(64) void k_finish_h(FinishArgs a) {
  const uint32_t per = a.pitch / 4;
  const uint64_t n = (uint64_t)a.rows * per;
  for (uint64_t at = (uint64_t)blockIdx.x * 64 + threadIdx.x; at < n; at += (uint64_t)gridDim.x * 64) {
    const uint32_t r = (uint32_t)(at / per), c = (uint32_t)(at - (uint64_t)r * per) * 4;
    f32x4 v{0, 0, 0, 0};
    const float* from = a.sums + (size_t)r * a.pitch + c;
    const size_t apart = (size_t)a.rows * a.pitch;
    uint32_t k = 0;
    for (; k + 16 <= a.splits; k += 16, from += 16 * apart) {
      f32x4 x[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) x[j] = *(const f32x4*)(from + j * apart);
#pragma unroll
      for (int j = 0; j < 16; ++j) v += x[j];
    }
    f32x4 x[16];
#pragma unroll
    for (uint32_t j = 0; j < 16; ++j) x[j] = k + j < a.splits ? *(const f32x4*)(from + j * apart) : f32x4{0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 16; ++j) v += x[j];
    // 0 x an infinity of W is not a gradient of a row without one.
    const uint32_t target = (uint32_t)a.targets[r];
    const bool none = target >= a.vocab || (a.weight && a.weight[r] == 0.f);
    const float rest = DT == TFE_F32 || none ? 0.f : a.rest[r];
    const uint16_t* const at_w = a.w + (size_t)(none ? 0 : target) * a.ldw;
    char* out = (char*)a.out + ((size_t)r * a.ldo) * sizeof(typename rows::Elem<DT>::T);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (c + j < a.dim) {
        const float x = DT == TFE_F32 ? v[j] : fmaf(rest, rows::load1<TFE_BF16>(at_w, c + j), v[j]);
        rows::store1<DT>(out, c + j, none ? 0.f : x);
      }
  }
}

struct GradWArgs {
  Matrix h;
  Dz dz;  // of a piece of the vocabulary
  uint32_t planes;
  uint32_t tiles_p, total, dim, vocab;  // vocab: of the piece
  uint32_t vocab0;
  const int32_t* targets;
  const float* rest;
  const uint32_t* start;
  const uint32_t* order;
  uint32_t buckets;
  const uint16_t* sums;   // of k_rests, pitch of h
  const uint32_t* place;
  void* out;
  int64_t ldo;
  bool add;
};
template <int TP, int TQ, int WP, int WQ, int DT>
__global__ __launch_bounds__(WP* WQ * 64) void k_grad_w(GradWArgs a) {
  typedef typename rows::Elem<DT>::T E;
  typedef Tile<Bf16, TP, TQ, WP, WQ, true, true, true> T;
  typedef f32x4 f4 __attribute__((aligned(4)));
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  T t;
  // A block's tiles, and of each its planes: one segment behind the other.
  struct Place {
    uint32_t t, plane, p0, q0;
  };
  auto find = [&](Place* x) {
    if (x->t >= a.total) return false;
    const uint32_t place = place_of(x->t, a.total);
    x->p0 = place % a.tiles_p * TP;
    x->q0 = place / a.tiles_p * TQ;
    return x->q0 < a.vocab;
  };
  auto segment = [&](const Place& x) {
    return gemm::Segment{across(a.h, x.p0), a.dz.across(x.plane, x.q0), 0, (a.h.rows + 63) / 64};
  };
  Place cur{blockIdx.x, 0, 0, 0}, nxt;
  if (!find(&cur)) return;
  constexpr int STORES = DT == TFE_F32 ? T::NT * T::MT : T::NT * T::MT / 2;
  static_assert(TQ / WQ == 64 && kListed <= 64, "a wave's columns lie in one bucket, its rows in a wave");
  t.clear();
  // The lane's numbers, worked out anew in each tile: kept over the steps, what follows from
  // them would take the registers of the sums.
  auto lane_of = [&](uint32_t* i, uint32_t* g) {
    uint32_t own = t.lane;
    asm volatile("" : "+v"(own));
    *i = own & 15;
    *g = own >> 4;
    return own;
  };
  auto add_rests = [&](uint32_t p0, uint32_t q0, const char* info) {
    if (q0 + t.wq >= a.vocab) return;  // behind the last bucket there is no start
    uint32_t i, g;
    const uint32_t lane = lane_of(&i, &g);
    // Of the tile's first bucket on.
    const uint32_t* starts = (const uint32_t*)info + (t.wq / kBucket);
    const uint32_t from = __builtin_amdgcn_readfirstlane(starts[0]);
    const uint32_t n = __builtin_amdgcn_readfirstlane(starts[1]) - from;
    if (n == 0) return;
    const uint32_t first = a.vocab0 + q0 + t.wq;
    // Small tiles: a lane's columns have a row of k_rests each, or none.  In large ones this way
    // beside the other takes the registers of the sums.
    constexpr bool EACH = TQ == 128;
    const bool many = n > kListed;
    if (EACH && many) {
#pragma unroll
      for (int m = 0; m < T::MT; ++m) {
        const uint32_t r = a.place[first + m * 16 + i];
        const uint16_t* x = a.sums + (size_t)r * a.h.ld + p0 + t.wp + g * 4;
        u32x2 y[T::NT];
#pragma unroll
        for (int n = 0; n < T::NT; ++n) y[n] = u32x2{0, 0};
        if (r != kNoRow) {
#pragma unroll
          for (int n = 0; n < T::NT; ++n)
            if (p0 + t.wp + n * 16 + g * 4 < a.h.cols) y[n] = *(const u32x2*)(x + n * 16);
        }
#pragma unroll
        for (int n = 0; n < T::NT; ++n)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            t.acc[n][m][j] += __uint_as_float(j & 1 ? y[n][j / 2] & 0xFFFF0000u : y[n][j / 2] << 16);
      }
      return;
    }
    uint32_t row = kNoRow, target = first + lane;
    float rest = 1.f;
    if (!EACH && many) {
      row = a.place[target];
    } else if (lane < n) {
      row = a.order[from + lane];
      target = (uint32_t)a.targets[row];
      rest = a.rest[row];
    }
    const uint16_t* const from_rows = !EACH && many ? a.sums : a.h.at;
    uint64_t mine = __builtin_amdgcn_ballot_w64(row != kNoRow && target - first < 64u);
    while (mine) {
      const int l = __builtin_ctzll(mine);
      mine &= mine - 1;
      const uint32_t r = __builtin_amdgcn_readlane(row, l), in = __builtin_amdgcn_readlane(target, l) - first;
      const float by = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(rest), l));
      const uint16_t* x = from_rows + (size_t)r * a.h.ld + p0 + t.wp + g * 4;
      u32x2 y[T::NT];
#pragma unroll
      for (int n = 0; n < T::NT; ++n)
        y[n] = p0 + t.wp + n * 16 + g * 4 < a.h.cols ? *(const u32x2*)(x + n * 16) : u32x2{0, 0};
      // Every sum is added to, most of them 0: a choice among them would put them in memory.
#pragma unroll
      for (int m = 0; m < T::MT; ++m) {
        const float f = in == (uint32_t)m * 16 + i ? by : 0.f;
#pragma unroll
        for (int n = 0; n < T::NT; ++n)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            t.acc[n][m][j] =
                fmaf(f, __uint_as_float(j & 1 ? y[n][j / 2] & 0xFFFF0000u : y[n][j / 2] << 16), t.acc[n][m][j]);
      }
    }
  };
  auto write = [&](uint32_t p0, uint32_t q0) {
    uint32_t i, g;
    lane_of(&i, &g);
    const bool all = p0 + TP <= a.dim && q0 + TQ <= a.vocab;
#pragma unroll
    for (int m = 0; m < T::MT; ++m) {
      const uint32_t v = q0 + t.wq + m * 16 + i;
      E* const row = (E*)a.out + (size_t)v * a.ldo + p0 + t.wp;
#pragma unroll
      for (int n = 0; n < T::NT; n += 2) {
        if (DT == TFE_F32 || !all) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t c = (n + h) * 16 + g * 4, left = a.dim - min(a.dim, p0 + t.wp + c);
            f32x4 x = t.acc[n + h][m];
            if (all || (v < a.vocab && left >= 4)) {
              if constexpr (DT == TFE_F32) {
                if (a.add) x += *(const f4*)(row + c);
                *(f4*)(row + c) = x;
              } else {
                typedef u32x2 u2 __attribute__((aligned(2)));
                *(u2*)(row + c) = u2{pack2(x[0], x[1]), pack2(x[2], x[3])};
              }
            } else if (v < a.vocab) {
#pragma unroll
              for (uint32_t j = 0; j < 4; ++j)
                if (j < left) {
                  const float old = DT == TFE_F32 && a.add ? rows::load1<DT>(row, c + j) : 0.f;
                  rows::store1<DT>(row, c + j, x[j] + old);
                }
            }
          }
        } else {
          // They pass by: nothing reads them soon.
          __builtin_nontemporal_store(pair_of((const float*)&t.acc[n][m], (const float*)&t.acc[n + 1][m]),
                                      (rows::u32x4_a2*)(row + n * 16 + piece_of(g)));
        }
      }
    }
    return all;
  };
  t.template run<STORES>(
      segment(cur),
      [&](gemm::Segment* s) {
        nxt = cur;
        if (++nxt.plane == a.planes) nxt.plane = 0, nxt.t += gridDim.x;
        const bool more = find(&nxt);
        if (more) *s = segment(nxt);
        return more;
      },
      [&](uint32_t odd) {
        if (DT == TFE_BF16 && t.wave == 0)
          gemm::load_numbers(a.start, (a.vocab0 + cur.q0) / kBucket, a.buckets + 1, 0, lds + T::LDS + odd * 256);
      },
      [&](uint32_t odd) {
        bool stored = false;
        if (cur.plane + 1 == a.planes) {
          if constexpr (DT == TFE_BF16) {
            add_rests(cur.p0, cur.q0, lds + T::LDS + odd * 256);
            __builtin_amdgcn_sched_barrier(0);
          }
          stored = write(cur.p0, cur.q0);
          t.clear();
        }
        cur = nxt;
        return stored;
      },
      lds);
}

// ---- launches ------------------------------------------------------------------------

// Rows of a tile of logits (the first rule that holds).  Loss and gradients in us with tiles of 64 / 128 / 256 rows
// (and 128 / 256 / 256 columns), dim 1024: 100 rows of vocabulary 3001 48 / 73 / 78, of 70000
// 166 / 194 / 190, of 151936 429 / 394 / 421; 200 rows of 20000 97 / 103 / 108, of 151936
// 647 / 549 / 452; 700 rows of 3000 70 / 90 / 98, of 20000 211 / 191 / 152.
uint32_t tile_of(uint32_t rows, uint32_t vocab) {
  const uint32_t cus = (uint32_t)compute_units(), wide = (vocab + 255) / 256;
  if (rows > 128 && wide * ((rows + 255) / 256) * 4 >= cus * 3) return 256;
  return rows > 64 && rows <= 128 && wide >= cus * 2 ? 128 : 64;
}
// Whether dW is cut into tiles of 128 x 128, of 256 x 256 otherwise.  Loss and gradients in
// us, so / otherwise: 64 rows of 151936 x 1024 289 / 315, of 40000 95 / 106; 100 rows of 151936
// 411 / 394, of 70000 166 / 181; 200 rows of 151936 495 / 452; 700 rows of 3000 70 / 77, of 20000
// 152 / 158; 2048 rows of 20000 354 / 351; 4096 rows of 3000 172 / 195.
bool small_w(uint32_t rows, uint32_t vocab, uint32_t dim) {
  const uint32_t cus = (uint32_t)compute_units(), tiles = ((vocab + 255) / 256) * ((dim + 255) / 256);
  return rows <= 64 || tiles * 4 < cus * 5 || (rows <= 128 && tiles < cus * 5);
}

// What lies where in the workspace, and how the work is cut.
struct Plan {
  uint32_t pitch;        // of packed rows and of dH's sums: dim rounded up to 64
  uint32_t piece;        // columns of the vocabulary at a time
  uint32_t chunk;        // rows at a time whose slabs' sums are kept
  uint32_t splits;       // of dH's sums over the vocabulary
  uint32_t tile;         // rows of a tile
  uint32_t log;          // dz is in blocks of 2^log = tile rows
  int64_t plane;         // its bytes, of which there are three for float32 gradients
  int64_t h, masked, w, part, picked, rest, start, order, longer, place, dz, sums, bytes;
};

int64_t take(int64_t* at, int64_t bytes) {
  const int64_t here = *at;
  *at += (bytes + 255) / 256 * 256;
  return here;
}
uint32_t up(uint32_t x, uint32_t to) { return (x + to - 1) / to * to; }

Plan plan_of(int64_t n_rows, int32_t n_vocab, int32_t n_dim) {
  const uint32_t rows = (uint32_t)n_rows, vocab = (uint32_t)n_vocab, dim = (uint32_t)n_dim;
  Plan p{};
  p.pitch = up(dim, 64);
  p.tile = tile_of(rows, vocab);
  const int64_t most = std::max<int64_t>(4096, (1 << 27) / n_rows / 256 * 256);
  p.piece = (uint32_t)std::min<int64_t>(most, up(vocab, 256));
  p.chunk = std::min<uint32_t>(rows, 16384);
  const uint32_t tiles = ((dim + 255) / 256) * ((rows + p.tile - 1) / p.tile);
  p.splits = std::max<uint32_t>(1, std::min<uint32_t>((uint32_t)compute_units() / tiles, p.piece / 128));
  int64_t at = 0;
  p.h = take(&at, (int64_t)rows * p.pitch * 2);
  p.masked = take(&at, (int64_t)rows * p.pitch * 2);
  p.w = take(&at, (int64_t)p.piece * p.pitch * 2);
  p.part = take(&at, (int64_t)((vocab + p.piece - 1) / p.piece * p.piece / kSlab) * p.chunk * 8);
  p.picked = take(&at, (int64_t)rows * 4);
  p.rest = take(&at, (int64_t)rows * 4);
  p.start = take(&at, (kMostBuckets + 1) * 4);
  p.order = take(&at, (int64_t)rows * 4);
  p.longer = take(&at, (int64_t)(1 + std::min(rows / (kListed + 1), kMostBuckets)) * 4);
  p.place = take(&at, (int64_t)up(vocab, kBucket) * 4);
  p.log = p.tile == 256 ? 8 : p.tile == 128 ? 7 : 6;
  p.plane = (int64_t)(up(rows, p.tile) / p.tile) * (p.piece / 64) * gemm::block_bytes(p.log);
  p.dz = take(&at, p.plane * planes_of(true));
  p.sums = take(&at, (int64_t)p.splits * rows * p.pitch * 4);
  p.bytes = at;
  return p;
}

// 16-byte loads of whole rows.
bool direct(const void* p, int64_t ld, uint32_t dim) {
  return ((uintptr_t)p & 15) == 0 && ld % 8 == 0 && dim % 8 == 0 && ld <= kXentMaxPitch;
}

hipError_t pack(const PackArgs& a, hipStream_t s) {
  const uint64_t n = (uint64_t)a.rows * (a.pitch / 8);
  k_pack<<<dim3((uint32_t)std::min<uint64_t>((n + 255) / 256, 8192)), dim3(256), 0, s>>>(a);
  return hipGetLastError();
}
hipError_t pack(const uint16_t* x, int64_t ldx, uint32_t rows, uint32_t cols, uint32_t pitch,
                uint16_t* out, hipStream_t s) {
  return pack(PackArgs{x, ldx, rows, cols, pitch, nullptr, nullptr, 0, out}, s);
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
#define LAUNCH(T, INFO, kernel, blocks, s, args)                                    \
  do {                                                                              \
    static std::atomic<uint64_t> told_{0};                                          \
    const hipError_t e_ = allow(kernel, T::LDS + INFO, &told_);                            \
    if (e_ != hipSuccess) return e_;                                                \
    kernel<<<dim3(blocks), dim3(T::THREADS), T::LDS + INFO, s>>>(args);             \
    return hipGetLastError();                                                       \
  } while (0)

// Blocks of a launch whose blocks take one tile after another.
template <class T> uint32_t blocks(uint32_t total, int info) {
  return std::min<uint32_t>(total, up(compute_units() * (163840 / (T::LDS + info)), 8));
}

template <int TP, int TQ, int WP, int WQ> hipError_t sums(LogitsArgs a, hipStream_t s) {
  typedef Tile<Bf16, TP, TQ, WP, WQ, false, false, false> T;
  a.tiles_q = (a.h.rows + TQ - 1) / TQ;
  a.total = up((a.w.rows + TP - 1) / TP * a.tiles_q, 8);
  auto* k = k_sums<TP, TQ, WP, WQ>;
  LAUNCH(T, 2 * kInfo<TQ>, k, blocks<T>(a.total, 2 * kInfo<TQ>), s, a);
}
template <int TP, int TQ, int WP, int WQ, int PLANES> hipError_t dz(LogitsArgs a, hipStream_t s) {
  typedef Tile<Bf16, TP, TQ, WP, WQ, false, false, false> T;
  a.tiles_q = (a.h.rows + TQ - 1) / TQ;
  a.total = up((a.w.rows + TP - 1) / TP * a.tiles_q, 8);
  auto* k = k_dz<TP, TQ, WP, WQ, PLANES>;
  LAUNCH(T, 2 * kInfo<TQ>, k, blocks<T>(a.total, 2 * kInfo<TQ>), s, a);
}
template <int TP, int TQ, int WP, int WQ> hipError_t grad_h(GradHArgs a, hipStream_t s) {
  typedef Tile<Bf16, TP, TQ, WP, WQ, true, false, true> T;
  a.tiles_p = (a.dim + TP - 1) / TP;
  a.tiles_q = (a.rows + TQ - 1) / TQ;
  a.total = up(a.tiles_p * a.tiles_q * a.splits, 8);
  auto* k = k_grad_h<TP, TQ, WP, WQ>;
  LAUNCH(T, 0, k, a.total, s, a);
}
template <int TP, int TQ, int WP, int WQ, int DT> hipError_t grad_w(GradWArgs a, hipStream_t s) {
  typedef Tile<Bf16, TP, TQ, WP, WQ, true, true, true> T;
  a.tiles_p = (a.dim + TP - 1) / TP;
  a.total = up(a.tiles_p * ((a.vocab + TQ - 1) / TQ), 8);
  auto* k = k_grad_w<TP, TQ, WP, WQ, DT>;
  LAUNCH(T, 512, k, blocks<T>(a.total, 512), s, a);
}

// dW of no rows.
__global__ __launch_bounds__(256) void k_zero(char* out, uint64_t pitch, uint32_t bytes) {
  char* row = out + blockIdx.x * pitch;
  for (uint32_t c = threadIdx.x * 2; c < bytes; c += 512) *(uint16_t*)(row + c) = 0;
}
hipError_t zero(const XentArgs& a, hipStream_t s) {
  const uint32_t size = a.gdtype == TFE_F32 ? 4 : 2;
  k_zero<<<dim3(a.vocab), dim3(256), 0, s>>>((char*)a.gw, (uint64_t)a.ldgw * size, a.dim * size);
  return hipGetLastError();
}

#define TRY_HIP(call)                        \
  do {                                       \
    const hipError_t te_ = (call);           \
    if (te_ != hipSuccess) return te_;       \
  } while (0)

// Rows [v0, v0 + n) of W as the tiles take them; `there`: a copy of them is in place.
hipError_t piece_of_w(const XentArgs& a, const Plan& p, uint32_t v0, uint32_t n, bool there, Matrix* m,
                      hipStream_t s) {
  const uint16_t* at = a.w + (size_t)v0 * a.ldw;
  if (direct(a.w, a.ldw, a.dim)) {
    *m = Matrix{at, (uint32_t)a.ldw, n, a.dim};
    return hipSuccess;
  }
  uint16_t* to = (uint16_t*)(a.space + p.w);
  *m = Matrix{to, p.pitch, n, p.pitch};
  return there ? hipSuccess : pack(at, a.ldw, n, a.dim, p.pitch, to, s);
}

}  // namespace

int64_t xent_space(int64_t rows, int32_t vocab, int32_t dim) {
  return rows == 0 ? 0 : plan_of(rows, vocab, dim).bytes;
}

hipError_t launch_xent_loss(const XentArgs& a, hipStream_t s) {
  const Plan p = plan_of(a.rows, a.vocab, a.dim);
  Matrix h{a.hidden, (uint32_t)a.ldh, a.rows, a.dim};
  if (!direct(a.hidden, a.ldh, a.dim)) {
    uint16_t* to = (uint16_t*)(a.space + p.h);
    TRY_HIP(pack(a.hidden, a.ldh, a.rows, a.dim, p.pitch, to, s));
    h = Matrix{to, p.pitch, a.rows, p.pitch};
  }
  const uint32_t step = direct(a.w, a.ldw, a.dim) ? a.vocab : p.piece;
  for (uint32_t r0 = 0; r0 < a.rows; r0 += p.chunk) {
    LogitsArgs l{};
    l.h = h;
    l.h.at += (size_t)r0 * h.ld;
    l.h.rows = std::min(p.chunk, a.rows - r0);
    l.targets = a.targets + r0;
    l.part = (f32x2*)(a.space + p.part);
    l.picked = (float*)(a.space + p.picked) + r0;
    for (uint32_t v0 = 0; v0 < a.vocab; v0 += step) {
      TRY_HIP(piece_of_w(a, p, v0, std::min(step, a.vocab - v0), r0 > 0 && step >= a.vocab, &l.w, s));
      l.vocab0 = v0;
      l.slab0 = v0 / kSlab;
      TRY_HIP((p.tile == 256   ? sums<256, 256, 2, 4>(l, s)
               : p.tile == 128 ? sums<256, 128, 2, 2>(l, s)
                               : sums<128, 64, 1, 4>(l, s)));
    }
    JoinArgs j{l.part, (a.vocab + kSlab - 1) / kSlab, l.h.rows, a.vocab, l.targets, l.picked,
               a.loss + r0, a.lse + r0};
    k_join<<<dim3((l.h.rows + 15) / 16), dim3(1024), 0, s>>>(j);
    TRY_HIP(hipGetLastError());
  }
  return hipSuccess;
}

hipError_t launch_xent_grad(const XentArgs& a, bool behind_loss, hipStream_t s) {
  if (a.rows == 0) return a.accumulate ? hipSuccess : zero(a, s);
  const Plan p = plan_of(a.rows, a.vocab, a.dim);
  const bool f32 = a.gdtype == TFE_F32;
  uint16_t* masked = (uint16_t*)(a.space + p.masked);
  const Matrix h{masked, p.pitch, a.rows, p.pitch};
  const PackArgs packed{a.hidden, a.ldh, a.rows, a.dim, p.pitch, a.targets, a.weight, a.vocab, masked};
  const ListArgs list{a.targets, a.weight, a.rows, a.vocab, (uint32_t*)(a.space + p.start),
                      (uint32_t*)(a.space + p.order), (uint32_t*)(a.space + p.longer)};
  if (f32) {
    TRY_HIP(pack(packed, s));
  } else {
    const uint64_t pieces = ((uint64_t)a.rows * (p.pitch / 8) + 1023) / 1024;
    static std::atomic<uint64_t> told{0};
    const int counts = (int)(listers_of(a.rows) * ((a.vocab + kBucket - 1) / kBucket) * 4);
    TRY_HIP(allow(k_prepare, (int)(kListers * kMostBuckets * 4), &told));
    k_prepare<<<dim3((uint32_t)std::min<uint64_t>(pieces, 2048) + 1), dim3(1024), counts, s>>>(packed, list);
    TRY_HIP(hipGetLastError());
  }
  for (uint32_t v0 = 0; v0 < a.vocab; v0 += p.piece) {
    const uint32_t n = std::min(p.piece, a.vocab - v0);
    LogitsArgs l{};
    l.h = h;
    TRY_HIP(piece_of_w(a, p, v0, n, behind_loss && p.piece >= a.vocab, &l.w, s));
    l.vocab0 = v0;
    l.targets = a.targets;
    l.lse = a.lse;
    l.weight = a.weight;
    l.vocab = a.vocab;
    l.rest = (float*)(a.space + p.rest);
    // Rows of whole tiles, columns of whole steps of this piece (memory: of whole tiles).
    l.dz = Dz{(uint16_t*)(a.space + p.dz), (uint64_t)p.plane / 2, p.log, p.piece / 64, up(a.rows, p.tile), up(n, 64)};
    l.h.cols = l.w.cols;  // zeros from dim on
    if (f32)
      TRY_HIP((p.tile == 256   ? dz<256, 256, 2, 4, planes_of(true)>(l, s)
               : p.tile == 128 ? dz<256, 128, 2, 2, planes_of(true)>(l, s)
                               : dz<128, 64, 1, 4, planes_of(true)>(l, s)));
    else
      TRY_HIP((p.tile == 256   ? dz<256, 256, 2, 4, planes_of(false)>(l, s)
               : p.tile == 128 ? dz<256, 128, 2, 2, planes_of(false)>(l, s)
                               : dz<128, 64, 1, 4, planes_of(false)>(l, s)));
    GradHArgs gh{};
    gh.w = l.w;
    gh.dz = l.dz;
    gh.rows = a.rows;
    gh.planes = planes_of(f32);
    gh.splits = p.splits;
    gh.dim = a.dim;
    gh.sums = (float*)(a.space + p.sums);
    gh.pitch = p.pitch;
    gh.add = v0 != 0;
    TRY_HIP((p.tile == 256   ? grad_h<256, 256, 2, 4>(gh, s)
             : p.tile == 128 ? grad_h<256, 128, 2, 2>(gh, s)
                             : grad_h<256, 64, 2, 2>(gh, s)));
    // p.h was the loss's.  Tokens of a block: a few thousand blocks at most.
    RestArgs rest{a.targets, l.rest, list.start, list.order, list.longer, masked, p.pitch, 1, v0 / kBucket,
                  (n + kBucket - 1) / kBucket, (uint16_t*)(a.space + p.h), (uint32_t*)(a.space + p.place)};
    if (!f32 && a.rows > kListed) {
      const uint32_t lists = std::min((a.vocab + kBucket - 1) / kBucket, a.rows / (kListed + 1)), across = (p.pitch + 511) / 512;
      while (rest.tokens < kBucket && lists * across * (kBucket / rest.tokens) > 8192) rest.tokens *= 2;
      k_rests<<<dim3(lists, across, kBucket / rest.tokens), dim3(kRestWaves * 64), 0, s>>>(rest);
      TRY_HIP(hipGetLastError());
    }
    GradWArgs gw{};
    gw.sums = rest.sums;
    gw.place = rest.place;
    gw.h = h;
    gw.dz = l.dz;
    gw.planes = gh.planes;
    gw.dim = a.dim;
    gw.vocab = n;
    gw.vocab0 = v0;
    gw.targets = a.targets;
    gw.rest = l.rest;
    gw.start = list.start;
    gw.order = list.order;
    gw.buckets = (a.vocab + kBucket - 1) / kBucket;
    gw.ldo = a.ldgw;
    gw.add = a.accumulate;
    gw.out = (char*)a.gw + (size_t)v0 * a.ldgw * (f32 ? 4 : 2);
    if (small_w(a.rows, n, a.dim))
      TRY_HIP((f32 ? grad_w<128, 128, 2, 2, TFE_F32>(gw, s) : grad_w<128, 128, 2, 2, TFE_BF16>(gw, s)));
    else
      TRY_HIP((f32 ? grad_w<256, 256, 2, 4, TFE_F32>(gw, s) : grad_w<256, 256, 2, 4, TFE_BF16>(gw, s)));
  }
  FinishArgs f{(float*)(a.space + p.sums), p.splits, a.rows, p.pitch, a.dim, a.gx, a.ldgx, a.targets,
               a.weight, a.vocab, (const float*)(a.space + p.rest), a.w, a.ldw};
  const uint32_t blocks = (uint32_t)std::min<uint64_t>(((uint64_t)a.rows * (p.pitch / 4) + 63) / 64, 32768);
  if (f32)
    k_finish_h<TFE_F32><<<dim3(blocks), dim3(64), 0, s>>>(f);
  else
    k_finish_h<TFE_BF16><<<dim3(blocks), dim3(64), 0, s>>>(f);
  return hipGetLastError();
}

}  // namespace tfe
