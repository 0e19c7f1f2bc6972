// The norm of many tensors taken as one vector, and their clipping by it.
// Bound by bytes: 155 million float32 numbers' norm 95 us (6.5 TB/s); of as many in bfloat16 the
// norm takes 53 us and the clipping 104 (6.0 TB/s read and written).  Tensors come as a launch's
// arguments, so that a call copies nothing to the device and can be captured.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "tfe_learn.h"
#include "tfe_rows.h"

namespace tfe {
namespace {

using namespace rows;

constexpr int kThreads = 256;
constexpr uint32_t kUnit = 1024;    // elements; a tensor begins a unit of its own
constexpr uint32_t kBlocks = 2048;  // of a launch at most
constexpr uint32_t kParts = 1024;   // of a launch of sums: a partial sum each
constexpr uint32_t kMostUnits = 1u << 30;  // of a launch, but for its last tensor
constexpr int kSlots = 160;         // tensors of a launch: its arguments stay below 4 KB
constexpr int kPitches = 16;        // of them with rows apart
constexpr int kDeep = 8;            // vectors of a thread under way

// A tensor of a launch, in 24 bytes: its elements are kUnit for each of its units but the last,
// and bits % 1024 + 1 there; then its dtype; then 0, or 1 + the place of its pitches.
struct Slot {
  const char* grad;
  char* out;
  uint32_t first;  // its first unit
  uint32_t bits;
};
struct Pitch {
  uint32_t cols, ldg, ldo;
};
template <int SLOTS> struct Batch {
  Slot slot[SLOTS];
  Pitch pitch[kPitches];
  uint32_t slots, units, pitches;
};
static_assert(sizeof(Batch<kSlots>) <= 4064, "a launch's arguments, with the others");
// The same as a run is worked on; cols 0: its elements lie one behind the other.
struct Tensor {
  const char* grad;
  char* out;
  uint64_t n;
  uint32_t cols, ldg, ldo;
  int32_t dtype;
};
// A launch's arguments are copied by the host: few tensors have short ones.
constexpr int kShort = 16;

// The last slot whose first unit is not behind `unit`: all are looked at by one to three
// loads, where a search would wait for one after another.
template <int SLOTS> __device__ __forceinline__ uint32_t find(const Batch<SLOTS>& b, uint32_t unit) {
  const uint32_t lane = threadIdx.x & 63;
  uint32_t n = 0;
#pragma unroll
  for (uint32_t k = 0; k < (SLOTS + 63) / 64; ++k) {
    const uint32_t i = k * 64 + lane;
    const bool at = i < b.slots && b.slot[min(i, (uint32_t)SLOTS - 1)].first <= unit;
    n += __popcll(__builtin_amdgcn_ballot_w64(at));
  }
  return n - 1;
}
// Element i of a tensor in its memory.
__device__ __forceinline__ uint64_t place(uint64_t i, uint32_t cols, uint32_t ld) {
  if (!cols) return i;
  if (i >> 32 == 0) {  // the 64-bit quotient is a long one
    const uint32_t row = (uint32_t)i / cols;
    return (uint64_t)row * ld + ((uint32_t)i - row * cols);
  }
  const uint64_t row = i / cols;
  return row * ld + (i - row * cols);
}
// The units [u0, u1) as runs of one tensor's elements [at, at + n).
template <int SLOTS, class F> __device__ __forceinline__ void runs(const Batch<SLOTS>& b, uint32_t u0, uint32_t u1, F go) {
  for (uint32_t k = find(b, u0); u0 < u1; ++k) {
    const Slot& x = b.slot[k];
    const uint32_t behind = k + 1 < b.slots ? b.slot[k + 1].first : b.units, end = min(u1, behind);
    const uint64_t at = (uint64_t)(u0 - x.first) * kUnit;
    const uint32_t apart = x.bits >> 11;
    const Pitch p = apart ? b.pitch[apart - 1] : Pitch{0, 0, 0};
    const Tensor t{x.grad, x.out, (uint64_t)(behind - x.first - 1) * kUnit + (x.bits & (kUnit - 1)) + 1,
                   p.cols, p.ldg, p.ldo, (int32_t)(x.bits >> 10 & 1)};
    go(t, at, min((uint64_t)(end - u0) * kUnit, t.n - at));
    u0 = end;
  }
}
// A block's part of the units: all blocks' are as long, to one unit.
template <int SLOTS, class F> __device__ __forceinline__ void part_of(const Batch<SLOTS>& b, uint32_t block, F go) {
  runs(b, (uint32_t)((uint64_t)b.units * block / gridDim.x),
       (uint32_t)((uint64_t)b.units * (block + 1) / gridDim.x), go);
}

// Elements of a run of n before `p` is at a 16-byte boundary.
template <int DT> __device__ __forceinline__ uint32_t head_of(const char* p, uint64_t n) {
  return (uint32_t)min((uint64_t)((-(uintptr_t)p & 15) / sizeof(typename Elem<DT>::T)), n);
}
// go(v, loaded vector) for the vectors of a run, kDeep of a thread under way at once.
// Returns the elements that they cover.
template <int DT, bool PASS>
__device__ __forceinline__ u32x4 loaded(const char* p, uint32_t v) {
  return PASS ? load_stream<DT>(p, v) : load_vec<DT>(p, v);
}
template <int DT, int THREADS, bool PASS, class F>
__device__ __forceinline__ uint64_t vectors(const char* p, uint64_t n, F go) {
  constexpr uint32_t N = Elem<DT>::N;
  const uint64_t all = n / N;
  uint64_t v0 = 0;
  for (; v0 + kDeep * THREADS <= all; v0 += kDeep * THREADS) {
    u32x4 x[kDeep];
#pragma unroll
    for (int k = 0; k < kDeep; ++k) x[k] = loaded<DT, PASS>(p + v0 * 16, k * THREADS + threadIdx.x);
#pragma unroll
    for (int k = 0; k < kDeep; ++k) go(v0 + k * THREADS + threadIdx.x, x[k]);
  }
  u32x4 x[kDeep];
  const uint32_t left = (uint32_t)(all - v0);
#pragma unroll
  for (int k = 0; k < kDeep; ++k)
    if (k * THREADS + threadIdx.x < left) x[k] = loaded<DT, PASS>(p + v0 * 16, k * THREADS + threadIdx.x);
#pragma unroll
  for (int k = 0; k < kDeep; ++k)
    if (k * THREADS + threadIdx.x < left) go(v0 + k * THREADS + threadIdx.x, x[k]);
  return all * N;
}

// Squares are summed in float64: neither large nor small gradients leave its range.
template <int DT, int THREADS, bool PASS>
__device__ __forceinline__ double squares(const Tensor& t, uint64_t at, uint64_t n) {
  constexpr uint32_t N = Elem<DT>::N;
  double sum = 0, sum2 = 0;
  uint32_t head = 0;
  uint64_t from = 0;
  if (t.cols == 0) {
    const char* p = t.grad + at * sizeof(typename Elem<DT>::T);
    head = head_of<DT>(p, n);
    from = vectors<DT, THREADS, PASS>(p + head * sizeof(typename Elem<DT>::T), n - head, [&](uint64_t, u32x4 x) {
      float f[N];
      unpack<DT>(x, f);
#pragma unroll
      for (uint32_t j = 0; j < N; j += 2) {
        sum += (double)f[j] * f[j];
        sum2 += (double)f[j + 1] * f[j + 1];
      }
    });
  } else if (t.cols % N == 0) {  // whole vectors in a row
    from = n;
    for (uint64_t e = threadIdx.x * N; e < n; e += THREADS * N) {
      float f[N];
      unpack<DT>(load_vec<DT>(t.grad + place(at + e, t.cols, t.ldg) * sizeof(typename Elem<DT>::T), 0), f);
#pragma unroll
      for (uint32_t j = 0; j < N; ++j) sum += (double)f[j] * f[j];
    }
  }
  // What the vectors leave, at either end.
  for (uint64_t i = threadIdx.x; i < n - from; i += THREADS) {
    const uint64_t e = i < head ? i : from + i;
    const double x = load1<DT>(t.grad, place(at + e, t.cols, t.ldg));
    sum += x * x;
  }
  return sum + sum2;
}
template <int THREADS, bool PASS>
__device__ __forceinline__ double squares(const Tensor& t, uint64_t at, uint64_t n) {
  return t.dtype == TFE_F32 ? squares<TFE_F32, THREADS, PASS>(t, at, n)
                            : squares<TFE_BF16, THREADS, PASS>(t, at, n);
}

// PASS: loads that pass the caches by.
template <int SLOTS, bool PASS>
__global__ __launch_bounds__(kThreads) void k_squares(Batch<SLOTS> b, double* part) {
  __shared__ double red[kThreads / 64];
  double sum = 0;
  part_of(b, blockIdx.x, [&](const Tensor& t, uint64_t at, uint64_t n) { sum += squares<kThreads, PASS>(t, at, n); });
  sum = block_add<double, kThreads>(sum, red);
  if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

// The norm of the partial sums, the same in every block that asks.
__device__ __forceinline__ float norm_of(const double* part, uint32_t parts, double* red) {
  double sum = 0;
  for (uint32_t k = threadIdx.x; k < parts; k += kThreads) sum += part[k];
  return (float)sqrt(block_add<double, kThreads>(sum, red));
}
__global__ __launch_bounds__(kThreads) void k_norm(const double* part, uint32_t parts, float* norm) {
  __shared__ double red[kThreads / 64];
  const float x = norm_of(part, parts, red);
  if (threadIdx.x == 0) *norm = x;
}

template <int DT, int THREADS>
__device__ __forceinline__ void scale(const Tensor& t, uint64_t at, uint64_t n, float by) {
  constexpr uint32_t N = Elem<DT>::N;
  uint32_t head = 0;
  uint64_t from = 0;
  if (t.cols == 0) {
    constexpr size_t SIZE = sizeof(typename Elem<DT>::T);
    head = head_of<DT>(t.out + at * SIZE, n);
    char* o = t.out + (at + head) * SIZE;
    from = vectors<DT, THREADS, false>(t.grad + (at + head) * SIZE, n - head, [&](uint64_t v, u32x4 x) {
      float f[N];
      unpack<DT>(x, f);
#pragma unroll
      for (uint32_t j = 0; j < N; ++j) f[j] *= by;
      __builtin_nontemporal_store(pack<DT>(f), (typename Elem<DT>::V*)(o + v * 16));
    });
  } else if (t.cols % N == 0) {
    constexpr size_t SIZE = sizeof(typename Elem<DT>::T);
    from = n;
    for (uint64_t e = threadIdx.x * N; e < n; e += THREADS * N) {
      float f[N];
      unpack<DT>(load_vec<DT>(t.grad + place(at + e, t.cols, t.ldg) * SIZE, 0), f);
#pragma unroll
      for (uint32_t j = 0; j < N; ++j) f[j] *= by;
      store_vec<DT>(t.out + place(at + e, t.cols, t.ldo) * SIZE, 0, pack<DT>(f));
    }
  }
  for (uint64_t i = threadIdx.x; i < n - from; i += THREADS) {
    const uint64_t e = i < head ? i : from + i;
    store1<DT>(t.out, place(at + e, t.cols, t.ldo), load1<DT>(t.grad, place(at + e, t.cols, t.ldg)) * by);
  }
}
struct Factor {
  bool clip;
  float by;
};
__device__ __forceinline__ Factor factor_of(float norm, float max_norm) {
  const bool clip = norm > max_norm && norm < INFINITY;
  return Factor{clip, clip ? max_norm / norm : 1.f};
}
template <int THREADS>
__device__ __forceinline__ void scale(const Tensor& t, uint64_t at, uint64_t n, Factor f) {
  if (!f.clip && t.grad == t.out) return;
  if (t.dtype == TFE_F32)
    scale<TFE_F32, THREADS>(t, at, n, f.by);
  else
    scale<TFE_BF16, THREADS>(t, at, n, f.by);
}

// The norm comes from partial sums (and is written), or from memory.
struct ClipArgs {
  const double* part;
  uint32_t parts;
  float* norm;
  float max_norm;
};
template <int SLOTS> __global__ __launch_bounds__(kThreads) void k_clip(Batch<SLOTS> b, ClipArgs a) {
  __shared__ double red[kThreads / 64];
  const float norm = a.part ? norm_of(a.part, a.parts, red) : *a.norm;
  if (a.part && blockIdx.x == 0 && threadIdx.x == 0) *a.norm = norm;
  const Factor f = factor_of(norm, a.max_norm);
  // What was read last is read first: it is still in the cache.
  part_of(b, gridDim.x - 1 - blockIdx.x,
          [&](const Tensor& t, uint64_t at, uint64_t n) { scale<kThreads>(t, at, n, f); });
}

// Runs `go` with batches of up to SLOTS tensors that have elements; `out`: theirs is used.
template <int SLOTS, class F> hipError_t batches_of(const GradArgs& a, bool out, F go) {
  Batch<SLOTS> b;
  b.slots = b.units = b.pitches = 0;
  for (int64_t k = 0; k < a.n; ++k) {
    const tfe_grad_tensor& g = a.tensors[k];
    const uint64_t n = (uint64_t)g.rows * g.cols;
    if (n == 0) continue;
    const bool whole = g.rows == 1 || (g.ldg == g.cols && (!out || g.ldo == g.cols));
    if (!whole) b.pitch[b.pitches++] = Pitch{(uint32_t)g.cols, (uint32_t)g.ldg, (uint32_t)g.ldo};
    b.slot[b.slots++] = Slot{(const char*)g.grad, (char*)g.out, b.units,
                             (uint32_t)((n - 1) % kUnit) | (uint32_t)g.dtype << 10 | (whole ? 0 : b.pitches) << 11};
    b.units += (uint32_t)((n + kUnit - 1) / kUnit);
    if (b.slots == SLOTS || b.pitches == kPitches || b.units >= kMostUnits) {
      const hipError_t e = go(b);
      if (e != hipSuccess) return e;
      b.slots = b.units = b.pitches = 0;
    }
  }
  return b.slots ? go(b) : hipSuccess;
}
template <class F> hipError_t batches(const GradArgs& a, bool out, F go) {
  return a.n <= kShort ? batches_of<kShort>(a, out, go) : batches_of<kSlots>(a, out, go);
}

template <int SLOTS, bool PASS> void sums(const Batch<SLOTS>& b, uint32_t blocks, double* part, hipStream_t s) {
  k_squares<SLOTS, PASS><<<dim3(blocks), dim3(kThreads), 0, s>>>(b, part);
}
hipError_t partials(const GradArgs& a, bool pass, uint32_t* parts, hipStream_t s) {
  *parts = 0;
  return batches(a, false, [&](const auto& b) {
    const uint32_t blocks = std::min(b.units, kParts);
    double* part = (double*)a.space + *parts;
    pass ? sums<sizeof(b.slot) / sizeof(Slot), true>(b, blocks, part, s)
         : sums<sizeof(b.slot) / sizeof(Slot), false>(b, blocks, part, s);
    *parts += blocks;
    return hipGetLastError();
  });
}
hipError_t join(const GradArgs& a, uint32_t parts, hipStream_t s) {
  k_norm<<<dim3(1), dim3(kThreads), 0, s>>>((const double*)a.space, parts, a.norm);
  return hipGetLastError();
}
hipError_t clip(const GradArgs& a, const double* part, uint32_t parts, hipStream_t s) {
  return batches(a, true, [&](const auto& b) {
    k_clip<<<dim3(std::min(b.units, kBlocks)), dim3(kThreads), 0, s>>>(
        b, ClipArgs{part, parts, a.norm, a.max_norm});
    return hipGetLastError();
  });
}

}  // namespace

// Sums of as many launches as there can be: each but the last has kSlots tensors (kShort of
// few), kPitches with rows apart or kMostUnits units.
int64_t grad_space(const tfe_grad_tensor* t, int64_t n) {
  int64_t units = 0, apart = 0;
  for (int64_t k = 0; k < n; ++k) {
    units += (int64_t)(((uint64_t)t[k].rows * t[k].cols + kUnit - 1) / kUnit);
    apart += t[k].rows > 1;
  }
  return ((n + kSlots - 1) / kSlots + apart / kPitches + units / kMostUnits) * (int64_t)kParts * 8;
}

hipError_t launch_grad_norm(const GradArgs& a, hipStream_t s) {
  // More than the last cache holds: it is not filled (622 MB of float32: 95 us instead of 110).
  int64_t bytes = 0;
  for (int64_t k = 0; k < a.n; ++k)
    bytes += a.tensors[k].rows * a.tensors[k].cols * (a.tensors[k].dtype == TFE_F32 ? 4 : 2);
  uint32_t parts;
  const hipError_t e = partials(a, bytes > (int64_t)256 << 20, &parts, s);
  return e == hipSuccess ? join(a, parts, s) : e;
}
hipError_t launch_grad_clip(const GradArgs& a, hipStream_t s) { return clip(a, nullptr, 0, s); }
hipError_t launch_grad_norm_clip(const GradArgs& a, hipStream_t s) {
  uint32_t parts;
  hipError_t e = partials(a, false, &parts, s);
  if (e != hipSuccess) return e;
  // One launch's sums are joined by every block that clips, more by a launch before.
  if (parts > 0 && parts <= kParts) return clip(a, (const double*)a.space, parts, s);
  e = join(a, parts, s);
  return e == hipSuccess ? clip(a, nullptr, 0, s) : e;
}

}  // namespace tfe
