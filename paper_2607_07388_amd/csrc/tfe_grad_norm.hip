// The norm of many tensors taken as one vector, and their clipping by it.
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
constexpr uint32_t kUnit = 8192;    // elements a block takes at a time
constexpr uint32_t kBlocks = 1024;  // of a launch at most, a partial sum each
constexpr int kSlots = 80;          // tensors of a launch: its arguments stay below 4 KB

// A tensor of a launch; cols 0: its elements lie one behind the other.
struct Slot {
  const char* grad;
  char* out;
  uint64_t n;
  uint32_t first;  // its first unit
  uint32_t cols, ldg, ldo;
  int32_t dtype;
};
struct Batch {
  Slot slot[kSlots];
  uint32_t slots, units;
};

__device__ __forceinline__ uint32_t find(const Batch& b, uint32_t unit) {
  uint32_t lo = 0, hi = b.slots;
  while (hi - lo > 1) {
    const uint32_t mid = (lo + hi) / 2;
    if (b.slot[mid].first <= unit) lo = mid;
    else hi = mid;
  }
  return lo;
}
// Element i of a tensor in its memory.
__device__ __forceinline__ uint64_t place(uint64_t i, uint32_t cols, uint32_t ld) {
  return cols ? i / cols * ld + i % cols : i;
}

// Squares are summed in float64: neither large nor small gradients leave its range.
template <int DT> __device__ __forceinline__ double squares(const Slot& t, uint64_t at, uint32_t n) {
  constexpr uint32_t N = Elem<DT>::N;
  double sum = 0;
  uint32_t from = 0;
  if (t.cols == 0) {
    const char* p = t.grad + at * sizeof(typename Elem<DT>::T);
    from = n / N * N;
    for (uint32_t v = threadIdx.x; v < n / N; v += kThreads) {
      float f[N];
      unpack<DT>(load_vec<DT>(p, v), f);
#pragma unroll
      for (uint32_t j = 0; j < N; ++j) sum += (double)f[j] * f[j];
    }
  }
  for (uint32_t e = from + threadIdx.x; e < n; e += kThreads) {
    const double x = load1<DT>(t.grad, place(at + e, t.cols, t.ldg));
    sum += x * x;
  }
  return sum;
}

__global__ __launch_bounds__(kThreads) void k_squares(Batch b, double* part) {
  __shared__ double red[kThreads / 64];
  double sum = 0;
  for (uint32_t u = blockIdx.x; u < b.units; u += gridDim.x) {
    const Slot& t = b.slot[find(b, u)];
    const uint64_t at = (uint64_t)(u - t.first) * kUnit;
    const uint32_t n = (uint32_t)min((uint64_t)kUnit, t.n - at);
    sum += t.dtype == TFE_F32 ? squares<TFE_F32>(t, at, n) : squares<TFE_BF16>(t, at, n);
  }
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

template <int DT>
__device__ __forceinline__ void scale(const Slot& t, uint64_t at, uint32_t n, float by) {
  constexpr uint32_t N = Elem<DT>::N;
  uint32_t from = 0;
  if (t.cols == 0) {
    const char* p = t.grad + at * sizeof(typename Elem<DT>::T);
    char* o = t.out + at * sizeof(typename Elem<DT>::T);
    from = n / N * N;
    for (uint32_t v = threadIdx.x; v < n / N; v += kThreads) {
      float f[N];
      unpack<DT>(load_vec<DT>(p, v), f);
#pragma unroll
      for (uint32_t j = 0; j < N; ++j) f[j] *= by;
      store_vec<DT>(o, v, pack<DT>(f));
    }
  }
  for (uint32_t e = from + threadIdx.x; e < n; e += kThreads)
    store1<DT>(t.out, place(at + e, t.cols, t.ldo), load1<DT>(t.grad, place(at + e, t.cols, t.ldg)) * by);
}

// The norm comes from partial sums (and is written), or from memory.
struct ClipArgs {
  const double* part;
  uint32_t parts;
  float* norm;
  float max_norm;
};
__global__ __launch_bounds__(kThreads) void k_clip(Batch b, ClipArgs a) {
  __shared__ double red[kThreads / 64];
  const float norm = a.part ? norm_of(a.part, a.parts, red) : *a.norm;
  if (a.part && blockIdx.x == 0 && threadIdx.x == 0) *a.norm = norm;
  const bool clip = norm > a.max_norm && norm < INFINITY;
  const float by = clip ? a.max_norm / norm : 1.f;
  for (uint32_t u = blockIdx.x; u < b.units; u += gridDim.x) {
    const Slot& t = b.slot[find(b, u)];
    if (!clip && t.grad == t.out) continue;
    const uint64_t at = (uint64_t)(u - t.first) * kUnit;
    const uint32_t n = (uint32_t)min((uint64_t)kUnit, t.n - at);
    if (t.dtype == TFE_F32)
      scale<TFE_F32>(t, at, n, by);
    else
      scale<TFE_BF16>(t, at, n, by);
  }
}

// Runs `go` with batches of up to kSlots tensors that have elements.
template <class F> hipError_t batches(const GradArgs& a, F go) {
  Batch b;
  b.slots = b.units = 0;
  for (int64_t k = 0; k < a.n; ++k) {
    const tfe_grad_tensor& g = a.tensors[k];
    const uint64_t n = (uint64_t)g.rows * g.cols;
    if (n == 0) continue;
    const bool whole = g.rows == 1 || (g.ldg == g.cols && g.ldo == g.cols);
    const uint64_t units = (n + kUnit - 1) / kUnit;
    b.slot[b.slots++] = Slot{(const char*)g.grad, (char*)g.out, n, b.units, whole ? 0 : (uint32_t)g.cols,
                             (uint32_t)g.ldg, (uint32_t)g.ldo, g.dtype};
    b.units += (uint32_t)units;
    if (b.slots == kSlots) {
      const hipError_t e = go(b);
      if (e != hipSuccess) return e;
      b.slots = b.units = 0;
    }
  }
  return b.slots ? go(b) : hipSuccess;
}

hipError_t partials(const GradArgs& a, uint32_t* parts, hipStream_t s) {
  *parts = 0;
  return batches(a, [&](const Batch& b) {
    const uint32_t blocks = std::min(b.units, kBlocks);
    k_squares<<<dim3(blocks), dim3(kThreads), 0, s>>>(b, (double*)a.space + *parts);
    *parts += blocks;
    return hipGetLastError();
  });
}
hipError_t clip(const GradArgs& a, const double* part, uint32_t parts, hipStream_t s) {
  return batches(a, [&](const Batch& b) {
    k_clip<<<dim3(std::min(b.units, kBlocks * 2)), dim3(kThreads), 0, s>>>(
        b, ClipArgs{part, parts, a.norm, a.max_norm});
    return hipGetLastError();
  });
}

}  // namespace

int64_t grad_space(const tfe_grad_tensor*, int64_t n) {
  return (n + kSlots - 1) / kSlots * (int64_t)kBlocks * 8;
}

hipError_t launch_grad_norm(const GradArgs& a, hipStream_t s) {
  uint32_t parts;
  const hipError_t e = partials(a, &parts, s);
  if (e != hipSuccess) return e;
  k_norm<<<dim3(1), dim3(kThreads), 0, s>>>((const double*)a.space, parts, a.norm);
  return hipGetLastError();
}
hipError_t launch_grad_clip(const GradArgs& a, hipStream_t s) { return clip(a, nullptr, 0, s); }
hipError_t launch_grad_norm_clip(const GradArgs& a, hipStream_t s) {
  uint32_t parts;
  const hipError_t e = partials(a, &parts, s);
  if (e != hipSuccess) return e;
  if (parts == 0) return launch_grad_norm(a, s);
  return clip(a, (const double*)a.space, parts, s);
}

}  // namespace tfe
