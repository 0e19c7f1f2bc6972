// Distillation from a teacher's top logits: the loss KL(q || p) of the
// teacher's softmax q over its K listed tokens against the student's softmax p
// over the vocabulary, both at temperature tau, and its gradient.
//   lse = log sum_v exp(s_v / tau)       (running maximum and sum, one pass)
//   loss = tau^2 sum_k q_k (log q_k - s_k / tau + lse)
//   d loss / d s_v = tau (p_v - q_v),    p_v = exp(s_v / tau - lse)
// Bound by the logits' bytes: the loss reads them, the gradient reads and
// writes them.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "tfe_logits.h"
#include "tfe_rows.h"

namespace tfe {
namespace {

using namespace rows;

constexpr int kThreads = 1024;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// Running maximum m and sum s of exp((x - m) c / log2 e).  While every element
// was -infinity, m stays -infinity and s 0.
struct Running {
  float m, s;
};
__device__ __forceinline__ float finite_max(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ Running join(Running a, Running b, float c) {
  Running r;
  r.m = fmaxf(a.m, b.m);
  const float ref = finite_max(r.m);
  r.s = a.s * exp2_hw((a.m - ref) * c) + b.s * exp2_hw((b.m - ref) * c);
  return r;
}

struct Shared {
  float q[kDistillMaxK];
  int32_t id[kDistillMaxK];
  float red[kThreads / 64], red2[kThreads / 64];
};

// The teacher's row: thread k < K gets its entry's log q and q, all of them
// in sh.  Padding has q = 0 and id -1; so has every entry of an empty row.
struct Entry {
  int32_t id;
  float q, logq;
};
template <int TDT> __device__ Entry teacher_row(const DistillArgs& a, uint32_t row, Shared& sh) {
  const uint32_t k = threadIdx.x;
  const size_t at = (size_t)row * a.K + k;
  Entry e{-1, 0.f, 0.f};
  float t = -INFINITY;
  if (k < a.K) {
    e.id = a.ids[at];
    if (e.id < 0 || (uint32_t)e.id >= a.vocab) e.id = -1;
    if (e.id >= 0) t = load1<TDT>(a.teacher, at) * a.inv_tau;
  }
  const float top = block_max<float, kThreads>(t, sh.red);
  const float some = block_max<float, kThreads>(t == -INFINITY ? 0.f : 1.f, sh.red);
  float x = t == -INFINITY ? 0.f : expf(t - top);
  const float sum = block_add<float, kThreads>(x, sh.red);
  if (some != 0.f) {
    e.q = x / sum;
    e.logq = (t - top) - logf(sum);
  }
  if (k < kDistillMaxK) {
    sh.q[k] = e.q;
    sh.id[k] = some != 0.f ? e.id : -1;
  }
  if (some == 0.f) e.id = -1;
  __syncthreads();
  return e;
}

// Maximum and sum of one row.
template <int DT> __device__ Running row_sum(const DistillArgs& a, const char* row, Shared& sh) {
  constexpr int N = Elem<DT>::N;
  const float c = a.inv_tau * kLog2e;
  Running r{-INFINITY, 0.f};
  const uint32_t nv = a.vocab / N;
  for (uint32_t v = threadIdx.x; v < nv; v += kThreads) {
    float x[N];
    unpack<DT>(load_vec<DT>(row, v), x);
    float top = x[0];
#pragma unroll
    for (int i = 1; i < N; ++i) top = fmaxf(top, x[i]);
    const float m = fmaxf(r.m, top), ref = finite_max(m);
    float s = r.s * exp2_hw((r.m - ref) * c);
#pragma unroll
    for (int i = 0; i < N; ++i) s += exp2_hw((x[i] - ref) * c);
    r = Running{m, s};
  }
  for (uint32_t i = nv * N + threadIdx.x; i < a.vocab; i += kThreads) {
    const float x = load1<DT>(row, i);
    r = join(r, Running{x, x == -INFINITY ? 0.f : (x == x ? 1.f : x)}, c);
  }
#pragma unroll
  for (int o = 32; o; o >>= 1)
    r = join(r, Running{__shfl_xor(r.m, o), __shfl_xor(r.s, o)}, c);
  if ((threadIdx.x & 63) == 0) {
    sh.red[threadIdx.x >> 6] = r.m;
    sh.red2[threadIdx.x >> 6] = r.s;
  }
  __syncthreads();
  r = Running{sh.red[0], sh.red2[0]};
  for (int w = 1; w < kThreads / 64; ++w) r = join(r, Running{sh.red[w], sh.red2[w]}, c);
  __syncthreads();
  return r;
}

__device__ __forceinline__ float lse_of(const DistillArgs& a, Running r) {
  return fmaf(r.m, a.inv_tau, __builtin_amdgcn_logf(r.s) * kLn2);
}

template <int DT>
__device__ void row_grad(const DistillArgs& a, const char* row, char* out, float lse, float g,
                         const Entry& e, float student, const Shared& sh) {
  constexpr int N = Elem<DT>::N;
  const uint32_t nv = a.vocab / N;
  // An empty teacher's row, or one that the loss' gradient leaves out.
  bool any = false;
  for (uint32_t k = 0; k < a.K; ++k) any |= sh.id[k] >= 0;
  const bool zero = !any || g == 0.f;
  const float f = g * a.tau;
  for (uint32_t v = threadIdx.x; v < nv; v += kThreads) {
    float x[N];
    if (zero) {
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = 0.f;
    } else {
      unpack<DT>(load_vec<DT>(row, v), x);
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = f * exp2_hw(fmaf(x[i], a.inv_tau, -lse) * kLog2e);
    }
    store_vec<DT>(out, v, pack<DT>(x));
  }
  for (uint32_t i = nv * N + threadIdx.x; i < a.vocab; i += kThreads)
    store1<DT>(out, i,
               zero ? 0.f : f * exp2_hw(fmaf(load1<DT>(row, i), a.inv_tau, -lse) * kLog2e));
  __syncthreads();
  // The listed tokens again, with their q (an id listed twice: each writer
  // adds the same entries in the same order).
  if (!zero && e.id >= 0) {
    float q = 0.f;
    for (uint32_t k = 0; k < a.K; ++k) q += sh.id[k] == e.id ? sh.q[k] : 0.f;
    store1<DT>(out, (uint32_t)e.id,
               f * (exp2_hw(fmaf(student, a.inv_tau, -lse) * kLog2e) - q));
  }
}

template <int DT, int TDT, bool LOSS, bool GRAD>
__global__ __launch_bounds__(kThreads) void k_distill(DistillArgs a) {
  __shared__ Shared sh;
  const uint32_t row = blockIdx.x;
  const char* x = (const char*)a.logits + (size_t)row * a.ld * sizeof(typename Elem<DT>::T);
  const Entry e = teacher_row<TDT>(a, row, sh);
  const float student = e.id >= 0 ? load1<DT>(x, (uint32_t)e.id) : 0.f;
  float lse;
  if (LOSS) {
    lse = lse_of(a, row_sum<DT>(a, x, sh));
    const float part =
        e.id < 0 || e.q == 0.f ? 0.f : e.q * (e.logq - fmaf(student, a.inv_tau, -lse));
    const float sum = block_add<float, kThreads>(part, sh.red);
    if (threadIdx.x == 0) {
      a.loss[row] = a.tau * a.tau * sum;
      a.lse[row] = lse;
    }
  } else {
    lse = a.lse[row];
  }
  if (GRAD) {
    const float g = a.weight ? a.weight[row] : 1.f;
    char* out = (char*)a.grad + (size_t)row * a.ldg * sizeof(typename Elem<DT>::T);
    row_grad<DT>(a, x, out, lse, g, e, student, sh);
  }
}

template <bool LOSS, bool GRAD>
hipError_t launch(const DistillArgs& a, int dtype, int tdtype, hipStream_t s) {
  const dim3 grid(a.rows), block(kThreads);
  if (dtype == TFE_F32 && tdtype == TFE_F32)
    k_distill<TFE_F32, TFE_F32, LOSS, GRAD><<<grid, block, 0, s>>>(a);
  else if (dtype == TFE_F32)
    k_distill<TFE_F32, TFE_BF16, LOSS, GRAD><<<grid, block, 0, s>>>(a);
  else if (tdtype == TFE_F32)
    k_distill<TFE_BF16, TFE_F32, LOSS, GRAD><<<grid, block, 0, s>>>(a);
  else
    k_distill<TFE_BF16, TFE_BF16, LOSS, GRAD><<<grid, block, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

int64_t distill_space(int64_t, int32_t) { return 0; }
hipError_t launch_distill_loss(const DistillArgs& a, int dtype, int tdtype, hipStream_t s) {
  return launch<true, false>(a, dtype, tdtype, s);
}
hipError_t launch_distill_grad(const DistillArgs& a, int dtype, int tdtype, hipStream_t s) {
  return launch<false, true>(a, dtype, tdtype, s);
}
hipError_t launch_distill_loss_grad(const DistillArgs& a, int dtype, int tdtype, hipStream_t s) {
  return launch<true, true>(a, dtype, tdtype, s);
}

}  // namespace tfe
