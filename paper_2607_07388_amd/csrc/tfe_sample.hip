// Sampling one token per row from its logits: temperature, top-k, top-p and
// min-p, then the inverse of the running sum at a given uniform number.
//   w_i = 2^31 exp((l_i - max) / T) rounded to an integer
// ordered by (w descending, token ascending).  Every step then asks for the
// element of that order at which a running count (top-k) or a running sum
// (top-p, the draw) reaches a target.  Sums are 64-bit integers (at most 2^18
// weights of at most 2^31: exact, and exact as doubles too), so the answer
// does not depend on the order of the additions.  2^-31 of the most likely
// token's weight is the resolution: finer than that of a float32 u.
// Bound by the logits' bytes.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "tfe_logits.h"
#include "tfe_rows.h"

namespace tfe {
namespace {

using namespace rows;

constexpr int kThreads = 1024;
// A weight w >= 1 is a float32 without error (it is one, or an integer below
// 2^24), and its bits order as it does.  The order's key: 28 bits of the
// weight's float bits above those of 1, then 18 bits of the token, lower
// first.  Larger keys come first; keys are distinct.
constexpr int kIdBits = 18, kKeyBits = 46;
constexpr uint32_t kOneBits = 127u << 23;
constexpr float kUnit = 2147483648.f;

__device__ __forceinline__ uint64_t key_of(float w, uint32_t id) {
  return ((uint64_t)(__float_as_uint(w) - kOneBits) << kIdBits) | ((1u << kIdBits) - 1 - id);
}
__device__ __forceinline__ float key_weight(uint64_t k) {
  return __uint_as_float((uint32_t)(k >> kIdBits) + kOneBits);
}
__device__ __forceinline__ uint32_t key_id(uint64_t k) {
  return (1u << kIdBits) - 1 - (uint32_t)(k & ((1u << kIdBits) - 1));
}

// A row's settings.
struct Row {
  float top, inv_t;  // largest logit, 1 / T
  bool greedy;
};
// The weight of logit l, an integer in float32; 0 for NaN and -infinity.
__device__ __forceinline__ float weight(const Row& r, float l) {
  if (l == r.top) return kUnit;
  if (r.greedy || !(l > -INFINITY)) return 0.f;
  const float e = rintf(expf((l - r.top) * r.inv_t) * kUnit);
  return e >= 1.f ? e : 0.f;  // NaN (0 x infinity) is no weight either
}

constexpr int kBins = 4096;
struct Shared {
  uint32_t cnt[kBins];
  unsigned long long sum[kBins];
  unsigned long long red[kThreads / 64];
  uint32_t redc[kThreads / 64];
  // What a scan of the bins found.
  uint32_t bin;
  uint64_t before_c, before_w, in_c, in_w;
};

// Calls f(l, id) for every logit of the row.
template <int DT, class F> __device__ __forceinline__ void each(const SampleArgs& a, const char* x, F f) {
  constexpr int N = Elem<DT>::N;
  const uint32_t nv = a.vocab / N;
  for (uint32_t v = threadIdx.x; v < nv; v += kThreads) {
    float l[N];
    unpack<DT>(load_vec<DT>(x, v), l);
#pragma unroll
    for (int i = 0; i < N; ++i) f(l[i], v * N + i);
  }
  for (uint32_t i = nv * N + threadIdx.x; i < a.vocab; i += kThreads) f(load1<DT>(x, i), i);
}

// The bin, from the highest down, in which the running count (by_count) or sum
// reaches `target`, what lies before it and in it.  target is at most the total.
__device__ void find_bin(Shared& sh, uint64_t target, bool by_count) {
  constexpr int PER = kBins / kThreads;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  uint32_t c[PER];
  uint64_t w[PER], cs = 0, ws = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int b = kBins - 1 - (t * PER + i);
    c[i] = sh.cnt[b];
    w[i] = sh.sum[b];
    cs += c[i];
    ws += w[i];
  }
  uint64_t pc = cs, pw = ws;  // inclusive over the wave
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint64_t xc = __shfl_up(pc, o), xw = __shfl_up(pw, o);
    if (lane >= o) {
      pc += xc;
      pw += xw;
    }
  }
  if (lane == 63) {
    sh.redc[wave] = (uint32_t)pc;
    sh.red[wave] = pw;
  }
  __syncthreads();
  for (int i = 0; i < wave; ++i) {
    pc += sh.redc[i];
    pw += sh.red[i];
  }
  pc -= cs;
  pw -= ws;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const uint64_t have = by_count ? pc : pw, get = by_count ? c[i] : w[i];
    if (have < target && target <= have + get) {
      sh.bin = (uint32_t)(kBins - 1 - (t * PER + i));
      sh.before_c = pc;
      sh.before_w = pw;
      sh.in_c = c[i];
      sh.in_w = w[i];
    }
    pc += c[i];
    pw += w[i];
  }
  __syncthreads();
}

// The element of the order at which the running count or sum reaches `target`
// (at least 1, at most the row's): its key, and the sum through it.  Twelve
// bits of the key at a time, over the elements that share the bits so far.
template <int DT>
__device__ uint64_t reach(const SampleArgs& a, const char* x, const Row& r, Shared& sh,
                          uint64_t target, bool by_count, uint64_t* sum) {
  uint64_t prefix = 0, base_w = 0;
  int left = kKeyBits;
  while (left > 0) {
    const int digit = left > 12 ? 12 : left, shift = left - digit;
    for (int b = threadIdx.x; b < kBins; b += kThreads) {
      sh.cnt[b] = 0;
      sh.sum[b] = 0;
    }
    __syncthreads();
    each<DT>(a, x, [&](float l, uint32_t id) {
      const float w = weight(r, l);
      if (w == 0.f) return;
      const uint64_t k = key_of(w, id);
      if (k >> left != prefix) return;
      const uint32_t b = (uint32_t)(k >> shift) & ((1u << digit) - 1);
      atomicAdd(&sh.cnt[b], 1u);
      atomicAdd(&sh.sum[b], (unsigned long long)w);
    });
    __syncthreads();
    find_bin(sh, target, by_count);
    prefix = (prefix << digit) | sh.bin;
    target -= by_count ? sh.before_c : sh.before_w;
    base_w += sh.before_w;
    left = shift;
    if (left == 0) base_w += sh.in_w;
    __syncthreads();
  }
  *sum = base_w;
  return prefix;
}

template <int DT> __global__ __launch_bounds__(kThreads) void k_sample(SampleArgs a) {
  __shared__ Shared sh;
  const uint32_t row = blockIdx.x;
  const char* x = (const char*)a.logits + (size_t)row * a.ld * sizeof(typename Elem<DT>::T);
  const float T = a.temperature ? a.temperature[row] : 1.f;
  Row r;
  r.greedy = !(T > 0.f);
  r.inv_t = 1.f / T;
  float top = -INFINITY;
  each<DT>(a, x, [&](float l, uint32_t) { top = fmaxf(top, l); });
  r.top = block_max<float, kThreads>(top, (float*)sh.red);
  if (r.top == -INFINITY) {
    if (threadIdx.x == 0) {
      a.token[row] = -1;
      if (a.prob) a.prob[row] = 0.f;
    }
    return;
  }
  uint64_t sum = 0, cnt = 0;
  each<DT>(a, x, [&](float l, uint32_t) {
    const float w = weight(r, l);
    sum += (uint64_t)w;
    cnt += w != 0.f;
  });
  sum = block_add<unsigned long long, kThreads>(sum, sh.red);
  cnt = block_add<unsigned long long, kThreads>(cnt, sh.red);
  uint64_t cut = 0;  // the last key kept so far
  const int32_t k = r.greedy ? 1 : a.top_k ? a.top_k[row] : 0;
  if (k > 0 && (uint64_t)k < cnt) cut = reach<DT>(a, x, r, sh, (uint64_t)k, true, &sum);
  const float p = a.top_p ? a.top_p[row] : 1.f;
  if (p < 1.f) {
    const uint64_t part = (uint64_t)((double)sum * (double)fmaxf(p, 0.f));
    cut = reach<DT>(a, x, r, sh, part > 1 ? part : 1, false, &sum);
  }
  const float mp = a.min_p ? a.min_p[row] : 0.f;
  const float least = mp > 0.f ? rintf(fminf(mp, 1.f) * kUnit) : 0.f;
  if (least > 1.f && (((uint64_t)(__float_as_uint(least) - kOneBits)) << kIdBits) > cut) {
    cut = (uint64_t)(__float_as_uint(least) - kOneBits) << kIdBits;
    uint64_t s = 0;
    each<DT>(a, x, [&](float l, uint32_t) {
      const float w = weight(r, l);
      s += w >= least ? (uint64_t)w : 0;
    });
    sum = block_add<unsigned long long, kThreads>(s, sh.red);
  }
  const float u = a.u[row];
  uint64_t at = (uint64_t)((double)sum * (double)(u > 0.f ? fminf(u, 1.f) : 0.f));
  at = at < sum ? at : sum - 1;
  uint64_t through;
  const uint64_t got = reach<DT>(a, x, r, sh, at + 1, false, &through);
  if (threadIdx.x == 0) {
    a.token[row] = (int32_t)key_id(got);
    if (a.prob) a.prob[row] = (float)((double)key_weight(got) / (double)sum);
  }
}

}  // namespace

int64_t sample_space(int64_t, int32_t) { return 0; }

hipError_t launch_sample(const SampleArgs& a, int dtype, hipStream_t s) {
  if (dtype == TFE_F32)
    k_sample<TFE_F32><<<dim3(a.rows), dim3(kThreads), 0, s>>>(a);
  else
    k_sample<TFE_BF16><<<dim3(a.rows), dim3(kThreads), 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace tfe
