// Sampling one token per row from its logits: temperature, top-k, top-p and
// min-p, then the inverse of the running sum at a given uniform number.
//   w_i = 2^31 exp((l_i - max) / T) rounded to an integer
// ordered by (w descending, token ascending).  Every step then asks for the
// element of that order at which a running count (top-k) or a running sum
// (top-p, the draw) reaches a target.  Sums are 64-bit integers (at most 2^18
// weights of at most 2^31: exact, and exact as doubles too), so the answer
// does not depend on the order of the additions.  2^-31 of the most likely
// token's weight is the resolution: finer than that of a float32 u.
//
// Nothing is sorted but a few hundred elements.  A histogram of the weights by
// their leading bits gives the running count and sum at every bin's edge; from
// those, and the settings, follows in which bins the answers to the four
// questions can lie (later ones depend on earlier ones, so a question can have
// a short range of bins).  Only those bins' elements are collected and sorted,
// and the questions answered in turn.  Three passes over the logits: their
// maximum, the histogram, the collection.
// Bound by the logits' bytes for the first pass, then by the weights' arithmetic
// (about 27 instruction slots a logit) and the LDS additions of the second.
// 151936 float32 logits a row, top-k and top-p: 1 row 25 us, 64 rows 52, 256 rows 83
// (top-p alone 96).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "tfe_logits.h"
#include "tfe_rows.h"

namespace tfe {
namespace {

using namespace rows;

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

// A row's largest logit and 1 / T.  The most likely token alone (T <= 0 or NaN)
// is 1 / T = infinity: every smaller logit has weight 0.
struct Scale {
  float top, inv_t;
};
__device__ __forceinline__ float inverse_temperature(const SampleArgs& a, uint32_t row) {
  const float T = a.temperature ? a.temperature[row] : 1.f;
  return T > 0.f ? 1.f / T : INFINITY;
}

// The weight of logit l, an integer in float32; 0 for NaN and -infinity.
// exp(d) is 2^(d log2 e) with the product in two parts (its rounding would be
// as much as |d| 2^-24 of the result) and the hardware's exponential: about an
// ulp in all.  The maximum with -30, where weights are 0, also takes the NaN
// of infinity - infinity and 0 x infinity.
// A weight never rises as d falls, nor above 1: so gfx950's exponential and this
// correction turned out when neighbours were compared for every float32 d from
// -30 to 0 (an error within an ulp alone would not give it).
__device__ __forceinline__ float weight(const Scale& r, float l) {
  const float d = fmaxf((l - r.top) * r.inv_t, -30.f);
  const float p = d * 1.44269504f;
  const float e = fmaf(d, 1.92596303e-8f, fmaf(d, 1.44269504f, -p));
  const float x = __builtin_amdgcn_exp2f(p);
  const float w = rintf(fmaf(x, e * 0.693147181f, x) * kUnit);
  return l == r.top ? kUnit : w;
}

// The histogram: 4096 bins of 1/128 of an octave, the leading 12 bits of the
// key.  An entry holds the number of its elements (from bit 43 on) and the sum
// of what their weights have above the bin's lowest (below 2^24 each, 2^42 in
// all): one 64-bit addition an element.
constexpr int kBins = 4096, kBinShift = 16, kCountShift = 43;
__device__ __forceinline__ uint32_t bin_of(float w) {
  return (__float_as_uint(w) - kOneBits) >> kBinShift;
}
__device__ __forceinline__ uint32_t bin_low(uint32_t bin) {
  return (uint32_t)__uint_as_float((bin << kBinShift) + kOneBits);
}
__device__ __forceinline__ uint64_t bin_entry(float w) {
  const uint32_t low = (uint32_t)__uint_as_float(__float_as_uint(w) & ~((1u << kBinShift) - 1));
  return ((uint64_t)1 << kCountShift) | ((uint32_t)w - low);
}
__device__ __forceinline__ uint32_t entry_count(uint64_t e) { return (uint32_t)(e >> kCountShift); }
__device__ __forceinline__ uint64_t entry_sum(uint64_t e, uint32_t bin) {
  return (e & (((uint64_t)1 << kCountShift) - 1)) + (uint64_t)entry_count(e) * bin_low(bin);
}

// Calls f(logit, token) for the logits that thread `from` of `threads` of a row
// takes, four 16-byte loads in flight.
template <int DT, class F>
__device__ __forceinline__ void each(const char* x, uint32_t vocab, uint32_t from, uint32_t threads,
                                     F f) {
  constexpr int N = Elem<DT>::N, U = 4;
  const uint32_t nv = vocab / N;
  uint32_t v = from;
  for (; v + (U - 1) * threads < nv; v += U * threads) {
    u32x4 q[U];
#pragma unroll
    for (int u = 0; u < U; ++u) q[u] = load_vec<DT>(x, v + u * threads);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float l[N];
      unpack<DT>(q[u], l);
#pragma unroll
      for (int i = 0; i < N; ++i) f(l[i], (v + u * threads) * N + i);
    }
  }
  for (; v < nv; v += threads) {
    float l[N];
    unpack<DT>(load_vec<DT>(x, v), l);
#pragma unroll
    for (int i = 0; i < N; ++i) f(l[i], v * N + i);
  }
  for (uint32_t i = nv * N + from; i < vocab; i += threads) f(load1<DT>(x, i), i);
}
template <int DT> __device__ __forceinline__ const char* row_of(const SampleArgs& a, uint32_t row) {
  return (const char*)a.logits + (size_t)row * a.ld * sizeof(typename Elem<DT>::T);
}

// Running counts and sums before each bin, bins in the order's direction
// (q = 4095 - bin), and in all at q = 4096.
struct Edges {
  uint64_t sum[kBins + 1];
  uint32_t cnt[kBins + 1];
};
template <int THREADS_, uint32_t LIST_> struct Shared {
  static constexpr int THREADS = THREADS_;
  static constexpr uint32_t LIST = LIST_;  // collected elements that are sorted in LDS
  Edges e;
  uint64_t list[LIST];
  uint64_t red[THREADS / 64];
  uint32_t redc[THREADS / 64];
  uint32_t n;
  // Answers of a search.
  uint32_t q[2];
  uint64_t key, sum;
};

// Edges from the histogram in sh.e.sum (in place) or in memory.
template <bool SHARED, class S> __device__ void make_edges(S& sh, unsigned long long* hist) {
  constexpr int THREADS = S::THREADS, PER = kBins / THREADS;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  uint32_t c[PER];
  uint64_t w[PER], ws = 0;
  uint32_t cs = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const uint32_t b = kBins - 1 - (t * PER + i);
    // SHARED: other blocks of the launch have added to it, device scope.
    const uint64_t x = SHARED ? __hip_atomic_load(hist + b, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)
                       : hist ? hist[b] : sh.e.sum[b];
    c[i] = entry_count(x);
    w[i] = entry_sum(x, b);
    cs += c[i];
    ws += w[i];
  }
  uint32_t pc = cs;
  uint64_t pw = ws;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t xc = __shfl_up(pc, o);
    const uint64_t xw = __shfl_up(pw, o);
    if (lane >= o) {
      pc += xc;
      pw += xw;
    }
  }
  if (lane == 63) {
    sh.redc[wave] = pc;
    sh.red[wave] = pw;
  }
  __syncthreads();  // also: the histogram has been read
  for (int i = 0; i < wave; ++i) {
    pc += sh.redc[i];
    pw += sh.red[i];
  }
  pc -= cs;
  pw -= ws;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    sh.e.cnt[t * PER + i] = pc;
    sh.e.sum[t * PER + i] = pw;
    pc += c[i];
    pw += w[i];
  }
  if (t == THREADS - 1) {
    sh.e.cnt[kBins] = pc;
    sh.e.sum[kBins] = pw;
  }
  __syncthreads();
}

// The bins in which the running sum reaches a and b (at least 1, at most the
// total; a <= b).
template <class S>
__device__ void bins_of_sums(S& sh, uint64_t a, uint64_t b, uint32_t* qa, uint32_t* qb) {
  for (int q = threadIdx.x; q < kBins; q += S::THREADS) {
    const uint64_t lo = sh.e.sum[q], hi = sh.e.sum[q + 1];
    if (lo < a && a <= hi) sh.q[0] = q;
    if (lo < b && b <= hi) sh.q[1] = q;
  }
  __syncthreads();
  *qa = sh.q[0];
  *qb = sh.q[1];
  __syncthreads();
}
template <class S> __device__ uint32_t bin_of_count(S& sh, uint32_t k) {
  for (int q = threadIdx.x; q < kBins; q += S::THREADS)
    if (sh.e.cnt[q] < k && k <= sh.e.cnt[q + 1]) sh.q[0] = q;
  __syncthreads();
  const uint32_t q = sh.q[0];
  __syncthreads();
  return q;
}

// A row's settings, the inactive ones at k = 0, p = 1, least = 0.
struct Settings {
  uint32_t k;
  float p, least, u;  // least: min-p's smallest weight
};
__device__ Settings settings_of(const SampleArgs& a, uint32_t row) {
  Settings s;
  const int32_t k = a.top_k ? a.top_k[row] : 0;
  s.k = k > 0 ? (uint32_t)k : 0;
  // The most likely token alone: of equal ones the first.
  if (a.temperature && !(a.temperature[row] > 0.f)) s.k = 1;
  const float p = a.top_p ? a.top_p[row] : 1.f;
  s.p = p < 1.f ? fmaxf(p, 0.f) : 1.f;
  const float m = a.min_p ? a.min_p[row] : 0.f;
  const float least = m > 0.f ? rintf(fminf(m, 1.f) * kUnit) : 0.f;
  s.least = least > 1.f ? least : 0.f;
  const float u = a.u[row];
  s.u = u > 0.f ? fminf(u, 1.f) : 0.f;
  return s;
}
template <class S> __device__ __forceinline__ bool cuts(const Settings& s, const S& sh) {
  return s.k && s.k < sh.e.cnt[kBins];
}
__device__ __forceinline__ uint64_t part_of(uint64_t sum, float p) {
  const uint64_t x = (uint64_t)((double)sum * (double)p);
  return x > 1 ? x : 1;
}
__device__ __forceinline__ uint64_t target_of(uint64_t sum, float u) {
  const uint64_t x = (uint64_t)((double)sum * (double)u);
  return (x < sum ? x : sum - 1) + 1;
}

// The bins that may hold an answer.
struct Ranges {
  uint32_t lo[4], n[4];  // q from lo on, n bins
  __device__ bool holds(uint32_t q) const {
    return q - lo[0] < n[0] || q - lo[1] < n[1] || q - lo[2] < n[2] || q - lo[3] < n[3];
  }
};
template <class S> __device__ Ranges ranges_of(S& sh, const Settings& s) {
  Ranges r{{0, 0, 0, 0}, {0, 0, 0, 0}};
  uint64_t lo = sh.e.sum[kBins], hi = lo;  // what is kept so far sums to something in lo .. hi
  if (cuts(s, sh)) {
    const uint32_t q = bin_of_count(sh, s.k);
    lo = sh.e.sum[q] + 1;
    hi = sh.e.sum[q + 1];
    r.lo[0] = q;
    r.n[0] = 1;
  }
  if (s.p < 1.f) {
    uint32_t qa, qb;
    lo = part_of(lo, s.p);
    bins_of_sums(sh, lo, part_of(hi, s.p), &qa, &qb);
    hi = min(hi, sh.e.sum[qb + 1]);
    r.lo[1] = qa;
    r.n[1] = qb - qa + 1;
  }
  if (s.least != 0.f) {
    const uint32_t q = kBins - 1 - bin_of(s.least);
    if (sh.e.sum[q] < hi) {
      r.lo[2] = q;
      r.n[2] = 1;
      hi = min(hi, sh.e.sum[q + 1]);
      lo = max((uint64_t)1, min(lo, sh.e.sum[q]));
    }
  }
  uint32_t qa, qb;
  bins_of_sums(sh, target_of(lo, s.u), target_of(hi, s.u), &qa, &qb);
  r.lo[3] = qa;
  r.n[3] = qb - qa + 1;
  return r;
}

// Sorts sh.list[0 .. n), larger keys first; n <= LIST.  A bitonic network; its
// steps within 64 neighbours run in a wave's registers (an element a lane), so
// only the longer ones need barriers.
template <class S> __device__ void sort_list(S& sh, uint32_t n) {
  constexpr uint32_t THREADS = S::THREADS;
  const uint32_t lane = threadIdx.x & 63;
  uint32_t size = 64;
  while (size < n) size <<= 1;
  for (uint32_t i = n + threadIdx.x; i < size; i += THREADS) sh.list[i] = 0;
  __syncthreads();
  // Steps j, j / 2, ... 1 of stage k, j <= 32, for the waves' runs of 64.
  auto within = [&](uint32_t k, uint32_t from) {
    for (uint32_t i = threadIdx.x; i < size; i += THREADS) {  // whole waves
      uint64_t x = sh.list[i];
      for (uint32_t kk = from; kk <= k; kk <<= 1)
        for (uint32_t j = min(kk >> 1, 32u); j; j >>= 1) {
          const uint64_t y = __shfl_xor(x, (int)j);
          // Descending runs where bit kk of i is clear: their lower half keeps the larger.
          const bool larger = ((i & kk) == 0) == ((lane & j) == 0);
          x = (x > y) == larger ? x : y;
        }
      sh.list[i] = x;
    }
    __syncthreads();
  };
  within(min(size, 64u), 2);
  for (uint32_t k = 128; k <= size; k <<= 1) {
    for (uint32_t j = k >> 1; j >= 64; j >>= 1) {
      for (uint32_t p = threadIdx.x; p < size / 2; p += THREADS) {
        const uint32_t i = 2 * p - (p & (j - 1)), o = i + j;  // i without bit j
        const uint64_t x = sh.list[i], y = sh.list[o];
        if ((x < y) == ((i & k) == 0)) {
          sh.list[i] = y;
          sh.list[o] = x;
        }
      }
      __syncthreads();
    }
    within(k, k);
  }
}

__device__ __forceinline__ uint32_t order_bin(uint64_t key) {
  return kBins - 1 - (uint32_t)(key >> (kKeyBits - 12));
}
__device__ void answer(const SampleArgs& a, uint32_t row, uint64_t key, uint64_t kept) {
  a.token[row] = (int32_t)key_id(key);
  if (a.prob) a.prob[row] = (float)((double)(uint64_t)key_weight(key) / (double)kept);
}

// Answers the four questions from the edges and the collected bins' n elements,
// sorted in sh.list.
template <class S>
__device__ void resolve(const SampleArgs& a, uint32_t row, S& sh, const Settings& s, uint32_t n) {
  constexpr int PER = S::LIST / S::THREADS;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const uint32_t qm = s.least != 0.f ? kBins - 1 - bin_of(s.least) : 0;
  const uint64_t total = sh.e.sum[kBins], edge_m = sh.e.sum[qm];
  const bool k_cuts = cuts(s, sh);
  // Running sums of the list.
  uint64_t key[PER], w[PER], cum[PER], run = 0;
  uint32_t cnt[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const uint32_t at = t * PER + i;
    key[i] = at < n ? sh.list[at] : 0;
    w[i] = at < n ? (uint64_t)key_weight(key[i]) : 0;
    run += w[i];
    cum[i] = run;
  }
  uint64_t pre = run;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint64_t x = __shfl_up(pre, o);
    if (lane >= o) pre += x;
  }
  if (lane == 63) sh.red[wave] = pre;
  __syncthreads();
  pre -= run;
  for (int i = 0; i < wave; ++i) pre += sh.red[i];
  // Of the order: an element's bin's edge, plus what the list has of its bin up
  // to it.  The first element of each bin makes the bin's edge relative to the list.
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const uint32_t at = t * PER + i;
    cum[i] += pre;
    if (at < n) {
      const uint32_t q = order_bin(key[i]);
      if (at == 0 || q != order_bin(sh.list[at - 1])) {
        sh.e.sum[q] -= cum[i] - w[i];
        sh.e.cnt[q] -= at;
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const uint32_t at = t * PER + i, q = order_bin(key[i]);
    if (at < n) {
      cum[i] += sh.e.sum[q];
      cnt[i] = at + 1 + sh.e.cnt[q];
    }
  }
  uint64_t kept = total, cut = 0;
  // The element that `is` holds for: its key and running sum.
  auto find = [&](auto is) {
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if ((uint32_t)(t * PER + i) < n && is(i)) {
        sh.key = key[i];
        sh.sum = cum[i];
      }
    __syncthreads();
    cut = sh.key;
    const uint64_t sum = sh.sum;
    __syncthreads();
    return sum;
  };
  if (k_cuts) kept = find([&](int i) { return cnt[i] == s.k; });
  if (s.p < 1.f) {
    const uint64_t part = part_of(kept, s.p);
    kept = find([&](int i) { return cum[i] >= part && cum[i] - w[i] < part; });
  }
  const uint64_t key_m = s.least != 0.f ? (uint64_t)(__float_as_uint(s.least) - kOneBits) << kIdBits : 0;
  if (key_m > cut) {  // through the last element of at least that weight
    if (t == 0) sh.sum = edge_m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if ((uint32_t)(t * PER + i) < n && order_bin(key[i]) == qm && key[i] >= key_m)
        atomicMax((unsigned long long*)&sh.sum, (unsigned long long)cum[i]);
    __syncthreads();
    kept = sh.sum;
    __syncthreads();
  }
  const uint64_t at = target_of(kept, s.u);
  find([&](int i) { return cum[i] >= at && cum[i] - w[i] < at; });
  if (t == 0) answer(a, row, cut, kept);
}

// Rows whose answers' bins hold more than LIST elements (many equal or nearly
// equal logits): the element at which the running count or sum reaches
// `target`, twelve bits of the key at a time over the elements that share the
// bits so far, each time over the whole row.  *sum: the sum through it.
// 151936 equal logits: 0.8 ms for the draw alone, 2.4 with top-k and top-p.
template <int DT, class S>
__device__ uint64_t reach(const char* x, uint32_t vocab, const Scale& r, S& sh,
                          uint64_t target, bool by_count, uint64_t* sum) {
  constexpr int kThreads = S::THREADS;
  uint64_t prefix = 0, base = 0;
  for (int left = kKeyBits; left > 0;) {
    const int digit = left > 12 ? 12 : left, shift = left - digit;
    __syncthreads();
    for (int b = threadIdx.x; b < kBins; b += kThreads) {
      sh.e.cnt[b] = 0;
      sh.e.sum[b] = 0;
    }
    __syncthreads();
    each<DT>(x, vocab, threadIdx.x, kThreads, [&](float l, uint32_t id) {
      const float w = weight(r, l);
      if (w == 0.f) return;
      const uint64_t k = key_of(w, id);
      if (k >> left != prefix) return;
      const uint32_t q = kBins - 1 - ((uint32_t)(k >> shift) & ((1u << digit) - 1));
      atomicAdd(&sh.e.cnt[q], 1u);
      atomicAdd((unsigned long long*)&sh.e.sum[q], (unsigned long long)w);
    });
    __syncthreads();
    // Edges of these bins (a thread's four in turn), and the one that holds the target.
    constexpr int PER = kBins / kThreads;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    uint64_t w[PER], ws = 0;
    uint32_t c[PER], cs = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      c[i] = sh.e.cnt[t * PER + i];
      w[i] = sh.e.sum[t * PER + i];
      cs += c[i];
      ws += w[i];
    }
    uint64_t pc = cs, pw = ws;
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
        sh.q[0] = t * PER + i;
        sh.key = have;
        sh.sum = base + pw + (shift == 0 ? w[i] : 0);
      }
      pc += c[i];
      pw += w[i];
    }
    __syncthreads();
    prefix = (prefix << digit) | ((kBins - 1 - sh.q[0]) & ((1u << digit) - 1));
    target -= sh.key;
    base = sh.sum;
    left = shift;
  }
  *sum = base;
  __syncthreads();
  return prefix;
}

template <int DT, class S>
__device__ void resolve_long(const SampleArgs& a, uint32_t row, const Scale& r, S& sh,
                             const Settings& s) {
  constexpr int kThreads = S::THREADS;
  const char* x = row_of<DT>(a, row);
  uint64_t kept = sh.e.sum[kBins], cut = 0;
  const bool k_cuts = cuts(s, sh);
  if (k_cuts) cut = reach<DT>(x, a.vocab, r, sh, s.k, true, &kept);
  if (s.p < 1.f) cut = reach<DT>(x, a.vocab, r, sh, part_of(kept, s.p), false, &kept);
  if (s.least != 0.f && (uint64_t)(__float_as_uint(s.least) - kOneBits) << kIdBits > cut) {
    uint64_t sum = 0;
    each<DT>(x, a.vocab, threadIdx.x, kThreads, [&](float l, uint32_t) {
      const float w = weight(r, l);
      sum += w >= s.least ? (uint64_t)w : 0;
    });
    kept = block_add<uint64_t, kThreads>(sum, sh.red);
  }
  uint64_t through;
  const uint64_t key = reach<DT>(x, a.vocab, r, sh, target_of(kept, s.u), false, &through);
  if (threadIdx.x == 0) answer(a, row, key, kept);
}

// Collects the elements of the ranges' bins that this thread's logits hold:
// f(key).  Logits surely below the last bin are passed over by a comparison
// (a thousandth of slack; the bins of the others are exact).
template <int DT, class F>
__device__ __forceinline__ void collect(const char* x, uint32_t vocab, uint32_t from,
                                        uint32_t threads, const Scale& r, const Ranges& g, F f) {
  uint32_t last = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) last = g.n[i] ? max(last, g.lo[i] + g.n[i] - 1) : last;
  const float low = fmaxf((float)bin_low(kBins - 1 - last) - 1.f, 0.25f);
  const float below = (__logf(low * (1.f / kUnit)) - 1e-3f) / r.inv_t;
  const float least = r.top == INFINITY ? r.top : r.top + below * (1.f + 1e-3f) - fabsf(r.top) * 1e-6f;
  each<DT>(x, vocab, from, threads, [&](float l, uint32_t id) {
    if (!(l >= least)) return;
    const float w = weight(r, l);
    if (w != 0.f && g.holds(kBins - 1 - bin_of(w))) f(key_of(w, id));
  });
}

__device__ void no_token(const SampleArgs& a, uint32_t row) {
  a.token[row] = -1;
  if (a.prob) a.prob[row] = 0.f;
}

// ---- bfloat16 rows -------------------------------------------------------------
// A bfloat16 logit has few values, so the values themselves are counted: a bin a
// value, for magnitudes from 2^-8 up to 2^8 (2048 of either sign), in one pass
// that needs neither the maximum nor a weight for each logit.  All elements of a
// bin have one weight, so the counts give the running sums exactly, and an
// answer is a bin and a number in it; bins whose weights are equal once rounded
// are one group, and neighbours, since weights fall with the logits.  A second pass finds the token, the group's j-th.
// Logits below 2^-8 in magnitude ("small") are kept one by one for their sum; a
// row whose answer they touch, or that has a logit of 2^8 or more, or one of
// -2^8 or less with a weight, takes the way of float32 rows.
// 256 rows of 151936, top-p: 50 us, that way 95; 300 of 33333: 30 and 41.
constexpr uint32_t kFirst = 119u << 7, kHalf = 2048, kSmall = kHalf;  // the bits of 2^-8
static_assert(2 * kHalf == kBins, "the values' counts lie where the edges do");
__device__ __forceinline__ float value_of(uint32_t q) {  // of a bin other than kSmall
  return __uint_as_float((q < kSmall ? kFirst + (kHalf - 1 - q) : 0x8000u | (kFirst + (q - kSmall - 1))) << 16);
}

template <class S>
__device__ bool row_of_values(const SampleArgs& a, uint32_t row, const char* x, float inv_t, S& sh) {
  constexpr int THREADS = S::THREADS, WAVES = THREADS / 64, PER = (kBins + THREADS) / THREADS;
  constexpr uint32_t MOST = S::LIST;
  const int t = threadIdx.x, lane = t & 63;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(t >> 6);
  uint32_t* cnt = sh.e.cnt;
  float* small = (float*)sh.list;
  for (int q = t; q <= kBins; q += THREADS) cnt[q] = 0;
  if (t == 0) {
    sh.n = 0;         // small logits
    sh.q[0] = 0;      // a logit of 2^8 or more
    sh.q[1] = 0xFFFFu;  // bits of the largest logit of -2^8 or less
  }
  __syncthreads();
  auto count = [&](uint32_t u) {
    const uint32_t m = (u & 0x7FFFu) - kFirst;
    if (m < kHalf) {
      atomicAdd(&cnt[(u & 0x8000u) ? kSmall + 1 + m : kHalf - 1 - m], 1u);
    } else if ((u & 0x7FFFu) < kFirst) {
      const uint32_t at = atomicAdd(&sh.n, 1u);
      if (at < MOST) small[at] = __uint_as_float(u << 16);
    } else if ((u & 0x7FFFu) <= 0x7F80u) {  // no NaN
      if (u & 0x8000u)
        atomicMin(&sh.q[1], u);
      else
        sh.q[0] = 1;
    }
  };
  const uint32_t nv = a.vocab / 8;
  {
    auto eight = [&](u32x4 q) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        count(q[i] & 0xFFFFu);
        count(q[i] >> 16);
      }
    };
    constexpr int U = 4;
    uint32_t i = t;
    for (; i + (U - 1) * THREADS < nv; i += U * THREADS) {
      u32x4 q[U];
#pragma unroll
      for (int u = 0; u < U; ++u) q[u] = load_vec<TFE_BF16>(x, i + u * THREADS);
#pragma unroll
      for (int u = 0; u < U; ++u) eight(q[u]);
    }
    for (; i < nv; i += THREADS) eight(load_vec<TFE_BF16>(x, i));
    for (uint32_t k = nv * 8 + t; k < a.vocab; k += THREADS) count(((const uint16_t*)x)[k]);
  }
  __syncthreads();
  // The largest logit.
  const uint32_t smalls = sh.n, far = sh.q[1];
  if (sh.q[0] || smalls > MOST) return false;
  uint32_t c[PER];
  float top = -INFINITY;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const uint32_t q = t * PER + i;
    c[i] = q <= kBins && q != kSmall ? cnt[q] : 0;
    if (c[i]) top = fmaxf(top, value_of(q));
  }
  for (uint32_t i = t; i < smalls; i += THREADS) top = fmaxf(top, small[i]);
  const Scale r{block_max<float, THREADS>(top, (float*)sh.red), inv_t};
  if (r.top == -INFINITY) return false;
  if (far != 0xFFFFu && weight(r, __uint_as_float(far << 16)) != 0.f) return false;
  // The small logits' sum, and their least and largest weight.
  uint64_t small_sum = 0;
  uint32_t small_cnt = 0;
  float small_most = 0.f, small_least = kUnit;
  if (smalls) {
    for (uint32_t i = t; i < smalls; i += THREADS) {
      const float w = weight(r, small[i]);
      small_sum += (uint64_t)w;
      small_cnt += w != 0.f;
      small_most = fmaxf(small_most, w);
      small_least = fminf(small_least, w);
    }
    small_sum = block_add<uint64_t, THREADS>(small_sum, sh.red);
    small_cnt = block_add<uint32_t, THREADS>(small_cnt, sh.redc);
    small_most = block_max<float, THREADS>(small_most, (float*)sh.red);
    small_least = -block_max<float, THREADS>(-small_least, (float*)sh.red);
  }
  // Whether the small logits' order matters to an answer of weight w.
  auto touched = [&](float w) { return smalls && w >= small_least && w <= small_most; };
  // Edges: this thread's bins' counts and sums, and those before them.
  float w[PER];
  uint64_t sum[PER], ws = 0, pw[PER];
  uint32_t cs = 0, pc[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const uint32_t q = t * PER + i;
    w[i] = c[i] ? weight(r, value_of(q)) : 0.f;
    if (w[i] == 0.f) c[i] = 0;
    sum[i] = (uint64_t)c[i] * (uint32_t)w[i];
    if (q == kSmall && smalls) {
      c[i] = small_cnt;
      sum[i] = small_sum;
    }
    cs += c[i];
    ws += sum[i];
  }
  uint32_t ic = cs;
  uint64_t iw = ws;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t xc = __shfl_up(ic, o);
    const uint64_t xw = __shfl_up(iw, o);
    if (lane >= o) {
      ic += xc;
      iw += xw;
    }
  }
  if (lane == 63) {
    sh.redc[wave] = ic;
    sh.red[wave] = iw;
  }
  __syncthreads();
  uint32_t all_c = 0;
  uint64_t kept = 0;
  ic -= cs;
  iw -= ws;
  for (uint32_t i = 0; i < (uint32_t)WAVES; ++i) {
    if (i < wave) {
      ic += sh.redc[i];
      iw += sh.red[i];
    }
    all_c += sh.redc[i];
    kept += sh.red[i];
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    pc[i] = ic;
    pw[i] = iw;
    ic += c[i];
    iw += sum[i];
  }
  // The group in which the running count or sum reaches `target`: its weight
  // (0: the small logits), and the count and sum before it.
  struct Group {
    float w;
    uint32_t cnt;
    uint64_t sum;
  };
  auto find = [&](uint64_t target, bool by_count) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const uint64_t have = by_count ? pc[i] : pw[i], get = by_count ? c[i] : sum[i];
      if (have < target && target <= have + get) sh.n = __float_as_uint(w[i]);
    }
    if (t == 0) {
      sh.sum = ~(uint64_t)0;
      sh.q[0] = ~0u;
    }
    __syncthreads();
    Group g;
    g.w = __uint_as_float(sh.n);
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (c[i] && w[i] == g.w) {
        atomicMin((unsigned long long*)&sh.sum, (unsigned long long)pw[i]);
        atomicMin(&sh.q[0], pc[i]);
      }
    __syncthreads();
    g.cnt = sh.q[0];
    g.sum = sh.sum;
    return g;
  };
  const Settings s = settings_of(a, row);
  if (s.k && s.k < all_c) {
    const Group g = find(s.k, true);
    if (g.w == 0.f || touched(g.w)) return false;
    kept = g.sum + (uint64_t)(s.k - g.cnt) * (uint32_t)g.w;
  }
  if (s.p < 1.f) {
    const uint64_t part = part_of(kept, s.p);
    const Group g = find(part, false);
    if (g.w == 0.f || touched(g.w)) return false;
    const uint32_t u = (uint32_t)g.w;
    kept = g.sum + (part - g.sum + u - 1) / u * u;
  }
  if (s.least != 0.f) {
    if (smalls && s.least > small_least && s.least <= small_most) return false;
    __syncthreads();
    if (t == 0) sh.sum = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (c[i] && (t * PER + i == (int)kSmall ? small_least : w[i]) >= s.least)
        atomicMax((unsigned long long*)&sh.sum, (unsigned long long)(pw[i] + sum[i]));
    __syncthreads();
    kept = min(kept, sh.sum);
  }
  const uint64_t at = target_of(kept, s.u);
  const Group g = find(at, false);
  if (g.w == 0.f || touched(g.w)) return false;
  const uint32_t nth = (uint32_t)((at - 1 - g.sum) / (uint32_t)g.w);
  // The group's values, and its nth element by token: a wave has consecutive logits.
  __syncthreads();
  if (t == 0) {
    sh.q[0] = ~0u;
    sh.q[1] = 0;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (c[i] && w[i] == g.w) {
      atomicMin(&sh.q[0], (uint32_t)(t * PER + i));
      atomicMax(&sh.q[1], (uint32_t)(t * PER + i));
    }
  __syncthreads();
  const float most = value_of(sh.q[0]), least = value_of(sh.q[1]);
  const uint32_t lo = (uint32_t)((uint64_t)nv * wave / WAVES), hi = (uint32_t)((uint64_t)nv * (wave + 1) / WAVES);
  const uint32_t tail = wave == WAVES - 1 && nv * 8 + lane < a.vocab ? nv * 8 + lane : ~0u;
  auto in = [&](float l) { return l >= least && l <= most; };
  auto matches = [&](u32x4 q) {
    float l[8];
    unpack<TFE_BF16>(q, l);
    uint32_t n = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) n += in(l[i]);
    return n;
  };
  uint32_t n = 0;
  {
    constexpr int U = 4;
    uint32_t i = lo + lane;
    for (; i + (U - 1) * 64 < hi; i += U * 64) {
      u32x4 q[U];
#pragma unroll
      for (int u = 0; u < U; ++u) q[u] = load_vec<TFE_BF16>(x, i + u * 64);
#pragma unroll
      for (int u = 0; u < U; ++u) n += matches(q[u]);
    }
    for (; i < hi; i += 64) n += matches(load_vec<TFE_BF16>(x, i));
    if (tail != ~0u) n += in(load1<TFE_BF16>(x, tail));
  }
  n = wave_add(n);
  if (lane == 0) sh.redc[wave] = n;
  __syncthreads();
  uint32_t before = 0;
  for (uint32_t i = 0; i < wave; ++i) before += sh.redc[i];
  if (nth >= before && nth < before + n) {
    // 64 vectors at a time, eight such loads in flight; their matches are counted
    // by ballots until the one that holds the element.
    constexpr int U = 8;
    bool found = false;
    for (uint32_t i = lo; i < hi && !found; i += U * 64) {
      u32x4 q[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        q[u] = u32x4{0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u};  // NaN: no match
        if (i + u * 64 + lane < hi) q[u] = load_vec<TFE_BF16>(x, i + u * 64 + lane);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float l[8];
        unpack<TFE_BF16>(q[u], l);
        uint32_t all = 0, below = 0;  // matches of the 64 vectors; of the lanes before
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint64_t m = __builtin_amdgcn_ballot_w64(in(l[j]));
          all += (uint32_t)__builtin_popcountll(m);
          below += (uint32_t)__builtin_popcountll(m & ((1ull << lane) - 1));
        }
        if (!found && nth < before + all) {
          uint32_t k = before + below;
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (in(l[j]) && k++ == nth) a.token[row] = (int32_t)((i + u * 64 + lane) * 8 + j);
          found = true;
        }
        before += all;
      }
    }
    const uint64_t last = __builtin_amdgcn_ballot_w64(tail != ~0u && in(load1<TFE_BF16>(x, tail != ~0u ? tail : 0)));
    if (!found && tail != ~0u && ((last >> lane) & 1) &&
        before + (uint32_t)__builtin_popcountll(last & ((1ull << lane) - 1)) == nth)
      a.token[row] = (int32_t)tail;
  }
  if (t == 0 && a.prob) a.prob[row] = (float)((double)(uint64_t)g.w / (double)kept);
  return true;
}

// One block a row.
template <int DT, int kThreads, uint32_t LIST>
__global__ __launch_bounds__(kThreads, 4) void k_row(SampleArgs a) {
  __shared__ Shared<kThreads, LIST> sh;
  const uint32_t row = blockIdx.x;
  const char* x = row_of<DT>(a, row);
  Scale r{-INFINITY, inverse_temperature(a, row)};
  if (DT == TFE_BF16 && row_of_values(a, row, x, r.inv_t, sh)) return;
  __syncthreads();
  for (int b = threadIdx.x; b < kBins; b += kThreads) sh.e.sum[b] = 0;
  if (threadIdx.x == 0) sh.n = 0;
  float top = -INFINITY;
  each<DT>(x, a.vocab, threadIdx.x, kThreads, [&](float l, uint32_t) { top = fmaxf(top, l); });
  r.top = block_max<float, kThreads>(top, (float*)sh.red);
  if (r.top == -INFINITY) {
    if (threadIdx.x == 0) no_token(a, row);
    return;
  }
  each<DT>(x, a.vocab, threadIdx.x, kThreads, [&](float l, uint32_t) {
    const float w = weight(r, l);
    if (w != 0.f) atomicAdd((unsigned long long*)&sh.e.sum[bin_of(w)], (unsigned long long)bin_entry(w));
  });
  __syncthreads();
  make_edges<false>(sh, nullptr);
  const Settings s = settings_of(a, row);
  const Ranges g = ranges_of(sh, s);
  collect<DT>(x, a.vocab, threadIdx.x, kThreads, r, g, [&](uint64_t key) {
    const uint32_t at = atomicAdd(&sh.n, 1u);
    if (at < LIST) sh.list[at] = key;
  });
  __syncthreads();
  const uint32_t n = sh.n;
  if (n <= LIST) {
    sort_list(sh, n);
    resolve(a, row, sh, s, n);
  } else {
    resolve_long<DT>(a, row, r, sh, s);
  }
}

// Few rows: a row's passes are split over `parts` blocks each (a launch a pass:
// the kernel's end is the barrier), and a block a row finishes.
constexpr uint32_t kMaxParts = 64;
constexpr uint32_t kList = 8192, kPartList = 2048;
constexpr int kMaxThreads = 512, kHistThreads = 1024, kCollectThreads = 512, kFinishThreads = 1024;
struct Part {  // a row's workspace
  unsigned long long hist[kBins];
  unsigned long long list[kList];
  float top[kMaxParts];
  Ranges ranges;
  uint32_t n, done, pad[2];
};

template <int DT>
__global__ __launch_bounds__(kMaxThreads) void k_part_max(SampleArgs a, uint32_t parts) {
  __shared__ float red[kMaxThreads / 64];
  const uint32_t row = blockIdx.y, part = blockIdx.x;
  Part& p = ((Part*)a.space)[row];
  for (uint32_t b = part * kMaxThreads + threadIdx.x; b < kBins; b += parts * kMaxThreads) p.hist[b] = 0;
  float top = -INFINITY;
  each<DT>(row_of<DT>(a, row), a.vocab, part * kMaxThreads + threadIdx.x, parts * kMaxThreads,
           [&](float l, uint32_t) { top = fmaxf(top, l); });
  top = block_max<float, kMaxThreads>(top, red);
  if (threadIdx.x == 0) {
    p.top[part] = top;
    if (part == 0) p.n = p.done = 0;
  }
}
__device__ __forceinline__ float top_of(const Part& p, uint32_t parts) {
  const uint32_t lane = threadIdx.x & 63;
  return wave_max(lane < parts ? p.top[lane] : -INFINITY);
}

template <int DT>
__global__ __launch_bounds__(kHistThreads) void k_part_hist(SampleArgs a, uint32_t parts) {
  __shared__ Shared<kHistThreads, 1> sh;
  const uint32_t row = blockIdx.y, part = blockIdx.x;
  Part& p = ((Part*)a.space)[row];
  const Scale r{top_of(p, parts), inverse_temperature(a, row)};
  if (r.top == -INFINITY) return;
  for (int b = threadIdx.x; b < kBins; b += kHistThreads) sh.e.sum[b] = 0;
  __syncthreads();
  each<DT>(row_of<DT>(a, row), a.vocab, part * kHistThreads + threadIdx.x, parts * kHistThreads,
           [&](float l, uint32_t) {
             const float w = weight(r, l);
             if (w != 0.f)
               atomicAdd((unsigned long long*)&sh.e.sum[bin_of(w)], (unsigned long long)bin_entry(w));
           });
  __syncthreads();
  for (int b = threadIdx.x; b < kBins; b += kHistThreads)
    if (sh.e.sum[b])
      __hip_atomic_fetch_add(&p.hist[b], sh.e.sum[b], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  // The last block to get here has the row's whole histogram: it finds the bins.
  // What blocks tell each other goes through device-scope atomics alone, and a
  // block counts itself in once its own are done: no fence (writing the L2s
  // back for one took 90 us at 64 rows).
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0)
    sh.n = __hip_atomic_fetch_add(&p.done, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  if (sh.n != parts - 1) return;
  make_edges<true>(sh, p.hist);
  const Ranges g = ranges_of(sh, settings_of(a, row));
  if (threadIdx.x == 0) p.ranges = g;
}

template <int DT>
__global__ __launch_bounds__(kCollectThreads) void k_part_collect(SampleArgs a, uint32_t parts) {
  __shared__ uint64_t list[kPartList];
  __shared__ uint32_t count, base;
  const uint32_t row = blockIdx.y, part = blockIdx.x;
  Part& p = ((Part*)a.space)[row];
  const Scale r{top_of(p, parts), inverse_temperature(a, row)};
  if (r.top == -INFINITY) return;
  if (threadIdx.x == 0) count = 0;
  __syncthreads();
  const Ranges g = p.ranges;
  collect<DT>(row_of<DT>(a, row), a.vocab, part * kCollectThreads + threadIdx.x,
              parts * kCollectThreads, r, g, [&](uint64_t key) {
                const uint32_t at = atomicAdd(&count, 1u);
                if (at < kPartList) list[at] = key;
              });
  __syncthreads();
  const uint32_t n = count;
  if (n == 0) return;
  // More than a list holds: the row's number is to exceed kList.
  if (threadIdx.x == 0) base = atomicAdd(&p.n, n <= kPartList ? n : kList + 1);
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < min(n, kPartList) && base + i < kList; i += kCollectThreads)
    p.list[base + i] = list[i];
}

template <int DT>
__global__ __launch_bounds__(kFinishThreads) void k_part_finish(SampleArgs a, uint32_t parts) {
  __shared__ Shared<kFinishThreads, kList> sh;
  const uint32_t row = blockIdx.x;
  Part& p = ((Part*)a.space)[row];
  const Scale r{top_of(p, parts), inverse_temperature(a, row)};
  if (r.top == -INFINITY) {
    if (threadIdx.x == 0) no_token(a, row);
    return;
  }
  const uint32_t n = p.n;
  const Settings s = settings_of(a, row);
  if (n <= kList) {
    for (uint32_t i = threadIdx.x; i < n; i += kFinishThreads) sh.list[i] = p.list[i];
    make_edges<false>(sh, p.hist);
    sort_list(sh, n);
    resolve(a, row, sh, s, n);
  } else {
    make_edges<false>(sh, p.hist);
    resolve_long<DT>(a, row, r, sh, s);
  }
}

// Blocks a row: about 512 in all, of at least 2048 logits each; one from 128 rows on.
// us split / one block a row, top-k and top-p, 151936 float32: 32 rows 43 / 46, 64 51 / 50,
// 100 64 / 53, 127 72 / 57, 128 66 / 56, 192 96 / 68, 256 106 / 83, 300 146 / 130; bfloat16: 32
// 40 / 38, 64 44 / 39, 127 58 / 43, 128 56 / 43, 256 77 / 61, 300 113 / 85; 33333 bfloat16: 32
// 34 / 22, 128 41 / 24, 256 45 / 38.  (Fewer than 64 rows, and 64 to 127, could gain from a
// block a row.)
uint32_t parts_of(int64_t rows, int32_t vocab) {
  if (rows >= 128) return 1;
  const uint32_t most = std::min<uint32_t>(kMaxParts, ((uint32_t)vocab + 2047) / 2048);
  return std::max(1u, std::min(most, (512 + (uint32_t)rows - 1) / (uint32_t)rows));
}

template <int DT> hipError_t launch(const SampleArgs& a, hipStream_t s) {
  const uint32_t parts = parts_of(a.rows, (int32_t)a.vocab);
  if (parts == 1) {
    // A short row's block leaves room for another on its compute unit.  us with 512 / 1024
    // threads, top-p: 300 rows of 33333 bfloat16 31 / 50, of 65000 40 / 68 (float32 72 / 86);
    // 128 rows of 151936 82 / 44 (101 / 80), 256 rows 86 / 50 (119 / 96), 300 rows, more than
    // compute units, 89 / 114 (156 / 164).
    if (a.vocab <= 65536)
      k_row<DT, 512, 2048><<<dim3(a.rows), dim3(512), 0, s>>>(a);
    else
      k_row<DT, 1024, 8192><<<dim3(a.rows), dim3(1024), 0, s>>>(a);
    return hipGetLastError();
  }
  const dim3 grid(parts, a.rows);
  k_part_max<DT><<<grid, dim3(kMaxThreads), 0, s>>>(a, parts);
  k_part_hist<DT><<<grid, dim3(kHistThreads), 0, s>>>(a, parts);
  k_part_collect<DT><<<grid, dim3(kCollectThreads), 0, s>>>(a, parts);
  k_part_finish<DT><<<dim3(a.rows), dim3(kFinishThreads), 0, s>>>(a, parts);
  return hipGetLastError();
}

}  // namespace

int64_t sample_space(int64_t rows, int32_t vocab) {
  return rows == 0 || parts_of(rows, vocab) == 1 ? 0 : rows * (int64_t)sizeof(Part);
}

hipError_t launch_sample(const SampleArgs& a, int dtype, hipStream_t s) {
  return dtype == TFE_F32 ? launch<TFE_F32>(a, s) : launch<TFE_BF16>(a, s);
}

}  // namespace tfe
