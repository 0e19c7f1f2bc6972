// Distillation from a teacher's top logits: the loss KL(q || p) of the
// teacher's softmax q over its K listed tokens against the student's softmax p
// over the vocabulary, both at temperature tau, and its gradient.
//   lse = log sum_v exp(s_v / tau)       (running maximum and sum, one pass)
//   loss = tau^2 sum_k q_k (log q_k - s_k / tau + lse)
//   d loss / d s_v = tau (p_v - q_v),    p_v = exp(s_v / tau - lse)
// A float32 lse far from zero does not show the sum: the loss uses the maximum
// and the sum themselves, and p does in rows with |lse| above kFar.
// Bound by the logits' bytes: the loss reads them, the gradient reads and
// writes them, and both together read and write them once.
//
// A row is split into parts of up to 2048 16-byte vectors, each a block of 256
// threads with eight vectors a thread in registers: many small blocks keep more
// of memory's latency hidden than few large ones (512 rows of 151936 bfloat16,
// loss alone: 30 us, 26 of them k_sum at 6.0 TB/s; one block of 1024 threads a row,
// the next row loaded while one is worked on: 41).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "tfe_logits.h"
#include "tfe_rows.h"

namespace tfe {
namespace {

using namespace rows;

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_hw(float x) { return __builtin_amdgcn_logf(x); }

// Maximum m and sum s of exp((x - m) / tau) of some logits.  While every one of
// them was -infinity, m is -infinity and s 0.  c = log2(e) / tau.
struct Running {
  float m, s;
};
__device__ __forceinline__ float finite_max(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ Running join(Running a, Running b, float c) {
  Running r;
  r.m = fmaxf(a.m, b.m);
  const float ref = finite_max(r.m);
  r.s = fmaf(a.s, exp2_hw((a.m - ref) * c), b.s * exp2_hw((b.m - ref) * c));
  return r;
}
__device__ __forceinline__ float lse_of(const DistillArgs& a, Running r) {
  return fmaf(r.m, a.inv_tau, log2_hw(r.s) * kLn2);
}
// Rounded by 2^-12 there, and so p by as much of itself.  Every probability of a
// row of -infinity is 0 (lse is -infinity; a row with NaN or +infinity has NaN).
constexpr float kFar = 4096.f;
__device__ __forceinline__ bool is_far(float lse) { return fabsf(lse) > kFar; }
// One vector's logits into r.  (Fused operations are written out here and in
// join: a sum has the same bits wherever it is computed.)
template <int DT> __device__ __forceinline__ void add(Running& r, u32x4 q, float c) {
  constexpr int N = Elem<DT>::N;
  float x[N];
  unpack<DT>(q, x);
  float m = r.m;
#pragma unroll
  for (int i = 0; i < N; ++i) m = fmaxf(m, x[i]);
  const float ref = finite_max(m);
  float s = fmaf(r.s, exp2_hw((r.m - ref) * c), exp2_hw((x[0] - ref) * c));
#pragma unroll
  for (int i = 1; i < N; ++i) s += exp2_hw((x[i] - ref) * c);
  r = Running{m, s};
}
__device__ __forceinline__ void add1(Running& r, float x, float c) {
  r = join(r, Running{x, x == -INFINITY ? 0.f : (x == x ? 1.f : x)}, c);
}

// The gradient's main part f p for one vector (f = upstream gradient x tau).
template <int DT>
__device__ __forceinline__ u32x4 scaled_softmax(const DistillArgs& a, u32x4 q, float lse, float f) {
  constexpr int N = Elem<DT>::N;
  float x[N];
  unpack<DT>(q, x);
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = f * exp2_hw(fmaf(x[i], a.inv_tau, -lse) * kLog2e);
  return pack<DT>(x);
}
__device__ __forceinline__ float scaled_softmax1(const DistillArgs& a, float x, float lse, float f) {
  return f * exp2_hw(fmaf(x, a.inv_tau, -lse) * kLog2e);
}

// The same in a row that is_far, from its maximum and sum (f: already over the sum).
template <int DT> __device__ __forceinline__ u32x4 far_softmax(u32x4 q, float ref, float c, float f) {
  constexpr int N = Elem<DT>::N;
  float x[N];
  unpack<DT>(q, x);
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = f * exp2_hw((x[i] - ref) * c);
  return pack<DT>(x);
}

// Entry k < K of a row is thread k's: its token (-1: padding), the teacher's
// logit (-infinity for padding) and the student's.
struct Entry {
  int32_t id;
  float t, s;
};
template <int DT, int TDT>
__device__ __forceinline__ Entry entry_of(const DistillArgs& a, uint32_t row, const char* x) {
  Entry e{-1, -INFINITY, 0.f};
  if (threadIdx.x >= a.K) return e;
  const size_t at = (size_t)row * a.K + threadIdx.x;
  e.id = a.ids[at];
  if (e.id < 0 || (uint32_t)e.id >= a.vocab) {
    e.id = -1;
    return e;
  }
  e.t = load1<TDT>(a.teacher, at);
  if (x) e.s = load1<DT>(x, (uint32_t)e.id);
  return e;
}

constexpr int kThreads = 256, kWaves = kThreads / 64;
static_assert(kDistillMaxK <= kThreads, "an entry a thread");
struct Shared {
  float q[kDistillMaxK];
  int32_t id[kDistillMaxK];
  float m[kWaves], s[kWaves], t[kWaves], some[kWaves], x[kWaves], y[kWaves];
  uint32_t ticket;
  unsigned long long missing;  // parts whose sums have not come
};
// What a row's entries come to.
struct Teacher {
  bool any;         // an entry has weight
  float q;          // this thread's entry's
  float gap;        // sum_k q_k (log q_k - (s_k - max) / tau), if the row's sum is given
};

// Joins the block's running sums and evaluates the entries; two barriers.  Nobody
// may still be reading `sh` from an earlier use.  Every thread gets the row's
// sum (if `r` is given) and its entry's q; sh.q and sh.id hold the entries'
// after the caller's next barrier.
__device__ __forceinline__ Teacher join_block(const DistillArgs& a, const Entry& e, Shared& sh,
                                              Running* r, float c) {
  const uint32_t wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  // NaN is weight, and stays NaN in the sums; fmaxf passes over it.
  const float top = wave_max(e.t == e.t ? e.t : -INFINITY);
  const bool some = __builtin_amdgcn_ballot_w64(!(e.t == -INFINITY)) != 0;
  if (r) {
#pragma unroll
    for (int o = 32; o; o >>= 1) *r = join(*r, Running{__shfl_xor(r->m, o), __shfl_xor(r->s, o)}, c);
  }
  if (lane == 0) {
    if (r) {
      sh.m[wave] = r->m;
      sh.s[wave] = r->s;
    }
    sh.t[wave] = top;
    sh.some[wave] = some ? 1.f : 0.f;
  }
  __syncthreads();
  if (r) {
    *r = Running{sh.m[0], sh.s[0]};
    for (int w = 1; w < kWaves; ++w) *r = join(*r, Running{sh.m[w], sh.s[w]}, c);
  }
  Teacher t;
  float tm = sh.t[0], any = sh.some[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) {
    tm = fmaxf(tm, sh.t[w]);
    any = fmaxf(any, sh.some[w]);
  }
  t.any = any != 0.f;
  // x = exp((t - max) / tau), their sum and that of x ((t - max) / tau - s).  Differences
  // before the division: t / tau of a list far from 0 may be rounded or infinite.
  const float s = r ? (e.s - finite_max(r->m)) * a.inv_tau : 0.f, d = (e.t - tm) * a.inv_tau;
  const float x = e.t == -INFINITY ? 0.f : expf(d);
  const float xs = wave_add(x), ys = wave_add(x == 0.f ? 0.f : x * (d - s));
  if (lane == 0) {
    sh.x[wave] = xs;
    sh.y[wave] = ys;
  }
  __syncthreads();
  float sum = sh.x[0], gap = sh.y[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) {
    sum += sh.x[w];
    gap += sh.y[w];
  }
  t.q = t.any ? x / sum : 0.f;
  t.gap = t.any ? gap / sum - logf(sum) : 0.f;
  if (threadIdx.x < kDistillMaxK) {
    sh.q[threadIdx.x] = t.q;
    sh.id[threadIdx.x] = t.any ? e.id : -1;
  }
  return t;
}
// The listed tokens again, with their q (an id listed twice: each writer adds
// the same entries in the same order); p: the token's probability.
template <int DT>
__device__ __forceinline__ void write_entry(const DistillArgs& a, const Entry& e, const Shared& sh,
                                            char* out, float p, float f) {
  float q = 0.f;
  for (uint32_t k = 0; k < a.K; ++k) q += sh.id[k] == e.id ? sh.q[k] : 0.f;
  store1<DT>(out, (uint32_t)e.id, f * (p - q));
}
__device__ __forceinline__ float p_of(const DistillArgs& a, float s, float lse) {
  return exp2_hw((s * a.inv_tau - lse) * kLog2e);
}

template <int DT> __device__ __forceinline__ const char* logits_of(const DistillArgs& a, uint32_t row) {
  return (const char*)a.logits + (size_t)row * a.ld * sizeof(typename Elem<DT>::T);
}
template <int DT> __device__ __forceinline__ char* grad_of(const DistillArgs& a, uint32_t row) {
  return (char*)a.grad + (size_t)row * a.ldg * sizeof(typename Elem<DT>::T);
}

// ---- parts of a row ------------------------------------------------------------

constexpr int kVectors = 8;  // of a thread
constexpr uint32_t kPart = kThreads * kVectors;
constexpr uint32_t kMaxParts = kLogitsMaxVocab / 4 / kPart;
static_assert(kMaxParts <= 64, "a part's sum a lane of the first wave");

// Workspace: a counter for each queue, then a record for each row of a launch: its parts' running
// sums (m in the low word, s in the high one).
struct Record {
  unsigned long long r[kMaxParts];
};
constexpr uint32_t kQueues = 8;
constexpr size_t kLine = 128, kRecords = kQueues * kLine;
__device__ __forceinline__ uint32_t* counter_of(const DistillArgs& a, uint32_t queue) {
  return (uint32_t*)(a.space + queue * kLine);
}
__device__ __forceinline__ Record& record_of(const DistillArgs& a, uint32_t row) {
  return ((Record*)(a.space + kRecords))[row];
}
// No sum looks like this: NaN is published as 0x7FC00000.
constexpr unsigned long long kUnset = ~0ull;
__device__ __forceinline__ unsigned long long packed(Running r) {
  const uint32_t s = r.s == r.s ? __float_as_uint(r.s) : 0x7FC00000u;
  return (unsigned long long)s << 32 | __float_as_uint(r.m);
}
__device__ __forceinline__ Running unpacked(unsigned long long x) {
  return Running{__uint_as_float((uint32_t)x), __uint_as_float((uint32_t)(x >> 32))};
}

// The running sum of a block's logits from those of its threads (r, of whole
// vectors) and the row's last few; in every thread.  `sh` may be reused after the
// last barrier.
template <int DT>
__device__ __forceinline__ Running block_sum(const DistillArgs& a, Running r, const char* x, bool last,
                                             float c, Shared& sh) {
  if (last)
    for (uint32_t i = a.vocab / Elem<DT>::N * Elem<DT>::N + threadIdx.x; i < a.vocab; i += kThreads)
      add1(r, load1<DT>(x, i), c);
#pragma unroll
  for (int o = 32; o; o >>= 1) r = join(r, Running{__shfl_xor(r.m, o), __shfl_xor(r.s, o)}, c);
  if ((threadIdx.x & 63) == 0) {
    sh.m[threadIdx.x >> 6] = r.m;
    sh.s[threadIdx.x >> 6] = r.s;
  }
  __syncthreads();
  r = Running{sh.m[0], sh.s[0]};
  for (int w = 1; w < kWaves; ++w) r = join(r, Running{sh.m[w], sh.s[w]}, c);
  __syncthreads();  // all have read: join_block writes the same words
  return r;
}

// The rest of a part's gradient: the row's last few logits, and the listed
// tokens among the part's.
template <int DT>
__device__ __forceinline__ void finish_grad(const DistillArgs& a, const char* x, char* out, bool last,
                                            bool zero, float lse, float f, const Entry& e, bool own,
                                            const Shared& sh) {
  if (last)
    for (uint32_t i = a.vocab / Elem<DT>::N * Elem<DT>::N + threadIdx.x; i < a.vocab; i += kThreads)
      store1<DT>(out, i, zero ? 0.f : scaled_softmax1(a, load1<DT>(x, i), lse, f));
  __syncthreads();
  if (!zero && own) write_entry<DT>(a, e, sh, out, p_of(a, e.s, lse), f);
}

// This thread's share of a part.
template <int DT> struct Share {
  int first, nv;  // its first vector; the row's
  u32x4 v[kVectors];
  __device__ __forceinline__ Share(const DistillArgs& a, uint32_t part)
      : first((int)(part * kPart + threadIdx.x)), nv((int)(a.vocab / Elem<DT>::N)) {}
  __device__ __forceinline__ bool has(int k) const { return first + k * kThreads < nv; }
  __device__ __forceinline__ void load(const char* x) {
#pragma unroll
    for (int k = 0; k < kVectors; ++k)
      if (has(k)) v[k] = load_stream<DT>(x, first + k * kThreads);
  }
  __device__ __forceinline__ Running sum(const DistillArgs& a, const char* x, bool last, float c,
                                         Shared& sh) const {
    Running r{-INFINITY, 0.f};
#pragma unroll
    for (int k = 0; k < kVectors; ++k)
      if (has(k)) add<DT>(r, v[k], c);
    return block_sum<DT>(a, r, x, last, c, sh);
  }
  // The part's gradient; the listed tokens among its logits last.
  __device__ __forceinline__ void grad(const DistillArgs& a, const char* x, char* out, bool last,
                                       bool zero, float lse, float f, const Entry& e, bool own,
                                       const Shared& sh) const {
#pragma unroll
    for (int k = 0; k < kVectors; ++k)
      if (has(k))
        store_stream<DT>(out, first + k * kThreads,
                         zero ? u32x4{0, 0, 0, 0} : scaled_softmax<DT>(a, v[k], lse, f));
    finish_grad<DT>(a, x, out, last, zero, lse, f, e, own, sh);
  }
};
// A part's running sum and its gradient, to the bit, without a place for its logits.
template <int DT>
__device__ __forceinline__ Running sum_of_part(const DistillArgs& a, const char* x, uint32_t part,
                                               bool last, float c, Shared& sh) {
  const uint32_t nv = a.vocab / Elem<DT>::N, first = part * kPart + threadIdx.x;
  Running r{-INFINITY, 0.f};
#pragma unroll 1
  for (uint32_t i = first; i < min(nv, first + kPart); i += kThreads) add<DT>(r, load_vec<DT>(x, i), c);
  return block_sum<DT>(a, r, x, last, c, sh);
}
template <int DT>
__device__ __forceinline__ void grad_of_part(const DistillArgs& a, const char* x, char* out, uint32_t part,
                                             bool last, bool zero, float lse, float f, const Entry& e,
                                             bool own, const Shared& sh) {
  const uint32_t nv = a.vocab / Elem<DT>::N, first = part * kPart + threadIdx.x;
#pragma unroll 1
  for (uint32_t i = first; i < min(nv, first + kPart); i += kThreads)
    store_vec<DT>(out, i, zero ? u32x4{0, 0, 0, 0} : scaled_softmax<DT>(a, load_vec<DT>(x, i), lse, f));
  finish_grad<DT>(a, x, out, last, zero, lse, f, e, own, sh);
}
// The gradient of vectors from .. to of a row that is_far, and of its last few logits.
template <int DT>
__device__ __forceinline__ void grad_of_far(const DistillArgs& a, const char* x, char* out, uint32_t from,
                                            uint32_t to, bool last, Running r, float f, const Entry& e,
                                            bool own, const Shared& sh) {
  const float c = a.inv_tau * kLog2e, ref = finite_max(r.m), inv = r.s == 0.f ? 0.f : 1.f / r.s;
#pragma unroll 1
  for (uint32_t i = from + threadIdx.x; i < to; i += kThreads)
    store_vec<DT>(out, i, far_softmax<DT>(load_vec<DT>(x, i), ref, c, f * inv));
  if (last)
    for (uint32_t i = a.vocab / Elem<DT>::N * Elem<DT>::N + threadIdx.x; i < a.vocab; i += kThreads)
      store1<DT>(out, i, f * inv * exp2_hw((load1<DT>(x, i) - ref) * c));
  __syncthreads();
  if (own) write_entry<DT>(a, e, sh, out, exp2_hw((e.s - ref) * c) * inv, f);
}
template <int DT>
__device__ __forceinline__ bool owns(const DistillArgs& a, const Entry& e, uint32_t part, uint32_t parts) {
  const uint32_t from = part * kPart * Elem<DT>::N;
  return e.id >= 0 && (uint32_t)e.id >= from && (part == parts - 1 || (uint32_t)e.id < from + kPart * Elem<DT>::N);
}
// No sum: the gap is infinite.
__device__ __forceinline__ void write_loss(const DistillArgs& a, uint32_t row, const Teacher& q, Running r) {
  const float sum = r.s == 0.f ? 0.f : log2_hw(r.s) * kLn2;
  a.loss[row] = q.any ? a.tau * a.tau * (q.gap + sum) : 0.f;
  a.lse[row] = lse_of(a, r);
}

// The loss of rows in several parts: the parts' sums, then a block a row.
template <int DT, int TDT>
__global__ __launch_bounds__(kThreads, 8) void k_sum(DistillArgs a) {
  __shared__ Shared sh;
  const uint32_t row = blockIdx.y, part = blockIdx.x;
  const char* x = logits_of<DT>(a, row);
  Share<DT> v(a, part);
  v.load(x);
  const Running r = v.sum(a, x, part == gridDim.x - 1, a.inv_tau * kLog2e, sh);
  if (threadIdx.x == 0) record_of(a, row).r[part] = packed(r);
}
template <int DT, int TDT>
__global__ __launch_bounds__(kThreads, 8) void k_loss(DistillArgs a, uint32_t parts) {
  __shared__ Shared sh;
  const uint32_t row = blockIdx.x;
  const Entry e = entry_of<DT, TDT>(a, row, logits_of<DT>(a, row));
  Running r{-INFINITY, 0.f};
  if (threadIdx.x < parts) r = unpacked(record_of(a, row).r[threadIdx.x]);
  const Teacher q = join_block(a, e, sh, &r, a.inv_tau * kLog2e);
  if (threadIdx.x == 0) write_loss(a, row, q, r);
}

// A row that is_far, by one block.
template <int DT, int TDT>
__device__ __noinline__ void grad_seldom(DistillArgs a, uint32_t row, uint32_t parts, float f) {
  __shared__ Shared sh;
  const float c = a.inv_tau * kLog2e;
  const char* x = logits_of<DT>(a, row);
  const Entry e = entry_of<DT, TDT>(a, row, x);
  Running r{-INFINITY, 0.f};
  for (uint32_t p = 0; p < parts; ++p) {
    const Running one = sum_of_part<DT>(a, x, p, p == parts - 1, c, sh);
    if (threadIdx.x == p) r = one;
  }
  join_block(a, e, sh, &r, c);
  grad_of_far<DT>(a, x, grad_of<DT>(a, row), 0, a.vocab / Elem<DT>::N, true, r, f, e, e.id >= 0, sh);
}

// The gradient from a known log-sum-exp.  1023 x 40001 float32: 63 us, 5.2 TB/s.
template <int DT, int TDT>
__global__ __launch_bounds__(kThreads, 8) void k_grad(DistillArgs a) {
  __shared__ Shared sh;
  const uint32_t row = blockIdx.y, part = blockIdx.x, parts = gridDim.x;
  const char* x = logits_of<DT>(a, row);
  Share<DT> v(a, part);
  v.load(x);
  Entry e = entry_of<DT, TDT>(a, row, nullptr);
  const bool own = owns<DT>(a, e, part, parts);
  if (own) e.s = load1<DT>(x, (uint32_t)e.id);
  const Teacher q = join_block(a, e, sh, nullptr, 0.f);
  const float g = a.weight ? a.weight[row] : 1.f, lse = a.lse[row];
  const bool zero = !q.any || g == 0.f;
  if (!zero && is_far(lse)) {
    // One block does the row, so that nobody writes where another reads.
    if (part == 0) grad_seldom<DT, TDT>(a, row, parts, g * a.tau);
    return;
  }
  v.grad(a, x, grad_of<DT>(a, row), part == parts - 1, zero, lse, g * a.tau, e, own, sh);
}

// Both at once, the logits read once.  The parts of a row exchange their sums
// while each keeps its logits in registers: a part publishes its sum and waits
// for the others'.
//   Nobody depends on a wait: sums that have not come after wait_limit polls, for
// lack of room for their blocks beside other kernels, a block computes itself,
// with the same bits.  For that the logits have to stay, so a gradient in their
// place goes the way of two readings (k_sum, k_loss, k_grad).
//   That waits are short: rows are dealt to queues, and a block takes the next
// part of its queue from a counter when it starts.  A queue's blocks that wait
// are therefore all of its newest row (fewer than the row has parts; those of
// its earlier rows have all their parts running and need nobody else).  There
// are so few queues (queues_of) that theirs together are fewer than the compute
// units, each of which has room for seven.  (One counter alone is the limit at about
// 100 parts a us.)
//   4096 x 151936 bfloat16: 459 us, 5.4 TB/s; as two launches over the same parts 645.
__global__ __launch_bounds__(256) void k_unset(DistillArgs a, uint32_t parts) {
  const uint32_t i = blockIdx.x * 256 + threadIdx.x, row = i / parts;
  if (i < kQueues) *counter_of(a, i) = 0;
  if (row < a.rows) record_of(a, row).r[i - row * parts] = kUnset;
}
// A part of a row that is_far or of which sums have not come (bits of `missing`;
// `got`: part t's sum).  The part is read again, a vector at a time, in a function
// of its own: within the kernel this cost every block registers (4096 x 151936
// bfloat16: 515 us where 485).
template <int DT, int TDT>
__device__ __noinline__ void joined_seldom(DistillArgs a, uint32_t row, uint32_t part, uint32_t parts,
                                           unsigned long long got, unsigned long long missing) {
  __shared__ Shared sh;
  const float c = a.inv_tau * kLog2e;
  const char* x = logits_of<DT>(a, row);
  const bool last = part == parts - 1;
  Entry e = entry_of<DT, TDT>(a, row, part == 0 ? x : nullptr);
  const bool own = owns<DT>(a, e, part, parts);
  if (part != 0 && own) e.s = load1<DT>(x, (uint32_t)e.id);
  for (unsigned long long m = missing; m; m &= m - 1) {
    const uint32_t p = (uint32_t)__builtin_ctzll(m);
    const Running other = sum_of_part<DT>(a, x, p, p == parts - 1, c, sh);
    if (threadIdx.x == p) got = packed(other);
  }
  Running r = unpacked(got);
  const Teacher q = join_block(a, e, sh, &r, c);
  if (part == 0 && threadIdx.x == 0) write_loss(a, row, q, r);
  const float g = a.weight ? a.weight[row] : 1.f, lse = lse_of(a, r);
  const bool zero = !q.any || g == 0.f;
  char* out = grad_of<DT>(a, row);
  const uint32_t from = part * kPart;
  if (!zero && is_far(lse))
    grad_of_far<DT>(a, x, out, from, min(a.vocab / Elem<DT>::N, from + kPart), last, r, g * a.tau, e, own, sh);
  else
    grad_of_part<DT>(a, x, out, part, last, zero, lse, g * a.tau, e, own, sh);
}
// Seven blocks a compute unit: 4096 x 151936 bfloat16 477 us where six take 498 (float32
// the same either way).
template <int DT, int TDT, bool GRAD>
__global__ __launch_bounds__(kThreads, 7) void k_joined(DistillArgs a, uint32_t parts, uint32_t queues) {
  __shared__ Shared sh;
  const uint32_t t = threadIdx.x;
  const float c = a.inv_tau * kLog2e;
  uint32_t row = blockIdx.x, part = 0;
  if (parts > 1) {
    // Eight neighbouring blocks, on the eight XCDs, share a queue.
    const uint32_t queue = blockIdx.x / 8 % queues;
    if (t == 0)
      sh.ticket = __hip_atomic_fetch_add(counter_of(a, queue), 1u, __ATOMIC_RELAXED,
                                         __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    const uint32_t ticket = __builtin_amdgcn_readfirstlane(sh.ticket);
    row = ticket / parts;
    part = ticket - row * parts;
    row = row * queues + queue;
    if (row >= a.rows) return;
  }
  const char* x = logits_of<DT>(a, row);
  const bool last = part == parts - 1;
  Share<DT> v(a, part);
  v.load(x);
  Entry e = entry_of<DT, TDT>(a, row, part == 0 ? x : nullptr);
  const bool own = owns<DT>(a, e, part, parts);
  if (part != 0 && own) e.s = load1<DT>(x, (uint32_t)e.id);
  Running r = v.sum(a, x, last, c, sh);
  unsigned long long got = packed(t == part ? r : Running{-INFINITY, 0.f});  // of part t
  if (parts > 1) {
    unsigned long long* slot = record_of(a, row).r;
    if (t == 0) __hip_atomic_store(slot + part, packed(r), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (t < parts && t != part) {
      got = kUnset;
      for (uint32_t n = 0; n < a.wait_limit && got == kUnset; ++n) {
        got = __hip_atomic_load(slot + t, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (got == kUnset) __builtin_amdgcn_s_sleep(16);
      }
    }
    const unsigned long long missing = __builtin_amdgcn_ballot_w64(got == kUnset);
    if (t == 0) sh.missing = missing;
  }
  r = unpacked(got);
  const Teacher q = join_block(a, e, sh, &r, c);
  const unsigned long long missing = parts > 1 ? sh.missing : 0;
  const float lse = lse_of(a, r);
  if (GRAD && (missing || is_far(lse))) return joined_seldom<DT, TDT>(a, row, part, parts, got, missing);
  if (part == 0 && t == 0) write_loss(a, row, q, r);
  if (GRAD) {
    const float g = a.weight ? a.weight[row] : 1.f;
    v.grad(a, x, grad_of<DT>(a, row), last, !q.any || g == 0.f, lse, g * a.tau, e, own, sh);
  }
}

// ---- launches ------------------------------------------------------------------

uint32_t parts_of(int dtype, int32_t vocab) {
  const uint32_t nv = (uint32_t)vocab / (dtype == TFE_F32 ? 4 : 8);
  return std::max(1u, (nv + kPart - 1) / kPart);
}

// The call for n rows from r0 on.
DistillArgs rows_from(DistillArgs a, uint32_t r0, uint32_t n, int dtype, int tdtype) {
  const size_t es = dtype == TFE_F32 ? 4 : 2, ts = tdtype == TFE_F32 ? 4 : 2;
  a.logits = (const char*)a.logits + (size_t)r0 * a.ld * es;
  if (a.grad) a.grad = (char*)a.grad + (size_t)r0 * a.ldg * es;
  a.ids += (size_t)r0 * a.K;
  a.teacher = (const char*)a.teacher + (size_t)r0 * a.K * ts;
  if (a.weight) a.weight += r0;
  if (a.loss) a.loss += r0;
  a.lse += r0;
  a.rows = n;
  return a;
}

// Rows of a launch: the grid's second axis, and 2^20 parts.
uint32_t launch_rows(uint32_t parts) { return std::min(32768u, (1u << 20) / parts); }

// Queues of the joined parts: the blocks that can wait are fewer than the compute units.
uint32_t queues_of(uint32_t parts) {
  return std::max(1u, std::min(kQueues, (uint32_t)compute_units() / parts));
}

template <int DT, int TDT, bool LOSS, bool GRAD> hipError_t launch(const DistillArgs& a, hipStream_t s) {
  const uint32_t parts = parts_of(DT, (int32_t)a.vocab), most = launch_rows(parts);
  const dim3 block(kThreads);
  for (uint32_t r0 = 0; r0 < a.rows; r0 += most) {
    const uint32_t n = std::min(most, a.rows - r0);
    const DistillArgs b = rows_from(a, r0, n, DT, TDT);
    const bool twice = parts > 1 && a.grad == a.logits;  // the gradient takes the logits' place
    if (LOSS && (GRAD ? !twice : parts == 1)) {
      if (parts > 1) k_unset<<<dim3((n * parts + 255) / 256), dim3(256), 0, s>>>(b, parts);
      // As many blocks for each queue, and enough for the longest.
      const uint32_t queues = queues_of(parts);
      const uint32_t rounds = ((n + queues - 1) / queues * parts + 7) / 8;
      k_joined<DT, TDT, GRAD><<<dim3(parts > 1 ? rounds * 8 * queues : n), block, 0, s>>>(b, parts, queues);
      continue;
    }
    if (LOSS) {
      k_sum<DT, TDT><<<dim3(parts, n), block, 0, s>>>(b);
      k_loss<DT, TDT><<<dim3(n), block, 0, s>>>(b, parts);
    }
    if (GRAD) k_grad<DT, TDT><<<dim3(parts, n), block, 0, s>>>(b);
  }
  return hipGetLastError();
}
template <bool LOSS, bool GRAD>
hipError_t launch_types(const DistillArgs& a, int dtype, int tdtype, hipStream_t s) {
  if (dtype == TFE_F32)
    return tdtype == TFE_F32 ? launch<TFE_F32, TFE_F32, LOSS, GRAD>(a, s)
                             : launch<TFE_F32, TFE_BF16, LOSS, GRAD>(a, s);
  return tdtype == TFE_F32 ? launch<TFE_BF16, TFE_F32, LOSS, GRAD>(a, s)
                           : launch<TFE_BF16, TFE_BF16, LOSS, GRAD>(a, s);
}

}  // namespace

int64_t distill_space(int64_t rows, int32_t vocab) {
  const uint32_t parts = parts_of(TFE_F32, vocab);  // bfloat16 rows have fewer
  if (rows == 0 || parts == 1) return 0;
  return (int64_t)kRecords + std::min<int64_t>(rows, 32768) * (int64_t)sizeof(Record);
}
hipError_t launch_distill_loss(const DistillArgs& a, int dtype, int tdtype, hipStream_t s) {
  return launch_types<true, false>(a, dtype, tdtype, s);
}
hipError_t launch_distill_grad(const DistillArgs& a, int dtype, int tdtype, hipStream_t s) {
  return launch_types<false, true>(a, dtype, tdtype, s);
}
hipError_t launch_distill_loss_grad(const DistillArgs& a, int dtype, int tdtype, hipStream_t s) {
  return launch_types<true, true>(a, dtype, tdtype, s);
}

}  // namespace tfe
