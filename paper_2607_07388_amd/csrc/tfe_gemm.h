// Tile products on the matrix cores, for the calls that learn and serve the
// head: sums over k of P(p, k) Q(q, k), P and Q of bfloat16 or 8-bit integers.
// An operand lies in memory with k along its rows (row p holds P(p, .)) or across
// them (row k holds P(., k)).  Steps of 128 bytes of k go from memory straight into
// LDS, two stages of them; a compute unit has one block with 256 x 256 sums (64 KB a
// stage) or several with fewer.
// LDS gives 247 bytes a cycle here (226 by the transposing reads), so that the 192 KB that
// a step of a large tile reads take 40% of its 2048 cycles of matrix products.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace tfe {
namespace gemm {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

struct Bf16 {
  typedef f32x4 Acc;
  static constexpr int BYTES = 2;
};
struct Int8 {
  typedef i32x4 Acc;
  static constexpr int BYTES = 1;
};

// Bytes from a block of 2^log rows x 128 bytes to the next: a power of two apart, the
// blocks that are read at once would lie in the same channels of memory.
__host__ __device__ constexpr uint32_t block_bytes(uint32_t log) { return (128u << log) + 1024; }

// An operand of one tile.  Rows along k: `at` is its first row, `rows` the rows
// there are from it on and `cols` the length of k.  k across: `at` is the
// tile's first column of row k = 0, `rows` the length of k and `cols` the
// columns there are from the tile's first on.  16-byte aligned, `pitch` in bytes
// a multiple of 16, and cols * BYTES a multiple of 16: a 16-byte load is inside
// or outside as a whole.
// In blocks (a Side's BLOCKS): 2^log rows x 128 bytes as one piece of memory each (pitch
// 128), `blocks` of them beside each other: what a step reads lies together whichever
// way it runs.  rows and cols are whole blocks, and all of it is there.
struct Operand {
  const char* at;
  uint32_t pitch, rows, cols;
  uint32_t log, blocks;
};

constexpr int kStep = 128;  // bytes of k a step: 64 bfloat16 or 128 integers

// T rows (or columns) of an operand, kStep bytes of k deep, in LDS.
// Rows along k: 128 bytes each, its eight 16-byte pieces exchanged by the row's
// number mod 8.  k across (bfloat16): 64 rows of T numbers, in 32-byte pieces (the
// 16 columns that a transposing read takes from a row) exchanged by the row's
// number, so that the eight rows that are read at once (k to k + 3 and k + 8 to
// k + 11) lie on different banks.
// HALF: the T rows are 64 of each 128, from `shift` (0 or 64) on.
template <class E, int T, bool ACROSS, bool BLOCKS, int WAVES, bool HALF = false> struct Side {
  static constexpr int SIZE = T * kStep;
  static constexpr int LOADS = SIZE / 1024 / WAVES;
  static_assert(SIZE % (1024 * WAVES) == 0, "whole loads of every wave");
  static_assert(!ACROSS || E::BYTES == 2, "the transposing read is one of 16-bit numbers");
  static_assert(!ACROSS || !BLOCKS || T == 64, "across blocks, a load is of one block");
  static constexpr uint32_t ROW = ACROSS ? T * 2 : kStep;  // bytes of an LDS row
  static constexpr uint32_t PER = 1024 / ROW;              // rows of a load instruction

  __device__ static __forceinline__ uint32_t turned(uint32_t k) {
    return T >= 128 ? (k & 3) | (k >> 1 & 4) : (k >> 1 & 1) | (k >> 2 & 2);
  }

  uint32_t from;   // this lane's byte offset within the rows of its first load
  uint32_t piece;  // its 16-byte piece of a row (rows along k), or byte of a row

  __device__ __forceinline__ void init(uint32_t wave, uint32_t lane, const Operand& o) {
    const uint32_t r = lane / (ROW / 16), c = lane % (ROW / 16);
    const uint32_t row = wave * PER + r;
    if (ACROSS) {
      // Rows of a wave's loads are turned alike, or alternately.
      static_assert(!ACROSS || WAVES * PER % 16 == 0 || (WAVES * PER == 8 && T >= 128), "16 rows repeat");
      piece = (((c >> 1) ^ turned(row)) << 5) + ((c & 1) << 4);
      if (HALF) piece += piece & 128;
    } else {
      piece = (c ^ (row & 7)) << 4;
    }
    from = row * o.pitch + piece;
  }

  // Where a step's k begins, and what is left of it (rows, or bytes along the rows), in
  // scalar registers (a limit may be applied by a vector instruction, and a descriptor in
  // vector registers is loaded with in a loop: told to be the same in all lanes).  A turn's scalar instructions take time that its loads do not have:
  // the next step's place is added up, not worked out.
  struct Cursor {
    const char* at;
    int left;
    uint32_t fixed;  // bytes to the last row, or of the columns that there are
    uint32_t step, pitch;
    uint32_t phase, phases, jump;  // across blocks of more rows than a step
  };
  __device__ static __forceinline__ Cursor start(const Operand& o, uint32_t s) {
    Cursor c{};
    c.pitch = o.pitch;
    if (ACROSS) {
      const uint32_t k = s * (kStep / 2);
      c.left = max((int)(o.rows - k), 0);
      if (BLOCKS) {
        const uint32_t wide = o.blocks * block_bytes(o.log);
        c.phases = 1u << (o.log - 6);
        c.phase = s & (c.phases - 1);
        c.step = 64 * 128;
        c.jump = wide - (128u << o.log);
        c.at = o.at + (size_t)(k >> o.log) * wide + c.phase * c.step;
        c.fixed = 128;
      } else {
        c.step = 64 * o.pitch;
        c.at = o.at + (size_t)k * o.pitch;
        c.fixed = min(o.cols * 2, o.pitch);
      }
    } else {
      c.left = max((int)(o.cols * E::BYTES - s * kStep), 0);
      c.step = BLOCKS ? block_bytes(o.log) : kStep;
      c.at = o.at + (size_t)s * c.step;
      const uint32_t rows = min(o.rows, (uint32_t)(HALF ? 2 * T : T));
      c.fixed = rows ? (rows - 1) * o.pitch : 0u;
      if (!rows) c.left = 0;
    }
    return c;
  }
  __device__ static __forceinline__ void advance(Cursor* c) {
    c->at += c->step;
    c->left = max(c->left - (ACROSS ? kStep / 2 : kStep), 0);
    if (ACROSS && BLOCKS) {
      c->phase = c->phase + 1 == c->phases ? 0 : c->phase + 1;
      if (c->phase == 0) c->at += c->jump;
    }
  }
#if defined(__HIP_DEVICE_COMPILE__)
  // A step's loads into `to`; across blocks `shift` is in bytes.
  __device__ __forceinline__ void load(const Cursor& o, char* to, uint32_t wave, uint32_t shift = 0) const {
    typedef __attribute__((address_space(3))) void* Lds;
    // Rows between a wave's loads.
    constexpr uint32_t APART = HALF && !ACROSS ? 128 : WAVES * PER;
    static_assert(!HALF || ACROSS || WAVES * PER == 64, "a load of every wave is 64 rows");
    if (ACROSS) {
      const int rows = min(o.left, 64);
      // (rows - 1) * pitch + fixed, of no rows 0.  All of the blocks is there.
      const int bytes = __builtin_amdgcn_readfirstlane(
          BLOCKS ? (rows ? 0x7FFFFFF0 : 0) : max((int)(rows * o.pitch - (o.pitch - o.fixed)), 0));
      const auto d = __builtin_amdgcn_make_buffer_rsrc((void*)o.at, 0, bytes, 0x00020000);
      const uint32_t start = from + (BLOCKS ? shift : shift * 2);
      const uint32_t other = WAVES * PER == 8 ? start - piece + (piece ^ 128) : start;
#pragma unroll
      for (int c = 0; c < LOADS; ++c)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(d, (Lds)(to + (c * WAVES + wave) * 1024), 16,
                                                 (int)((c & 1 ? other : start) + c * APART * o.pitch), 0, 0, 0);
    } else {
      const int bytes = __builtin_amdgcn_readfirstlane((int)o.fixed + min(o.left, kStep));
      const auto d = __builtin_amdgcn_make_buffer_rsrc((void*)o.at, 0, bytes, 0x00020000);
      // Past the row's end: an offset beyond every descriptor's range.
      const uint32_t start = (int)piece < o.left ? from + shift * o.pitch : 0x70000000u;
#pragma unroll
      for (int c = 0; c < LOADS; ++c)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(d, (Lds)(to + (c * WAVES + wave) * 1024), 16,
                                                 (int)(start + c * APART * o.pitch), 0, 0, 0);
    }
  }
  // The 16 rows (columns) from 16 t + `first` on, `first` a multiple of the
  // wave's part: lane (g, i) gets row i's 16 bytes of k at 64 h + 16 g.
  __device__ static __forceinline__ u32x4 operand(const char* lds, uint32_t first, int t, int h,
                                                  uint32_t i, uint32_t g) {
    if (ACROSS) {
      typedef __attribute__((address_space(3))) s16x4* Lds;
      const uint32_t k = g * 8 + (i >> 2);
      u32x4 r;
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const char* p = lds + (k + h * 32 + q * 4) * ROW + (((first / 16 + t) ^ turned(k)) << 5) + (i & 3) * 8;
        const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)p);
        const u32x2 w = __builtin_bit_cast(u32x2, v);
        r[2 * q] = w[0];
        r[2 * q + 1] = w[1];
      }
      return r;
    }
    return *(const u32x4*)(lds + (first + t * 16 + i) * kStep + (((h * 4 + g) ^ (i & 7)) << 4));
  }
#endif
};

template <class E>
__device__ __forceinline__ typename E::Acc multiply(u32x4 p, u32x4 q, typename E::Acc c) {
#if defined(__HIP_DEVICE_COMPILE__)
  if constexpr (E::BYTES == 2)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, p),
                                                   __builtin_bit_cast(bf16x8, q), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, p),
                                                 __builtin_bit_cast(i32x4, q), c, 0, 0, 0);
#else
  return c;
#endif
}

// Numbers of four bytes from `first` on (those that there are, and zeros) into LDS:
// 64 of each wave that takes part, 64 `part` behind the first.
__device__ __forceinline__ void load_numbers(const void* array, uint32_t first, uint32_t count, uint32_t part,
                                             char* to) {
#if defined(__HIP_DEVICE_COMPILE__)
  typedef __attribute__((address_space(3))) void* Lds;
  const uint32_t left = count > first ? min(count - first, 1u << 20) : 0u;
  const auto d = __builtin_amdgcn_make_buffer_rsrc((void*)((const char*)array + (size_t)first * 4), 0,
                                                   (int)(left * 4), 0x00020000);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(d, (Lds)(to + part * 256), 4,
                                           (int)(part * 256 + (threadIdx.x & 63) * 4), 0, 0, 0);
#endif
}

// Asks for a share of `rows` rows of `len` bytes that blocks of this XCD read soon, so that
// they are in its L2 by then: a number of each 128 bytes, into 256 bytes of LDS that nobody
// reads.  Thread t of THREADS of share `part` of `parts`; more than a number a thread: none.
template <int THREADS>
__device__ __forceinline__ void warm(const Operand& o, uint32_t most, uint32_t len, uint32_t part, uint32_t parts,
                                     char* to) {
#if defined(__HIP_DEVICE_COMPILE__)
  typedef __attribute__((address_space(3))) void* Lds;
  const uint32_t lines = (len + 127) / 128, rows = min(o.rows, most), all = rows * lines;
  if (all > parts * THREADS) return;
  const uint32_t line = part * THREADS + threadIdx.x, row = line / lines;
  const int bytes = __builtin_amdgcn_readfirstlane(rows ? (int)((rows - 1) * o.pitch + len) : 0);
  const auto d = __builtin_amdgcn_make_buffer_rsrc((void*)o.at, 0, bytes, 0x00020000);
  const uint32_t at = line < all ? row * o.pitch + (line - row * lines) * 128 : 0x70000000u;
  __builtin_amdgcn_raw_ptr_buffer_load_lds(d, (Lds)to, 4, (int)at, 0, 0, 0);
#endif
}

// Steps [s0, s1) of a tile's operands.
struct Segment {
  Operand p, q;
  uint32_t s0, s1;
};
__device__ __forceinline__ Segment no_segment(const Segment& like) {
  Segment r = like;  // reads as zeros
  r.p.rows = r.p.cols = r.q.rows = r.q.cols = 0;
  return r;
}

// A block of WP x WQ waves and its tile of TP x TQ sums.  Lane (g, i) of a wave
// holds in acc[n][m][j] the sum at p = wp + 16 n + 4 g + j, q = wq + 16 m + i.
// PA, QA: k runs across P, Q; QB: Q lies in blocks.
template <class E, int TP, int TQ, int WP, int WQ, bool PA, bool QA, bool QB> struct Tile {
  static constexpr int WAVES = WP * WQ, NT = TP / WP / 16, MT = TQ / WQ / 16;
  static constexpr int THREADS = WAVES * 64;
  typedef Side<E, TP, PA, false, WAVES> P;
  typedef Side<E, QA && QB ? 64 : TQ, QA, QB, WAVES> Q;
  static constexpr bool LARGE = TP == 256 && TQ == 256 && WP == 2 && WQ == 4;
  static constexpr int PARTS = QA && QB ? TQ / 64 : 1;  // blocks of a step across them
  static_assert(PARTS == 1 || TQ / WQ == 64, "a wave's columns are a block's");
  static constexpr int STAGE = P::SIZE + Q::SIZE * PARTS;
  // Behind the stages: two tiles' numbers of their rows and columns, INFO bytes each.
  static constexpr int LDS = 2 * STAGE;
  // Steps of a segment: fewer are followed by zeros.
  static constexpr uint32_t LEAST = 4;
  typename E::Acc acc[NT][MT];
  uint32_t wave, lane, i, g, wp, wq;

  __device__ __forceinline__ Tile() {
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    lane = threadIdx.x & 63;
    i = lane & 15;
    g = lane >> 4;
    wp = (wave % WP) * (TP / WP);
    wq = (wave / WP) * (TQ / WQ);
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int m = 0; m < MT; ++m) acc[n][m] = typename E::Acc{0, 0, 0, 0};
  }
  // Adds one segment after another: `next` gives the one behind (false: none), `begin`
  // is called when a segment's first step is about to be read, and may ask for loads into
  // the LDS behind the stages, of a place for odd and one for even segments; `done` when a
  // segment's sums are in acc, where those loads have come.  Neither may wait for other
  // waves.  `done` returns whether it has stored at least STORES times (memory operations
  // of each wave), which then need not have landed when the next segment's first step is.
  // A segment of fewer than LEAST steps ends where its operands end.
  template <int STORES, class Next, class Begin, class Done>
  __device__ __forceinline__ void run(Segment cur, Next next, Begin begin, Done done, char* lds) {
    if constexpr (LARGE) {
      in_turns<STORES>(cur, next, begin, done, lds);
    } else {
      uint32_t odd = 0;
      for (bool more = true; more; odd ^= 1) {
        Segment nxt = cur;
        more = next(&nxt);
        begin(odd);
        together(cur.p, cur.q, cur.s0, cur.s1, lds);
        done(odd);
        cur = nxt;
      }
    }
  }

 private:
  // Large tiles: the waves take turns.  While the four of one group (one on each
  // SIMD) multiply, the other four read LDS and ask for loads; a barrier ends each
  // turn.  A wave's step is two such pairs of turns: its rows of P's first half with
  // all of Q, then P's second half.  A place in LDS is loaded again, for the step
  // after next, in the turn after every wave has read it, so a load is a whole step
  // under way.  Loads run on over the segments: a tile's first ones are under way
  // while the last one's results are written.
  template <int STORES, class Next, class Begin, class Done>
  __device__ __forceinline__ void in_turns(Segment cur, Next next, Begin begin, Done done, char* lds) {
#if defined(__HIP_DEVICE_COMPILE__)
    typedef Side<E, 128, PA, false, WAVES, true> Half;
    constexpr int HALF = Half::SIZE;
    static_assert(NT == 8 && MT == 4 && Half::LOADS == 2 && Q::LOADS * PARTS == 4, "what the waits count");
    Half sp;
    Q sq;
    sp.init(wave, lane, cur.p);
    sq.init(wave, lane, cur.q);
    const uint32_t block = block_bytes(cur.q.log);
    u32x4 pv[2][4], qv[2][4];
    // A stage: P's halves, then Q.
    auto read_p = [&](const char* from) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int n = 0; n < 4; ++n) pv[h][n] = Half::operand(from, wp / 2, n, h, i, g);
    };
    auto read_q = [&](const char* from) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int m = 0; m < 4; ++m)
          qv[h][m] = q_operand(from + 2 * HALF, m, h);
    };
    auto load_q = [&](const typename Q::Cursor& c, char* to) {
#pragma unroll
      for (int k = 0; k < PARTS; ++k) sq.load(c, to + k * Q::SIZE, wave, k * block);
    };
    auto products = [&](int half) {
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
          for (int m = 0; m < 4; ++m) {
            typename E::Acc& c = acc[half * 4 + n][m];
            c = multiply<E>(pv[h][n], qv[h][m], c);
          }
      __builtin_amdgcn_s_setprio(0);
    };
    auto turn = [] {
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_sched_barrier(0);
    };
    // The next loads' places: P's first half and Q two steps on, P's second half one.
    auto first = Half::start(cur.p, cur.s0), other = first;
    auto cq = Q::start(cur.q, cur.s0);
    sp.load(first, lds, wave, 0);
    load_q(cq, lds + 2 * HALF);
    sp.load(other, lds + HALF, wave, 64);
    Half::advance(&first);
    Half::advance(&other);
    Q::advance(&cq);
    sp.load(first, lds + STAGE, wave, 0);
    load_q(cq, lds + STAGE + 2 * HALF);
    Half::advance(&first);
    Q::advance(&cq);
    wait_loads<6>();  // the first step is there
    __builtin_amdgcn_s_barrier();
    const bool second = wave >= 4;
    if (second) turn();
    uint32_t at = 0, odd = 0;
    bool stored = false, ahead = false;
    for (bool more = true; more; odd ^= 1) {
      Segment nxt = cur;
      more = next(&nxt);
      if (!more) nxt = no_segment(cur);
      begin(odd);
      const uint32_t steps = max(cur.s1 - cur.s0, LEAST);
      for (uint32_t j = 0; j < steps; ++j) {
        char* const from = lds + at;
        read_p(from);
        read_q(from);
        if (j + 1 == steps) other = Half::start(nxt.p, nxt.s0);
        if (!ahead) {
          sp.load(other, lds + (STAGE - at) + HALF, wave, 64);
          Half::advance(&other);
        }
        ahead = false;
        // This step's second half of P is there: behind it were asked for the next step's
        // first half and Q (6), and its second half (2).
        if (STORES && stored && j < 2)
          wait_loads<(8 + STORES < 63 ? 8 + STORES : 63)>();
        else
          wait_loads<8>();
        turn();
        products(0);
        turn();
        read_p(from + HALF);
        if (j + 2 == steps) {
          first = Half::start(nxt.p, nxt.s0);
          cq = Q::start(nxt.q, nxt.s0);
        }
        sp.load(first, from, wave, 0);
        load_q(cq, from + 2 * HALF);
        Half::advance(&first);
        Q::advance(&cq);
        // The next step's first half and Q are there: behind them were asked for its second
        // half (2) and what this turn asked for (6).
        if (STORES && stored && j == 0)
          wait_loads<(8 + STORES < 63 ? 8 + STORES : 63)>();
        else
          wait_loads<8>();
        turn();
        products(1);
        turn();
        at = STAGE - at;
      }
      // The next segment's second step: every wave has read what lies in its place, and
      // asked for now it does not wait for the results' stores.
      if (STORES) {
        sp.load(other, lds + (STAGE - at) + HALF, wave, 64);
        Half::advance(&other);
        ahead = true;
      }
      __builtin_amdgcn_sched_barrier(0);
      stored = done(odd);
      __builtin_amdgcn_sched_barrier(0);
      cur = nxt;
    }
    if (!second) turn();
    // Loads of zeros may still be under way.
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#endif
  }
#if defined(__HIP_DEVICE_COMPILE__)
  __device__ __forceinline__ u32x4 q_operand(const char* from, int m, int h) const {
    if (PARTS > 1) return Q::operand(from + wq / 64 * Q::SIZE, 0, m, h, i, g);
    return Q::operand(from, wq, m, h, i, g);
  }
#endif
  // This wave's LDS reads have returned, and all but its last N memory operations.
  template <int N> __device__ static __forceinline__ void wait_loads() {
    static_assert(N < 64, "the counter's range");
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
    __builtin_amdgcn_sched_barrier(0);
  }

  // Smaller tiles: one step's loads are under way while the one before is
  // multiplied.
  __device__ __forceinline__ void together(const Operand& p, const Operand& q, uint32_t s0, uint32_t s1,
                                           char* lds) {
#if defined(__HIP_DEVICE_COMPILE__)
    if (s0 >= s1) return;
    P sp;
    Q sq;
    sp.init(wave, lane, p);
    sq.init(wave, lane, q);
    auto cp = P::start(p, s0);
    auto cq = Q::start(q, s0);
    const uint32_t block = block_bytes(q.log);
    auto load = [&](char* to) {
      sp.load(cp, to, wave);
#pragma unroll
      for (int k = 0; k < PARTS; ++k) sq.load(cq, to + P::SIZE + k * Q::SIZE, wave, k * block);
      P::advance(&cp);
      Q::advance(&cq);
    };
    load(lds);
    uint32_t at = 0;
    for (uint32_t s = s0; s < s1; ++s) {
      // The stage has arrived, and every wave's reads of the other one have returned.
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_sched_barrier(0);
      const char* from = lds + at;
      at = STAGE - at;
      if (s + 1 < s1) load(lds + at);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        u32x4 qv[MT];
#pragma unroll
        for (int m = 0; m < MT; ++m) qv[m] = q_operand(from + P::SIZE, m, h);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const u32x4 pv = P::operand(from, wp, n, h, i, g);
#pragma unroll
          for (int m = 0; m < MT; ++m) acc[n][m] = multiply<E>(pv, qv[m], acc[n][m]);
        }
      }
    }
    // The LDS may be written again, by loads or by the caller.
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
#endif
  }
};

}  // namespace gemm
}  // namespace tfe
