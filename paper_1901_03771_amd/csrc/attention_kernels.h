// Device parts that the attention kernels share: products of 32 x 32 blocks on the matrix cores, tiles in LDS, scores.
//
// One layout carries all of them.  v_mfma_f32_32x32x16_bf16 leaves its result with a column per lane (lane & 31) and, in
// register r of the lane's half hi = lane >> 5, row (r & 3) + 8 (r >> 2) + 4 hi; its operands hold row (or column) lane & 31
// and the eight places 8 hi .. 8 hi + 7 of the summed dimension.  A sum may run in any order, so registers 8 t .. 8 t + 7 of a
// result ARE the operand of the next product over its rows, if the other operand takes the rows of step t in the order
//   place j of half hi  =  row 16 t + (j & 3) + 8 (j >> 2) + 4 hi,
// which is two groups of four neighbouring rows: what ds_read_b64_tr_b16 returns from a row-major tile.  So scores are formed with
// the side that is normalised along the lanes (queries for the output and dq, keys for dk and dv), the softmax needs one
// exchange between the two halves of a wave, and neither scores nor probabilities ever pass through LDS.
// float32 uses the same layout, as three bfloat16 pieces.
#pragma once

#include <hip/hip_runtime.h>

#include "attention.h"

#define GR_DEVICE_MATH_SOURCE(...) __VA_ARGS__
#include "device_tanh.h"
#undef GR_DEVICE_MATH_SOURCE

namespace gr {
namespace attn {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 b16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 b16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 b16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

#define GR_LDS __attribute__((address_space(3)))

constexpr float LIFT = 32.0f, UNLIFT = 0x1p-32f;   // see attention_backward.h
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

template <class T> struct Frag;
template <> struct Frag<__bf16> { typedef b16x8 type; };
template <> struct Frag<float> { typedef f32x8 type; };

static __device__ __forceinline__ f32x16 mma(b16x8 a, b16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
// float32 as bfloat16 pieces: x = h + m + l to 2^-26 of x, each piece the rounding of what the ones before it leave, and x y = the six products
// of pieces that count (m l, l m and l l are below 2^-25 of it).  Six products of bfloat16 take 192 cycles of a SIMD's matrix core, eight steps of
// v_mfma_f32_32x32x2_f32 512; the pieces cost 44 vector instructions for an operand of eight values, beside them (8 heads of 4096 rows twice, 64 values: 564 us
// on the float32 products, 365 so; the results are no further from binary64).  An infinity has no pieces: it gives NaN, and so does what rounds to one, from
// 2^128 - 2^119 on (holding h below it, an instruction more per value, cost float32 calls 4 to 7 %).
struct Pieces { b16x8 h, m, l; };
static __device__ __forceinline__ Pieces pieces(f32x8 x) {
  Pieces p;
#pragma unroll
  for (int j = 0; j < 8; j += 2) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    f32x2 v = {x[j], x[j + 1]};
    const b16x2 h = __builtin_convertvector(v, b16x2);
    v[0] -= (float)h[0]; v[1] -= (float)h[1];
    const b16x2 m = __builtin_convertvector(v, b16x2);
    v[0] -= (float)m[0]; v[1] -= (float)m[1];
    const b16x2 l = __builtin_convertvector(v, b16x2);
    p.h[j] = h[0]; p.h[j + 1] = h[1]; p.m[j] = m[0]; p.m[j + 1] = m[1]; p.l[j] = l[0]; p.l[j + 1] = l[1];
  }
  return p;
}
static __device__ __forceinline__ f32x16 mma(f32x8 a, f32x8 b, f32x16 c) {
  const Pieces x = pieces(a), y = pieces(b);
  c = mma(x.l, y.h, c);
  c = mma(x.h, y.l, c);
  c = mma(x.m, y.m, c);
  c = mma(x.m, y.h, c);
  c = mma(x.h, y.m, c);
  return mma(x.h, y.h, c);
}
// Keeps the pieces of an operand from being formed ahead of a loop, for lack of registers to hold them.
static __device__ __forceinline__ void anew(f32x8& f) { asm volatile("" : "+v"(f)); }
static __device__ __forceinline__ void anew(b16x8&) {}

// Results of the matrix cores that branches may stand before the use of: a vector instruction reads such a register 19 issue slots after
// its product at the earliest, and the compiler, which counts them, has been seen to count along one of several paths that meet
// (float32, 64 values a head: the last of 64 products was missing from a score).  Here the slots are spent.
static __device__ __forceinline__ void finished(f32x16& x) { asm volatile("s_nop 7\n\ts_nop 7\n\ts_nop 2" : "+v"(x)); }
static __device__ __forceinline__ void finished(f32x16& x, f32x16& y) { asm volatile("s_nop 7\n\ts_nop 7\n\ts_nop 2" : "+v"(x), "+v"(y)); }
template <int N>
static __device__ __forceinline__ void finished(f32x16 (&x)[N]) {
#pragma unroll
  for (int i = 1; i < N; ++i) asm volatile("" : "+v"(x[i]));   // (their products come before the wait ..)
  finished(x[0]);
#pragma unroll
  for (int i = 1; i < N; ++i) asm volatile("" : "+v"(x[i]));   // (.. and their uses after it)
}

static __device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
static __device__ __forceinline__ float log2_(float x) { return __builtin_amdgcn_logf(x); }
// A value that the compiler takes to be new wherever this stands: what is computed from it is computed there, instead of once before the
// loop at the price of registers that are full.
static __device__ __forceinline__ int fresh(int x) { asm volatile("" : "+v"(x)); return x; }

// Makes the compiler wait here for values that it has loaded, before a loop: it knows nothing of the loads into LDS of the statements below, and a wait of its own
// within the loop, for what was loaded before it, would be for all of those too.
static __device__ __forceinline__ void loaded(float& x) { asm volatile("" : "+v"(x)); }
template <class F, int N>
static __device__ __forceinline__ void loaded(F (&f)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+v"(f[i]));
}

constexpr float INF = __builtin_inff();

// The value of the lane's partner in the other half of the wave.
static __device__ __forceinline__ float max_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __builtin_fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
static __device__ __forceinline__ float sum_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// ---- tiles in LDS -------------------------------------------------------------------------------------------------------
// Rows of row_values(DP) values without padding, in chunks of 16 bytes; chunk c of row r lies in place c ^ twist(r), chosen so that
// both kinds of reads spread over all 64 banks: the same chunk of 16 neighbouring rows (rows as operands: 16 different places), and 64
// bytes each of four neighbouring rows (transposed reads: four different groups of four places).
template <class T, int DP>
struct Tile {
  static constexpr int VALUES = row_values(DP), ROW = VALUES * (int)sizeof(T), CHUNKS = ROW / 16, EACH = 16 / (int)sizeof(T);
  static constexpr int STEPS = DP / 16, BLOCKS = DP / 32;

  static __device__ __forceinline__ int twist(int r) {
    return CHUNKS == 8 ? ((r >> 1) & 1) << 2 | ((r >> 2) & 3) : (r & 3) << 2 | ((r >> 2) & 3);
  }

  // Row `r` as an operand: the values 16 s + 8 hi .. + 7.
  static __device__ __forceinline__ typename Frag<T>::type row(const GR_LDS char* tile, int r, int s, int hi) {
    const GR_LDS char* at = tile + r * ROW;
    if constexpr (sizeof(T) == 2) {
      return *(const GR_LDS b16x8*)(at + (((2 * s + hi) ^ twist(r)) << 4));
    } else {
      const f32x4 x = *(const GR_LDS f32x4*)(at + (((4 * s + 2 * hi) ^ twist(r)) << 4));
      const f32x4 y = *(const GR_LDS f32x4*)(at + (((4 * s + 2 * hi + 1) ^ twist(r)) << 4));
      return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
    }
  }

  // Column 32 block + (lane & 31) as an operand: rows r0 + (j & 3) + 8 (j >> 2) + 4 hi, r0 a multiple of 16.
  static __device__ __forceinline__ typename Frag<T>::type column(const GR_LDS char* tile, int r0, int block, int lane) {
    const int hi = lane >> 5;
    if constexpr (sizeof(T) == 2) {
      const int r = r0 + 4 * hi + ((lane & 15) >> 2), c = 4 * block + ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
      const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((GR_LDS s16x4*)(tile + r * ROW + ((c ^ twist(r)) << 4) + (lane & 1) * 8));
      const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((GR_LDS s16x4*)(tile + (r + 8) * ROW + ((c ^ twist(r + 8)) << 4) + (lane & 1) * 8));
      return __builtin_bit_cast(b16x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      const int col = 32 * block + (lane & 31);
      f32x8 f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int r = r0 + (j & 3) + 8 * (j >> 2) + 4 * hi;
        f[j] = *(const GR_LDS float*)(tile + r * ROW + (((col >> 2) ^ twist(r)) << 4) + (col & 3) * 4);
      }
      return f;
    }
  }

  // Rows [0, valid) of the tensor at `base` (uniform) into a tile of ROWS rows; the rest of the tile, and what lies behind D in a
  // row, become zeros.  Where the tensor allows it the loads go straight into LDS (buffer_load_dwordx4 .. lds: lane L of a wave
  // fills the 16 bytes at L of its kilobyte, so the twist is in the lane's address; a place without a value reads behind the
  // buffer's end, which gives zeros) and the caller waits for them; else every value is fetched by itself.
  // The caller has no more than one such tile of each kind under way, and a barrier on either side.
  template <int ROWS, int THREADS>
  static __device__ __forceinline__ void load(GR_LDS char* tile, const T* base, int64_t stride, int valid, int D, int tid, int direct) {
    constexpr int N = ROWS * CHUNKS / THREADS;
    static_assert(N * THREADS == ROWS * CHUNKS, "whole chunks for every thread");
    if (direct) {
      // (the buffer ends with its last valid row: rows do not overlap, see Tensor::direct)
      const uint64_t b = (uint64_t)base;
      const int sbytes = (int)stride * (int)sizeof(T);
      const int bytes = valid > 0 ? (valid - 1) * sbytes + D * (int)sizeof(T) : 0;
      i32x4 rsrc = {__builtin_amdgcn_readfirstlane((int)b), __builtin_amdgcn_readfirstlane((int)(b >> 32) & 0xffff), __builtin_amdgcn_readfirstlane(bytes), 0x00027000};
      const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)tile + (tid & ~63) * 16);
      // a thread's chunks are STEP rows apart; the twist comes back after 16 rows
      constexpr int STEP = THREADS / CHUNKS, PERIOD = STEP >= 16 ? 1 : 16 / STEP;
      uint32_t first[PERIOD];
#pragma unroll
      for (int n = 0; n < PERIOD && n < N; ++n) {
        const int r = n * STEP + tid / CHUNKS, c = (tid % CHUNKS) ^ twist(r);
        first[n] = c * EACH < D ? (uint32_t)(r * sbytes + c * 16) : 0x80000000u;
      }
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const uint32_t off = first[n % PERIOD] + (uint32_t)(n / PERIOD * PERIOD * STEP * sbytes);
        // (the statement leaves the scalar condition code alone; wait states: M0, and a base that a vector instruction wrote)
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" : : "v"(off), "s"(rsrc), "s"(lds0 + n * THREADS * 16) : "memory", "m0");
      }
    } else {
#pragma unroll 1
      for (int n = 0; n < N; ++n) {
        const int i = n * THREADS + tid, r = i / CHUNKS, c = (i % CHUNKS) ^ twist(r);
        T x[EACH];
#pragma unroll
        for (int e = 0; e < EACH; ++e) x[e] = r < valid && c * EACH + e < D ? base[r * stride + c * EACH + e] : (T)0.0f;
        GR_LDS T* to = (GR_LDS T*)(tile + i * 16);
#pragma unroll
        for (int e = 0; e < EACH; ++e) to[e] = x[e];
      }
    }
  }

  // Values 16 s + 8 hi .. + 7 of a row in memory.
  static __device__ __forceinline__ typename Frag<T>::type fetch(const T* p, int s, int hi, int D, bool valid, int aligned) {
    typename Frag<T>::type f;
    const int d = 16 * s + 8 * hi;
    if (aligned) {
      // (d is a multiple of 8 and D one of a vector: a float32 row may end within the eight)
      if constexpr (sizeof(T) == 2) {
        f = valid && d < D ? *(const b16x8*)(p + d) : (b16x8)(__bf16)0.0f;
      } else {
        const f32x4 z = {0.f, 0.f, 0.f, 0.f};
        const f32x4 x = valid && d < D ? *(const f32x4*)(p + d) : z, y = valid && d + 4 < D ? *(const f32x4*)(p + d + 4) : z;
        f = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = valid && d + e < D ? p[d + e] : (T)0.0f;
    }
    return f;
  }
};

// A whole number at an address that is the same for the wave, written before this kernel began: a scalar load.  (A vector load would have to be
// waited for behind all the tile's loads under way.)
static __device__ __forceinline__ int scalar(const int* p, int64_t i) { return ((const __attribute__((address_space(4))) int*)p)[i]; }

static __device__ __forceinline__ float scalar_float(const float* p, int64_t i) { return ((const __attribute__((address_space(4))) float*)p)[i]; }

// One wave loads up to 64 neighbouring 4-byte values straight into LDS.
static __device__ __forceinline__ void load_words(GR_LDS float* to, const void* from, int lane, int count) {
  const uint64_t b = (uint64_t)from;
  i32x4 rsrc = {__builtin_amdgcn_readfirstlane((int)b), __builtin_amdgcn_readfirstlane((int)(b >> 32) & 0xffff), 0x7fffffff, 0x00027000};
  const uint32_t lds = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)to);
  if (lane < count) asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tbuffer_load_dword %0, %1, 0 offen lds" : : "v"(lane * 4), "s"(rsrc), "s"(lds) : "memory", "m0");
}

// Waits for this wave's loads into LDS, then for everybody's.
static __device__ __forceinline__ void arrive() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// ---- operands from results ----------------------------------------------------------------------------------------------
// Registers 8 t .. 8 t + 7 of a result as an operand.  To bfloat16 by round to nearest even: a probability or a score's gradient
// loses at most 2^-8 of itself (half a step of 8 bits), as the result does when it is stored; sums and statistics are taken before this rounding.  Taken as two
// such numbers, as the forward kernel does where `rest` is wanted, they cost its second product twice (16 heads of 8192 causal rows of 128 values 0.30 -> 0.40 ms): so out
// is up to 1.4 times as far from binary64 as with probabilities of 32 bits, and no further than a rounding of the result or two.
static __device__ __forceinline__ void operand(const f32x16& x, int t, b16x8& f) {
#pragma unroll
  for (int j = 0; j < 8; j += 2) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const f32x2 p = {x[8 * t + j], x[8 * t + j + 1]};
    const b16x2 b = __builtin_convertvector(p, b16x2);
    f[j] = b[0];
    f[j + 1] = b[1];
  }
}
static __device__ __forceinline__ void operand(const f32x16& x, int t, f32x8& f) {
#pragma unroll
  for (int j = 0; j < 8; ++j) f[j] = x[8 * t + j];
}

// ---- scores -------------------------------------------------------------------------------------------------------------
// A product q.k becomes y, the score in units in which c y is its binary logarithm: q.k itself; its tanh where scores are capped; the
// whole exponent (c = 1) where a bias is added.  tanh(a) = 1 - 2 / (1 + e^2a) by the hardware's power of two and reciprocal takes 11 units of
// issue against about 25, but its error, 2^-22 at most, is one of 1 also where the tanh is small, and the score is off by cap times as much.  Up to
// SHORT_CAP that is 2^-12, a sixteenth of what rounding a probability to bfloat16 may do to it; larger caps (MODE_WIDE) and float32 take the library's own
// tanh, right to the last place for small scores too (a prompt of 8192 rows, 16 heads of 256 values on 8: 0.69 ms with the short form, 1.02 with this one).
template <class T, int MODE>
static __device__ __forceinline__ float capped(float s, float cin) {
  if constexpr (sizeof(T) == 2 && !(MODE & MODE_WIDE)) return __builtin_fmaf(-2.0f, __builtin_amdgcn_rcpf(1.0f + exp2_(s * cin)), 1.0f);
  else return gr_tanhf(s * cin);
}

// How many keys a query sees at most: its causal part, the prefix and the length are beginnings of the row of keys.
static __device__ __forceinline__ int keys_seen(const Args& a, int i, int len, int pre) {
  if (!a.causal) return len;
  return min(max(max(a.place + i + 1, pre), 0), len);
}

// The first query whose causal part holds `key`; 2^31 - 1 if none does.
static __device__ __forceinline__ int first_seeing(const Args& a, int key) {
  const int f = max(key - a.place, 0);
  return f < a.N ? f : 0x7fffffff;
}

static __device__ __forceinline__ int length_of(const Args& a, int b) {
  const int n = a.lengths ? scalar(a.lengths, b * a.lengths_s) : a.M;
  return n < 0 ? 0 : n < a.M ? n : a.M;
}

// A row of the queries of one head of k: query and head of q (a row behind the last stands for the last).
struct Row { int i, h; bool valid; };
static __device__ __forceinline__ Row row_of(const Args& a, int hk, int row) {
  const int R = a.N * a.G;
  Row r;
  r.valid = row < R;
  const int n = r.valid ? row : R - 1;
  r.i = n / a.G;
  r.h = hk * a.G + (n - r.i * a.G);
  return r;
}

// Which (batch, head of k) and which block of it a workgroup takes.  Workgroups go round the eight XCDs in turn, each with an L2 of its
// own: those of one head stay on one XCD (or on 8 / pairs of them) where the number of heads allows it.
struct Place { int pair, block; };
static __device__ __forceinline__ Place place_of(unsigned id, int pairs, int blocks) {
  if (pairs % 8 == 0) { const int x = id & 7, r = id >> 3; return {x + 8 * (r / blocks), r % blocks}; }
  if (8 % pairs == 0) { const int x = id & 7, per = 8 / pairs; return {x / per, (int)(id >> 3) * per + x % per}; }
  return {(int)(id / (unsigned)blocks), (int)(id % (unsigned)blocks)};
}

// Tiles of 32 * UNIT entries of a row of document numbers that hold a number between lo and hi, found 256 at a time.
template <int UNIT>
struct Finder {
  const int* ranges;   // nullptr: every tile
  int count;           // 32-entry pieces
  int lo, hi;          // lo > hi: none
  int base = -1;
  uint64_t mask[4] = {0, 0, 0, 0};
  __device__ __forceinline__ void look(int t, int end, int lane) {
    base = t;
    int l[4][UNIT], u[4][UNIT];
#pragma unroll
    for (int w = 0; w < 4; ++w)
#pragma unroll
      for (int x = 0; x < UNIT; ++x) {
        const int i = min((t + 64 * w + lane) * UNIT + x, count - 1);
        l[w][x] = ranges[2 * i];
        u[w][x] = ranges[2 * i + 1];
      }
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      bool some = false;
#pragma unroll
      for (int x = 0; x < UNIT; ++x) some |= (l[w][x] <= hi) & (u[w][x] >= lo);
      mask[w] = __ballot(some & (t + 64 * w + lane < end) & (lo <= hi));
    }
  }
  __device__ __forceinline__ int next(int t, int end, int lane) {
    if (!ranges) return t < end ? t : end;
    while (t < end) {
      if (base < 0 || t < base || t >= base + 256) look(t, end, lane);
      const int w = (t - base) >> 6;
      const uint64_t m = (w == 0 ? mask[0] : w == 1 ? mask[1] : w == 2 ? mask[2] : mask[3]) >> ((t - base) & 63);
      if (m) { const int f = t + __builtin_ctzll(m); return f < end ? f : end; }
      t = base + (w + 1) * 64;
    }
    return end;
  }
};

// Smallest (below zero counts as none: 0) and largest document of the 32-entry pieces that entries first .. last lie in, and whether all of
// them are one document's.
struct Span { int lo, hi; bool one; };
static __device__ __forceinline__ Span span_of(const int* ranges, int first, int last) {
  Span s = {0x7fffffff, -1, true};
  int all = 0x7fffffff;
  for (int e = first / 32; e <= last / 32; ++e) {
    const int l = scalar(ranges, 2 * e), u = scalar(ranges, 2 * e + 1);
    all = min(all, l);
    if (u >= 0) { s.lo = min(s.lo, max(l, 0)); s.hi = max(s.hi, u); }
  }
  s.one = all == s.hi && s.hi >= 0;
  return s;
}

// Four neighbouring values of a row of a tensor (of those below D).
template <class T>
static __device__ __forceinline__ void store4(T* p, int d, int D, const float* x, int aligned) {
  if (aligned) {
    if (d < D) {   // (D and the strides are multiples of 4 values)
      if constexpr (sizeof(T) == 2) { b16x4 v; for (int e = 0; e < 4; ++e) v[e] = (__bf16)x[e]; *(b16x4*)(p + d) = v; }
      else { f32x4 v = {x[0], x[1], x[2], x[3]}; *(f32x4*)(p + d) = v; }
    }
  } else {
    for (int e = 0; e < 4; ++e) if (d + e < D) p[d + e] = (T)x[e];
  }
}

template <class T>
static __device__ __forceinline__ T* at(const Tensor& t, int64_t b, int64_t n, int64_t h) { return (T*)t.p + b * t.sb + n * t.sn + h * t.sh; }

}  // namespace attn
}  // namespace gr
