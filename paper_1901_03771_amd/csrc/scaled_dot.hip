// Products of 8-bit tensors with scales: out[m][n] = sum over blocks of 128 places of sa[m] sb[n] (sum of a[m][k] b[n][k]).
//
// The matrix cores take 128 places of 16 x 16 results at once (v_mfma_f32_16x16x128_f8f6f4, 32 cycles of a SIMD): one such product from zero is a
// block's sum, and four vector instructions a lane add it to the result in float32, times the scales.  b goes in as the first operand, so that a lane
// has ONE row of a, in four neighbouring columns of the result: where b's scales are of 128 rows together, the lane's factor is one number for all its results of a block.
//
// That instruction (like every 8-bit one of this card, at any of its sizes) aligns eight neighbouring products to the largest of them and drops what lies more than 13
// places below its leading one: sums of normal numbers are off by 1.5e-5 of themselves, at most by 7 x 2^-13 of the sum of their sizes.  A result rounded to bfloat16 does not show it (half a
// step of it is 2^-8; 1.7e-3 from binary64 with and without).  For a float32 result the operands become bfloat16 on their way from LDS, which holds e4m3 exactly, and four products of 32 places
// each are summed in float32 proper: 2^-24, at twice the cycles.
//
// Large products are bound by the card's power (8192^3: 445 to 465 us, 2.4 PFLOP/s, the matrix cores busy 62 % of the cycles at 1.8 GHz; of zeros 344 us), those into float32 by vector
// instructions beside the products (4096 x 6144 x 16384 with factors of rows: 750 us, 1.1 PFLOP/s, vector units 69 %, matrix cores 53 %), few rows by reading b.
#include <type_traits>

#include "scaled_kernels.h"

namespace gr {
namespace scaled {

#define GR_LDS __attribute__((address_space(3)))
#define GR_INLINE __attribute__((always_inline))

// 32 places of a row a lane, as the matrix cores take them: 8-bit, or bfloat16 where sums are to be float32 proper.
template <bool PROPER> struct Operand;
template <> struct Operand<false> {
  i32x8 v;
  __device__ __forceinline__ void set(i32x8 x) { v = x; }
};
template <> struct Operand<true> {
  b16x8 v[4];
  __device__ __forceinline__ void set(i32x8 x) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const b16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[i], 1.0f, false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[i], 1.0f, true);
      v[i / 2][i % 2 * 4] = lo[0]; v[i / 2][i % 2 * 4 + 1] = lo[1];
      v[i / 2][i % 2 * 4 + 2] = hi[0]; v[i / 2][i % 2 * 4 + 3] = hi[1];
    }
  }
};
static __device__ __forceinline__ f32x4 block_product(const Operand<false>& a, const Operand<false>& b) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a.v, b.v, f32x4{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0, 0, 0, 0);
}
static __device__ __forceinline__ f32x4 block_product(const Operand<true>& a, const Operand<true>& b) {
  f32x4 z = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int s = 0; s < 4; ++s) z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v[s], b.v[s], z, 0, 0, 0);
  return z;
}

// 16 bytes k .. k + 15 of a row of K bytes at any address, zeros behind its end, in two steps without a branch between loads: what is loaded ends with the row, and is moved
// to its place once it is needed.
template <bool LONG = false>
static __device__ __forceinline__ i32x4 bytes_until(const uint8_t* row, int k, int K) {
  typedef int anywhere __attribute__((ext_vector_type(4), aligned(1)));
  if (LONG || K >= 16) return *(const __attribute__((address_space(1))) anywhere*)(uintptr_t)(row + min(k, K - 16));
  i32x4 v = {0, 0, 0, 0};
#pragma unroll
  for (int e = 0; e < 15; ++e) v[e / 4] |= (e < K ? (int)row[min(e, K - 1)] : 0) << (8 * (e % 4));
  return v;
}
static __device__ __forceinline__ i32x4 in_place(i32x4 v, int k, int K) {
  const int off = K >= 16 ? k - min(k, K - 16) : k;   // bytes that are too many in front
  uint64_t lo = (uint32_t)v[0] | (uint64_t)(uint32_t)v[1] << 32, hi = (uint32_t)v[2] | (uint64_t)(uint32_t)v[3] << 32;
  const int bits = 8 * (off & 7);
  if (off >= 8) { lo = hi; hi = 0; }
  lo = bits ? lo >> bits | hi << (64 - bits) : lo;
  hi >>= bits;
  if (off >= 16) lo = hi = 0;
  return i32x4{(int)lo, (int)(lo >> 32), (int)hi, (int)(hi >> 32)};
}

// The same of rows at odd addresses: whole words, each of which holds a byte of the row, and a fifth one where the bytes stand across five.  (Vector loads at addresses that are no
// multiple of four bytes take this card 2.7 times as long: 4 rows by 4096, 4095 places, 20 us.)
struct Words { i32x4 v; int more; };
static __device__ __forceinline__ Words words_until(const uint8_t* row, int k, int K) {
  if (K < 16) return {bytes_until(row, k, K), 0};
  typedef int anywhere __attribute__((ext_vector_type(4), aligned(4)));
  const uint8_t* const p = row + min(k, K - 16);
  const int off = (int)(uintptr_t)p & 3;
  return {*(const anywhere*)(p - off), *(const int*)(p - off + (off ? 16 : 12))};
}
static __device__ __forceinline__ i32x4 joined(const Words& w, const uint8_t* row, int k, int K) {
  const uint32_t off = K < 16 ? 0 : (uint32_t)(uintptr_t)(row + min(k, K - 16)) & 3;
  i32x4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = (int)__builtin_amdgcn_alignbyte((uint32_t)(e < 3 ? w.v[e + 1] : w.more), (uint32_t)w.v[e], off);
  return v;
}

// Tiles in LDS: rows of 128 bytes, chunks of 16; chunk c of row r lies in place c ^ twist(r): a chunk of 16 neighbouring rows, which is what 16 lanes
// read at once, then stands in all 64 banks.
static __device__ __forceinline__ int twist(int r) { return (r >> 1) & 7; }

// Row r of a tile as an operand.  The order of the 128 places is free as long as both operands have the same: lane group g takes chunks g and g + 4.
static __device__ __forceinline__ i32x8 operand(const GR_LDS char* tile, int r, int g) {
  const int at = r * 128 + ((g ^ twist(r)) << 4);
  const i32x4 x = *(const GR_LDS i32x4*)(tile + at), y = *(const GR_LDS i32x4*)(tile + (at ^ 64));
  return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
}

// Waits for this wave's loads and LDS accesses, then for everybody's.
static __device__ __forceinline__ void arrive() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

template <class T>
static __device__ __forceinline__ void store4(T* row, int n, int N, f32x4 v) {
  if (n + 4 <= N) {
    typedef T anywhere __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    anywhere z;
#pragma unroll
    for (int e = 0; e < 4; ++e) z[e] = (T)v[e];
    *(anywhere*)(row + n) = z;
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e) if (n + e < N) row[n + e] = (T)v[e];
  }
}

// The same where only LDS is waited for: what is under way to registers stays so.
static __device__ __forceinline__ void arrive_in_lds() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Which tile and which split a workgroup takes.  Workgroups go round the eight XCDs in turn, each with an L2 of its own: an XCD takes neighbouring
// tiles, eight rows of them at a time.
struct Place { int n, m, split; };
static __device__ __forceinline__ Place place_of(const Dot& d) {
  const unsigned all = gridDim.x, id = blockIdx.x, each = all / 8, rest = all % 8, x = id % 8;
  unsigned k = x * each + (x < rest ? x : rest) + id / 8;
  Place p;
  const unsigned tiles = (unsigned)d.mt * d.nt;
  p.split = (int)(k / tiles);
  k -= p.split * tiles;
  const unsigned band = k / (8u * d.nt), rows = min(8u, d.mt - band * 8), in = k - band * 8 * d.nt;
  p.n = (int)(in / rows);
  p.m = (int)(band * 8 + in % rows);
  return p;
}

// A tile of rows in flight straight into LDS (buffer_load_dwordx4 .. lds: lane L of a wave fills the 16 bytes at L of its kilobyte, so the twist is in the lane's
// address).  Each of a thread's chunks has a buffer of its own, in scalar registers, so that one vector register holds its place in all of them; a buffer ends with the last
// valid row, and a place behind the end of a row is given an address behind it: both read zeros.
template <int ROWS, int THREADS>
struct Flight {
  static constexpr int N = ROWS * 8 / THREADS, STEP = THREADS / 8;
  static_assert(N * THREADS == ROWS * 8 && STEP % 16 == 0, "whole chunks for every thread, the same twist for all of them");
  i32x4 rsrc[N];
  uint32_t first;            // of the thread's first chunk
  int at;                    // of the chunk in the row
  uint32_t lds0;
  __device__ __forceinline__ Flight(const uint8_t* base, int64_t stride, int rows, int K, int tid, GR_LDS char* tile) {
    const int r = tid / 8;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const uint64_t b = (uint64_t)base + n * STEP * stride;
      const int left = rows - n * STEP;
      rsrc[n] = i32x4{__builtin_amdgcn_readfirstlane((int)b), __builtin_amdgcn_readfirstlane((int)(b >> 32) & 0xffff),
                      __builtin_amdgcn_readfirstlane(left > 0 ? (left - 1) * (int)stride + K : 0), 0x00027000};
    }
    at = ((tid % 8) ^ twist(r)) * 16;
    first = r * (uint32_t)stride + at;
    lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)tile + (tid & ~63) * 16);
  }
  __device__ __forceinline__ uint32_t place(int kb, int K) const { return kb * 128 + at < K ? first + kb * 128 : 0x80000000u; }
  __device__ __forceinline__ void go(int n, uint32_t off, uint32_t stage) const {
    // (the statement leaves the scalar condition code alone; wait states: M0)
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" : : "v"(off), "s"(rsrc[n]), "s"(lds0 + stage + n * THREADS * 16) : "memory", "m0");
  }
};

// A tile of TM rows of a by TN rows of b, waves WM x WN.  Stages of a block each in LDS: while one is multiplied, the others are under way, through registers (any strides) or straight
// into LDS (DIRECT).  Two of them, or three for tiles of 64 rows, which have few products to hide a load behind (512 x 4096 x 4096: 15.7 us, with two 23, with four, whose LDS leaves a compute unit
// one workgroup, 18.7; of 128 x 128, 26 with two and 28 with three).  Four waves, or eight through registers, where a
// SIMD's second wave works while one moves bytes into place (777 x 1291 x 1003 in float32: 11.7 us, with four 13.6; 1024 x 4096 x 4095 33 and 40, but 4000 x 6000 x 3001 146 and 135; straight into
// LDS, 192 x 4096 x 14336: 25.7 and 24.9).
template <int TM, int TN, int WM, int WN, bool DIRECT, int STAGES, bool BLOCKS, class OUT>
__global__ __launch_bounds__(WM * WN * 64, 2) void gr_dot_scaled_kernel(const Dot d) {
  constexpr int THREADS = WM * WN * 64, I = TN / WN / 16, J = TM / WM / 16, NB = TN / BLOCK;
  constexpr int CA = TM * 8 / THREADS, CB = TN * 8 / THREADS;               // chunks of a thread
  static_assert(CA * THREADS == TM * 8 && CB * THREADS == TN * 8, "whole chunks for every thread");
  constexpr int STAGE = (TM + TN) * 128;
  // factors of a stage: of the rows of a, for each block of rows of b (BLOCKS, two stages) or apart from those of b
  constexpr int USED = !BLOCKS ? TM + TN : STAGES > 2 ? TM + NB : NB * TM, FACTORS = USED > THREADS ? USED : THREADS;
  __shared__ __attribute__((aligned(1024))) char memory[STAGES * (STAGE + FACTORS * 4)];
  GR_LDS char* const lds = (GR_LDS char*)memory;
  GR_LDS float* const factors = (GR_LDS float*)(lds + STAGES * STAGE);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l = lane & 15, g = lane >> 4;
  const int wm = wave % WM * (TM / WM), wn = wave / WM * (TN / WN);
  const Place p = place_of(d);
  const int m0 = p.m * TM, n0 = p.n * TN, rows_a = min(TM, d.M - m0), rows_b = min(TN, d.N - n0);
  const int first = (int)((int64_t)d.KB * p.split / d.splits), last = (int)((int64_t)d.KB * (p.split + 1) / d.splits);
  const uint8_t* const a = d.a + (int64_t)m0 * d.a_s;
  const uint8_t* const b = d.b + (int64_t)n0 * d.b_s;

  constexpr int SETS = DIRECT ? 1 : 2;   // blocks on their way through registers at once (512 x 4096 x 4095 with four waves: 29 us with two, 37 with one)
  i32x4 staged[SETS][DIRECT ? 1 : CA + CB];
  const Flight<TM, THREADS> fa(a, d.a_s, rows_a, d.K, tid, lds);
  const Flight<TN, THREADS> fb(b, d.b_s, rows_b, d.K, tid, lds + TM * 128);
  // Chunk c of a tile on its way into LDS.
  auto send = [&](int c, int kb, int stage) GR_INLINE {
    if (c < CA) fa.go(c, fa.place(kb, d.K), stage * STAGE);
    else fb.go(c - CA, fb.place(kb, d.K), stage * STAGE);
  };
  // (a row behind the last is read as the last: its results go nowhere; a block behind the last as the last, which nothing takes.  MORE: of more than one, so that rows have 16 bytes, or none
  // of them is taken and it reads the kernel's arguments: no branch makes the loads before it wait.)
  const uint8_t* const some = (const uint8_t*)__builtin_amdgcn_kernarg_segment_ptr();
  auto fetch = [&](int kb, int set, auto more) GR_INLINE {
    constexpr bool MORE = decltype(more)::value;
    if (MORE) kb = min(kb, last - 1);
    const bool there = !MORE || d.K >= 16;
    const uint8_t *const from_a = there ? a : some, *const from_b = there ? b : some;
    const int64_t step_a = there ? d.a_s : 0, step_b = there ? d.b_s : 0;
    const int K = there ? d.K : 16;
#pragma unroll
    for (int c = 0; c < CA; ++c) staged[set][c] = bytes_until<MORE>(from_a + min((c * THREADS + tid) / 8, rows_a - 1) * step_a, kb * 128 + tid % 8 * 16, K);
#pragma unroll
    for (int c = 0; c < CB; ++c) staged[set][CA + c] = bytes_until<MORE>(from_b + min((c * THREADS + tid) / 8, rows_b - 1) * step_b, kb * 128 + tid % 8 * 16, K);
  };
  auto settle = [&](int kb, int stage, int set) GR_INLINE {
    if (kb * 128 + 128 > d.K) {
#pragma unroll
      for (int c = 0; c < CA + CB; ++c) staged[set][c] = in_place(staged[set][c], kb * 128 + tid % 8 * 16, d.K);
    }
#pragma unroll
    for (int c = 0; c < CA + CB; ++c) {
      const int i = (c < CA ? c : c - CA) * THREADS + tid, r = i / 8;
      *(GR_LDS i32x4*)(lds + stage * STAGE + (c < CA ? 0 : TM * 128) + r * 128 + ((i % 8 ^ twist(r)) << 4)) = staged[set][c];
    }
  };
  // The factors of a block, a thread each.  (Rows behind the last have the last one's: their results go nowhere.  Threads without a factor of their own write one that
  // nothing reads: between a product and its use stands no branch, where the compiler has been seen to count too few wait states.)
  static_assert(FACTORS == THREADS && TM % 64 == 0, "a factor a thread, of the same operand across a wave");
  constexpr bool DEEP = STAGES > 2;
  static_assert(STAGES == 2 || (STAGES == 3 && DIRECT), "tiles that pass through registers have two stages");
  const bool of_a = (BLOCKS && !DEEP) || tid < TM;
  const int64_t of_b = BLOCKS ? min(n0 / BLOCK + tid - TM, (d.N - 1) / BLOCK) : n0 + min(tid - TM, rows_b - 1);
  const float* const row_factor = of_a ? d.sa + (int64_t)(m0 + min(tid % TM, rows_a - 1)) * d.sa_m : d.sb + of_b * d.sb_n;
  const int64_t row_step = of_a ? d.sa_k : d.sb_k;
  const float* const block_factor = d.sb + (int64_t)min(n0 / BLOCK + __builtin_amdgcn_readfirstlane(tid / TM), (d.N - 1) / BLOCK) * d.sb_n;
  float factor = 0.0f;
  auto fetch_factors = [&](int kb) GR_INLINE { factor = row_factor[min(kb, last - 1) * row_step]; };
  auto settle_factors = [&](int kb, int stage) GR_INLINE {
    if constexpr (BLOCKS) factor *= ((const __attribute__((address_space(4))) float*)block_factor)[min(kb, last - 1) * d.sb_k];
    factors[stage * FACTORS + tid] = factor;
  };
  // Three stages: factors go straight into LDS like the tiles, those of a's rows and those of b apart, and a wait leaves the tile after the next under way.
  const uint32_t factors0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(factors + (tid & ~63)));
  auto send_factors = [&](int kb, int stage) GR_INLINE {
    const float* const from = row_factor + min(kb, last - 1) * row_step;
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 4\n\tglobal_load_lds_dword %0, off" : : "v"(from), "s"(factors0 + stage * FACTORS * 4) : "memory", "m0");
  };
  constexpr int UNDER_WAY = (STAGES - 2) * (CA + CB + 1);   // loads of the tile after the next, and of its factors
  auto arrive_but_one = [&]() GR_INLINE { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(UNDER_WAY) : "memory"); };

  // Steps that operands of b are read ahead: a read from LDS takes longer than one step's products (8192^3: 465 us with one, 445 with two).  (With factors of their own for b's rows the
  // registers hold one, of tiles of 256 x 256; waves with two steps a block read one ahead.)
  constexpr int AHEAD = (I == 8 && !BLOCKS) || I == 2 ? 1 : 2, RING = 2 * AHEAD;
  constexpr int EARLY = AHEAD + I / 8;   // steps over which a tile is sent for
  constexpr bool PROPER = sizeof(OUT) == 4;
  f32x4 acc[I][J];
#pragma unroll
  for (int i = 0; i < I; ++i)
#pragma unroll
    for (int j = 0; j < J; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  // A block begins with the operands of a's rows in registers, and the first of b's; they are read while the last step of the block before it is multiplied, each once the
  // product that had its registers is on its way.
  static_assert(I % RING == 0 && EARLY <= I - AHEAD, "operands of b go round their registers, and a tile has time to come");
  i32x8 raw[J], y[RING];
  f32x4 t[BLOCKS ? 1 : RING];
  float s[STAGES][J];
  auto read_a = [&](int j, auto parity) GR_INLINE {
    constexpr int P = decltype(parity)::value;
    raw[j] = operand(lds + P * STAGE, wm + 16 * j + l, g);
    s[P][j] = factors[P * FACTORS + (BLOCKS && !DEEP ? wn / BLOCK * TM : 0) + wm + 16 * j + l];
    if constexpr (BLOCKS && DEEP) s[P][j] *= factors[P * FACTORS + TM + wn / BLOCK];
  };
  auto read_b = [&](int i, auto parity) GR_INLINE {
    constexpr int P = decltype(parity)::value;
    y[i % RING] = operand(lds + P * STAGE + TM * 128, wn + 16 * i + l, g);
    if constexpr (!BLOCKS) t[i % RING] = *(const GR_LDS f32x4*)(factors + P * FACTORS + TM + wn + 16 * i + 4 * g);
  };
  auto block = [&](int kb, auto parity) GR_INLINE {
    constexpr int P = decltype(parity)::value;
    constexpr std::integral_constant<int, (P + 1) % STAGES> other;
    Operand<PROPER> x[J];
    f32x4 z[J], before = {1.0f, 1.0f, 1.0f, 1.0f};
#pragma unroll
    for (int j = 0; j < J; ++j) x[j].set(raw[j]);
    if constexpr (!DIRECT) {   // (has branches: before the first product)
      settle(kb + 1, P ^ 1, (P ^ 1) % SETS);
      fetch(kb + 1 + SETS, (P ^ 1) % SETS, std::true_type());
    }
    // Columns 16 at a time: four sums of the step before are added, then the registers take the next product.
#pragma unroll
    for (int i = 0; i <= I; ++i) {
      if (i == I - AHEAD) {
        // All operands of this block have been read: everybody waits for the next one's tiles, and the one after it takes this one's place.
        if constexpr (DEEP) {
          arrive_but_one();
          send_factors(kb + STAGES, P);
        } else {
          settle_factors(kb + 1, P ^ 1);
          if constexpr (DIRECT) arrive();
          else arrive_in_lds();
          fetch_factors(kb + 2);
        }
      }
      Operand<PROPER> o;
      if (i < I) o.set(y[i % RING]);
      f32x4 last_t = {1.0f, 1.0f, 1.0f, 1.0f};
      if constexpr (!BLOCKS) { last_t = before; before = t[i % RING]; }
      if (i + AHEAD < I) read_b(i + AHEAD, parity);
      else if (i < I) read_b(i + AHEAD - I, other);
#pragma unroll
      for (int j = 0; j < J; ++j) {
        if (i > 0) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float v = z[j][e];
            if constexpr (!BLOCKS) v *= last_t[e];
            acc[i - 1][j][e] = __builtin_fmaf(v, s[P][j], acc[i - 1][j][e]);
          }
          // (kept here: moved behind a block's end, the sums would leave all its products in registers, and a branch between them and their use)
          asm volatile("" : "+v"(acc[i - 1][j]));
        }
        if (i < I) z[j] = block_product(o, x[j]);
        if constexpr (DIRECT) {
          // A tile is sent for a few chunks at a time, from where its place is free: all at once would keep the waves from multiplying until they are under way.
          // (behind the last block: another split's or zeros, which nothing takes)
          constexpr int SLOTS = EARLY * J;
          const int slot = i >= I ? SLOTS : i >= I - AHEAD ? (i - I + AHEAD) * J + j : i < EARLY - AHEAD ? (i + AHEAD) * J + j : SLOTS;
          if (slot < SLOTS)
#pragma unroll
            for (int c = slot * (CA + CB) / SLOTS; c < (slot + 1) * (CA + CB) / SLOTS; ++c) {
              if (i >= I - AHEAD) send(c, kb + STAGES, P);
              else send(c, kb + STAGES - 1, (P + STAGES - 1) % STAGES);
            }
        }
        if (i == I - 1) read_a(j, other);
      }
      if (i > 0 && i < I) {
#pragma unroll
        for (int j = 0; j < J; ++j) {
          __builtin_amdgcn_sched_group_barrier(0x2, BLOCKS ? 4 : 8, 0);   // vector instructions
          __builtin_amdgcn_sched_group_barrier(0x8, PROPER ? 4 : 1, 0);   // products
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  if (first < last) {
    constexpr int SENT = AHEAD * J * (CA + CB) / (EARLY * J);   // of a tile before its first block begins
    if constexpr (DEEP) {
#pragma unroll
      for (int t = 0; t < STAGES - 1; ++t) {
        send_factors(first + t, t);
#pragma unroll
        for (int c = 0; c < CA + CB; ++c) send(c, first + t, t);
      }
      arrive_but_one();
      send_factors(first + STAGES - 1, STAGES - 1);
    } else {
      fetch_factors(first);
      if constexpr (DIRECT) {
#pragma unroll
        for (int c = 0; c < CA + CB; ++c) send(c, first, 0);
      } else {
        fetch(first, 0, std::false_type());
        settle(first, 0, 0);
      }
      settle_factors(first, 0);
      arrive();
      if constexpr (!DIRECT) {
#pragma unroll
        for (int t = 1; t <= SETS; ++t) fetch(first + t, t % SETS, std::true_type());
      }
      fetch_factors(first + 1);
    }
    if constexpr (DIRECT) {
#pragma unroll
      for (int c = 0; c < SENT; ++c) send(c, first + STAGES - 1, STAGES - 1);
    }
    constexpr std::integral_constant<int, 0> even;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) read_b(i, even);
#pragma unroll
    for (int j = 0; j < J; ++j) read_a(j, even);
    constexpr std::integral_constant<int, 1> odd;
    if constexpr (SETS > 1) {
      // (one way out of the loop: with two, the compiler waits for the later set of loads, too)
      int kb = first;
      for (; kb + 1 < last; kb += 2) {
        block(kb, even);
        block(kb + 1, odd);
      }
      if (kb < last) block(kb, even);
    } else for (int kb = first;;) {
      block(kb, even);
      if (++kb >= last) break;
      block(kb, odd);
      if (++kb >= last) break;
      if constexpr (DEEP) {
        block(kb, std::integral_constant<int, 2>());
        if (++kb >= last) break;
      }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // (loads into LDS that nothing takes end before the workgroup does)
  }

#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int m = m0 + wm + 16 * j + l;
    if (m >= d.M) continue;
#pragma unroll
    for (int i = 0; i < I; ++i) {
      const int n = n0 + wn + 16 * i + 4 * g;
      if (d.splits > 1) store4<float>(d.parts + ((int64_t)p.split * d.M + m) * d.N, n, d.N, acc[i][j]);
      else store4<OUT>((OUT*)d.out + m * d.out_s, n, d.N, acc[i][j]);
    }
  }
}

// Few rows of a (16 MT at most): b is what is read, at the rate of the memory.  A workgroup has 32 rows of b, its eight waves take blocks of 128 places in turn, U of them in
// flight at once, straight from memory to the registers that the matrix cores read; the waves' sums are added in order.  (4 rows by 14336 x 4096: 13.3 us, 4.4 TB/s; with U = 4, whose registers leave
// a compute unit one workgroup, 14.3, and by 16384 x 2048 14.1, 8.1 so.)
template <bool WORDS> struct Chunk;
template <> struct Chunk<false> {
  i32x4 v;
  __device__ __forceinline__ void load(const uint8_t* row, int k, int K) { v = bytes_until(row, k, K); }
  __device__ __forceinline__ i32x4 get(const uint8_t*, int, int) const { return v; }
};
template <> struct Chunk<true> {
  Words w;
  __device__ __forceinline__ void load(const uint8_t* row, int k, int K) { w = words_until(row, k, K); }
  __device__ __forceinline__ i32x4 get(const uint8_t* row, int k, int K) const { return joined(w, row, k, K); }
};

template <int MT, bool WORDS, bool BLOCKS, class OUT>
__global__ __launch_bounds__(512) void gr_dot_scaled_few_kernel(const Dot d) {
  constexpr bool PROPER = sizeof(OUT) == 4;
  constexpr int WAVES = 8, NT = 2, U = 2, PITCH = 16 * NT + 4;
  __shared__ __attribute__((aligned(16))) float part[WAVES][16 * MT][PITCH];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = lane & 15, g = lane >> 4;
  const int tile = blockIdx.x % d.nt, split = blockIdx.x / d.nt, n0 = tile * 16 * NT;
  const int first = (int)((int64_t)d.KB * split / d.splits), last = (int)((int64_t)d.KB * (split + 1) / d.splits);
  const uint8_t *a[MT], *b[NT];
  const float* sa[MT];
  const float* sb[NT][BLOCKS ? 1 : 4];
#pragma unroll
  for (int j = 0; j < MT; ++j) {
    const int m = min(16 * j + l, d.M - 1);
    a[j] = d.a + m * d.a_s;
    sa[j] = d.sa + m * d.sa_m;
  }
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    b[i] = d.b + min(n0 + 16 * i + l, d.N - 1) * d.b_s;
    if constexpr (BLOCKS) {
      sb[i][0] = d.sb + min(n0 + 16 * i, d.N - 1) / BLOCK * d.sb_n;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) sb[i][e] = d.sb + min(n0 + 16 * i + 4 * g + e, d.N - 1) * d.sb_n;
    }
  }
  f32x4 acc[NT][MT];
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < MT; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  for (int kb0 = first + wave; kb0 < last; kb0 += WAVES * U) {
    Chunk<WORDS> x[U][MT][2], y[U][NT][2];
    float s[U][MT], t[U][NT][BLOCKS ? 1 : 4];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int kb = min(kb0 + u * WAVES, last - 1), k = kb * 128 + 16 * g;   // (behind the last block: the last again, which is left out of the sums)
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        y[u][i][0].load(b[i], k, d.K);
        y[u][i][1].load(b[i], k + 64, d.K);
#pragma unroll
        for (int e = 0; e < (BLOCKS ? 1 : 4); ++e) t[u][i][e] = sb[i][e][kb * d.sb_k];
      }
#pragma unroll
      for (int j = 0; j < MT; ++j) {
        x[u][j][0].load(a[j], k, d.K);
        x[u][j][1].load(a[j], k + 64, d.K);
        s[u][j] = sa[j][kb * d.sa_k];
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int kb = min(kb0 + u * WAVES, last - 1), k = kb * 128 + 16 * g;
      const bool there = kb0 + u * WAVES < last;
      i32x4 v[NT + MT][2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int i = 0; i < NT; ++i) v[i][h] = y[u][i][h].get(b[i], k + 64 * h, d.K);
#pragma unroll
        for (int j = 0; j < MT; ++j) v[NT + j][h] = x[u][j][h].get(a[j], k + 64 * h, d.K);
      }
      if (kb * 128 + 128 > d.K) {
#pragma unroll
        for (int i = 0; i < NT + MT; ++i)
#pragma unroll
          for (int h = 0; h < 2; ++h) v[i][h] = in_place(v[i][h], k + 64 * h, d.K);
      }
      Operand<PROPER> p[NT], q[MT];
#pragma unroll
      for (int i = 0; i < NT; ++i) p[i].set(__builtin_shufflevector(v[i][0], v[i][1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
      for (int j = 0; j < MT; ++j) q[j].set(__builtin_shufflevector(v[NT + j][0], v[NT + j][1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j) {
          const f32x4 z = block_product(p[i], q[j]);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float sum = __builtin_fmaf(z[e], s[u][j] * t[u][i][BLOCKS ? 0 : e], acc[i][j][e]);
            acc[i][j][e] = there ? sum : acc[i][j][e];
          }
          asm volatile("" : "+v"(acc[i][j]));   // (no branch between a product and its use)
        }
    }
  }
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < MT; ++j) *(f32x4*)&part[wave][16 * j + l][16 * i + 4 * g] = acc[i][j];
  __syncthreads();
  const int m = threadIdx.x / (4 * NT), n = threadIdx.x % (4 * NT) * 4;
  if (m >= 16 * MT || m >= d.M) return;
  f32x4 z = *(const f32x4*)&part[0][m][n];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) z += *(const f32x4*)&part[w][m][n];
  if (d.splits > 1) store4<float>(d.parts + ((int64_t)split * d.M + m) * d.N, n0 + n, d.N, z);
  else store4<OUT>((OUT*)d.out + m * d.out_s, n0 + n, d.N, z);
}

// The sum of the splits, in order.
template <class OUT>
__global__ __launch_bounds__(256) void gr_dot_scaled_join_kernel(const Dot d) {
  const int64_t n4 = (d.N + 3) / 4, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= d.M * n4) return;
  const int64_t m = i / n4;
  const int n = (int)(i - m * n4) * 4;
  f32x4 z = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int s0 = 0; s0 < d.splits; s0 += 8) {   // (eight in flight)
    f32x4 v[8];
#pragma unroll
    for (int s = 0; s < 8; ++s) v[s] = s0 + s < d.splits ? get<float>(d.parts + ((s0 + s) * (int64_t)d.M + m) * d.N, n, d.N) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int s = 0; s < 8; ++s) z += v[s];
  }
  store4<OUT>((OUT*)d.out + m * d.out_s, n, d.N, z);
}

template <int TM, int TN, int WM, int WN, bool DIRECT, int STAGES, bool BLOCKS, class OUT>
static hipError_t launch(const Dot& d, hipStream_t stream) {
  gr_dot_scaled_kernel<TM, TN, WM, WN, DIRECT, STAGES, BLOCKS, OUT><<<dim3((unsigned)(d.mt * d.nt * d.splits)), dim3(WM * WN * 64), 0, stream>>>(d);
  return hipGetLastError();
}

template <int MT, bool WORDS, bool BLOCKS, class OUT>
static hipError_t launch_few(const Dot& d, hipStream_t stream) {
  gr_dot_scaled_few_kernel<MT, WORDS, BLOCKS, OUT><<<dim3((unsigned)(d.nt * d.splits)), dim3(512), 0, stream>>>(d);
  return hipGetLastError();
}

template <bool BLOCKS, class OUT>
static hipError_t dot_of(const Dot& d, int form, hipStream_t stream) {
  if (form == DOT_FEW) return d.M <= 16 ? launch_few<1, false, BLOCKS, OUT>(d, stream) : launch_few<2, false, BLOCKS, OUT>(d, stream);
  if (form == DOT_FEW_WORDS) return d.M <= 16 ? launch_few<1, true, BLOCKS, OUT>(d, stream) : launch_few<2, true, BLOCKS, OUT>(d, stream);
  if constexpr (sizeof(OUT) == 2) if (form == DOT_LARGE) return launch<256, 256, 4, 2, true, 2, BLOCKS, OUT>(d, stream);
  if (form == DOT_LOW) return launch<64, 128, 2, 2, true, 3, BLOCKS, OUT>(d, stream);
  if (form == DOT_DIRECT) return launch<128, 128, 2, 2, true, 2, BLOCKS, OUT>(d, stream);
  if (form == DOT_STAGED_LOW) return launch<64, 128, 2, 4, false, 2, BLOCKS, OUT>(d, stream);
  if (form == DOT_STAGED) return launch<128, 128, 4, 2, false, 2, BLOCKS, OUT>(d, stream);
  return hipErrorInvalidValue;
}

hipError_t dot(const Dot& d, int form, bool blocks, int out_type, hipStream_t stream) {
  if (out_type == BF16) return blocks ? dot_of<true, __bf16>(d, form, stream) : dot_of<false, __bf16>(d, form, stream);
  return blocks ? dot_of<true, float>(d, form, stream) : dot_of<false, float>(d, form, stream);
}

hipError_t dot_join(const Dot& d, int out_type, hipStream_t stream) {
  const int64_t n = (int64_t)d.M * ((d.N + 3) / 4);
  const dim3 grid((unsigned)((n + 255) / 256));
  if (out_type == BF16) gr_dot_scaled_join_kernel<__bf16><<<grid, dim3(256), 0, stream>>>(d);
  else gr_dot_scaled_join_kernel<float><<<grid, dim3(256), 0, stream>>>(d);
  return hipGetLastError();
}

}  // namespace scaled
}  // namespace gr
