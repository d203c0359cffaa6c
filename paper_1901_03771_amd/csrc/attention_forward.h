// The output of attention: out = sum over the keys a query sees of exp(score - lse) v, lse = log(sum of exp(score)).
//
// One pass over the keys with a running maximum m and sum l per query (a lane's column, see attention_kernels.h):
// scores^T = K Q^T, p = 2^(score - m), out^T += V^T p.  m only moves when a score exceeds it by 2^8 or more: any m serves, since it
// cancels, and p <= 2^8 is far from overflow, so the products so far are rescaled a few times per row and not per tile.
//
// The rows of one head of k and v are the queries of all its G heads, query by query: k and v are read once for all of them, and a
// causal block of 128 rows spans 128 / G positions.  Two forms:
//   own rows  (DIVIDED = false): each of four waves has 32 rows, all waves walk the same tiles of keys;
//   own keys  (DIVIDED = true):  up to 32 rows, each wave takes 32 keys of every tile, and the waves' sums are joined at the end:
//              single tokens and other calls of at most 32 rows per head, whose time is that of reading k and v.
// Either may split the keys over workgroups as well (a.splits), which leaves (m, l, sums) for combine().
//
// Measured, bfloat16: 16 heads of 8192 causal rows of 128 values, a beginning seen whole, 0.40 ms (own rows: matrix cores busy 61 % of the cycles, vector units 55 %, the card's power
// lowers the clock to 1.65 GHz); a capped prompt of 8192 rows of 256 values 0.70 to 0.73 ms (vector units 59 %: a tanh and an exponential per score; matrix cores 35 %, waves wait 42 %); single tokens of
// 32 sequences of 4096 to 8192 keys 0.165 ms (own keys: 4.9 TB/s of the 6.0 of a copy).
#pragma once

#include "attention_kernels.h"

namespace gr {
namespace attn {

template <class T, int DP, bool DIVIDED>
struct Shape {
  static constexpr int WAVES = DIVIDED ? shared_waves(sizeof(T), DP) : 4;
  static constexpr int THREADS = 64 * WAVES;
  static constexpr int KEYS = DIVIDED ? 32 * WAVES : tile_rows(sizeof(T), DP);   // of a tile
  static constexpr int KB = DIVIDED ? 1 : KEYS / 32;                              // blocks of 32 keys a wave multiplies
  static constexpr int ROWS = DIVIDED ? 32 : 32 * WAVES;
  static constexpr int TILE = KEYS * Tile<T, DP>::ROW;
  // two stages of a tile of k and one of v (the joining waves' sums lie over them), two stages of the keys' documents
  static constexpr int LDS = 4 * TILE + 2 * KEYS * 4;
  static_assert(!DIVIDED || WAVES * 32 * (DP + 4) * 4 <= 4 * TILE, "the waves' sums fit the stages");
  // registers: operands of q, sums, scores
  static constexpr int REGS = DP / 16 * (sizeof(T) == 2 ? 4 : 12) + DP / 2 + 16 * KB;
  static constexpr bool TIGHT = REGS > (sizeof(T) == 2 ? 128 : 100);   // of registers: addresses within tiles are formed anew for each tile
  static constexpr int PER_CU = forward_per_cu(sizeof(T), DP);
  static_assert(DIVIDED || PER_CU * LDS <= 160 * 1024, "LDS of a compute unit");
};

// PRECISE (bfloat16): a probability enters its product as the sum of two bfloat16 numbers, so that the sum is right to 2^-16 and not only what 8 bits of every
// probability give.  Taken where `rest` is wanted, since the gradient's dp - delta nearly cancels for queries that see few keys (0.30 -> 0.40 ms in the pass of 16
// heads above), and in all calls of own keys, whose time is the memory's: out is then as near to binary64 as its own rounding lets it be (1.7e-3 in norm, 2.0e-3 to
// 2.3e-3 without) for 1 to 3 % (32 sequences of 4096 to 8192 keys 164.8 -> 167.6 us; 256 values a head, 16 sequences of 2048 to 4096 keys, 61.7 -> 65.9).
template <class T, int DP, int MODE, bool DIVIDED, bool PRECISE>
__global__ __launch_bounds__((Shape<T, DP, DIVIDED>::THREADS), (Shape<T, DP, DIVIDED>::PER_CU)) void gr_attention_kernel(const Args a) {
  typedef Shape<T, DP, DIVIDED> S;
  typedef Tile<T, DP> L;
  typedef typename Frag<T>::type F;
  extern __shared__ char smem_[];
  GR_LDS char* const smem = (GR_LDS char*)smem_;
  GR_LDS int* const documents = (GR_LDS int*)(smem + 4 * S::TILE);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, hi = lane >> 5;
  const int pairs = a.B * a.HK;
  const Place place = place_of(blockIdx.x, pairs, a.blocks * a.splits);
  if (place.block >= a.blocks * a.splits) return;
  // the last blocks of rows see the most keys: they start first
  const int split = place.block % a.splits, rb = a.blocks - 1 - place.block / a.splits;
  const int b = place.pair / a.HK, hk = place.pair - b * a.HK;
  const int R = a.N * a.G, row0 = rb * S::ROWS, wrow0 = row0 + (DIVIDED ? 0 : wave * 32);
  const int len = length_of(a, b), pre = a.prefix ? scalar(a.prefix, b * a.prefix_s) : 0;
  const Row mine = row_of(a, hk, wrow0 + col);   // (not kept beyond the operands: registers are full)
  // of the workgroup's rows, and of this wave's: how many keys the last one sees, the first one
  const int i_last = (row0 + S::ROWS <= R ? row0 + S::ROWS - 1 : R - 1) / a.G;
  const int end = keys_seen(a, i_last, len, pre);
  const int w_first = wrow0 < R ? keys_seen(a, wrow0 / a.G, len, pre) : 0;
  const int w_last = wrow0 < R ? keys_seen(a, (wrow0 + 31 < R ? wrow0 + 31 : R - 1) / a.G, len, pre) : 0;

  // documents: what the pieces of the wave's and the workgroup's queries hold
  Span w = {0, 0, true}, all = {0, 0, true};
  if (a.kdoc) {
    const int* const qr = a.qranges + (int64_t)b * ((a.N + 31) / 32) * 2;
    all = span_of(qr, row0 / a.G, i_last);
    w = span_of(qr, min(wrow0, R - 1) / a.G, min(wrow0 + 31, R - 1) / a.G);
  }
  const int pieces = (a.M + 31) / 32;
  const int* const ranges = a.kdoc ? a.kranges + (int64_t)b * pieces * 2 : nullptr;
  Finder<S::KEYS / 32> find{ranges, pieces, all.lo, all.hi};

  // the rows' operands
  F qf[L::STEPS];
  {
    const T* q = at<T>(a.q, b, mine.i, mine.h);
#pragma unroll
    for (int s = 0; s < L::STEPS; ++s) qf[s] = L::fetch(q, s, hi, a.D, mine.valid, a.q.aligned);
  }
  float slope = MODE & MODE_BIAS ? a.slopes[mine.h * a.slopes_s] * LOG2E : 0.0f;
  const int64_t pos = MODE & MODE_BIAS ? (a.step ? (int64_t)len - 1 : a.position + mine.i) : 0;
  const float c = MODE & MODE_BIAS ? 1.0f : a.c;

  f32x16 o[L::BLOCKS];
#pragma unroll
  for (int d = 0; d < L::BLOCKS; ++d) o[d] = (f32x16)0.0f;
  float my = -INF, m = -INF, l = 0.0f;   // the running maximum, as y and in binary logarithms

  const int tiles = (end + S::KEYS - 1) / S::KEYS, per = (tiles + a.splits - 1) / a.splits;
  const int t1 = min(tiles, (split + 1) * per);
  const T* const kbase = at<T>(a.k, b, 0, hk);
  const T* const vbase = at<T>(a.v, b, 0, hk);
  // (rows from the length on are never read: what a cache holds there has no say, not even infinities times zero)
  auto load = [&](int t, int stage) {
    const int64_t k0 = (int64_t)t * S::KEYS;
    const int rows = min(S::KEYS, len - (int)k0);
    L::template load<S::KEYS, S::THREADS>(smem + 2 * stage * S::TILE, kbase + k0 * a.k.sn, a.k.sn, rows, a.D, S::TIGHT ? fresh(tid) : tid, a.k.direct);
    L::template load<S::KEYS, S::THREADS>(smem + (2 * stage + 1) * S::TILE, vbase + k0 * a.v.sn, a.v.sn, rows, a.D, S::TIGHT ? fresh(tid) : tid, a.v.direct);
    if (a.kdoc && wave * 64 < S::KEYS) load_words((GR_LDS float*)(documents + stage * S::KEYS + wave * 64), a.kdocs + b * padded_rows(a.M) + k0 + wave * 64, lane, S::KEYS - wave * 64);
  };
  int t = find.next(split * per, t1, lane), stage = 0;
  if (t < t1) load(t, 0);
  loaded(qf);
  if constexpr (MODE & MODE_BIAS) loaded(slope);
  while (t < t1) {
    const int after = find.next(t + 1, t1, lane);
    arrive();
    if (after < t1) load(after, stage ^ 1);
    const GR_LDS char* const kt = smem + 2 * stage * S::TILE + (DIVIDED ? wave * 32 * L::ROW : 0);
    const GR_LDS char* const vt = kt + S::TILE;
    const int key0 = t * S::KEYS + (DIVIDED ? wave * 32 : 0);
    if (key0 < w_last) {
      bool whole = key0 + 32 * S::KB <= w_first, one = true;   // one: all keys and all of the wave's rows belong to one document
      if (ranges) {
#pragma unroll
        for (int kb = 0; kb < S::KB; ++kb) {
          const int e = min(key0 / 32 + kb, pieces - 1);
          one &= w.one & (scalar(ranges, 2 * e) == w.hi) & (scalar(ranges, 2 * e + 1) == w.hi);
        }
        whole = whole && one;
      }
      const int tcol = S::TIGHT ? fresh(col) : col, tlane = S::TIGHT ? fresh(lane) : lane;
      // (the wave that multiplies goes first: its next product is what the other one's exponentials run beside)
      __builtin_amdgcn_s_setprio(1);
      f32x16 s[S::KB];
#pragma unroll
      for (int kb = 0; kb < S::KB; ++kb) {
        s[kb] = (f32x16)0.0f;
#pragma unroll
        for (int st = 0; st < L::STEPS; ++st) {
          if constexpr (DP == 256) anew(qf[st]);
          s[kb] = mma(L::row(kt, kb * 32 + tcol, st, hi), qf[st], s[kb]);
        }
      }
      __builtin_amdgcn_s_setprio(0);
      if constexpr (S::KB == 2) finished(s[0], s[1]);
      else finished(s[0]);
      if constexpr (MODE != 0) {
        const float away = MODE & MODE_BIAS ? (float)(pos - key0 - 4 * (tlane >> 5)) : 0.0f;   // from the first key of this half
#pragma unroll
        for (int kb = 0; kb < S::KB; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            float y = s[kb][r];
            if constexpr (MODE & MODE_CAP) y = capped<T, MODE>(y, a.cin);
            if constexpr (MODE & MODE_BIAS) y = __builtin_fmaf(y, a.c, -slope * __builtin_fabsf(away - (float)(kb * 32 + (r & 3) + 8 * (r >> 2))));
            s[kb][r] = y;
          }
      }
      if (!whole) {
        const int flane = fresh(lane);
        const Row me = row_of(a, hk, wrow0 + (flane & 31));
        const int see = (me.valid ? keys_seen(a, me.i, len, pre) : 0) - key0 - 4 * (flane >> 5);
#pragma unroll
        for (int kb = 0; kb < S::KB; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[kb][r] = kb * 32 + (r & 3) + 8 * (r >> 2) < see ? s[kb][r] : -INF;
        if (!one) {
          const int doc = me.valid ? a.qdocs[b * padded_rows(a.N) + me.i] : -1;
          const GR_LDS int* const kd = documents + stage * S::KEYS + (DIVIDED ? wave * 32 : 0) + 4 * (flane >> 5);
#pragma unroll
          for (int kb = 0; kb < S::KB; ++kb)
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4) {
              const i32x4 n = *(const GR_LDS i32x4*)(kd + kb * 32 + 8 * r4);
#pragma unroll
              for (int e = 0; e < 4; ++e) s[kb][4 * r4 + e] = (n[e] == doc) & (doc >= 0) ? s[kb][4 * r4 + e] : -INF;
            }
        }
      }
      float top = s[0][0];
#pragma unroll
      for (int kb = 0; kb < S::KB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) top = __builtin_fmaxf(top, s[kb][r]);
      top = max_halves(top);
      if (__any(top * c > m + 8.0f)) {
        const float to = __builtin_fmaxf(my, top), by = to == -INF ? 1.0f : exp2_((my - to) * c);
        my = to;
        m = to * c;
        l *= by;
#pragma unroll
        for (int d = 0; d < L::BLOCKS; ++d) o[d] *= by;
      }
      float less = m == -INF ? 0.0f : m;
      // (scores of 2^20 and more: m is rounded by as much as an exponent counts, so the difference is taken before the product; of those rows
      // only, which leaves every row the bits that it would have beside any others)
      if (__any(__builtin_fabsf(less) > 1048576.0f)) {
        const bool far = __builtin_fabsf(less) > 1048576.0f;
        const float by = far ? my : 0.0f;
        less = far ? 0.0f : less;
#pragma unroll
        for (int kb = 0; kb < S::KB; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[kb][r] -= by;
      }
#pragma unroll
      for (int kb = 0; kb < S::KB; ++kb) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          s[kb][r] = exp2_(__builtin_fmaf(s[kb][r], c, -less));
          l += s[kb][r];
        }
#pragma unroll
        for (int st = 0; st < 2; ++st) {
          F p, low;
          operand(s[kb], st, p);
          if constexpr (PRECISE) {
#pragma unroll
            for (int j = 0; j < 8; ++j) s[kb][8 * st + j] -= (float)p[j];
            operand(s[kb], st, low);
          }
#pragma unroll
          for (int d = 0; d < L::BLOCKS; ++d) {
            const F v = L::column(vt, kb * 32 + st * 16, d, tlane);
            o[d] = mma(v, p, o[d]);
            if constexpr (PRECISE) o[d] = mma(v, low, o[d]);
          }
        }
      }
    }
    t = after;
    stage ^= 1;
  }
  finished(o);
  l = sum_halves(l);
  // A maximum passes over scores that are not numbers, the sum does not: where it is none, the maximum is made none too, so that a row or a part
  // of one that saw NaN is told from one that saw nothing (m = -inf, l = 0) wherever they are joined.
  if (l != l) m = l;

  if constexpr (DIVIDED) {
    // the waves' sums: each scaled to the largest maximum, added in the order of the waves
    GR_LDS float* const sums = (GR_LDS float*)smem;          // [wave][row][DP + 4]
    constexpr int PITCH = DP + 4;
    __syncthreads();
    if (hi == 0) { sums[(wave * 32 + col) * PITCH + DP] = m; sums[(wave * 32 + col) * PITCH + DP + 1] = l; }
    __syncthreads();
    float top = -INF, total = 0.0f;
#pragma unroll
    for (int w = 0; w < S::WAVES; ++w) top = __builtin_fmaxf(top, sums[(w * 32 + col) * PITCH + DP]);
#pragma unroll
    for (int w = 0; w < S::WAVES; ++w) {
      const float mw = sums[(w * 32 + col) * PITCH + DP];
      total += sums[(w * 32 + col) * PITCH + DP + 1] * (mw == -INF ? 0.0f : exp2_(mw - top));
    }
    const float by = m == -INF ? 0.0f : exp2_(m - top);
#pragma unroll
    for (int d = 0; d < L::BLOCKS; ++d)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const f32x4 x = {o[d][r] * by, o[d][r + 1] * by, o[d][r + 2] * by, o[d][r + 3] * by};
        *(GR_LDS f32x4*)(sums + (wave * 32 + col) * PITCH + d * 32 + 2 * r + 4 * hi) = x;
      }
    __syncthreads();
    // wave w finishes the blocks d = w, w + WAVES, ..: its lanes keep the rows they had
#pragma unroll
    for (int d = 0; d < L::BLOCKS; ++d) {
      if (d % S::WAVES != wave) continue;
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        f32x4 x = (f32x4)0.0f;
#pragma unroll
        for (int w = 0; w < S::WAVES; ++w) x += *(const GR_LDS f32x4*)(sums + (w * 32 + col) * PITCH + d * 32 + 2 * r + 4 * hi);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[d][r + e] = x[e];
      }
    }
    m = total != total ? total : top;
    l = total;
  }

  const Row me = row_of(a, hk, wrow0 + col);
  if (!me.valid) return;
  const bool first = !DIVIDED || wave == 0;
  if (a.splits > 1) {
    const int64_t at_row = ((int64_t)split * pairs + place.pair) * R + wrow0 + col;
    float* const po = a.part_o + at_row * DP;
#pragma unroll
    for (int d = 0; d < L::BLOCKS; ++d) {
      if (DIVIDED && d % S::WAVES != wave) continue;
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const f32x4 x = {o[d][r], o[d][r + 1], o[d][r + 2], o[d][r + 3]};
        *(f32x4*)(po + d * 32 + 2 * r + 4 * hi) = x;
      }
    }
    if (first && hi == 0) { a.part_ml[2 * at_row] = m; a.part_ml[2 * at_row + 1] = l; }
    return;
  }
  // a row that sees nothing: out = 0, lse = -inf
  const float inv = m == -INF ? 0.0f : 1.0f / l;
  T* const out = at<T>(a.out, b, me.i, me.h);
  T* const rest = a.rest.p ? at<T>(a.rest, b, me.i, me.h) : nullptr;
#pragma unroll
  for (int d = 0; d < L::BLOCKS; ++d) {
    if (DIVIDED && d % S::WAVES != wave) continue;
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      float x[4], y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) { x[e] = o[d][r + e] * inv; y[e] = x[e] - (float)(T)x[e]; }
      store4(out, d * 32 + 2 * r + 4 * hi, a.D, x, a.out.aligned);
      if (rest) store4(rest, d * 32 + 2 * r + 4 * hi, a.D, y, a.rest.aligned);
    }
  }
  if (a.lse && first && hi == 0) a.lse[((int64_t)b * a.H + me.h) * a.N + me.i] = m == -INF ? -INF : (m + log2_(l)) * LN2;
}

template <class T, int DP, int MODE, bool DIVIDED>
static hipError_t forward_one(const Args& a, unsigned grid, hipStream_t stream) {
  typedef Shape<T, DP, DIVIDED> S;
  if constexpr (sizeof(T) == 2) {
    if (DIVIDED || a.rest.p) {
      gr_attention_kernel<T, DP, MODE, DIVIDED, true><<<dim3(grid), dim3(S::THREADS), S::LDS, stream>>>(a);
      return hipGetLastError();
    }
  }
  if constexpr (sizeof(T) == 4 || !DIVIDED) gr_attention_kernel<T, DP, MODE, DIVIDED, false><<<dim3(grid), dim3(S::THREADS), S::LDS, stream>>>(a);
  return hipGetLastError();
}
template <class T, int DP, bool DIVIDED>
static hipError_t forward_mode(const Args& a, int mode, unsigned grid, hipStream_t stream) {
  switch (mode) {
    case 0: return forward_one<T, DP, 0, DIVIDED>(a, grid, stream);
    case 1: return forward_one<T, DP, 1, DIVIDED>(a, grid, stream);
    case 2: return forward_one<T, DP, 2, DIVIDED>(a, grid, stream);
    case 3: return forward_one<T, DP, 3, DIVIDED>(a, grid, stream);
  }
  if constexpr (sizeof(T) == 2) return mode == 5 ? forward_one<T, DP, 5, DIVIDED>(a, grid, stream) : forward_one<T, DP, 7, DIVIDED>(a, grid, stream);
  return hipErrorInvalidValue;
}
template <class T>
static hipError_t forward_all(const Args& a, int dp, int mode, bool divided, unsigned grid, hipStream_t stream) {
  switch (dp) {
    case 64: return divided ? forward_mode<T, 64, true>(a, mode, grid, stream) : forward_mode<T, 64, false>(a, mode, grid, stream);
    case 96: return divided ? forward_mode<T, 96, true>(a, mode, grid, stream) : forward_mode<T, 96, false>(a, mode, grid, stream);
    case 128: return divided ? forward_mode<T, 128, true>(a, mode, grid, stream) : forward_mode<T, 128, false>(a, mode, grid, stream);
    default: return divided ? forward_mode<T, 256, true>(a, mode, grid, stream) : forward_mode<T, 256, false>(a, mode, grid, stream);
  }
}

}  // namespace attn
}  // namespace gr
