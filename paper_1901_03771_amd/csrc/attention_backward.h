// The gradient of attention.  With p = exp(score - lse), t the tanh of a capped score and delta = sum over d of dout * out:
//   dv = p^T dout,   dp = dout v^T,   ds = p (dp - delta) (1 - t^2) scale,   dq = ds k,   dk = ds^T q.
// p is formed again from q, k and lse.  Two kernels, so that every sum stays in registers of one workgroup and its order is fixed
// (no atomic additions, the same bits from call to call):
//   gr_attention_grad_q   walks the keys for 128 rows of queries, as the forward kernel does;
//   gr_attention_grad_kv  walks the queries of all heads that share a head of k and v for a block of keys.
// Probabilities are carried 2^32 times as large (UNLIFT takes it out of the sums in the end), so that those below float32's normal numbers
// still count in the gradients of keys that every query all but ignores; there is room for it above.  With bfloat16 tensors LIFT stands in the
// exponent, which rounds it like a number near 32: 2^-20 of a probability that is rounded to 2^-8 next.  For float32 that would be the largest error of
// all (a pass over 777 rows of 80 values 7.2e-7 from binary64 where a plain one is at 4.2e-7): there the kernels form e = 2^(half the exponent), which never
// leaves the normal numbers, and the probability as (2^32 e) e.
// They form q k^T and dout v^T twice, 7 products of the size of q k^T where a single kernel would have 5 and an addition to dq in memory
// per tile.
//
// Measured, bfloat16, 16 heads of 8192 causal rows of 128 values, a beginning seen whole: dq 0.45 ms (matrix cores busy 53 % of the cycles), dk and dv 0.73 ms (42 %, waiting 49 %: operands of
// both sides and both sums fill 256 registers a lane, nothing is read ahead from LDS).
#pragma once

#include "attention_kernels.h"

namespace gr {
namespace attn {

// Of exponents, and what stands for them (less, c, slopes): the whole for bfloat16, the half for float32.
template <class T> constexpr float EXPONENT = sizeof(T) == 4 ? 0.5f : 1.0f;
template <class T>
static __device__ __forceinline__ float lifted(float x) {
  const float e = exp2_(x);
  if constexpr (sizeof(T) == 4) return (e * 0x1p32f) * e;
  else return e;
}

template <class T, int DP>
struct ShapeQ {
  static constexpr int THREADS = 256, KEYS = tile_rows(sizeof(T), DP), ROWS = 128, TILE = KEYS * Tile<T, DP>::ROW;
  static constexpr int LDS = 4 * TILE + 2 * KEYS * 4;   // two stages of k and v, two stages of the keys' documents
  static constexpr int REGS = DP / 16 * (sizeof(T) == 2 ? 8 : 24) + DP / 2 + 32;   // operands of q and dout, sums, two blocks of scores
  static constexpr bool TIGHT = REGS > (sizeof(T) == 2 ? 160 : 128);   // of registers: addresses within tiles are formed anew for each tile
  static constexpr int PER_CU = grad_q_per_cu(sizeof(T), DP);
  static_assert(PER_CU * LDS <= 160 * 1024, "LDS of a compute unit");
};

template <class T, int DP, int MODE>
__global__ __launch_bounds__(256, (ShapeQ<T, DP>::PER_CU)) void gr_attention_grad_q_kernel(const Args a) {
  typedef ShapeQ<T, DP> S;
  typedef Tile<T, DP> L;
  typedef typename Frag<T>::type F;
  extern __shared__ char smem_[];
  GR_LDS char* const smem = (GR_LDS char*)smem_;
  GR_LDS int* const documents = (GR_LDS int*)(smem + 4 * S::TILE);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, hi = lane >> 5;
  const int pairs = a.B * a.HK;
  const Place place = place_of(blockIdx.x, pairs, a.blocks * a.splits);
  if (place.block >= a.blocks * a.splits) return;
  const int split = place.block % a.splits, rb = a.blocks - 1 - place.block / a.splits;
  const int b = place.pair / a.HK, hk = place.pair - b * a.HK;
  const int R = a.N * a.G, row0 = rb * S::ROWS, wrow0 = row0 + wave * 32;
  const int len = length_of(a, b), pre = a.prefix ? scalar(a.prefix, b * a.prefix_s) : 0;
  const Row mine = row_of(a, hk, wrow0 + col);   // (not kept beyond the operands: registers are full)
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

  F qf[L::STEPS], df[L::STEPS];
  {
    const T* q = at<T>(a.q, b, mine.i, mine.h);
    const T* d = at<T>(a.dout, b, mine.i, mine.h);
#pragma unroll
    for (int s = 0; s < L::STEPS; ++s) { qf[s] = L::fetch(q, s, hi, a.D, mine.valid, a.q.aligned); df[s] = L::fetch(d, s, hi, a.D, mine.valid, a.dout.aligned); }
  }
  const int64_t stat = ((int64_t)b * a.H + mine.h) * padded_rows(a.N) + mine.i;
  float less = mine.valid ? a.less[stat] : INF, delta = mine.valid ? a.delta[stat] : 0.0f;
  float slope = MODE & MODE_BIAS ? a.slopes[mine.h * a.slopes_s] * (LOG2E * EXPONENT<T>) : 0.0f;
  const int64_t pos = MODE & MODE_BIAS ? a.position + mine.i : 0;

  f32x16 o[L::BLOCKS];
#pragma unroll
  for (int d = 0; d < L::BLOCKS; ++d) o[d] = (f32x16)0.0f;

  const int most = (end + S::KEYS - 1) / S::KEYS, per = (most + a.splits - 1) / a.splits, tiles = min(most, (split + 1) * per);
  const T* const kbase = at<T>(a.k, b, 0, hk);
  const T* const vbase = at<T>(a.v, b, 0, hk);
  auto load = [&](int t, int stage) {
    const int64_t k0 = (int64_t)t * S::KEYS;
    const int rows = min(S::KEYS, len - (int)k0);
    L::template load<S::KEYS, 256>(smem + 2 * stage * S::TILE, kbase + k0 * a.k.sn, a.k.sn, rows, a.D, S::TIGHT ? fresh(tid) : tid, a.k.direct);
    L::template load<S::KEYS, 256>(smem + (2 * stage + 1) * S::TILE, vbase + k0 * a.v.sn, a.v.sn, rows, a.D, S::TIGHT ? fresh(tid) : tid, a.v.direct);
    if (a.kdoc && wave == 0) load_words((GR_LDS float*)(documents + stage * S::KEYS), a.kdocs + b * padded_rows(a.M) + k0, lane, S::KEYS);
  };
  int t = find.next(split * per, tiles, lane), stage = 0;
  if (t < tiles) load(t, 0);
  loaded(qf);
  loaded(df);
  loaded(less);
  loaded(delta);
  if constexpr (MODE & MODE_BIAS) loaded(slope);
  while (t < tiles) {
    const int after = find.next(t + 1, tiles, lane);
    arrive();
    if (after < tiles) load(after, stage ^ 1);
    const GR_LDS char* const kt = smem + 2 * stage * S::TILE;
    const GR_LDS char* const vt = kt + S::TILE;
#pragma unroll 1
    for (int kb = 0; kb < S::KEYS / 32; ++kb) {
      const int key0 = t * S::KEYS + kb * 32;
      if (key0 >= w_last) break;
      bool whole = key0 + 32 <= w_first, one = true;
      if (ranges) {
        one = w.one & (scalar(ranges, 2 * (key0 / 32)) == w.hi) & (scalar(ranges, 2 * (key0 / 32) + 1) == w.hi);
        whole = whole && one;
      }
      const int tcol = S::TIGHT ? fresh(col) : col, tlane = S::TIGHT ? fresh(lane) : lane;
      f32x16 s = (f32x16)0.0f, dp = (f32x16)0.0f;
#pragma unroll
      for (int st = 0; st < L::STEPS; ++st) {
        if constexpr (DP == 256) { anew(qf[st]); anew(df[st]); }
        s = mma(L::row(kt, kb * 32 + tcol, st, hi), qf[st], s);
        dp = mma(L::row(vt, kb * 32 + tcol, st, hi), df[st], dp);
      }
      finished(s, dp);
      const float away = MODE & MODE_BIAS ? (float)(pos - key0 - 4 * (tlane >> 5)) : 0.0f;   // from the first key of this half
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        float y = s[r], bend = 1.0f;
        if constexpr (MODE & MODE_CAP) { y = capped<T, MODE>(y, a.cin); bend = __builtin_fmaf(-y, y, 1.0f); }
        if constexpr (MODE & MODE_BIAS) y = __builtin_fmaf(y, a.c, __builtin_fmaf(-slope, __builtin_fabsf(away - (float)((r & 3) + 8 * (r >> 2))), -less));
        else y = __builtin_fmaf(y, a.c, -less);
        s[r] = y;
        dp[r] -= delta;
        if constexpr (MODE & MODE_CAP) dp[r] *= bend;
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = lifted<T>(s[r]) * dp[r];
      if (!whole) {
        const int flane = fresh(lane);
        const Row me = row_of(a, hk, wrow0 + (flane & 31));
        const int see = (me.valid ? keys_seen(a, me.i, len, pre) : 0) - key0 - 4 * (flane >> 5);
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = (r & 3) + 8 * (r >> 2) < see ? s[r] : 0.0f;
        if (!one) {
          const int doc = me.valid ? a.qdocs[b * padded_rows(a.N) + me.i] : -1;
          const GR_LDS int* const kd = documents + stage * S::KEYS + kb * 32 + 4 * (flane >> 5);
#pragma unroll
          for (int r4 = 0; r4 < 4; ++r4) {
            const i32x4 n = *(const GR_LDS i32x4*)(kd + 8 * r4);
#pragma unroll
            for (int e = 0; e < 4; ++e) s[4 * r4 + e] = (n[e] == doc) & (doc >= 0) ? s[4 * r4 + e] : 0.0f;
          }
        }
      }
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        F f;
        operand(s, st, f);
#pragma unroll
        for (int d = 0; d < L::BLOCKS; ++d) o[d] = mma(L::column(kt, kb * 32 + st * 16, d, tlane), f, o[d]);
      }
    }
    t = after;
    stage ^= 1;
  }
  finished(o);
  const Row me = row_of(a, hk, wrow0 + col);
  if (!me.valid) return;
  if (a.splits > 1) {
    // (splits, B * HK, N * G, DP)
    float* const to = a.part_o + (((int64_t)split * pairs + place.pair) * R + wrow0 + col) * DP;
#pragma unroll
    for (int d = 0; d < L::BLOCKS; ++d)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const f32x4 x = {o[d][r], o[d][r + 1], o[d][r + 2], o[d][r + 3]};
        *(f32x4*)(to + d * 32 + 2 * r + 4 * hi) = x;
      }
    return;
  }
  T* const dq = at<T>(a.dq, b, me.i, me.h);
#pragma unroll
  for (int d = 0; d < L::BLOCKS; ++d)
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      const float by = a.scale * UNLIFT, x[4] = {o[d][r] * by, o[d][r + 1] * by, o[d][r + 2] * by, o[d][r + 3] * by};
      store4(dq, d * 32 + 2 * r + 4 * hi, a.D, x, a.dq.aligned);
    }
}

// Which of dk and dv a launch forms: both, or, where the operands and sums of both do not fit a lane's registers, one each.
enum { BOTH = 0, ONLY_V = 1, ONLY_K = 2 };

template <class T, int DP, int WHICH>
struct ShapeKV {
  static constexpr int ROWS = tile_rows(sizeof(T), DP), KEYS = 128, TILE = ROWS * Tile<T, DP>::ROW;   // rows: of a tile of queries
  static constexpr int STATS = 4 * ROWS;                     // less, delta and document of every row
  static constexpr int LDS = 4 * TILE + 2 * STATS * 4;       // two stages of q and dout, and of these
  static constexpr int PER_CU = WHICH == ONLY_V && sizeof(T) == 2 ? 2 : grad_kv_per_cu(sizeof(T), DP);
  static_assert(PER_CU * LDS <= 160 * 1024, "LDS of a compute unit");
};

template <class T, int DP, int MODE, int WHICH>
__global__ __launch_bounds__(256, (ShapeKV<T, DP, WHICH>::PER_CU)) void gr_attention_grad_kv_kernel(const Args a) {
  typedef ShapeKV<T, DP, WHICH> S;
  typedef Tile<T, DP> L;
  typedef typename Frag<T>::type F;
  constexpr bool WANT_K = WHICH != ONLY_V, WANT_V = WHICH != ONLY_K;
  extern __shared__ char smem_[];
  GR_LDS char* const smem = (GR_LDS char*)smem_;
  GR_LDS float* const stats = (GR_LDS float*)(smem + 4 * S::TILE);   // [stage][less, delta, document][row]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, hi = lane >> 5;
  const int pairs = a.B * a.HK;
  const Place place = place_of(blockIdx.x, pairs, a.blocks * a.splits);
  if (place.block >= a.blocks * a.splits) return;
  const int split = place.block % a.splits, kblock = place.block / a.splits;   // the first keys are seen by the most queries
  const int b = place.pair / a.HK, hk = place.pair - b * a.HK;
  const int len = length_of(a, b), pre = a.prefix ? scalar(a.prefix, b * a.prefix_s) : 0;
  const int block0 = kblock * S::KEYS, key0 = block0 + wave * 32, key = key0 + col;
  const bool valid = key < len;

  int lo = 0, up = 0, w_doc = -1;
  bool w_one = false;
  const int kpieces = (a.M + 31) / 32, qpieces = (a.N + 31) / 32;
  if (a.kdoc) {
    lo = 0x7fffffff; up = -1;
    const int* kr = a.kranges + (int64_t)b * kpieces * 2;
    for (int e = block0 / 32; e < block0 / 32 + 4 && e < kpieces; ++e) {
      // (numbers below zero belong to no document; a piece of nothing else has no largest)
      const int all = scalar(kr, 2 * e), l = all < 0 ? 0 : all, u = scalar(kr, 2 * e + 1);
      if (u >= 0) { lo = min(lo, l); up = max(up, u); }
      if (e == key0 / 32) { w_one = all == u && u >= 0; w_doc = u; }
    }
  }
  const int* const ranges = a.kdoc ? a.qranges + (int64_t)b * qpieces * 2 : nullptr;

  F kf[L::STEPS], vf[WANT_K ? L::STEPS : 1];
  {
    const T* k = at<T>(a.k, b, valid ? key : 0, hk);
    const T* v = at<T>(a.v, b, valid ? key : 0, hk);
#pragma unroll
    for (int s = 0; s < L::STEPS; ++s) {
      kf[s] = L::fetch(k, s, hi, a.D, valid, a.k.aligned);
      if constexpr (WANT_K) vf[s] = L::fetch(v, s, hi, a.D, valid, a.v.aligned);
    }
  }
  f32x16 ok[WANT_K ? L::BLOCKS : 1], ov[WANT_V ? L::BLOCKS : 1];
#pragma unroll
  for (int d = 0; d < L::BLOCKS; ++d) {
    if constexpr (WANT_K) ok[d] = (f32x16)0.0f;
    if constexpr (WANT_V) ov[d] = (f32x16)0.0f;
  }

  // The queries that see a key of the block: all from the first one that does, since what a query sees grows with its place.
  int first = 0;
  if (block0 >= len) first = a.N;
  else if (a.causal && block0 >= pre) first = min(first_seeing(a, block0), a.N);
  const int t0 = first / S::ROWS, tiles = (a.N + S::ROWS - 1) / S::ROWS, span = first < a.N ? tiles - t0 : 0;
  // units: tiles of the first head, of the second, ..; a split takes a run of them
  const int64_t units = (int64_t)span * a.G;
  const int u0 = (int)(units * split / a.splits), u1 = (int)(units * (split + 1) / a.splits);
  struct Unit { int u, g, t; };   // running number, head of the group, tile
  Finder<S::ROWS / 32> find{ranges, qpieces, lo, up};
  // the unit at or after x that has something to do
  auto next = [&](Unit x) {
    while (x.u < u1) {
      if (x.t >= tiles) { x.t = t0; ++x.g; }
      const int n = find.next(x.t, tiles, lane);
      x.u += n - x.t;
      x.t = n;
      if (n < tiles) return x;
    }
    return x;
  };
  auto load = [&](const Unit& x, int stage) {
    const int t = x.t, h = hk * a.G + x.g;
    const int64_t i0 = (int64_t)t * S::ROWS;
    const int rows = min(S::ROWS, a.N - (int)i0);
    L::template load<S::ROWS, 256>(smem + 2 * stage * S::TILE, at<T>(a.q, b, i0, h), a.q.sn, rows, a.D, fresh(tid), a.q.direct);
    L::template load<S::ROWS, 256>(smem + (2 * stage + 1) * S::TILE, at<T>(a.dout, b, i0, h), a.dout.sn, rows, a.D, fresh(tid), a.dout.direct);
    // (a tile's rows behind the last are there: +inf, 0, -1)
    const int64_t np = padded_rows(a.N), stat = ((int64_t)b * a.H + h) * np + i0;
    GR_LDS float* const to = stats + stage * S::STATS;
    if (wave == 0) load_words(to, a.less + stat, lane, S::ROWS);
    else if (wave == 1) load_words(to + S::ROWS, a.delta + stat, lane, S::ROWS);
    else if (wave == 2 && a.kdoc) load_words(to + 2 * S::ROWS, a.qdocs + b * np + i0, lane, S::ROWS);
  };
  Unit now{u0, span > 0 ? u0 / span : 0, 0};
  now.t = t0 + (u0 - now.g * span);
  now = next(now);
  int stage = 0;
  if (now.u < u1) load(now, 0);
  loaded(kf);
  if constexpr (WANT_K) loaded(vf);
  while (now.u < u1) {
    const Unit after = next({now.u + 1, now.g, now.t + 1});
    arrive();
    if (after.u < u1) load(after, stage ^ 1);
    const int t = now.t, h = hk * a.G + now.g;
    const GR_LDS char* const qt = smem + 2 * stage * S::TILE;
    const GR_LDS char* const dt = qt + S::TILE;
    const GR_LDS float* const st = stats + stage * S::STATS;
    const float slope = MODE & MODE_BIAS ? scalar_float(a.slopes, h * a.slopes_s) * (LOG2E * EXPONENT<T>) : 0.0f;
    
#pragma unroll 1
    for (int rb = 0; rb < S::ROWS / 32; ++rb) {
      const int i0 = t * S::ROWS + rb * 32;
      if (i0 >= a.N) break;
      const int see_last = keys_seen(a, min(i0 + 31, a.N - 1), len, pre);
      if (see_last <= key0) continue;
      // from this lane's key to the tile's first query
      const float away = MODE & MODE_BIAS ? (float)(a.position + t * S::ROWS - key0 - (fresh(tid) & 31)) : 0.0f;
      // (registers are full: what depends on the lane is formed here)
      const int flane = fresh(tid) & 63, fcol = flane & 31, fhi = flane >> 5;
      // (rows behind the last query need no mask: their lse is none)
      bool whole = keys_seen(a, i0, len, pre) >= key0 + 32, one = true;
      if (ranges) {
        one = w_one & (scalar(ranges, 2 * (i0 / 32)) == w_doc) & (scalar(ranges, 2 * (i0 / 32) + 1) == w_doc);
        whole = whole && one;
      }
      f32x16 s = (f32x16)0.0f, dp = (f32x16)0.0f;
#pragma unroll
      for (int x = 0; x < L::STEPS; ++x) {
        if constexpr (DP == 256) { anew(kf[x]); if constexpr (WANT_K) anew(vf[x]); }
        s = mma(L::row(qt, rb * 32 + fcol, x, fhi), kf[x], s);
        if constexpr (WANT_K) dp = mma(L::row(dt, rb * 32 + fcol, x, fhi), vf[x], dp);
      }
      if constexpr (WANT_K) finished(s, dp);
      else finished(s);
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        const int rr = rb * 32 + 8 * r4 + 4 * fhi;
        const f32x4 less = *(const GR_LDS f32x4*)(st + rr), delta = *(const GR_LDS f32x4*)(st + S::ROWS + rr);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = 4 * r4 + e;
          float y = s[r], bend = 1.0f;
          if constexpr (MODE & MODE_CAP) { y = capped<T, MODE>(y, a.cin); bend = __builtin_fmaf(-y, y, 1.0f); }
          if constexpr (MODE & MODE_BIAS) y = __builtin_fmaf(y, a.c, __builtin_fmaf(-slope, __builtin_fabsf(away + (float)(rr + e)), -less[e]));
          else y = __builtin_fmaf(y, a.c, -less[e]);
          s[r] = lifted<T>(y);
          if constexpr (WANT_K) {
            dp[r] = s[r] * (dp[r] - delta[e]);
            if constexpr (MODE & MODE_CAP) dp[r] *= bend;
          }
        }
      }
      if (!whole) {
        // the first query that sees this lane's key
        const int key = key0 + fcol, i = i0 + 4 * fhi;
        int from = a.causal && key >= pre ? first_seeing(a, key) : 0;
        from = key < len ? from : 0x7fffffff;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const bool seen = i + (r & 3) + 8 * (r >> 2) >= from;
          s[r] = seen ? s[r] : 0.0f;
          if constexpr (WANT_K) dp[r] = seen ? dp[r] : 0.0f;
        }
        if (!one) {
          const int doc = key < a.M ? a.kdocs[b * padded_rows(a.M) + key] : -1;
#pragma unroll
          for (int r4 = 0; r4 < 4; ++r4) {
            const i32x4 docs = *(const GR_LDS i32x4*)(st + 2 * S::ROWS + rb * 32 + 8 * r4 + 4 * fhi);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const bool seen = (docs[e] == doc) & (doc >= 0);
              s[4 * r4 + e] = seen ? s[4 * r4 + e] : 0.0f;
              if constexpr (WANT_K) dp[4 * r4 + e] = seen ? dp[4 * r4 + e] : 0.0f;
            }
          }
        }
      }
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        F f;
        if constexpr (WANT_V) {
          operand(s, x, f);
#pragma unroll
          for (int d = 0; d < L::BLOCKS; ++d) ov[d] = mma(L::column(dt, rb * 32 + x * 16, d, flane), f, ov[d]);
        }
        if constexpr (WANT_K) {
          operand(dp, x, f);
#pragma unroll
          for (int d = 0; d < L::BLOCKS; ++d) ok[d] = mma(L::column(qt, rb * 32 + x * 16, d, flane), f, ok[d]);
        }
      }
    }
    now = after;
    stage ^= 1;
  }
  if constexpr (WANT_K) finished(ok);
  if constexpr (WANT_V) finished(ov);
  const int lane_ = fresh(tid) & 63, key_ = key0 + (lane_ & 31), hi_ = lane_ >> 5;
  if (key_ >= a.M) return;
  if (a.splits > 1) {
    // (splits, 2, B * HK, M, DP)
    const int64_t plane = (int64_t)pairs * a.M * DP, to = ((int64_t)place.pair * a.M + key_) * DP + 2 * split * plane;
#pragma unroll
    for (int d = 0; d < L::BLOCKS; ++d)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const int n = d * 32 + 2 * r + 4 * hi_;
        if constexpr (WANT_K) { const f32x4 x = {ok[d][r], ok[d][r + 1], ok[d][r + 2], ok[d][r + 3]}; *(f32x4*)(a.part_o + to + n) = x; }
        if constexpr (WANT_V) { const f32x4 x = {ov[d][r], ov[d][r + 1], ov[d][r + 2], ov[d][r + 3]}; *(f32x4*)(a.part_o + plane + to + n) = x; }
      }
    return;
  }
#pragma unroll
  for (int d = 0; d < L::BLOCKS; ++d)
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      const int n = d * 32 + 2 * r + 4 * hi_;
      if constexpr (WANT_K) {
        const float by = a.scale * UNLIFT, x[4] = {ok[d][r] * by, ok[d][r + 1] * by, ok[d][r + 2] * by, ok[d][r + 3] * by};
        store4(at<T>(a.dk, b, key_, hk), n, a.D, x, a.dk.aligned);
      }
      if constexpr (WANT_V) {
        const float x[4] = {ov[d][r] * UNLIFT, ov[d][r + 1] * UNLIFT, ov[d][r + 2] * UNLIFT, ov[d][r + 3] * UNLIFT};
        store4(at<T>(a.dv, b, key_, hk), n, a.D, x, a.dv.aligned);
      }
    }
}

template <class T, int DP, int MODE>
static hipError_t grad_q_one(const Args& a, unsigned grid, hipStream_t stream) {
  gr_attention_grad_q_kernel<T, DP, MODE><<<dim3(grid), dim3(256), ShapeQ<T, DP>::LDS, stream>>>(a);
  return hipGetLastError();
}
template <class T, int DP, int MODE, int WHICH>
static hipError_t grad_kv_part(const Args& a, unsigned grid, hipStream_t stream) {
  gr_attention_grad_kv_kernel<T, DP, MODE, WHICH><<<dim3(grid), dim3(256), ShapeKV<T, DP, WHICH>::LDS, stream>>>(a);
  return hipGetLastError();
}
template <class T, int DP, int MODE>
static hipError_t grad_kv_one(const Args& a, unsigned grid, hipStream_t stream) {
  if constexpr (DP == 256) {
    const hipError_t e = grad_kv_part<T, DP, MODE, ONLY_V>(a, grid, stream);
    return e != hipSuccess ? e : grad_kv_part<T, DP, MODE, ONLY_K>(a, grid, stream);
  } else {
    return grad_kv_part<T, DP, MODE, BOTH>(a, grid, stream);
  }
}

#define GR_BY_MODE(F, DP)                                                                                         \
  switch (mode) {                                                                                                 \
    case 0: return F<T, DP, 0>(a, grid, stream); case 1: return F<T, DP, 1>(a, grid, stream);                     \
    case 2: return F<T, DP, 2>(a, grid, stream); case 3: return F<T, DP, 3>(a, grid, stream);                     \
  }                                                                                                               \
  if constexpr (sizeof(T) == 2) return mode == 5 ? F<T, DP, 5>(a, grid, stream) : F<T, DP, 7>(a, grid, stream);   \
  return hipErrorInvalidValue;
#define GR_BY_SHAPE(F)                                                                                            \
  switch (dp) {                                                                                                   \
    case 64: { GR_BY_MODE(F, 64) } case 96: { GR_BY_MODE(F, 96) }                                                 \
    case 128: { GR_BY_MODE(F, 128) } default: { GR_BY_MODE(F, 256) }                                              \
  }
template <class T>
static hipError_t grad_q_all(const Args& a, int dp, int mode, unsigned grid, hipStream_t stream) { GR_BY_SHAPE(grad_q_one) }
template <class T>
static hipError_t grad_kv_all(const Args& a, int dp, int mode, unsigned grid, hipStream_t stream) { GR_BY_SHAPE(grad_kv_one) }
#undef GR_BY_MODE
#undef GR_BY_SHAPE

}  // namespace attn
}  // namespace gr
