// The small kernels around attention: joining the splits of the keys, document ranges, the gradient's statistics of a row, summing the parts of dk and dv.
#include "attention_kernels.h"

namespace gr {
namespace attn {

// out and lse of a row from the splits' (m, l, sums): each scaled to the largest m, added in the order of the splits.  With more than 16 splits a
// workgroup has one row: its threads read the splits' (m, l) once, a split each, then 256 / quads runs of splits are summed side by side for every four
// values and joined in order.  (Threads that each walked all splits of four values took 68 us for 128 splits of 8 rows, a chain of 128 reads.)
// A split that saw nothing has m = -inf and counts for nothing; one that saw NaN has m = l = NaN, which a maximum passes over and every sum keeps:
// l = 0 is a row that saw nothing.
template <class T>
static __device__ __forceinline__ void finish_row(const Args& a, int64_t row, int d, const f32x4& x, float m, float l) {
  const int R = a.N * a.G;
  const int pair = (int)(row / R), r = (int)(row - (int64_t)pair * R), i = r / a.G, g = r - i * a.G, b = pair / a.HK, h = (pair - b * a.HK) * a.G + g;
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  float o[4], y[4];
  for (int e = 0; e < 4; ++e) { o[e] = x[e] * inv; y[e] = o[e] - (float)(T)o[e]; }
  store4(at<T>(a.out, b, i, h), d, a.D, o, a.out.aligned);
  if (a.rest.p) store4(at<T>(a.rest, b, i, h), d, a.D, y, a.rest.aligned);
  if (a.lse && d == 0) a.lse[((int64_t)b * a.H + h) * a.N + i] = l == 0.0f ? -INF : (m + log2_(l)) * LN2;
}

template <class T>
__global__ __launch_bounds__(256) void gr_attention_combine_few_kernel(const Args a, int dp) {
  const int quads = dp / 4;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, rows = (int64_t)a.B * a.HK * a.N * a.G;
  const int64_t row = id / quads;
  const int d = (int)(id - row * quads) * 4;
  if (row >= rows) return;
  float m = -INF, l = 0.0f;
#pragma unroll 8
  for (int s = 0; s < a.splits; ++s) m = __builtin_fmaxf(m, a.part_ml[2 * (s * rows + row)]);
  f32x4 x = (f32x4)0.0f;
#pragma unroll 8
  for (int s = 0; s < a.splits; ++s) {
    const float ms = a.part_ml[2 * (s * rows + row)], by = ms == -INF ? 0.0f : exp2_(ms - m);
    l = __builtin_fmaf(a.part_ml[2 * (s * rows + row) + 1], by, l);
    const f32x4 p = *(const f32x4*)(a.part_o + (s * rows + row) * dp + d);
    for (int e = 0; e < 4; ++e) x[e] = by == 0.0f ? x[e] : __builtin_fmaf(p[e], by, x[e]);
  }
  finish_row<T>(a, row, d, x, m, l);
}

template <class T>
__global__ __launch_bounds__(256) void gr_attention_combine_kernel(const Args a, int dp) {
  __shared__ float by_[MAX_SPLITS];
  __shared__ f32x4 sums[256];
  __shared__ float tops[4], totals[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, quads = dp / 4, R = a.N * a.G, pairs = a.B * a.HK;
  const int64_t rows = (int64_t)pairs * R, row = blockIdx.x;
  static_assert(MAX_SPLITS <= 256, "a split per thread");
  const bool have = tid < a.splits;
  const float ms = have ? a.part_ml[2 * (tid * rows + row)] : -INF, ls = have ? a.part_ml[2 * (tid * rows + row) + 1] : 0.0f;
  float m = ms;
  for (int x = 32; x; x >>= 1) m = __builtin_fmaxf(m, __shfl_xor(m, x));
  if (lane == 0) tops[wave] = m;
  __syncthreads();
  m = __builtin_fmaxf(__builtin_fmaxf(tops[0], tops[1]), __builtin_fmaxf(tops[2], tops[3]));
  const float by = ms == -INF ? 0.0f : exp2_(ms - m);
  if (have) by_[tid] = by;
  float l = ms == -INF ? 0.0f : ls * by;
  for (int x = 32; x; x >>= 1) l += __shfl_xor(l, x);
  if (lane == 0) totals[wave] = l;
  __syncthreads();
  l = (totals[0] + totals[1]) + (totals[2] + totals[3]);
  const int runs = 256 / quads, run = tid / quads, d = (tid - run * quads) * 4;
  f32x4 x = (f32x4)0.0f;
  if (run < runs) {
    const int per = (a.splits + runs - 1) / runs, s1 = min(a.splits, (run + 1) * per);
    const float* p = a.part_o + row * dp + d;
#pragma unroll 4
    for (int s = run * per; s < s1; ++s) {
      const float w = by_[s];
      const f32x4 v = *(const f32x4*)(p + (int64_t)s * rows * dp);
      // (a split that saw nothing: whatever its sums hold counts for nothing)
      for (int e = 0; e < 4; ++e) x[e] = w == 0.0f ? x[e] : __builtin_fmaf(v[e], w, x[e]);
    }
    sums[tid] = x;
  }
  __syncthreads();
  if (run != 0) return;
  for (int u = 1; u < runs; ++u) x += sums[u * quads + tid];
  finish_row<T>(a, row, d, x, m, l);
}

// Smallest and largest document number of 32 neighbours, half a wave each, and the numbers themselves side by side in rows of a multiple of
// 128: of the keys, then of the queries.
__global__ __launch_bounds__(256) void gr_attention_ranges_kernel(const Args a, int64_t key_pieces) {
  int64_t id = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 5;
  const bool keys = id < key_pieces;
  if (!keys) id -= key_pieces;
  const int N = keys ? a.M : a.N, pieces = (N + 31) / 32;
  if (id >= (int64_t)a.B * pieces) return;
  const int64_t sb = keys ? a.kdoc_sb : a.qdoc_sb, sn = keys ? a.kdoc_sn : a.qdoc_sn, np = padded_rows(N);
  const int* const docs = keys ? a.kdoc : a.qdoc;
  const int b = (int)(id / pieces), n = (int)(id - (int64_t)b * pieces) * 32 + (threadIdx.x & 31);
  int* const rows = (keys ? a.kdocs : a.qdocs) + b * np;
  int* const to = keys ? a.kranges : a.qranges;
  int lo = n < N ? docs[b * sb + n * sn] : 0x7fffffff, hi = n < N ? lo : -1;
  rows[n] = hi;
  for (int64_t r = n + 32; r >= (int64_t)pieces * 32 && r < np; r += 32) rows[r] = -1;
  for (int m = 16; m; m >>= 1) { lo = min(lo, __shfl_xor(lo, m)); hi = max(hi, __shfl_xor(hi, m)); }
  if ((threadIdx.x & 31) == 0) { to[2 * id] = lo; to[2 * id + 1] = hi; }
}

// less and delta of the gradient, 16 lanes a row of (batch, query, head).  delta = sum over d of dout (out + rest); rest is what the rounding of
// out to 16 bits lost: with it delta is that of the unrounded output, which matters for queries that see few keys, where dp - delta nearly
// cancels.  An lse of 2^28 and more is rounded by more than 2^4: it is taken a little larger, so that no probability passes 1 by so much
// that its lifted value could overflow.
template <class T>
__global__ __launch_bounds__(256) void gr_attention_statistics_kernel(const Args a) {
  const int64_t np = padded_rows(a.N), id = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 4, rows = a.B * np * a.H;
  if (id >= rows) return;   // (16 lanes leave together)
  const int part = threadIdx.x & 15;
  const int h = (int)(id % a.H);
  const int64_t bn = id / a.H;
  const int i = (int)(bn % np), b = (int)(bn / np);
  const int64_t to = ((int64_t)b * a.H + h) * np + i;
  if (i >= a.N) {
    if (part == 0) { a.less[to] = INF; a.delta[to] = 0.0f; }
    return;
  }
  const T* o = at<T>(a.out, b, i, h);
  const T* r = a.rest.p ? at<T>(a.rest, b, i, h) : nullptr;
  const T* g = at<T>(a.dout, b, i, h);
  float x = 0.0f;
  constexpr int V = 16 / (int)sizeof(T);
  if (a.out.aligned && a.dout.aligned && (!r || a.rest.aligned)) {
    typedef T vec __attribute__((ext_vector_type(V)));
    for (int d = part * V; d < a.D; d += 16 * V) {
      const vec ov = *(const vec*)(o + d), gv = *(const vec*)(g + d), rv = r ? *(const vec*)(r + d) : (vec)(T)0.0f;
      for (int e = 0; e < V; ++e) x = __builtin_fmaf((float)gv[e], (float)ov[e] + (float)rv[e], x);
    }
  } else {
    for (int d = part; d < a.D; d += 16) x = __builtin_fmaf((float)g[d], (float)o[d] + (r ? (float)r[d] : 0.0f), x);
  }
  for (int m = 8; m; m >>= 1) x += __shfl_xor(x, m);
  if (part != 0) return;
  const float e = a.lse[((int64_t)b * a.H + h) * a.N + i];
  float less = e == -INF ? INF : sizeof(T) == 4 ? e * LOG2E : e * LOG2E - LIFT;
  const float size = __builtin_fabsf(less);
  if (size >= 0x1p28f && size < INF) less += size * 0x1p-22f;
  a.less[to] = sizeof(T) == 4 ? 0.5f * less : less;   // (see EXPONENT in attention_backward.h)
  a.delta[to] = x;
}

// dq (WHICH = 0), or dk and dv (1), from the parts of the splits, in the order of the splits.  A thread has four values of a row.
template <class T, int WHICH>
__global__ __launch_bounds__(256) void gr_attention_sum_parts_kernel(const Args a, int dp) {
  const int quads = dp / 4, each = WHICH == 0 ? a.N * a.G : a.M;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, rows = (int64_t)a.B * a.HK * each, plane = rows * dp;
  const int64_t row = id / quads;
  const int d = (int)(id - row * quads) * 4;
  if (row >= rows) return;
  const float* const p = a.part_o + row * dp + d;
  const float by = a.scale * UNLIFT;
  const int64_t pair = row / each, n = row - pair * each, b = pair / a.HK, hk = pair - b * a.HK;
  f32x4 x = (f32x4)0.0f, y = (f32x4)0.0f;
  if constexpr (WHICH == 0) {
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s) x += *(const f32x4*)(p + s * plane);
    const float q[4] = {x[0] * by, x[1] * by, x[2] * by, x[3] * by};
    const int64_t i = n / a.G;
    store4(at<T>(a.dq, b, i, hk * a.G + (n - i * a.G)), d, a.D, q, a.dq.aligned);
  } else {
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s) {
      x += *(const f32x4*)(p + 2 * s * plane);
      y += *(const f32x4*)(p + (2 * s + 1) * plane);
    }
    const float k[4] = {x[0] * by, x[1] * by, x[2] * by, x[3] * by}, v[4] = {y[0] * UNLIFT, y[1] * UNLIFT, y[2] * UNLIFT, y[3] * UNLIFT};
    store4(at<T>(a.dk, b, n, hk), d, a.D, k, a.dk.aligned);
    store4(at<T>(a.dv, b, n, hk), d, a.D, v, a.dv.aligned);
  }
}

static dim3 blocks_of(int64_t threads) { return dim3((unsigned)((threads + 255) / 256)); }

hipError_t combine(const Args& a, int type, int dp, hipStream_t stream) {
  const int64_t rows = (int64_t)a.B * a.HK * a.N * a.G;
  if (a.splits <= 16) {
    const dim3 grid = blocks_of(rows * (dp / 4));
    if (type == TYPE_BF16) gr_attention_combine_few_kernel<__bf16><<<grid, dim3(256), 0, stream>>>(a, dp);
    else gr_attention_combine_few_kernel<float><<<grid, dim3(256), 0, stream>>>(a, dp);
  } else {
    const dim3 grid((unsigned)rows);
    if (type == TYPE_BF16) gr_attention_combine_kernel<__bf16><<<grid, dim3(256), 0, stream>>>(a, dp);
    else gr_attention_combine_kernel<float><<<grid, dim3(256), 0, stream>>>(a, dp);
  }
  return hipGetLastError();
}

hipError_t ranges(const Args& a, hipStream_t stream) {
  const int64_t keys = (int64_t)a.B * ((a.M + 31) / 32), queries = (int64_t)a.B * ((a.N + 31) / 32);
  gr_attention_ranges_kernel<<<blocks_of((keys + queries) * 32), dim3(256), 0, stream>>>(a, keys);
  return hipGetLastError();
}

hipError_t statistics(const Args& a, int type, hipStream_t stream) {
  const dim3 grid = blocks_of(a.B * padded_rows(a.N) * a.H * 16);
  if (type == TYPE_BF16) gr_attention_statistics_kernel<__bf16><<<grid, dim3(256), 0, stream>>>(a);
  else gr_attention_statistics_kernel<float><<<grid, dim3(256), 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t sum_parts(const Args& a, int type, int dp, bool queries, hipStream_t stream) {
  const dim3 grid = blocks_of((int64_t)a.B * a.HK * (queries ? (int64_t)a.N * a.G : a.M) * (dp / 4));
  if (type == TYPE_BF16) {
    if (queries) gr_attention_sum_parts_kernel<__bf16, 0><<<grid, dim3(256), 0, stream>>>(a, dp);
    else gr_attention_sum_parts_kernel<__bf16, 1><<<grid, dim3(256), 0, stream>>>(a, dp);
  } else {
    if (queries) gr_attention_sum_parts_kernel<float, 0><<<grid, dim3(256), 0, stream>>>(a, dp);
    else gr_attention_sum_parts_kernel<float, 1><<<grid, dim3(256), 0, stream>>>(a, dp);
  }
  return hipGetLastError();
}

}  // namespace attn
}  // namespace gr
