// The small kernels around attention: joining the splits of the keys, document ranges, delta, summing the parts of dk and dv.
#include "attention_kernels.h"

namespace gr {
namespace attn {

// out and lse of a row from the splits' (m, l, sums): each scaled to the largest m, added in the order of the splits.  A thread has four
// values of a row.
template <class T>
__global__ __launch_bounds__(256) void gr_attention_combine_kernel(const Args a, int dp) {
  const int quads = dp / 4, R = a.N * a.G, pairs = a.B * a.HK;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, rows = (int64_t)pairs * R;
  const int64_t row = id / quads;
  const int d = (int)(id - row * quads) * 4;
  if (row >= rows) return;
  float m = -INF, l = 0.0f;
  for (int s = 0; s < a.splits; ++s) m = __builtin_fmaxf(m, a.part_ml[2 * (s * rows + row)]);
  f32x4 x = (f32x4)0.0f;
  for (int s = 0; s < a.splits; ++s) {
    const float ms = a.part_ml[2 * (s * rows + row)], by = ms == -INF ? 0.0f : exp2_(ms - m);
    l = __builtin_fmaf(a.part_ml[2 * (s * rows + row) + 1], by, l);
    const f32x4 p = *(const f32x4*)(a.part_o + (s * rows + row) * dp + d);
    if (ms != -INF) for (int e = 0; e < 4; ++e) x[e] = __builtin_fmaf(p[e], by, x[e]);
  }
  const int pair = (int)(row / R), r = (int)(row - (int64_t)pair * R), i = r / a.G, g = r - i * a.G, b = pair / a.HK, h = (pair - b * a.HK) * a.G + g;
  const float inv = m == -INF ? 0.0f : 1.0f / l;
  float o[4], y[4];
  for (int e = 0; e < 4; ++e) { o[e] = x[e] * inv; y[e] = o[e] - (float)(T)o[e]; }
  store4(at<T>(a.out, b, i, h), d, a.D, o, a.out.aligned);
  if (a.rest.p) store4(at<T>(a.rest, b, i, h), d, a.D, y, a.rest.aligned);
  if (a.lse && d == 0) a.lse[((int64_t)b * a.H + h) * a.N + i] = m == -INF ? -INF : (m + log2_(l)) * LN2;
}

// Smallest and largest document number of 32 neighbours: half a wave each.
__global__ __launch_bounds__(256) void gr_attention_ranges_kernel(const int* docs, int64_t sb, int64_t sn, int B, int N, int* to) {
  const int pieces = (N + 31) / 32;
  const int64_t id = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 5;
  if (id >= (int64_t)B * pieces) return;
  const int b = (int)(id / pieces), n = (int)(id - (int64_t)b * pieces) * 32 + (threadIdx.x & 31);
  int lo = n < N ? docs[b * sb + n * sn] : 0x7fffffff, hi = n < N ? lo : -1;
  for (int m = 16; m; m >>= 1) { lo = min(lo, __shfl_xor(lo, m)); hi = max(hi, __shfl_xor(hi, m)); }
  if ((threadIdx.x & 31) == 0) { to[2 * id] = lo; to[2 * id + 1] = hi; }
}

// delta = sum over d of dout (out + rest), 16 lanes a row of (batch, query, head).  rest is what the rounding of out to 16 bits lost:
// with it delta is that of the unrounded output, which matters for queries that see few keys, where dp - delta nearly cancels.
template <class T>
__global__ __launch_bounds__(256) void gr_attention_delta_kernel(const Args a, float* to) {
  const int64_t id = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 4, rows = (int64_t)a.B * a.N * a.H;
  if (id >= rows) return;   // (16 lanes leave together)
  const int part = threadIdx.x & 15;
  const int h = (int)(id % a.H);
  const int64_t bn = id / a.H;
  const int i = (int)(bn % a.N), b = (int)(bn / a.N);
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
  if (part == 0) to[((int64_t)b * a.H + h) * a.N + i] = x;
}

// dk and dv from the parts of the splits of the queries, in the order of the splits.
template <class T>
__global__ __launch_bounds__(256) void gr_attention_sum_parts_kernel(const Args a, int dp) {
  const int quads = dp / 4;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, rows = (int64_t)a.B * a.HK * a.M, plane = rows * dp;
  const int64_t row = id / quads;
  const int d = (int)(id - row * quads) * 4;
  if (row >= rows) return;
  f32x4 k = (f32x4)0.0f, v = (f32x4)0.0f;
  for (int s = 0; s < a.splits; ++s) {
    k += *(const f32x4*)(a.part_o + 2 * s * plane + row * dp + d);
    v += *(const f32x4*)(a.part_o + (2 * s + 1) * plane + row * dp + d);
  }
  const int64_t pair = row / a.M;
  const int64_t key = row - pair * a.M, b = pair / a.HK, hk = pair - b * a.HK;
  const float by = a.scale * UNLIFT, x[4] = {k[0] * by, k[1] * by, k[2] * by, k[3] * by}, y[4] = {v[0] * UNLIFT, v[1] * UNLIFT, v[2] * UNLIFT, v[3] * UNLIFT};
  store4(at<T>(a.dk, b, key, hk), d, a.D, x, a.dk.aligned);
  store4(at<T>(a.dv, b, key, hk), d, a.D, y, a.dv.aligned);
}

static dim3 blocks_of(int64_t threads) { return dim3((unsigned)((threads + 255) / 256)); }

hipError_t combine(const Args& a, int type, int dp, hipStream_t stream) {
  const dim3 grid = blocks_of((int64_t)a.B * a.HK * a.N * a.G * (dp / 4));
  if (type == TYPE_BF16) gr_attention_combine_kernel<__bf16><<<grid, dim3(256), 0, stream>>>(a, dp);
  else gr_attention_combine_kernel<float><<<grid, dim3(256), 0, stream>>>(a, dp);
  return hipGetLastError();
}

hipError_t ranges(const Args& a, hipStream_t stream) {
  gr_attention_ranges_kernel<<<blocks_of((int64_t)a.B * ((a.M + 31) / 32) * 32), dim3(256), 0, stream>>>(a.kdoc, a.kdoc_sb, a.kdoc_sn, a.B, a.M, a.kranges);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.qranges) return e;
  gr_attention_ranges_kernel<<<blocks_of((int64_t)a.B * ((a.N + 31) / 32) * 32), dim3(256), 0, stream>>>(a.qdoc, a.qdoc_sb, a.qdoc_sn, a.B, a.N, a.qranges);
  return hipGetLastError();
}

hipError_t delta(const Args& a, int type, float* to, hipStream_t stream) {
  const dim3 grid = blocks_of((int64_t)a.B * a.N * a.H * 16);
  if (type == TYPE_BF16) gr_attention_delta_kernel<__bf16><<<grid, dim3(256), 0, stream>>>(a, to);
  else gr_attention_delta_kernel<float><<<grid, dim3(256), 0, stream>>>(a, to);
  return hipGetLastError();
}

hipError_t sum_parts(const Args& a, int type, int dp, hipStream_t stream) {
  const dim3 grid = blocks_of((int64_t)a.B * a.HK * a.M * (dp / 4));
  if (type == TYPE_BF16) gr_attention_sum_parts_kernel<__bf16><<<grid, dim3(256), 0, stream>>>(a, dp);
  else gr_attention_sum_parts_kernel<float><<<grid, dim3(256), 0, stream>>>(a, dp);
  return hipGetLastError();
}

}  // namespace attn
}  // namespace gr
