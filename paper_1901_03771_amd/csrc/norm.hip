// Root-mean-square norms: r = 1 / sqrt(mean(t^2) + eps), y = t r (offset + weight) of t = x or of the rounded sum x + residual; and the gradient
//   g = dout (offset + weight),  dx = r g - t r^3 mean(g t) + dtotal,  dweight = sum over rows of dout t r.
// What is read and written of the tensors bounds them.  A row is shared by 16 to 1024 threads and stays in their registers between the sum and its
// use, so that every tensor passes once; a workgroup goes through rows with the weights, and the sums for dweight, in registers too.  1024 threads of 128 registers hold that up to 16384 values (a
// gradient's in f32: 8192); of longer rows part of it lies in scratch memory, which every row reads, and gradients over 16384 values write too (1000 rows of 16384 and 32768 values: gradients in bf16 31 and
// 168 us, in f32 62 and 246; bf16 to 8 bits 17.0 and 36.7).
// 16384 rows of 8192 bf16 values with a residual, to 8 bits: 165 us, 5.7 TB/s; the gradient of 8192 rows of 4096: 52 us, 5.2 TB/s.
#include "scaled_kernels.h"

namespace gr {
namespace scaled {

template <class T>
static __device__ __forceinline__ T* row_at(const Rows& r, const Norm& a, int64_t row) {
  if (a.n1 == 1 && a.n2 == 1) return (T*)r.p + row * r.s0;
  const uint32_t n = (uint32_t)row, i = n / (uint32_t)a.n2, k = n - i * (uint32_t)a.n2, h = i / (uint32_t)a.n1, j = i - h * (uint32_t)a.n1;
  return (T*)r.p + h * r.s0 + j * r.s1 + k * r.s2;
}

// The weights of the thread's values, to which the offset is added where they are used: so the first row's loads need not wait for them.  1 where there are none.  Only f32 ones side by side come as vectors (8
// rows of 4096 bf16 values to 8 bits: 3.6 us, with bf16 weights 5.2).
template <int TPR, int V, int N>
static __device__ __forceinline__ void weights(const Norm& a, int t, float (&w)[V][N]) {
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int d = (j * TPR + t) * N;
    if (a.weight && a.weight_s == 1) {
#pragma unroll
      for (int q = 0; q < N; q += 4) {
        const f32x4 v = get<float>(a.weight, d + q, a.D);
#pragma unroll
        for (int e = 0; e < 4; ++e) w[j][q + e] = v[e];
      }
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const int64_t at = (d + e) * a.weight_s;
        w[j][e] = d + e >= a.D ? 0.0f : a.weight ? a.weight[at] : a.weight16 ? (float)((const __bf16*)a.weight16)[at] : 1.0f;
      }
    }
  }
}
// (a number that the compiler takes to be new in every turn of the loop)
static __device__ __forceinline__ float anew(float x) { asm volatile("" : "+s"(x)); return x; }

// The sums of a row over the TPR threads that share it, in all of them.  One barrier a row: `turn` alternates between two places in LDS.
template <int TPR, int COUNT>
static __device__ __forceinline__ void row_sums(float (&s)[COUNT], int turn) {
#pragma unroll
  for (int c = 0; c < COUNT; ++c) s[c] = sum_across<(TPR < 64 ? TPR : 64)>(s[c]);
  if constexpr (TPR > 64) {
    constexpr int WAVES = TPR / 64;
    __shared__ float part[2][COUNT][WAVES];
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int c = 0; c < COUNT; ++c) part[turn][c][threadIdx.x >> 6] = s[c];
    __syncthreads();
#pragma unroll
    for (int c = 0; c < COUNT; ++c) {
      s[c] = part[turn][c][0];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) s[c] += part[turn][c][w];
    }
  }
}

template <class T, bool EIGHT, bool PAST, int TPR, int V>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void gr_rms_norm_kernel(const Norm a) {
  constexpr int N = Vec<T>::N, THREADS = TPR < 256 ? 256 : TPR, PER = THREADS / TPR;
  const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  float w[V][N];
  weights<TPR, V, N>(a, t, w);
  int turn = 0;
  // Workgroups go round the eight XCDs in turn, each with an L2 of its own: eight neighbouring rows go to one XCD, so that the scales of a block, which may lie side by side, are written
  // to memory together.
  unsigned place = blockIdx.x;
  if (EIGHT && gridDim.x % 64 == 0) place = place / 64 * 64 + place % 8 * 8 + place / 8 % 8;
  for (int64_t row0 = (int64_t)place * PER; row0 < a.rows; row0 += (int64_t)gridDim.x * PER) {
    const int64_t row = row0 + sub < a.rows ? row0 + sub : a.rows - 1;
    const bool mine = row0 + sub < a.rows;
    const int D = mine ? a.D : 0;             // (a row behind the last is neither read nor written)
    typename Vec<T>::type x[V];
    const T* const xr = row_at<const T>(a.x, a, row);
#pragma unroll
    for (int j = 0; j < V; ++j) x[j] = get<T, PAST>(xr, (j * TPR + t) * N, D);
    if (a.residual.p) {
      const T* const rr = row_at<const T>(a.residual, a, row);
      typename Vec<T>::type more[V];
#pragma unroll
      for (int j = 0; j < V; ++j) more[j] = get<T, PAST>(rr, (j * TPR + t) * N, D);
      // (rounded to the type before the norm: that is the stream as the next layer, and the gradient, find it)
#pragma unroll
      for (int j = 0; j < V; ++j)
#pragma unroll
        for (int e = 0; e < N; ++e) x[j][e] = (T)((float)x[j][e] + (float)more[j][e]);
      if (a.total.p) {
        T* const to = row_at<T>(a.total, a, row);
#pragma unroll
        for (int j = 0; j < V; ++j) put<T, PAST>(to, (j * TPR + t) * N, D, x[j]);
      }
    }
    const float offset = anew(a.offset);
    float s[1] = {0.0f};
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
      for (int e = 0; e < N; ++e) s[0] = __builtin_fmaf((float)x[j][e], (float)x[j][e], s[0]);
    row_sums<TPR, 1>(s, turn);
    turn ^= 1;
    const float r = 1.0f / sqrtf(s[0] / (float)a.D + a.eps);
    if constexpr (EIGHT) {
      uint8_t* const to = row_at<uint8_t>(a.out, a, row);
      float* const scales = row_at<float>(a.scales, a, row);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int d = (j * TPR + t) * N;
        float y[N];
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < N; ++e) {
          y[e] = (float)x[j][e] * r * (offset + w[j][e]);
          const uint32_t b = d + e < D ? size_bits(y[e]) : 0;   // (r may be infinite or NaN: not behind the row's end)
          top = b > top ? b : top;
        }
        top = max_across<BLOCK / N>(top);
        const float scale = scale_of(top), inverse = inverse_of(scale);
        const bool some = top < 0x7f800000u;
        uint32_t q[N / 4];
#pragma unroll
        for (int e = 0; e < N; e += 4) q[e / 4] = some ? eight(y[e], y[e + 1], y[e + 2], y[e + 3], scale, inverse) : NO_NUMBERS;
        if (d + N <= D) {
          typedef uint32_t anywhere __attribute__((ext_vector_type(N / 4), aligned(1)));
          anywhere v;
#pragma unroll
          for (int e = 0; e < N / 4; ++e) v[e] = q[e];
          if constexpr (PAST) __builtin_nontemporal_store(v, (anywhere*)(to + d));
          else *(anywhere*)(to + d) = v;
        } else {
#pragma unroll
          for (int e = 0; e < N; ++e) if (d + e < D) to[d + e] = (uint8_t)(q[e / 4] >> (8 * (e % 4)));
        }
        if (t % (BLOCK / N) == 0 && d < D) scales[d / BLOCK * a.scales_s] = scale;
      }
    } else {
      T* const to = row_at<T>(a.out, a, row);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        typename Vec<T>::type y;
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] = (T)((float)x[j][e] * r * (offset + w[j][e]));
        put<T, PAST>(to, (j * TPR + t) * N, D, y);
      }
    }
  }
}

template <class T, bool PAST, int TPR, int V>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void gr_rms_norm_grad_kernel(const Norm a) {
  constexpr int N = Vec<T>::N, THREADS = TPR < 256 ? 256 : TPR, PER = THREADS / TPR;
  const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  float w[V][N], dw[V][N];
  weights<TPR, V, N>(a, t, w);
#pragma unroll
  for (int j = 0; j < V; ++j)
#pragma unroll
    for (int e = 0; e < N; ++e) dw[j][e] = 0.0f;
  int turn = 0;
  for (int64_t row0 = (int64_t)blockIdx.x * PER; row0 < a.rows; row0 += (int64_t)gridDim.x * PER) {
    const int64_t row = row0 + sub < a.rows ? row0 + sub : a.rows - 1;
    const bool mine = row0 + sub < a.rows;
    const int D = mine ? a.D : 0;
    typename Vec<T>::type x[V], y[V], more[V];
    const T* const xr = row_at<const T>(a.x, a, row);
    const T* const yr = row_at<const T>(a.dout, a, row);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      x[j] = get<T, PAST>(xr, (j * TPR + t) * N, D);
      y[j] = get<T, PAST>(yr, (j * TPR + t) * N, D);
    }
    if (a.residual.p) {
      const T* const rr = row_at<const T>(a.residual, a, row);
#pragma unroll
      for (int j = 0; j < V; ++j) more[j] = get<T, PAST>(rr, (j * TPR + t) * N, D);
    }
    const float offset = anew(a.offset);
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float v = (float)x[j][e];
        s[0] = __builtin_fmaf(v, v, s[0]);
        s[1] = __builtin_fmaf((float)y[j][e] * (offset + w[j][e]), v, s[1]);
      }
    row_sums<TPR, 2>(s, turn);
    turn ^= 1;
    const float r = 1.0f / sqrtf(s[0] / (float)a.D + a.eps), pull = s[1] / (float)a.D * r * r;   // dx = r (g - pull t)
    T* const to = row_at<T>(a.dx, a, row);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      typename Vec<T>::type dx;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float v = (float)x[j][e], g = (float)y[j][e];
        float z = r * __builtin_fmaf(-pull, v, g * (offset + w[j][e]));
        if (a.residual.p) z += (float)more[j][e];
        dx[e] = (T)z;
        if (mine) dw[j][e] = __builtin_fmaf(g, v * r, dw[j][e]);
      }
      put<T, PAST>(to, (j * TPR + t) * N, D, dx);
    }
  }
  if (!a.parts) return;
  // the sums of the workgroup's rows; of rows side by side, in order
  if constexpr (PER > 1) {
    __shared__ float side[PER][V * TPR * N + 4];
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
      for (int e = 0; e < N; ++e) side[sub][(j * TPR + t) * N + e] = dw[j][e];
    __syncthreads();
    for (int d = threadIdx.x; d < a.D; d += THREADS) {
      float z = side[0][d];
#pragma unroll
      for (int p = 1; p < PER; ++p) z += side[p][d];
      a.parts[(int64_t)blockIdx.x * a.D + d] = z;
    }
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
      for (int q = 0; q < N; q += 4) put<float>(a.parts + (int64_t)blockIdx.x * a.D, (j * TPR + t) * N + q, a.D, f32x4{dw[j][q], dw[j][q + 1], dw[j][q + 2], dw[j][q + 3]});
  }
}

// dweight: the sums of all workgroups, in order; 32 columns a workgroup, 32 threads for each.
__global__ __launch_bounds__(1024) void gr_rms_norm_sum_kernel(const Norm a) {
  __shared__ float side[32][32];
  const int c = threadIdx.x & 31, g = threadIdx.x >> 5, d = blockIdx.x * 32 + c;
  const int each = (a.groups + 31) / 32, to = min((g + 1) * each, a.groups);
  float z = 0.0f;
  if (d < a.D) {
#pragma unroll 8
    for (int p = g * each; p < to; ++p) z += a.parts[(int64_t)p * a.D + d];
  }
  side[g][c] = z;
  __syncthreads();
  if (g == 0 && d < a.D) {
#pragma unroll
    for (int p = 1; p < 32; ++p) z += side[p][c];
    a.dweight[d * a.dweight_s] = z;
  }
}

// Tensors of 32 MiB and more go past the caches, which they have left by the time that anything reads them (16384 rows of 8192 bf16 values with a residual, to 8 bits: 177 us, 165 so; of 1024
// values, to bf16: 27 and 25; 65536 rows of 128 values, 16 MiB: 7.6 and 8.1).
static bool goes_past(const Norm& a, size_t size) { return a.rows * a.D * (int64_t)size >= (int64_t)32 << 20; }

template <class T, bool EIGHT>
static hipError_t norm_of(const Norm& a, Shape s, unsigned grid, hipStream_t stream) {
  const bool past = goes_past(a, sizeof(T));
#define CASE(THREADS, VECTORS)                                                                                                               \
  if (s.threads == THREADS && s.vectors == VECTORS) {                                                                                         \
    constexpr int GROUP = THREADS < 256 ? 256 : THREADS;                                                                                      \
    if (past && THREADS >= 64) gr_rms_norm_kernel<T, EIGHT, THREADS >= 64, THREADS, VECTORS><<<dim3(grid), dim3(GROUP), 0, stream>>>(a);      \
    else gr_rms_norm_kernel<T, EIGHT, false, THREADS, VECTORS><<<dim3(grid), dim3(GROUP), 0, stream>>>(a);                                    \
    return hipGetLastError();                                                                                                                 \
  }
  CASE(BLOCK / Vec<T>::N, 1) CASE(64, 1) CASE(64, 2) CASE(64, 4) CASE(256, 2) CASE(512, 2) CASE(1024, 2) CASE(1024, 4)
  if constexpr (sizeof(T) == 4) { CASE(1024, 8) }
#undef CASE
  return hipErrorInvalidValue;
}
template <class T>
static hipError_t grad_of(const Norm& a, Shape s, unsigned grid, hipStream_t stream) {
  const bool past = goes_past(a, sizeof(T));
#define CASE(THREADS, VECTORS)                                                                                                          \
  if (s.threads == THREADS && s.vectors == VECTORS) {                                                                                    \
    constexpr int GROUP = THREADS < 256 ? 256 : THREADS;                                                                                 \
    if (past && THREADS >= 64) gr_rms_norm_grad_kernel<T, THREADS >= 64, THREADS, VECTORS><<<dim3(grid), dim3(GROUP), 0, stream>>>(a);   \
    else gr_rms_norm_grad_kernel<T, false, THREADS, VECTORS><<<dim3(grid), dim3(GROUP), 0, stream>>>(a);                                 \
    return hipGetLastError();                                                                                                            \
  }
  CASE(BLOCK / Vec<T>::N, 1) CASE(64, 1) CASE(64, 2) CASE(64, 4) CASE(256, 2) CASE(256, 4) CASE(1024, 2) CASE(1024, 4)
  if constexpr (sizeof(T) == 4) { CASE(1024, 8) }
#undef CASE
  return hipErrorInvalidValue;
}

// Short rows: as few threads as hold them, so that no barrier stands between a row's loads and its use (16384 rows of 2048 bf16 values: 45.6 us on 64 threads, 48 on 256).  Longer ones: few
// registers a thread in the norm (8192 values: 512 threads 165 us, 256 with twice as many vectors 170); in the gradient, whose every thread keeps its part of dweight, as many vectors as 256
// registers hold (8192 bf16 values, 4096 rows: 256 threads 55 us, 512 57; 5003 float32 values, 777 rows: 1024 threads 17, 512 22).
Shape norm_shape(int type, int D, bool gradient) {
  const int n = type == BF16 ? 8 : 4, vectors = (D + n - 1) / n, narrow = BLOCK / n;
  if (vectors <= narrow) return {narrow, 1};
  if (vectors <= 64) return {64, 1};
  if (vectors <= 128) return {64, 2};
  if (vectors <= 256) return {64, 4};
  if (vectors <= 512) return {256, 2};
  if (vectors <= 1024) return gradient ? Shape{256, 4} : Shape{512, 2};
  if (vectors <= 2048) return {1024, 2};
  return vectors <= 4096 ? Shape{1024, 4} : Shape{1024, 8};
}

hipError_t norm(const Norm& a, int type, bool eight, Shape s, unsigned grid, hipStream_t stream) {
  if (type == BF16) return eight ? norm_of<__bf16, true>(a, s, grid, stream) : norm_of<__bf16, false>(a, s, grid, stream);
  return eight ? norm_of<float, true>(a, s, grid, stream) : norm_of<float, false>(a, s, grid, stream);
}
hipError_t norm_grad(const Norm& a, int type, Shape s, unsigned grid, hipStream_t stream) {
  return type == BF16 ? grad_of<__bf16>(a, s, grid, stream) : grad_of<float>(a, s, grid, stream);
}
hipError_t norm_sum(const Norm& a, hipStream_t stream) {
  gr_rms_norm_sum_kernel<<<dim3((a.D + 31) / 32), dim3(1024), 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace scaled
}  // namespace gr
