// 8-bit tensors with scales: q = round(x / s), s = max|x| / 448 over 128 neighbours of a row, or over 128 x 128 values; and the same of the
// transposed tensor.  A read of x and a write of a byte per value bound it (14336 x 4096 bf16 values, transposed, in blocks: 32 us, 5.5 TB/s).
#include "scaled_kernels.h"

namespace gr {
namespace scaled {

// Rows as they lie: BLOCK / N neighbouring lanes have a block of a row, U of them under way at once where there are many; those beside them the same blocks of the next rows, whose scales
// may lie side by side (14336 x 4096 bf16 values: 37 us with four blocks of a row, 31 so; 4096 x 2048 float32 values, 8192 workgroups with a block each: 9.3 us, 10.1 with four).
template <class T, bool PAST, int U>
__global__ __launch_bounds__(256) void gr_quantize_rows_kernel(const Quantize a) {
  constexpr int N = Vec<T>::N, LANES = BLOCK / N, PER = 256 / LANES;
  const int t = threadIdx.x % LANES, sub = threadIdx.x / LANES, d = t * N;
  const int64_t KU = (a.K + BLOCK * U - 1) / (BLOCK * U), group = blockIdx.x / KU, k0 = (blockIdx.x - group * KU) * U;
  const int64_t row = group * PER + sub, m = row < a.M ? row : a.M - 1;
  typename Vec<T>::type x[U];
  int D[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t left = a.K - (k0 + u) * BLOCK;
    // (a block behind the last has no values, and is not written)
    D[u] = row >= a.M || left <= 0 ? 0 : left < BLOCK ? (int)left : BLOCK;
    x[u] = get<T, PAST>((const T*)a.x + m * a.x_s + (k0 + u) * BLOCK, d, D[u]);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < N; ++e) { const uint32_t b = size_bits((float)x[u][e]); top = b > top ? b : top; }
    top = max_across<LANES>(top);
    const float scale = scale_of(top), inverse = inverse_of(scale);
    uint32_t q[N / 4];
#pragma unroll
    for (int e = 0; e < N; e += 4) q[e / 4] = top < 0x7f800000u ? eight((float)x[u][e], (float)x[u][e + 1], (float)x[u][e + 2], (float)x[u][e + 3], scale, inverse) : NO_NUMBERS;
    uint8_t* const to = (uint8_t*)a.out + m * a.out_s + (k0 + u) * BLOCK;
    if (d + N <= D[u]) {
      typedef uint32_t anywhere __attribute__((ext_vector_type(N / 4), aligned(1)));
      anywhere v;
#pragma unroll
      for (int e = 0; e < N / 4; ++e) v[e] = q[e];
      *(anywhere*)(to + d) = v;
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) if (d + e < D[u]) to[d + e] = (uint8_t)(q[e / 4] >> (8 * (e % 4)));
    }
    if (t == 0 && D[u] > 0) a.scales[m * a.scales_sm + (k0 + u) * a.scales_sk] = scale;
  }
}

// Tiles of 128 x 128 values: a workgroup has one in registers, finds what shares a scale (the whole, or each column, which is a row of the transposed
// tensor), and writes it as it lies or, through LDS, transposed.  512 threads: 4099 x 2051 float32 values to columns 11.6 us, 12.2 with 256; 1000 x 3000 bf16 values 6.0 and 8.0.
constexpr int TILE_THREADS = 512;
template <class T, bool BLOCKS, bool TRANSPOSED, bool PAST>
__global__ __launch_bounds__(TILE_THREADS) void gr_quantize_tiles_kernel(const Quantize a) {
  static_assert(BLOCKS || TRANSPOSED, "rows as they lie need no tiles");
  constexpr int N = Vec<T>::N, LANES = BLOCK / N, HIGH = TILE_THREADS / LANES, V = BLOCK / HIGH;   // HIGH rows at a time, V times
  __shared__ uint32_t tops[HIGH][BLOCK];
  __shared__ uint32_t tile[TRANSPOSED ? BLOCK * (BLOCK / 4 + 1) : 1];                         // [column][row / 4]
  const int t = threadIdx.x % LANES, h = threadIdx.x / LANES;
  const int64_t KB = (a.K + BLOCK - 1) / BLOCK, mb = blockIdx.x / KB, kb = blockIdx.x - mb * KB;
  const int64_t m0 = mb * BLOCK, k0 = kb * BLOCK;
  const int rows = (int)(a.M - m0 < BLOCK ? a.M - m0 : BLOCK), cols = (int)(a.K - k0 < BLOCK ? a.K - k0 : BLOCK);
  // a thread's rows: h V .. h V + V - 1, so that four of them are neighbours in the transposed tensor
  typename Vec<T>::type x[V];
  const T* const from = (const T*)a.x + m0 * a.x_s + k0;
#pragma unroll
  for (int j = 0; j < V; ++j) x[j] = get<T, PAST>(from + (h * V + j) * a.x_s, t * N, h * V + j < rows ? cols : 0);
  uint32_t top[N];
#pragma unroll
  for (int e = 0; e < N; ++e) top[e] = 0;
#pragma unroll
  for (int j = 0; j < V; ++j)
#pragma unroll
    for (int e = 0; e < N; ++e) { const uint32_t b = size_bits((float)x[j][e]); top[e] = b > top[e] ? b : top[e]; }
  if constexpr (BLOCKS) {
#pragma unroll
    for (int e = 1; e < N; ++e) top[0] = top[e] > top[0] ? top[e] : top[0];
    top[0] = max_across<64>(top[0]);
    if ((threadIdx.x & 63) == 0) tops[0][threadIdx.x >> 6] = top[0];
    __syncthreads();
    uint32_t all = tops[0][0];
#pragma unroll
    for (int w = 1; w < TILE_THREADS / 64; ++w) all = tops[0][w] > all ? tops[0][w] : all;
#pragma unroll
    for (int e = 0; e < N; ++e) top[e] = all;
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) tops[h][t * N + e] = top[e];
    __syncthreads();
    if (threadIdx.x < BLOCK) {
      uint32_t all = tops[0][threadIdx.x];
#pragma unroll
      for (int w = 1; w < HIGH; ++w) { const uint32_t b = tops[w][threadIdx.x]; all = b > all ? b : all; }
      tops[0][threadIdx.x] = all;
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < N; ++e) top[e] = tops[0][t * N + e];
  }
  float scale[N], inverse[N];
  bool some[N];
#pragma unroll
  for (int e = 0; e < N; ++e) {
    scale[e] = scale_of(top[e]);
    inverse[e] = inverse_of(scale[e]);
    some[e] = top[e] < 0x7f800000u;
  }
  if constexpr (BLOCKS) {
    if (threadIdx.x == 0) a.scales[(TRANSPOSED ? kb : mb) * a.scales_sm + (TRANSPOSED ? mb : kb) * a.scales_sk] = scale[0];
  } else {
    if (threadIdx.x < cols) a.scales[(k0 + threadIdx.x) * a.scales_sm + mb * a.scales_sk] = scale_of(tops[0][threadIdx.x]);
  }
  if constexpr (!TRANSPOSED) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int m = h * V + j, d = t * N;
      if (m >= rows) continue;
      uint8_t* const to = (uint8_t*)a.out + (m0 + m) * a.out_s + k0;
      uint32_t q[N / 4];
#pragma unroll
      for (int e = 0; e < N; e += 4) q[e / 4] = some[e] ? eight((float)x[j][e], (float)x[j][e + 1], (float)x[j][e + 2], (float)x[j][e + 3], scale[e], inverse[e]) : NO_NUMBERS;
      if (d + N <= cols) {
        typedef uint32_t anywhere __attribute__((ext_vector_type(N / 4), aligned(1)));
        anywhere v;
#pragma unroll
        for (int e = 0; e < N / 4; ++e) v[e] = q[e];
        *(anywhere*)(to + d) = v;
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e) if (d + e < cols) to[d + e] = (uint8_t)(q[e / 4] >> (8 * (e % 4)));
      }
    }
  } else {
    constexpr int PITCH = BLOCK / 4 + 1;
#pragma unroll
    for (int e = 0; e < N; ++e)
#pragma unroll
      for (int j = 0; j < V; j += 4)
        tile[(t * N + e) * PITCH + (h * V + j) / 4] = some[e] ? eight((float)x[j][e], (float)x[j + 1][e], (float)x[j + 2][e], (float)x[j + 3][e], scale[e], inverse[e]) : NO_NUMBERS;
    __syncthreads();
    // rows of the transposed tensor: 16 bytes a thread, 8 threads a row
#pragma unroll
    for (int j = 0; j < BLOCK * 8 / TILE_THREADS; ++j) {
      const int k = j * (TILE_THREADS / 8) + threadIdx.x / 8, m = threadIdx.x % 8 * 16;
      if (k >= cols || m >= rows) continue;
      uint32_t v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = tile[k * PITCH + m / 4 + e];
      uint8_t* const to = (uint8_t*)a.out + (k0 + k) * a.out_s + m0 + m;
      if (m + 16 <= rows) {
        typedef uint32_t anywhere __attribute__((ext_vector_type(4), aligned(1)));
        *(anywhere*)to = anywhere{v[0], v[1], v[2], v[3]};
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) if (m + e < rows) to[e] = (uint8_t)(v[e / 4] >> (8 * (e % 4)));
      }
    }
  }
}

template <class T, bool PAST>
static hipError_t quantize_of(const Quantize& a, bool blocks, bool transposed, hipStream_t stream) {
  const int64_t KB = blocks_of(a.K);
  if (!blocks && !transposed) {
    constexpr int PER = 256 / (BLOCK / Vec<T>::N);
    const int64_t high = (a.M + PER - 1) / PER;
    if (high * KB >= 16384) gr_quantize_rows_kernel<T, PAST, 4><<<dim3((unsigned)(high * ((KB + 3) / 4))), dim3(256), 0, stream>>>(a);
    else gr_quantize_rows_kernel<T, PAST, 1><<<dim3((unsigned)(high * KB)), dim3(256), 0, stream>>>(a);
    return hipGetLastError();
  }
  const dim3 grid((unsigned)(blocks_of(a.M) * KB)), group(TILE_THREADS);
  if (!transposed) gr_quantize_tiles_kernel<T, true, false, PAST><<<grid, group, 0, stream>>>(a);
  else if (blocks) gr_quantize_tiles_kernel<T, true, true, PAST><<<grid, group, 0, stream>>>(a);
  else gr_quantize_tiles_kernel<T, false, true, PAST><<<grid, group, 0, stream>>>(a);
  return hipGetLastError();
}

// Tensors of 64 MiB and more are read past the caches (14336 x 4096 bf16 values, transposed in blocks: 37 us, 33 so; 4096 x 2048 float32 values: 9.2 and 10.0); the result, half of it or a
// quarter, is left to them for the product that takes it.
hipError_t quantize(const Quantize& a, int type, bool blocks, bool transposed, hipStream_t stream) {
  const bool past = a.M * a.K * (type == BF16 ? 2 : 4) >= (int64_t)64 << 20;
  if (type == BF16) return past ? quantize_of<__bf16, true>(a, blocks, transposed, stream) : quantize_of<__bf16, false>(a, blocks, transposed, stream);
  return past ? quantize_of<float, true>(a, blocks, transposed, stream) : quantize_of<float, false>(a, blocks, transposed, stream);
}

}  // namespace scaled
}  // namespace gr
