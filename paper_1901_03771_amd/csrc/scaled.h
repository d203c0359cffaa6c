// What the host side of the norms, the 8-bit tensors and their products (scaled.cpp) hands to their kernels (norm.hip, quantize.hip,
// scaled_dot.hip).
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstdint>

namespace gr {
namespace scaled {

enum { F32 = 0, BF16 = 1, E4M3 = 2 };

constexpr int BLOCK = 128;                       // values that share a scale
constexpr float LARGEST = 448.0f;                // of e4m3
constexpr float LEAST_SCALE = 0x1p-126f;         // so that 1 / scale is a number
static inline int64_t blocks_of(int64_t n) { return (n + BLOCK - 1) / BLOCK; }

// A tensor of up to three axes of rows, the values of a row neighbours: row (i, j, k) lies i s0 + j s1 + k s2 elements from p.
struct Rows {
  void* p = nullptr;
  int64_t s0 = 0, s1 = 0, s2 = 0;
};

// Root-mean-square norm and its gradient of `rows` rows of D values: row = (i * n1 + j) * n2 + k.
struct Norm {
  Rows x, residual, total, out, dout, dx;         // the gradient: x = total, residual = dtotal
  Rows scales;                                    // of an 8-bit out, and the step from one block's to the next
  int64_t scales_s = 0;
  const float* weight = nullptr;                  // f32 or bf16 (weight16)
  const void* weight16 = nullptr;
  int64_t weight_s = 0;
  float* dweight = nullptr;
  int64_t dweight_s = 0;
  float* parts = nullptr;                         // (groups, D): sums of a workgroup's rows
  int64_t rows = 0;
  int n1 = 1, n2 = 1, D = 0, groups = 0;
  float eps = 0.0f, offset = 0.0f;
};

// The threads that share a row, and the vectors of 16 bytes that each of them holds of it.
struct Shape { int threads, vectors; };
constexpr int MOST_VALUES = 32768;                // of a row
Shape norm_shape(int type, int D, bool gradient);
hipError_t norm(const Norm& a, int type, bool eight, Shape s, unsigned grid, hipStream_t stream);
hipError_t norm_grad(const Norm& a, int type, Shape s, unsigned grid, hipStream_t stream);
hipError_t norm_sum(const Norm& a, hipStream_t stream);

struct Quantize {
  const void* x = nullptr;
  int64_t x_s = 0;                                // from row to row
  void* out = nullptr;
  int64_t out_s = 0;
  float* scales = nullptr;
  int64_t scales_sm = 0, scales_sk = 0;           // along the rows of out (or blocks of them), along the blocks of a row
  int64_t M = 0, K = 0;                           // of x
};
hipError_t quantize(const Quantize& a, int type, bool blocks, bool transposed, hipStream_t stream);

// out (M, N) = a (M, K) times b (N, K), the scales between
struct Dot {
  const uint8_t *a = nullptr, *b = nullptr;
  int64_t a_s = 0, b_s = 0;
  const float *sa = nullptr, *sb = nullptr;
  int64_t sa_m = 0, sa_k = 0, sb_n = 0, sb_k = 0;
  void* out = nullptr;
  int64_t out_s = 0;
  float* parts = nullptr;                         // (splits, M, N)
  int M = 0, N = 0, K = 0, KB = 0;                // KB = blocks of K
  int splits = 1;                                 // of the blocks of K
  int mt = 0, nt = 0;                             // tiles
};
enum { DOT_STAGED, DOT_DIRECT, DOT_LOW, DOT_STAGED_LOW, DOT_LARGE, DOT_FEW, DOT_FEW_WORDS };
hipError_t dot(const Dot& d, int form, bool blocks, int out_type, hipStream_t stream);
hipError_t dot_join(const Dot& d, int out_type, hipStream_t stream);

}  // namespace scaled
}  // namespace gr
