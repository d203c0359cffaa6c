// What the host side of the attention and rotary calls (attention.cpp) hands to their kernels
// (attention_kernels.h, rotary.hip).
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstdint>

namespace gr {
namespace attn {

// A (batch, row, head, d) tensor whose d are neighbours: strides in elements.
struct Tensor {
  void* p = nullptr;
  int64_t sb = 0, sn = 0, sh = 0;
  int aligned = 0;  // address and strides are multiples of 16 bytes, and so are d elements: whole vectors
  int direct = 0;   // ... and rows follow one another without overlap, those of a tile within 2^31 bytes: buffer loads straight into LDS
};

struct Args {
  Tensor q, k, v, out, rest, dout, dq, dk, dv;
  float* lse = nullptr;          // (B, H, N)
  // of the gradient, (B, H, NP) with NP = N rounded up to whole tiles: less = lse in binary logarithms - LIFT, of float32 half of it without (rows that see nothing, and
  // rows behind the last: +inf), delta = sum over d of dout * out
  float *less = nullptr, *delta = nullptr;
  float* part_o = nullptr;       // (splits, B * HK, N * G, DP) unnormalised sums of a split's keys; parts of dq, or of dk and dv, likewise
  float* part_ml = nullptr;      // (splits, B * HK, N * G, 2) maximum (binary logarithms) and sum
  const float* slopes = nullptr; // (H), stride slopes_s
  int64_t slopes_s = 0;
  const int* prefix = nullptr;   // (B)
  int64_t prefix_s = 0;
  const int* lengths = nullptr;  // (B)
  int64_t lengths_s = 0;
  const int* qdoc = nullptr;     // (B, N)
  const int* kdoc = nullptr;     // (B, M)
  int64_t qdoc_sb = 0, qdoc_sn = 0, kdoc_sb = 0, kdoc_sn = 0;
  int* kranges = nullptr;        // (B, ceil(M / 32), 2): smallest and largest document number of 32 keys
  int* qranges = nullptr;        // (B, ceil(N / 32), 2), the same of 32 queries
  int *qdocs = nullptr, *kdocs = nullptr;   // (B, NP) and (B, MP), the documents of queries and keys side by side, -1 behind the last
  int64_t position = 0;          // of query 0
  int place = 0;                 // the same within 2^30 of key 0: all that masks can tell (N and M are smaller)
  int B = 0, N = 0, M = 0, H = 0, HK = 0, G = 0, D = 0;
  int causal = 0, step = 0;      // step: a query stands at its sequence's last key
  int splits = 1, blocks = 0;    // splits of the keys (for dk and dv: of the queries), blocks of rows (of keys) of a head
  float scale = 1.0f;
  float c = 0.0f;                // binary logarithm units: scale * log2(e), or cap * log2(e) where scores are capped
  float cin = 0.0f;              // a product times this is the argument of the tanh, in the unit that its form takes
};

enum { MODE_CAP = 1, MODE_BIAS = 2, MODE_WIDE = 4 };   // wide: bfloat16 with a cap beyond SHORT_CAP, see capped() in attention_kernels.h
constexpr double SHORT_CAP = 1024.0;
enum { TYPE_F32 = 0, TYPE_BF16 = 1 };

constexpr int64_t padded_rows(int64_t n) { return (n + 127) / 128 * 128; }   // no tile is taller

// Sizes that host and kernels share, for an element of `size` bytes and heads padded to `dp` values.
constexpr int row_values(int dp) { return dp <= 64 ? 64 : dp <= 128 ? 128 : 256; }                 // of a row in LDS
constexpr int tile_rows(int size, int dp) { return size * row_values(dp) <= 256 ? 64 : 32; }       // of a tile that waves share
// Workgroups of a kernel that fit a compute unit together: two where a wave's operands, sums and scores leave 256 registers enough.
constexpr int forward_per_cu(int size, int dp) { return size == 2 || dp <= 96 ? 2 : 1; }
constexpr int grad_q_per_cu(int size, int dp) { return size == 2 && dp <= 128 ? 2 : 1; }
constexpr int grad_kv_per_cu(int size, int dp) { return size == 2 ? (dp <= 128 ? 2 : 1) : (dp <= 64 ? 2 : 1); }
constexpr int MAX_SPLITS = 256;
// Waves that divide a tile's keys.  bfloat16: tiles of 16 KiB, so that two workgroups and more fit a compute unit and one's loads are under way
// while another multiplies (32 sequences of 4096 to 8192 keys, 128 values: 200 us with one workgroup of four waves per compute unit, 172 so).  float32,
// where the matrix cores are the bound: 32 KiB, for fewer parts to join (65537 keys, 64 values: 23 and 20 us).
constexpr int shared_waves(int size, int dp) { return (size == 2 ? 16384 : 32768) / (32 * size * row_values(dp)) > 4 ? 4 : (size == 2 ? 16384 : 32768) / (32 * size * row_values(dp)); }

// Workgroups that place_of (attention_kernels.h) deals `blocks` of each of `pairs` heads to.
static inline unsigned grid_of(int pairs, int64_t blocks) {
  if (pairs % 8 != 0 && 8 % pairs == 0) { const int per = 8 / pairs; return (unsigned)((blocks + per - 1) / per * 8); }
  return (unsigned)(pairs * blocks);
}

hipError_t forward_f32(const Args& a, int dp, int mode, bool divided, unsigned grid, hipStream_t stream);
hipError_t forward_bf16(const Args& a, int dp, int mode, bool divided, unsigned grid, hipStream_t stream);
hipError_t combine(const Args& a, int type, int dp, hipStream_t stream);
hipError_t ranges(const Args& a, hipStream_t stream);
hipError_t statistics(const Args& a, int type, hipStream_t stream);
hipError_t grad_q_f32(const Args& a, int dp, int mode, unsigned grid, hipStream_t stream);
hipError_t grad_q_bf16(const Args& a, int dp, int mode, unsigned grid, hipStream_t stream);
hipError_t grad_kv_f32(const Args& a, int dp, int mode, unsigned grid, hipStream_t stream);
hipError_t grad_kv_bf16(const Args& a, int dp, int mode, unsigned grid, hipStream_t stream);
hipError_t sum_parts(const Args& a, int type, int dp, bool queries, hipStream_t stream);

constexpr int MAX_PAIRS = 256;
struct Rotary {
  Tensor x, y;
  const int* positions = nullptr;  // (B, N)
  int64_t positions_sb = 0, positions_sn = 0, position = 0;
  int B = 0, N = 0, H = 0, D = 0, pairs = 0, interleaved = 0, inverse = 0, tokens = 1, heads = 1;
  float factor = 1.0f;
  double turns[MAX_PAIRS];         // of each pair per position
};
hipError_t rotary(const Rotary& r, int type, hipStream_t stream);

}  // namespace attn
}  // namespace gr
