// Rotary positions: pair i of a head at position p turns by the angle p f_i,
//   lo' = factor (lo cos - hi sin),  hi' = factor (hi cos + lo sin);
// the gradient is the same turn backwards.  A read and a write of the tensor bound it.
//
// A workgroup takes a few tokens and a run of heads.  It forms their sines and cosines once, in LDS, for all its heads, and where the tokens
// lie, then moves whole 16-byte vectors: a thread has a place in the heads and goes through the tokens with it, so that nothing is divided
// on the way (4611 tokens of 12 heads of 80 float32 values: 13.6 us with three divisions a vector).  The angle is formed in turns, in 64 bits, and its whole turns are taken off there: at position 10^6 an angle
// held in 32 bits is off by 0.06.  What is left, an eighth of a turn at most around a quarter, is small enough for Taylor's
// polynomials in 32 bits (sine to x^9: 2e-9 off at pi / 4; cosine to x^10: 1e-10).
#include "attention_kernels.h"

namespace gr {
namespace attn {

static __device__ __forceinline__ void turn(double turns, float& c, float& s) {
  const double r = turns - __builtin_rint(turns);           // [-1/2, 1/2]
  const double q = __builtin_rint(4.0 * r);
  const float x = (float)((r - 0.25 * q) * 6.283185307179586);
  const float z = x * x;
  float u = 1.0f / 362880.0f;
  u = __builtin_fmaf(u, z, -1.0f / 5040.0f);
  u = __builtin_fmaf(u, z, 1.0f / 120.0f);
  u = __builtin_fmaf(u, z, -1.0f / 6.0f);
  const float sn = __builtin_fmaf(x * z, u, x);
  float w = -1.0f / 3628800.0f;
  w = __builtin_fmaf(w, z, 1.0f / 40320.0f);
  w = __builtin_fmaf(w, z, -1.0f / 720.0f);
  w = __builtin_fmaf(w, z, 1.0f / 24.0f);
  w = __builtin_fmaf(w, z, -0.5f);
  const float cs = __builtin_fmaf(z, w, 1.0f);
  const int k = (int)q & 3;
  c = k & 1 ? sn : cs;
  s = k & 1 ? cs : sn;
  if (k == 1 || k == 2) c = -c;
  if (k >= 2) s = -s;
}

template <bool STREAM, class V>
static __device__ __forceinline__ V get(const V* p) {
  if constexpr (STREAM) return __builtin_nontemporal_load(p);
  else return *p;
}
template <bool STREAM, class V>
static __device__ __forceinline__ void put(V* p, V x) {
  if constexpr (STREAM) __builtin_nontemporal_store(x, p);
  else *p = x;
}

// VECTORS: rows of whole aligned vectors, halves (or neighbouring pairs) and the part behind them of whole vectors too
// STREAM: loads and stores that leave the caches alone
template <class T, bool VECTORS, bool STREAM>
__global__ __launch_bounds__(256) void gr_rotary_kernel(const Rotary r) {
  // [token] offset in x, in y, position; then [token][cos of the pairs, sin of the pairs]
  extern __shared__ int64_t places[];
  int64_t* const to = places + r.tokens;
  int64_t* const pos = to + r.tokens;
  float* const table = (float*)(pos + r.tokens);
  const int tid = threadIdx.x, P = r.pairs;
  const int64_t token0 = (int64_t)blockIdx.x * r.tokens, all = (int64_t)r.B * r.N;
  const int tokens = (int)(all - token0 < r.tokens ? all - token0 : r.tokens);
  const int head0 = blockIdx.y * r.heads, heads = r.H - head0 < r.heads ? r.H - head0 : r.heads;
  for (int n = tid; n < tokens; n += 256) {
    const int t = (int)token0 + n, b = t / r.N, i = t - b * r.N;
    places[n] = b * r.x.sb + i * r.x.sn;
    to[n] = b * r.y.sb + i * r.y.sn;
    pos[n] = r.positions ? (int64_t)r.positions[b * r.positions_sb + i * r.positions_sn] : r.position + i;
  }
  __syncthreads();
  for (int k = tid; k < tokens * P; k += 256) {
    const int n = k / P, i = k - n * P;
    float c, s;
    turn((double)pos[n] * r.turns[i], c, s);
    table[2 * n * P + i] = c * r.factor;
    table[2 * n * P + P + i] = r.inverse ? -s * r.factor : s * r.factor;
  }
  __syncthreads();
  constexpr int V = VECTORS ? 16 / (int)sizeof(T) : 1;
  typedef T vec __attribute__((ext_vector_type(VECTORS ? 16 / (int)sizeof(T) : 2)));
  // units of a head: pairs (V at a time, V / 2 where pairs are neighbours), then what is not turned
  const int turned = r.interleaved ? (VECTORS ? 2 * P / V : P) : P / V, units = turned + (r.D - 2 * P) / V;
  const bool in_place = r.x.p == r.y.p;
  // the threads side by side over the units of the heads, and over tokens where those are fewer
  const int wide = heads * units, side = wide < 256 ? wide : 256, rows = 256 / side, row = tid / side;
  if (row >= rows) return;
  for (int k = tid - row * side; k < wide; k += side) {
    const int h = k / units, u = k - h * units;
    const T* const xh = (const T*)r.x.p + (head0 + h) * r.x.sh;
    T* const yh = (T*)r.y.p + (head0 + h) * r.y.sh;
#pragma unroll 1
    for (int n = row; n < tokens; n += rows) {
      const T* x = xh + places[n];
      T* y = yh + to[n];
      const float* cs = table + 2 * n * P;
      const float* sn = cs + P;
      if constexpr (VECTORS) {
        if (u >= turned) {
          const int d = 2 * P + (u - turned) * V;
          if (!in_place) put<STREAM>((vec*)(y + d), get<STREAM>((const vec*)(x + d)));
        } else if (r.interleaved) {
          const vec v = get<STREAM>((const vec*)(x + u * V));
          vec w;
#pragma unroll
          for (int e = 0; e < V; e += 2) {
            const float c = cs[u * (V / 2) + e / 2], s = sn[u * (V / 2) + e / 2], lo = (float)v[e], hi = (float)v[e + 1];
            w[e] = (T)__builtin_fmaf(lo, c, -hi * s);
            w[e + 1] = (T)__builtin_fmaf(hi, c, lo * s);
          }
          put<STREAM>((vec*)(y + u * V), w);
        } else {
          const vec v = get<STREAM>((const vec*)(x + u * V)), w = get<STREAM>((const vec*)(x + P + u * V));
          vec p, q;
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const float c = cs[u * V + e], s = sn[u * V + e], lo = (float)v[e], hi = (float)w[e];
            p[e] = (T)__builtin_fmaf(lo, c, -hi * s);
            q[e] = (T)__builtin_fmaf(hi, c, lo * s);
          }
          put<STREAM>((vec*)(y + u * V), p);
          put<STREAM>((vec*)(y + P + u * V), q);
        }
      } else {
        if (u >= turned) {
          const int d = 2 * P + u - turned;
          if (!in_place) y[d] = x[d];
        } else {
          const int a = r.interleaved ? 2 * u : u, c = r.interleaved ? 2 * u + 1 : P + u;
          const float lo = (float)x[a], hi = (float)x[c];
          y[a] = (T)__builtin_fmaf(lo, cs[u], -hi * sn[u]);
          y[c] = (T)__builtin_fmaf(hi, cs[u], lo * sn[u]);
        }
      }
    }
  }
}

template <class T>
static hipError_t rotary_of(Rotary r, hipStream_t stream) {
  constexpr int V = 16 / (int)sizeof(T);
  const bool vectors = r.x.aligned && r.y.aligned && (r.interleaved ? 2 * r.pairs % V == 0 : r.pairs % V == 0);
  const int64_t tokens = (int64_t)r.B * r.N;
  const dim3 grid((unsigned)((tokens + r.tokens - 1) / r.tokens), (unsigned)((r.H + r.heads - 1) / r.heads));
  const size_t lds = (size_t)r.tokens * (24 + r.pairs * 8);
  // A tensor of 64 MiB and more will have left the caches by the time that anything reads it: it goes past them (2 x 8192 tokens of 32 heads of 128
  // bfloat16 values 60 -> 54 us, 4 x 8192 105 -> 97); a smaller one is read by attention from there (2 x 2048 15 us, 16 past them).
  const bool past = tokens * r.H * r.D * (int64_t)sizeof(T) >= (int64_t)64 << 20;
  if (!vectors) gr_rotary_kernel<T, false, false><<<grid, dim3(256), lds, stream>>>(r);
  else if (past) gr_rotary_kernel<T, true, true><<<grid, dim3(256), lds, stream>>>(r);
  else gr_rotary_kernel<T, true, false><<<grid, dim3(256), lds, stream>>>(r);
  return hipGetLastError();
}

hipError_t rotary(const Rotary& r, int type, hipStream_t stream) { return type == TYPE_BF16 ? rotary_of<__bf16>(r, stream) : rotary_of<float>(r, stream); }

}  // namespace attn
}  // namespace gr
