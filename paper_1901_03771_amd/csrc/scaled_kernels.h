// Device parts that the kernels of the norms and of 8-bit tensors share: vectors of a row at any alignment, sums and maxima over lanes,
// 8-bit values.
#pragma once

#include <hip/hip_runtime.h>

#include "scaled.h"

namespace gr {
namespace scaled {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 b16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 b16x8 __attribute__((ext_vector_type(8)));

// 16 bytes of a row in registers; in memory they stand at any place that its elements may stand at (global loads and stores of vectors take
// every address).
template <class T> struct Vec;
template <> struct Vec<float> {
  static constexpr int N = 4;
  typedef float type __attribute__((ext_vector_type(4)));
  typedef float anywhere __attribute__((ext_vector_type(4), aligned(4)));
};
template <> struct Vec<__bf16> {
  static constexpr int N = 8;
  typedef __bf16 type __attribute__((ext_vector_type(8)));
  typedef __bf16 anywhere __attribute__((ext_vector_type(8), aligned(2)));
};

// Values d .. d + N - 1 of a row of D; zeros behind its end.  PAST: leaves the caches alone.
template <class T, bool PAST = false>
static __device__ __forceinline__ typename Vec<T>::type get(const T* row, int d, int D) {
  constexpr int N = Vec<T>::N;
  typename Vec<T>::type v = (T)0.0f;
  if (d + N <= D) {
    if constexpr (PAST) v = __builtin_nontemporal_load((const typename Vec<T>::anywhere*)(row + d));
    else v = *(const typename Vec<T>::anywhere*)(row + d);
  } else if (d < D) {
#pragma unroll
    for (int e = 0; e < N - 1; ++e) if (d + e < D) v[e] = row[d + e];
  }
  return v;
}
template <class T, bool PAST = false>
static __device__ __forceinline__ void put(T* row, int d, int D, typename Vec<T>::type v) {
  constexpr int N = Vec<T>::N;
  if (d + N <= D) {
    if constexpr (PAST) __builtin_nontemporal_store((typename Vec<T>::anywhere)v, (typename Vec<T>::anywhere*)(row + d));
    else *(typename Vec<T>::anywhere*)(row + d) = v;
  } else if (d < D) {
#pragma unroll
    for (int e = 0; e < N - 1; ++e) if (d + e < D) row[d + e] = v[e];
  }
}

// ---- over neighbouring lanes: every lane of the group gets the result ----------------------------------------------------
template <int CONTROL>
static __device__ __forceinline__ uint32_t rotated(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CONTROL, 0xf, 0xf, false); }

struct Sum {
  static __device__ __forceinline__ uint32_t of(uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }
};
// (of the bits of a size: a NaN's are above an infinity's, and those above all numbers')
struct Max {
  static __device__ __forceinline__ uint32_t of(uint32_t a, uint32_t b) { return a > b ? a : b; }
};
template <class OP, int LANES>
static __device__ __forceinline__ uint32_t across(uint32_t x) {
  static_assert(LANES == 16 || LANES == 32 || LANES == 64, "a row of lanes, or a power of two of them");
  x = OP::of(x, rotated<0x128>(x));   // row_ror:8, 4, 2, 1
  x = OP::of(x, rotated<0x124>(x));
  x = OP::of(x, rotated<0x122>(x));
  x = OP::of(x, rotated<0x121>(x));
  if constexpr (LANES >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = OP::of(r[0], r[1]);
  }
  if constexpr (LANES >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    x = OP::of(r[0], r[1]);
  }
  return x;
}
template <int LANES>
static __device__ __forceinline__ float sum_across(float x) { return __uint_as_float(across<Sum, LANES>(__float_as_uint(x))); }
template <int LANES>
static __device__ __forceinline__ uint32_t max_across(uint32_t x) { return across<Max, LANES>(x); }

static __device__ __forceinline__ uint32_t size_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// ---- 8-bit values -----------------------------------------------------------------------------------------------------------
// The scale of 128 values, of which `top` are the bits of the largest size: NaN where one is infinite or NaN, so that none of them stands for a number.
static __device__ __forceinline__ float scale_of(uint32_t top) {
  const float s = __builtin_fmaxf(__uint_as_float(top) / LARGEST, LEAST_SCALE);
  return top < 0x7f800000u ? s : __uint_as_float(0x7fc00000u);
}

// Four values over their scale, to the nearest e4m3, even ones in the middle.  The quotient of the hardware's reciprocal is put right by what is left of the value (two more instructions, of which
// the memory leaves time for many): values of few bits often lie in the middle, and fall to the side that their float32 quotient is on.  It may pass 448 by a last place: it is held there.
static __device__ __forceinline__ uint32_t eight(float a, float b, float c, float d, float scale, float inverse) {
  const auto held = [&](float x) {
    const float q = x * inverse, left = __builtin_fmaf(-q, scale, x);
    return __builtin_amdgcn_fmed3f(__builtin_fmaf(left, inverse, q), -LARGEST, LARGEST);
  };
  int v = __builtin_amdgcn_cvt_pk_fp8_f32(held(a), held(b), 0, false);
  v = __builtin_amdgcn_cvt_pk_fp8_f32(held(c), held(d), v, true);
  return (uint32_t)v;
}
constexpr uint32_t NO_NUMBERS = 0x7f7f7f7fu;
static __device__ __forceinline__ float inverse_of(float scale) { return __builtin_amdgcn_rcpf(scale); }

}  // namespace scaled
}  // namespace gr
