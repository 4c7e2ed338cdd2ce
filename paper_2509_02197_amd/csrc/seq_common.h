// Device helpers shared by the kernels of the sequence and token operators:
// element types and their accumulation type,
// 16-byte vectors at any element's address, wave reductions.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "adst.h"

namespace adst {
namespace {

typedef __bf16 bf16;
typedef _Float16 f16;

// What sums, states and statistics of a type are held in.
template <class T>
struct AccOf {
  typedef float type;
};
template <>
struct AccOf<double> {
  typedef double type;
};
template <class T>
using Acc = typename AccOf<T>::type;

template <class T>
__device__ inline Acc<T> up(T v) {
  return (Acc<T>)v;
}
// Rounds to nearest, ties to even.
template <class T>
__device__ inline T down(Acc<T> v) {
  return (T)v;
}
// By bits: the hardware's conversion instruction where it has one, and the
// exact widening shift.
template <>
__device__ inline float up<bf16>(bf16 v) {
  return __builtin_bit_cast(float, (uint32_t)__builtin_bit_cast(uint16_t, v) << 16);
}

// 16 bytes of T. The alignment is one element's: gfx950 loads and stores
// 16-byte vectors at any such address, so rows of any length, stride and
// start take the same path.
template <class T>
struct Vec {
  static constexpr int N = 16 / (int)sizeof(T);
  typedef T type __attribute__((ext_vector_type(N)));
  typedef T unaligned __attribute__((ext_vector_type(N), aligned(sizeof(T))));
  type v;
};

template <class T>
__device__ inline Vec<T> load_vec(const T* p) {
  Vec<T> r;
  r.v = *reinterpret_cast<const typename Vec<T>::unaligned*>(p);
  return r;
}
template <class T>
__device__ inline void store_vec(T* p, Vec<T> v) {
  *reinterpret_cast<typename Vec<T>::unaligned*>(p) = v.v;
}
// The first n of the vector's elements (the others are zero, and untouched).
template <class T>
__device__ inline Vec<T> load_part(const T* p, int n) {
  Vec<T> r;
  if (n >= Vec<T>::N) return load_vec(p);
#pragma unroll
  for (int i = 0; i < Vec<T>::N; ++i) r.v[i] = i < n ? p[i] : T(0);
  return r;
}
template <class T>
__device__ inline void store_part(T* p, Vec<T> v, int n) {
  if (n >= Vec<T>::N) {
    store_vec(p, v);
    return;
  }
#pragma unroll
  for (int i = 0; i < Vec<T>::N; ++i)
    if (i < n) p[i] = v.v[i];
}

__device__ inline float fma_(float a, float b, float c) { return __builtin_fmaf(a, b, c); }
__device__ inline double fma_(double a, double b, double c) { return __builtin_fma(a, b, c); }

__device__ inline float exp_full(float x) { return expf(x); }
__device__ inline double exp_full(double x) { return exp(x); }
__device__ inline float inverse(float x) { return __builtin_amdgcn_rcpf(x); }  // within 1 ulp
__device__ inline double inverse(double x) { return 1.0 / x; }

// s = 1 / (1 + exp(-a)) and q = 1 - s = 1 / (1 + exp(a)), each to full
// relative precision down to the type's smallest normal value, and 0 and 1 are
// reached. Behind a 16-bit value the exponential may be off by |a| units of
// 2^-24.
template <class T>
__device__ inline void gates(Acc<T> a, Acc<T>* s, Acc<T>* q) {
  typedef Acc<T> A;
  if constexpr (sizeof(T) == 2) {
    const float e = __builtin_amdgcn_exp2f(-1.44269504f * a);
    *s = inverse(1.0f + e);
    *q = e > 0x1p126f ? 1.0f : e * *s;  // beyond, 1 / e is no normal value; NaN stays
  } else {  // with e = exp(-|a|) in [0, 1] nothing overflows, and 0 and 1 are reached
    const A e = exp_full(-__builtin_elementwise_abs(a));
    const A big = inverse(A(1) + e), small = e * big;
    *s = __builtin_signbit(a) ? small : big;
    *q = __builtin_signbit(a) ? big : small;
  }
}

__device__ inline int64_t row_length(const int32_t* lens, int64_t b, int64_t T) {
  if (!lens) return T;
  const int64_t n = lens[b];
  return n < 0 ? 0 : n > T ? T : n;
}

// Sum over groups of W consecutive lanes (16 or 64), in every lane, in an
// order that is the same for all of them. Within a row of 16 lanes the values
// go through the vector instructions' lane permutations (pairs, quads, halves,
// the row), and between rows through row exchanges: nothing goes through LDS.
template <int CTRL>
__device__ inline float permuted(float v) {
  return __builtin_bit_cast(
      float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
// Sum of the wave's four rows, lane by lane.
__device__ inline float sum_rows(float v) {
  const uint32_t b = __builtin_bit_cast(uint32_t, v);
  const auto rows = __builtin_amdgcn_permlane16_swap(b, b, false, false);
  // (named words: a bit cast of a vector's element takes its first one)
  const uint32_t even = rows[0], odd = rows[1];
  v = __builtin_bit_cast(float, even) + __builtin_bit_cast(float, odd);
  const uint32_t c = __builtin_bit_cast(uint32_t, v);
  const auto halves = __builtin_amdgcn_permlane32_swap(c, c, false, false);
  const uint32_t low = halves[0], high = halves[1];
  return __builtin_bit_cast(float, low) + __builtin_bit_cast(float, high);
}
__device__ inline double sum_rows(double v) {
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}
template <int W>
__device__ inline float lane_sum(float v) {
  v += permuted<0xb1>(v);   // lanes 1 0 3 2
  v += permuted<0x4e>(v);   // lanes 2 3 0 1
  v += permuted<0x141>(v);  // the half row, mirrored
  v += permuted<0x140>(v);  // the row, mirrored
  return W > 16 ? sum_rows(v) : v;
}
template <int W>
__device__ inline double lane_sum(double v) {
#pragma unroll
  for (int off = 1; off < 16; off <<= 1) v += __shfl_xor(v, off, 64);
  return W > 16 ? sum_rows(v) : v;
}

}  // namespace
}  // namespace adst
