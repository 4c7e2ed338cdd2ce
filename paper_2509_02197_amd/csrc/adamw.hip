// One AdamW step over many tensors, with states in the parameters' type or in
// blocks of 8-bit codes.
//
// Per value the step reads and writes p, m, v, reads the gradient and writes
// the copy: 28 bytes with 32-bit states, a 16-bit gradient and a 16-bit copy,
// 16 with 8-bit states, against some 20 to 40 instructions: HBM bandwidth
// bounds it. One launch covers as many tensors as its arguments hold (their
// descriptors travel in the kernel's arguments: no device table has to be
// built, kept or copied), cut into chunks of 512 values, a workgroup each. A
// lane handles four consecutive values, so a wave holds one block of 256 codes
// and finds its scale with a wave reduction, without LDS or barrier. Short
// workgroups with one vector of each array a lane were the fastest: 70 million
// values with 32-bit states take 318 us in chunks of 512, 336 to 346 of 1024 to
// 4096, 352 and 358 with two and four vectors a lane.
// Measured at 70.5 million values in 61 tensors, 16-bit gradients and copies:
// 32-bit states 318 us, 6.2 TB/s; 8-bit 190 us, 6.0 TB/s (a plain copy: 6.35).
// 35 million F64 values with F64 gradients, no copies: 376 us, 5.2 TB/s.

#include <cmath>

#include "seq_common.h"
#include "seq_kernels.h"
#include "seq_launch.h"

namespace adst {
namespace {

constexpr int kThreads = 128;
constexpr int kChunk = kThreads * 4;  // values of a workgroup
constexpr int kBlock = ADST_STATE_BLOCK;
static_assert(kBlock == 64 * 4, "a wave's vectors are one block of codes");
constexpr float kCodeMax = 448.0f;   // the largest e4m3 value
constexpr float kCodeMin = 0x1p-9f;  // the smallest positive one
constexpr float kTiny = 0x1p-100f;

// A tensor as the kernel sees it; P is the parameters' type.
template <class P, bool BITS8>
struct Entry {
  void* p;
  const void* g;
  void* m;
  void* v;
  void* copy;
  int64_t n;
  P decay, rate;  // 1 - lr * weight_decay, lr / (1 - beta1^t)
};
template <class P>
struct Entry<P, true> : Entry<P, false> {
  float* m_scale;
  float* v_scale;
};

template <class P>
struct Coefs {
  P b1, b2, c1, c2;  // betas and 1 - beta
  P root, eps;       // 1 / sqrt(1 - beta2^t)
};

constexpr int kArgBytes = 4096;  // of one launch
template <class P, bool BITS8>
struct Table {
  static constexpr int kMost =
      (kArgBytes - (int)sizeof(Coefs<P>) - 32) / (int)(sizeof(Entry<P, BITS8>) + 4);
  Coefs<P> k;
  const float* scale;  // of the gradients, on the device (or null)
  int n;
  int first[kMost + 1];  // first chunk of each tensor
  Entry<P, BITS8> e[kMost];
};

// Four values of T, at any element's address.
template <class T>
struct Four {
  typedef T type __attribute__((ext_vector_type(4)));
  typedef T unaligned __attribute__((ext_vector_type(4), aligned(sizeof(T))));
};
template <bool NT, class T>
__device__ inline typename Four<T>::type load4(const T* p, int n) {
  if (n >= 4) {
    const auto* at = reinterpret_cast<const typename Four<T>::unaligned*>(p);
    if constexpr (NT) return __builtin_nontemporal_load(at);
    else return *at;
  }
  typename Four<T>::type r = {T(0), T(0), T(0), T(0)};
#pragma unroll
  for (int i = 0; i < 3; ++i)
    if (i < n) r[i] = p[i];
  return r;
}
template <bool NT, class T>
__device__ inline void store4(T* p, typename Four<T>::type v, int n) {
  if (n >= 4) {
    auto* at = reinterpret_cast<typename Four<T>::unaligned*>(p);
    if constexpr (NT) __builtin_nontemporal_store(v, at);
    else *at = v;
    return;
  }
#pragma unroll
  for (int i = 0; i < 3; ++i)
    if (i < n) p[i] = v[i];
}

__device__ inline float sqrt_(float x) { return __builtin_sqrtf(x); }
__device__ inline double sqrt_(double x) { return __builtin_sqrt(x); }

// Magnitudes as integers: their bits are in the values' order, and a NaN's
// are above every other's, so that the largest is NaN where any value is.
__device__ inline int magnitude(float x) { return __builtin_bit_cast(int, x) & 0x7fffffff; }
__device__ inline float wave_top(int b) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) b = max(b, __shfl_xor(b, off, 64));
  return __builtin_bit_cast(float, b);
}

// Codes of a lane's four values, whose block's largest magnitude is top; the
// block's scale. Hardware conversions: round to nearest even, OCP e4m3.
template <bool ROOT>
__device__ inline uint32_t encode(const float (&x)[4], float top, float* scale) {
  const bool none = top < kTiny;
  const float to = none ? 0.0f : (1.0f / top) * kCodeMax;
  *scale = none ? 0.0f : top * (1.0f / kCodeMax);
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[i] = x[i] * to;
    if (ROOT && y[i] > 0.0f && y[i] < kCodeMin) y[i] = kCodeMin;
  }
  int c = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], c, true);
}

template <int I>
__device__ inline float decode(uint32_t c) {
  return __builtin_amdgcn_cvt_f32_fp8((int)c, I);
}

// Evaluated operation by operation in P, as the header states the formula.
template <class P, class G, class C, bool BITS8, bool NT>
__global__ __launch_bounds__(kThreads) void adamw_many(const Table<P, BITS8> tb) {
  const float gs = tb.scale ? *tb.scale : 1.0f;
  if (!(gs - gs == 0.0f)) return;
  int at = 0, past = tb.n;  // the tensor whose chunks include this one
  while (past - at > 1) {
    const int mid = (at + past) / 2;
    if (tb.first[mid] <= (int)blockIdx.x) at = mid;
    else past = mid;
  }
  const Entry<P, BITS8>& e = tb.e[at];
  const Coefs<P>& k = tb.k;
  const int64_t i = (int64_t)((int)blockIdx.x - tb.first[at]) * kChunk + threadIdx.x * 4;
  const int n = (int)min((int64_t)4, e.n - i);  // this lane's values, none beyond the end
  const bool in = n > 0;

  typename Four<P>::type p{}, m32{}, v32{};
  typename Four<G>::type g{};
  P m[4], v[4], root[4];
  if constexpr (BITS8) {
    uint32_t mc = 0, vc = 0;
    float ms = 0.0f, vs = 0.0f;
    if (in) {
      p = load4<NT>((const P*)e.p + i, n);
      g = load4<NT>((const G*)e.g + i, n);
      mc = __builtin_bit_cast(uint32_t, load4<NT>((const uint8_t*)e.m + i, n));
      vc = __builtin_bit_cast(uint32_t, load4<NT>((const uint8_t*)e.v + i, n));
      ms = e.m_scale[i / kBlock];
      vs = e.v_scale[i / kBlock];
    }
    m[0] = decode<0>(mc);
    m[1] = decode<1>(mc);
    m[2] = decode<2>(mc);
    m[3] = decode<3>(mc);
    v[0] = decode<0>(vc);
    v[1] = decode<1>(vc);
    v[2] = decode<2>(vc);
    v[3] = decode<3>(vc);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      m[j] *= ms;
      v[j] *= vs;
      v[j] *= v[j];
    }
  } else {
    if (in) {
      p = load4<NT>((const P*)e.p + i, n);
      g = load4<NT>((const G*)e.g + i, n);
      m32 = load4<NT>((const P*)e.m + i, n);
      v32 = load4<NT>((const P*)e.v + i, n);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) m[j] = m32[j], v[j] = v32[j];
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const P gj = (P)up(g[j]) * (P)gs;
    m[j] = k.b1 * m[j] + k.c1 * gj;
    v[j] = k.b2 * v[j] + k.c2 * (gj * gj);
    root[j] = sqrt_(v[j]);
    const P update = m[j] / (root[j] * k.root + k.eps);
    p[j] = p[j] * e.decay - e.rate * update;
  }
  if constexpr (BITS8) {
    // lanes beyond the tensor hold zeros: they do not change the largest
    int tm = 0, tv = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      tm = max(tm, magnitude(m[j]));
      tv = max(tv, magnitude(root[j]));
    }
    float sm, sv;
    const uint32_t cm = encode<false>(m, wave_top(tm), &sm);
    const uint32_t cv = encode<true>(root, wave_top(tv), &sv);
    if (in) {
      store4<NT>((uint8_t*)e.m + i, __builtin_bit_cast(Four<uint8_t>::type, cm), n);
      store4<NT>((uint8_t*)e.v + i, __builtin_bit_cast(Four<uint8_t>::type, cv), n);
      if (threadIdx.x % 64 == 0) {
        e.m_scale[i / kBlock] = sm;
        e.v_scale[i / kBlock] = sv;
      }
    }
  } else if (in) {
#pragma unroll
    for (int j = 0; j < 4; ++j) m32[j] = m[j], v32[j] = v[j];
    store4<NT>((P*)e.m + i, m32, n);
    store4<NT>((P*)e.v + i, v32, n);
  }
  if (!in) return;
  store4<NT>((P*)e.p + i, p, n);
  if (e.copy) {
    typename Four<C>::type c;
#pragma unroll
    for (int j = 0; j < 4; ++j) c[j] = down<C>((float)p[j]);
    store4<NT>((C*)e.copy + i, c, n);
  }
}

template <class P, class G, class C, bool BITS8, bool NT>
hipError_t launch(const adst_adamw_problem& pr, const adst_adamw_tensor* t, int32_t n,
                  hipStream_t st) {
  Table<P, BITS8> tb;
  static_assert(sizeof(tb) <= kArgBytes, "the kernel's arguments");
  const double b1t = 1 - std::pow(pr.beta1, (double)pr.t);
  const double b2t = 1 - std::pow(pr.beta2, (double)pr.t);
  tb.k = {(P)pr.beta1, (P)pr.beta2, (P)(1 - pr.beta1), (P)(1 - pr.beta2),
          P(1) / (P)std::sqrt(b2t), (P)pr.eps};
  tb.scale = pr.grad_scale;
  tb.n = 0;
  int64_t chunks = 0;
  constexpr int64_t kMostChunks = (int64_t(1) << 32) / kThreads - 1;  // of a launch's grid
  for (int32_t i = 0; i < n; ++i) {
    // a tensor goes in whole, or in parts that a launch holds each
    for (int64_t from = 0; from < t[i].n;) {
      const int64_t want = (t[i].n - from + kChunk - 1) / kChunk;
      const int64_t take = want < kMostChunks ? want : kMostChunks;
      if (tb.n == Table<P, BITS8>::kMost || chunks + take > kMostChunks) {
        tb.first[tb.n] = (int)chunks;
        const hipError_t e =
            start(adamw_many<P, G, C, BITS8, NT>, (unsigned)chunks, kThreads, st, tb);
        if (e != hipSuccess) return e;
        tb.n = 0;
        chunks = 0;
      }
      const int64_t all = t[i].n - from, part = take * kChunk < all ? take * kChunk : all;
      Entry<P, BITS8>& e = tb.e[tb.n];
      e.p = (P*)t[i].p + from;
      e.g = (const G*)t[i].grad + from;
      const int64_t code = BITS8 ? 1 : (int64_t)sizeof(P);
      e.m = (char*)t[i].m + from * code;
      e.v = (char*)t[i].v + from * code;
      e.copy = t[i].copy ? (C*)t[i].copy + from : nullptr;
      e.n = part;
      e.decay = (P)(1 - t[i].lr * t[i].weight_decay);
      e.rate = (P)(t[i].lr / b1t);
      if constexpr (BITS8) {
        e.m_scale = t[i].m_scale + from / kBlock;
        e.v_scale = t[i].v_scale + from / kBlock;
      }
      tb.first[tb.n++] = (int)chunks;
      chunks += take;
      from += part;
    }
  }
  if (chunks == 0) return hipSuccess;
  tb.first[tb.n] = (int)chunks;
  return start(adamw_many<P, G, C, BITS8, NT>, (unsigned)chunks, kThreads, st, tb);
}

// Non-temporal loads and stores for calls that move more than the caches hold
// between two steps: 70 million values take 314 us with them and 350 without
// (32-bit states; 181 and 192 with 8-bit ones), 20 million 90 and 84 (56 and 51).
constexpr int64_t kStreamBytes = int64_t(768) << 20;

template <class P, class G, class C, bool BITS8>
hipError_t by_size(const adst_adamw_problem& p, const adst_adamw_tensor* t, int32_t n,
                   hipStream_t st) {
  const int64_t per = 2 * sizeof(P) + sizeof(G) + (BITS8 ? 4 : 4 * sizeof(P));
  int64_t bytes = 0;
  for (int32_t i = 0; i < n; ++i) bytes += t[i].n * (per + (t[i].copy ? (int64_t)sizeof(C) : 0));
  return bytes >= kStreamBytes ? launch<P, G, C, BITS8, true>(p, t, n, st)
                               : launch<P, G, C, BITS8, false>(p, t, n, st);
}

template <class P, class G, bool BITS8>
hipError_t by_copy(const adst_adamw_problem& p, const adst_adamw_tensor* t, int32_t n,
                   hipStream_t st) {
  if (p.copy_dtype == ADST_BF16) return by_size<P, G, bf16, BITS8>(p, t, n, st);
  if (p.copy_dtype == ADST_F16) return by_size<P, G, f16, BITS8>(p, t, n, st);
  return by_size<P, G, float, BITS8>(p, t, n, st);
}

template <class G>
hipError_t by_bits(const adst_adamw_problem& p, const adst_adamw_tensor* t, int32_t n,
                   hipStream_t st) {
  return p.bits == 8 ? by_copy<float, G, true>(p, t, n, st) : by_copy<float, G, false>(p, t, n, st);
}

}  // namespace

hipError_t adamw(const adst_adamw_problem& p, const adst_adamw_tensor* t, int32_t n,
                 hipStream_t st) {
  if (p.dtype == ADST_F64) return by_copy<double, double, false>(p, t, n, st);
  if (p.grad_dtype == ADST_F32) return by_bits<float>(p, t, n, st);
  return p.grad_dtype == ADST_BF16 ? by_bits<bf16>(p, t, n, st) : by_bits<f16>(p, t, n, st);
}

}  // namespace adst
