// Gated linear recurrence: h_t = c_t h_{t-1} + d_t per channel, with
// (c, d) = (a, u) or (s, (1 - s) u), s = 1 / (1 + exp(-a)); its VJP, which
// recomputes the states from checkpoints; and one step on a pool of states.

#include "seq_common.h"
#include "seq_kernels.h"

namespace adst {
namespace {

constexpr int kThreads = 64;
constexpr int kSpan = 16;  // steps between checkpoints: a thread keeps their states

__device__ inline float exp_(float x) { return expf(x); }
__device__ inline double exp_(double x) { return exp(x); }

// s = 1 / (1 + exp(-a)) and q = 1 - s = 1 / (1 + exp(a)), each to full
// relative precision: with e = exp(-|a|) in [0, 1] nothing overflows.
template <class A>
__device__ inline void sigmoid(A a, A* s, A* q) {
  const A e = exp_(-__builtin_elementwise_abs(a));
  const A big = A(1) / (A(1) + e), small = e * big;
  *s = a >= A(0) ? big : small;
  *q = a >= A(0) ? small : big;
}

__device__ inline int64_t row_length(const int32_t* lens, int64_t b, int64_t T) {
  if (!lens) return T;
  const int64_t n = lens[b];
  return n < 0 ? 0 : n > T ? T : n;
}

template <class T, bool SIG>
__global__ __launch_bounds__(kThreads) void rec_fwd(RecArgs r, int64_t spans) {
  typedef Acc<T> A;
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i >= r.B * r.D) return;
  const int64_t b = i / r.D, d = i % r.D;
  const T* a = (const T*)r.a + b * r.sa_b + d;
  const T* u = (const T*)r.u + b * r.su_b + d;
  T* h = r.h ? (T*)r.h + b * r.T * r.D + d : nullptr;
  A* ck = r.ck ? (A*)r.ck + b * spans * r.D + d : nullptr;
  const int64_t n = row_length(r.lens, b, r.T);
  A x = r.h0 ? ((const A*)r.h0)[i] : A(0);
  for (int64_t t = 0; t < n; ++t) {
    if (ck && t % kSpan == 0) ck[t / kSpan * r.D] = x;
    A c = up(a[t * r.sa_t]), v = up(u[t * r.su_t]);
    if (SIG) {
      A s, q;
      sigmoid(c, &s, &q);
      c = s;
      v = q * v;
    }
    x = fma_(c, x, v);
    if (h) h[t * r.D] = down<T>(x);
  }
  if (h)
    for (int64_t t = n; t < r.T; ++t) h[t * r.D] = T(0);
  if (r.hT) ((A*)r.hT)[i] = x;
}

template <class T, bool SIG>
__global__ __launch_bounds__(kThreads) void rec_rev(RecArgs r, int64_t spans) {
  typedef Acc<T> A;
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i >= r.B * r.D) return;
  const int64_t b = i / r.D, d = i % r.D;
  const T* a = (const T*)r.a + b * r.sa_b + d;
  const T* u = (const T*)r.u + b * r.su_b + d;
  const T* dh = (const T*)r.dh + b * r.sd_b + d;
  T* da = (T*)r.da + b * r.T * r.D + d;
  T* du = (T*)r.du + b * r.T * r.D + d;
  const A* ck = (const A*)r.ck + b * spans * r.D + d;
  const int64_t n = row_length(r.lens, b, r.T);
  for (int64_t t = n; t < r.T; ++t) da[t * r.D] = du[t * r.D] = T(0);
  A carry = r.dhT ? ((const A*)r.dhT)[i] : A(0);
  for (int64_t k = (n + kSpan - 1) / kSpan - 1; k >= 0; --k) {
    A old[kSpan];
    A x = ck[k * r.D];
#pragma unroll
    for (int j = 0; j < kSpan; ++j) {
      const int64_t t = k * kSpan + j;
      old[j] = x;
      if (t < n) {
        A c = up(a[t * r.sa_t]), v = up(u[t * r.su_t]);
        if (SIG) {
          A s, q;
          sigmoid(c, &s, &q);
          c = s;
          v = q * v;
        }
        x = fma_(c, x, v);
      }
    }
#pragma unroll
    for (int j = kSpan - 1; j >= 0; --j) {
      const int64_t t = k * kSpan + j;
      if (t >= n) continue;
      const A g = up(dh[t * r.sd_t]) + carry;
      A c = up(a[t * r.sa_t]);
      if (SIG) {
        A s, q;
        sigmoid(c, &s, &q);
        da[t * r.D] = down<T>(g * ((old[j] - up(u[t * r.su_t])) * (s * q)));
        du[t * r.D] = down<T>(g * q);
        c = s;
      } else {
        da[t * r.D] = down<T>(g * old[j]);
        du[t * r.D] = down<T>(g);
      }
      carry = c * g;
    }
  }
  if (r.dh0) ((A*)r.dh0)[i] = carry;
}

template <class T, bool SIG>
__global__ __launch_bounds__(kThreads) void rec_one(RecStep r) {
  typedef Acc<T> A;
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i >= r.B * r.D) return;
  const int64_t b = i / r.D, d = i % r.D;
  const int64_t slot = r.slots ? r.slots[b] : b;
  A x = A(0);
  if (slot >= 0 && slot < r.nstates) {
    A* at = (A*)r.state + slot * r.D + d;
    A c = up(((const T*)r.a)[b * r.sa + d]), v = up(((const T*)r.u)[b * r.su + d]);
    if (SIG) {
      A s, q;
      sigmoid(c, &s, &q);
      c = s;
      v = q * v;
    }
    x = fma_(c, *at, v);
    *at = x;
  }
  if (r.h) ((T*)r.h)[i] = down<T>(x);
}

template <class F>
hipError_t by_type(int32_t dtype, F f) {
  switch (dtype) {
    case ADST_F64: f(double()); break;
    case ADST_F32: f(float()); break;
    case ADST_BF16: f(bf16()); break;
    default: f(f16()); break;
  }
  return hipGetLastError();
}

unsigned blocks(int64_t n) { return (unsigned)((n + kThreads - 1) / kThreads); }

}  // namespace

RecPlan rec_plan(int32_t dtype, int64_t B, int64_t T, int64_t D) {
  RecPlan p;
  p.span = kSpan;
  p.spans = T > 0 ? (T + kSpan - 1) / kSpan : 1;
  p.ck_bytes = (uint64_t)(B * D * p.spans) * (dtype == ADST_F64 ? 8 : 4);
  p.ws_bytes = 0;
  p.fits = B * D < (int64_t(1) << 31);
  return p;
}

hipError_t rec_forward(const RecArgs& r, void*, hipStream_t st) {
  const RecPlan p = rec_plan(r.dtype, r.B, r.T, r.D);
  return by_type(r.dtype, [&](auto t) {
    typedef decltype(t) T;
    if (r.gate == ADST_GATE_SIGMOID)
      rec_fwd<T, true><<<blocks(r.B * r.D), kThreads, 0, st>>>(r, p.spans);
    else
      rec_fwd<T, false><<<blocks(r.B * r.D), kThreads, 0, st>>>(r, p.spans);
  });
}

hipError_t rec_vjp(const RecArgs& r, void*, hipStream_t st) {
  const RecPlan p = rec_plan(r.dtype, r.B, r.T, r.D);
  return by_type(r.dtype, [&](auto t) {
    typedef decltype(t) T;
    if (r.gate == ADST_GATE_SIGMOID)
      rec_rev<T, true><<<blocks(r.B * r.D), kThreads, 0, st>>>(r, p.spans);
    else
      rec_rev<T, false><<<blocks(r.B * r.D), kThreads, 0, st>>>(r, p.spans);
  });
}

hipError_t rec_step(const RecStep& r, hipStream_t st) {
  return by_type(r.dtype, [&](auto t) {
    typedef decltype(t) T;
    if (r.gate == ADST_GATE_SIGMOID)
      rec_one<T, true><<<blocks(r.B * r.D), kThreads, 0, st>>>(r);
    else
      rec_one<T, false><<<blocks(r.B * r.D), kThreads, 0, st>>>(r);
  });
}

}  // namespace adst
