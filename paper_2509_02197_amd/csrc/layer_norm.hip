// Layer norm over rows, its VJP, and the weights' gradients summed over rows.

#include "seq_common.h"
#include "seq_kernels.h"

namespace adst {
namespace {

constexpr int kThreads = 256;
constexpr int kParts = 256;  // row groups of the weights' gradients

template <class A>
__device__ inline A block_sum(A v) {
  __shared__ A part[kThreads / 64];
  v = lane_sum<64>(v);
  __syncthreads();  // earlier sums are read
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  return (part[0] + part[1]) + (part[2] + part[3]);
}

__device__ inline float sqrt_(float x) { return __builtin_sqrtf(x); }
__device__ inline double sqrt_(double x) { return __builtin_sqrt(x); }

template <class T, class W>
__global__ __launch_bounds__(kThreads) void norm_fwd(NormArgs p) {
  typedef Acc<T> A;
  const int64_t row = blockIdx.x;
  const T* x = (const T*)p.x + row * p.sx;
  T* y = (T*)p.y + row * p.n;
  A s = 0;
  for (int64_t i = threadIdx.x; i < p.n; i += kThreads) s += up(x[i]);
  const A mean = block_sum(s) / A(p.n);
  s = 0;
  for (int64_t i = threadIdx.x; i < p.n; i += kThreads) {
    const A d = up(x[i]) - mean;
    s = fma_(d, d, s);
  }
  const A rstd = A(1) / sqrt_(block_sum(s) / A(p.n) + A(p.eps));
  for (int64_t i = threadIdx.x; i < p.n; i += kThreads) {
    const A w = p.w ? (A)up(((const W*)p.w)[i]) : A(1), b = p.b ? (A)up(((const W*)p.b)[i]) : A(0);
    y[i] = down<T>(fma_((up(x[i]) - mean) * rstd, w, b));
  }
  if (threadIdx.x == 0) {
    if (p.mean) ((A*)p.mean)[row] = mean;
    if (p.rstd) ((A*)p.rstd)[row] = rstd;
  }
}

template <class T, class W>
__global__ __launch_bounds__(kThreads) void norm_dx(NormArgs p) {
  typedef Acc<T> A;
  const int64_t row = blockIdx.x;
  const T* x = (const T*)p.x + row * p.sx;
  const T* dy = (const T*)p.dy + row * p.sdy;
  T* dx = (T*)p.dx + row * p.n;
  const A mean = ((const A*)p.mean)[row], rstd = ((const A*)p.rstd)[row];
  A s = 0, q = 0;
  for (int64_t i = threadIdx.x; i < p.n; i += kThreads) {
    const A w = p.w ? (A)up(((const W*)p.w)[i]) : A(1);
    const A e = up(dy[i]) * w;
    s += e;
    q = fma_(e, (up(x[i]) - mean) * rstd, q);
  }
  s = block_sum(s) / A(p.n);
  q = block_sum(q) / A(p.n);
  for (int64_t i = threadIdx.x; i < p.n; i += kThreads) {
    const A w = p.w ? (A)up(((const W*)p.w)[i]) : A(1);
    const A e = up(dy[i]) * w;
    dx[i] = down<T>(fma_(-q, (up(x[i]) - mean) * rstd, e - s) * rstd);
  }
}

// Partial sums of dw and db of rows blockIdx.y, + kParts, ..., one column a thread.
template <class T>
__global__ __launch_bounds__(kThreads) void norm_dw_part(NormArgs p, Acc<T>* part) {
  typedef Acc<T> A;
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i >= p.n) return;
  A sw = 0, sb = 0;
  for (int64_t row = blockIdx.y; row < p.rows; row += kParts) {
    const A d = up(((const T*)p.dy)[row * p.sdy + i]);
    const A xh = (up(((const T*)p.x)[row * p.sx + i]) - ((const A*)p.mean)[row]) *
                 ((const A*)p.rstd)[row];
    sw = fma_(d, xh, sw);
    sb += d;
  }
  part[(2 * (int64_t)blockIdx.y) * p.n + i] = sw;
  part[(2 * (int64_t)blockIdx.y + 1) * p.n + i] = sb;
}

template <class T, class W>
__global__ __launch_bounds__(kThreads) void norm_dw_sum(NormArgs p, const Acc<T>* part, int parts) {
  typedef Acc<T> A;
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i >= p.n) return;
  A sw = 0, sb = 0;
  for (int64_t k = 0; k < parts; ++k) {
    sw += part[2 * k * p.n + i];
    sb += part[(2 * k + 1) * p.n + i];
  }
  if (p.dw) ((W*)p.dw)[i] = down<W>(sw);
  if (p.db) ((W*)p.db)[i] = down<W>(sb);
}

template <class F>
hipError_t by_type(int32_t dtype, int32_t wtype, F f) {
  switch (dtype) {
    case ADST_F64: f(double(), double()); break;
    case ADST_F32: f(float(), float()); break;
    case ADST_BF16:
      if (wtype == ADST_F32) f(bf16(), float());
      else f(bf16(), bf16());
      break;
    default:
      if (wtype == ADST_F32) f(f16(), float());
      else f(f16(), f16());
      break;
  }
  return hipGetLastError();
}

int parts_of(int64_t rows) { return (int)(rows < kParts ? rows : kParts); }

}  // namespace

hipError_t norm_forward(const NormArgs& a, hipStream_t st) {
  return by_type(a.dtype, a.wtype, [&](auto t, auto w) {
    norm_fwd<decltype(t), decltype(w)><<<(unsigned)a.rows, kThreads, 0, st>>>(a);
  });
}

uint64_t norm_workspace_bytes(int32_t dtype, int64_t rows, int64_t n) {
  return 2ull * parts_of(rows) * (uint64_t)n * (dtype == ADST_F64 ? 8 : 4);
}

hipError_t norm_vjp(const NormArgs& a, void* ws, hipStream_t st) {
  return by_type(a.dtype, a.wtype, [&](auto t, auto w) {
    typedef decltype(t) T;
    typedef decltype(w) W;
    if (a.dx && a.rows > 0) norm_dx<T, W><<<(unsigned)a.rows, kThreads, 0, st>>>(a);
    if (a.dw || a.db) {
      const int parts = parts_of(a.rows);
      const unsigned cols = (unsigned)((a.n + kThreads - 1) / kThreads);
      Acc<T>* part = (Acc<T>*)ws;
      if (parts > 0)
        norm_dw_part<T><<<dim3(cols, parts), kThreads, 0, st>>>(a, part);
      norm_dw_sum<T, W><<<cols, kThreads, 0, st>>>(a, part, parts);
    }
  });
}

}  // namespace adst
