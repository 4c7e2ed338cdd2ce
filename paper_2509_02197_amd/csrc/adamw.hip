// One AdamW step over many tensors, with states in the parameters' type or in
// blocks of 8-bit codes.

#include <cmath>

#include "seq_common.h"
#include "seq_kernels.h"

namespace adst {
namespace {

constexpr int kBlock = ADST_STATE_BLOCK;
constexpr float kCodeMax = 448.0f;       // the largest e4m3 value
constexpr float kCodeMin = 0x1p-9f;      // the smallest positive one
constexpr float kTiny = 0x1p-100f;

struct Coefs {
  double b1, b2, c1, c2;  // betas and 1 - beta
  double root2, eps;      // sqrt(1 - beta2^t)
  const float* scale;
};
struct OneTensor {
  adst_adamw_tensor t;
  double decay, rate;  // 1 - lr * weight_decay, lr / (1 - beta1^t)
};

__device__ inline float sqrt_(float x) { return __builtin_sqrtf(x); }
__device__ inline double sqrt_(double x) { return __builtin_sqrt(x); }

// e4m3 codes by the hardware's conversions, two at a time.
__device__ inline float code_up(uint8_t c) {
  return __builtin_amdgcn_cvt_f32_fp8((int)c, 0);
}
__device__ inline uint8_t code_down(float v) {
  return (uint8_t)(__builtin_amdgcn_cvt_pk_fp8_f32(v, 0.0f, 0, false) & 0xff);
}

// NaN where any is NaN.
__device__ inline float block_max(float v) {
  __shared__ float part[kBlock / 64];
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    const float o = __shfl_xor(v, off, 64);
    v = o != o || o > v ? o : v;
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  v = part[0];
  for (int k = 1; k < kBlock / 64; ++k) v = part[k] != part[k] || part[k] > v ? part[k] : v;
  return v;
}

__device__ inline uint8_t encode(float x, float top, bool root, float* scale) {
  const bool none = top < kTiny;
  *scale = none ? 0.0f : top / kCodeMax;
  float y = none ? 0.0f : x * (kCodeMax / top);
  if (root && y > 0.0f && y < kCodeMin) y = kCodeMin;
  return code_down(y);
}

template <class P, class G, class C, bool BITS8>
__global__ __launch_bounds__(kBlock) void adamw_one(OneTensor one, Coefs k) {
  const adst_adamw_tensor& t = one.t;
  const int64_t block = blockIdx.x, i = block * kBlock + threadIdx.x;
  const float gs = k.scale ? *k.scale : 1.0f;
  if (!(gs - gs == 0.0f)) return;
  const bool in = i < t.n;
  P p = 0, m = 0, v = 0;
  if (in) {
    p = ((const P*)t.p)[i];
    const P g = (P)up(((const G*)t.grad)[i]) * (P)gs;
    if constexpr (BITS8) {
      m = code_up(((const uint8_t*)t.m)[i]) * t.m_scale[block];
      const float r = code_up(((const uint8_t*)t.v)[i]) * t.v_scale[block];
      v = r * r;
    } else {
      m = ((const P*)t.m)[i];
      v = ((const P*)t.v)[i];
    }
    m = (P)k.b1 * m + (P)k.c1 * g;
    v = (P)k.b2 * v + (P)k.c2 * (g * g);
  }
  const P root = sqrt_(v);
  if constexpr (BITS8) {
    const float top_m = block_max(__builtin_fabsf(m)), top_v = block_max(root);
    float sm, sv;
    const uint8_t cm = encode(m, top_m, false, &sm), cv = encode(root, top_v, true, &sv);
    if (in) {
      ((uint8_t*)t.m)[i] = cm;
      ((uint8_t*)t.v)[i] = cv;
    }
    if (threadIdx.x == 0) {
      t.m_scale[block] = sm;
      t.v_scale[block] = sv;
    }
  }
  if (!in) return;
  if constexpr (!BITS8) {
    ((P*)t.m)[i] = m;
    ((P*)t.v)[i] = v;
  }
  const P update = m / (root / (P)k.root2 + (P)k.eps);
  p = p * (P)one.decay - (P)one.rate * update;
  ((P*)t.p)[i] = p;
  if (t.copy) ((C*)t.copy)[i] = down<C>((float)p);
}

template <class P, class G, bool BITS8>
void launch(const OneTensor& o, const Coefs& k, int32_t copy, hipStream_t st) {
  const unsigned blocks = (unsigned)((o.t.n + kBlock - 1) / kBlock);
  if (copy == ADST_BF16)
    adamw_one<P, G, bf16, BITS8><<<blocks, kBlock, 0, st>>>(o, k);
  else if (copy == ADST_F16)
    adamw_one<P, G, f16, BITS8><<<blocks, kBlock, 0, st>>>(o, k);
  else
    adamw_one<P, G, float, BITS8><<<blocks, kBlock, 0, st>>>(o, k);
}

}  // namespace

hipError_t adamw(const adst_adamw_problem& p, const adst_adamw_tensor* tensors, int32_t n,
                 hipStream_t st) {
  const Coefs k = {p.beta1, p.beta2, 1 - p.beta1, 1 - p.beta2,
                   std::sqrt(1 - std::pow(p.beta2, (double)p.t)), p.eps, p.grad_scale};
  for (int32_t i = 0; i < n; ++i) {
    if (tensors[i].n == 0) continue;
    OneTensor o = {tensors[i], 1 - tensors[i].lr * tensors[i].weight_decay,
                   tensors[i].lr / (1 - std::pow(p.beta1, (double)p.t))};
    if (p.dtype == ADST_F64)
      launch<double, double, false>(o, k, p.copy_dtype, st);
    else if (p.grad_dtype == ADST_F32)
      p.bits == 8 ? launch<float, float, true>(o, k, p.copy_dtype, st)
                  : launch<float, float, false>(o, k, p.copy_dtype, st);
    else if (p.grad_dtype == ADST_BF16)
      p.bits == 8 ? launch<float, bf16, true>(o, k, p.copy_dtype, st)
                  : launch<float, bf16, false>(o, k, p.copy_dtype, st);
    else
      p.bits == 8 ? launch<float, f16, true>(o, k, p.copy_dtype, st)
                  : launch<float, f16, false>(o, k, p.copy_dtype, st);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace adst
