// How the vocabulary's cross entropy is cut into pieces, and its launches by
// element type.

#include "token_kernels.h"

namespace adst {

namespace {

int64_t parts(int64_t n, int64_t by) { return (n + by - 1) / by; }
int64_t up_to(int64_t n, int64_t by) { return parts(n, by) * by; }

// g of a piece of the vocabulary, one of its two orders, at most: both then stay in the
// 256 MB cache between the products.
constexpr int64_t kPieceBytes = 128 << 20;

// Parts of the long axis of an m x n product whose tiles leave CUs without work.
int64_t splits_of(int64_t m, int64_t n, int64_t steps) {
  const int64_t tiles = parts(m, 128) * parts(n, 128);
  int64_t s = tiles >= 192 ? 1 : 256 / tiles;
  if (s > steps / 8) s = steps / 8;
  return s < 1 ? 1 : s;
}

}  // namespace

XentPlan xent_plan(int32_t dtype, int64_t M, int64_t V, int64_t K, bool reverse) {
  XentPlan p{};
  const int64_t e = dtype == ADST_F64 ? 8 : dtype == ADST_F32 ? 4 : 2, acc = e == 8 ? 8 : 4;
  const int64_t step = 128 / e;
  p.m_pad = up_to(M, step);
  uint64_t at = 0;
  const auto take = [&](int64_t bytes) {
    const uint64_t here = at;
    at += (uint64_t)up_to(bytes, 256);
    return here;
  };
  if (!reverse) {
    p.stats = take(parts(V, 64) * M * 2 * acc);
    p.target = take(M * acc);
    p.bytes = at;
    return p;
  }
  int64_t most = kPieceBytes / (e * (M > 0 ? M : 1)) / 256 * 256;
  if (most < 1024) most = 1024;
  p.pieces = parts(V, most);
  p.piece = up_to(parts(V, p.pieces), p.pieces > 1 ? 256 : step);
  p.pieces = parts(V, p.piece);
  p.dx_splits = splits_of(M, K, p.piece / step);
  p.dw_splits = splits_of(p.piece, K, p.m_pad / step);
  p.dx_direct = p.pieces == 1 && p.dx_splits == 1;
  p.scale = take(2 * 4);
  p.xt = take(K * p.m_pad * e);
  p.wt = take(K * p.piece * e);
  p.g = take(M * p.piece * e);
  p.gt = take(p.piece * p.m_pad * e);
  p.dx_sums = take(p.dx_direct ? 0 : p.dx_splits * M * K * acc);
  p.dw_sums = take(p.dw_splits > 1 ? p.dw_splits * p.piece * K * acc : 0);
  p.bytes = at;
  return p;
}

hipError_t xent_forward(const XentArgs& a, void* ws, hipStream_t st) {
  const XentPlan p = xent_plan(a.dtype, a.M, a.V, a.K, false);
  switch (a.dtype) {
    case ADST_F64: return xent_forward_f64(a, p, ws, st);
    case ADST_F32: return xent_forward_f32(a, p, ws, st);
    case ADST_BF16: return xent_forward_bf16(a, p, ws, st);
    default: return xent_forward_f16(a, p, ws, st);
  }
}

hipError_t xent_vjp(const XentArgs& a, void* ws, hipStream_t st) {
  const XentPlan p = xent_plan(a.dtype, a.M, a.V, a.K, true);
  switch (a.dtype) {
    case ADST_F64: return xent_vjp_f64(a, p, ws, st);
    case ADST_F32: return xent_vjp_f32(a, p, ws, st);
    case ADST_BF16: return xent_vjp_bf16(a, p, ws, st);
    default: return xent_vjp_f16(a, p, ws, st);
  }
}

}  // namespace adst
