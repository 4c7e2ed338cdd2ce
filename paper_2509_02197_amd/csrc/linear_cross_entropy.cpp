// How the vocabulary's cross entropy is cut into pieces, and its launches by
// element type.

#include "token_kernels.h"

namespace adst {

namespace {

int64_t parts(int64_t n, int64_t by) { return (n + by - 1) / by; }
int64_t up_to(int64_t n, int64_t by) { return parts(n, by) * by; }

// g of a piece of the vocabulary, one of its two orders, where a piece has more than 1024 words:
// both then stay in the 256 MB cache between the products. With more rows than 65536 (16-bit types;
// 32768 of F32) a piece has 1024 words, whatever they take: 2 GB an order at 2^20 rows of bf16.
constexpr int64_t kPieceBytes = 128 << 20;

// The tiles of an m x n product, and the parts of its long axis (of `steps` steps) where it
// may be split: what takes the least time by the work of the CU that has the most
// tiles. The rates are those of large products measured here (F32 128, F64 55 TFLOP/s, and
// 1050 of 16-bit types with 256 x 256 tiles); smaller tiles read more of LDS for each
// product, and a CU with less than two waves a SIMD waits for its loads. (999 x 515 x 10007 F32:
// the whole step 590 us with 128 x 128 tiles everywhere, 555 with the ones chosen here. Up to 16
// rows have tiles of their own: 7 x 2383 over 52952 words F32 forward 120 us, 219 with 64 x 64.)
XentPlan::Product product_of(int64_t e, int64_t m, int64_t n, int64_t steps, bool split) {
  static const struct {
    int64_t bm, bn, waves;
    double speed;
  } tiles[] = {{256, 256, 8, 1.0}, {128, 128, 4, 0.85}, {128, 64, 4, 0.7}, {64, 64, 4, 0.5},
               {16, 128, 2, 0.3}};
  if (m <= 64 && !split) return {m <= 16 ? 4 : 3, 1};
  const double flops_per_us = (e == 2 ? 1050e6 : e == 4 ? 128e6 : 55e6) / 256;  // of a CU
  XentPlan::Product best{1, 1};
  double least = -1;
  for (int k = e == 8 ? 1 : 0; k < (m <= 16 ? 5 : 4); ++k) {
    const auto& t = tiles[k];
    const int64_t count = parts(m, t.bm) * parts(n, t.bn);
    // (the matrix cores, not LDS, bound the wider types)
    const double speed = e == 2 ? t.speed : 1 - (1 - t.speed) / 3;
    const double step = 2.0 * t.bm * t.bn * (128 / e) / flops_per_us / speed;
    for (int64_t s = 1; s == 1 || (split && s <= 64 && s <= steps / 8); ++s) {
      const int64_t of_cu = parts(count * s, 256);
      double us = (double)(of_cu * parts(steps, s)) * step;
      if (of_cu * t.waves < 8) us *= 1.3;
      if (s > 1) us += 4 + 2.0 * (double)(s * m * n * (e == 8 ? 8 : 4)) / 5e6;
      if (least < 0 || us < least) {
        least = us;
        best = {k, s};
      }
    }
  }
  return best;
}

// The logits' product: split, into tiles of 64 x 64, where those are fewer than a quarter of the
// CUs and have as many steps as take longer one after another than a launch and the sums (64
// rows over 4096 words, forward, split and not: F32 of 16 steps 20 and 21 us, of 32 22 and 33;
// bf16 of 16 18 and 15, of 32 18 and 21).
XentPlan::Product logits_of(int64_t e, int64_t M, int64_t V, int64_t steps) {
  const int64_t count = parts(M, 64) * parts(V, 64);
  if (count < 1 || count > 64 || steps < (e == 2 ? 24 : 16)) return product_of(e, M, V, steps, false);
  const int64_t fill = 256 / count;
  return {3, fill < steps / 4 ? fill : steps / 4};
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
  p.logits = logits_of(e, M, V, parts(K, step));
  if (p.logits.splits > 1) p.few = take(p.logits.splits * M * V * acc);
  if (!reverse) {
    if (p.logits.splits > 1) {
      p.bytes = at;
      return p;
    }
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
  // (few logits are one piece)
  if (p.logits.splits == 1) p.logits = product_of(e, p.m_pad, p.piece, parts(K, step), false);
  p.dx = product_of(e, M, K, p.piece / step, true);
  p.dw = product_of(e, p.piece, K, p.m_pad / step, true);
  p.dx_direct = p.pieces == 1 && p.dx.splits == 1;
  p.scale = take(2 * 4);
  p.xt = take(K * p.m_pad * e);
  p.wt = take(K * p.piece * e);
  p.g = take(M * p.piece * e);
  p.gt = take(p.piece * p.m_pad * e);
  p.dx_sums = take(p.dx_direct ? 0 : p.dx.splits * M * K * acc);
  p.dw_sums = take(p.dw.splits > 1 ? p.dw.splits * p.piece * K * acc : 0);
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
