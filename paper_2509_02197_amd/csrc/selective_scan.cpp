// How the selective scan is laid out, and its launches by element type.

#include "token_kernels.h"

namespace adst {

namespace {

int64_t up_to(int64_t n, int64_t by) { return (n + by - 1) / by; }

// Segments are cut below kEnoughWaves of the card's 1024 SIMDs, into kWaves, and are at least
// kLeastSegment steps long.
constexpr int64_t kEnoughWaves = 768, kWaves = 2048, kLeastSegment = 128;

}  // namespace

ScanGrid scan_grid(int32_t dtype, int64_t B, int64_t T, int64_t D, int64_t N, int64_t G) {
  ScanGrid g{};
  const int acc = dtype == ADST_F64 ? 8 : 4;
  const bool wide = dtype == ADST_F64;
  if (wide) {
    g.states = N <= 16 ? 2 : 4;
    g.waves = N <= 8 ? 2 : N <= 32 ? 4 : 8;
  } else {
    g.states = N <= 4 ? 1 : N <= 16 ? 2 : N <= 32 ? 4 : N <= 64 ? 8 : 16;
    g.waves = N <= 8 ? 2 : 4;
  }
  g.chunk = (wide ? 16 : 32) / (g.states < 2 ? 2 : g.states);
  g.slab = 32;
  g.chunks = up_to(T, g.chunk);
  g.group_slabs = up_to(D / G, g.slab);
  g.slabs = g.group_slabs * G;
  // Segments only where the batch's rows and channels leave SIMDs without work: a segment's
  // map is a second sweep over its inputs. 6 x 777 x 1000 F16 of 16 states, 768 waves: 63 us
  // in one segment, 52 + 29 (map) in two, 37 + 29 in four. 1 x 16384 x 2048 bf16, 256 waves:
  // 152 + 211 in eight; a wave of one segment has four times the steps of 4 x 4096 x 2048's 301.
  const int64_t waves = g.slabs * B * g.waves;
  int64_t segments = 1;
  if (waves > 0 && waves < kEnoughWaves) {
    segments = up_to(kWaves, waves);
    const int64_t most = T / kLeastSegment;
    if (segments > most) segments = most;
    if (segments < 1) segments = 1;
  }
  g.seg_chunks = up_to(g.chunks, segments);
  if (g.seg_chunks < 1) g.seg_chunks = 1;
  g.segments = up_to(g.chunks, g.seg_chunks);
  if (g.segments < 1) g.segments = 1;
  // dA's partial sums are one for each row of workgroups: many batch rows share one
  const int64_t most_rows = up_to(4096, g.slabs * g.segments > 0 ? g.slabs * g.segments : 1);
  g.rows = B < most_rows ? B : most_rows;
  if (g.rows < 1) g.rows = 1;
  const int64_t padded = 2 * g.waves * g.states;
  g.ck_bytes = (uint64_t)(B * g.chunks * N * D) * acc;
  g.map_bytes = g.segments > 1 ? (uint64_t)(up_to(B * g.segments * (N + 1) * D * acc, 16) * 16) : 0;
  g.rev_bytes = (uint64_t)(g.slabs * B * g.chunks * g.chunk * padded * 2 +
                           g.rows * g.segments * (N + 2) * D) * acc;
  const int64_t limit = int64_t(1) << 32;  // work-items of a launch
  g.fits = g.slabs * g.segments * B * g.waves * 64 < limit &&
           B * g.chunks * g.chunk * 2 * padded * G < limit && (N + 2) * D < limit;
  return g;
}

namespace {

ScanGrid grid_of(const ScanArgs& a) { return scan_grid(a.dtype, a.B, a.T, a.D_, a.N, a.G); }

}  // namespace

hipError_t scan_forward(const ScanArgs& a, void* ws, hipStream_t st) {
  const ScanGrid g = grid_of(a);
  switch (a.dtype) {
    case ADST_F64: return scan_forward_f64(a, g, ws, st);
    case ADST_F32: return scan_forward_f32(a, g, ws, st);
    case ADST_BF16: return scan_forward_bf16(a, g, ws, st);
    default: return scan_forward_f16(a, g, ws, st);
  }
}

hipError_t scan_vjp(const ScanArgs& a, void* ws, hipStream_t st) {
  const ScanGrid g = grid_of(a);
  switch (a.dtype) {
    case ADST_F64: return scan_vjp_f64(a, g, ws, st);
    case ADST_F32: return scan_vjp_f32(a, g, ws, st);
    case ADST_BF16: return scan_vjp_bf16(a, g, ws, st);
    default: return scan_vjp_f16(a, g, ws, st);
  }
}

hipError_t scan_step(const ScanStep& s, hipStream_t st) {
  switch (s.a.dtype) {
    case ADST_F64: return scan_step_f64(s, st);
    case ADST_F32: return scan_step_f32(s, st);
    case ADST_BF16: return scan_step_bf16(s, st);
    default: return scan_step_f16(s, st);
  }
}

}  // namespace adst
