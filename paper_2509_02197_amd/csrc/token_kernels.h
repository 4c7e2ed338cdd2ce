// Launchers of the token operators' kernels. Arguments are checked by the
// callers (token_abi.cpp); every launcher only enqueues and returns the launch
// status.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstdint>

#include "adst.h"

namespace adst {

struct ConvArgs {
  const void* x;
  const void* w;
  const void* bias;
  const void* x0;
  const int32_t* lens;
  int64_t sx_b, sx_t;  // strides in elements: batch rows, steps
  int64_t B, T, D;
  int32_t dtype, wtype, act, taps;
  // forward
  void* y;
  void* xT;
  // reverse
  const void* dy;
  const void* dxT;
  int64_t sd_b, sd_t;
  void* dx;
  void* dw;
  void* dbias;
  void* dx0;
};
hipError_t conv_forward(const ConvArgs& a, hipStream_t st);
uint64_t conv_workspace_bytes(int32_t dtype, int64_t B, int64_t T, int64_t D, int32_t taps);
hipError_t conv_vjp(const ConvArgs& a, void* ws, hipStream_t st);

struct ConvStep {
  const void* x;
  const void* w;
  const void* bias;
  int64_t sx;
  const int32_t* slots;
  void* window;
  int64_t nstates;
  void* y;
  int64_t B, D;
  int32_t dtype, wtype, act, taps;
};
hipError_t conv_step(const ConvStep& a, hipStream_t st);

struct ScanArgs {
  const void* x;
  const void* delta;
  const void* A;
  const void* Bm;
  const void* Cm;
  const void* D;
  const void* z;
  const void* bias;
  const void* h0;
  const int32_t* lens;
  // strides in elements: batch rows, steps
  int64_t sx_b, sx_t, sl_b, sl_t, sb_b, sb_t, sc_b, sc_t, sz_b, sz_t, sd_b, sd_t;
  int64_t B, T, D_;
  int32_t N, G, dtype, softplus;
  // forward
  void* y;
  void* hT;
  void* ck;  // [B][chunks][N][channels] accumulation type; read by the reverse
  // reverse
  const void* dy;
  const void* dhT;
  adst_scan_gradients out;
};

// How a problem is laid out: slabs of channels, chunks of steps, and segments
// of chunks that are worked on at the same time.
struct ScanGrid {
  int32_t chunk;          // steps
  int32_t slab;           // channels
  int32_t states;         // states of a lane
  int32_t waves;          // of a workgroup
  int64_t chunks;         // of a batch row
  int64_t group_slabs;    // of a group of channels
  int64_t slabs;          // of a batch row
  int64_t seg_chunks;     // chunks of a segment
  int64_t segments;       // of a batch row
  int64_t rows;           // of workgroups along the batch in the reverse sweep
  uint64_t ck_bytes;
  uint64_t map_bytes;     // segments' maps
  uint64_t rev_bytes;     // the reverse sweep's sums
  bool fits;
};
ScanGrid scan_grid(int32_t dtype, int64_t B, int64_t T, int64_t D, int64_t N, int64_t G);
hipError_t scan_forward(const ScanArgs& a, void* ws, hipStream_t st);
hipError_t scan_vjp(const ScanArgs& a, void* ws, hipStream_t st);

struct ScanStep {
  ScanArgs a;  // x, delta, A, Bm, Cm, D, z, bias, y and the strides along the batch
  const int32_t* slots;
  void* state;
  int64_t nstates;
};
hipError_t scan_step(const ScanStep& s, hipStream_t st);

// By type: each is compiled by itself.
#define ADST_SCAN_OF(type)                                                                     \
  hipError_t scan_forward_##type(const ScanArgs& a, const ScanGrid& g, void* ws, hipStream_t st); \
  hipError_t scan_vjp_##type(const ScanArgs& a, const ScanGrid& g, void* ws, hipStream_t st);     \
  hipError_t scan_step_##type(const ScanStep& s, hipStream_t st);
ADST_SCAN_OF(f64)
ADST_SCAN_OF(f32)
ADST_SCAN_OF(bf16)
ADST_SCAN_OF(f16)

struct XentArgs {
  const void* x;
  const void* w;
  int64_t sx, sw;  // elements between rows
  int64_t M, V, K; // rows, vocabulary, width
  const int32_t* labels;
  int32_t dtype;
  void* loss;
  void* lse;       // written by the forward, read by the reverse
  const void* dloss;
  void* dx;
  void* dw;
};

// Sizes and the workspace's parts (bytes from its start). Rows and pieces that
// are the long axis of a product are padded to whole steps of it (128 bytes).
struct XentPlan {
  int64_t piece, pieces;   // of the vocabulary: columns (padded) and their number
  int64_t m_pad;           // rows, padded
  // each product's tiles, and the parts of its long axis that are summed afterwards
  struct Product {
    int tiles;  // 0: 256 x 256, 1: 128 x 128, 2: 128 x 64; for few rows 3: 64 x 64, 4: 16 x 128
    int64_t splits;
  } logits, dx, dw;
  bool dx_direct;          // dx leaves its product in the element type
  uint64_t stats, target, scale, xt, wt, g, gt, dx_sums, dw_sums;
  uint64_t few;            // the logits' sums, where their product is split
  uint64_t bytes;
};
XentPlan xent_plan(int32_t dtype, int64_t M, int64_t V, int64_t K, bool reverse);
hipError_t xent_forward(const XentArgs& a, void* ws, hipStream_t st);
hipError_t xent_vjp(const XentArgs& a, void* ws, hipStream_t st);

#define ADST_XENT_OF(type)                                                                       \
  hipError_t xent_forward_##type(const XentArgs& a, const XentPlan& p, void* ws, hipStream_t st); \
  hipError_t xent_vjp_##type(const XentArgs& a, const XentPlan& p, void* ws, hipStream_t st);
ADST_XENT_OF(f64)
ADST_XENT_OF(f32)
ADST_XENT_OF(bf16)
ADST_XENT_OF(f16)

}  // namespace adst
