// Launchers of the sequence operators' kernels. Arguments are checked by the
// callers (seq_abi.cpp); every launcher only enqueues and returns the launch
// status.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstdint>

#include "adst.h"

namespace adst {

struct RecArgs {
  const void* a;
  const void* u;
  const void* h0;
  const int32_t* lens;
  int64_t sa_b, sa_t, su_b, su_t;  // strides in elements: batch rows, steps
  int64_t B, T, D;
  int32_t dtype, gate;
  // forward
  void* h;
  void* hT;
  void* ck;  // [B][checkpoints][D] accumulation type
  // reverse (ck: read)
  const void* dh;
  const void* dhT;
  int64_t sd_b, sd_t;
  void* da;
  void* du;
  void* dh0;
};

struct RecPlan {
  int64_t span;  // steps between checkpoints
  bool fits;     // the launches hold the problem
  uint64_t ck_bytes, ws_bytes;
};
RecPlan rec_plan(int32_t dtype, int64_t B, int64_t T, int64_t D);
hipError_t rec_forward(const RecArgs& r, void* ws, hipStream_t st);
hipError_t rec_vjp(const RecArgs& r, void* ws, hipStream_t st);

struct RecStep {
  const void* a;
  const void* u;
  int64_t sa, su;
  const int32_t* slots;
  void* state;
  int64_t nstates;
  void* h;
  int64_t B, D;
  int32_t dtype, gate;
};
hipError_t rec_step(const RecStep& r, hipStream_t st);

struct NormArgs {
  const void* x;
  const void* dy;
  const void* w;
  const void* b;
  int64_t sx, sdy;
  int64_t rows, n;
  double eps;
  int32_t dtype, wtype;
  void* y;
  void* mean;  // written by the forward, read by the reverse
  void* rstd;
  void* dx;
  void* dw;
  void* db;
};
hipError_t norm_forward(const NormArgs& a, hipStream_t st);
uint64_t norm_workspace_bytes(int32_t dtype, int64_t rows, int64_t n);
hipError_t norm_vjp(const NormArgs& a, void* ws, hipStream_t st);

hipError_t adamw(const adst_adamw_problem& prob, const adst_adamw_tensor* tensors, int32_t n,
                 hipStream_t st);

}  // namespace adst
