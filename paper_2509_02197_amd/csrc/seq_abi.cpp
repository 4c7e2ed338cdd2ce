// C boundary of the sequence operators: every argument is checked before the
// first HIP call, and nothing here throws.

#include <hip/hip_runtime_api.h>

#include <cmath>
#include <cstdarg>
#include <cstdint>
#include <cstdio>

#include "adst.h"
#include "errors.h"
#include "seq_kernels.h"

namespace adst {
namespace {

typedef __int128 Wide;  // extents are products of caller-given 64-bit numbers

adst_status fail(adst_status st, const char* format, ...) {
  char text[256];
  va_list v;
  va_start(v, format);
  std::vsnprintf(text, sizeof(text), format, v);
  va_end(v);
  return report(st, text);
}

adst_status done(hipError_t e, const char* what) {
  if (e != hipSuccess) return fail(ADST_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
  return report_ok();
}

bool known(int32_t dtype) { return dtype >= ADST_F64 && dtype <= ADST_F16; }
int size_of(int32_t dtype) { return dtype == ADST_F64 ? 8 : dtype == ADST_F32 ? 4 : 2; }
int acc_size(int32_t dtype) { return dtype == ADST_F64 ? 8 : 4; }

// The arrays of one call: each output overlaps no other array, except where
// `same` allows it.
class Ranges {
 public:
  void in(const char* name, const void* p, Wide bytes) { add(name, p, bytes, false); }
  void out(const char* name, const void* p, Wide bytes) { add(name, p, bytes, true); }
  adst_status check() const {
    if (wild_) return fail(ADST_ERR_ARG, "%s: more bytes than the address space", wild_);
    for (int i = 0; i < n_; ++i)
      for (int j = 0; j < i; ++j) {
        if (!r_[i].out && !r_[j].out) continue;
        if (r_[i].lo < r_[j].hi && r_[j].lo < r_[i].hi && r_[i].lo != r_[i].hi &&
            r_[j].lo != r_[j].hi)
          return fail(ADST_ERR_ARG, "%s and %s overlap", r_[j].name, r_[i].name);
      }
    return ADST_OK;
  }

 private:
  struct One {
    const char* name;
    Wide lo, hi;
    bool out;
  };
  One r_[16];
  int n_ = 0;
  const char* wild_ = nullptr;
  void add(const char* name, const void* p, Wide bytes, bool out) {
    if (bytes > (Wide(1) << 62)) wild_ = name;
    if (!p) return;
    const Wide lo = (Wide)reinterpret_cast<uintptr_t>(p);
    r_[n_++] = {name, lo, lo + bytes, out};
  }
};

// Bytes that [batch][steps][channels] with these strides spans.
Wide span_bytes(int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t n2, int size) {
  if (n0 == 0 || n1 == 0 || n2 == 0) return 0;
  return (Wide(n0 - 1) * s0 + Wide(n1 - 1) * s1 + n2) * size;
}

bool aligned(const void* p, int size) { return reinterpret_cast<uintptr_t>(p) % size == 0; }

constexpr int64_t kMost = (int64_t(1) << 31) - (1 << 16);

adst_status check_recurrence(const adst_recurrence_problem* p, RecPlan* plan) {
  if (!p) return fail(ADST_ERR_ARG, "problem is NULL");
  if (!known(p->dtype)) return fail(ADST_ERR_ARG, "unknown dtype %d", p->dtype);
  if (p->gate != ADST_GATE_COEFF && p->gate != ADST_GATE_SIGMOID)
    return fail(ADST_ERR_ARG, "unknown gate %d", p->gate);
  if (p->batch < 0 || p->steps < 0 || p->channels < 0)
    return fail(ADST_ERR_ARG, "batch, steps and channels must be >= 0");
  for (int i = 0; i < 2; ++i)
    if (p->stride_a[i] < 0 || p->stride_u[i] < 0 || p->stride_dh[i] < 0)
      return fail(ADST_ERR_ARG, "strides must be >= 0");
  if (p->steps >= kMost || p->channels >= kMost || p->batch >= kMost)
    return fail(ADST_ERR_UNSUPPORTED, "batch, steps and channels must be below 2^31 - 2^16");
  if (Wide(p->batch) * p->channels * (p->steps + 1) > (Wide(1) << 58))
    return fail(ADST_ERR_UNSUPPORTED, "more values than the address space");
  *plan = rec_plan(p->dtype, p->batch, p->steps, p->channels);
  if (!plan->fits) return fail(ADST_ERR_UNSUPPORTED, "more spans than one launch holds");
  return ADST_OK;
}

RecArgs rec_args(const adst_recurrence_problem* p, const void* a, const void* u, const void* h0,
                 const int32_t* lens) {
  RecArgs r{};
  r.a = a;
  r.u = u;
  r.h0 = h0;
  r.lens = lens;
  r.sa_b = p->stride_a[0];
  r.sa_t = p->stride_a[1];
  r.su_b = p->stride_u[0];
  r.su_t = p->stride_u[1];
  r.sd_b = p->stride_dh[0];
  r.sd_t = p->stride_dh[1];
  r.B = p->batch;
  r.T = p->steps;
  r.D = p->channels;
  r.dtype = p->dtype;
  r.gate = p->gate;
  return r;
}

void rec_inputs(const adst_recurrence_problem* p, const void* a, const void* u, const void* h0,
                const int32_t* lens, Ranges* rs) {
  const int e = size_of(p->dtype), s = acc_size(p->dtype);
  const Wide state = Wide(p->batch) * p->channels * s;
  rs->in("a", a, span_bytes(p->batch, p->stride_a[0], p->steps, p->stride_a[1], p->channels, e));
  rs->in("u", u, span_bytes(p->batch, p->stride_u[0], p->steps, p->stride_u[1], p->channels, e));
  rs->in("h0", h0, state);
  rs->in("lens", lens, Wide(p->batch) * 4);
}

adst_status check_aligned(const char* name, const void* p, int size) {
  if (p && !aligned(p, size))
    return fail(ADST_ERR_ARG, "%s is not aligned to its elements of %d bytes", name, size);
  return ADST_OK;
}

#define CHECK(call)                       \
  do {                                    \
    const adst_status st_ = (call);       \
    if (st_ != ADST_OK) return st_;       \
  } while (0)

adst_status check_norm(const adst_norm_problem* p) {
  if (!p) return fail(ADST_ERR_ARG, "problem is NULL");
  if (!known(p->dtype)) return fail(ADST_ERR_ARG, "unknown dtype %d", p->dtype);
  const bool half = p->dtype == ADST_BF16 || p->dtype == ADST_F16;
  if (p->weight_dtype != p->dtype && !(half && p->weight_dtype == ADST_F32))
    return fail(ADST_ERR_ARG, "weight_dtype must be the dtype, or F32 beside BF16 and F16");
  if (p->rows < 0 || p->n < 1) return fail(ADST_ERR_ARG, "rows must be >= 0 and n >= 1");
  if (p->stride_x < 0 || p->stride_dy < 0) return fail(ADST_ERR_ARG, "strides must be >= 0");
  if (!std::isfinite(p->eps) || p->eps < 0)
    return fail(ADST_ERR_ARG, "eps must be finite and >= 0");
  if (p->rows >= kMost || p->n >= kMost)
    return fail(ADST_ERR_UNSUPPORTED, "rows and n must be below 2^31 - 2^16");
  return ADST_OK;
}

NormArgs norm_args(const adst_norm_problem* p) {
  NormArgs a{};
  a.sx = p->stride_x;
  a.sdy = p->stride_dy;
  a.rows = p->rows;
  a.n = p->n;
  a.eps = p->eps;
  a.dtype = p->dtype;
  a.wtype = p->weight_dtype;
  return a;
}

}  // namespace
}  // namespace adst

using namespace adst;

extern "C" {

adst_status adst_recurrence_plan(const adst_recurrence_problem* prob, adst_recurrence_info* out) {
  if (!out) return fail(ADST_ERR_ARG, "out is NULL");
  RecPlan plan;
  CHECK(check_recurrence(prob, &plan));
  out->span = plan.span;
  out->ck_bytes = plan.ck_bytes;
  out->workspace_bytes = plan.ws_bytes;
  out->vjp_workspace_bytes = plan.ws_bytes + plan.ck_bytes;
  return report_ok();
}

adst_status adst_recurrence_forward(const adst_recurrence_problem* prob, const void* a,
                                    const void* u, const void* h0, const int32_t* lens, void* h,
                                    void* hT, void* ck, void* ws, uint64_t ws_bytes,
                                    hipStream_t stream) {
  RecPlan plan;
  CHECK(check_recurrence(prob, &plan));
  const adst_recurrence_problem& p = *prob;
  const int e = size_of(p.dtype), s = acc_size(p.dtype);
  const bool some = p.batch > 0 && p.steps > 0 && p.channels > 0;
  if (some && (!a || !u)) return fail(ADST_ERR_ARG, "a and u are required");
  CHECK(check_aligned("a", a, e));
  CHECK(check_aligned("u", u, e));
  CHECK(check_aligned("h", h, e));
  CHECK(check_aligned("h0", h0, s));
  CHECK(check_aligned("hT", hT, s));
  CHECK(check_aligned("ck", ck, s));
  CHECK(check_aligned("lens", lens, 4));
  if (plan.ws_bytes && (!ws || ws_bytes < plan.ws_bytes))
    return fail(ADST_ERR_WORKSPACE, "adst_recurrence_forward needs %llu workspace bytes",
                (unsigned long long)plan.ws_bytes);
  if (plan.ws_bytes) CHECK(check_aligned("ws", ws, 16));
  Ranges rs;
  rec_inputs(prob, a, u, h0, lens, &rs);
  rs.out("h", h, Wide(p.batch) * p.steps * p.channels * e);
  rs.out("hT", hT, Wide(p.batch) * p.channels * s);
  rs.out("ck", ck, plan.ck_bytes);
  if (plan.ws_bytes) rs.out("ws", ws, plan.ws_bytes);
  CHECK(rs.check());
  if (p.batch == 0 || p.channels == 0) return report_ok();
  RecArgs r = rec_args(prob, a, u, h0, lens);
  r.h = h;
  r.hT = hT;
  r.ck = ck;
  return done(rec_forward(r, ws, stream), "recurrence");
}

adst_status adst_recurrence_vjp(const adst_recurrence_problem* prob, const void* a, const void* u,
                                const void* h0, const int32_t* lens, const void* ck,
                                const void* dh, const void* dhT, void* da, void* du, void* dh0,
                                void* ws, uint64_t ws_bytes, hipStream_t stream) {
  RecPlan plan;
  CHECK(check_recurrence(prob, &plan));
  const adst_recurrence_problem& p = *prob;
  const int e = size_of(p.dtype), s = acc_size(p.dtype);
  const bool some = p.batch > 0 && p.steps > 0 && p.channels > 0;
  if (some && (!a || !u || !dh || !da || !du))
    return fail(ADST_ERR_ARG, "a, u, dh, da and du are required");
  CHECK(check_aligned("a", a, e));
  CHECK(check_aligned("u", u, e));
  CHECK(check_aligned("dh", dh, e));
  CHECK(check_aligned("da", da, e));
  CHECK(check_aligned("du", du, e));
  CHECK(check_aligned("h0", h0, s));
  CHECK(check_aligned("ck", ck, s));
  CHECK(check_aligned("dhT", dhT, s));
  CHECK(check_aligned("dh0", dh0, s));
  CHECK(check_aligned("lens", lens, 4));
  const uint64_t need = plan.ws_bytes + (ck ? 0 : plan.ck_bytes);
  if (need && (!ws || ws_bytes < need))
    return fail(ADST_ERR_WORKSPACE, "adst_recurrence_vjp needs %llu workspace bytes",
                (unsigned long long)need);
  if (need) CHECK(check_aligned("ws", ws, 16));
  Ranges rs;
  const Wide state = Wide(p.batch) * p.channels * s;
  const Wide values = Wide(p.batch) * p.steps * p.channels * e;
  rec_inputs(prob, a, u, h0, lens, &rs);
  rs.in("dh", dh, span_bytes(p.batch, p.stride_dh[0], p.steps, p.stride_dh[1], p.channels, e));
  rs.in("dhT", dhT, state);
  rs.in("ck", ck, plan.ck_bytes);
  rs.out("da", da, values);
  rs.out("du", du, values);
  rs.out("dh0", dh0, state);
  if (need) rs.out("ws", ws, need);
  CHECK(rs.check());
  if (p.batch == 0 || p.channels == 0) return report_ok();
  RecArgs r = rec_args(prob, a, u, h0, lens);
  char* const at = static_cast<char*>(ws);
  if (!ck) {  // the states again, from the start: checkpoints only
    r.ck = at + plan.ws_bytes;
    const hipError_t err = rec_forward(r, ws, stream);
    if (err != hipSuccess) return done(err, "recurrence");
  } else {
    r.ck = const_cast<void*>(ck);
  }
  r.dh = dh;
  r.dhT = dhT;
  r.da = da;
  r.du = du;
  r.dh0 = dh0;
  return done(rec_vjp(r, ws, stream), "recurrence gradient");
}

adst_status adst_recurrence_step(const adst_recurrence_problem* prob, const void* a, const void* u,
                                 const int32_t* slots, void* state, int64_t nstates, void* h,
                                 hipStream_t stream) {
  RecPlan plan;
  CHECK(check_recurrence(prob, &plan));
  const adst_recurrence_problem& p = *prob;
  const int e = size_of(p.dtype), s = acc_size(p.dtype);
  if (p.steps != 1) return fail(ADST_ERR_ARG, "steps must be 1");
  if (nstates < 0 || (!slots && nstates < p.batch))
    return fail(ADST_ERR_ARG, "nstates must be >= 0, and >= batch without slots");
  const bool some = p.batch > 0 && p.channels > 0;
  if (some && (!a || !u || (nstates > 0 && !state)))
    return fail(ADST_ERR_ARG, "a, u and state are required");
  CHECK(check_aligned("a", a, e));
  CHECK(check_aligned("u", u, e));
  CHECK(check_aligned("h", h, e));
  CHECK(check_aligned("state", state, s));
  CHECK(check_aligned("slots", slots, 4));
  Ranges rs;
  rec_inputs(prob, a, u, nullptr, nullptr, &rs);
  rs.in("slots", slots, Wide(p.batch) * 4);
  rs.out("state", state, Wide(nstates) * p.channels * s);
  rs.out("h", h, Wide(p.batch) * p.channels * e);
  CHECK(rs.check());
  if (!some) return report_ok();
  RecStep r{a,       u, p.stride_a[0], p.stride_u[0], slots, state,
            nstates, h, p.batch,       p.channels,    p.dtype, p.gate};
  return done(rec_step(r, stream), "recurrence step");
}

adst_status adst_layer_norm_forward(const adst_norm_problem* prob, const void* x, const void* w,
                                    const void* b, void* y, void* mean, void* rstd,
                                    hipStream_t stream) {
  CHECK(check_norm(prob));
  const adst_norm_problem& p = *prob;
  const int e = size_of(p.dtype), s = acc_size(p.dtype), we = size_of(p.weight_dtype);
  if (p.rows > 0 && (!x || !y)) return fail(ADST_ERR_ARG, "x and y are required");
  CHECK(check_aligned("x", x, e));
  CHECK(check_aligned("y", y, e));
  CHECK(check_aligned("w", w, we));
  CHECK(check_aligned("b", b, we));
  CHECK(check_aligned("mean", mean, s));
  CHECK(check_aligned("rstd", rstd, s));
  Ranges rs;
  // each row is read whole before it is written, so y may be x itself
  const bool in_place = x == y && p.stride_x == p.n;
  if (!in_place) rs.in("x", x, span_bytes(1, 0, p.rows, p.stride_x, p.n, e));
  rs.in("w", w, Wide(p.n) * we);
  rs.in("b", b, Wide(p.n) * we);
  rs.out("y", y, Wide(p.rows) * p.n * e);
  rs.out("mean", mean, Wide(p.rows) * s);
  rs.out("rstd", rstd, Wide(p.rows) * s);
  CHECK(rs.check());
  if (p.rows == 0) return report_ok();
  NormArgs a = norm_args(prob);
  a.x = x;
  a.w = w;
  a.b = b;
  a.y = y;
  a.mean = mean;
  a.rstd = rstd;
  return done(norm_forward(a, stream), "layer norm");
}

uint64_t adst_layer_norm_workspace_bytes(const adst_norm_problem* prob) {
  if (!prob || !known(prob->dtype) || prob->rows < 1 || prob->n < 1 || prob->rows >= kMost ||
      prob->n >= kMost)
    return 0;
  return norm_workspace_bytes(prob->dtype, prob->rows, prob->n);
}

adst_status adst_layer_norm_vjp(const adst_norm_problem* prob, const void* x, const void* dy,
                                const void* w, const void* mean, const void* rstd, void* dx,
                                void* dw, void* db, void* ws, uint64_t ws_bytes,
                                hipStream_t stream) {
  CHECK(check_norm(prob));
  const adst_norm_problem& p = *prob;
  const int e = size_of(p.dtype), s = acc_size(p.dtype), we = size_of(p.weight_dtype);
  if (p.rows > 0 && (!x || !dy || !mean || !rstd))
    return fail(ADST_ERR_ARG, "x, dy, mean and rstd are required");
  CHECK(check_aligned("x", x, e));
  CHECK(check_aligned("dy", dy, e));
  CHECK(check_aligned("dx", dx, e));
  CHECK(check_aligned("w", w, we));
  CHECK(check_aligned("dw", dw, we));
  CHECK(check_aligned("db", db, we));
  CHECK(check_aligned("mean", mean, s));
  CHECK(check_aligned("rstd", rstd, s));
  const uint64_t need = dw || db ? adst_layer_norm_workspace_bytes(prob) : 0;
  if (need && (!ws || ws_bytes < need))
    return fail(ADST_ERR_WORKSPACE, "adst_layer_norm_vjp needs %llu workspace bytes",
                (unsigned long long)need);
  if (need) CHECK(check_aligned("ws", ws, 16));
  Ranges rs;
  rs.in("x", x, span_bytes(1, 0, p.rows, p.stride_x, p.n, e));
  rs.in("dy", dy, span_bytes(1, 0, p.rows, p.stride_dy, p.n, e));
  rs.in("w", w, Wide(p.n) * we);
  rs.in("mean", mean, Wide(p.rows) * s);
  rs.in("rstd", rstd, Wide(p.rows) * s);
  rs.out("dx", dx, Wide(p.rows) * p.n * e);
  rs.out("dw", dw, Wide(p.n) * we);
  rs.out("db", db, Wide(p.n) * we);
  if (need) rs.out("ws", ws, need);
  CHECK(rs.check());
  if (!dx && !dw && !db) return report_ok();
  if (p.rows == 0 && !dw && !db) return report_ok();
  NormArgs a = norm_args(prob);
  a.x = x;
  a.dy = dy;
  a.w = w;
  a.mean = const_cast<void*>(mean);
  a.rstd = const_cast<void*>(rstd);
  a.dx = dx;
  a.dw = dw;
  a.db = db;
  return done(norm_vjp(a, ws, stream), "layer norm gradient");
}

adst_status adst_adamw(const adst_adamw_problem* prob, const adst_adamw_tensor* tensors,
                       int32_t n_tensors, hipStream_t stream) {
  if (!prob) return fail(ADST_ERR_ARG, "problem is NULL");
  const adst_adamw_problem& p = *prob;
  if (p.dtype != ADST_F32 && p.dtype != ADST_F64)
    return fail(ADST_ERR_ARG, "parameters must be F32 or F64");
  if (!known(p.grad_dtype) || (p.dtype == ADST_F64) != (p.grad_dtype == ADST_F64))
    return fail(ADST_ERR_ARG, "gradients must be F32, BF16 or F16, and F64 with F64 parameters");
  if (p.bits != 32 && !(p.bits == 8 && p.dtype == ADST_F32))
    return fail(ADST_ERR_ARG, "bits must be 32, or 8 with F32 parameters");
  if (p.copy_dtype != ADST_F32 && p.copy_dtype != ADST_BF16 && p.copy_dtype != ADST_F16)
    return fail(ADST_ERR_ARG, "copies must be F32, BF16 or F16");
  if (p.t < 1) return fail(ADST_ERR_ARG, "t counts from 1");
  if (!(p.beta1 >= 0 && p.beta1 < 1) || !(p.beta2 >= 0 && p.beta2 < 1))
    return fail(ADST_ERR_ARG, "betas must be in [0, 1)");
  if (!std::isfinite(p.eps) || p.eps < 0) return fail(ADST_ERR_ARG, "eps must be finite and >= 0");
  CHECK(check_aligned("grad_scale", p.grad_scale, 4));
  if (n_tensors < 0 || (n_tensors > 0 && !tensors))
    return fail(ADST_ERR_ARG, "tensors is NULL");
  const int e = size_of(p.dtype), ge = size_of(p.grad_dtype), ce = size_of(p.copy_dtype);
  const int se = p.bits == 8 ? 1 : e;
  for (int32_t i = 0; i < n_tensors; ++i) {
    const adst_adamw_tensor& t = tensors[i];
    if (t.n < 0) return fail(ADST_ERR_ARG, "tensor %d: n must be >= 0", i);
    if (t.n >= (int64_t(1) << 40)) return fail(ADST_ERR_UNSUPPORTED, "tensor %d: too large", i);
    if (!std::isfinite(t.lr) || !std::isfinite(t.weight_decay))
      return fail(ADST_ERR_ARG, "tensor %d: lr and weight_decay must be finite", i);
    if (t.n == 0) continue;
    if (!t.p || !t.grad || !t.m || !t.v || (p.bits == 8 && (!t.m_scale || !t.v_scale)))
      return fail(ADST_ERR_ARG, "tensor %d: p, grad, m, v and their scales are required", i);
    if (!aligned(t.p, e) || !aligned(t.grad, ge) || !aligned(t.m, se) || !aligned(t.v, se) ||
        (p.bits == 8 && (!aligned(t.m_scale, 4) || !aligned(t.v_scale, 4))) ||
        (t.copy && !aligned(t.copy, ce)))
      return fail(ADST_ERR_ARG, "tensor %d: an array is not aligned to its elements", i);
    // fewer than 2^40 values at a 64-bit address: sums of 64 bits do
    struct One {
      const char* name;
      const void* at;
      uint64_t bytes;
    };
    const uint64_t n = (uint64_t)t.n, scales = (n + ADST_STATE_BLOCK - 1) / ADST_STATE_BLOCK * 4;
    const One r[8] = {{"p", t.p, n * e},
                      {"m", t.m, n * se},
                      {"v", t.v, n * se},
                      {"copy", t.copy, n * ce},
                      {"m_scale", p.bits == 8 ? t.m_scale : nullptr, scales},
                      {"v_scale", p.bits == 8 ? t.v_scale : nullptr, scales},
                      {"grad", t.grad, n * ge},
                      {"grad_scale", p.grad_scale, 4}};
    for (int k = 0; k < 6; ++k)  // what is written overlaps nothing
      for (int j = k + 1; j < 8; ++j) {
        const uint64_t x = (uint64_t)(uintptr_t)r[k].at, y = (uint64_t)(uintptr_t)r[j].at;
        if (x && y && x < y + r[j].bytes && y < x + r[k].bytes)
          return fail(ADST_ERR_ARG, "tensor %d: %s and %s overlap", i, r[k].name, r[j].name);
      }
  }
  if (n_tensors == 0) return report_ok();
  return done(adamw(p, tensors, n_tensors, stream), "adamw");
}

}  // extern "C"
