// C boundary of the token operators: every argument is checked before the
// first HIP call, and nothing here throws.

#include "abi_checks.h"
#include "token_kernels.h"

namespace adst {
namespace {

bool half(int32_t dtype) { return dtype == ADST_BF16 || dtype == ADST_F16; }

adst_status check_strides(const int64_t (&s)[2]) {
  if (s[0] < 0 || s[1] < 0) return fail(ADST_ERR_ARG, "strides must be >= 0");
  return ADST_OK;
}

// [batch][steps][channels] as every operator here takes it.
adst_status check_extents(int64_t batch, int64_t steps, int64_t channels) {
  if (batch < 0 || steps < 0 || channels < 0)
    return fail(ADST_ERR_ARG, "batch, steps and channels must be >= 0");
  if (steps >= kMost || batch >= kMost || channels >= (int64_t(1) << 26))
    return fail(ADST_ERR_UNSUPPORTED,
                "batch and steps must be below 2^31 - 2^16, channels below 2^26");
  if (Wide(batch) * channels * (steps + 16) > (Wide(1) << 52))
    return fail(ADST_ERR_UNSUPPORTED, "more values than the address space");
  return ADST_OK;
}

// ------------------------------------------------------------- convolution
adst_status check_conv(const adst_conv_problem* p) {
  if (!p) return fail(ADST_ERR_ARG, "problem is NULL");
  if (!known(p->dtype)) return fail(ADST_ERR_ARG, "unknown dtype %d", p->dtype);
  if (p->weight_dtype != p->dtype && !(half(p->dtype) && p->weight_dtype == ADST_F32))
    return fail(ADST_ERR_ARG, "weight_dtype must be the dtype, or F32 beside BF16 and F16");
  if (p->act != ADST_ACT_NONE && p->act != ADST_ACT_SILU)
    return fail(ADST_ERR_ARG, "unknown act %d", p->act);
  if (p->taps < 1 || p->taps > ADST_CONV_MAX_TAPS)
    return fail(ADST_ERR_ARG, "taps must be 1..%d", ADST_CONV_MAX_TAPS);
  CHECK(check_strides(p->stride_x));
  CHECK(check_strides(p->stride_dy));
  return check_extents(p->batch, p->steps, p->channels);
}

ConvArgs conv_args(const adst_conv_problem* p, const void* x, const void* w, const void* bias,
                   const void* x0, const int32_t* lens) {
  ConvArgs a{};
  a.x = x;
  a.w = w;
  a.bias = bias;
  a.x0 = x0;
  a.lens = lens;
  a.sx_b = p->stride_x[0];
  a.sx_t = p->stride_x[1];
  a.sd_b = p->stride_dy[0];
  a.sd_t = p->stride_dy[1];
  a.B = p->batch;
  a.T = p->steps;
  a.D = p->channels;
  a.dtype = p->dtype;
  a.wtype = p->weight_dtype;
  a.act = p->act;
  a.taps = p->taps;
  return a;
}

// Alignment and extents of the inputs that the convolution's calls share.
adst_status conv_inputs(const adst_conv_problem* p, const void* x, const void* w, const void* bias,
                        const void* x0, const int32_t* lens, Ranges* rs) {
  const int e = size_of(p->dtype), we = size_of(p->weight_dtype);
  CHECK(check_aligned("x", x, e));
  CHECK(check_aligned("w", w, we));
  CHECK(check_aligned("bias", bias, we));
  CHECK(check_aligned("x0", x0, e));
  CHECK(check_aligned("lens", lens, 4));
  rs->in("x", x, span_bytes(p->batch, p->stride_x[0], p->steps, p->stride_x[1], p->channels, e));
  rs->in("w", w, Wide(p->taps) * p->channels * we);
  rs->in("bias", bias, Wide(p->channels) * we);
  rs->in("x0", x0, Wide(p->batch) * (p->taps - 1) * p->channels * e);
  rs->in("lens", lens, Wide(p->batch) * 4);
  return ADST_OK;
}

// ------------------------------------------------------------ selective scan
adst_status check_scan(const adst_scan_problem* p, ScanGrid* grid) {
  if (!p) return fail(ADST_ERR_ARG, "problem is NULL");
  if (!known(p->dtype)) return fail(ADST_ERR_ARG, "unknown dtype %d", p->dtype);
  if (p->softplus != 0 && p->softplus != 1) return fail(ADST_ERR_ARG, "softplus must be 0 or 1");
  CHECK(check_strides(p->stride_x));
  CHECK(check_strides(p->stride_delta));
  CHECK(check_strides(p->stride_b));
  CHECK(check_strides(p->stride_c));
  CHECK(check_strides(p->stride_z));
  CHECK(check_strides(p->stride_dy));
  if (p->states < 1 || p->groups < 1)
    return fail(ADST_ERR_ARG, "states and groups must be >= 1");
  const int64_t most = p->dtype == ADST_F64 ? ADST_SCAN_MAX_STATES / 2 : ADST_SCAN_MAX_STATES;
  if (p->states > most)
    return fail(ADST_ERR_UNSUPPORTED, "at most %lld states", (long long)most);
  CHECK(check_extents(p->batch, p->steps, p->channels));
  if (p->channels % p->groups != 0) return fail(ADST_ERR_ARG, "groups must divide channels");
  // (without channels nothing else bounds the groups, whose B and C are still read and cleared)
  if (Wide(p->batch) * p->channels * (p->steps + 16) * p->states > (Wide(1) << 52) ||
      p->groups >= (int64_t(1) << 26) ||
      Wide(p->batch) * (p->steps + 16) * p->groups * p->states > (Wide(1) << 52))
    return fail(ADST_ERR_UNSUPPORTED, "more values than the address space");
  *grid = scan_grid(p->dtype, p->batch, p->steps, p->channels, p->states, p->groups);
  if (!grid->fits) return fail(ADST_ERR_UNSUPPORTED, "more rows and channels than a launch holds");
  return ADST_OK;
}

ScanArgs scan_args(const adst_scan_problem* p, const adst_scan_inputs* in) {
  ScanArgs a{};
  a.x = in->x;
  a.delta = in->delta;
  a.A = in->A;
  a.Bm = in->B;
  a.Cm = in->C;
  a.D = in->D;
  a.z = in->z;
  a.bias = in->delta_bias;
  a.h0 = in->h0;
  a.lens = in->lens;
  a.sx_b = p->stride_x[0];
  a.sx_t = p->stride_x[1];
  a.sl_b = p->stride_delta[0];
  a.sl_t = p->stride_delta[1];
  a.sb_b = p->stride_b[0];
  a.sb_t = p->stride_b[1];
  a.sc_b = p->stride_c[0];
  a.sc_t = p->stride_c[1];
  a.sz_b = p->stride_z[0];
  a.sz_t = p->stride_z[1];
  a.sd_b = p->stride_dy[0];
  a.sd_t = p->stride_dy[1];
  a.B = p->batch;
  a.T = p->steps;
  a.D_ = p->channels;
  a.N = (int32_t)p->states;
  a.G = (int32_t)p->groups;
  a.dtype = p->dtype;
  a.softplus = p->softplus;
  return a;
}

// The inputs that the scan's calls share.
adst_status scan_inputs(const adst_scan_problem* p, const adst_scan_inputs* in, Ranges* rs) {
  const int e = size_of(p->dtype), s = acc_size(p->dtype);
  const Wide channels = Wide(p->channels) * s;
  const auto seq = [&](const char* name, const void* at, const int64_t (&stride)[2], int64_t n) {
    rs->in(name, at, span_bytes(p->batch, stride[0], p->steps, stride[1], n, e));
    return check_aligned(name, at, e);
  };
  const auto held = [&](const char* name, const void* at, Wide bytes) {
    rs->in(name, at, bytes);
    return check_aligned(name, at, s);
  };
  CHECK(seq("x", in->x, p->stride_x, p->channels));
  CHECK(seq("delta", in->delta, p->stride_delta, p->channels));
  CHECK(seq("z", in->z, p->stride_z, p->channels));
  CHECK(seq("B", in->B, p->stride_b, p->groups * p->states));
  CHECK(seq("C", in->C, p->stride_c, p->groups * p->states));
  CHECK(held("A", in->A, channels * p->states));
  CHECK(held("D", in->D, channels));
  CHECK(held("delta_bias", in->delta_bias, channels));
  CHECK(held("h0", in->h0, channels * p->states * p->batch));
  rs->in("lens", in->lens, Wide(p->batch) * 4);
  CHECK(check_aligned("lens", in->lens, 4));
  if (p->batch > 0 && p->steps > 0 && p->channels > 0 &&
      (!in->x || !in->delta || !in->A || !in->B || !in->C))
    return fail(ADST_ERR_ARG, "x, delta, A, B and C are required");
  return ADST_OK;
}

// ------------------------------------------------------------ cross entropy
adst_status check_xent(const adst_xent_problem* p) {
  if (!p) return fail(ADST_ERR_ARG, "problem is NULL");
  if (!known(p->dtype)) return fail(ADST_ERR_ARG, "unknown dtype %d", p->dtype);
  if (p->reserved != 0) return fail(ADST_ERR_ARG, "reserved must be 0");
  if (p->rows < 0 || p->width < 1 || p->vocab < 1)
    return fail(ADST_ERR_ARG, "rows must be >= 0, width and vocab >= 1");
  if (p->stride_x < 0 || p->stride_w < 0) return fail(ADST_ERR_ARG, "strides must be >= 0");
  // tiles of 64 x 64 and up, their work-items counted in 32 bits, and 256 values of a
  // result to a workgroup
  constexpr int64_t most = int64_t(1) << 31;
  if (p->rows >= kMost || p->width >= kMost || p->vocab >= kMost ||
      Wide(p->rows) * (p->width + 64) >= most || Wide(p->vocab) * (p->width + 64) >= most ||
      Wide(p->rows + 256) * (p->vocab + 256) >= Wide(1) << 35)
    return fail(ADST_ERR_UNSUPPORTED,
                "rows and vocab times width + 64 must be below 2^31, (rows + 256) * (vocab + 256) "
                "below 2^35");
  return ADST_OK;
}

adst_status xent_inputs(const adst_xent_problem* p, const void* x, const void* w,
                        const int32_t* labels, Ranges* rs) {
  const int e = size_of(p->dtype);
  if (p->rows > 0 && (!x || !w || !labels))
    return fail(ADST_ERR_ARG, "x, w and labels are required");
  CHECK(check_aligned("x", x, e));
  CHECK(check_aligned("w", w, e));
  CHECK(check_aligned("labels", labels, 4));
  rs->in("x", x, span_bytes(1, 0, p->rows, p->stride_x, p->width, e));
  rs->in("w", w, span_bytes(1, 0, p->vocab, p->stride_w, p->width, e));
  rs->in("labels", labels, Wide(p->rows) * 4);
  return ADST_OK;
}

XentArgs xent_args(const adst_xent_problem* p, const void* x, const void* w,
                   const int32_t* labels) {
  XentArgs a{};
  a.x = x;
  a.w = w;
  a.sx = p->stride_x;
  a.sw = p->stride_w;
  a.M = p->rows;
  a.V = p->vocab;
  a.K = p->width;
  a.labels = labels;
  a.dtype = p->dtype;
  return a;
}

}  // namespace
}  // namespace adst

using namespace adst;

extern "C" {

adst_status adst_causal_conv_forward(const adst_conv_problem* prob, const void* x, const void* w,
                                     const void* bias, const void* x0, const int32_t* lens,
                                     void* y, void* xT, hipStream_t stream) {
  CHECK(check_conv(prob));
  const adst_conv_problem& p = *prob;
  const int e = size_of(p.dtype);
  if (p.batch > 0 && p.steps > 0 && p.channels > 0 && (!x || !w))
    return fail(ADST_ERR_ARG, "x and w are required");
  Ranges rs;
  CHECK(conv_inputs(prob, x, w, bias, x0, lens, &rs));
  CHECK(check_aligned("y", y, e));
  CHECK(check_aligned("xT", xT, e));
  rs.out("y", y, Wide(p.batch) * p.steps * p.channels * e);
  rs.out("xT", xT, Wide(p.batch) * (p.taps - 1) * p.channels * e);
  CHECK(rs.check());
  if (p.batch == 0 || p.channels == 0) return report_ok();
  ConvArgs a = conv_args(prob, x, w, bias, x0, lens);
  a.y = y;
  a.xT = xT;
  return done(conv_forward(a, stream), "causal convolution");
}

uint64_t adst_causal_conv_workspace_bytes(const adst_conv_problem* prob) {
  if (check_conv(prob) != ADST_OK || prob->channels == 0) return 0;
  return conv_workspace_bytes(prob->dtype, prob->batch, prob->steps, prob->channels, prob->taps);
}

adst_status adst_causal_conv_vjp(const adst_conv_problem* prob, const void* x, const void* dy,
                                 const void* w, const void* bias, const void* x0,
                                 const int32_t* lens, const void* dxT, void* dx, void* dw,
                                 void* dbias, void* dx0, void* ws, uint64_t ws_bytes,
                                 hipStream_t stream) {
  CHECK(check_conv(prob));
  const adst_conv_problem& p = *prob;
  const int e = size_of(p.dtype), we = size_of(p.weight_dtype);
  if (p.batch > 0 && p.steps > 0 && p.channels > 0 && (!x || !w || !dy))
    return fail(ADST_ERR_ARG, "x, dy and w are required");
  const bool launches = p.channels > 0 && (dx || dw || dbias || dx0);
  if (launches && !w) return fail(ADST_ERR_ARG, "w is required");  // it is read before any step
  Ranges rs;
  CHECK(conv_inputs(prob, x, w, bias, x0, lens, &rs));
  CHECK(check_aligned("dy", dy, e));
  CHECK(check_aligned("dxT", dxT, e));
  CHECK(check_aligned("dx", dx, e));
  CHECK(check_aligned("dx0", dx0, e));
  CHECK(check_aligned("dw", dw, we));
  CHECK(check_aligned("dbias", dbias, we));
  const uint64_t need = dw || dbias ? adst_causal_conv_workspace_bytes(prob) : 0;
  if (need && (!ws || ws_bytes < need))
    return fail(ADST_ERR_WORKSPACE, "adst_causal_conv_vjp needs %llu workspace bytes",
                (unsigned long long)need);
  if (need) CHECK(check_aligned("ws", ws, 16));
  const Wide window = Wide(p.batch) * (p.taps - 1) * p.channels * e;
  rs.in("dy", dy, span_bytes(p.batch, p.stride_dy[0], p.steps, p.stride_dy[1], p.channels, e));
  rs.in("dxT", dxT, window);
  rs.out("dx", dx, Wide(p.batch) * p.steps * p.channels * e);
  rs.out("dx0", dx0, window);
  rs.out("dw", dw, Wide(p.taps) * p.channels * we);
  rs.out("dbias", dbias, Wide(p.channels) * we);
  if (need) rs.out("ws", ws, need);
  CHECK(rs.check());
  if (!launches) return report_ok();
  ConvArgs a = conv_args(prob, x, w, bias, x0, lens);
  a.dy = dy;
  a.dxT = dxT;
  a.dx = dx;
  a.dw = dw;
  a.dbias = dbias;
  a.dx0 = dx0;
  return done(conv_vjp(a, ws, stream), "causal convolution's gradient");
}

adst_status adst_causal_conv_step(const adst_conv_problem* prob, const void* x, const void* w,
                                  const void* bias, const int32_t* slots, void* window,
                                  int64_t nstates, void* y, hipStream_t stream) {
  CHECK(check_conv(prob));
  const adst_conv_problem& p = *prob;
  const int e = size_of(p.dtype);
  if (p.steps != 1) return fail(ADST_ERR_ARG, "steps must be 1");
  if (nstates < 0 || (!slots && nstates < p.batch))
    return fail(ADST_ERR_ARG, "nstates must be >= 0, and >= batch without slots");
  if (Wide(p.batch) * p.channels >= (Wide(1) << 31))
    return fail(ADST_ERR_UNSUPPORTED, "more rows and channels than one launch holds");
  const bool some = p.batch > 0 && p.channels > 0;
  if (some && (!x || !w || (nstates > 0 && p.taps > 1 && !window)))
    return fail(ADST_ERR_ARG, "x, w and window are required");
  Ranges rs;
  CHECK(conv_inputs(prob, x, w, bias, nullptr, nullptr, &rs));
  CHECK(check_aligned("slots", slots, 4));
  CHECK(check_aligned("window", window, e));
  CHECK(check_aligned("y", y, e));
  rs.in("slots", slots, Wide(p.batch) * 4);
  rs.out("window", window, Wide(nstates) * (p.taps - 1) * p.channels * e);
  rs.out("y", y, Wide(p.batch) * p.channels * e);
  CHECK(rs.check());
  if (!some) return report_ok();
  const ConvStep a{x,       w, bias,    p.stride_x[0], slots,  window,        nstates,
                   y,       p.batch, p.channels,  p.dtype, p.weight_dtype, p.act, p.taps};
  return done(conv_step(a, stream), "causal convolution's step");
}

adst_status adst_selective_scan_plan(const adst_scan_problem* prob, adst_scan_info* out) {
  if (!out) return fail(ADST_ERR_ARG, "out is NULL");
  ScanGrid g;
  CHECK(check_scan(prob, &g));
  out->span = g.chunk;
  out->ck_bytes = g.ck_bytes;
  out->workspace_bytes = g.map_bytes;
  out->vjp_workspace_bytes = g.map_bytes + (g.rev_bytes + 15) / 16 * 16;
  return report_ok();
}

adst_status adst_selective_scan_forward(const adst_scan_problem* prob, const adst_scan_inputs* in,
                                        void* y, void* hT, void* ck, void* ws, uint64_t ws_bytes,
                                        hipStream_t stream) {
  ScanGrid g;
  CHECK(check_scan(prob, &g));
  if (!in) return fail(ADST_ERR_ARG, "inputs are NULL");
  const adst_scan_problem& p = *prob;
  const int e = size_of(p.dtype), s = acc_size(p.dtype);
  Ranges rs;
  CHECK(scan_inputs(prob, in, &rs));
  CHECK(check_aligned("y", y, e));
  CHECK(check_aligned("hT", hT, s));
  CHECK(check_aligned("ck", ck, s));
  if (g.map_bytes && (!ws || ws_bytes < g.map_bytes))
    return fail(ADST_ERR_WORKSPACE, "adst_selective_scan_forward needs %llu workspace bytes",
                (unsigned long long)g.map_bytes);
  if (g.map_bytes) CHECK(check_aligned("ws", ws, 16));
  rs.out("y", y, Wide(p.batch) * p.steps * p.channels * e);
  rs.out("hT", hT, Wide(p.batch) * p.channels * p.states * s);
  rs.out("ck", ck, g.ck_bytes);
  if (g.map_bytes) rs.out("ws", ws, g.map_bytes);
  CHECK(rs.check());
  if (p.batch == 0 || p.channels == 0 || (!y && !hT && !ck)) return report_ok();
  if (!in->A) return fail(ADST_ERR_ARG, "A is required");  // it is read before any step
  ScanArgs a = scan_args(prob, in);
  a.y = y;
  a.hT = hT;
  a.ck = ck;
  return done(scan_forward(a, ws, stream), "selective scan");
}

adst_status adst_selective_scan_vjp(const adst_scan_problem* prob, const adst_scan_inputs* in,
                                    const void* ck, const void* dy, const void* dhT,
                                    const adst_scan_gradients* out, void* ws, uint64_t ws_bytes,
                                    hipStream_t stream) {
  ScanGrid g;
  CHECK(check_scan(prob, &g));
  if (!in || !out) return fail(ADST_ERR_ARG, "inputs or gradients are NULL");
  const adst_scan_problem& p = *prob;
  const int e = size_of(p.dtype), s = acc_size(p.dtype);
  Ranges rs;
  CHECK(scan_inputs(prob, in, &rs));
  const bool some = p.batch > 0 && p.steps > 0 && p.channels > 0;
  if (some && (!dy || !out->dx || !out->ddelta))
    return fail(ADST_ERR_ARG, "dy, dx and ddelta are required");
  if (p.batch > 0 && p.steps > 0 && (!out->dB || !out->dC))
    return fail(ADST_ERR_ARG, "dB and dC are required");
  if (p.channels > 0 && (!in->A || !out->dA)) return fail(ADST_ERR_ARG, "A and dA are required");
  if (some && in->z && !out->dz) return fail(ADST_ERR_ARG, "dz is required with z");
  if (!in->z && out->dz) return fail(ADST_ERR_ARG, "dz without z");
  const Wide values = Wide(p.batch) * p.steps * p.channels * e;
  const Wide coefficients = Wide(p.batch) * p.steps * p.groups * p.states * e;
  const Wide channels = Wide(p.channels) * s;
  const struct {
    const char* name;
    const void* at;
    Wide bytes;
    int size;
  } outs[] = {{"dx", out->dx, values, e},
              {"ddelta", out->ddelta, values, e},
              {"dz", out->dz, values, e},
              {"dB", out->dB, coefficients, e},
              {"dC", out->dC, coefficients, e},
              {"dA", out->dA, channels * p.states, s},
              {"dD", out->dD, channels, s},
              {"ddelta_bias", out->ddelta_bias, channels, s},
              {"dh0", out->dh0, channels * p.states * p.batch, s}};
  for (const auto& o : outs) {
    CHECK(check_aligned(o.name, o.at, o.size));
    rs.out(o.name, o.at, o.bytes);
  }
  CHECK(check_aligned("dy", dy, e));
  CHECK(check_aligned("dhT", dhT, s));
  CHECK(check_aligned("ck", ck, s));
  rs.in("dy", dy, span_bytes(p.batch, p.stride_dy[0], p.steps, p.stride_dy[1], p.channels, e));
  rs.in("dhT", dhT, channels * p.states * p.batch);
  rs.in("ck", ck, g.ck_bytes);
  const uint64_t given = g.map_bytes + (g.rev_bytes + 15) / 16 * 16;
  const uint64_t need = given + (ck ? 0 : g.ck_bytes);
  if (need && (!ws || ws_bytes < need))
    return fail(ADST_ERR_WORKSPACE, "adst_selective_scan_vjp needs %llu workspace bytes",
                (unsigned long long)need);
  if (need) CHECK(check_aligned("ws", ws, 16));
  if (need) rs.out("ws", ws, need);
  CHECK(rs.check());
  // without channels dB and dC, sums over them, are still to be cleared
  if (p.channels == 0 && (p.batch == 0 || p.steps == 0)) return report_ok();
  ScanArgs a = scan_args(prob, in);
  if (!ck) {  // the checkpoints again
    a.ck = static_cast<char*>(ws) + given;
    if (some) {
      const hipError_t err = scan_forward(a, ws, stream);
      if (err != hipSuccess) return done(err, "selective scan");
    }
  } else {
    a.ck = const_cast<void*>(ck);
  }
  a.dy = dy;
  a.dhT = dhT;
  a.out = *out;
  return done(scan_vjp(a, ws, stream), "selective scan's gradient");
}

adst_status adst_selective_scan_step(const adst_scan_problem* prob, const adst_scan_inputs* in,
                                     const int32_t* slots, void* state, int64_t nstates, void* y,
                                     hipStream_t stream) {
  ScanGrid g;
  CHECK(check_scan(prob, &g));
  if (!in) return fail(ADST_ERR_ARG, "inputs are NULL");
  const adst_scan_problem& p = *prob;
  const int e = size_of(p.dtype), s = acc_size(p.dtype);
  if (p.steps != 1) return fail(ADST_ERR_ARG, "steps must be 1");
  if (in->h0 || in->lens) return fail(ADST_ERR_ARG, "a step has neither h0 nor lens");
  if (nstates < 0 || (!slots && nstates < p.batch))
    return fail(ADST_ERR_ARG, "nstates must be >= 0, and >= batch without slots");
  if (Wide(p.batch) * p.channels >= (Wide(1) << 26))
    return fail(ADST_ERR_UNSUPPORTED, "more rows and channels than one launch holds");
  Ranges rs;
  CHECK(scan_inputs(prob, in, &rs));
  const bool some = p.batch > 0 && p.channels > 0;
  if (some && nstates > 0 && !state) return fail(ADST_ERR_ARG, "state is required");
  CHECK(check_aligned("slots", slots, 4));
  CHECK(check_aligned("state", state, s));
  CHECK(check_aligned("y", y, e));
  rs.in("slots", slots, Wide(p.batch) * 4);
  rs.out("state", state, Wide(nstates) * p.channels * p.states * s);
  rs.out("y", y, Wide(p.batch) * p.channels * e);
  CHECK(rs.check());
  if (!some) return report_ok();
  ScanStep q{scan_args(prob, in), slots, state, nstates};
  q.a.y = y;
  return done(scan_step(q, stream), "selective scan's step");
}

adst_status adst_linear_cross_entropy_plan(const adst_xent_problem* prob, adst_xent_info* out) {
  if (!out) return fail(ADST_ERR_ARG, "out is NULL");
  CHECK(check_xent(prob));
  out->workspace_bytes = out->vjp_workspace_bytes = 0;
  if (prob->rows > 0) {
    const adst_xent_problem& p = *prob;
    out->workspace_bytes = xent_plan(p.dtype, p.rows, p.vocab, p.width, false).bytes;
    out->vjp_workspace_bytes = xent_plan(p.dtype, p.rows, p.vocab, p.width, true).bytes;
  }
  return report_ok();
}

adst_status adst_linear_cross_entropy_forward(const adst_xent_problem* prob, const void* x,
                                              const void* w, const int32_t* labels, void* loss,
                                              void* lse, void* ws, uint64_t ws_bytes,
                                              hipStream_t stream) {
  adst_xent_info info;
  CHECK(adst_linear_cross_entropy_plan(prob, &info));
  const adst_xent_problem& p = *prob;
  const int s = acc_size(p.dtype);
  Ranges rs;
  CHECK(xent_inputs(prob, x, w, labels, &rs));
  CHECK(check_aligned("loss", loss, s));
  CHECK(check_aligned("lse", lse, s));
  const uint64_t need = info.workspace_bytes;
  if (need && (!ws || ws_bytes < need))
    return fail(ADST_ERR_WORKSPACE, "adst_linear_cross_entropy_forward needs %llu workspace bytes",
                (unsigned long long)need);
  if (need) CHECK(check_aligned("ws", ws, 16));
  rs.out("loss", loss, Wide(p.rows) * s);
  rs.out("lse", lse, Wide(p.rows) * s);
  if (need) rs.out("ws", ws, need);
  CHECK(rs.check());
  if (p.rows == 0 || (!loss && !lse)) return report_ok();
  XentArgs a = xent_args(prob, x, w, labels);
  a.loss = loss;
  a.lse = lse;
  return done(xent_forward(a, ws, stream), "cross entropy");
}

adst_status adst_linear_cross_entropy_vjp(const adst_xent_problem* prob, const void* x,
                                          const void* w, const int32_t* labels, const void* lse,
                                          const void* dloss, void* dx, void* dw, void* ws,
                                          uint64_t ws_bytes, hipStream_t stream) {
  adst_xent_info info;
  CHECK(adst_linear_cross_entropy_plan(prob, &info));
  const adst_xent_problem& p = *prob;
  const int e = size_of(p.dtype), s = acc_size(p.dtype);
  Ranges rs;
  CHECK(xent_inputs(prob, x, w, labels, &rs));
  if (p.rows > 0 && !lse) return fail(ADST_ERR_ARG, "lse is required");
  CHECK(check_aligned("lse", lse, s));
  CHECK(check_aligned("dloss", dloss, s));
  CHECK(check_aligned("dx", dx, e));
  CHECK(check_aligned("dw", dw, e));
  const uint64_t need = info.vjp_workspace_bytes;
  if (need && (!ws || ws_bytes < need))
    return fail(ADST_ERR_WORKSPACE, "adst_linear_cross_entropy_vjp needs %llu workspace bytes",
                (unsigned long long)need);
  if (need) CHECK(check_aligned("ws", ws, 16));
  rs.in("lse", lse, Wide(p.rows) * s);
  rs.in("dloss", dloss, Wide(p.rows) * s);
  rs.out("dx", dx, Wide(p.rows) * p.width * e);
  rs.out("dw", dw, Wide(p.vocab) * p.width * e);
  if (need) rs.out("ws", ws, need);
  CHECK(rs.check());
  if ((!dx && !dw) || (p.rows == 0 && !dw)) return report_ok();
  XentArgs a = xent_args(prob, x, w, labels);
  a.lse = const_cast<void*>(lse);
  a.dloss = dloss;
  a.dx = dx;
  a.dw = dw;
  return done(xent_vjp(a, ws, stream), "cross entropy's gradient");
}

}  // extern "C"
