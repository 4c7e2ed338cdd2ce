// The selective scan's kernels as host code, of every type, on guarded arrays: a
// read or write past an array, the workspace among them, ends the program. Results are
// compared with the definition. Arguments: dtype batch steps channels states groups
// ragged optional (1: with D, z and delta_bias).

#include "token_lanes.h"

#include "selective_scan_f32.host.inc"

#include <memory>
#include <vector>

#include "guard.h"
#include "values.h"

namespace adst {
#define OF(name, T)                                                                              \
  hipError_t scan_forward_##name(const ScanArgs& a, const ScanGrid& g, void* ws, hipStream_t st) { \
    return forward_of<T>(a, g, ws, st);                                                          \
  }                                                                                              \
  hipError_t scan_vjp_##name(const ScanArgs& a, const ScanGrid& g, void* ws, hipStream_t st) {   \
    return vjp_of<T>(a, g, ws, st);                                                              \
  }                                                                                              \
  hipError_t scan_step_##name(const ScanStep& s, hipStream_t st) { return step_of<T>(s, st); }
OF(f64, double)
OF(bf16, bf16)
OF(f16, f16)
}  // namespace adst
#include "selective_scan.cpp"

using namespace adst;

namespace {

double softplus_of(double v) { return std::fmax(v, 0) + std::log1p(std::exp(-std::fabs(v))); }
double sigmoid_of(double v) { return 1 / (1 + std::exp(-v)); }

template <class T>
void check(int dtype, int64_t B, int64_t T_, int64_t D, int N, int G, bool ragged, bool optional,
           bool at_end) {
  typedef Acc<T> A;
  const double tol = sizeof(T) == 8 ? 1e-9 : sizeof(T) == 4 ? 3e-4 : 3e-2;
  const int64_t n = B * T_ * D, gn = G * N, nb = B * T_ * gn, nh = B * D * N;
  const ScanGrid grid = scan_grid(dtype, B, T_, D, N, G);
  const auto values = [&](int64_t count, uint64_t from, double scale, double shift) {
    auto g = std::make_unique<Guarded>(count * sizeof(T), at_end);
    for (int64_t i = 0; i < count; ++i)
      g->template as<T>()[i] = (T)((2 * noise(i + from) - 1) * scale + shift);
    return g;
  };
  const auto held = [&](int64_t count, uint64_t from, double scale, double shift) {
    auto g = std::make_unique<Guarded>(count * sizeof(A), at_end);
    for (int64_t i = 0; i < count; ++i)
      g->template as<A>()[i] = (A)((2 * noise(i + from) - 1) * scale + shift);
    return g;
  };
  // s A stays <= 0, as the products of coefficients need
  const auto x = values(n, 1, 1, 0), delta = values(n, 10 * n, optional ? 1 : 0.25, optional ? -1 : 0.3), z = values(n, 20 * n, 2, 0),
             dy = values(n, 30 * n, 1, 0), Bm = values(nb, 40 * n, 1, 0),
             Cm = values(nb, 50 * n, 1, 0);
  const auto Am = held(D * N, 60 * n + 7, 0.5, -0.6), skip = held(D, 70 * n + 7, 1, 0),
             bias = held(D, 80 * n + 7, 0.5, 0), h0 = held(nh, 90 * n + 7, 1, 0),
             dhT = held(nh, 95 * n + 7, 1, 0);
  Guarded y(n * sizeof(T), at_end), dx(n * sizeof(T), at_end), ddelta(n * sizeof(T), at_end),
      dz(n * sizeof(T), at_end), dB(nb * sizeof(T), at_end), dC(nb * sizeof(T), at_end),
      dA(D * N * sizeof(A), at_end), dD(D * sizeof(A), at_end), dbias(D * sizeof(A), at_end),
      dh0(nh * sizeof(A), at_end), hT(nh * sizeof(A), at_end), lens(B * 4, at_end),
      ck(grid.ck_bytes, at_end), ws(grid.map_bytes + grid.rev_bytes, at_end);
  for (int64_t b = 0; b < B; ++b)
    lens.as<int32_t>()[b] = b == B - 1 ? (int32_t)T_ : (int32_t)(noise(b + 7 * n) * (double)T_);
  ScanArgs a{};
  a.x = x->get();
  a.delta = delta->get();
  a.A = Am->get();
  a.Bm = Bm->get();
  a.Cm = Cm->get();
  if (optional) {
    a.D = skip->get();
    a.z = z->get();
    a.bias = bias->get();
  }
  a.h0 = h0->get();
  a.lens = ragged ? lens.as<int32_t>() : nullptr;
  a.sx_b = a.sl_b = a.sz_b = a.sd_b = T_ * D;
  a.sx_t = a.sl_t = a.sz_t = a.sd_t = D;
  a.sb_b = a.sc_b = T_ * gn;
  a.sb_t = a.sc_t = gn;
  a.B = B;
  a.T = T_;
  a.D_ = D;
  a.N = N;
  a.G = G;
  a.dtype = dtype;
  a.softplus = optional;
  a.y = y.get();
  a.hT = hT.get();
  a.ck = ck.get();
  if (B > 0 && scan_forward(a, ws.get(), nullptr) != hipSuccess) std::exit(3);
  a.dy = dy->get();
  a.dhT = dhT->get();
  a.out = {dx.get(), ddelta.get(), optional ? dz.get() : nullptr, dB.get(), dC.get(), dA.get(),
           dD.get(), dbias.get(), dh0.get()};
  if (scan_vjp(a, ws.get(), nullptr) != hipSuccess) std::exit(3);
  std::vector<double> sB(nb, 0.0), sC(nb, 0.0);
  for (int64_t d = 0; d < D; ++d) {
    const int64_t g = d / (D / G);
    std::vector<double> sA(N, 0.0);
    double sD = 0, sbias = 0;
    for (int64_t b = 0; b < B; ++b) {
      const int64_t len = ragged ? lens.as<int32_t>()[b] : T_;
      std::vector<double> h((len + 1) * N), s(len), e(len), pre(len);
      for (int i = 0; i < N; ++i) h[i] = (double)h0->template as<A>()[(b * D + d) * N + i];
      const auto at = [&](int64_t t) { return (b * T_ + t) * D + d; };
      const auto of = [&](int64_t t) { return (b * T_ + t) * gn + g * N; };
      const auto val = [&](const auto& v, int64_t i) { return (double)(A)v->template as<T>()[i]; };
      const auto rate_of = [&](int i) { return (double)Am->template as<A>()[d * N + i]; };
      for (int64_t t = 0; t < T_; ++t) {
        double out = 0;
        if (t < len) {
          double raw = val(delta, at(t));
          if (optional) raw += (double)bias->template as<A>()[d];
          s[t] = optional ? softplus_of(raw) : raw;
          e[t] = optional ? sigmoid_of(raw) : 1;
          for (int i = 0; i < N; ++i) {
            h[(t + 1) * N + i] = std::exp(s[t] * rate_of(i)) * h[t * N + i] +
                                 s[t] * val(x, at(t)) * val(Bm, of(t) + i);
            out += val(Cm, of(t) + i) * h[(t + 1) * N + i];
          }
          if (optional) out += (double)skip->template as<A>()[d] * val(x, at(t));
          pre[t] = out;
          if (optional) out *= val(z, at(t)) * sigmoid_of(val(z, at(t)));
        }
        near("y", at(t), (double)(A)y.as<T>()[at(t)], out, tol);
      }
      for (int i = 0; i < N; ++i)
        near("hT", (b * D + d) * N + i, (double)hT.as<A>()[(b * D + d) * N + i], h[len * N + i],
             tol);
      std::vector<double> G_(N);
      for (int i = 0; i < N; ++i) G_[i] = (double)dhT->template as<A>()[(b * D + d) * N + i];
      for (int64_t t = T_ - 1; t >= 0; --t) {
        double ox = 0, od = 0, oz = 0;
        if (t < len) {
          double d_out = val(dy, at(t));
          if (optional) {
            const double f = sigmoid_of(val(z, at(t)));
            oz = d_out * pre[t] * f * (1 + val(z, at(t)) * (1 - f));
            d_out *= val(z, at(t)) * f;
            sD += d_out * val(x, at(t));
            ox = d_out * (double)skip->template as<A>()[d];
          } else {
            sD += d_out * val(x, at(t));
          }
          for (int i = 0; i < N; ++i) {
            const double grow = std::exp(s[t] * rate_of(i));
            G_[i] += d_out * val(Cm, of(t) + i);
            sC[of(t) + i] += d_out * h[(t + 1) * N + i];
            sB[of(t) + i] += G_[i] * s[t] * val(x, at(t));
            ox += s[t] * G_[i] * val(Bm, of(t) + i);
            od += val(x, at(t)) * G_[i] * val(Bm, of(t) + i);
            G_[i] *= grow;
            od += rate_of(i) * G_[i] * h[t * N + i];
            sA[i] += s[t] * G_[i] * h[t * N + i];
          }
          od *= e[t];
          sbias += od;
        }
        near("dx", at(t), (double)(A)dx.as<T>()[at(t)], ox, tol);
        near("ddelta", at(t), (double)(A)ddelta.as<T>()[at(t)], od, tol);
        if (optional) near("dz", at(t), (double)(A)dz.as<T>()[at(t)], oz, tol);
      }
      for (int i = 0; i < N; ++i)
        near("dh0", (b * D + d) * N + i, (double)dh0.as<A>()[(b * D + d) * N + i], G_[i], tol);
    }
    for (int i = 0; i < N; ++i) near("dA", d * N + i, (double)dA.as<A>()[d * N + i], sA[i], 10 * tol);
    near("dD", d, (double)dD.as<A>()[d], sD, 10 * tol);
    near("dbias", d, (double)dbias.as<A>()[d], sbias, 10 * tol);
  }
  for (int64_t i = 0; i < nb; ++i) {
    near("dB", i, (double)(A)dB.as<T>()[i], sB[i], 10 * tol);
    near("dC", i, (double)(A)dC.as<T>()[i], sC[i], 10 * tol);
  }
}

}  // namespace

int main(int argc, char** argv) {
  if (argc != 9) return 2;
  const int dtype = std::atoi(argv[1]), N = std::atoi(argv[5]), G = std::atoi(argv[6]);
  const int64_t B = std::atoll(argv[2]), T = std::atoll(argv[3]), D = std::atoll(argv[4]);
  const bool ragged = std::atoi(argv[7]) != 0, optional = std::atoi(argv[8]) != 0;
  for (const bool at_end : {true, false}) {
    if (dtype == 0) check<double>(dtype, B, T, D, N, G, ragged, optional, at_end);
    else if (dtype == 1) check<float>(dtype, B, T, D, N, G, ragged, optional, at_end);
    else if (dtype == 2) check<bf16>(dtype, B, T, D, N, G, ragged, optional, at_end);
    else check<f16>(dtype, B, T, D, N, G, ragged, optional, at_end);
  }
  return done();
}
