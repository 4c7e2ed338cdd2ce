// The causal convolution's kernels as host code, on guarded arrays: a read or
// write past an array, the workspace among them, ends the program. Results are
// compared with the definition. Arguments: dtype weight_dtype act taps batch steps
// channels ragged.

#include "causal_conv.host.inc"

#include <vector>

#include "guard.h"
#include "values.h"

using namespace adst;

namespace {

template <class T>
void check(int dtype, int wtype, int act, int K, int64_t B, int64_t T_, int64_t D, bool ragged,
           bool at_end) {
  typedef Acc<T> A;
  const double tol = sizeof(T) == 8 ? 1e-9 : sizeof(T) == 4 ? 1e-4 : 3e-2;
  const int64_t n = B * T_ * D, m = B * (K - 1) * D;
  const bool same = dtype == wtype;
  const int we = same ? sizeof(T) : 4;
  Guarded x(n * sizeof(T), at_end), dy(n * sizeof(T), at_end), y(n * sizeof(T), at_end),
      dx(n * sizeof(T), at_end), x0(m * sizeof(T), at_end), xT(m * sizeof(T), at_end),
      dx0(m * sizeof(T), at_end), dxT(m * sizeof(T), at_end), w(K * D * we, at_end),
      bias(D * we, at_end), dw(K * D * we, at_end), db(D * we, at_end), lens(B * 4, at_end);
  const auto weight = [&](const Guarded& g, int64_t i) {
    return same ? (double)(A)g.as<T>()[i] : (double)g.as<float>()[i];
  };
  const auto set = [&](const Guarded& g, int64_t i, double v) {
    if (same) g.as<T>()[i] = (T)v;
    else g.as<float>()[i] = (float)v;
  };
  for (int64_t i = 0; i < n; ++i) {
    x.as<T>()[i] = (T)(2 * noise(i) - 1);
    dy.as<T>()[i] = (T)(2 * noise(i + n) - 1);
  }
  for (int64_t i = 0; i < m; ++i) {
    x0.as<T>()[i] = (T)(2 * noise(i + 2 * n) - 1);
    dxT.as<T>()[i] = (T)(2 * noise(i + 3 * n) - 1);
  }
  for (int64_t i = 0; i < K * D; ++i) set(w, i, 2 * noise(i + 4 * n) - 1);
  for (int64_t i = 0; i < D; ++i) set(bias, i, 2 * noise(i + 5 * n) - 1);
  for (int64_t b = 0; b < B; ++b)
    lens.as<int32_t>()[b] = b == B - 1 ? (int32_t)T_ : (int32_t)(noise(b + 7 * n) * (double)T_);
  ConvArgs a{};
  a.x = x.get();
  a.w = w.get();
  a.bias = bias.get();
  a.x0 = x0.get();
  a.lens = ragged ? lens.as<int32_t>() : nullptr;
  a.sx_b = a.sd_b = T_ * D;
  a.sx_t = a.sd_t = D;
  a.B = B;
  a.T = T_;
  a.D = D;
  a.dtype = dtype;
  a.wtype = wtype;
  a.act = act;
  a.taps = K;
  a.y = y.get();
  a.xT = xT.get();
  if (conv_forward(a, nullptr) != hipSuccess) std::exit(3);
  Guarded ws(conv_workspace_bytes(dtype, B, T_, D, K), at_end);
  a.dy = dy.get();
  a.dxT = dxT.get();
  a.dx = dx.get();
  a.dw = dw.get();
  a.dbias = db.get();
  a.dx0 = dx0.get();
  if (conv_vjp(a, ws.get(), nullptr) != hipSuccess) std::exit(3);
  for (int64_t d = 0; d < D; ++d) {
    std::vector<double> sw(K + 1, 0.0);
    for (int64_t b = 0; b < B; ++b) {
      const int64_t len = ragged ? lens.as<int32_t>()[b] : T_;
      std::vector<double> seen(len + K - 1), g(len + K - 1, 0.0);
      for (int64_t t = 0; t < len + K - 1; ++t)
        seen[t] = t < K - 1 ? (double)(A)x0.as<T>()[(b * (K - 1) + t) * D + d]
                            : (double)(A)x.as<T>()[(b * T_ + t - K + 1) * D + d];
      for (int j = 0; j < K - 1; ++j) {
        near("xT", j, (double)(A)xT.as<T>()[(b * (K - 1) + j) * D + d], seen[len + j], 0);
        g[len + j] += (double)(A)dxT.as<T>()[(b * (K - 1) + j) * D + d];
      }
      for (int64_t t = 0; t < T_; ++t) {
        const int64_t at = (b * T_ + t) * D + d;
        double v = 0, s = 1, slope = 1;
        if (t < len) {
          v = weight(bias, d);
          for (int k = 0; k < K; ++k) v += weight(w, k * D + d) * seen[t + k];
          if (act) {
            s = 1 / (1 + std::exp(-v));
            slope = s * (1 + v * (1 - s));
          }
          const double e = (double)(A)dy.as<T>()[at] * slope;
          for (int k = 0; k < K; ++k) {
            g[t + k] += weight(w, k * D + d) * e;
            sw[k] += e * seen[t + k];
          }
          sw[K] += e;
        }
        near("y", at, (double)(A)y.as<T>()[at], t < len ? (act ? v * s : v) : 0, tol);
      }
      for (int64_t t = 0; t < T_; ++t)
        near("dx", t, (double)(A)dx.as<T>()[(b * T_ + t) * D + d], t < len ? g[t + K - 1] : 0, tol);
      for (int j = 0; j < K - 1; ++j)
        near("dx0", j, (double)(A)dx0.as<T>()[(b * (K - 1) + j) * D + d], g[j], tol);
    }
    const double wide = tol * 4;
    for (int k = 0; k < K; ++k) near("dw", k * D + d, weight(dw, k * D + d), sw[k], wide);
    near("db", d, weight(db, d), sw[K], wide);
  }
}

// One step of rows whose windows are in a pool, idle ones among them.
template <class T>
void check_step(int dtype, int wtype, int act, int K, int64_t B, int64_t D, bool at_end) {
  typedef Acc<T> A;
  const double tol = sizeof(T) == 8 ? 1e-9 : sizeof(T) == 4 ? 1e-4 : 3e-2;
  const bool same = dtype == wtype;
  const int we = same ? sizeof(T) : 4;
  const int64_t pool = B + 3;
  Guarded x(B * D * sizeof(T), at_end), y(B * D * sizeof(T), at_end), w(K * D * we, at_end),
      window(pool * (K - 1) * D * sizeof(T), at_end), slots(B * 4, at_end);
  std::vector<double> before(pool * (K - 1) * D);
  for (int64_t i = 0; i < B * D; ++i) x.as<T>()[i] = (T)(2 * noise(i) - 1);
  for (int64_t i = 0; i < pool * (K - 1) * D; ++i)
    before[i] = (double)(A)(window.as<T>()[i] = (T)(2 * noise(i + 9999) - 1));
  for (int64_t i = 0; i < K * D; ++i) {
    if (same) w.as<T>()[i] = (T)(2 * noise(i + 777) - 1);
    else w.as<float>()[i] = (float)(2 * noise(i + 777) - 1);
  }
  for (int64_t b = 0; b < B; ++b)
    slots.as<int32_t>()[b] = b % 3 == 1 ? (b % 2 ? -1 : (int32_t)pool) : (int32_t)(pool - 1 - b);
  const ConvStep q{x.get(), w.get(), nullptr, D, slots.as<int32_t>(), window.get(), pool,
                   y.get(), B, D, dtype, wtype, act, K};
  if (conv_step(q, nullptr) != hipSuccess) std::exit(3);
  for (int64_t b = 0; b < B; ++b)
    for (int64_t d = 0; d < D; ++d) {
      const int64_t slot = slots.as<int32_t>()[b];
      const bool on = slot >= 0 && slot < pool;
      double v = 0;
      for (int k = 0; k < K && on; ++k) {
        const double seen = k == K - 1 ? (double)(A)x.as<T>()[b * D + d]
                                       : before[(slot * (K - 1) + k) * D + d];
        v += (same ? (double)(A)w.as<T>()[k * D + d] : (double)w.as<float>()[k * D + d]) * seen;
        if (k > 0)
          near("window", d, (double)(A)window.as<T>()[(slot * (K - 1) + k - 1) * D + d], seen, 0);
      }
      if (act) v = v / (1 + std::exp(-v));
      near("step", b * D + d, (double)(A)y.as<T>()[b * D + d], v, tol);
    }
}

}  // namespace

int main(int argc, char** argv) {
  if (argc != 9) return 2;
  const int dtype = std::atoi(argv[1]), wtype = std::atoi(argv[2]), act = std::atoi(argv[3]),
            K = std::atoi(argv[4]);
  const int64_t B = std::atoll(argv[5]), T = std::atoll(argv[6]), D = std::atoll(argv[7]);
  const bool ragged = std::atoi(argv[8]) != 0;
  for (const bool at_end : {true, false}) {
    (void)by_type(dtype, [&](auto t) {
      check<decltype(t)>(dtype, wtype, act, K, B, T, D, ragged, at_end);
      if (B > 0) check_step<decltype(t)>(dtype, wtype, act, K, B, D, at_end);
      return hipSuccess;
    });
  }
  return done();
}
