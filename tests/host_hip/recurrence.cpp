// The recurrence's kernels as host code, on guarded arrays: a read or write
// past an array, the workspace among them, ends the program. Results are
// compared with the definition. Arguments: dtype gate batch steps channels ragged.

#include "recurrence.host.inc"

#include <vector>

#include "guard.h"
#include "values.h"

using namespace adst;

namespace {

template <class T>
void check(int dtype, int gate, int64_t B, int64_t T_, int64_t D, bool ragged, bool at_end) {
  typedef Acc<T> A;
  const double tol = sizeof(T) == 8 ? 1e-9 : sizeof(T) == 4 ? 1e-4 : 2e-2;
  const int64_t n = B * T_ * D;
  const RecPlan plan = rec_plan(dtype, B, T_, D);
  Guarded a(n * sizeof(T), at_end), u(n * sizeof(T), at_end), dh(n * sizeof(T), at_end),
      h(n * sizeof(T), at_end), da(n * sizeof(T), at_end), du(n * sizeof(T), at_end),
      h0(B * D * sizeof(A), at_end), hT(B * D * sizeof(A), at_end), dhT(B * D * sizeof(A), at_end),
      dh0(B * D * sizeof(A), at_end), lens(B * 4, at_end), ck(plan.ck_bytes, at_end),
      ws(plan.ws_bytes, at_end);
  for (int64_t i = 0; i < n; ++i) {
    a.as<T>()[i] = (T)(gate ? 4 * noise(i) - 1 : 0.5 + 0.5 * noise(i));
    u.as<T>()[i] = (T)(2 * noise(i + n) - 1);
    dh.as<T>()[i] = (T)(2 * noise(i + 2 * n) - 1);
  }
  for (int64_t i = 0; i < B * D; ++i) {
    h0.as<A>()[i] = (A)(2 * noise(i + 3 * n) - 1);
    dhT.as<A>()[i] = (A)(2 * noise(i + 4 * n) - 1);
  }
  for (int64_t b = 0; b < B; ++b)
    lens.as<int32_t>()[b] = b == B - 1 ? (int32_t)T_ : (int32_t)(noise(b + 5 * n) * (double)T_);
  RecArgs r{};
  r.a = a.get();
  r.u = u.get();
  r.h0 = h0.get();
  r.lens = ragged ? lens.as<int32_t>() : nullptr;
  r.sa_b = r.su_b = r.sd_b = T_ * D;
  r.sa_t = r.su_t = r.sd_t = D;
  r.B = B;
  r.T = T_;
  r.D = D;
  r.dtype = dtype;
  r.gate = gate;
  r.h = h.get();
  r.hT = hT.get();
  r.ck = ck.get();
  if (rec_forward(r, ws.get(), nullptr) != hipSuccess) std::exit(3);
  r.dh = dh.get();
  r.dhT = dhT.get();
  r.da = da.get();
  r.du = du.get();
  r.dh0 = dh0.get();
  if (rec_vjp(r, ws.get(), nullptr) != hipSuccess) std::exit(3);
  std::vector<double> x(T_ + 1);
  for (int64_t b = 0; b < B; ++b)
    for (int64_t d = 0; d < D; ++d) {
      const int64_t len = ragged ? lens.as<int32_t>()[b] : T_;
      const auto at = [&](int64_t t) { return (b * T_ + t) * D + d; };
      const auto coeff = [&](int64_t t) {
        const double v = (double)(A)a.as<T>()[at(t)];
        return gate ? 1 / (1 + std::exp(-v)) : v;
      };
      x[0] = (double)h0.as<A>()[b * D + d];
      for (int64_t t = 0; t < T_; ++t) {
        const double c = coeff(t), v = (double)(A)u.as<T>()[at(t)];
        x[t + 1] = t < len ? c * x[t] + (gate ? (1 - c) * v : v) : x[t];
        near("h", at(t), (double)(A)h.as<T>()[at(t)], t < len ? x[t + 1] : 0, tol);
      }
      near("hT", b * D + d, (double)hT.as<A>()[b * D + d], x[T_], tol);
      double G = (double)dhT.as<A>()[b * D + d];
      for (int64_t t = T_ - 1; t >= 0; --t) {
        double ga = 0, gu = 0;
        if (t < len) {
          const double c = coeff(t), v = (double)(A)u.as<T>()[at(t)];
          G += (double)(A)dh.as<T>()[at(t)];
          ga = gate ? G * (x[t] - v) * c * (1 - c) : G * x[t];
          gu = gate ? G * (1 - c) : G;
          G *= c;
        }
        near("da", at(t), (double)(A)da.as<T>()[at(t)], ga, tol);
        near("du", at(t), (double)(A)du.as<T>()[at(t)], gu, tol);
      }
      near("dh0", b * D + d, (double)dh0.as<A>()[b * D + d], G, tol);
    }
}

}  // namespace

int main(int argc, char** argv) {
  if (argc != 7) return 2;
  const int dtype = std::atoi(argv[1]), gate = std::atoi(argv[2]);
  const int64_t B = std::atoll(argv[3]), T = std::atoll(argv[4]), D = std::atoll(argv[5]);
  const bool ragged = std::atoi(argv[6]) != 0;
  for (const bool at_end : {true, false}) {
    std::printf("dtype %d gate %d: %lld x %lld x %lld%s, arrays %s a guarded page\n", dtype, gate,
                (long long)B, (long long)T, (long long)D, ragged ? " ragged" : "",
                at_end ? "before" : "behind");
    std::fflush(stdout);
    (void)by_type(dtype, [&](auto t) {
      check<decltype(t)>(dtype, gate, B, T, D, ragged, at_end);
      return hipSuccess;
    });
  }
  return done();
}
