// Layer norm's kernels as host code, on guarded arrays: a read or write past an
// array, the workspace among them, ends the program. Results are compared with
// the definition. Arguments: dtype weight_dtype rows n gap (between rows), or
// rows n: nothing runs, but every type's launches have to fit a dispatch.

#include "layer_norm.host.inc"

#include <vector>

#include "guard.h"
#include "values.h"

using namespace adst;

namespace {

template <class T, class W>
void check(int dtype, int wtype, int64_t M, int64_t N, int64_t gap, bool at_end) {
  typedef Acc<T> A;
  const double tol = sizeof(T) == 8 ? 1e-9 : sizeof(T) == 4 ? 1e-3 : 2e-2, eps = 1e-5;
  const double wtol = sizeof(W) == 2 ? 2e-2 : tol;
  const int64_t s = N + gap, span = M ? (M - 1) * s + N : 0;
  Guarded x(span * sizeof(T), at_end), dy(span * sizeof(T), at_end), w(N * sizeof(W), at_end),
      b(N * sizeof(W), at_end), y(M * N * sizeof(T), at_end), dx(M * N * sizeof(T), at_end),
      mean(M * sizeof(A), at_end), rstd(M * sizeof(A), at_end), dw(N * sizeof(W), at_end),
      db(N * sizeof(W), at_end), ws(M ? norm_workspace_bytes(dtype, M, N) : 0, at_end);
  for (int64_t i = 0; i < span; ++i) {
    x.as<T>()[i] = (T)(2 * noise(i) + noise(i / s));
    dy.as<T>()[i] = (T)(2 * noise(i + span) - 1);
  }
  for (int64_t c = 0; c < N; ++c) {
    w.as<W>()[c] = (W)(0.5 + noise(c + 2 * span));
    b.as<W>()[c] = (W)(noise(c + 3 * span) - 0.5);
  }
  NormArgs a{};
  a.x = x.get();
  a.dy = dy.get();
  a.w = w.get();
  a.b = b.get();
  a.sx = a.sdy = s;
  a.rows = M;
  a.n = N;
  a.eps = eps;
  a.dtype = dtype;
  a.wtype = wtype;
  a.y = y.get();
  a.mean = mean.get();
  a.rstd = rstd.get();
  if (M > 0 && norm_forward(a, nullptr) != hipSuccess) std::exit(3);
  a.dx = dx.get();
  a.dw = dw.get();
  a.db = db.get();
  if (norm_vjp(a, ws.get(), nullptr) != hipSuccess) std::exit(3);
  std::vector<double> sw(N), sb(N);
  for (int64_t r = 0; r < M; ++r) {
    const T *xr = x.as<T>() + r * s, *dr = dy.as<T>() + r * s;
    double mu = 0, var = 0, e1 = 0, e2 = 0;
    for (int64_t c = 0; c < N; ++c) mu += (double)(A)xr[c] / N;
    for (int64_t c = 0; c < N; ++c) var += ((double)(A)xr[c] - mu) * ((double)(A)xr[c] - mu) / N;
    const double inv = 1 / std::sqrt(var + eps);
    for (int64_t c = 0; c < N; ++c) {
      const double h = ((double)(A)xr[c] - mu) * inv, d = (double)(A)dr[c];
      e1 += d * (double)(A)w.as<W>()[c] / N;
      e2 += d * (double)(A)w.as<W>()[c] * h / N;
      sw[c] += d * h;
      sb[c] += d;
    }
    near("mean", r, (double)mean.as<A>()[r], mu, tol);
    near("rstd", r, (double)rstd.as<A>()[r], inv, tol);
    for (int64_t c = 0; c < N; ++c) {
      const double h = ((double)(A)xr[c] - mu) * inv, wc = (double)(A)w.as<W>()[c];
      near("y", r * N + c, (double)(A)y.as<T>()[r * N + c], h * wc + (double)(A)b.as<W>()[c], tol);
      near("dx", r * N + c, (double)(A)dx.as<T>()[r * N + c],
           ((double)(A)dr[c] * wc - e1 - h * e2) * inv, tol);
    }
  }
  for (int64_t c = 0; c < N; ++c) {
    near("dw", c, (double)(A)dw.as<W>()[c], sw[c], wtol);
    near("db", c, (double)(A)db.as<W>()[c], sb[c], wtol);
  }
}

int grids(int64_t rows, int64_t n) {
  host_hip::only_grids = true;
  char here;  // in place of every array
  int failed = 0;
  for (int dtype = ADST_F64; dtype <= ADST_F16; ++dtype) {
    NormArgs a{};
    a.x = a.dy = a.w = a.b = &here;
    a.y = a.mean = a.rstd = a.dx = a.dw = a.db = &here;
    a.sx = a.sdy = a.n = n;
    a.rows = rows;
    a.dtype = a.wtype = dtype;
    const bool forward = norm_forward(a, nullptr) == hipSuccess;
    const bool reverse = norm_vjp(a, &here, nullptr) == hipSuccess;
    if (!forward || !reverse) ++failed, std::printf("dtype %d: a launch does not fit\n", dtype);
  }
  return failed != 0;
}

}  // namespace

int main(int argc, char** argv) {
  if (argc == 3) return grids(std::atoll(argv[1]), std::atoll(argv[2]));
  if (argc != 6) return 2;
  const int dtype = std::atoi(argv[1]), wtype = std::atoi(argv[2]);
  const int64_t M = std::atoll(argv[3]), N = std::atoll(argv[4]), gap = std::atoll(argv[5]);
  for (const bool at_end : {true, false}) {
    std::printf("dtype %d, weights %d: %lld x %lld, arrays %s a guarded page\n", dtype, wtype,
                (long long)M, (long long)N, at_end ? "before" : "behind");
    std::fflush(stdout);
    (void)by_type(dtype, wtype, [&](auto t, auto w) {
      check<decltype(t), decltype(w)>(dtype, wtype, M, N, gap, at_end);
      return hipSuccess;
    });
  }
  return done();
}
