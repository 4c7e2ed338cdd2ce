// The vocabulary's cross entropy as host code, of every type: its kernels on guarded arrays,
// each part of the workspace among them, so that a read or write past any of them ends the
// program; results are compared with the definition. Arguments:
//   run dtype rows words width apart shift tiles piece uneven
// apart: elements between rows beyond the width; shift: elements that the inputs are moved by;
// tiles: of all products, or -1 for the plan's; piece: words of a piece, or 0 for the plan's;
// uneven: rows with weights of their own, and rows without one.
//   empty
// the VJP of no rows: dw is cleared, at widths on both sides of every rule.
//   plans
// plans over a range of sizes: their tiles, splits, pieces and workspaces.

#include "matrix_lanes.h"
#include "seq_launch.h"

#include "linear_cross_entropy.h"

#include <memory>
#include <string>
#include <vector>

#include "guard.h"
#include "values.h"

namespace adst {
#define OF(name, T)                                                                             \
  hipError_t xent_forward_##name(const XentArgs& a, const XentPlan& p, void* ws, hipStream_t st) { \
    return forward_of<T>(a, p, ws, st);                                                         \
  }                                                                                             \
  hipError_t xent_vjp_##name(const XentArgs& a, const XentPlan& p, void* ws, hipStream_t st) {   \
    return vjp_of<T>(a, p, ws, st);                                                             \
  }
OF(f64, double)
OF(f32, float)
OF(bf16, bf16)
OF(f16, f16)
}  // namespace adst

using namespace adst;

namespace {

int64_t up_to(int64_t n, int64_t by) { return (n + by - 1) / by * by; }
int64_t size_of(int dtype) { return dtype == ADST_F64 ? 8 : dtype == ADST_F32 ? 4 : 2; }

// The workspace's parts: what each has to hold.
struct Part {
  const char* name;
  uint64_t XentPlan::*at;
  int64_t bytes;
};
std::vector<Part> parts_of(const XentPlan& p, int dtype, int64_t M, int64_t V, int64_t K,
                           bool reverse) {
  const int64_t e = size_of(dtype), acc = e == 8 ? 8 : 4;
  static const int64_t bn[] = {256, 128, 64, 64, 128};
  std::vector<Part> v;
  if (p.logits.splits > 1) v.push_back({"few", &XentPlan::few, p.logits.splits * M * V * acc});
  if (!reverse) {
    if (p.logits.splits == 1) {
      v.push_back({"stats", &XentPlan::stats,
                   (V + bn[p.logits.tiles] - 1) / bn[p.logits.tiles] * M * 2 * acc});
      v.push_back({"target", &XentPlan::target, M * acc});
    }
    return v;
  }
  v.push_back({"scale", &XentPlan::scale, 8});
  v.push_back({"xt", &XentPlan::xt, K * p.m_pad * e});
  v.push_back({"wt", &XentPlan::wt, K * p.piece * e});
  v.push_back({"g", &XentPlan::g, M * p.piece * e});
  v.push_back({"gt", &XentPlan::gt, p.piece * p.m_pad * e});
  if (!p.dx_direct) v.push_back({"dx_sums", &XentPlan::dx_sums, p.dx.splits * M * K * acc});
  if (p.dw.splits > 1) v.push_back({"dw_sums", &XentPlan::dw_sums, p.dw.splits * p.piece * K * acc});
  return v;
}

// The parts as arrays of their own: their places are counted from address 0.
std::vector<std::unique_ptr<Guarded>> place(XentPlan& p, int dtype, int64_t M, int64_t V,
                                            int64_t K, bool reverse, bool at_end) {
  std::vector<std::unique_ptr<Guarded>> held;
  for (const Part& q : parts_of(p, dtype, M, V, K, reverse)) {
    held.push_back(std::make_unique<Guarded>(q.bytes, at_end));
    p.*q.at = (uint64_t)(uintptr_t)held.back()->get();
  }
  return held;
}

template <class T>
void check(int dtype, int64_t M, int64_t V, int64_t K, int64_t apart, int64_t shift, int tiles,
           int64_t piece, bool uneven, bool at_end) {
  typedef Acc<T> A;
  const int64_t stride = K + apart;
  Guarded xs(((M - 1) * stride + K + shift) * sizeof(T), at_end),
      wsp(((V - 1) * stride + K + shift) * sizeof(T), at_end), labels(M * 4, at_end),
      loss(M * sizeof(A), at_end), lse(M * sizeof(A), at_end), dloss(M * sizeof(A), at_end),
      dx(M * K * sizeof(T), at_end), dw(V * K * sizeof(T), at_end);
  T *x = xs.as<T>() + shift, *w = wsp.as<T>() + shift;
  const double scale = 3 / std::sqrt((double)K);
  for (int64_t m = 0; m < M; ++m) {
    for (int64_t k = 0; k < K; ++k) x[m * stride + k] = (T)(2 * noise(m * K + k) - 1);
    int label = (int)(noise(m + 777) * (double)V);
    if (uneven && m % 5 == 3) label = m % 2 ? -1 : (int)V;
    labels.as<int32_t>()[m] = label;
    dloss.as<A>()[m] = (A)(!uneven ? 1 : m % 7 == 6 ? 0 : 2 * noise(m + 999) - 1);
  }
  for (int64_t v = 0; v < V; ++v)
    for (int64_t k = 0; k < K; ++k)
      w[v * stride + k] = (T)((2 * noise(v * K + k + 123456) - 1) * scale);
  XentArgs a{};
  a.x = x;
  a.w = w;
  a.sx = a.sw = stride;
  a.M = M;
  a.V = V;
  a.K = K;
  a.labels = labels.as<int32_t>();
  a.dtype = dtype;
  a.loss = loss.get();
  a.lse = lse.get();
  {
    XentPlan p = xent_plan(dtype, M, V, K, false);
    if (tiles >= 0) p.logits = {tiles, 1};
    const auto held = place(p, dtype, M, V, K, false, at_end);
    if (forward_of<T>(a, p, nullptr, nullptr) != hipSuccess) std::exit(3);
  }
  a.dloss = uneven ? dloss.get() : nullptr;
  a.dx = dx.get();
  a.dw = dw.get();
  {
    XentPlan p = xent_plan(dtype, M, V, K, true);
    if (tiles >= 0) {
      p.logits = {tiles, 1};
      p.dx.tiles = p.dw.tiles = tiles;
    }
    if (piece) {
      p.piece = piece;
      p.pieces = (V + piece - 1) / piece;
      p.dx_direct = p.dx_direct && p.pieces == 1;
    }
    const auto held = place(p, dtype, M, V, K, true, at_end);
    if (vjp_of<T>(a, p, nullptr, nullptr) != hipSuccess) std::exit(3);
  }
  // How far a result may be off, with u the type's half step and a the accumulation type's: a
  // logit of K products, (K + 2) a sum |x w|; lse, that of the largest and (V + 8) a for the sum
  // and logarithm, a rounding of each size; p = exp(logit - lse), p times its argument's error and
  // 2 |argument| + 4 roundings; g, the -1, the weight and its scale, 4 a, and u once where it is
  // held in 16 bits (F16: or 2^-38 of the largest weight, below its normal range); a sum of n
  // terms, (n + 8) a of their sizes; the result's own rounding, u.
  const double ua = sizeof(A) == 8 ? 0x1p-53 : 0x1p-24;
  const double u = sizeof(T) == 8 ? 0x1p-53 : sizeof(T) == 4 ? 0x1p-24
                   : dtype == ADST_BF16 ? 0x1p-8 : 0x1p-11;
  const double of_g = sizeof(T) == 2 ? u : 0;
  double most = 0;
  for (int64_t m = 0; m < M; ++m) most = std::fmax(most, std::fabs((double)dloss.as<A>()[m]));
  const double least = dtype == ADST_F16 ? 0x1p-38 * most : 0;
  struct Sum {
    double v = 0, size = 0, off = 0;
    void add(double g, double far, double by) {
      v += g * by;
      size += (std::fabs(g) + far) * std::fabs(by);
      off += far * std::fabs(by);
    }
  };
  std::vector<Sum> want_dx(M * K), want_dw(V * K);
  std::vector<double> logit(V), size(V);
  const auto within = [&](const char* name, int64_t i, double got, double want, double bound) {
    near(name, i, got, want, bound / (1 + std::fabs(want)));
  };
  for (int64_t m = 0; m < M; ++m) {
    double top = -INFINITY, sum = 0, off = 0;
    for (int64_t v = 0; v < V; ++v) {
      double s = 0, abs = 0;
      for (int64_t k = 0; k < K; ++k) {
        const double term = (double)(A)x[m * stride + k] * (double)(A)w[v * stride + k];
        s += term;
        abs += std::fabs(term);
      }
      logit[v] = s;
      top = std::fmax(top, s);
      off = std::fmax(off, (K + 2) * ua * abs);
    }
    for (int64_t v = 0; v < V; ++v) sum += std::exp(logit[v] - top);
    const double z = top + std::log(sum);
    const int64_t label = labels.as<int32_t>()[m];
    const bool has = label >= 0 && label < V;
    double low = 0;  // the farthest argument of an exponential
    for (int64_t v = 0; v < V; ++v) low = std::fmax(low, std::fabs(logit[v] - z));
    const double of_z = off + (V + 8 + 2 * low + 4) * ua + 4 * ua * (std::fabs(z) + std::fabs(top) + 1);
    within("lse", m, (double)lse.as<A>()[m], z, of_z);
    const double loss_ = has ? z - logit[label] : 0;
    within("loss", m, (double)loss.as<A>()[m], loss_,
           has ? of_z + off + ua * (std::fabs(z) + std::fabs(logit[label])) : 0);
    const double weight = has ? uneven ? (double)dloss.as<A>()[m] : 1 : 0;
    if (weight == 0) continue;
    for (int64_t v = 0; v < V; ++v) {
      const double p = std::exp(logit[v] - z), hot = v == label, g = (p - hot) * weight;
      const double arg = std::fabs(logit[v] - z);
      double far = (p * (off + of_z + ua * (std::fabs(logit[v]) + std::fabs(z)) + (2 * arg + 4) * ua) +
                    4 * ua * (p + hot)) * std::fabs(weight);
      far += of_g * (std::fabs(g) + far) + least;
      for (int64_t k = 0; k < K; ++k) {
        want_dx[m * K + k].add(g, far, (double)(A)w[v * stride + k]);
        want_dw[v * K + k].add(g, far, (double)(A)x[m * stride + k]);
      }
    }
  }
  const auto sums = [&](const char* name, const T* got, const std::vector<Sum>& want, int64_t n) {
    for (size_t i = 0; i < want.size(); ++i) {
      const double bound = want[i].off + (n + 8) * ua * want[i].size;
      within(name, i, (double)(A)got[i], want[i].v, bound + u * (std::fabs(want[i].v) + bound) +
                                                        (dtype == ADST_F16 ? 0x1p-25 : 0));
    }
  };
  sums("dx", dx.as<T>(), want_dx, V);
  sums("dw", dw.as<T>(), want_dw, M);
}

// No rows: through the same call as any other.
template <class T>
void empty(int dtype, int64_t K, int64_t V) {
  Guarded dw(V * K * sizeof(T), true);
  XentArgs a{};
  a.sx = a.sw = K;
  a.V = V;
  a.K = K;
  a.dtype = dtype;
  a.dw = dw.get();
  std::printf("no rows, dtype %d, width %lld, %lld words\n", dtype, (long long)K, (long long)V);
  std::fflush(stdout);
  if (xent_vjp(a, nullptr, nullptr) != hipSuccess) std::exit(3);
  for (int64_t i = 0; i < V * K; ++i) near("dw", i, (double)(Acc<T>)dw.as<T>()[i], 0, 0);
}

void wrong_plan(const char* what, int dtype, int64_t M, int64_t V, int64_t K) {
  if (wrong++ < 8)
    std::printf("%s: dtype %d, %lld rows, %lld words, width %lld\n", what, dtype, (long long)M,
                (long long)V, (long long)K);
}

void check_plan(int dtype, int64_t M, int64_t V, int64_t K) {
  const int64_t e = size_of(dtype), step = 128 / e;
  for (const bool reverse : {false, true}) {
    const XentPlan p = xent_plan(dtype, M, V, K, reverse);
    const auto product = [&](const XentPlan::Product& q, int64_t steps) {
      if (q.tiles < (dtype == ADST_F64) || q.tiles > 4 || q.splits < 1 || q.splits > steps)
        wrong_plan("tiles or splits", dtype, M, V, K);
    };
    product(p.logits, up_to(K, step) / step);
    if (reverse) {
      product(p.dx, p.piece / step);
      product(p.dw, p.m_pad / step);
      if (p.piece < 1 || p.piece % step || p.pieces * p.piece < V || (p.pieces - 1) * p.piece >= V ||
          (p.pieces > 1 && p.piece % 256))
        wrong_plan("pieces", dtype, M, V, K);
      if (p.logits.splits > 1 && p.pieces > 1) wrong_plan("few logits", dtype, M, V, K);
      if (p.m_pad < M || p.m_pad % step) wrong_plan("rows", dtype, M, V, K);
      // 128 MB of g, or the 1024 words that a piece has at least
      if (M * p.piece * e > (128 << 20) && p.piece > 1024) wrong_plan("a piece's size", dtype, M, V, K);
    }
    // each part within the workspace, and apart from the others
    const auto parts = parts_of(p, dtype, M, V, K, reverse);
    for (const Part& q : parts) {
      if (p.*q.at % 256 || p.*q.at + (uint64_t)q.bytes > p.bytes)
        wrong_plan(q.name, dtype, M, V, K);
      for (const Part& r : parts)
        if (q.at != r.at && p.*q.at <= p.*r.at && p.*r.at < p.*q.at + (uint64_t)q.bytes &&
            r.bytes > 0)
          wrong_plan(r.name, dtype, M, V, K);
    }
  }
}

}  // namespace

int main(int argc, char** argv) {
  const std::string what = argc > 1 ? argv[1] : "";
  if (what == "plans") {
    const int64_t rows[] = {1, 2, 15, 16, 17, 63, 64, 65, 500, 999, 4096, 8192, 65537, 1 << 20};
    const int64_t words[] = {1, 2, 7, 64, 65, 300, 1024, 4096, 4097, 32000, 65537, 1 << 20};
    const int64_t widths[] = {1, 8, 63, 255, 256, 257, 512, 767, 768, 1024, 1536, 2048, 4096, 20000};
    for (int dtype = 0; dtype < 4; ++dtype)
      for (const int64_t M : rows)
        for (const int64_t V : words)
          for (const int64_t K : widths)
            if (M * (K + 64) < int64_t(1) << 31 && V * (K + 64) < int64_t(1) << 31 &&
                (M + 256) * (V + 256) < int64_t(1) << 35)
              check_plan(dtype, M, V, K);
    return done();
  }
  if (what == "empty") {
    for (const int64_t K : {1, 8, 255, 256, 511, 512, 1535, 1536, 2048, 4096})
      for (const int64_t V : {1, 20, 64, 5000})
        if (K * V < 200000) {
          empty<double>(ADST_F64, K, V);
          empty<float>(ADST_F32, K, V);
          empty<bf16>(ADST_BF16, K, V);
          empty<f16>(ADST_F16, K, V);
        }
    return done();
  }
  if (what != "run" || argc != 11) return 2;
  int64_t n[9];
  for (int i = 0; i < 9; ++i) n[i] = std::atoll(argv[i + 2]);
  for (const bool at_end : {true, false}) {
    const auto go = [&](auto t) {
      check<decltype(t)>((int)n[0], n[1], n[2], n[3], n[4], n[5], (int)n[6], n[7], n[8] != 0,
                         at_end);
    };
    switch (n[0]) {
      case ADST_F64: go(double()); break;
      case ADST_F32: go(float()); break;
      case ADST_BF16: go(bf16()); break;
      default: go(f16());
    }
  }
  return done();
}
