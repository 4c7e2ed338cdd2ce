// Selective scan: per channel d and state n
//   h_t[n] = exp(s_t A[n]) h_{t-1}[n] + s_t x_t B_t[n],  s_t = softplus(delta_t + bias),
//   y_t = (sum_n C_t[n] h_t[n] + D x_t) z_t / (1 + exp(-z_t)),
// its VJP, and one step on a pool of states.
//
// A value of x, delta, z and y takes part in 7 operations for each of its N
// states, an exponential among them that costs as much as four others: with 16
// states the vector units' work bounds it, not memory. A lane holds NS states of
// a channel, half a wave 32 channels, and a workgroup all states of its 32
// channels, so each exponential is taken once. Steps go in chunks through LDS:
// the workgroup's threads first share the work that a step has once for all
// states (softplus, s x), then every lane runs its states over the chunk's steps
// and leaves its share of y's sum over the states, then the threads share the
// sums, the gate and the stores. The next chunk's inputs are requested before a
// chunk is worked on.
//
// Where a batch's rows and channels do not fill the card the time axis is cut
// into segments. A segment's map h -> exp(A sum_t s_t) h + H takes one sweep from
// h = 0; every segment then starts from the maps of those before it, applied in
// order.
//
// In reverse G_t = C_t dy'_t + exp(s_{t+1} A) G_{t+1}, dy' = dy times the gate, and
//   dC_t = sum_d dy'_t h_t,  dB_t = sum_d G_t s_t x_t,  u_t = sum_n G_t B_t,
//   dx_t = s_t u_t + D dy'_t,  ds_t = x_t u_t + sum_n A q_t,  dA = sum_t s_t q_t,
// with q_t = G_t exp(s_t A) h_{t-1}. A chunk's states are recomputed in registers
// from the checkpoint at its start, which the forward sweep left. The sums over
// channels are taken across lanes as a transposition: five exchanges that halve the
// number of registers each, after which a lane holds one step's and state's sum.
// They and dA leave the workgroup as partial sums that later kernels add in an
// order which the sizes alone set.
#pragma once

#include "packs.h"
#include "seq_common.h"
#include "token_kernels.h"

namespace adst {
namespace {

constexpr int kSlab = 32;  // channels of a workgroup: half a wave

// NS states of a lane, W waves of a workgroup, which hold up to 2 NS W states.
template <class T, int NS_, int W_>
struct ScanShape {
  typedef Acc<T> A;
  static constexpr int NS = NS_, W = W_;
  // Steps of a chunk: their states' registers are what the reverse sweep has most of.
  static constexpr int R = (sizeof(T) == 8 ? 16 : 32) / (NS < 2 ? 2 : NS);
  static constexpr int NT = 64 * W;
  static constexpr int SG = 2 * W;             // lanes that share a channel
  static constexpr int NP = SG * NS;           // states, those that are not there included
  static constexpr int E = R * kSlab >= NT ? R * kSlab / NT : 1;  // a thread's channels of a step
  static constexpr int kRowThreads = kSlab / E;
  static constexpr int kLoaders = R * kRowThreads;  // threads that load and store
  static constexpr int NB = (R * NP + NT - 1) / NT;  // values of B, and of C, a thread loads
  typedef Pack<T, E> P;
};

// The number of a chunk's steps, known to the compiler where the chunk is whole.
template <bool WHOLE, int R>
struct Steps {
  static constexpr bool kWhole = WHOLE;
  int n;
  __device__ bool has(int r) const { return WHOLE || r < n; }
};

__device__ inline float exp2_(float v) { return __builtin_amdgcn_exp2f(v); }
// exp(s A) from the coefficient that `rate` makes of A.
__device__ inline float rate(float a) { return a * 1.44269504f; }
__device__ inline double rate(double a) { return a; }
__device__ inline float decay(float s, float rate) { return exp2_(s * rate); }
__device__ inline double decay(double s, double rate) { return exp(s * rate); }
template <class A>
__device__ inline A of_rate(A v) {  // a sum of rates, as one of A's values
  return sizeof(A) == 4 ? v * A(0.69314718f) : v;
}

// log(1 + exp(v)): max(v, 0) + log(1 + e), e = exp(-|v|), and log(1 + e) = 2 atanh(e / (2 + e))
// by its series, whose argument is at most 1/3 (the ninth term is below 2^-29 of the first).
__device__ inline float softplus(float v) {
  const float e = exp2_(-1.44269504f * __builtin_fabsf(v));
  const float s = e * inverse(2.0f + e), q = s * s;
  float p = 1.0f / 15;
  p = fma_(p, q, 1.0f / 13);
  p = fma_(p, q, 1.0f / 11);
  p = fma_(p, q, 1.0f / 9);
  p = fma_(p, q, 1.0f / 7);
  p = fma_(p, q, 1.0f / 5);
  p = fma_(p, q, 1.0f / 3);
  p = fma_(p, q, 1.0f);
  return fma_(2.0f * s, p, v > 0 ? v : 0.0f);
}
__device__ inline double softplus(double v) {
  return (v > 0 ? v : 0.0) + log1p(exp(-__builtin_fabs(v)));
}

// Where a workgroup is.
struct Place {
  int64_t slab, group, segment, b;
  int64_t d0;  // first channel
  int channels;
};
__device__ inline Place place_of(const ScanArgs& a, const ScanGrid& g, int64_t id) {
  Place p;
  p.slab = id % g.slabs;
  p.segment = id / g.slabs % g.segments;
  p.b = id / (g.slabs * g.segments);
  p.group = p.slab / g.group_slabs;
  const int64_t of_group = a.D_ / a.G, at = p.slab % g.group_slabs * kSlab;
  p.d0 = p.group * of_group + at;
  p.channels = (int)(of_group - at < kSlab ? of_group - at : kSlab);
  return p;
}
// Consecutive workgroups go to the 8 XCDs in turn; each XCD gets neighbouring slabs, which
// share cache lines.
__device__ inline int64_t work_id(int64_t n) {
  const int64_t x = blockIdx.x;
  return n % 8 == 0 ? x % 8 * (n / 8) + x / 8 : x;
}

// What a thread loads and stores of a chunk: E channels of step `row`. FULL: every slab has
// all of its channels. Loads need no bounds: steps that are not there are read as the
// first one, channels as the last one, and their values are not used.
template <class S, bool FULL>
struct Loader {
  int row, c, last, n;  // n: channels that exist
  bool stores;
  __device__ Loader(const Place& p) {
    row = threadIdx.x / S::kRowThreads % S::R;
    c = threadIdx.x % S::kRowThreads * S::E;
    last = p.channels - 1;
    n = FULL ? S::E : p.channels - c < S::E ? p.channels - c : S::E;
    stores = threadIdx.x < S::kLoaders && (FULL || n > 0);
  }
  template <class T>
  __device__ Pack<T, S::E> load(const T* from) const {  // from: of the slab's first channel
    Pack<T, S::E> v;
    if constexpr (FULL) {
      v = load_pack<T, S::E>(from + c, S::E);
    } else {
#pragma unroll
      for (int i = 0; i < S::E; ++i) v.v[i] = from[c + i < last ? c + i : last];
    }
    return v;
  }
  template <class T>
  __device__ void store(T* to, const Pack<T, S::E>& v) const {
    store_pack<T, S::E>(to + c, v, n);
  }
  template <class A>
  __device__ void constants(const void* from, int64_t d0, A (&to)[S::E]) const {
#pragma unroll
    for (int i = 0; i < S::E; ++i)
      to[i] = from ? static_cast<const A*>(from)[d0 + (c + i < last ? c + i : last)] : A(0);
  }
};

// An input [batch][step][channel] as a thread goes through it, chunk after chunk.
template <class T>
struct Walk {
  const T *first, *at;  // step t0 of the segment; the thread's step of the next chunk
  int64_t stride;
  __device__ Walk(const void* p, int64_t b, int64_t sb, int64_t st, int64_t t0, int64_t d0)
      : first(p ? static_cast<const T*>(p) + b * sb + t0 * st + d0 : nullptr), stride(st) {}
  __device__ void go(int64_t step) { at = first + step * stride; }  // steps after t0
  __device__ const T* next(bool there, int steps) {
    const T* const now = there ? at : first;
    at += steps * stride;
    return now;
  }
};

// B and C of a chunk, {B, C} of a lane's states together in LDS.
template <class S>
struct Coefficients {
  typedef typename S::A A;
  struct alignas(2 * S::NS * sizeof(A)) Of {
    A b[S::NS], c[S::NS];
  };
};
template <class T, class S>
struct CoefficientLoader {
  Walk<T> b, c;
  int row[S::NB], n[S::NB];
  int64_t of_b[S::NB], of_c[S::NB];
  __device__ CoefficientLoader(const ScanArgs& a, const Place& p, int64_t t0)
      : b(a.Bm, p.b, a.sb_b, a.sb_t, t0, p.group * a.N),
        c(a.Cm, p.b, a.sc_b, a.sc_t, t0, p.group * a.N) {
#pragma unroll
    for (int i = 0; i < S::NB; ++i) {
      const int k = threadIdx.x + i * S::NT;
      row[i] = k / S::NP;
      n[i] = k % S::NP;
      const int state = n[i] < a.N ? n[i] : 0;
      of_b[i] = row[i] * a.sb_t + state;
      of_c[i] = row[i] * a.sc_t + state;
    }
  }
};

// A chunk's inputs on their way.
template <class T, class S>
struct Inputs {
  Pack<T, S::E> x, delta, z, dy;
  T b[S::NB], c[S::NB];
  typename S::A before[S::NS];
  // `left`: the steps from the chunk's first on
  __device__ void request(CoefficientLoader<T, S>& l, int64_t left, int steps) {
#pragma unroll
    for (int i = 0; i < S::NB; ++i) {
      const bool there = l.row[i] < left;
      b[i] = *(there ? l.b.at + l.of_b[i] : l.b.first);
      c[i] = *(there ? l.c.at + l.of_c[i] : l.c.first);
    }
    l.b.at += steps * l.b.stride;
    l.c.at += steps * l.c.stride;
  }
  __device__ void put(const CoefficientLoader<T, S>& l, int states,
                      typename Coefficients<S>::Of (&bc)[S::R][S::SG]) const {
    typedef typename S::A A;
#pragma unroll
    for (int i = 0; i < S::NB; ++i)
      if (S::R * S::NP % S::NT == 0 || l.row[i] < S::R) {
        const bool there = l.n[i] < states;
        bc[l.row[i]][l.n[i] / S::NS].b[l.n[i] % S::NS] = there ? up(b[i]) : A(0);
        bc[l.row[i]][l.n[i] / S::NS].c[l.n[i] % S::NS] = there ? up(c[i]) : A(0);
      }
  }
};

// The sums of R values over the lanes that share a channel: first over a wave's two
// halves, after which the lower one holds the chunk's first steps and the upper one the others.
__device__ inline float add_halves(float first, float second) {
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, first),
                                                  __builtin_bit_cast(uint32_t, second), false,
                                                  false);
  const uint32_t low = r[0], high = r[1];
  return __builtin_bit_cast(float, low) + __builtin_bit_cast(float, high);
}
__device__ inline double add_halves(double first, double second) {
  const bool upper = threadIdx.x & 32;
  return (upper ? second : first) + __shfl_xor(upper ? first : second, 32, 64);
}
template <class S>
__device__ inline void leave(const typename S::A (&sums)[S::R],
                             typename S::A (&part)[S::R][S::W][kSlab]) {
  constexpr int H = S::R / 2;
  const int wave = threadIdx.x / 64, c = threadIdx.x % kSlab, half = threadIdx.x / kSlab % 2 * H;
#pragma unroll
  for (int r = 0; r < H; ++r) part[half + r][wave][c] = add_halves(sums[r], sums[r + H]);
}
template <class S>
__device__ inline void gather(const typename S::A (&part)[S::R][S::W][kSlab], int row, int c,
                              typename S::A (&sums)[S::E]) {
  typedef typename S::A A;
  typedef A V __attribute__((ext_vector_type(S::E), aligned(sizeof(A) * (S::E < 4 ? S::E : 4))));
#pragma unroll
  for (int q = 0; q < S::W; ++q) {
    const V v = *reinterpret_cast<const V*>(&part[row][q][c]);
#pragma unroll
    for (int i = 0; i < S::E; ++i) sums[i] = q == 0 ? (A)v[i] : sums[i] + (A)v[i];
  }
}

// A lane's states: their channel, the first state and how many of them there are.
struct Lane {
  int c, group, first, count;
  bool channel;
};
template <class S>
__device__ inline Lane lane_of(const ScanArgs& a, const Place& p) {
  Lane l;
  l.c = threadIdx.x % kSlab;
  l.group = threadIdx.x / kSlab;
  l.first = l.group * S::NS;
  const int left = a.N - l.first;
  l.channel = l.c < p.channels;
  l.count = l.channel ? (left < 0 ? 0 : left < S::NS ? left : S::NS) : 0;
  return l;
}

// Maps of segments: [b][segment][state][channel], and the sums of s [b][segment][channel].
template <class A>
struct Maps {
  A* h;
  A* s;
  __device__ Maps(void* ws, const ScanArgs& a, const ScanGrid& g) {
    h = static_cast<A*>(ws);
    s = h + a.B * g.segments * a.N * a.D_;
  }
};

// What a sweep starts from: `from` taken through the maps of the segments first,
// first + by, ... up to but not including `end`.
template <class A, int NS>
__device__ inline void through(const Maps<A>& m, const ScanArgs& a, const ScanGrid& g, int64_t b,
                               int64_t first, int64_t end, int by, const Lane& l, int64_t d,
                               const A (&rates)[NS], A (&h)[NS]) {
  constexpr int kAhead = 4;  // maps whose loads are in flight together
  for (int64_t q = first; q != end;) {
    A s[kAhead], m_[kAhead][NS];
    int count = 0;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int64_t seg = q + k * by;
      const bool there = by > 0 ? seg < end : seg > end;
      const int64_t row = b * g.segments + (there ? seg : q);
      s[k] = l.channel ? m.s[row * a.D_ + d] : A(0);
#pragma unroll
      for (int i = 0; i < NS; ++i)
        m_[k][i] = i < l.count ? m.h[(row * a.N + l.first + i) * a.D_ + d] : A(0);
      count += there;
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (k < count)
#pragma unroll
        for (int i = 0; i < NS; ++i) h[i] = fma_(decay(s[k], rates[i]), h[i], m_[k][i]);
    q += count * by;
  }
}

// ------------------------------------------------------------------- forward
// In LDS a chunk's prepared inputs and sums have a place for each parity of the chunk's
// number: while a chunk is swept the next one is prepared and the one before is finished,
// in one stretch of independent instructions between two barriers. (4 x 4096 x 2048 bf16
// of 16 states: 301 us forward and 852 in reverse, 323 and 949 with a barrier after each of the
// three: a SIMD has one wave there, so what a wave waits for nothing hides.) The arrays are
// variables of their own, so that the compiler knows that they do not overlap.
//
// A sweep's LDS reads go a batch of steps ahead of its arithmetic, held there by
// scheduling barriers.
template <class S, bool BACK, class In, int BATCH>
struct Ahead {
  static constexpr int kBatch = BATCH;
  In in[2][kBatch];
  typename Coefficients<S>::Of bc[2][kBatch];
  static constexpr int kBatches = S::R / kBatch;
  __device__ static int step(int batch, int k) {
    const int r = batch * kBatch + k;
    return BACK ? S::R - 1 - r : r;
  }
  __device__ void read(int batch, const In (&ins)[S::R][kSlab],
                       const typename Coefficients<S>::Of (&bcs)[S::R][S::SG], const Lane& l) {
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      in[batch & 1][k] = ins[step(batch, k)][l.c];
      bc[batch & 1][k] = bcs[step(batch, k)][l.group];
    }
  }
  // f(step, inputs, coefficients) of the chunk's steps in order; of a whole chunk the first
  // batch has been read.
  template <class F, class N>
  __device__ void each(N steps, const In (&ins)[S::R][kSlab],
                       const typename Coefficients<S>::Of (&bcs)[S::R][S::SG], const Lane& l, F f) {
    if constexpr (N::kWhole) {
#pragma unroll
      for (int b = 0; b < kBatches; ++b) {
        if (b + 1 < kBatches) read(b + 1, ins, bcs, l);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int k = 0; k < kBatch; ++k) f(step(b, k), in[b & 1][k], bc[b & 1][k]);
      }
    } else {
#pragma unroll
      for (int b = 0; b < kBatches; ++b)
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
          const int r = step(b, k);
          if (steps.has(r)) f(r, ins[r][l.c], bcs[r][l.group]);
        }
    }
  }
};
template <int P>
struct Parity {
  static constexpr int p = P, q = 1 - P;  // of the chunk that is swept; of its neighbours
};
template <class X>
__device__ inline X& of_parity(X& even, X& odd, int p) {
  return p ? odd : even;
}
template <class A>
struct alignas(2 * sizeof(A)) Two {
  A s, sx;
};
template <class A>
struct alignas(4 * sizeof(A)) Four {
  A s, sx, dy, pad;
};

// MAP: the segment's map alone.
template <class T, int NS, int W, bool MAP, bool FULL>
__global__ __launch_bounds__(64 * W) void scan_fwd(ScanArgs a, ScanGrid g, void* ws) {
  typedef ScanShape<T, NS, W> S;
  typedef Acc<T> A;
  constexpr int R = S::R, E = S::E;
  __shared__ typename Coefficients<S>::Of bc0[R][S::SG], bc1[R][S::SG];
  __shared__ Two<A> in0[R][kSlab], in1[R][kSlab];
  __shared__ A part0[R][S::W][kSlab], part1[R][S::W][kSlab];
  const Place p = place_of(a, g, work_id((int64_t)gridDim.x));
  const int64_t len = row_length(a.lens, p.b, a.T);
  const int64_t span = g.seg_chunks * R, t0 = p.segment * span;
  const int64_t t1 = a.T - t0 < span ? a.T : t0 + span;
  if (MAP && len <= t1) return;  // no segment follows
  const int64_t live = len < t1 ? len : t1;
  const Loader<S, FULL> at(p);
  const Lane l = lane_of<S>(a, p);
  const int64_t d = p.d0 + l.c;
  A rates[NS], h[NS], total = A(0);
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    rates[i] = i < l.count ? rate(static_cast<const A*>(a.A)[d * a.N + l.first + i]) : A(0);
    h[i] = !MAP && a.h0 && i < l.count
               ? static_cast<const A*>(a.h0)[(p.b * a.D_ + d) * a.N + l.first + i] : A(0);
  }
  const Maps<A> maps(ws, a, g);
  if (!MAP && p.segment > 0 && t0 < live)
    through(maps, a, g, p.b, 0, p.segment, 1, l, d, rates, h);
  A skip[E], bias[E];
  at.constants(a.D, p.d0, skip);
  at.constants(a.bias, p.d0, bias);
  T* y = a.y ? static_cast<T*>(a.y) + (p.b * a.T + t0 + at.row) * a.D_ + p.d0 : nullptr;
  A* ck = static_cast<A*>(a.ck) + ((p.b * g.chunks + t0 / R) * a.N + l.first) * a.D_ + d;
  // without z its loads are of x, and their values are not used
  const bool gated = a.z;
  Walk<T> xs(a.x, p.b, a.sx_b, a.sx_t, t0, p.d0), deltas(a.delta, p.b, a.sl_b, a.sl_t, t0, p.d0);
  Walk<T> zs(gated ? a.z : a.x, p.b, gated ? a.sz_b : a.sx_b, gated ? a.sz_t : a.sx_t, t0, p.d0);
  CoefficientLoader<T, S> coefficients(a, p, t0);
  const auto go = [&](int64_t t) {  // the next request is of step t
    xs.go(t - t0 + at.row);
    deltas.go(t - t0 + at.row);
    zs.go(t - t0 + at.row);
    coefficients.b.go(t - t0);
    coefficients.c.go(t - t0);
  };
  const auto request = [&](Inputs<T, S>& in, int64_t t) {  // chunk after chunk
    const bool there = t + at.row < live;
    in.x = at.load(xs.next(there, R));
    in.delta = at.load(deltas.next(there, R));
    if (!MAP) in.z = at.load(zs.next(there, R));
    in.request(coefficients, live - t, R);
    __builtin_amdgcn_sched_barrier(0);  // loads are waited for in the order of their requests
  };
  Inputs<T, S> even, odd;
  A x[2][E], gate[2][E];
  const auto prepare = [&](const Inputs<T, S>& in, auto parity) {
    constexpr int P = decltype(parity)::p;
    auto& to = of_parity(in0, in1, P);
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const A raw = up((T)in.delta.v[i]) + bias[i], smooth = softplus(raw);
      const A s = a.softplus ? smooth : raw;
      x[P][i] = up((T)in.x.v[i]);
      if (!MAP) {
        A f, rest;
        const A z = up((T)in.z.v[i]);
        gates<T>(z, &f, &rest);
        gate[P][i] = gated ? z * f : A(1);
      }
      if (S::kLoaders == S::NT || threadIdx.x < S::kLoaders) to[at.row][at.c + i] = {s, s * x[P][i]};
    }
    in.put(coefficients, a.N, of_parity(bc0, bc1, P));
  };
  Ahead<S, false, Two<A>, R < 4 ? R : 4> ahead;
  const auto sweep = [&](auto steps, auto parity) {
    constexpr int P = decltype(parity)::p;
    A sums[R];
#pragma unroll
    for (int r = 0; r < R; ++r) sums[r] = A(0);
    ahead.each(steps, of_parity(in0, in1, P), of_parity(bc0, bc1, P), l,
               [&](int r, const Two<A>& now, const typename Coefficients<S>::Of& bc) {
#pragma unroll
                 for (int i = 0; i < NS; ++i) {
                   h[i] = fma_(decay(now.s, rates[i]), h[i], now.sx * bc.b[i]);
                   if (!MAP) sums[r] = fma_(bc.c[i], h[i], sums[r]);
                 }
                 if (MAP) total += now.s;
               });
    if (!MAP) leave<S>(sums, of_parity(part0, part1, P));
  };
  const auto finish = [&](auto parity) {
    constexpr int P = decltype(parity)::p;
    Pack<T, E> out;
    if (!MAP) {
      A v[E];
      gather<S>(of_parity(part0, part1, P), at.row, at.c, v);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const A all = a.D ? fma_(skip[i], x[P][i], v[i]) : v[i];  // (0 x is not 0 for every x)
        out.v[i] = down<T>(all * gate[P][i]);
      }
    }
    return out;
  };
  const auto checkpoint = [&] {  // of the chunk that h is the start of
    if (!MAP && a.ck) {
#pragma unroll
      for (int i = 0; i < NS; ++i)
        if (i < l.count) ck[i * a.D_] = h[i];
      ck += a.N * a.D_;
    }
  };
  const auto store = [&](const Pack<T, E>& out, bool there) {
    if (!MAP && y) {
      if (at.stores && there) at.store(y, out);
      y += R * a.D_;
    }
  };
  int64_t t = t0;
  if (t + 2 * R <= live) {
    go(t);
    request(even, t);
    request(odd, t + R);
    checkpoint();
    prepare(even, Parity<0>());
    request(even, t + 2 * R);
    __syncthreads();
    // the sweep of chunk t, whose parity is named, the end of the one before, the start of
    // the one behind: of the last pair's that is none, and what is prepared is not used
    const auto turn = [&](Inputs<T, S>& next, auto parity, bool first, int64_t at_t) {
      constexpr int P = decltype(parity)::p, Q = decltype(parity)::q;
      ahead.read(0, of_parity(in0, in1, P), of_parity(bc0, bc1, P), l);
      const Pack<T, E> out = finish(Parity<Q>());
      prepare(next, Parity<Q>());
      sweep(Steps<true, R>{R}, parity);
      if (!first) store(out, true);
      if (at_t + R < live) checkpoint();
      request(next, at_t + 3 * R);
      __syncthreads();
    };
    turn(odd, Parity<0>(), true, t);
    turn(even, Parity<1>(), false, t + R);
    for (t += 2 * R; t + 2 * R <= live; t += 2 * R) {
      turn(odd, Parity<0>(), false, t);
      turn(even, Parity<1>(), false, t + R);
    }
    store(finish(Parity<1>()), true);
  } else if (t < live) {
    checkpoint();
  }
  for (; t < live; t += R) {  // the row's last one or two
    go(t);
    request(even, t);
    prepare(even, Parity<0>());
    __syncthreads();
    const Steps<false, R> steps{(int)(live - t < R ? live - t : R)};
    sweep(steps, Parity<0>());
    __syncthreads();
    store(finish(Parity<0>()), steps.has(at.row));
    if (t + R < live) checkpoint();
  }
  if (MAP) {
#pragma unroll
    for (int i = 0; i < NS; ++i)
      if (i < l.count)
        maps.h[((p.b * g.segments + p.segment) * a.N + l.first + i) * a.D_ + d] = h[i];
    if (l.channel && l.group == 0) maps.s[(p.b * g.segments + p.segment) * a.D_ + d] = total;
    return;
  }
  // the row's last state: of the segment that it ends in
  if (a.hT && (t0 < live ? len <= t1 : p.segment == 0 && len == 0))
#pragma unroll
    for (int i = 0; i < NS; ++i)
      if (i < l.count)
        static_cast<A*>(a.hT)[(p.b * a.D_ + d) * a.N + l.first + i] = h[i];
  if (a.y && at.stores) {
    Pack<T, E> zero;
#pragma unroll
    for (int i = 0; i < E; ++i) zero.v[i] = T(0);
    for (int64_t t = (live > t0 ? live : t0) + at.row; t < t1; t += R)
      at.store(static_cast<T*>(a.y) + (p.b * a.T + t) * a.D_ + p.d0, zero);
  }
}

// ------------------------------------------------------------------- reverse
// Sums over the 32 channels of each half wave. A first exchange between rows of 16 lanes
// takes two registers into one, whose upper row then is the second's; the others go on from
// there, until of each 16 registers every lane has one, that of its own number in the row.
template <int BIT>
__device__ inline float folded(float u, float v, bool upper) {
  // lanes without the bit hold u's sum over the pair, those with it v's
  if constexpr (BIT == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, u),
                                                    __builtin_bit_cast(uint32_t, v), false, false);
    const uint32_t even = r[0], odd = r[1];
    return __builtin_bit_cast(float, even) + __builtin_bit_cast(float, odd);
  } else {
    const float mine = upper ? v : u, other = upper ? u : v;
    if constexpr (BIT == 8) return mine + permuted<0x140>(other);
    if constexpr (BIT == 4) return mine + permuted<0x141>(other);
    if constexpr (BIT == 2) return mine + permuted<0x4e>(other);
    return mine + permuted<0xb1>(other);
  }
}
template <int BIT>
__device__ inline double folded(double u, double v, bool upper) {
  return (upper ? v : u) + __shfl_xor(upper ? u : v, BIT, 64);
}
template <int BIT, int V, class A>
__device__ inline void fold(A (&x)[V]) {
  const bool upper = threadIdx.x & BIT;
#pragma unroll
  for (int base = 0; base < V; base += 2 * BIT)
#pragma unroll
    for (int k = 0; k < BIT; ++k) x[base + k] = folded<BIT>(x[base + k], x[base + k + BIT], upper);
}
template <int J, class A>
__device__ inline void sum_channels(A (&x)[J]) {
  static_assert(J == 8 || J % 16 == 0, "");
  if constexpr (J >= 16) {
    fold<8>(x);
  } else {  // the lanes that differ in this bit add up
#pragma unroll
    for (int k = 0; k < J; ++k) x[k] += __shfl_xor(x[k], 8, 64);
  }
  fold<4>(x);
  fold<2>(x);
  fold<1>(x);
}

// The partial sums that leave a workgroup.
template <class A>
struct Sums {
  A* bc;  // [slab][b][chunk][lanes of a channel][B or C][a lane's steps and states]
  A* a;   // [row of workgroups][state][channel]
  A* d;   // [row of workgroups][D or bias][channel]
  __device__ __host__ Sums(void* ws, int64_t B, int64_t D, int64_t N, const ScanGrid& g) {
    const int64_t padded = 2 * g.waves * g.states;
    bc = static_cast<A*>(ws);
    a = bc + g.slabs * B * g.chunks * g.chunk * padded * 2;
    d = a + g.rows * g.segments * N * D;
  }
};

// MAP: the segment's map of G alone.
template <class T, int NS, int W, bool MAP, bool FULL>
__global__ __launch_bounds__(64 * W) void scan_rev(ScanArgs a, ScanGrid g, void* ws, void* sums_ws) {
  typedef ScanShape<T, NS, W> S;
  typedef Acc<T> A;
  constexpr int R = S::R, E = S::E, V = R * NS, H = R / 2, J = H * NS;
  constexpr int kAhead = 2, kBack = 2;  // batches of the two sweeps
  __shared__ typename Coefficients<S>::Of bc0[R][S::SG], bc1[R][S::SG];
  __shared__ Four<A> in0[R][kSlab], in1[R][kSlab];
  // of u, of sum A q, of y before skip and gate
  __shared__ A part0[MAP ? 1 : 3][R][S::W][kSlab], part1[MAP ? 1 : 3][R][S::W][kSlab];
  Place p = place_of(a, g, work_id((int64_t)gridDim.x));
  const int64_t row = p.b;  // of workgroups: in the reverse sweep they take several batch rows
  const int64_t span = g.seg_chunks * R, t0 = p.segment * span;
  const int64_t t1 = a.T - t0 < span ? a.T : t0 + span;
  const Loader<S, FULL> at(p);
  const Lane l = lane_of<S>(a, p);
  const int64_t d = p.d0 + l.c;
  A rates[NS];
#pragma unroll
  for (int i = 0; i < NS; ++i)
    rates[i] = i < l.count ? rate(static_cast<const A*>(a.A)[d * a.N + l.first + i]) : A(0);
  A skip[E], bias[E];
  at.constants(a.D, p.d0, skip);
  at.constants(a.bias, p.d0, bias);
  // Sums over steps, a few chunks' at a time: one sum over thousands of steps is 1.5 times as
  // far off (dA of 4 x 4096 x 2048 bf16: 2.7e-6 of it, two levels 1.9e-6; 852 us, not 833).
  A dA[NS], dD[E], dbias[E], all_dA[NS], all_dD[E], all_dbias[E];
#pragma unroll
  for (int i = 0; i < NS; ++i) dA[i] = all_dA[i] = A(0);
#pragma unroll
  for (int i = 0; i < E; ++i) dD[i] = dbias[i] = all_dD[i] = all_dbias[i] = A(0);
  const auto keep_sums = [&] {
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      all_dA[i] += dA[i];
      dA[i] = A(0);
    }
#pragma unroll
    for (int i = 0; i < E; ++i) {
      all_dD[i] += dD[i];
      all_dbias[i] += dbias[i];
      dD[i] = dbias[i] = A(0);
    }
  };
  const Maps<A> maps(ws, a, g);
  const Sums<A> sums(sums_ws, a.B, a.D_, a.N, g);
  for (p.b = row; p.b < a.B; p.b += MAP ? a.B : g.rows) {
    const int64_t len = row_length(a.lens, p.b, a.T), live = len < t1 ? len : t1;
    const int64_t active = len > 0 ? (len - 1) / span + 1 : 1;  // segments of this row
    if (MAP && (p.segment == 0 || p.segment >= active)) return;
    A G[NS], total = A(0);
#pragma unroll
    for (int i = 0; i < NS; ++i)
      G[i] = !MAP && a.dhT && i < l.count
                 ? static_cast<const A*>(a.dhT)[(p.b * a.D_ + d) * a.N + l.first + i] : A(0);
    if (!MAP && p.segment + 1 < active)
      through(maps, a, g, p.b, active - 1, p.segment, -1, l, d, rates, G);
    const int64_t last = live > t0 ? t0 + (live - t0 - 1) / R * R : t0 - R;
    // without z its loads are of dy, and their values are not used
    const bool gated = a.z;
    Walk<T> xs(a.x, p.b, a.sx_b, a.sx_t, t0, p.d0), deltas(a.delta, p.b, a.sl_b, a.sl_t, t0, p.d0),
        zs(gated ? a.z : a.dy, p.b, gated ? a.sz_b : a.sd_b, gated ? a.sz_t : a.sd_t, t0, p.d0),
        dys(a.dy, p.b, a.sd_b, a.sd_t, t0, p.d0);
    CoefficientLoader<T, S> coefficients(a, p, t0);
    const A* const ck0 =
        static_cast<const A*>(a.ck) + (p.b * g.chunks + t0 / R) * a.N * a.D_;
    const A* ck = ck0;
    // a lane's states in a checkpoint; lanes without them read the first
    const int64_t of_ck = l.count > 0 ? l.first * a.D_ + d : 0;
    const auto go = [&](int64_t t) {  // the next request is of step t
      xs.go(t - t0 + at.row);
      deltas.go(t - t0 + at.row);
      zs.go(t - t0 + at.row);
      dys.go(t - t0 + at.row);
      coefficients.b.go(t - t0);
      coefficients.c.go(t - t0);
      ck = ck0 + (t - t0) / R * a.N * a.D_;
    };
    const auto request = [&](Inputs<T, S>& in, int64_t t) {
      const bool there = t >= t0 && t + at.row < live;
      in.delta = at.load(deltas.next(there, -R));
      in.dy = at.load(dys.next(there, -R));
      in.z = at.load(zs.next(there, -R));
      if (!MAP) {
        in.x = at.load(xs.next(there, -R));
        const A* const from = t >= t0 ? ck : ck0;
#pragma unroll
        for (int i = 0; i < NS; ++i) in.before[i] = from[of_ck + (i < l.count ? i * a.D_ : 0)];
        ck -= a.N * a.D_;
      }
      in.request(coefficients, t >= t0 ? live - t : 0, -R);
      __builtin_amdgcn_sched_barrier(0);  // loads are waited for in the order of their requests
    };
    Inputs<T, S> even, odd;
    // of a chunk, from its preparation to its end; and its first states
    A s_[2][E], x_[2][E], dy_[2][E], gate[2][E], of_gate[2][E], slope[2][E], start_[2][NS];
    const auto prepare = [&](const Inputs<T, S>& in, auto parity) {
      constexpr int P = decltype(parity)::p;
      auto& to = of_parity(in0, in1, P);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const A raw = up((T)in.delta.v[i]) + bias[i], smooth = softplus(raw);
        const A s = a.softplus ? smooth : raw, x = MAP ? A(0) : up((T)in.x.v[i]);
        const A dy = up((T)in.dy.v[i]), z = up((T)in.z.v[i]);
        A f, rest, g1, g2;
        gates<T>(z, &f, &rest);
        const A open = gated ? z * f : A(1);
        if (!MAP) {
          gates<T>(raw, &g1, &g2);
          slope[P][i] = a.softplus ? g1 : A(1);
          of_gate[P][i] = f * fma_(z, rest, A(1));
          s_[P][i] = s;
          x_[P][i] = x;
          dy_[P][i] = dy;
          gate[P][i] = open;
        }
        if (S::kLoaders == S::NT || threadIdx.x < S::kLoaders) {
          // channels that are not there add nothing to the sums over channels
          const bool there = FULL || at.c + i <= at.last;
          to[at.row][at.c + i] = {there ? s : A(0), there ? s * x : A(0), there ? dy * open : A(0),
                                  A(0)};
        }
      }
      in.put(coefficients, a.N, of_parity(bc0, bc1, P));
      if (!MAP)
#pragma unroll
        for (int i = 0; i < NS; ++i) start_[P][i] = i < l.count ? in.before[i] : A(0);
    };
    A ofB[J], ofC[J];  // sums over the channels
    Ahead<S, false, Four<A>, kAhead> ahead;
    Ahead<S, true, Four<A>, kBack> back;
    const auto sweep = [&](auto steps, auto parity) {
      constexpr int P = decltype(parity)::p;
      auto& in = of_parity(in0, in1, P);
      auto& bcs = of_parity(bc0, bc1, P);
      typedef typename Coefficients<S>::Of Of;
      if constexpr (MAP) {
        back.each(steps, in, bcs, l, [&](int, const Four<A>& now, const Of& bc) {
          total += now.s;
#pragma unroll
          for (int i = 0; i < NS; ++i)
            G[i] = decay(now.s, rates[i]) * fma_(bc.c[i], now.dy, G[i]);
        });
      } else {
        auto& part = of_parity(part0, part1, P);
        // What a step leaves for sums over lanes is taken together with that of the step
        // half a chunk away as soon as both are there: it would take 6 R registers otherwise.
        A e[R][NS], old[R][NS], yp[R], h[NS], otherB[J], otherC[J], other_u[H], other_aq[H];
        const int wave = threadIdx.x / 64, half = threadIdx.x / kSlab % 2 * H;
#pragma unroll
        for (int i = 0; i < NS; ++i) h[i] = start_[P][i];
        if (!steps.kWhole) {  // steps that are not there
#pragma unroll
          for (int r = 0; r < R; ++r) yp[r] = A(0);
#pragma unroll
          for (int r = 0; r < H; ++r) other_u[r] = other_aq[r] = A(0);
#pragma unroll
          for (int k = 0; k < J; ++k) otherB[k] = otherC[k] = ofB[k] = ofC[k] = A(0);
        }
        ahead.each(steps, in, bcs, l, [&](int r, const Four<A>& now, const Of& bc) {
          yp[r] = A(0);
#pragma unroll
          for (int i = 0; i < NS; ++i) {
            e[r][i] = decay(now.s, rates[i]);
            old[r][i] = h[i];
            h[i] = fma_(e[r][i], h[i], now.sx * bc.b[i]);
            yp[r] = fma_(bc.c[i], h[i], yp[r]);
          }
          if (steps.kWhole && r >= H) part[2][half + r - H][wave][l.c] = add_halves(yp[r - H], yp[r]);
        });
        if (!steps.kWhole) leave<S>(yp, part[2]);
        if (steps.kWhole) back.read(0, in, bcs, l);
        back.each(steps, in, bcs, l, [&](int r, const Four<A>& now, const Of& bc) {
          A u = A(0), aq = A(0);
#pragma unroll
          for (int i = 0; i < NS; ++i) {
            G[i] = fma_(bc.c[i], now.dy, G[i]);
            const A c = now.dy * h[i], b = G[i] * now.sx;
            u = fma_(G[i], bc.b[i], u);
            G[i] *= e[r][i];
            h[i] = old[r][i];
            const A q = G[i] * h[i];
            dA[i] = fma_(now.s, q, dA[i]);
            aq = fma_(rates[i], q, aq);
            if (r >= H) {
              otherB[(r - H) * NS + i] = b;
              otherC[(r - H) * NS + i] = c;
            } else {
              ofB[r * NS + i] = folded<16>(b, otherB[r * NS + i], threadIdx.x & 16);
              ofC[r * NS + i] = folded<16>(c, otherC[r * NS + i], threadIdx.x & 16);
            }
          }
          if (r >= H) {
            other_u[r - H] = u;
            other_aq[r - H] = aq;
          } else {
            part[0][half + r][wave][l.c] = add_halves(u, other_u[r]);
            part[1][half + r][wave][l.c] = add_halves(aq, other_aq[r]);
          }
        });
        sum_channels(ofB);
        sum_channels(ofC);
      }
    };
    struct Out {
      Pack<T, E> dx, ddelta, dz;
    };
    const auto finish = [&](auto parity, bool there) {
      constexpr int P = decltype(parity)::p;
      Out o;
      if constexpr (!MAP) {
        auto& part = of_parity(part0, part1, P);
        A u[E], aq[E], yp[E];
        gather<S>(part[0], at.row, at.c, u);
        gather<S>(part[1], at.row, at.c, aq);
        gather<S>(part[2], at.row, at.c, yp);
#pragma unroll
        for (int i = 0; i < E; ++i) {
          const A dy = dy_[P][i], through_gate = dy * gate[P][i];
          const A of_raw = fma_(u[i], x_[P][i], of_rate(aq[i])) * slope[P][i];
          o.dx.v[i] = down<T>(fma_(s_[P][i], u[i], skip[i] * through_gate));
          o.ddelta.v[i] = down<T>(of_raw);
          const A all = a.D ? fma_(skip[i], x_[P][i], yp[i]) : yp[i];
          o.dz.v[i] = down<T>(dy * all * of_gate[P][i]);
          dD[i] = there ? fma_(through_gate, x_[P][i], dD[i]) : dD[i];
          dbias[i] = there ? dbias[i] + of_raw : dbias[i];
        }
      }
      return o;
    };
    const auto store = [&](const Out& o, int64_t t, bool there) {
      if (!MAP && there && at.stores) {
        const int64_t to = (p.b * a.T + t + at.row) * a.D_ + p.d0;
        at.store(static_cast<T*>(a.out.dx) + to, o.dx);
        at.store(static_cast<T*>(a.out.ddelta) + to, o.ddelta);
        if (gated) at.store(static_cast<T*>(a.out.dz) + to, o.dz);
      }
    };
    const auto store_bc = [&](int64_t t) {
      if constexpr (!MAP) {
        constexpr int L = J < 16 ? J : 16;  // values of a register in half of a slab's lanes
        A* const to = sums.bc +
                      ((((p.slab * a.B + p.b) * g.chunks + t / R) * S::SG + l.group) * 2) * V;
        const int lane = l.c / 16 * L + l.c % 16;
#pragma unroll
        for (int k = 0; k < J; k += 16)
          if (L == 16 || l.c % 16 < L) {
            to[2 * k + lane] = ofB[k];
            to[V + 2 * k + lane] = ofC[k];
          }
      }
    };
    int64_t t = last;
    // the row's last one or two, until pairs of whole chunks are left
    for (; t >= t0 && ((t - t0) / R % 2 == 0 || live - t < R); t -= R) {
      go(t);
      request(even, t);
      prepare(even, Parity<0>());
      __syncthreads();
      const Steps<false, R> steps{(int)(live - t < R ? live - t : R)};
      sweep(steps, Parity<0>());
      store_bc(t);
      __syncthreads();
      const bool there = steps.has(at.row);
      store(finish(Parity<0>(), there), t, there);
    }
    if (t > t0) {
      go(t);
      request(even, t);
      request(odd, t - R);
      prepare(even, Parity<0>());
      request(even, t - 2 * R);
      __syncthreads();
      const auto turn = [&](Inputs<T, S>& next, auto parity, bool first, int64_t now) {
        constexpr int P = decltype(parity)::p, Q = decltype(parity)::q;
        if (MAP) back.read(0, of_parity(in0, in1, P), of_parity(bc0, bc1, P), l);
        else ahead.read(0, of_parity(in0, in1, P), of_parity(bc0, bc1, P), l);
        const Out o = finish(Parity<Q>(), !first);
        prepare(next, Parity<Q>());
        sweep(Steps<true, R>{R}, parity);
        store_bc(now);
        if (!first) store(o, now + R, true);
        request(next, now - 3 * R);
        __syncthreads();
      };
      turn(odd, Parity<0>(), true, t);
      turn(even, Parity<1>(), false, t - R);
      for (t -= 2 * R; t > t0; t -= 2 * R) {
        turn(odd, Parity<0>(), false, t);
        turn(even, Parity<1>(), false, t - R);
        if (!MAP && (t - t0) / R % 8 == 1) keep_sums();
      }
      store(finish(Parity<1>(), true), t0, true);
      __syncthreads();  // the next row's chunks take its place
    }
    if (MAP) {
#pragma unroll
      for (int i = 0; i < NS; ++i)
        if (i < l.count)
          maps.h[((p.b * g.segments + p.segment) * a.N + l.first + i) * a.D_ + d] = G[i];
      if (l.channel && l.group == 0) maps.s[(p.b * g.segments + p.segment) * a.D_ + d] = total;
      return;
    }
    keep_sums();
    if (p.segment == 0 && a.out.dh0)
#pragma unroll
      for (int i = 0; i < NS; ++i)
        if (i < l.count)
          static_cast<A*>(a.out.dh0)[(p.b * a.D_ + d) * a.N + l.first + i] = G[i];
    if (at.stores) {
      Pack<T, E> zero;
#pragma unroll
      for (int i = 0; i < E; ++i) zero.v[i] = T(0);
      for (int64_t t = (live > t0 ? live : t0) + at.row; t < t1; t += R) {
        const int64_t to = (p.b * a.T + t) * a.D_ + p.d0;
        at.store(static_cast<T*>(a.out.dx) + to, zero);
        at.store(static_cast<T*>(a.out.ddelta) + to, zero);
        if (a.z) at.store(static_cast<T*>(a.out.dz) + to, zero);
      }
    }
  }
  const int64_t part = row * g.segments + p.segment;
#pragma unroll
  for (int i = 0; i < NS; ++i)
    if (i < l.count) sums.a[(part * a.N + l.first + i) * a.D_ + d] = all_dA[i];
  // the loaders' sums of a channel, step after step of the chunk
  A(*const rows_of)[2][kSlab] = reinterpret_cast<A(*)[2][kSlab]>(&part0[0][0][0][0]);
  __syncthreads();
  if (threadIdx.x < S::kLoaders)
#pragma unroll
    for (int i = 0; i < E; ++i) {
      rows_of[at.row][0][at.c + i] = all_dD[i];
      rows_of[at.row][1][at.c + i] = all_dbias[i];
    }
  __syncthreads();
  if (threadIdx.x < 2 * kSlab && (int)threadIdx.x % kSlab < p.channels) {
    const int which = threadIdx.x / kSlab, c = threadIdx.x % kSlab;
    double v = 0;
    for (int r = 0; r < R; ++r) v += rows_of[r][which][c];
    sums.d[(part * 2 + which) * a.D_ + p.d0 + c] = (A)v;
  }
}

constexpr int kSumThreads = 256;

// dB and dC: over the slabs of a group. A work-item: one value of a chunk's, in
// the order in which the workgroups wrote them.
template <class T>
__global__ __launch_bounds__(kSumThreads) void scan_sum_bc(ScanArgs a, ScanGrid g, void* ws) {
  typedef Acc<T> A;
  const Sums<A> sums(ws, a.B, a.D_, a.N, g);
  const int64_t V = (int64_t)g.chunk * g.states, lanes = 2 * g.waves;
  const int64_t of_row = g.chunks * lanes * 2 * V, of_slab = a.B * of_row;
  const int64_t id = (int64_t)blockIdx.x * kSumThreads + threadIdx.x;
  if (id >= of_slab * a.G) return;
  const int64_t group = id / of_slab, at = id % of_slab;
  const int64_t b = at / of_row, k = at % V;
  const int64_t rest = at / V, which = rest % 2, lane = rest / 2 % lanes;
  const int64_t chunk = rest / 2 / lanes % g.chunks;
  // registers of 16 (or fewer) steps and states in the lower row of lanes, and those of half
  // a chunk later in the upper one
  const int64_t of_half = V / 2, L = of_half < 16 ? of_half : 16;
  const int64_t upper = k % (2 * L) / L, j = k / (2 * L) * L + k % L;
  const int64_t t = chunk * g.chunk + upper * (g.chunk / 2) + j / g.states;
  const int64_t n = lane * g.states + j % g.states;
  if (t >= a.T || n >= a.N) return;
  A v = A(0);
  if (t < row_length(a.lens, b, a.T)) {
    const A* from = sums.bc + group * g.group_slabs * of_slab + at;
#pragma unroll 8
    for (int64_t s = 0; s < g.group_slabs; ++s) v += from[s * of_slab];
  }
  static_cast<T*>(which ? a.out.dC : a.out.dB)[((b * a.T + t) * a.G + group) * a.N + n] =
      down<T>(v);
}

// dA, dD and dbias: over the rows of workgroups and the segments, in 64 bits: a part is a sum over
// steps already, and what is 2^-24 of another one is not to be lost beside it.
template <class T>
__global__ __launch_bounds__(kSumThreads) void scan_sum_a(ScanArgs a, ScanGrid g, void* ws) {
  typedef Acc<T> A;
  const Sums<A> sums(ws, a.B, a.D_, a.N, g);
  const int64_t id = (int64_t)blockIdx.x * kSumThreads + threadIdx.x, parts = g.rows * g.segments;
  if (id >= (a.N + 2) * a.D_) return;
  const int64_t n = id / a.D_, d = id % a.D_;
  const A* from = n < a.N ? sums.a + n * a.D_ + d : sums.d + (n - a.N) * a.D_ + d;
  const int64_t by = (n < a.N ? a.N : 2) * a.D_;
  double sum = 0;
#pragma unroll 8
  for (int64_t k = 0; k < parts; ++k) sum += from[k * by];
  const A v = (A)sum;
  if (n < a.N) static_cast<A*>(a.out.dA)[d * a.N + n] = v;
  else if (n == a.N && a.out.dD) static_cast<A*>(a.out.dD)[d] = v;
  else if (n > a.N && a.out.ddelta_bias) static_cast<A*>(a.out.ddelta_bias)[d] = v;
}

// ------------------------------------------------------------------ one step
// A lane: four neighbouring states of a channel; LANES lanes, a power of two, share a
// channel. A workgroup's row of the batch is its second index.
template <int LANES, class A>
__device__ inline A sum_lanes(A v) {
  if constexpr (sizeof(A) == 4) {
    if (LANES > 1) v += permuted<0xb1>(v);
    if (LANES > 2) v += permuted<0x4e>(v);
    if (LANES > 4) v += permuted<0x141>(v);
    if (LANES > 8) v += permuted<0x140>(v);
    if (LANES > 16) v += __shfl_xor(v, 16, 64);
  } else {
#pragma unroll
    for (int by = 1; by < LANES; by <<= 1) v += __shfl_xor(v, by, 64);
  }
  return v;
}
// Rows of the batch that a lane takes, whose loads are in flight together.
constexpr int kStepRows = 2;
template <class T, int LANES>
__global__ __launch_bounds__(256) void scan_one(ScanStep q, int64_t row) {
  typedef Acc<T> A;
  const ScanArgs& a = q.a;
  const int first = (int)(threadIdx.x % LANES) * 4;
  const int64_t d = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  const bool channel = d < a.D_;
  const int left = channel ? a.N - first : 0, n = left < 0 ? 0 : left < 4 ? left : 4;
  const int64_t c = channel ? d : 0;  // (loads of lanes that have no channel are of the first)
  const int64_t group = (uint32_t)c / (uint32_t)(a.D_ / a.G);
  const Pack<A, 4> r = load_pack<A, 4>(static_cast<const A*>(a.A) + c * a.N + first, n);
  const A bias = a.bias ? static_cast<const A*>(a.bias)[c] : A(0);
  const A skip = a.D ? static_cast<const A*>(a.D)[c] : A(0);
  Pack<A, 4> h[kStepRows];
  Pack<T, 4> B[kStepRows], C[kStepRows];
  A x[kStepRows], s[kStepRows], z[kStepRows];
  A* state[kStepRows];
  bool on[kStepRows];
  const int64_t b0 = row + (int64_t)blockIdx.y * kStepRows;
#pragma unroll
  for (int k = 0; k < kStepRows; ++k) {
    const int64_t b = b0 + k < a.B ? b0 + k : b0;
    const int64_t slot = q.slots ? q.slots[b] : b;
    on[k] = b0 + k < a.B && slot >= 0 && slot < q.nstates;
    state[k] = static_cast<A*>(q.state) + ((on[k] ? slot : 0) * a.D_ + c) * a.N + first;
    const int m = on[k] ? n : 0;
    h[k] = load_pack<A, 4>(state[k], m);
    B[k] = load_pack<T, 4>(static_cast<const T*>(a.Bm) + b * a.sb_b + group * a.N + first, m);
    C[k] = load_pack<T, 4>(static_cast<const T*>(a.Cm) + b * a.sc_b + group * a.N + first, m);
    x[k] = up(static_cast<const T*>(a.x)[b * a.sx_b + c]);
    s[k] = up(static_cast<const T*>(a.delta)[b * a.sl_b + c]) + bias;
    z[k] = a.z ? up(static_cast<const T*>(a.z)[b * a.sz_b + c]) : A(0);
  }
#pragma unroll
  for (int k = 0; k < kStepRows; ++k) {
    if (a.softplus) s[k] = softplus(s[k]);
    A sum = A(0);
    if (on[k]) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i < n) {
          h[k].v[i] = fma_(decay(s[k], rate((A)r.v[i])), (A)h[k].v[i], s[k] * x[k] * up((T)B[k].v[i]));
          sum = fma_(up((T)C[k].v[i]), (A)h[k].v[i], sum);
        }
      store_pack<A, 4>(state[k], h[k], n);
    }
    sum = sum_lanes<LANES>(sum);
    if (first > 0 || !channel || b0 + k >= a.B || !a.y) continue;
    A v = A(0);
    if (on[k]) {
      v = a.D ? fma_(skip, x[k], sum) : sum;
      if (a.z) {
        A f, rest;
        gates<T>(z[k], &f, &rest);
        v *= z[k] * f;
      }
    }
    static_cast<T*>(a.y)[(b0 + k) * a.D_ + d] = down<T>(v);
  }
}

// ------------------------------------------------------------------ launches
// f(shape) for the shape that the grid names.
template <class T, class F>
hipError_t by_shape(const ScanGrid& g, F f) {
  if (g.states == 2 && g.waves == 2) return f(ScanShape<T, 2, 2>());
  if (g.states == 2 && g.waves == 4) return f(ScanShape<T, 2, 4>());
  if (g.states == 4 && g.waves == 4) return f(ScanShape<T, 4, 4>());
  if constexpr (sizeof(T) == 8) {
    if (g.states == 4 && g.waves == 8) return f(ScanShape<T, 4, 8>());
  } else {
    if (g.states == 1 && g.waves == 2) return f(ScanShape<T, 1, 2>());
    if (g.states == 8 && g.waves == 4) return f(ScanShape<T, 8, 4>());
    if (g.states == 16 && g.waves == 4) return f(ScanShape<T, 16, 4>());
  }
  return hipErrorInvalidValue;
}

// Every slab has all of its channels, and rows of B and C exist.
inline bool full_slabs(const ScanArgs& a) { return a.D_ / a.G % kSlab == 0; }

template <class T>
hipError_t forward_of(const ScanArgs& a, const ScanGrid& g, void* ws, hipStream_t st) {
  return by_shape<T>(g, [&](auto shape) {
    typedef decltype(shape) S;
    constexpr int N = S::NS, W = S::W;
    const dim3 groups((unsigned)(g.slabs * g.segments * a.B));
    const bool full = full_slabs(a);
    if (g.segments > 1) {
      const hipError_t e = start(full ? scan_fwd<T, N, W, true, true> : scan_fwd<T, N, W, true, false>,
                                 groups, S::NT, st, a, g, ws);
      if (e != hipSuccess) return e;
    }
    return start(full ? scan_fwd<T, N, W, false, true> : scan_fwd<T, N, W, false, false>, groups,
                 S::NT, st, a, g, ws);
  });
}

template <class T>
hipError_t vjp_of(const ScanArgs& a, const ScanGrid& g, void* ws, hipStream_t st) {
  void* const sums = static_cast<char*>(ws) + g.map_bytes;
  return by_shape<T>(g, [&](auto shape) {
    typedef decltype(shape) S;
    constexpr int N = S::NS, W = S::W;
    const bool full = full_slabs(a);
    hipError_t e = hipSuccess;
    if (g.segments > 1) {
      e = start(full ? scan_rev<T, N, W, true, true> : scan_rev<T, N, W, true, false>,
                dim3((unsigned)(g.slabs * g.segments * a.B)), S::NT, st, a, g, ws, sums);
      if (e != hipSuccess) return e;
    }
    if (a.D_ > 0) {
      e = start(full ? scan_rev<T, N, W, false, true> : scan_rev<T, N, W, false, false>,
                dim3((unsigned)(g.slabs * g.segments * g.rows)), S::NT, st, a, g, ws, sums);
      if (e != hipSuccess) return e;
    }
    const int64_t bc = a.B * g.chunks * g.chunk * 2 * S::NP * a.G;
    if (bc > 0) {
      e = start(scan_sum_bc<T>, dim3((unsigned)((bc + kSumThreads - 1) / kSumThreads)), kSumThreads,
                st, a, g, sums);
      if (e != hipSuccess) return e;
    }
    const int64_t rest = (a.N + 2) * a.D_;
    if (rest == 0) return e;
    return start(scan_sum_a<T>, dim3((unsigned)((rest + kSumThreads - 1) / kSumThreads)),
                 kSumThreads, st, a, g, sums);
  });
}

template <class T, int LANES>
hipError_t step_with(const ScanStep& q, hipStream_t st) {
  constexpr int64_t kMostRows = 65535 * kStepRows;  // of a launch's second axis
  const int64_t of_group = 256 / LANES, groups = (q.a.D_ + of_group - 1) / of_group;
  for (int64_t b = 0; b < q.a.B; b += kMostRows) {
    const int64_t rows = q.a.B - b < kMostRows ? q.a.B - b : kMostRows;
    const dim3 grid((unsigned)groups, (unsigned)((rows + kStepRows - 1) / kStepRows));
    const hipError_t e = start(scan_one<T, LANES>, grid, 256, st, q, b);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <class T>
hipError_t step_of(const ScanStep& q, hipStream_t st) {
  const int N = q.a.N;
  if (N <= 4) return step_with<T, 1>(q, st);
  if (N <= 8) return step_with<T, 2>(q, st);
  if (N <= 16) return step_with<T, 4>(q, st);
  if (N <= 32) return step_with<T, 8>(q, st);
  if (N <= 64) return step_with<T, 16>(q, st);
  return step_with<T, 32>(q, st);
}

}  // namespace
}  // namespace adst
