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
  static constexpr int R = sizeof(T) == 8 || NS == 8 ? 8 : 16;  // steps of a chunk
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

// The chunk's steps of one input, as a thread has them: E channels of step `row`.
template <class S>
struct Loader {
  int row, c, n;  // n: channels that exist
  __device__ Loader(const Place& p) {
    row = threadIdx.x / S::kRowThreads;
    c = threadIdx.x % S::kRowThreads * S::E;
    const int left = p.channels - c;
    n = threadIdx.x < S::kLoaders && left > 0 ? (left < S::E ? left : S::E) : 0;
  }
  template <class T>
  __device__ Pack<T, S::E> load(const void* from, int64_t at, bool there) const {
    return load_pack<T, S::E>(static_cast<const T*>(from) + at, there ? n : 0);
  }
  template <class A>
  __device__ void constants(const void* from, int64_t d0, A (&to)[S::E]) const {
#pragma unroll
    for (int i = 0; i < S::E; ++i)
      to[i] = from && i < n ? static_cast<const A*>(from)[d0 + c + i] : A(0);
  }
};

// B and C of a chunk: [step][B or C][state] in LDS, zero where there is none.
template <class T, class S>
struct Coefficients {
  typedef Acc<T> A;
  T v[2][S::NB];
  __device__ void load(const ScanArgs& a, const Place& p, int64_t t0, int rows, bool with_b) {
    const T* const at[2] = {
        static_cast<const T*>(a.Bm) + p.b * a.sb_b + t0 * a.sb_t + p.group * a.N,
        static_cast<const T*>(a.Cm) + p.b * a.sc_b + t0 * a.sc_t + p.group * a.N};
#pragma unroll
    for (int i = 0; i < S::NB; ++i) {
      const int k = threadIdx.x + i * S::NT, r = k / S::NP, n = k % S::NP;
      const bool there = r < rows && n < a.N;
      v[0][i] = there && with_b ? at[0][r * a.sb_t + n] : T(0);
      v[1][i] = there ? at[1][r * a.sc_t + n] : T(0);
    }
  }
  __device__ void put(A (&bc)[S::R][2][S::NP]) const {
#pragma unroll
    for (int i = 0; i < S::NB; ++i) {
      const int k = threadIdx.x + i * S::NT, r = k / S::NP, n = k % S::NP;
      if (r < S::R) {
        bc[r][0][n] = up(v[0][i]);
        bc[r][1][n] = up(v[1][i]);
      }
    }
  }
};

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
template <class S>
struct ForwardLds {
  typedef typename S::A A;
  struct Two {
    A s, sx;
  };
  Two in[S::R][kSlab];
  A bc[S::R][2][S::NP];
  A part[S::R][S::SG][kSlab];
};

// MAP: the segment's map alone.
template <class T, int NS, int W, bool MAP>
__global__ __launch_bounds__(64 * W) void scan_fwd(ScanArgs a, ScanGrid g, void* ws) {
  typedef ScanShape<T, NS, W> S;
  typedef Acc<T> A;
  constexpr int R = S::R, E = S::E;
  __shared__ ForwardLds<S> lds;
  const Place p = place_of(a, g, work_id((int64_t)gridDim.x));
  const int64_t len = row_length(a.lens, p.b, a.T);
  const int64_t span = g.seg_chunks * R, t0 = p.segment * span;
  const int64_t t1 = a.T - t0 < span ? a.T : t0 + span;
  if (MAP && len <= t1) return;  // no segment follows
  const int64_t live = len < t1 ? len : t1;
  const Loader<S> at(p);
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
  const int64_t from = p.d0 + at.c;
  T* const y = static_cast<T*>(a.y);
  Pack<T, E> x, delta, z;
  Coefficients<T, S> bc;
  const auto request = [&](int64_t t) {  // a chunk's inputs
    const bool there = t + at.row < live;
    x = at.template load<T>(a.x, p.b * a.sx_b + (t + at.row) * a.sx_t + from, there);
    delta = at.template load<T>(a.delta, p.b * a.sl_b + (t + at.row) * a.sl_t + from, there);
    if (!MAP && a.z)
      z = at.template load<T>(a.z, p.b * a.sz_b + (t + at.row) * a.sz_t + from, there);
    bc.load(a, p, t, (int)(live - t < R ? live - t : R), true);
  };
  if (t0 < live) request(t0);
  for (int64_t t = t0; t < live; t += R) {
    const int rows = (int)(live - t < R ? live - t : R);
    if (threadIdx.x < S::kLoaders) {
#pragma unroll
      for (int i = 0; i < E; ++i) {
        A s = up((T)delta.v[i]) + bias[i];
        if (a.softplus) s = softplus(s);
        lds.in[at.row][at.c + i] = {s, s * up((T)x.v[i])};
      }
    }
    bc.put(lds.bc);
    __syncthreads();
    const Pack<T, E> old_x = x, old_z = z;
    if (t + R < live) request(t + R);
    if (!MAP && a.ck) {
      A* const ck = static_cast<A*>(a.ck) + (p.b * g.chunks + t / R) * a.N * a.D_;
#pragma unroll
      for (int i = 0; i < NS; ++i)
        if (i < l.count) ck[(l.first + i) * a.D_ + d] = h[i];
    }
    const auto sweep = [&](auto steps) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if (!steps.has(r)) break;
        const auto in = lds.in[r][l.c];
        A sum = A(0);
#pragma unroll
        for (int i = 0; i < NS; ++i) {
          h[i] = fma_(decay(in.s, rates[i]), h[i], in.sx * lds.bc[r][0][l.first + i]);
          if (!MAP) sum = fma_(lds.bc[r][1][l.first + i], h[i], sum);
        }
        if (MAP) total += in.s;
        else lds.part[r][l.group][l.c] = sum;
      }
    };
    if (rows == R) sweep(Steps<true, R>{R});
    else sweep(Steps<false, R>{rows});
    __syncthreads();
    if (!MAP && y && t + at.row < live && at.n > 0) {
      Pack<T, E> out;
#pragma unroll
      for (int i = 0; i < E; ++i) {
        A v = lds.part[at.row][0][at.c + i];
#pragma unroll
        for (int q = 1; q < S::SG; ++q) v += lds.part[at.row][q][at.c + i];
        v = fma_(skip[i], up((T)old_x.v[i]), v);
        if (a.z) {
          A f, rest;
          const A zi = up((T)old_z.v[i]);
          gates<T>(zi, &f, &rest);
          v *= zi * f;
        }
        out.v[i] = down<T>(v);
      }
      store_pack<T, E>(y + (p.b * a.T + t + at.row) * a.D_ + from, out, at.n);
    }
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
  if (y && at.n > 0) {
    Pack<T, E> zero;
#pragma unroll
    for (int i = 0; i < E; ++i) zero.v[i] = T(0);
    for (int64_t t = (live > t0 ? live : t0) + at.row; t < t1; t += R)
      store_pack<T, E>(y + (p.b * a.T + t) * a.D_ + from, zero, at.n);
  }
}

// ------------------------------------------------------------------- reverse
// Sums over the 32 lanes of each half wave: of V registers (a multiple of 32) each
// lane gets the V / 32 whose index, modulo 32, is its own in the half.
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
// Where there are fewer than 32 registers the lanes that differ in the other bits add up first.
template <int V, class A>
__device__ inline void sum_channels(A (&x)[V]) {
  static_assert(V >= 16, "");
  if constexpr (V >= 32) {
    fold<16>(x);
  } else {
#pragma unroll
    for (int k = 0; k < V; ++k) x[k] += __shfl_xor(x[k], 16, 64);
  }
  fold<8>(x);
  fold<4>(x);
  fold<2>(x);
  fold<1>(x);
}

template <class S>
struct ReverseLds {
  typedef typename S::A A;
  struct Four {
    A s, sx, dy, pad;
  };
  Four in[S::R][kSlab];
  A bc[S::R][2][S::NP];
  A part[3][S::R][S::SG][kSlab];  // of u, of sum A q, of y before skip and gate
};

// The partial sums that leave a workgroup.
template <class A>
struct Sums {
  A* bc;  // [slab][b][chunk][lanes of a channel][B or C][step][state of a lane]
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
template <class T, int NS, int W, bool MAP>
__global__ __launch_bounds__(64 * W) void scan_rev(ScanArgs a, ScanGrid g, void* ws, void* sums_ws) {
  typedef ScanShape<T, NS, W> S;
  typedef Acc<T> A;
  constexpr int R = S::R, E = S::E, V = R * NS;
  __shared__ ReverseLds<S> lds;
  Place p = place_of(a, g, work_id((int64_t)gridDim.x));
  const int64_t row = p.b;  // of workgroups: in the reverse sweep they take several batch rows
  const int64_t span = g.seg_chunks * R, t0 = p.segment * span;
  const int64_t t1 = a.T - t0 < span ? a.T : t0 + span;
  const Loader<S> at(p);
  const Lane l = lane_of<S>(a, p);
  const int64_t d = p.d0 + l.c;
  const int64_t from = p.d0 + at.c;
  A rates[NS], dA[NS];
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    rates[i] = i < l.count ? rate(static_cast<const A*>(a.A)[d * a.N + l.first + i]) : A(0);
    dA[i] = A(0);
  }
  A skip[E], bias[E], dD[E], dbias[E];
  at.constants(a.D, p.d0, skip);
  at.constants(a.bias, p.d0, bias);
#pragma unroll
  for (int i = 0; i < E; ++i) dD[i] = dbias[i] = A(0);
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
    Pack<T, E> x, delta, z, dy;
    Coefficients<T, S> bc;
    A before[NS];
    const auto request = [&](int64_t t) {
      const bool there = t + at.row < live;
      delta = at.template load<T>(a.delta, p.b * a.sl_b + (t + at.row) * a.sl_t + from, there);
      dy = at.template load<T>(a.dy, p.b * a.sd_b + (t + at.row) * a.sd_t + from, there);
      if (a.z) z = at.template load<T>(a.z, p.b * a.sz_b + (t + at.row) * a.sz_t + from, there);
      if (!MAP) {
        x = at.template load<T>(a.x, p.b * a.sx_b + (t + at.row) * a.sx_t + from, there);
        const A* const ck = static_cast<const A*>(a.ck) + (p.b * g.chunks + t / R) * a.N * a.D_;
#pragma unroll
        for (int i = 0; i < NS; ++i)
          before[i] = i < l.count ? ck[(l.first + i) * a.D_ + d] : A(0);
      }
      bc.load(a, p, t, (int)(live - t < R ? live - t : R), !MAP);
    };
    const int64_t last = live > t0 ? t0 + (live - t0 - 1) / R * R : t0 - R;
    if (last >= t0) request(last);
    for (int64_t t = last; t >= t0; t -= R) {
      const int rows = (int)(live - t < R ? live - t : R);
      A s_[E], x_[E], dy_[E], gate[E], of_gate[E], slope[E];
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const A raw = up((T)delta.v[i]) + bias[i];
        s_[i] = a.softplus ? softplus(raw) : raw;
        slope[i] = A(1);
        if (!MAP && a.softplus) {
          A rest;
          gates<T>(raw, &slope[i], &rest);
        }
        x_[i] = MAP ? A(0) : up((T)x.v[i]);
        dy_[i] = up((T)dy.v[i]);
        gate[i] = A(1);
        of_gate[i] = A(0);
        if (a.z) {
          A f, rest;
          const A zi = up((T)z.v[i]);
          gates<T>(zi, &f, &rest);
          gate[i] = zi * f;
          of_gate[i] = f * fma_(zi, rest, A(1));
        }
        if (threadIdx.x < S::kLoaders)
          lds.in[at.row][at.c + i] = {s_[i], s_[i] * x_[i], dy_[i] * gate[i], A(0)};
      }
      bc.put(lds.bc);
      A h[NS];
#pragma unroll
      for (int i = 0; i < NS; ++i) h[i] = MAP ? A(0) : before[i];
      __syncthreads();
      if (t > t0) request(t - R);
      const auto sweep = [&](auto steps) {
        if constexpr (MAP) {
#pragma unroll
          for (int r = R - 1; r >= 0; --r) {
            if (!steps.has(r)) continue;
            const auto in = lds.in[r][l.c];
            total += in.s;
#pragma unroll
            for (int i = 0; i < NS; ++i)
              G[i] = decay(in.s, rates[i]) * fma_(lds.bc[r][1][l.first + i], in.dy, G[i]);
          }
        } else {
          A e[R][NS], old[R][NS], ofB[V], ofC[V];
#pragma unroll
          for (int r = 0; r < R; ++r) {
            if (!steps.has(r)) break;
            const auto in = lds.in[r][l.c];
            A sum = A(0);
#pragma unroll
            for (int i = 0; i < NS; ++i) {
              e[r][i] = decay(in.s, rates[i]);
              old[r][i] = h[i];
              h[i] = fma_(e[r][i], h[i], in.sx * lds.bc[r][0][l.first + i]);
              sum = fma_(lds.bc[r][1][l.first + i], h[i], sum);
            }
            if (a.z) lds.part[2][r][l.group][l.c] = sum;
          }
#pragma unroll
          for (int r = R - 1; r >= 0; --r) {
#pragma unroll
            for (int i = 0; i < NS; ++i) ofB[r * NS + i] = ofC[r * NS + i] = A(0);
            if (!steps.has(r)) continue;
            const auto in = lds.in[r][l.c];
            A u = A(0), aq = A(0);
#pragma unroll
            for (int i = 0; i < NS; ++i) {
              G[i] = fma_(lds.bc[r][1][l.first + i], in.dy, G[i]);
              ofC[r * NS + i] = in.dy * h[i];
              ofB[r * NS + i] = G[i] * in.sx;
              u = fma_(G[i], lds.bc[r][0][l.first + i], u);
              G[i] *= e[r][i];
              h[i] = old[r][i];
              const A q = G[i] * h[i];
              dA[i] = fma_(in.s, q, dA[i]);
              aq = fma_(rates[i], q, aq);
            }
            lds.part[0][r][l.group][l.c] = u;
            lds.part[1][r][l.group][l.c] = aq;
          }
          sum_channels(ofB);
          sum_channels(ofC);
          A* const to = sums.bc + ((((p.slab * a.B + p.b) * g.chunks + t / R) * S::SG + l.group) * 2)
                                      * V;
#pragma unroll
          for (int k = 0; k < V; k += kSlab)
            if (k + l.c < V) {
              to[k + l.c] = ofB[k];
              to[V + k + l.c] = ofC[k];
            }
        }
      };
      if (rows == R) sweep(Steps<true, R>{R});
      else sweep(Steps<false, R>{rows});
      __syncthreads();
      if (!MAP && t + at.row < live && at.n > 0) {
        Pack<T, E> ox, od, oz;
#pragma unroll
        for (int i = 0; i < E; ++i) {
          A u = A(0), aq = A(0), yp = A(0);
#pragma unroll
          for (int q = 0; q < S::SG; ++q) {
            u += lds.part[0][at.row][q][at.c + i];
            aq += lds.part[1][at.row][q][at.c + i];
            if (a.z) yp += lds.part[2][at.row][q][at.c + i];
          }
          const A through_gate = dy_[i] * gate[i];
          const A of_raw = fma_(u, x_[i], of_rate(aq)) * slope[i];
          ox.v[i] = down<T>(fma_(s_[i], u, skip[i] * through_gate));
          od.v[i] = down<T>(of_raw);
          oz.v[i] = down<T>(dy_[i] * fma_(skip[i], x_[i], yp) * of_gate[i]);
          dD[i] = fma_(through_gate, x_[i], dD[i]);
          dbias[i] += of_raw;
        }
        const int64_t to = (p.b * a.T + t + at.row) * a.D_ + from;
        store_pack<T, E>(static_cast<T*>(a.out.dx) + to, ox, at.n);
        store_pack<T, E>(static_cast<T*>(a.out.ddelta) + to, od, at.n);
        if (a.z) store_pack<T, E>(static_cast<T*>(a.out.dz) + to, oz, at.n);
      }
    }
    if (MAP) {
#pragma unroll
      for (int i = 0; i < NS; ++i)
        if (i < l.count)
          maps.h[((p.b * g.segments + p.segment) * a.N + l.first + i) * a.D_ + d] = G[i];
      if (l.channel && l.group == 0) maps.s[(p.b * g.segments + p.segment) * a.D_ + d] = total;
      return;
    }
    if (p.segment == 0 && a.out.dh0)
#pragma unroll
      for (int i = 0; i < NS; ++i)
        if (i < l.count)
          static_cast<A*>(a.out.dh0)[(p.b * a.D_ + d) * a.N + l.first + i] = G[i];
    if (at.n > 0) {
      Pack<T, E> zero;
#pragma unroll
      for (int i = 0; i < E; ++i) zero.v[i] = T(0);
      for (int64_t t = (live > t0 ? live : t0) + at.row; t < t1; t += R) {
        const int64_t to = (p.b * a.T + t) * a.D_ + from;
        store_pack<T, E>(static_cast<T*>(a.out.dx) + to, zero, at.n);
        store_pack<T, E>(static_cast<T*>(a.out.ddelta) + to, zero, at.n);
        if (a.z) store_pack<T, E>(static_cast<T*>(a.out.dz) + to, zero, at.n);
      }
    }
  }
  const int64_t part = row * g.segments + p.segment;
#pragma unroll
  for (int i = 0; i < NS; ++i)
    if (i < l.count) sums.a[(part * a.N + l.first + i) * a.D_ + d] = dA[i];
  // the loaders' sums of a channel, step after step of the chunk
  A(*const rows_of)[2][kSlab] = reinterpret_cast<A(*)[2][kSlab]>(&lds.part[0][0][0][0]);
  __syncthreads();
  if (threadIdx.x < S::kLoaders)
#pragma unroll
    for (int i = 0; i < E; ++i) {
      rows_of[at.row][0][at.c + i] = dD[i];
      rows_of[at.row][1][at.c + i] = dbias[i];
    }
  __syncthreads();
  if (threadIdx.x < 2 * kSlab && (int)threadIdx.x % kSlab < p.channels) {
    const int which = threadIdx.x / kSlab, c = threadIdx.x % kSlab;
    A v = A(0);
    for (int r = 0; r < R; ++r) v += rows_of[r][which][c];
    sums.d[(part * 2 + which) * a.D_ + p.d0 + c] = v;
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
  const int64_t t = chunk * g.chunk + k / g.states, n = lane * g.states + k % g.states;
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

// dA, dD and dbias: over the rows of workgroups and the segments.
template <class T>
__global__ __launch_bounds__(kSumThreads) void scan_sum_a(ScanArgs a, ScanGrid g, void* ws) {
  typedef Acc<T> A;
  const Sums<A> sums(ws, a.B, a.D_, a.N, g);
  const int64_t id = (int64_t)blockIdx.x * kSumThreads + threadIdx.x, parts = g.rows * g.segments;
  if (id >= (a.N + 2) * a.D_) return;
  const int64_t n = id / a.D_, d = id % a.D_;
  const A* from = n < a.N ? sums.a + n * a.D_ + d : sums.d + (n - a.N) * a.D_ + d;
  const int64_t by = (n < a.N ? a.N : 2) * a.D_;
  A v = A(0);
#pragma unroll 8
  for (int64_t k = 0; k < parts; ++k) v += from[k * by];
  if (n < a.N) static_cast<A*>(a.out.dA)[d * a.N + n] = v;
  else if (n == a.N && a.out.dD) static_cast<A*>(a.out.dD)[d] = v;
  else if (n > a.N && a.out.ddelta_bias) static_cast<A*>(a.out.ddelta_bias)[d] = v;
}

// ------------------------------------------------------------------ one step
// A lane: four neighbouring states of a channel; `lanes` lanes, a power of two, share
// a channel.
template <class T>
__global__ __launch_bounds__(256) void scan_one(ScanStep q, int lanes) {
  typedef Acc<T> A;
  const ScanArgs& a = q.a;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int first = (int)(id % lanes) * 4;
  const int64_t channel = id / lanes, b = channel / a.D_, d = channel % a.D_;
  const int64_t slot = b < a.B ? (q.slots ? q.slots[b] : b) : -1;
  const bool on = slot >= 0 && slot < q.nstates;
  A sum = A(0), x = A(0);
  if (on) {
    const int left = a.N - first, n = left < 0 ? 0 : left < 4 ? left : 4;
    x = up(static_cast<const T*>(a.x)[b * a.sx_b + d]);
    A s = up(static_cast<const T*>(a.delta)[b * a.sl_b + d]);
    if (a.bias) s += static_cast<const A*>(a.bias)[d];
    if (a.softplus) s = softplus(s);
    const int64_t group = d / (a.D_ / a.G);
    A* const state = static_cast<A*>(q.state) + (slot * a.D_ + d) * a.N + first;
    Pack<A, 4> h = load_pack<A, 4>(state, n);
    const Pack<A, 4> r = load_pack<A, 4>(static_cast<const A*>(a.A) + d * a.N + first, n);
    const Pack<T, 4> B = load_pack<T, 4>(
        static_cast<const T*>(a.Bm) + b * a.sb_b + group * a.N + first, n);
    const Pack<T, 4> C = load_pack<T, 4>(
        static_cast<const T*>(a.Cm) + b * a.sc_b + group * a.N + first, n);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) {
        h.v[i] = fma_(decay(s, rate((A)r.v[i])), (A)h.v[i], s * x * up((T)B.v[i]));
        sum = fma_(up((T)C.v[i]), (A)h.v[i], sum);
      }
    store_pack<A, 4>(state, h, n);
  }
  for (int by = 1; by < lanes; by <<= 1) sum += __shfl_xor(sum, by, 64);
  if (first > 0 || b >= a.B || !a.y) return;
  A v = A(0);
  if (on) {
    v = a.D ? fma_(static_cast<const A*>(a.D)[d], x, sum) : sum;
    if (a.z) {
      A f, rest;
      const A z = up(static_cast<const T*>(a.z)[b * a.sz_b + d]);
      gates<T>(z, &f, &rest);
      v *= z * f;
    }
  }
  static_cast<T*>(a.y)[b * a.D_ + d] = down<T>(v);
}

// ------------------------------------------------------------------ launches
// f(shape) for the shape that the grid names.
template <class T, class F>
hipError_t by_shape(const ScanGrid& g, F f) {
  if (g.states == 2 && g.waves == 1) return f(ScanShape<T, 2, 1>());
  if (g.states == 2 && g.waves == 2) return f(ScanShape<T, 2, 2>());
  if (g.states == 2 && g.waves == 4) return f(ScanShape<T, 2, 4>());
  if (g.states == 4 && g.waves == 4) return f(ScanShape<T, 4, 4>());
  if (g.states == 4 && g.waves == 8) return f(ScanShape<T, 4, 8>());
  if constexpr (sizeof(T) < 8)
    if (g.states == 8 && g.waves == 8) return f(ScanShape<T, 8, 8>());
  return hipErrorInvalidValue;
}

template <class T>
hipError_t forward_of(const ScanArgs& a, const ScanGrid& g, void* ws, hipStream_t st) {
  return by_shape<T>(g, [&](auto shape) {
    typedef decltype(shape) S;
    const dim3 groups((unsigned)(g.slabs * g.segments * a.B));
    if (g.segments > 1) {
      const hipError_t e = start(scan_fwd<T, S::NS, S::W, true>, groups, S::NT, st, a, g, ws);
      if (e != hipSuccess) return e;
    }
    return start(scan_fwd<T, S::NS, S::W, false>, groups, S::NT, st, a, g, ws);
  });
}

template <class T>
hipError_t vjp_of(const ScanArgs& a, const ScanGrid& g, void* ws, hipStream_t st) {
  void* const sums = static_cast<char*>(ws) + g.map_bytes;
  return by_shape<T>(g, [&](auto shape) {
    typedef decltype(shape) S;
    if (g.segments > 1) {
      const hipError_t e = start(scan_rev<T, S::NS, S::W, true>,
                                 dim3((unsigned)(g.slabs * g.segments * a.B)), S::NT, st, a, g, ws,
                                 sums);
      if (e != hipSuccess) return e;
    }
    hipError_t e = start(scan_rev<T, S::NS, S::W, false>,
                         dim3((unsigned)(g.slabs * g.segments * g.rows)), S::NT, st, a, g, ws, sums);
    if (e != hipSuccess) return e;
    const int64_t bc = a.B * g.chunks * g.chunk * 2 * S::NP * a.G;
    if (bc > 0) {
      e = start(scan_sum_bc<T>, dim3((unsigned)((bc + kSumThreads - 1) / kSumThreads)), kSumThreads,
                st, a, g, sums);
      if (e != hipSuccess) return e;
    }
    const int64_t rest = (a.N + 2) * a.D_;
    return start(scan_sum_a<T>, dim3((unsigned)((rest + kSumThreads - 1) / kSumThreads)),
                 kSumThreads, st, a, g, sums);
  });
}

template <class T>
hipError_t step_of(const ScanStep& q, hipStream_t st) {
  int lanes = 1;
  while (lanes * 4 < q.a.N) lanes *= 2;
  const int64_t groups = (q.a.B * q.a.D_ * lanes + 255) / 256;
  return start(scan_one<T>, dim3((unsigned)groups), 256, st, q, lanes);
}

}  // namespace
}  // namespace adst
