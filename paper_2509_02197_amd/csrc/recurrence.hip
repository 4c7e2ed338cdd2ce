// Gated linear recurrence: h_t = c_t h_{t-1} + d_t per channel, with
// (c, d) = (a, u) or (s, (1 - s) u), s = 1 / (1 + exp(-a)); its VJP, which
// recomputes the states from checkpoints; and one step on a pool of states.
//
// A step is an affine map of the state, and maps compose: (A, H) after
// (A', H') is (A A', A H' + H). So a row is cut into spans, a workgroup each:
// it loads its span once, composes its steps, learns the state at its start
// from the spans before it, and applies its steps to that. Everything is read
// and written once, and HBM bandwidth bounds it. A workgroup's lanes lie along
// channels (16 lanes of 16 bytes: 256 consecutive bytes of a step) and its
// groups of 16 lanes along time, each with R consecutive steps in registers;
// maps are composed within a lane, over the wave by lane shifts, and over the
// waves through LDS. The reverse sweep is the same recurrence backwards
// (G_t = dh_t + c_{t+1} G_{t+1}); it recomputes its span's states in registers
// from the checkpoint at its start, so the forward's h is not needed: reading
// a, u and dh and writing da and du is all it moves.
//
// Between spans: a workgroup publishes its span's map (A, H) as soon as it has
// it, and the state at its end as soon as it knows that. To learn the state at
// its start it takes the nearest published state before it and applies the
// published maps of the spans between, in order: state' = A state + H. That is
// what each of those spans computes for itself, bit for bit, so the result
// does not depend on which states happened to be there. Spans are taken from a
// counter per row in the order of time, so a workgroup only ever waits for
// workgroups that have started before it, whose maps depend on nothing: every
// wait ends. What is published is complete in itself (each word is written
// whole, and its initial pattern is never a value), so no fence is needed; the
// accesses are of agent scope, which the caches of the XCDs keep coherent.

#include "seq_common.h"
#include "seq_kernels.h"

namespace adst {
namespace {

constexpr int kLanes = 16;  // along channels

template <class T>
struct Shape {
  static constexpr int V = Vec<T>::N;               // channels of a lane
  static constexpr int R = sizeof(T) == 2 ? 4 : 8;  // steps of a lane
  static constexpr int C = kLanes * V;              // channels of a workgroup
  static constexpr int span(int threads) { return threads / kLanes * R; }
};

// How a problem is laid out over workgroups of `threads`.
struct Grid {
  int threads;
  int span;    // steps
  int spans;   // per batch row
  int slabs;   // of C channels
  uint32_t chains;  // batch rows times slabs
};

// What a launch of several spans publishes in, all ones at its start.
struct Board {
  int32_t* next;  // a counter per chain, 32 bytes apart, from -1
  void* state;    // [chain][span][C] accumulation type
  void* map;      // [chain][span][C] two of it
};
constexpr int kCounterInts = 8;

// ---------------------------------------------------------------- the gates
__device__ inline float exp_full(float x) { return expf(x); }
__device__ inline double exp_full(double x) { return exp(x); }
__device__ inline float inverse(float x) { return __builtin_amdgcn_rcpf(x); }  // within 1 ulp
__device__ inline double inverse(double x) { return 1.0 / x; }

// min(s, 1 - s) to full relative precision, with the sign of a: with
// e = exp(-|a|) in [0, 1], it is e / (1 + e), and the other one is 1 less it,
// which loses nothing as it is at least a half. Behind a 16-bit value the
// exponential may be off by |a| units of 2^-24.
template <class T>
__device__ inline Acc<T> gate_of(Acc<T> a) {
  typedef Acc<T> A;
  A e;
  if constexpr (sizeof(T) == 2)
    e = __builtin_amdgcn_exp2f(-1.44269504f * __builtin_fabsf(a));
  else
    e = exp_full(-__builtin_elementwise_abs(a));
  return __builtin_elementwise_copysign(e * inverse(A(1) + e), a);
}
// The compiler treats the values as new ones: it does not keep what it
// derived from them before, which would take more registers than there are.
template <class A, int R, int V>
__device__ inline void forget(A (&x)[R][V]) {
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int i = 0; i < V; ++i) asm volatile("" : "+v"(x[r][i]));
}
template <class A>
__device__ inline bool negative(A x) {
  return __builtin_signbit(x);
}
template <class A>
__device__ inline void open_gate(A gate, A* s, A* q) {
  const A small = __builtin_elementwise_abs(gate), big = A(1) - small;
  *s = negative(gate) ? small : big;
  *q = negative(gate) ? big : small;
}

__device__ inline int64_t row_length(const int32_t* lens, int64_t b, int64_t T) {
  if (!lens) return T;
  const int64_t n = lens[b];
  return n < 0 ? 0 : n > T ? T : n;
}

// ------------------------------------------------------- maps along the time
// Inclusive composition over the wave's groups of lanes, each group's map
// applied after those of the groups before it (FORWARD) or after it.
template <bool FORWARD, class A, int V>
__device__ inline void compose_wave(A (&a)[V], A (&h)[V]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int off = kLanes; off < 64; off <<= 1) {
    const bool has = FORWARD ? lane >= off : lane + off < 64;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const A oa = FORWARD ? __shfl_up(a[i], off, 64) : __shfl_down(a[i], off, 64);
      const A oh = FORWARD ? __shfl_up(h[i], off, 64) : __shfl_down(h[i], off, 64);
      h[i] = has ? fma_(a[i], oh, h[i]) : h[i];
      a[i] = has ? a[i] * oa : a[i];
    }
  }
}
// The composition of the groups before (after) this one, from the inclusive one.
template <bool FORWARD, class A, int V>
__device__ inline void exclude_own(A (&a)[V], A (&h)[V]) {
  const int lane = threadIdx.x & 63;
  const bool has = FORWARD ? lane >= kLanes : lane + kLanes < 64;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const A oa = FORWARD ? __shfl_up(a[i], kLanes, 64) : __shfl_down(a[i], kLanes, 64);
    const A oh = FORWARD ? __shfl_up(h[i], kLanes, 64) : __shfl_down(h[i], kLanes, 64);
    a[i] = has ? oa : A(1);
    h[i] = has ? oh : A(0);
  }
}

// Per wave and channel, in LDS: first each wave's map, then the composition of
// the waves before (after) it.
template <class A, int W, int C>
struct Maps {
  A a[W][C], h[W][C];
};
// One thread a channel: from the waves' maps to exclusive ones, in place, and
// the workgroup's map.
template <bool FORWARD, class A, int W, int C>
__device__ inline void compose_waves(Maps<A, W, C>& m, int c, A* a_out, A* h_out) {
  A a = A(1), h = A(0);
#pragma unroll
  for (int k = 0; k < W; ++k) {
    const int w = FORWARD ? k : W - 1 - k;
    const A wa = m.a[w][c], wh = m.h[w][c];
    m.a[w][c] = a;
    m.h[w][c] = h;
    h = fma_(wa, h, wh);
    a = wa * a;
  }
  *a_out = a;
  *h_out = h;
}

// ------------------------------------------------------------- between spans
template <class A>
struct WordOf {
  typedef uint32_t type;
  static constexpr uint32_t kNan = 0x7fc00000u;
};
template <>
struct WordOf<double> {
  typedef uint64_t type;
  static constexpr uint64_t kNan = 0x7ff8000000000000ull;
};
template <class A>
using Word = typename WordOf<A>::type;

template <class W>
__device__ inline W agent_load(const W* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <class W>
__device__ inline void agent_store(W* p, W v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// A value's word: its bits, and another NaN's for the NaN that means "empty".
template <class A>
__device__ inline Word<A> word_of(A v) {
  const Word<A> w = __builtin_bit_cast(Word<A>, v);
  return w == ~Word<A>(0) ? WordOf<A>::kNan : w;
}

// (A, H) in one word of 8 bytes, or in two for double precision.
template <class A>
struct MapWords;
template <>
struct MapWords<float> {
  uint64_t w;
  __device__ bool full() const { return ~w != 0; }
  __device__ static MapWords load(const void* base, int64_t i) {
    return {agent_load((const uint64_t*)base + i)};
  }
  __device__ static void store(void* base, int64_t i, float a, float h) {
    agent_store((uint64_t*)base + i, (uint64_t)word_of(h) << 32 | word_of(a));
  }
  __device__ float apply(float x) const {
    return fma_(__builtin_bit_cast(float, (uint32_t)w), x,
                __builtin_bit_cast(float, (uint32_t)(w >> 32)));
  }
};
template <>
struct MapWords<double> {
  uint64_t a, h;
  __device__ bool full() const { return ~a != 0 && ~h != 0; }
  __device__ static MapWords load(const void* base, int64_t i) {
    const uint64_t* p = (const uint64_t*)base + 2 * i;
    return {agent_load(p), agent_load(p + 1)};
  }
  __device__ static void store(void* base, int64_t i, double a, double h) {
    uint64_t* p = (uint64_t*)base + 2 * i;
    agent_store(p, word_of(a));
    agent_store(p + 1, word_of(h));
  }
  __device__ double apply(double x) const {
    return fma_(__builtin_bit_cast(double, a), x, __builtin_bit_cast(double, h));
  }
};

// The state that enters this span, one thread a channel. `at`: this span's
// and channel's place on the board; the span before (FORWARD) or after it is
// `step` places away, the wave's first channel's place is `first`; `before`:
// how many spans there are on that side, at least 1, the last of which
// publishes its end state without waiting. Whole waves call this; a lane
// without a channel (mine false) only takes part in the looking.
template <class A>
__device__ inline A enter(const Board& bd, int64_t at, int64_t first, int64_t step, int before,
                          bool mine) {
  const Word<A>* states = (const Word<A>*)bd.state;
  // Lane l looks at the span l + 1 away: the nearest one with a state, and
  // whether all maps up to it are there.
  const int lane = threadIdx.x & 63;
  const bool there = lane < before;
  const int64_t seen = first + (int64_t)(lane + 1) * step;
  int k;
  for (;;) {
    const bool s = there && ~agent_load(states + seen) != 0;
    const bool m = there && MapWords<A>::load(bd.map, seen).full();
    const uint64_t with_state = __ballot(s), with_map = __ballot(m);
    if (with_state) {
      k = __ffsll((unsigned long long)with_state) - 1;
      const uint64_t need = (uint64_t(1) << k) - 1;
      if ((with_map & need) == need) break;
    }
    __builtin_amdgcn_s_sleep(1);
  }
  A x = A(0);
  if (!mine) return x;
  // The words of this lane's own channel were written with those looked at;
  // each is checked all the same.
  int64_t j = at + (int64_t)(k + 1) * step;
  Word<A> w;
  do w = agent_load(states + j);
  while (~w == 0);
  x = __builtin_bit_cast(A, w);
  constexpr int kAhead = 8;  // maps under way at a time
  while (k > 0) {
    const int n = k < kAhead ? k : kAhead;
    MapWords<A> m[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (i < n) m[i] = MapWords<A>::load(bd.map, j - (int64_t)(i + 1) * step);
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (i < n) {
        while (!m[i].full()) m[i] = MapWords<A>::load(bd.map, j - (int64_t)(i + 1) * step);
        x = m[i].apply(x);
      }
    j -= (int64_t)n * step;
    k -= n;
  }
  return x;
}

// -------------------------------------------------------------- the kernels
// Where a workgroup works, and how much of it exists.
template <class T, int NT>
struct Place {
  typedef Shape<T> S;
  int64_t b, len;  // the batch row and its steps
  int slab, span;
  int64_t t0;     // the span's first step
  int64_t mine;   // this lane's first step
  int c0, n;      // this lane's first channel, and how many it has
  bool whole;     // every step and channel of the workgroup exists
  __device__ Place(const RecArgs& r, const Grid& g, uint32_t chain, int span_) {
    span = span_;
    b = chain / (uint32_t)g.slabs;
    slab = (int)(chain % (uint32_t)g.slabs);
    len = row_length(r.lens, b, r.T);
    constexpr int kSpan = S::span(NT);
    t0 = (int64_t)span * kSpan;
    mine = t0 + threadIdx.x / kLanes * S::R;
    c0 = slab * S::C + (int)(threadIdx.x % kLanes) * S::V;
    const int64_t left = r.D - c0;
    n = left < 0 ? 0 : left < S::V ? (int)left : S::V;
    whole = (int64_t)(slab + 1) * S::C <= r.D && t0 + kSpan <= len;
  }
};

// This lane's R vectors of a strided array; zero where steps or channels end.
template <class T, int NT>
__device__ inline void load_steps(const void* base, int64_t sb, int64_t stp,
                                  const Place<T, NT>& at, Vec<T> (&v)[Shape<T>::R]) {
  const T* p = (const T*)base + at.b * sb + at.mine * stp + at.c0;
  if (at.whole) {
#pragma unroll
    for (int r = 0; r < Shape<T>::R; ++r) v[r] = load_vec(p + r * stp);
    return;
  }
#pragma unroll
  for (int r = 0; r < Shape<T>::R; ++r) {
    v[r].v = typename Vec<T>::type{};
    if (at.mine + r < at.len && at.n > 0) v[r] = load_part(p + r * stp, at.n);
  }
}
// Stores them to a contiguous array: up to T, zeros from len on.
template <class T, int NT>
__device__ inline void store_steps(void* base, const RecArgs& q, const Place<T, NT>& at,
                                   const Vec<T> (&v)[Shape<T>::R]) {
  T* p = (T*)base + (at.b * q.T + at.mine) * q.D + at.c0;
  if (at.whole) {
#pragma unroll
    for (int r = 0; r < Shape<T>::R; ++r) store_vec(p + r * q.D, v[r]);
    return;
  }
#pragma unroll
  for (int r = 0; r < Shape<T>::R; ++r)
    if (at.mine + r < q.T && at.n > 0) {
      Vec<T> x = v[r];
      if (at.mine + r >= at.len) x.v = typename Vec<T>::type{};
      store_part(p + r * q.D, x, at.n);
    }
}

template <class T, bool SIG, bool MULTI, int NT>
__global__ __launch_bounds__(NT) void rec_fwd(RecArgs q, Grid g, Board bd) {
  typedef Acc<T> A;
  typedef Shape<T> S;
  constexpr int V = S::V, R = S::R, C = S::C, W = NT / 64;
  __shared__ Maps<A, W, C> maps;
  __shared__ A start[C];
  __shared__ int ticket;
  const uint32_t chain = blockIdx.x % g.chains;
  if (MULTI) {
    if (threadIdx.x == 0) ticket = atomicAdd(bd.next + (int64_t)chain * kCounterInts, 1) + 1;
    __syncthreads();
  }
  const Place<T, NT> at(q, g, chain, MULTI ? ticket : 0);
  if (at.t0 >= at.len && at.span > 0) {  // nothing but zeros, and nobody asks for its state
    Vec<T> zero[R];
#pragma unroll
    for (int r = 0; r < R; ++r) zero[r].v = typename Vec<T>::type{};
    if (q.h) store_steps<T, NT>(q.h, q, at, zero);
    return;
  }
  Vec<T> va[R], vu[R];
  load_steps<T, NT>(q.a, q.sa_b, q.sa_t, at, va);
  load_steps<T, NT>(q.u, q.su_b, q.su_t, at, vu);

  A c[R][V], d[R][V], a[V], h[V];
#pragma unroll
  for (int i = 0; i < V; ++i) a[i] = A(1), h[i] = A(0);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const bool live = at.whole || (at.mine + r < at.len);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      A cc = up(va[r].v[i]), dd = up(vu[r].v[i]);
      if (SIG) {
        A s, o;
        open_gate(gate_of<T>(cc), &s, &o);
        cc = s;
        dd = o * dd;
      }
      c[r][i] = live ? cc : A(1);
      d[r][i] = live ? dd : A(0);
      h[i] = fma_(c[r][i], h[i], d[r][i]);
      a[i] *= c[r][i];
    }
  }
  compose_wave<true>(a, h);
  const int wave = threadIdx.x / 64, lane = threadIdx.x & 63;
  const int col = (threadIdx.x % kLanes) * V;
  if (lane >= 64 - kLanes) {
#pragma unroll
    for (int i = 0; i < V; ++i) maps.a[wave][col + i] = a[i], maps.h[wave][col + i] = h[i];
  }
  exclude_own<true>(a, h);
  __syncthreads();
  for (int k = threadIdx.x; k < C; k += NT) {
    A ma, mh;
    compose_waves<true>(maps, k, &ma, &mh);
    const int64_t ch = (int64_t)at.slab * C + k;
    const bool mine = ch < q.D;
    const bool last = at.t0 + S::span(NT) >= at.len;
    const int64_t place = ((int64_t)chain * g.spans + at.span) * C + k;
    A x = A(0);
    if (!MULTI || at.span == 0) {
      if (mine && q.h0) x = ((const A*)q.h0)[at.b * q.D + ch];
    } else {
      if (mine && !last) MapWords<A>::store(bd.map, place, ma, mh);
      asm volatile("" ::: "memory");  // published before this wave waits
      if ((int64_t)at.slab * C + (k & ~63) < q.D)
        x = enter<A>(bd, place, place - (k & 63), -C, at.span, mine);
    }
    const A end = fma_(ma, x, mh);
    if (MULTI && mine && !last) agent_store((Word<A>*)bd.state + place, word_of(end));
    if (mine && q.ck) ((A*)q.ck)[(at.b * g.spans + at.span) * q.D + ch] = x;
    if (mine && last && q.hT) ((A*)q.hT)[at.b * q.D + ch] = end;
    start[k] = x;
  }
  if (!q.h) return;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const A x = fma_(maps.a[wave][col + i], start[col + i], maps.h[wave][col + i]);
    h[i] = fma_(a[i], x, h[i]);
  }
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      h[i] = fma_(c[r][i], h[i], d[r][i]);
      va[r].v[i] = down<T>(h[i]);
    }
  store_steps<T, NT>(q.h, q, at, va);
}

template <class T, bool SIG, bool MULTI, int NT>
__global__ __launch_bounds__(NT) void rec_rev(RecArgs q, Grid g, Board bd) {
  typedef Acc<T> A;
  typedef Shape<T> S;
  constexpr int V = S::V, R = S::R, C = S::C, W = NT / 64;
  __shared__ Maps<A, W, C> maps, rmaps;
  __shared__ A start[C], finish[C];
  __shared__ int ticket;
  const uint32_t chain = blockIdx.x % g.chains;
  if (MULTI) {
    if (threadIdx.x == 0) ticket = atomicAdd(bd.next + (int64_t)chain * kCounterInts, 1) + 1;
    __syncthreads();
  }
  const Place<T, NT> at(q, g, chain, MULTI ? g.spans - 1 - ticket : 0);
  Vec<T> va[R], vu[R], vd[R];
  if (at.t0 >= at.len && at.span > 0) {
#pragma unroll
    for (int r = 0; r < R; ++r) va[r].v = typename Vec<T>::type{};
    store_steps<T, NT>(q.da, q, at, va);
    store_steps<T, NT>(q.du, q, at, va);
    return;
  }
  load_steps<T, NT>(q.a, q.sa_b, q.sa_t, at, va);
  load_steps<T, NT>(q.u, q.su_b, q.su_t, at, vu);
  load_steps<T, NT>(q.dh, q.sd_b, q.sd_t, at, vd);

  // gate[r][i]: the coefficient, or gate_of it. Steps beyond the end keep the
  // state and the gradient: coefficient 1, input 0.
  A gate[R][V], a[V], h[V], ra[V], rh[V];
  constexpr A kKeep = SIG ? A(0) : A(1);
#pragma unroll
  for (int i = 0; i < V; ++i) a[i] = A(1), h[i] = A(0), rh[i] = A(0);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const bool live = at.whole || (at.mine + r < at.len);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      A cc = up(va[r].v[i]), dd = up(vu[r].v[i]);
      if (SIG) cc = gate_of<T>(cc);
      gate[r][i] = live ? cc : kKeep;
      A s = gate[r][i];
      if (SIG) {
        A o;
        open_gate(gate[r][i], &s, &o);
        dd = o * dd;
      }
      h[i] = fma_(s, h[i], dd);
      a[i] *= s;
    }
  }
  if (SIG) forget(gate);
#pragma unroll
  for (int r = R - 1; r >= 0; --r)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      A s = gate[r][i], o;
      if (SIG) open_gate(gate[r][i], &s, &o);
      rh[i] = s * (up(vd[r].v[i]) + rh[i]);
    }
#pragma unroll
  for (int i = 0; i < V; ++i) ra[i] = a[i];
  compose_wave<true>(a, h);
  compose_wave<false>(ra, rh);
  const int wave = threadIdx.x / 64, lane = threadIdx.x & 63;
  const int col = (threadIdx.x % kLanes) * V;
  if (lane >= 64 - kLanes) {
#pragma unroll
    for (int i = 0; i < V; ++i) maps.a[wave][col + i] = a[i], maps.h[wave][col + i] = h[i];
  }
  if (lane < kLanes) {
#pragma unroll
    for (int i = 0; i < V; ++i) rmaps.a[wave][col + i] = ra[i], rmaps.h[wave][col + i] = rh[i];
  }
  exclude_own<true>(a, h);
  exclude_own<false>(ra, rh);
  __syncthreads();
  for (int k = threadIdx.x; k < C; k += NT) {
    A ma, mh;
    compose_waves<true>(maps, k, &ma, &mh);
    compose_waves<false>(rmaps, k, &ma, &mh);
    const int64_t ch = (int64_t)at.slab * C + k;
    const bool mine = ch < q.D;
    // the row's last span, where the gradient of the last state enters
    const int last = at.len > 0 ? (int)((at.len - 1) / S::span(NT)) : 0;
    const int64_t place = ((int64_t)chain * g.spans + at.span) * C + k;
    A x = A(0);
    if (!MULTI || at.span == last) {
      if (mine && q.dhT) x = ((const A*)q.dhT)[at.b * q.D + ch];
    } else {
      if (mine && at.span > 0) MapWords<A>::store(bd.map, place, ma, mh);
      asm volatile("" ::: "memory");  // published before this wave waits
      if ((int64_t)at.slab * C + (k & ~63) < q.D)
        x = enter<A>(bd, place, place - (k & 63), C, last - at.span, mine);
    }
    const A end = fma_(ma, x, mh);
    if (MULTI && mine && at.span > 0) agent_store((Word<A>*)bd.state + place, word_of(end));
    if (mine && at.span == 0 && q.dh0) ((A*)q.dh0)[at.b * q.D + ch] = end;
    finish[k] = x;
    start[k] = mine ? ((const A*)q.ck)[(at.b * g.spans + at.span) * q.D + ch] : A(0);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const A x = fma_(maps.a[wave][col + i], start[col + i], maps.h[wave][col + i]);
    h[i] = fma_(a[i], x, h[i]);
    const A y = fma_(rmaps.a[wave][col + i], finish[col + i], rmaps.h[wave][col + i]);
    rh[i] = fma_(ra[i], y, rh[i]);
  }
  if (SIG) forget(gate);
  // e[r][i]: what G_t is multiplied with in da_t
  A e[R][V];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const A x = h[i], u = up(vu[r].v[i]);
      if (SIG) {
        A s, o;
        open_gate(gate[r][i], &s, &o);
        e[r][i] = (x - u) * (s * o);
        h[i] = fma_(s, x, o * u);
      } else {
        e[r][i] = x;
        h[i] = fma_(gate[r][i], x, u);
      }
    }
  if (SIG) forget(gate);
#pragma unroll
  for (int r = R - 1; r >= 0; --r)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const A G = up(vd[r].v[i]) + rh[i];
      A s = gate[r][i], o = A(1);
      if (SIG) open_gate(gate[r][i], &s, &o);
      va[r].v[i] = down<T>(G * e[r][i]);
      vu[r].v[i] = down<T>(SIG ? G * o : G);
      rh[i] = s * G;
    }
  store_steps<T, NT>(q.da, q, at, va);
  store_steps<T, NT>(q.du, q, at, vu);
}

// One step of B rows on a pool of states, V channels a thread. Latency bounds
// it: a row's slot, then its state.
constexpr int kStepThreads = 64;
template <class T, bool SIG>
__global__ __launch_bounds__(kStepThreads) void rec_one(RecStep q, int64_t per_row) {
  typedef Acc<T> A;
  constexpr int V = Vec<T>::N;
  const int64_t i = (int64_t)blockIdx.x * kStepThreads + threadIdx.x;
  if (i >= q.B * per_row) return;
  const int64_t b = i / per_row, d = i % per_row * V;
  const int n = (int)min((int64_t)V, q.D - d);
  const Vec<T> a = load_part((const T*)q.a + b * q.sa + d, n);
  const Vec<T> u = load_part((const T*)q.u + b * q.su + d, n);
  const int64_t slot = q.slots ? q.slots[b] : b;
  Vec<T> out;
  out.v = typename Vec<T>::type{};
  if (slot >= 0 && slot < q.nstates) {
    A* const state = (A*)q.state + slot * q.D + d;
    constexpr int N = Vec<A>::N;
    Vec<A> x[V / N];
#pragma unroll
    for (int k = 0; k < V / N; ++k)
      x[k] = load_part(state + k * N, n - k * N);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      A c = up(a.v[j]), v = up(u.v[j]);
      if (SIG) {
        A s, o;
        open_gate(gate_of<T>(c), &s, &o);
        c = s;
        v = o * v;
      }
      const A y = fma_(c, x[j / N].v[j % N], v);
      x[j / N].v[j % N] = y;
      out.v[j] = down<T>(y);
    }
#pragma unroll
    for (int k = 0; k < V / N; ++k) store_part(state + k * N, x[k], n - k * N);
  }
  if (q.h) store_part((T*)q.h + b * q.D + d, out, n);
}

constexpr int kFillThreads = 256;
__global__ __launch_bounds__(kFillThreads) void fill_ones(uint4* p, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * kFillThreads + threadIdx.x;
  if (i < n) p[i] = make_uint4(~0u, ~0u, ~0u, ~0u);
}

// -------------------------------------------------------------- on the host
int type_steps(int32_t dtype) { return dtype == ADST_BF16 || dtype == ADST_F16 ? 4 : 8; }
int type_size(int32_t dtype) { return dtype == ADST_F64 ? 8 : dtype == ADST_F32 ? 4 : 2; }

Grid grid_of(int32_t dtype, int64_t B, int64_t T, int64_t D) {
  const int C = kLanes * 16 / type_size(dtype);
  Grid g;
  g.slabs = (int)((D + C - 1) / C);
  g.chains = (uint32_t)(B * g.slabs);
  g.threads = 512;
  if (T <= 64 / kLanes * type_steps(dtype)) g.threads = 64;
  g.span = g.threads / kLanes * type_steps(dtype);
  g.spans = T > 0 ? (int)((T + g.span - 1) / g.span) : 1;
  return g;
}

int64_t round16(int64_t n) { return (n + 15) / 16 * 16; }

Board board_of(int32_t dtype, const Grid& g, void* ws, int64_t* bytes) {
  const int64_t C = kLanes * 16 / type_size(dtype), A = dtype == ADST_F64 ? 8 : 4;
  const int64_t counters = (int64_t)g.chains * kCounterInts * 4;
  const int64_t words = round16((int64_t)g.chains * g.spans * C * A);
  char* p = static_cast<char*>(ws);
  *bytes = g.spans > 1 ? counters + 3 * words : 0;
  return {reinterpret_cast<int32_t*>(p), p + counters, p + counters + words};
}

template <class F>
void by_type(int32_t dtype, F f) {
  switch (dtype) {
    case ADST_F64: f(double()); break;
    case ADST_F32: f(float()); break;
    case ADST_BF16: f(bf16()); break;
    default: f(f16()); break;
  }
}

template <bool FORWARD, class T, bool SIG, bool MULTI, int NT>
void launch(const RecArgs& q, const Grid& g, const Board& bd, hipStream_t st) {
  const unsigned blocks = (unsigned)(g.chains * g.spans);
  if (FORWARD) rec_fwd<T, SIG, MULTI, NT><<<blocks, NT, 0, st>>>(q, g, bd);
  else rec_rev<T, SIG, MULTI, NT><<<blocks, NT, 0, st>>>(q, g, bd);
}
template <bool FORWARD, class T, bool SIG>
void by_grid(const RecArgs& q, const Grid& g, const Board& bd, hipStream_t st) {
  if (g.threads == 64)
    launch<FORWARD, T, SIG, false, 64>(q, g, bd, st);
  else if (g.spans == 1)
    launch<FORWARD, T, SIG, false, 512>(q, g, bd, st);
  else
    launch<FORWARD, T, SIG, true, 512>(q, g, bd, st);
}

template <bool FORWARD>
hipError_t sweep(const RecArgs& q, void* ws, hipStream_t st) {
  const Grid g = grid_of(q.dtype, q.B, q.T, q.D);
  int64_t bytes;
  const Board bd = board_of(q.dtype, g, ws, &bytes);
  if (bytes) {
    const int64_t n = bytes / 16;
    fill_ones<<<(unsigned)((n + kFillThreads - 1) / kFillThreads), kFillThreads, 0, st>>>(
        static_cast<uint4*>(ws), n);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  by_type(q.dtype, [&](auto t) {
    typedef decltype(t) T;
    if (q.gate == ADST_GATE_SIGMOID) by_grid<FORWARD, T, true>(q, g, bd, st);
    else by_grid<FORWARD, T, false>(q, g, bd, st);
  });
  return hipGetLastError();
}

}  // namespace

RecPlan rec_plan(int32_t dtype, int64_t B, int64_t T, int64_t D) {
  const Grid g = grid_of(dtype, B, T, D);
  RecPlan p;
  p.span = g.span;
  p.spans = g.spans;
  p.ck_bytes = (uint64_t)(B * D * g.spans) * (dtype == ADST_F64 ? 8 : 4);
  int64_t bytes;
  board_of(dtype, g, nullptr, &bytes);
  p.ws_bytes = (uint64_t)bytes;
  // work-items of a launch, and of the step's, in the 32-bit dispatch grid
  const int64_t per_row = (D + 16 / type_size(dtype) - 1) / (16 / type_size(dtype));
  p.fits = (double)B * g.slabs * g.spans * g.threads < 4294967296.0 &&
           (double)B * per_row < 4294967296.0 - 64 && bytes / 16 < (int64_t(1) << 32) - 256;
  return p;
}

hipError_t rec_forward(const RecArgs& q, void* ws, hipStream_t st) {
  return sweep<true>(q, ws, st);
}

hipError_t rec_vjp(const RecArgs& q, void* ws, hipStream_t st) { return sweep<false>(q, ws, st); }

hipError_t rec_step(const RecStep& q, hipStream_t st) {
  by_type(q.dtype, [&](auto t) {
    typedef decltype(t) T;
    const int64_t per_row = (q.D + Vec<T>::N - 1) / Vec<T>::N;
    const unsigned blocks = (unsigned)((q.B * per_row + kStepThreads - 1) / kStepThreads);
    if (q.gate == ADST_GATE_SIGMOID) rec_one<T, true><<<blocks, kStepThreads, 0, st>>>(q, per_row);
    else rec_one<T, false><<<blocks, kStepThreads, 0, st>>>(q, per_row);
  });
  return hipGetLastError();
}

}  // namespace adst
