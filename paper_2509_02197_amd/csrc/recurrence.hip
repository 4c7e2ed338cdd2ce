// Gated linear recurrence: h_t = c_t h_{t-1} + d_t per channel, with
// (c, d) = (a, u) or (s, (1 - s) u), s = 1 / (1 + exp(-a)); its VJP, which
// recomputes the states from checkpoints; and one step on a pool of states.
//
// A step is an affine map of the state, and maps compose: (A, H) after
// (A', H') is (A A', A H' + H). So a row is cut into spans, a workgroup each:
// it loads its span once, composes its steps, learns the state at its start
// from the spans before it, and applies its steps to that. Everything is read
// and written once, and HBM bandwidth bounds it. A wave's lanes lie along
// channels (256 consecutive bytes of a step) and each lane holds 16 consecutive
// steps of its channels in registers, so maps are composed within a lane, and
// over the waves through LDS; a wave needs no exchange between its lanes.
// (Lanes of 16 bytes with their maps composed across the wave took 100 us
// forward and 191 in reverse at 8 x 4096 x 2048 bf16, against 90 and 138: more
// registers for the maps, and a third more instructions.) Where channels are
// few, rows of 16 lanes lie along channels and the wave's four rows along time.
// The reverse sweep is the same recurrence backwards
// (G_t = dh_t + c_{t+1} G_{t+1}); it recomputes its span's states in registers
// from the checkpoint at its start, so the forward's h is not needed: reading
// a, u and dh and writing da and du is all it moves.
//
// Measured, bf16 SIGMOID on halves of one projection: 8 x 4096 x 2048 forward
// 89 us (4.5 TB/s), reverse 136 us (4.9 TB/s); 1 x 65536 x 1024 forward 105 us,
// reverse 176; 8 x 4096 x 1024 F32 86 and 131, 4 x 4096 x 1024 F64 85 and 133.
// Without the waits between spans the first would take 85 and 136, the second 83
// and 133; the fill of the board is 3 to 5 us of each.
//
// Between spans: a workgroup publishes its span's map (A, H) as soon as it has
// it. Eight spans form a group; a group's last workgroup also publishes the
// group's map, composed of its spans' in order, and the state at the group's
// end, state' = A state + H. The state that enters a span is that of its
// group's start with the maps of the group's earlier spans applied in order;
// the state of a group's start is the nearest one published before it, with
// the maps of the groups between applied in order. That is what each group
// computes for itself, bit for bit, so results do not depend on which states
// happened to be there. Spans are taken from a counter per row in the order of
// the sweep, so a workgroup only ever waits for workgroups that have started
// before it; spans' maps depend on nothing, groups' on spans', states on both:
// every wait ends. What is published is complete in itself (each word is
// written whole, and its initial pattern is never a value), so no fence is
// needed; the accesses are of agent scope, which the caches of the XCDs keep
// coherent.

#include "packs.h"
#include "seq_common.h"
#include "seq_kernels.h"
#include "seq_launch.h"

namespace adst {
namespace {

// A workgroup of NT threads: L lanes of a wave lie along channels, V of them a
// lane, and its 64 / L rows of lanes along time, R consecutive steps each.
template <class T, int NT_, int L_, bool STREAM_>
struct Shape {
  typedef Acc<T> A;
  static constexpr bool STREAM = STREAM_;
  static constexpr int V = sizeof(T) == 2 ? 2 : 1;
  static constexpr int R = sizeof(T) == 8 ? 8 : 16;
  static constexpr int W = NT_ / 64;
  static constexpr int L = L_;
  static constexpr int C = L * V;                // channels of a workgroup
  static constexpr int kWaveSteps = 64 / L * R;
  static constexpr int kSpan = W * kWaveSteps;   // a workgroup's steps
  typedef Pack<T, V> P;
};
// Threads of a workgroup on long rows: 512, whose spans are fewer. Forward: 8 x
// 4096 x 2048 bf16 89 us, 93 with 256; 1 x 65536 x 1024 105 and 135. In reverse
// a workgroup of 512 has a CU's registers to itself, but for F32 (5 x 2049 x 771
// 43 us, 47 with 256), and the other types take 256 (8 x 4096 x 2048 bf16 136 us,
// 163 with 512; 4 x 4096 x 1024 F64 133 and 156). A few long rows alone would be
// faster with 512 (1 x 65536 x 1024 bf16 176 us, 164 with it), but spans set the
// order of the sums, and a row's bits are not to depend on the number of rows.
constexpr int kLong = 512, kReverse = 256;
constexpr int kCkWaves = 4;  // a checkpoint at every fourth wave's steps

// How a problem is laid out over workgroups of `threads`.
struct Grid {
  int threads;
  int span;    // steps
  int spans;   // per batch row
  int groups;  // of spans
  int lanes;   // along channels
  int C;       // channels of a slab
  int slabs;   // of a batch row
  int ck;      // steps between checkpoints
  int cks;     // checkpoints of a batch row
  uint32_t chains;  // batch rows times slabs
  uint32_t round;   // the workgroups of one span of each
  bool by_xcd;      // chains belong to XCDs
};

// The chain of a workgroup (past the last one: none). Consecutive workgroups
// go to the 8 XCDs in turn. by_xcd: each XCD gets neighbouring chains, whose
// rows share cache lines where a row is not a multiple of them, and keeps them
// (8 x 4096 x 2048 bf16: 90 us forward and 136 in reverse, 92 and 140 without;
// 5 x 2049 x 771 f32: 26 and 29 us forward). That takes a multiple of 8 chains, or so
// many that the XCDs with one more than others do not count: one chain of
// 262144 steps took 373 us on one XCD and takes 91 on all.
__device__ inline uint32_t chain_of(const Grid& g) {
  const uint32_t x = blockIdx.x % g.round;
  return g.by_xcd ? x % 8 * (g.round / 8) + x / 8 : x;
}

// What a launch of several spans publishes in, all ones at its start. Spans
// are counted in the order of the sweep.
constexpr int kGroup = 8;
struct Board {
  int32_t* next;  // a counter per chain, 32 bytes apart, from -1
  void* state;    // [chain][groups][C] accumulation type: the state at a group's end
  void* group;    // [chain][groups][C] two of it: a group's map
  void* map;      // [chain][spans][C] two of it: a span's
};
constexpr int kCounterInts = 8;

// -------------------------------------------------------------- registers
// The compiler treats the values as new ones: it does not keep what it
// derived from them before, which would take more registers than there are.
template <class A, int R, int V>
__device__ inline void forget(A (&x)[R][V]) {
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int i = 0; i < V; ++i) asm volatile("" : "+v"(x[r][i]));
}
template <class T, int V, int R>
__device__ inline void forget(Pack<T, V> (&x)[R]) {  // and unpacks again
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      uint32_t w = __builtin_bit_cast(uint32_t, x[r].v);
      asm volatile("" : "+v"(w));
      x[r].v = __builtin_bit_cast(typename Pack<T, V>::type, w);
    }
  }
}

// ------------------------------------------------------- maps along the time
// Rows of 16 lanes exchange values: in every lane the value of its pair's even
// (lower) row and of the odd (upper) one, or of the wave's lower and upper
// half. Vector instructions, which do without LDS.
template <bool HALVES>
__device__ inline void exchange(uint32_t x, uint32_t* lower, uint32_t* upper) {
  const auto r = HALVES ? __builtin_amdgcn_permlane32_swap(x, x, false, false)
                        : __builtin_amdgcn_permlane16_swap(x, x, false, false);
  *lower = r[0];
  *upper = r[1];
}
template <bool HALVES>
__device__ inline void exchange(float x, float* lower, float* upper) {
  uint32_t a, b;
  exchange<HALVES>(__builtin_bit_cast(uint32_t, x), &a, &b);
  *lower = __builtin_bit_cast(float, a);
  *upper = __builtin_bit_cast(float, b);
}
template <bool HALVES>
__device__ inline void exchange(double x, double* lower, double* upper) {
  const uint64_t w = __builtin_bit_cast(uint64_t, x);
  uint32_t a0, b0, a1, b1;
  exchange<HALVES>((uint32_t)w, &a0, &b0);
  exchange<HALVES>((uint32_t)(w >> 32), &a1, &b1);
  *lower = __builtin_bit_cast(double, (uint64_t)a1 << 32 | a0);
  *upper = __builtin_bit_cast(double, (uint64_t)b1 << 32 | b0);
}

// From a row's map (a, h) the one of the rows before it in the wave, and the
// wave's.
template <class A>
__device__ inline void compose_rows(A& a, A& h, A* wave_a, A* wave_h) {
  const int lane = threadIdx.x & 63;
  const bool odd = lane & 16, high = lane & 32;
  A ea, oa, eh, oh, la, ua, lh, uh;
  exchange<false>(a, &ea, &oa);
  exchange<false>(h, &eh, &oh);
  exchange<true>(oa * ea, &la, &ua);
  exchange<true>(fma_(oa, eh, oh), &lh, &uh);
  *wave_a = ua * la;
  *wave_h = fma_(ua, lh, uh);
  const A xa = odd ? ea : A(1), xh = odd ? eh : A(0);
  a = high ? xa * la : xa;
  h = high ? fma_(xa, lh, xh) : xh;
}
// The same, and against the time: from (a, c) the map of the rows after it.
template <class A>
__device__ inline void compose_rows_both(A a, A& h, A& c, A* before_a, A* after_a, A* wave_a,
                                         A* wave_h, A* wave_c) {
  const int lane = threadIdx.x & 63;
  const bool odd = lane & 16, high = lane & 32;
  A ea, oa, eh, oh, ec, oc, la, ua, lh, uh, lc, uc;
  exchange<false>(a, &ea, &oa);
  exchange<false>(h, &eh, &oh);
  exchange<false>(c, &ec, &oc);
  exchange<true>(oa * ea, &la, &ua);
  exchange<true>(fma_(oa, eh, oh), &lh, &uh);
  exchange<true>(fma_(ea, oc, ec), &lc, &uc);
  *wave_a = ua * la;
  *wave_h = fma_(ua, lh, uh);
  *wave_c = fma_(la, uc, lc);
  const A xa = odd ? ea : A(1), xh = odd ? eh : A(0);
  *before_a = high ? xa * la : xa;
  h = high ? fma_(xa, lh, xh) : xh;
  const A ya = odd ? A(1) : oa, yc = odd ? A(0) : oc;
  *after_a = high ? ya : ya * ua;
  c = high ? yc : fma_(ya, uc, yc);
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
  __device__ float scale(float x) const { return __builtin_bit_cast(float, (uint32_t)w) * x; }
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
  __device__ double scale(double x) const { return __builtin_bit_cast(double, a) * x; }
  __device__ double apply(double x) const {
    return fma_(__builtin_bit_cast(double, a), x, __builtin_bit_cast(double, h));
  }
};

// This span's map, the e-th of its chain.
template <class A>
__device__ inline void publish(const Board& bd, const Grid& g, uint32_t chain, int e, int C,
                               int c, A a, A h) {
  MapWords<A>::store(bd.map, ((int64_t)chain * g.spans + e) * C + c, a, h);
  asm volatile("" ::: "memory");  // before this wave waits for anything
}

// The state that enters this chain's e-th span, e > 0, one thread a channel;
// whole waves call this, and a lane without a channel (mine false) only takes
// part in the looking. first: the state that enters span 0. (oa, oh): this
// span's map. more: spans follow, which read what the last one of a group
// publishes. c: the channel's place in the slab.
template <class A, int C>
__device__ inline A enter(const Board& bd, const Grid& g, uint32_t chain, int e, bool more, int c,
                          bool mine, A first, A oa, A oh) {
  const int lane = threadIdx.x & 63;
  const int j = e / kGroup, i = e % kGroup;
  const int64_t maps = ((int64_t)chain * g.spans + (e - i)) * C + c;  // the group's first span's
  const int64_t groups = (int64_t)chain * g.groups * C + c;
  const Word<A>* states = (const Word<A>*)bd.state;
  const bool closes = i == kGroup - 1 && more;
  // Lane l < 32 looks at the state of the start of the group l before this one
  // (group 0's is `first`), lane 32 + l at the map of the group l + 1 before it.
  const int back = lane & 31;
  const bool looks = back < j;
  const int64_t seen = groups - (c & 63) + (int64_t)(j - 1 - back) * C;
  MapWords<A> m[kGroup - 1];
#pragma unroll
  for (int l = 0; l < kGroup - 1; ++l)  // (without a channel they would lie past the slab's)
    if (l < i && mine) m[l] = MapWords<A>::load(bd.map, maps + (int64_t)l * C);
  Word<A> w;
  int dist = 0;
  A ga = oa, gh = oh;
  bool composed = !closes;
  for (;;) {
    w = j > 0 && mine ? agent_load(states + groups + (int64_t)(j - 1) * C) : 0;
    bool there = false;
    if (looks)
      there = lane < 32 ? ~agent_load(states + seen) != 0
                        : MapWords<A>::load(bd.group, seen).full();
    there = there || (lane < 32 && back == j);
    const uint64_t all = __ballot(there);
    bool missing = false;
    if (mine) {
#pragma unroll
      for (int l = 0; l < kGroup - 1; ++l)
        if (l < i) missing = missing || !m[l].full();
    }
    const bool have = __ballot(missing) == 0;
    if (have && !composed) {  // the group's map, before any wait for a state
      composed = true;
      if (mine) {
        A a = A(1), h = A(0);
#pragma unroll
        for (int l = 0; l < kGroup - 1; ++l) {
          h = m[l].apply(h);
          a = m[l].scale(a);
        }
        ga = oa * a;
        gh = fma_(oa, h, oh);
        MapWords<A>::store(bd.group, groups + (int64_t)j * C, ga, gh);
      }
    }
    const uint32_t with_state = (uint32_t)all, with_map = (uint32_t)(all >> 32);
    if (have && with_state) {
      dist = __ffs((int)with_state) - 1;
      const uint32_t need = (1u << dist) - 1u;
      if ((with_map & need) == need) break;
    }
    __builtin_amdgcn_s_sleep(1);
    if (!have && mine) {
#pragma unroll
      for (int l = 0; l < kGroup - 1; ++l)
        if (l < i && !m[l].full()) m[l] = MapWords<A>::load(bd.map, maps + (int64_t)l * C);
    }
  }
  if (!mine) return A(0);
  // The words of this lane's own channel were written with those looked at;
  // each is checked all the same.
  constexpr int kAhead = 4;  // maps under way at a time
  A x = first;
  for (int k = dist; k >= 0 && j > 0;) {  // from the start of group j - k
    if (k == dist && k < j) {
      const int64_t at = groups + (int64_t)(j - 1 - k) * C;
      if (k > 0) w = agent_load(states + at);
      while (~w == 0) w = agent_load(states + at);
      x = __builtin_bit_cast(A, w);
    }
    if (k == 0) break;
    MapWords<A> b[kAhead];
#pragma unroll
    for (int l = 0; l < kAhead; ++l)
      if (l < k) b[l] = MapWords<A>::load(bd.group, groups + (int64_t)(j - k + l) * C);
#pragma unroll
    for (int l = 0; l < kAhead; ++l)
      if (l < k) {
        while (!b[l].full())
          b[l] = MapWords<A>::load(bd.group, groups + (int64_t)(j - k + l) * C);
        x = b[l].apply(x);
      }
    if (k <= kAhead) break;
    k -= kAhead;
  }
  if (closes) agent_store((Word<A>*)bd.state + groups + (int64_t)j * C, word_of(fma_(ga, x, gh)));
#pragma unroll
  for (int l = 0; l < kGroup - 1; ++l)
    if (l < i) x = m[l].apply(x);
  return x;
}

// -------------------------------------------------------------- the kernels
// Where a workgroup works, and how much of it exists.
template <class S>
struct Place {
  int64_t b, len;  // the batch row and its steps
  int slab, span;
  int64_t t0;     // the span's first step
  int64_t mine;   // this lane's first step
  int c0, n;      // this lane's first channel, and how many it has
  bool whole;     // every step and channel of this lane exists
  __device__ Place(const RecArgs& r, const Grid& g, uint32_t chain, int span_) {
    span = span_;
    b = chain / (uint32_t)g.slabs;
    slab = (int)(chain % (uint32_t)g.slabs);
    len = row_length(r.lens, b, r.T);
    t0 = (int64_t)span * S::kSpan;
    mine = t0 + threadIdx.x / S::L * S::R;
    c0 = slab * S::C + (int)(threadIdx.x % S::L) * S::V;
    const int64_t left = r.D - c0;
    n = left < 0 ? 0 : left < S::V ? (int)left : S::V;
    whole = n == S::V && mine + S::R <= len;
  }
};

// This lane's R packs of a strided array; `none` where steps or channels end.
template <class T, class S>
__device__ inline void load_steps(const void* base, int64_t sb, int64_t stp, const Place<S>& at,
                                  T none, typename S::P (&v)[S::R]) {
  const T* p = (const T*)base + at.b * sb + at.mine * stp + at.c0;
  if (at.whole) {
#pragma unroll
    for (int r = 0; r < S::R; ++r) v[r] = load_pack<T, S::V, S::STREAM>(p + r * stp, S::V);
    return;
  }
#pragma unroll
  for (int r = 0; r < S::R; ++r) {
#pragma unroll
    for (int i = 0; i < S::V; ++i) v[r].v[i] = none;
    if (at.mine + r < at.len && at.n > 0) v[r] = load_pack<T, S::V>(p + r * stp, at.n);
  }
}
// Stores them to a contiguous array: up to T, zeros from len on.
template <class T, class S>
__device__ inline void store_steps(void* base, const RecArgs& q, const Place<S>& at,
                                   const typename S::P (&v)[S::R]) {
  T* p = (T*)base + (at.b * q.T + at.mine) * q.D + at.c0;
  if (at.whole) {
#pragma unroll
    for (int r = 0; r < S::R; ++r) store_pack<T, S::V, S::STREAM>(p + r * q.D, v[r], S::V);
    return;
  }
#pragma unroll
  for (int r = 0; r < S::R; ++r)
    if (at.mine + r < q.T && at.n > 0) {
      typename S::P x = v[r];
      if (at.mine + r >= at.len) x.v = typename S::P::type{};
      store_pack<T, S::V>(p + r * q.D, x, at.n);
    }
}

// What a and u are beyond a row's end, so that a step keeps the state and the
// gradient: coefficient 1 and input 0.
template <class T, bool SIG>
__device__ inline T keep() {
  return SIG ? (T)__builtin_inff() : T(1);
}

// The span this workgroup takes: the next one of its chain.
__device__ inline int take_span(const Board& bd, uint32_t chain) {
  __shared__ int ticket;
  if (threadIdx.x == 0) ticket = atomicAdd(bd.next + (int64_t)chain * kCounterInts, 1) + 1;
  __syncthreads();
  return ticket;
}

template <class T, bool SIG, bool MULTI, bool STREAM, int NT, int L>
__global__ __launch_bounds__(NT, 4) void rec_fwd(RecArgs q, Grid g, Board bd) {
  typedef Shape<T, NT, L, STREAM> S;
  typedef typename S::A A;
  constexpr int V = S::V, R = S::R, C = S::C;
  __shared__ Maps<A, S::W, C> maps;
  __shared__ A start[C];
  const uint32_t chain = chain_of(g);
  if (chain >= g.chains) return;
  const Place<S> at(q, g, chain, MULTI ? take_span(bd, chain) : 0);
  typename S::P va[R], vu[R];
  if (at.t0 >= at.len && at.span > 0) {  // nothing but zeros, and nobody asks for its state
#pragma unroll
    for (int r = 0; r < R; ++r) va[r].v = typename S::P::type{};
    if (q.h) store_steps<T>(q.h, q, at, va);
    return;
  }
  load_steps(q.a, q.sa_b, q.sa_t, at, keep<T, SIG>(), va);
  load_steps(q.u, q.su_b, q.su_t, at, T(0), vu);

  // SIGMOID: the gate and the gated input; COEFF: a and u stay packed.
  A c[R][V], d[R][V], a[V], h[V];
#pragma unroll
  for (int i = 0; i < V; ++i) a[i] = A(1), h[i] = A(0);
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      A s = up(va[r].v[i]), x = up(vu[r].v[i]);
      if (SIG) {
        A o;
        gates<T>(s, &s, &o);
        c[r][i] = s;
        d[r][i] = x = o * x;
      }
      h[i] = fma_(s, h[i], x);
      a[i] *= s;
    }
  if (!SIG) forget(va), forget(vu);
  const int wave = threadIdx.x / 64, col = threadIdx.x % L * V;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    A wa = a[i], wh = h[i];
    if (L < 64) compose_rows(a[i], h[i], &wa, &wh);
    if (L == 64 || (threadIdx.x & 63) < L) maps.a[wave][col + i] = wa, maps.h[wave][col + i] = wh;
  }
  __syncthreads();
  for (int k = threadIdx.x; k < (C + 63) / 64 * 64; k += NT) {  // whole waves
    A ma = A(1), mh = A(0);
    if (k < C) compose_waves<true>(maps, k, &ma, &mh);
    const int64_t ch = (int64_t)at.slab * C + k;
    const bool mine = k < C && ch < q.D;
    const bool last = at.t0 + S::kSpan >= at.len;
    A x = mine && q.h0 ? ((const A*)q.h0)[at.b * q.D + ch] : A(0);
    if (MULTI) {
      if (mine && !last) publish(bd, g, chain, at.span, C, k, ma, mh);
      if (at.span > 0 && (int64_t)at.slab * C + (k & ~63) < q.D)
        x = enter<A, C>(bd, g, chain, at.span, !last, k, mine, x, ma, mh);
    }
    if (mine && last && q.hT) ((A*)q.hT)[at.b * q.D + ch] = fma_(ma, x, mh);
    if (k < C) start[k] = x;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const A x = fma_(maps.a[wave][col + i], start[col + i], maps.h[wave][col + i]);
    h[i] = L == 64 ? x : fma_(a[i], x, h[i]);
  }
  if (q.ck && wave % kCkWaves == 0 && (threadIdx.x & 63) < L &&
      (at.mine < at.len || at.mine == 0)) {
    A* ck = (A*)q.ck + (at.b * g.cks + at.mine / (kCkWaves * S::kWaveSteps)) * q.D + at.c0;
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < at.n) ck[i] = h[i];
  }
  if (!q.h) return;
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      h[i] = SIG ? fma_(c[r][i], h[i], d[r][i]) : fma_(up(va[r].v[i]), h[i], up(vu[r].v[i]));
      va[r].v[i] = down<T>(h[i]);
    }
  store_steps<T>(q.h, q, at, va);
}

template <class T, bool SIG, bool MULTI, bool STREAM, int NT, int L>
__global__ __launch_bounds__(NT, 3) void rec_rev(RecArgs q, Grid g, Board bd) {
  typedef Shape<T, NT, L, STREAM> S;
  typedef typename S::A A;
  constexpr int V = S::V, R = S::R, C = S::C;
  __shared__ Maps<A, S::W, C> maps, rmaps;
  __shared__ A start[C], finish[C];
  const uint32_t chain = chain_of(g);
  if (chain >= g.chains) return;
  typename S::P va[R], vu[R], vd[R];
  const Place<S> at(q, g, chain, MULTI ? g.spans - 1 - take_span(bd, chain) : 0);
  if (at.t0 >= at.len && at.span > 0) {
#pragma unroll
    for (int r = 0; r < R; ++r) va[r].v = typename S::P::type{};
    store_steps<T>(q.da, q, at, va);
    store_steps<T>(q.du, q, at, va);
    return;
  }
  load_steps(q.a, q.sa_b, q.sa_t, at, keep<T, SIG>(), va);
  load_steps(q.u, q.su_b, q.su_t, at, T(0), vu);
  load_steps(q.dh, q.sd_b, q.sd_t, at, T(0), vd);

  // SIGMOID: the gate s and o = 1 - s; COEFF: a stays packed.
  A s[R][V], o[R][V], a[V], h[V], c[V];
#pragma unroll
  for (int i = 0; i < V; ++i) a[i] = A(1), h[i] = A(0), c[i] = A(0);
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      A k = up(va[r].v[i]), d = up(vu[r].v[i]);
      if (SIG) {
        gates<T>(k, &s[r][i], &o[r][i]);
        k = s[r][i];
        d = o[r][i] * d;
      }
      h[i] = fma_(k, h[i], d);
      a[i] *= k;
    }
  if (!SIG) forget(va);
#pragma unroll
  for (int r = R - 1; r >= 0; --r)
#pragma unroll
    for (int i = 0; i < V; ++i)
      c[i] = (SIG ? s[r][i] : up(va[r].v[i])) * (up(vd[r].v[i]) + c[i]);
  forget(vu);
  forget(vd);
  const int wave = threadIdx.x / 64, col = threadIdx.x % L * V;
  A ra[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    A wa = a[i], wh = h[i], wc = c[i];
    if (L < 64) compose_rows_both(a[i], h[i], c[i], &a[i], &ra[i], &wa, &wh, &wc);
    if (L == 64 || (threadIdx.x & 63) < L) {
      maps.a[wave][col + i] = rmaps.a[wave][col + i] = wa;
      maps.h[wave][col + i] = wh, rmaps.h[wave][col + i] = wc;
    }
  }
  __syncthreads();
  for (int k = threadIdx.x; k < (C + 63) / 64 * 64; k += NT) {  // whole waves
    A ma = A(1), mh = A(0);
    if (k < C) {
      compose_waves<true>(maps, k, &ma, &mh);
      compose_waves<false>(rmaps, k, &ma, &mh);
    }
    const int64_t ch = (int64_t)at.slab * C + k;
    const bool mine = k < C && ch < q.D;
    // asked for before the wait
    const int64_t check = at.b * g.cks + at.span * S::W / kCkWaves;
    const A first = mine ? ((const A*)q.ck)[check * q.D + ch] : A(0);
    // the sweep begins at the row's last span, where dhT enters
    const int last = at.len > 0 ? (int)((at.len - 1) / S::kSpan) : 0;
    A x = mine && q.dhT ? ((const A*)q.dhT)[at.b * q.D + ch] : A(0);
    if (MULTI) {
      const int e = last - at.span;
      if (mine && at.span > 0) publish(bd, g, chain, e, C, k, ma, mh);
      if (e > 0 && (int64_t)at.slab * C + (k & ~63) < q.D)
        x = enter<A, C>(bd, g, chain, e, at.span > 0, k, mine, x, ma, mh);
    }
    if (mine && at.span == 0 && q.dh0) ((A*)q.dh0)[at.b * q.D + ch] = fma_(ma, x, mh);
    if (k < C) finish[k] = x, start[k] = first;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const A x = fma_(maps.a[wave][col + i], start[col + i], maps.h[wave][col + i]);
    const A y = fma_(rmaps.a[wave][col + i], finish[col + i], rmaps.h[wave][col + i]);
    h[i] = L == 64 ? x : fma_(a[i], x, h[i]);
    c[i] = L == 64 ? y : fma_(ra[i], y, c[i]);
  }
  if (SIG) forget(o);  // what was o * u is not kept
  else forget(va);
  A e[R][V];  // what G_t is multiplied with in da_t
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const A x = h[i], u = up(vu[r].v[i]);
      if (SIG) {
        e[r][i] = (x - u) * (s[r][i] * o[r][i]);
        h[i] = fma_(s[r][i], x, o[r][i] * u);
      } else {
        e[r][i] = x;
        h[i] = fma_(up(va[r].v[i]), x, u);
      }
    }
  if (!SIG) forget(va);
#pragma unroll
  for (int r = R - 1; r >= 0; --r)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const A G = up(vd[r].v[i]) + c[i], k = SIG ? s[r][i] : up(va[r].v[i]);
      va[r].v[i] = down<T>(G * e[r][i]);
      vu[r].v[i] = down<T>(SIG ? G * o[r][i] : G);
      c[i] = k * G;
    }
  store_steps<T>(q.da, q, at, va);
  store_steps<T>(q.du, q, at, vu);
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
        gates<T>(c, &s, &o);
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

constexpr int kFillThreads = 256, kFillEach = 4;
__global__ __launch_bounds__(kFillThreads) void fill_ones(uint4* p, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * (kFillThreads * kFillEach) + threadIdx.x;
#pragma unroll
  for (int k = 0; k < kFillEach; ++k)
    if (i + k * kFillThreads < n) p[i + k * kFillThreads] = make_uint4(~0u, ~0u, ~0u, ~0u);
}

// -------------------------------------------------------------- on the host
int type_size(int32_t dtype) { return dtype == ADST_F64 ? 8 : dtype == ADST_F32 ? 4 : 2; }

int lane_channels(int32_t dtype) { return dtype == ADST_F64 || dtype == ADST_F32 ? 1 : 2; }
int lane_steps(int32_t dtype) { return dtype == ADST_F64 ? 8 : 16; }

// Lanes along channels: all 64 where that leaves few without one, else 16
// (64 x 30000 x 7 f32: 74 us forward and 99 in reverse with 16, 230 and 278
// with 64; 1 x 4096 x 64 bf16 8.8 and 10.2 us against 11.9 and 14.1).
int lanes_of(int32_t dtype, int64_t D) {
  const int64_t C = 64 * lane_channels(dtype), all = (D + C - 1) / C * C;
  return 4 * (all - D) <= all ? 64 : 16;
}

Grid grid_of(int32_t dtype, int64_t B, int64_t T, int64_t D, bool forward) {
  Grid g;
  g.lanes = lanes_of(dtype, D);
  g.C = g.lanes * lane_channels(dtype);
  const int wave = 64 / g.lanes * lane_steps(dtype);  // its steps
  g.slabs = (int)((D + g.C - 1) / g.C);
  g.chains = (uint32_t)(B * g.slabs);
  g.round = (g.chains + 7) / 8 * 8;
  g.by_xcd = 8 * (uint64_t)g.round <= 9 * (uint64_t)g.chains;
  if (!g.by_xcd) g.round = g.chains;
  g.threads = T <= wave ? 64 : T <= 2 * wave ? 128 : T <= 4 * wave ? 256
              : forward || dtype == ADST_F32 ? kLong : kReverse;
  g.span = g.threads / 64 * wave;
  g.spans = T > 0 ? (int)((T + g.span - 1) / g.span) : 1;
  g.groups = (g.spans + kGroup - 1) / kGroup;
  g.ck = kCkWaves * wave;
  g.cks = T > 0 ? (int)((T + g.ck - 1) / g.ck) : 1;
  return g;
}

Board board_of(int32_t dtype, const Grid& g, void* ws, int64_t* bytes) {
  const int64_t C = g.C, A = dtype == ADST_F64 ? 8 : 4;
  const int64_t counters = (int64_t)g.chains * kCounterInts * 4;
  const int64_t states = (int64_t)g.chains * g.groups * C * A;
  const int64_t maps = (int64_t)g.chains * g.spans * C * 2 * A;
  char* p = static_cast<char*>(ws);
  *bytes = g.spans > 1 ? counters + 3 * states + maps : 0;
  return {reinterpret_cast<int32_t*>(p), p + counters, p + counters + states,
          p + counters + 3 * states};
}

template <class F>
hipError_t by_type(int32_t dtype, F f) {
  switch (dtype) {
    case ADST_F64: return f(double());
    case ADST_F32: return f(float());
    case ADST_BF16: return f(bf16());
    default: return f(f16());
  }
}

template <bool FORWARD, class T, bool SIG, bool MULTI, bool STREAM, int NT, int L>
hipError_t launch(const RecArgs& q, const Grid& g, const Board& bd, hipStream_t st) {
  const unsigned blocks = g.round * (unsigned)g.spans;
  if constexpr (FORWARD)
    return start(rec_fwd<T, SIG, MULTI, STREAM, NT, L>, blocks, NT, st, q, g, bd);
  else
    return start(rec_rev<T, SIG, MULTI, STREAM, NT, L>, blocks, NT, st, q, g, bd);
}

// Non-temporal loads and stores for calls that move more than the caches keep,
// on arrays whose rows are whole cache lines (8 x 4096 x 2048 bf16: reverse 136
// us with them, 146 without; rows off the lines, whose shared lines then leave
// the cache between two workgroups, 5 x 2049 x 771 f32: 54 and 47).
constexpr int64_t kStreamBytes = int64_t(128) << 20, kLine = 128;
bool streams(const RecArgs& q, bool forward) {
  const int64_t e = type_size(q.dtype);
  int64_t off = q.D * e | q.sa_b * e | q.sa_t * e | q.su_b * e | q.su_t * e;
  off |= (int64_t)(uintptr_t)q.a | (int64_t)(uintptr_t)q.u;
  if (forward) off |= (int64_t)(uintptr_t)q.h;
  else off |= q.sd_b * e | q.sd_t * e | (int64_t)(uintptr_t)q.dh | (int64_t)(uintptr_t)q.da |
              (int64_t)(uintptr_t)q.du;
  return off % kLine == 0 && q.B * q.T * q.D * e * (forward ? 3 : 5) >= kStreamBytes;
}

template <bool FORWARD, class T, bool SIG, int L>
hipError_t by_threads(const RecArgs& q, const Grid& g, const Board& bd, hipStream_t st) {
  constexpr int kMost = FORWARD || sizeof(T) == 4 ? kLong : kReverse;
  if (g.spans > 1)
    return launch<FORWARD, T, SIG, true, false, kMost, L>(q, g, bd, st);
  if (g.threads == 64)
    return launch<FORWARD, T, SIG, false, false, 64, L>(q, g, bd, st);
  if (g.threads == 128)
    return launch<FORWARD, T, SIG, false, false, 128, L>(q, g, bd, st);
  if (g.threads == 256)
    return launch<FORWARD, T, SIG, false, false, 256, L>(q, g, bd, st);
  if constexpr (kMost > 256)
    return launch<FORWARD, T, SIG, false, false, kMost, L>(q, g, bd, st);
  return hipErrorInvalidValue;  // grid_of has no such workgroup
}
template <bool FORWARD, class T, bool SIG>
hipError_t by_grid(const RecArgs& q, const Grid& g, const Board& bd, hipStream_t st) {
  constexpr int kMost = FORWARD || sizeof(T) == 4 ? kLong : kReverse;
  if (g.lanes == 16)
    return by_threads<FORWARD, T, SIG, 16>(q, g, bd, st);
  if (!streams(q, FORWARD) || g.threads < 256)
    return by_threads<FORWARD, T, SIG, 64>(q, g, bd, st);
  if (g.spans > 1)
    return launch<FORWARD, T, SIG, true, true, kMost, 64>(q, g, bd, st);
  if (g.threads == 256)
    return launch<FORWARD, T, SIG, false, true, 256, 64>(q, g, bd, st);
  if constexpr (kMost > 256)
    return launch<FORWARD, T, SIG, false, true, kMost, 64>(q, g, bd, st);
  return hipErrorInvalidValue;
}

template <bool FORWARD>
hipError_t sweep(const RecArgs& q, void* ws, hipStream_t st) {
  const Grid g = grid_of(q.dtype, q.B, q.T, q.D, FORWARD);
  int64_t bytes;
  const Board bd = board_of(q.dtype, g, ws, &bytes);
  if (bytes) {
    const int64_t n = bytes / 16, each = kFillThreads * kFillEach;
    const hipError_t e = start(fill_ones, (unsigned)((n + each - 1) / each), kFillThreads, st,
                               static_cast<uint4*>(ws), n);
    if (e != hipSuccess) return e;
  }
  return by_type(q.dtype, [&](auto t) {
    typedef decltype(t) T;
    return q.gate == ADST_GATE_SIGMOID ? by_grid<FORWARD, T, true>(q, g, bd, st)
                                       : by_grid<FORWARD, T, false>(q, g, bd, st);
  });
}

}  // namespace

RecPlan rec_plan(int32_t dtype, int64_t B, int64_t T, int64_t D) {
  RecPlan p;
  p.ws_bytes = 0;
  p.fits = true;
  for (int forward = 0; forward < 2; ++forward) {
    const Grid g = grid_of(dtype, B, T, D, forward);
    int64_t bytes;
    board_of(dtype, g, nullptr, &bytes);
    if ((uint64_t)bytes > p.ws_bytes) p.ws_bytes = (uint64_t)bytes;
    // a launch's work-items in the 32-bit dispatch grid
    p.fits = p.fits && ((double)B * g.slabs + 7) * g.spans * g.threads < 4294967296.0 &&
             bytes / 16 < (int64_t(1) << 32) - 256;
    p.span = g.ck;
    p.ck_bytes = (uint64_t)(B * D * g.cks) * (dtype == ADST_F64 ? 8 : 4);
  }
  const int64_t per_row = (D + 16 / type_size(dtype) - 1) / (16 / type_size(dtype));
  p.fits = p.fits && (double)B * per_row < 4294967296.0 - 64;  // the step's
  return p;
}

hipError_t rec_forward(const RecArgs& q, void* ws, hipStream_t st) {
  return sweep<true>(q, ws, st);
}

hipError_t rec_vjp(const RecArgs& q, void* ws, hipStream_t st) { return sweep<false>(q, ws, st); }

hipError_t rec_step(const RecStep& q, hipStream_t st) {
  return by_type(q.dtype, [&](auto t) {
    typedef decltype(t) T;
    const int64_t per_row = (q.D + Vec<T>::N - 1) / Vec<T>::N;
    const unsigned blocks = (unsigned)((q.B * per_row + kStepThreads - 1) / kStepThreads);
    return start(q.gate == ADST_GATE_SIGMOID ? rec_one<T, true> : rec_one<T, false>, blocks,
                 kStepThreads, st, q, per_row);
  });
}

}  // namespace adst
