// Causal convolution of a few taps per channel, y_t = act(bias + sum_k w_k
// x_{t-K+1+k}); its VJP; and one step on a pool of windows.
//
// A thread takes V neighbouring channels of a segment of steps and keeps the
// last K-1 inputs in registers, so an input is loaded once but for the K-1
// before each segment. HBM bandwidth bounds it: one value read and one written.
// The VJP computes the sum before the activation again, as its derivative needs
// it: with g_t = dy_t act'(pre_t),
//   dx_t = sum_k w_k g_{t+K-1-k},  dw_k = sum_t g_t x_{t-K+1+k},  db = sum_t g_t,
// so x and dy are read, dx is written, and dw and db are summed in registers over
// a thread's segments, over a workgroup through LDS, and over workgroups by a
// second kernel in an order that the sizes alone set.

#include "packs.h"
#include "seq_common.h"
#include "seq_launch.h"
#include "token_kernels.h"

namespace adst {
namespace {

constexpr int kThreads = 256;
constexpr int kBatch = 4;      // steps whose loads are in flight together
constexpr int kSegment = 32;   // steps of a thread, where there are enough threads
constexpr int kFewSegment = 8;
constexpr int64_t kManyThreads = 1 << 17;  // 8 waves a CU

template <int K>
struct Count {
  static constexpr int value = K;
};

// Channels of a thread. The forward has registers for three waves a SIMD or more with these (8 x
// 4096 x 2048 bf16 64 us with 4 channels, 67 with 8). The reverse has three up to 4 taps of 16
// bits, and two from 5 on (bf16 of 8 taps with SiLU one); F32 two at 3 and 4 taps, and above them
// three, with half the channels (8 x 4096 x 2048 with SiLU: 8 taps 246 us, 295 with 4 channels; 5
// taps 225 and 200); F64 two from 3 taps on and one from 6.
template <class T, int K>
constexpr int lanes_of(bool reverse) {
  return sizeof(T) == 8 || (sizeof(T) == 4 && reverse && K > 4) ? 2 : 4;
}

// A weight: of T, or of float beside 16-bit T.
template <class T>
__device__ inline Acc<T> weight(const void* w, bool same, int64_t i) {
  if (same) return up(static_cast<const T*>(w)[i]);
  return (Acc<T>)static_cast<const float*>(w)[i];
}

template <class T, int K, int V>
struct Taps {
  Acc<T> w[K][V], b[V];
  __device__ Taps(const ConvArgs& a, int64_t d0) {
    const bool same = a.wtype == a.dtype;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      b[i] = a.bias ? weight<T>(a.bias, same, d0 + i) : Acc<T>(0);
#pragma unroll
      for (int k = 0; k < K; ++k) w[k][i] = weight<T>(a.w, same, k * a.D + d0 + i);
    }
  }
};

// A thread's first channel. V channels are there at every thread: the last one of a row
// takes the row's last V, and computes what its neighbour does once more.
template <int V>
__device__ inline int64_t first_channel(int64_t c, int64_t D) {
  return c * V + V <= D ? c * V : D - V;
}
template <class T, int V>
__device__ inline Pack<T, V> zeros() {
  Pack<T, V> z;
#pragma unroll
  for (int i = 0; i < V; ++i) z.v[i] = T(0);
  return z;
}

// Input t of a row, those of the window before it where t < 0 (t >= 1 - K).
template <class T, int V>
__device__ inline Pack<T, V> input(const ConvArgs& a, int64_t b, int64_t t, int64_t d0) {
  if (t >= 0) return load_pack<T, V>(static_cast<const T*>(a.x) + b * a.sx_b + t * a.sx_t + d0, V);
  if (a.x0)
    return load_pack<T, V>(
        static_cast<const T*>(a.x0) + (b * (a.taps - 1) + t + a.taps - 1) * a.D + d0, V);
  return zeros<T, V>();
}

// ------------------------------------------------------------------- forward
// A thread: V channels of one segment of a row; the last segment's index copies
// the window that follows the row.
template <class T, int K, int V, bool SILU>
__global__ __launch_bounds__(kThreads) void conv_fwd(ConvArgs a, int64_t nvec, int64_t segments,
                                                     int segment) {
  typedef Acc<T> A;
  constexpr int H = K > 1 ? K - 1 : 1;
  const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t c = id % nvec, rest = id / nvec;
  const int64_t b = rest / (segments + 1), s = rest % (segments + 1);
  if (b >= a.B) return;
  const int64_t d0 = first_channel<V>(c, a.D);
  const int64_t len = row_length(a.lens, b, a.T);
  if (s == segments) {
    if (a.xT)
      for (int j = 0; j < K - 1; ++j)
        store_pack<T, V>(static_cast<T*>(a.xT) + (b * (K - 1) + j) * a.D + d0,
                         input<T, V>(a, b, len + j - (K - 1), d0), V);
    return;
  }
  if (!a.y) return;
  const int64_t first = s * segment, all = a.T - first < segment ? a.T - first : segment;
  const int64_t end = first + all, live = len < end ? len : end;
  T* y = static_cast<T*>(a.y) + (b * a.T + first) * a.D + d0;
  if (first < live) {
    const Taps<T, K, V> taps(a, d0);
    Pack<T, V> seen[H];  // inputs t-K+1 .. t-1
#pragma unroll
    for (int k = 0; k < K - 1; ++k) seen[k] = input<T, V>(a, b, first - (K - 1) + k, d0);
    const T* x = static_cast<const T*>(a.x) + b * a.sx_b + first * a.sx_t + d0;
    Pack<T, V> in[kBatch];
    const auto request = [&](int64_t t) {  // (of steps that are not there the segment's first)
#pragma unroll
      for (int r = 0; r < kBatch; ++r)
        in[r] = load_pack<T, V>(x + (t + r < live ? t + r - first : 0) * a.sx_t, V);
    };
    const auto batch = [&](int64_t t, auto whole) {
      Pack<T, V> now[kBatch];
#pragma unroll
      for (int r = 0; r < kBatch; ++r) now[r] = in[r];
      request(t + kBatch);
#pragma unroll
      for (int r = 0; r < kBatch; ++r) {
        Pack<T, V> out;
#pragma unroll
        for (int i = 0; i < V; ++i) {
          A v = taps.b[i];
#pragma unroll
          for (int k = 0; k < K - 1; ++k) v = fma_(taps.w[k][i], up((T)seen[k].v[i]), v);
          v = fma_(taps.w[K - 1][i], up((T)now[r].v[i]), v);
          if (SILU) {
            A g, q;
            gates<T>(v, &g, &q);
            v *= g;
          }
          out.v[i] = down<T>(v);
        }
        if (decltype(whole)::value || t + r < live) store_pack<T, V>(y + r * a.D, out, V);
#pragma unroll
        for (int k = 0; k + 1 < K - 1; ++k) seen[k] = seen[k + 1];
        if (K > 1) seen[H - 1] = now[r];
      }
      y += kBatch * a.D;
    };
    request(first);
    int64_t t = first;
    for (; t + kBatch <= live; t += kBatch) batch(t, Count<1>());
    if (t < live) batch(t, Count<0>());
  }
  y = static_cast<T*>(a.y) + b * a.T * a.D + d0;
  for (int64_t t = live > first ? live : first; t < end; ++t)
    store_pack<T, V>(y + t * a.D, zeros<T, V>(), V);
}

// ------------------------------------------------------------------- reverse
// How the VJP is laid out: `columns` lanes along channels, the workgroup's other
// threads and `workers` workgroups along segments.
struct Layout {
  int columns;
  int64_t slabs, workers, segments;
};
Layout layout_of(int64_t B, int64_t T_, int64_t D, int V) {
  const int64_t nvec = (D + V - 1) / V;
  Layout l;
  l.columns = 1;
  while (l.columns < nvec && l.columns < 64) l.columns *= 2;
  l.slabs = (nvec + l.columns - 1) / l.columns;
  l.segments = T_ > 0 ? (T_ + kSegment - 1) / kSegment : 1;
  const int64_t rows = kThreads / l.columns, all = (B * l.segments + rows - 1) / rows;
  const int64_t most = (1024 + l.slabs - 1) / l.slabs;
  l.workers = all < most ? all : most;
  if (l.workers < 1) l.workers = 1;
  return l;
}

template <class T, int K, int V, bool SILU>
__global__ __launch_bounds__(kThreads) void conv_rev(ConvArgs a, Layout l, void* sums) {
  typedef Acc<T> A;
  constexpr int H = K > 1 ? K - 1 : 1;
  __shared__ A part[kThreads][V];
  const int rows = kThreads / l.columns;
  const int column = threadIdx.x % l.columns, row = threadIdx.x / l.columns;
  const int64_t slab = blockIdx.x % l.slabs, worker = blockIdx.x / l.slabs;
  const int64_t c = slab * l.columns + column, d0 = first_channel<V>(c, a.D);
  const bool works = c * V < a.D;
  const Taps<T, K, V> taps(a, d0);
  A dw[K][V], db[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    db[i] = A(0);
#pragma unroll
    for (int k = 0; k < K; ++k) dw[k][i] = A(0);
  }
  const int64_t all = works ? a.B * l.segments : 0;
  for (int64_t item = worker * rows + row; item < all; item += l.workers * rows) {
    const int64_t b = item / l.segments, first = item % l.segments * kSegment;
    const int64_t end = a.T - first < kSegment ? a.T : first + kSegment;
    const int64_t len = row_length(a.lens, b, a.T);
    // the first value whose gradient is this segment's: the window's before the row's start
    const int64_t low = first > 0 ? first : -(K - 1);
    const int64_t most = end + K - 1 < len ? end + K - 1 : len;  // steps that are needed
    Pack<T, V> seen[H];
    const bool any = first < most;
    if (any) {
#pragma unroll
      for (int k = 0; k < K - 1; ++k) seen[k] = input<T, V>(a, b, first - (K - 1) + k, d0);
    }
    A acc[K][V];  // of the gradients of inputs t-K+1 .. t
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) acc[k][i] = A(0);
    const T* x = static_cast<const T*>(a.x) + b * a.sx_b + first * a.sx_t + d0;
    const T* dy = static_cast<const T*>(a.dy) + b * a.sd_b + first * a.sd_t + d0;
    Pack<T, V> in[kBatch], d[kBatch];
    const auto request = [&](int64_t t0) {  // (of steps that are not there the segment's first)
#pragma unroll
      for (int r = 0; r < kBatch; ++r) {
        const int64_t t = t0 + r < most ? t0 + r - first : 0;
        in[r] = load_pack<T, V>(x + t * a.sx_t, V);
        d[r] = load_pack<T, V>(dy + t * a.sd_t, V);
      }
    };
    if (any) request(first);
    // one step: WHOLE: it is there; OWN: one of the segment's, whose dw and db it adds to, 0 where
    // that is to be asked
    const auto step = [&](int64_t t, const Pack<T, V>& now, const Pack<T, V>& e, auto whole,
                          auto own) {
      constexpr bool kWhole = decltype(whole)::value, kOwn = decltype(own)::value;
      if (kWhole || t < most) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          A g = up((T)e.v[i]);
          if (SILU) {
            A v = taps.b[i], s, q;
#pragma unroll
            for (int k = 0; k < K - 1; ++k) v = fma_(taps.w[k][i], up((T)seen[k].v[i]), v);
            v = fma_(taps.w[K - 1][i], up((T)now.v[i]), v);
            gates<T>(v, &s, &q);
            g *= s * fma_(v, q, A(1));
          }
#pragma unroll
          for (int k = 0; k < K; ++k) acc[k][i] = fma_(taps.w[k][i], g, acc[k][i]);
          if (kOwn || (!kWhole && t < end)) {
            db[i] += g;
#pragma unroll
            for (int k = 0; k < K - 1; ++k) dw[k][i] = fma_(g, up((T)seen[k].v[i]), dw[k][i]);
            dw[K - 1][i] = fma_(g, up((T)now.v[i]), dw[K - 1][i]);
          }
        }
      }
#pragma unroll
      for (int k = 0; k + 1 < K - 1; ++k) seen[k] = seen[k + 1];
      if (K > 1) seen[H - 1] = now;
    };
    // the gradient of input t - (K - 1) is whole
    const auto leave = [&](int64_t t, auto inside) {
      const int64_t at = t - (K - 1);
      if (decltype(inside)::value || (at >= low && at < end)) {
        Pack<T, V> out, of;
        const bool held =
            !decltype(inside)::value && a.dxT && at >= len - (K - 1) && at < len;
        if (held)
          of = load_pack<T, V>(static_cast<const T*>(a.dxT) +
                                   (b * (K - 1) + at + (K - 1) - len) * a.D + d0, V);
#pragma unroll
        for (int i = 0; i < V; ++i)
          out.v[i] = down<T>(held ? acc[0][i] + up((T)of.v[i]) : acc[0][i]);
        if (decltype(inside)::value || at >= 0) {
          if (a.dx) store_pack<T, V, true>(static_cast<T*>(a.dx) + (b * a.T + at) * a.D + d0, out, V);
        } else if (a.dx0) {
          store_pack<T, V>(static_cast<T*>(a.dx0) + (b * (K - 1) + at + (K - 1)) * a.D + d0, out, V);
        }
      }
#pragma unroll
      for (int k = 0; k + 1 < K; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) acc[k][i] = acc[k + 1][i];
#pragma unroll
      for (int i = 0; i < V; ++i) acc[K - 1][i] = A(0);
    };
    const auto batch = [&](int64_t t0, auto whole, auto own, auto inside) {
      Pack<T, V> now[kBatch], e[kBatch];
#pragma unroll
      for (int r = 0; r < kBatch; ++r) {
        now[r] = in[r];
        e[r] = d[r];
      }
      if (any) request(t0 + kBatch);
#pragma unroll
      for (int r = 0; r < kBatch; ++r) {
        step(t0 + r, now[r], e[r], whole, own);
        leave(t0 + r, inside);
      }
    };
    const int64_t stop = end + K - 1;  // every gradient has left by then
    int64_t t0 = first;
    typedef Count<1> Yes;
    typedef Count<0> No;
    if (first + kSegment + K - 1 <= len) {  // nothing of the segment or after it is missing
      constexpr int kLead = (K - 1 + kBatch - 1) / kBatch;  // batches whose gradients start before
#pragma unroll
      for (int k = 0; k < kLead; ++k, t0 += kBatch) batch(t0, Yes(), Yes(), No());
      for (; t0 < end; t0 += kBatch) batch(t0, Yes(), Yes(), Yes());
    }
    for (; t0 < stop; t0 += kBatch) batch(t0, No(), No(), No());
  }
  if (!sums) return;
  // [worker][K + 1][D]: over the workgroup's rows in turn
  A* const out = static_cast<A*>(sums) + worker * (K + 1) * a.D;
#pragma unroll
  for (int k = 0; k <= K; ++k) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < V; ++i) part[threadIdx.x][i] = k < K ? dw[k < K ? k : 0][i] : db[i];
    __syncthreads();
    if (row == 0 && works)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        double v = 0;
        for (int r = 0; r < rows; ++r) v += part[r * l.columns + column][i];
        out[k * a.D + d0 + i] = (A)v;
      }
  }
}

// dw and dbias from the workers' sums: 64 columns, four rows of threads that
// take every fourth worker. In 64 bits: threads' sums are of a few segments, what is added up here
// and over a workgroup's rows may be a thousand times as long (5 x 2049 x 771 F32: dw and db
// 1.4e-7 off in 32 bits, 1.1e-7 so; 4.2 us both).
template <class T>
__global__ __launch_bounds__(kThreads) void conv_sum(const Acc<T>* sums, int64_t workers, int64_t D,
                                                     int taps, void* dw, void* dbias, bool same) {
  __shared__ double part[4][64];
  const int64_t i = (int64_t)blockIdx.x * 64 + threadIdx.x % 64, all = (taps + 1) * D;
  const int row = threadIdx.x / 64;
  double v = 0;
  if (i < all) {
#pragma unroll 8
    for (int64_t k = row; k < workers; k += 4) v += sums[k * all + i];
  }
  part[row][threadIdx.x % 64] = v;
  __syncthreads();
  if (row > 0 || i >= all) return;
  v = (part[0][threadIdx.x] + part[1][threadIdx.x]) + (part[2][threadIdx.x] + part[3][threadIdx.x]);
  void* const to = i < taps * D ? dw : dbias;
  const int64_t at = i < taps * D ? i : i - taps * D;
  if (!to) return;
  if (same) static_cast<T*>(to)[at] = (T)v;
  else static_cast<float*>(to)[at] = (float)v;
}

// ------------------------------------------------------------------ one step
template <class T, int V>
__global__ __launch_bounds__(kThreads) void conv_one(ConvStep a, int64_t first) {
  typedef Acc<T> A;
  const int64_t b = first + blockIdx.y, d0 = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * V;
  if (d0 >= a.D) return;
  const int n = (int)(a.D - d0 < V ? a.D - d0 : V), K = a.taps;
  const bool same = a.wtype == a.dtype;
  const int64_t slot = a.slots ? a.slots[b] : b;
  Pack<T, V> out;
  if (slot < 0 || slot >= a.nstates) {
#pragma unroll
    for (int i = 0; i < V; ++i) out.v[i] = T(0);
    if (a.y) store_pack<T, V>(static_cast<T*>(a.y) + b * a.D + d0, out, n);
    return;
  }
  T* const window = static_cast<T*>(a.window) + slot * (K - 1) * a.D + d0;
  Pack<T, V> seen[ADST_CONV_MAX_TAPS];
  A w[ADST_CONV_MAX_TAPS][V], v[V];
  const auto weights = [&](const void* from, int64_t at, A (&to)[V]) {
    if (same) {
      const Pack<T, V> p = load_pack<T, V>(static_cast<const T*>(from) + at, n);
#pragma unroll
      for (int i = 0; i < V; ++i) to[i] = up((T)p.v[i]);
    } else {
      const Pack<float, V> p = load_pack<float, V>(static_cast<const float*>(from) + at, n);
#pragma unroll
      for (int i = 0; i < V; ++i) to[i] = (A)p.v[i];
    }
  };
#pragma unroll
  for (int k = 0; k < ADST_CONV_MAX_TAPS; ++k)
    if (k < K) {
      seen[k] = load_pack<T, V>(k < K - 1 ? window + k * a.D
                                          : static_cast<const T*>(a.x) + b * a.sx + d0, n);
      weights(a.w, k * a.D + d0, w[k]);
    }
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = A(0);
  if (a.bias) weights(a.bias, d0, v);
#pragma unroll
  for (int k = 0; k < ADST_CONV_MAX_TAPS; ++k)
    if (k < K) {
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = fma_(w[k][i], up((T)seen[k].v[i]), v[i]);
      if (k > 0) store_pack<T, V>(window + (k - 1) * a.D, seen[k], n);
    }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    if (a.act == ADST_ACT_SILU) {
      A g, q;
      gates<T>(v[i], &g, &q);
      v[i] *= g;
    }
    out.v[i] = down<T>(v[i]);
  }
  if (a.y) store_pack<T, V>(static_cast<T*>(a.y) + b * a.D + d0, out, n);
}

// ------------------------------------------------------------------ launches
template <class F>
hipError_t by_type(int32_t dtype, F f) {
  switch (dtype) {
    case ADST_F64: return f(double());
    case ADST_F32: return f(float());
    case ADST_BF16: return f(bf16());
    default: return f(f16());
  }
}
template <class F>
hipError_t by_taps(int taps, F f) {
  switch (taps) {
    case 1: return f(Count<1>());
    case 2: return f(Count<2>());
    case 3: return f(Count<3>());
    case 4: return f(Count<4>());
    case 5: return f(Count<5>());
    case 6: return f(Count<6>());
    case 7: return f(Count<7>());
    default: return f(Count<8>());
  }
}

// f(the channels of a thread): one where a row has fewer than V.
template <int V, class F>
hipError_t by_lanes(int64_t D, F f) {
  return D >= V ? f(Count<V>()) : f(Count<1>());
}

// Workgroups of one launch at most: its work-items are counted in 32 bits.
constexpr int64_t kMostGroups = (int64_t(1) << 32) / kThreads - 1;
constexpr int64_t kMostRows = 65535;  // of a launch's second axis

}  // namespace

hipError_t conv_forward(const ConvArgs& q, hipStream_t st) {
  return by_type(q.dtype, [&](auto t) {
    return by_taps(q.taps, [&](auto k) {
      typedef decltype(t) T;
      constexpr int K = decltype(k)::value;
      return by_lanes<lanes_of<T, K>(false)>(q.D, [&](auto lanes) {
        constexpr int V = decltype(lanes)::value;
        const int64_t nvec = (q.D + V - 1) / V;
        const int segment =
            nvec * q.B * ((q.T + kSegment - 1) / kSegment) >= kManyThreads ? kSegment : kFewSegment;
        const int64_t segments = q.y ? (q.T + segment - 1) / segment : 0;
        // rows of the batch in several launches where one does not hold them
        const int64_t row = nvec * (segments + 1), rows = kMostGroups * kThreads / row;
        if (rows < 1) return hipErrorInvalidValue;
        for (int64_t b = 0; b < q.B; b += rows) {
          ConvArgs a = q;
          a.B = q.B - b < rows ? q.B - b : rows;
          a.x = q.x ? static_cast<const T*>(q.x) + b * q.sx_b : nullptr;
          a.x0 = q.x0 ? static_cast<const T*>(q.x0) + b * (K - 1) * q.D : nullptr;
          a.lens = q.lens ? q.lens + b : nullptr;
          a.y = q.y ? static_cast<T*>(q.y) + b * q.T * q.D : nullptr;
          a.xT = q.xT ? static_cast<T*>(q.xT) + b * (K - 1) * q.D : nullptr;
          const unsigned groups = (unsigned)((a.B * row + kThreads - 1) / kThreads);
          const hipError_t e = start(a.act == ADST_ACT_SILU ? conv_fwd<T, K, V, true>
                                                            : conv_fwd<T, K, V, false>,
                                     dim3(groups), kThreads, st, a, nvec, segments, segment);
          if (e != hipSuccess) return e;
        }
        return hipSuccess;
      });
    });
  });
}

uint64_t conv_workspace_bytes(int32_t dtype, int64_t B, int64_t T_, int64_t D, int32_t taps) {
  uint64_t bytes = 0;
  (void)by_type(dtype, [&](auto t) {
    return by_taps(taps, [&](auto k) {
      typedef decltype(t) T;
      constexpr int K = decltype(k)::value;
      return by_lanes<lanes_of<T, K>(true)>(D, [&](auto lanes) {
        bytes = (uint64_t)layout_of(B, T_, D, decltype(lanes)::value).workers * (K + 1) * D *
                sizeof(Acc<T>);
        return hipSuccess;
      });
    });
  });
  return bytes;
}

hipError_t conv_vjp(const ConvArgs& q, void* ws, hipStream_t st) {
  return by_type(q.dtype, [&](auto t) {
    return by_taps(q.taps, [&](auto k) {
      typedef decltype(t) T;
      constexpr int K = decltype(k)::value;
      return by_lanes<lanes_of<T, K>(true)>(q.D, [&](auto lanes) {
        constexpr int V = decltype(lanes)::value;
        const Layout l = layout_of(q.B, q.T, q.D, V);
        const bool sums = q.dw || q.dbias;
        const hipError_t e = start(q.act == ADST_ACT_SILU ? conv_rev<T, K, V, true>
                                                          : conv_rev<T, K, V, false>,
                                   dim3((unsigned)(l.slabs * l.workers)), kThreads, st, q, l,
                                   sums ? ws : nullptr);
        if (e != hipSuccess || !sums) return e;
        return start(conv_sum<T>, dim3((unsigned)(((K + 1) * q.D + 63) / 64)), kThreads, st,
                     static_cast<const Acc<T>*>(ws), l.workers, q.D, K, q.dw, q.dbias,
                     q.wtype == q.dtype);
      });
    });
  });
}

hipError_t conv_step(const ConvStep& q, hipStream_t st) {
  return by_type(q.dtype, [&](auto t) {
    typedef decltype(t) T;
    constexpr int V = sizeof(T) == 8 ? 1 : sizeof(T) == 4 ? 2 : 4;
    const int64_t nvec = (q.D + V - 1) / V, groups = (nvec + kThreads - 1) / kThreads;
    for (int64_t b = 0; b < q.B; b += kMostRows) {
      const int64_t rows = q.B - b < kMostRows ? q.B - b : kMostRows;
      const hipError_t e = start(conv_one<T, V>, dim3((unsigned)groups, (unsigned)rows), kThreads,
                                 st, q, b);
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  });
}

}  // namespace adst
