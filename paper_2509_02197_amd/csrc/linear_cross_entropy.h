// Softmax cross entropy of rows x [M][K] over a vocabulary w [V][K] without its
// logits in memory: lse = log sum_v exp(x w_v), loss = lse - x w_label; and its
// VJP, g = (exp(x w_v - lse) - [v = label]) dloss, dx = g w, dw = g^T x.
//
// Four products of 2 M V K operations (one forward, three in reverse) and little
// else: the matrix cores bound it, or the read of w where rows are few. Every product
// is vocab_gemm.h's, with both operands contiguous along the axis that is summed; what
// follows a product happens in its registers:
//   forward   a tile's rows to their largest logit and sum of exponentials (online
//             softmax across tiles: a second kernel joins the tiles in order)
//   reverse   for a piece of the vocabulary at a time, the logits again and from them g,
//             written in both orders, rows and columns; then dw of the piece = g^T x and
//             dx += g w, for which x and the piece of w are transposed once each (with many
//             rows a hundredth of a product's time, against a second kind of product).
// g is rounded to the element type, which the matrix cores need (a caller who wants 32 bits of it
// passes x and w in F32); each of its elements enters sums of thousands in 32 bits, and its
// roundings are independent, all but those of the -1 at the labels: there g is close to -dloss.
// What leaves -1 exact differs by order. In rows, for dx, g is held without dloss, which a row of
// dx is multiplied by at its end: -1 and a row's small probabilities do not depend on other rows'
// weights. In columns, for dw, whose sums go over rows, g has its weight, beside 16-bit types
// scaled to make the largest |dloss| a power of two, which leaves the -1 exact under a mean. F16's
// range would lose small probabilities: both orders are held times 2^14. (dw and dx of 4096 x
// 4096 x 65537 F16 under a mean: 4.0e-4 off without, of which 2.1e-4 are their own rounding. bf16
// 8192 x 2048 x 32000: the results are as far from 64 bits as with 32 bits of g, 1.7e-3, to 1%.)
#pragma once

#include "vocab_gemm.h"

namespace adst {
namespace {

constexpr int kJoinThreads = 256;

__device__ inline float exp_(float v) { return __builtin_amdgcn_exp2f(v * 1.44269504f); }
__device__ inline double exp_(double v) { return exp(v); }
__device__ inline float log_(float v) { return logf(v); }
__device__ inline double log_(double v) { return log(v); }
// What exponentials are taken relative to: 0 where the largest logit is infinite, so that
// no infinity is subtracted from itself.
template <class A>
__device__ inline A pivot(A top) {
  return __builtin_isinf(top) ? A(0) : top;
}
template <class A>
__device__ inline A larger(A a, A b) {  // a NaN stays
  return a > b || a != a ? a : b;
}

// Over the 16 lanes of a row of the wave.
__device__ inline float row_sum(float v) { return lane_sum<16>(v); }
__device__ inline double row_sum(double v) { return lane_sum<16>(v); }
__device__ inline float row_top(float v) {
  v = larger(v, permuted<0xb1>(v));
  v = larger(v, permuted<0x4e>(v));
  v = larger(v, permuted<0x141>(v));
  return larger(v, permuted<0x140>(v));
}
__device__ inline double row_top(double v) {
#pragma unroll
  for (int off = 1; off < 16; off <<= 1) v = larger(v, __shfl_xor(v, off, 64));
  return v;
}

template <class A>
struct Stat {
  A top, sum;  // the sum of exponentials relative to pivot(top)
};
template <class A>
__device__ inline A relative_to(A from, Stat<A> s) {
  return s.sum == A(0) ? A(0) : s.sum * exp_(pivot(s.top) - from);
}

struct Tiles {
  int64_t m, n;       // tiles
  int64_t K, steps;   // the long axis: elements and steps
  int64_t splits;     // parts of the steps, along the grid
};

// ------------------------------------------------------------------- forward
// [tile column][row] statistics and each row's target logit.
template <class S, bool DIRECT>
__global__ __launch_bounds__(S::kThreads) void xent_stats(Rows x, Rows w, Tiles t,
                                                          const int32_t* labels, void* stats,
                                                          void* target) {
  typedef typename S::T T;
  typedef Acc<T> A;
  typedef Tile<T> C;
  __shared__ __attribute__((aligned(16))) char lds[S::ST * S::kStageBytes];
  const TileAt tile = tile_at(t.m, t.n, blockIdx.x);
  const int64_t m0 = tile.m * S::BM, n0 = tile.n * S::BN;
  S s;
  multiply<S, DIRECT>(s, lds, x, w, t.K, m0, n0, 0, t.steps);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wm = wave / S::WN, wn = wave % S::WN, col = lane & 15;
  Stat<A>(*const part)[S::WN] = reinterpret_cast<Stat<A>(*)[S::WN]>(lds);  // [row of the tile]
  int* const label_of = reinterpret_cast<int*>(part + S::BM);  // a column of the tile, or -1
  for (int row = threadIdx.x; row < S::BM; row += S::kThreads) {
    const int64_t at = m0 + row < x.n ? labels[m0 + row] - n0 : -1;
    label_of[row] = at >= 0 && at < S::BN && n0 + at < w.n ? (int)at : -1;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < S::MT; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = (wm * S::MT + i) * 16 + C::at(lane, r);
      const int label = label_of[row];
      A top = -__builtin_inf();
#pragma unroll
      for (int j = 0; j < S::NT; ++j) {
        const int n = (wn * S::NT + j) * 16 + col;
        const A v = s.acc[i][j][r];
        if (n == label) static_cast<A*>(target)[m0 + row] = v;
        if (n0 + n < w.n) top = larger(v, top);
      }
      top = row_top(top);
      const A from = pivot(top);
      A sum = A(0);
#pragma unroll
      for (int j = 0; j < S::NT; ++j) {
        const int64_t n = n0 + (wn * S::NT + j) * 16 + col;
        if (n < w.n) sum += exp_(s.acc[i][j][r] - from);
      }
      sum = row_sum(sum);
      if (col == 0) part[row][wn] = {top, sum};
    }
  __syncthreads();
  for (int row = threadIdx.x; row < S::BM; row += S::kThreads) {
    if (m0 + row >= x.n) continue;
    A top = part[row][0].top;
#pragma unroll
    for (int k = 1; k < S::WN; ++k) top = larger(part[row][k].top, top);
    const A from = pivot(top);
    A sum = A(0);
#pragma unroll
    for (int k = 0; k < S::WN; ++k) sum += relative_to(from, part[row][k]);
    static_cast<Stat<A>*>(stats)[tile.n * x.n + m0 + row] = {top, sum};
  }
}

// loss and lse from the tiles' statistics. W lanes of a wave share a row.
template <class T, int W>
__global__ __launch_bounds__(kJoinThreads) void xent_join(const void* stats, const void* target,
                                                          const int32_t* labels, int64_t M,
                                                          int64_t V, int64_t columns, void* loss,
                                                          void* lse) {
  typedef Acc<T> A;
  constexpr int kAhead = 8;  // statistics whose loads are in flight together
  const int64_t m = ((int64_t)blockIdx.x * kJoinThreads + threadIdx.x) / W;
  const int lane = threadIdx.x % W;
  const int64_t row = m < M ? m : M - 1;
  const Stat<A>* const from = static_cast<const Stat<A>*>(stats) + row;
  Stat<A> all = {A(-__builtin_inf()), A(0)};
  for (int64_t k = lane; k < columns; k += W * kAhead) {
    Stat<A> some[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int64_t at = k + i * W;
      some[i] = from[(at < columns ? at : k) * M];
      if (at >= columns) some[i].sum = A(0);  // of one that was there already
    }
    A top = all.top;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) top = larger(some[i].top, top);
    A sum = relative_to(pivot(top), all);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) sum += relative_to(pivot(top), some[i]);
    all = {top, sum};
  }
  A top = all.top;
#pragma unroll
  for (int by = 1; by < W; by <<= 1) top = larger(top, __shfl_xor(top, by, 64));
  const A at = pivot(top);
  A sum = relative_to(at, all);
#pragma unroll
  for (int by = 1; by < W; by <<= 1) sum += __shfl_xor(sum, by, 64);
  if (m >= M || lane > 0) return;
  const A v = at + log_(sum);
  if (lse) static_cast<A*>(lse)[m] = v;
  if (loss) {
    const bool has = labels[m] >= 0 && labels[m] < V;
    static_cast<A*>(loss)[m] = has ? v - static_cast<const A*>(target)[m] : A(0);
  }
}

// ------------------------------------------------------------------- reverse
// What a row's g is multiplied by: 0 where it takes no part.
template <class A>
__device__ inline A row_weight(const int32_t* labels, const void* dloss, int64_t m, int64_t V) {
  const int64_t label = labels[m];
  const A weight = dloss ? static_cast<const A*>(dloss)[m] : A(1);  // loaded beside the label
  return label < 0 || label >= V ? A(0) : weight;
}

// What g in rows is held times.
template <class T>
constexpr float kUnit = 1.0f;
template <>
inline constexpr float kUnit<f16> = 0x1p14f;

// scale[0]: what takes the largest finite |dloss| of the rows that take part to `to`;
// scale[1]: its inverse. One workgroup.
__global__ __launch_bounds__(1024) void xent_scale(const int32_t* labels, const void* dloss,
                                                   int64_t M, int64_t V, float to, float* scale) {
  __shared__ float part[16];
  float top = 0.0f;
#pragma unroll 4
  for (int64_t m = threadIdx.x; m < M; m += 1024) {
    const float v = __builtin_fabsf(row_weight<float>(labels, dloss, m, V));
    if (v > top && !__builtin_isinf(v)) top = v;
  }
  for (int by = 1; by < 64; by <<= 1) {
    const float other = __shfl_xor(top, by, 64);
    top = other > top ? other : top;
  }
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = top;
  __syncthreads();
  if (threadIdx.x > 0) return;
  for (int k = 1; k < 16; ++k) top = part[k] > top ? part[k] : top;
  // both stay normal numbers
  top = top == 0.0f ? to : top < 0x1p-100f ? 0x1p-100f : top > 0x1p100f ? 0x1p100f : top;
  scale[0] = to / top;
  scale[1] = top / to;
}

// to [cols][pad] = from [rows][cols] transposed, zeros from `rows` to `pad`. KEEP: rows
// without a weight are zeros, whatever they hold.
constexpr int kTurn = 64;
template <class T, bool KEEP>
__global__ __launch_bounds__(256) void xent_turn(Rows from, int64_t cols, int64_t pad, void* to,
                                                 const int32_t* labels, const void* dloss,
                                                 int64_t V) {
  constexpr int N = Vec<T>::N, kAcross = kTurn / N;  // vectors of 16 bytes across a tile
  __shared__ __attribute__((aligned(16))) T tile[kTurn][kTurn + N];  // [column][row]
  const int64_t across = (cols + kTurn - 1) / kTurn;
  const int64_t r0 = blockIdx.x / across * kTurn, c0 = blockIdx.x % across * kTurn;
#pragma unroll
  for (int k = threadIdx.x; k < kTurn * kAcross; k += 256) {
    const int r = k / kAcross, c = k % kAcross * N;
    const int64_t row = r0 + r, left = cols - c0 - c;
    bool there = row < from.n && left > 0;
    if (KEEP && there) there = row_weight<Acc<T>>(labels, dloss, row, V) != Acc<T>(0);
    const T* const at = static_cast<const T*>(from.p) + row * from.stride + c0 + c;
    const Vec<T> v = load_part(at, there ? (int)(left < N ? left : N) : 0);
#pragma unroll
    for (int i = 0; i < N; ++i) tile[c + i][r] = v.v[i];
  }
  __syncthreads();
#pragma unroll
  for (int k = threadIdx.x; k < kTurn * kAcross; k += 256) {
    const int c = k / kAcross, r = k % kAcross * N;
    // (pad is whole steps of 128 bytes, and so whole vectors)
    if (c0 + c < cols && r0 + r < pad)
      *reinterpret_cast<U4*>(static_cast<T*>(to) + (c0 + c) * pad + r0 + r) =
          *reinterpret_cast<const U4*>(&tile[c][r]);
  }
}

// g of a piece of the vocabulary, whose first word is v0: without weights times kUnit
// [rows][piece] and, with them and transposed, [piece][m_pad]. Both are whole: zeros beyond the
// vocabulary and the rows.
struct GArgs {
  const int32_t* labels;
  const void* lse;
  const void* dloss;
  const float* scale;  // or NULL
  int64_t v0, V, piece, m_pad;
  void* g;
  void* gt;
};
template <class S, bool DIRECT>
__global__ __launch_bounds__(S::kThreads) void xent_grad(Rows x, Rows w, Tiles t, GArgs q) {
  typedef typename S::T T;
  typedef Acc<T> A;
  typedef Tile<T> C;
  __shared__ __attribute__((aligned(16))) char lds[S::ST * S::kStageBytes];
  const TileAt tile = tile_at(t.m, t.n, blockIdx.x);
  const int64_t m0 = tile.m * S::BM, n0 = tile.n * S::BN;
  S s;
  multiply<S, DIRECT>(s, lds, x, w, t.K, m0, n0, 0, t.steps);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wm = wave / S::WN, wn = wave % S::WN, col = lane & 15;
  const A scale = q.scale ? (A)q.scale[0] : A(1);
  struct Row {
    A lse, weight;
    int label;
    bool in;  // takes part
  };
  Row* const row_of = reinterpret_cast<Row*>(lds);
  for (int row = threadIdx.x; row < S::BM; row += S::kThreads) {
    const int64_t m = m0 + row;
    Row one = {A(0), A(0), -1, false};
    if (m < x.n) {
      const int64_t at = q.labels[m] - q.v0 - n0;
      const A weight = row_weight<A>(q.labels, q.dloss, m, q.V);
      one.in = weight != A(0);
      one.weight = weight * scale;
      one.lse = static_cast<const A*>(q.lse)[m];
      one.label = at >= 0 && at < S::BN ? (int)at : -1;
    }
    row_of[row] = one;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < S::MT; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const Row row = row_of[(wm * S::MT + i) * 16 + C::at(lane, r)];
#pragma unroll
      for (int j = 0; j < S::NT; ++j) {
        const int n = (wn * S::NT + j) * 16 + col;
        A v = A(0);
        if (row.in && n0 + n < w.n)
          v = exp_(s.acc[i][j][r] - row.lse) - (n == row.label ? A(1) : A(0));
        s.acc[i][j][r] = v;
      }
    }
  // transposed: a lane has four neighbouring rows of a column (every fourth, for F64)
#pragma unroll
  for (int i = 0; i < S::MT; ++i) {
    A weight[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) weight[r] = row_of[(wm * S::MT + i) * 16 + C::at(lane, r)].weight;
#pragma unroll
    for (int j = 0; j < S::NT; ++j) {
      const int64_t n = n0 + (wn * S::NT + j) * 16 + col, m = m0 + (wm * S::MT + i) * 16;
      if (m >= q.m_pad || n >= q.piece) continue;  // (both are multiples of 16)
      T* const to = static_cast<T*>(q.gt) + n * q.m_pad + m;
      if constexpr (sizeof(T) == 8) {
#pragma unroll
        for (int r = 0; r < 4; ++r) to[C::at(lane, r)] = down<T>(s.acc[i][j][r] * weight[r]);
      } else {
        typedef T Four __attribute__((ext_vector_type(4)));
        Four v;
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = down<T>(s.acc[i][j][r] * weight[r]);
        *reinterpret_cast<Four*>(to + C::at(lane, 0)) = v;
      }
    }
  }
  __syncthreads();
  store_tile<S>(lds, static_cast<T*>(q.g) + m0 * q.piece + n0, q.piece, x.n - m0, q.piece - n0,
                [&](int i, int r, int j) { return down<T>(s.acc[i][j][r] * A(kUnit<T>)); });
}

// What the rows of a product are multiplied by at its end: for dw what scales it back (1 if
// NULL), for dx (labels given) the rows' weights and what takes kUnit back.
struct Back {
  const float* scale;
  const int32_t* labels;
  const void* dloss;
  int64_t V;
};
template <class T>
__device__ inline Acc<T> back_of(const Back& q, int64_t row) {
  typedef Acc<T> A;
  if (q.labels) return row_weight<A>(q.labels, q.dloss, row, q.V) * A(1 / kUnit<T>);
  return q.scale ? (A)q.scale[1] : A(1);
}

// C [rows][n] from a product (DIRECT: of whole steps): rounded to `out`, or added to (`add`: after
// earlier pieces) its split's sums [split][rows][n].
struct OutArgs {
  void* out;
  void* sums;
  Back back;
  bool add;
};
template <class S, bool DIRECT>
__global__ __launch_bounds__(S::kThreads) void xent_product(Rows a, Rows b, Tiles t, OutArgs q) {
  typedef typename S::T T;
  typedef Acc<T> A;
  typedef Tile<T> C;
  __shared__ __attribute__((aligned(16))) char lds[S::ST * S::kStageBytes];
  const int64_t split = blockIdx.x % t.splits;
  const TileAt tile = tile_at(t.m, t.n, blockIdx.x / t.splits);
  const int64_t m0 = tile.m * S::BM, n0 = tile.n * S::BN;
  S s;
  multiply<S, DIRECT>(s, lds, a, b, t.K, m0, n0, t.steps * split / t.splits,
                      t.steps * (split + 1) / t.splits);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wm = wave / S::WN, wn = wave % S::WN, col = lane & 15;
  if (q.out) {
#pragma unroll
    for (int i = 0; i < S::MT; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int64_t m = m0 + (wm * S::MT + i) * 16 + C::at(lane, r);
        const A back = back_of<T>(q.back, m < a.n ? m : a.n - 1);
#pragma unroll
        for (int j = 0; j < S::NT; ++j) s.acc[i][j][r] *= back;
      }
    store_tile<S>(lds, static_cast<T*>(q.out) + m0 * b.n + n0, b.n, a.n - m0, b.n - n0,
                  [&](int i, int r, int j) { return down<T>(s.acc[i][j][r]); });
    return;
  }
  A* const to = static_cast<A*>(q.sums) + (split * a.n + m0) * b.n + n0;
  const int64_t rows = a.n - m0, columns = b.n - n0;
#pragma unroll
  for (int i = 0; i < S::MT; ++i) {
    A old[4][S::NT];  // the loads of a row of tiles are in flight together
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int j = 0; j < S::NT; ++j) {
        const int m = (wm * S::MT + i) * 16 + C::at(lane, r), n = (wn * S::NT + j) * 16 + col;
        const bool there = m < rows && n < columns;
        old[r][j] = q.add && there ? to[m * b.n + n] : A(0);
      }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int j = 0; j < S::NT; ++j) {
        const int m = (wm * S::MT + i) * 16 + C::at(lane, r), n = (wn * S::NT + j) * 16 + col;
        if (m < rows && n < columns) to[m * b.n + n] = old[r][j] + s.acc[i][j][r];
      }
  }
}

// out [n / width][width] = the splits' sums added in order, rounded. n is below 2^31. A thread takes
// EACH values, whose loads, and those of four splits, are in flight together.
constexpr int kSumThreads = 256;
template <class T, int EACH>
__global__ __launch_bounds__(kSumThreads) void xent_sum(const void* sums, int64_t n, int64_t width,
                                                        int64_t splits, Back back, void* out) {
  typedef Acc<T> A;
  const int64_t first = (int64_t)blockIdx.x * (kSumThreads * EACH) + threadIdx.x;
  A v[EACH], by[EACH];
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int64_t at = first + i * kSumThreads < n ? first + i * kSumThreads : n - 1;
    by[i] = back_of<T>(back, back.labels ? (uint32_t)at / (uint32_t)width : 0);
    v[i] = A(0);
  }
#pragma unroll 4
  for (int64_t k = 0; k < splits; ++k)
#pragma unroll
    for (int i = 0; i < EACH; ++i)
      if (first + i * kSumThreads < n)
        v[i] += static_cast<const A*>(sums)[k * n + first + i * kSumThreads];
#pragma unroll
  for (int i = 0; i < EACH; ++i)
    if (first + i * kSumThreads < n)
      static_cast<T*>(out)[first + i * kSumThreads] = down<T>(v[i] * by[i]);
}
// Four values where there is one split (dx of 8192 x 2048: 32 us, 43 with one value), one where
// there are more, whose loads fill the time (999 x 515 of 7 splits: 5 us, 11 with four).
template <class T>
hipError_t sum_up(const void* sums, int64_t n, int64_t width, int64_t splits, const Back& back,
                  void* out, hipStream_t st) {
  const int64_t each = kSumThreads * (splits > 1 ? 1 : 4);
  return start(splits > 1 ? xent_sum<T, 1> : xent_sum<T, 4>, dim3((unsigned)((n + each - 1) / each)),
               kSumThreads, st, sums, n, width, splits, back, out);
}

// --------------------------------------------------------------- few logits
// Where the tiles of the logits are fewer than the CUs and the rows long, the product is
// split along them, into sums in memory [split][row][word], and what follows a product is a
// kernel of its own (5 x 4014 over 728 words F32, 12 tiles of 126 steps: forward 16 us, 108 in
// one part).
template <class A>
__device__ inline A few_logit(const A* sums, int64_t splits, int64_t all, int64_t at) {
  A v = A(0);
#pragma unroll 8
  for (int64_t k = 0; k < splits; ++k) v += sums[k * all + at];
  return v;
}

// loss and lse: NT threads a row.
template <class T, int NT>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void xent_few_stats(
    const void* sums, int64_t splits, const int32_t* labels, int64_t M, int64_t V, void* loss,
    void* lse) {
  typedef Acc<T> A;
  constexpr int kRows = NT < 256 ? 256 / NT : 1, kWaves = NT / 64;
  __shared__ Stat<A> part[kWaves];
  __shared__ A part_target[kWaves];
  const int lane = threadIdx.x % NT;
  const int64_t m = (int64_t)blockIdx.x * kRows + threadIdx.x / NT, row = m < M ? m : M - 1;
  const int64_t label = labels[row];
  const A* const from = static_cast<const A*>(sums) + row * V;
  Stat<A> all = {A(-__builtin_inf()), A(0)};
  A target = A(0);
  for (int64_t n = lane; n < V; n += NT) {
    const A v = few_logit(from, splits, M * V, n);
    if (n == label) target = v;
    const A top = larger(v, all.top);
    all = {top, relative_to(pivot(top), all) + exp_(v - pivot(top))};
  }
  const auto join = [&](Stat<A> other) {
    const A top = larger(other.top, all.top), at = pivot(top);
    all = {top, relative_to(at, all) + relative_to(at, other)};
  };
#pragma unroll
  for (int by = 1; by < 64; by <<= 1) {
    join({__shfl_xor(all.top, by, 64), __shfl_xor(all.sum, by, 64)});
    target += __shfl_xor(target, by, 64);
  }
  if constexpr (kWaves > 1) {
    if (lane % 64 == 0) {
      part[lane / 64] = all;
      part_target[lane / 64] = target;
    }
    __syncthreads();
    if (lane > 0) return;
    all = part[0];
    target = part_target[0];
    for (int k = 1; k < kWaves; ++k) {
      join(part[k]);
      target += part_target[k];
    }
  }
  if (m >= M || lane > 0) return;
  const A v = pivot(all.top) + log_(all.sum);
  if (lse) static_cast<A*>(lse)[m] = v;
  if (loss) static_cast<A*>(loss)[m] = label >= 0 && label < V ? v - target : A(0);
}

// g of the whole vocabulary in both orders, as xent_grad leaves it. A thread: one value.
template <class T>
__global__ __launch_bounds__(256) void xent_few_grad(const void* sums, int64_t splits, int64_t M,
                                                     GArgs q) {
  typedef Acc<T> A;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (id >= q.m_pad * q.piece) return;
  const int64_t m = id / q.piece, n = id % q.piece;
  A v = A(0), weight = A(0);
  if (m < M && n < q.V) {
    weight = row_weight<A>(q.labels, q.dloss, m, q.V);
    if (weight != A(0)) {
      const A logit = few_logit(static_cast<const A*>(sums), splits, M * q.V, m * q.V + n);
      v = exp_(logit - static_cast<const A*>(q.lse)[m]) - (n == q.labels[m] ? A(1) : A(0));
    }
  }
  if (m < M) static_cast<T*>(q.g)[m * q.piece + n] = down<T>(v * A(kUnit<T>));
  const A scale = q.scale ? (A)q.scale[0] : A(1);
  static_cast<T*>(q.gt)[n * q.m_pad + m] = down<T>(v * (weight * scale));
}

// ------------------------------------------------------------------ launches
inline int64_t parts(int64_t n, int64_t by) { return (n + by - 1) / by; }
template <class S>
Tiles tiles_of(int64_t m, int64_t n, int64_t K, int64_t splits) {
  return {parts(m, S::BM), parts(n, S::BN), K, parts(K, S::kStep), splits};
}

// f(shape) for the tiles that the plan names.
template <class T, class F>
hipError_t by_tiles(int tiles, F f) {
  if constexpr (sizeof(T) < 8)
    if (tiles == 0) return f(GemmShape<T, 2, 4, 8, 4, 2>());  // 256 x 256
  if (tiles == 1) return f(GemmShape<T, 2, 2, 4, 4, 2>());    // 128 x 128
  if (tiles == 2) return f(GemmShape<T, 2, 2, 4, 2, 2>());    // 128 x 64
  if (tiles == 3) return f(GemmShape<T, 1, 4, 4, 1, 4>());  // 64 x 64, three steps ahead
  return f(GemmShape<T, 1, 2, 1, 4, 4>());  // 16 x 128
}

template <class T>
bool whole_pieces(const void* p, int64_t stride, int64_t K) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * (int64_t)sizeof(T) % 16 == 0 &&
         K * (int64_t)sizeof(T) % kStepBytes == 0 &&
         stride < (int64_t(1) << 28) / (int64_t)sizeof(T);  // offsets of 7 rows in 31 bits
}

// The logits' sums of a plan with few of them.
template <class T>
hipError_t few_logits(const XentArgs& a, const XentPlan& p, const Rows& x, const Rows& w,
                      bool direct, void* sums, hipStream_t st) {
  return by_tiles<T>(p.logits.tiles, [&](auto shape) {
    typedef decltype(shape) S;
    const Tiles t = tiles_of<S>(a.M, a.V, a.K, p.logits.splits);
    return start(direct ? xent_product<S, true> : xent_product<S, false>,
                 dim3((unsigned)(t.m * t.n * t.splits)), S::kThreads, st, x, w, t,
                 OutArgs{nullptr, sums, Back{}, false});
  });
}

template <class T>
hipError_t forward_of(const XentArgs& a, const XentPlan& p, void* ws, hipStream_t st) {
  char* const at = static_cast<char*>(ws);
  const bool direct = whole_pieces<T>(a.x, a.sx, a.K) && whole_pieces<T>(a.w, a.sw, a.K);
  const Rows x{a.x, a.sx, a.M}, w{a.w, a.sw, a.V};
  if (p.logits.splits > 1) {
    const hipError_t e = few_logits<T>(a, p, x, w, direct, at + p.few, st);
    if (e != hipSuccess) return e;
    const void* const sums = at + p.few;
    if (a.V <= 256)
      return start(xent_few_stats<T, 64>, dim3((unsigned)parts(a.M, 4)), 256, st, sums,
                   p.logits.splits, a.labels, a.M, a.V, a.loss, a.lse);
    return start(xent_few_stats<T, 1024>, dim3((unsigned)a.M), 1024, st, sums, p.logits.splits,
                 a.labels, a.M, a.V, a.loss, a.lse);
  }
  return by_tiles<T>(p.logits.tiles, [&](auto shape) {
    typedef decltype(shape) S;
    const Tiles t = tiles_of<S>(a.M, a.V, a.K, 1);
    hipError_t e = start(direct ? xent_stats<S, true> : xent_stats<S, false>,
                         dim3((unsigned)(t.m * t.n)), S::kThreads, st, x, w, t, a.labels,
                         at + p.stats, at + p.target);
    if (e != hipSuccess) return e;
    const void *stats = at + p.stats, *target = at + p.target;
    // (few rows: a wave for each, whose lanes take the tiles' statistics at once)
    if (a.M < 2048)
      return start(xent_join<T, 64>, dim3((unsigned)parts(a.M * 64, kJoinThreads)), kJoinThreads,
                   st, stats, target, a.labels, a.M, a.V, t.n, a.loss, a.lse);
    return start(xent_join<T, 8>, dim3((unsigned)parts(a.M * 8, kJoinThreads)), kJoinThreads, st,
                 stats, target, a.labels, a.M, a.V, t.n, a.loss, a.lse);
  });
}

template <class T>
hipError_t vjp_of(const XentArgs& a, const XentPlan& p, void* ws, hipStream_t st) {
  if (a.M == 0)  // no rows: dw is zero, a sum of nothing
    return sum_up<T>(nullptr, a.V * a.K, a.K, 0, Back{}, a.dw, st);
  char* const at = static_cast<char*>(ws);
  const Rows x{a.x, a.sx, a.M};
  hipError_t e = hipSuccess;
  const float* scale = nullptr;
  if (sizeof(T) == 2) {
    scale = reinterpret_cast<const float*>(at + p.scale);
    e = start(xent_scale, dim3(1), 1024, st, a.labels, a.dloss, a.M, a.V,
              kUnit<T>, reinterpret_cast<float*>(at + p.scale));
    if (e != hipSuccess) return e;
  }
  const Back of_dw{scale, nullptr, nullptr, a.V}, of_dx{nullptr, a.labels, a.dloss, a.V};
  if (a.dw) {
    e = start(xent_turn<T, true>,
              dim3((unsigned)(parts(p.m_pad, kTurn) * parts(a.K, kTurn))), 256, st, x, a.K, p.m_pad,
              at + p.xt, a.labels, a.dloss, a.V);
    if (e != hipSuccess) return e;
  }
  for (int64_t v0 = 0; v0 < a.V; v0 += p.piece) {
    const int64_t words = a.V - v0 < p.piece ? a.V - v0 : p.piece;
    const Rows w{static_cast<const T*>(a.w) + v0 * a.sw, a.sw, words};
    const bool direct = whole_pieces<T>(x.p, x.stride, a.K) && whole_pieces<T>(w.p, w.stride, a.K);
    const GArgs q{a.labels, a.lse, a.dloss, scale, v0, a.V, p.piece, p.m_pad, at + p.g, at + p.gt};
    // the products' long axes: this piece's words, and the rows, in whole steps
    if (p.logits.splits > 1) {
      e = few_logits<T>(a, p, x, w, direct, at + p.few, st);
      if (e != hipSuccess) return e;
      const void* const logits = at + p.few;
      e = start(xent_few_grad<T>, dim3((unsigned)parts(p.m_pad * p.piece, 256)), 256, st, logits,
                p.logits.splits, a.M, q);
    } else {
      e = by_tiles<T>(p.logits.tiles, [&](auto shape) {
        typedef decltype(shape) S;
        const Tiles t = tiles_of<S>(p.m_pad, p.piece, a.K, 1);
        return start(direct ? xent_grad<S, true> : xent_grad<S, false>,
                     dim3((unsigned)(t.m * t.n)), S::kThreads, st, x, w, t, q);
      });
    }
    if (e != hipSuccess) return e;
    if (a.dw) {
      const Rows gt{at + p.gt, p.m_pad, words}, xt{at + p.xt, p.m_pad, a.K};
      T* const out = static_cast<T*>(a.dw) + v0 * a.K;
      const bool split = p.dw.splits > 1;
      e = by_tiles<T>(p.dw.tiles, [&](auto shape) {
        typedef decltype(shape) S;
        const Tiles t = tiles_of<S>(words, a.K, p.m_pad, p.dw.splits);
        return start(xent_product<S, true>, dim3((unsigned)(t.m * t.n * t.splits)), S::kThreads, st, gt,
                     xt, t, OutArgs{split ? nullptr : out, at + p.dw_sums, of_dw, false});
      });
      if (e != hipSuccess) return e;
      if (split) {
        e = sum_up<T>(at + p.dw_sums, words * a.K, a.K, p.dw.splits, of_dw, out, st);
        if (e != hipSuccess) return e;
      }
    }
    if (a.dx) {
      e = start(xent_turn<T, false>,
                dim3((unsigned)(parts(p.piece, kTurn) * parts(a.K, kTurn))), 256, st, w, a.K,
                p.piece, at + p.wt, a.labels, a.dloss, a.V);
      if (e != hipSuccess) return e;
      const Rows g{at + p.g, p.piece, a.M}, wt{at + p.wt, p.piece, a.K};
      e = by_tiles<T>(p.dx.tiles, [&](auto shape) {
        typedef decltype(shape) S;
        const Tiles t = tiles_of<S>(a.M, a.K, p.piece, p.dx.splits);
        return start(xent_product<S, true>, dim3((unsigned)(t.m * t.n * t.splits)), S::kThreads, st, g,
                     wt, t, OutArgs{p.dx_direct ? a.dx : nullptr, at + p.dx_sums, of_dx, v0 > 0});
      });
      if (e != hipSuccess) return e;
    }
  }
  if (a.dx && !p.dx_direct)
    return sum_up<T>(at + p.dx_sums, a.M * a.K, a.K, p.dx.splits, of_dx, a.dx, st);
  return hipSuccess;
}

}  // namespace
}  // namespace adst
