// Layer norm over rows, its VJP, and the weights' gradients summed over rows.
//
// The forward reads x and writes y, the VJP reads x and dy and writes dx:
// HBM bandwidth bounds both. A row is held in the registers of a group of
// lanes, so that its mean, its spread about that mean (two passes, which lose
// nothing to a large mean) and its result need one read: 16 or 64 lanes of a
// wave, or the waves of a workgroup that join their sums through LDS. A group
// takes R rows at a time, to have their reads under way together and to wait
// once for their sums. The weights stay in registers over all of a
// workgroup's rows, and so do, in the VJP, the sums of dw and db of the
// group's columns; each workgroup writes its sums once, and a second kernel
// adds those of all workgroups. Their number, and so the order of all sums,
// depends on the sizes alone. In large calls the VJP's next rows are on their
// way to LDS while the ones before are worked on. Rows longer than the
// registers hold are read again for each pass (norm_fwd_long, norm_rev_long),
// from the caches mostly; the VJP of rows longer than its kernel holds with the
// sums reads x and dy again for them (norm_dw_long).
//
// Measured, forward and VJP with its sums: bf16 32768 x 2048 48 and 71 us (5.6
// and 5.7 TB/s), 16384 x 4096 50 and 74, 8192 x 8192 47 and 76, 4096 x 16384 48
// and 84, 2000 x 30001 60 and 174; F32 16384 x 2048 47 and 71, 8192 x 8192 91 and
// 145, 4096 x 16384 95 and 154, 1024 x 30000 68 and 144; F64 16384 x 2048 93 and
// 142, 4096 x 8000 99 and 242.

#include "seq_common.h"
#include "seq_kernels.h"
#include "seq_launch.h"

namespace adst {
namespace {

__device__ inline float sqrt_(float x) { return __builtin_sqrtf(x); }
__device__ inline double sqrt_(double x) { return __builtin_sqrt(x); }

// N values of W, at any element's address.
template <class W, int N>
struct Pack {
  typedef W type __attribute__((ext_vector_type(N)));
  typedef W unaligned __attribute__((ext_vector_type(N), aligned(sizeof(W))));
  type v;
};
template <class W, int N>
__device__ inline Pack<W, N> load_pack(const W* p, int n, W none) {
  Pack<W, N> r;
  if (p && n >= N) {
    r.v = *reinterpret_cast<const typename Pack<W, N>::unaligned*>(p);
    return r;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) r.v[i] = p && i < n ? p[i] : none;
  return r;
}

// Has the compiler keep 16-bit vectors as they are and unpack them again
// later: unpacked, they take twice the registers.
template <class T, int R, int K>
__device__ inline void keep_packed(Vec<T> (&x)[R][K]) {
  if constexpr (sizeof(T) == 2) {
    typedef uint32_t Four __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int k = 0; k < K; ++k) {
        Four w = __builtin_bit_cast(Four, x[r][k].v);
        asm volatile("" : "+v"(w));
        x[r][k].v = __builtin_bit_cast(typename Vec<T>::type, w);
      }
  }
}

// The compiler does not mix the vectors before with those after: their
// intermediate values share registers.
__device__ inline void one_at_a_time() { __builtin_amdgcn_sched_barrier(0); }
template <class W, int N, int K>
__device__ inline void keep_packed(Pack<W, N> (&w)[K]) {
  if constexpr (sizeof(W) == 2) {
    typedef uint32_t Words __attribute__((ext_vector_type(N / 2)));
#pragma unroll
    for (int k = 0; k < K; ++k) {
      Words x = __builtin_bit_cast(Words, w[k].v);
      asm volatile("" : "+v"(x));
      w[k].v = __builtin_bit_cast(typename Pack<W, N>::type, x);
    }
  }
}

// A workgroup of NT threads in groups of L lanes; a lane holds K vectors of
// each of R rows.
template <class T, int NT_, int L_, int K_, int R_>
struct Shape {
  typedef Acc<T> A;
  static constexpr int NT = NT_, L = L_, K = K_, R = R_;
  static constexpr int V = Vec<T>::N;
  static constexpr int G = NT / L;             // groups
  static constexpr int W = L > 64 ? L / 64 : 1;  // waves of a group
  static constexpr int kRows = G * R;          // rows of a workgroup at a time
};

// How rows are read and written: vectors at a row's end in part (PARTS), or
// all of them whole (WHOLE), then also with non-temporal hints (STREAM), and
// the next rows requested into LDS while the ones before are worked on (AHEAD).
enum Mode { PARTS, WHOLE, STREAM, AHEAD };

// A group's R rows, this lane's vectors of them: n[k] columns of the k-th,
// zeros beyond a row's end and the last row.
template <class S, Mode M, class T>
__device__ inline void load_rows(const void* base, int64_t stride, int64_t row, int64_t rows,
                                 const int (&n)[S::K], Vec<T> (&v)[S::R][S::K]) {
  const T* p = (const T*)base + row * stride + threadIdx.x % S::L * S::V;
#pragma unroll
  for (int r = 0; r < S::R; ++r)
#pragma unroll
    for (int k = 0; k < S::K; ++k) {
      v[r][k].v = typename Vec<T>::type{};
      if (row + r < rows && n[k] > 0) {
        const T* at = p + r * stride + k * S::L * S::V;
        if constexpr (M == STREAM)
          v[r][k].v = __builtin_nontemporal_load(
              reinterpret_cast<const typename Vec<T>::unaligned*>(at));
        else if constexpr (M == WHOLE) v[r][k] = load_vec(at);
        else v[r][k] = load_part(at, n[k]);
      }
    }
}
template <class S, Mode M, class T>
__device__ inline void store_row(void* base, int64_t row, int64_t columns,
                                 const int (&n)[S::K], const Vec<T> (&v)[S::K]) {
  T* p = (T*)base + row * columns + threadIdx.x % S::L * S::V;
#pragma unroll
  for (int k = 0; k < S::K; ++k)
    if (n[k] > 0) {
      T* at = p + k * S::L * S::V;
      if constexpr (M >= STREAM)
        __builtin_nontemporal_store(v[k].v, reinterpret_cast<typename Vec<T>::unaligned*>(at));
      else if constexpr (M == WHOLE) store_vec(at, v[k]);
      else store_part(at, v[k], n[k]);
    }
}

// Rows on their way through LDS, for AHEAD. Each wave has its own lanes' part
// of its rows there, R * K vectors of x and as many of dy, so that only its own
// wait counts. The compiler would wait for every request before any read of
// LDS and at every barrier; so LDS is read by instructions that it does not
// see as such, with their wait, and the barrier leaves the requests under way.
__device__ inline int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ inline void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
typedef uint32_t Words4 __attribute__((ext_vector_type(4)));
__device__ inline uint32_t lds_address(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}
// Four times 16 bytes, STEP apart.
template <int STEP>
__device__ inline void read_lds(uint32_t at, Words4 (&v)[4]) {
  asm volatile(
      "ds_read_b128 %0, %4\n\t"
      "ds_read_b128 %1, %4 offset:%5\n\t"
      "ds_read_b128 %2, %4 offset:%6\n\t"
      "ds_read_b128 %3, %4 offset:%7\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3])
      : "v"(at), "n"(STEP), "n"(2 * STEP), "n"(3 * STEP)
      : "memory");
}
__device__ inline void write_lds(uint32_t at, const float (&v)[2]) {
  typedef float Two __attribute__((ext_vector_type(2)));
  asm volatile("ds_write_b64 %0, %1" : : "v"(at), "v"(Two{v[0], v[1]}) : "memory");
}
__device__ inline void write_lds(uint32_t at, const float (&v)[4]) {
  typedef float Four __attribute__((ext_vector_type(4)));
  asm volatile("ds_write_b128 %0, %1" : : "v"(at), "v"(Four{v[0], v[1], v[2], v[3]}) : "memory");
}
// A value that no kernel of the launch writes, the same for the wave: through
// the scalar cache, whose loads do not queue behind the requests.
template <class A>
__device__ inline A uniform_load(const A* p) {
  return *(const __attribute__((address_space(4))) A*)p;
}
// Now, and not in the loop, where the wait would be for the requests too.
template <class W, int N, int K>
__device__ inline void wait_for(Pack<W, N> (&w)[K]) {
  typedef uint32_t Words __attribute__((ext_vector_type(N * sizeof(W) / 4)));
#pragma unroll
  for (int k = 0; k < K; ++k) {
    Words x = __builtin_bit_cast(Words, w[k].v);
    asm volatile("" : "+v"(x));
    w[k].v = __builtin_bit_cast(typename Pack<W, N>::type, x);
  }
}
// Until at most `later` of this wave's newest loads and stores are under way.
__device__ inline void wait_all_but(int later) {
  switch (later) {
    case 1: __builtin_amdgcn_s_waitcnt(0x0f71); break;
    case 2: __builtin_amdgcn_s_waitcnt(0x0f72); break;
    case 3: __builtin_amdgcn_s_waitcnt(0x0f73); break;
    case 4: __builtin_amdgcn_s_waitcnt(0x0f74); break;
    default: __builtin_amdgcn_s_waitcnt(0x0f70); break;
  }
}
template <class S, class T, bool USED>
struct Ahead {
  Words4 words[USED ? S::NT / 64 : 1][USED ? 2 * S::R * S::K : 1][64];
};
// Requests this lane's vectors of a group's rows; beyond a row's end and the
// last row, of the last ones that are there.
template <class S, class T>
__device__ inline void request_rows(const void* base, int64_t stride, int64_t row, int64_t rows,
                                    int64_t columns, Words4 (*slots)[64]) {
#pragma unroll
  for (int r = 0; r < S::R; ++r) {
    const T* p = (const T*)base + (row + r < rows ? row + r : rows - 1) * stride;
#pragma unroll
    for (int k = 0; k < S::K; ++k) {
      const int c = (k * S::L + (int)threadIdx.x % S::L) * S::V, end = (int)columns - S::V;
      __builtin_amdgcn_global_load_lds(
          (const __attribute__((address_space(1))) void*)(p + (c < end ? c : end)),
          (__attribute__((address_space(3))) void*)slots[r * S::K + k], 16, 0, 2);
    }
  }
}
// They arrive: x, then dy; zeros beyond a row's end and the last row.
template <class S, class T>
__device__ inline void take_rows(const Words4 (*slots)[64], int64_t row, int64_t rows,
                                 const int (&n)[S::K], Vec<T> (&x)[S::R][S::K],
                                 Vec<T> (&y)[S::R][S::K]) {
  constexpr int N = S::R * S::K;
  static_assert(N % 2 == 0);
  const uint32_t at = lds_address(slots) + (threadIdx.x & 63) * 16;
#pragma unroll
  for (int j = 0; j < 2 * N; j += 4) {
    Words4 v[4];
    read_lds<1024>(at + j * 1024, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = (j + i) % N / S::K, k = (j + i) % S::K;
      if (!(row + r < rows && n[k] > 0)) v[i] = Words4{};
      const auto got = __builtin_bit_cast(typename Vec<T>::type, v[i]);
      if (j + i < N) x[r][k].v = got;
      else y[r][k].v = got;
    }
  }
}

// Sums over a group, of N values each, in every lane. Calls alternate between
// two buffers, so that one barrier a call is enough.
template <class S, int N>
struct Sums {
  typename S::A part[2][S::G][S::W][N];
};
template <class S, int N, Mode M = PARTS>
__device__ inline void group_sum(Sums<S, N>& sm, int& turn, typename S::A (&v)[N]) {
#pragma unroll
  for (int r = 0; r < N; ++r) v[r] = lane_sum<(S::L < 64 ? S::L : 64)>(v[r]);
  if constexpr (S::W > 1) {
    const int g = threadIdx.x / S::L, w = threadIdx.x % S::L / 64;
    if ((threadIdx.x & 63) == 0) {
      if constexpr (M == AHEAD) {
        write_lds(lds_address(&sm.part[turn][g][w][0]), v);
      } else {
#pragma unroll
        for (int r = 0; r < N; ++r) sm.part[turn][g][w][r] = v[r];
      }
    }
    if constexpr (M == AHEAD) {
      static_assert(S::W * N % 16 == 0);
      meet();
      const uint32_t at = lds_address(&sm.part[turn][g][0][0]);
#pragma unroll
      for (int r = 0; r < N; ++r) v[r] = 0;
#pragma unroll
      for (int j = 0; j < S::W * N; j += 16) {
        Words4 p[4];
        read_lds<16>(at + j * 4, p);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const uint32_t word = p[i / 4][i % 4];
          const float f = __builtin_bit_cast(float, word);
          if (j + i < N) v[i] = f;
          else v[(j + i) % N] += f;
        }
      }
      turn ^= 1;
      return;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < N; ++r) {
      v[r] = sm.part[turn][g][0][r];
#pragma unroll
      for (int k = 1; k < S::W; ++k) v[r] += sm.part[turn][g][k][r];
    }
    turn ^= 1;
  }
}

template <class T, class W, int NT, int L, int K, int R_, Mode M>
__global__ __launch_bounds__(NT) void norm_fwd(NormArgs p) {
  typedef Shape<T, NT, L, K, R_> S;
  typedef typename S::A A;
  constexpr int V = S::V, R = S::R;
  __shared__ Sums<S, R> sm;
  int turn = 0;
  const int lane = threadIdx.x % L, group = threadIdx.x / L;
  constexpr bool kHoldsWeights = K < 8;
  int n[K];  // columns of each of this lane's vectors
  Pack<W, V> w[K], b[K];
  const auto weights = [&](int k) {
    const int64_t c = (int64_t)(k * L + lane) * V;
    w[k] = load_pack<W, V>(p.w ? (const W*)p.w + c : nullptr, n[k], W(1));
    b[k] = load_pack<W, V>(p.b ? (const W*)p.b + c : nullptr, n[k], W(0));
  };
#pragma unroll
  for (int k = 0; k < K; ++k) {
    n[k] = (int)min((int64_t)V, p.n - (int64_t)(k * L + lane) * V);
    if (kHoldsWeights) weights(k);
  }
  const A inv = A(1) / A(p.n);
  for (int64_t row0 = (int64_t)blockIdx.x * S::kRows; row0 < p.rows;
       row0 += (int64_t)gridDim.x * S::kRows) {
    const int64_t row = row0 + group * R;
    Vec<T> x[R][K];
    A s[R], mean[R];
    load_rows<S, M>(p.x, p.sx, row, p.rows, n, x);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      s[r] = A(0);
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) s[r] += up(x[r][k].v[i]);
    }
    keep_packed(x);
    group_sum<S>(sm, turn, s);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      mean[r] = s[r] * inv;
      s[r] = A(0);
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const A d = (M != PARTS ? n[k] > 0 : i < n[k]) ? up(x[r][k].v[i]) - mean[r] : A(0);
          s[r] = fma_(d, d, s[r]);
        }
    }
    keep_packed(x);
    group_sum<S>(sm, turn, s);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (row + r >= p.rows) continue;
      const A rstd = A(1) / sqrt_(s[r] * inv + A(p.eps));
#pragma unroll
      for (int k = 0; k < K; ++k) {
        if (!kHoldsWeights) weights(k);
#pragma unroll
        for (int i = 0; i < V; ++i)
          x[r][k].v[i] = down<T>(fma_((up(x[r][k].v[i]) - mean[r]) * rstd, (A)up(w[k].v[i]),
                                      (A)up(b[k].v[i])));
      }
      store_row<S, M>(p.y, row + r, p.n, n, x[r]);
      if (lane == 0) {
        if (p.mean) ((A*)p.mean)[row + r] = mean[r];
        if (p.rstd) ((A*)p.rstd)[row + r] = rstd;
      }
    }
  }
}

// dx (where asked for), and with SUMS and where part is given this workgroup's
// sums of dw and db in part[blockIdx.x][2][n].
template <class T, class W, int NT, int L, int K, int R_, Mode M, bool SUMS>
__global__ __launch_bounds__(NT) void norm_rev(NormArgs p, Acc<T>* part) {
  typedef Shape<T, NT, L, K, R_> S;
  typedef typename S::A A;
  constexpr int V = S::V, R = S::R;
  __shared__ alignas(M == AHEAD ? 16 : sizeof(A)) Sums<S, 2 * R> sm;
  int turn = 0;
  const int lane = threadIdx.x % L, group = threadIdx.x / L;
  int n[K];
  Pack<W, V> w[K];
  A dw[K][V], db[K][V];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int64_t c = (int64_t)(k * L + lane) * V;
    n[k] = (int)min((int64_t)V, p.n - c);
    w[k] = load_pack<W, V>(p.w ? (const W*)p.w + c : nullptr, n[k], W(1));
#pragma unroll
    for (int i = 0; i < V; ++i) dw[k][i] = db[k][i] = A(0);
  }
  if constexpr (M == AHEAD) wait_for(w);
  const A inv = A(1) / A(p.n);
  __shared__ Ahead<S, T, M == AHEAD> ahead;
  Words4 (*const slots)[64] =
      ahead.words[M == AHEAD ? uniform((int)threadIdx.x / 64) : 0];
  A next_mean[R], next_rstd[R];
  int stores = 0;  // of this wave since its last request
  const auto request = [&](int64_t row) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t at = row + r < p.rows ? row + r : p.rows - 1;
      next_mean[r] = uniform_load((const A*)p.mean + at);
      next_rstd[r] = uniform_load((const A*)p.rstd + at);
    }
    request_rows<S, T>(p.x, p.sx, row, p.rows, p.n, slots);
    request_rows<S, T>(p.dy, p.sdy, row, p.rows, p.n, slots + R * K);
  };
  if constexpr (M == AHEAD)
    if ((int64_t)blockIdx.x * S::kRows < p.rows)
      request((int64_t)blockIdx.x * S::kRows + uniform(group) * R);
  for (int64_t row0 = (int64_t)blockIdx.x * S::kRows; row0 < p.rows;
       row0 += (int64_t)gridDim.x * S::kRows) {
    const int64_t row = row0 + (M == AHEAD ? uniform(group) : group) * R;
    Vec<T> x[R][K], y[R][K];
    A s[2 * R], mean[R], rstd[R];  // sums of e, then of e * xhat
    if constexpr (M == AHEAD) {
      wait_all_but(stores);
      take_rows<S, T>(slots, row, p.rows, n, x, y);
#pragma unroll
      for (int r = 0; r < R; ++r) mean[r] = next_mean[r], rstd[r] = next_rstd[r];
      if (row0 + (int64_t)gridDim.x * S::kRows < p.rows)
        request(row + (int64_t)gridDim.x * S::kRows);
      stores = 0;
    } else {
      load_rows<S, M>(p.x, p.sx, row, p.rows, n, x);
      load_rows<S, M>(p.dy, p.sdy, row, p.rows, n, y);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        mean[r] = row + r < p.rows ? ((const A*)p.mean)[row + r] : A(0);
        rstd[r] = row + r < p.rows ? ((const A*)p.rstd)[row + r] : A(0);
      }
    }
    // columns beyond the end have dy = 0 and add nothing; rows beyond it too
#pragma unroll
    for (int r = 0; r < R; ++r) {
      s[r] = s[R + r] = A(0);
#pragma unroll
      for (int k = 0; k < K; ++k) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const A d = up(y[r][k].v[i]), h = (up(x[r][k].v[i]) - mean[r]) * rstd[r];
          const A e = d * (A)up(w[k].v[i]);
          s[r] += e;
          s[R + r] = fma_(e, h, s[R + r]);
          if (SUMS) {
            dw[k][i] = fma_(d, h, dw[k][i]);
            db[k][i] += d;
          }
        }
        one_at_a_time();
      }
    }
    if (!p.dx) continue;
    keep_packed(x);
    keep_packed(y);
    keep_packed(w);
    group_sum<S, 2 * R, M>(sm, turn, s);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (row + r >= p.rows) continue;
      const A ms = s[r] * inv, mq = s[R + r] * inv;
#pragma unroll
      for (int k = 0; k < K; ++k) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const A h = (up(x[r][k].v[i]) - mean[r]) * rstd[r];
          const A e = up(y[r][k].v[i]) * (A)up(w[k].v[i]);
          x[r][k].v[i] = down<T>(fma_(-mq, h, e - ms) * rstd[r]);
        }
        one_at_a_time();
      }
      store_row<S, M>(p.dx, row + r, p.n, n, x[r]);
      if constexpr (M == AHEAD) {
#pragma unroll
        for (int k = 0; k < K; ++k) stores += uniform(n[k]) > 0;
      }
    }
    keep_packed(w);
  }
  if constexpr (SUMS) {
    if (!part) return;
    // The groups' sums (of 16 lanes: first the wave's four), added in their
    // order through LDS.
    constexpr int kShare = L < 64 ? 64 : L, kShares = NT / kShare;
    A* const out = part + (int64_t)blockIdx.x * 2 * p.n;
    if constexpr (L < 64) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        dw[0][i] = sum_rows(dw[0][i]);
        db[0][i] = sum_rows(db[0][i]);
      }
    }
    const int share = threadIdx.x / kShare;
    if constexpr (kShares > 1) {
      __shared__ A total[kShares][L * K * V];
#pragma unroll
      for (int which = 0; which < 2; ++which) {
        __syncthreads();
        if (L >= 64 || (threadIdx.x & 63) < L) {
#pragma unroll
          for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i)
              total[share][(k * L + lane) * V + i] = which ? db[k][i] : dw[k][i];
        }
        __syncthreads();
        for (int c = threadIdx.x; c < p.n; c += NT) {
          A t = total[0][c];
#pragma unroll
          for (int g = 1; g < kShares; ++g) t += total[g][c];
          out[which * p.n + c] = t;
        }
      }
    } else {
      // whole vectors: value by value a wave's store touches 16 lines, and the
      // VJP of 4096 x 16384 f16 took 105 us, of 32 such rows 24 (now 92 and 12)
      constexpr int N = Vec<A>::N;
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < V; i += N) {
          A* const at = out + (k * L + lane) * V + i;
          Vec<A> sw, sb;
#pragma unroll
          for (int j = 0; j < N; ++j) sw.v[j] = dw[k][i + j], sb.v[j] = db[k][i + j];
          store_part(at, sw, n[k] - i);
          store_part(at + p.n, sb, n[k] - i);
        }
    }
  }
}

// Rows of any length, read again for each pass; a workgroup a row at a time.
constexpr int kLongThreads = 1024;
template <class T>
struct LongShape : Shape<T, kLongThreads, kLongThreads, 1, 1> {};

template <class T, class W>
__global__ __launch_bounds__(kLongThreads) void norm_fwd_long(NormArgs p) {
  typedef LongShape<T> S;
  typedef typename S::A A;
  constexpr int V = S::V;
  __shared__ Sums<S, 1> sm;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
    const T* x = (const T*)p.x + row * p.sx;
    T* y = (T*)p.y + row * p.n;
    A s[1] = {A(0)};
    for (int64_t c = threadIdx.x * V; c < p.n; c += kLongThreads * V) {
      const Vec<T> v = load_part(x + c, (int)min((int64_t)V, p.n - c));
#pragma unroll
      for (int i = 0; i < V; ++i) s[0] += up(v.v[i]);
    }
    group_sum<S>(sm, turn, s);
    const A mean = s[0] / A(p.n);
    s[0] = A(0);
    for (int64_t c = threadIdx.x * V; c < p.n; c += kLongThreads * V) {
      const int n = (int)min((int64_t)V, p.n - c);
      const Vec<T> v = load_part(x + c, n);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const A d = i < n ? up(v.v[i]) - mean : A(0);
        s[0] = fma_(d, d, s[0]);
      }
    }
    group_sum<S>(sm, turn, s);
    const A rstd = A(1) / sqrt_(s[0] / A(p.n) + A(p.eps));
    for (int64_t c = threadIdx.x * V; c < p.n; c += kLongThreads * V) {
      const int n = (int)min((int64_t)V, p.n - c);
      Vec<T> v = load_part(x + c, n);
      const Pack<W, V> w = load_pack<W, V>(p.w ? (const W*)p.w + c : nullptr, n, W(1));
      const Pack<W, V> b = load_pack<W, V>(p.b ? (const W*)p.b + c : nullptr, n, W(0));
#pragma unroll
      for (int i = 0; i < V; ++i)
        v.v[i] = down<T>(fma_((up(v.v[i]) - mean) * rstd, (A)up(w.v[i]), (A)up(b.v[i])));
      store_part(y + c, v, n);
    }
    if (threadIdx.x == 0) {
      if (p.mean) ((A*)p.mean)[row] = mean;
      if (p.rstd) ((A*)p.rstd)[row] = rstd;
    }
  }
}

template <class T, class W>
__global__ __launch_bounds__(kLongThreads) void norm_rev_long(NormArgs p) {
  typedef LongShape<T> S;
  typedef typename S::A A;
  constexpr int V = S::V;
  __shared__ Sums<S, 2> sm;
  int turn = 0;
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
    const T* x = (const T*)p.x + row * p.sx;
    const T* dy = (const T*)p.dy + row * p.sdy;
    T* dx = (T*)p.dx + row * p.n;
    const A mean = ((const A*)p.mean)[row], rstd = ((const A*)p.rstd)[row];
    A s[2] = {A(0), A(0)};
    for (int64_t c = threadIdx.x * V; c < p.n; c += kLongThreads * V) {
      const int n = (int)min((int64_t)V, p.n - c);
      const Vec<T> v = load_part(x + c, n), d = load_part(dy + c, n);
      const Pack<W, V> w = load_pack<W, V>(p.w ? (const W*)p.w + c : nullptr, n, W(1));
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const A e = up(d.v[i]) * (A)up(w.v[i]);
        s[0] += e;
        s[1] = fma_(e, (up(v.v[i]) - mean) * rstd, s[1]);
      }
    }
    group_sum<S>(sm, turn, s);
    const A ms = s[0] / A(p.n), mq = s[1] / A(p.n);
    for (int64_t c = threadIdx.x * V; c < p.n; c += kLongThreads * V) {
      const int n = (int)min((int64_t)V, p.n - c);
      Vec<T> v = load_part(x + c, n);
      const Vec<T> d = load_part(dy + c, n);
      const Pack<W, V> w = load_pack<W, V>(p.w ? (const W*)p.w + c : nullptr, n, W(1));
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const A h = (up(v.v[i]) - mean) * rstd, e = up(d.v[i]) * (A)up(w.v[i]);
        v.v[i] = down<T>(fma_(-mq, h, e - ms) * rstd);
      }
      store_part(dx + c, v, n);
    }
  }
}

// The same rows' sums of dw and db: a vector of columns a thread, of the rows
// blockIdx.y, + gridDim.y, ...
constexpr int kColumnThreads = 64;
template <class T>
__global__ __launch_bounds__(kColumnThreads) void norm_dw_long(NormArgs p, Acc<T>* part) {
  typedef Acc<T> A;
  constexpr int V = Vec<T>::N;
  const int64_t c = ((int64_t)blockIdx.x * kColumnThreads + threadIdx.x) * V;
  const int n = (int)min((int64_t)V, p.n - c);
  if (n <= 0) return;
  A sw[V], sb[V];
#pragma unroll
  for (int i = 0; i < V; ++i) sw[i] = sb[i] = A(0);
#pragma unroll 4
  for (int64_t row = blockIdx.y; row < p.rows; row += gridDim.y) {
    const Vec<T> v = load_part((const T*)p.x + row * p.sx + c, n);
    const Vec<T> d = load_part((const T*)p.dy + row * p.sdy + c, n);
    const A mean = ((const A*)p.mean)[row], rstd = ((const A*)p.rstd)[row];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      sw[i] = fma_(up(d.v[i]), (up(v.v[i]) - mean) * rstd, sw[i]);
      sb[i] += up(d.v[i]);
    }
  }
  A* const out = part + (int64_t)blockIdx.y * 2 * p.n + c;
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (i < n) out[i] = sw[i], out[p.n + i] = sb[i];
}

// dw and db from the workgroups' sums, from column `first` on (of dw's columns,
// then db's): 32 columns a workgroup, 32 shares of the parts.
constexpr int kSumColumns = 32, kShares = 32;
template <class T, class W>
__global__ __launch_bounds__(kSumColumns * kShares) void norm_dw_sum(NormArgs p,
                                                                     const Acc<T>* part,
                                                                     int parts, int64_t first) {
  typedef Acc<T> A;
  __shared__ A sums[kShares][kSumColumns];
  const int column = threadIdx.x % kSumColumns, share = threadIdx.x / kSumColumns;
  const int64_t c = first + (int64_t)blockIdx.x * kSumColumns + column;
  A s = A(0);
  if (c < 2 * p.n) {
    const int each = (parts + kShares - 1) / kShares;
    const int from = share * each, to = min(from + each, parts);
#pragma unroll 16
    for (int k = from; k < to; ++k) s += part[(int64_t)k * 2 * p.n + c];
  }
  sums[share][column] = s;
  __syncthreads();
  if (share > 0 || c >= 2 * p.n) return;
#pragma unroll
  for (int k = 1; k < kShares; ++k) s += sums[k][column];
  if (c < p.n) {
    if (p.dw) ((W*)p.dw)[c] = down<W>((Acc<W>)s);
  } else if (p.db) {
    ((W*)p.db)[c - p.n] = down<W>((Acc<W>)s);
  }
}

// -------------------------------------------------------------- on the host
template <class F>
hipError_t by_type(int32_t dtype, int32_t wtype, F f) {
  switch (dtype) {
    case ADST_F64: return f(double(), double());
    case ADST_F32: return f(float(), float());
    case ADST_BF16: return wtype == ADST_F32 ? f(bf16(), float()) : f(bf16(), bf16());
    default: return wtype == ADST_F32 ? f(f16(), float()) : f(f16(), f16());
  }
}

int64_t vectors_of(int32_t dtype, int64_t n) {
  const int64_t v = dtype == ADST_F64 ? 2 : dtype == ADST_F32 ? 4 : 8;
  return (n + v - 1) / v;
}
// Vectors of a row that one kernel of the VJP takes with the sums of dw and db:
// what its registers hold (a few of F16 and F64 are 2 to 8 of 128 short), and of
// F32 twice as many. There the weights and both sums beside x and dy leave 13
// (rows requested ahead) to 75 (PARTS) registers to scratch memory, which costs
// less than a second kernel that reads x and dy again: 4096 x 16384 154 us, 297
// with two; 2000 x 9001 67 and 114.
int64_t held_in_vjp(int32_t dtype) { return dtype == ADST_F32 ? 4096 : 2048; }

// Non-temporal accesses where a call moves more than the caches keep for the
// next one (32768 x 2048 bf16: forward 47 us against 49, VJP 77 against 83).
constexpr int64_t kStreamBytes = int64_t(128) << 20;
Mode mode_of(const NormArgs& a, int64_t size, int64_t arrays) {
  if (a.n % (16 / size) != 0) return PARTS;
  return a.rows * a.n * size * arrays >= kStreamBytes ? STREAM : WHOLE;
}

// Workgroups of the forward: enough to fill the chip several times over, each
// with several rows to keep its weights for.
template <class T, class W, int NT, int L, int K, int R>
hipError_t forward(const NormArgs& a, hipStream_t st) {
  const int64_t per = (int64_t)NT / L * R, all = (a.rows + per - 1) / per;
  const int64_t most = 256 * 2048 / NT;
  const unsigned grid = (unsigned)(all < most ? all : most);
  const Mode m = mode_of(a, sizeof(T), 2);
  return start(m == PARTS   ? norm_fwd<T, W, NT, L, K, R, PARTS>
               : m == WHOLE ? norm_fwd<T, W, NT, L, K, R, WHOLE>
                            : norm_fwd<T, W, NT, L, K, R, STREAM>,
               grid, NT, st, a);
}
unsigned long_grid(int64_t rows) { return (unsigned)(rows < 4096 ? rows : 4096); }
template <class T, class W>
hipError_t forward_by_length(const NormArgs& a, int64_t nv, hipStream_t st) {
  if (nv <= 16) return forward<T, W, 256, 16, 1, 2>(a, st);
  if (nv <= 64) return forward<T, W, 256, 64, 1, 4>(a, st);
  if (nv <= 128) return forward<T, W, 256, 64, 2, 2>(a, st);
  if (nv <= 256) return forward<T, W, 256, 64, 4, 1>(a, st);
  if (nv <= 512) return forward<T, W, 256, 256, 2, 1>(a, st);
  if (nv <= 1024) return forward<T, W, 256, 256, 4, 1>(a, st);
  if (nv <= 2048) return forward<T, W, 512, 512, 4, 1>(a, st);
  if (nv <= 4096) return forward<T, W, 1024, 1024, 4, 1>(a, st);
  // eight vectors of a row and their weights are 24 registers more than there
  // are: neither this nor reading the row again is the faster throughout (1024 x
  // 30000 68 us and 75, 1000 x 30001 76 and 72, 2000 x 20000 96 and 88)
  if constexpr (sizeof(T) == 4)
    if (nv <= 8192) return forward<T, W, 1024, 1024, 8, 1>(a, st);
  return start(norm_fwd_long<T, W>, long_grid(a.rows), kLongThreads, st, a);
}

// Groups of rows that sum dw and db apart.
constexpr int kParts = 512, kLongParts = 128;
int parts_of(int32_t dtype, int64_t rows, int64_t nv) {
  // rows that the VJP's workgroups take at a time (reverse_by_length)
  const int64_t at_once = nv <= 16 ? 64 : nv <= 64 ? 32 : nv <= 128 ? 16
                          : nv <= 512 ? 4 : nv <= 1024 ? 2 : 1;
  const int64_t all = (rows + at_once - 1) / at_once;
  const int64_t most = nv > held_in_vjp(dtype) ? kLongParts : nv > 256 ? kParts / 2 : kParts;
  return (int)(all < most ? all : most);
}

// Rows requested ahead of their use, where a workgroup joins its sums through
// LDS and so has all its waves wait at the same time, and the requests' 16 bytes
// are aligned (VJP in bf16 with, without: 32768 x 2048 71 and 74 us, 16384 x 4096
// 74 and 81, 8192 x 8192 76 and 81, 4096 x 16384 84 and 92). A second turn of
// rows under way gained nothing more.
template <class T, int L, int K, int R>
constexpr bool kAheadFits = sizeof(T) < 8 && L >= 256 && R * K <= 4;
bool requests(const NormArgs& a) {
  const int64_t e = a.dtype == ADST_F32 ? 4 : 2;
  return (((int64_t)(uintptr_t)a.x | (int64_t)(uintptr_t)a.dy | a.sx * e | a.sdy * e) & 15) == 0;
}

template <class T, class W, int NT, int L, int K, int R, bool SUMS>
hipError_t reverse_sums(const NormArgs& a, unsigned grid, Acc<T>* part, hipStream_t st) {
  const Mode m = mode_of(a, sizeof(T), 3);
  if constexpr (kAheadFits<T, L, K, R>)
    if (m == STREAM && requests(a))
      return start(norm_rev<T, W, NT, L, K, R, AHEAD, SUMS>, grid, NT, st, a, part);
  return start(m == PARTS   ? norm_rev<T, W, NT, L, K, R, PARTS, SUMS>
               : m == WHOLE ? norm_rev<T, W, NT, L, K, R, WHOLE, SUMS>
                            : norm_rev<T, W, NT, L, K, R, STREAM, SUMS>,
               grid, NT, st, a, part);
}
template <class T, class W, int NT, int L, int K, int R>
hipError_t reverse(const NormArgs& a, unsigned grid, Acc<T>* part, hipStream_t st) {
  return reverse_sums<T, W, NT, L, K, R, true>(a, grid, part, st);
}

template <class T, class W>
hipError_t reverse_by_length(const NormArgs& a, int64_t nv, int parts, Acc<T>* part, hipStream_t st) {
  const unsigned g = (unsigned)parts;
  if (nv <= 16) return reverse<T, W, 512, 16, 1, 2>(a, g, part, st);
  if (nv <= 64) return reverse<T, W, 512, 64, 1, 4>(a, g, part, st);
  if (nv <= 128) return reverse<T, W, 512, 64, 2, 2>(a, g, part, st);
  if (nv <= 256) return reverse<T, W, 512, 256, 1, 2>(a, g, part, st);
  if (nv <= 512) return reverse<T, W, 1024, 512, 1, 2>(a, g, part, st);
  if (nv <= 1024) return reverse<T, W, 1024, 512, 2, 1>(a, g, part, st);
  if (nv <= 2048) return reverse<T, W, 512, 512, 4, 1>(a, g, part, st);
  if constexpr (sizeof(T) == 4)
    if (nv <= held_in_vjp(a.dtype)) return reverse<T, W, 1024, 1024, 4, 1>(a, g, part, st);
  // dx without the sums' registers, as long as those hold the row (of F32's eight
  // vectors but 64 of 128: 1024 x 30000 144 us, 149 with norm_rev_long)
  hipError_t e = hipSuccess;
  if (a.dx) {
    const unsigned rows = long_grid(a.rows);
    constexpr int K = sizeof(T) == 4 ? 8 : 4;
    e = nv <= K * 1024 ? reverse_sums<T, W, 1024, 1024, K, 1, false>(a, rows, nullptr, st)
                       : start(norm_rev_long<T, W>, rows, kLongThreads, st, a);
  }
  if (e != hipSuccess || !part) return e;
  const unsigned columns = (unsigned)((nv + kColumnThreads - 1) / kColumnThreads);
  return start(norm_dw_long<T>, dim3(columns, g), kColumnThreads, st, a, part);
}

}  // namespace

hipError_t norm_forward(const NormArgs& a, hipStream_t st) {
  const int64_t nv = vectors_of(a.dtype, a.n);
  return by_type(a.dtype, a.wtype, [&](auto t, auto w) {
    return forward_by_length<decltype(t), decltype(w)>(a, nv, st);
  });
}

uint64_t norm_workspace_bytes(int32_t dtype, int64_t rows, int64_t n) {
  const uint64_t parts = (uint64_t)parts_of(dtype, rows, vectors_of(dtype, n));
  return 2 * parts * (uint64_t)n * (dtype == ADST_F64 ? 8 : 4);
}

hipError_t norm_vjp(const NormArgs& a, void* ws, hipStream_t st) {
  const int64_t nv = vectors_of(a.dtype, a.n);
  const int parts = parts_of(a.dtype, a.rows, nv);
  const bool sums = a.dw || a.db;
  return by_type(a.dtype, a.wtype, [&](auto t, auto w) {
    typedef decltype(t) T;
    typedef decltype(w) W;
    Acc<T>* const part = sums ? (Acc<T>*)ws : nullptr;
    hipError_t e = parts > 0 ? reverse_by_length<T, W>(a, nv, parts, part, st) : hipSuccess;
    if (!sums) return e;
    // a launch has fewer than 2^32 threads
    constexpr int64_t kMostGroups = (int64_t(1) << 32) / (kSumColumns * kShares) - 1;
    const int64_t groups = (2 * a.n + kSumColumns - 1) / kSumColumns;
    for (int64_t done = 0; e == hipSuccess && done < groups; done += kMostGroups) {
      const int64_t now = groups - done < kMostGroups ? groups - done : kMostGroups;
      e = start(norm_dw_sum<T, W>, (unsigned)now, kSumColumns * kShares, st, a, part, parts,
                done * kSumColumns);
    }
    return e;
  });
}

}  // namespace adst
