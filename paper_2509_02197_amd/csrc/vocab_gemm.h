// Products of matrices whose long axis is contiguous in both, C[m][n] = sum_k
// A[m][k] B[n][k], on the matrix cores, with what the cross entropy does to a
// tile of C before it leaves the registers (linear_cross_entropy.h).
//
// A workgroup computes BM x BN of C in steps of 128 bytes of k. A step's rows go
// to LDS by loads that write it directly, 16 bytes a lane, ST - 1 steps ahead; in LDS
// a row's eight pieces of 16 bytes are permuted by half the row's number, so that the
// reads of 16 neighbouring rows fall into all 64 banks. A wave's lane reads 16 bytes of
// a row of A and of B for each matrix instruction (four for F32, two for F64): lanes
// 16 q .. 16 q + 15 hold piece q of rows 0..15. The sum over k does not ask in which
// order the pieces' elements are taken as long as A and B agree.
#pragma once

#include "seq_common.h"
#include "token_kernels.h"

namespace adst {
namespace {

typedef float F4 __attribute__((ext_vector_type(4)));
typedef double D4 __attribute__((ext_vector_type(4)));
typedef uint32_t U4 __attribute__((ext_vector_type(4)));

// 16 x 16 of C from 16 rows' pieces of 16 bytes, in kParts instructions. at(lane, i): the row of
// a lane's value i; its column is lane % 16.
template <class T>
struct Tile;
template <>
struct Tile<bf16> {
  typedef F4 C;
  typedef bf16 V __attribute__((ext_vector_type(8)));
  static constexpr int kParts = 1;
  __device__ static C mul(U4 a, U4 b, C c, int) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(V, a),
                                                   __builtin_bit_cast(V, b), c, 0, 0, 0);
  }
  __device__ static int at(int lane, int i) { return lane / 16 * 4 + i; }
};
template <>
struct Tile<f16> {
  typedef F4 C;
  typedef f16 V __attribute__((ext_vector_type(8)));
  static constexpr int kParts = 1;
  __device__ static C mul(U4 a, U4 b, C c, int) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(V, a),
                                                  __builtin_bit_cast(V, b), c, 0, 0, 0);
  }
  __device__ static int at(int lane, int i) { return lane / 16 * 4 + i; }
};
template <>
struct Tile<float> {
  typedef F4 C;
  static constexpr int kParts = 4;
  __device__ static C mul(U4 a, U4 b, C c, int part) {
    const F4 x = __builtin_bit_cast(F4, a), y = __builtin_bit_cast(F4, b);
    return __builtin_amdgcn_mfma_f32_16x16x4f32(x[part], y[part], c, 0, 0, 0);
  }
  __device__ static int at(int lane, int i) { return lane / 16 * 4 + i; }
};
template <>
struct Tile<double> {
  typedef D4 C;
  typedef double V __attribute__((ext_vector_type(2)));
  static constexpr int kParts = 2;
  __device__ static C mul(U4 a, U4 b, C c, int part) {
    const V x = __builtin_bit_cast(V, a), y = __builtin_bit_cast(V, b);
    return __builtin_amdgcn_mfma_f64_16x16x4f64(x[part], y[part], c, 0, 0, 0);
  }
  __device__ static int at(int lane, int i) { return i * 4 + lane / 16; }
};

// A matrix whose rows are contiguous.
struct Rows {
  const void* p;
  int64_t stride;  // elements between rows
  int64_t n;       // rows
};

constexpr int kStepBytes = 128;
constexpr int kXcds = 8;
constexpr int kTileGroup = 8;  // rows of tiles that neighbouring workgroups go through together

// WM x WN waves, each MT x NT tiles of 16 x 16. ST steps in LDS.
template <class T_, int WM_, int WN_, int MT_, int NT_, int ST_>
struct GemmShape {
  typedef T_ T;
  static constexpr int WM = WM_, WN = WN_, MT = MT_, NT = NT_, ST = ST_;
  static constexpr int BM = WM * MT * 16, BN = WN * NT * 16, kThreads = 64 * WM * WN;
  static constexpr int kStep = kStepBytes / (int)sizeof(T);  // elements of k
  static constexpr int kStageBytes = (BM + BN) * kStepBytes;
  static constexpr int kLoads = kStageBytes / 16 / kThreads;  // of a thread, per step
  // Steps that are on their way in registers where they cannot go to LDS directly.
  static constexpr int kHold = BM * BN <= 64 * 64 ? 3 : BM * BN <= 128 * 128 ? 2 : 1;
  static_assert(kStageBytes % (16 * kThreads) == 0 && BM % 8 == 0, "");
  typename Tile<T>::C acc[MT][NT];
};

// The tile of a workgroup. Consecutive workgroups go to the XCDs in turn; each XCD
// takes a run of tiles, kTileGroup rows of them column after column, whose rows and
// columns its cache then holds.
struct TileAt {
  int64_t m, n;
};
__device__ inline TileAt tile_at(int64_t tiles_m, int64_t tiles_n, int64_t id) {
  const int64_t all = tiles_m * tiles_n, q = all / kXcds, r = all % kXcds;
  const int64_t xcd = id % kXcds, k = xcd * q + (xcd < r ? xcd : r) + id / kXcds;
  const int64_t per = kTileGroup * tiles_n, group = k / per, in = k % per;
  const int64_t first = group * kTileGroup;
  const int64_t height = tiles_m - first < kTileGroup ? tiles_m - first : kTileGroup;
  return {first + in % height, in / height};
}

__device__ inline uint32_t lds_at(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}

// Of a lane's row from the first of eight, in bytes.
template <bool DIRECT>
struct Offset {
  typedef int64_t type;
};
template <>
struct Offset<true> {
  typedef uint32_t type;
};

template <int N>
struct Behind {
  static constexpr int n = N;
};

// Steps first .. end of k into s.acc, for the tile whose first rows of A and B are m0, n0.
// DIRECT: k is whole steps, rows and their starts are multiples of 16 bytes, rows less than
// 2^28 bytes apart.
template <class S, bool DIRECT>
__device__ inline void multiply(S& s, char* lds, const Rows& A, const Rows& B, int64_t K,
                                int64_t m0, int64_t n0, int64_t first, int64_t end) {
  typedef typename S::T T;
  typedef Tile<T> C;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / S::WN, wn = wave % S::WN;
#pragma unroll
  for (int i = 0; i < S::MT; ++i)
#pragma unroll
    for (int j = 0; j < S::NT; ++j) s.acc[i][j] = typename C::C{0, 0, 0, 0};
  if (first >= end) return;

  // A load of a wave fills 8 rows of a step: lane l row l / 8, piece l % 8 of LDS, which
  // holds the row's piece (l % 8) ^ (row / 2 % 8). Rows beyond the matrix are read as its last
  // one, and their results are not used.
  constexpr int kWaves = S::kThreads / 64;
  static_assert(S::BM % (kWaves * 8) == 0 && kWaves % 2 == 0, "a load is of A or of B");
  const int row8 = lane >> 3, piece = (lane & 7) ^ (row8 >> 1 | (wave & 1) << 2);
  const char* from[S::kLoads];  // the first of the 8 rows, at step `first`
  typename Offset<DIRECT>::type offset[S::kLoads];
#pragma unroll
  for (int j = 0; j < S::kLoads; ++j) {
    const bool of_a = j < S::BM / (kWaves * 8);
    const Rows& X = of_a ? A : B;
    const int64_t r0 = (of_a ? m0 : n0 - S::BM) + (j * kWaves + wave) * 8;
    const int64_t row = r0 < X.n ? r0 : X.n - 1, left = X.n - 1 - row;
    const int down_to = row8 < left ? row8 : (int)left;
    from[j] = static_cast<const char*>(X.p) +
              (row * X.stride + first * S::kStep) * (int64_t)sizeof(T);
    offset[j] = (typename Offset<DIRECT>::type)(down_to * X.stride * (int64_t)sizeof(T) + piece * 16);
  }
  // What a lane reads: its row of 16 and, for each half of a step, the piece lane / 16.
  uint32_t at[2];
#pragma unroll
  for (int h = 0; h < 2; ++h)
    at[h] = (lane & 15) * kStepBytes + (((h * 4 + (lane >> 4)) ^ (lane >> 1 & 7)) * 16);
  // Two halves' pieces in registers where an instruction takes 16 bytes; the wider types
  // take 128 and 256 cycles for them, beside which a read is short.
  constexpr bool kAcross = DIRECT && C::kParts == 1;
  constexpr int kHalves = kAcross ? 2 : 1;
  U4 a[kHalves][S::MT], b[kHalves][S::NT];
  const auto read = [&](const char* stage, int half) {
    const int h = half % kHalves;
    stage += at[half];
#pragma unroll
    for (int j = 0; j < S::NT; ++j)
      b[h][j] = *reinterpret_cast<const U4*>(stage + (S::BM + (wn * S::NT + j) * 16) * kStepBytes);
#pragma unroll
    for (int i = 0; i < S::MT; ++i)
      a[h][i] = *reinterpret_cast<const U4*>(stage + (wm * S::MT + i) * 16 * kStepBytes);
  };
  const auto compute = [&](int half) {
    const int h = half % kHalves;
    // (an instruction's result is ready some instructions later: no two in a row share one)
#pragma unroll
    for (int part = 0; part < C::kParts; ++part)
#pragma unroll
      for (int i = 0; i < S::MT; ++i)
#pragma unroll
        for (int j = 0; j < S::NT; ++j) s.acc[i][j] = C::mul(a[h][i], b[h][j], s.acc[i][j], part);
  };
  if constexpr (DIRECT) {
    // While a half of a step is multiplied the next half is read from LDS, across the
    // barrier between steps too. (8192 x 8192 x 2048 bf16: 232 us, and 254
    // where they are read as they are used.)
    const uint32_t base = lds_at(lds);
    const auto request = [&](int stage) {
#pragma unroll
      for (int j = 0; j < S::kLoads; ++j) {
        const uint32_t to = base + stage * S::kStageBytes + (j * kWaves + wave) * 1024;
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                     : : "s"(to), "v"(offset[j]), "s"(from[j]) : "memory");
        from[j] += kStepBytes;
      }
    };
    // A step is in LDS when no more loads than those of the `behind` steps after it are under
    // way; and this wave has read all that it has asked LDS for.
    const auto arrived = [&](bool behind, auto steps) {
      if (behind)
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" : : "n"(decltype(steps)::n * S::kLoads)
                     : "memory");
      else
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" : : : "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" : : : "memory");
    };
#pragma unroll
    for (int k = 0; k < S::ST; ++k)
      if (first + k < end) request(k);
    arrived(first + S::ST <= end, Behind<S::ST - 1>());
    if (kAcross) read(lds, 0);
    int stage = 0;
    for (int64_t k = first; k < end; ++k) {
      const char* const here = lds + stage * S::kStageBytes;
      const int next = stage + 1 == S::ST ? 0 : stage + 1;
      if constexpr (kAcross) {
        read(here, 1);
        __builtin_amdgcn_sched_barrier(0);
        compute(0);
        __builtin_amdgcn_sched_barrier(0);
      } else {
        read(here, 0);
        compute(0);
        read(here, 1);
        compute(1);
      }
      if (k + 1 < end) {
        arrived(k + S::ST <= end, Behind<S::ST - 2>());
        if (k + S::ST < end) request(stage);  // every wave has read the step
        if (kAcross) read(lds + next * S::kStageBytes, 0);
      }
      if constexpr (kAcross) {
        __builtin_amdgcn_sched_barrier(0);
        compute(1);
      }
      stage = next;
    }
  } else {
    // Through registers, kHold steps ahead; two stages of LDS are in use.
    constexpr int D = S::kHold;
    Vec<T> hold[D][S::kLoads];
    const auto request = [&](Vec<T>(&to)[S::kLoads], int64_t k) {
#pragma unroll
      for (int j = 0; j < S::kLoads; ++j) {
        const int64_t left = K - k * S::kStep - piece * Vec<T>::N;
        to[j] = load_part(reinterpret_cast<const T*>(from[j] + offset[j]),
                          (int)(left < 0 ? 0 : left < Vec<T>::N ? left : Vec<T>::N));
        from[j] += kStepBytes;
      }
    };
#pragma unroll
    for (int d = 0; d < D; ++d)
      if (first + d < end) request(hold[d], first + d);
    char *here = lds, *other = lds + S::kStageBytes;
    for (int64_t k0 = first; k0 < end; k0 += D)
#pragma unroll
      for (int d = 0; d < D; ++d) {
        const int64_t k = k0 + d;
        if (k >= end) break;
#pragma unroll
        for (int j = 0; j < S::kLoads; ++j)
          *reinterpret_cast<U4*>(here + (j * kWaves + wave) * 1024 + lane * 16) =
              __builtin_bit_cast(U4, hold[d][j].v);
        if (k + D < end) request(hold[d], k + D);
        __syncthreads();  // and every wave has read the step before, whose stage is next
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          read(here, h);
          compute(h);
        }
        char* const next = other;
        other = here;
        here = next;
      }
  }
  __syncthreads();  // LDS is free
}

// f(tile row i, value r, tile column j) of a wave's tiles as rows of T in global memory, through
// LDS: to [row][column] from the workgroup's tile on, `rows` x `columns` of which exist, in whole
// vectors where the rows allow it. All of the workgroup's threads.
template <class S, class F>
__device__ inline void store_tile(char* lds, typename S::T* to, int64_t stride, int64_t rows,
                                  int64_t columns, F f) {
  typedef typename S::T T;
  typedef Tile<T> C;
  constexpr int kAll = S::BM * S::BN * (int)sizeof(T), kHave = S::ST * S::kStageBytes;
  constexpr int P = (kAll + kHave - 1) / kHave;  // parts of a wave's rows of tiles
  static_assert(S::MT % P == 0, "");
  constexpr int M = S::MT / P, N = Vec<T>::N, kPieces = S::BN / N;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wm = wave / S::WN, wn = wave % S::WN;
  // a row's pieces of 16 bytes are permuted by the number of its row of four
  const auto place = [](int row, int piece) {
    return (row * kPieces + (piece ^ (row / 4 % 4 * 2 % kPieces))) * 16;
  };
#pragma unroll
  for (int p = 0; p < P; ++p) {
    if (p > 0) __syncthreads();
#pragma unroll
    for (int i = 0; i < M; ++i)
#pragma unroll
      for (int j = 0; j < S::NT; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = (wm * M + i) * 16 + C::at(lane, r);
          const int column = (wn * S::NT + j) * 16 + (lane & 15);
          *reinterpret_cast<T*>(lds + place(row, column / N) + column % N * (int)sizeof(T)) =
              f(p * M + i, r, j);
        }
    __syncthreads();
    for (int k = threadIdx.x; k < S::BM / P * kPieces; k += S::kThreads) {
      const int row = k / kPieces, piece = k % kPieces;
      // the tile's row that this row of the part is
      const int of = row / (M * 16) * S::MT * 16 + p * M * 16 + row % (M * 16);
      const int64_t left = columns - piece * N;
      if (of >= rows || left <= 0) continue;
      Vec<T> v;
      v.v = __builtin_bit_cast(typename Vec<T>::type,
                               *reinterpret_cast<const U4*>(lds + place(row, piece)));
      store_part(to + of * stride + piece * N, v, (int)(left < N ? left : N));
    }
  }
}

}  // namespace
}  // namespace adst
