// Products of matrices whose long axis is contiguous in both, C[m][n] = sum_k
// A[m][k] B[n][k], on the matrix cores, with what the cross entropy does to a
// tile of C before it leaves the registers (linear_cross_entropy.h).
//
// A workgroup computes BM x BN of C in steps of 128 bytes of k. A step's rows go
// to LDS by loads that write it directly, 16 bytes a lane, one step ahead (ST - 1
// steps); in LDS a row's eight pieces of 16 bytes are permuted by the row's number, so
// that the reads of eight neighbouring rows fall into different banks. A wave's
// lane reads 16 bytes of a row of A and of B for each matrix instruction (four for
// F32, two for F64): lanes 16 q .. 16 q + 15 hold piece q of rows 0..15. The sum
// over k does not ask in which order the pieces' elements are taken as long as A
// and B agree.
#pragma once

#include "seq_common.h"
#include "token_kernels.h"

namespace adst {
namespace {

typedef float F4 __attribute__((ext_vector_type(4)));
typedef double D4 __attribute__((ext_vector_type(4)));
typedef uint32_t U4 __attribute__((ext_vector_type(4)));

// 16 x 16 of C from 16 rows' pieces of 16 bytes, in kParts instructions. at(lane, i): the row of a lane's
// value i; its column is lane % 16.
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

// Steps first .. end of k into s.acc, for the tile whose first rows of A and B are m0, n0.
// DIRECT: k is whole steps, rows and their starts are multiples of 16 bytes.
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
  // holds the row's piece (l % 8) ^ (l / 8).
  const int row8 = lane >> 3, piece = (lane & 7) ^ row8;
  const T* from[S::kLoads];
#pragma unroll
  for (int j = 0; j < S::kLoads; ++j) {
    const int r = (j * (S::kThreads / 64) + wave) * 8 + row8;
    const bool of_a = r < S::BM;
    const Rows& X = of_a ? A : B;
    const int64_t want = of_a ? m0 + r : n0 + r - S::BM;
    const int64_t row = want < X.n ? want : X.n - 1;  // beyond: any row, its results are not used
    from[j] = static_cast<const T*>(X.p) + row * X.stride + piece * (16 / (int)sizeof(T));
  }
  // What a lane reads: its row of 16 and, for each half of a step, the piece lane / 16.
  uint32_t read[2];
#pragma unroll
  for (int h = 0; h < 2; ++h)
    read[h] = (lane & 15) * kStepBytes + (((h * 4 + (lane >> 4)) ^ (lane & 7)) * 16);
  const auto compute = [&](const char* stage) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      U4 a[S::MT], b[S::NT];
#pragma unroll
      for (int j = 0; j < S::NT; ++j)
        b[j] = *reinterpret_cast<const U4*>(stage + read[h] +
                                            (S::BM + (wn * S::NT + j) * 16) * kStepBytes);
#pragma unroll
      for (int i = 0; i < S::MT; ++i)
        a[i] = *reinterpret_cast<const U4*>(stage + read[h] + (wm * S::MT + i) * 16 * kStepBytes);
      // (an instruction's result is ready some instructions later: no two in a row share one)
#pragma unroll
      for (int part = 0; part < C::kParts; ++part)
#pragma unroll
        for (int i = 0; i < S::MT; ++i)
#pragma unroll
          for (int j = 0; j < S::NT; ++j) s.acc[i][j] = C::mul(a[i], b[j], s.acc[i][j], part);
    }
  };
  if constexpr (DIRECT) {
    const uint32_t base = lds_at(lds);
    const auto request = [&](int64_t k, int stage) {
#pragma unroll
      for (int j = 0; j < S::kLoads; ++j) {
        const uint32_t to = base + stage * S::kStageBytes + (j * (S::kThreads / 64) + wave) * 1024;
        const T* const at = from[j] + k * S::kStep;
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                     : : "s"(to), "v"(at) : "memory");
      }
    };
    constexpr int kAhead = S::ST - 1;
    for (int k = 0; k < kAhead; ++k)
      if (first + k < end) request(first + k, k);
    int stage = 0;
    for (int64_t k = first; k < end; ++k) {
      // the step's loads are done when no more than those of the steps behind it are under
      // way; and this wave has read all of the step before, whose place is filled next
      if (k + kAhead - 1 < end && kAhead > 1)
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" : : "n"((kAhead - 1) * S::kLoads) : "memory");
      else
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" : : : "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" : : : "memory");
      const int free_stage = stage == 0 ? S::ST - 1 : stage - 1;
      if (k + kAhead < end) request(k + kAhead, free_stage);
      compute(lds + stage * S::kStageBytes);
      stage = stage + 1 == S::ST ? 0 : stage + 1;
    }
  } else {
    Vec<T> hold[S::kLoads];
    const auto request = [&](int64_t k) {
#pragma unroll
      for (int j = 0; j < S::kLoads; ++j) {
        const int64_t left = K - k * S::kStep - piece * Vec<T>::N;
        hold[j] = load_part(from[j] + k * S::kStep,
                            (int)(left < 0 ? 0 : left < Vec<T>::N ? left : Vec<T>::N));
      }
    };
    const auto put = [&](char* stage) {
#pragma unroll
      for (int j = 0; j < S::kLoads; ++j)
        *reinterpret_cast<U4*>(stage + (j * (S::kThreads / 64) + wave) * 1024 + lane * 16) =
            __builtin_bit_cast(U4, hold[j].v);
    };
    request(first);
    put(lds);
    for (int64_t k = first; k < end; ++k) {
      const int stage = (int)((k - first) & 1);
      __syncthreads();
      if (k + 1 < end) request(k + 1);
      compute(lds + stage * S::kStageBytes);
      if (k + 1 < end) put(lds + (stage ^ 1) * S::kStageBytes);
    }
  }
  __syncthreads();  // LDS is free
}

}  // namespace
}  // namespace adst
