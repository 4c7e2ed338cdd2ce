// What the matrix products use beside hip/hip_runtime.h and token_lanes.h: a wave's 16 x 16
// products from lanes' pieces of rows, and loads that write LDS, which are done at once.
#pragma once

#include "token_lanes.h"

namespace host_hip {

// c[i] += the product of row `row of i` of a and column lane % 16 of b, whose pieces of the long
// axis are in lanes 16 q + row. FOURS: a lane's values are every fourth row, else four
// neighbouring ones.
template <int N, bool FOURS, class V, class C>
C matrix_product(V a, V b, C c) {
  struct Both {
    V a, b;
  } mine{a, b};
  const int lane = group().now->index % 64;
  uint64_t at[64];
  std::memcpy(at, lanes_meet((uint64_t)(uintptr_t)&mine), sizeof(at));
  for (int i = 0; i < 4; ++i) {
    const int row = FOURS ? i * 4 + lane / 16 : lane / 16 * 4 + i;
    for (int q = 0; q < 4; ++q) {
      const Both& of_a = *reinterpret_cast<const Both*>(at[q * 16 + row]);
      const Both& of_b = *reinterpret_cast<const Both*>(at[q * 16 + lane % 16]);
      typedef decltype(c[0] + c[0]) A;
      if constexpr (N == 1) {
        c[i] += (A)of_a.a * (A)of_b.b;
      } else {
        for (int k = 0; k < N; ++k) c[i] += (A)of_a.a[k] * (A)of_b.b[k];
      }
    }
  }
  lanes_meet(0);  // every lane has read the others'
  return c;
}

inline char* lds = nullptr;
inline uint32_t lds_at(const void* p) {
  lds = static_cast<char*>(const_cast<void*>(p));
  return 0;
}
inline void load_lds(uint32_t to, const char* from) {
  std::memcpy(lds + to + group().now->index % 64 * 16, from, 16);
}

}  // namespace host_hip

#define __builtin_amdgcn_s_barrier() host_hip::threads_meet()
#define __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, x, y, z) \
  host_hip::matrix_product<8, false>(a, b, c)
#define __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, x, y, z) \
  host_hip::matrix_product<8, false>(a, b, c)
#define __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, x, y, z) \
  host_hip::matrix_product<1, false>(a, b, c)
#define __builtin_amdgcn_mfma_f64_16x16x4f64(a, b, c, x, y, z) \
  host_hip::matrix_product<1, true>(a, b, c)
