// Exchanges between lanes that the token operators' kernels use beside those of
// hip/hip_runtime.h: rows of two different registers.
#pragma once

#include <hip/hip_runtime.h>

namespace host_hip {

// The odd rows of a and the even rows of b change places: {a's even rows and, in the odd
// ones, b's even rows; a's odd rows in the even ones, and b's odd rows}.
inline Pair rows_swap(uint32_t a, uint32_t b, int row) {
  const int lane = group().now->index % 64;
  const uint64_t* v = lanes_meet((uint64_t)b << 32 | a);
  const int even = lane & ~row, odd = lane | row;
  return lane & row ? Pair{{(uint32_t)(v[even] >> 32), (uint32_t)(v[odd] >> 32)}}
                    : Pair{{(uint32_t)v[even], (uint32_t)v[odd]}};
}

}  // namespace host_hip

#undef __builtin_amdgcn_permlane16_swap
#define __builtin_amdgcn_permlane16_swap(a, b, x, y) host_hip::rows_swap(a, b, 16)
#undef __builtin_amdgcn_permlane32_swap
#define __builtin_amdgcn_permlane32_swap(a, b, x, y) host_hip::rows_swap(a, b, 32)
