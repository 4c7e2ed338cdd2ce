// Checks of arguments that the C boundaries of the sequence and token operators
// share (seq_abi.cpp, token_abi.cpp).
#pragma once

#include <hip/hip_runtime_api.h>

#include <cmath>
#include <cstdarg>
#include <cstdint>
#include <cstdio>

#include "adst.h"
#include "errors.h"

namespace adst {
namespace {

typedef __int128 Wide;  // extents are products of caller-given 64-bit numbers

adst_status fail(adst_status st, const char* format, ...) {
  char text[256];
  va_list v;
  va_start(v, format);
  std::vsnprintf(text, sizeof(text), format, v);
  va_end(v);
  return report(st, text);
}

adst_status done(hipError_t e, const char* what) {
  if (e != hipSuccess) return fail(ADST_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
  return report_ok();
}

[[maybe_unused]] bool known(int32_t dtype) { return dtype >= ADST_F64 && dtype <= ADST_F16; }
[[maybe_unused]] int size_of(int32_t dtype) { return dtype == ADST_F64 ? 8 : dtype == ADST_F32 ? 4 : 2; }
[[maybe_unused]] int acc_size(int32_t dtype) { return dtype == ADST_F64 ? 8 : 4; }

// The arrays of one call: each output overlaps no other array, except where
// `same` allows it.
class Ranges {
 public:
  void in(const char* name, const void* p, Wide bytes) { add(name, p, bytes, false); }
  void out(const char* name, const void* p, Wide bytes) { add(name, p, bytes, true); }
  adst_status check() const {
    if (wild_) return fail(ADST_ERR_ARG, "%s: more bytes than the address space", wild_);
    for (int i = 0; i < n_; ++i)
      for (int j = 0; j < i; ++j) {
        if (!r_[i].out && !r_[j].out) continue;
        if (r_[i].lo < r_[j].hi && r_[j].lo < r_[i].hi && r_[i].lo != r_[i].hi &&
            r_[j].lo != r_[j].hi)
          return fail(ADST_ERR_ARG, "%s and %s overlap", r_[j].name, r_[i].name);
      }
    return ADST_OK;
  }

 private:
  struct One {
    const char* name;
    Wide lo, hi;
    bool out;
  };
  One r_[32];
  int n_ = 0;
  const char* wild_ = nullptr;
  void add(const char* name, const void* p, Wide bytes, bool out) {
    if (bytes > (Wide(1) << 62)) wild_ = name;
    if (!p) return;
    const Wide lo = (Wide)reinterpret_cast<uintptr_t>(p);
    r_[n_++] = {name, lo, lo + bytes, out};
  }
};

// Bytes that [batch][steps][channels] with these strides spans.
Wide span_bytes(int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t n2, int size) {
  if (n0 == 0 || n1 == 0 || n2 == 0) return 0;
  return (Wide(n0 - 1) * s0 + Wide(n1 - 1) * s1 + n2) * size;
}

bool aligned(const void* p, int size) { return reinterpret_cast<uintptr_t>(p) % size == 0; }

constexpr int64_t kMost = (int64_t(1) << 31) - (1 << 16);

adst_status check_aligned(const char* name, const void* p, int size) {
  if (p && !aligned(p, size))
    return fail(ADST_ERR_ARG, "%s is not aligned to its elements of %d bytes", name, size);
  return ADST_OK;
}

#define CHECK(call)                       \
  do {                                    \
    const adst_status st_ = (call);       \
    if (st_ != ADST_OK) return st_;       \
  } while (0)

}  // namespace
}  // namespace adst
