// Inputs and comparisons of the programs.
#pragma once

#include <cmath>
#include <cstdint>
#include <cstdio>

inline double noise(uint64_t i) {  // in [0, 1)
  i = (i + 1) * 0x9e3779b97f4a7c15ull;
  i = (i ^ (i >> 30)) * 0xbf58476d1ce4e5b9ull;
  i = (i ^ (i >> 27)) * 0x94d049bb133111ebull;
  return (double)((i ^ (i >> 31)) >> 11) * 0x1p-53;
}

inline int wrong = 0;
inline void near(const char* what, int64_t i, double got, double want, double tol) {
  if (!(std::fabs(got - want) <= tol * (1 + std::fabs(want))) && wrong++ < 8)
    std::printf("%s[%lld]: %.9g, not %.9g\n", what, (long long)i, got, want);
}
inline int done() {
  if (wrong) std::printf("%d wrong values\n", wrong);
  return wrong != 0;
}
