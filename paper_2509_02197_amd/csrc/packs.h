// Vectors of any number of channels at any element's address (recurrence.hip
// and the token operators).
#pragma once

#include "seq_common.h"

namespace adst {
namespace {

// V consecutive channels of T, at any element's address.
template <class T, int V>
struct Pack {
  typedef T type __attribute__((ext_vector_type(V)));
  typedef T unaligned __attribute__((ext_vector_type(V), aligned(sizeof(T))));
  type v;
};
template <class T, int V, bool STREAM = false>
__device__ inline Pack<T, V> load_pack(const T* p, int n) {
  Pack<T, V> r;
  if (n >= V) {
    const auto* at = reinterpret_cast<const typename Pack<T, V>::unaligned*>(p);
    if constexpr (STREAM) r.v = __builtin_nontemporal_load(at);
    else r.v = *at;
    return r;
  }
#pragma unroll
  for (int i = 0; i < V; ++i) r.v[i] = i < n ? p[i] : T(0);
  return r;
}
template <class T, int V, bool STREAM = false>
__device__ inline void store_pack(T* p, Pack<T, V> x, int n) {
  if (n >= V) {
    auto* at = reinterpret_cast<typename Pack<T, V>::unaligned*>(p);
    if constexpr (STREAM) __builtin_nontemporal_store(x.v, at);
    else *at = x.v;
    return;
  }
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (i < n) p[i] = x.v[i];
}

}  // namespace
}  // namespace adst
