// The vocabulary's cross entropy (linear_cross_entropy.h) of one element type.

#include "seq_launch.h"
#include "linear_cross_entropy.h"

namespace adst {

hipError_t xent_forward_f32(const XentArgs& a, const XentPlan& p, void* ws, hipStream_t st) {
  return forward_of<float>(a, p, ws, st);
}
hipError_t xent_vjp_f32(const XentArgs& a, const XentPlan& p, void* ws, hipStream_t st) {
  return vjp_of<float>(a, p, ws, st);
}

}  // namespace adst
