// The selective scan (selective_scan.h) of one element type.

#include "seq_launch.h"
#include "selective_scan.h"

namespace adst {

hipError_t scan_forward_f32(const ScanArgs& a, const ScanGrid& g, void* ws, hipStream_t st) {
  return forward_of<float>(a, g, ws, st);
}
hipError_t scan_vjp_f32(const ScanArgs& a, const ScanGrid& g, void* ws, hipStream_t st) {
  return vjp_of<float>(a, g, ws, st);
}
hipError_t scan_step_f32(const ScanStep& s, hipStream_t st) { return step_of<float>(s, st); }

}  // namespace adst
