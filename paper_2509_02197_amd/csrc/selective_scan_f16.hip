// The selective scan (selective_scan.h) of one element type.

#include "seq_launch.h"
#include "selective_scan.h"

namespace adst {

hipError_t scan_forward_f16(const ScanArgs& a, const ScanGrid& g, void* ws, hipStream_t st) {
  return forward_of<f16>(a, g, ws, st);
}
hipError_t scan_vjp_f16(const ScanArgs& a, const ScanGrid& g, void* ws, hipStream_t st) {
  return vjp_of<f16>(a, g, ws, st);
}
hipError_t scan_step_f16(const ScanStep& s, hipStream_t st) { return step_of<f16>(s, st); }

}  // namespace adst
