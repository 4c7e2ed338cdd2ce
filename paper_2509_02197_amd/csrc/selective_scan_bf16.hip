// The selective scan (selective_scan.h) of one element type.

#include "seq_launch.h"
#include "selective_scan.h"

namespace adst {

hipError_t scan_forward_bf16(const ScanArgs& a, const ScanGrid& g, void* ws, hipStream_t st) {
  return forward_of<bf16>(a, g, ws, st);
}
hipError_t scan_vjp_bf16(const ScanArgs& a, const ScanGrid& g, void* ws, hipStream_t st) {
  return vjp_of<bf16>(a, g, ws, st);
}
hipError_t scan_step_bf16(const ScanStep& s, hipStream_t st) { return step_of<bf16>(s, st); }

}  // namespace adst
