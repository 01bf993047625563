// The gated scan's kernels for bf16 elements, given coefficients
#include "scan_tile.cuh"

namespace mg {
template int launch_scan<__nv_bfloat16, kGiven>(ScanArgs&, bool, bool, void*, cudaStream_t);
}  // namespace mg
