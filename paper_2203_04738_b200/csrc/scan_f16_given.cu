// The gated scan's kernels for f16 elements, given coefficients
#include "scan_tile.cuh"

namespace mg {
template int launch_scan<__half, kGiven>(ScanArgs&, bool, bool, void*, cudaStream_t);
}  // namespace mg
