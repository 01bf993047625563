// The gated scan's kernels for f32 elements, given coefficients
#include "scan_tile.cuh"

namespace mg {
template int launch_scan<float, kGiven>(ScanArgs&, bool, bool, void*, cudaStream_t);
}  // namespace mg
