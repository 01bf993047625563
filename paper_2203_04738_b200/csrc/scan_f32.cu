// The gated scan's kernels for f32 elements
#include "scan_tile.cuh"

namespace mg {
template int launch_scan<float>(ScanArgs&, bool, int, bool, void*, cudaStream_t);
}  // namespace mg
