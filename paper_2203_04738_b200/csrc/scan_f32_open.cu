// The gated scan's kernels for f32 elements, other cells
#include "scan_tile.cuh"

namespace mg {
template int launch_scan<float, kOpen>(ScanArgs&, bool, bool, void*, cudaStream_t);
template int launch_scan<float, kLarge>(ScanArgs&, bool, bool, void*, cudaStream_t);
}  // namespace mg
