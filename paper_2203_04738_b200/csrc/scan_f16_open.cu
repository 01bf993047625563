// The gated scan's kernels for f16 elements, other cells
#include "scan_tile.cuh"

namespace mg {
template int launch_scan<__half, kOpen>(ScanArgs&, bool, bool, void*, cudaStream_t);
template int launch_scan<__half, kLarge>(ScanArgs&, bool, bool, void*, cudaStream_t);
}  // namespace mg
