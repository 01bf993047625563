// The gated scan's kernels for f16 elements, cells with q <= 1/2
#include "scan_tile.cuh"

namespace mg {
template int launch_scan<__half, kCells>(ScanArgs&, bool, bool, void*, cudaStream_t);
}  // namespace mg
