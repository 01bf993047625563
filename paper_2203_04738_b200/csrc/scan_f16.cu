// The gated scan's kernels for f16 elements
#include "scan_tile.cuh"

namespace mg {
template int launch_scan<__half>(ScanArgs&, bool, int, bool, void*, cudaStream_t);
}  // namespace mg
