// The gated scan's kernels for bf16 elements
#include "scan_tile.cuh"

namespace mg {
template int launch_scan<__nv_bfloat16>(ScanArgs&, bool, int, bool, void*, cudaStream_t);
}  // namespace mg
