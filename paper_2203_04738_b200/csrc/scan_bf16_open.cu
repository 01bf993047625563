// The gated scan's kernels for bf16 elements, other cells
#include "scan_tile.cuh"

namespace mg {
template int launch_scan<__nv_bfloat16, kOpen>(ScanArgs&, bool, bool, void*, cudaStream_t);
template int launch_scan<__nv_bfloat16, kLarge>(ScanArgs&, bool, bool, void*, cudaStream_t);
}  // namespace mg
