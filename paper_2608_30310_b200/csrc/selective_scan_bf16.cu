// The selective scan's instances for bf16 (the two dtypes compile side by side).
#include "selective_scan.cuh"

namespace gdn {
cudaError_t launch_scan_bf16(const ScanArgs& a, int states, cudaStream_t stream) { return scan::launch_type<__nv_bfloat16>(a, states, stream); }
}  // namespace gdn
