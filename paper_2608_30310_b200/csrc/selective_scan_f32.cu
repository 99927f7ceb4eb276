// The selective scan's instances for fp32, and the choice of the dtype.
#include "selective_scan.cuh"

namespace gdn {
cudaError_t launch_scan_bf16(const ScanArgs& a, int states, cudaStream_t stream);
cudaError_t launch_scan(const ScanArgs& a, int io_dtype, int states, cudaStream_t stream)
{
    return io_dtype == GDN_BF16 ? launch_scan_bf16(a, states, stream) : scan::launch_type<float>(a, states, stream);
}
}  // namespace gdn
