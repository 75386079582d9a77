// Attention over a bf16 cache.
#include "pldp_attend.cuh"

namespace pldp {

cudaError_t launch_attend_bf16(const AttendArgs& a, const Maps& m, int nt, int ctas, cudaStream_t s) {
    return launch_dims<false>(a, m, nt, ctas, s);
}

}  // namespace pldp
