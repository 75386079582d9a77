// Attention over an e4m3 cache.
#include "pldp_attend.cuh"

namespace pldp {

cudaError_t launch_attend_e4m3(const AttendArgs& a, const Maps& m, int nt, int ctas, cudaStream_t s) {
    return launch_dims<true>(a, m, nt, ctas, s);
}

}  // namespace pldp
