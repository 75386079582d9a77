// Attention of prompts over a bf16 cache.
#include "pldp_prompt.cuh"

namespace pldp {

cudaError_t launch_prompt_bf16(const PromptArgs& a, const PromptMaps& m, int ctas, cudaStream_t s) {
    return launch_prompt_dims<false>(a, m, ctas, s);
}

}  // namespace pldp
