// Attention of prompts over an e4m3 cache.
#include "pldp_prompt.cuh"

namespace pldp {

cudaError_t launch_prompt_e4m3(const PromptArgs& a, const PromptMaps& m, int ctas, cudaStream_t s) {
    return launch_prompt_dims<true>(a, m, ctas, s);
}

}  // namespace pldp
