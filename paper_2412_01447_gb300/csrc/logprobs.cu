// Log probabilities of tokens, entropy and alternatives: pldp_token_logprobs.
#include <math.h>

#include "pldp_internal.cuh"

namespace pldp {
namespace {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxTop = 32;

struct LogprobArgs {
    const int32_t* tokens;
    float *logprob, *entropy, *top_logprob;
    int32_t* top_id;
    int V, top;
    float inv_t;
};

// One CTA a row: the maximum, the sums against it, then the alternatives one by one.
template <typename T>
__global__ void __launch_bounds__(kThreads) logprobs_kernel(const T* __restrict__ logits, const LogprobArgs a) {
    pdl_enter();
    __shared__ unsigned long long keys[kWarps];
    __shared__ float sums[2][kWarps];
    const int64_t r = blockIdx.x;
    const T* x = logits + r * a.V;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    unsigned long long last = ~0ull;
    float m = -INFINITY, l = 0.f, t = 0.f, lse = -INFINITY;
    for (int k = 0; k <= a.top; ++k) {                  // turn 0 is the maximum, which turn 1 finds again
        unsigned long long best = 0;
        for (int v = threadIdx.x; v < a.V; v += kThreads) {
            const unsigned long long key = pack_key(to_f32(x[v]), v);
            if (key < last && key > best) best = key;
        }
        best = warp_max_u64(best);
        __syncthreads();
        if (lane == 0) keys[warp] = best;
        __syncthreads();
        best = warp_max_u64(lane < kWarps ? keys[lane] : 0ull);
        if (k == 0) {
            m = key_value(best) * a.inv_t;
            if (m > -INFINITY)
                for (int v = threadIdx.x; v < a.V; v += kThreads) {
                    const float d = to_f32(x[v]) * a.inv_t - m, e = expf(d);
                    l += e;
                    if (e > 0.f) t += e * d;
                }
            l = warp_sum(l), t = warp_sum(t);
            __syncthreads();
            if (lane == 0) sums[0][warp] = l, sums[1][warp] = t;
            __syncthreads();
            l = warp_sum(lane < kWarps ? sums[0][lane] : 0.f);
            t = warp_sum(lane < kWarps ? sums[1][lane] : 0.f);
            if (m > -INFINITY) lse = m + logf(l);
            if (threadIdx.x == 0) {
                if (a.entropy) a.entropy[r] = m > -INFINITY ? logf(l) - t / l : 0.f;
                if (a.logprob && a.tokens) {
                    const int tok = a.tokens[r];
                    a.logprob[r] = tok >= 0 && tok < a.V && m > -INFINITY ? to_f32(x[tok]) * a.inv_t - lse : -INFINITY;
                }
            }
        } else {
            last = best;
            if (threadIdx.x == 0) {
                if (a.top_id) a.top_id[r * a.top + k - 1] = static_cast<int>(key_index(best));
                if (a.top_logprob) a.top_logprob[r * a.top + k - 1] = m > -INFINITY ? key_value(best) * a.inv_t - lse : -INFINITY;
            }
        }
    }
}

}  // namespace
}  // namespace pldp

using namespace pldp;

extern "C" {

PLDP_API size_t pldp_token_logprobs_workspace_size(int64_t rows, int V) {
    if (rows < 0 || V < 1) return 0;
    return 256;
}

PLDP_API pldp_status pldp_token_logprobs(const void* logits, pldp_dtype dtype, int64_t rows, int V, float temperature,
                                         const int32_t* tokens, float* logprob, float* entropy, int top, int32_t* top_id,
                                         float* top_logprob, void* workspace, size_t workspace_bytes, void* stream) {
    const char* fn = "token_logprobs";
    if (rows < 0 || V < 1) return fail(PLDP_ERR_INVALID_ARG, "%s: rows < 0 or V < 1", fn);
    if (dtype != PLDP_F32 && dtype != PLDP_BF16)
        return fail(PLDP_ERR_UNSUPPORTED, "%s: dtype %d", fn, static_cast<int>(dtype));
    if (!(temperature > 0.f) || !isfinite(temperature))
        return fail(PLDP_ERR_INVALID_ARG, "%s: temperature must be positive and finite", fn);
    if (top < 0 || top > V || top > kMaxTop)
        return fail(PLDP_ERR_INVALID_ARG, "%s: top must be 0..%d and at most V", fn, kMaxTop);
    if (rows > (int64_t(1) << 31) - 1) return fail(PLDP_ERR_UNSUPPORTED, "%s: 2^31 rows or more", fn);
    if ((tokens == nullptr) != (logprob == nullptr))
        return fail(PLDP_ERR_INVALID_ARG, "%s: tokens and logprob go together", fn);
    if (rows == 0) return PLDP_OK;
    if (!logits || !workspace) return fail(PLDP_ERR_INVALID_ARG, "%s: null pointer", fn);
    const size_t need = pldp_token_logprobs_workspace_size(rows, V);
    if (workspace_bytes < need)
        return fail(PLDP_ERR_INVALID_ARG, "%s: workspace needs %zu bytes, has %zu", fn, need, workspace_bytes);
    if (!aligned16(workspace)) return fail(PLDP_ERR_INVALID_ARG, "%s: workspace is not 16-byte aligned", fn);
    LogprobArgs a = {tokens, logprob, entropy, top_logprob, top_id, V, top_id || top_logprob ? top : 0, 1.f / temperature};
    auto s = static_cast<cudaStream_t>(stream);
    const dim3 grid(static_cast<unsigned>(rows));
    const cudaError_t e =
        dtype == PLDP_F32
            ? launch_pdl(logprobs_kernel<float>, grid, dim3(kThreads), 0, s, 0, static_cast<const float*>(logits), a)
            : launch_pdl(logprobs_kernel<__nv_bfloat16>, grid, dim3(kThreads), 0, s, 0,
                         static_cast<const __nv_bfloat16*>(logits), a);
    if (e != cudaSuccess) return fail(PLDP_ERR_CUDA, "%s: launch failed: %s", fn, cudaGetErrorString(e));
    return check_launch(fn);
}

}  // extern "C"
