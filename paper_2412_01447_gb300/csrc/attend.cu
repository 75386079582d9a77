// Attention of a step's tokens over the paged cache: pldp_attend_cache.
#include <cuda_fp8.h>
#include <math.h>

#include "pldp_cache.cuh"

namespace pldp {
namespace {

struct AttendArgs {
    CacheView c;
    const __nv_bfloat16* q;
    __nv_bfloat16* out;
    int64_t q_seq, q_tok, q_head, o_seq, o_tok, o_head;
    const int32_t *seq_len, *draft_len;
    float* lse;
    uint32_t* status;
    int n, q_heads;
    float scale;
};

constexpr int kThreads = 128;

__device__ __forceinline__ float element(const uint8_t* v, int e, bool e4m3) {
    if (!e4m3) return __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(v)[e]);
    const __half_raw h = __nv_cvt_fp8_to_halfraw(v[e], __NV_E4M3);
    return __half2float(*reinterpret_cast<const __half*>(&h));
}

// One warp a query row: the keys in turn, lanes over the head's elements.
template <bool E4M3>
__global__ void __launch_bounds__(kThreads) attend_kernel(const AttendArgs a) {
    pdl_enter();
    const CacheView& c = a.c;
    const int b = blockIdx.z, i = blockIdx.y, h = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (h >= a.q_heads) return;
    constexpr int PER = kMaxHeadDim / 32;
    const int D = c.head_dim, kv = h / (a.q_heads / c.heads);
    uint32_t st;
    const StepTokens tk = step_tokens(a.seq_len, a.draft_len, b, a.n, c.capacity, st);
    const int32_t* table = c.pages + b * c.pages_stride;
    const int keys = i < tk.count ? tk.first + i + 1 : 0;
    float q[PER], o[PER], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int t = 0; t < PER; ++t) {
        const int e = lane + 32 * t;
        q[t] = keys > 0 && e < D ? a.scale * to_f32(a.q[b * a.q_seq + i * a.q_tok + h * a.q_head + e]) : 0.f;
        o[t] = 0.f;
    }
    for (int j = 0; j < keys; ++j) {
        int64_t scale_at;
        const int64_t off = locate(c, table, j, scale_at);
        if (off < 0) {
            st |= PLDP_ST_PAGE;
            continue;
        }
        const uint8_t *key = c.k + off + kv * c.head_stride, *val = c.v + off + kv * c.head_stride;
        const int64_t sc = scale_at + static_cast<int64_t>(kv) * c.page_size;
        float s = 0.f;
#pragma unroll
        for (int t = 0; t < PER; ++t)
            if (lane + 32 * t < D) s = fmaf(q[t], element(key, lane + 32 * t, E4M3), s);
        s = warp_sum(s);
        if (E4M3) s *= __ldg(c.k_scale + sc);
        const float mn = fmaxf(m, s), w = expf(m - mn), p = expf(s - mn), pv = E4M3 ? p * __ldg(c.v_scale + sc) : p;
        l = l * w + p;
#pragma unroll
        for (int t = 0; t < PER; ++t)
            if (lane + 32 * t < D) o[t] = o[t] * w + pv * element(val, lane + 32 * t, E4M3);
        m = mn;
    }
    if (st && lane == 0 && a.status) atomicOr(a.status + b, st);
#pragma unroll
    for (int t = 0; t < PER; ++t) {
        const int e = lane + 32 * t;
        if (e < D) a.out[b * a.o_seq + i * a.o_tok + h * a.o_head + e] = __float2bfloat16(l > 0.f ? o[t] / l : 0.f);
    }
    if (lane == 0 && a.lse) a.lse[(static_cast<int64_t>(b) * a.n + i) * a.q_heads + h] = l > 0.f ? m + logf(l) : -INFINITY;
}

}  // namespace
}  // namespace pldp

using namespace pldp;

extern "C" {

PLDP_API size_t pldp_attend_workspace_size(int B, int n, int q_heads, int heads, int head_dim) {
    if (B < 0 || n < 1 || q_heads < 1 || heads < 1 || q_heads % heads || head_dim < 1) return 0;
    return 256;
}

PLDP_API pldp_status pldp_attend_cache(const pldp_attend_args* p, void* stream) {
    const char* fn = "attend_cache";
    if (!p) return fail(PLDP_ERR_INVALID_ARG, "%s: null argument block", fn);
    if (p->B < 0 || p->n < 1 || p->q_heads < 1)
        return fail(PLDP_ERR_INVALID_ARG, "%s: B < 0, n < 1 or q_heads < 1", fn);
    if (!isfinite(p->scale)) return fail(PLDP_ERR_INVALID_ARG, "%s: scale must be finite", fn);
    AttendArgs a = {};
    pldp_status st = cache_view(fn, p->cache, p->B, &a.c);
    if (st != PLDP_OK) return st;
    if (p->q_heads % p->cache.heads)
        return fail(PLDP_ERR_INVALID_ARG, "%s: q_heads must be a multiple of the cache's heads", fn);
    if (p->B > 65535 || p->n > 65535) return fail(PLDP_ERR_UNSUPPORTED, "%s: B or n above 65535", fn);
    if (p->B == 0) return PLDP_OK;
    if (!p->q || !p->out || !p->seq_len || !p->workspace) return fail(PLDP_ERR_INVALID_ARG, "%s: null pointer", fn);
    if ((st = check_rows(fn, "q", p->q, p->q_strides, 2)) != PLDP_OK) return st;
    if ((st = check_rows(fn, "out", p->out, p->out_strides, 2)) != PLDP_OK) return st;
    const size_t need = pldp_attend_workspace_size(p->B, p->n, p->q_heads, p->cache.heads, p->cache.head_dim);
    if (p->workspace_bytes < need)
        return fail(PLDP_ERR_INVALID_ARG, "%s: workspace needs %zu bytes, has %zu", fn, need, p->workspace_bytes);
    if (reinterpret_cast<uintptr_t>(p->workspace) & 255u)
        return fail(PLDP_ERR_INVALID_ARG, "%s: workspace is not 256-byte aligned", fn);
    a.q = static_cast<const __nv_bfloat16*>(p->q);
    a.out = static_cast<__nv_bfloat16*>(p->out);
    a.q_seq = p->q_strides[0], a.q_tok = p->q_strides[1], a.q_head = p->q_strides[2];
    a.o_seq = p->out_strides[0], a.o_tok = p->out_strides[1], a.o_head = p->out_strides[2];
    a.seq_len = p->seq_len, a.draft_len = p->draft_len;
    a.lse = p->lse;
    a.status = p->status;
    a.n = p->n, a.q_heads = p->q_heads;
    a.scale = p->scale;
    const dim3 grid((p->q_heads + kThreads / 32 - 1) / (kThreads / 32), p->n, p->B);
    auto s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = p->cache.dtype == PLDP_E4M3 ? launch_pdl(attend_kernel<true>, grid, dim3(kThreads), 0, s, 0, a)
                                                      : launch_pdl(attend_kernel<false>, grid, dim3(kThreads), 0, s, 0, a);
    if (e != cudaSuccess) return fail(PLDP_ERR_CUDA, "%s: launch failed: %s", fn, cudaGetErrorString(e));
    return check_launch(fn);
}

}  // extern "C"
