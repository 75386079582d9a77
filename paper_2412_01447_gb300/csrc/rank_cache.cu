// Ranking by attentions (Eq. 2) straight from a layer's cache: pldp_rank_cache.
#include <cuda_fp8.h>
#include <math.h>

#include "pldp_cache.cuh"

namespace pldp {
namespace {

struct RankArgs {
    CacheView c;
    const __nv_bfloat16* q;
    int64_t q_seq, q_tok, q_head;
    const int32_t *row, *kv_len, *heads, *cand_pos, *cand_count;
    const float* lse;
    float *scores, *best_score;
    int32_t* best_pos;
    uint32_t* status;
    int n, q_heads, n_sel, C_cap, accumulate, sum;
    float scale;
};

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;

__device__ __forceinline__ float element(const uint8_t* v, int e, bool e4m3) {
    if (!e4m3) return __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(v)[e]);
    const __half_raw h = __nv_cvt_fp8_to_halfraw(v[e], __NV_E4M3);
    return __half2float(*reinterpret_cast<const __half*>(&h));
}

// One CTA a sequence, one warp a candidate.
template <bool E4M3>
__global__ void __launch_bounds__(kThreads) rank_cache_kernel(const RankArgs a) {
    pdl_enter();
    extern __shared__ __align__(16) float qs[];                    // [n_sel][head_dim], scaled
    __shared__ unsigned long long best_of[kWarps];
    const CacheView& c = a.c;
    const int b = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, D = c.head_dim;
    const int row = a.row ? __ldg(a.row + b) : 0, len = __ldg(a.kv_len + b);
    int count = __ldg(a.cand_count + b);
    count = count < 0 ? 0 : min(count, a.C_cap);
    uint32_t st = 0;
    if (row < 0 || row >= a.n) st |= PLDP_ST_ROW_INDEX;
    if (len < 0 || len > c.capacity) st |= PLDP_ST_SEQ_LEN;
    const bool ok = st == 0;
    const float* lse = a.lse + (static_cast<int64_t>(b) * a.n + (ok ? row : 0)) * a.q_heads;
    if (ok)
        for (int t = threadIdx.x; t < a.n_sel * D; t += kThreads) {
            const int r = t / D, e = t - r * D;
            const int h = a.heads ? __ldg(a.heads + r) : r;
            qs[t] = h >= 0 && h < a.q_heads
                        ? a.scale * to_f32(a.q[b * a.q_seq + row * a.q_tok + h * a.q_head + e])
                        : 0.f;
            if (e == 0 && (h < 0 || h >= a.q_heads) && a.status) atomicOr(a.status + b, PLDP_ST_ROW_INDEX);
        }
    if (st && a.status) atomicOr(a.status + b, st);
    __syncthreads();
    const int32_t* table = c.pages + b * c.pages_stride;
    const int group = a.q_heads / c.heads;
    unsigned long long best = 0;
    for (int i = warp; i < count; i += kWarps) {
        const int j = __ldg(a.cand_pos + static_cast<int64_t>(b) * a.C_cap + i);
        float* out = a.scores ? a.scores + static_cast<int64_t>(b) * a.C_cap + i : nullptr;
        float score = a.sum ? 0.f : -INFINITY;
        bool live = ok && j >= 0 && j < len;
        int64_t scale_at = 0, off = -1;
        if (live) off = locate(c, table, j, scale_at);
        if (live && off < 0 && lane == 0 && a.status) atomicOr(a.status + b, PLDP_ST_PAGE);
        live = live && off >= 0;
        if (live) {
            for (int r = 0; r < a.n_sel; ++r) {
                const int h = a.heads ? __ldg(a.heads + r) : r;
                if (h < 0 || h >= a.q_heads) continue;
                const int kv = h / group;
                const uint8_t* key = c.k + off + kv * c.head_stride;
                float dot = 0.f;
                for (int e = lane; e < D; e += 32) dot = fmaf(qs[r * D + e], element(key, e, E4M3), dot);
                dot = warp_sum(dot);
                if (E4M3) dot *= __ldg(c.k_scale + scale_at + static_cast<int64_t>(kv) * c.page_size);
                const float l = __ldg(lse + h);
                const float p = l > -INFINITY ? expf(dot - l) : 0.f;
                score = a.sum ? score + p : fmaxf(score, p);
            }
        } else {
            score = -INFINITY;
        }
        if (a.accumulate) {
            const float before = *out;
            score = live ? (a.sum ? before + score : fmaxf(before, score)) : before;
        }
        if (out && lane == 0) *out = score;
        if (score > -INFINITY) {
            const unsigned long long key = pack_key(score, static_cast<uint32_t>(j));
            best = key > best ? key : best;
        }
    }
    if (lane == 0) best_of[warp] = best;
    __syncthreads();
    if (warp == 0) {
        best = warp_max_u64(lane < kWarps ? best_of[lane] : 0ull);
        if (lane == 0) {
            a.best_pos[b] = best ? static_cast<int>(key_index(best)) : -1;
            if (a.best_score) a.best_score[b] = best ? key_value(best) : -INFINITY;
        }
    }
}

}  // namespace
}  // namespace pldp

using namespace pldp;

extern "C" PLDP_API pldp_status pldp_rank_cache(const pldp_rank_cache_args* p, void* stream) {
    const char* fn = "rank_cache";
    if (!p) return fail(PLDP_ERR_INVALID_ARG, "%s: null argument block", fn);
    if (p->B < 0 || p->n < 1 || p->q_heads < 1 || p->C_cap < 0)
        return fail(PLDP_ERR_INVALID_ARG, "%s: B < 0, n < 1, q_heads < 1 or C_cap < 0", fn);
    if (p->agg != PLDP_AGG_MAX && p->agg != PLDP_AGG_SUM)
        return fail(PLDP_ERR_INVALID_ARG, "%s: agg %d", fn, static_cast<int>(p->agg));
    if (!isfinite(p->scale)) return fail(PLDP_ERR_INVALID_ARG, "%s: scale must be finite", fn);
    RankArgs a = {};
    pldp_status st = cache_view(fn, p->cache, p->B, &a.c);
    if (st != PLDP_OK) return st;
    if (p->q_heads % p->cache.heads)
        return fail(PLDP_ERR_INVALID_ARG, "%s: q_heads must be a multiple of the cache's heads", fn);
    const int n_sel = p->heads ? p->n_sel : p->q_heads;
    if (n_sel < 1) return fail(PLDP_ERR_INVALID_ARG, "%s: n_sel < 1", fn);
    if (static_cast<int64_t>(n_sel) * p->cache.head_dim > 49152)
        return fail(PLDP_ERR_UNSUPPORTED, "%s: n_sel * head_dim above 49152", fn);
    if (p->accumulate && !p->scores) return fail(PLDP_ERR_INVALID_ARG, "%s: accumulate needs scores", fn);
    if (p->B == 0) return PLDP_OK;
    if (!p->q || !p->kv_len || !p->lse || !p->cand_pos || !p->cand_count || !p->best_pos)
        return fail(PLDP_ERR_INVALID_ARG, "%s: null pointer", fn);
    if ((st = check_rows(fn, "q", p->q, p->q_strides, 2)) != PLDP_OK) return st;
    a.q = static_cast<const __nv_bfloat16*>(p->q);
    a.q_seq = p->q_strides[0], a.q_tok = p->q_strides[1], a.q_head = p->q_strides[2];
    a.row = p->row, a.kv_len = p->kv_len, a.heads = p->heads;
    a.cand_pos = p->cand_pos, a.cand_count = p->cand_count;
    a.lse = p->lse;
    a.scores = p->scores, a.best_score = p->best_score, a.best_pos = p->best_pos;
    a.status = p->status;
    a.n = p->n, a.q_heads = p->q_heads, a.n_sel = n_sel, a.C_cap = p->C_cap;
    a.accumulate = p->accumulate != 0, a.sum = p->agg == PLDP_AGG_SUM;
    a.scale = p->scale;
    const size_t smem = static_cast<size_t>(n_sel) * p->cache.head_dim * sizeof(float);
    auto s = static_cast<cudaStream_t>(stream);
    auto kernel = p->cache.dtype == PLDP_E4M3 ? rank_cache_kernel<true> : rank_cache_kernel<false>;
    if (smem > kOptInShared) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
        if (e != cudaSuccess) return fail(PLDP_ERR_CUDA, "%s: %s", fn, cudaGetErrorString(e));
    }
    const cudaError_t e = launch_pdl(kernel, dim3(p->B), dim3(kThreads), smem, s, 0, a);
    if (e != cudaSuccess) return fail(PLDP_ERR_CUDA, "%s: launch failed: %s", fn, cudaGetErrorString(e));
    return check_launch(fn);
}
