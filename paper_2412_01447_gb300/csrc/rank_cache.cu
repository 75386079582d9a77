// Ranking by attentions (Eq. 2) straight from a layer's cache: pldp_rank_cache.
#include <cuda_fp8.h>
#include <cuda_fp16.h>
#include <math.h>

#include <utility>

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

// A cluster of CTAs a sequence, which deal its candidates among them.  The selected heads' queries lie in shared
// memory, ordered by the key/value head they read, so that a unit of work (one candidate, one key/value head) reads
// that key once, 16 bytes a lane, for all of its heads.  Bound by latency: a candidate's position, its page,
// its key and the queries each wait for the one before.  The first two are looked up for 64 candidates at once, and
// four units' keys are on their way a group of lanes.
// 16 x 341..512 candidates, 8 heads of an e4m3 cache: 15.5 us (one CTA a sequence and a warp a candidate: 191 us);
// 8 x 8..16 candidates, 32 heads: 9.7 us (23 us).
constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kChunk = 64;           // candidates looked up at once
constexpr int kParts = 1024;         // scores of (candidate, key/value head) held
constexpr int kInFlight = 4;
constexpr int64_t kNoCandidate = -2;   // in the place of a key's offset (locate()'s -1 is a missing page)

// Elements that 16 bytes hold, as floats, times q and added up.
template <bool E4M3>
__device__ __forceinline__ float dot16(const uint4& x, const float* q) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    float d = 0.f;
    if constexpr (E4M3) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const __half2_raw lo = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(w[k] & 0xFFFFu), __NV_E4M3);
            const __half2_raw hi = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(w[k] >> 16), __NV_E4M3);
            const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&lo)), b = __half22float2(*reinterpret_cast<const __half2*>(&hi));
            const float4 y = *reinterpret_cast<const float4*>(q + 4 * k);
            d = fmaf(a.x, y.x, fmaf(a.y, y.y, fmaf(b.x, y.z, fmaf(b.y, y.w, d))));
        }
    } else {
#pragma unroll
        for (int k = 0; k < 4; k += 2) {
            const float4 y = *reinterpret_cast<const float4*>(q + 2 * k);
            d = fmaf(__uint_as_float(w[k] << 16), y.x, fmaf(__uint_as_float(w[k] & 0xFFFF0000u), y.y, d));
            d = fmaf(__uint_as_float(w[k + 1] << 16), y.z, fmaf(__uint_as_float(w[k + 1] & 0xFFFF0000u), y.w, d));
        }
    }
    return d;
}

// GS lanes a unit: the power of two that covers a vector's 16-byte pieces.
template <bool E4M3, int GS>
__global__ void __launch_bounds__(kThreads) rank_cache_kernel(const RankArgs a) {
    pdl_enter();
    extern __shared__ __align__(16) uint8_t raw[];
    __shared__ int64_t off[kChunk], scale_at[kChunk];
    __shared__ float part[kParts];
    __shared__ int pos[kChunk];
    __shared__ int groups, chunk_size;
    __shared__ unsigned long long best_of[kWarps], cluster_best[16];
    cg::cluster_group cluster = cg::this_cluster();
    auto started = cluster.barrier_arrive();                // nothing is written to a CTA that has not begun
    const CacheView& c = a.c;
    const int S = cluster.num_blocks(), rank = cluster.block_rank(), b = blockIdx.x / S;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, D = c.head_dim, group = a.q_heads / c.heads;
    float* qs = reinterpret_cast<float*>(raw);                                       // [selected, in order][head_dim], scaled
    float* lses = qs + a.n_sel * D;                                                  // [selected, in order]
    const int most = min(c.heads, a.n_sel);
    uint16_t* first = reinterpret_cast<uint16_t*>(lses + a.n_sel);                   // [groups + 1]: where a key/value head's begin
    uint16_t* kv_of = first + most + 1;                                              // [groups]: which one it is
    uint16_t* order = kv_of + most;                                                  // [selected]: the n_sel entries in order
    const int row = a.row ? __ldg(a.row + b) : 0, len = __ldg(a.kv_len + b);
    int count = __ldg(a.cand_count + b);
    count = count < 0 ? 0 : min(count, a.C_cap);
    uint32_t st = 0;
    if (row < 0 || row >= a.n) st |= PLDP_ST_ROW_INDEX;
    if (len < 0 || len > c.capacity) st |= PLDP_ST_SEQ_LEN;
    const bool ok = st == 0;
    if (st && a.status && threadIdx.x == 0) atomicOr(a.status + b, st);
    const float* lse = a.lse + (static_cast<int64_t>(b) * a.n + (ok ? row : 0)) * a.q_heads;
    const int32_t* table = c.pages + b * c.pages_stride;

    // the selected heads by key/value head (entries outside [0, q_heads) last), each with its queries
    auto head_at = [&](int r) { return a.heads ? __ldg(a.heads + r) : r; };
    auto key_head = [&](int h) { return h >= 0 && h < a.q_heads ? h / group : c.heads; };
    if (threadIdx.x == 0) groups = 0;
    if (a.heads) {
        for (int r = threadIdx.x; r < a.n_sel; r += kThreads) {
            const int kv = key_head(head_at(r));
            int at = 0;
            for (int o = 0; o < a.n_sel; ++o) {
                const int other = key_head(head_at(o));
                at += other < kv || (other == kv && o < r);
            }
            order[at] = static_cast<uint16_t>(r);
            if (kv == c.heads && a.status) atomicOr(a.status + b, PLDP_ST_ROW_INDEX);
        }
    } else {
        for (int r = threadIdx.x; r < a.n_sel; r += kThreads) order[r] = static_cast<uint16_t>(r);
    }
    __syncthreads();
    if (warp == 0) {                                        // where a key/value head's entries begin
        int n = 0;
        for (int r0 = 0; r0 < a.n_sel; r0 += 32) {
            const int r = r0 + lane;
            const int kv = r < a.n_sel ? key_head(head_at(order[r])) : -1;
            const int before = r > 0 && r < a.n_sel ? key_head(head_at(order[r - 1])) : -1;
            const bool starts = r < a.n_sel && kv != before && kv < c.heads, ends = r < a.n_sel && kv != before && kv == c.heads;
            const unsigned m = __ballot_sync(0xFFFFFFFFu, starts), e = __ballot_sync(0xFFFFFFFFu, ends);
            if (starts) {
                const int k = n + __popc(m & ((1u << lane) - 1u));
                first[k] = static_cast<uint16_t>(r);
                kv_of[k] = static_cast<uint16_t>(kv);
            }
            n += __popc(m);
            if (ends) first[n] = static_cast<uint16_t>(r);
            if (e) break;
            if (r0 + 32 >= a.n_sel && lane == 0) first[n] = static_cast<uint16_t>(a.n_sel);
        }
        if (lane == 0) {
            groups = n;
            chunk_size = n > 0 ? min(kChunk, max(1, kParts / n)) : kChunk;
        }
    }
    if (ok)
        for (int t = threadIdx.x; t < a.n_sel * (D / 8); t += kThreads) {
            const int r = t / (D / 8), e = t - r * (D / 8), h = head_at(order[r]);
            if (h < 0 || h >= a.q_heads) continue;
            if (e == 0) lses[r] = __ldg(lse + h);
            const uint4 x = *reinterpret_cast<const uint4*>(a.q + b * a.q_seq + row * a.q_tok + h * a.q_head + e * 8);
            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
            float* to = qs + r * D + e * 8;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                to[2 * k] = a.scale * __uint_as_float(w[k] << 16);
                to[2 * k + 1] = a.scale * __uint_as_float(w[k] & 0xFFFF0000u);
            }
        }
    __syncthreads();

    const int n_groups = groups, per = chunk_size;
    const int g = threadIdx.x / GS, at = threadIdx.x % GS, pieces = c.vec_bytes / 16;
    const unsigned mates = GS == 32 ? 0xFFFFFFFFu : ((1u << (GS % 32)) - 1u) << (lane / GS * GS);
    constexpr int kGroups = kThreads / GS;
    unsigned long long best = 0;
    // this CTA's candidates: rank, rank + S, ...
    const int mine = count > rank ? (count - rank + S - 1) / S : 0;
    for (int i0 = 0; i0 < mine; i0 += per) {
        const int here = min(per, mine - i0);
        for (int t = threadIdx.x; t < here; t += kThreads) {
            const int j = __ldg(a.cand_pos + static_cast<int64_t>(b) * a.C_cap + rank + (i0 + t) * S);
            pos[t] = j;
            off[t] = kNoCandidate;
            if (ok && j >= 0 && j < len) {
                off[t] = locate(c, table, j, scale_at[t]);
                if (off[t] < 0 && a.status) atomicOr(a.status + b, PLDP_ST_PAGE);
            }
        }
        __syncthreads();
        const int units = here * n_groups;
        for (int u0 = g; u0 < units; u0 += kGroups * kInFlight) {
            uint4 x[kInFlight];
            float ks[kInFlight];
#pragma unroll
            for (int p = 0; p < kInFlight; ++p) {
                const int u = u0 + p * kGroups;
                x[p] = make_uint4(0u, 0u, 0u, 0u);
                ks[p] = 1.f;
                if (u >= units) continue;
                const int t = u / n_groups, kv = kv_of[u - t * n_groups];
                if (off[t] < 0) continue;
                if (at < pieces) x[p] = ld_stream16(c.k + off[t] + kv * c.head_stride + at * 16);
                if constexpr (E4M3) ks[p] = __ldg(c.k_scale + scale_at[t] + static_cast<int64_t>(kv) * c.page_size);
            }
#pragma unroll
            for (int p = 0; p < kInFlight; ++p) {
                const int u = u0 + p * kGroups;
                if (u >= units) continue;                   // the whole group of lanes
                const int t = u / n_groups, gr = u - t * n_groups, r1 = first[gr + 1];
                float score = a.sum ? 0.f : -INFINITY;
                for (int r = first[gr]; r < r1; ++r) {
                    float d = at < pieces ? dot16<E4M3>(x[p], qs + r * D + at * (E4M3 ? 16 : 8)) : 0.f;
#pragma unroll
                    for (int o = GS / 2; o > 0; o >>= 1) d += __shfl_xor_sync(mates, d, o, GS);
                    if constexpr (E4M3) d *= ks[p];
                    const float l = lses[r];
                    const float w = l > -INFINITY ? expf(d - l) : 0.f;
                    score = a.sum ? score + w : fmaxf(score, w);
                }
                if (at == 0) part[u] = score;
            }
        }
        __syncthreads();
        for (int t = threadIdx.x; t < here; t += kThreads) {
            float* out = a.scores ? a.scores + static_cast<int64_t>(b) * a.C_cap + rank + (i0 + t) * S : nullptr;
            // A candidate without a page, or where no selected head is one, has no score of this layer: that of the
            // others stands.  One outside the context, or of a sequence that is refused, has none at all.
            const bool live = off[t] >= 0 && n_groups > 0;
            float score = live && a.sum ? 0.f : -INFINITY;
            if (live)
                for (int k = 0; k < n_groups; ++k) score = a.sum ? score + part[t * n_groups + k] : fmaxf(score, part[t * n_groups + k]);
            if (a.accumulate && off[t] != kNoCandidate) {
                const float before = *out;
                score = live ? (a.sum ? before + score : fmaxf(before, score)) : before;
            }
            if (out) *out = score;
            if (score > -INFINITY) {
                const unsigned long long key = pack_key(score, static_cast<uint32_t>(pos[t]));
                best = key > best ? key : best;
            }
        }
        __syncthreads();
    }
    best = warp_max_u64(best);
    if (lane == 0) best_of[warp] = best;
    __syncthreads();
    cluster.barrier_wait(std::move(started));
    if (threadIdx.x == 0) {
        for (int w = 1; w < kWarps; ++w) best = best_of[w] > best ? best_of[w] : best;
        *cluster.map_shared_rank(&cluster_best[rank], 0) = best;
    }
    cluster.sync();
    if (rank == 0 && threadIdx.x == 0) {
        for (int k = 0; k < S; ++k) best = cluster_best[k] > best ? cluster_best[k] : best;
        a.best_pos[b] = best ? static_cast<int>(key_index(best)) : -1;
        if (a.best_score) a.best_score[b] = best ? key_value(best) : -INFINITY;
    }
}

template <bool E4M3, int GS>
cudaError_t launch(const RankArgs& a, int B, int S, size_t smem, cudaStream_t s) {
    if (smem > kOptInShared - 24 * 1024) {                  // the kernel's own shared memory counts too
        const cudaError_t e =
            cudaFuncSetAttribute(rank_cache_kernel<E4M3, GS>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
        if (e != cudaSuccess) return e;
    }
    return launch_pdl(rank_cache_kernel<E4M3, GS>, dim3(static_cast<unsigned>(B) * S), dim3(kThreads), smem, s, S, a);
}
template <bool E4M3>
cudaError_t launch_group(const RankArgs& a, int B, int S, size_t smem, cudaStream_t s) {
    const int pieces = a.c.vec_bytes / 16;
    if (pieces <= 8) return launch<E4M3, 8>(a, B, S, smem, s);
    if (pieces <= 16) return launch<E4M3, 16>(a, B, S, smem, s);
    return launch<E4M3, 32>(a, B, S, smem, s);
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
    const size_t smem = (static_cast<size_t>(n_sel) * (p->cache.head_dim + 1) * sizeof(float) +
                         (static_cast<size_t>(n_sel) + 2 * (n_sel < p->cache.heads ? n_sel : p->cache.heads) + 1) * sizeof(uint16_t) + 15) / 16 * 16;
    // CTAs a sequence: up to eight, as many as fill the GPU, each with four candidates at least
    int S = 1;
    while (S < 8 && 2 * S * p->B <= 2 * sm_count() && 8 * S <= p->C_cap) S *= 2;
    if (static_cast<int64_t>(p->B) * S > INT32_MAX) return fail(PLDP_ERR_UNSUPPORTED, "%s: too many sequences", fn);
    auto s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = p->cache.dtype == PLDP_E4M3 ? launch_group<true>(a, p->B, S, smem, s) : launch_group<false>(a, p->B, S, smem, s);
    return launched(fn, e);
}
