// Causal attention of packed prompts over the paged cache: pldp_attend_prompt, and the join of units that CTAs share.
#include <math.h>

#include "pldp_prompt.cuh"

namespace pldp {
namespace {

constexpr size_t kCutBytes = 8192;
static_assert(kPromptCtas * sizeof(CutUnit) <= kCutBytes, "cuts");

// The queries as a tensor of (element, head, row), in boxes of 64 elements of the heads of one kv head and as many rows as
// make 128 with them.
bool query_map(CUtensorMap* map, const PromptArgs& a, int head_dim) {
    const auto encode = tensor_map_encoder();
    if (!encode) return false;
    const auto used = [&](int64_t stride, int size) { return static_cast<cuuint64_t>(size == 1 ? head_dim : stride) * 2; };
    const cuuint64_t dims[4] = {static_cast<cuuint64_t>(head_dim), static_cast<cuuint64_t>(a.q_heads), static_cast<cuuint64_t>(a.R), 1};
    const cuuint64_t strides[3] = {used(a.q_head, a.q_heads), used(a.q_tok, a.R), static_cast<cuuint64_t>(head_dim) * 2};
    const cuuint32_t size[4] = {64u, static_cast<cuuint32_t>(a.group), static_cast<cuuint32_t>(128 / a.group), 1u}, step[4] = {1u, 1u, 1u, 1u};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<__nv_bfloat16*>(a.q), dims, strides, size, step,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Keys or values of heads of 256 with all four panels of 64 elements of `box` positions in one box: (element, position of 8, panel,
// 8 positions, page).  Two places are all that shared memory has for such tiles, so the time that a box's issue takes
// is not hidden: pages of 24 positions (boxes of 8), three prompts of 2000 behind 4096: 231 us with a box a panel, 183 to 188 so.  (Heads
// of 128, which have six places: nothing.)
bool whole_map(CUtensorMap* map, void* base, const CacheView& c, int box, int* whole) {
    const auto encode = tensor_map_encoder();
    constexpr int panels = 4;
    if (!encode || c.head_dim != panels * 64 || box % 8) return false;
    *whole = c.heads == 1 || c.head_stride == c.vec_bytes ? 1 : c.head_stride == c.page_size * c.pos_stride ? 2 : 0;
    if (!*whole) return false;
    const cuuint64_t p = c.page_size / 8, h = c.heads, n = panels;
    const cuuint64_t dims[5] = {64, 8, *whole == 1 ? n * h : n, *whole == 1 ? p : p * h, static_cast<cuuint64_t>(c.n_pages)};
    const cuuint64_t pos = static_cast<cuuint64_t>(c.pos_stride), page = c.n_pages == 1 ? pos * 8 : static_cast<cuuint64_t>(c.page_stride);
    const cuuint64_t strides[4] = {pos, 128, pos * 8, page};
    const cuuint32_t size[5] = {64u, 8u, static_cast<cuuint32_t>(panels), static_cast<cuuint32_t>(box / 8), 1u}, step[5] = {1u, 1u, 1u, 1u, 1u};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, base, dims, strides, size, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int prompt_ctas() {
    const int n = sm_count();
    return n < kPromptCtas ? n : kPromptCtas;
}

// The parts of a unit joined: 32 rows a block, a row a lane; the warps share the head's elements.
constexpr int kJoinThreads = 256;

template <int DP>
__global__ void __launch_bounds__(kJoinThreads) prompt_join_kernel(const PromptArgs a) {
    pdl_enter();
    const CutUnit cut = a.cuts[blockIdx.x];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, row = blockIdx.y * 32 + lane, D = a.c.head_dim;
    if (cut.parts == 0 || row >= cut.rows) return;
    const int q = row >> 7, j = row & 127;
    auto place = [&](int k) {
        return a.parts + static_cast<int64_t>(2 * (cut.first_cta + k) + (k == 0 ? 1 : 0)) * prompt_part(DP) + q * 128 * (DP + 2);
    };
    float M = -INFINITY, sum = 0.f;
#pragma unroll 1
    for (int k0 = 0; k0 < cut.parts; k0 += 8) {
        float m[8], l[8], top = M;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            m[i] = -INFINITY, l[i] = 0.f;
            if (k0 + i < cut.parts) m[i] = __ldcg(place(k0 + i) + 128 * DP + j), l[i] = __ldcg(place(k0 + i) + 128 * DP + 128 + j);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, m[i]);
        if (!(top > -INFINITY)) continue;
        sum *= ex2(M - top);                                     // (2^-inf of the first)
        M = top;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = fmaf(ex2(m[i] - M), l[i], sum);
    }
    const int r = cut.row0 + row, tok = r / a.group;
    const int64_t at = cut.row_base + static_cast<int64_t>(tok), head = static_cast<int64_t>(cut.kv) * a.group + (r - tok * a.group);
    if (warp == 0 && a.lse) a.lse[at * a.q_heads + head] = sum == 0.f ? -INFINITY : (log2f(sum) + M) * 0.69314718055994531f;
    const float inverse = sum == 0.f ? 0.f : 1.f / sum;
    __nv_bfloat16* out = a.out + at * a.o_tok + head * a.o_head;
#pragma unroll 1
    for (int d = warp * 8; d < D; d += kJoinThreads / 32 * 8) {
        float o[8] = {};
#pragma unroll 1
        for (int k0 = 0; k0 < cut.parts; k0 += 4) {
            float4 x[4][2];
            float by[4], l[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                by[i] = -INFINITY, l[i] = 0.f;
                if (k0 + i < cut.parts) {
                    const float* p = place(k0 + i);
                    by[i] = __ldcg(p + 128 * DP + j), l[i] = __ldcg(p + 128 * DP + 128 + j);
                    x[i][0] = __ldcg(reinterpret_cast<const float4*>(p + (d / 4 * 128 + j) * 4));
                    x[i][1] = __ldcg(reinterpret_cast<const float4*>(p + ((d / 4 + 1) * 128 + j) * 4));
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float f = sum == 0.f ? 0.f : ex2(by[i] - M) * l[i] * inverse;            // the part's share, 1 at most
                if (f == 0.f) continue;
                o[0] = fmaf(f, x[i][0].x, o[0]), o[1] = fmaf(f, x[i][0].y, o[1]), o[2] = fmaf(f, x[i][0].z, o[2]), o[3] = fmaf(f, x[i][0].w, o[3]);
                o[4] = fmaf(f, x[i][1].x, o[4]), o[5] = fmaf(f, x[i][1].y, o[5]), o[6] = fmaf(f, x[i][1].z, o[6]), o[7] = fmaf(f, x[i][1].w, o[7]);
            }
        }
        *reinterpret_cast<uint4*>(out + d) = make_uint4(pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3]), pack_bf16(o[4], o[5]), pack_bf16(o[6], o[7]));
    }
}

}  // namespace
}  // namespace pldp

using namespace pldp;

extern "C" {

PLDP_API size_t pldp_attend_prompt_workspace_size(int q_heads, int heads, int head_dim) {
    if (q_heads < 1 || heads < 1 || q_heads % heads || head_dim < 1 || head_dim > kMaxHeadDim) return 0;
    return kCutBytes + static_cast<size_t>(2 * prompt_ctas()) * prompt_part(prompt_dim(head_dim)) * sizeof(float);
}

PLDP_API pldp_status pldp_attend_prompt(const pldp_attend_prompt_args* p, void* stream) {
    const char* fn = "attend_prompt";
    if (!p) return fail(PLDP_ERR_INVALID_ARG, "%s: null argument block", fn);
    if (p->B < 0 || p->R < 0 || p->q_heads < 1)
        return fail(PLDP_ERR_INVALID_ARG, "%s: B < 0, R < 0 or q_heads < 1", fn);
    if (!isfinite(p->scale)) return fail(PLDP_ERR_INVALID_ARG, "%s: scale must be finite", fn);
    PromptArgs a = {};
    pldp_status st = cache_view(fn, p->cache, p->B, &a.c);
    if (st != PLDP_OK) return st;
    // (tiles are counted past the last position)
    if (a.c.capacity > INT32_MAX - 4095)
        return fail(PLDP_ERR_UNSUPPORTED, "%s: more than 2^31 - 4096 positions a sequence", fn);
    if (p->q_heads % p->cache.heads)
        return fail(PLDP_ERR_INVALID_ARG, "%s: q_heads must be a multiple of the cache's heads", fn);
    a.group = p->q_heads / p->cache.heads;
    if (p->R > INT32_MAX - 256 || static_cast<int64_t>(p->R) * a.group > INT32_MAX - 4095)
        return fail(PLDP_ERR_UNSUPPORTED, "%s: too many rows", fn);
    if (p->B == 0) return PLDP_OK;
    if (!p->rows || !p->workspace || (p->R > 0 && (!p->q || !p->out))) return fail(PLDP_ERR_INVALID_ARG, "%s: null pointer", fn);
    const int64_t qs[3] = {0, p->q_strides[0], p->q_strides[1]}, os[3] = {0, p->out_strides[0], p->out_strides[1]};
    if ((st = check_rows(fn, "q", p->q, qs, 2)) != PLDP_OK) return st;
    if ((st = check_rows(fn, "out", p->out, os, 2)) != PLDP_OK) return st;
    const size_t need = pldp_attend_prompt_workspace_size(p->q_heads, p->cache.heads, p->cache.head_dim);
    if (p->workspace_bytes < need)
        return fail(PLDP_ERR_INVALID_ARG, "%s: workspace needs %zu bytes, has %zu", fn, need, p->workspace_bytes);
    if (reinterpret_cast<uintptr_t>(p->workspace) & 255u)
        return fail(PLDP_ERR_INVALID_ARG, "%s: workspace is not 256-byte aligned", fn);
    a.q = static_cast<const __nv_bfloat16*>(p->q);
    a.out = static_cast<__nv_bfloat16*>(p->out);
    a.q_tok = p->q_strides[0], a.q_head = p->q_strides[1], a.o_tok = p->out_strides[0], a.o_head = p->out_strides[1];
    a.rows = p->rows, a.start = p->start;
    a.lse = p->lse;
    a.status = p->status;
    a.cuts = static_cast<CutUnit*>(p->workspace);
    a.parts = reinterpret_cast<float*>(static_cast<uint8_t*>(p->workspace) + kCutBytes);
    a.B = p->B, a.R = p->R, a.q_heads = p->q_heads;
    divide_by(a.group, &a.group_mul, &a.group_shift);
    // A negative scale turns the queries' signs, so that larger scores are larger weights; one of zero is the least that
    // keeps a masked score at -infinity (as it is once an e4m3 cache's kernel has taken its queries' power of two out).
    a.scale2 = fmaxf(fabsf(p->scale) * 1.4426950408889634f, 0x1p-126f);
    a.flip = p->scale < 0.f ? 0x80008000u : 0u;
    a.box = kTile;                                           // the largest power of two that divides the page, up to a tile
    while (p->cache.page_size % a.box) a.box /= 2;
    const bool e4m3 = p->cache.dtype == PLDP_E4M3;
    const int dp = prompt_dim(p->cache.head_dim);
    if (e4m3 && dp == 256 && a.box > 64) a.box = 64;         // (a stage holds half a tile)
    // a copy starts at a multiple of 128 bytes of shared memory: vectors side by side where a box of them is one
    a.pitch = p->cache.head_dim * a.box % 128 == 0 ? p->cache.head_dim : p->cache.head_dim <= 128 ? 128 : 256;
    PromptMaps maps = {};
    bool head_first = false;
    a.group_step = 1024, a.panel_step = kTile * 128;
    if (!e4m3 && whole_map(&maps.pool.k, a.c.k, a.c, a.box, &a.whole) && whole_map(&maps.pool.v, a.c.v, a.c, a.box, &a.whole))
        a.group_step = dp / 64 * 1024, a.panel_step = 1024;
    else if (a.whole = 0, !pool_map(&maps.pool.k, a.c.k, a.c, e4m3, a.box, a.pitch, &head_first) || !pool_map(&maps.pool.v, a.c.v, a.c, e4m3, a.box, a.pitch, &head_first))
        return fail(PLDP_ERR_UNSUPPORTED, "%s: the cache's strides cannot be described to the copy engine", fn);
    a.head_first = head_first;
    // (signs are turned on the way by the other form)
    a.q_boxes = 128 % a.group == 0 && (e4m3 || !a.flip) && p->R > 0 && query_map(&maps.q, a, p->cache.head_dim);
    // No more CTAs than the most tiles make parts for (rows that several sequences claim, which is none of their uses, make
    // parts longer), and no join where no unit is long enough to be cut: 47 tokens, 32 heads over 8, 19.6 us before and
    // 17.5 with both, from a cold L2.
    const int64_t positions = p->start || p->R > a.c.capacity ? a.c.capacity : p->R, tiles = (positions + kTile - 1) / kTile;
    const int64_t units = p->cache.heads * (static_cast<int64_t>(p->R) * a.group / prompt_rows(dp) + p->B);
    const int64_t parts = (units * (tiles + kUnitCost) + kLeast - 1) / kLeast;
    const int most = prompt_ctas(), ctas = parts < most ? static_cast<int>(parts > 0 ? parts : 1) : most;
    auto s = static_cast<cudaStream_t>(stream);
    cudaError_t e = e4m3 ? launch_prompt_e4m3(a, maps, ctas, s) : launch_prompt_bf16(a, maps, ctas, s);
    if (e != cudaSuccess || tiles <= kWhole) return launched(fn, e);
    const dim3 grid(ctas, prompt_rows(dp) / 32);
    e = dp == 64    ? launch_pdl(prompt_join_kernel<64>, grid, dim3(kJoinThreads), 0, s, 0, a)
        : dp == 128 ? launch_pdl(prompt_join_kernel<128>, grid, dim3(kJoinThreads), 0, s, 0, a)
                    : launch_pdl(prompt_join_kernel<256>, grid, dim3(kJoinThreads), 0, s, 0, a);
    return launched(fn, e);
}

}  // extern "C"
