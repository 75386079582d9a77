// Attention of a step's tokens over the paged cache: pldp_attend_cache.
#include <math.h>

#include "pldp_attend.cuh"

namespace pldp {
namespace {

// Rows a CTA takes at once: the fewest columns that hold them all (one pass over the keys; a tile takes 1.0 us with 16
// columns, 1.3 with 48, 1.4 with 64, heads of 64 in e4m3), up to
// 128, or 32 for heads above 128 elements, whose tiles leave no more shared memory.
int columns_of(int rows, int head_dim) {
    const int most = head_dim > 128 ? 32 : 128;
    for (const int nt : {16, 32, 48, 64, 96})
        if (rows <= nt && nt <= most) return nt;
    return most;
}
int padded_dim(int head_dim) { return head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256; }

// The workspace: a ticket for each CTA, at a place that no shape moves, so that calls of any shapes find them zeroed;
// then the parts, which need not be.
constexpr size_t kTicketBytes = 1024;
static_assert(kMaxCtas * sizeof(uint32_t) <= kTicketBytes, "tickets");
size_t space_of(int64_t n, int64_t q_heads, int64_t heads, int head_dim) {
    const int64_t rows = n * (q_heads / heads);
    const int nt = columns_of(rows > 128 ? 128 : static_cast<int>(rows), head_dim);
    return kTicketBytes + static_cast<size_t>(2 * kMaxCtas) * nt * (padded_dim(head_dim) + 2) * sizeof(float);
}

}  // namespace

TensorMapEncoder tensor_map_encoder() {
    static const auto encode = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            f = nullptr;
        return reinterpret_cast<TensorMapEncoder>(f);
    }();
    return encode;
}

// The pool as a tensor of (element, position, head, page), its middle dimensions by ascending
// stride, copied in boxes of `box` positions of one head of one page: 64 elements of bf16, swizzled as the
// matrix instructions read them, or a whole vector of codes.
bool pool_map(CUtensorMap* map, void* base, const CacheView& c, bool e4m3, int box, int pitch, bool* head_first) {
    const auto encode = tensor_map_encoder();
    if (!encode) return false;
    // the stride of a dimension of one is never used; any that the map takes will do
    const auto used = [&](int64_t stride, int size) { return static_cast<cuuint64_t>(size == 1 ? c.vec_bytes : stride); };
    const cuuint64_t pos = used(c.pos_stride, c.page_size), head = used(c.head_stride, c.heads);
    *head_first = head < pos;
    const cuuint64_t d = c.head_dim, p = c.page_size, h = c.heads;
    const cuuint64_t dims[4] = {d, *head_first ? h : p, *head_first ? p : h, static_cast<cuuint64_t>(c.n_pages)};
    const cuuint64_t strides[3] = {*head_first ? head : pos, *head_first ? pos : head, used(c.page_stride, c.n_pages)};
    const cuuint32_t inner = e4m3 ? pitch : 64, rows = box;
    const cuuint32_t size[4] = {inner, *head_first ? 1u : rows, *head_first ? rows : 1u, 1u}, step[4] = {1u, 1u, 1u, 1u};
    return encode(map, e4m3 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, base, dims, strides, size, step,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, e4m3 ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace pldp

using namespace pldp;

extern "C" {

PLDP_API size_t pldp_attend_workspace_size(int B, int n, int q_heads, int heads, int head_dim) {
    if (B < 0 || n < 1 || q_heads < 1 || heads < 1 || q_heads % heads || head_dim < 1) return 0;
    return (space_of(n, q_heads, heads, head_dim) + 255) / 256 * 256;
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
    // (tiles are counted past the last position)
    if (a.c.capacity > INT32_MAX - 4095)
        return fail(PLDP_ERR_UNSUPPORTED, "%s: more than 2^31 - 4096 positions a sequence", fn);
    if (p->q_heads % p->cache.heads)
        return fail(PLDP_ERR_INVALID_ARG, "%s: q_heads must be a multiple of the cache's heads", fn);
    const int64_t rows = static_cast<int64_t>(p->n) * (p->q_heads / p->cache.heads);
    if (rows > (1 << 24) || static_cast<int64_t>(p->B) * p->cache.heads * ((rows + 15) / 16) > INT32_MAX)
        return fail(PLDP_ERR_UNSUPPORTED, "%s: too many rows", fn);
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
    a.B = p->B, a.n = p->n, a.q_heads = p->q_heads, a.group = p->q_heads / p->cache.heads;
    a.scale2 = p->scale * 1.4426950408889634f;
    const int nt = columns_of(static_cast<int>(rows), p->cache.head_dim);
    a.row_tiles = static_cast<int>((rows + nt - 1) / nt);
    a.tickets = static_cast<uint32_t*>(p->workspace);
    a.parts = reinterpret_cast<float*>(static_cast<uint8_t*>(p->workspace) + kTicketBytes);
    const int64_t most = static_cast<int64_t>(p->B) * p->cache.heads * a.row_tiles * ((a.c.capacity + int64_t(kTile) - 1) / kTile);
    int ctas = sm_count() < kMaxCtas ? sm_count() : kMaxCtas;
    if (most < ctas) ctas = static_cast<int>(most);
    const bool e4m3 = p->cache.dtype == PLDP_E4M3;
    a.box = kTile;                                           // the largest power of two that divides the page, up to a tile
    while (p->cache.page_size % a.box) a.box /= 2;
    // a copy starts at a multiple of 128 bytes of shared memory: vectors side by side where a box of them is one
    a.pitch = p->cache.head_dim * a.box % 128 == 0 ? p->cache.head_dim : p->cache.head_dim <= 128 ? 128 : 256;
    Maps maps;
    bool head_first = false;
    if (!pool_map(&maps.k, a.c.k, a.c, e4m3, a.box, a.pitch, &head_first) || !pool_map(&maps.v, a.c.v, a.c, e4m3, a.box, a.pitch, &head_first))
        return fail(PLDP_ERR_UNSUPPORTED, "%s: the cache's strides cannot be described to the copy engine", fn);
    a.head_first = head_first;
    auto s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = e4m3 ? launch_attend_e4m3(a, maps, nt, ctas, s) : launch_attend_bf16(a, maps, nt, ctas, s);
    return launched(fn, e);
}

}  // extern "C"
