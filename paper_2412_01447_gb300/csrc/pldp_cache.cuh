// The paged cache as the kernels see it, and the host's checks of its description.
#pragma once

#include "pldp_internal.cuh"

namespace pldp {

constexpr int kMaxHeadDim = 256;
// The smallest scale of an e4m3 vector, which vectors of zeros have as well.  Attention rounds weights relative to the
// largest of weight x scale, so a value of zeros must not count as if it were large; and its sums hold weight / scale up to
// 2^15 2^80 for each of 2^31 keys, which is below 2^127.
constexpr float kLeastScale = 0x1p-80f;

// One cache.  Offsets and strides in bytes; positions are below 2^31.
struct CacheView {
    uint8_t* k;
    uint8_t* v;
    float* k_scale;
    float* v_scale;
    const int32_t* pages;
    int64_t pages_stride, page_stride, pos_stride, head_stride;
    int n_pages, page_size, heads, head_dim, max_pages;
    int capacity;                 // max_pages * page_size
    uint32_t div_mul, div_shift;  // p / page_size = (umulhi(p, div_mul) + p) >> div_shift
    int vec_bytes;                // of one vector
};

// p / page_size for 0 <= p < 2^31, by the round-up method of division by invariant
// integers (Granlund and Montgomery 1994): the sum stays below 2^32.
__host__ __device__ __forceinline__ uint32_t page_of(uint32_t p, uint32_t mul, uint32_t shift) {
#ifdef __CUDA_ARCH__
    return (__umulhi(p, mul) + p) >> shift;
#else
    return static_cast<uint32_t>(((static_cast<uint64_t>(p) * mul >> 32) + p) >> shift);
#endif
}

// Where position p of a sequence lies: byte offset of head 0's vector, or -1 where the page
// table holds no page; `scale_at` the index of head 0's scale.
__device__ __forceinline__ int64_t locate(const CacheView& c, const int32_t* table, int p, int64_t& scale_at) {
    const uint32_t pg = page_of(p, c.div_mul, c.div_shift);
    const int slot = p - static_cast<int>(pg) * c.page_size;
    const int page = __ldg(table + pg);
    scale_at = static_cast<int64_t>(page) * c.heads * c.page_size + slot;
    if (static_cast<unsigned>(page) >= static_cast<unsigned>(c.n_pages)) return -1;
    return page * c.page_stride + slot * c.pos_stride;
}

// Checks a cache description; fills the view.  `B` sequences read it.
pldp_status cache_view(const char* fn, const pldp_cache& c, int B, CacheView* out);
// Strides (sequence, token, head) of a tensor of elements of es bytes: multiples of 16 bytes.
pldp_status check_rows(const char* fn, const char* name, const void* p, const int64_t* strides, size_t es);

// The tokens that a sequence's step holds.
struct StepTokens {
    int first;   // position of x_t
    int count;   // tokens with a position below the capacity; 0: nothing to do
};
__device__ __forceinline__ StepTokens step_tokens(const int32_t* seq_len, const int32_t* draft_len, int b, int n,
                                                  int capacity, uint32_t& status) {
    const int L = __ldg(seq_len + b);
    int d = draft_len ? __ldg(draft_len + b) : n - 1;
    status = 0;
    if (L < 0 || L > capacity) {
        status = PLDP_ST_SEQ_LEN;
        return {0, 0};
    }
    if (L == 0) return {0, 0};
    if (d < 0 || d > n - 1) {
        status |= PLDP_ST_DRAFT_LEN;
        d = d < 0 ? 0 : n - 1;
    }
    int count = d + 1;
    if (count > capacity - (L - 1)) {
        status |= PLDP_ST_CAPACITY;
        count = capacity - (L - 1);
    }
    return {L - 1, count};
}

}  // namespace pldp
