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

// page_of's constants for a divisor from 1 on.
inline void divide_by(int d, uint32_t* mul, uint32_t* shift) {
    uint32_t l = 0;
    while ((uint64_t(1) << l) < static_cast<uint64_t>(d)) ++l;
    *shift = l;
    *mul = static_cast<uint32_t>((((uint64_t(1) << l) - d) << 32) / d + 1);
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

// The packed tokens of one sequence.
struct PackedRows {
    int row;     // its first one
    int first;   // the position of that
    int count;   // tokens with a position below the capacity; 0: nothing to do
    int given;   // and the rows that it has in all
};
__device__ __forceinline__ PackedRows packed_rows(const int32_t* rows, const int32_t* start, int b, int R, int capacity,
                                                  uint32_t& status) {
    const int r0 = __ldg(rows + b), r1 = __ldg(rows + b + 1), p = start ? __ldg(start + b) : 0;
    status = 0;
    if (r0 < 0 || r1 < r0 || r1 > R) {
        status = PLDP_ST_SEQ_LEN;
        return {0, 0, 0, 0};
    }
    if (p < 0 || p > capacity) {
        status = PLDP_ST_SEQ_LEN;
        return {r0, 0, 0, r1 - r0};
    }
    int count = r1 - r0;
    if (count > capacity - p) {
        status = PLDP_ST_CAPACITY;
        count = capacity - p;
    }
    return {r0, p, count, r1 - r0};
}

// The sequence that a row belongs to, one whose pair lies within [0, R] and holds it, or -1; `hint` is looked at first.  Where
// the list ascends, bisection finds the one pair that can be it.  Where it does not, bisection may end elsewhere, and all pairs are
// looked at by the GS lanes (`lane` of `mates`) that ask together; `ascends` (-1: not known yet) is theirs to keep, so that the rows
// behind the last sequence pay for that look once.
template <int GS>
__device__ __forceinline__ int sequence_of(const int32_t* rows, int B, int R, int row, int hint, int lane, unsigned mates, int& ascends) {
    auto holds = [&](int b) {
        const int r0 = __ldg(rows + b), r1 = __ldg(rows + b + 1);
        return r0 >= 0 && r0 <= row && row < r1 && r1 <= R;
    };
    if (holds(hint)) return hint;
    int lo = 0, hi = B;
    while (hi - lo > 1) {
        const int mid = lo + ((hi - lo) >> 1);
        if (__ldg(rows + mid) <= row) lo = mid;
        else hi = mid;
    }
    if (holds(lo)) return lo;
    if (ascends < 0) {
        bool up = true;
#pragma unroll 1
        for (int64_t b = lane; b < B; b += GS) up = up && __ldg(rows + b) <= __ldg(rows + b + 1);
        ascends = __all_sync(mates, up);
    }
    if (ascends) return -1;
    unsigned found = 0xFFFFFFFFu;
#pragma unroll 1
    for (int64_t b = lane; b < B && found == 0xFFFFFFFFu; b += GS)
        if (holds(static_cast<int>(b))) found = static_cast<unsigned>(b);
    return static_cast<int>(__reduce_min_sync(mates, found));
}

}  // namespace pldp
