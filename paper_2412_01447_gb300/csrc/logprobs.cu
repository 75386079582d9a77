// Log probabilities of tokens, entropy and alternatives: pldp_token_logprobs.
#include <float.h>
#include <math.h>

#include "pldp_internal.cuh"

namespace pldp {
namespace {

// With x = logits / T in units of log2 (y = logit * c, c = log2(e) / T) and the row's maximum M,
//   L = sum 2^(y - M),  U = sum 2^(y - M) (y - M):
//   logprob = ln2 (y_token - M - log2 L),   entropy = ln2 (log2 L - U / L).
//
// 1. A pass reads the logits once, in units of 2 KB of a row, a warp a unit (four 16-byte loads a lane):
//    L and U against the unit's own maximum, and the maximum of each 512 bytes.
// 2. One CTA a row joins them.  The row's top k elements lie in the k chunks of 512 bytes whose maxima
//    are largest (ties to the lower chunk): each element elsewhere has k such maxima before it.  So only
//    those are read again (4% of a row of 128256 bf16 for k = 20).
//
// Bound by reading the logits, then by the second pass's chain of a row (its units' sums, k chunks, their elements).
// 1664 rows of 128256 bf16 (427 MB), k = 20, L2 flushed: 86 us, 5.0 TB/s (the pass 72); 11 rows of
// 32000 fp32, k = 5: 5.5 us.
constexpr int kThreads = 256, kWarps = kThreads / 32, kLoads = 4;
constexpr int kBlocksPerSm = 5, kWaves = 11;
constexpr int kMaxTop = 32;
constexpr int kUnitBytes = kLoads * 32 * 16;

struct LogprobArgs {
    const int32_t* tokens;
    float *logprob, *entropy, *top_logprob;
    int32_t* top_id;
    float4* maxima;      // [rows * units]: of each load
    float2* sums;        // [rows * units]: L, U against the largest of them
    int64_t rows;
    uint32_t V, units;   // units a row
    uint32_t step_rows, step_units;   // of the grid's warps: their number in rows and units
    uint32_t lead;       // elements from a 16-byte boundary to the first logit
    int top;
    float c;
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float warp_max(float v) {
    float m;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(m) : "f"(v));
    return m;
}
__device__ __forceinline__ void unpack(const uint4& x, float (&e)[8]) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        e[2 * k] = __uint_as_float(w[k] << 16);
        e[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void unpack(const uint4& x, float (&e)[4]) {
    e[0] = __uint_as_float(x.x), e[1] = __uint_as_float(x.y), e[2] = __uint_as_float(x.z), e[3] = __uint_as_float(x.w);
}

// Rows that are not whole vectors, or do not start at one: a row starts `head` elements into a
// vector, units are cut at whole vectors all the same, and the two vectors that other rows share are
// read element by element, -inf in the place of what is not the row's.
template <typename T>
__device__ __forceinline__ uint32_t head_of(const LogprobArgs& a, int64_t r) {
    return static_cast<uint32_t>((static_cast<uint64_t>(r) * a.V + a.lead) % (16 / sizeof(T)));
}
template <typename T>
__device__ __noinline__ uint4 cut_vector(const T* row, int64_t at, int64_t V) {   // elements at.. of a row, some outside [0, V)
    uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int j = 0; j < static_cast<int>(16 / sizeof(T)); ++j) {
        const bool in = at + j >= 0 && at + j < V;
        if constexpr (sizeof(T) == 2)
            w[j / 2] |= (in ? static_cast<uint32_t>(__bfloat16_as_ushort(row[at + j])) : 0xFF80u) << (16 * (j % 2));
        else
            w[j] = in ? __float_as_uint(row[at + j]) : 0xFF800000u;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// The vector at element `at` of a row (relative to its first, head elements before it a vector's start).
template <typename T, bool CUT>
__device__ __forceinline__ uint4 row_vector(const T* row, int64_t at, int64_t V) {
    if (CUT && (at < 0 || at + static_cast<int>(16 / sizeof(T)) > V)) return cut_vector<T>(row, at, V);
    return ld_stream16(row + at);
}

template <typename T, bool CUT>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm) logprob_sums_kernel(const T* __restrict__ logits, const LogprobArgs a) {
    pdl_wait_only();
    constexpr int VW = 16 / sizeof(T), P = kUnitBytes / sizeof(T);
    const int lane = threadIdx.x & 31;
    // the grid's warps take units in turn: each turn is step_rows rows and step_units units further
    const uint32_t start = blockIdx.x * kWarps + (threadIdx.x >> 5), V = a.V;
    uint32_t r = start / a.units, k = start - r * a.units;
#pragma unroll 1
    for (; r < a.rows; r += a.step_rows, k += a.step_units) {
        if (k >= a.units) {
            k -= a.units;
            if (++r >= a.rows) break;
        }
        const uint32_t head = CUT ? head_of<T>(a, r) : 0u;
        const T* row = logits + static_cast<int64_t>(r) * V;
        const int32_t e0 = static_cast<int32_t>(k * P - head + lane * VW);      // (V + a unit is below 2^31)
        uint4 raw[kLoads];
#pragma unroll
        for (int q = 0; q < kLoads; ++q) {
            const int32_t at = e0 + q * 32 * VW;
            raw[q] = sizeof(T) == 2 ? make_uint4(0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u)
                                    : make_uint4(0xFF800000u, 0xFF800000u, 0xFF800000u, 0xFF800000u);
            if (at < static_cast<int32_t>(V)) raw[q] = row_vector<T, CUT>(row, at, V);
        }
        float top[kLoads], m = -INFINITY;
#pragma unroll
        for (int q = 0; q < kLoads; ++q) {
            top[q] = vmax(raw[q], T());
            m = fmaxf(m, top[q]);
        }
        // a lane's sums against its own maximum, the differences first (l - m) and the factor after, so that
        // large offsets and the lowest values cost nothing; what weighs nothing must not make 0 * inf
        float L = 0.f, U = 0.f;
        if (m > -INFINITY) {
            const uint64_t c2 = pack_f32x2(a.c, a.c), m2 = pack_f32x2(-m, -m);
            uint64_t l2 = 0, u2 = 0;
            auto add = [&](bool far) {
#pragma unroll
                for (int q = 0; q < kLoads; ++q) {
                    float e[VW];
                    unpack(raw[q], e);
#pragma unroll
                    for (int j = 0; j < VW; j += 2) {
                        uint64_t y = fma_f32x2(add_f32x2(pack_f32x2(e[j], e[j + 1]), m2), c2, 0ull);
                        if (far) y = pack_f32x2(fmaxf(lo_f32(y), -1000.f), fmaxf(hi_f32(y), -1000.f));
                        const uint64_t w = pack_f32x2(ex2(lo_f32(y)), ex2(hi_f32(y)));
                        l2 = add_f32x2(l2, w);
                        u2 = fma_f32x2(w, y, u2);
                    }
                }
            };
            add(false);
            if (!(hi_f32(u2) + lo_f32(u2) > -INFINITY)) {          // 0 * inf somewhere
                l2 = u2 = 0;
                add(true);
            }
            L = lo_f32(l2) + hi_f32(l2);
            U = lo_f32(u2) + hi_f32(u2);
        }
        float4 best;
        best.x = warp_max(top[0]);
        best.y = warp_max(top[1]);
        best.z = warp_max(top[2]);
        best.w = warp_max(top[3]);
        const float M = fmaxf(fmaxf(best.x, best.y), fmaxf(best.z, best.w));
        if (L != 0.f) {
            const float d = fmaxf((m - M) * a.c, -1000.f), by = ex2(d);
            U = (U + L * d) * by;
            L *= by;
        }
        L = warp_sum(L);
        U = warp_sum(U);
        if (lane == 0) {
            const int64_t u = static_cast<int64_t>(r) * a.units + k;
            a.maxima[u] = best;
            a.sums[u] = make_float2(L, U);
        }
    }
}

__device__ __forceinline__ unsigned long long warp_best(unsigned long long v) {   // the largest key of the warp
    const uint32_t hi = __reduce_max_sync(0xFFFFFFFFu, static_cast<uint32_t>(v >> 32));
    const uint32_t lo = __reduce_max_sync(0xFFFFFFFFu, static_cast<uint32_t>(v >> 32) == hi ? static_cast<uint32_t>(v) : 0u);
    return static_cast<unsigned long long>(hi) << 32 | lo;
}

// The k best elements of a row by one warp, whatever the row holds: the k chunks with the largest maxima in
// order, then their elements into a list of the best, one a lane.  (Each turn waits for the last.)
template <typename T, bool CUT>
__device__ __noinline__ unsigned long long best_in_turn(const T* row, const float* chunk_max, uint32_t chunks, uint32_t head, int64_t V,
                                                        int top) {
    constexpr int VW = 16 / sizeof(T), CE = 32 * VW;              // elements of a chunk
    const int lane = threadIdx.x & 31;
    unsigned long long last = ~0ull, own = 0, list = 0;
    uint32_t mine = 0;
    const int want = min(static_cast<uint32_t>(top), chunks);
    auto best_own = [&] {                                         // this lane's next chunk
        own = 0;
        for (uint32_t ch = lane; ch < chunks; ch += 32) {
            const unsigned long long key = pack_key(__ldcg(chunk_max + ch), ch);
            if (key < last && key > own) own = key;
        }
    };
    best_own();
    for (int i = 0; i < want; ++i) {
        last = warp_best(own);
        if (lane == i) mine = key_index(last);
        if (own == last) best_own();
    }
    for (int i = 0; i < want; ++i) {
        const int64_t first = static_cast<int64_t>(__shfl_sync(0xFFFFFFFFu, mine, i)) * CE - head + lane * VW;
        uint4 raw = make_uint4(0u, 0u, 0u, 0u);
        if (first < V) raw = row_vector<T, CUT>(row, first, V);
        float e[VW];
        unpack(raw, e);
        unsigned taken = 0;
        while (true) {
            const unsigned long long kth = __shfl_sync(0xFFFFFFFFu, list, top - 1);
            unsigned long long cand = 0;
            int which = 0;
#pragma unroll
            for (int j = 0; j < VW; ++j) {
                const int64_t v = first + j;
                const unsigned long long key = pack_key(e[j], static_cast<uint32_t>(v));
                if (v >= 0 && v < V && !(taken >> j & 1u) && key > kth && key > cand) cand = key, which = j;
            }
            if (!__any_sync(0xFFFFFFFFu, cand != 0)) break;
            const unsigned long long best = warp_best(cand);
            if (cand == best) taken |= 1u << which;
            const int place = __popc(__ballot_sync(0xFFFFFFFFu, list > best));
            const unsigned long long above = __shfl_up_sync(0xFFFFFFFFu, list, 1);
            if (lane > place) list = above;
            if (lane == place) list = best;
        }
    }
    return list;
}

constexpr int kFinishThreads = 128, kFinishWarps = kFinishThreads / 32;
// A row is a chain of loads that wait for one another, so the more rows an SM has at once the better, as long as
// registers do (1664 rows, both passes: 86.3 us; with 9 CTAs an SM 89.2, with 16 87.2).
constexpr int kFinishBlocks = 12;
static_assert(kMaxTop * kLoads <= kFinishThreads, "a chunk a thread");
constexpr int kChunkList = 64, kElementList = 256;    // chunks and elements that a row's alternatives are picked from

// One CTA a row.  The k-th largest of the threads' own largest chunk maxima is a value that k elements reach: the
// chunks that reach it (k, or a few more) are read again, the elements that reach it counted against one
// another for their places.  Rows that have more of either (few distinct values) take them in turn.
template <typename T, bool CUT>
__global__ void __launch_bounds__(kFinishThreads, kFinishBlocks) logprob_finish_kernel(const T* __restrict__ logits, const LogprobArgs a) {
    pdl_enter();
    constexpr int VW = 16 / sizeof(T), CE = 32 * VW;
    __shared__ __align__(16) uint32_t maxima_of[kFinishThreads];
    __shared__ float part[3][kFinishWarps];
    __shared__ uint32_t list[kChunkList];
    __shared__ unsigned long long elements[kElementList];
    __shared__ int chunk_count, element_count;
    __shared__ float floor_value;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int64_t r = blockIdx.x, V = a.V;
    const T* row = logits + r * V;
    const float4* maxima = a.maxima + r * a.units;
    const float* chunk_max = reinterpret_cast<const float*>(maxima);
    const float2* sums = a.sums + r * a.units;
    const uint32_t chunks = a.units * kLoads;
    float at_token = -INFINITY;
    if (tid == 0 && a.tokens) {
        const int token = __ldg(a.tokens + r);
        if (token >= 0 && token < static_cast<int>(a.V)) at_token = to_f32(row[token]);
    }
    // a thread's first unit stays in registers: rows of up to 128 units are read once
    auto top_of = [](const float4& t) { return fmaxf(fmaxf(t.x, t.y), fmaxf(t.z, t.w)); };
    float4 mine = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
    float2 mine_sums = make_float2(0.f, 0.f);
    if (tid < a.units) mine = __ldcg(maxima + tid), mine_sums = __ldcg(sums + tid);
    float own = top_of(mine);
    // (of few units a chunk each: `top` threads have to have one)
    if (a.units <= kMaxTop) own = tid < chunks ? __ldcg(chunk_max + tid) : -INFINITY;
    for (uint32_t k = tid + kFinishThreads; k < a.units; k += kFinishThreads) own = fmaxf(own, top_of(__ldcg(maxima + k)));
    // (a float's order, its last seven bits given up for the thread's: all different, lower threads first)
    const uint32_t own_key = (ordered_key(own) & ~127u) | (127u - tid);
    maxima_of[tid] = own_key;
    const float top_of_warp = warp_max(own);
    if (lane == 0) part[0][warp] = top_of_warp;
    if (tid == 0) {
        chunk_count = element_count = 0;
        floor_value = -INFINITY;
    }
    __syncthreads();
    const float M = fmaxf(fmaxf(part[0][0], part[0][1]), fmaxf(part[0][2], part[0][3]));
    float L = 0.f, U = 0.f;
    if (M > -INFINITY) {
        auto add = [&](const float4& t, const float2& s) {
            const float d = fmaxf((top_of(t) - M) * a.c, -1000.f), by = ex2(d);
            if (s.x != 0.f) {
                L = fmaf(s.x, by, L);
                U = fmaf(s.y + s.x * d, by, U);
            }
        };
        add(mine, mine_sums);
        for (uint32_t k = tid + kFinishThreads; k < a.units; k += kFinishThreads) add(__ldcg(maxima + k), __ldcg(sums + k));
    }
    L = warp_sum(L);
    U = warp_sum(U);
    if (lane == 0) part[1][warp] = L, part[2][warp] = U;
    // this thread's place among the maxima
    if (a.top) {
        int place = 0;
#pragma unroll 8
        for (int t = 0; t < kFinishThreads; t += 4) {
            const uint4 o = *reinterpret_cast<const uint4*>(maxima_of + t);
            place += (o.x > own_key) + (o.y > own_key) + (o.z > own_key) + (o.w > own_key);
        }
        if (place == a.top - 1) {
            const uint32_t low = own_key & ~127u;          // at most this thread's maximum, as at most the others before it
            floor_value = __uint_as_float(low & 0x80000000u ? low & 0x7FFFFFFFu : ~low);
            if (!(own > -INFINITY)) floor_value = -INFINITY;
        }
    }
    __syncthreads();
    constexpr float kLn2 = 0.69314718055994531f;
    L = (part[1][0] + part[1][1]) + (part[1][2] + part[1][3]);
    U = (part[2][0] + part[2][1]) + (part[2][2] + part[2][3]);
    const float log_l = log2f(L);                                 // L >= 1 unless the row is empty
    if (tid == 0) {
        if (a.logprob) a.logprob[r] = at_token > -INFINITY ? ((at_token - M) * a.c - log_l) * kLn2 : -INFINITY;
        if (a.entropy) a.entropy[r] = M > -INFINITY ? (log_l - U / L) * kLn2 : 0.f;
    }
    if (a.top == 0) return;
    const float reach = floor_value;
    auto pick = [&](float top, uint32_t ch) {
        if (top >= reach) {
            const int at = atomicAdd(&chunk_count, 1);
            if (at < kChunkList) list[at] = ch;
        }
    };
    for (uint32_t k = tid; k < a.units; k += kFinishThreads) {
        const float4 t = k == tid ? mine : __ldcg(maxima + k);
        pick(t.x, 4 * k);
        pick(t.y, 4 * k + 1);
        pick(t.z, 4 * k + 2);
        pick(t.w, 4 * k + 3);
    }
    __syncthreads();
    const uint32_t head = CUT ? head_of<T>(a, r) : 0u;
    const int n = chunk_count;
    if (n <= kChunkList) {
        constexpr int kAhead = 4;
        for (int i0 = warp; i0 < n; i0 += kFinishWarps * kAhead) {
            uint4 raw[kAhead];
            int64_t first[kAhead];
#pragma unroll
            for (int p = 0; p < kAhead; ++p) {
                const int i = i0 + p * kFinishWarps;
                first[p] = V;
                if (i < n) first[p] = static_cast<int64_t>(list[i]) * CE - head + lane * VW;
                if (first[p] < V) raw[p] = row_vector<T, CUT>(row, first[p], V);
            }
#pragma unroll
            for (int p = 0; p < kAhead; ++p) {
                if (first[p] >= V) continue;
                float e[VW];
                unpack(raw[p], e);
#pragma unroll
                for (int j = 0; j < VW; ++j) {
                    const int64_t v = first[p] + j;
                    if (e[j] >= reach && v >= 0 && v < V) {
                        const int at = atomicAdd(&element_count, 1);
                        if (at < kElementList) elements[at] = pack_key(e[j], static_cast<uint32_t>(v));
                    }
                }
            }
        }
    }
    __syncthreads();
    const int m = element_count;
    auto put = [&](int place, unsigned long long key) {
        if (a.top_id) a.top_id[r * a.top + place] = static_cast<int>(key_index(key));
        if (a.top_logprob) {
            const float x = key_value(key);
            a.top_logprob[r * a.top + place] = x > -INFINITY ? ((x - M) * a.c - log_l) * kLn2 : -INFINITY;
        }
    };
    if (n <= kChunkList && m <= kElementList && m >= a.top) {       // (fewer reach it only where logits are NaN)
        // (the order in which they came into the list does not matter: the keys are all different)
        for (int i = tid; i < m; i += kFinishThreads) {
            const unsigned long long key = elements[i];
            int place = 0;
            for (int t = 0; t < m; ++t) place += elements[t] > key;
            if (place < a.top) put(place, key);
        }
    } else if (warp == 0) {
        const unsigned long long key = best_in_turn<T, CUT>(row, chunk_max, chunks, head, V, a.top);
        if (lane < a.top) put(lane, key);
    }
}

// Units of a row: whole vectors from the one that holds its first element, wherever in it that is.
int64_t units_of(int64_t V, size_t es, bool cut) {
    const int64_t VW = 16 / static_cast<int64_t>(es), P = kUnitBytes / static_cast<int64_t>(es);
    return (V + (cut ? VW - 1 : 0) + P - 1) / P;
}

template <typename T, bool CUT>
cudaError_t launch(const void* logits, LogprobArgs a, cudaStream_t s) {
    const T* x = static_cast<const T*>(logits);
    const int64_t total = a.rows * a.units, most = static_cast<int64_t>(kBlocksPerSm) * kWaves * sm_count();
    int64_t blocks = (total + kWarps - 1) / kWarps;
    if (blocks > most) blocks = most;
    a.step_rows = static_cast<uint32_t>(blocks * kWarps / a.units);
    a.step_units = static_cast<uint32_t>(blocks * kWarps % a.units);
    const cudaError_t e = launch_pdl(logprob_sums_kernel<T, CUT>, dim3(static_cast<unsigned>(blocks)), dim3(kThreads), 0, s, 0, x, a);
    if (e != cudaSuccess) return e;
    return launch_pdl(logprob_finish_kernel<T, CUT>, dim3(static_cast<unsigned>(a.rows)), dim3(kFinishThreads), 0, s, 0, x, a);
}

}  // namespace
}  // namespace pldp

using namespace pldp;

extern "C" {

PLDP_API size_t pldp_token_logprobs_workspace_size(int64_t rows, int V) {
    if (rows < 0 || V < 1) return 0;
    const size_t units = static_cast<size_t>(rows) * units_of(V, 4, true);     // fp32 has the most
    return (units * (sizeof(float4) + sizeof(float2)) + 255) / 256 * 256;
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
    if (rows >= int64_t(1) << 31 || V > INT32_MAX - 4096)
        return fail(PLDP_ERR_UNSUPPORTED, "%s: 2^31 rows, or 2^31 - 4096 logits a row, or more", fn);
    if ((tokens == nullptr) != (logprob == nullptr))
        return fail(PLDP_ERR_INVALID_ARG, "%s: tokens and logprob go together", fn);
    if (rows == 0) return PLDP_OK;
    if (!logits || !workspace) return fail(PLDP_ERR_INVALID_ARG, "%s: null pointer", fn);
    const size_t need = pldp_token_logprobs_workspace_size(rows, V);
    if (workspace_bytes < need)
        return fail(PLDP_ERR_INVALID_ARG, "%s: workspace needs %zu bytes, has %zu", fn, need, workspace_bytes);
    if (!aligned16(workspace)) return fail(PLDP_ERR_INVALID_ARG, "%s: workspace is not 16-byte aligned", fn);
    const size_t es = dtype == PLDP_F32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(logits) % es) return fail(PLDP_ERR_INVALID_ARG, "%s: logits are not aligned to their elements", fn);
    LogprobArgs a = {};
    a.tokens = tokens, a.logprob = logprob, a.entropy = entropy;
    a.top_id = top_id, a.top_logprob = top_logprob, a.top = top_id || top_logprob ? top : 0;
    a.rows = rows, a.V = static_cast<uint32_t>(V);
    a.lead = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(logits) % 16 / es);
    const bool cut = a.lead != 0 || static_cast<size_t>(V) * es % 16 != 0;
    a.units = static_cast<uint32_t>(units_of(V, es, cut));
    a.maxima = static_cast<float4*>(workspace);
    a.sums = reinterpret_cast<float2*>(a.maxima + rows * a.units);
    a.c = fminf(1.4426950408889634f / temperature, FLT_MAX);       // (infinity would make the maximum's own exponent 0 * inf)
    auto s = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (dtype == PLDP_F32) e = cut ? launch<float, true>(logits, a, s) : launch<float, false>(logits, a, s);
    else e = cut ? launch<__nv_bfloat16, true>(logits, a, s) : launch<__nv_bfloat16, false>(logits, a, s);
    return launched(fn, e);
}

}  // extern "C"
