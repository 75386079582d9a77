// Attention of a step's tokens over the paged cache: the kernel of pldp_attend_cache (attend.cu).
#pragma once

#include <cuda_fp8.h>
#include <cuda_fp16.h>
#include <math.h>

#include "pldp_cache.cuh"
#include "pldp_tcgen05.cuh"

namespace pldp {

constexpr int kTile = 128;                // keys a tile
constexpr int kMaxCtas = 192;             // parts of the list at most
#ifdef PLDP_TEST_STUCK_SCORES
constexpr uint32_t kPolls = 1u << 12;     // test build: a short bound on every wait
#else
constexpr uint32_t kPolls = kMbarPolls;
#endif

struct AttendArgs {
    CacheView c;
    const __nv_bfloat16* q;
    __nv_bfloat16* out;
    int64_t q_seq, q_tok, q_head, o_seq, o_tok, o_head;
    const int32_t *seq_len, *draft_len;
    float *lse, *parts;
    uint32_t *status, *tickets;
    int B, n, q_heads, group, row_tiles;
    int box;                               // positions of a page that one copy takes
    int pitch;                             // e4m3: bytes from one position's codes to the next in a stage
    int head_first;                        // the maps' second dimension is the head, not the position
    float scale2;                          // scale * log2(e)
};

struct Maps {
    CUtensorMap k, v;
};
// cuTensorMapEncodeTiled, or null where the driver has none.
using TensorMapEncoder = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                      const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                      CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
TensorMapEncoder tensor_map_encoder();
bool pool_map(CUtensorMap* map, void* base, const CacheView& c, bool e4m3, int box, int pitch, bool* head_first);

// One launch for nt columns; one translation unit a cache type.
cudaError_t launch_attend_bf16(const AttendArgs& a, const Maps& m, int nt, int ctas, cudaStream_t s);
cudaError_t launch_attend_e4m3(const AttendArgs& a, const Maps& m, int nt, int ctas, cudaStream_t s);

namespace {

// ---------------------------------------------------------------------------
// One pass over the keys, 128 at a time, all query rows of one key/value head at once (the
// tokens' G = q_heads / heads heads each: up to NT rows, padded).  Both products have the
// keys or the head's elements as the tensor core's 128 rows and the query rows as its columns,
// so a few query rows waste nothing:
//   S^T [128 keys, NT]  = K [128, D] Q^T [D, NT]
//   O^T [D, NT]        += V^T [D, 128] P^T [128, NT]
// S^T and O^T stay in tensor memory.  A thread owns one key (a lane of S^T) and half of the
// columns: it applies the key's scale and the masks, takes weights w = 2^(x - m), adds them to
// its own sums and writes them to shared memory as the next product's operand.  The running
// maximum m of a column only moves when a score passes it by more than 2^8: then the column's
// sums and its accumulators in tensor memory are scaled; otherwise no thread needs another's
// scores, and the 128 of them agree on that with one barrier.  bf16 weights have fp32's range: there the
// maximum may be passed by 2^64, and m starts as the first key's score, whose weight is then 1, so that the
// sums cannot vanish.
//
// Weights are rounded to 16 bits for the second product: in a bf16 cache as a sum of two bf16
// (2^-17 of the weight; one alone would add as much error as the result's own rounding), the second
// ones as NT more columns, which cost the product little beside reading V^T; in an
// e4m3 cache as f16 (2^-11, where the cache rounds each element by up to 2^-4; the error against 64 bits is 0.00167 for
// 0.00166 with weights in 32 bits), in which the codes, at most 448, are exact as well.  The scales of an
// e4m3 cache never touch its codes: k's multiplies the key's scores, v's goes into the exponent
// (w = vs 2^(x - m), m the maximum of x + log2 vs) and is divided out of the sums.
//
// The keys of all sequences and heads form one list of tiles, cut into equal parts, one a CTA
// (one a SM), so that ragged lengths and few long sequences keep every SM reading to the end.
// What a CTA holds of a unit (sequence, head, rows) that others share goes to the workspace, and
// the last of them, by the ticket of the CTA in which the unit begins, joins the parts in order.
//
// Warps: 8 for the softmax (a key a thread, half of the columns each four), one that issues the matrix
// instructions, two that copy (tensor copies, one a page's positions: keys, values), one that looks the
// keys' pages and scales up, and for e4m3 four that turn codes into f16.  They meet at mbarriers; a wait for
// one that is over takes some 120 cycles, so waits are asked together or ahead, and code is kept short:
// all of these loops share one instruction cache.
//
// Bound by memory where a tile is large: 2 x 131072 keys of 8 heads of 128, bf16, one token: 141..146 us (0.95..0.98
// of the measured copy rate); 64 x 16384, 17 tokens, 5 query heads a head: 502..517 us (0.93..0.95).  Short
// tiles are bound by the warps' own work, 0.95 us a tile of 128 keys of 64 elements in e4m3 with up to 16
// columns (the conversion), 1.3 us with 48 (the softmax): 32 x 8192 keys, 8 heads, 11 tokens: 106..109 us (2.0 TB/s).
// Of a prompt every tile of rows walks all of its sequence's keys, those that it sees none of too: 4 x 4095 tokens, 32 query
// heads, bf16: 2.2 ms (209 of 1922 TFLOP/s for what the mask leaves).
// ---------------------------------------------------------------------------
constexpr int kSoftmaxThreads = 256, kConvertThreads = 128;
constexpr int kMaxShared = 232448;        // bytes a CTA, static and dynamic

template <int NT, int DP, bool E4M3>
struct Shape {
    // warps: 8 softmax, (e4m3: 4 that convert,) one of matrix instructions, two of copies, one that looks up keys
    static constexpr int kMmaWarp = E4M3 ? 12 : 8, kCopyWarp = kMmaWarp + 1, kKeyWarp = kMmaWarp + 3;
    static constexpr int kThreads = (E4M3 ? 16 : 12) * 32;
    static constexpr int kPanels = DP / 64;                    // of 64 elements (128 bytes) each
    static constexpr int kSlot = kPanels * kTile * 128;        // one tile of keys or values
    static constexpr int kQ = kPanels * NT * 128;
    static constexpr int kRow = NT % 64 == 0 ? 128 : NT % 32 == 0 ? 64 : 32;   // bytes of a row of a panel of P^T
    static constexpr int kP = NT * 2 * kTile;                  // weights of a tile, 16 bits each
    static constexpr int kWeights = E4M3 ? NT : 2 * NT;        // columns of the second product
    static constexpr int kStage = E4M3 ? kTile * (DP < 128 ? 128 : DP) : 0;    // one tile's codes
    static constexpr int kPs = kP * (E4M3 ? 1 : 2);            // with the low parts
    static constexpr int kWeightTiles = NT <= 64 && DP <= 128 ? 2 : 1;     // tiles of weights held
    static constexpr int kRest = kQ + kPs * kWeightTiles;
    static constexpr int kColumns = NT * 56 + 2688 + (E4M3 ? 4096 : 0);    // static: Columns
    static constexpr int kRoom = kMaxShared - 1024 - kColumns - kRest;
    // e4m3: what three stages leave
    static constexpr int kMost = E4M3 ? (kRoom - 3 * kStage) / kSlot : kRoom / kSlot;
    static constexpr int kSlots = kMost > (E4M3 ? 6 : 8) ? (E4M3 ? 6 : 8) : kMost < 2 ? 2 : kMost;
    static constexpr int kStages = E4M3 ? ((kRoom - kSlots * kSlot) / kStage < 7 ? (kRoom - kSlots * kSlot) / kStage : 7) : 0;
    // Keys and values take the slots in turn, so in an odd ring a slot is both's.  Two warps that copy on their own could
    // then ask a slot's barrier for a phase while it is two behind, and the parity of that answers at once: of three
    // slots, the values of tile 3 would overwrite those of tile 0.  There one warp copies both, in order (as fast: heads
    // of 128, 25 tokens a step 235 us, and of 256, one token 248 us, 32 sequences of 8192 tokens).  The rings of codes
    // are read in order by one group of warps and may be odd.
    static constexpr bool kOneCopyWarp = !E4M3 && kSlots % 2 == 1;
    static constexpr int kBlocks = DP == 256 ? 2 : 1;          // of 128 rows of O^T
    static constexpr int kCols = 2 * NT + kBlocks * kWeights;
    static constexpr int kTmem = kCols <= 64 ? 64 : kCols <= 128 ? 128 : kCols <= 256 ? 256 : 512;
    static constexpr int kUsed = kSlots * kSlot + kRest + kStages * kStage;
    // V^T's 128 rows read two panels: with one (64 elements) the second lies behind the slot
    static constexpr int kBytes = (kPanels > 1 || kUsed > (kSlots + 1) * kSlot ? kUsed : (kSlots + 1) * kSlot) + 1024;
    static_assert(kCols <= 512, "tensor memory");
    static_assert(kSlots >= 2 && (!E4M3 || kStages >= 2) && kBytes <= kMaxShared - kColumns, "shared memory");
};

// What a column (query row) and the CTA's roles share.
template <int NT, bool E4M3>
struct Columns {
    int64_t q_at[NT], o_at[NT];     // element offsets, -1: no such row
    float neg_m[NT], factor[NT], sum[NT], inverse[NT];
    float part[4][NT];
    // of the keys of four tiles: 0 or, where there is none, -inf; e4m3: the scales of the key and of the value
    alignas(16) float key[4][kTile], key_scale[E4M3 ? 4 : 1][E4M3 ? kTile : 4], value_scale[E4M3 ? 4 : 1][E4M3 ? kTile : 4];
    int limit[NT];                  // last position that the row sees
    int seen[NT];                   // whether m has been set
    uint64_t full[8], empty[8], stage_full[8], stage_empty[8], s_full[2], p_full[2], pv_done[2], q_full, key_empty[4], drained;
#ifdef PLDP_TEST_STUCK_SCORES
    uint64_t never;                 // test build: a barrier that nothing arrives on
#endif
    uint32_t tmem, amax;
    int dead, last;
    int ended[2];                   // entries of the ring that the copy warps have come to
    int b, unit, tile;              // where this CTA's part of the list starts
    long long at, count;            // its first tile in the list, tiles in it
    long long each, extra;          // tiles a CTA, and CTAs that have one more
    long long warp_sum[16];
};

// Whether a phase is over; the answer takes some 120 cycles, which other questions and work can share.
__device__ __forceinline__ bool over(uint64_t* bar, uint32_t parity) { return mbar_wait(bar, parity & 1u, 1); }
// Waits, with a limit; after one has run out no wait of this CTA blocks for long any more, and its results
// are marked as none.  From then on a role may be ahead of the others, so no copy starts any more (its place may be in
// use), the warp of keys still waits for the softmax, which meets it at barriers without a limit, and what is in flight is
// waited for before the CTA ends.
__device__ __forceinline__ void wait_more(bool done, uint64_t* bar, uint32_t parity, int* dead) {
    // (one statement: the loop as C++ came to a hundred instructions at each of its places)
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b32 n, x;\n\t"
        "mov.u32 n, 0;\n\t"
        "setp.ne.u32 p, %0, 0;\n\t"
        "@p bra DONE;\n\t"
        "AGAIN:\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "@p bra DONE;\n\t"
        "add.u32 n, n, 1;\n\t"
        "ld.volatile.shared.u32 x, [%3];\n\t"
        "setp.ne.u32 p, x, 0;\n\t"
        "@p bra DONE;\n\t"
        "setp.lt.u32 p, n, %4;\n\t"
        "@p bra AGAIN;\n\t"
        "st.volatile.shared.u32 [%3], 1;\n\t"
        "DONE:\n\t}" ::"r"(static_cast<uint32_t>(done)),
        "r"(smem_u32(bar)), "r"(parity & 1u), "r"(smem_u32(dead)), "n"(kPolls)
        : "memory");
}
__device__ __forceinline__ void wait_for(uint64_t* bar, uint32_t parity, int* dead) {
    wait_more(over(bar, parity), bar, parity, dead);
}

// The CTA's part of the list, unit by unit.
struct Walk {
    int b, unit, t0;
    long long at, left;
    // the unit's
    int T, t1, first, tokens, keys;

    __device__ __forceinline__ bool next(const AttendArgs& a, uint32_t* status) {
        if (left <= 0) return false;
        const StepTokens tk = step_tokens(a.seq_len, a.draft_len, b, a.n, a.c.capacity, *status);
        first = tk.first, tokens = tk.count, keys = tk.first + tk.count;
        T = keys > 0 ? (keys + kTile - 1) / kTile : 1;
        t1 = left < T - t0 ? t0 + static_cast<int>(left) : T;
        return true;
    }
    __device__ __forceinline__ void step(const AttendArgs& a) {
        at += t1 - t0;
        left -= t1 - t0;
        t0 = 0;
        if (++unit == a.c.heads * a.row_tiles) unit = 0, ++b;
    }
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&p);
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
    const __half2 p = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&p);
}
// Four e4m3 codes as four f16.
__device__ __forceinline__ uint2 four_codes(uint32_t codes) {
    uint2 h;
    asm("{\n\t.reg .b16 lo, hi;\n\t"
        "mov.b32 {lo, hi}, %2;\n\t"
        "cvt.rn.f16x2.e4m3x2 %0, lo;\n\t"
        "cvt.rn.f16x2.e4m3x2 %1, hi;\n\t}"
        : "=r"(h.x), "=r"(h.y)
        : "r"(codes));
    return h;
}
__device__ __forceinline__ float warp_max(float v) {
    const uint32_t k = __reduce_max_sync(0xFFFFFFFFu, ordered_key(v));
    return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}

// A load that stays where it is written, ahead of its use.
__device__ __forceinline__ int load_now(const int32_t* p) {
    int v;
    asm volatile("ld.global.nc.b32 %0, [%1];" : "=r"(v) : "l"(p));
    return v;
}
__device__ __forceinline__ float load_now(const float* p) {
    float v;
    asm volatile("ld.global.nc.f32 %0, [%1];" : "=f"(v) : "l"(p));
    return v;
}
__device__ __forceinline__ float reciprocal(float x) {
    float y;
    asm("rcp.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// N words (one, or four on a boundary of 16 bytes) from global to shared memory, later; and until all copies but
// those of the last N groups, this one with them, are done.
template <int N>
__device__ __forceinline__ void copy_words(float* to, const float* from) {
    if constexpr (N == 4) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(to)), "l"(from) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(to)), "l"(from) : "memory");
}
template <int N>
__device__ __forceinline__ void copies_but() {
    asm volatile("cp.async.commit_group;" ::: "memory");
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// Sums v[0..C) over the warp's lanes, C a multiple of 8: each lane ends with the sums of the
// columns from the returned one on, in v[0..]; `lanes` neighbouring lanes hold the same.
template <int C>
struct ColumnSums {
    static constexpr int kHalvings = C % 32 == 0 ? 5 : C % 16 == 0 ? 4 : 3;
    static constexpr int kOwn = C >> kHalvings, kLanes = 1 << (5 - kHalvings);
};
template <int C>
__device__ __forceinline__ int warp_columns(float (&v)[C], int lane) {
    int first = 0;
#pragma unroll
    for (int k = 0; k < 5; ++k) {
        const int o = 16 >> k;
        if (k < ColumnSums<C>::kHalvings) {
            const int n = C >> (k + 1);
            const bool up = lane & o;
#pragma unroll
            for (int i = 0; i < n; ++i) {
                const float keep = up ? v[i + n] : v[i], send = up ? v[i] : v[i + n];
                v[i] = keep + __shfl_xor_sync(0xFFFFFFFFu, send, o);
            }
            if (up) first += n;
        } else {
#pragma unroll
            for (int i = 0; i < ColumnSums<C>::kOwn; ++i) v[i] += __shfl_xor_sync(0xFFFFFFFFu, v[i], o);
        }
    }
    return first;
}

template <int NT, int DP, bool E4M3>
__global__ void __launch_bounds__(Shape<NT, DP, E4M3>::kThreads, 1)
attend_kernel(const AttendArgs a, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map) {
    using S = Shape<NT, DP, E4M3>;
    constexpr int kThreads = S::kThreads;
    static_assert(sizeof(Columns<NT, E4M3>) <= S::kColumns, "shared memory");
    extern __shared__ uint8_t raw[];
    __shared__ __align__(16) Columns<NT, E4M3> col;
    uint8_t* ring = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
    uint8_t* const q_smem = ring + S::kSlots * S::kSlot;
    uint8_t* const p_smem = q_smem + S::kQ;                     // (high part, and behind it the low part)
    [[maybe_unused]] uint8_t* const stages = q_smem + S::kRest;
    const CacheView& c = a.c;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, D = c.head_dim;
    const int units = c.heads * a.row_tiles;

    if (warp == S::kMmaWarp) tmem_alloc(&col.tmem, S::kTmem);
    if (threadIdx.x == 0) {
        for (int i = 0; i < 8; ++i) {
            mbar_init(&col.full[i], E4M3 ? kConvertThreads / 32 : 1);
            mbar_init(&col.empty[i], 1);
            mbar_init(&col.stage_full[i], 1);
            mbar_init(&col.stage_empty[i], kConvertThreads / 32);
        }
        mbar_init(&col.s_full[0], 1);
        mbar_init(&col.s_full[1], 1);
        for (int i = 0; i < 4; ++i) {
            mbar_init(&col.key_empty[i], kSoftmaxThreads / 32);
        }
        mbar_init(&col.p_full[0], kSoftmaxThreads / 32);
        mbar_init(&col.p_full[1], kSoftmaxThreads / 32);
        mbar_init(&col.pv_done[0], 1);
        mbar_init(&col.pv_done[1], 1);
        mbar_init(&col.q_full, kSoftmaxThreads / 32);
        mbar_init(&col.drained, 1);
#ifdef PLDP_TEST_STUCK_SCORES
        mbar_init(&col.never, 1);
#endif
        fence_mbar_init();
        col.dead = 0;
    }
    pdl_enter();

    // the list: every thread counts the tiles of a strip of sequences
    {
        const int strip = (a.B + kThreads - 1) / kThreads;
        const int lo = min(a.B, static_cast<int>(threadIdx.x) * strip), hi = min(a.B, lo + strip);
        long long mine = 0;
        auto tiles_of = [&](int b) {
            uint32_t st;
            const StepTokens tk = step_tokens(a.seq_len, a.draft_len, b, a.n, c.capacity, st);
            const int keys = tk.first + tk.count;
            return keys > 0 ? (keys + kTile - 1) / kTile : 1;
        };
#pragma unroll 1
        for (int b = lo; b < hi; ++b) mine += tiles_of(b);
        long long upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long t = __shfl_up_sync(0xFFFFFFFFu, upto, o);
            if (lane >= o) upto += t;
        }
        if (lane == 31) col.warp_sum[warp] = upto;
        __syncthreads();
        long long total = 0;
#pragma unroll 1
        for (int w = 0; w < kThreads / 32; ++w) {
            if (w == warp) upto += total;
            total += col.warp_sum[w];
        }
        total *= units;
        const int ctas = static_cast<int>(total < gridDim.x ? total : gridDim.x);
        // the first `extra` CTAs take one tile more than the others
        const long long each = total >> 32 ? total / ctas : static_cast<uint32_t>(total) / static_cast<uint32_t>(ctas);
        const long long extra = total - each * ctas;
        const long long g0 = each * blockIdx.x + min(static_cast<long long>(blockIdx.x), extra);
        const long long g1 = g0 + each + (blockIdx.x < extra ? 1 : 0);
        long long before = (upto - mine) * units;
        if (blockIdx.x < ctas && before <= g0 && g0 < before + mine * units) {     // one thread's
            int b = lo;
#pragma unroll 1
            for (;; ++b) {
                const long long t = static_cast<long long>(tiles_of(b)) * units;
                if (g0 < before + t) break;
                before += t;
            }
            const int T = tiles_of(b);
            col.b = b;
            const long long in = g0 - before;
            const int unit = in >> 32 ? static_cast<int>(in / T) : static_cast<int>(static_cast<uint32_t>(in) / static_cast<uint32_t>(T));
            col.unit = unit;
            col.tile = static_cast<int>(in - static_cast<long long>(unit) * T);
            col.at = g0;
            col.count = g1 - g0;
        }
        if (threadIdx.x == 0) {
            col.each = each;
            col.extra = extra;
            if (blockIdx.x >= ctas) col.count = 0;
        }
    }
    tmem_before_sync();
    __syncthreads();
    tmem_after_sync();
    const uint32_t tmem = col.tmem;
    Walk w = {col.b, col.unit, col.tile, col.at, col.count, 0, 0, 0, 0, 0};
    uint32_t st;

    if (warp >= S::kMmaWarp) {
        // e4m3: 16 warps start with 128 registers a thread; the softmax takes what the others leave:
        // 256 * 176 + 128 * 88 + 128 * 64 = 64512 of 65536
        if constexpr (E4M3) fewer_registers<64>();
        if (warp == S::kCopyWarp || (!S::kOneCopyWarp && warp == S::kCopyWarp + 1)) {
            // ---- copies: one warp the tiles of keys, one those of values; a box (positions of one page) a lane ----
            constexpr int kDepth = E4M3 ? S::kStages : S::kSlots;
            uint64_t* const arrived = E4M3 ? col.stage_full : col.full;
            uint64_t* const left = E4M3 ? col.stage_empty : col.empty;
            const int boxes = kTile / a.box;                               // of a tile, 1..128
            int kv = warp - S::kCopyWarp;
            int e = kv;                                                    // entries of the ring: keys and values in turn
            constexpr int kStep = S::kOneCopyWarp ? 1 : 2;
            bool on = true;                                                // no wait has run out
#pragma unroll 1
            while (on && w.next(a, &st)) {
                if (kv == 0 && w.t0 == 0 && w.unit == 0 && lane == 0 && st && a.status) atomicOr(a.status + w.b, st);
                const int head = w.unit / a.row_tiles;
                const int32_t* table = c.pages + w.b * c.pages_stride;
                auto look = [&](int tile, int box) {
                    const int pos = tile * kTile + box * a.box;
                    return tile < w.t1 && box < boxes && pos < w.keys ? load_now(table + page_of(pos, c.div_mul, c.div_shift)) : 0;
                };
                // pages are looked up two tiles ahead, into two registers in turn: a copy from one to the other would
                // wait for the load
                auto turn = [&](int tile, int& page) {
                    // boxes that hold a position below the sequence's end
                    const int full = max(0, min(boxes, (w.keys - tile * kTile + a.box - 1) / a.box));
                    const CUtensorMap* map = kv ? &v_map : &k_map;
                    const int at = e % kDepth;
                    if (e >= kDepth) wait_for(&left[at], e / kDepth - 1, &col.dead);
                    on = !__any_sync(0xFFFFFFFFu, *static_cast<volatile int*>(&col.dead));
                    if (!on) return;
                    if (lane == 0) mbar_arrive_expect_tx(&arrived[at], full * a.box * (E4M3 ? a.pitch : S::kPanels * 128));
                    __syncwarp();
                    uint8_t* dst = E4M3 ? stages + at * S::kStage : ring + at * S::kSlot;
#pragma unroll 1
                    for (int box = lane; box < full; box += 32) {
                        const int pos = tile * kTile + box * a.box;
                        const int slot = pos - static_cast<int>(page_of(pos, c.div_mul, c.div_shift)) * c.page_size;
                        int pg = box < 32 ? page : look(tile, box);        // (pages that 4 does not divide have more)
                        if (static_cast<unsigned>(pg) >= static_cast<unsigned>(c.n_pages)) {
                            pg = c.n_pages;                                // outside the tensor: zeros
                            if (kv == 0 && a.status) atomicOr(a.status + w.b, PLDP_ST_PAGE);
                        }
                        const int c1 = a.head_first ? head : slot, c2 = a.head_first ? slot : head;
                        if constexpr (E4M3) {
                            tma_box(dst + box * a.box * a.pitch, map, 0, c1, c2, pg, &arrived[at]);
                        } else {
#pragma unroll 1
                            for (int p = 0; p < S::kPanels; ++p)
                                tma_box(dst + p * (kTile * 128) + box * a.box * 128, map, p * 64, c1, c2, pg, &arrived[at]);
                        }
                    }
                    __syncwarp();
                    if (!S::kOneCopyWarp || kv) page = look(tile + 2, lane);
                    e += kStep;
                };
                auto both = [&](int tile, int& page) {
                    turn(tile, page);
                    if constexpr (S::kOneCopyWarp) {
                        if (!on) return;
                        kv = 1;
                        turn(tile, page);
                        kv = 0;
                    }
                };
                int page = look(w.t0, lane), page_b = look(w.t0 + 1, lane);
#pragma unroll 1
                for (int tile = w.t0; on && tile < w.t1; tile += 2) {
                    both(tile, page);
                    if (on && tile + 1 < w.t1) both(tile + 1, page_b);
                }
                w.step(a);
            }
            // The last copy into each place arrives before this CTA ends, whether or not its reader has waited for it: the
            // last entry of either warp there, by the parity of its turn.
            if (lane == 0) col.ended[warp - S::kCopyWarp] = e;
            if constexpr (S::kOneCopyWarp) __syncwarp();
            else bar_sync(13, 64);
            if (warp == S::kCopyWarp && lane < kDepth) {
                const int ended[2] = {col.ended[0], S::kOneCopyWarp ? col.ended[0] : col.ended[1]};   // (each warp's next one)
                const int top = max(ended[0], ended[1]) - 1;
                int x = top - (top - lane + kDepth) % kDepth;
                while (x >= 0 && x >= ended[x & 1]) x -= kDepth;
                if (x >= 0) mbar_wait(&arrived[lane], (x / kDepth) & 1, kMbarPolls);
            }
        } else if (warp == S::kKeyWarp) {
            // ---- the keys of each tile, four a lane: whether there is one, and e4m3's scales ----
            // Four neighbours lie in one page where 4 divides the page size; their scales are then 16 bytes (if the
            // tensors start on such a boundary).  This warp's own instructions bound short tiles: with a page, two
            // addresses and two loads for every key a turn took 1900 cycles.
            const uintptr_t scales = reinterpret_cast<uintptr_t>(c.k_scale) | reinterpret_cast<uintptr_t>(c.v_scale);
            const bool four = c.page_size % 4 == 0 && (!E4M3 || scales % 16 == 0);
            int tile_no = 0;
#pragma unroll 1
            while (w.next(a, &st)) {
                const int kv = w.unit / a.row_tiles;
                const int32_t* table = c.pages + w.b * c.pages_stride;
                auto look = [&](int tile, int pos) {
                    return tile < w.t1 && pos < w.keys ? load_now(table + page_of(pos, c.div_mul, c.div_shift)) : -1;
                };
                auto exists = [&](int page) { return static_cast<unsigned>(page) < static_cast<unsigned>(c.n_pages); };
                auto scales_at = [&](int page, int pos) {
                    const int slot = pos - static_cast<int>(page_of(pos, c.div_mul, c.div_shift)) * c.page_size;
                    return (static_cast<int64_t>(page) * c.heads + kv) * c.page_size + slot;
                };
                // e4m3: a tile's scales are asked for (straight into shared memory) two turns before they are handed on,
                // and the pages two turns before that.
                constexpr int kLate = E4M3 ? 2 : 0;
                auto turn = [&](int tile, int& page) {
                    const int at = tile_no & 3;
                    if (tile < w.t1) {
                        if (tile_no >= 4 && !over(&col.key_empty[at], (tile_no >> 2) - 1)) {
                            wait_more(false, &col.key_empty[at], (tile_no >> 2) - 1, &col.dead);
                            // ahead of the softmax this warp would arrive on a barrier before they have left it
                            if (*static_cast<volatile int*>(&col.dead)) mbar_wait(&col.key_empty[at], ((tile_no >> 2) - 1) & 1, kMbarPolls);
                        }
                        const int pos = tile * kTile + 4 * lane;
                        if (four) {
                            const int there = exists(page) ? w.keys - pos : 0;
                            if (E4M3 && there > 0) {
                                const int64_t from = scales_at(page, pos);
                                copy_words<4>(&col.key_scale[at][4 * lane], c.k_scale + from);
                                copy_words<4>(&col.value_scale[at][4 * lane], c.v_scale + from);
                            }
                            *reinterpret_cast<float4*>(&col.key[at][4 * lane]) =
                                make_float4(there > 0 ? 0.f : -INFINITY, there > 1 ? 0.f : -INFINITY, there > 2 ? 0.f : -INFINITY,
                                            there > 3 ? 0.f : -INFINITY);
                            page = look(tile + 2, pos + 2 * kTile);
                        } else {
#pragma unroll 1
                            for (int i = 0; i < 4; ++i) {
                                const int pg = look(tile, pos + i);
                                if (E4M3 && exists(pg)) {
                                    const int64_t from = scales_at(pg, pos + i);
                                    copy_words<1>(&col.key_scale[at][4 * lane + i], c.k_scale + from);
                                    copy_words<1>(&col.value_scale[at][4 * lane + i], c.v_scale + from);
                                }
                                col.key[at][4 * lane + i] = exists(pg) ? 0.f : -INFINITY;
                            }
                        }
                    }
                    if constexpr (E4M3) copies_but<kLate>();
                    if (tile - kLate >= w.t0) {
                        const int on = (tile_no - kLate) & 3;
                        bar_arrive(5 + on, 160);         // for the one half of the columns, and for the other
                        bar_arrive(9 + on, 160);
                    }
                    ++tile_no;
                };
                // two registers in turn: a copy from one to the other would wait for the load
                int page = look(w.t0, w.t0 * kTile + 4 * lane), page_b = look(w.t0 + 1, (w.t0 + 1) * kTile + 4 * lane);
#pragma unroll 1
                for (int tile = w.t0; tile < w.t1 + kLate; tile += 2) {
                    turn(tile, page);
                    if (tile + 1 < w.t1 + kLate) turn(tile + 1, page_b);
                }
                tile_no -= kLate;
                w.step(a);
            }
        } else if (warp == S::kMmaWarp) {
            // ---- matrix instructions: one lane issues them, three ask the barriers ----
            // the operands' descriptors in two words: addresses move the low one, in units of 16 bytes
            const uint64_t q_op = smem_operand(smem_u32(q_smem), 16, 1024, swizzle_mode(128));
            const uint64_t p_op = smem_operand(smem_u32(p_smem), kTile * S::kRow, 8 * S::kRow, swizzle_mode(S::kRow));
            const uint64_t k_op = smem_operand(smem_u32(ring), 16, 1024, swizzle_mode(128));
            const uint64_t v_op = smem_operand(smem_u32(ring), kTile * 128, 1024, swizzle_mode(128));
            const uint32_t q_lo = static_cast<uint32_t>(q_op), q_hi = q_op >> 32, p_lo = static_cast<uint32_t>(p_op), p_hi = p_op >> 32;
            const uint32_t k_lo = static_cast<uint32_t>(k_op), k_hi = k_op >> 32, v_lo = static_cast<uint32_t>(v_op), v_hi = v_op >> 32;
            constexpr uint32_t kScores = mma_form(128, NT, !E4M3, false, false), kValues = mma_form(128, S::kWeights, !E4M3, true, true);
            // Each lane's own barrier (or none): until all are over.  One wait for three costs what one does.
            auto wait_all = [&](uint64_t* bar, uint32_t parity) {
                bool done = bar == nullptr || over(bar, parity);
                uint32_t polls = 0;
#pragma unroll 1
                while (!__all_sync(0xFFFFFFFFu, done)) {
                    if (++polls >= kPolls || *static_cast<volatile int*>(&col.dead)) {
                        *static_cast<volatile int*>(&col.dead) = 1;
                        break;
                    }
                    if (!done) done = over(bar, parity);
                }
                __syncwarp();
            };
            const uint32_t lead = elect_lane(), base = __shfl_sync(0xFFFFFFFFu, tmem, 0);
            // where the next tile's keys, values, weights and scores lie, and the parities of their arrivals
            uint32_t k_slot = 0, k_parity = 0, v_slot = 1, v_parity = 0, place = 0, p_parity = 0, scores_at = 0, segment = 0;
            auto second = [](uint32_t& slot, uint32_t& parity) {       // entries go two by two: keys and values in turn
                slot += 2;
                if (slot >= S::kSlots) slot -= S::kSlots, parity ^= 1u;
            };
#pragma unroll 1
            while (w.next(a, &st)) {
                const int count = __shfl_sync(0xFFFFFFFFu, w.t1 - w.t0, 0);
                // (In a short ring the keys of tile i + 2, or the values before them, come only when the
                // values of tile i have gone: their wait cannot come first.)
                constexpr bool kTogether = S::kSlots >= 6;
                // Turn i: the second product of the unit's tile i, then the scores of tile i + 2, whose place in
                // tensor memory tile i's weights have left; turns -2 and -1 have scores only.  (In this order the
                // scores' arrival also says that the second product two tiles before is done.)
#pragma unroll 1
                for (int i = -2; i < count; ++i) {
                    const bool scores = i + 2 < count, values = i >= 0;
                    uint64_t* bar = nullptr;
                    uint32_t parity = 0;
                    if (kTogether && lane == 0 && scores) bar = &col.full[k_slot], parity = k_parity;
                    if (lane == 1 && values) bar = &col.full[v_slot], parity = v_parity;
                    if (lane == 2 && values) bar = &col.p_full[place], parity = p_parity;
                    if (lane == 2 && i == -2) bar = &col.q_full, parity = segment;
                    wait_all(bar, parity);
                    tmem_after_sync();
                    if (values) {
                        const uint32_t op = __shfl_sync(0xFFFFFFFFu, v_lo + v_slot * (S::kSlot / 16), 0);
                        const uint32_t from = __shfl_sync(0xFFFFFFFFu, p_lo + place * (S::kPs / 16), 0), more = i > 0;
#pragma unroll
                        for (int m = 0; m < S::kBlocks; ++m)
#pragma unroll
                            for (int s = 0; s < kTile / 16; ++s)
                                mma_f16(base + 2 * NT + m * S::kWeights, op + m * 2 * (kTile * 8) + s * 128, v_hi, from + s * S::kRow, p_hi,
                                        kValues, s > 0 ? 1u : more, lead);
                        mma_commit(&col.pv_done[scores_at], lead);
                        mma_commit(&col.empty[v_slot], lead);
                        second(v_slot, v_parity);
                        if (S::kWeightTiles == 1 || (place ^= 1u) == 0) p_parity ^= 1u;
                    }
                    if (scores) {
                        if (!kTogether) {
                            wait_all(lane == 0 ? &col.full[k_slot] : nullptr, k_parity);
                            tmem_after_sync();
                        }
                        const uint32_t op = __shfl_sync(0xFFFFFFFFu, k_lo + k_slot * (S::kSlot / 16), 0);
                        const uint32_t to = __shfl_sync(0xFFFFFFFFu, tmem + scores_at * NT, 0);
#pragma unroll
                        for (int s = 0; s < DP / 16; ++s)
                            if (s == 0 || s * 16 < D)
                                mma_f16(to, op + (s >> 2) * (kTile * 8) + (s & 3) * 2, k_hi, q_lo + (s >> 2) * (NT * 8) + (s & 3) * 2, q_hi,
                                        kScores, s > 0, lead);
                        mma_commit(&col.s_full[scores_at], lead);
                        mma_commit(&col.empty[k_slot], lead);
                        second(k_slot, k_parity);
                    }
                    scores_at ^= 1u;                                  // (of tile i + 2, as of tile i)
                }
                ++segment;
                w.step(a);
            }
            // nothing reads shared memory or writes tensor memory any more when they are given back
            mma_commit(&col.drained, lead);
            mbar_wait(&col.drained, 0, kMbarPolls);
        }
    } else if (E4M3 && warp >= 8) {
        // ---- e4m3: the codes of a tile of keys or values to f16, 16 at a time ----
        if constexpr (E4M3) {
            fewer_registers<88>();
            const int t = threadIdx.x - kSoftmaxThreads;
            constexpr int kRowChunks = DP / 16, kRows = kConvertThreads / kRowChunks, kTurns = kTile / kRows;
            const int chunk = t % kRowChunks, row0 = t / kRowChunks;
            const bool in = chunk * 16 < D;
            // where this thread's pieces of a tile lie: kRows rows apart, a multiple of 8, so all with the same swizzle
            static_assert(kRows % 8 == 0 && kTurns % 4 == 0, "rows");
            const int first = row0 * a.pitch + chunk * 16, step = kRows * a.pitch;
            const int line = (chunk >> 2) * (kTile * 128) + row0 * 128;
            const int low = line + ((((chunk & 3) * 2) ^ (row0 & 7)) << 4), high = low ^ 16;
            int e = 0;
#pragma unroll 1
            while (w.next(a, &st)) {
#pragma unroll 1
                for (int tile = w.t0; tile < w.t1; ++tile) {
                    const int rows = min(kTile, w.keys - tile * kTile);          // the rest is zeros
#pragma unroll 1
                    for (int kv = 0; kv < 2; ++kv, ++e) {
                        const int slot = e % S::kSlots, stage = e % S::kStages;
                        const uint8_t* from = stages + stage * S::kStage + first;
                        uint8_t* const to = ring + slot * S::kSlot;
                        const bool codes = over(&col.stage_full[stage], e / S::kStages);
                        const bool room = e < S::kSlots || over(&col.empty[slot], e / S::kSlots - 1);
                        wait_more(codes, &col.stage_full[stage], e / S::kStages, &col.dead);
                        wait_more(room, &col.empty[slot], e / S::kSlots - 1, &col.dead);
                        if (in) {
                            constexpr int kAtOnce = kTurns < 8 ? kTurns : 8;
#pragma unroll 1
                            for (int turn = 0; turn < kTurns; turn += kAtOnce) {
                                uint4 x[kAtOnce];
#pragma unroll
                                for (int i = 0; i < kAtOnce; ++i, from += step) x[i] = *reinterpret_cast<const uint4*>(from);
#pragma unroll
                                for (int i = 0; i < kAtOnce; ++i) {
                                    const uint2 h0 = four_codes(x[i].x), h1 = four_codes(x[i].y), h2 = four_codes(x[i].z), h3 = four_codes(x[i].w);
                                    const int at = (turn + i) * (kRows * 128);
                                    *reinterpret_cast<uint4*>(to + low + at) = make_uint4(h0.x, h0.y, h1.x, h1.y);
                                    *reinterpret_cast<uint4*>(to + high + at) = make_uint4(h2.x, h2.y, h3.x, h3.y);
                                }
                            }
                            // past the end a stage holds anything: zeros, in the sequence's last tile
                            if (rows < kTile)
#pragma unroll 1
                                for (int i = 0; i < kTurns; ++i)
                                    if (row0 + i * kRows >= rows) {
                                        *reinterpret_cast<uint4*>(to + low + i * (kRows * 128)) = make_uint4(0u, 0u, 0u, 0u);
                                        *reinterpret_cast<uint4*>(to + high + i * (kRows * 128)) = make_uint4(0u, 0u, 0u, 0u);
                                    }
                        }
                        fence_smem_async();
                        __syncwarp();
                        mbar_arrive_if(&col.full[slot], lane == 0);
                        mbar_arrive_if(&col.stage_empty[stage], lane == 0);
                    }
                }
                w.step(a);
            }
        }
    } else {
        if constexpr (E4M3) more_registers<176>();
        // ---- softmax: two groups of 128 threads, each half of the columns, a key a thread ----
        constexpr int C = NT / 2, CH = C <= 48 ? C : 32, NCH = C / CH;      // columns, and those held at once
        const int grp = warp >> 2, quad = warp & 3, j = quad * 32 + lane, c0 = grp * C, tid = threadIdx.x;
        const uint32_t my_s = tmem + (static_cast<uint32_t>(quad * 32) << 16) + c0, my_o = my_s + 2 * NT;
        constexpr float kLift = E4M3 ? 7.f : 0.f;       // f16 weights up to 2^15 instead of 2^8: fewer of them vanish
        constexpr float kRoomUp = E4M3 ? 8.f + kLift : 64.f;
        int tile_no = 0;
        auto values_done = [&](int k) { wait_for(&col.pv_done[k & 1], k >> 1, &col.dead); };   // the second product of tile k
#pragma unroll 1
        while (w.next(a, &st)) {
            const int kv = w.unit / a.row_tiles, r0 = (w.unit - kv * a.row_tiles) * NT;
            // the columns of this unit
            if (tid < NT) {
                const int r = r0 + tid, i = r / a.group, h = kv * a.group + (r - i * a.group);
                const bool row = i < a.n;
                col.q_at[tid] = row && i < w.tokens ? w.b * a.q_seq + i * a.q_tok + h * a.q_head : -1;
                col.o_at[tid] = row ? w.b * a.o_seq + i * a.o_tok + h * a.o_head : -1;
                col.limit[tid] = row && i < w.tokens ? w.first + i : -1;
                col.neg_m[tid] = 0.f;
                col.seen[tid] = !(row && i < w.tokens);        // rows that take no part need no maximum
            }
            if (tid == 0) col.amax = 0;
            bar_sync(4, kSoftmaxThreads);
            // the queries: 16-byte pieces, rows of 128 bytes swizzled
            constexpr int kPieces = NT * DP / 8, kPer = (kPieces + kSoftmaxThreads - 1) / kSoftmaxThreads;
            float back = 1.f;                               // what the scores are multiplied by for a scaled Q
            {
                uint4 x[kPer];
#pragma unroll
                for (int p = 0; p < kPer; ++p) {
                    const int id = tid + p * kSoftmaxThreads, row = id / (DP / 8), piece = id % (DP / 8);
                    x[p] = make_uint4(0u, 0u, 0u, 0u);
                    if (id < kPieces && piece * 8 < D && col.q_at[row] >= 0)
                        x[p] = *reinterpret_cast<const uint4*>(a.q + col.q_at[row] + piece * 8);
                }
                if constexpr (E4M3) {
                    // bf16 to f16 exactly: the largest element to 2^14..2^15 by a power of two
                    uint32_t most = 0;
#pragma unroll
                    for (int p = 0; p < kPer; ++p) {
                        const uint32_t q4[4] = {x[p].x, x[p].y, x[p].z, x[p].w};
#pragma unroll
                        for (int k = 0; k < 4; ++k) most = max(most, max((q4[k] << 16) & 0x7FFF0000u, q4[k] & 0x7FFF0000u));
                    }
                    most = __reduce_max_sync(0xFFFFFFFFu, most);
                    if (lane == 0) atomicMax(&col.amax, most);
                    bar_sync(4, kSoftmaxThreads);
                    const int ex = static_cast<int>(col.amax >> 23);                    // biased exponent
                    const int up = ex == 0 || ex == 255 ? 0 : min(14 - (ex - 127), 120);
                    const float lift = __uint_as_float(static_cast<uint32_t>(up + 127) << 23);
                    back = __uint_as_float(static_cast<uint32_t>(127 - up) << 23);
#pragma unroll
                    for (int p = 0; p < kPer; ++p) {
                        uint32_t q4[4] = {x[p].x, x[p].y, x[p].z, x[p].w};
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            q4[k] = pack_f16(__uint_as_float(q4[k] << 16) * lift, __uint_as_float(q4[k] & 0xFFFF0000u) * lift);
                        x[p] = make_uint4(q4[0], q4[1], q4[2], q4[3]);
                    }
                }
#pragma unroll
                for (int p = 0; p < kPer; ++p) {
                    const int id = tid + p * kSoftmaxThreads, row = id / (DP / 8), piece = id % (DP / 8);
                    if (id < kPieces)
                        *reinterpret_cast<uint4*>(q_smem + (piece >> 3) * (NT * 128) + row * 128 + (((piece & 7) ^ (row & 7)) << 4)) = x[p];
                }
            }
            fence_smem_async();
            tmem_before_sync();
            __syncwarp();
            mbar_arrive_if(&col.q_full, lane == 0);

            float l[C];
#pragma unroll
            for (int i = 0; i < C; ++i) l[i] = 0.f;
            bool settled = false;
            [[maybe_unused]] const float f0 = a.scale2;
            const int seen_by_all = w.first + r0 / a.group;    // the unit's first row sees positions up to here
#pragma unroll 1
            for (int tile = w.t0; tile < w.t1; ++tile, ++tile_no) {
                const uint32_t s_at = my_s + (tile_no & 1) * NT;
                uint8_t* const p_now = p_smem + tile_no % S::kWeightTiles * S::kPs;
                const int pos = tile * kTile + j;
                const bool masked = tile * kTile + kTile - 1 > seen_by_all;
                // this thread's key: the factor of its scores, log2 of its values' scale (-inf: no key) and its inverse
                const int at = tile_no & 3;
                const bool scored = over(&col.s_full[tile_no & 1], tile_no >> 1);       // (asked early: see above)
                bar_sync(5 + 4 * grp + at, 160);
                float g = col.key[at][j], f = f0;
                [[maybe_unused]] float inv = 1.f;
                if constexpr (E4M3) {
                    // (where there is no key nothing was loaded, or what lies past the end; the logarithm is 2^-22 off
                    // at most, as much as the weight's own exponential, and the reciprocal one unit)
                    const float v = g == 0.f ? fmaxf(col.value_scale[at][j], kLeastScale) : 1.f;
                    f = g == 0.f ? col.key_scale[at][j] * a.scale2 * back : 0.f;
                    g += __log2f(v);
                    inv = reciprocal(v);
                }
                __syncwarp();
                mbar_arrive_if(&col.key_empty[at], lane == 0);
                const uint64_t f2 = pack_f32x2(f, f);
                [[maybe_unused]] const uint64_t g2 = pack_f32x2(g, g), inv2 = pack_f32x2(inv, inv);
                float x[CH];
                // exponents of the weights of chunk ch against the present m
                auto load = [&](int ch) {
                    tmem_load(s_at + ch * CH, x);
#pragma unroll
                    for (int i = 0; i < CH; i += 4) {
                        // (two columns an instruction)
                        const float4 nm = *reinterpret_cast<const float4*>(&col.neg_m[c0 + ch * CH + i]);
                        uint64_t lo = pack_f32x2(nm.x, nm.y), hi = pack_f32x2(nm.z, nm.w);
                        if constexpr (E4M3) {
                            lo = add_f32x2(lo, g2);
                            hi = add_f32x2(hi, g2);
                        }
                        lo = fma_f32x2(pack_f32x2(x[i], x[i + 1]), f2, lo);
                        hi = fma_f32x2(pack_f32x2(x[i + 2], x[i + 3]), f2, hi);
                        x[i] = lo_f32(lo), x[i + 1] = hi_f32(lo);
                        x[i + 2] = lo_f32(hi), x[i + 3] = hi_f32(hi);
                    }
                    if constexpr (!E4M3) {
                        if (g != 0.f) {                            // no such page
#pragma unroll
                            for (int i = 0; i < CH; ++i) x[i] = -INFINITY;
                        }
                    }
                    if (masked) {
#pragma unroll
                        for (int i = 0; i < CH; ++i)
                            if (pos > col.limit[c0 + ch * CH + i]) x[i] = -INFINITY;
                    }
                };
#ifdef PLDP_TEST_STUCK_SCORES
                wait_for(&col.never, 0, &col.dead);
#endif
                wait_more(scored, &col.s_full[tile_no & 1], tile_no >> 1, &col.dead);
                tmem_after_sync();
                bool up = E4M3 && !settled;
                if (!E4M3 && !settled) {
                    // the first key's scores do for a maximum: its own weight is then 1 (2^kLift)
#pragma unroll
                    for (int ch = 0; ch < NCH; ++ch) {
                        load(ch);
                        if (j == 0)
#pragma unroll
                            for (int i = 0; i < CH; ++i) {
                                const int n = c0 + ch * CH + i;
                                if (!col.seen[n] && x[i] > -INFINITY && x[i] < INFINITY) col.neg_m[n] = kLift - x[i], col.seen[n] = 1;
                            }
                        __syncwarp();
                    }
                    bar_sync(2 + grp, 128);
                    settled = !bar_any(2 + grp, 128, (tid & 127) < C && !col.seen[c0 + (tid & 127)]);
                    up = !settled;
                }
#pragma unroll
                for (int ch = 0; ch < NCH; ++ch) {
                    load(ch);
                    float most = x[0];
#pragma unroll
                    for (int i = 1; i < CH; ++i) most = fmaxf(most, x[i]);
                    up = up || most > kRoomUp;
                }
                auto sum = [&](int ch) {
#pragma unroll
                    for (int i = 0; i < CH; i += 2) {
                        const uint64_t w2 = pack_f32x2(x[i], x[i + 1]);
                        uint64_t l2 = pack_f32x2(l[ch * CH + i], l[ch * CH + i + 1]);
                        if constexpr (E4M3) l2 = fma_f32x2(w2, inv2, l2);
                        else l2 = add_f32x2(w2, l2);
                        l[ch * CH + i] = lo_f32(l2), l[ch * CH + i + 1] = hi_f32(l2);
                    }
                };
                auto weights = [&] {
#pragma unroll
                    for (int ch = 0; ch < NCH; ++ch) {
                        if (NCH > 1) load(ch);
#pragma unroll
                        for (int i = 0; i < CH; i += 8) {
                            float* v = x + i;
#pragma unroll
                            for (int k = 0; k < 8; ++k) v[k] = ex2(v[k]);
                            const int byte = (c0 + ch * CH + i) * 2;                      // within the key's weights
                            const int panel = byte / S::kRow, in_row = byte % S::kRow;
                            constexpr int kMask = S::kRow / 16 - 1;
                            const int line = j * S::kRow + in_row;
                            // the swizzle: 16-byte pieces, by the address's bits from 128 bytes up
                            uint8_t* to = p_now + panel * (kTile * S::kRow) + (line ^ (((line >> 7) & kMask) << 4));
                            if constexpr (E4M3) {
                                *reinterpret_cast<uint4*>(to) = make_uint4(pack_f16(v[0], v[1]), pack_f16(v[2], v[3]), pack_f16(v[4], v[5]), pack_f16(v[6], v[7]));
                            } else {
                                uint32_t hi[4], lo[4];
#pragma unroll
                                for (int k = 0; k < 4; ++k) {
                                    hi[k] = pack_bf16(v[2 * k], v[2 * k + 1]);
                                    lo[k] = pack_bf16(v[2 * k] - __uint_as_float(hi[k] << 16),
                                                      v[2 * k + 1] - __uint_as_float(hi[k] & 0xFFFF0000u));
                                }
                                *reinterpret_cast<uint4*>(to) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                                *reinterpret_cast<uint4*>(to + S::kP) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                            }
                        }
                        if (NCH > 1) sum(ch);
                    }
                };
                if (bar_any(2 + grp, 128, up)) {
                    // some column's maximum moves
#pragma unroll
                    for (int ch = 0; ch < NCH; ++ch) {
                        load(ch);
                        float mine = -INFINITY;
#pragma unroll
                        for (int i = 0; i < CH; ++i) {
                            const float top = warp_max(x[i]);
                            if (lane == (i & 31)) mine = top;
                            if (((i & 31) == 31 || i == CH - 1) && lane <= (i & 31)) col.part[quad][c0 + ch * CH + (i & ~31) + lane] = mine;
                        }
                    }
                    bar_sync(2 + grp, 128);
                    const int t = tid & 127;
                    bool unset = false;
                    if (t < C) {
                        const int n = c0 + t;
                        const float top = fmaxf(fmaxf(col.part[0][n], col.part[1][n]), fmaxf(col.part[2][n], col.part[3][n]));
                        float by = 1.f;
                        if (top > -INFINITY && top < INFINITY) {
                            if (!col.seen[n]) {
                                col.seen[n] = 1;
                                col.neg_m[n] = kLift - top;
                            } else if (top > kLift) {
                                by = ex2(kLift - top);
                                col.neg_m[n] += kLift - top;
                            }
                        }
                        col.factor[n] = by;
                        unset = !col.seen[n];
                    }
                    settled = !bar_any(2 + grp, 128, unset);
#pragma unroll
                    for (int i = 0; i < C; ++i) l[i] *= col.factor[c0 + i];
                    if (tile > w.t0) {
                        values_done(tile_no - 1);
                        tmem_after_sync();
#pragma unroll
                        for (int m = 0; m < S::kCols / NT - 2; ++m)             // blocks and parts
#pragma unroll
                            for (int i = 0; i < C; i += 8) {
                                float o[8];
                                tmem_load(my_o + m * NT + i, o);
#pragma unroll
                                for (int k = 0; k < 8; ++k) o[k] *= col.factor[c0 + i + k];
                                tmem_store8(my_o + m * NT + i, o);
                            }
                        tmem_store_wait();
                    }
                    if (NCH == 1) load(0);
                }
                // The weights that were in their place have been read: of two tiles' places, by the second product of
                // tile_no - 2, which was issued before the first one of tile_no.
                if (S::kWeightTiles == 1 && tile_no > 0) values_done(tile_no - 1);
                weights();
                if constexpr (!E4M3) {
                    // what the pages hold past the end is not used: zeros, in the values' tile
                    if (tile * kTile + kTile > w.keys) {
                        const int e = 2 * tile_no + 1, slot = e % S::kSlots;
                        wait_for(&col.full[slot], e / S::kSlots, &col.dead);
                        if (pos >= w.keys)
#pragma unroll 1
                            for (int p = grp; p < 8 * S::kPanels; p += 2)
                                *reinterpret_cast<uint4*>(ring + slot * S::kSlot + (p >> 3) * (kTile * 128) + j * 128 + (p & 7) * 16) =
                                    make_uint4(0u, 0u, 0u, 0u);
                    }
                }
                fence_smem_async();
                tmem_before_sync();
                __syncwarp();
                mbar_arrive_if(&col.p_full[tile_no % S::kWeightTiles], lane == 0);
                if (NCH == 1) sum(0);
            }
            // the sums over the keys
            {
                const int at = warp_columns<C>(l, lane);
                if ((lane & (ColumnSums<C>::kLanes - 1)) == 0)
#pragma unroll
                    for (int i = 0; i < ColumnSums<C>::kOwn; ++i) col.part[quad][c0 + at + i] = l[i];
                bar_sync(2 + grp, 128);
                const int t = tid & 127;
                if (t < C) {
                    const int n = c0 + t;
                    const float s = col.part[0][n] + col.part[1][n] + col.part[2][n] + col.part[3][n];
                    col.sum[n] = s;
                    col.inverse[n] = s == 0.f || col.limit[n] < 0 ? 0.f : 1.f / s;      // 0: an empty row
                }
            }
            values_done(tile_no - 1);
            tmem_after_sync();
            bar_sync(4, kSoftmaxThreads);
            const bool whole = w.t0 == 0 && w.t1 == w.T;
            const int rows = min(NT, a.n * a.group - r0);           // columns that are rows of the output
            const long long unit_at = w.at - w.t0;
            // which of this CTA's two places in the workspace: the unit began in another's part, or in this one's
            constexpr int kPart = NT * (DP + 2);
            float* part = a.parts + static_cast<int64_t>(2 * blockIdx.x + (w.t0 == 0 ? 1 : 0)) * kPart;
            auto lse_at = [&](int n) {
                const int r = r0 + n, i = r / a.group;
                return (static_cast<int64_t>(w.b) * a.n + i) * a.q_heads + kv * a.group + (r - i * a.group);
            };
            if (whole) {
                if (tid < NT && a.lse && col.o_at[tid] >= 0) {
                    const float s = col.limit[tid] >= 0 ? col.sum[tid] : 0.f;
                    a.lse[lse_at(tid)] = s == 0.f ? -INFINITY : (log2f(s) - col.neg_m[tid]) * 0.69314718055994531f;
                }
            } else if (tid < NT) {
                part[NT * DP + tid] = col.seen[tid] ? -col.neg_m[tid] : -INFINITY;
                part[NT * DP + NT + tid] = col.sum[tid];
            }
#pragma unroll
            for (int m = 0; m < S::kBlocks; ++m) {
                const int d = m * 128 + j;
#pragma unroll
                for (int ch = 0; ch < NCH; ++ch) {
                    float o[CH];
                    tmem_load(my_o + m * S::kWeights + ch * CH, o);
                    if constexpr (!E4M3) {
                        float low[CH];
                        tmem_load(my_o + m * S::kWeights + NT + ch * CH, low);
#pragma unroll
                        for (int i = 0; i < CH; ++i) o[i] += low[i];
                    }
                    if (d >= D) {
                    } else if (whole) {
#pragma unroll
                        for (int i = 0; i < CH; ++i) {
                            const int n = c0 + ch * CH + i;
                            const float by = col.inverse[n];
                            if (n < rows) a.out[col.o_at[n] + d] = __float2bfloat16(by == 0.f ? 0.f : o[i] * by);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < CH; ++i)
                            if (c0 + ch * CH + i < rows) part[(c0 + ch * CH + i) * DP + d] = o[i];
                    }
                    __syncwarp();
                }
            }
            if (!whole) {
                // the last of the unit's CTAs joins the parts
                const long long each = col.each, extra = col.extra;
                auto owner = [&](long long at) {                         // the CTA whose part holds a tile
                    const long long edge = (each + 1) * extra;
                    const long long x = at < edge ? at : at - edge, y = at < edge ? each + 1 : each;
                    const long long q = (x | y) >> 32 ? x / y : static_cast<uint32_t>(x) / static_cast<uint32_t>(y);
                    return static_cast<int>(at < edge ? q : extra + q);
                };
                const int c_first = owner(unit_at), c_last = owner(unit_at + w.T - 1);
                bar_sync(4, kSoftmaxThreads);
                if (tid == 0) {
                    // after all that the barrier has seen written, before what the others wrote is read
                    uint32_t* ticket = a.tickets + c_first;      // (of the units that begin there it is the only one cut)
                    uint32_t before;
                    asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;" : "=r"(before) : "l"(ticket) : "memory");
                    const bool is_last = before == static_cast<uint32_t>(c_last - c_first);
                    if (is_last) *ticket = 0u;
                    col.last = is_last;
                }
                bar_sync(4, kSoftmaxThreads);
                if (col.last) {
                    // The parts' factors 2^(m - M) / sum first, in the weights' place (64 parts a turn at most), then
                    // sums over the parts, V elements of a row a thread.
                    constexpr int V = 4, kRowItems = DP / V, kFactors = 64;
                    static_assert(kFactors * NT * 4 <= S::kPs * S::kWeightTiles, "factors");
                    float* factors = reinterpret_cast<float*>(p_smem);               // [part][row]
                    const int parts = c_last - c_first + 1;
                    auto place = [&](int k) { return a.parts + static_cast<int64_t>(2 * (c_first + k) + (k == 0 ? 1 : 0)) * kPart; };
                    float M = -INFINITY, sum = 0.f;
                    if (tid < rows) {
                        const bool live = col.limit[tid] >= 0;
#pragma unroll 1
                        for (int k0 = 0; k0 < parts; k0 += 8) {                      // eight parts' m and sum in flight
                            float m[8], part_sum[8], top = M;
#pragma unroll
                            for (int q = 0; q < 8; ++q) {
                                m[q] = -INFINITY, part_sum[q] = 0.f;
                                if (live && k0 + q < parts) {
                                    m[q] = __ldcg(place(k0 + q) + NT * DP + tid);
                                    part_sum[q] = __ldcg(place(k0 + q) + NT * DP + NT + tid);
                                }
                            }
#pragma unroll
                            for (int q = 0; q < 8; ++q) {
                                top = fmaxf(top, m[q]);
                                if (k0 + q < min(parts, kFactors)) factors[(k0 + q) * NT + tid] = m[q];
                            }
                            if (!(top > -INFINITY)) continue;
                            sum *= ex2(M - top);                                     // (2^-inf of the first)
                            M = top;
#pragma unroll
                            for (int q = 0; q < 8; ++q)
                                if (m[q] > -INFINITY) sum = fmaf(ex2(m[q] - M), part_sum[q], sum);
                        }
                        if (a.lse) a.lse[lse_at(tid)] = sum == 0.f ? -INFINITY : (log2f(sum) + M) * 0.69314718055994531f;
                    }
                    const float inverse = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll 1
                    for (int k0 = 0; k0 < parts; k0 += kFactors) {
                        const int k1 = min(parts, k0 + kFactors);
                        if (tid < rows)
#pragma unroll 1
                            for (int k = k0; k < k1; ++k) {
                                const float m = k0 == 0 ? factors[k * NT + tid] : __ldcg(place(k) + NT * DP + tid);
                                factors[(k - k0) * NT + tid] = inverse == 0.f ? 0.f : ex2(m - M) * inverse;
                            }
                        bar_sync(4, kSoftmaxThreads);
#pragma unroll 1
                        for (int item = tid; item < rows * kRowItems; item += kSoftmaxThreads) {
                            const int n = item / kRowItems, d = item % kRowItems * V;
                            if (d >= D) continue;
                            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
                            const float* sums = place(0) + n * DP + d;               // the first round's sums stay in its place
                            if (k0 > 0) o = __ldcg(reinterpret_cast<const float4*>(sums));
#pragma unroll 1
                            for (int k = k0; k < k1; k += 8) {                       // eight parts in flight
                                float4 x[8];
#pragma unroll
                                for (int q = 0; q < 8; ++q)
                                    if (k + q < k1) x[q] = __ldcg(reinterpret_cast<const float4*>(place(k + q) + n * DP + d));
#pragma unroll
                                for (int q = 0; q < 8; ++q) {
                                    if (k + q >= k1) break;
                                    const float by = factors[(k + q - k0) * NT + n];
                                    if (by == 0.f) continue;                          // (its part may hold anything)
                                    o.x = fmaf(by, x[q].x, o.x);
                                    o.y = fmaf(by, x[q].y, o.y);
                                    o.z = fmaf(by, x[q].z, o.z);
                                    o.w = fmaf(by, x[q].w, o.w);
                                }
                            }
                            if (k1 < parts)
                                __stcg(reinterpret_cast<float4*>(const_cast<float*>(sums)), o);
                            else
                                *reinterpret_cast<uint2*>(a.out + col.o_at[n] + d) = make_uint2(pack_bf16(o.x, o.y), pack_bf16(o.z, o.w));
                        }
                        bar_sync(4, kSoftmaxThreads);
                    }
                }
            }
            if (col.dead && tid == 0 && a.status) atomicOr(a.status + w.b, PLDP_ST_TIMEOUT);
            tmem_before_sync();
            bar_sync(4, kSoftmaxThreads);
            w.step(a);
        }
    }
    tmem_before_sync();
    __syncthreads();
    if (warp == S::kMmaWarp) {
        tmem_after_sync();
        tmem_free(tmem, S::kTmem);
    }
}

template <int NT, int DP, bool E4M3>
cudaError_t launch(const AttendArgs& a, const Maps& m, int ctas, cudaStream_t s) {
    constexpr int bytes = Shape<NT, DP, E4M3>::kBytes;
    const cudaError_t e = cudaFuncSetAttribute(attend_kernel<NT, DP, E4M3>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != cudaSuccess) return e;
    return launch_pdl(attend_kernel<NT, DP, E4M3>, dim3(ctas), dim3(Shape<NT, DP, E4M3>::kThreads), bytes, s, 0, a, m.k, m.v);
}
template <int DP, bool E4M3>
cudaError_t launch_columns(const AttendArgs& a, const Maps& m, int nt, int ctas, cudaStream_t s) {
    if (nt == 16) return launch<16, DP, E4M3>(a, m, ctas, s);
    if (nt == 32) return launch<32, DP, E4M3>(a, m, ctas, s);
    if constexpr (DP <= 128) {
        if (nt == 48) return launch<48, DP, E4M3>(a, m, ctas, s);
        if (nt == 64) return launch<64, DP, E4M3>(a, m, ctas, s);
        if (nt == 96) return launch<96, DP, E4M3>(a, m, ctas, s);
        return launch<128, DP, E4M3>(a, m, ctas, s);
    } else {
        return cudaErrorInvalidValue;
    }
}
template <bool E4M3>
cudaError_t launch_dims(const AttendArgs& a, const Maps& m, int nt, int ctas, cudaStream_t s) {
    if (a.c.head_dim <= 64) return launch_columns<64, E4M3>(a, m, nt, ctas, s);
    if (a.c.head_dim <= 128) return launch_columns<128, E4M3>(a, m, nt, ctas, s);
    return launch_columns<256, E4M3>(a, m, nt, ctas, s);
}

}  // namespace
}  // namespace pldp
