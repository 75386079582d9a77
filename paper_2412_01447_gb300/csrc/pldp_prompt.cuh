// Causal attention of packed prompts over the paged cache: the kernel of pldp_attend_prompt (prompt.cu).
#pragma once

#include "pldp_attend.cuh"

namespace pldp {

struct PromptArgs {
    CacheView c;
    const __nv_bfloat16* q;
    __nv_bfloat16* out;
    int64_t q_tok, q_head, o_tok, o_head;
    const int32_t *rows, *start;
    float* lse;
    uint32_t* status;
    float* parts;                          // [2 a CTA][Part]
    struct CutUnit* cuts;                  // [CTAs]
    int B, R, q_heads, group;
    uint32_t group_mul, group_shift;       // division by group, as CacheView's by the page
    int box, pitch;                        // as AttendArgs
    int head_first;
    // bf16, heads above 128 elements: a box holds all of a vector's panels of 64 elements (1: their places in the map go on
    // with the next head's, 2: a head's positions with the next head's), or (0) one of them
    int whole;
    int group_step, panel_step;            // bytes of shared memory from 8 positions to the next ones, and from panel to panel
    int q_boxes;                           // queries by boxes of whole tokens
    float scale2;                          // |scale| * log2(e)
    uint32_t flip;                         // what turns the signs of two queries for a negative scale
};

// A unit that several CTAs have parts of, written by the CTA in which it begins: what the join needs.
struct CutUnit {
    int parts;                             // 0: none
    int first_cta;
    int row0, rows;                        // the unit's rows of the sequence and kv head (token * group + head)
    int row_base, kv;                      // the sequence's first row
};

struct PromptMaps {
    Maps pool;
    CUtensorMap q;
};
// One launch; one translation unit a cache type.
cudaError_t launch_prompt_bf16(const PromptArgs& a, const PromptMaps& m, int ctas, cudaStream_t s);
cudaError_t launch_prompt_e4m3(const PromptArgs& a, const PromptMaps& m, int ctas, cudaStream_t s);

__host__ __device__ constexpr int prompt_dim(int head_dim) { return head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256; }
__host__ __device__ constexpr int prompt_rows(int dp) { return dp == 256 ? 128 : 256; }       // rows of a unit
// What a part of a unit leaves: per 128 rows the averages [DP / 4][128][4], then the maxima [128] and the weights' sums [128].
__host__ __device__ constexpr int prompt_part(int dp) { return prompt_rows(dp) * (dp + 2); }
constexpr int kPromptCtas = 192;           // at most

namespace {

#ifdef __CUDACC__
#define PLDP_ONE_COPY __noinline__
#endif
// (32 bits where they do: a division of 64 takes some 100 cycles, and these are done before anything else can start)
__host__ __device__ inline uint64_t quotient(uint64_t x, uint64_t y) {
    return (x | y) >> 32 ? x / y : (uint32_t)x / (uint32_t)y;
}
// sum over i < n of floor((c + i) / d): the first x numbers from 0 on have quotients of 0 to x / d - 1, d of each, and then the
// last one.  (What both sums have above 2^64 is the same.  One copy of its code: at a kernel's start every new line of code is a miss
// in the instruction cache, which takes longer than what it holds.)
__host__ __device__ inline PLDP_ONE_COPY uint64_t quotients_sum(uint64_t n, uint64_t c, uint64_t d) {
    const uint64_t q1 = quotient(c + n, d), q0 = quotient(c, d);
    return d * (q1 * (q1 - 1) / 2) + q1 * (c + n - q1 * d) - d * (q0 * (q0 - 1) / 2) - q0 * (c - q0 * d);
}
// sum over i < n of floor((a i + b) / m), for an `a` of 128 or 256 and an m that 128 divides: by 128 these are the quotients above, or
// of 2 i + c, for which floor(2 x) = floor(x) + floor(x + 1/2).
__host__ __device__ inline uint64_t floor_sum(uint64_t n, uint64_t m, uint64_t a, uint64_t b) {
    const uint64_t d = m / 128, c = b / 128;
    if (a == 128) return quotients_sum(n, c, d);
    return quotients_sum(n, c / 2, d) + quotients_sum(n, (c + d) / 2, d);
}

// The rows of a sequence and kv head, token * group + head, cut into units of `UR`; unit u sees the keys up to its last
// row's token, T(u) tiles.  tiles_before: those of the units before u, u up to the number of units.
struct Units {
    int64_t N;         // rows
    int group, start, count;
};
__device__ __forceinline__ Units units_of(const PackedRows& p, int group) {
    return {static_cast<int64_t>(p.count) * group, group, p.first, p.count};
}
template <int UR>
__host__ __device__ __forceinline__ int unit_count(const Units& s) { return static_cast<int>((s.N + UR - 1) / UR); }
template <int UR>
__host__ __device__ __forceinline__ int unit_tiles(const Units& s, int u) {
    const int64_t end = min(s.N, (static_cast<int64_t>(u) + 1) * UR);
    return (s.start + static_cast<int>(static_cast<uint32_t>(end - 1) / static_cast<uint32_t>(s.group)) + kTile) / kTile;
}
template <int UR>
__host__ __device__ __forceinline__ int64_t tiles_before(const Units& s, int u) {
    if (u == 0) return 0;
    const int whole = static_cast<int64_t>(u) * UR > s.N ? u - 1 : u;          // the last unit may have fewer rows
    static_assert(kTile == 128 && (UR == kTile || UR == 2 * kTile), "rows of a unit");
    const uint64_t m = static_cast<uint64_t>(kTile) * s.group;
    int64_t n = 0;
    if (whole > 0) n = floor_sum(whole, m, UR, static_cast<uint64_t>(s.start) * s.group + UR - 1 + m);
    if (whole < u) n += unit_tiles<UR>(s, whole);
    return n;
}
// What a unit costs beside its tiles, in tiles: its queries' way in, the first scores' and the last weights' latency, its
// results' way out.  The list counts it, so that a part of many short units is not the last to end.
constexpr int kUnitCost = 2;
template <int UR>
__host__ __device__ PLDP_ONE_COPY int64_t cost_before(const Units& s, int u) { return tiles_before<UR>(s, u) + static_cast<int64_t>(u) * kUnitCost; }
// The unit that holds place x of the list of one kv head: cost_before(u) <= x < cost_before(u + 1).
template <int UR>
__host__ __device__ __forceinline__ int unit_at(const Units& s, int units, int64_t x, int64_t* before) {
    // tiles grow linearly from unit to unit: the root of their sum, and from there to the unit itself
    const float a2 = UR / (2.f * kTile * s.group), b = kUnitCost + (s.start + 0.5f * UR / s.group) / kTile + 0.5f;
    int u = static_cast<int>((sqrtf(b * b + 4.f * a2 * static_cast<float>(x)) - b) / (2.f * a2));
    u = max(0, min(u, units - 1));
    int64_t at = cost_before<UR>(s, u);
    while (at > x) at -= kUnitCost + unit_tiles<UR>(s, --u);
    for (int next; at + (next = kUnitCost + unit_tiles<UR>(s, u)) <= x; ++u) at += next;
    *before = at;
    return u;
}
// Units of so few tiles are one CTA's, that of the place in the list where they begin.
constexpr int kWhole = 4;
// And there are no more parts than make some this many tiles each (never fewer than two): of a unit that several have, a few tiles
// each pay for the join.
constexpr int kLeast = 3;

template <int DP, bool E4M3>
struct PromptShape {
    static constexpr int kQ = DP == 256 ? 1 : 2;               // tiles of 128 rows
    static constexpr int kRows = kQ * 128;
    static constexpr int kSoftmaxWarps = 4 * kQ;
    static constexpr int kConvertWarps = E4M3 ? 4 : 0;
    // warps: softmax, matrix instructions, keys' scales, copies, queries, conversion
    static constexpr int kMmaWarp = kSoftmaxWarps, kKeyWarp = kMmaWarp + 1, kCopyWarp = kMmaWarp + 2, kQueryWarp = kMmaWarp + 3;
    static constexpr int kConvertWarp = kMmaWarp + 4;
    static constexpr int kThreads = (kSoftmaxWarps + 4 + kConvertWarps) * 32;
    static constexpr int kPanels = DP / 64;
    static constexpr int kSlot = kPanels * kTile * 128;
    static constexpr int kQBytes = kQ * kPanels * 128 * 128;
    static constexpr int kStatic = E4M3 ? 8192 : 2048;         // PromptShared
    // Rows of the result pass through shared memory, 32 rows of a warp and kOutBytes of each at a time, to be written whole
    // lines at a time.
    static constexpr int kOutBytes = E4M3 && DP >= 128 ? 64 : 128;
    static constexpr int kOut = kSoftmaxWarps * 32 * kOutBytes;
    // e4m3: codes as they are, a tile (heads above 128 elements: half of one) a stage
    static constexpr int kStageRows = DP == 256 ? 64 : kTile, kStage = E4M3 ? kStageRows * (DP < 128 ? 128 : DP) : 0;
    static constexpr int kRoom = kMaxShared - 1024 - kStatic - kQBytes - kOut;
    static constexpr int kMost = (kRoom - (DP == 256 ? 1 : 2) * kStage) / kSlot;
    static constexpr int kSlots = kMost > 6 ? 6 : kMost;
    static constexpr int kFit = E4M3 ? (kRoom - kSlots * kSlot) / kStage : 0;
    static constexpr int kStages = kFit > 6 ? 6 : kFit;
    static constexpr int kBytes = kQBytes + kSlots * kSlot + kStages * kStage + kOut + 1024;
    static constexpr int kO = 256;                             // column of the first sums
    // 384 threads start with 168 registers each (640: 96); the softmax takes what the others leave
    static constexpr int kSoftmaxRegs = E4M3 ? 184 : 192, kOtherRegs = E4M3 ? 72 : 120, kConvertRegs = 72;
    static_assert(kSlots >= 2 && (!E4M3 || kStages >= 1) && kBytes + kStatic <= kMaxShared, "shared memory");
};

constexpr int kApart = INT32_MAX;
constexpr int kAbove = 7;                  // a scale may be this many powers of two above the unit: 448 * 2^7 is f16
// A positive float is below 2^(exponent_of it); 0: -126.
__device__ __forceinline__ int exponent_of(float x) { return static_cast<int>(__float_as_uint(x) >> 23) - 126; }

constexpr int kAhead = 8;                  // tiles whose holes are kept (more than the ring of keys holds)

// A unit, or what a CTA has of it, as one warp works it out for the others (rows: token * group + head).
struct alignas(16) PromptUnit {
    int b, kv;
    int row, start, end;         // the sequence's first row, that one's position, and the first position that is not its
    int r0, rows;                // the unit's first row of the sequence and kv head, and how many (below 256 or 128 in the last)
    int t0, t1, T;               // this CTA's tiles of keys, of all; T 0: there is no more
    int last_cta;                // where the unit begins and others have the rest: the CTA of its last tile
    int unused;
};
constexpr int kUnits = 8;                  // worked out and not yet done by all

template <bool E4M3>
struct PromptShared {
    // of the keys of four tiles: the scale of the key, that of the value, and by 2^-unit as two f16
    alignas(16) float key_scale[E4M3 ? 4 : 1][E4M3 ? kTile : 4], value[E4M3 ? 4 : 1][E4M3 ? kTile : 4];
    uint32_t value_scale[E4M3 ? 4 : 1][E4M3 ? kTile : 4];
    int unit_of[4];                        // kApart: the weights take the values' scales, each row in a unit of its own
    uint32_t live[kAhead][4];              // whether a page holds the key, a bit each; looked at where `holes` is set
    int holes[kAhead];
    PromptUnit units[kUnits];
    uint64_t unit_full[kUnits], unit_empty[kUnits], full[8], empty[8], stage_full[6], stage_empty[6], q_raw[2], s_full[2], p_full[2][2], pv_half[2], pv_done[2], q_full[2], q_empty[2], tail, drained,
        key_full[4], key_empty[4];
#ifdef PLDP_TEST_STUCK_SCORES
    uint64_t never;                        // test build: a barrier that nothing arrives on
#endif
    uint32_t tmem;
    int dead, zeros;
    long long warp_sum[24];
    long long total;
    // where this CTA's part of the list starts
    int b, kv, unit, in;                   // (in: how far into the unit, its own cost first)
    long long at, count, each, extra;
};

// The CTA's part of the list, unit by unit: sequences, their kv heads, the units of one of those.
template <int UR>
struct PromptWalk {
    int b, kv, unit, t0;
    int pre;           // what is left of the unit's own cost
    long long at, left;
    // the unit's
    PackedRows p;
    Units s;
    int units, T, t1;
    int64_t r0;
    int rows;          // below UR only in the last unit
    int end;           // positions from here on are not the sequence's

    __device__ __forceinline__ bool next(const PromptArgs& a) {
        if (left <= 0) return false;
        uint32_t st;
        while (true) {                                           // (sequences without rows hold no tiles)
            p = packed_rows(a.rows, a.start, b, a.R, a.c.capacity, st);
            if (p.count > 0) break;
            ++b;
        }
        s = units_of(p, a.group);
        units = unit_count<UR>(s);
        end = s.start + s.count;
        T = unit_tiles<UR>(s, unit);
        if (T <= kWhole) {
            t1 = T;
        } else {
            if (left <= pre) return false;
            t1 = left - pre < T - t0 ? t0 + static_cast<int>(left - pre) : T;
        }
        r0 = static_cast<int64_t>(unit) * UR;
        rows = static_cast<int>(min(static_cast<int64_t>(UR), s.N - r0));
        return true;
    }
    // Where a part begins inside a unit that is another CTA's whole, it begins behind it.
    __device__ __forceinline__ bool first(const PromptArgs& a, int in) {
        if (in > 0) {
            uint32_t st;
            p = packed_rows(a.rows, a.start, b, a.R, a.c.capacity, st);
            s = units_of(p, a.group);
            units = unit_count<UR>(s);
            T = unit_tiles<UR>(s, unit);
            if (T <= kWhole) {
                t0 = 0, t1 = T, pre = kUnitCost - in;                   // (what of the unit lies in this part goes with it)
                step(a);
            }
        }
        return next(a);
    }
    __device__ __forceinline__ void step(const PromptArgs& a) {
        at += pre + (t1 - t0);
        left -= pre + (t1 - t0);
        t0 = 0, pre = kUnitCost;
        if (++unit == units) {
            unit = 0;
            if (++kv == a.c.heads) kv = 0, ++b;
        }
    }
};

// tma_box by the lane that leads, all lanes with the same values.
__device__ __forceinline__ void tma_box_if(void* dst, const CUtensorMap* map, int c0, int c1, int c2, int c3, uint64_t* bar, uint32_t lead) {
    asm volatile(
        "{\n\t.reg .pred q;\n\t"
        "setp.ne.u32 q, %7, 0;\n\t"
        "@q cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];\n\t}"
        ::"r"(smem_u32(dst)), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(smem_u32(bar)), "r"(lead)
        : "memory");
}
__device__ __forceinline__ void tma_box5_if(void* dst, const CUtensorMap* map, int c2, int c3, int c4, uint64_t* bar, uint32_t lead) {
    asm volatile(
        "{\n\t.reg .pred q;\n\t.reg .b32 z;\n\t"
        "mov.u32 z, 0;\n\t"
        "setp.ne.u32 q, %6, 0;\n\t"
        "@q cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {z, z, %2, %3, %4}], [%5];\n\t}"
        ::"r"(smem_u32(dst)), "l"(map), "r"(c2), "r"(c3), "r"(c4), "r"(smem_u32(bar)), "r"(lead)
        : "memory");
}
// D += A B with A in tensor memory.
__device__ __forceinline__ void mma_f16_tmem(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t b_hi, uint32_t form, uint32_t accumulate,
                                             uint32_t lead) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t.reg .b64 b;\n\t"
        "mov.b64 b, {%2, %3};\n\t"
        "setp.ne.u32 p, %5, 0;\n\t"
        "setp.ne.u32 q, %6, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %4, p;\n\t}"
        ::"r"(d), "r"(a), "r"(b_lo), "r"(b_hi), "r"(form), "r"(accumulate), "r"(lead)
        : "memory");
}
__device__ __forceinline__ void tmem_store32(uint32_t addr, const uint32_t* v) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};"
        ::"r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]),
          "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]),
          "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]),
          "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31]), "r"(addr)
        : "memory");
}
// 16 bytes from global to shared memory, later, or zeros.
__device__ __forceinline__ void copy_or_zeros(void* to, const void* from, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(to)), "l"(from), "r"(there ? 16 : 0) : "memory");
}
// 2^e, -126 <= e <= 127.
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint64_t mul_f32x2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
// The arithmetic of the weights, where it is written.
__device__ __forceinline__ float ordered_ex2(float x) {
    float y;
    asm volatile("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float ordered_max3(float a, float b, float c) {
    float d;
    asm volatile("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ uint64_t ordered_fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm volatile("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t ordered_add2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm volatile("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint32_t ordered_bf16(float lo, float hi) {
    uint32_t d;
    asm volatile("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
__device__ __forceinline__ uint32_t ordered_f16(float lo, float hi) {
    uint32_t d;
    asm volatile("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
// A tile of keys (e4m3) of which some rows see only a part, and whose other values are so much larger that a unit for all of them
// would cost these rows theirs.  The values' codes go into the product as they are (by 1/4), and each weight takes its value's
// scale: weights w_j = 2^(x_j - m + 7) become w_j 4 v_j / 2^unit, where unit is the row's own, above the largest scale that it
// sees.  Done here in the scores, so that the loops over tiles need not know of it: x_j (by f, the queries' factor) becomes
// x_j + log2(4 v_j / 2^unit), and the sum of the weights takes the difference in advance, the w_j and not what the loop will add.  The
// scores are divided by the keys' scales, as the loop multiplies by them, and f is 1 from here on.  (A function, as the loops of all
// roles share one instruction cache: 24 short prompts, which never come here, 139 us without it, 145 so, 157 with its code in the
// loop over tiles.)
struct ApartRow {
    float m, l;
    int unit;
};
template <int DP>
__device__ __noinline__ ApartRow apart_tile(uint32_t s_at, uint32_t o_at, const float* key_scale, const float* value, float f, bool sums, ApartRow r) {
    constexpr float kLift = 7.f, kRoomUp = 8.f;
    float top = -INFINITY, largest = 0.f;
#pragma unroll 1
    for (int i = 0; i < kTile; i += 8) {
        float y[8];
        tmem_load(s_at + i, y);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float x = y[k] * key_scale[i + k] * f;
            top = fmaxf(top, x);
            if (x > -INFINITY) largest = fmaxf(largest, value[i + k]);
        }
    }
    float by = 1.f;
    if (top > r.m + kRoomUp || (r.m == -INFINITY && top > -INFINITY)) {
        by = r.m == -INFINITY ? 0.f : ex2(r.m - top);
        r.m = top;
    }
    r.l *= by;
    if (top > -INFINITY) {                                     // (a row that sees nothing of the tile stays as it is)
        const int now = max(r.unit, min(exponent_of(largest) + 2, 126));
        if (now != r.unit && r.unit != INT32_MIN) by *= power_of_two(max(r.unit - now, -126));
        r.unit = now;
    }
    __syncwarp();
    tmem_after_sync();
    if (sums && __any_sync(0xFFFFFFFFu, by != 1.f)) {
#pragma unroll 1
        for (int i = 0; i < DP; i += 8) {
            float o[8];
            tmem_load(o_at + i, o);
#pragma unroll
            for (int k = 0; k < 8; ++k) o[k] *= by;
            tmem_store8(o_at + i, o);
        }
    }
    const float less = r.m == -INFINITY ? 0.f : kLift - r.m, lift = top > -INFINITY ? power_of_two(2 - r.unit) : 0.f;
#pragma unroll 1
    for (int i = 0; i < kTile; i += 8) {
        float y[8];
        tmem_load(s_at + i, y);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float scale = key_scale[i + k], x = y[k] * scale * f;
            // (keys that the row does not see: -infinity)
            y[k] = x > -INFINITY ? (x + log2f(value[i + k] * lift)) / scale : -INFINITY;
            r.l += ex2(x + less) - ex2(__fmaf_rn(__fmul_rn(y[k], scale), 1.f, less));
        }
        tmem_store8(s_at + i, y);
    }
    tmem_store_wait();
    return r;
}

// ---------------------------------------------------------------------------
// One pass over the keys that a unit sees, 128 at a time.  A unit is 256 (heads above 128 elements: 128) rows of one
// sequence and key/value head: the rows of all of its query heads, token by token, so short prompts with grouped heads
// fill the tensor core's 128 rows and only the last tokens' keys are masked.
//   S [128 rows, 128 keys] = Q K^T       P = 2^(x - m)       O [128 rows, D] += P V
// S and O of two row tiles stay in tensor memory (512 columns); P, 16 bits a weight, overwrites S and is the second
// product's operand from there, so only queries, keys and values pass through shared memory.  A thread owns a row: its
// maximum, sum and rescaling need no other thread.  While one tile of rows is in the softmax, the tensor core works for
// the other.  The running maximum m of a row moves only when a score passes it by more than 2^64 (2^8 where weights are
// f16): weights may be large, their rounding is relative.
//
// Weights are rounded to bf16 (2^-8 of each) over a bf16 cache, whose values need bf16's range: two terms, as a step's attention takes
// them, would make the second product, half of the work here, twice as long.  Over an e4m3 cache codes are converted by warps
// of their own and weights are f16 (2^-11): keys as f16, which holds every code, their scales multiplying the scores; values
// times scale / 2^unit, each rounded to f16 (2^-11), where 2^unit is above the largest scale that the unit has met of keys that its
// rows see, and O is multiplied when that rises (apart_tile: where keys that only some of them see are much larger).
//
// What bounds it: the matrix unit, 64 cycles for each 16 elements of a product of 128 rows and 128 columns, and beside it
// the special functions' rate, 4 cycles a warp's 32 exponentials, and the hand-over of each tile between the roles.  Measured, bf16, heads of
// 128, 32 over 8: a prompt of 8192 tokens 374 to 394 us (1400 to 1470 TFLOP/s, 0.74 to 0.78 of the rate measured for one large matrix
// product), four of 16384 3.2 to 3.5 ms (1420 to 1520, where the clock falls under the power limit); 40 over 8, whose groups of five do
// not divide 128 rows, 4.6 to 4.9 ms (1260 to 1350).  Steps on the way there, the former's us:
// 2530 as one CTA's products and softmax in turn; 685 by two tiles of rows, queries asynchronous; 428 with weights in halves, of
// which the first is multiplied while the second is taken; 370 with the units worked out by one warp and seldom-run code kept
// short, as every new line of it is a miss in the instruction cache.  Tried and not kept: a warp for each tile of rows'
// products (494 for 425), their issue as a loop (522 for 364), a tile's maximum before its weights (two passes over the scores).
// e4m3: 550 us; there the conversion (without its work 8 % less) and the scales of the keys (6 %, which each warp reads for
// each of its rows' tiles) take issue slots and shared memory's bandwidth, all of which the first product's operands need,
// from the softmax, whose halves take 1000 cycles each.  Keys as codes in an 8-bit product, the queries split into two of
// them, would save no more than the keys' half of the conversion, 3 %.
//
// The tiles of all units form one list, cut into equal parts, one a CTA (one a SM), whatever the lengths are; what
// a part holds of a unit that others share goes to the workspace, and the join, a kernel behind this one, adds them in order.
// ---------------------------------------------------------------------------
template <int DP, bool E4M3>
__global__ void __launch_bounds__(PromptShape<DP, E4M3>::kThreads, 1)
prompt_kernel(const PromptArgs a, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map,
              const __grid_constant__ CUtensorMap q_map) {
    using S = PromptShape<DP, E4M3>;
    constexpr int UR = S::kRows, NQ = S::kQ, kThreads = S::kThreads;
    static_assert(sizeof(PromptShared<E4M3>) <= S::kStatic, "shared memory");
    extern __shared__ uint8_t raw[];
    __shared__ __align__(16) PromptShared<E4M3> sh;
    uint8_t* ring = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
    uint8_t* const q_smem = ring + S::kSlots * S::kSlot;
    uint8_t* const out_smem = q_smem + S::kQBytes;
    [[maybe_unused]] uint8_t* const stages = out_smem + S::kOut;
    const CacheView& c = a.c;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, D = c.head_dim;

    if (warp == S::kMmaWarp) tmem_alloc(&sh.tmem, 512);
    if (threadIdx.x == 0) {
        for (int i = 0; i < 8; ++i) {
            mbar_init(&sh.full[i], E4M3 ? S::kConvertWarps : 1);
            mbar_init(&sh.empty[i], 1);
        }
        for (int i = 0; i < 6; ++i) {
            mbar_init(&sh.stage_full[i], 1);
            mbar_init(&sh.stage_empty[i], E4M3 ? S::kConvertWarps : 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sh.q_raw[i], 1);
            mbar_init(&sh.s_full[i], 1);
            mbar_init(&sh.p_full[i][0], 4);
            mbar_init(&sh.p_full[i][1], 4);
            mbar_init(&sh.pv_half[i], 1);
            mbar_init(&sh.pv_done[i], 1);
            mbar_init(&sh.q_full[i], E4M3 ? 4 : 1);
            mbar_init(&sh.q_empty[i], 1);
        }
        for (int i = 0; i < 4; ++i) {
            mbar_init(&sh.key_full[i], 1);
            mbar_init(&sh.key_empty[i], S::kSoftmaxWarps + S::kConvertWarps);
        }
        for (int i = 0; i < kUnits; ++i) {
            mbar_init(&sh.unit_full[i], 1);
            mbar_init(&sh.unit_empty[i], kThreads / 32 - 1);
        }
        mbar_init(&sh.tail, 1);
        mbar_init(&sh.drained, 1);
#ifdef PLDP_TEST_STUCK_SCORES
        mbar_init(&sh.never, 1);
#endif
        fence_mbar_init();
        sh.dead = 0;
        sh.zeros = 0;
    }
    pdl_enter();
    __syncthreads();

    // the list: every thread counts the costs of a strip of sequences
    {
        const int strip = (a.B + kThreads - 1) / kThreads;
        const int lo = min(a.B, static_cast<int>(threadIdx.x) * strip), hi = min(a.B, lo + strip);
        long long mine = 0;
#pragma unroll 1
        for (int b = lo; b < hi; ++b) {
            uint32_t st;
            const PackedRows p = packed_rows(a.rows, a.start, b, a.R, c.capacity, st);
            if (st && blockIdx.x == 0 && a.status) atomicOr(a.status + b, st);
            if (p.count < p.given) sh.zeros = 1;
            if (p.count == 0) continue;
            const Units s = units_of(p, a.group);
            mine += c.heads * cost_before<UR>(s, unit_count<UR>(s));
        }
        long long upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long t = __shfl_up_sync(0xFFFFFFFFu, upto, o);
            if (lane >= o) upto += t;
        }
        if (lane == 31) sh.warp_sum[warp] = upto;
        __syncthreads();
        long long total = 0;
#pragma unroll 1
        for (int w = 0; w < kThreads / 32; ++w) {
            if (w == warp) upto += total;
            total += sh.warp_sum[w];
        }
        // equal parts; the first `extra` CTAs take one more than the others
        const long long most = quotient(total + kLeast - 1, kLeast);
        const int ctas = static_cast<int>(most < gridDim.x ? most : gridDim.x);
        const long long each = ctas ? quotient(total, ctas) : 0, extra = ctas ? total - each * ctas : 0;
        const long long g0 = each * blockIdx.x + min(static_cast<long long>(blockIdx.x), extra);
        const long long g1 = g0 + each + (blockIdx.x < extra ? 1 : 0);
        long long before = upto - mine;
        if (blockIdx.x < ctas && before <= g0 && g0 < before + mine) {              // one thread's
#pragma unroll 1
            for (int b = lo;; ++b) {
                uint32_t st;
                const Units s = units_of(packed_rows(a.rows, a.start, b, a.R, c.capacity, st), a.group);
                if (s.N == 0) continue;
                const int units = unit_count<UR>(s);
                const long long per = strip == 1 ? quotient(mine, c.heads) : cost_before<UR>(s, units);
                if (g0 >= before + per * c.heads) {
                    before += per * c.heads;
                    continue;
                }
                const int kv = static_cast<int>(quotient(g0 - before, per));
                int64_t at;
                sh.unit = unit_at<UR>(s, units, g0 - before - kv * per, &at);
                sh.b = b, sh.kv = kv;
                sh.in = static_cast<int>(g0 - before - kv * per - at);
                sh.at = g0, sh.count = g1 - g0;
                break;
            }
        }
        if (threadIdx.x == 0) {
            sh.each = each, sh.extra = extra;
            if (blockIdx.x >= ctas) sh.count = 0;
        }
    }
    tmem_before_sync();
    __syncthreads();
    tmem_after_sync();
    const uint32_t tmem = sh.tmem;
    // The query warp works the units out for all: the sequence's rows, divisions and the cut, which every role would fetch
    // code for and wait for loads for at every unit.
    PromptUnit w;
    int unit_no = 0;
    // Whether a wait has run out, as all lanes of a warp see it together: another warp may set it between their looks, and lanes
    // that left a loop alone would be waited for by the rest at the next vote.
    auto given_up = [&] { return __any_sync(0xFFFFFFFFu, *static_cast<volatile int*>(&sh.dead)); };
    auto next_unit = [&] {
        wait_for(&sh.unit_full[unit_no % kUnits], unit_no / kUnits, &sh.dead);
        if (given_up()) return false;
        w = sh.units[unit_no % kUnits];
        return w.T > 0;
    };
    auto unit_done = [&] {
        __syncwarp();
        mbar_arrive_if(&sh.unit_empty[unit_no % kUnits], lane == 0);
        ++unit_no;
    };
    if (sh.zeros) {
        // tokens that take no part: their rows, of all heads
#pragma unroll 1
        for (int b = 0; b < a.B; ++b) {
            uint32_t st;
            const PackedRows p = packed_rows(a.rows, a.start, b, a.R, c.capacity, st);
            const int64_t heads = a.q_heads, chunks = D / 8, items = (p.given - p.count) * heads * chunks;
            for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < items; i += static_cast<int64_t>(gridDim.x) * kThreads) {
                const int64_t vec = i / chunks, row = p.row + p.count + vec / heads, h = vec % heads;
                *reinterpret_cast<uint4*>(a.out + row * a.o_tok + h * a.o_head + (i - vec * chunks) * 8) = make_uint4(0u, 0u, 0u, 0u);
                if (i == vec * chunks && a.lse) a.lse[row * heads + h] = -INFINITY;
            }
        }
    }

    if (warp >= S::kMmaWarp && warp < S::kConvertWarp) {
    if constexpr (NQ == 2) fewer_registers<S::kOtherRegs>();
    // bf16: a warp the keys and one the values (issuing bounds small pages: 16 positions, heads of 128, 8192 tokens 519 us with
    // one warp); where the queries need a warp for each tile of rows, one warp both
    const bool two_copy = !E4M3 && (NQ == 1 || a.q_boxes);
    if (warp == S::kCopyWarp || (two_copy && warp == S::kKeyWarp)) {
        // ---- copies: keys and values in turn, a box (positions of one page) at a time ----
        static_assert(E4M3 || S::kSlots % 2 == 0, "a slot is the keys' or the values'");
        const int first_kv = warp == S::kCopyWarp ? 0 : 1, last_kv = two_copy ? first_kv : 1;
        constexpr int kDepth = E4M3 ? S::kStages : S::kSlots, kParts = E4M3 ? kTile / S::kStageRows : 1, kPartRows = kTile / kParts;
        const uint32_t lead = elect_lane();
        uint64_t* const arrived = E4M3 ? sh.stage_full : sh.full;
        uint64_t* const left = E4M3 ? sh.stage_empty : sh.empty;
        const int boxes = kTile / a.box, part_boxes = kPartRows / a.box;
        int e = 0, tile_no = 0, tails = 0;
        bool on = true;
#pragma unroll 1
        while (on && next_unit()) {
            const int32_t* table = c.pages + w.b * c.pages_stride;
            // the page of box `box` of a tile; those of the next tile, a box a lane, are asked for before this one's
            // copies (pages that 4 does not divide have more boxes than lanes)
            auto look = [&](int tile, int box) {
                const int pos = tile * kTile + box * a.box;
                return tile < w.t1 && box < boxes && pos < w.end ? load_now(table + page_of(pos, c.div_mul, c.div_shift)) : 0;
            };
            int page = look(w.t0, lane);
#pragma unroll 1
            for (int tile = w.t0; on && tile < w.t1; ++tile, ++tile_no) {
                const bool tail = !E4M3 && tile * kTile + kTile > w.end;
                const int page_ahead = look(tile + 1, lane);
#pragma unroll 1
                for (int part = 0; on && part < 2 * kParts; ++part, ++e) {
                    const int kv = part / kParts, first = part % kParts * part_boxes;
                    // boxes that hold a position of the sequence
                    const int full = max(0, min(part_boxes, (w.end - tile * kTile + a.box - 1) / a.box - first));
                    const CUtensorMap* map = kv ? &v_map : &k_map;
                    const int at = e % kDepth;
                    if (kv < first_kv || kv > last_kv) continue;
                    if (e >= kDepth) wait_for(&left[at], e / kDepth - 1, &sh.dead);
                    on = !given_up();
                    if (!on) break;
                    uint64_t* const bar = tail && kv ? &sh.tail : &arrived[at];
                    // (bf16 keys: behind their flags of missing pages, which the softmax reads once the scores are there; until
                    // this arrival the phase stays open, whatever has been copied)
                    const bool flags = !E4M3 && kv == 0;
                    auto arrive = [&] {
                        if (lane == 0) mbar_arrive_expect_tx(bar, full * a.box * (E4M3 ? a.pitch : S::kPanels * 128));
                        __syncwarp();
                    };
                    if (!flags) arrive();
                    uint8_t* dst = E4M3 ? stages + at * S::kStage : ring + at * S::kSlot;
                    bool hole = false;
                    // issued one after the other by the lane that leads: a branch around the copy would make every
                    // operand one lane's
#pragma unroll 1
                    for (int b0 = 0; b0 < full; b0 += 32) {
                        const int box = first + b0 + lane, pos = tile * kTile + box * a.box;
                        const int slot = pos - static_cast<int>(page_of(pos, c.div_mul, c.div_shift)) * c.page_size;
                        int pg = boxes <= 32 ? __shfl_sync(0xFFFFFFFFu, page, box & 31) : look(tile, box);
                        if (static_cast<unsigned>(pg) >= static_cast<unsigned>(c.n_pages)) {
                            pg = c.n_pages;                                // outside the tensor: zeros
                            hole = hole || b0 + lane < full;
                        }
                        const int count = min(32, full - b0);
                        // (several at once: a box's way from its lanes to the copy is a chain of some 100 cycles.  8192 tokens, heads of
                        // 128, pages of 8: 454 us one at a time, 411 with two, 382 with four (392 with the keys' arrival behind the boxes), 376 with
                        // eight, of which 24 short prompts in pages of 32 take 118 us for 114; e4m3: 698, 638, 566, and 142, 144 and 151
                        // there, as code crowds the instruction cache)
                        if (S::kPanels == 4 && !E4M3 && a.whole) {
#pragma unroll 8
                            for (int i = 0; i < count; ++i) {
                                const int i_slot = __shfl_sync(0xFFFFFFFFu, slot, i), i_pg = __shfl_sync(0xFFFFFFFFu, pg, i);
                                tma_box5_if(dst + (b0 + i) * a.box * (S::kPanels * 128), map, a.whole == 1 ? w.kv * S::kPanels : 0,
                                            (a.whole == 1 ? 0 : w.kv * (c.page_size >> 3)) + (i_slot >> 3), i_pg, bar, lead);
                            }
                        } else {
#pragma unroll (E4M3 ? DP == 256 ? 4 : 2 : S::kPanels == 4 ? 1 : 4)
                            for (int i = 0; i < count; ++i) {
                                const int i_slot = __shfl_sync(0xFFFFFFFFu, slot, i), i_pg = __shfl_sync(0xFFFFFFFFu, pg, i);
                                const int c1 = a.head_first ? w.kv : i_slot, c2 = a.head_first ? i_slot : w.kv;
                                if constexpr (E4M3) {
                                    tma_box_if(dst + (b0 + i) * a.box * a.pitch, map, 0, c1, c2, i_pg, bar, lead);
                                } else {
#pragma unroll
                                    for (int p = 0; p < S::kPanels; ++p)
                                        tma_box_if(dst + p * (kTile * 128) + (b0 + i) * a.box * 128, map, p * 64, c1, c2, i_pg, bar, lead);
                                }
                            }
                        }
                    }
                    if (flags) {
                        hole = __any_sync(0xFFFFFFFFu, hole);
                        if (hole) {
#pragma unroll 1
                            for (int i = 0; i < 4; ++i) {
                                const int pos = tile * kTile + 32 * i + lane;
                                const int pg = pos < w.end ? __ldg(table + page_of(pos, c.div_mul, c.div_shift)) : 0;
                                const uint32_t bits = __ballot_sync(0xFFFFFFFFu, static_cast<unsigned>(pg) < static_cast<unsigned>(c.n_pages));
                                if (lane == 0) sh.live[tile_no % kAhead][i] = bits;
                            }
                            if (lane == 0 && a.status) atomicOr(a.status + w.b, PLDP_ST_PAGE);
                        }
                        if (lane == 0) sh.holes[tile_no % kAhead] = hole;
                        arrive();
                    }
                    if (tail && kv) {
                        // what the pages hold past the end is not used: zeros, in the values' tile
                        const int group_step = S::kPanels == 4 ? a.group_step : 1024, panel_step = S::kPanels == 4 ? a.panel_step : kTile * 128;
                        wait_for(&sh.tail, tails, &sh.dead);
                        ++tails;
#pragma unroll 1
                        for (int r = w.end - tile * kTile; r < kTile; ++r)
#pragma unroll 1
                            for (int p = lane; p < 8 * S::kPanels; p += 32)
                                *reinterpret_cast<uint4*>(dst + (p >> 3) * panel_step + (r >> 3) * group_step + (r & 7) * 128 + (p & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
                        fence_smem_async();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&arrived[at]);
                    }
                    __syncwarp();
                }
                page = page_ahead;
            }
            unit_done();
        }
        // the last copy into each place arrives before this CTA ends, whether or not its reader has waited for it
        if (lane < kDepth) {
            const int x = e - 1 - ((e - 1 - lane) % kDepth + kDepth) % kDepth;
            if (x >= 0 && (!two_copy || (x & 1) == first_kv)) mbar_wait(&arrived[lane], (x / kDepth) & 1, kMbarPolls);
        } else if (lane == 31 && tails > 0) {
            mbar_wait(&sh.tail, (tails - 1) & 1, kMbarPolls);
        }
    } else if (warp == S::kQueryWarp || (!E4M3 && warp == S::kKeyWarp)) {
        // ---- queries of the next unit, as soon as the last scores of this one are done; those without boxes of bf16: a tile of rows a warp ----
        const uint32_t lead = elect_lane();
        int seg0 = 0, seg1 = 0;
        auto queries = [&](int q) {
            if (q * 128 >= w.rows) return;
            int& seg = q ? seg1 : seg0;
            if (seg > 0) wait_for(&sh.q_empty[q], seg - 1, &sh.dead);
            if (given_up()) return;
            uint64_t* const bar = E4M3 ? &sh.q_raw[q] : &sh.q_full[q];
            uint8_t* const to = q_smem + q * (S::kPanels * 128 * 128);
            const uint32_t first = static_cast<uint32_t>(w.r0) + q * 128, group = a.group;
            if (a.q_boxes) {
                // whole tokens: boxes of their heads (what lies behind the sequence's rows is not used)
                if (lane == 0) mbar_arrive_expect_tx(bar, S::kPanels * 128 * 128);
                __syncwarp();
#pragma unroll
                for (int p = 0; p < S::kPanels; ++p)
                    tma_box_if(to + p * (128 * 128), &q_map, p * 64, w.kv * a.group, w.row + static_cast<int>(page_of(first, a.group_mul, a.group_shift)), 0, bar, lead);
            } else {
                // all of the tile's pieces of 16 bytes are asked for before the first is waited for
                constexpr int kLanes = DP / 8, kAt = 32 / kLanes;          // lanes a row, and rows at once
                const int piece = lane % kLanes;
                const bool in = piece * 8 < D;
                uint8_t* const mine = to + (piece >> 3) * (128 * 128);
                uint32_t tok = (first + lane / kLanes) / group, h = first + lane / kLanes - tok * group;
                const __nv_bfloat16* from = a.q + w.row * a.q_tok + static_cast<int64_t>(w.kv) * a.group * a.q_head + piece * 8;
#pragma unroll 2
                for (int row = lane / kLanes; row < 128; row += kAt) {
                    const bool there = in && q * 128 + row < w.rows;
                    copy_or_zeros(mine + row * 128 + (((piece & 7) ^ (row & 7)) << 4), there ? from + tok * a.q_tok + h * a.q_head : a.q, there);
                    h += kAt;
                    while (h >= group) h -= group, ++tok;
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
                asm volatile("cp.async.wait_group 0;" ::: "memory");
                if (!E4M3 && a.flip) {
                    // (each lane its own pieces)
#pragma unroll 1
                    for (int row = lane / kLanes; row < 128; row += kAt) {
                        uint4* const at = reinterpret_cast<uint4*>(mine + row * 128 + (((piece & 7) ^ (row & 7)) << 4));
                        uint4 x = *at;
                        x.x ^= a.flip, x.y ^= a.flip, x.z ^= a.flip, x.w ^= a.flip;
                        *at = x;
                    }
                }
                if constexpr (!E4M3) fence_smem_async();
                __syncwarp();
                mbar_arrive_if(bar, lane == 0);
            }
            ++seg;
        };
        auto tile_rows = [&](int from, int to) {
#pragma unroll 1
            for (int q = from; q < to; ++q) queries(q);
        };
        if (warp == S::kQueryWarp) {
            PromptWalk<UR> walk;
            walk.b = sh.b, walk.kv = sh.kv, walk.unit = sh.unit, walk.at = sh.at, walk.left = sh.count;
            walk.pre = max(0, kUnitCost - sh.in), walk.t0 = max(0, sh.in - kUnitCost);
            bool more = walk.left > 0;
            bool ended = false;
            int ahead = 0;
#pragma unroll 1
            while (true) {
                // units are three ahead of their queries, which wait for the last ones' scores
#pragma unroll 1
                for (; !ended && ahead <= unit_no + 3; ++ahead) {
                    if (ahead >= kUnits) wait_for(&sh.unit_empty[ahead % kUnits], ahead / kUnits - 1, &sh.dead);
                    // (after a wait that ran out a place may still be read: half of one unit and half of another would put
                    // results anywhere)
                    if (given_up()) break;
                    if (more) more = ahead == 0 ? walk.first(a, sh.in) : walk.next(a);
                    PromptUnit u = {};
                    if (more) {
                        u = {walk.b, walk.kv, walk.p.row, walk.s.start, walk.end, static_cast<int>(walk.r0), walk.rows, walk.t0, walk.t1, walk.T, 0, 0};
                        if (walk.t0 == 0 && walk.t1 < walk.T) {
                            const long long last = walk.at + walk.pre + walk.T - 1, edge = (sh.each + 1) * sh.extra;
                            u.last_cta = static_cast<int>(last < edge ? last / (sh.each + 1) : sh.extra + (last - edge) / sh.each);
                        }
                        walk.step(a);
                    } else {
                        ended = true;
                    }
                    if (lane == 0) sh.units[ahead % kUnits] = u;
                    __syncwarp();
                    mbar_arrive_if(&sh.unit_full[ahead % kUnits], lane == 0);
                }
                w = sh.units[unit_no % kUnits];
                ++unit_no;
                if (w.T == 0 || given_up()) break;
                tile_rows(0, NQ == 2 && (E4M3 || a.q_boxes) ? 2 : 1);
            }
        } else {
#pragma unroll 1
            while (next_unit()) {
                tile_rows(1, 2);
                unit_done();
            }
        }
        // boxes that nothing has waited for arrive before this CTA ends
        const int last = lane ? seg1 : seg0;
        if (a.q_boxes && lane < NQ && last > 0) mbar_wait(E4M3 ? &sh.q_raw[lane] : &sh.q_full[lane], (last - 1) & 1, kMbarPolls);
    } else if (warp == S::kKeyWarp) {
        // ---- e4m3: the scales of each tile, four keys a lane ----
        if constexpr (E4M3) {
            int tile_no = 0, unit = 0;
#pragma unroll 1
            while (next_unit()) {
                const int32_t* table = c.pages + w.b * c.pages_stride;
                const int first = w.start + static_cast<int>(page_of(static_cast<uint32_t>(w.r0), a.group_mul, a.group_shift));
                bool apart = false;
#pragma unroll 1
                for (int tile = w.t0; tile < w.t1; ++tile, ++tile_no) {
                    const int at = tile_no & 3;
                    float f[4], v[4];
                    bool gone[4], hole = false;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int pos = tile * kTile + 4 * lane + i;
                        f[i] = 1.f, v[i] = 0.f;                     // (a masked score stays -infinity by 1, not by 0)
                        gone[i] = false;
                        if (pos < w.end) {
                            const int pg_at = page_of(pos, c.div_mul, c.div_shift), pg = __ldg(table + pg_at);
                            gone[i] = static_cast<unsigned>(pg) >= static_cast<unsigned>(c.n_pages);
                            hole |= gone[i];
                            if (!gone[i]) {
                                const int64_t from = (static_cast<int64_t>(pg) * c.heads + w.kv) * c.page_size + (pos - pg_at * c.page_size);
                                f[i] = __ldg(c.k_scale + from), v[i] = __ldg(c.v_scale + from);
                            }
                        }
                    }
                    // The values' unit 2^unit: above the largest scale of a unit's first tile, and of a later one that passes it.
                    // Of a tile that some rows see in part only the keys count that all of those rows see, and only where it is
                    // the first, so that no row's result depends on later tokens' values; where that leaves a scale too far above
                    // the unit, from there on the weights take the scales.
                    const int all = __reduce_max_sync(0xFFFFFFFFu, exponent_of(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3]))));
                    const int partly = first - tile * kTile;                  // keys up to here: all rows see them that see any
                    if (tile == w.t0 || (all > unit && partly >= kTile - 1)) {
                        const int mine = max(partly, 0) - 4 * lane;
                        unit = min(2 + __reduce_max_sync(0xFFFFFFFFu, exponent_of(fmaxf(fmaxf(mine >= 0 ? v[0] : 0.f, mine >= 1 ? v[1] : 0.f),
                                                                                        fmaxf(mine >= 2 ? v[2] : 0.f, mine >= 3 ? v[3] : 0.f)))), 126);
                    }
                    apart = apart || (all > unit + kAbove && partly < kTile - 1);
                    const float by = power_of_two(-unit);
                    if (tile_no >= 4) wait_for(&sh.key_empty[at], (tile_no >> 2) - 1, &sh.dead);
                    // (keys' scales never 0: scores are divided by them where the weights take the values')
                    *reinterpret_cast<float4*>(&sh.key_scale[at][4 * lane]) = make_float4(fmaxf(f[0], 0x1p-120f), fmaxf(f[1], 0x1p-120f),
                                                                                          fmaxf(f[2], 0x1p-120f), fmaxf(f[3], 0x1p-120f));
                    *reinterpret_cast<float4*>(&sh.value[at][4 * lane]) = make_float4(v[0], v[1], v[2], v[3]);
                    // (codes / 4 are exact)
                    uint32_t h[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float x = apart ? 0.25f : v[i] * by;
                        h[i] = pack_f16(x, x);
                    }
                    *reinterpret_cast<uint4*>(&sh.value_scale[at][4 * lane]) = make_uint4(h[0], h[1], h[2], h[3]);
                    if (lane == 0) sh.unit_of[at] = apart ? kApart : unit;
                    hole = __any_sync(0xFFFFFFFFu, hole);
                    if (hole) {
                        // (this lane's four keys are bits 4 (lane & 7) and on of a word)
                        uint32_t bits = (gone[0] ? 0u : 1u) | (gone[1] ? 0u : 2u) | (gone[2] ? 0u : 4u) | (gone[3] ? 0u : 8u);
                        bits <<= 4 * (lane & 7);
#pragma unroll
                        for (int o = 1; o < 8; o <<= 1) bits |= __shfl_xor_sync(0xFFFFFFFFu, bits, o);
                        if ((lane & 7) == 0) sh.live[tile_no % kAhead][lane >> 3] = bits;
                        if (lane == 0 && a.status) atomicOr(a.status + w.b, PLDP_ST_PAGE);
                    }
                    if (lane == 0) sh.holes[tile_no % kAhead] = hole;
                    __syncwarp();
                    mbar_arrive_if(&sh.key_full[at], lane == 0);
                }
                unit_done();
            }
        }
    } else if (warp == S::kMmaWarp) {
        // ---- matrix instructions ----
        const uint64_t q_op = smem_operand(smem_u32(q_smem), 16, 1024, swizzle_mode(128));
        const int group_step = !E4M3 && S::kPanels == 4 ? a.group_step : 1024, panel_step = !E4M3 && S::kPanels == 4 ? a.panel_step : kTile * 128;
        const uint64_t k_op = smem_operand(smem_u32(ring), 16, group_step, swizzle_mode(128));
        const uint64_t v_op = smem_operand(smem_u32(ring), panel_step, group_step, swizzle_mode(128));
        const uint32_t q_lo = static_cast<uint32_t>(q_op), q_hi = q_op >> 32, k_lo = static_cast<uint32_t>(k_op), k_hi = k_op >> 32;
        const uint32_t v_lo = static_cast<uint32_t>(v_op), v_hi = v_op >> 32;
        constexpr uint32_t kScores = mma_form(128, 128, !E4M3, false, false);
        const uint32_t values = mma_form(128, D, !E4M3, false, true);
        const uint32_t lead = elect_lane();
        int e = 0;                                       // entry of the ring
        int seg0 = 0, seg1 = 0, s_no = 0, p_no0 = 0, p_no1 = 0;      // units and weights of each tile of rows so far, and (of one) scores
        // Two barriers, a lane each: a wait for two costs what one does.
        auto wait_both = [&](uint64_t* x, uint32_t x_parity, uint64_t* y, uint32_t y_parity) {
            uint64_t* const bar = lane == 0 ? x : lane == 1 ? y : nullptr;
            const uint32_t parity = lane == 0 ? x_parity : y_parity;
            bool done = bar == nullptr || over(bar, parity);
            uint32_t polls = 0;
#pragma unroll 1
            while (!__all_sync(0xFFFFFFFFu, done)) {
                if (++polls >= kPolls || given_up()) {
                    *static_cast<volatile int*>(&sh.dead) = 1;
                    break;
                }
                if (!done) done = over(bar, parity);
            }
            __syncwarp();
            tmem_after_sync();
        };
        auto full = [&](int entry) { return &sh.full[entry % S::kSlots]; };
        auto scores = [&](int q, int slot, int at) {     // to place `at`
            const uint32_t op = __shfl_sync(0xFFFFFFFFu, k_lo + slot * (S::kSlot / 16), 0), to = __shfl_sync(0xFFFFFFFFu, tmem + at * 128, 0);
            const uint32_t qo = __shfl_sync(0xFFFFFFFFu, q_lo + q * (S::kPanels * 128 * 128 / 16), 0);
#pragma unroll
            for (int s = 0; s < DP / 16; ++s)
                if (s * 16 < D)
                    mma_f16(to, qo + (s >> 2) * (128 * 8) + (s & 3) * 2, q_hi, op + (s >> 2) * (panel_step / 16) + (s & 3) * 2, k_hi, kScores, s > 0, lead);
            mma_commit(&sh.s_full[at], lead);
        };
        auto sums = [&](int q, int half, int slot, int at, bool more) {
            const uint32_t op = __shfl_sync(0xFFFFFFFFu, v_lo + slot * (S::kSlot / 16), 0), from = __shfl_sync(0xFFFFFFFFu, tmem + at * 128, 0);
            const uint32_t to = __shfl_sync(0xFFFFFFFFu, tmem + S::kO + q * DP, 0);
            if (half == 0) {
#pragma unroll
                for (int s = 0; s < 4; ++s) mma_f16_tmem(to, from + s * 8, op + s * (group_step / 8), v_hi, values, s > 0 || more, lead);
            } else {
#pragma unroll
                for (int s = 4; s < 8; ++s) mma_f16_tmem(to, from + s * 8, op + s * (group_step / 8), v_hi, values, 1u, lead);
            }
        };
        // Of each tile: the product of the first half of its weights, then of the second, then (two tiles of rows) the next
        // tile's scores, whose place the weights have left; one tile of rows has two places in turn for scores, and the
        // next tile's come first.
#pragma unroll 1
        while (next_unit()) {
            const int n = w.t1 - w.t0, nq = w.rows > 128 ? 2 : 1;
#pragma unroll 1
            for (int q = 0; q < nq; ++q) {
                wait_both(q == 0 ? full(e) : nullptr, e / S::kSlots, &sh.q_full[q], q ? seg1 : seg0);
                scores(q, e % S::kSlots, NQ == 2 ? q : s_no++ & 1);
                if (n == 1) mma_commit(&sh.q_empty[q], lead);
            }
            mma_commit(&sh.empty[e % S::kSlots], lead);
#pragma unroll 1
            for (int i = 0; i < n; ++i) {
                const int v = e + 2 * i + 1, k = v + 1, v_slot = v % S::kSlots, k_slot = k % S::kSlots;
                const bool next = i + 1 < n;
                if (NQ == 1 && next) {
                    wait_both(full(k), k / S::kSlots, nullptr, 0);
                    scores(0, k_slot, s_no++ & 1);
                    if (i + 2 == n) mma_commit(&sh.q_empty[0], lead);
                    mma_commit(&sh.empty[k_slot], lead);
                }
#pragma unroll 1
                for (int q = 0; q < nq; ++q) {
                    const int at = NQ == 2 ? q : p_no0 & 1;
                    const uint32_t turn = NQ == 1 ? p_no0 >> 1 : q ? p_no1 : p_no0;
                    wait_both(q == 0 ? full(v) : nullptr, v / S::kSlots, &sh.p_full[at][0], turn);
                    sums(q, 0, v_slot, at, i > 0);
                    mma_commit(&sh.pv_half[q], lead);
                    wait_both(NQ == 2 && next && q == 0 ? full(k) : nullptr, k / S::kSlots, &sh.p_full[at][1], turn);
                    sums(q, 1, v_slot, at, true);
                    if (NQ == 1 || !next) mma_commit(&sh.pv_done[NQ == 1 ? p_no0 & 1 : q], lead);
                    if (q + 1 == nq) mma_commit(&sh.empty[v_slot], lead);
                    if (NQ == 2 && next) {
                        scores(q, k_slot, q);
                        if (i + 2 == n) mma_commit(&sh.q_empty[q], lead);
                        if (q + 1 == nq) mma_commit(&sh.empty[k_slot], lead);
                    }
                }
                ++p_no0;
                if (nq == 2) ++p_no1;
            }
            ++seg0;
            if (nq == 2) ++seg1;
            e += 2 * n;
            unit_done();
        }
        // nothing reads shared memory or writes tensor memory any more when they are given back
        mma_commit(&sh.drained, lead);
        mbar_wait(&sh.drained, 0, kMbarPolls);
    }
    } else if (E4M3 && warp >= S::kConvertWarp) {
        // ---- e4m3: the codes of a tile of keys or values to f16, 16 at a time ----
        if constexpr (E4M3) {
            if constexpr (NQ == 2) fewer_registers<S::kConvertRegs>();
            constexpr int kConvert = S::kConvertWarps * 32, kParts = kTile / S::kStageRows;
            const int t = threadIdx.x - S::kConvertWarp * 32;
            constexpr int kRowChunks = DP / 16, kStepRows = kConvert / kRowChunks, kTurns = S::kStageRows / kStepRows;
            const int chunk = t % kRowChunks, row0 = t / kRowChunks;
            const bool in = chunk * 16 < D, upper = chunk >> 2 & 1;
            static_assert(kStepRows % 8 == 0, "rows");
            const int first = row0 * a.pitch + chunk * 16, step = kStepRows * a.pitch;
            const int line = (chunk >> 2) * (kTile * 128) + row0 * 128;
            const int low = line + ((((chunk & 3) * 2) ^ (row0 & 7)) << 4), high = low ^ 16;
            int e = 0, tile_no = 0;                              // parts, tiles
#pragma unroll 1
            while (next_unit()) {
#pragma unroll 1
                for (int tile = w.t0; tile < w.t1; ++tile, ++tile_no) {
                    const int key_at = tile_no & 3;
#pragma unroll 1
                    for (int part = 0; part < 2 * kParts; ++part, ++e) {
                        const int entry = e / kParts, slot = entry % S::kSlots, stage = e % S::kStages, base = part % kParts * S::kStageRows;
                        const bool values = part >= kParts;
                        const int rows = w.end - tile * kTile - base;           // the rest is zeros
                        const uint8_t* from = stages + stage * S::kStage + first;
                        uint8_t* const to = ring + slot * S::kSlot + base * 128;
                        const bool codes = over(&sh.stage_full[stage], e / S::kStages);
                        const bool room = entry < S::kSlots || over(&sh.empty[slot], entry / S::kSlots - 1);
                        // (waited for before the keys go on, so that the softmax, to which their scores come, need not ask)
                        if (part == 0) wait_for(&sh.key_full[key_at], tile_no >> 2, &sh.dead);
                        wait_more(codes, &sh.stage_full[stage], e / S::kStages, &sh.dead);
                        wait_more(room, &sh.empty[slot], entry / S::kSlots - 1, &sh.dead);
                        if (in) {
                            constexpr int kAtOnce = kTurns < 4 ? kTurns : 4;
#pragma unroll 1
                            for (int turn = 0; turn < kTurns; turn += kAtOnce) {
                                uint4 x[kAtOnce];
#pragma unroll
                                for (int i = 0; i < kAtOnce; ++i, from += step) x[i] = *reinterpret_cast<const uint4*>(from);
                                if (rows < S::kStageRows)
#pragma unroll
                                    for (int i = 0; i < kAtOnce; ++i)
                                        if (row0 + (turn + i) * kStepRows >= rows) x[i] = make_uint4(0u, 0u, 0u, 0u);
                                uint32_t by[kAtOnce];
                                if (values)
#pragma unroll
                                    for (int i = 0; i < kAtOnce; ++i) by[i] = sh.value_scale[key_at][base + row0 + (turn + i) * kStepRows];
#pragma unroll
                                for (int i = 0; i < kAtOnce; ++i) {
                                    uint2 h0 = four_codes(x[i].x), h1 = four_codes(x[i].y), h2 = four_codes(x[i].z), h3 = four_codes(x[i].w);
                                    if (values) {
                                        h0.x = mul_f16x2(h0.x, by[i]), h0.y = mul_f16x2(h0.y, by[i]), h1.x = mul_f16x2(h1.x, by[i]), h1.y = mul_f16x2(h1.y, by[i]);
                                        h2.x = mul_f16x2(h2.x, by[i]), h2.y = mul_f16x2(h2.y, by[i]), h3.x = mul_f16x2(h3.x, by[i]), h3.y = mul_f16x2(h3.y, by[i]);
                                    }
                                    const uint4 a0 = make_uint4(h0.x, h0.y, h1.x, h1.y), a1 = make_uint4(h2.x, h2.y, h3.x, h3.y);
                                    const int at = (turn + i) * (kStepRows * 128);
                                    // (eight neighbours' pieces into all banks: of the second panel the upper one first)
                                    *reinterpret_cast<uint4*>(to + at + (upper ? high : low)) = upper ? a1 : a0;
                                    *reinterpret_cast<uint4*>(to + at + (upper ? low : high)) = upper ? a0 : a1;
                                }
                            }
                        }
                        fence_smem_async();
                        __syncwarp();
                        mbar_arrive_if(&sh.stage_empty[stage], lane == 0);
                        if (part == 2 * kParts - 1) mbar_arrive_if(&sh.key_empty[key_at], lane == 0);
                        if (part % kParts == kParts - 1) mbar_arrive_if(&sh.full[slot], lane == 0);
                    }
                }
                unit_done();
            }
        }
    } else {
        // ---- softmax: a row a thread ----
        if constexpr (NQ == 2) more_registers<S::kSoftmaxRegs>();
        const int q = warp >> 2, quad = warp & 3, j = quad * 32 + lane;
        const uint32_t lanes = static_cast<uint32_t>(quad * 32) << 16, my_o = tmem + lanes + S::kO + q * DP;
        constexpr float kLift = E4M3 ? 7.f : 0.f;       // f16 weights up to 2^15 instead of 2^8: fewer of them vanish
        constexpr float kRoomUp = E4M3 ? 8.f : 64.f;
        int tile_no = 0, mine = 0;                      // tiles of this CTA, and those of this warp's rows
        int seg = 0;                                    // and its units
        bool cut_here = false;
#pragma unroll 1
        while (next_unit()) {
            if (q * 128 >= w.rows) {                    // no rows for these warps
                if constexpr (E4M3)
#pragma unroll 1
                    for (int tile = w.t0; tile < w.t1; ++tile, ++tile_no) {
                        wait_for(&sh.key_full[tile_no & 3], tile_no >> 2, &sh.dead);
                        __syncwarp();
                        mbar_arrive_if(&sh.key_empty[tile_no & 3], lane == 0);
                    }
                else tile_no += w.t1 - w.t0;
                unit_done();
                continue;
            }
            const uint32_t r = static_cast<uint32_t>(w.r0) + q * 128 + j;
            const bool is_row = q * 128 + j < w.rows;
            const uint32_t tok = is_row ? page_of(r, a.group_mul, a.group_shift) : 0u;
            const uint32_t head = is_row ? static_cast<uint32_t>(w.kv) * a.group + (r - tok * a.group) : 0u;
            const int limit = is_row ? w.start + static_cast<int>(tok) : -1;         // last position that the row sees
            // (e4m3: by all rows of the unit, as the values' units go)
            const int seen_by_all = w.start + static_cast<int>(page_of(static_cast<uint32_t>(w.r0) + (E4M3 ? 0 : q * 128), a.group_mul, a.group_shift));
            float m = -INFINITY;                        // (of x, in powers of two)
            [[maybe_unused]] int unit = INT32_MIN;      // the values' in the sums (none yet)
            uint64_t l2 = 0, l3 = 0;
            float f = a.scale2;
            if constexpr (E4M3) {
                // the row's queries, bf16 to f16: its largest element to 2^14..2^15 by a power of two
                wait_for(&sh.q_raw[q], seg, &sh.dead);
                uint8_t* const mine_q = q_smem + q * (S::kPanels * 128 * 128) + j * 128;
                uint32_t most = 0;
                auto piece = [&](int ch) { return reinterpret_cast<uint4*>(mine_q + (ch >> 3) * (128 * 128) + (((ch & 7) ^ (j & 7)) << 4)); };
                // (D / 8 pieces, an even number)
#pragma unroll 1
                for (int c0 = 0; c0 < D / 8; c0 += 4) {
                    uint4 x[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[i] = c0 + i < D / 8 ? *piece(c0 + i) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t v[4] = {x[i].x & 0x7FFF7FFFu, x[i].y & 0x7FFF7FFFu, x[i].z & 0x7FFF7FFFu, x[i].w & 0x7FFF7FFFu};
#pragma unroll
                        for (int k = 0; k < 4; ++k) most = __vmaxu2(most, v[k]);
                    }
                }
                const int ex = static_cast<int>(max(most & 0xFFFFu, most >> 16) >> 7);
                const int up = ex == 0 || ex == 255 ? 0 : min(14 - (ex - 127), 120);
                const float lift = __uint_as_float((static_cast<uint32_t>(up + 127) << 23) ^ (a.flip & 0x80000000u));
                // (never 0, so that a masked score stays -infinity: what is left of so small a scale moves no weight)
                f = fmaxf(f * __uint_as_float(static_cast<uint32_t>(127 - up) << 23), 0x1p-126f);
#pragma unroll 1
                for (int c0 = 0; c0 < D / 8; c0 += 4) {
                    uint4 x[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[i] = c0 + i < D / 8 ? *piece(c0 + i) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t v[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            v[k] = pack_f16(__uint_as_float(v[k] << 16) * lift, __uint_as_float(v[k] & 0xFFFF0000u) * lift);
                        if (c0 + i < D / 8) *piece(c0 + i) = make_uint4(v[0], v[1], v[2], v[3]);
                    }
                }
                fence_smem_async();
                __syncwarp();
                mbar_arrive_if(&sh.q_full[q], lane == 0);
            }
            [[maybe_unused]] const float scale_f = f;
            uint64_t f2 = pack_f32x2(f, f);
#pragma unroll 1
            for (int tile = w.t0; tile < w.t1; ++tile, ++tile_no, ++mine) {
                const int at = NQ == 2 ? q : mine & 1;
                const uint32_t s_at = tmem + lanes + at * 128;
                const uint32_t s_turn = NQ == 2 ? mine : mine >> 1;
                [[maybe_unused]] const int k_at = tile_no & 3;
#ifdef PLDP_TEST_STUCK_SCORES
                wait_for(&sh.never, 0, &sh.dead);
#endif
                wait_for(&sh.s_full[at], s_turn, &sh.dead);
                __syncwarp();
                tmem_after_sync();
                const bool masked = tile * kTile + kTile - 1 > seen_by_all;
                const bool holes = sh.holes[tile_no % kAhead];
                // (asked for here: at the end of each half it would be waited for, 566 us for 542)
                [[maybe_unused]] int now = E4M3 ? sh.unit_of[k_at] : 0;
                if (masked || holes) {
                    // scores of keys that the row does not see become -infinity where they are (code that is seldom run is
                    // kept short: it is fetched anew every time)
#pragma unroll 1
                    for (int i = 0; i < kTile; i += 16) {
                        const int most = limit - tile * kTile - i;                    // keys up to here
                        uint32_t bits = most >= 15 ? 0xFFFFu : most < 0 ? 0u : (2u << most) - 1u;
                        if (holes) bits &= sh.live[tile_no % kAhead][i >> 5] >> (i & 16);
                        if (!__any_sync(0xFFFFFFFFu, (bits & 0xFFFFu) != 0xFFFFu)) continue;
                        float y[16];
                        tmem_load(s_at + i, y);
#pragma unroll
                        for (int k = 0; k < 16; ++k)
                            if (!(bits >> k & 1u)) y[k] = -INFINITY;
                        tmem_store8(s_at + i, y);
                        tmem_store8(s_at + i + 8, y + 8);
                    }
                    tmem_store_wait();
                    if constexpr (E4M3)
                        if (now == kApart) {
                            if (NQ == 1 && tile > w.t0) wait_for(&sh.pv_done[(mine - 1) & 1], (mine - 1) >> 1, &sh.dead);
                            const ApartRow x = apart_tile<DP>(s_at, my_o, sh.key_scale[k_at], sh.value[k_at], scale_f, tile > w.t0,
                                                              {m, (lo_f32(l2) + hi_f32(l2)) + (lo_f32(l3) + hi_f32(l3)), unit});
                            m = x.m, l2 = pack_f32x2(x.l, 0.f), l3 = 0, unit = now = x.unit;
                            f = 1.f, f2 = pack_f32x2(1.f, 1.f);
                        }
                }
                // Keys in two halves: the first's weights are in the product while the second's are taken.
#pragma unroll 1
                for (int half = 0; half < 2; ++half) {
                    float y[64];
                    tmem_load(s_at + half * 64, y);
                    // The weights with the m that there is, while the maximum is found; where m has to move, which it hardly
                    // ever does, they are taken again.
                    uint32_t p[32];
                    uint64_t s2, s3;
                    bool again = false;
#pragma unroll 1
                    while (true) {
                        const float less = m == -INFINITY ? 0.f : kLift - m;
                        const uint64_t less2 = pack_f32x2(less, less);
                        float t0 = -INFINITY, t1 = -INFINITY;
                        s2 = l2, s3 = l3;
#pragma unroll
                        for (int i = 0; i < 64; i += 4) {
                            uint64_t x0 = pack_f32x2(y[i], y[i + 1]), x1 = pack_f32x2(y[i + 2], y[i + 3]);
                            if constexpr (E4M3) {
                                const float4 k = *reinterpret_cast<const float4*>(&sh.key_scale[k_at][half * 64 + i]);
                                x0 = mul_f32x2(x0, pack_f32x2(k.x, k.y)), x1 = mul_f32x2(x1, pack_f32x2(k.z, k.w));
                            }
                            const uint64_t e0 = ordered_fma2(x0, f2, less2), e1 = ordered_fma2(x1, f2, less2);
                            const float p0 = ordered_ex2(lo_f32(e0)), p1 = ordered_ex2(hi_f32(e0));
                            t0 = ordered_max3(t0, lo_f32(x0), hi_f32(x0)), t1 = ordered_max3(t1, lo_f32(x1), hi_f32(x1));
                            const float p2 = ordered_ex2(lo_f32(e1)), p3 = ordered_ex2(hi_f32(e1));
                            s2 = ordered_add2(s2, pack_f32x2(p0, p1));
                            s3 = ordered_add2(s3, pack_f32x2(p2, p3));
                            p[i / 2] = E4M3 ? ordered_f16(p0, p1) : ordered_bf16(p0, p1);
                            p[i / 2 + 1] = E4M3 ? ordered_f16(p2, p3) : ordered_bf16(p2, p3);
                        }
                        if (again) break;
                        float top = fmaxf(t0, t1);
                        top = top > -INFINITY ? top * f : top;
                        const bool up = top > m + kRoomUp || (m == -INFINITY && top > -INFINITY);
                        if (!__any_sync(0xFFFFFFFFu, up) && (!E4M3 || now == unit)) break;
                        again = true;
                        float by = 1.f;
                        if (up) {
                            by = m == -INFINITY ? 0.f : ex2(m - top);
                            m = top;
                        }
                        l2 = mul_f32x2(l2, pack_f32x2(by, by)), l3 = mul_f32x2(l3, pack_f32x2(by, by));
                        if constexpr (E4M3) {
                            if (now != unit && tile > w.t0) by *= power_of_two(max(unit - now, -126));
                            unit = now;
                        }
                        if (tile > w.t0 || half) {
                            // (Of two tiles of rows the scores came behind the last tile's product.  Of one they came behind
                            // that of the one before, and the last one's may be over or not: a barrier for every other tile,
                            // as one asked for a phase that is two ahead or behind answers wrongly.)
                            if (NQ == 1 && tile > w.t0) wait_for(&sh.pv_done[(mine - 1) & 1], (mine - 1) >> 1, &sh.dead);
                            if (half) wait_for(&sh.pv_half[q], mine, &sh.dead);
                            __syncwarp();
                            tmem_after_sync();
#pragma unroll 1
                            for (int i = 0; i < DP; i += 8) {
                                float o[8];
                                tmem_load(my_o + i, o);
#pragma unroll
                                for (int k = 0; k < 8; ++k) o[k] *= by;
                                tmem_store8(my_o + i, o);
                            }
                            tmem_store_wait();
                        }
                    }
                    l2 = s2, l3 = s3;
                    tmem_store32(s_at + half * 32, p);
                    tmem_store_wait();
                    tmem_before_sync();
                    __syncwarp();
                    mbar_arrive_if(&sh.p_full[at][half], lane == 0);
                }
                if constexpr (E4M3) mbar_arrive_if(&sh.key_empty[k_at], lane == 0);
            }
            // ---- the unit's end ----
            if constexpr (NQ == 1) wait_for(&sh.pv_done[(mine - 1) & 1], (mine - 1) >> 1, &sh.dead);
            else wait_for(&sh.pv_done[q], seg, &sh.dead);
            __syncwarp();
            tmem_after_sync();
            const float l = (lo_f32(l2) + hi_f32(l2)) + (lo_f32(l3) + hi_f32(l3));
            const bool whole = w.t0 == 0 && w.t1 == w.T;
            // (l 0: a row that sees nothing; NaN: a query that holds it)
            const float inverse = l == 0.f ? 0.f : (E4M3 ? power_of_two(unit) : 1.f) / l;
            if (whole) {
                const int64_t row = w.row + static_cast<int64_t>(tok);
                if (is_row && a.lse) a.lse[row * a.q_heads + head] = l == 0.f ? -INFINITY : (log2f(l) + m - kLift) * 0.69314718055994531f;
                // kOutBytes of each of the warp's 32 rows at a time: a row a lane into shared memory, whole pieces of rows out of it
                constexpr int kCols = S::kOutBytes / 2, kPieces = kCols / 8, kAt = 32 / kPieces;
                uint8_t* const room = out_smem + warp * (32 * S::kOutBytes);
                const int wrows = w.rows - q * 128 - quad * 32, piece = lane % kPieces;
                const int64_t at_out = row * a.o_tok + static_cast<int64_t>(head) * a.o_head;
#pragma unroll 1
                for (int i = 0; i < D; i += kCols) {
                    // (e4m3, where more roles share the instruction cache: short code; bf16: 111 us for 24 short prompts, heads of
                    // 128, with 64 columns at once, 114 with 16; e4m3, heads of 64: 151 and 145)
                    constexpr int kLoad = E4M3 ? 16 : kCols;
#pragma unroll 1
                    for (int k = 0; k < kCols; k += kLoad) {
                        float o[kLoad];
                        tmem_load(my_o + i + k, o);
#pragma unroll
                        for (int h = 0; h < kLoad; h += 8)
                            *reinterpret_cast<uint4*>(room + lane * S::kOutBytes + (((k + h) / 8 ^ (lane & (kPieces - 1))) << 4)) =
                                make_uint4(pack_bf16(o[h] * inverse, o[h + 1] * inverse), pack_bf16(o[h + 2] * inverse, o[h + 3] * inverse),
                                           pack_bf16(o[h + 4] * inverse, o[h + 5] * inverse), pack_bf16(o[h + 6] * inverse, o[h + 7] * inverse));
                    }
                    __syncwarp();
#pragma unroll (E4M3 ? 2 : 4)
                    for (int k = 0; k < kPieces; ++k) {
                        const int rr = k * kAt + lane / kPieces;
                        const int64_t to = __shfl_sync(0xFFFFFFFFu, at_out, rr) + i + piece * 8;
                        const uint4 y = *reinterpret_cast<const uint4*>(room + rr * S::kOutBytes + ((piece ^ (rr & (kPieces - 1))) << 4));
                        if (rr < wrows && i + piece * 8 < D) *reinterpret_cast<uint4*>(a.out + to) = y;
                    }
                    __syncwarp();
                }
            } else {
                // (which of this CTA's two places: the unit began in another's part, or in this one's.  Averages, as sums of values
                // near fp32's largest pass it)
                float* part = a.parts + static_cast<int64_t>(2 * blockIdx.x + (w.t0 == 0 ? 1 : 0)) * prompt_part(DP) + q * 128 * (DP + 2);
#pragma unroll 1
                for (int i = 0; i < D; i += 16) {
                    float o[16];
                    tmem_load(my_o + i, o);
#pragma unroll
                    for (int k = 0; k < 16; ++k) o[k] *= inverse;
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        *reinterpret_cast<float4*>(part + ((i / 4 + k) * 128 + j) * 4) = make_float4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]);
                    __syncwarp();
                }
                part[128 * DP + j] = l == 0.f ? -INFINITY : m == -INFINITY ? 0.f : m - kLift;            // (of NaN a number, so that it counts)
                part[128 * DP + 128 + j] = l;
                if (w.t0 == 0) cut_here = true;
                if (w.t0 == 0 && threadIdx.x == 0)
                    a.cuts[blockIdx.x] = {w.last_cta - static_cast<int>(blockIdx.x) + 1, static_cast<int>(blockIdx.x), w.r0, w.rows, w.row, w.kv};
            }
            tmem_before_sync();
            ++seg;
            unit_done();
        }
        if (threadIdx.x == 0 && !cut_here) a.cuts[blockIdx.x].parts = 0;
        if (sh.dead && a.status)
#pragma unroll 1
            for (int b = threadIdx.x; b < a.B; b += S::kSoftmaxWarps * 32) atomicOr(a.status + b, PLDP_ST_TIMEOUT);
    }
    tmem_before_sync();
    __syncthreads();
    if (warp == S::kMmaWarp) {
        tmem_after_sync();
        tmem_free(tmem, 512);
    }
}

template <int DP, bool E4M3>
cudaError_t launch_prompt(const PromptArgs& a, const PromptMaps& m, int ctas, cudaStream_t s) {
    using Shape = PromptShape<DP, E4M3>;
    const cudaError_t e = cudaFuncSetAttribute(prompt_kernel<DP, E4M3>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape::kBytes);
    if (e != cudaSuccess) return e;
    // what the warps take must be what the block was launched with: more would be waited for without end
    static const int regs = [] {
        cudaFuncAttributes attr;
        return cudaFuncGetAttributes(&attr, prompt_kernel<DP, E4M3>) == cudaSuccess ? attr.numRegs : 0;
    }();
    constexpr int kSplit = (Shape::kSoftmaxWarps * Shape::kSoftmaxRegs + 4 * Shape::kOtherRegs + Shape::kConvertWarps * Shape::kConvertRegs) * 32;
    if (Shape::kQ == 2 && regs * Shape::kThreads < kSplit) return cudaErrorLaunchOutOfResources;
    return launch_pdl(prompt_kernel<DP, E4M3>, dim3(ctas), dim3(Shape::kThreads), Shape::kBytes, s, 0, a, m.pool.k, m.pool.v, m.q);
}
template <bool E4M3>
cudaError_t launch_prompt_dims(const PromptArgs& a, const PromptMaps& m, int ctas, cudaStream_t s) {
    const int dp = prompt_dim(a.c.head_dim);
    return dp == 64 ? launch_prompt<64, E4M3>(a, m, ctas, s) : dp == 128 ? launch_prompt<128, E4M3>(a, m, ctas, s) : launch_prompt<256, E4M3>(a, m, ctas, s);
}

}  // namespace
}  // namespace pldp
