// The paged cache around a step: pldp_cache_append and pldp_cache_read.
#include <cuda_fp8.h>
#include <math.h>

#include "pldp_cache.cuh"

namespace pldp {

pldp_status check_rows(const char* fn, const char* name, const void* p, const int64_t* strides, size_t es) {
    if (!aligned16(p)) return fail(PLDP_ERR_INVALID_ARG, "%s: %s is not 16-byte aligned", fn, name);
    const int64_t v = static_cast<int64_t>(16 / es);
    for (int i = 0; i < 3; ++i)
        if (strides[i] < 0 || strides[i] % v)
            return fail(PLDP_ERR_INVALID_ARG, "%s: %s strides must be multiples of 16 bytes", fn, name);
    return PLDP_OK;
}

pldp_status cache_view(const char* fn, const pldp_cache& c, int B, CacheView* out) {
    if (c.dtype != PLDP_BF16 && c.dtype != PLDP_E4M3)
        return fail(PLDP_ERR_UNSUPPORTED, "%s: cache dtype %d", fn, static_cast<int>(c.dtype));
    if (c.heads < 1 || c.heads > 1024 || c.head_dim < 16 || c.head_dim > kMaxHeadDim || c.head_dim % 16)
        return fail(PLDP_ERR_UNSUPPORTED, "%s: %d cache heads of %d (1..1024 heads, a multiple of 16 up to %d)", fn,
                    c.heads, c.head_dim, kMaxHeadDim);
    if (c.n_pages < 1 || c.page_size < 1 || c.max_pages < 1 || c.pages_stride < c.max_pages)
        return fail(PLDP_ERR_INVALID_ARG, "%s: n_pages, page_size and max_pages must be >= 1, pages_stride >= max_pages", fn);
    const int64_t capacity = static_cast<int64_t>(c.max_pages) * c.page_size;
    if (capacity > INT32_MAX) return fail(PLDP_ERR_INVALID_ARG, "%s: max_pages * page_size must be below 2^31", fn);
    const int es = c.dtype == PLDP_BF16 ? 2 : 1;
    const int64_t strides[3] = {c.page_stride, c.pos_stride, c.head_stride};
    if (B > 0) {
        if (!c.k || !c.v || !c.pages) return fail(PLDP_ERR_INVALID_ARG, "%s: null cache pointer", fn);
        if (c.dtype == PLDP_E4M3 && (!c.k_scale || !c.v_scale))
            return fail(PLDP_ERR_INVALID_ARG, "%s: a PLDP_E4M3 cache needs k_scale and v_scale", fn);
        pldp_status st = check_rows(fn, "cache.k", c.k, strides, es);
        if (st == PLDP_OK) st = check_rows(fn, "cache.v", c.v, strides, es);
        if (st != PLDP_OK) return st;
    }
    CacheView& w = *out;
    w.k = static_cast<uint8_t*>(c.k);
    w.v = static_cast<uint8_t*>(c.v);
    w.k_scale = c.k_scale;
    w.v_scale = c.v_scale;
    w.pages = c.pages;
    w.pages_stride = c.pages_stride;
    w.page_stride = c.page_stride * es;
    w.pos_stride = c.pos_stride * es;
    w.head_stride = c.head_stride * es;
    w.n_pages = c.n_pages;
    w.page_size = c.page_size;
    w.heads = c.heads;
    w.head_dim = c.head_dim;
    w.max_pages = c.max_pages;
    w.capacity = static_cast<int>(capacity);
    w.vec_bytes = c.head_dim * es;
    uint32_t l = 0;
    while ((uint64_t(1) << l) < static_cast<uint64_t>(c.page_size)) ++l;
    w.div_shift = l;
    w.div_mul = static_cast<uint32_t>((((uint64_t(1) << l) - c.page_size) << 32) / c.page_size + 1);
    return PLDP_OK;
}

namespace {

// ---------------------------------------------------------------------------
// append
// ---------------------------------------------------------------------------
struct Strides {
    int64_t seq, tok, head;
};

struct AppendArgs {
    CacheView c;
    const void *q, *k, *v, *q_norm, *k_norm;
    void* q_out;
    Strides qs, ks, vs, os;
    const float *cos, *sin;
    const int32_t *seq_len, *draft_len;
    uint32_t* status;
    int n, q_heads, rot, interleaved, capacity;
    uint32_t tokens, at_once;           // tokens in all, and a CTA's at a time
    int share;                          // groups of lanes a token
    float eps, inverse_dim;
};

constexpr int kAppendThreads = 256, kAppendBlocks = 4;

// Eight elements as floats.
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&x)[8]) {
    const uint4 r = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w;
    x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&p);
}
__device__ __forceinline__ uint4 bf16_8(const float (&x)[8]) {
    return make_uint4(bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]), bf16_pair(x[4], x[5]), bf16_pair(x[6], x[7]));
}
__device__ __forceinline__ uint32_t e4m3_quad(float a, float b, float c, float d) {
    return static_cast<uint32_t>(__nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3)) |
           static_cast<uint32_t>(__nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3)) << 16;
}

template <typename T>
struct Raw {                            // eight elements as they are in memory
    uint4 x[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T* p) {
#pragma unroll
        for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) x[i] = *(reinterpret_cast<const uint4*>(p) + i);
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < static_cast<int>(sizeof(T) / 2); ++i) x[i] = make_uint4(0u, 0u, 0u, 0u);
    }
    __device__ __forceinline__ void unpack(float (&y)[8]) const { load8(reinterpret_cast<const T*>(x), y); }
};

// A vector (a query, key or value head of one token) is GS lanes', eight elements a lane.  Of many tokens a quarter of a
// CTA takes one, its vectors in turn, the next one's elements on their way while one is worked on, and then its next
// token.  Instructions are what bounds it, so what a token's vectors share (its position, its page, the rotation's
// cosines and sines of this lane's elements) is worked out once a token.
// 4 x 4095 tokens of 48 heads of 128, bf16 to e4m3, with the read of the last positions behind it: 99 us (428 MB,
// 4.3 TB/s); 1 x 11 tokens, fp32 to bf16: 5.3 us, two launches' latency.
template <typename T, int GS, bool E4M3>
__global__ void __launch_bounds__(kAppendThreads, kAppendBlocks) cache_append_kernel(const AppendArgs a) {
    pdl_enter();
    constexpr int kGroups = kAppendThreads / GS;
    __shared__ __align__(16) float stage[2][kGroups][GS * 8];
    const CacheView& c = a.c;
    const int D = c.head_dim, g = threadIdx.x / GS, at = threadIdx.x % GS, e0 = at * 8;
    const int sub = g / a.share, first = g - sub * a.share + blockIdx.y * a.share, step = a.share * gridDim.y;   // this group's vectors
    if (sub >= static_cast<int>(a.at_once)) return;
    const int k_first = a.q_heads, v_first = a.q_heads + c.heads, total = v_first + c.heads;
    const bool live = e0 < D;
    // the lanes of this vector's group: they take the same branches
    const unsigned mates = GS == 32 ? 0xFFFFFFFFu : ((1u << (GS % 32)) - 1u) << ((threadIdx.x & 31) / GS * GS);
    const int half = a.rot >> 1;
    // where this lane's partners in the rotation are, when its eight elements rotate alike (or not at all)
    const bool alike = a.interleaved || (half & 7) == 0;
    const int partner = e0 < half ? e0 + half : e0 < a.rot ? e0 - half : e0;
    // The stage's two places, in turn from one rotated vector to the next, over the end of a token as well: the one barrier
    // between a place's write and its reads then also lies between those reads and the write after next.
    int turn = 0;
#pragma unroll 1
    for (uint32_t token = blockIdx.x * a.at_once + sub; token < a.tokens; token += gridDim.x * a.at_once) {
        const int b = token / static_cast<uint32_t>(a.n), i = token - b * a.n;
        const T* q = static_cast<const T*>(a.q) + (b * a.qs.seq + i * a.qs.tok + e0);
        const T* k = static_cast<const T*>(a.k) + (b * a.ks.seq + i * a.ks.tok + e0);
        const T* v = static_cast<const T*>(a.v) + (b * a.vs.seq + i * a.vs.tok + e0);
        auto source = [&](int h) {
            return h < k_first ? q + h * a.qs.head : h < v_first ? k + (h - k_first) * a.ks.head : v + (h - v_first) * a.vs.head;
        };
        Raw<T> next;
        if (first < total && live) next.load(source(first));
        uint32_t st;
        const StepTokens tk = step_tokens(a.seq_len, a.draft_len, b, a.n, a.capacity, st);
        if (i == 0 && first == 0 && at == 0 && st && a.status) atomicOr(a.status + b, st);
        if (i >= tk.count) continue;
        const int pos = tk.first + i;
        // y' = y cs + partner sn; an element that does not rotate is its own partner, cs = 1, sn = 0
        float cs[8], sn[8];
        {
            const float* cr = a.cos + static_cast<int64_t>(pos) * half;
            const float* sr = a.sin + static_cast<int64_t>(pos) * half;
#pragma unroll
            for (int j = 0; j < 8; ++j) cs[j] = 1.f, sn[j] = 0.f;
            if (alike && (half & 3) == 0) {                // whole vectors of the tables' rows
                if (e0 < a.rot) {
                    if (a.interleaved) {
                        const float4 x = __ldg(reinterpret_cast<const float4*>(cr + (e0 >> 1))), y = __ldg(reinterpret_cast<const float4*>(sr + (e0 >> 1)));
                        if (e0 + 8 <= a.rot) {
                            cs[0] = cs[1] = x.x, cs[2] = cs[3] = x.y, cs[4] = cs[5] = x.z, cs[6] = cs[7] = x.w;
                            sn[0] = -y.x, sn[1] = y.x, sn[2] = -y.y, sn[3] = y.y, sn[4] = -y.z, sn[5] = y.z, sn[6] = -y.w, sn[7] = y.w;
                        }
                    } else {
                        const int p = e0 < half ? e0 : e0 - half;
                        const float sign = e0 < half ? -1.f : 1.f;
#pragma unroll
                        for (int j = 0; j < 8; j += 4) {
                            const float4 x = __ldg(reinterpret_cast<const float4*>(cr + p + j)), y = __ldg(reinterpret_cast<const float4*>(sr + p + j));
                            cs[j] = x.x, cs[j + 1] = x.y, cs[j + 2] = x.z, cs[j + 3] = x.w;
                            sn[j] = sign * y.x, sn[j + 1] = sign * y.y, sn[j + 2] = sign * y.z, sn[j + 3] = sign * y.w;
                        }
                    }
                }
            } else {
#pragma unroll 1
                for (int j = 0; j < 8; ++j) {
                    const int e = e0 + j;
                    if (e >= a.rot) break;
                    const int p = a.interleaved ? e >> 1 : e < half ? e : e - half;
                    const float s = __ldg(sr + p), x = __ldg(cr + p), y = (a.interleaved ? e & 1 : e >= half) ? s : -s;
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if (k == j) cs[k] = x, sn[k] = y;
                }
            }
        }
        int64_t scale_at;
        const int64_t off = locate(c, c.pages + b * c.pages_stride, pos, scale_at);
        if (off < 0 && first == 0 && at == 0 && a.status) atomicOr(a.status + b, PLDP_ST_PAGE);
        auto unpack = [&](float (&y)[8]) {
            if (live) {
                next.unpack(y);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = 0.f;
            }
        };
        auto normed = [&](float (&y)[8], const Raw<T>& norm) {
            float w[8], sum = 0.f;
            norm.unpack(w);
            uint64_t two = 0;                              // (two elements an instruction)
#pragma unroll
            for (int j = 0; j < 8; j += 2) two = fma_f32x2(pack_f32x2(y[j], y[j + 1]), pack_f32x2(y[j], y[j + 1]), two);
            sum = lo_f32(two) + hi_f32(two);
#pragma unroll
            for (int o = GS / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(mates, sum, o, GS);
            const float r = rsqrtf(fmaf(sum, a.inverse_dim, a.eps));
            const uint64_t r2 = pack_f32x2(r, r);
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                const uint64_t z = fma_f32x2(fma_f32x2(pack_f32x2(y[j], y[j + 1]), r2, 0ull), pack_f32x2(w[j], w[j + 1]), 0ull);
                y[j] = lo_f32(z), y[j + 1] = hi_f32(z);
            }
        };
        auto rotated = [&](float (&y)[8]) {
            if (a.interleaved) {
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    const float p = y[j];
                    y[j] = p * cs[j] + y[j + 1] * sn[j];
                    y[j + 1] = y[j + 1] * cs[j + 1] + p * sn[j + 1];
                }
            } else {
                float* row = stage[turn][g];
                turn ^= 1;
                *reinterpret_cast<float4*>(row + e0) = make_float4(y[0], y[1], y[2], y[3]);
                *reinterpret_cast<float4*>(row + e0 + 4) = make_float4(y[4], y[5], y[6], y[7]);
                __syncwarp(mates);
                if (alike) {
                    const float4 lo = *reinterpret_cast<const float4*>(row + partner), hi = *reinterpret_cast<const float4*>(row + partner + 4);
                    y[0] = y[0] * cs[0] + lo.x * sn[0], y[1] = y[1] * cs[1] + lo.y * sn[1];
                    y[2] = y[2] * cs[2] + lo.z * sn[2], y[3] = y[3] * cs[3] + lo.w * sn[3];
                    y[4] = y[4] * cs[4] + hi.x * sn[4], y[5] = y[5] * cs[5] + hi.y * sn[5];
                    y[6] = y[6] * cs[6] + hi.z * sn[6], y[7] = y[7] * cs[7] + hi.w * sn[7];
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int e = e0 + j;
                        if (e < a.rot) y[j] = y[j] * cs[j] + row[e < half ? e + half : e - half] * sn[j];
                    }
                }
            }
        };
        // the queries, most of the vectors: nothing in their loop depends on which one it is
        int h = first;
        {
            Raw<T> norm;
            norm.clear();
            if (a.q_norm && live) norm.load(static_cast<const T*>(a.q_norm) + e0);
            const T* from = q + h * a.qs.head;
            const int64_t from_step = step * a.qs.head, to_step = step * a.os.head;
            __nv_bfloat16* to = static_cast<__nv_bfloat16*>(a.q_out) + (b * a.os.seq + i * a.os.tok + h * a.os.head + e0);
#pragma unroll 1
            for (; h < k_first; h += step, to += to_step) {
                float y[8];
                unpack(y);
                from += from_step;
                if (live && h + step < total) next.load(h + step < k_first ? from : source(h + step));
                if (a.q_norm) normed(y, norm);
                if (a.rot) rotated(y);
                if (live) *reinterpret_cast<uint4*>(to) = bf16_8(y);
            }
        }
#pragma unroll 1
        for (; h < total; h += step) {
            float y[8];
            unpack(y);
            if (live && h + step < total) next.load(source(h + step));
            const bool key = h < v_first;
            if (key) {
                if (a.k_norm) {
                    Raw<T> norm;
                    norm.clear();
                    if (live) norm.load(static_cast<const T*>(a.k_norm) + e0);
                    normed(y, norm);
                }
                if (a.rot) rotated(y);
            }
            if (off < 0) continue;
            const int head = key ? h - k_first : h - v_first;
            uint8_t* dst = (key ? c.k : c.v) + off + head * c.head_stride;
            if constexpr (E4M3) {
                float m = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) m = fmaxf(m, fabsf(y[j]));
#pragma unroll
                for (int o = GS / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(mates, m, o, GS));
                // Codes are quotients as 32-bit division rounds them, on which ties between codes depend: a product with the inverse,
                // put right by its remainder (Markstein 1990), two elements an instruction.
                const float scale = fmaxf(m * (1.f / 448.f), kLeastScale), inverse = 1.f / scale;
                if (live) {
                    const uint64_t by = pack_f32x2(inverse, inverse), less = pack_f32x2(-scale, -scale);
#pragma unroll
                    for (int j = 0; j < 8; j += 2) {
                        const uint64_t x = pack_f32x2(y[j], y[j + 1]), first = fma_f32x2(x, by, 0ull);
                        const uint64_t z = fma_f32x2(fma_f32x2(first, less, x), by, first);
                        y[j] = lo_f32(z), y[j + 1] = hi_f32(z);
                    }
                    *reinterpret_cast<uint2*>(dst + e0) = make_uint2(e4m3_quad(y[0], y[1], y[2], y[3]), e4m3_quad(y[4], y[5], y[6], y[7]));
                    if (at == 0) (key ? c.k_scale : c.v_scale)[scale_at + static_cast<int64_t>(head) * c.page_size] = scale;
                }
            } else if (live) {
                *reinterpret_cast<uint4*>(dst + 2 * e0) = bf16_8(y);
            }
        }
    }
}

template <typename T, int GS, bool E4M3>
cudaError_t launch_append_group(AppendArgs a, cudaStream_t s) {
    // few tokens: a token's vectors over as many CTAs as take them at once (1 x 11 tokens of 48: 1 us less than with
    // one CTA a token)
    constexpr uint32_t groups = kAppendThreads / GS;
    const uint32_t most = kAppendBlocks * sm_count(), total = a.q_heads + 2 * a.c.heads;
    const uint32_t turns = (total + groups - 1) / groups;
    a.share = static_cast<int>(total < groups ? total : groups);
    a.at_once = groups / a.share;
    uint32_t ctas = (a.tokens + a.at_once - 1) / a.at_once;
    const bool few = static_cast<uint64_t>(ctas) * turns <= most;
    // otherwise a quarter of a CTA a token, which then works out a token's common part less often: 4 x 4095 tokens of 48
    // vectors 23 us less (a half 23, an eighth 21), of shorter ones (64 elements) 37, 64 x 17 tokens 3
    constexpr uint32_t kMany = groups / 4;
    if (!few && total > kMany) {
        a.share = kMany;
        a.at_once = groups / a.share;
        ctas = (a.tokens + a.at_once - 1) / a.at_once;
    }
    return launch_pdl(cache_append_kernel<T, GS, E4M3>, dim3(ctas < most ? ctas : most, few ? turns : 1), dim3(kAppendThreads), 0, s, 0, a);
}
template <typename T, bool E4M3>
cudaError_t launch_append(const AppendArgs& a, cudaStream_t s) {
    if (a.c.head_dim <= 64) return launch_append_group<T, 8, E4M3>(a, s);
    if (a.c.head_dim <= 128) return launch_append_group<T, 16, E4M3>(a, s);
    return launch_append_group<T, 32, E4M3>(a, s);
}

// ---------------------------------------------------------------------------
// read
// ---------------------------------------------------------------------------
struct ReadArgs {
    CacheView c;
    const int32_t *start, *count;
    void *k_out, *v_out;
    Strides os;
    uint32_t* status;
    int n, per;   // per: positions a CTA takes
};

constexpr int kReadThreads = 256;

__device__ __forceinline__ float2 e4m3_two(uint32_t codes) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(codes), __NV_E4M3);
    return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

// The elements (8 of bf16, 4 of fp32) that 16 bytes of output hold, from the cache's.
template <bool E4M3>
struct Piece;
template <>
struct Piece<false> {
    uint4 x = make_uint4(0u, 0u, 0u, 0u);
    __device__ __forceinline__ void load(const uint8_t* p, const __nv_bfloat16*) { x = ld_stream16(p); }
    __device__ __forceinline__ void load(const uint8_t* p, const float*) {
        const uint2 y = __ldcs(reinterpret_cast<const uint2*>(p));
        x.x = y.x, x.y = y.y;
    }
    __device__ __forceinline__ void store(__nv_bfloat16* p, float) const { *reinterpret_cast<uint4*>(p) = x; }
    __device__ __forceinline__ void store(float* p, float) const {
        *reinterpret_cast<uint4*>(p) = make_uint4(x.x << 16, x.x & 0xFFFF0000u, x.y << 16, x.y & 0xFFFF0000u);
    }
};
template <>
struct Piece<true> {
    uint2 x = make_uint2(0u, 0u);
    __device__ __forceinline__ void load(const uint8_t* p, const __nv_bfloat16*) { x = __ldcs(reinterpret_cast<const uint2*>(p)); }
    __device__ __forceinline__ void load(const uint8_t* p, const float*) { x.x = __ldcs(reinterpret_cast<const unsigned int*>(p)); }
    __device__ __forceinline__ void store(__nv_bfloat16* p, float scale) const {
        const float2 a = e4m3_two(x.x & 0xFFFFu), b = e4m3_two(x.x >> 16), c = e4m3_two(x.y & 0xFFFFu), d = e4m3_two(x.y >> 16);
        *reinterpret_cast<uint4*>(p) = make_uint4(bf16_pair(a.x * scale, a.y * scale), bf16_pair(b.x * scale, b.y * scale),
                                                  bf16_pair(c.x * scale, c.y * scale), bf16_pair(d.x * scale, d.y * scale));
    }
    __device__ __forceinline__ void store(float* p, float scale) const {
        const float2 a = e4m3_two(x.x & 0xFFFFu), b = e4m3_two(x.x >> 16);
        *reinterpret_cast<float4*>(p) = make_float4(a.x * scale, a.y * scale, b.x * scale, b.y * scale);
    }
};

// One thread takes 16 bytes of output of one vector of keys and the same of values, so that neighbours write side by
// side, and steps from piece to piece without divisions.  Bound by memory: 8 x 4096 positions of 8 heads of 128, e4m3
// to bf16, 159 MB in 28.6 us (5.6 TB/s); 33.5 with 16 bytes of codes a thread and two divisions a piece.
template <typename O, bool E4M3>
__global__ void __launch_bounds__(kReadThreads) cache_read_kernel(const ReadArgs a) {
    pdl_enter();
    const CacheView& c = a.c;
    const int b = blockIdx.y;
    int first = a.start ? __ldg(a.start + b) : 0, count = __ldg(a.count + b);
    uint32_t st = 0;
    if (count < 0 || count > a.n) {
        st |= PLDP_ST_SEQ_LEN;
        count = count < 0 ? 0 : a.n;
    }
    if (first < 0 || first > c.capacity) {
        st |= PLDP_ST_CAPACITY;
        count = 0;
    } else if (count > c.capacity - first) {
        st |= PLDP_ST_CAPACITY;
        count = c.capacity - first;
    }
    if (blockIdx.x == 0 && threadIdx.x == 0 && st && a.status) atomicOr(a.status + b, st);
    const int lo = blockIdx.x * a.per;                  // below n
    constexpr int kElements = 16 / sizeof(O), kBytes = kElements * (E4M3 ? 1 : 2);
    const uint32_t rows = lo < count ? min(a.per, count - lo) : 0, heads = c.heads, chunks = static_cast<uint32_t>(c.head_dim) / kElements;
    const int32_t* table = c.pages + b * c.pages_stride;
    // this thread's piece (position, head, chunk), and from one to its next
    uint32_t ch = threadIdx.x % chunks, r = threadIdx.x / chunks, head = r % heads;
    r /= heads;
    const uint32_t ch_step = kReadThreads % chunks, vectors = kReadThreads / chunks, head_step = vectors % heads, r_step = vectors / heads;
    while (r < rows) {
        const int i = lo + static_cast<int>(r);
        int64_t scale_at;
        const int64_t off = locate(c, table, first + i, scale_at);
        if (off < 0 && head == 0 && ch == 0 && a.status) atomicOr(a.status + b, PLDP_ST_PAGE);
        const int64_t from = off + head * c.head_stride + ch * kBytes;
        const int64_t to = b * a.os.seq + i * a.os.tok + head * a.os.head + ch * kElements;
        Piece<E4M3> x[2];
        float scale[2] = {0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            if (off < 0 || !(w ? a.v_out : a.k_out)) continue;
            x[w].load((w ? c.v : c.k) + from, static_cast<const O*>(nullptr));
            if constexpr (E4M3) scale[w] = __ldg((w ? c.v_scale : c.k_scale) + scale_at + static_cast<int64_t>(head) * c.page_size);
        }
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            O* out = static_cast<O*>(w ? a.v_out : a.k_out);
            if (out) x[w].store(out + to, scale[w]);
        }
        ch += ch_step, head += head_step, r += r_step;
        if (ch >= chunks) ch -= chunks, ++head;
        if (head >= heads) head -= heads, ++r;
    }
}

Strides strides_of(const int64_t (&s)[3]) { return {s[0], s[1], s[2]}; }

}  // namespace
}  // namespace pldp

using namespace pldp;

extern "C" {

PLDP_API pldp_status pldp_cache_append(const pldp_cache_append_args* p, void* stream) {
    const char* fn = "cache_append";
    if (!p) return fail(PLDP_ERR_INVALID_ARG, "%s: null argument block", fn);
    if (p->B < 0 || p->n < 1 || p->q_heads < 1)
        return fail(PLDP_ERR_INVALID_ARG, "%s: B < 0, n < 1 or q_heads < 1", fn);
    if (p->dtype != PLDP_F32 && p->dtype != PLDP_BF16)
        return fail(PLDP_ERR_UNSUPPORTED, "%s: dtype %d", fn, static_cast<int>(p->dtype));
    if (p->q_heads > 65536) return fail(PLDP_ERR_UNSUPPORTED, "%s: more than 65536 query heads", fn);
    AppendArgs a = {};
    pldp_status st = cache_view(fn, p->cache, p->B, &a.c);
    if (st != PLDP_OK) return st;
    if ((p->cos == nullptr) != (p->sin == nullptr)) return fail(PLDP_ERR_INVALID_ARG, "%s: cos and sin go together", fn);
    if (p->cos && (p->rot < 2 || p->rot > p->cache.head_dim || p->rot % 2 || p->rot_rows < 1))
        return fail(PLDP_ERR_INVALID_ARG, "%s: rot must be even, 2..head_dim, and rot_rows >= 1", fn);
    if (!(p->eps >= 0.f) || !isfinite(p->eps)) return fail(PLDP_ERR_INVALID_ARG, "%s: eps must be finite and >= 0", fn);
    if (static_cast<int64_t>(p->B) * p->n > INT32_MAX)
        return fail(PLDP_ERR_UNSUPPORTED, "%s: B * n must be below 2^31", fn);
    if (p->B == 0) return PLDP_OK;
    if (!p->q || !p->k || !p->v || !p->q_out || !p->seq_len) return fail(PLDP_ERR_INVALID_ARG, "%s: null pointer", fn);
    const size_t es = p->dtype == PLDP_F32 ? 4 : 2;
    if ((st = check_rows(fn, "q", p->q, p->q_strides, es)) != PLDP_OK) return st;
    if ((st = check_rows(fn, "k", p->k, p->k_strides, es)) != PLDP_OK) return st;
    if ((st = check_rows(fn, "v", p->v, p->v_strides, es)) != PLDP_OK) return st;
    if ((st = check_rows(fn, "q_out", p->q_out, p->q_out_strides, 2)) != PLDP_OK) return st;
    if (!aligned16(p->q_norm) || !aligned16(p->k_norm) || !aligned16(p->cos) || !aligned16(p->sin))
        return fail(PLDP_ERR_INVALID_ARG, "%s: norms, cos and sin must be 16-byte aligned", fn);
    a.q = p->q, a.k = p->k, a.v = p->v;
    a.q_norm = p->q_norm, a.k_norm = p->k_norm;
    a.q_out = p->q_out;
    a.qs = strides_of(p->q_strides), a.ks = strides_of(p->k_strides), a.vs = strides_of(p->v_strides);
    a.os = strides_of(p->q_out_strides);
    a.cos = p->cos, a.sin = p->sin;
    a.seq_len = p->seq_len, a.draft_len = p->draft_len;
    a.status = p->status;
    a.n = p->n, a.q_heads = p->q_heads;
    a.rot = p->cos ? p->rot : 0, a.interleaved = p->interleaved != 0;
    a.capacity = a.c.capacity;
    if (p->cos && p->rot_rows < a.capacity) a.capacity = static_cast<int>(p->rot_rows);
    a.eps = p->eps;
    a.tokens = p->B * p->n;
    a.inverse_dim = 1.f / p->cache.head_dim;
    auto s = static_cast<cudaStream_t>(stream);
    const bool q8 = p->cache.dtype == PLDP_E4M3;
    cudaError_t e;
    if (p->dtype == PLDP_F32) e = q8 ? launch_append<float, true>(a, s) : launch_append<float, false>(a, s);
    else e = q8 ? launch_append<__nv_bfloat16, true>(a, s) : launch_append<__nv_bfloat16, false>(a, s);
    return launched(fn, e);
}

PLDP_API pldp_status pldp_cache_read(const pldp_cache_read_args* p, void* stream) {
    const char* fn = "cache_read";
    if (!p) return fail(PLDP_ERR_INVALID_ARG, "%s: null argument block", fn);
    if (p->B < 0 || p->n < 0) return fail(PLDP_ERR_INVALID_ARG, "%s: B < 0 or n < 0", fn);
    if (p->B > 65535) return fail(PLDP_ERR_UNSUPPORTED, "%s: more than 65535 sequences", fn);
    if (p->dtype != PLDP_F32 && p->dtype != PLDP_BF16)
        return fail(PLDP_ERR_UNSUPPORTED, "%s: dtype %d", fn, static_cast<int>(p->dtype));
    ReadArgs a = {};
    pldp_status st = cache_view(fn, p->cache, p->B, &a.c);
    if (st != PLDP_OK) return st;
    if (p->B == 0 || p->n == 0) return PLDP_OK;
    if (!p->count) return fail(PLDP_ERR_INVALID_ARG, "%s: null pointer", fn);
    const size_t es = p->dtype == PLDP_F32 ? 4 : 2;
    if ((st = check_rows(fn, "k_out", p->k_out, p->out_strides, es)) != PLDP_OK) return st;
    if ((st = check_rows(fn, "v_out", p->v_out, p->out_strides, es)) != PLDP_OK) return st;
    a.start = p->start, a.count = p->count;
    a.k_out = p->k_out, a.v_out = p->v_out;
    a.os = strides_of(p->out_strides);
    a.status = p->status;
    a.n = p->n;
    // about four pieces a thread (159 MB: 28.6 us; eight 31.0, two 29.8, one 35.5), at least one position a CTA; one a
    // thread where that leaves SMs without a CTA (an append of 11 tokens and their read: 5.3 us; four 6.2)
    const int row = a.c.head_dim * (p->dtype == PLDP_F32 ? 4 : 2) / 16 * a.c.heads;
    const bool few = static_cast<int64_t>(p->n) * p->B * row < static_cast<int64_t>(4 * kReadThreads) * sm_count();
    a.per = (few ? 1 : 4) * kReadThreads / row;
    if (a.per < 1) a.per = 1;
    const dim3 grid(static_cast<unsigned>((static_cast<int64_t>(p->n) + a.per - 1) / a.per), p->B);
    auto s = static_cast<cudaStream_t>(stream);
    const bool q8 = p->cache.dtype == PLDP_E4M3;
    cudaError_t e;
    if (p->dtype == PLDP_F32)
        e = q8 ? launch_pdl(cache_read_kernel<float, true>, grid, dim3(kReadThreads), 0, s, 0, a)
               : launch_pdl(cache_read_kernel<float, false>, grid, dim3(kReadThreads), 0, s, 0, a);
    else
        e = q8 ? launch_pdl(cache_read_kernel<__nv_bfloat16, true>, grid, dim3(kReadThreads), 0, s, 0, a)
               : launch_pdl(cache_read_kernel<__nv_bfloat16, false>, grid, dim3(kReadThreads), 0, s, 0, a);
    return launched(fn, e);
}

}  // extern "C"
