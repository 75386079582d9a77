// The pages of a cache: giving them out, sharing, giving back, moving and copying them.
#include "pldp_cache.cuh"

namespace pldp {
namespace {

struct Table {
    int32_t* pages;
    int64_t stride;
    int32_t* refs;
    int B, max_pages, page_size, n_pages;
};

__device__ __forceinline__ bool is_page(const Table& t, int x) { return static_cast<unsigned>(x) < static_cast<unsigned>(t.n_pages); }

// ---------------------------------------------------------------------------
// free and fork: an entry a thread, one launch's latency (1.0-1.3 and 1.3-1.6 us a call in a graph, the larger of 256 sequences
// of 258 entries)
// ---------------------------------------------------------------------------
constexpr int kEntryThreads = 256;

__global__ void __launch_bounds__(kEntryThreads) pages_free_kernel(const Table t, const int32_t* keep_len) {
    pdl_enter();
    const int b = blockIdx.y, keep = __ldg(keep_len + b), e = blockIdx.x * kEntryThreads + threadIdx.x;
    if (keep < 0 || e >= t.max_pages || static_cast<int64_t>(e) * t.page_size < keep) return;
    int32_t* entry = t.pages + b * t.stride + e;
    const int old = *entry;
    if (is_page(t, old)) atomicSub(t.refs + old, 1);
    if (old != -1) *entry = -1;
}

__global__ void __launch_bounds__(kEntryThreads) pages_fork_kernel(const Table t, const int32_t* parent, const int32_t* len,
                                                                   uint32_t* status) {
    pdl_enter();
    const int b = blockIdx.y, p = __ldg(parent + b), e = blockIdx.x * kEntryThreads + threadIdx.x;
    if (p == -1 || p == b) return;
    uint32_t st = 0;
    if (p < 0 || p >= t.B) {
        st = PLDP_ST_ROW_INDEX;
    } else {
        // (a row that is read must not be written)
        const int above = __ldg(parent + p), n = __ldg(len + b);
        if (above >= 0 && above < t.B && above != p) st = PLDP_ST_ROW_INDEX;
        if (n < 0 || n > static_cast<int64_t>(t.max_pages) * t.page_size) st |= PLDP_ST_SEQ_LEN;
    }
    if (st) {
        if (e == 0 && status) atomicOr(status + b, st);
        return;
    }
    if (e >= t.max_pages) return;
    int32_t* entry = t.pages + b * t.stride + e;
    const int old = *entry;
    int now = -1;
    if (static_cast<int64_t>(e) * t.page_size < __ldg(len + b)) now = t.pages[p * t.stride + e];
    if (!is_page(t, now)) now = -1;
    if (now == old) return;
    if (now >= 0) atomicAdd(t.refs + now, 1);
    if (is_page(t, old)) atomicSub(t.refs + old, 1);
    *entry = now;
}

// ---------------------------------------------------------------------------
// reserve and compact: one cluster that looks at all pages
// ---------------------------------------------------------------------------
// Which page is the k-th free one is a running count over refs.  A cluster of eight CTAs counts: every warp has a run of
// neighbouring pages, the counts of warps and CTAs are added up between cluster barriers (shared memory of one another),
// and a second look at the run gives each page its number.  All of it is latency: a launch, three barriers, two
// looks; one launch of a cluster saves the workspace's way through a second and third one.  A step's wants are one word a
// sequence and are counted with the free pages, a barrier less: 4.9 us for 5 sequences, 6.5 for 256 and 9000 pages;
// compacting 4.5 and, 12000 pages, 5.4.  2^20 pages: 13.4 us to reserve, 48 to compact, as eight SMs read them.
constexpr int kCluster = 8, kThreads = 1024, kWarps = kThreads / 32;

struct Counts {
    int warp[kWarps];      // of this CTA's warps, then what lies before each of them
    int total;             // of this CTA
};

// Every warp's count -> the count before this warp in the whole cluster (`before`) and of all (`all`); where they may
// pass `most`, they stay there.  A cluster barrier lies between the two halves, once for each `c`.
__device__ __forceinline__ void give_count(Counts& c, int mine, int most) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0) c.warp[warp] = mine;
    __syncthreads();
    if (warp == 0) {
        unsigned upto = c.warp[lane];                        // (two of them stay below 2^32)
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned y = __shfl_up_sync(0xFFFFFFFFu, upto, o);
            if (lane >= o) upto = min(upto + y, static_cast<unsigned>(most));
        }
        const unsigned prior = __shfl_up_sync(0xFFFFFFFFu, upto, 1);
        c.warp[lane] = lane ? prior : 0;
        if (lane == 31) c.total = upto;
    }
}
__device__ __forceinline__ void take_count(cg::cluster_group& cluster, Counts& c, int most, int& before, int& all) {
    unsigned ahead = 0, sum = 0;
#pragma unroll
    for (int k = 0; k < kCluster; ++k) {
        const unsigned x = *cluster.map_shared_rank(&c.total, k);
        if (k < static_cast<int>(cluster.block_rank())) ahead = min(ahead + x, static_cast<unsigned>(most));
        sum = min(sum + x, static_cast<unsigned>(most));
    }
    before = min(ahead + c.warp[threadIdx.x >> 5], static_cast<unsigned>(most)), all = sum;
}

// A warp's run of pages, four neighbours a lane.
struct Run {
    int lo, hi;
};
__device__ __forceinline__ Run run_of(int n_pages, int rank) {
    const int w = rank * kWarps + (threadIdx.x >> 5);
    const int64_t each = (static_cast<int64_t>(n_pages) + kCluster * kWarps * 128 - 1) / (kCluster * kWarps * 128) * 128;
    const int64_t lo = each * w, hi = lo + each;
    return {static_cast<int>(lo < n_pages ? lo : n_pages), static_cast<int>(hi < n_pages ? hi : n_pages)};
}
// Bits of this lane's four pages p..p+3 that exist and are held (or free).
template <bool HELD>
__device__ __forceinline__ unsigned four_pages(const int32_t* refs, bool vectors, int p, int hi) {
    int r[4] = {};
    if (vectors && p + 3 < hi) {
        const int4 x = *reinterpret_cast<const int4*>(refs + p);
        r[0] = x.x, r[1] = x.y, r[2] = x.z, r[3] = x.w;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (p + i < hi) r[i] = refs[p + i];
    }
    unsigned bits = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (p + i < hi && (r[i] > 0) == HELD) bits |= 1u << i;
    return bits;
}
__device__ __forceinline__ int warp_total(int x) { return __reduce_add_sync(0xFFFFFFFFu, x); }
__device__ __forceinline__ int lanes_before(int x, int lane) {
    int upto = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xFFFFFFFFu, upto, o);
        if (lane >= o) upto += y;
    }
    return upto - x;
}

struct ReserveArgs {
    Table t;
    const int32_t *start, *count;
    int n;
    int32_t* copies;
    uint32_t* status;
    int32_t* list;       // [n_pages] the free pages that are given out
    int32_t* base;       // [B] number of a sequence's first one, -1: it gets none
    uint32_t* words;     // [B][W] which entries of a sequence's range need a page
    int W;
};

// The entries that sequence b wants to write: first..first+entries-1.
struct Range {
    int first, entries, start;
    uint32_t status;
};
__device__ __forceinline__ Range range_of(const ReserveArgs& a, int b) {
    const int s = __ldg(a.start + b), c = a.count ? __ldg(a.count + b) : a.n;
    if (s < 0 || c < 0 || c > a.n) return {0, 0, 0, PLDP_ST_SEQ_LEN};
    if (c == 0) return {0, 0, 0, 0u};
    if (static_cast<int64_t>(s) + c > static_cast<int64_t>(a.t.max_pages) * a.t.page_size) return {0, 0, 0, PLDP_ST_CAPACITY};
    const int first = s / a.t.page_size;
    return {first, (s + (c - 1)) / a.t.page_size - first + 1, s, 0u};
}

__global__ void __launch_bounds__(kThreads, 1) __cluster_dims__(kCluster, 1, 1) pages_reserve_kernel(const ReserveArgs a) {
    pdl_enter();
    __shared__ Counts free_pages, wanted;
    cg::cluster_group cluster = cg::this_cluster();
    const Table& t = a.t;
    const int rank = cluster.block_rank(), warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const bool vectors = (reinterpret_cast<uintptr_t>(t.refs) & 15u) == 0;
    const Run run = run_of(t.n_pages, rank);

    // which entries need a page, a word of 32 a warp
    const int64_t items = static_cast<int64_t>(t.B) * a.W;
    auto look = [&](int b, int w) {
        const Range r = range_of(a, b);
        const int k = w * 32 + lane;
        bool need = false;
        if (k < r.entries) {
            const int page = t.pages[b * t.stride + r.first + k];
            need = !is_page(t, page) || t.refs[page] > 1;
        }
        const uint32_t word = __ballot_sync(0xFFFFFFFFu, need);
        if (lane == 0) a.words[static_cast<int64_t>(b) * a.W + w] = word;
        return __popc(word);
    };
    // how many pages each sequence needs: CTAs have runs of sequences, their warps neighbouring ones
    // (no more than there are pages count: sums stay in range, and more are not given out)
    const int most = t.n_pages + 1;
    auto plus = [&](int x, int y) { return static_cast<int>(min(static_cast<unsigned>(x) + static_cast<unsigned>(y), static_cast<unsigned>(most))); };
    const int each = (t.B + kCluster * kWarps - 1) / (kCluster * kWarps);
    const int b0 = min(t.B, (rank * kWarps + warp) * each), b1 = min(t.B, b0 + each);
    auto needs = [&](int b) {
        int n = 0;
        for (int w = lane; w < a.W; w += 32) n += __popc(__ldcg(a.words + static_cast<int64_t>(b) * a.W + w));
        return warp_total(n);
    };
    int warp_needs = 0;
    if (a.W == 1) {                                          // (a step: its counts go with those of the free pages)
        for (int b = b0; b < b1; ++b) warp_needs = plus(warp_needs, look(b, 0));
    } else {
        for (int64_t i = rank * kWarps + warp; i < items; i += kCluster * kWarps) {
            const int b = static_cast<int>(i / a.W);
            look(b, static_cast<int>(i - static_cast<int64_t>(b) * a.W));
        }
    }
    int mine = 0;
    for (int p = run.lo + 4 * lane; p - 4 * lane < run.hi; p += 128) mine += __popc(four_pages<false>(t.refs, vectors, p, run.hi));
    give_count(free_pages, warp_total(mine), INT32_MAX);
    if (a.W == 1) give_count(wanted, warp_needs, most);
    cluster.sync();
    int before, all, need_before, need_all;
    take_count(cluster, free_pages, INT32_MAX, before, all);
    if (a.W > 1) {
        for (int b = b0; b < b1; ++b) warp_needs = plus(warp_needs, needs(b));
        give_count(wanted, warp_needs, most);
        cluster.sync();
    }
    take_count(cluster, wanted, most, need_before, need_all);
    for (int b = b0; b < b1; ++b) {
        const int n = needs(b);
        const bool served = n == 0 || static_cast<int64_t>(need_before) + n <= all;
        if (lane == 0) {
            a.base[b] = served ? need_before : -1;
            const uint32_t st = range_of(a, b).status | (served ? 0u : static_cast<uint32_t>(PLDP_ST_CAPACITY));
            if (st && a.status) atomicOr(a.status + b, st);
        }
        need_before = plus(need_before, n);
    }
    // the free pages that are given out, by number
    const int given = min(need_all, all);
    for (int p = run.lo + 4 * lane; p - 4 * lane < run.hi && before < given; p += 128) {
        const unsigned bits = four_pages<false>(t.refs, vectors, p, run.hi);
        const int n = __popc(bits);
        int at = before + lanes_before(n, lane);
        before += warp_total(n);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (bits >> i & 1u) {
                if (at < given) a.list[at] = p + i;
                ++at;
            }
    }
    cluster.sync();

    for (int64_t i = rank * kWarps + warp; i < items; i += kCluster * kWarps) {
        const int b = static_cast<int>(i / a.W), w = static_cast<int>(i - static_cast<int64_t>(b) * a.W);
        const uint32_t word = __ldcg(a.words + i);
        const int base = __ldcg(a.base + b);
        const Range r = range_of(a, b);
        int from = -1, to = -1;
        if (base >= 0 && word) {
            int at = 0;
            for (int x = lane; x < w; x += 32) at += __popc(__ldcg(a.words + static_cast<int64_t>(b) * a.W + x));
            at = base + warp_total(at) + __popc(word & ((1u << lane) - 1u));
            if (word >> lane & 1u) {
                int32_t* entry = t.pages + b * t.stride + r.first + w * 32 + lane;
                const int old = *entry, now = __ldcg(a.list + at);
                *entry = now;
                t.refs[now] = 1;
                if (is_page(t, old)) {
                    atomicSub(t.refs + old, 1);
                    if (w == 0 && lane == 0 && r.start % t.page_size) from = old, to = now;
                }
            }
        }
        if (w == 0 && lane == 0) *reinterpret_cast<int2*>(a.copies + 2 * static_cast<int64_t>(b)) = make_int2(from, to);
    }
    cluster.sync();        // (shared memory of a CTA that another one still reads)
}

struct CompactArgs {
    Table t;
    int32_t *copies, *n_copies, *used;
    int32_t* head;       // U and the number of moves
    int32_t *to, *holes, *movers;
};

__global__ void __launch_bounds__(kThreads, 1) __cluster_dims__(kCluster, 1, 1) pages_compact_kernel(const CompactArgs a) {
    pdl_enter();
    __shared__ Counts held;
    __shared__ int moves;
    cg::cluster_group cluster = cg::this_cluster();
    const Table& t = a.t;
    const int rank = cluster.block_rank(), lane = threadIdx.x & 31;
    const bool vectors = (reinterpret_cast<uintptr_t>(t.refs) & 15u) == 0;
    const Run run = run_of(t.n_pages, rank);
    if (threadIdx.x == 0) moves = 0;
    int mine = 0;
    for (int p = run.lo + 4 * lane; p - 4 * lane < run.hi; p += 128) mine += __popc(four_pages<true>(t.refs, vectors, p, run.hi));
    give_count(held, warp_total(mine), INT32_MAX);
    cluster.sync();
    int before, U;
    take_count(cluster, held, INT32_MAX, before, U);

    // free pages below U by ascending number, held ones from U on by descending number
    int moving = 0;
    for (int p = run.lo + 4 * lane; p - 4 * lane < run.hi; p += 128) {
        const unsigned bits = four_pages<true>(t.refs, vectors, p, run.hi);
        const int n = __popc(bits);
        int at = before + lanes_before(n, lane);           // held pages before this one
        before += warp_total(n);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int page = p + i;
            if (page >= run.hi) break;
            const bool is_held = bits >> i & 1u;
            if (page < U) {
                if (!is_held) a.holes[page - at] = page;
            } else {
                a.to[page] = page;
                if (is_held) {
                    a.movers[U - 1 - at] = page;
                    ++moving;
                }
            }
            at += is_held;
        }
    }
    moving = warp_total(moving);
    if (lane == 0 && moving) atomicAdd(cluster.map_shared_rank(&moves, 0), moving);
    cluster.sync();
    const int n = *cluster.map_shared_rank(&moves, 0);
    for (int i = rank * kThreads + threadIdx.x; i < n; i += kCluster * kThreads) {
        const int from = __ldcg(a.movers + i), to = __ldcg(a.holes + i);
        *reinterpret_cast<int2*>(a.copies + 2 * static_cast<int64_t>(i)) = make_int2(from, to);
        a.to[from] = to;
        t.refs[to] = t.refs[from];
        t.refs[from] = 0;
    }
    if (rank == 0 && threadIdx.x == 0) {
        a.head[0] = U, a.head[1] = n;
        *a.n_copies = n;
        if (a.used) *a.used = U;
    }
    cluster.sync();
}

// The table's entries after the moves, an entry a thread.
__global__ void __launch_bounds__(kEntryThreads) pages_moved_kernel(const Table t, const int32_t* head, const int32_t* to) {
    pdl_enter();
    const int U = head[0], moves = head[1], e = blockIdx.x * kEntryThreads + threadIdx.x;
    if (moves == 0 || e >= t.max_pages) return;
    int32_t* entry = t.pages + blockIdx.y * t.stride + e;
    const int page = *entry;
    if (is_page(t, page) && page >= U) *entry = to[page];
}

// ---------------------------------------------------------------------------
// copy
// ---------------------------------------------------------------------------
struct CopyArgs {
    CacheView c;
    const int32_t *copies, *n_copies;
    int n;
    bool e4m3;
    int64_t run, inner_stride, outer_stride;   // bytes that lie together, and between two such of either order
    int64_t inner, runs;                       // runs of the inner order, and in all
    int64_t pieces;                            // of one page's keys (or values)
};

// A piece is 16 KB of one page's keys or values, sixteen bytes a thread four times, all loaded before the first is stored:
// memory bounds it (1.22 GB read and written in 184 us, 6.6 TB/s).
constexpr int kCopyThreads = 256, kCopyLoads = 4, kPiece = kCopyThreads * kCopyLoads * 16;

__global__ void __launch_bounds__(kCopyThreads) copy_pages_kernel(const CopyArgs a) {
    pdl_enter();
    const CacheView& c = a.c;
    int n = a.n;
    if (a.n_copies) n = max(0, min(n, __ldg(a.n_copies)));
    const int64_t items = static_cast<int64_t>(n) * 2 * a.pieces, chunks = a.runs * (a.run / 16), per_run = a.run / 16;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t part = item / a.pieces, piece = item - part * a.pieces;
        const int pair = static_cast<int>(part >> 1), kv = part & 1;
        const int from = __ldg(a.copies + 2 * static_cast<int64_t>(pair)), to = __ldg(a.copies + 2 * static_cast<int64_t>(pair) + 1);
        if (static_cast<unsigned>(from) >= static_cast<unsigned>(c.n_pages) || static_cast<unsigned>(to) >= static_cast<unsigned>(c.n_pages) ||
            from == to)
            continue;
        uint8_t* base = kv ? c.v : c.k;
        const uint8_t* src = base + from * c.page_stride;
        uint8_t* dst = base + to * c.page_stride;
        uint4 x[kCopyLoads];
        int64_t at[kCopyLoads];
#pragma unroll
        for (int i = 0; i < kCopyLoads; ++i) {
            const int64_t ch = piece * (kPiece / 16) + i * kCopyThreads + threadIdx.x;
            at[i] = -1;
            if (ch < chunks) {
                if (a.runs == 1) {
                    at[i] = ch * 16;
                } else {
                    const int64_t r = ch / per_run, outer = r / a.inner;
                    at[i] = (ch - r * per_run) * 16 + (r - outer * a.inner) * a.inner_stride + outer * a.outer_stride;
                }
                x[i] = ld_stream16(src + at[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < kCopyLoads; ++i)
            if (at[i] >= 0) *reinterpret_cast<uint4*>(dst + at[i]) = x[i];
        if (a.e4m3 && piece == 0) {
            float* scale = kv ? c.v_scale : c.k_scale;
            const int64_t each = static_cast<int64_t>(c.heads) * c.page_size;
            for (int64_t i = threadIdx.x; i < each; i += kCopyThreads) scale[to * each + i] = scale[from * each + i];
        }
    }
}

pldp_status table_of(const char* fn, const pldp_page_table* p, Table* t) {
    if (!p) return fail(PLDP_ERR_INVALID_ARG, "%s: null table", fn);
    if (p->B < 0 || p->max_pages < 1 || p->page_size < 1 || p->n_pages < 1 || p->pages_stride < p->max_pages)
        return fail(PLDP_ERR_INVALID_ARG, "%s: B < 0, max_pages, page_size or n_pages < 1, or pages_stride < max_pages", fn);
    if (static_cast<int64_t>(p->max_pages) * p->page_size > INT32_MAX)
        return fail(PLDP_ERR_INVALID_ARG, "%s: max_pages * page_size must be below 2^31", fn);
    if (p->B > 65535) return fail(PLDP_ERR_UNSUPPORTED, "%s: more than 65535 rows", fn);
    // (pages are counted past the last one)
    if (p->n_pages > INT32_MAX - 4095) return fail(PLDP_ERR_UNSUPPORTED, "%s: more than 2^31 - 4096 pages", fn);
    if (p->B > 0 && (!p->pages || !p->refs)) return fail(PLDP_ERR_INVALID_ARG, "%s: null pointer", fn);
    *t = {p->pages, p->pages_stride, p->refs, p->B, p->max_pages, p->page_size, p->n_pages};
    return PLDP_OK;
}
dim3 entries_grid(const Table& t) {
    return dim3(static_cast<unsigned>((static_cast<int64_t>(t.max_pages) + kEntryThreads - 1) / kEntryThreads), t.B);
}
pldp_status check_workspace(const char* fn, const pldp_page_table* p, const void* ws, size_t bytes) {
    const size_t need = pldp_pages_workspace_size(p->B, p->max_pages, p->n_pages);
    if (!ws) return fail(PLDP_ERR_INVALID_ARG, "%s: null pointer", fn);
    if (bytes < need) return fail(PLDP_ERR_INVALID_ARG, "%s: workspace needs %zu bytes, has %zu", fn, need, bytes);
    if (!aligned16(ws)) return fail(PLDP_ERR_INVALID_ARG, "%s: workspace is not 16-byte aligned", fn);
    return PLDP_OK;
}

}  // namespace
}  // namespace pldp

using namespace pldp;

extern "C" {

PLDP_API size_t pldp_pages_workspace_size(int B, int max_pages, int n_pages) {
    if (B < 0 || max_pages < 1 || n_pages < 1) return 0;
    const size_t reserve = static_cast<size_t>(n_pages) + B + static_cast<size_t>(B) * ((static_cast<size_t>(max_pages) + 31) / 32);
    const size_t compact = 2 * static_cast<size_t>(n_pages) + 8;
    return ((reserve > compact ? reserve : compact) * sizeof(int32_t) + 255) / 256 * 256;
}

PLDP_API pldp_status pldp_pages_free(const pldp_page_table* table, const int32_t* keep_len, void* stream) {
    const char* fn = "pages_free";
    Table t;
    const pldp_status st = table_of(fn, table, &t);
    if (st != PLDP_OK) return st;
    if (t.B == 0) return PLDP_OK;
    if (!keep_len) return fail(PLDP_ERR_INVALID_ARG, "%s: null pointer", fn);
    return launched(fn, launch_pdl(pages_free_kernel, entries_grid(t), dim3(kEntryThreads), 0, static_cast<cudaStream_t>(stream), 0, t, keep_len));
}

PLDP_API pldp_status pldp_pages_fork(const pldp_page_table* table, const int32_t* parent, const int32_t* len,
                                     uint32_t* status, void* stream) {
    const char* fn = "pages_fork";
    Table t;
    const pldp_status st = table_of(fn, table, &t);
    if (st != PLDP_OK) return st;
    if (t.B == 0) return PLDP_OK;
    if (!parent || !len) return fail(PLDP_ERR_INVALID_ARG, "%s: null pointer", fn);
    return launched(fn, launch_pdl(pages_fork_kernel, entries_grid(t), dim3(kEntryThreads), 0, static_cast<cudaStream_t>(stream), 0, t, parent,
                                   len, status));
}

PLDP_API pldp_status pldp_pages_reserve(const pldp_page_table* table, const int32_t* start, const int32_t* count, int n,
                                        int32_t* copies, uint32_t* status, void* workspace, size_t workspace_bytes,
                                        void* stream) {
    const char* fn = "pages_reserve";
    ReserveArgs a = {};
    pldp_status st = table_of(fn, table, &a.t);
    if (st != PLDP_OK) return st;
    if (n < 0) return fail(PLDP_ERR_INVALID_ARG, "%s: n < 0", fn);
    if (a.t.B == 0) return PLDP_OK;
    if (!start || !copies) return fail(PLDP_ERR_INVALID_ARG, "%s: null pointer", fn);
    if (reinterpret_cast<uintptr_t>(copies) & 7u) return fail(PLDP_ERR_INVALID_ARG, "%s: copies is not 8-byte aligned", fn);
    if ((st = check_workspace(fn, table, workspace, workspace_bytes)) != PLDP_OK) return st;
    a.start = start, a.count = count, a.n = n;
    a.copies = copies, a.status = status;
    // entries that a range of n positions reaches into, at most the row's
    int64_t entries = (static_cast<int64_t>(n) + a.t.page_size - 2) / a.t.page_size + 1;
    if (entries > a.t.max_pages) entries = a.t.max_pages;
    if (entries < 1) entries = 1;
    a.W = static_cast<int>((entries + 31) / 32);
    a.list = static_cast<int32_t*>(workspace);
    a.base = a.list + a.t.n_pages;
    a.words = reinterpret_cast<uint32_t*>(a.base + a.t.B);
    return launched(fn, launch_pdl(pages_reserve_kernel, dim3(kCluster), dim3(kThreads), 0, static_cast<cudaStream_t>(stream), 0, a));
}

PLDP_API pldp_status pldp_pages_compact(const pldp_page_table* table, int32_t* copies, int copies_cap, int32_t* n_copies,
                                        int32_t* used, void* workspace, size_t workspace_bytes, void* stream) {
    const char* fn = "pages_compact";
    CompactArgs a = {};
    pldp_status st = table_of(fn, table, &a.t);
    if (st != PLDP_OK) return st;
    if (copies_cap < a.t.n_pages / 2)
        return fail(PLDP_ERR_INVALID_ARG, "%s: room for %d moves, needs n_pages / 2 = %d", fn, copies_cap, a.t.n_pages / 2);
    if (!a.t.refs || !copies || !n_copies) return fail(PLDP_ERR_INVALID_ARG, "%s: null pointer", fn);
    if (reinterpret_cast<uintptr_t>(copies) & 7u) return fail(PLDP_ERR_INVALID_ARG, "%s: copies is not 8-byte aligned", fn);
    if ((st = check_workspace(fn, table, workspace, workspace_bytes)) != PLDP_OK) return st;
    a.copies = copies, a.n_copies = n_copies, a.used = used;
    a.head = static_cast<int32_t*>(workspace);
    a.to = a.head + 2;
    a.holes = a.to + a.t.n_pages;
    a.movers = a.holes + a.t.n_pages / 2 + 1;
    auto s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = launch_pdl(pages_compact_kernel, dim3(kCluster), dim3(kThreads), 0, s, 0, a);
    if (e != cudaSuccess || a.t.B == 0) return launched(fn, e);
    return launched(fn, launch_pdl(pages_moved_kernel, entries_grid(a.t), dim3(kEntryThreads), 0, s, 0, a.t, a.head, a.to));
}

PLDP_API pldp_status pldp_cache_copy_pages(const pldp_cache* cache, const int32_t* copies, int n, const int32_t* n_copies,
                                           void* stream) {
    const char* fn = "cache_copy_pages";
    if (!cache) return fail(PLDP_ERR_INVALID_ARG, "%s: null cache", fn);
    if (n < 0) return fail(PLDP_ERR_INVALID_ARG, "%s: n < 0", fn);
    CopyArgs a = {};
    const pldp_status st = cache_view(fn, *cache, 1, &a.c);
    if (st != PLDP_OK) return st;
    if (n == 0) return PLDP_OK;
    if (!copies) return fail(PLDP_ERR_INVALID_ARG, "%s: null pointer", fn);
    a.copies = copies, a.n_copies = n_copies, a.n = n;
    a.e4m3 = cache->dtype == PLDP_E4M3;
    // positions and heads by ascending stride; what lies side by side is one run
    const bool head_first = a.c.heads > 1 && (a.c.page_size == 1 || a.c.head_stride < a.c.pos_stride);
    a.inner = head_first ? a.c.heads : a.c.page_size;
    a.runs = static_cast<int64_t>(a.c.heads) * a.c.page_size;
    a.inner_stride = head_first ? a.c.head_stride : a.c.pos_stride;
    a.outer_stride = head_first ? a.c.pos_stride : a.c.head_stride;
    a.run = a.c.vec_bytes;
    if (a.inner == 1 || a.inner_stride == a.run) {
        a.run *= a.inner, a.runs /= a.inner;
        a.inner = a.runs, a.inner_stride = a.outer_stride;
        if (a.runs == 1 || a.inner_stride == a.run) a.run *= a.runs, a.runs = a.inner = 1;
    }
    a.pieces = (a.run * a.runs + kPiece - 1) / kPiece;
    const int64_t items = static_cast<int64_t>(n) * 2 * a.pieces, most = static_cast<int64_t>(8) * sm_count();
    return launched(fn, launch_pdl(copy_pages_kernel, dim3(static_cast<unsigned>(items < most ? items : most)), dim3(kCopyThreads), 0,
                                   static_cast<cudaStream_t>(stream), 0, a));
}

}  // extern "C"
