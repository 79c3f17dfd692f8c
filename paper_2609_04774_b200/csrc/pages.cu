// The care of the pages of a paged cache: extend, evict, free, fork, compact, copy.
//
// A pool's state is one reference count per page (0: free); page tables and lengths live on the device, so a serving step
// can be captured into a graph.  Whatever hands out pages takes the free ones with the lowest ids, in the order of the rows that
// ask, so the result is a pure function of the inputs.
//
// Choosing pages is a prefix sum over the rows' needs and one over the pool's counts.  One CTA of 1024 threads does both:
// the counts are 4 bytes a page (64 KB for a pool of a million tokens in pages of 64), the scan stops at the last page needed, and a
// second CTA would cost a grid-wide wait that is longer than the scan.  Extend for one token of 64 rows takes 5.2 us (4.6 without the look at
// what the entries hold), for a prompt of 2048 pages 15 us: a warp walks a long row together, 32 entries at a time.  Moving pages is HBM-bound (2x the moved bytes): the
// list of moves stays in the workspace, a second launch (set up while the first one runs) copies them for all layers, 32 KB per CTA step
// with eight 16-byte vectors in flight per thread.  1 GB of moved pages: 171 us with the choosing and the tables, 6.1 TB/s; with four
// vectors 174, with eight CTAs per SM in one wave 184.
#include <algorithm>

#include "device_util.cuh"
#include "internal.h"

using namespace cpattn;

namespace {

constexpr int kMetaThreads = 1024;
constexpr int kScanItems = 8;                             // counts per thread and step of the free-page scan
constexpr int kScanStep = kMetaThreads * kScanItems;
constexpr int kCopyThreads = 256;
constexpr int kCopyVectors = 8;                           // 16-byte vectors in flight per thread
constexpr int kCopyCtas = 32;                             // most CTAs of a copy launch per SM: four waves even out what fixed shares do not
constexpr int kPieceVectors = kCopyThreads * kCopyVectors;

struct Move {
    int32_t src, dst, n_tok, pad;
};
static_assert(sizeof(Move) == 16, "Move layout");

// Workspace: header {n_moves}, then the moves, then a list of page ids (free pages chosen, or holes).
constexpr size_t kPagesHeader = 256;
struct PagesLayout {
    size_t moves, ids, total;
};
PagesLayout pages_layout(int64_t num_pages, int64_t n) {
    PagesLayout l;
    l.moves = kPagesHeader;
    l.ids = l.moves + (size_t)std::max<int64_t>(num_pages, n) * sizeof(Move);
    l.total = (l.ids + (size_t)num_pages * sizeof(int32_t) + 255) / 256 * 256;
    return l;
}

struct PoolGeom {
    int64_t num_pages, stride_page, stride_tok, stride_head;   // bytes
    int32_t page_size, page_shift, Hkv, row_vec_shift;         // row_vec_shift: log2(16-byte vectors per head row)
    int32_t n_layers, contiguous;                              // contiguous: the tokens of a page are one run of bytes
};
struct LayerPtrs {
    void* k[CP_POOL_MAX_LAYERS];
    void* v[CP_POOL_MAX_LAYERS];
};

// Exclusive prefix sum of one value per thread over the CTA; `total` is the sum.  Two barriers.
template <typename T>
__device__ __forceinline__ T block_scan(T x, int64_t* scratch, T& total) {
    T* warp_sums = reinterpret_cast<T*>(scratch);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    T inc = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const T y = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += y;
    }
    __syncthreads();                                       // the previous use of the scratch is over
    if (lane == 31) warp_sums[warp] = inc;
    __syncthreads();
    T sums = warp_sums[lane];                              // kMetaThreads / 32 = 32 warps: one sum per lane, scanned by every warp
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const T y = __shfl_up_sync(0xffffffffu, sums, o);
        if (lane >= o) sums += y;
    }
    total = __shfl_sync(0xffffffffu, sums, 31);
    const T before = __shfl_sync(0xffffffffu, sums, warp > 0 ? warp - 1 : 0);
    return (warp > 0 ? before : 0) + inc - x;
}
static_assert(kMetaThreads == 1024, "block_scan: one warp sum per lane");

// The ids of the `want` lowest pages of [begin, end) whose count is zero (kFree) or not (!kFree), ascending: emit(rank, page) is
// called once for each.  Returns how many there are (at most `want`).  Every thread of the CTA calls it with the same arguments.
template <bool kFree, typename Emit>
__device__ __forceinline__ int32_t scan_pages(const int32_t* __restrict__ refcount, int32_t begin, int32_t end, int64_t want_all, int64_t* scratch,
                                              Emit emit) {
    const int32_t want = (int32_t)min(want_all, (int64_t)end);
    int32_t found = 0;
    // counts of this thread's pages of a step as a bit mask: bit i set if page base + i is one of those looked for
    auto fetch = [&](int64_t base) {
        int32_t c[kScanItems];
        const int64_t at = base + (int64_t)threadIdx.x * kScanItems;
#pragma unroll
        for (int i = 0; i < kScanItems; ++i) c[i] = at + i < end ? refcount[at + i] : (kFree ? 1 : 0);
        uint32_t hit = 0;
#pragma unroll
        for (int i = 0; i < kScanItems; ++i) hit |= (uint32_t)((c[i] <= 0) == kFree) << i;
        return hit;
    };
    for (int64_t base = begin; base < end && found < want; base += kScanStep) {
        uint32_t hit = fetch(base);
        int32_t total;
        int32_t rank = found + block_scan<int32_t>(__popc(hit), scratch, total);
        while (hit != 0 && rank < want) {
            const int i = __ffs(hit) - 1;
            hit &= hit - 1;
            emit(rank++, (int32_t)(base + (int64_t)threadIdx.x * kScanItems + i));
        }
        found += total;
    }
    return min(found, want);
}

// Entries [first, first + count) of a row are those that [kv_len, kv_len + add) needs beyond the pages that hold tokens; count -1: the
// request cannot be served.
struct Span {
    int64_t first, count;
};
__device__ __forceinline__ Span span_of(int32_t len, int32_t add, int page_shift, int64_t capacity) {
    if (len < 0 || add < 0 || (int64_t)len + add > capacity) return {0, -1};
    const int64_t m = (1ll << page_shift) - 1;
    const int64_t first = ((int64_t)len + m) >> page_shift;
    return {first, (((int64_t)len + add + m) >> page_shift) - first};
}

// An entry behind a row's end may name a page still (the row was longer before: rejected draft tokens).  The row's own page is used again; of
// one that is shared only the reference is given up, later (give_up_shared: all decisions look at the counts as the call found them); one
// that names no used page counts as -1.  Returns whether the entry needs a fresh page.
__device__ __forceinline__ bool settle_entry(int32_t* entry, int32_t page, const int32_t* refcount, int64_t num_pages, bool& shared) {
    if (page == -1) return true;
    const int32_t count = page >= 0 && page < num_pages ? refcount[page] : 0;
    if (count == 1) return false;
    *entry = count > 1 ? -2 - page : -1;
    shared |= count > 1;
    return true;
}
__device__ __forceinline__ void give_up_shared(int32_t* entry, int32_t mark, int32_t* refcount) {
    if (mark >= -1) return;
    atomicSub(refcount + (-2 - mark), 1);
    *entry = -1;
}

// Calls f(entry, its value) -> bool for the entries of this lane's span and returns how often it was true.  Long spans (prompts) are walked by
// the warp together, kBatch loads in flight: every lane of it makes the call.
constexpr int kOwnEntries = 4;
template <typename F>
__device__ __forceinline__ int64_t count_entries(int32_t* row, const Span& sp, F f) {
    constexpr int kBatch = 8;
    const int lane = threadIdx.x & 31;
    int64_t n = 0;
    if (sp.count <= kOwnEntries)
        for (int i = 0; i < sp.count; ++i) n += f(row + sp.first + i, row[sp.first + i]);
    for (uint32_t todo = __ballot_sync(0xffffffffu, sp.count > kOwnEntries); todo != 0; todo &= todo - 1) {
        const int src = __ffs(todo) - 1;
        int32_t* at = reinterpret_cast<int32_t*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(row + sp.first), src));
        const int64_t count = __shfl_sync(0xffffffffu, (long long)sp.count, src);
        int32_t hits = 0;
        for (int64_t i0 = lane; i0 < count; i0 += 32 * kBatch) {
            int32_t value[kBatch];
#pragma unroll
            for (int i = 0; i < kBatch; ++i) value[i] = i0 + 32 * i < count ? at[i0 + 32 * i] : -1;
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                if (i0 + 32 * i < count) hits += f(at + i0 + 32 * i, value[i]);
        }
        hits = __reduce_add_sync(0xffffffffu, hits);
        if (lane == src) n = hits;
    }
    return n;
}

// The entries of this lane's span that hold -1, n of them, take the pages ids[0 .. n).  Every lane of the warp makes the call.
__device__ __forceinline__ void fill_entries(int32_t* row, const Span& sp, int64_t n, const int32_t* ids, int32_t* refcount) {
    const int lane = threadIdx.x & 31;
    if (sp.count <= kOwnEntries)
        for (int i = 0; i < sp.count; ++i)
            if (row[sp.first + i] == -1) {
                row[sp.first + i] = *ids;
                refcount[*ids++] = 1;
            }
    for (uint32_t todo = __ballot_sync(0xffffffffu, sp.count > kOwnEntries && n > 0); todo != 0; todo &= todo - 1) {
        const int src = __ffs(todo) - 1;
        int32_t* at = reinterpret_cast<int32_t*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(row + sp.first), src));
        const int32_t* next = reinterpret_cast<const int32_t*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(ids), src));
        const int64_t count = __shfl_sync(0xffffffffu, (long long)sp.count, src);
        const bool all = __shfl_sync(0xffffffffu, (int)(n == sp.count), src);
        for (int64_t i0 = 0; i0 < count; i0 += 32) {
            const int64_t i = i0 + lane;
            const bool take = i < count && (all || at[i] == -1);
            const uint32_t takers = __ballot_sync(0xffffffffu, take);
            if (take) {
                const int32_t page = next[__popc(takers & ((1u << lane) - 1))];
                at[i] = page;
                refcount[page] = 1;
            }
            next += __popc(takers);
        }
    }
}

__global__ void __launch_bounds__(kMetaThreads, 1)      // the only CTA: registers for all of it
extend_kernel(PoolGeom g, int32_t* refcount, int32_t* table, int64_t rows, int64_t stride, int32_t* kv_len, const int32_t* add, int32_t* ids,
              int32_t* status) {
    __shared__ int64_t scratch[kMetaThreads / 32];
    const int64_t capacity = stride << g.page_shift;
    auto span = [&](int64_t r) { return r < rows ? span_of(kv_len[r], add[r], g.page_shift, capacity) : Span{0, 0}; };
    // pages wanted by all rows; those of the first kMetaThreads rows stay in registers
    int64_t mine = 0, total, first_need = 0;
    const Span first_span = span(threadIdx.x);
    bool shared = false;
    for (int64_t r0 = 0; r0 < rows; r0 += kMetaThreads) {
        const int64_t r = r0 + threadIdx.x;
        const int64_t n = count_entries(table + r * stride, r0 == 0 ? first_span : span(r),
                                        [&](int32_t* e, int32_t v) { return settle_entry(e, v, refcount, g.num_pages, shared); });
        if (r0 == 0) first_need = n;
        mine += n;
    }
    if (__syncthreads_or(shared)) {
        for (int64_t r0 = 0; r0 < rows; r0 += kMetaThreads) {
            const int64_t r = r0 + threadIdx.x;
            count_entries(table + r * stride, span(r), [&](int32_t* e, int32_t v) { give_up_shared(e, v, refcount); return false; });
        }
        __syncthreads();
    }
    block_scan<int64_t>(mine, scratch, total);
    const int64_t got = total > 0 ? scan_pages<true>(refcount, 0, (int32_t)g.num_pages, total, scratch, [&](int32_t k, int32_t page) { ids[k] = page; }) : 0;
    __syncthreads();
    // rows in order take theirs; a row that does not get all its pages gets none and keeps its length
    int64_t base = 0;
    for (int64_t r0 = 0; r0 < rows; r0 += kMetaThreads) {
        const int64_t r = r0 + threadIdx.x;
        int32_t* row = table + r * stride;
        const Span sp = r0 == 0 ? first_span : span(r);
        const int64_t n = r0 == 0 ? first_need : count_entries(row, sp, [&](int32_t*, int32_t v) { return v == -1; });
        int64_t step;
        const int64_t at = base + block_scan<int64_t>(n, scratch, step);
        base += step;
        const bool served = r < rows && sp.count >= 0 && (n == 0 || at + n <= got);
        fill_entries(row, served ? sp : Span{0, 0}, n, ids + at, refcount);
        if (served) kv_len[r] += add[r];
        else if (r < rows) report_status(status, CP_ERR_BOUNDS, r, sp.count < 0 ? add[r] : -1);
    }
}

// One table entry is given up: -1 is written first, so an entry named twice is released once.
__device__ __forceinline__ void release_entry(int32_t* entry, int32_t* refcount, int64_t num_pages, int64_t index, int32_t* status) {
    const int32_t page = atomicExch(entry, -1);
    if (page == -1) return;
    if (page < 0 || page >= num_pages) {
        report_status(status, CP_ERR_BOUNDS, index, page);
        return;
    }
    if (atomicSub(refcount + page, 1) <= 0) {              // the page was free already: its count stays what it was
        atomicAdd(refcount + page, 1);
        report_status(status, CP_ERR_BOUNDS, index, page);
    }
}

// The next token of row r sits at position kv_len and sees keys from kv_len + 1 - window on, and the sinks: pages that hold
// none of these, now or later, are given back.
__global__ void __launch_bounds__(kCopyThreads)
evict_kernel(PoolGeom g, int32_t* refcount, int32_t* table, int64_t rows, int64_t stride, const int32_t* kv_len, int64_t window, int64_t sinks,
             int32_t* status) {
    const int64_t first = (sinks + g.page_size - 1) >> g.page_shift;
    const int64_t r = blockIdx.y + (int64_t)blockIdx.z * gridDim.y;
    if (r >= rows) return;
    const int64_t len = kv_len[r];
    const int64_t last = len + 1 > window ? min((len + 1 - window) >> g.page_shift, stride) : 0;
    for (int64_t e = first + (int64_t)blockIdx.x * kCopyThreads + threadIdx.x; e < last; e += (int64_t)gridDim.x * kCopyThreads)
        if (table[r * stride + e] != -1) release_entry(table + r * stride + e, refcount, g.num_pages, r * stride + e, status);
}

__global__ void __launch_bounds__(kCopyThreads)
free_kernel(PoolGeom g, int32_t* refcount, int32_t* table, int64_t rows, int64_t stride, int32_t* kv_len, const int32_t* which, int32_t* status) {
    const int64_t r = which[blockIdx.x];
    if (r < 0 || r >= rows) {
        if (threadIdx.x == 0) report_status(status, CP_ERR_BOUNDS, blockIdx.x, r);
        return;
    }
    for (int64_t e = threadIdx.x; e < stride; e += kCopyThreads)
        if (table[r * stride + e] != -1) release_entry(table + r * stride + e, refcount, g.num_pages, r * stride + e, status);
    if (threadIdx.x == 0) kv_len[r] = 0;
}

// Fork, first launch: a fresh page for every child whose parent ends inside a page.  moves[i] = {parent's page, fresh page, tokens};
// dst -1: nothing to copy.  n_moves is the number of forks.
__device__ __forceinline__ bool fork_ok(const PoolGeom& g, int64_t rows, int64_t stride, const int32_t* kv_len, int32_t parent, int32_t child) {
    return parent >= 0 && parent < rows && child >= 0 && child < rows && parent != child && kv_len[parent] >= 0 &&
           kv_len[parent] <= (stride << g.page_shift);
}
__global__ void __launch_bounds__(kMetaThreads)
fork_choose_kernel(PoolGeom g, const int32_t* refcount, const int32_t* table, int64_t rows, int64_t stride, const int32_t* kv_len,
                   const int32_t* parent, const int32_t* child, int64_t n, int32_t* n_moves, Move* moves, int32_t* ids, int32_t* status) {
    let_next_launch_begin();
    __shared__ int64_t scratch[kMetaThreads / 32];
    auto tail = [&](int64_t i, int32_t& page, int32_t& used) {
        page = -1;
        used = 0;
        if (!fork_ok(g, rows, stride, kv_len, parent[i], child[i])) return false;
        const int32_t len = kv_len[parent[i]];
        used = len & (g.page_size - 1);
        if (used == 0) return false;
        page = table[parent[i] * stride + (len >> g.page_shift)];
        return page >= 0 && page < g.num_pages;
    };
    int64_t mine = 0, total;
    int32_t page, used;
    for (int64_t i = threadIdx.x; i < n; i += kMetaThreads) mine += tail(i, page, used) ? 1 : 0;
    block_scan<int64_t>(mine, scratch, total);
    const int64_t got = total > 0 ? scan_pages<true>(refcount, 0, (int32_t)g.num_pages, total, scratch, [&](int32_t k, int32_t id) { ids[k] = id; }) : 0;
    __syncthreads();
    int64_t base = 0;
    for (int64_t i0 = 0; i0 < n; i0 += kMetaThreads) {
        const int64_t i = i0 + threadIdx.x;
        page = -1;
        used = 0;
        const bool need = i < n && tail(i, page, used);
        int64_t step;
        const int64_t at = base + block_scan<int64_t>(need ? 1 : 0, scratch, step);
        base += step;
        if (i < n) {
            const bool served = need && at < got;
            // no page left, or the parent's partly filled page is not one of the pool
            if (!served && (need || used != 0)) report_status(status, CP_ERR_BOUNDS, i, need ? -1 : page);
            moves[i] = {need ? page : -1, served ? ids[at] : -1, need ? used : 0, 0};
        }
    }
    if (threadIdx.x == 0) *n_moves = (int32_t)n;
}

// Copies the first n_tok tokens of page src to page dst, K and V of every layer, for the moves of the list: CTA steps of kPieceVectors.
__device__ __forceinline__ void copy_moves(const PoolGeom& g, const LayerPtrs& layers, const Move* moves, int64_t n_moves, int64_t cta, int64_t ctas) {
    const int32_t vec_per_tok = g.Hkv << g.row_vec_shift;                                            // at most 4096 * 16
    const uint32_t pieces = ((vec_per_tok << g.page_shift) + kPieceVectors - 1) / kPieceVectors;     // of a whole page, at most 2^13
    const uint32_t per_move = pieces * g.n_layers * 2;                                               // at most 2^21
    int64_t m = cta / per_move;
    uint32_t rest = (uint32_t)(cta - m * per_move);
    const int64_t m_step = ctas / per_move;
    const uint32_t rest_step = (uint32_t)(ctas - m_step * per_move);
    for (; m < n_moves; m += m_step, rest += rest_step) {
        if (rest >= per_move) {
            rest -= per_move;
            if (++m >= n_moves) break;
        }
        const Move mv = moves[m];
        if (mv.dst < 0) continue;
        const uint32_t lv = rest / pieces;
        const int32_t v0 = (int32_t)(rest - lv * pieces) * kPieceVectors, n_vec = vec_per_tok * mv.n_tok;
        if (v0 >= n_vec) continue;
        uint8_t* pool = static_cast<uint8_t*>((lv & 1) ? layers.v[lv >> 1] : layers.k[lv >> 1]);
        const uint8_t* src = pool + mv.src * g.stride_page;
        uint8_t* dst = pool + mv.dst * g.stride_page;
        uint4 x[kCopyVectors];
        int64_t off[kCopyVectors];
#pragma unroll
        for (int i = 0; i < kCopyVectors; ++i) {
            const int32_t v = v0 + i * kCopyThreads + threadIdx.x;
            off[i] = -1;
            if (v < n_vec) {
                if (g.contiguous) {
                    off[i] = (int64_t)v * 16;
                } else {
                    const int32_t row = v >> g.row_vec_shift, c = v - (row << g.row_vec_shift);
                    const int32_t tok = row / g.Hkv;
                    off[i] = tok * g.stride_tok + (row - tok * g.Hkv) * g.stride_head + c * 16;
                }
                x[i] = *reinterpret_cast<const uint4*>(src + off[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < kCopyVectors; ++i)
            if (off[i] >= 0) *reinterpret_cast<uint4*>(dst + off[i]) = x[i];
    }
}

// Fork, second launch: blocks [0, n) write the children's rows and take the references, the others copy.
__global__ void __launch_bounds__(kCopyThreads)
fork_apply_kernel(PoolGeom g, const __grid_constant__ LayerPtrs layers, int32_t* refcount, int32_t* table, int64_t rows, int64_t stride,
                  int32_t* kv_len, const int32_t* parent, const int32_t* child, int64_t n, const int32_t* n_moves, const Move* moves,
                  int32_t* status) {
    wait_for_launch_before();
    if (blockIdx.x >= n) {
        copy_moves(g, layers, moves, *n_moves, blockIdx.x - n, gridDim.x - n);
        return;
    }
    const int64_t i = blockIdx.x;
    const int32_t p = parent[i], c = child[i];
    if (!fork_ok(g, rows, stride, kv_len, p, c)) {
        if (threadIdx.x == 0) report_status(status, CP_ERR_BOUNDS, i, c);
        return;
    }
    const int32_t len = kv_len[p];
    const int64_t full = len >> g.page_shift;
    const Move mv = moves[i];
    for (int64_t e = threadIdx.x; e < stride; e += kCopyThreads) {
        int32_t page = -1;
        if (e < full) {
            page = table[p * stride + e];
            if (page >= 0 && page < g.num_pages) atomicAdd(refcount + page, 1);
            else if (page != -1) {                         // evicted entries (-1) stay what they are; anything else is an error
                report_status(status, CP_ERR_BOUNDS, p * stride + e, page);
                page = -1;
            }
        } else if (e == full && mv.dst >= 0) {
            page = mv.dst;
            refcount[page] = 1;
        }
        table[c * stride + e] = page;
    }
    // without a page for its partly filled tail the child ends with the last full page
    if (threadIdx.x == 0) kv_len[c] = (len & (g.page_size - 1)) && mv.dst < 0 ? (int32_t)(full << g.page_shift) : len;
}

// Compact, first launch.  n_live pages are in use; the k-th used page at or behind n_live moves to the k-th hole before it.
__global__ void __launch_bounds__(kMetaThreads)
compact_choose_kernel(PoolGeom g, int32_t* refcount, int32_t* page_map, int32_t* n_live_out, int32_t* n_moves, Move* moves, int32_t* ids) {
    let_next_launch_begin();
    __shared__ int64_t scratch[kMetaThreads / 32];
    const int64_t N = g.num_pages;
    int64_t mine = 0, n_live;
    for (int64_t i = threadIdx.x; i < N; i += kMetaThreads) {
        const bool used = refcount[i] > 0;
        mine += used;
        page_map[i] = used ? (int32_t)i : -1;              // movers are overwritten below
    }
    block_scan<int64_t>(mine, scratch, n_live);
    const int64_t holes = scan_pages<true>(refcount, 0, (int32_t)n_live, n_live, scratch, [&](int32_t k, int32_t page) { ids[k] = page; });
    __syncthreads();
    // as many used pages lie at or behind n_live as there are holes before it
    scan_pages<false>(refcount, (int32_t)n_live, (int32_t)N, holes, scratch, [&](int32_t k, int32_t page) {
        const int32_t dst = ids[k];
        moves[k] = {page, dst, g.page_size, 0};
        page_map[page] = dst;
    });
    __syncthreads();
    for (int64_t k = threadIdx.x; k < holes; k += kMetaThreads) {
        const Move mv = moves[k];
        refcount[mv.dst] = refcount[mv.src];
        refcount[mv.src] = 0;
    }
    if (threadIdx.x == 0) {
        *n_live_out = (int32_t)n_live;
        *n_moves = (int32_t)holes;
    }
}

// Compact, second launch: the tables follow the map, the pages move.
__global__ void __launch_bounds__(kCopyThreads)
compact_apply_kernel(PoolGeom g, const __grid_constant__ LayerPtrs layers, int32_t* table, int64_t entries, const int32_t* page_map,
                     const int32_t* n_moves, const Move* moves) {
    wait_for_launch_before();
    for (int64_t e = (int64_t)blockIdx.x * kCopyThreads + threadIdx.x; e < entries; e += (int64_t)gridDim.x * kCopyThreads) {
        const int32_t page = table[e];
        if (page >= 0 && page < g.num_pages) {
            const int32_t to = page_map[page];
            if (to >= 0 && to != page) table[e] = to;      // an entry that names a free page stays
        }
    }
    copy_moves(g, layers, moves, *n_moves, blockIdx.x, gridDim.x);
}

// Listed copies: the ids are checked while the list is made.
__global__ void __launch_bounds__(kCopyThreads)
copy_list_kernel(PoolGeom g, const int32_t* src, const int32_t* dst, int64_t n, int32_t* n_moves, Move* moves, int32_t* status) {
    let_next_launch_begin();
    for (int64_t i = (int64_t)blockIdx.x * kCopyThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kCopyThreads) {
        const int32_t a = src[i], b = dst[i];
        const bool bad_a = a < 0 || a >= g.num_pages, bad = bad_a || b < 0 || b >= g.num_pages;
        if (bad) report_status(status, CP_ERR_BOUNDS, i, bad_a ? a : b);
        moves[i] = {a, (bad || a == b) ? -1 : b, g.page_size, 0};
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) *n_moves = (int32_t)n;
}
__global__ void __launch_bounds__(kCopyThreads)
copy_apply_kernel(PoolGeom g, const __grid_constant__ LayerPtrs layers, const int32_t* n_moves, const Move* moves) {
    wait_for_launch_before();
    copy_moves(g, layers, moves, *n_moves, blockIdx.x, gridDim.x);
}

int check_pool(const cp_page_pool* p, bool copies, PoolGeom& g, LayerPtrs* layers, const char* who) {
    if (!p || p->num_pages < 1) return set_error(CP_ERR_INVALID_ARG, "%s: pool is NULL or empty", who);
    if (p->page_size != 16 && p->page_size != 32 && p->page_size != 64 && p->page_size != 128)
        return set_error(CP_ERR_UNSUPPORTED, "%s: page_size=%d; supported: pages of 16, 32, 64 or 128 tokens", who, p->page_size);
    if (p->num_pages > 0x7ffffff0ll) return set_error(CP_ERR_UNSUPPORTED, "%s: more than 2^31 pages", who);
    g = PoolGeom{};
    g.num_pages = p->num_pages;
    g.page_size = p->page_size;
    g.page_shift = log2_exact(p->page_size);
    if (!copies) return CP_OK;
    if (p->n_layers < 1 || !p->k || !p->v || p->Hkv < 1)
        return set_error(CP_ERR_INVALID_ARG, "%s: pool without layers or heads", who);
    if (p->n_layers > CP_POOL_MAX_LAYERS || p->Hkv > 4096)
        return set_error(CP_ERR_UNSUPPORTED, "%s: %d layers (at most %d), %d heads", who, p->n_layers, CP_POOL_MAX_LAYERS, p->Hkv);
    if (p->row_bytes != 256 && p->row_bytes != 128)
        return set_error(CP_ERR_UNSUPPORTED, "%s: row_bytes=%d; a head row has 256 (bf16) or 128 bytes (E4M3)", who, p->row_bytes);
    if (((p->stride_page | p->stride_tok | p->stride_head) & 15) || p->stride_page < 1 || p->stride_tok < 1 || p->stride_head < 1)
        return set_error(CP_ERR_UNSUPPORTED, "%s: strides must be positive multiples of 16 bytes", who);
    for (int32_t l = 0; l < p->n_layers; ++l) {
        if (!p->k[l] || !p->v[l]) return set_error(CP_ERR_INVALID_ARG, "%s: layer %d has a null pointer", who, l);
        if (((uintptr_t)p->k[l] | (uintptr_t)p->v[l]) & 15)
            return set_error(CP_ERR_UNSUPPORTED, "%s: k and v of layer %d must be 16-byte aligned", who, l);
        layers->k[l] = p->k[l];
        layers->v[l] = p->v[l];
    }
    g.stride_page = p->stride_page;
    g.stride_tok = p->stride_tok;
    g.stride_head = p->stride_head;
    g.Hkv = p->Hkv;
    g.row_vec_shift = p->row_bytes == 256 ? 4 : 3;
    g.n_layers = p->n_layers;
    g.contiguous = p->stride_head == p->row_bytes && p->stride_tok == (int64_t)p->Hkv * p->row_bytes;
    return CP_OK;
}

int check_table(const int32_t* table, int64_t rows, int64_t stride, const PoolGeom& g, const char* who) {
    if (!table || rows < 1 || stride < 1) return set_error(CP_ERR_INVALID_ARG, "%s: no page table, or rows=%lld stride=%lld", who,
                                                           (long long)rows, (long long)stride);
    if (rows > 0x7fffffffll || stride > (0x7fffffffll >> g.page_shift) || rows * stride > (1ll << 40))
        return set_error(CP_ERR_UNSUPPORTED, "%s: a page table of %lld x %lld entries", who, (long long)rows, (long long)stride);
    return CP_OK;
}

int check_workspace(void* ws, size_t bytes, int64_t num_pages, int64_t n, const char* who) {
    const size_t need = pages_layout(num_pages, n).total;
    if (!ws || ((uintptr_t)ws & 255) || bytes < need)
        return set_error(CP_ERR_WORKSPACE, "%s: workspace %p of %zu bytes; need %zu bytes, 256-byte aligned", who, ws, bytes, need);
    return CP_OK;
}

// CTAs of a copy launch: enough for the largest list, at most kCopyCtas per SM.
int copy_grid(const cp_ctx* ctx, const PoolGeom& g, int64_t moves) {
    const int64_t pieces = ((((int64_t)g.Hkv << g.row_vec_shift) << g.page_shift) + kPieceVectors - 1) / kPieceVectors * g.n_layers * 2;
    const int64_t most = (int64_t)ctx->num_sms * kCopyCtas;
    return (int)std::max<int64_t>(1, moves > most / pieces ? most : std::min(most, moves * pieces));
}

}  // namespace

extern "C" size_t cp_workspace_bytes_pages(int64_t num_pages, int64_t n) {
    if (num_pages < 1 || num_pages > 0x7ffffff0ll || n < 0 || n > 0x7fffffffll) return 0;
    return pages_layout(num_pages, n).total;
}

extern "C" int cp_pages_extend(cp_ctx* ctx, const cp_page_pool* pool, int32_t* refcount, int32_t* page_table, int64_t table_rows,
                               int64_t table_stride, int32_t* kv_len, const int32_t* new_tokens, void* workspace,
                               size_t workspace_bytes, void* stream) {
    const char* who = "cp_pages_extend";
    PoolGeom g;
    if (int rc = check_pool(pool, false, g, nullptr, who)) return rc;
    if (int rc = check_table(page_table, table_rows, table_stride, g, who)) return rc;
    if (!refcount || !kv_len || !new_tokens) return set_error(CP_ERR_INVALID_ARG, "%s: null pointer", who);
    if (int rc = check_workspace(workspace, workspace_bytes, pool->num_pages, 0, who)) return rc;
    if (!ctx) return set_error(CP_ERR_INVALID_ARG, "%s: ctx is NULL", who);
    DeviceGuard guard(ctx->device);
    if (guard.rc()) return guard.rc();
    const PagesLayout l = pages_layout(pool->num_pages, 0);
    extend_kernel<<<1, kMetaThreads, 0, static_cast<cudaStream_t>(stream)>>>(
        g, refcount, page_table, table_rows, table_stride, kv_len, new_tokens,
        reinterpret_cast<int32_t*>(static_cast<uint8_t*>(workspace) + l.ids), ctx->d_status);
    return check_cuda(cudaGetLastError(), who);
}

extern "C" int cp_pages_evict(cp_ctx* ctx, const cp_page_pool* pool, int32_t* refcount, int32_t* page_table, int64_t table_rows,
                              int64_t table_stride, const int32_t* kv_len, int64_t window, int64_t sinks, void* stream) {
    const char* who = "cp_pages_evict";
    PoolGeom g;
    if (int rc = check_pool(pool, false, g, nullptr, who)) return rc;
    if (int rc = check_table(page_table, table_rows, table_stride, g, who)) return rc;
    if (!refcount || !kv_len || window < 1 || sinks < 0)
        return set_error(CP_ERR_INVALID_ARG, "%s: null pointer, window=%lld or sinks=%lld", who, (long long)window, (long long)sinks);
    if (!ctx) return set_error(CP_ERR_INVALID_ARG, "%s: ctx is NULL", who);
    DeviceGuard guard(ctx->device);
    if (guard.rc()) return guard.rc();
    sinks = std::min<int64_t>(sinks, 1ll << 40);
    const int64_t first = (sinks + g.page_size - 1) >> g.page_shift;
    if (first >= table_stride) return CP_OK;               // the sinks cover every row
    const unsigned x = (unsigned)std::min<int64_t>((table_stride - first + kCopyThreads - 1) / kCopyThreads, 64);
    const unsigned y = (unsigned)std::min<int64_t>(table_rows, 32768), z = (unsigned)((table_rows + y - 1) / y);
    if (z > 65535) return set_error(CP_ERR_UNSUPPORTED, "%s: %lld rows", who, (long long)table_rows);
    evict_kernel<<<dim3(x, y, z), kCopyThreads, 0, static_cast<cudaStream_t>(stream)>>>(
        g, refcount, page_table, table_rows, table_stride, kv_len, window, sinks, ctx->d_status);
    return check_cuda(cudaGetLastError(), who);
}

extern "C" int cp_pages_free(cp_ctx* ctx, const cp_page_pool* pool, int32_t* refcount, int32_t* page_table, int64_t table_rows,
                             int64_t table_stride, int32_t* kv_len, const int32_t* rows, int32_t n, void* stream) {
    const char* who = "cp_pages_free";
    PoolGeom g;
    if (int rc = check_pool(pool, false, g, nullptr, who)) return rc;
    if (int rc = check_table(page_table, table_rows, table_stride, g, who)) return rc;
    if (!refcount || !kv_len || (!rows && n > 0) || n < 0) return set_error(CP_ERR_INVALID_ARG, "%s: null pointer or n=%d", who, n);
    if (!ctx) return set_error(CP_ERR_INVALID_ARG, "%s: ctx is NULL", who);
    if (n == 0) return CP_OK;
    DeviceGuard guard(ctx->device);
    if (guard.rc()) return guard.rc();
    free_kernel<<<(unsigned)n, kCopyThreads, 0, static_cast<cudaStream_t>(stream)>>>(g, refcount, page_table, table_rows, table_stride,
                                                                                   kv_len, rows, ctx->d_status);
    return check_cuda(cudaGetLastError(), who);
}

extern "C" int cp_pages_fork(cp_ctx* ctx, const cp_page_pool* pool, int32_t* refcount, int32_t* page_table, int64_t table_rows,
                             int64_t table_stride, int32_t* kv_len, const int32_t* parent, const int32_t* child, int32_t n,
                             void* workspace, size_t workspace_bytes, void* stream) {
    const char* who = "cp_pages_fork";
    PoolGeom g;
    LayerPtrs layers;
    if (int rc = check_pool(pool, true, g, &layers, who)) return rc;
    if (int rc = check_table(page_table, table_rows, table_stride, g, who)) return rc;
    if (n > (1 << 24)) return set_error(CP_ERR_UNSUPPORTED, "%s: %d forks in one call", who, n);
    if (!refcount || !kv_len || (n > 0 && (!parent || !child)) || n < 0) return set_error(CP_ERR_INVALID_ARG, "%s: null pointer or n=%d", who, n);
    if (int rc = check_workspace(workspace, workspace_bytes, pool->num_pages, n, who)) return rc;
    if (!ctx) return set_error(CP_ERR_INVALID_ARG, "%s: ctx is NULL", who);
    if (n == 0) return CP_OK;
    DeviceGuard guard(ctx->device);
    if (guard.rc()) return guard.rc();
    const PagesLayout l = pages_layout(pool->num_pages, n);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    int32_t* n_moves = reinterpret_cast<int32_t*>(ws);
    Move* moves = reinterpret_cast<Move*>(ws + l.moves);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    fork_choose_kernel<<<1, kMetaThreads, 0, s>>>(g, refcount, page_table, table_rows, table_stride, kv_len, parent, child, n, n_moves,
                                                  moves, reinterpret_cast<int32_t*>(ws + l.ids), ctx->d_status);
    if (int rc = check_cuda(cudaGetLastError(), who)) return rc;
    return launch_behind(fork_apply_kernel, dim3((unsigned)n + copy_grid(ctx, g, n)), kCopyThreads, s, who, g, layers, refcount, page_table,
                         table_rows, table_stride, kv_len, parent, child, (int64_t)n, (const int32_t*)n_moves, (const Move*)moves, ctx->d_status);
}

extern "C" int cp_pages_compact(cp_ctx* ctx, const cp_page_pool* pool, int32_t* refcount, int32_t* page_table, int64_t table_rows,
                                int64_t table_stride, int32_t* page_map, int32_t* n_live, void* workspace, size_t workspace_bytes,
                                void* stream) {
    const char* who = "cp_pages_compact";
    PoolGeom g;
    LayerPtrs layers;
    if (int rc = check_pool(pool, true, g, &layers, who)) return rc;
    if (int rc = check_table(page_table, table_rows, table_stride, g, who)) return rc;
    if (!refcount || !page_map || !n_live) return set_error(CP_ERR_INVALID_ARG, "%s: null pointer", who);
    if (int rc = check_workspace(workspace, workspace_bytes, pool->num_pages, 0, who)) return rc;
    if (!ctx) return set_error(CP_ERR_INVALID_ARG, "%s: ctx is NULL", who);
    DeviceGuard guard(ctx->device);
    if (guard.rc()) return guard.rc();
    const PagesLayout l = pages_layout(pool->num_pages, 0);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    int32_t* n_moves = reinterpret_cast<int32_t*>(ws);
    Move* moves = reinterpret_cast<Move*>(ws + l.moves);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    compact_choose_kernel<<<1, kMetaThreads, 0, s>>>(g, refcount, page_map, n_live, n_moves, moves, reinterpret_cast<int32_t*>(ws + l.ids));
    if (int rc = check_cuda(cudaGetLastError(), who)) return rc;
    return launch_behind(compact_apply_kernel, dim3(copy_grid(ctx, g, pool->num_pages)), kCopyThreads, s, who, g, layers, page_table,
                         table_rows * table_stride, (const int32_t*)page_map, (const int32_t*)n_moves, (const Move*)moves);
}

extern "C" int cp_pages_copy(cp_ctx* ctx, const cp_page_pool* pool, const int32_t* src, const int32_t* dst, int32_t n, void* workspace,
                             size_t workspace_bytes, void* stream) {
    const char* who = "cp_pages_copy";
    PoolGeom g;
    LayerPtrs layers;
    if (int rc = check_pool(pool, true, g, &layers, who)) return rc;
    if ((n > 0 && (!src || !dst)) || n < 0) return set_error(CP_ERR_INVALID_ARG, "%s: null pointer or n=%d", who, n);
    if (int rc = check_workspace(workspace, workspace_bytes, pool->num_pages, n, who)) return rc;
    if (!ctx) return set_error(CP_ERR_INVALID_ARG, "%s: ctx is NULL", who);
    if (n == 0) return CP_OK;
    DeviceGuard guard(ctx->device);
    if (guard.rc()) return guard.rc();
    const PagesLayout l = pages_layout(pool->num_pages, n);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    int32_t* n_moves = reinterpret_cast<int32_t*>(ws);
    Move* moves = reinterpret_cast<Move*>(ws + l.moves);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    copy_list_kernel<<<(unsigned)std::min<int64_t>((n + kCopyThreads - 1) / kCopyThreads, 256), kCopyThreads, 0, s>>>(g, src, dst, n, n_moves, moves,
                                                                                                                ctx->d_status);
    if (int rc = check_cuda(cudaGetLastError(), who)) return rc;
    return launch_behind(copy_apply_kernel, dim3(copy_grid(ctx, g, n)), kCopyThreads, s, who, g, layers, (const int32_t*)n_moves, (const Move*)moves);
}
