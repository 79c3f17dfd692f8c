// Decode attention: one or a few new tokens per request over a paged cache (bf16 or E4M3), full or with a sliding window and
// sinks; lengths and page tables are read on the device.
//
//   O = sum_j p_j v_j / sum_j p_j,   p_j = 2^(c q.k_j - m),   c = scale log2(e),   LSE = ln sum_j e^(scale q.k_j)
//
// HBM-bound: every visible key and value is read once (512 bytes a key and KV head in bf16, 256 in E4M3) and serves the n_q * G query
// rows of its head group, 4 * 128 flops a row: 8 flops a byte for 8 rows, which the legacy warp MMA (m16n8k16) covers many
// times over.  What counts is bytes in flight, so the kernel is built around the load stream:
//   - 8 warps a CTA, one or two CTAs per SM (Shape).  The work is the list of tiles of all (request, KV head, row group) units, cut into
//     equal runs, one per CTA, whatever the lengths; a unit counts four tiles more than it has, for its queries and its merge (ragged
//     batches of short requests: 95 us with one, 87 with two, 81 with four, 85 with eight).  A warp owns 16 keys of every tile and a
//     ring of slots that it fills with cp.async and reads by itself: no barrier in the loop, 128 KB in flight per SM, across
//     unit boundaries as well.
//   - Products with the keys as the M side: S^T[16 keys x 8 rows] = K Q^T, and O^T[16 dims x 8 rows] += V^T P^T, so 8 query rows
//     fill an MMA (with the rows on the M side half of it would be padding).  K goes through ldmatrix, V through its transposed form;
//     the weights turn from accumulator to operand layout with one movmatrix per 8 x 8 block.
//   - Every warp keeps its own running maximum and sum; the maximum is only raised (and O rescaled) when a score exceeds it by more
//     than 2^8, which one vote per 16 keys finds out.
//   - At the end of a unit's run the warps' partial results are merged, in a fixed order, through the ring slots that were just read.  A
//     unit that lies in one run is written out; the pieces of a cut unit go to the workspace as unnormalised fp32 rows with their
//     maximum and sum, and a second launch, set up under the first, joins them (done by the CTA that finishes last instead, a single
//     request took 18 us on the device against 10).
// E4M3: codes are widened exactly to fp16 in registers; the queries become fp16 after a power-of-two scaling per row (bf16's 8 bits of
// mantissa fit; what falls below 2^-24 of the row's largest is lost), weights are fp16 after a scaling by 2^7, so the
// result has fp16 weights (2^-11) where the bf16 cache has bf16 ones (2^-8).  Sums, maxima and accumulators are fp32.
//
// Measured (device time from a graph; a copy reaches 6.45 TB/s, reading alone somewhat more): 64 requests of 257..16384 keys, 32 / 8 heads: 177 us,
// 6.6 TB/s; E4M3 101 us, 5.8 TB/s; 128 requests with a window of 4096, 64 / 8 heads: 276 us, 6.7 TB/s, E4M3 158 us, 5.9 TB/s; four contexts of
// 100K..128K keys, four draft tokens each, 32 / 4 heads: 143 us, 6.2 TB/s, E4M3 140 us (bound by the fp16 widening and the fragments' shared-memory
// traffic); one request of 4097 keys: 9.7 us, the latency of two launches.  More than 32 rows per KV head are several units, each reading K and V
// (from L2 where it can): four contexts of 64K keys, four draft tokens, 64 / 4 heads: 170 us against 93 for 32 / 4, E4M3 160 against 99.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include <algorithm>

#include "device_util.cuh"
#include "internal.h"

using namespace cpattn;

namespace {

constexpr int kDim = 128;
constexpr int kGroups = 8;                                 // warps of a CTA: key groups of a tile, times heads
constexpr int kThreads = kGroups * 32;
constexpr int kSubKeys = 16;                               // keys of a group
constexpr int kJoinThreads = 256;
constexpr int kUnitCost = 4;                               // fixed cost of a unit in tiles (see Cursor)
constexpr float kLag = 8.0f;                               // the running maximum may lag by a factor 2^8
constexpr float kF16Shift = 7.0f;                          // fp16 weights carry 2^7: at most 2^15 with the lag
constexpr float kNoKey = -1.5e38f;                         // reference of a row that has seen no key: finite, so that hidden scores (-inf) give weight 0
// NT: query rows of a unit and KV head in blocks of 8; HP: KV heads of a unit, so a tile is 128 / HP keys of each.
// Up to 16 rows the queries' fragments stay in registers; the E4M3 form of up to 8 rows fits an SM twice (128 registers a thread, half
// the ring each).  With 32 rows the fragments are read from shared memory for every 16 keys.  Two warps per key group that share the
// rows and the ring slots were slower: 16 rows 190 us either way, E4M3 160 -> 175 us (every code is widened twice), 32 rows 147 -> 174 us.
// E4M3 rows are 128 bytes: two heads together make a token's loads 256 contiguous bytes, as they are in bf16 (the loads of one head alone
// reach 5.4 TB/s; 128 requests with a window 183 us with one head, 160 with two, 172 with four; bf16 278, 283 with two).
template <int NT, int HP, bool kFp8>
struct Shape {
    static constexpr int kCtas = kFp8 && NT == 1 ? 2 : 1;                    // per SM
    static constexpr int kHeadGroups = kGroups / HP;                         // key groups per head
    static constexpr int kTile = kHeadGroups * kSubKeys;                     // keys of a tile
    static constexpr int kRows = NT * 8;                                     // query rows of a unit, per head
    static constexpr int kRowBytes = kFp8 ? 128 : 256;                       // one key's row of one head
    static constexpr int kHalf = kSubKeys * kRowBytes;                       // the K half of a warp's ring slot
    static constexpr int kRing = 196608 / kCtas;
    static constexpr int kStages = kRing / (kGroups * 2 * kHalf);            // 3, or 6 in the E4M3 forms with one CTA
    static constexpr int kMl = kGroups * kRows * 8;                          // maximum and sum of every warp's rows
    static constexpr int kQ = 2 * HP * kRows * kDim * 2;                     // two units' queries
    static constexpr int kSmem = kRing + kMl + kQ + 512;
    static constexpr int kPassTiles = std::min(8, 2 * kHalf / (NT * 4 * 32 * 4));      // 16-dim blocks of O that fit a slot
    static_assert(kCtas * (kSmem + 1024) <= 228 * 1024, "shared memory of an SM");
    static_assert(kPassTiles >= 1, "the merge goes through the slots");
};

struct DecodeParams {
    const __nv_bfloat16* q;
    const uint8_t* k;
    const uint8_t* v;
    const float* k_scale;
    const float* v_scale;
    const int32_t* table;
    const int32_t* kv_len;
    int64_t table_stride, num_pages, stride_page, stride_tok, stride_head;     // strides in bytes
    int32_t page_shift;
    int32_t B, n_q, Hq, Hkv, G;
    int32_t rows;              // n_q * G
    int32_t row_groups;        // units per (request, KV head)
    int32_t window, sinks;
    int32_t capacity;          // tokens a table row can hold
    float scale_log2;
    __nv_bfloat16* out;
    float* lse;
    float* part_o;             // [2 * grid][rows of a unit][128]
    float* part_ml;            // [2 * grid][rows of a unit][2]
    int32_t* meta;             // [grid][4]: request, unit, CTAs, valid
    int32_t* status;
};

// ---------------------------------------------------------------------------------------------- PTX
__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async16_or_zeros(uint32_t dst, const void* src, bool valid) {
    const int n = valid ? 16 : 0;                          // 0: nothing is read, the 16 bytes become zeros
    asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
    uint4 r;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(addr) : "memory");
    return r;
}
__device__ __forceinline__ void sts128(uint32_t addr, const uint4& r) {
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(r.x), "r"(r.y), "r"(r.z), "r"(r.w) : "memory");
}
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
template <bool kF16>
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if (kF16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Four E4M3 codes -> two pairs of fp16 values (low codes, high codes), exact.
__device__ __forceinline__ void widen4(uint32_t codes, uint32_t& lo, uint32_t& hi) {
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}" : "=r"(lo), "=r"(hi) : "r"(codes));
}
template <bool kF16>
__device__ __forceinline__ uint32_t pack_weights(float lo, float hi) {
    if (kF16) {
        const __half2 h = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// The sign bits of the elements of a word that are infinite or NaN: those whose exponent (E4M3: exponent and mantissa) is all ones carry.
template <bool kFp8>
__device__ __forceinline__ uint32_t not_finite(uint32_t w) {
    return kFp8 ? ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u : ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
}
template <bool kFp8>
__device__ __forceinline__ uint32_t finite_part(uint32_t w) {
    const uint32_t top = not_finite<kFp8>(w);
    return w & ~(top | (top - (top >> (kFp8 ? 7 : 15))));
}

// ---------------------------------------------------------------------------------------------- work list
// Tiles of one unit of a request: those that some of its rows see, at least one (an empty request still writes its rows).
struct Request {
    int32_t len;               // keys of the request
    int32_t n;                 // tiles of a unit
    int32_t sink_tiles, skip;
};
template <int kTile>
__device__ __forceinline__ Request request_of(const DecodeParams& p, int b) {
    Request r;
    r.len = min(max(p.kv_len[b], 0), p.capacity);
    const int low = r.len - p.n_q + 1 - p.window;          // lowest key of the first row's window
    r.sink_tiles = p.sinks / kTile + (p.sinks % kTile != 0);
    r.skip = max(0, max(low, 0) / kTile - r.sink_tiles);   // tiles between sinks and window
    r.n = max(1, (r.len + kTile - 1) / kTile - r.skip);
    return r;
}
// A position in the list: request, unit (KV head major, then row group), tile.  On the axis that is cut into equal runs a unit
// takes kUnitCost + n places, starting at x: its fixed cost (queries, merge), then its tiles.
template <int kTile>
struct Cursor {
    int32_t b, u, t;
    int64_t x;
    Request r;
    __device__ __forceinline__ int64_t place() const { return x + kUnitCost + t; }
    __device__ __forceinline__ void next(const DecodeParams& p, int units) {
        if (++t < r.n) return;
        t = 0;
        x += kUnitCost + r.n;
        if (++u < units) return;
        u = 0;
        if (++b < p.B) r = request_of<kTile>(p, b);
    }
    __device__ __forceinline__ int first_key(int key_group) const {
        return (t < r.sink_tiles ? t : t + r.skip) * kTile + key_group * kSubKeys;
    }
};

// The infinities and NaN of V, at one dim, among the listed keys (late: from the first token's limit on, early: from its window's first
// key on) that token t of request b sees.  Only those are nonzero: 0 + inf, whatever the weight.
template <bool kFp8>
__device__ __forceinline__ float odd_values(const DecodeParams& p, const unsigned long long* keys, int b, int len, int h, int t, int dim) {
    const int lim_min = len - p.n_q + 1, lim = lim_min + t;
    float sum = 0.f;
#pragma unroll 1
    for (int early = 0; early < 2; ++early) {
#pragma unroll 1
        for (unsigned long long todo = keys[early]; todo != 0; todo &= todo - 1) {
            const int key = lim_min - (early ? p.window : 0) + __ffsll(todo) - 1;
            if (key >= lim || (key < lim - p.window && key >= p.sinks)) continue;
            const int64_t page = p.table[b * p.table_stride + (key >> p.page_shift)];      // of the pool: it was read
            const uint8_t* v = p.v + page * p.stride_page + (key & ((1 << p.page_shift) - 1)) * p.stride_tok + h * p.stride_head;
            const uint32_t x = kFp8 ? v[dim] : reinterpret_cast<const uint16_t*>(v)[dim];
            if (not_finite<kFp8>(x)) sum += kFp8 ? NAN : __uint_as_float(x << 16);
        }
    }
    return sum;
}

__device__ __forceinline__ int64_t run_begin(int64_t total, int64_t cta, int64_t ctas) { return total * cta / ctas; }

// NT, HP: see Shape.  kFp8: E4M3 cache.  kDrafts: n_q > 1, so the rows of a unit differ in the keys they see; only then is V looked at for
// infinities and NaN, in the groups that some row does not see in full (two of a unit as a rule).  These have a loop of their own: with the
// check inside the common one every group got slower (four contexts of 128K keys, E4M3, 32 rows: 157 us; 144 without the check, 141 like this;
// short requests of two tokens: 109 us without, 117 like this).
template <int NT, int HP, bool kFp8, bool kDrafts>
__global__ void __launch_bounds__(kThreads, Shape<NT, HP, kFp8>::kCtas)
decode_kernel(const __grid_constant__ DecodeParams p) {
    using Sh = Shape<NT, HP, kFp8>;
    constexpr int kHeadGroups = Sh::kHeadGroups, kTile = Sh::kTile;
    constexpr int kRowBytes = Sh::kRowBytes, kHalf = Sh::kHalf, kStages = Sh::kStages, kRows = Sh::kRows, kPassTiles = Sh::kPassTiles;
    constexpr float kShift = kFp8 ? kF16Shift : 0.f;
    constexpr bool kQRegs = NT <= 2;                       // query fragments stay in registers (else they are read from shared memory per tile)
    extern __shared__ __align__(1024) uint8_t smem[];
    float* ml = reinterpret_cast<float*>(smem + Sh::kRing);                                    // [warp][row][2]
    uint8_t* q_buf = smem + Sh::kRing + Sh::kMl;                                               // 2 x [row][256 B], chunks swizzled
    int64_t* scan = reinterpret_cast<int64_t*>(q_buf + Sh::kQ);                                // warp sums, then the run's start
    float* row_inv = reinterpret_cast<float*>(q_buf + Sh::kQ + 256);                           // 1 / sum of a unit's rows
    // [q_cur][head][2]: keys from the first row's limit on, from its window's first key on, whose V holds infinities or NaN (n_q <= 64)
    unsigned long long* odd_keys = reinterpret_cast<unsigned long long*>(q_buf + Sh::kQ + 128);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int sub = warp / kHeadGroups, key_group = warp % kHeadGroups;                        // the unit's head, the tile's keys
    const int g = lane >> 2, qd = lane & 3;
    const int units = p.Hkv / HP * p.row_groups;
    let_next_launch_begin();                               // the join

    // where this CTA's run starts: requests are dealt to the threads in order, a prefix sum over their tiles finds it
    const int per = (p.B + kThreads - 1) / kThreads;
    int64_t mine = 0;
    for (int i = 0; i < per; ++i) {
        const int b = tid * per + i;
        if (b < p.B) {
            mine += request_of<kTile>(p, b).n + kUnitCost;
            if (blockIdx.x == 0 && (p.kv_len[b] > p.capacity || p.kv_len[b] < 0)) report_status(p.status, CP_ERR_BOUNDS, b, p.kv_len[b]);
        }
    }
    int64_t inc = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += y;
    }
    if (lane == 31) scan[warp] = inc;
    if (kDrafts && tid < 4 * HP) odd_keys[tid] = 0;
    __syncthreads();
    int64_t before = inc - mine, total = 0;
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
        if (i < warp) before += scan[i];
        total += scan[i];
    }
    total *= units;
    before *= units;
    const int64_t ctas = min((int64_t)gridDim.x, total);   // no run is empty
    const int64_t x0 = blockIdx.x < ctas ? run_begin(total, blockIdx.x, ctas) : total;
    const int64_t x1 = blockIdx.x < ctas ? run_begin(total, blockIdx.x + 1, ctas) : total;
    int32_t* start = reinterpret_cast<int32_t*>(scan + kGroups);
    if (x0 >= before && x0 < before + mine * units) {
        int b = tid * per;
        int64_t at = before;
        while (true) {
            const int64_t n = (int64_t)(request_of<kTile>(p, b).n + kUnitCost) * units;
            if (x0 < at + n) break;
            at += n;
            ++b;
        }
        const int n = request_of<kTile>(p, b).n + kUnitCost;
        start[0] = b;
        start[1] = (int32_t)((x0 - at) / n);
        start[2] = (int32_t)((x0 - at) % n);               // places into the unit
    }
    if (tid == 0) p.meta[blockIdx.x * 4 + 3] = 0;
    __syncthreads();
    if (x0 >= x1) return;

    Cursor<kTile> ld, cur;                                        // the load stream runs kStages - 1 tiles ahead
    ld.b = start[0];
    ld.u = start[1];
    ld.t = max(0, start[2] - kUnitCost);
    ld.x = x0 - start[2];
    ld.r = request_of<kTile>(p, ld.b);
    cur = ld;
    if (cur.place() >= x1) return;                         // a run of fixed costs alone

    // ------------------------------------------------------------------ loads
    auto visible_group = [&](const Request& r, int key0) {
        const int low = r.len - p.n_q + 1 - p.window;      // lowest key of the first row's window
        return key0 < r.len && (key0 + kSubKeys > low || key0 < p.sinks);
    };
    // what the load stream keeps of its request and unit: this lane's offset into a page for the head, the table row
    const int ld_c = lane % (kRowBytes / 16), ld_k = lane / (kRowBytes / 16);
    const int page_mask = (1 << p.page_shift) - 1;
    const int32_t* ld_row = nullptr;
    int64_t ld_head = 0;
    int ld_low = 0, ld_key0 = 0, next_page = -1;
    auto enter_unit = [&]() {
        ld_row = p.table + ld.b * p.table_stride;
        ld_head = (int64_t)(ld.u / p.row_groups * HP + sub) * p.stride_head + ld_k * p.stride_tok + ld_c * 16;
        ld_low = ld.r.len - p.n_q + 1 - p.window;
    };
    auto look_up = [&]() {                                 // first key of this warp in the tile to load, and its page (-1: none to read)
        ld_key0 = ld.first_key(key_group);
        next_page = -1;
        if (visible_group(ld.r, ld_key0)) next_page = __ldg(ld_row + (ld_key0 >> p.page_shift));
    };
    const uint32_t ring_s = smem_addr(smem) + warp * (kStages * 2 * kHalf);
    int slot_ld = 0, slot_cur = 0;
    bool more = true;
    enter_unit();
    look_up();
    // copies: a row of kRowBytes is kChunks lanes, kKeysPerStep keys a step; chunk c of key k sits at chunk c ^ (k & 7)
    constexpr int kChunks = kRowBytes / 16, kKeysPerStep = 32 / kChunks, kSteps = kSubKeys / kKeysPerStep, kPeriod = 8 / kKeysPerStep;
    uint32_t ld_off[kPeriod];
#pragma unroll
    for (int i = 0; i < kPeriod; ++i) {
        const int kk = i * kKeysPerStep + ld_k;
        ld_off[i] = kk * kRowBytes + ((ld_c ^ (kk & 7)) << 4);
    }
    const int64_t step_bytes = kKeysPerStep * p.stride_tok;
    auto load_tile = [&]() {
        if (more) {
            const int key0 = ld_key0, len = ld.r.len;
            if (visible_group(ld.r, key0)) {
                const bool in_pool = (uint32_t)next_page < (uint32_t)p.num_pages;
                const int64_t off = next_page * p.stride_page + (key0 & page_mask) * p.stride_tok + ld_head;
                const uint8_t* ks = p.k + off;
                const uint8_t* vs = p.v + off;
                const uint32_t dst = ring_s + slot_ld * (2 * kHalf);
                if (in_pool && key0 + kSubKeys <= len && (key0 >= ld_low || key0 + kSubKeys <= p.sinks)) {
#pragma unroll
                    for (int i = 0; i < kSteps; ++i) {
                        const uint32_t d = dst + ld_off[i % kPeriod] + (i / kPeriod) * 8 * kRowBytes;
                        cp_async16(d, ks);
                        cp_async16(d + kHalf, vs);
                        ks += step_bytes;
                        vs += step_bytes;
                    }
                } else {                                   // some keys have no slot, or nobody sees them: zeros
#pragma unroll
                    for (int i = 0; i < kSteps; ++i) {
                        const uint32_t d = dst + ld_off[i % kPeriod] + (i / kPeriod) * 8 * kRowBytes;
                        const int key = key0 + i * kKeysPerStep + ld_k;
                        const bool ok = in_pool && key < len && (key >= ld_low || key < p.sinks);
                        cp_async16_or_zeros(d, ok ? ks + i * step_bytes : p.k, ok);
                        cp_async16_or_zeros(d + kHalf, ok ? vs + i * step_bytes : p.v, ok);
                    }
                }
            }
            ld.next(p, units);
            more = ld.place() < x1;
            if (more) {
                if (ld.t == 0) enter_unit();
                look_up();
            }
            slot_ld = slot_ld + 1 == kStages ? 0 : slot_ld + 1;
        }
        cp_commit();
    };
    // the query rows of unit (b, u) into buffer `buf`; rows behind the last are zeros
    auto load_q = [&](int b, int u, int buf) {
        const int hb = u / p.row_groups, r0 = (u - hb * p.row_groups) * kRows;
        for (int i = tid; i < HP * kRows * 16; i += kThreads) {
            const int at = i >> 4, c = i & 15, hs = at / kRows, r = r0 + at - hs * kRows;      // a row of head hb * HP + hs
            const bool ok = r < p.rows;
            const int t = kDrafts && ok ? r / p.G : 0;
            const int64_t o = ok ? (((int64_t)b * p.n_q + t) * p.Hq + (hb * HP + hs) * p.G + (r - t * p.G)) * kDim + c * 8 : 0;
            cp_async16_or_zeros(smem_addr(q_buf + buf * (HP * kRows * 256) + at * 256 + ((c ^ (at & 7)) << 4)), p.q + o, ok);
        }
    };

    load_q(cur.b, cur.u, 0);
    for (int i = 0; i < kStages - 1; ++i) load_tile();
    cp_wait<kStages - 2>();                                // the first group carries the queries
    __syncthreads();

    // ------------------------------------------------------------------ units
    int q_cur = 0;
    bool last_unit;
    do {
        const int b = cur.b, u = cur.u, t_begin = cur.t;
        const Request rq = cur.r;
        const int n_tiles = (int)min((int64_t)rq.n, x1 - cur.x - kUnitCost) - t_begin;
        last_unit = cur.x + 2 * kUnitCost + rq.n >= x1;    // the run ends before the next unit's first tile
        const int hb = u / p.row_groups, r0 = (u - hb * p.row_groups) * kRows, h0 = hb * HP;
        const uint8_t* qb = q_buf + q_cur * (HP * kRows * 256);
        // the next unit's queries travel under this unit's tiles (with the group of the next tile load)
        if (!last_unit) {
            if (u + 1 < units) load_q(b, u + 1, q_cur ^ 1);
            else load_q(b + 1, 0, q_cur ^ 1);
        }
        float c_row[NT][2];                                // scores -> log2 units, per query row of this thread
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) c_row[nt][0] = c_row[nt][1] = p.scale_log2;
        auto c_col = [&](int nt, int c) { return kFp8 ? c_row[nt][c] : p.scale_log2; };
        if (kFp8) {
            // fp16 queries: scaled per row by a power of two that brings the largest element to [2^10, 2^11); in place
            for (int row = warp; row < HP * kRows; row += kGroups) {
                const float k_scale = p.k_scale[h0 + row / kRows];
                uint8_t* at = const_cast<uint8_t*>(qb) + row * 256;
                const uint2 x = *reinterpret_cast<const uint2*>(at + (((lane >> 1) ^ (row & 7)) << 4) + (lane & 1) * 8);
                const float f0 = __uint_as_float(x.x << 16), f1 = __uint_as_float(x.x & 0xffff0000u);
                const float f2 = __uint_as_float(x.y << 16), f3 = __uint_as_float(x.y & 0xffff0000u);
                float amax = fmaxf(fmaxf(fabsf(f0), fabsf(f1)), fmaxf(fabsf(f2), fabsf(f3)));
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
                int e = 0;
                if (amax > 0.f && amax < INFINITY) e = min(max(10 - ilogbf(amax), -126), 126);
                const float up = copysignf(__uint_as_float((uint32_t)(127 + e) << 23), k_scale), down = __uint_as_float((uint32_t)(127 - e) << 23);
                // dims 4q .. 4q + 3 of a step's 16 are the operand's (2q, 2q + 1 | 2q + 8, 2q + 9), as the codes of K come out of a register
                __syncwarp();
                const int ks = lane >> 2;
                *reinterpret_cast<uint32_t*>(at + (((2 * ks) ^ (row & 7)) << 4) + (lane & 3) * 4) = pack_weights<true>(f0 * up, f1 * up);
                *reinterpret_cast<uint32_t*>(at + (((2 * ks + 1) ^ (row & 7)) << 4) + (lane & 3) * 4) = pack_weights<true>(f2 * up, f3 * up);
                if (lane == 0) ml[row] = down;             // the merge area is free between units
            }
            __syncthreads();
            // c > 0: the sign of a scale is in the queries; with a scale of zero (all scores 0) hidden keys must still be -inf * c = -inf
            const float ks = fabsf(p.k_scale[h0 + sub]) * p.scale_log2;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                c_row[nt][0] = fmaxf(ks * ml[sub * kRows + nt * 8 + 2 * qd], 1e-35f);
                c_row[nt][1] = fmaxf(ks * ml[sub * kRows + nt * 8 + 2 * qd + 1], 1e-35f);
            }
            __syncthreads();
        }
        // query fragments: one ldmatrix brings (two steps of one row block) or (one step of two row blocks)
        const uint32_t q_lane = smem_addr(qb) + sub * kRows * 256 + (NT == 1 ? (lane & 7) * 256 + (((lane >> 3) ^ (lane & 7)) << 4)
                                                        : ((lane & 7) + 8 * (lane >> 4)) * 256 + ((((lane >> 3) & 1) ^ (lane & 7)) << 4));
        uint32_t qf[kQRegs ? NT : 1][kQRegs ? 8 : 1][2];
        if (NT == 1) {
#pragma unroll
            for (int ks = 0; ks < 8; ks += 2) {
                uint32_t r4[4];
                ldsm4(r4, q_lane ^ (ks << 5));
                qf[0][ks][0] = r4[0];
                qf[0][ks][1] = r4[1];
                qf[0][ks + 1][0] = r4[2];
                qf[0][ks + 1][1] = r4[3];
            }
        } else if (kQRegs) {
#pragma unroll
            for (int ks = 0; ks < 8; ++ks) {
                uint32_t r4[4];
                ldsm4(r4, q_lane ^ (ks << 5));
                qf[0][ks][0] = r4[0];
                qf[0][ks][1] = r4[1];
                qf[NT > 1 ? 1 : 0][ks][0] = r4[2];
                qf[NT > 1 ? 1 : 0][ks][1] = r4[3];
            }
        }
        // S^T += K Q^T of one step of 16 dims
        auto score_step = [&](float (&sc)[NT][4], const uint32_t (&a)[4], int ks) {
            if (kQRegs) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) mma16816<kFp8>(sc[nt], a, qf[kQRegs ? nt : 0][kQRegs ? ks : 0][0], qf[kQRegs ? nt : 0][kQRegs ? ks : 0][1]);
            } else {
#pragma unroll
                for (int nt = 0; nt < NT; nt += 2) {
                    uint32_t r4[4];
                    ldsm4(r4, (q_lane + nt * 8 * 256) ^ (ks << 5));
                    mma16816<kFp8>(sc[nt], a, r4[0], r4[1]);
                    mma16816<kFp8>(sc[nt + 1 < NT ? nt + 1 : nt], a, r4[2], r4[3]);
                }
            }
        };
        // keys visible to each of this thread's rows: [lim - window, lim), and the sinks below lim
        int lim[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int r = r0 + nt * 8 + 2 * qd + c;
                lim[nt][c] = r < p.rows ? rq.len - p.n_q + (kDrafts ? r / p.G : 0) + 1 : 0;
            }
        float o[8][NT][4], l[NT][2];
        float m[NT][2];                                    // reference of the weights, p = 2^(c s - m): the running maximum, less kShift
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[i][nt][j] = 0.f;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            l[nt][0] = l[nt][1] = 0.f;
            m[nt][0] = m[nt][1] = kNoKey;
        }
        const int lim_min = rq.len - p.n_q + 1, low_max = rq.len - p.window;
        // this lane's row and chunk of the first ldmatrix of K and of V; later ones flip chunk bits
        const int mi = lane >> 3, mr = lane & 7;           // which 8 x 8 matrix of an ldmatrix this lane addresses, and its row
        const uint32_t k_lane = (mr + 8 * (mi & 1)) * kRowBytes + (((mi >> 1) ^ mr) << 4);
        const uint32_t v_lane = kFp8 ? k_lane : (mr + 8 * (mi >> 1)) * kRowBytes + (((mi & 1) ^ mr) << 4);

        int key0 = 0;                                      // the current tile: this warp's first key, its slot
        uint32_t kt = 0, vt = 0;
        bool full = false;                                 // every row sees all its keys
        // this warp's 16 keys of the current tile; masked: some row does not see some of them
        auto take = [&](bool masked) __attribute__((always_inline)) {
            // A key that only some of the rows see (draft tokens among themselves, the edge of their windows) may hold a V that is no finite
            // number, and a zero weight times that would reach the rows that do not see it: such elements are cleared here, and put into
            // the rows that do see them when the unit's result is written.
            if (kDrafts && masked) {
                // two lanes a key, each half a row, from another chunk on in every lane (banks)
                const uint32_t half_row = vt - v_lane + lane * (kRowBytes / 2) + ((kFp8 ? lane >> 1 & 3 : lane & 7) << 4);
                uint32_t odd = 0;
#pragma unroll
                for (int i = 0; i < kRowBytes / 2; i += 16) {
                    const uint4 w = lds128(half_row ^ i);
                    odd |= not_finite<kFp8>(w.x) | not_finite<kFp8>(w.y) | not_finite<kFp8>(w.z) | not_finite<kFp8>(w.w);
                }
                if (__any_sync(0xffffffffu, odd != 0)) {
                    const int key = key0 + (lane >> 1);
                    const bool late = key >= lim_min, early = key >= lim_min - p.window && key < low_max && key >= p.sinks;
                    if (odd != 0 && (late || early)) {
#pragma unroll 1
                        for (int i = 0; i < kRowBytes / 2; i += 16) {
                            const uint4 w = lds128(half_row ^ i);
                            sts128(half_row ^ i, make_uint4(finite_part<kFp8>(w.x), finite_part<kFp8>(w.y), finite_part<kFp8>(w.z), finite_part<kFp8>(w.w)));
                        }
                        atomicOr(&odd_keys[(q_cur * HP + sub) * 2 + (late ? 0 : 1)], 1ull << (key - lim_min + (late ? 0 : p.window)));
                    }
                    __syncwarp();
                }
            }
            float s[NT][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 4; ++j) s[nt][j] = 0.f;
            if (kFp8) {
#pragma unroll
                for (int ks = 0; ks < 8; ks += 2) {        // one ldmatrix brings two steps: codes of 16 dims x (keys 0-7, 8-15)
                    uint32_t r4[4];
                    ldsm4(r4, kt ^ (ks << 4));
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        uint32_t a[4];
                        widen4(r4[2 * half], a[0], a[2]);
                        widen4(r4[2 * half + 1], a[1], a[3]);
                        score_step(s, a, ks + half);
                    }
                }
            } else {
#pragma unroll
                for (int ks = 0; ks < 8; ++ks) {
                    uint32_t a[4];
                    ldsm4(a, kt ^ (ks << 5));
                    score_step(s, a, ks);
                }
            }
            // s[nt][j]: key g + 8 (j >> 1), row 2 qd + (j & 1); scores and maxima stay unscaled, c joins in the exponent
            if (masked) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int key = key0 + g + 8 * (j >> 1), lm = lim[nt][j & 1];
                        if (key >= lm || (key < lm - p.window && key >= p.sinks)) s[nt][j] = -INFINITY;
                    }
            }
            // exponents; is a weight about to exceed 2^kLag times its row's reference?
            float x[NT][4];
            bool grow = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    x[nt][j] = fmaf(s[nt][j], c_col(nt, j & 1), -m[nt][j & 1]);
                    grow |= x[nt][j] > kLag + kShift;
                }
            if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float top = fmaxf(s[nt][c], s[nt][c + 2]) * c_col(nt, c) - kShift;
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                        const float mn = fmaxf(m[nt][c], top), alpha = exp2_fast(m[nt][c] - mn);
                        m[nt][c] = mn;
                        l[nt][c] *= alpha;
                        x[nt][c] = fmaf(s[nt][c], c_col(nt, c), -mn);
                        x[nt][c + 2] = fmaf(s[nt][c + 2], c_col(nt, c), -mn);
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            o[i][nt][c] *= alpha;
                            o[i][nt][c + 2] *= alpha;
                        }
                    }
            }
            // weights, their sums (unrounded), and the weights as the B operand of V^T P^T
            uint32_t pb[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float w[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = exp2_fast(x[nt][j]);
                l[nt][0] += w[0] + w[2];
                l[nt][1] += w[1] + w[3];
                pb[nt][0] = transpose8x8(pack_weights<kFp8>(w[0], w[1]));
                pb[nt][1] = transpose8x8(pack_weights<kFp8>(w[2], w[3]));
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (kFp8) {
                    if ((i & 1) == 0) {
                        // two chunks of 16 dims: codes [16-bit pair of dims][keys], (keys 0-7, 8-15) of chunk i, then of chunk i + 1
                        uint32_t r4[4];
                        ldsm4_t(r4, vt ^ (i << 4));
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            uint32_t w[4];                 // dim 2g, keys 2q, 2q+1 | dim 2g + 1 | the same of keys 2q + 8, 2q + 9
                            widen4(__byte_perm(r4[2 * half], 0, 0x3120), w[0], w[1]);
                            widen4(__byte_perm(r4[2 * half + 1], 0, 0x3120), w[2], w[3]);
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) mma16816<true>(o[i + half][nt], w, pb[nt][0], pb[nt][1]);
                        }
                    }
                } else {
                    uint32_t a[4];
                    ldsm4_t(a, vt ^ (i << 5));
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma16816<false>(o[i][nt], a, pb[nt][0], pb[nt][1]);
                }
            }
        };
        // on to the next tile; false: no row sees its keys
        auto next_tile = [&]() {
            cp_wait<kStages - 2>();
            __syncwarp();                                  // this tile has landed, and every lane has read the slot that is filled next
            load_tile();
            key0 = cur.first_key(key_group);
            ++cur.t;
            kt = ring_s + slot_cur * (2 * kHalf) + k_lane;
            vt = ring_s + slot_cur * (2 * kHalf) + kHalf + v_lane;
            slot_cur = slot_cur + 1 == kStages ? 0 : slot_cur + 1;
            full = key0 + kSubKeys <= lim_min && (key0 >= low_max || key0 + kSubKeys <= p.sinks);
            return visible_group(rq, key0);
        };
        int it = 0;
        if (kDrafts) {
            while (true) {
                bool part = false;
                while (it < n_tiles) {
                    ++it;
                    if (!next_tile()) continue;
                    if (!full) {
                        part = true;
                        break;
                    }
                    take(false);
                }
                if (!part) break;
                take(true);
            }
        } else {
            for (; it < n_tiles; ++it)
                if (next_tile()) take(!full);
        }

        // -------------------------------------------------------------- the warps' partial results become one
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], d);
                if (g == 0) {
                    const int row = nt * 8 + 2 * qd + c;
                    ml[(warp * kRows + row) * 2] = m[nt][c];
                    ml[(warp * kRows + row) * 2 + 1] = l[nt][c];
                }
            }
        if (n_tiles < kStages) cp_wait<0>();               // the next unit's queries have landed before the barrier
        __syncthreads();
        unsigned long long any_odd = 0;
        if (kDrafts)
            for (int i = 0; i < 2 * HP; ++i) any_odd |= odd_keys[q_cur * HP * 2 + i];
        if (kDrafts && tid < 2 * HP) odd_keys[(q_cur ^ 1) * HP * 2 + tid] = 0;      // for the next unit
        const bool whole = t_begin == 0 && n_tiles == rq.n;
        const int slot = 2 * blockIdx.x + (t_begin > 0 ? 0 : 1);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int row = nt * 8 + 2 * qd + c;
                float mx = kNoKey;
#pragma unroll
                for (int w = 0; w < kHeadGroups; ++w) mx = fmaxf(mx, ml[((sub * kHeadGroups + w) * kRows + row) * 2]);
                const float f = exp2_fast(m[nt][c] - mx);  // a warp that saw no key of the row: 0 (or 1, on zeros)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    o[i][nt][c] *= f;
                    o[i][nt][c + 2] *= f;
                }
            }
        if (tid < HP * kRows && r0 + tid % kRows < p.rows) {
            const int hs = tid / kRows, row = tid % kRows, h = h0 + hs;
            const float* mine_ml = ml + (hs * kHeadGroups * kRows + row) * 2;
            float mx = kNoKey, sum = 0.f;
#pragma unroll
            for (int w = 0; w < kHeadGroups; ++w) mx = fmaxf(mx, mine_ml[w * kRows * 2]);
#pragma unroll
            for (int w = 0; w < kHeadGroups; ++w) sum += mine_ml[w * kRows * 2 + 1] * exp2_fast(mine_ml[w * kRows * 2] - mx);
            // a sum of zero: the row sees nothing; one that is no number (of a key or the query) makes the row NaN
            row_inv[tid] = sum == 0.f ? 0.f : (kFp8 ? p.v_scale[h] : 1.f) / sum;     // read behind the barrier below
            const int r = r0 + row, t = kDrafts ? r / p.G : 0;
            if (whole) {
                p.lse[(int64_t)(h * p.G + r - t * p.G) * ((int64_t)p.B * p.n_q) + (int64_t)b * p.n_q + t] =
                    sum == 0.f ? -INFINITY : (mx + log2f(sum)) * 0.6931471805599453f;
            } else {
                p.part_ml[((int64_t)slot * (HP * kRows) + tid) * 2] = mx;
                p.part_ml[((int64_t)slot * (HP * kRows) + tid) * 2 + 1] = sum;
            }
        }
        // through the slots that were read last: they are filled again only after the next unit has begun
        const int slot_free = slot_cur == 0 ? kStages - 1 : slot_cur - 1;
        float* mine_o = reinterpret_cast<float*>(smem + (warp * kStages + slot_free) * (2 * kHalf));
        const float* all_o = reinterpret_cast<const float*>(smem + slot_free * (2 * kHalf));
        constexpr int kPassRegs = kPassTiles * NT * 4, kGroupFloats = kStages * 2 * kHalf / 4;
#pragma unroll
        for (int pass = 0; pass < 8 / kPassTiles; ++pass) {
            if (pass > 0) __syncthreads();                 // the previous pass has been summed
#pragma unroll
            for (int i = 0; i < kPassTiles; ++i)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int j = 0; j < 4; ++j) mine_o[((i * NT + nt) * 4 + j) * 32 + lane] = o[pass * kPassTiles + i][nt][j];
            __syncthreads();
#pragma unroll
            for (int x = 0; x < kPassRegs * 32 * HP / kThreads; ++x) {
                const int all = x * kThreads + tid, hs = all / (kPassRegs * 32);       // head
                const int at = all - hs * (kPassRegs * 32);                            // lane at & 31 of register (at >> 5)
                float sum = 0.f;
#pragma unroll
                for (int w = 0; w < kHeadGroups; ++w) sum += all_o[(hs * kHeadGroups + w) * kGroupFloats + at];
                const int ln = at & 31, reg = at >> 5, j = reg & 3, nt = (reg >> 2) % NT, i = (reg >> 2) / NT;
                const int gg = ln >> 2, row = nt * 8 + 2 * (ln & 3) + (j & 1);
                const int dim = (pass * kPassTiles + i) * 16 + (kFp8 ? 2 * gg + (j >> 1) : gg + 8 * (j >> 1));
                const int r = r0 + row;
                if (r < p.rows) {
                    const int t = kDrafts ? r / p.G : 0;
                    if (whole) {
                        p.out[(((int64_t)b * p.n_q + t) * p.Hq + (h0 + hs) * p.G + r - t * p.G) * kDim + dim] = __float2bfloat16_rn(sum * row_inv[hs * kRows + row]);
                    } else {
                        p.part_o[((int64_t)slot * (HP * kRows) + hs * kRows + row) * kDim + dim] = sum;
                    }
                }
            }
        }
        if (kDrafts && any_odd != 0) {                     // what was cleared joins the rows just written
            __syncthreads();
#pragma unroll 1
            for (int i = tid; i < HP * kRows * kDim; i += kThreads) {
                const int at = i / kDim, dim = i % kDim, hs = at / kRows, r = r0 + at % kRows, t = r / p.G;
                if (r >= p.rows) continue;
                const float x = odd_values<kFp8>(p, odd_keys + (q_cur * HP + hs) * 2, b, rq.len, h0 + hs, t, dim);
                if (x == 0.f) continue;
                if (whole) {
                    __nv_bfloat16* o = p.out + (((int64_t)b * p.n_q + t) * p.Hq + (h0 + hs) * p.G + r - t * p.G) * kDim + dim;
                    *o = __float2bfloat16_rn(__bfloat162float(*o) + x);
                } else {
                    p.part_o[((int64_t)slot * (HP * kRows) + at) * kDim + dim] += x;
                }
            }
        }
        if (tid == 0 && !whole && t_begin == 0) {
            // this CTA holds the unit's first piece: the last one ends with the unit's last tile, at place x_end - 1
            const int64_t x_end = cur.x + kUnitCost + rq.n;
            int64_t last = min((x_end * ctas - 1) / total, ctas - 1);
            while (run_begin(total, last, ctas) >= x_end) --last;
            while (run_begin(total, last + 1, ctas) < x_end) ++last;
            p.meta[blockIdx.x * 4 + 0] = b;
            p.meta[blockIdx.x * 4 + 1] = u;
            p.meta[blockIdx.x * 4 + 2] = (int32_t)(last - blockIdx.x + 1);
            p.meta[blockIdx.x * 4 + 3] = 1;
        }
        __syncthreads();                                   // ml, the slots and the old query buffer are free again
        if (!last_unit) {
            --cur.t;                                       // back on the unit's last tile, then to the next unit
            cur.next(p, units);
        }
        q_cur ^= 1;
    } while (!last_unit);
    cp_wait<0>();
}

// Joins the pieces of the units that were cut: block (c, row) takes the unit whose first piece CTA c holds.  Pieces: slot 2c + 1, then slot
// 2c' of the following CTAs.  Warps take the pieces in turn, and are summed in a fixed order.
template <bool kFp8>
__global__ void __launch_bounds__(kJoinThreads)
decode_join_kernel(const __grid_constant__ DecodeParams p, int heads, int rows_per_head) {
    constexpr int kJoinWarps = kJoinThreads / 32;
    __shared__ float acc[kJoinWarps][kDim];
    __shared__ float sums[kJoinWarps];
    wait_for_launch_before();
    const int c = blockIdx.x, row = blockIdx.y, rows_per_unit = heads * rows_per_head;
    const int4 me = *reinterpret_cast<const int4*>(p.meta + 4 * c);
    if (me.w == 0) return;
    const int hb = me.y / p.row_groups, hs = row / rows_per_head, h = hb * heads + hs;
    const int r = (me.y - hb * p.row_groups) * rows_per_head + row - hs * rows_per_head;
    if (r >= p.rows) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    auto slot_of = [&](int k) { return k == 0 ? 2 * c + 1 : 2 * (c + k); };
    float mx = kNoKey;
    for (int k = lane; k < me.z; k += 32) mx = fmaxf(mx, p.part_ml[((int64_t)slot_of(k) * rows_per_unit + row) * 2]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
    float sum = 0.f;
#pragma unroll 4
    for (int k = warp; k < me.z; k += kJoinWarps) {
        const int64_t at = (int64_t)slot_of(k) * rows_per_unit + row;
        const float2 v = *reinterpret_cast<const float2*>(p.part_ml + at * 2);
        const float4 x = *reinterpret_cast<const float4*>(p.part_o + at * kDim + lane * 4);
        const float f = exp2_fast(v.x - mx);
        sum += f * v.y;
        a.x += f * x.x;
        a.y += f * x.y;
        a.z += f * x.z;
        a.w += f * x.w;
    }
    *reinterpret_cast<float4*>(&acc[warp][lane * 4]) = a;
    if (lane == 0) sums[warp] = sum;
    __syncthreads();
    float total = 0.f;
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) total += sums[w];
    const int t = r / p.G, head = h * p.G + r - t * p.G;
    const int64_t token = (int64_t)me.x * p.n_q + t;
    if (threadIdx.x < kDim) {
        float x = 0.f;
#pragma unroll
        for (int w = 0; w < kJoinWarps; ++w) x += acc[w][threadIdx.x];
        const float inv = total == 0.f ? 0.f : (kFp8 ? p.v_scale[h] : 1.f) / total;
        p.out[(token * p.Hq + head) * kDim + threadIdx.x] = __float2bfloat16_rn(x * inv);
    }
    if (threadIdx.x == 0)
        p.lse[(int64_t)head * ((int64_t)p.B * p.n_q) + token] =
            total == 0.f ? -INFINITY : (mx + log2f(total)) * 0.6931471805599453f;
}

constexpr int kMaxDecodeGrid = 2 * kMaxGrid;
constexpr int kMaxHeads = 2;                               // largest HP
constexpr int kMaxDecodeTokens = 64, kMaxDecodeRows = 1024, kMaxDecodeBatch = 65536;      // limits of a call: n_q, rows per KV head, B
inline int row_blocks(int rows) { return rows <= 8 ? 1 : (rows <= 16 ? 2 : 4); }

// Workspace: partial rows and their (maximum, sum) of two pieces per CTA, and four words per CTA.
size_t decode_workspace(int rows) {
    const size_t n = 2 * (size_t)kMaxDecodeGrid * kMaxHeads * row_blocks(rows) * 8;
    return (n * (kDim + 2) * sizeof(float) + kMaxDecodeGrid * 16 + 255) / 256 * 256;
}

template <int NT, int HP, bool kFp8, bool kDrafts>
int launch_decode(cp_ctx* ctx, const DecodeParams& p, cudaStream_t s, const char* who) {
    using Sh = Shape<NT, HP, kFp8>;
    const int grid = std::min(ctx->num_sms, kMaxGrid) * Sh::kCtas;
    const uint32_t variant = 1u << (8 * (NT / 2) + 4 * (HP - 1) + (kFp8 ? 2 : 0) + (kDrafts ? 1 : 0));      // NT 1, 2 or 4; HP 1 or 2
    if (!(ctx->decode_attr_set & variant)) {
        if (int rc = check_cuda(cudaFuncSetAttribute(decode_kernel<NT, HP, kFp8, kDrafts>, cudaFuncAttributeMaxDynamicSharedMemorySize, Sh::kSmem),
                                "cudaFuncSetAttribute(decode)")) return rc;
        ctx->decode_attr_set |= variant;
    }
    decode_kernel<NT, HP, kFp8, kDrafts><<<grid, kThreads, Sh::kSmem, s>>>(p);
    if (int rc = check_cuda(cudaGetLastError(), who)) return rc;
    return launch_behind(decode_join_kernel<kFp8>, dim3((unsigned)grid, (unsigned)(HP * Sh::kRows)), kJoinThreads, s, who, p, HP, (int)Sh::kRows);
}

template <int HP, bool kFp8, bool kDrafts>
int launch_rows(int blocks, cp_ctx* ctx, const DecodeParams& p, cudaStream_t s, const char* who) {
    if (blocks == 1) return launch_decode<1, HP, kFp8, kDrafts>(ctx, p, s, who);
    if (blocks == 2) return launch_decode<2, HP, kFp8, kDrafts>(ctx, p, s, who);
    return launch_decode<4, HP, kFp8, kDrafts>(ctx, p, s, who);
}

int decode_attn(cp_ctx* ctx, const void* q, const void* k, const void* v, const float* k_scale, const float* v_scale, int64_t num_pages,
                int32_t page_size, int32_t Hkv, int64_t stride_page, int64_t stride_tok, int64_t stride_head, bool fp8,
                const int32_t* page_table, int64_t table_stride, const int32_t* kv_len, int32_t B, int32_t n_q, int32_t Hq,
                int64_t window, int64_t sinks, float scale, void* out, float* lse, void* workspace, size_t workspace_bytes,
                void* stream, const char* who) {
    if (B < 0 || n_q < 1 || Hq < 1 || table_stride < 1)
        return set_error(CP_ERR_INVALID_ARG, "%s: B=%d n_q=%d Hq=%d table_stride=%lld", who, B, n_q, Hq, (long long)table_stride);
    if (Hq % Hkv != 0) return set_error(CP_ERR_INVALID_ARG, "%s: Hq=%d is not a multiple of Hkv=%d", who, Hq, Hkv);
    if (B > 0 && (!q || !page_table || !kv_len || !out || !lse)) return set_error(CP_ERR_INVALID_ARG, "%s: null pointer", who);
    if (!(scale > 0.f) || !isfinite(scale)) return set_error(CP_ERR_INVALID_ARG, "%s: scale must be positive", who);
    if (window < 1 || sinks < 0)
        return set_error(CP_ERR_INVALID_ARG, "%s: window=%lld sinks=%lld", who, (long long)window, (long long)sinks);
    if (((uintptr_t)q | (uintptr_t)out) & 15) return set_error(CP_ERR_INVALID_ARG, "%s: q and out must be 16-byte aligned", who);
    const int shift = log2_exact(page_size);
    const int64_t rows = (int64_t)n_q * (Hq / Hkv);
    if (n_q > kMaxDecodeTokens || rows > kMaxDecodeRows)
        return set_error(CP_ERR_UNSUPPORTED, "%s: n_q=%d, %lld query rows per KV head; at most 64 and 1024 (more: a prefill call)", who, n_q,
                         (long long)rows);
    if (B > kMaxDecodeBatch || table_stride > (0x7fffff00ll >> shift) || num_pages > 0x7fffffffll)
        return set_error(CP_ERR_UNSUPPORTED, "%s: B=%d (at most 65536), a table row of %lld entries or %lld pages", who, B,
                         (long long)table_stride, (long long)num_pages);
    const size_t need = decode_workspace((int)rows);
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < need)
        return set_error(CP_ERR_WORKSPACE, "%s: workspace %p of %zu bytes; need %zu bytes, 256-byte aligned", who, workspace, workspace_bytes, need);
    if (!ctx) return set_error(CP_ERR_INVALID_ARG, "%s: ctx is NULL", who);
    if (B == 0) return CP_OK;
    DeviceGuard guard(ctx->device);
    if (guard.rc()) return guard.rc();
    DecodeParams p;
    p.q = static_cast<const __nv_bfloat16*>(q);
    p.k = static_cast<const uint8_t*>(k);
    p.v = static_cast<const uint8_t*>(v);
    p.k_scale = k_scale;
    p.v_scale = v_scale;
    p.table = page_table;
    p.kv_len = kv_len;
    p.table_stride = table_stride;
    p.num_pages = num_pages;
    p.stride_page = stride_page;
    p.stride_tok = stride_tok;
    p.stride_head = stride_head;
    p.page_shift = shift;
    p.B = B;
    p.n_q = n_q;
    p.Hq = Hq;
    p.Hkv = Hkv;
    p.G = Hq / Hkv;
    p.rows = (int32_t)rows;
    const int nt = row_blocks(p.rows);
    p.row_groups = (p.rows + nt * 8 - 1) / (nt * 8);
    p.window = (int32_t)std::min<int64_t>(window, 0x7fffff00);
    p.sinks = (int32_t)std::min<int64_t>(sinks, 0x7fffff00);
    p.capacity = (int32_t)(table_stride << shift);
    p.scale_log2 = scale * 1.4426950408889634f;
    p.out = static_cast<__nv_bfloat16*>(out);
    p.lse = lse;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    const size_t n = 2 * (size_t)kMaxDecodeGrid * kMaxHeads * nt * 8;
    p.part_o = reinterpret_cast<float*>(ws);
    p.part_ml = p.part_o + n * kDim;
    p.meta = reinterpret_cast<int32_t*>(p.part_ml + n * 2);
    p.status = ctx->d_status;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (fp8 && Hkv % 2 == 0) return n_q > 1 ? launch_rows<2, true, true>(nt, ctx, p, s, who) : launch_rows<2, true, false>(nt, ctx, p, s, who);
    if (fp8) return n_q > 1 ? launch_rows<1, true, true>(nt, ctx, p, s, who) : launch_rows<1, true, false>(nt, ctx, p, s, who);
    return n_q > 1 ? launch_rows<1, false, true>(nt, ctx, p, s, who) : launch_rows<1, false, false>(nt, ctx, p, s, who);
}

}  // namespace

extern "C" size_t cp_workspace_bytes_decode(int32_t B, int32_t n_q, int32_t Hq, int32_t Hkv) {
    if (B < 0 || n_q < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0) return 0;
    const int64_t rows = (int64_t)n_q * (Hq / Hkv);
    if (B > kMaxDecodeBatch || n_q > kMaxDecodeTokens || rows > kMaxDecodeRows) return 0;
    return decode_workspace((int)rows);
}

extern "C" int cp_decode_attn(cp_ctx* ctx, const void* q, const cp_kv_cache* cache, const int32_t* page_table, int64_t table_stride,
                              const int32_t* kv_len, int32_t B, int32_t n_q, int32_t Hq, int64_t window, int64_t sinks, float scale,
                              void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    const char* who = "cp_decode_attn";
    if (int rc = validate_kv_cache(cache, who)) return rc;
    return decode_attn(ctx, q, cache->k, cache->v, nullptr, nullptr, cache->num_pages, cache->page_size, cache->Hkv, cache->stride_page * 2,
                       cache->stride_tok * 2, cache->stride_head * 2, false, page_table, table_stride, kv_len, B, n_q, Hq, window, sinks,
                       scale, out, lse, workspace, workspace_bytes, stream, who);
}

extern "C" int cp_decode_attn_fp8(cp_ctx* ctx, const void* q, const cp_kv_cache_fp8* cache, const int32_t* page_table,
                                  int64_t table_stride, const int32_t* kv_len, int32_t B, int32_t n_q, int32_t Hq, int64_t window,
                                  int64_t sinks, float scale, void* out, float* lse, void* workspace, size_t workspace_bytes,
                                  void* stream) {
    const char* who = "cp_decode_attn_fp8";
    if (int rc = validate_kv_cache_fp8(cache, who)) return rc;
    return decode_attn(ctx, q, cache->k, cache->v, cache->k_scale, cache->v_scale, cache->num_pages, cache->page_size, cache->Hkv,
                       cache->stride_page, cache->stride_tok, cache->stride_head, true, page_table, table_stride, kv_len, B, n_q, Hq,
                       window, sinks, scale, out, lse, workspace, workspace_bytes, stream, who);
}
