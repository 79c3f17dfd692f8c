// Attention of drafted trees with many query rows per KV head, n_q * Hq / Hkv of them, on the tcgen05 tensor cores, over paged caches
// with lengths, masks and page tables on the device.
//
// With r rows a key costs 512 r flops and 512 bytes (bf16; E4M3 256, 4-bit 136): at 128 rows half of what the tensor cores can do while the keys
// arrive, at 264 as much.  The narrow form (decode_kernel.cuh) works such rows off in units of 32 with mma.sync, each reading (and, of one-byte and 4-bit
// caches, widening) the keys again; here a CTA takes up to 256 rows, so every key is brought to shared memory once for all of them.
//   - Query row t * G + h of a KV head (token t, head h of the group) is a row of the M side.  Up to 256 rows are two 128-row score tiles that share the K/V
//     tiles, one softmax warpgroup each.  Up to 128 rows are one, and the warpgroups take the K/V tiles in turn, each with an accumulator of its own; the
//     two are added at the end of a unit (one warpgroup alone needs twice the time that the keys do to arrive).
//   - More than 256 rows are several classes of equal height, whose CTAs walk the same runs of the key axis side by side: they
//     read the same keys at the same time and all but one find them in L2.  So do the CTAs of up to four KV heads of E4M3 and 4-bit caches, whose rows of 128 and 64 bytes
//     lie side by side (and share the exponents' 16 bytes): 64 requests with a window of 4096, 96 rows, E4M3 202 us with a head by itself, 186 with two or four;
//     28 rows, 4-bit 217 / 209 / 208; bf16 no change.
//   - The key axis is all (request, KV head) units one after the other, 128 keys a step, cut into equal runs, one per CTA of a class, whatever
//     the lengths are (the scheme of the narrow form: Cursor); pieces of cut units are joined by a second launch.
//   - Warps: two softmax warpgroups; a producer that fetches K/V tiles page by page; the issuers of S = Q K^T and of O += P V; a warp that gathers the
//     unit's query rows with cp.async.  S, P and O live in TMEM: S | P0 | P1 | O0 | O1.  S is one buffer that the tiles use in turn, read
//     into registers at once, so the next product runs under the exponentials.
//   - K and V come by TMA, page by page.  E4M3 and 4-bit rows land in a ring of raw tiles, and a fourth warpgroup (with the softmax warps that have no rows, for 4-bit rows) widens them into the tiles of the products:
//     E4M3 to fp16 (queries and weights are then fp16 as in the narrow form), 4-bit codes and exponents to bf16, both exactly.  (Copied by the widening warps
//     with cp.async, an E4M3 tile takes 3 us: with 64 registers a thread the copies wait for one another's addresses.)
//   - Only the last tiles of a unit and those at a window's edge hide keys from rows.  Their masks are bits: of the tree's mask and of the window.  A hidden
//     key's weight is zero, but zero times an infinity is not: the issuer of P V looks through the V of these tiles and clears what is no
//     finite number; what some rows do see of it is added to their results when they are written.
// Every wait is bounded, as in the prefill kernel.
// Measured, 37 requests of 8192 keys, 32 / 8 heads, pages of 64 (the copy rate needs 193 / 96 / 51 us): bf16 199, 208 and 294 us with 64, 128 and 256 rows (6.2 TB/s up to
// 128 rows, then the tensor and MUFU pipes: 1080 TFLOP/s of visible pairs); E4M3 190, 192, 298 and 4-bit 202, 235, 315 us, bound by the chain from a raw tile to the second product,
// in which shared memory's data pipe is the busiest (57 %: 33 by the warps that widen, 24 by the tensor cores).  A unit costs 9 to 22 us beside its tiles: 4 until its queries are there, 2 of epilogue, 1 to 3 where the warpgroups wait for one another.
#pragma once

#include "decode_kernel.cuh"
#include "tc_ptx.cuh"

namespace {

constexpr int kWideRows = 256;                             // query rows of a unit
constexpr int kWideCost = 3;                               // fixed cost of a unit in tiles: queries, epilogue
constexpr float kWideLag = 8.0f;                           // the running maximum may lag by a factor 2^8
constexpr int kWideSplit = 3;                              // P is handed over in two pieces: three quarters of the keys, then the rest
constexpr int kConvWarps = 4;
constexpr int kMaxRing = 3, kMaxRaw = 6;
constexpr int kUnitBytes = 80;

// kTiles: score tiles of a unit; with one, the warpgroups take the K/V tiles in turn.
template <Kind kKind, int kTiles>
struct Wide {
    static constexpr bool kRawTiles = kKind != kBf16, kTurns = kTiles == 1, kHelp = kKind == kMx4 && kTurns;
    static constexpr int kThreads = kRawTiles ? 512 : 384;
    // register budgets after the roles split; they stay below the register file by one step at least
    static constexpr int kRegsSoftmax = kRawTiles ? 184 : 200, kRegsOther = kRawTiles ? 64 : 104;
    static_assert(256 * kRegsSoftmax + (kThreads - 256) * kRegsOther <= 65536 - 1024, "leave slack in the register file");
    // Rings of 32 KB tiles, one for K and one for V: a full barrier has one waiter, who has waited for each of its phases.  (With K and V in turn in one ring the
    // issuer of S can be at a slot whose V has not landed yet, when the tiles are taken in turn; its wait would take the phase before that for its own.)
    static constexpr int kStagesK = kRawTiles ? 2 : 3, kStagesV = 2, kStages = kStagesK + kStagesV;
    static constexpr uint32_t kRawCodes = kKind == kE4m3 ? 16384u : 8192u;                         // of the 128 keys of a tile
    static constexpr uint32_t kRawBytes = kRawCodes + (kKind == kMx4 ? 2048u : 0u);                // 4-bit: then 16 bytes a key with the exponents of four heads
    static constexpr int kRaw = kKind == kBf16 ? 0 : (kKind == kE4m3 ? (kTurns ? 3 : 2) : (kTurns ? 6 : 3));      // slots of the ring of raw tiles
    // shared memory: the query tiles, the ring, the raw tiles, what the warpgroups tell one another, barriers and small areas
    static constexpr uint32_t kQ = 0, kKV = kTiles * kTileBytes, kRawAt = kKV + kStages * kTileBytes;
    static constexpr uint32_t kMl = kRawAt + kRaw * kRawBytes;                        // [unit parity][warpgroup][row]: maximum and sum
    static constexpr uint32_t kBar = kMl + (kTurns ? 2 * 2 * kBlockM * 8 : 0);
    static constexpr uint32_t kOdd = kBar + 48 * 8;        // [unit parity][2] keys whose V is no finite number (see odd_values)
    static constexpr uint32_t kScan = kOdd + 32;           // sums of the warps, then the run's start
    static constexpr uint32_t kExp = kScan + 16 * 8 + 16;  // [unit parity][row]: exponent by which a row of E4M3 queries was scaled up
    static constexpr uint32_t kUnits = (kExp + (kKind == kE4m3 ? 2 * kWideRows : 0) + 15) / 16 * 16;      // a copy per warp
    static constexpr uint32_t kTmemPtr = kUnits + kThreads / 32 * kUnitBytes, kAbort = kTmemPtr + 4;
    static constexpr uint32_t kSmem = kAbort + 12;
    static_assert(kSmem <= 227 * 1024, "shared memory of a CTA");
};
enum WideBar : uint32_t {
    kWQFull = 0, kWQEmpty = 1,
    kWKFull = 2,                             // + stage
    kWKEmpty = kWKFull + kMaxRing,           // + stage
    kWVFull = kWKEmpty + kMaxRing,           // + stage
    kWVEmpty = kWVFull + kMaxRing,           // + stage
    kWSReady = kWVEmpty + kMaxRing,          // + warpgroup: its scores are in the S buffer
    kWSFree = kWSReady + 2,                  // + warpgroup: it has read the S buffer
    kWPReady = kWSFree + 2,                  // + 2 warpgroup + piece
    kWPvDone = kWPReady + 4,                 // + warpgroup: P V of a step has finished
    kWOFree = kWPvDone + 2,                  // + warpgroup: O has been read
    kWOdd = kWOFree + 2,                     // the unit's list of odd keys is complete
    kWMl = kWOdd + 1,                        // + warpgroup: its accumulator, maxima and sums of the unit are complete (tiles in turn)
    kWQRaw = kWMl + 2,                       // the query rows are there, to be converted
    kWRawFull = kWQRaw + 1,                  // + raw slot
    kWRawEmpty = kWRawFull + kMaxRaw,        // + raw slot
    kNumWideBars = kWRawEmpty + kMaxRaw
};
static_assert(kNumWideBars <= 48, "barrier area");

constexpr uint32_t kWTmemS = 0, kWTmemP = 128, kWTmemO = 256;      // columns; + 64 and + 128 for the second tile

struct WideParams {
    DecodeParams d;
    int32_t classes;           // row classes of a KV head
    int32_t class_rows;        // rows of a class (the last may have fewer)
    int32_t heads;             // KV heads whose units are walked side by side
    int32_t runs;              // CTAs of a class and head
    // CTA (x, y, z): row class, head of the group, run; x counts fastest, so what reads the same tokens starts together
    __device__ __forceinline__ int cls() const { return (int)blockIdx.x; }
    __device__ __forceinline__ int head() const { return (int)blockIdx.y; }
    __device__ __forceinline__ int run() const { return (int)blockIdx.z; }
    __device__ __forceinline__ int64_t place() const { return (int64_t)(head() * classes + cls()) * runs + run(); }       // in the workspace: runs side by side
};

// The units of this CTA, one after the other: request b, KV head u, tiles [t_begin, t_end).  Every warp has a copy in shared memory that it steps by itself, which
// keeps a score of registers free in every role.
struct WideUnits {
    Cursor<kBlockN, true> cur;
    int64_t x1;
    int t_begin, t_end, heads;
    bool whole, valid;
    // by one lane
    __device__ __forceinline__ void begin(const WideParams& w, const int32_t* start, int64_t x0, int64_t end) {
        const DecodeParams& p = w.d;
        heads = w.heads;
        cur.b = start[0];
        cur.u = start[1] * heads + w.head();
        cur.t = max(0, start[2] - kWideCost);
        cur.x = x0 - start[2];
        cur.r = request_of<kBlockN, true>(p, cur.b);
        x1 = end;
        span();
    }
    __device__ __forceinline__ void span() {
        t_begin = cur.t;
        t_end = (int)min((int64_t)cur.r.n, x1 - cur.x - kWideCost);
        whole = t_begin == 0 && t_end == cur.r.n;
        valid = cur.x + kWideCost + cur.t < x1;
    }
    // by the warp
    __device__ __forceinline__ void next(const DecodeParams& p) {
        __syncwarp();
        if ((threadIdx.x & 31) == 0) {
            cur.t = 0;
            cur.x += kWideCost + cur.r.n;
            cur.u += heads;
            if (cur.u >= p.Hkv) {
                cur.u -= p.Hkv;
                if (++cur.b < p.B) cur.r = request_of<kBlockN, true>(p, cur.b);
            }
            span();
        }
        __syncwarp();
    }
    __device__ __forceinline__ int key_of(int t) const { return (t < cur.r.sink_tiles ? t : t + cur.r.skip) * kBlockN; }
    // every row of the tree sees all keys of the tile
    __device__ __forceinline__ bool full(const DecodeParams& p, int key0) const {
        return key0 + kBlockN <= cur.r.base && (key0 >= cur.r.len - p.window || key0 + kBlockN <= p.sinks);
    }
};

static_assert(sizeof(WideUnits) <= kUnitBytes, "room for the units");

struct WideCtx {
    uint32_t smem, bars, tmem;
    uint8_t* gen;              // the same shared memory
    volatile uint32_t* abort_flag;
    int32_t* status;
    __device__ __forceinline__ void wait(uint32_t id, uint32_t parity, int iter) const { mbar_wait(bars, id, parity, abort_flag, status, iter); }
    // some wait has given up: whoever starts copies or products stops, so that little is in flight when the CTA ends (by the warp)
    __device__ __forceinline__ bool given_up() const { return __any_sync(0xffffffffu, *abort_flag != 0); }
};
// Warps of a warpgroup that have rows of the CTA's class, one at least.  The others stay out (they would poll beside the widening warps: 8192 4-bit keys of 37 requests,
// 64 rows 275 us, 255 like this), or help to widen 4-bit tiles.
template <int kTiles>
__device__ __forceinline__ int wide_warps(const WideParams& w, int wg) {
    const int rows = min(w.class_rows, w.d.rows - w.cls() * w.class_rows) - (kTiles == 2 ? wg * kBlockM : 0);
    return min(max((rows + 31) >> 5, 1), 4);
}
// Warps that widen: a warpgroup, and of 4-bit tiles of up to 128 rows the softmax warps without rows (28 rows 205 -> 175 us, 64 rows 225 -> 196 us).
template <Kind kKind, int kTiles>
__device__ __forceinline__ int wide_widening(const WideParams& w) {
    return kConvWarps + (Wide<kKind, kTiles>::kHelp ? 8 - wide_warps<kTiles>(w, 0) - wide_warps<kTiles>(w, 1) : 0);
}
// A position in a ring: slot, and the parity of the phase that ends when it is filled (for the side that fills: when it was emptied).
template <int kStages>
struct WideRing {
    uint32_t slot, par;
    __device__ __forceinline__ void advance() {
        if (++slot == (uint32_t)kStages) {
            slot = 0;
            par ^= 1u;
        }
    }
};

// ---------------------------------------------------------------------------------------------- producer
struct WideMaps {
    const CUtensorMap *k, *v, *k_exp, *v_exp;              // the last two: exponents of 4-bit rows
};
// Lane i < pages of a tile holds a page id; those of the next K tile are fetched while the current ones are used.  Pages that no row sees anything of are read as
// zeros.  bf16: loads in order of first use, K(j0), then K(j + 1) before V(j), into the rings; the others K(j), V(j) into the raw ring.
template <Kind kKind, int kTiles>
__device__ __forceinline__ void wide_producer(const WideParams& w, const WideCtx& c, WideUnits& units, const WideMaps& maps) {
    using W = Wide<kKind, kTiles>;
    const DecodeParams& p = w.d;
    const int lane = threadIdx.x & 31;
    const int page_tokens = 1 << p.page_shift, per_tile = kBlockN >> p.page_shift;
    const int outside = (int)p.num_pages;                  // a page coordinate behind the tensor: TMA fills zeros
    WideRing<W::kStagesK> kr = {0, 1};
    WideRing<W::kStagesV> vr = {0, 1};
    WideRing<W::kRawTiles ? W::kRaw : 1> raw = {0, 1};
    for (; units.valid; units.next(p)) {
        const int len = units.cur.r.len, low = units.cur.r.low(p), head = units.cur.u;
        const int32_t* row = p.table + units.cur.b * p.table_stride;
        auto fetch = [&](int t) {
            const int key0 = units.key_of(t), key = key0 + lane * page_tokens;
            int id = outside;
            if (lane < per_tile && key < len && (key + page_tokens > low || key < p.sinks)) id = __ldg(row + (key >> p.page_shift));
            return id;                                     // looked at when it is used: the load travels meanwhile
        };
        int ahead = fetch(units.t_begin), k_ids = 0, v_ids = 0;
        const int n_loads = 2 * (units.t_end - units.t_begin);
        int j = units.t_begin;                             // next K tile
        for (int ld = 0; ld < n_loads; ++ld) {
            if (c.given_up()) return;
            const bool is_v = W::kRawTiles ? ld & 1 : ld == n_loads - 1 || (ld > 0 && (ld & 1) == 0);
            int ids;
            if (!is_v) {
                v_ids = k_ids;
                k_ids = ids = (uint32_t)ahead < (uint32_t)outside ? ahead : outside;
                if (++j < units.t_end) ahead = fetch(j);
            } else {
                ids = W::kRawTiles || ld == n_loads - 1 ? k_ids : v_ids;
            }
            if constexpr (W::kRawTiles) {
                const uint32_t fbar = c.bars + (kWRawFull + raw.slot) * 8, dst = c.smem + W::kRawAt + raw.slot * W::kRawBytes;
                if (lane == 0) {
                    c.wait(kWRawEmpty + raw.slot, raw.par, ld);
                    mbar_expect_tx(fbar, W::kRawBytes);
                }
                __syncwarp();
                if (lane < per_tile) {
                    const uint32_t row_bytes = kKind == kE4m3 ? 128u : 64u;
                    tma_load_4d(dst + lane * page_tokens * row_bytes, is_v ? maps.v : maps.k, fbar, 0, head, 0, ids);
                    if (kKind == kMx4)
                        tma_load_3d(dst + W::kRawCodes + lane * page_tokens * 16, is_v ? maps.v_exp : maps.k_exp, fbar, head * 4 & ~15, 0, ids);
                }
                raw.advance();
            } else {
                const uint32_t slot = is_v ? W::kStagesK + vr.slot : kr.slot;
                const uint32_t fbar = c.bars + (is_v ? kWVFull + vr.slot : kWKFull + kr.slot) * 8, dst = c.smem + W::kKV + slot * kTileBytes;
                if (lane == 0) {
                    c.wait(is_v ? kWVEmpty + vr.slot : kWKEmpty + kr.slot, is_v ? vr.par : kr.par, ld);
                    mbar_expect_tx(fbar, kTileBytes);
                }
                __syncwarp();
                if (lane < per_tile) {
#pragma unroll
                    for (int half = 0; half < 2; ++half)
                        tma_load_4d(dst + half * kHalfBytes + lane * page_tokens * 128, is_v ? maps.v : maps.k, fbar, half * 64, head, 0, ids);
                }
                if (is_v) vr.advance();
                else kr.advance();
            }
            __syncwarp();
        }
    }
}

// 16-byte chunk (of 16) of query row i: lines of 64 dims with the 128-byte swizzle, tiles of 128 rows
__device__ __forceinline__ uint32_t wide_place(uint32_t q, int i, int chunk) {
    const int in = i & (kBlockM - 1);
    return q + (i / kBlockM) * kTileBytes + (chunk >> 3) * kHalfBytes + in * 128 + (((chunk & 7) ^ (in & 7)) << 4);
}

// ---------------------------------------------------------------------------------------------- widening
// The query rows of a unit, in place, two a step of a warp.  E4M3: to fp16, scaled per row by a power of two that brings the largest element to [2^10, 2^11)
// (what falls below 2^-24 of it is lost); the sign of the keys' scale joins here.  4-bit: elements i and i + 4 of every eight side by side.  Spread over the
// widening warps, as the one that gathers the rows needs 9 us for 64 rows of E4M3.
template <Kind kKind, int kTiles>
__device__ __forceinline__ void wide_convert(const WideParams& w, const WideCtx& c, const WideUnits& units, int cw, int warps, int round) {
    using W = Wide<kKind, kTiles>;
    constexpr int kBatch = 4;                              // steps that go together
    const DecodeParams& p = w.d;
    const int lane = threadIdx.x & 31, chunk = lane & 15, sub = lane >> 4;
    const int rows = min(w.class_rows, p.rows - w.cls() * w.class_rows);
    const float sign = kKind == kE4m3 ? p.k_scale[units.cur.u] : 1.f;
    c.wait(kWQRaw, round & 1, round);
    __syncwarp();
#pragma unroll 1
    for (int i0 = 2 * cw; i0 < rows; i0 += 2 * warps * kBatch) {      // the same for all lanes
        uint4 x[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const int i = i0 + 2 * warps * k + sub;
            x[k] = make_uint4(0, 0, 0, 0);
            if (i < rows) x[k] = lds128(wide_place(c.smem + W::kQ, i, chunk));
        }
        // E4M3: the largest magnitude of every row, as bits: the exponent is enough, and infinities and NaN stay the largest
        uint32_t top[kBatch];
        if (kKind == kE4m3) {
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const uint32_t two = __vmaxu2(__vmaxu2(x[k].x & 0x7fff7fffu, x[k].y & 0x7fff7fffu), __vmaxu2(x[k].z & 0x7fff7fffu, x[k].w & 0x7fff7fffu));
                top[k] = max(two & 0xffffu, two >> 16);
            }
#pragma unroll
            for (int o = 8; o > 0; o >>= 1)
#pragma unroll
                for (int k = 0; k < kBatch; ++k) top[k] = max(top[k], __shfl_xor_sync(0xffffffffu, top[k], o));
        }
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const int i = i0 + 2 * warps * k + sub;
            if (i >= rows) continue;
            const uint32_t at = wide_place(c.smem + W::kQ, i, chunk);
            if (kKind == kMx4) {
                sts128(at, make_uint4(__byte_perm(x[k].x, x[k].z, 0x5410), __byte_perm(x[k].x, x[k].z, 0x7632),
                                      __byte_perm(x[k].y, x[k].w, 0x5410), __byte_perm(x[k].y, x[k].w, 0x7632)));
            } else {
                const int field = (int)(top[k] >> 7);      // of a zero or subnormal row 0
                const int e = top[k] == 0 || field == 255 ? 0 : min(137 - max(field, 1), 126);
                const float up = copysignf(__uint_as_float((uint32_t)(127 + e) << 23), sign);
                const uint32_t word[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
                uint32_t o[4];
#pragma unroll
                for (int n = 0; n < 4; ++n) o[n] = pack_weights<true>(__uint_as_float(word[n] << 16) * up, __uint_as_float(word[n] & 0xffff0000u) * up);
                sts128(at, make_uint4(o[0], o[1], o[2], o[3]));
                if (chunk == 0) reinterpret_cast<int8_t*>(c.gen + W::kExp)[(round & 1) * kWideRows + i] = (int8_t)e;
            }
        }
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) mbar_arrive(c.bars + kWQFull * 8);
}

// A share of every raw tile each.  16 E4M3 codes -> 16 fp16 values; a block of 32 4-bit codes -> 32 bf16 values, in whose groups of eight elements i and
// i + 4 stand side by side (the queries are laid out alike, and the columns of O are taken in that order).  The copies leave 16-byte chunk x of key k at
// chunk x ^ (k & 7) of its row (4-bit rows of four chunks: x ^ (k / 2 & 3)), so that eight lanes with eight keys and the same chunk meet no bank twice.
template <Kind kKind, int kTiles>
__device__ __forceinline__ void wide_widen(const WideParams& w, const WideCtx& c, WideUnits& units, int cw) {
    using W = Wide<kKind, kTiles>;
    const int lane = threadIdx.x & 31, warps = W::kHelp ? wide_widening<kKind, kTiles>(w) : kConvWarps;
    WideRing<W::kRawTiles ? W::kRaw : 1> raw = {0, 0};
    WideRing<W::kStagesK> kr = {0, 1};
    WideRing<W::kStagesV> vr = {0, 1};
    for (int round = 0; units.valid; units.next(w.d), ++round) {
        const int n = 2 * (units.t_end - units.t_begin);
        const int exp_byte = W::kRawCodes + (units.cur.u & 3) * 4;
#pragma unroll 1
        for (int ld = 0; ld < n; ++ld) {
            const bool is_v = ld & 1;
            if (ld == 1) wide_convert<kKind, kTiles>(w, c, units, cw, warps, round);
            c.wait(kWRawFull + raw.slot, raw.par, ld);
            c.wait(is_v ? kWVEmpty + vr.slot : kWKEmpty + kr.slot, is_v ? vr.par : kr.par, ld);
            __syncwarp();
            const uint32_t src = c.smem + W::kRawAt + raw.slot * W::kRawBytes;
            const uint32_t tile = c.smem + W::kKV + (is_v ? W::kStagesK + vr.slot : kr.slot) * kTileBytes;
            if (kKind == kE4m3) {
                // a step is 8 keys x all 8 chunks of 16 codes, two a lane
                const int k7 = lane & 7, x = lane >> 3;
                const uint32_t in0 = ((x ^ k7) << 4), in1 = (((x + 4) ^ k7) << 4), out0 = (((2 * x & 7) ^ k7) << 4), out1 = (((2 * x + 1 & 7) ^ k7) << 4);
                uint32_t from = src + (cw * 8 + k7) * 128, row = tile + (cw * 8 + k7) * 128;
                uint4 q0 = lds128(from + in0), q1 = lds128(from + in1);
#pragma unroll 1
                for (int i = cw; i < 16; i += warps) {
                    const uint4 a = q0, b = q1;
                    if (i + warps < 16) {
                        from += warps * 8 * 128;
                        q0 = lds128(from + in0);
                        q1 = lds128(from + in1);
                    }
                    // chunks 0 to 3 are the first 64 dims
                    uint4 lo, hi;
                    widen4(a.x, lo.x, lo.y);
                    widen4(a.y, lo.z, lo.w);
                    widen4(a.z, hi.x, hi.y);
                    widen4(a.w, hi.z, hi.w);
                    sts128(row + out0, lo);
                    sts128(row + out1, hi);
                    widen4(b.x, lo.x, lo.y);
                    widen4(b.y, lo.z, lo.w);
                    widen4(b.z, hi.x, hi.y);
                    widen4(b.w, hi.z, hi.w);
                    sts128(row + kHalfBytes + out0, lo);
                    sts128(row + kHalfBytes + out1, hi);
                    row += warps * 8 * 128;
                }
            } else {
                // a step is 8 keys x 4 blocks
                const int k7 = lane & 7, x = lane >> 3;
                uint32_t from = src + (cw * 8 + k7) * 64 + ((x ^ (k7 >> 1)) << 4), e_from = src + exp_byte + (cw * 8 + k7) * 16;
                uint32_t row = tile + (x >> 1) * kHalfBytes + (cw * 8 + k7) * 128;
                uint4 q = lds128(from);
                uint32_t word = lds32(e_from);
#pragma unroll 1
                for (int i = cw; i < 16; i += warps) {
                    const uint32_t codes[4] = {q.x, q.y, q.z, q.w}, e = word >> (8 * x) & 255;
                    if (i + warps < 16) {
                        q = lds128(from += warps * 8 * 64);
                        word = lds32(e_from += warps * 8 * 16);
                    }
                    // one factor of 2^(e - 127 + 126) while it is a bf16 number, else 2^126 and 2^(e - 127)
                    const bool near = __all_sync(0xffffffffu, e - 1 < 128u);
                    const uint32_t f = near ? (e + 126) * 0x00800080u : 0x7e807e80u;
                    uint4 o[4];
#pragma unroll
                    for (int n4 = 0; n4 < 4; ++n4)
                        o[n4] = make_uint4(mul_bf16x2(small_bf16<0>(codes[n4]), f), mul_bf16x2(small_bf16<1>(codes[n4]), f),
                                           mul_bf16x2(small_bf16<2>(codes[n4]), f), mul_bf16x2(small_bf16<3>(codes[n4]), f));
                    if (!near) {
                        const uint32_t f2 = e == 0 ? 0x00400040u : (e == 255 ? 0x7fc07fc0u : e * 0x00800080u);
#pragma unroll
                        for (int n4 = 0; n4 < 4; ++n4) o[n4] = make_uint4(mul_bf16x2(o[n4].x, f2), mul_bf16x2(o[n4].y, f2), mul_bf16x2(o[n4].z, f2), mul_bf16x2(o[n4].w, f2));
                    }
#pragma unroll
                    for (int n4 = 0; n4 < 4; ++n4) sts128(row + (((4 * x + n4 & 7) ^ k7) << 4), o[n4]);
                    row += warps * 8 * 128;
                }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");          // the tensor cores read what these lanes wrote
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(c.bars + (is_v ? kWVFull + vr.slot : kWKFull + kr.slot) * 8);
                mbar_arrive(c.bars + (kWRawEmpty + raw.slot) * 8);
            }
            raw.advance();
            if (is_v) vr.advance();
            else kr.advance();
        }
    }
}

// ---------------------------------------------------------------------------------------------- queries
// Row i of the unit's class is token (r0 + i) / G, head (r0 + i) % G of the group; rows without a token are zeros.  The widening warps convert them.
template <Kind kKind, int kTiles>
__device__ __forceinline__ void wide_queries(const WideParams& w, const WideCtx& c, WideUnits& units) {
    using W = Wide<kKind, kTiles>;
    const DecodeParams& p = w.d;
    const int lane = threadIdx.x & 31, chunk = lane & 15, sub = lane >> 4;
    const int r0 = w.cls() * w.class_rows, rows = min(w.class_rows, p.rows - r0);
    auto place = [&](int i) { return wide_place(c.smem + W::kQ, i, chunk); };
    for (int i = sub; i < kTiles * kBlockM; i += 2)        // rows behind the class's last stay zeros
        if (i >= rows) sts128(place(i), make_uint4(0, 0, 0, 0));
    if (kKind == kE4m3)
        for (int i = lane; i < 2 * kWideRows; i += 32) reinterpret_cast<int8_t*>(c.gen + W::kExp)[i] = 0;
    const int t0 = (r0 + sub) / p.G, h0 = r0 + sub - t0 * p.G;            // token and head of this lane's first row
    const int64_t wrap = (int64_t)(p.Hq - p.G) * kDim;     // elements from the group's heads of a token to the next token's
    for (int round = 0; units.valid && !c.given_up(); units.next(p), ++round) {
        const int b = units.cur.b, m = units.cur.r.len - units.cur.r.base;
        const int live = min(rows, m * p.G - r0);
        const __nv_bfloat16* src = p.q + (((int64_t)b * p.n_q + t0) * p.Hq + (int64_t)units.cur.u * p.G + h0) * kDim + chunk * 8;
        c.wait(kWQEmpty, (round & 1) ^ 1, round);
        __syncwarp();
        int h = h0;
#pragma unroll 4
        for (int i = sub; i < rows; i += 2) {
            const bool ok = i < live;
            cp_async16_or_zeros(place(i), ok ? src : p.q, ok);
            src += 2 * kDim;
            for (h += 2; h >= p.G; h -= p.G) src += wrap;
        }
        cp_commit();
        cp_wait<0>();
        __syncwarp();
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // the tensor cores read what these lanes wrote
        __syncwarp();
        if (lane == 0) mbar_arrive(c.bars + (W::kRawTiles ? kWQRaw : kWQFull) * 8);
    }
}

// ---------------------------------------------------------------------------------------------- issuers
template <Kind kKind, int kTiles>
__device__ __forceinline__ void wide_scores(const WideParams& w, const WideCtx& c, WideUnits& units) {
    using W = Wide<kKind, kTiles>;
    constexpr uint32_t kIdesc = kKind == kE4m3 ? kIdescS & ~((1u << 7) | (1u << 10)) : kIdescS;      // fp16 or bf16 operands
    WideRing<W::kStagesK> pos = {0, 0};
    uint32_t f_par0 = 0, f_par1 = 0;   // parity of "the scores are read", per warpgroup
    int prev = -1;                     // whose scores are in S
    const uint64_t q_desc = make_desc(c.smem + W::kQ, 16, 1024), k_desc = make_desc(c.smem + W::kKV, 16, 1024);
    for (int round = 0; units.valid; units.next(w.d), ++round) {
        const int j0 = units.t_begin, n = units.t_end;
        c.wait(kWQFull, round & 1, round);
#pragma unroll 1
        for (int j = j0; j < n; ++j) {
            if (c.given_up()) return;
            c.wait(kWKFull + pos.slot, pos.par, j);
            for (int q = 0; q < kTiles; ++q) {
                if (prev >= 0) {
                    c.wait(kWSFree + prev, prev ? f_par1 : f_par0, j);
                    if (prev) f_par1 ^= 1u;
                    else f_par0 ^= 1u;
                }
                prev = kTiles == 2 ? q : (j - j0) & 1;
                tc_fence_after();
                if (elect_one()) {
#pragma unroll
                    for (int ks = 0; ks < kD / 16; ++ks) {
                        const uint32_t off = ((ks >> 2) * kHalfBytes + (ks & 3) * 32) >> 4;
                        mma_ss(c.tmem + kWTmemS, q_desc + q * (kTileBytes >> 4) + off, k_desc + pos.slot * (kTileBytes >> 4) + off, kIdesc, ks > 0);
                    }
                    tc_commit(c.bars + (kWSReady + prev) * 8);
                    if (q == kTiles - 1) {
                        tc_commit(c.bars + (kWKEmpty + pos.slot) * 8);
                        if (j == n - 1) tc_commit(c.bars + kWQEmpty * 8);
                    }
                }
                __syncwarp();
            }
            pos.advance();
        }
    }
}

// The V of a tile that hides keys from some row: keys that no row sees lose what is no finite number; so do those that only some rows
// see, which are listed (as odd_values takes them).  Those that every row sees keep it: every row becomes that.
template <bool kF16>
__device__ __forceinline__ uint32_t odd_halves(uint32_t w) {
    return kF16 ? ((w & 0x7c007c00u) + 0x04000400u) & 0x80008000u : not_finite<false>(w);
}
template <bool kF16>
__device__ __forceinline__ uint32_t finite_halves(uint32_t w) {
    const uint32_t top = odd_halves<kF16>(w);
    return w & ~(top | (top - (top >> 15)));
}
// x * 0 + acc of two values: NaN from the first infinity or NaN on
template <bool kF16>
__device__ __forceinline__ uint32_t times_zero(uint32_t x, uint32_t acc) {
    if (kF16) asm("fma.rn.f16x2 %0, %1, %2, %0;" : "+r"(acc) : "r"(x), "r"(0u));
    else asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(acc) : "r"(x), "r"(0u));
    return acc;
}
template <bool kF16>
__device__ __forceinline__ void wide_clear(const DecodeParams& p, const Request& r, uint32_t v_tile, int key0, unsigned long long* odd) {
    const int lane = threadIdx.x & 31, low = r.low(p), low_max = r.len - p.window;
    uint32_t a0 = 0, a1 = 0, a2 = 0, a3 = 0;
#pragma unroll 8
    for (int i = lane; i < 2 * (int)kHalfBytes / 16; i += 32) {
        const uint4 x = lds128(v_tile + i * 16);
        a0 = times_zero<kF16>(x.x, a0);
        a1 = times_zero<kF16>(x.y, a1);
        a2 = times_zero<kF16>(x.z, a2);
        a3 = times_zero<kF16>(x.w, a3);
    }
    const uint32_t any = odd_halves<kF16>(a0) | odd_halves<kF16>(a1) | odd_halves<kF16>(a2) | odd_halves<kF16>(a3);
    if (!__any_sync(0xffffffffu, any != 0)) return;        // the rule
#pragma unroll 1
    for (int i = lane; i < 2 * (int)kHalfBytes / 16; i += 32) {
        const uint4 x = lds128(v_tile + i * 16);
        const uint32_t bad = odd_halves<kF16>(x.x) | odd_halves<kF16>(x.y) | odd_halves<kF16>(x.z) | odd_halves<kF16>(x.w);
        if (bad == 0) continue;
        const int key = key0 + (i >> 3 & (kBlockN - 1));
        const bool nobody = key >= r.len || (key < low && key >= p.sinks);
        const bool late = key >= r.base, early = key < low_max && key >= p.sinks;
        if (!nobody && !late && !early) continue;
        sts128(v_tile + i * 16, make_uint4(finite_halves<kF16>(x.x), finite_halves<kF16>(x.y), finite_halves<kF16>(x.z), finite_halves<kF16>(x.w)));
        if (!nobody) atomicOr(odd + (late ? 0 : 1), 1ull << (late ? key - r.base : key - low));
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
}

template <Kind kKind, int kTiles>
__device__ __forceinline__ void wide_outputs(const WideParams& w, const WideCtx& c, WideUnits& units) {
    using W = Wide<kKind, kTiles>;
    constexpr uint32_t kIdesc = kKind == kE4m3 ? kIdescPV & ~((1u << 7) | (1u << 10)) : kIdescPV;
    const DecodeParams& p = w.d;
    const int lane = threadIdx.x & 31;
    WideRing<W::kStagesV> pos = {0, 0};
    uint32_t p_par0 = 0, p_par1 = 0;   // parity of "P is there", per warpgroup
    const uint64_t v_desc = make_desc(c.smem + W::kKV + W::kStagesK * kTileBytes, kHalfBytes, 1024);
    for (int round = 0; units.valid; units.next(p), ++round) {
        const int j0 = units.t_begin, n = units.t_end;
        unsigned long long* odd = reinterpret_cast<unsigned long long*>(c.gen + W::kOdd) + 2 * (round & 1);
        // Its readers, of the unit before the last, took their copies before they arrived at kWOFree, which the first tiles of the last unit waited for: with
        // two score tiles one barrier for each of the warpgroups, with one the first tile's for both.
        if (lane < 2) odd[lane] = 0;
        __syncwarp();
#pragma unroll 1
        for (int j = j0; j < n; ++j) {
            if (c.given_up()) return;
            c.wait(kWVFull + pos.slot, pos.par, j);
            const int key0 = units.key_of(j);
            if (!units.full(p, key0)) wide_clear<kKind == kE4m3>(p, units.cur.r, c.smem + W::kKV + (W::kStagesK + pos.slot) * kTileBytes, key0, odd);
            for (int q = 0; q < kTiles; ++q) {
                const int h = kTiles == 2 ? q : (j - j0) & 1;
                const bool fresh = kTiles == 2 ? j == j0 : j - j0 < 2;             // the accumulator's first tile of the unit
                if (fresh && round > 0) c.wait(kWOFree + h, (round - 1) & 1, j);
                const uint32_t p_par = h ? p_par1 : p_par0;
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    c.wait(kWPReady + 2 * h + part, p_par, j);
                    tc_fence_after();
                    if (elect_one()) {
#pragma unroll
                        for (int ks = 0; ks < 8; ++ks)
                            if ((ks < 2 * kWideSplit) == (part == 0))
                                mma_ts(c.tmem + kWTmemO + h * 128, c.tmem + kWTmemP + h * 64 + ks * 8, v_desc + pos.slot * (kTileBytes >> 4) + ks * (2048 >> 4),
                                       kIdesc, !fresh || ks > 0);
                        if (part == 1) {
                            tc_commit(c.bars + (kWPvDone + h) * 8);
                            if (q == kTiles - 1) tc_commit(c.bars + (kWVEmpty + pos.slot) * 8);
                        }
                    }
                    __syncwarp();
                }
                if (h) p_par1 ^= 1u;
                else p_par0 ^= 1u;
            }
            pos.advance();
        }
        if (lane == 0) mbar_arrive(c.bars + kWOdd * 8);
    }
}

// ---------------------------------------------------------------------------------------------- softmax
// Keys [k, k + 32) that a row sees: before base those of its window and the sinks, from base on those of its mask.
__device__ __forceinline__ uint32_t wide_seen(int k, int base, int low, int sinks, unsigned long long mask) {
    const uint32_t before = bits_below(base - k) & (~bits_below(low - k) | bits_below(sinks - k));
    const int d = k - base;
    const uint32_t drafts = d >= 64 || d <= -32 ? 0u : (d >= 0 ? (uint32_t)(mask >> d) : (uint32_t)(mask << -d));
    return before | drafts;
}
__device__ __forceinline__ void wide_hide(float (&s)[32], uint32_t seen) {
#pragma unroll
    for (int i = 0; i < 32; ++i)
        if (!(seen >> i & 1u)) s[i] = -INFINITY;
}

// What wide_clear took out of the V that a row sees joins the elements [d0, d1) of the row just written.
template <Kind kKind>
__device__ __forceinline__ void wide_odd_row(const DecodeParams& p, unsigned long long late, unsigned long long early, int b, int base, int len, int u, int t, bool whole,
                                             int64_t at, int d0, int d1) {
#pragma unroll 1
    for (int dim = d0; dim < d1; ++dim) {
        const float x = odd_values<kKind, true>(p, late, early, b, base, len, u, t, dim);
        if (x == 0.f) continue;
        if (whole) p.out[at + dim] = __float2bfloat16_rn(__bfloat162float(p.out[at + dim]) + x);
        else p.part_o[at + dim] += x;
    }
}

#define CP_LOAD_S3(a0, a1, a2)       \
    TMEM_LD32(s_tmem + 0, a0, 0);    \
    TMEM_LD32(s_tmem + 32, a1, 0);   \
    TMEM_LD32(s_tmem + 64, a2, 0);

// 2^(s c - m) of 32 keys as 16 packed pairs, and their sums (unrounded).
template <bool kF16>
__device__ __forceinline__ void wide_exp32(const float (&s)[32], uint32_t (&pk)[16], float2 c2, float2 nm2, float2& sum0, float2& sum1, float2& sum2, float2& sum3) {
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
        float2 e[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 x = __ffma2_rn(make_float2(s[2 * (i + k)], s[2 * (i + k) + 1]), c2, nm2);
            e[k] = make_float2(ex2(x.x), ex2(x.y));
            pk[i + k] = pack_weights<kF16>(e[k].x, e[k].y);
        }
        sum0 = __fadd2_rn(sum0, e[0]);
        sum1 = __fadd2_rn(sum1, e[1]);
        sum2 = __fadd2_rn(sum2, e[2]);
        sum3 = __fadd2_rn(sum3, e[3]);
    }
}

// One score tile (in c0..c3): the row's maximum, the rescaling of O where it grows by more than the lag, the weights in four pieces.  If the unit has another
// tile, its scores replace the current ones before the function returns.
template <bool kF16>
__device__ __forceinline__ void wide_softmax_tile(const WideCtx& cx, float (&c0)[32], float (&c1)[32], float (&c2)[32], float (&c3)[32], int wg, bool more,
                                                  bool first, uint32_t& s_par, uint32_t pv_par, uint32_t s_tmem, uint32_t p_tmem, uint32_t o_tmem, float c,
                                                  float& m, float& l, int iter) {
    float mx0 = -INFINITY, mx1 = -INFINITY, mx2 = -INFINITY, mx3 = -INFINITY;
    max32(c0, mx0, mx1, mx2, mx3);
    max32(c1, mx0, mx1, mx2, mx3);
    max32(c2, mx0, mx1, mx2, mx3);
    max32(c3, mx0, mx1, mx2, mx3);
    const float m_new = fmaxf(m, fmaxf(fmaxf(mx0, mx1), fmaxf(mx2, mx3)) * c);
    if (first) {
        m = m_new;                     // O is overwritten by the first product
    } else {
        cx.wait(kWPvDone + wg, pv_par, iter);
        __syncwarp();
        tc_fence_after();
        const bool grow = m_new - m > kWideLag;
        if (__any_sync(0xffffffffu, grow)) {
            const float m_upd = grow ? m_new : m, alpha = ex2(m - m_upd);
            l *= alpha;
            m = m_upd;
#pragma unroll 1
            for (int cc = 0; cc < 4; ++cc) {
                float o[32];
                TMEM_LD32(o_tmem + cc * 32, o, 0);
                tc_wait_ld();
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] *= alpha;
                TMEM_ST32F(o_tmem + cc * 32, o, 0);
            }
        }
    }
    const float2 c2f = make_float2(c, c), nm2 = make_float2((kF16 ? kF16Shift : 0.f) - m, (kF16 ? kF16Shift : 0.f) - m);      // fp16 weights carry 2^7
    float2 sum0 = make_float2(0.f, 0.f), sum1 = sum0, sum2 = sum0, sum3 = sum0;
    uint32_t pk[16];
    const uint32_t p_bar = cx.bars + (kWPReady + 2 * wg) * 8;
#define CP_WIDE_PIECE(cur, q)                                                           \
    wide_exp32<kF16>(cur, pk, c2f, nm2, sum0, sum1, sum2, sum3);                            \
    TMEM_ST16R(p_tmem + (q) * 16, pk, 0);                                               \
    if ((q) + 1 == kWideSplit || (q) == 3) {                                            \
        tc_wait_st();                                                                   \
        tc_fence_before();                                                              \
        __syncwarp();                                                                   \
        if ((threadIdx.x & 31) == 0) mbar_arrive(p_bar + ((q) == 3 ? 8 : 0));    \
    }
    CP_WIDE_PIECE(c0, 0)
    CP_WIDE_PIECE(c1, 1)
    CP_WIDE_PIECE(c2, 2)
    bool early = false;                // is the next score tile there already?  (the same answer in the whole warp)
    if (more) {
        early = __all_sync(0xffffffffu, mbar_test(cx.bars + (kWSReady + wg) * 8, s_par));
        if (early) {
            tc_fence_after();
            CP_LOAD_S3(c0, c1, c2)
        }
    }
    CP_WIDE_PIECE(c3, 3)
#undef CP_WIDE_PIECE
    if (more) {
        if (!early) {
            cx.wait(kWSReady + wg, s_par, iter);
            __syncwarp();
            tc_fence_after();
            CP_LOAD_S3(c0, c1, c2)
        }
        TMEM_LD32(s_tmem + 96, c3, 0);
        tc_wait_ld();
        tc_fence_before();
        __syncwarp();
        if ((threadIdx.x & 31) == 0) mbar_arrive(cx.bars + (kWSFree + wg) * 8);
        s_par ^= 1u;
    }
    const float2 st = __fadd2_rn(__fadd2_rn(sum0, sum1), __fadd2_rn(sum2, sum3));
    l += st.x + st.y;
}

// Column of O that holds element i of a head (see wide_widen).
template <Kind kKind>
__device__ __forceinline__ constexpr int wide_column(int i) { return kKind == kMx4 ? (i & ~7) | (i & 3) << 1 | (i >> 2 & 1) : i; }

template <Kind kKind, int kTiles>
__device__ __forceinline__ void wide_softmax(const WideParams& w, const WideCtx& cx, WideUnits& units, int wg, int64_t total, int ctas) {
    using W = Wide<kKind, kTiles>;
    constexpr bool kF16 = kKind == kE4m3;
    const DecodeParams& p = w.d;
    const int lane = threadIdx.x & 31, warp_in_wg = threadIdx.x >> 5 & 3;
    const uint32_t lane_addr = (uint32_t)(warp_in_wg * 32) << 16;
    const uint32_t s_tmem = cx.tmem + lane_addr + kWTmemS, p_tmem = cx.tmem + lane_addr + kWTmemP + wg * 64, o_tmem = cx.tmem + lane_addr + kWTmemO + wg * 128;
    const int cls = w.cls(), run = w.run();
    constexpr bool turns = W::kTurns;
    const int tile_row = warp_in_wg * 32 + lane, row = (turns ? 0 : wg * kBlockM) + tile_row;      // of the class
    const int r = cls * w.class_rows + row, t = r / p.G;                  // of the KV head; its token
    const bool in_class = row < w.class_rows && r < p.rows;
    constexpr int step = turns ? 2 : 1;
    if (!W::kHelp && warp_in_wg >= wide_warps<kTiles>(w, wg)) return;
    float c = p.scale_log2;
    uint32_t s_par = 0, tile_cnt = 0;
    for (int round = 0; units.valid; ++round) {
        const Request rq = units.cur.r;
        const int b = units.cur.b, u = units.cur.u, j0 = units.t_begin, n = units.t_end, m_tree = rq.len - rq.base;
                const bool live = in_class && t < m_tree;                         // rows without a token: zeros, -inf
        TreeRow tr;
        tr.mask = 0;
        tr.lim = 0;
        if (live) tr = tree_row(p, b, t, rq.base, m_tree);
        const int low = (live ? tr.lim : rq.len) - p.window;
        const int j1 = j0 + (turns ? wg : 0);                             // this warpgroup's first tile
        const bool some = j1 < n;
        float m = kNoKey, l = 0.f;
        if (some && !__any_sync(0xffffffffu, live)) {                     // none of this warp's rows: whatever P and O hold there, nobody takes it
#pragma unroll 1
            for (int j = j1; j < n; j += step) {
                cx.wait(kWSReady + wg, s_par, j);
                s_par ^= 1u;
                __syncwarp();
                if (lane == 0) mbar_arrive(cx.bars + (kWSFree + wg) * 8);
                if (j > j1) cx.wait(kWPvDone + wg, (tile_cnt - 1) & 1, j);
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(cx.bars + (kWPReady + 2 * wg) * 8);
                    mbar_arrive(cx.bars + (kWPReady + 2 * wg + 1) * 8);
                }
                ++tile_cnt;
            }
            cx.wait(kWPvDone + wg, (tile_cnt - 1) & 1, n);
            __syncwarp();
            tc_fence_after();
        } else if (some) {
            float s0[32], s1[32], s2[32], s3[32];
            int e = 0;
            cx.wait(kWSReady + wg, s_par, j1);
            __syncwarp();
            s_par ^= 1u;
            tc_fence_after();
            CP_LOAD_S3(s0, s1, s2)
            TMEM_LD32(s_tmem + 96, s3, 0);
            // before this warp says that S is free: the next unit's scores may then be computed, and the queries of the one behind it overwrite the exponent
            if (kF16) e = reinterpret_cast<const volatile int8_t*>(cx.gen + W::kExp)[(round & 1) * kWideRows + row];
            tc_wait_ld();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(cx.bars + (kWSFree + wg) * 8);
            // c > 0: the sign of a scale is in the queries; with a scale of zero hidden keys must still be -inf
            if (kF16) c = fmaxf(fabsf(p.k_scale[u]) * p.scale_log2 * __uint_as_float((uint32_t)(127 - e) << 23), 1e-35f);
#pragma unroll 1
            for (int j = j1; j < n; j += step) {
                const int key0 = units.key_of(j);
                if (!units.full(p, key0)) {
                    wide_hide(s0, wide_seen(key0, rq.base, low, p.sinks, tr.mask));
                    wide_hide(s1, wide_seen(key0 + 32, rq.base, low, p.sinks, tr.mask));
                    wide_hide(s2, wide_seen(key0 + 64, rq.base, low, p.sinks, tr.mask));
                    wide_hide(s3, wide_seen(key0 + 96, rq.base, low, p.sinks, tr.mask));
                }
                wide_softmax_tile<kF16>(cx, s0, s1, s2, s3, wg, j + step < n, j == j1, s_par, (tile_cnt - 1) & 1, s_tmem, p_tmem, o_tmem, c, m, l, j);
                ++tile_cnt;
            }
            cx.wait(kWPvDone + wg, (tile_cnt - 1) & 1, n);
            __syncwarp();
            tc_fence_after();
        }
        const bool whole = units.whole;
        const int64_t x_end = units.cur.x + kWideCost + rq.n;
        float f0 = 1.f, f1 = 0.f;                                         // factors of the accumulators
        const bool both = turns && n - j0 > 1;
        if (turns) {
            // the warpgroups tell one another their maxima and sums; then each reads half of the columns of both accumulators, which lie in the same lanes
            // Without a tile of this unit nothing has kept this warp behind the others: one of them may still be in the last unit, and this one's arrival would be taken
            // for the other's there.  (With a tile, the first product onto the accumulator has waited for the same barrier.)
            if (!some && round > 0) cx.wait(kWOFree + wg, (round - 1) & 1, n);
            float2* ml = reinterpret_cast<float2*>(cx.gen + W::kMl) + (round & 1) * 2 * kBlockM;
            ml[wg * kBlockM + tile_row] = make_float2(m, l);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(cx.bars + (kWMl + wg) * 8);
            cx.wait(kWMl + (wg ^ 1), round & 1, n);
            __syncwarp();
            tc_fence_after();
            const float2 o = ml[(wg ^ 1) * kBlockM + tile_row];
            const float mx = fmaxf(m, o.x), own = ex2(m - mx), other = ex2(o.x - mx);
            l = l * own + o.y * other;
            m = mx;
            f0 = wg == 0 ? own : other;
            f1 = wg == 0 ? other : own;
        }
        cx.wait(kWOdd, round & 1, n);
        __syncwarp();
        // a copy of the list, before this warp arrives at kWOFree: from then on it may be cleared for the unit after the next
        const volatile unsigned long long* odd = reinterpret_cast<const volatile unsigned long long*>(cx.gen + W::kOdd) + 2 * (round & 1);
        const unsigned long long odd_late = odd[0], odd_early = odd[1];
        const bool any_odd = live && (odd_late | odd_early) != 0;
        const float inv = !whole ? 1.f : (l == 0.f ? 0.f : (kF16 ? p.v_scale[u] : 1.f) / l);
        f0 *= inv;
        f1 *= inv;
        const int64_t slot = 2 * w.place() + (j0 > 0 ? 0 : 1);
        const int head = u * p.G + r - t * p.G;
        // offset of this row in the destination, -1: none
        const int64_t at = !in_class ? -1 : (whole ? (((int64_t)b * p.n_q + t) * p.Hq + head) * kD : (slot * kWideRows + row) * kD);
        const int qt = lane & 3;
        const uint32_t acc0 = turns ? cx.tmem + lane_addr + kWTmemO : o_tmem, acc1 = cx.tmem + lane_addr + kWTmemO + 128;
        int64_t to[4];                 // of the rows of this lane's quad: the lanes swap 16-byte pieces, so that a store writes 64 contiguous bytes of a row
#pragma unroll
        for (int i = 0; i < 4; ++i) to[i] = __shfl_sync(0xffffffffu, at, (lane & ~3) + i);
        const int cc0 = turns ? 2 * wg : 0, cc1 = turns ? cc0 + 2 : 4;
#pragma unroll 1
        for (int cc = cc0; cc < cc1; ++cc) {
            float o[32];
            TMEM_LD32(acc0 + cc * 32, o, 0);
            if (both) {
                float o1[32];
                TMEM_LD32(acc1 + cc * 32, o1, 0);
                tc_wait_ld();
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = live ? o[i] * f0 + o1[i] * f1 : 0.f;
            } else {
                tc_wait_ld();
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = live ? o[i] * f0 : 0.f;
            }
            if (whole) {
                uint4 v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
#define CP_O(k) o[wide_column<kKind>(8 * i + (k))]
                    v[i] = make_uint4(pack_bf16(CP_O(0), CP_O(1)), pack_bf16(CP_O(2), CP_O(3)), pack_bf16(CP_O(4), CP_O(5)), pack_bf16(CP_O(6), CP_O(7)));
#undef CP_O
                }
                quad_transpose(v, qt);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (to[i] >= 0) *reinterpret_cast<uint4*>(p.out + to[i] + cc * 32 + qt * 8) = v[i];
            } else {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    uint4 v[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int k = half * 16 + 4 * i;
                        v[i] = make_uint4(__float_as_uint(o[wide_column<kKind>(k)]), __float_as_uint(o[wide_column<kKind>(k + 1)]),
                                          __float_as_uint(o[wide_column<kKind>(k + 2)]), __float_as_uint(o[wide_column<kKind>(k + 3)]));
                    }
                    quad_transpose(v, qt);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (to[i] >= 0) *reinterpret_cast<uint4*>(p.part_o + to[i] + cc * 32 + half * 16 + qt * 4) = v[i];
                }
            }
        }
        tc_fence_before();
        __syncwarp();                  // also: the rows are written, by the lanes of their quads
        if (lane == 0) {
            if (turns) {
                mbar_arrive(cx.bars + kWOFree * 8);
                mbar_arrive(cx.bars + (kWOFree + 1) * 8);
            } else {
                mbar_arrive(cx.bars + (kWOFree + wg) * 8);
            }
        }
        if (any_odd) wide_odd_row<kKind>(p, odd_late, odd_early, b, rq.base, rq.len, u, t, whole, at, cc0 * 32, cc1 * 32);
        if (in_class && (!turns || wg == 0)) {
            if (whole) {
                p.lse[(int64_t)head * ((int64_t)p.B * p.n_q) + (int64_t)b * p.n_q + t] =
                    live && l != 0.f ? (m + log2f(l) - (kF16 ? kF16Shift : 0.f)) * 0.6931471805599453f : -INFINITY;
            } else {
                p.part_ml[(slot * kWideRows + row) * 2] = live ? m : kNoKey;
                p.part_ml[(slot * kWideRows + row) * 2 + 1] = live ? l : 0.f;
            }
        }
        if (threadIdx.x == 0 && !whole && j0 == 0) {
            // this CTA holds the unit's first piece: the last one ends with the unit's last tile, at place x_end - 1
            int64_t last = min((x_end * ctas - 1) / total, (int64_t)ctas - 1);
            while (run_begin(total, last, ctas) >= x_end) --last;
            while (run_begin(total, last + 1, ctas) < x_end) ++last;
            int32_t* meta = p.meta + w.place() * 4;
            meta[0] = b;
            meta[1] = u;
            meta[2] = (int32_t)(last - run + 1);
            meta[3] = 1;
        }
        units.next(p);
    }
}
#undef CP_LOAD_S3

template <Kind kKind, int kTiles>
__global__ void __launch_bounds__(Wide<kKind, kTiles>::kThreads, 1)
tree_wide_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_ke,
                 const __grid_constant__ CUtensorMap tm_ve, const __grid_constant__ WideParams w) {
    using W = Wide<kKind, kTiles>;
    constexpr int kThreadsHere = W::kThreads;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    const DecodeParams& p = w.d;
    WideCtx c;
    c.smem = smem_u32(smem_raw);
    c.gen = smem_raw;
    c.bars = c.smem + W::kBar;
    c.abort_flag = reinterpret_cast<volatile uint32_t*>(c.gen + W::kAbort);
    c.status = p.status;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int run = w.run();
    if (tid == 0) {
        const int widening = W::kRawTiles ? wide_widening<kKind, kTiles>(w) : 1;
        mbar_init(c.bars + kWQFull * 8, widening);
        mbar_init(c.bars + kWQRaw * 8, 1);
        mbar_init(c.bars + kWQEmpty * 8, 1);
        for (int s = 0; s < kMaxRing; ++s) {
            mbar_init(c.bars + (kWKFull + s) * 8, widening);
            mbar_init(c.bars + (kWKEmpty + s) * 8, 1);
            mbar_init(c.bars + (kWVFull + s) * 8, widening);
            mbar_init(c.bars + (kWVEmpty + s) * 8, 1);
        }
        for (int s = 0; s < W::kRaw; ++s) {
            mbar_init(c.bars + (kWRawFull + s) * 8, 1);
            mbar_init(c.bars + (kWRawEmpty + s) * 8, widening);
        }
        for (int h = 0; h < 2; ++h) {
            const int warps = wide_warps<kTiles>(w, h);    // one arrival per warp
            mbar_init(c.bars + (kWSReady + h) * 8, 1);
            mbar_init(c.bars + (kWSFree + h) * 8, warps);
            for (int q = 0; q < 2; ++q) mbar_init(c.bars + (kWPReady + 2 * h + q) * 8, warps);
            mbar_init(c.bars + (kWPvDone + h) * 8, 1);
            mbar_init(c.bars + (kWOFree + h) * 8, W::kTurns ? 2 * warps : warps);
            mbar_init(c.bars + (kWMl + h) * 8, warps);
        }
        mbar_init(c.bars + kWOdd * 8, 1);
        *c.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(c.smem + W::kTmemPtr), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    // where this CTA's run starts: requests are dealt to the threads in order, a prefix sum over their places finds it
    int64_t* scan = reinterpret_cast<int64_t*>(c.gen + W::kScan);
    int32_t* start = reinterpret_cast<int32_t*>(scan + kThreadsHere / 32);
    const int per = (p.B + kThreadsHere - 1) / kThreadsHere;
    int64_t mine = 0;
    for (int i = 0; i < per; ++i) {
        const int b = tid * per + i;
        if (b >= p.B) break;
        mine += request_of<kBlockN, true>(p, b).n + kWideCost;
        if ((blockIdx.x | blockIdx.y | blockIdx.z) == 0) {
            const int len = p.kv_len[b];
            if (len > p.capacity || len < 0) report_status(p.status, CP_ERR_BOUNDS, b, len);
            if (p.tree_len && (p.tree_len[b] < 0 || p.tree_len[b] > min(p.n_q, len))) report_status(p.status, CP_ERR_BOUNDS, b, p.tree_len[b]);
        }
    }
    int64_t inc = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += y;
    }
    if (lane == 31) scan[warp] = inc;
    if (tid == 0) p.meta[w.place() * 4 + 3] = 0;
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    c.tmem = *reinterpret_cast<volatile uint32_t*>(c.gen + W::kTmemPtr);
    int64_t before = inc - mine, total = 0;
    for (int i = 0; i < kThreadsHere / 32; ++i) {
        if (i < warp) before += scan[i];
        total += scan[i];
    }
    const int groups = p.Hkv / w.heads;
    total *= groups;
    before *= groups;
    const int ctas = (int)min((int64_t)w.runs, total);
    const int64_t x0 = run < ctas ? run_begin(total, run, ctas) : total, x1 = run < ctas ? run_begin(total, run + 1, ctas) : total;
    if (x0 >= before && x0 < before + mine * groups) {
        int b = tid * per;
        int64_t at = before;
        while (true) {
            const int64_t n = (int64_t)(request_of<kBlockN, true>(p, b).n + kWideCost) * groups;
            if (x0 < at + n) break;
            at += n;
            ++b;
        }
        const int n = request_of<kBlockN, true>(p, b).n + kWideCost;
        start[0] = b;
        start[1] = (int32_t)((x0 - at) / n);
        start[2] = (int32_t)((x0 - at) % n);
    }
    __syncthreads();
    if (x0 < x1) {
        WideUnits& units = *reinterpret_cast<WideUnits*>(c.gen + W::kUnits + warp * kUnitBytes);
        if (lane == 0) units.begin(w, start, x0, x1);
        __syncwarp();
        int widener = warp >= 12 ? warp - 12 : -1;
        if (W::kHelp && warp < 8) {
            const int wg = warp >> 2, spare = (warp & 3) - wide_warps<kTiles>(w, wg);
            if (spare >= 0) widener = kConvWarps + spare + (wg ? 4 - wide_warps<kTiles>(w, 0) : 0);
        }
        if (warp < 8) {
            asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(W::kRegsSoftmax));
            if (!W::kHelp || widener < 0) wide_softmax<kKind, kTiles>(w, c, units, warp >> 2, total, ctas);
        } else {
            asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(W::kRegsOther));
            if (warp == 9) {
                wide_scores<kKind, kTiles>(w, c, units);
            } else if (warp == 10) {
                wide_outputs<kKind, kTiles>(w, c, units);
            } else if (warp == 11) {
                wide_queries<kKind, kTiles>(w, c, units);
            } else if (warp == 8) {
                const WideMaps maps = {&tm_k, &tm_v, &tm_ke, &tm_ve};
                wide_producer<kKind, kTiles>(w, c, units, maps);
            } else if constexpr (W::kRawTiles && !W::kHelp) {
                wide_widen<kKind, kTiles>(w, c, units, warp - 12);
            }
        }
        if constexpr (W::kHelp) {
            if (widener >= 0) wide_widen<kKind, kTiles>(w, c, units, widener);     // one place, so one copy of the code
        }
    }
    let_next_launch_begin();           // not earlier: nothing is to be set up beside a block whose warps pass registers on
    tc_fence_before();
    __syncthreads();
    if (*c.abort_flag) {
        for (int i = 0; i < 200; ++i) __nanosleep(1000);   // copies in flight land before shared memory is released
        __syncthreads();
    }
    if (warp == 0) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(c.tmem), "r"(512u) : "memory");
    }
}

// Joins the pieces of cut units: CTA (v, y), v = class * runs + run of a unit's first piece; a warp a row.  Pieces: slot 2v + 1, then slots 2v', v' = v + 1, ..
constexpr int kWideJoinRows = 8;
template <Kind kKind>
__global__ void __launch_bounds__(32 * kWideJoinRows)
tree_join_kernel(const __grid_constant__ WideParams w) {
    const DecodeParams& p = w.d;
    wait_for_launch_before();
    const int v = blockIdx.x, row = blockIdx.y * kWideJoinRows + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    const int4 me = *reinterpret_cast<const int4*>(p.meta + 4 * v);
    const int r = v / w.runs % w.classes * w.class_rows + row;
    if (me.w == 0 || row >= w.class_rows || r >= p.rows) return;
    auto slot_of = [&](int k) { return (int64_t)(k == 0 ? 2 * v + 1 : 2 * (v + k)) * kWideRows + row; };
    float mx = kNoKey;
    for (int k = lane; k < me.z; k += 32) mx = fmaxf(mx, p.part_ml[slot_of(k) * 2]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
    float sum = 0.f;
#pragma unroll 4
    for (int k = 0; k < me.z; ++k) {
        const float2 ml = *reinterpret_cast<const float2*>(p.part_ml + slot_of(k) * 2);
        const float4 x = *reinterpret_cast<const float4*>(p.part_o + slot_of(k) * kD + lane * 4);
        const float f = exp2_fast(ml.x - mx);
        sum += f * ml.y;
        a.x += f * x.x;
        a.y += f * x.y;
        a.z += f * x.z;
        a.w += f * x.w;
    }
    const int t = r / p.G, head = me.y * p.G + r - t * p.G;
    const int64_t token = (int64_t)me.x * p.n_q + t;
    const float inv = sum == 0.f ? 0.f : (kKind == kE4m3 ? p.v_scale[me.y] : 1.f) / sum;
    uint2 out;
    out.x = pack_bf16(a.x * inv, a.y * inv);
    out.y = pack_bf16(a.z * inv, a.w * inv);
    *reinterpret_cast<uint2*>(p.out + (token * p.Hq + head) * kD + lane * 4) = out;
    if (lane == 0) p.lse[(int64_t)head * ((int64_t)p.B * p.n_q) + token] = sum == 0.f ? -INFINITY : (mx + log2f(sum) - (kKind == kE4m3 ? kF16Shift : 0.f)) * 0.6931471805599453f;
}

}  // namespace
