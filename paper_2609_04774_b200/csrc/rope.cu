// cp_rope_append: rotary positions with one to four axes applied to q and k, the rotated k and the v rows written to the
// paged cache (bf16, or E4M3 with a scale per head) in the same pass.
//
// Pair i of a head is a point (a, b) that is turned by the angle pos[axis(i)] * freq(i):
//     a' = a cos - b sin,   b' = b cos + a sin.
// Angles are kept in turns, as 64-bit fixed point: step(i) = freq(i) / 2 pi mod 1, scaled by 2^64, and the product
// pos * step wraps modulo one turn by itself, so a position of 10^6 or 2^31 loses nothing (an fp32 product would be off by
// 0.06 radians at 10^6).  The top 32 bits, read as a signed fraction in [-1/2, 1/2), go to sincospif as an fp32 number of half turns, whose
// rounding is the largest error of the angle: 2^-26 of a turn (cutting the bits off adds 2^-32, the step's own 2^-64 up to 2^-33).
//
// HBM-bound: q is read and written once, k and v are read once and written once (24 KB per token at 32 / 8 heads).  A warp takes
// the heads of one token in steps of four (8 lanes a head, two 16-byte vectors a lane), so the 64 sines and cosines of a token
// are computed once (two pairs a lane, handed round by shuffles) for all its heads.  With few tokens the steps of a
// token are dealt to several warps instead (the sines are then computed by each): see rope_append.
// Measured (device time): 16384 tokens, three axes, 74 us, 5.4 TB/s (E4M3 75 us), 65536 tokens 6.2 TB/s of the 6.45 that a copy reaches: at
// 16384 the last of 3.5 waves of warps costs the rest.  Steps cut into equal runs, one wave of warps: 72 us, but 1024 tokens 8.3 -> 10.1 us.
// 64 tokens: 3.4 us, one launch.  4-bit: 16384 tokens 97 us (three blocks an SM; 109 with two, 126 with four and spills; 90 without the check of every key's codes), 64
// tokens 5 us.
#include <cuda_bf16.h>
#include <math.h>

#include <algorithm>

#include "device_util.cuh"
#include "internal.h"

using namespace cpattn;

namespace {

constexpr int kHeadDim = 128;
constexpr int kRopeThreads = 256;

struct RopeParams {
    uint64_t step[64];          // turns per position step, 2^64 = one turn
    uint8_t axis[64];
    int32_t n_chunks;           // 16-byte chunks of a head that hold first elements of pairs (half layout); interleaved: rotated chunks
    int32_t n;                  // tokens
    int32_t Hq, Hkv;
    int32_t q_steps, kv_steps;  // steps of four heads
    int32_t steps_per_warp;     // steps one warp takes (of q_steps + 2 kv_steps)
    int32_t parts;              // warps per token
    const uint4* q;
    uint4* q_out;
    const uint4* k_rows;
    const uint4* v_rows;
    const int32_t* positions;   // [n_axes, n]
    const int32_t* seq;         // [n] row of the page table, < 0: the token is padding
    const int32_t* slot;        // [n] logical token of the sequence
    const int32_t* page_table;  // [rows, stride]
    int64_t table_rows, table_stride;
    uint8_t* cache_k;
    uint8_t* cache_v;
    const float* k_scale;
    const float* v_scale;
    int64_t num_pages, stride_page, stride_tok, stride_head;      // bytes
    int32_t page_shift;
    int32_t* status;
};

__device__ __forceinline__ void unpack8(const uint4& r, float (&x)[8]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);      // the one rounding of a rotated element
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
    return make_uint4(pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7]));
}
// E4M3 bytes of x / scale: IEEE quotient, round to nearest even, saturating at 448.
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
    return (uint32_t)lo | ((uint32_t)hi << 16);
}
__device__ __forceinline__ uint2 quantize8(const float (&x)[8], float sc, float inv) {
    // x * inv is within 2^-22 of the quotient (inv and the product are rounded once each); where 2^-21 less and 2^-21 more round to the
    // same code, so does the quotient.  The others divide: a border of the format in between (one element in 10^5), or a scale whose
    // reciprocal is no normal number.  16384 tokens at 32 / 8 heads: 83 -> 75 us.
    float lo[8], hi[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float y = x[i] * inv;
        lo[i] = y * 0.9999995f;
        hi[i] = y * 1.0000005f;
    }
    uint2 a = make_uint2(e4m3x4(lo[0], lo[1], lo[2], lo[3]), e4m3x4(lo[4], lo[5], lo[6], lo[7]));
    const uint2 b = make_uint2(e4m3x4(hi[0], hi[1], hi[2], hi[3]), e4m3x4(hi[4], hi[5], hi[6], hi[7]));
    if (a.x != b.x || a.y != b.y || !(fabsf(inv) >= 1.17549435e-38f && fabsf(inv) < INFINITY)) {
        a.x = e4m3x4(__fdiv_rn(x[0], sc), __fdiv_rn(x[1], sc), __fdiv_rn(x[2], sc), __fdiv_rn(x[3], sc));
        a.y = e4m3x4(__fdiv_rn(x[4], sc), __fdiv_rn(x[5], sc), __fdiv_rn(x[6], sc), __fdiv_rn(x[7], sc));
    }
    return a;
}

// ---- 4-bit blocks.  A head is owned by eight lanes, two chunks of eight elements each, which may lie in any of its four blocks.
// A code depends on where a value lies between the format's few borders and an exponent on which side of a power of two the block's largest
// is, so the fp32 rotation (off by less than kTurnError times the pair's magnitudes: 2^-23 from the angle, 2^-23 from the sine and cosine, three
// roundings of 2^-24; among the subnormals the roundings are half a step each of 2^-149, a product's and the sum's, hence kTurnStep) is only trusted where values that much smaller and larger give the same codes and exponents; otherwise the head is
// rotated again in fp64 (about one head in ten thousand).  16384 tokens: see the figures above.
constexpr float kTurnError = 5e-7f, kTurnStep = 0x1p-149f;

// E2M1 codes of two values, the first in the low half: nearest, ties to even, saturating at 6.
__device__ __forceinline__ uint32_t e2m1x2(float a, float b) {
    uint32_t d;
    asm("{\n\t.reg .b8 c;\n\tcvt.rn.satfinite.e2m1x2.f32 c, %2, %1;\n\tcvt.u32.u8 %0, c;\n\t}" : "=r"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ uint32_t e2m1x8(const float (&x)[8]) {
    return e2m1x2(x[0], x[1]) | e2m1x2(x[2], x[3]) << 8 | e2m1x2(x[4], x[5]) << 16 | e2m1x2(x[6], x[7]) << 24;
}
// Largest exponent field (255: an infinity or NaN is there) of eight values, each changed by `by` towards larger (by > 0) or smaller magnitudes.
__device__ __forceinline__ uint32_t exponent8(const float (&x)[8], float by) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
    if (top >= 0x7f800000u) return 255;
    return __float_as_uint(fmaxf(__uint_as_float(top) + by, 0.f)) >> 23;
}
// Exponents of the head's four blocks, a byte each, from those of this lane's two chunks.
__device__ __forceinline__ uint32_t block_exponents(uint32_t ea, int ca, uint32_t eb, int cb, uint32_t lanes) {
    uint32_t w = ca >> 2 == cb >> 2 ? max(ea, eb) << (8 * (ca >> 2)) : ea << (8 * (ca >> 2)) | eb << (8 * (cb >> 2));
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) w = __vmaxu4(w, __shfl_xor_sync(lanes, w, o));
    return w;
}
// Exponent byte of a block whose largest magnitude has exponent field f: two less (6 = 1.5 2^2 is the largest code), at least 0.
__device__ __forceinline__ uint32_t scale_byte(uint32_t f) { return f == 255 ? 255u : (f > 2 ? f - 2 : 0u); }
// 2^(127 - byte), exact; byte <= 252 (255: any)
__device__ __forceinline__ float scale_up(uint32_t byte) { return __uint_as_float((byte > 253 ? 1u : 254u - byte) << 23); }
// x as fp32 so that every border of a shorter format is on the right side: inexact values get an odd last bit.  Finite values beyond the range become the largest
// fp32 number: exponent byte 252, code 6.
__device__ __forceinline__ float to_odd(double x) {
    const float f = __double2float_rz(x);
    return (double)f == x || !(fabsf(f) < INFINITY) ? f : __uint_as_float(__float_as_uint(f) | 1u);
}

// kPairs: pair i is elements (2i, 2i + 1) of a head, else (i, i + rot / 2).  A lane owns two chunks of 8 elements of a head, ca and
// cb, and eight pairs: interleaved, four in each chunk; half layout, element j of ca with element j of cb.  Lanes whose chunks lie
// behind the rotated part copy them.
// The codes and exponent fields of a lane's two chunks from a rotation in fp64 (one lane of every eight that own a head asks for it).
template <bool kPairs>
__device__ __noinline__ void exact_codes(const RopeParams& p, int t, uint4 ra, uint4 rb, int ca, int cb, bool turn_a, bool turn_b, uint32_t lanes,
                                         uint32_t& f, uint32_t& codes_a, uint32_t& codes_b) {
    float ia[8], ib[8];
    unpack8(ra, ia);
    unpack8(rb, ib);
    double xa[8], xb[8];
#pragma unroll 1
    for (int j = 0; j < 8; ++j) {
        xa[j] = ia[j];
        xb[j] = ib[j];
    }
    auto turn = [&](int pair, double& a, double& b) {
        const int64_t pos = p.positions[(int64_t)p.axis[pair] * p.n + t];
        double s, c;
        sincospi((double)(int64_t)((uint64_t)pos * p.step[pair]) * 1.08420217248550443400745280086994171e-19, &s, &c);      // 2^-63: half turns
        const double u = a * c - b * s, w = b * c + a * s;
        a = u;
        b = w;
    };
#pragma unroll 1
    for (int j = 0; j < 4; ++j) {
        if (kPairs) {
            if (turn_a) turn(4 * ca + j, xa[2 * j], xa[2 * j + 1]);
            if (turn_b) turn(4 * cb + j, xb[2 * j], xb[2 * j + 1]);
        } else if (turn_a) {
            turn(8 * ca + j, xa[j], xb[j]);
            turn(8 * ca + j + 4, xa[j + 4], xb[j + 4]);
        }
    }
    float ya[8], yb[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        ya[j] = to_odd(xa[j]);
        yb[j] = to_odd(xb[j]);
    }
    f = block_exponents(exponent8(ya, 0.f), ca, exponent8(yb, 0.f), cb, lanes);
    const float ua = scale_up(scale_byte(f >> (8 * (ca >> 2)) & 255)), ub = scale_up(scale_byte(f >> (8 * (cb >> 2)) & 255));
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        ya[j] *= ua;
        yb[j] *= ub;
    }
    codes_a = e2m1x8(ya);
    codes_b = e2m1x8(yb);
}

enum Form : int { kRows16, kRows8, kRows4 };       // bf16, E4M3, 4-bit blocks
template <bool kPairs, Form kForm>
__global__ void __launch_bounds__(kRopeThreads, kForm == kRows4 ? 3 : 4)
rope_append_kernel(const __grid_constant__ RopeParams p) {
    constexpr bool kFp8 = kForm == kRows8, kMx = kForm == kRows4;
    const int lane = threadIdx.x & 31;
    const int sub = lane & 7, grp = lane >> 3;
    const int64_t w = ((int64_t)blockIdx.x * kRopeThreads + threadIdx.x) >> 5;
    const int t = (int)(w / p.parts), part = (int)(w - (int64_t)t * p.parts);
    if (t >= p.n) return;
    const int seq = p.seq[t];
    if (seq < 0) return;                                    // a padding row: nothing of it is touched
    // this lane's chunks
    int ca, cb;
    bool turn_a, turn_b;
    if (kPairs) {
        ca = sub;
        cb = sub + 8;
        turn_a = ca < p.n_chunks;
        turn_b = cb < p.n_chunks;
    } else {
        turn_a = turn_b = sub < p.n_chunks;
        ca = turn_a ? sub : 2 * sub;                        // behind the pairs: chunks 2 n .. 15, two per lane
        cb = turn_a ? sub + p.n_chunks : 2 * sub + 1;
    }
    const int s_begin = part * p.steps_per_warp, s_end = min(s_begin + p.steps_per_warp, p.q_steps + 2 * p.kv_steps);
    // head of this lane in step s: kind 0 = q, 1 = k, 2 = v
    auto locate = [&](int s, int& kind, int& h, int& heads) {
        kind = s < p.q_steps ? 0 : (s < p.q_steps + p.kv_steps ? 1 : 2);
        heads = kind == 0 ? p.Hq : p.Hkv;
        h = 4 * (kind == 0 ? s : s - p.q_steps - (kind == 2 ? p.kv_steps : 0)) + grp;
        return h < heads;
    };
    auto fetch = [&](int s, uint4& a, uint4& b) {
        int kind, h, heads;
        if (s < s_end && locate(s, kind, h, heads)) {
            const uint4* src = (kind == 0 ? p.q : (kind == 1 ? p.k_rows : p.v_rows)) + ((int64_t)t * heads + h) * (kHeadDim / 8);
            a = src[ca];
            b = src[cb];
        }
    };
    // the first rows, the slot and the positions are all on their way before any of them is used
    uint4 na = make_uint4(0, 0, 0, 0), nb = na;
    fetch(s_begin, na, nb);
    int64_t tok_off = -1, entry = -1, slot = 0;
    int32_t page = -1;
    if (s_end > p.q_steps) {
        slot = p.slot[t];
        entry = slot >> p.page_shift;
        if (seq < p.table_rows && slot >= 0 && entry < p.table_stride) page = p.page_table[seq * p.table_stride + entry];
        else entry = -1;
    }
    // cosines and sines: lane l computes pairs 2l and 2l + 1, then every lane fetches its eight
    float cs[8], sn[8];
    {
        float c2[2], s2[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int pair = 2 * lane + i;
            const int64_t pos = p.positions[(int64_t)p.axis[pair] * p.n + t];
            const uint64_t turns = (uint64_t)pos * p.step[pair];
            const float f = (float)(int32_t)(uint32_t)(turns >> 32) * 4.656612873077392578125e-10f;      // 2^-31: half turns in [-1, 1)
            sincospif(f, &s2[i], &c2[i]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int pair = kPairs ? (j < 4 ? 4 * ca + j : 4 * cb + j - 4) : 8 * sub + j;
            const int src = (pair >> 1) & 31;
            cs[j] = __shfl_sync(0xffffffffu, (j & 1) ? c2[1] : c2[0], src);
            sn[j] = __shfl_sync(0xffffffffu, (j & 1) ? s2[1] : s2[0], src);
        }
    }
    if (s_end > p.q_steps) {
        if (entry < 0) {
            if (lane == 0) report_status(p.status, CP_ERR_BOUNDS, t, slot);
        } else if (page < 0 || page >= p.num_pages) {
            if (lane == 0) report_status(p.status, CP_ERR_BOUNDS, seq * p.table_stride + entry, page);
        } else {
            tok_off = page * p.stride_page + (slot & ((1ll << p.page_shift) - 1)) * p.stride_tok;
        }
    }
    for (int s = s_begin; s < s_end; ++s) {
        const uint4 ra = na, rb = nb;
        fetch(s + 1, na, nb);                               // the next step's rows travel under this step's arithmetic
        int kind, h, heads;
        if (!locate(s, kind, h, heads) || (kind > 0 && tok_off < 0)) continue;
        uint4 oa = ra, ob = rb;
        float xa[8], xb[8];
        if (kind < 2 || kFp8 || kMx) {
            unpack8(ra, xa);
            unpack8(rb, xb);
        }
        if (kind < 2) {
            if (kPairs) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (turn_a) {
                        const float a = xa[2 * j], b = xa[2 * j + 1];
                        xa[2 * j] = a * cs[j] - b * sn[j];
                        xa[2 * j + 1] = b * cs[j] + a * sn[j];
                    }
                    if (turn_b) {
                        const float a = xb[2 * j], b = xb[2 * j + 1];
                        xb[2 * j] = a * cs[4 + j] - b * sn[4 + j];
                        xb[2 * j + 1] = b * cs[4 + j] + a * sn[4 + j];
                    }
                }
            } else if (turn_a) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float a = xa[j], b = xb[j];
                    xa[j] = a * cs[j] - b * sn[j];
                    xb[j] = b * cs[j] + a * sn[j];
                }
            }
            if (turn_a) oa = pack8(xa);       // chunks behind the rotated part keep their bits
            if (turn_b) ob = pack8(xb);
        }
        if (kind == 0) {
            uint4* dst = p.q_out + ((int64_t)t * heads + h) * (kHeadDim / 8);
            dst[ca] = oa;
            dst[cb] = ob;
        } else {
            uint8_t* dst = (kind == 1 ? p.cache_k : p.cache_v) + tok_off + (int64_t)h * p.stride_head;
            if (kMx) {
                const uint32_t lanes = 0xffu << (8 * grp);
                // how far xa, xb may be off: a lane's pairs have one element in each chunk (half layout) or both in one
                float err_a = 0.f, err_b = 0.f;
                if (kind == 1 && (turn_a || turn_b)) {
                    float in_a[8], in_b[8];
                    unpack8(ra, in_a);
                    unpack8(rb, in_b);
                    float ma = 0.f, mb = 0.f;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        ma = fmaxf(ma, fabsf(in_a[j]));
                        mb = fmaxf(mb, fabsf(in_b[j]));
                    }
                    err_a = turn_a ? fmaf(kTurnError, kPairs ? 2.f * ma : ma + mb, kTurnStep) : 0.f;
                    err_b = turn_b ? fmaf(kTurnError, kPairs ? 2.f * mb : ma + mb, kTurnStep) : 0.f;
                }
                uint32_t f = block_exponents(exponent8(xa, -err_a), ca, exponent8(xb, -err_b), cb, lanes);
                // a field of 255: an infinity or NaN of the input, or a rotation that left the fp32 range, which only the way through fp64 tells apart
                bool unsure = false;
                if (kind == 1) unsure = f != block_exponents(exponent8(xa, err_a), ca, exponent8(xb, err_b), cb, lanes) || __vcmpeq4(f, 0xffffffffu) != 0;
                uint32_t codes_a, codes_b;
                auto code8 = [&](const float (&x)[8], int chunk, float err, bool& differ) {
                    const float up = scale_up(scale_byte(f >> (8 * (chunk >> 2)) & 255));
                    float y[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) y[j] = x[j] * up;
                    const uint32_t c = e2m1x8(y);
                    if (kind == 1) {
                        float lo[8], hi[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            lo[j] = y[j] - err * up;
                            hi[j] = y[j] + err * up;
                        }
                        // A sign that is not decided counts unless both ends are zeros: what lies between them is one, of either sign.  (Counted for zeros too, keys with
                        // zero pairs went through fp64: 16384 tokens, 8 heads, half of the pairs zero 117 us where dense keys take 70.)
                        const uint32_t l = e2m1x8(lo), u = e2m1x8(hi), d = l ^ u;
                        differ = (d & 0x77777777u) != 0 || (d & 0x88888888u & (l << 1 | l << 2 | l << 3)) != 0;
                    }
                    return c;
                };
                bool da = false, db = false;
                codes_a = code8(xa, ca, err_a, da);
                codes_b = code8(xb, cb, err_b, db);
                if (kind == 1 && __any_sync(lanes, unsure || da || db)) {
                    exact_codes<kPairs>(p, t, ra, rb, ca, cb, turn_a, turn_b, lanes, f, codes_a, codes_b);
                }
                reinterpret_cast<uint32_t*>(dst)[ca] = codes_a;
                reinterpret_cast<uint32_t*>(dst)[cb] = codes_b;
                if (sub == 0) {
                    const uint32_t e = scale_byte(f & 255) | scale_byte(f >> 8 & 255) << 8 | scale_byte(f >> 16 & 255) << 16 | scale_byte(f >> 24) << 24;
                    *reinterpret_cast<uint32_t*>(dst + (int64_t)(p.Hkv - h) * p.stride_head + h * 4) = e;
                }
            } else if (kFp8) {
                const float sc = kind == 1 ? p.k_scale[h] : p.v_scale[h];
                const float inv = __frcp_rn(sc);
                reinterpret_cast<uint2*>(dst)[ca] = quantize8(xa, sc, inv);
                reinterpret_cast<uint2*>(dst)[cb] = quantize8(xb, sc, inv);
            } else {
                reinterpret_cast<uint4*>(dst)[ca] = oa;
                reinterpret_cast<uint4*>(dst)[cb] = ob;
            }
        }
    }
}

int rope_append(cp_ctx* ctx, const cp_rope* rope, const void* q, const void* k_rows, const void* v_rows, int64_t n, int32_t Hq,
                const int32_t* positions, const int32_t* token_seq, const int32_t* token_slot, const int32_t* page_table,
                int64_t table_rows, int64_t table_stride, void* q_out, const void* ck, const void* cv, const float* k_scale,
                const float* v_scale, int64_t num_pages, int32_t page_size, int32_t Hkv, int64_t stride_page, int64_t stride_tok,
                int64_t stride_head, Form form, void* stream, const char* who) {
    if (!rope || n < 0 || (n > 0 && (!positions || !token_seq)))
        return set_error(CP_ERR_INVALID_ARG, "%s: null pointer or negative token count", who);
    if (rope->n_axes < 1 || rope->n_axes > CP_ROPE_MAX_AXES || rope->rot_dims < 2 || rope->rot_dims > kHeadDim)
        return set_error(CP_ERR_INVALID_ARG, "%s: n_axes=%d rot_dims=%d", who, rope->n_axes, rope->rot_dims);
    if (rope->rot_dims % 16 != 0)
        return set_error(CP_ERR_UNSUPPORTED, "%s: rot_dims=%d; supported: multiples of 16", who, rope->rot_dims);
    for (int i = 0; i < rope->rot_dims / 2; ++i) {
        if (rope->axis[i] < 0 || rope->axis[i] >= rope->n_axes)
            return set_error(CP_ERR_INVALID_ARG, "%s: pair %d is on axis %d of %d", who, i, rope->axis[i], rope->n_axes);
        if (!isfinite(rope->freq[i])) return set_error(CP_ERR_INVALID_ARG, "%s: freq[%d] is not finite", who, i);
    }
    if (n == 0) return ctx ? CP_OK : set_error(CP_ERR_INVALID_ARG, "%s: ctx is NULL", who);      // empty tensors have no address
    if (!q != !q_out) return set_error(CP_ERR_INVALID_ARG, "%s: q and q_out come together or not at all", who);
    if (q && Hq < 1) return set_error(CP_ERR_INVALID_ARG, "%s: Hq=%d", who, Hq);
    if (!k_rows != !v_rows) return set_error(CP_ERR_INVALID_ARG, "%s: k_rows and v_rows come together or not at all", who);
    if (!q && !k_rows) return set_error(CP_ERR_INVALID_ARG, "%s: neither q nor k_rows", who);
    if (k_rows && (!token_slot || !page_table || table_rows < 1 || table_stride < 1))
        return set_error(CP_ERR_INVALID_ARG, "%s: k_rows need token_slot and a page table of at least one row and column", who);
    if (((uintptr_t)q | (uintptr_t)q_out | (uintptr_t)k_rows | (uintptr_t)v_rows) & 15)
        return set_error(CP_ERR_INVALID_ARG, "%s: q, q_out, k_rows and v_rows must be 16-byte aligned", who);
    if (n > 0x7fffffffll / 64 || (q && Hq > 4096) || (k_rows && Hkv > 4096))
        return set_error(CP_ERR_UNSUPPORTED, "%s: %lld tokens, %d / %d heads", who, (long long)n, Hq, Hkv);
    const size_t q_bytes = (size_t)n * (q ? Hq : 0) * kHeadDim * 2;
    if (q && q != q_out && ranges_overlap(q, q_bytes, q_out, q_bytes))
        return set_error(CP_ERR_INVALID_ARG, "%s: q_out overlaps q without being q", who);
    if (!ctx) return set_error(CP_ERR_INVALID_ARG, "%s: ctx is NULL", who);
    DeviceGuard guard(ctx->device);
    if (guard.rc()) return guard.rc();
    RopeParams p;
    const int pairs = rope->rot_dims / 2;
    for (int i = 0; i < 64; ++i) {
        // turns per step: modulo one turn (positions are whole numbers), as a fraction of 2^64
        long double turns = i < pairs ? (long double)rope->freq[i] * 0.159154943091895335768883763372514362L : 0.0L;
        if (turns < 0.0L || turns >= 1.0L) turns -= floorl(turns);
        const long double scaled = turns * 18446744073709551616.0L;
        p.step[i] = scaled >= 18446744073709551615.0L ? 0ull : (uint64_t)scaled;
        p.axis[i] = i < pairs ? (uint8_t)rope->axis[i] : 0;
    }
    p.n_chunks = rope->interleaved ? rope->rot_dims / 8 : rope->rot_dims / 16;
    p.n = (int32_t)n;
    p.Hq = q ? Hq : 0;
    p.Hkv = k_rows ? Hkv : 0;
    p.q_steps = (p.Hq + 3) / 4;
    p.kv_steps = (p.Hkv + 3) / 4;
    p.q = static_cast<const uint4*>(q);
    p.q_out = static_cast<uint4*>(q_out);
    p.k_rows = static_cast<const uint4*>(k_rows);
    p.v_rows = static_cast<const uint4*>(v_rows);
    p.positions = positions;
    p.seq = token_seq;
    p.slot = token_slot;
    p.page_table = page_table;
    p.table_rows = table_rows;
    p.table_stride = table_stride;
    p.cache_k = static_cast<uint8_t*>(const_cast<void*>(ck));
    p.cache_v = static_cast<uint8_t*>(const_cast<void*>(cv));
    p.k_scale = k_scale;
    p.v_scale = v_scale;
    p.num_pages = num_pages;
    p.stride_page = stride_page;
    p.stride_tok = stride_tok;
    p.stride_head = stride_head;
    p.page_shift = log2_exact(page_size);
    p.status = ctx->d_status;
    // few tokens: deal the steps of a token to several warps until the SMs have about 16 warps each
    const int steps = p.q_steps + 2 * p.kv_steps;
    const int64_t want = (int64_t)ctx->num_sms * 16;
    int per = (int)std::min<int64_t>(steps, std::max<int64_t>(1, n * steps / want));
    p.steps_per_warp = per;
    p.parts = (steps + per - 1) / per;
    const int64_t blocks = (n * p.parts + kRopeThreads / 32 - 1) / (kRopeThreads / 32);
    if (blocks > 0x7fffffffll) return set_error(CP_ERR_UNSUPPORTED, "%s: %lld blocks", who, (long long)blocks);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool pairs_of_two = rope->interleaved != 0;
    void (*kernel)(const RopeParams) = form == kRows4 ? (pairs_of_two ? rope_append_kernel<true, kRows4> : rope_append_kernel<false, kRows4>)
                                       : form == kRows8 ? (pairs_of_two ? rope_append_kernel<true, kRows8> : rope_append_kernel<false, kRows8>)
                                                        : (pairs_of_two ? rope_append_kernel<true, kRows16> : rope_append_kernel<false, kRows16>);
    kernel<<<(unsigned)blocks, kRopeThreads, 0, s>>>(p);
    return check_cuda(cudaGetLastError(), who);
}

}  // namespace

extern "C" int cp_rope_init(cp_rope* rope, int32_t n_axes, const int32_t* sections, double base, int32_t interleaved) {
    if (!rope || !sections || n_axes < 1 || n_axes > CP_ROPE_MAX_AXES || !(base > 0.0) || !isfinite(base))
        return set_error(CP_ERR_INVALID_ARG, "cp_rope_init: null pointer, n_axes=%d or base=%g", n_axes, base);
    int64_t pairs = 0;
    for (int32_t a = 0; a < n_axes; ++a) {
        if (sections[a] < 0) return set_error(CP_ERR_INVALID_ARG, "cp_rope_init: section %d is negative", a);
        pairs += sections[a];
    }
    if (pairs < 1 || pairs > 64)
        return set_error(CP_ERR_INVALID_ARG, "cp_rope_init: %lld rotated pairs, between 1 and 64", (long long)pairs);
    cp_rope r = {};
    r.n_axes = n_axes;
    r.rot_dims = (int32_t)(2 * pairs);
    r.interleaved = interleaved ? 1 : 0;
    int i = 0;
    for (int32_t a = 0; a < n_axes; ++a)
        for (int32_t k = 0; k < sections[a]; ++k, ++i) {
            r.axis[i] = a;
            r.freq[i] = pow(base, -(double)i / (double)pairs);
        }
    *rope = r;
    return CP_OK;
}

extern "C" int cp_rope_append(cp_ctx* ctx, const cp_rope* rope, const void* q, const void* k_rows, const void* v_rows, int64_t n,
                              int32_t Hq, const int32_t* positions, const int32_t* token_seq, const int32_t* token_slot,
                              const cp_kv_cache* cache, const int32_t* page_table, int64_t table_rows, int64_t table_stride,
                              void* q_out, void* stream) {
    const char* who = "cp_rope_append";
    if (int rc = validate_kv_cache(cache, who)) return rc;
    return rope_append(ctx, rope, q, k_rows, v_rows, n, Hq, positions, token_seq, token_slot, page_table, table_rows, table_stride,
                       q_out, cache->k, cache->v, nullptr, nullptr, cache->num_pages, cache->page_size, cache->Hkv,
                       cache->stride_page * 2, cache->stride_tok * 2, cache->stride_head * 2, kRows16, stream, who);
}

extern "C" int cp_rope_append_fp8(cp_ctx* ctx, const cp_rope* rope, const void* q, const void* k_rows, const void* v_rows, int64_t n,
                                  int32_t Hq, const int32_t* positions, const int32_t* token_seq, const int32_t* token_slot,
                                  const cp_kv_cache_fp8* cache, const int32_t* page_table, int64_t table_rows,
                                  int64_t table_stride, void* q_out, void* stream) {
    const char* who = "cp_rope_append_fp8";
    if (int rc = validate_kv_cache_fp8(cache, who)) return rc;
    return rope_append(ctx, rope, q, k_rows, v_rows, n, Hq, positions, token_seq, token_slot, page_table, table_rows, table_stride,
                       q_out, cache->k, cache->v, cache->k_scale, cache->v_scale, cache->num_pages, cache->page_size, cache->Hkv,
                       cache->stride_page, cache->stride_tok, cache->stride_head, kRows8, stream, who);
}

extern "C" int cp_rope_append_mx4(cp_ctx* ctx, const cp_rope* rope, const void* q, const void* k_rows, const void* v_rows, int64_t n,
                                  int32_t Hq, const int32_t* positions, const int32_t* token_seq, const int32_t* token_slot,
                                  const cp_kv_cache_mx4* cache, const int32_t* page_table, int64_t table_rows, int64_t table_stride,
                                  void* q_out, void* stream) {
    const char* who = "cp_rope_append_mx4";
    if (int rc = validate_kv_cache_mx4(cache, who)) return rc;
    return rope_append(ctx, rope, q, k_rows, v_rows, n, Hq, positions, token_seq, token_slot, page_table, table_rows, table_stride,
                       q_out, cache->k, cache->v, nullptr, nullptr, cache->num_pages, cache->page_size, cache->Hkv, cache->stride_page,
                       cache->stride_tok, 64, kRows4, stream, who);
}
