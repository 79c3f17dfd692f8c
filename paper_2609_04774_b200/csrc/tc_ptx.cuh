// What the tensor-core attention kernels share: PTX wrappers (mbarriers, TMA, tcgen05), the tiles' layouts and descriptors, bounded waits, and the
// exponentials of a score tile.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>

#include "internal.h"

using namespace cpattn;

namespace {

constexpr int kD = 128;
constexpr int kBlockM = 128;
constexpr int kBlockN = 128;
constexpr uint32_t kTileBytes = kBlockN * kD * 2;  // 32768
constexpr uint32_t kHalfBytes = kTileBytes / 2;    // one 64-dim half: 128 rows x 128 B
constexpr uint32_t kTryWaitHintNs = 200000;             // the thread may stay suspended this long per try
constexpr long long kWaitLimitCycles = 4000000000ll;   // about two seconds
constexpr int kPolyOf4 = 0;                            // pairs out of every four whose exp2 runs on the FMA pipe instead of MUFU:
                                                       // 0 since both softmax warpgroups run all the time (issue slots are the
                                                       // scarcer resource: 1 costs 3 %, 2 costs 12 %); 1 was best while they alternated

// ------------------------------------------------------------------------------------------
// PTX wrappers
// ------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mbar_expect_tx(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool mbar_try_wait(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(bar), "r"(parity), "r"(kTryWaitHintNs) : "memory");
    return ok != 0;
}

// Non-blocking test of a phase; the result comes back asynchronously, so a test issued before a block
// of MMAs costs nothing by the time it is looked at.
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
        ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2) : "memory");
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2,
                                            int c3) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
        ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3) : "memory");
}

// True in exactly one lane of the (converged) warp.
__device__ __forceinline__ bool elect_one() {
    uint32_t pred;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "elect.sync _|p, 0xffffffff;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(pred));
    return pred != 0;
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// D[tmem] (+)= A[smem desc] * B[smem desc]
__device__ __forceinline__ void mma_ss(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(acc) : "memory");
}
// D[tmem] (+)= A[tmem] * B[smem desc]
__device__ __forceinline__ void mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(acc) : "memory");
}

// the same two forms for one-byte operands (E4M3 x E4M3, fp32 accumulation; K = 32 per instruction)
__device__ __forceinline__ void mma_ss_f8(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(acc) : "memory");
}
__device__ __forceinline__ void mma_ts_f8(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(acc) : "memory");
}

#define CP_R8(a, o) "=f"(a[o + 0]), "=f"(a[o + 1]), "=f"(a[o + 2]), "=f"(a[o + 3]), "=f"(a[o + 4]), "=f"(a[o + 5]), "=f"(a[o + 6]), "=f"(a[o + 7])
#define CP_W8F(a, o) "f"(a[o + 0]), "f"(a[o + 1]), "f"(a[o + 2]), "f"(a[o + 3]), "f"(a[o + 4]), "f"(a[o + 5]), "f"(a[o + 6]), "f"(a[o + 7])
#define CP_W8R(a, o) "r"(a[o + 0]), "r"(a[o + 1]), "r"(a[o + 2]), "r"(a[o + 3]), "r"(a[o + 4]), "r"(a[o + 5]), "r"(a[o + 6]), "r"(a[o + 7])

// 32 consecutive fp32 columns of this thread's TMEM lane -> registers v[o .. o+31]
#define TMEM_LD32(taddr, v, o)                                                                            \
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "                                                \
                 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"                                  \
                 "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"                 \
                 : CP_R8(v, o), CP_R8(v, o + 8), CP_R8(v, o + 16), CP_R8(v, o + 24) : "r"(taddr) : "memory")
#define TMEM_ST32F(taddr, v, o)                                                                           \
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "                                         \
                 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"                                  \
                 "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};"                        \
                 ::CP_W8F(v, o), CP_W8F(v, o + 8), CP_W8F(v, o + 16), CP_W8F(v, o + 24), "r"(taddr) : "memory")
#define TMEM_ST16R(taddr, v, o)                                                                           \
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "                                         \
                 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"                                 \
                 ::CP_W8R(v, o), CP_W8R(v, o + 8), "r"(taddr) : "memory")
#define TMEM_ST8R(taddr, v, o)                                                                            \
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};"                    \
                 ::CP_W8R(v, o), "r"(taddr) : "memory")
#define TMEM_ST32R(taddr, v, o)                                                                           \
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "                                         \
                 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"                                  \
                 "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};"                        \
                 ::CP_W8R(v, o), CP_W8R(v, o + 8), CP_W8R(v, o + 16), CP_W8R(v, o + 24), "r"(taddr) : "memory")

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float lg2(float x) {
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// 2^x for a pair of arguments x <= 0 on the FMA pipe (no MUFU): round to nearest integer with the
// 1.5*2^23 trick, cubic minimax polynomial of 2^f on [-0.5, 0.5] (relative error 7.5e-5, far below
// the bf16 rounding of P), integer part added into the exponent field.
__device__ __forceinline__ float2 ex2_poly2(float2 x) {
    const float kMagic = 12582912.f;
    x.x = fmaxf(x.x, -126.f);
    x.y = fmaxf(x.y, -126.f);
    const float2 r = __fadd2_rn(x, make_float2(kMagic, kMagic));
    const float2 xi = __fadd2_rn(r, make_float2(-kMagic, -kMagic));
    const float2 f = __fadd2_rn(x, make_float2(-xi.x, -xi.y));
    float2 p = __ffma2_rn(f, make_float2(0.0551716648f, 0.0551716648f), make_float2(0.2426111251f, 0.2426111251f));
    p = __ffma2_rn(p, f, make_float2(0.6932609677f, 0.6932609677f));
    p = __ffma2_rn(p, f, make_float2(0.9999280572f, 0.9999280572f));
    float2 out;
    out.x = __int_as_float(__float_as_int(p.x) + (__float_as_int(r.x) << 23));
    out.y = __int_as_float(__float_as_int(p.y) + (__float_as_int(r.y) << 23));
    return out;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&b);
}

// Four weights -> four E4M3 bytes of one TMEM column, lowest key in the lowest byte (round to nearest even,
// saturating at 448).  cvt packs its first source into the upper byte of the pair.
__device__ __forceinline__ uint32_t pack_e4m3x4(float e0, float e1, float e2, float e3) {
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(e1), "f"(e0));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(e3), "f"(e2));
    return (uint32_t)lo | ((uint32_t)hi << 16);
}

// tcgen05 shared-memory matrix descriptor, 128-byte swizzle (layout type 2), descriptor version 1.
// K-major operand (Q, K): rows of 128 B, 8-row groups 1024 B apart (SBO); LBO unused.
// MN-major operand (V): 64 dims contiguous per key row (128 B), 8-key groups 1024 B apart (SBO),
// the next 64 dims one half-tile (16 KB) further (LBO).
__device__ __forceinline__ uint64_t make_desc(uint32_t saddr, uint32_t lbo_bytes, uint32_t sbo_bytes) {
    uint64_t d = (uint64_t)((saddr & 0x3FFFFu) >> 4);
    d |= (uint64_t)(lbo_bytes >> 4) << 16;
    d |= (uint64_t)(sbo_bytes >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}

// instruction descriptor: fp32 accumulate, bf16 A and B, M = 128, N = 128; bit 16 = B is MN-major
constexpr uint32_t kIdescS = (1u << 4) | (1u << 7) | (1u << 10) | ((kBlockN >> 3) << 17) | ((kBlockM >> 4) << 24);
constexpr uint32_t kIdescPV = kIdescS | (1u << 16);
// one-byte operands: A and B format fields 0 = E4M3; same shape; K = 32 per instruction
constexpr uint32_t kIdescS8 = (1u << 4) | ((kBlockN >> 3) << 17) | ((kBlockM >> 4) << 24);
constexpr uint32_t kIdescPV8 = kIdescS8 | (1u << 16);

// Bounded wait on an mbarrier phase.  The fast path is a single try; the slow path spins with a cycle
// limit.  When the limit runs out the first thread to notice records {code, barrier id, block,
// iteration} in the status word and raises the CTA's abort flag; from then on every wait of the CTA
// gives up after one failed try, so all roles run off the end of their loops without blocking (the
// results are garbage, the status word says so) and the kernel returns normally.
__device__ __forceinline__ void mbar_wait(uint32_t bar_base, uint32_t bar_id, uint32_t parity, volatile uint32_t* abort_flag,
                                          int32_t* status, int iter, long long limit_cycles = kWaitLimitCycles) {
    const uint32_t bar = bar_base + bar_id * 8;
    if (mbar_try_wait(bar, parity)) return;
    const long long t0 = clock64();
    while (true) {
        if (*abort_flag) return;
#pragma unroll 1
        for (int i = 0; i < 64; ++i)
            if (mbar_try_wait(bar, parity)) return;
        if (clock64() - t0 > limit_cycles) {
            *abort_flag = 1;
            if (atomicCAS(status, 0, CP_ERR_TIMEOUT) == 0) {
                status[1] = (int32_t)bar_id;
                status[2] = (int32_t)blockIdx.x;
                status[3] = iter;
            }
            return;
        }
    }
}

// Row max of 32 raw scores into four independent chains.
__device__ __forceinline__ void max32(const float (&s)[32], float& a0, float& a1, float& a2, float& a3) {
#pragma unroll
    for (int i = 0; i < 32; i += 8) {
        a0 = max3(a0, s[i], s[i + 1]);
        a1 = max3(a1, s[i + 2], s[i + 3]);
        a2 = max3(a2, s[i + 4], s[i + 5]);
        a3 = max3(a3, s[i + 6], s[i + 7]);
    }
}
__device__ __forceinline__ uint32_t bits_below(int x) { return x <= 0 ? 0u : (x >= 32 ? 0xffffffffu : (1u << x) - 1u); }
// p = 2^(s*c - m) for 32 keys -> 16 packed bf16 pairs; row sums into four accumulators.  With kPoly,
// kPolyOf4 of every four pairs take the FMA-pipe polynomial instead of MUFU; masked tiles do not (the
// polynomial clamps a masked score, -inf, to 2^-126, which is not the exact zero a hidden key needs).
template <bool kPoly>
__device__ __forceinline__ void exp32(const float (&s)[32], uint32_t (&pk)[16], float2 c2, float2 nm2, float2& sum0,
                                      float2& sum1, float2& sum2, float2& sum3) {
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
        const float2 x0 = __ffma2_rn(make_float2(s[2 * i + 0], s[2 * i + 1]), c2, nm2);
        const float2 x1 = __ffma2_rn(make_float2(s[2 * i + 2], s[2 * i + 3]), c2, nm2);
        const float2 x2 = __ffma2_rn(make_float2(s[2 * i + 4], s[2 * i + 5]), c2, nm2);
        const float2 x3 = __ffma2_rn(make_float2(s[2 * i + 6], s[2 * i + 7]), c2, nm2);
        const float2 p0 = make_float2(ex2(x0.x), ex2(x0.y));
        const float2 p1 = make_float2(ex2(x1.x), ex2(x1.y));
        const float2 p2 = (kPoly && kPolyOf4 >= 2) ? ex2_poly2(x2) : make_float2(ex2(x2.x), ex2(x2.y));
        const float2 p3 = (kPoly && kPolyOf4 >= 1) ? ex2_poly2(x3) : make_float2(ex2(x3.x), ex2(x3.y));
        sum0 = __fadd2_rn(sum0, p0);
        sum1 = __fadd2_rn(sum1, p1);
        sum2 = __fadd2_rn(sum2, p2);
        sum3 = __fadd2_rn(sum3, p3);
        pk[i + 0] = pack_bf16(p0.x, p0.y);
        pk[i + 1] = pack_bf16(p1.x, p1.y);
        pk[i + 2] = pack_bf16(p2.x, p2.y);
        pk[i + 3] = pack_bf16(p3.x, p3.y);
    }
}

// 4 x 4 transpose of 16-byte items inside every group of four lanes: on return v[s] holds what lane (quad * 4 + s)
// had in v[t], t = this lane's position in its quad.  Two exchange stages (lane ^ 1, lane ^ 2), 16 shuffles.
__device__ __forceinline__ uint4 shfl_xor16(uint4 a, int mask) {
    a.x = __shfl_xor_sync(0xffffffffu, a.x, mask);
    a.y = __shfl_xor_sync(0xffffffffu, a.y, mask);
    a.z = __shfl_xor_sync(0xffffffffu, a.z, mask);
    a.w = __shfl_xor_sync(0xffffffffu, a.w, mask);
    return a;
}
__device__ __forceinline__ void quad_transpose(uint4 (&v)[4], int t) {
    {
        const bool hi = t & 1;
        const uint4 r0 = shfl_xor16(hi ? v[0] : v[1], 1), r1 = shfl_xor16(hi ? v[2] : v[3], 1);
        if (hi) { v[0] = r0; v[2] = r1; } else { v[1] = r0; v[3] = r1; }
    }
    {
        const bool hi = t & 2;
        const uint4 r0 = shfl_xor16(hi ? v[0] : v[2], 2), r1 = shfl_xor16(hi ? v[1] : v[3], 2);
        if (hi) { v[0] = r0; v[1] = r1; } else { v[2] = r0; v[3] = r1; }
    }
}

}  // namespace
