// 4-bit K/V caches (blocks of 32 E2M1 codes with an exponent byte): cp_decode_attn_mx4 (see decode_kernel.cuh) and cp_kv_gather_mx4.
#include "decode_kernel.cuh"

namespace {

// Chains of drafts with more than 16 rows a KV head stay in this form, though each 32 rows read and widen the keys again: the many-row kernel (tree_wide.cuh) has no mode for
// chains.  37 requests of 4096 keys: 24 rows 158 us where a tree takes 105, 48 rows 253 / 109; of 700 keys 42 / 35, 78 / 36; one of 4096 18.8 / 19.0, 22.5 / 20.1.
int decode_attn_mx4(cp_ctx* ctx, const DecodeParams& p, cudaStream_t s, const char* who) {
    return p.n_q > 1 ? launch_mx4<kChain>(ctx, p, s, who) : launch_mx4<kToken>(ctx, p, s, who);
}

// ---------------------------------------------------------------------------------------------- gather
// HBM-bound: 68 bytes of a head's row become 256.  A thread turns eight codes into a 16-byte vector, so a warp's stores are 512
// contiguous bytes; four vectors are in flight per thread.
constexpr int kGatherThreads = 256;
constexpr int kGatherItems = 4;

struct GatherParams {
    const uint8_t* cache[2];
    uint4* rows[2];
    const int32_t* table;
    int64_t t_begin, items;            // items: vectors of one of K and V, n * Hkv * 16
    int64_t num_pages, stride_page, stride_tok;
    int32_t page_shift, Hkv, first, count;      // tensors [first, first + count) of K, V
    int32_t* status;
};

__device__ __forceinline__ uint4 widen_bf16(uint32_t codes, uint32_t e) {
    // the scale in fp32 (2^-127 is a subnormal, e = 255 a NaN): the products are exact, and so is their rounding up to e = 252
    const float scale = __uint_as_float(e == 0 ? 0x00400000u : (e == 255 ? 0x7fc00000u : e << 23));
    uint32_t h[4];
    widen8(codes, h[0], h[1], h[2], h[3]);
    uint32_t out[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
        out[i] = pack_weights<false>(x.x * scale, x.y * scale);
    }
    return make_uint4(out[0], out[1], out[2], out[3]);
}

__global__ void __launch_bounds__(kGatherThreads)
gather_mx4_kernel(const __grid_constant__ GatherParams p) {
    const int which = p.first + blockIdx.y;
    const uint8_t* cache = p.cache[which];
    uint4* rows = p.rows[which];
    const int64_t step = (int64_t)gridDim.x * kGatherThreads * kGatherItems;
    const uint32_t per_token = p.Hkv * 16;
    for (int64_t base = (int64_t)blockIdx.x * kGatherThreads * kGatherItems; base < p.items; base += step) {
        uint32_t codes[kGatherItems], e[kGatherItems];
        bool ok[kGatherItems];
        const int64_t token0 = base / per_token;           // one division in 64 bits, then offsets
        const uint32_t rest = (uint32_t)(base - token0 * per_token);
#pragma unroll
        for (int i = 0; i < kGatherItems; ++i) {
            const int64_t at = base + i * kGatherThreads + threadIdx.x;
            ok[i] = at < p.items;
            if (!ok[i]) continue;
            const uint32_t off = rest + i * kGatherThreads + threadIdx.x, tokens = off / per_token;
            const int64_t t = p.t_begin + token0 + tokens;
            const uint32_t vec = off - tokens * per_token;                // head * 16 + eighth of the codes' bytes
            const int64_t entry = t >> p.page_shift;
            const int32_t page = __ldg(p.table + entry);
            ok[i] = page >= 0 && page < p.num_pages;
            if (!ok[i]) {
                report_status(p.status, CP_ERR_BOUNDS, entry, page);
                continue;
            }
            const uint8_t* row = cache + page * p.stride_page + (t & ((1ll << p.page_shift) - 1)) * p.stride_tok;
            codes[i] = __ldg(reinterpret_cast<const uint32_t*>(row) + vec);
            e[i] = __ldg(row + p.Hkv * 64 + (vec >> 2));
        }
#pragma unroll
        for (int i = 0; i < kGatherItems; ++i)
            if (ok[i]) rows[base + i * kGatherThreads + threadIdx.x] = widen_bf16(codes[i], e[i]);
    }
}

}  // namespace

namespace cpattn {

int validate_kv_cache_mx4(const cp_kv_cache_mx4* c, const char* who) {
    if (!c || !c->k || !c->v) return set_error(CP_ERR_INVALID_ARG, "%s: cache or its K/V pointers are NULL", who);
    if (c->D != 128) return set_error(CP_ERR_UNSUPPORTED, "%s: D=%d; only 128 is supported", who, c->D);
    if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64 && c->page_size != 128)
        return set_error(CP_ERR_UNSUPPORTED, "%s: page_size=%d; supported: pages of 16, 32, 64 or 128 tokens", who, c->page_size);
    if (c->num_pages < 1 || c->Hkv < 1) return set_error(CP_ERR_INVALID_ARG, "%s: num_pages=%lld Hkv=%d", who, (long long)c->num_pages, c->Hkv);
    if (c->Hkv > 4096) return set_error(CP_ERR_UNSUPPORTED, "%s: %d KV heads", who, c->Hkv);
    if (c->stride_tok < (int64_t)c->Hkv * 68 || c->stride_page < 1)
        return set_error(CP_ERR_INVALID_ARG, "%s: stride_tok=%lld (a token's row has %d bytes), stride_page=%lld", who, (long long)c->stride_tok,
                         c->Hkv * 68, (long long)c->stride_page);
    if (((c->stride_page | c->stride_tok) & 15) || (((uintptr_t)c->k | (uintptr_t)c->v) & 15))
        return set_error(CP_ERR_UNSUPPORTED, "%s: k, v and the strides must be multiples of 16 bytes", who);
    return CP_OK;
}

}  // namespace cpattn

extern "C" int cp_decode_attn_mx4(cp_ctx* ctx, const void* q, const cp_kv_cache_mx4* cache, const int32_t* page_table, int64_t table_stride,
                                  const int32_t* kv_len, int32_t B, int32_t n_q, int32_t Hq, int64_t window, int64_t sinks, float scale,
                                  void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    const char* who = "cp_decode_attn_mx4";
    if (int rc = validate_kv_cache_mx4(cache, who)) return rc;
    DecodeParams p;
    if (int rc = decode_params(ctx, q, view_of(cache), page_table, table_stride, kv_len, B, n_q, Hq, window, sinks, scale, out, lse, workspace,
                               workspace_bytes, p, who)) return rc;
    if (B == 0) return CP_OK;
    DeviceGuard guard(ctx->device);
    if (guard.rc()) return guard.rc();
    return decode_attn_mx4(ctx, p, static_cast<cudaStream_t>(stream), who);
}

extern "C" int cp_kv_gather_mx4(cp_ctx* ctx, const cp_kv_cache_mx4* cache, const int32_t* page_table, int64_t t_begin, int64_t n,
                                void* k_rows, void* v_rows, void* stream) {
    const char* who = "cp_kv_gather_mx4";
    if (int rc = validate_kv_cache_mx4(cache, who)) return rc;
    if (!page_table || t_begin < 0 || n < 0) return set_error(CP_ERR_INVALID_ARG, "%s: null pointer or negative range", who);
    if (t_begin > (1ll << 40) || n > (1ll << 40)) return set_error(CP_ERR_UNSUPPORTED, "%s: %lld tokens from %lld", who, (long long)n, (long long)t_begin);
    if (((uintptr_t)k_rows | (uintptr_t)v_rows) & 15) return set_error(CP_ERR_INVALID_ARG, "%s: k_rows and v_rows must be 16-byte aligned", who);
    if (!ctx) return set_error(CP_ERR_INVALID_ARG, "%s: ctx is NULL", who);
    if (n == 0 || (!k_rows && !v_rows)) return CP_OK;
    DeviceGuard guard(ctx->device);
    if (guard.rc()) return guard.rc();
    GatherParams p;
    p.cache[0] = static_cast<const uint8_t*>(cache->k);
    p.cache[1] = static_cast<const uint8_t*>(cache->v);
    p.rows[0] = static_cast<uint4*>(k_rows);
    p.rows[1] = static_cast<uint4*>(v_rows);
    p.table = page_table;
    p.t_begin = t_begin;
    p.items = n * cache->Hkv * 16;
    p.num_pages = cache->num_pages;
    p.stride_page = cache->stride_page;
    p.stride_tok = cache->stride_tok;
    p.page_shift = log2_exact(cache->page_size);
    p.Hkv = cache->Hkv;
    p.first = k_rows ? 0 : 1;
    p.count = (k_rows ? 1 : 0) + (v_rows ? 1 : 0);
    p.status = ctx->d_status;
    const int64_t per_block = kGatherThreads * kGatherItems;
    const unsigned blocks = (unsigned)std::min<int64_t>((p.items + per_block - 1) / per_block, (int64_t)ctx->num_sms * 64);
    gather_mx4_kernel<<<dim3(blocks, (unsigned)p.count), kGatherThreads, 0, static_cast<cudaStream_t>(stream)>>>(p);
    return check_cuda(cudaGetLastError(), who);
}
