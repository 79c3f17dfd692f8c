// cp_decode_attn, cp_decode_attn_fp8: attention of one or a few new tokens per request over a paged cache; see decode_kernel.cuh.
#include "decode_kernel.cuh"

namespace {

int decode_attn(cp_ctx* ctx, const void* q, const CacheView& cache, bool fp8, const int32_t* page_table, int64_t table_stride, const int32_t* kv_len, int32_t B,
                int32_t n_q, int32_t Hq, int64_t window, int64_t sinks, float scale, void* out, float* lse, void* workspace,
                size_t workspace_bytes, void* stream, const char* who) {
    DecodeParams p;
    if (int rc = decode_params(ctx, q, cache, page_table, table_stride, kv_len, B, n_q, Hq, window, sinks, scale, out, lse, workspace, workspace_bytes, p, who))
        return rc;
    if (B == 0) return CP_OK;
    DeviceGuard guard(ctx->device);
    if (guard.rc()) return guard.rc();
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (fp8 && cache.Hkv % 2 == 0) return n_q > 1 ? launch_rows<2, kE4m3, kChain>(ctx, p, s, who) : launch_rows<2, kE4m3, kToken>(ctx, p, s, who);
    if (fp8) return n_q > 1 ? launch_rows<1, kE4m3, kChain>(ctx, p, s, who) : launch_rows<1, kE4m3, kToken>(ctx, p, s, who);
    return n_q > 1 ? launch_rows<1, kBf16, kChain>(ctx, p, s, who) : launch_rows<1, kBf16, kToken>(ctx, p, s, who);
}

}  // namespace

extern "C" size_t cp_workspace_bytes_decode(int32_t B, int32_t n_q, int32_t Hq, int32_t Hkv) {
    if (B < 0 || n_q < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0) return 0;
    const int64_t rows = (int64_t)n_q * (Hq / Hkv);
    if (B > kMaxDecodeBatch || n_q > kMaxDecodeTokens || rows > kMaxDecodeRows) return 0;
    return decode_workspace((int)rows, Hkv % 4 == 0);      // of every kind of cache
}

extern "C" int cp_decode_attn(cp_ctx* ctx, const void* q, const cp_kv_cache* cache, const int32_t* page_table, int64_t table_stride,
                              const int32_t* kv_len, int32_t B, int32_t n_q, int32_t Hq, int64_t window, int64_t sinks, float scale,
                              void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    const char* who = "cp_decode_attn";
    if (int rc = validate_kv_cache(cache, who)) return rc;
    return decode_attn(ctx, q, view_of(cache), false, page_table, table_stride, kv_len, B, n_q, Hq, window, sinks, scale, out, lse, workspace,
                       workspace_bytes, stream, who);
}

extern "C" int cp_decode_attn_fp8(cp_ctx* ctx, const void* q, const cp_kv_cache_fp8* cache, const int32_t* page_table,
                                  int64_t table_stride, const int32_t* kv_len, int32_t B, int32_t n_q, int32_t Hq, int64_t window,
                                  int64_t sinks, float scale, void* out, float* lse, void* workspace, size_t workspace_bytes,
                                  void* stream) {
    const char* who = "cp_decode_attn_fp8";
    if (int rc = validate_kv_cache_fp8(cache, who)) return rc;
    return decode_attn(ctx, q, view_of(cache), true, page_table, table_stride, kv_len, B, n_q, Hq, window, sinks, scale, out, lse, workspace,
                       workspace_bytes, stream, who);
}
