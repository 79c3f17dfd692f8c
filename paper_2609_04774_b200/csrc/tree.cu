// Trees of drafted tokens: cp_tree_plan (masks, positions and slots from the parents) and cp_tree_attn[_fp8|_mx4].
#include "decode_kernel.cuh"

namespace {

// ---------------------------------------------------------------------------------------------- plan
constexpr int kMaxTree = 64;

// One CTA per sequence, one thread per drafted token.  A token's ancestors by pointer doubling: after round i a mask holds the nearest 2^i
// of them and the pointer is at the next one, so six rounds do for 64 tokens.  The call is one launch of a few microseconds.
__global__ void __launch_bounds__(kMaxTree)
tree_plan_kernel(const int32_t* parent, const int32_t* tree_len, const int32_t* kv_len, int32_t B, int32_t n_q, int32_t n_axes,
                 unsigned long long* mask, int32_t* positions, int32_t* token_seq, int32_t* token_slot, int32_t* status) {
    __shared__ unsigned long long seen[kMaxTree];
    __shared__ int up[kMaxTree];
    const int b = blockIdx.x, t = threadIdx.x;
    const int len = max(kv_len[b], 0), asked = tree_len ? tree_len[b] : n_q;
    const int m = min(max(asked, 0), min(n_q, len));
    if (t == 0 && tree_len && m != asked) report_status(status, CP_ERR_BOUNDS, b, asked);
    int to = -1;
    if (t < m) {
        to = parent[(int64_t)b * n_q + t];
        if (to < -1 || to >= t) {
            report_status(status, CP_ERR_BOUNDS, (int64_t)b * n_q + t, to);
            to = -1;
        }
    }
    unsigned long long mine = t < m ? 1ull << t : 0;
    seen[t] = mine;
    up[t] = to;
#pragma unroll
    for (int i = 0; i < 6; ++i) {
        __syncthreads();
        unsigned long long theirs = 0;
        int next = -1;
        if (to >= 0) {
            theirs = seen[to];
            next = up[to];
        }
        __syncthreads();
        mine |= theirs;
        to = next;
        seen[t] = mine;
        up[t] = to;
    }
    if (t >= n_q) return;
    const int64_t at = (int64_t)b * n_q + t;
    const int base = len - m;
    mask[at] = mine;
    for (int a = 0; a < n_axes; ++a) positions[(int64_t)a * B * n_q + at] = t < m ? base + __popcll(mine) - 1 : 0;
    token_seq[at] = t < m ? b : -1;
    token_slot[at] = t < m ? base + t : 0;
}

// Rows per KV head up to which the narrow form is taken (us narrow / wide; B requests x keys, 32 / 8 heads).
//          16 rows: 37 x 4096  37 x 700   1 x 4096     24 rows: 37 x 4096  37 x 700   1 x 4096     32 rows: 37 x 4096  37 x 700   1 x 4096
//   bf16            98 / 103    27 / 31    13 / 17             108 / 104    39 / 31    17 / 18             109 / 106    39 / 31    18 / 18
//   E4M3            66 / 101    22 / 34    18 / 19              97 / 101    34 / 34    25 / 19              99 / 101    35 / 35    26 / 20
//   4-bit          103 / 105    29 / 35    15 / 19             165 / 105    45 / 35    20 / 19             174 / 105    46 / 36    20 / 20
// Up to 16 rows the narrow form is faster for every kind.  Its 32-row form costs more than the loads of a tile for 4-bit rows and somewhat for bf16; with E4M3 it is 2 to 4 % ahead on long
// batches, level on short ones and behind on a single request.  Behind 32 rows it reads the keys again (48 rows, 37 x 4096: 208 / 107, 183 / 102, 261 / 108).
constexpr int kNarrowRows[3] = {16, 32, 16};
constexpr int kLeastNarrowRows = 16;               // a workspace serves every kind

template <typename Cache>
int tree_attn(cp_ctx* ctx, const void* q, const Cache* cache, const int32_t* page_table, int64_t table_stride, const int32_t* kv_len,
              const int32_t* tree_len, const uint64_t* mask, int32_t B, int32_t n_q, int32_t Hq, int64_t window, int64_t sinks, float scale,
              void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream, Kind kind, const char* who) {
    if (B > 0 && !mask) return set_error(CP_ERR_INVALID_ARG, "%s: null pointer", who);
    if (workspace && workspace_bytes < cp_workspace_bytes_tree(B, n_q, Hq, cache->Hkv))
        return set_error(CP_ERR_WORKSPACE, "%s: workspace of %zu bytes; need %zu", who, workspace_bytes, cp_workspace_bytes_tree(B, n_q, Hq, cache->Hkv));
    if ((uintptr_t)mask & 7) return set_error(CP_ERR_INVALID_ARG, "%s: mask must be 8-byte aligned", who);
    DecodeParams p;
    if (int rc = decode_params(ctx, q, view_of(cache), page_table, table_stride, kv_len, B, n_q, Hq, window, sinks, scale, out, lse, workspace,
                               workspace_bytes, p, who)) return rc;
    if (B == 0) return CP_OK;
    p.tree_len = tree_len;
    p.tree_mask = reinterpret_cast<const unsigned long long*>(mask);
    DeviceGuard guard(ctx->device);
    if (guard.rc()) return guard.rc();
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const CacheView view = view_of(cache);
    if (p.rows > kNarrowRows[kind]) return launch_tree_wide(ctx, kind, &p, &view, workspace, stream, who);
    if (kind == kBf16) return launch_rows<1, kBf16, kTree>(ctx, p, s, who);
    if (kind == kE4m3) return p.Hkv % 2 == 0 ? launch_rows<2, kE4m3, kTree>(ctx, p, s, who) : launch_rows<1, kE4m3, kTree>(ctx, p, s, who);
    return launch_mx4<kTree>(ctx, p, s, who);
}

}  // namespace

extern "C" int cp_tree_plan(cp_ctx* ctx, const int32_t* parent, const int32_t* tree_len, const int32_t* kv_len, int32_t B, int32_t n_q,
                            int32_t n_axes, uint64_t* mask, int32_t* positions, int32_t* token_seq, int32_t* token_slot, void* stream) {
    const char* who = "cp_tree_plan";
    if (B < 0 || n_q < 1 || n_axes < 1 || n_axes > CP_ROPE_MAX_AXES)
        return set_error(CP_ERR_INVALID_ARG, "%s: B=%d n_q=%d n_axes=%d", who, B, n_q, n_axes);
    if (B > 0 && (!parent || !kv_len || !mask || !positions || !token_seq || !token_slot)) return set_error(CP_ERR_INVALID_ARG, "%s: null pointer", who);
    if ((uintptr_t)mask & 7) return set_error(CP_ERR_INVALID_ARG, "%s: mask must be 8-byte aligned", who);
    if (n_q > kMaxTree || B > kMaxDecodeBatch) return set_error(CP_ERR_UNSUPPORTED, "%s: n_q=%d (at most 64), B=%d (at most 65536)", who, n_q, B);
    if (!ctx) return set_error(CP_ERR_INVALID_ARG, "%s: ctx is NULL", who);
    if (B == 0) return CP_OK;
    DeviceGuard guard(ctx->device);
    if (guard.rc()) return guard.rc();
    tree_plan_kernel<<<(unsigned)B, kMaxTree, 0, static_cast<cudaStream_t>(stream)>>>(
        parent, tree_len, kv_len, B, n_q, n_axes, reinterpret_cast<unsigned long long*>(mask), positions, token_seq, token_slot, ctx->d_status);
    return check_cuda(cudaGetLastError(), who);
}

extern "C" size_t cp_workspace_bytes_tree(int32_t B, int32_t n_q, int32_t Hq, int32_t Hkv) {
    const size_t narrow = cp_workspace_bytes_decode(B, n_q, Hq, Hkv);
    return narrow == 0 || (int64_t)n_q * (Hq / Hkv) <= kLeastNarrowRows ? narrow : std::max(narrow, tree_wide_workspace());
}

extern "C" int cp_tree_attn(cp_ctx* ctx, const void* q, const cp_kv_cache* cache, const int32_t* page_table, int64_t table_stride,
                            const int32_t* kv_len, const int32_t* tree_len, const uint64_t* mask, int32_t B, int32_t n_q, int32_t Hq,
                            int64_t window, int64_t sinks, float scale, void* out, float* lse, void* workspace, size_t workspace_bytes,
                            void* stream) {
    const char* who = "cp_tree_attn";
    if (int rc = validate_kv_cache(cache, who)) return rc;
    return tree_attn(ctx, q, cache, page_table, table_stride, kv_len, tree_len, mask, B, n_q, Hq, window, sinks, scale, out, lse, workspace,
                     workspace_bytes, stream, kBf16, who);
}

extern "C" int cp_tree_attn_fp8(cp_ctx* ctx, const void* q, const cp_kv_cache_fp8* cache, const int32_t* page_table, int64_t table_stride,
                                const int32_t* kv_len, const int32_t* tree_len, const uint64_t* mask, int32_t B, int32_t n_q, int32_t Hq,
                                int64_t window, int64_t sinks, float scale, void* out, float* lse, void* workspace, size_t workspace_bytes,
                                void* stream) {
    const char* who = "cp_tree_attn_fp8";
    if (int rc = validate_kv_cache_fp8(cache, who)) return rc;
    return tree_attn(ctx, q, cache, page_table, table_stride, kv_len, tree_len, mask, B, n_q, Hq, window, sinks, scale, out, lse, workspace,
                     workspace_bytes, stream, kE4m3, who);
}

extern "C" int cp_tree_attn_mx4(cp_ctx* ctx, const void* q, const cp_kv_cache_mx4* cache, const int32_t* page_table, int64_t table_stride,
                                const int32_t* kv_len, const int32_t* tree_len, const uint64_t* mask, int32_t B, int32_t n_q, int32_t Hq,
                                int64_t window, int64_t sinks, float scale, void* out, float* lse, void* workspace, size_t workspace_bytes,
                                void* stream) {
    const char* who = "cp_tree_attn_mx4";
    if (int rc = validate_kv_cache_mx4(cache, who)) return rc;
    return tree_attn(ctx, q, cache, page_table, table_stride, kv_len, tree_len, mask, B, n_q, Hq, window, sinks, scale, out, lse, workspace,
                     workspace_bytes, stream, kMx4, who);
}
