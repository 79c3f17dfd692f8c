// Launch of the wide form of tree attention (tree_wide.cuh).
#include "tree_wide.cuh"

namespace {

int encode(cp_ctx* ctx, CUtensorMap* map, CUtensorMapDataType type, int rank, const void* base, const cuuint64_t* dims, const cuuint64_t* strides,
           const cuuint32_t* box, CUtensorMapSwizzle swizzle, CUtensorMapL2promotion promotion, const char* who) {
    const cuuint32_t es[4] = {1, 1, 1, 1};
    const CUresult r = ctx->encode_tiled(map, type, rank, const_cast<void*>(base), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                                         promotion, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? CP_OK : set_error(CP_ERR_CUDA, "%s: cuTensorMapEncodeTiled failed with %d", who, (int)r);
}

// One box is a page of one head: 64 bf16 dims, or the whole row of codes; 4-bit: a second box for 16 bytes of exponents a token.
// L2 fetches no more than a row (with 256 bytes for all kinds, E4M3 read 704 MB where 480 are needed and 37 requests of 8192 keys with 128 rows took 201 us, not 192).
template <Kind kKind>
int encode_cache(cp_ctx* ctx, const CacheView& v, bool second, CUtensorMap* map, CUtensorMap* exps, const char* who) {
    const uint8_t* base = static_cast<const uint8_t*>(second ? v.v : v.k);
    const cuuint64_t dims[4] = {kKind == kMx4 ? 64u : 128u, (cuuint64_t)v.Hkv, (cuuint64_t)v.page_size, (cuuint64_t)v.num_pages};
    const cuuint64_t strides[3] = {(cuuint64_t)v.stride_head, (cuuint64_t)v.stride_tok, (cuuint64_t)v.stride_page};
    const cuuint32_t box[4] = {kKind == kE4m3 ? 128u : 64u, 1, (cuuint32_t)v.page_size, 1};
    if (int rc = encode(ctx, map, kKind == kBf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, base, dims, strides, box,
                        kKind == kMx4 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B,
                        kKind == kBf16 ? CU_TENSOR_MAP_L2_PROMOTION_L2_256B
                                       : (kKind == kE4m3 ? CU_TENSOR_MAP_L2_PROMOTION_L2_128B : CU_TENSOR_MAP_L2_PROMOTION_L2_64B), who)) return rc;
    if (kKind != kMx4) return CP_OK;
    const cuuint64_t edims[3] = {(cuuint64_t)v.Hkv * 4, (cuuint64_t)v.page_size, (cuuint64_t)v.num_pages};
    const cuuint64_t estrides[2] = {(cuuint64_t)v.stride_tok, (cuuint64_t)v.stride_page};
    const cuuint32_t ebox[3] = {16, (cuuint32_t)v.page_size, 1};
    return encode(ctx, exps, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, base + (int64_t)v.Hkv * 64, edims, estrides, ebox, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_NONE, who);
}

template <Kind kKind, int kTiles>
int launch(cp_ctx* ctx, const WideParams& w, const CacheView& view, cudaStream_t s, const char* who) {
    using W = Wide<kKind, kTiles>;
    CUtensorMap k, v, ke = {}, ve = {};
    if (int rc = encode_cache<kKind>(ctx, view, false, &k, &ke, who)) return rc;
    if (int rc = encode_cache<kKind>(ctx, view, true, &v, &ve, who)) return rc;
    if (!ctx->tree_attr_set[kKind][kTiles - 1]) {
        if (int rc = check_cuda(cudaFuncSetAttribute(tree_wide_kernel<kKind, kTiles>, cudaFuncAttributeMaxDynamicSharedMemorySize, W::kSmem),
                                "cudaFuncSetAttribute(tree)")) return rc;
        ctx->tree_attr_set[kKind][kTiles - 1] = true;
    }
    tree_wide_kernel<kKind, kTiles><<<dim3((unsigned)w.classes, (unsigned)w.heads, (unsigned)w.runs), W::kThreads, W::kSmem, s>>>(k, v, ke, ve, w);
    if (int rc = check_cuda(cudaGetLastError(), who)) return rc;
    const unsigned y = (unsigned)((w.class_rows + kWideJoinRows - 1) / kWideJoinRows);
    return launch_behind(tree_join_kernel<kKind>, dim3((unsigned)(w.runs * w.classes * w.heads), y), 32 * kWideJoinRows, s, who, w);
}

}  // namespace

namespace cpattn {

size_t tree_wide_workspace() {
    const size_t n = 2 * (size_t)kMaxGrid * kWideRows;
    return (n * (kD + 2) * sizeof(float) + kMaxGrid * 16 + 255) / 256 * 256;
}

int launch_tree_wide(cp_ctx* ctx, int kind, const void* decode_params, const void* cache_view, void* workspace, void* stream, const char* who) {
    WideParams w;
    w.d = *static_cast<const DecodeParams*>(decode_params);
    const CacheView& view = *static_cast<const CacheView*>(cache_view);
    const int grid = std::min(ctx->num_sms, kMaxGrid);
    w.classes = (w.d.rows + kWideRows - 1) / kWideRows;
    w.class_rows = (w.d.rows + w.classes - 1) / w.classes;
    w.heads = kind == kBf16 || w.classes > 1 ? 1 : (w.d.Hkv % 4 == 0 ? 4 : (w.d.Hkv % 2 == 0 ? 2 : 1));
    w.runs = grid / (w.classes * w.heads);
    const size_t n = 2 * (size_t)kMaxGrid * kWideRows;
    w.d.part_o = static_cast<float*>(workspace);
    w.d.part_ml = w.d.part_o + n * kD;
    w.d.meta = reinterpret_cast<int32_t*>(w.d.part_ml + n * 2);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool two = w.class_rows > kBlockM;
    if (kind == kE4m3) return two ? launch<kE4m3, 2>(ctx, w, view, s, who) : launch<kE4m3, 1>(ctx, w, view, s, who);
    if (kind == kMx4) return two ? launch<kMx4, 2>(ctx, w, view, s, who) : launch<kMx4, 1>(ctx, w, view, s, who);
    return two ? launch<kBf16, 2>(ctx, w, view, s, who) : launch<kBf16, 1>(ctx, w, view, s, who);
}

}  // namespace cpattn
