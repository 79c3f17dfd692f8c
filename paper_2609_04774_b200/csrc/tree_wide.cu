// Launch of the wide form of tree attention (tree_wide.cuh).
#include "tree_wide.cuh"

namespace {

int encode_kv(cp_ctx* ctx, const CacheView& v, bool second, CUtensorMap* map, const char* who) {
    cuuint64_t dims[4] = {(cuuint64_t)kD, (cuuint64_t)v.Hkv, (cuuint64_t)v.page_size, (cuuint64_t)v.num_pages};
    cuuint64_t strides[3] = {(cuuint64_t)v.stride_head, (cuuint64_t)v.stride_tok, (cuuint64_t)v.stride_page};
    cuuint32_t box[4] = {64, 1, (cuuint32_t)v.page_size, 1}, es[4] = {1, 1, 1, 1};
    const CUresult r = ctx->encode_tiled(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(second ? v.v : v.k), dims, strides, box, es,
                                         CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return set_error(CP_ERR_CUDA, "%s: cuTensorMapEncodeTiled(%s) failed with %d", who, second ? "v" : "k", (int)r);
    return CP_OK;
}

template <Kind kKind, int kTiles>
int launch(cp_ctx* ctx, const WideParams& w, const CacheView& view, cudaStream_t s, const char* who) {
    using W = Wide<kKind, kTiles>;
    CUtensorMap k = {}, v = {};
    if (kKind == kBf16) {
        if (int rc = encode_kv(ctx, view, false, &k, who)) return rc;
        if (int rc = encode_kv(ctx, view, true, &v, who)) return rc;
    }
    if (!ctx->tree_attr_set[kKind][kTiles - 1]) {
        if (int rc = check_cuda(cudaFuncSetAttribute(tree_wide_kernel<kKind, kTiles>, cudaFuncAttributeMaxDynamicSharedMemorySize, W::kSmem),
                                "cudaFuncSetAttribute(tree)")) return rc;
        ctx->tree_attr_set[kKind][kTiles - 1] = true;
    }
    tree_wide_kernel<kKind, kTiles><<<(unsigned)(w.runs * w.classes), W::kThreads, W::kSmem, s>>>(k, v, w);
    if (int rc = check_cuda(cudaGetLastError(), who)) return rc;
    const unsigned y = (unsigned)((w.class_rows + kWideJoinRows - 1) / kWideJoinRows);
    return launch_behind(tree_join_kernel<kKind>, dim3((unsigned)(w.runs * w.classes), y), 32 * kWideJoinRows, s, who, w);
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
    w.runs = grid / w.classes;
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
