// Host side of gemm16.cuh: tensor maps, tile choice and launch.
#pragma once

#include "gemm16.cuh"

namespace csrt {

// Scratch of the split products: slabs of 128 x BN floats. A product takes splits only while they all fit.
constexpr size_t kPartialBytes = (size_t)24 << 20;

inline int dt_size(int dtype) { return dtype == CSRT_DT_F32 ? 4 : 2; }

// Rows that TMA (and 16-byte vector access) can take in place.
inline bool tma_rows_ok(const void *p, int64_t ld, int size) {
    return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld * size % 16 == 0;
}

struct GOperand {
    void *p;
    int64_t rows, cols, ld;   // as stored, row-major
    int64_t stride = 0;       // elements between batch matrices
};

struct GProduct {
    GOperand a, b;
    bool a_mn, b_mn;
    int64_t reduction;
};

// 3D map (columns, rows, batch) of row-major 16-byte aligned rows.
inline bool make_map3(CUtensorMap *map, const void *base, int dtype, int64_t rows, int64_t cols, int64_t ld,
                      int64_t batch, int64_t stride, int box_cols, int box_rows, CUtensorMapSwizzle swizzle) {
    auto fn = encode_fn();
    if (!fn) return false;
    const int size = dt_size(dtype);
    if (batch <= 1) stride = ld;   // any multiple of 16 bytes: never stepped over
    cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)batch};
    cuuint64_t strides[2] = {(cuuint64_t)(ld * size), (cuuint64_t)(stride * size)};
    cuuint32_t box[3] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows, 1u};
    cuuint32_t estr[3] = {1, 1, 1};
    const CUtensorMapDataType t = dtype == CSRT_DT_F32   ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                  : dtype == CSRT_DT_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16
                                                         : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    return fn(map, t, 3, const_cast<void *>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

inline bool operand_map(CUtensorMap *map, const GOperand &o, bool mn, int box_rows, int dtype, int batch) {
    return make_map3(map, o.p, dtype, o.rows, o.cols, o.ld, batch, o.stride, 64, mn ? kGBK : box_rows,
                     CU_TENSOR_MAP_SWIZZLE_128B);
}

inline bool out_map(CUtensorMap *map, const GMat &o, int m, int n, int batch) {
    return make_map3(map, o.p, o.dtype, m, n, o.ld, batch, o.stride, 32, 32,
                     o.dtype == CSRT_DT_F32 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B);
}

template <int CG, int BN, int EPI, bool PROMOTE>
int launch_tile(const GProduct &p, GArgs a, cudaStream_t s) {
    const int dtype = a.f16 ? CSRT_DT_F16 : CSRT_DT_BF16;
    GMaps maps = {};
    a.a_mn = p.a_mn;
    a.b_mn = p.b_mn;
    a.kb = (int32_t)ceil_div<int64_t>(p.reduction, kGBK);
    a.tiles_m = (int32_t)ceil_div<int64_t>(a.m, 128 * CG);
    a.tiles_n = (int32_t)ceil_div<int64_t>(a.n, BN);
    const bool sym = EPI == kEpiGram || EPI == kEpiPoly;
    const int64_t tiles = (int64_t)a.batch * (sym ? (int64_t)a.tiles_m * (a.tiles_m + 1) / 2 : (int64_t)a.tiles_m * a.tiles_n);
    if (a.splits < 1) a.splits = 1;
    a.kb_split = ceil_div<int32_t>(imax(a.kb, 1), a.splits);
    a.splits = ceil_div<int32_t>(imax(a.kb, 1), a.kb_split);
    CSRT_ARG(tiles * a.splits < ((int64_t)1 << 31), "product too large");
    a.units = (int32_t)(tiles * a.splits);
    // an empty reduction loads nothing; its maps still have to be valid, so they are left out
    if (a.kb > 0 && (!operand_map(&maps.a, p.a, p.a_mn, 128, dtype, a.batch) ||
                     !operand_map(&maps.b, p.b, p.b_mn, BN / CG, dtype, a.batch)))
        return fail(CSRT_ERR_CUDA, "cuTensorMapEncodeTiled refused an operand");
    if (a.out0.vec && !out_map(&maps.out0, a.out0, a.m, a.n, a.batch))
        return fail(CSRT_ERR_CUDA, "cuTensorMapEncodeTiled refused an output");
    if (a.out1.vec && !out_map(&maps.out1, a.out1, a.m, a.n, a.batch))
        return fail(CSRT_ERR_CUDA, "cuTensorMapEncodeTiled refused an output");
    auto kernel = gemm16_kernel<CG, BN, EPI, PROMOTE>;
    constexpr int smem = gsmem_bytes<CG, BN>();
    static bool attr_set[64] = {false};
    int dev = 0;
    CSRT_CHECK_CUDA(cudaGetDevice(&dev));
    if (dev < 0 || dev >= 64 || !attr_set[dev]) {
        CSRT_CHECK_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
        if (dev >= 0 && dev < 64) attr_set[dev] = true;
    }
    const int grid = imin(a.units, imax(1, num_sms() / CG)) * CG;
    launch_pdl(kernel, dim3(grid), dim3(kGThreads), smem, s, maps, a);
    count_launch();
    return check_launch("gemm16_kernel");
}

template <int EPI, bool PROMOTE>
int launch_gemm16(const GProduct &p, const GArgs &a, cudaStream_t s) {
    if (!device_is_sm10x()) return fail(CSRT_ERR_CUDA, "the dense products need a GPU with tcgen05");
    return launch_tile<1, 128, EPI, PROMOTE>(p, a, s);
}

}  // namespace csrt
