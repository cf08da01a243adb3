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

// Rows that TMA may store: it writes whole units of 16 bytes, so one that ends inside a unit would write into the gap
// before the next (a load stops at the element).
inline bool tma_store_ok(const void *p, int64_t ld, int64_t cols, int size) {
    return tma_rows_ok(p, ld, size) && cols * size % 16 == 0;
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

// Tiles of a product; `sym`: those that reach above the diagonal, `ratio` tile columns to a tile row.
inline int64_t tile_count(bool sym, int64_t tm, int64_t tn, int64_t ratio) {
    return sym ? tm * tn - ratio * (tm * (tm - 1) / 2) : tm * tn;
}

inline bool operand_map(CUtensorMap *map, const GOperand &o, bool mn, int box_rows, int dtype, int batch) {
    return make_map3(map, o.p, dtype, o.rows, o.cols, o.ld, batch, o.stride, 64, mn ? kGBK : box_rows,
                     CU_TENSOR_MAP_SWIZZLE_128B);
}

inline bool out_map(CUtensorMap *map, const GMat &o, int m, int n, int batch) {
    return make_map3(map, o.p, o.dtype, m, n, o.ld, batch, o.stride, 32, 32,
                     o.dtype == CSRT_DT_F32 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B);
}

// Dimensions and maps of one product on CG x 128 x BN tiles.
template <int CG, int BN, int EPI, bool PROMOTE>
int fill_set(const GProduct &p, GArgs &a, GMaps &maps) {
    const int dtype = a.f16 ? CSRT_DT_F16 : CSRT_DT_BF16;
    a.a_mn = p.a_mn;
    a.b_mn = p.b_mn;
    a.kb = (int32_t)ceil_div<int64_t>(p.reduction, kGBK);
    a.tiles_m = (int32_t)ceil_div<int64_t>(a.m, 128 * CG);
    a.tiles_n = (int32_t)ceil_div<int64_t>(a.n, BN);
    const int64_t tiles = a.batch * tile_count(a.sym, a.tiles_m, a.tiles_n, 128 * CG / BN);
    if (a.splits < 1) a.splits = 1;
    a.kb_split = ceil_div<int32_t>(imax(a.kb, 1), a.splits);
    a.splits = ceil_div<int32_t>(imax(a.kb, 1), a.kb_split);
    CSRT_ARG(tiles * a.splits < ((int64_t)1 << 31), "product too large");
    a.units = (int32_t)(a.splits == 1 ? tiles : a.whole + (tiles - a.whole) * a.splits);
    // an empty reduction loads nothing; its maps still have to be valid, so they are left out
    if (a.kb > 0 && (!operand_map(&maps.a, p.a, p.a_mn, 128, dtype, a.batch) ||
                     !operand_map(&maps.b, p.b, p.b_mn, BN / CG, dtype, a.batch)))
        return fail(CSRT_ERR_CUDA, "cuTensorMapEncodeTiled refused an operand");
    if (a.out0.vec && !out_map(&maps.out0, a.out0, a.m, a.n, a.batch))
        return fail(CSRT_ERR_CUDA, "cuTensorMapEncodeTiled refused an output");
    if (a.out1.vec && !out_map(&maps.out1, a.out1, a.m, a.n, a.batch))
        return fail(CSRT_ERR_CUDA, "cuTensorMapEncodeTiled refused an output");
    // one aligned 16-bit output, at most one operand: a group needs half the staging; a float32 output has it
    // twice (PROMOTE)
    const bool two_in = a.c0.p != nullptr && a.c1.p != nullptr;
    a.slots = PROMOTE || (EPI != kEpiNs && a.out0.dtype != CSRT_DT_F32 && a.out1.p == nullptr && !two_in && a.out0.vec) ? 2 : 1;
    return CSRT_OK;
}

template <auto kernel>
int allow_smem(int smem) {
    static bool done[64] = {false};
    int dev = 0;
    CSRT_CHECK_CUDA(cudaGetDevice(&dev));
    if (dev < 0 || dev >= 64 || !done[dev]) {
        CSRT_CHECK_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
        if (dev >= 0 && dev < 64) done[dev] = true;
    }
    return CSRT_OK;
}

// Time of a product in microseconds by a simple model of gemm16_kernel: waves of units, each loading its stages and
// then running an epilogue that overlaps the next unit's stages but not the last's; joining slices costs their
// partial tiles' trip through L2. The constants are fitted to measured times of 69 products of 64 to 9216 rows and
// columns on every tile and up to 16 slices; the choice they give is within 1.2% of the best on average. The longer
// epilogues are fitted to 24 products of odd sizes: dx of 4096 x 1777 from 1000 rows takes 21.9 us on 128 x 128 tiles
// and 24.9 on the 256 x 256 that the short one would choose, aligned with z and a residual 22.8 and 27.2.
struct GTile {
    int cg, bn;
    double stage, epi;   // us per stage, us per unit's epilogue
    double epi_more;     // the same in the general kernel, or with z or two more matrices to read and write
};
constexpr int kTileKinds = 4;
constexpr GTile kTiles[kTileKinds] = {
    {2, 256, 0.34, 5.7, 8.8}, {1, 128, 0.245, 4.3, 5.9}, {1, 64, 0.206, 3.6, 4.0}, {2, 128, 0.228, 4.4, 6.6}};
inline double model_us(const GTile &t, int64_t tiles, int64_t kb, int64_t whole, int64_t splits) {
    const int64_t slots = imax(1, num_sms() / t.cg);
    const double tile = (double)imax<int64_t>(kb, 1) * t.stage;
    double us = t.epi - 1.75;
    if (whole > 0) us += ceil_div(whole, slots) * (tile > t.epi ? tile : t.epi);
    if (tiles > whole) {
        const double unit = (double)ceil_div(imax<int64_t>(kb, 1), splits) * t.stage;
        us += ceil_div((tiles - whole) * splits, slots) * (unit > t.epi ? unit : t.epi);
    }
    if (splits > 1) us += 3.9 + 0.446 * splits * t.bn / 64;
    return us;
}

// Best sharing of a product's reductions on tiles t, and its time: all tiles in one number of slices, or (tail) those
// that are left over after whole waves.
struct GSplit {
    int whole, splits;
    double us;
};
inline GSplit best_splits(const GTile &t, const GArgs &a, int64_t reduction, bool tail) {
    const int64_t kb = ceil_div<int64_t>(reduction, kGBK), slots = imax(1, num_sms() / t.cg);
    const int64_t tiles = a.batch * tile_count(a.sym, ceil_div<int64_t>(a.m, 128 * t.cg), ceil_div<int64_t>(a.n, t.bn),
                                               128 * t.cg / t.bn);
    GSplit best = {0, 1, model_us(t, tiles, kb, 0, 1)};
    const int64_t waves = tail && tiles < ((int64_t)1 << 30) ? tiles / slots : 0;
    for (int64_t whole = 0; whole <= waves * slots; whole += imax<int64_t>(1, waves * slots)) {
        const int64_t rest = tiles - whole;
        for (int64_t sp = 2; sp <= 32 && sp * 2 <= kb && rest > 0 && rest * (sp - 1) < 2 * slots; ++sp) {
            if ((size_t)(rest * sp) * t.cg * 128 * t.bn * sizeof(float) > kPartialBytes ||
                rest * t.cg * kGEpiWarps > (int64_t)kWsCounterInts)
                break;
            const double us = model_us(t, tiles, kb, whole, sp);
            if (us < best.us) best = {(int)whole, (int)sp, us};
        }
    }
    return best;
}

// Whether the kernel for aligned matrices serves: every epilogue matrix 16-byte aligned and of the kernel's own types,
// and its operands readable in units of 16 bytes up to the end of a row.
inline bool aligned_set(const GArgs &a, bool wide) {
    auto fine = [&](const GMat &c, bool w) {
        return c.p == nullptr || (c.vec && (c.dtype == CSRT_DT_F32) == w && (w ? a.n % 4 == 0 : c.pad || a.n % 8 == 0));
    };
    return a.out0.vec && (a.out0.dtype == CSRT_DT_F32) == wide && (a.out1.p == nullptr || a.out1.vec) && fine(a.c0, false) &&
           fine(a.c1, wide);
}

template <int CG, int BN, int EPI, bool PROMOTE, bool GEN>
int launch_tile(const GProduct &p, const GArgs &a, cudaStream_t s) {
    GLaunch<EPI> l = {};
    l.args[0] = a;
    l.phases = 1;
    int rc = fill_set<CG, BN, EPI, PROMOTE>(p, l.args[0], l.maps[0]);
    if (rc != CSRT_OK) return rc;
    constexpr auto kernel = gemm16_kernel<CG, BN, EPI, PROMOTE, GEN, false>;
    constexpr int smem = gsmem_bytes<CG, BN, EPI, PROMOTE>();
    rc = allow_smem<kernel>(smem);
    if (rc != CSRT_OK) return rc;
    const int grid = imin(l.args[0].units, imax(1, num_sms() / CG)) * CG;
    launch_pdl(kernel, dim3(grid), dim3(kGThreads), smem, s, l);
    count_launch();
    return check_launch("gemm16_kernel");
}

// The tile and slices of a product by the model.
struct GChoice {
    int tile;
    GSplit split;
};
inline GChoice choose_tile(const GArgs &a, int64_t reduction, bool aligned) {
    const bool more = !aligned || a.c0.p != nullptr || (a.c1.p != nullptr && a.out1.p != nullptr);
    GChoice best = {0, {0, 1, 1e30}};
    for (int c = 0; c < kTileKinds; ++c) {
        GTile t = kTiles[c];
        if (more) t.epi = t.epi_more;
        const GSplit s = best_splits(t, a, reduction, true);
        if (s.us < best.split.us) best = {c, s};
    }
    return best;
}

// Stages of the longest accumulation that sharing `s` leaves of a reduction.
inline int64_t longest(const GSplit &s, int64_t reduction) {
    const int64_t kb = ceil_div<int64_t>(reduction, kGBK);
    return s.splits == 1 || s.whole > 0 ? kb : ceil_div<int64_t>(kb, s.splits);
}

// A 16-bit result of sums too long for one accumulation is the promoting kernel's, in its general form.
template <int EPI, bool PROMOTE>
int launch_gemm16(const GProduct &p, GArgs a, cudaStream_t s) {
    if (!device_is_sm10x()) return fail(CSRT_ERR_CUDA, "the dense products need a GPU with tcgen05");
    const bool aligned = aligned_set(a, PROMOTE);
    const GChoice choice = choose_tile(a, p.reduction, aligned);
    if constexpr (!PROMOTE)
        if (longest(choice.split, p.reduction) > (a.f16 ? kLongF16 : kLongBf16)) return launch_gemm16<EPI, true>(p, a, s);
    const int best = choice.tile;
    a.whole = choice.split.whole;
    a.splits = choice.split.splits;
    if (aligned) {
        if (best == 0) return launch_tile<2, 256, EPI, PROMOTE, false>(p, a, s);
        if (best == 1) return launch_tile<1, 128, EPI, PROMOTE, false>(p, a, s);
        if (best == 3) return launch_tile<2, 128, EPI, PROMOTE, false>(p, a, s);
        return launch_tile<1, 64, EPI, PROMOTE, false>(p, a, s);
    }
    if (best == 0) return launch_tile<2, 256, EPI, PROMOTE, true>(p, a, s);
    if (best == 1) return launch_tile<1, 128, EPI, PROMOTE, true>(p, a, s);
    if (best == 3) return launch_tile<2, 128, EPI, PROMOTE, true>(p, a, s);
    return launch_tile<1, 64, EPI, PROMOTE, true>(p, a, s);
}

}  // namespace csrt
