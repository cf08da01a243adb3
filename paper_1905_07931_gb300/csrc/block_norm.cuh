// The norms around a block of a residual network (include/csrtrain.h, csrt_block_norm_*): arguments of the kernels.
#pragma once

#include "gemm16.cuh"

namespace csrt {

struct NormSide {
    int32_t kind;                 // CSRT_NORM_*, -1: no such norm
    float eps;
    const float *w, *b;
    float *mean, *rstd;
    float *dw, *db;
};

// p == nullptr: the matrix is not given.
struct NormMat {
    char *p;
    int64_t ld;
};

struct NormArgs {
    int32_t d, n;
    int32_t gate_act;
    int32_t accumulate;
    float r_scale;
    NormSide post, pre;
    NormMat y, g, r, h, v;         // r is dh in the backward pass
    NormMat dv, dr, dy, dg;
    float *partial;                // backward: row sums of a group of tokens, [group][4][d] (post dw, db; pre dw, db)
    int32_t cluster;               // blocks that share the features of a tile
    int32_t chunk, box, boxes;     // features of a block, and the loads that bring them
    WsHeader *hdr;               // takes the flag of a wait that ran out, may be nullptr
    int32_t groups;                // blocks (or clusters) along the tokens, each with row sums of its own
};

constexpr int kNormGroups = 304;   // two for each SM of a GB300
enum { kSumPostW = 0, kSumPostB = 1, kSumPreW = 2, kSumPreB = 3 };

template <typename T>
__device__ __forceinline__ float to_f(T v);
template <>
__device__ __forceinline__ float to_f(float v) { return v; }
template <>
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
template <>
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T>
__device__ __forceinline__ T from_f(float v);
template <>
__device__ __forceinline__ float from_f(float v) { return v; }
template <>
__device__ __forceinline__ __half from_f(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f(float v) { return __float2bfloat16_rn(v); }

// silu and its slope are products with sigmoid's tails, which are 0 to float32 from |g| = 104 on: with the factor g held to 128
// an infinite gate has its limits there (-0, and a slope of 0 or 1) instead of 0 times infinity. A NaN stays.
__device__ __forceinline__ float above_m128(float g) {
    asm("max.NaN.f32 %0, %0, 0fC3000000;" : "+f"(g));
    return g;
}
__device__ __forceinline__ float within_128(float g) {
    asm("min.NaN.xorsign.abs.f32 %0, %0, 0f43000000;" : "+f"(g));   // min(|g|, 128) with g's sign
    return g;
}

// a(g) and a'(g). FAST, by the type of g, takes the fast exponential and quotient: the sigmoid is off by (4 + 1.2 |g|) 2^-23 of
// itself, in a float32 h and the norms' float32 gradients too. g is then a value of 16 bits, whose own half step moves the sigmoid
// by (1 - p) |g| 2^-9 (bfloat16) or 2^-12. float32 gates take the others.
template <bool FAST>
__device__ __forceinline__ void gate_both(float g, int act, float &value, float &slope) {
    value = g;
    slope = 1.f;
    if (act == CSRT_GATE_NONE) return;
    const float e = FAST ? __expf(-g) : expf(-g);
    const float p = FAST ? __fdividef(1.f, 1.f + e) : 1.f / (1.f + e);
    const float q = fminf(e * p, 1.f);   // 1 - p, with all digits where p is near 1; 1 where e is infinite (and the product NaN)
    value = act == CSRT_GATE_SIGMOID ? p : above_m128(g) * p;
    slope = act == CSRT_GATE_SIGMOID ? p * q : p * (1.f + within_128(g) * q);
}
template <bool FAST>
__device__ __forceinline__ float gate_value(float g, int act) {
    float value, slope;
    gate_both<FAST>(g, act, value, slope);
    return value;
}

// Tiles of the kernels that read every matrix once: tokens wide, features a thread.
enum NormTile { kTileColumns, kTile1x4, kTile1x16, kTile32x8, kTile32x4, kTile32x2, kTile16x5, kTile16x4, kTile16x2, kTile8x4, kTile8x2 };
// By the type of the block's matrices and, where it is another, of the stream. in, out: the rows of all inputs, or results,
// are 16-byte aligned.
typedef int NormFwd(const NormArgs &a, NormTile t, bool in, bool out, cudaStream_t s);
typedef int NormBwd(NormArgs &a, NormTile t, bool in, bool out, cudaStream_t s);   // sets a.groups
NormFwd norm_fwd_bf16, norm_fwd_bf16_f32, norm_fwd_f16, norm_fwd_f16_f32, norm_fwd_f32;
NormBwd norm_bwd_bf16, norm_bwd_bf16_f32, norm_bwd_f16, norm_bwd_f16_f32, norm_bwd_f32;

}  // namespace csrt
