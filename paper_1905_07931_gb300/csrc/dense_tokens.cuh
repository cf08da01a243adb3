// The few-token forward product, see dense_tokens.cu.
#pragma once

#include "gemm16.cuh"

namespace csrt {

constexpr int kTokensMax = 4;

struct TokenArgs {
    const uint16_t *w, *x;
    int64_t ldw, ldx;
    int32_t m, k, wpr;      // wpr: warps that share a pair of rows
    const float *bias;
    int32_t act;
    GMat res, z, y;
};

// vec: k % 8 == 0, rows of w 16-byte aligned, x without gaps between its rows and 16-byte aligned.
int dense_tokens(TokenArgs a, int n, bool f16, bool vec, cudaStream_t s);

}  // namespace csrt
