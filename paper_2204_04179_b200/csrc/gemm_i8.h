// Rows in 8 bits with a scale each, and their products.
#pragma once
#include "gram_internal.h"

gram_status quantize_rows_launch(gram_ctx* ctx, const void* x, int dtype, int64_t ld, int64_t rows, int32_t cols, int8_t* codes, int64_t ld_codes,
                                 float* scale, cudaStream_t st);
// C[m, n] = scale_a[m] scale_b[n] sum_k A[m, k] B[n, k] + bias[n]
gram_status gemm_i8_launch(gram_ctx* ctx, const int8_t* A, int64_t lda, const float* scale_a, const int8_t* B, int64_t ldb, const float* scale_b,
                           const float* bias, void* C, int c_dtype, int64_t ldc, int64_t M, int32_t N, int32_t K, cudaStream_t st);
