// Rows of logits over a pool of items or a vocabulary: log probabilities and what else is read from them, their gradient,
// distillation, and the same answers from the vectors whose products the logits are.
#pragma once
#include "gram_internal.h"

// What is asked of each of N rows (see gram_logprobs); null pointers: not asked.
struct RowAnswers {
  const int32_t* targets = nullptr;   // [N, C]
  float* logp = nullptr;              // [N, C]
  float* stats = nullptr;             // [N, 2]
  float* entropy = nullptr;           // [N]
  float* top_logp = nullptr;          // [N, k]
  int32_t* top_ids = nullptr;         // [N, k]
  int32_t C = 0, k = 0;
};

gram_status logprobs_launch(gram_ctx* ctx, const void* logits, int dtype, int64_t ld, int64_t N, int32_t V, float scale,
                            const RowAnswers& ask, cudaStream_t st);
gram_status logprobs_backward_launch(gram_ctx* ctx, const void* logits, int dtype, int64_t ld, int64_t N, int32_t V, float scale,
                                     const int32_t* targets, int32_t C, const float* stats, const float* entropy, const float* dlogp,
                                     const float* dentropy, void* dlogits, int64_t ld_out, cudaStream_t st);
gram_status distill_launch(gram_ctx* ctx, const void* logits, int dtype, int64_t ld, int64_t N, int32_t V, float scale,
                           const int32_t* teacher_ids, const float* teacher_logits, int32_t k, float* loss, const float* weight,
                           void* dlogits, int64_t ld_out, cudaStream_t st);
gram_status score_logprobs_launch(gram_ctx* ctx, const void* users, int64_t ld_users, const void* items, int64_t ld_items,
                                  const float* bias, int64_t N, int32_t V, int32_t d, float scale, const RowAnswers& ask, void* ws,
                                  size_t ws_bytes, cudaStream_t st);
// the logits themselves, [N, ld_logits] (ld_logits >= V, a multiple of 8, 32-byte aligned): what N x V are few enough for
gram_status score_logits_launch(gram_ctx* ctx, const void* users, int64_t ld_users, const void* items, int64_t ld_items, const float* bias, int64_t N,
                                int32_t V, int32_t d, float* logits, int64_t ld_logits, cudaStream_t st);
