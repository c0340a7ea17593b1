// Softmax cross entropy of users against an item table, with its gradients (gram_score_loss).
#pragma once
#include "gram_internal.h"

struct ScoreLoss {
  const void* users;                  // bf16 [N, d]
  const void* items;                  // bf16 [V, d]
  int64_t ld_users, ld_items;
  const float* bias;                  // [V] or null
  int64_t N;
  int32_t V, d;
  float scale;
  const int32_t* targets;             // [N]
  const float* weight;                // [N] or null
  float* loss;                        // [N]
  int grad_dtype;
  void *dusers, *ditems;              // null: not asked
  int64_t ld_dusers, ld_ditems;
  float* dbias;                       // [V] or null
};

// bytes of the caller's workspace: the least that serves, and beyond `best` nothing is gained
void score_loss_workspace(int64_t N, int32_t V, int32_t d, int grad_dtype, size_t* least, size_t* best);
// ws: the caller's; score_ws: the context's workspace for products (the answers without alternatives take it)
gram_status score_loss_launch(gram_ctx* ctx, const ScoreLoss& a, void* ws, size_t ws_bytes, void* score_ws, size_t score_ws_bytes, cudaStream_t st);
