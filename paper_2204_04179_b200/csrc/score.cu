// Answers over an item table from the vectors themselves (gram_score_logprobs).
#include "logits.h"

namespace {

constexpr int SC_TILE = 32, SC_K = 32;

// z[n, v] = users[n] . items[v] + bias[v], a 32 x 32 tile per block
__global__ void __launch_bounds__(SC_TILE * SC_TILE) score_tile_kernel(const bf16* users, int64_t ld_u, const bf16* items, int64_t ld_i,
                                                                      const float* bias, int64_t N, int32_t V, int32_t d, float* z) {
  if (!chain_begin()) return;
  __shared__ float u[SC_TILE][SC_K + 1], w[SC_TILE][SC_K + 1];
  const int tx = threadIdx.x % SC_TILE, ty = threadIdx.x / SC_TILE;
  const int64_t n0 = (int64_t)blockIdx.y * SC_TILE, v0 = (int64_t)blockIdx.x * SC_TILE;
  float acc = 0.f;
  for (int k0 = 0; k0 < d; k0 += SC_K) {
    const bool in = k0 + tx < d;
    u[ty][tx] = in && n0 + ty < N ? __bfloat162float(users[(n0 + ty) * ld_u + k0 + tx]) : 0.f;
    w[ty][tx] = in && v0 + ty < V ? __bfloat162float(items[(v0 + ty) * ld_i + k0 + tx]) : 0.f;
    __syncthreads();
    for (int k = 0; k < SC_K; ++k) acc = fmaf(u[ty][k], w[tx][k], acc);
    __syncthreads();
  }
  if (n0 + ty < N && v0 + tx < V) z[(n0 + ty) * V + v0 + tx] = acc + (bias ? bias[v0 + tx] : 0.f);
}

}  // namespace

gram_status score_logprobs_launch(gram_ctx* ctx, const void* users, int64_t ld_users, const void* items, int64_t ld_items,
                                  const float* bias, int64_t N, int32_t V, int32_t d, float scale, const RowAnswers& ask, void* ws,
                                  size_t ws_bytes, cudaStream_t st) {
  const int64_t rows = (int64_t)(ws_bytes / sizeof(float)) / V;
  if (rows < 1) return gram_set_error(ctx, "gram_score_logprobs: %d items", V), GRAM_ERR_UNSUPPORTED;
  for (int64_t n = 0; n < N; n += rows) {
    const int64_t now = N - n < rows ? N - n : rows;
    launch_chain(score_tile_kernel, dim3((unsigned)ceil_div(V, SC_TILE), (unsigned)ceil_div64(now, SC_TILE)), SC_TILE * SC_TILE, 0, st,
                 (const bf16*)users + n * ld_users, ld_users, (const bf16*)items, ld_items, bias, now, V, d, (float*)ws);
    GRAM_LAUNCH_CHECK(ctx);
    RowAnswers part = ask;
    if (ask.C) { part.targets += n * ask.C; part.logp += n * ask.C; }
    if (ask.stats) part.stats += 2 * n;
    if (ask.entropy) part.entropy += n;
    if (ask.k) { part.top_logp += n * ask.k; part.top_ids += n * ask.k; }
    GRAM_TRY(logprobs_launch(ctx, ws, GRAM_F32, V, now, V, scale, part, st));
  }
  return GRAM_OK;
}
