// Answers read from rows of logits, and their gradients (gram_logprobs, gram_logprobs_backward, gram_distill).
#include "logits.h"
#include "row_softmax.cuh"

namespace {

constexpr int LP_THREADS = 256, LP_WARPS = LP_THREADS / 32;

// the block's statistics, in every thread
__device__ __forceinline__ RowStat join_block(RowStat r, float c, RowStat* part) {
  r = row_join_warp(r, c);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = r;
  __syncthreads();
  r = part[0];
  for (int w = 1; w < LP_WARPS; ++w) r = row_join(r, part[w], c);
  return r;
}
template <typename T> __device__ __forceinline__ RowStat row_statistics(const T* z, int V, float c, RowStat* part) {
  RowStat r = row_empty();
  for (int v = threadIdx.x; v < V; v += LP_THREADS) row_add(r, row_load(z + v), c);
  return join_block(r, c, part);
}

template <typename T>
__global__ void __launch_bounds__(LP_THREADS) logprobs_kernel(const T* logits, int64_t ld, int32_t V, float scale, RowAnswers ask,
                                                              int32_t* status) {
  if (!chain_begin()) return;
  __shared__ RowStat part[LP_WARPS];
  __shared__ uint64_t best[LP_WARPS];
  const int64_t n = blockIdx.x;
  const T* z = logits + n * ld;
  const RowStat r = row_statistics(z, V, scale * kLog2e, part);
  const float log_s = row_log_sum(r);
  if (threadIdx.x == 0) {
    if (ask.stats) { ask.stats[2 * n] = r.m; ask.stats[2 * n + 1] = log_s; }
    if (ask.entropy) ask.entropy[n] = row_entropy(r);
  }
  for (int i = threadIdx.x; i < ask.C; i += LP_THREADS) {
    const int32_t t = ask.targets[n * ask.C + i];
    if (t < -1 || t >= V) gram_device_fail(status, GRAM_ERR_ID_RANGE);
    ask.logp[n * ask.C + i] = t >= 0 && t < V ? row_logp(row_load(z + t), r.m, log_s, scale) : 0.f;
  }
  uint64_t last = ~0ull;
  for (int j = 0; j < ask.k; ++j) {                 // the largest key below the last one
    uint64_t b = 0;
    for (int v = threadIdx.x; v < V; v += LP_THREADS) {
      const float x = row_load(z + v);
      const uint64_t key = row_key(x, v);
      if (x > ROW_NEG_INF && key < last && key > b) b = key;
    }
    for (int o = 16; o > 0; o >>= 1) b = max(b, __shfl_xor_sync(0xffffffffu, b, o));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) best[threadIdx.x >> 5] = b;
    __syncthreads();
    for (int w = 0; w < LP_WARPS; ++w) b = max(b, best[w]);
    if (threadIdx.x == 0) {
      ask.top_ids[n * ask.k + j] = b ? row_key_place(b) : -1;
      ask.top_logp[n * ask.k + j] = b ? row_logp(row_key_logit(b), r.m, log_s, scale) : ROW_NEG_INF;
    }
    last = b;
  }
}

struct BackwardArgs {
  const int32_t* targets;
  const float* stats;
  const float* entropy;
  const float* dlogp;
  const float* dentropy;
  int64_t ld, ld_out;
  int32_t V, C;
  float scale;
  int32_t* status;
};

// dz = scale (sum of g at the given places - p (sum of all g + h (log p + H))), 0 at masked places
template <typename T>
__global__ void __launch_bounds__(LP_THREADS) logprobs_backward_kernel(const T* logits, T* dlogits, BackwardArgs a) {
  if (!chain_begin()) return;
  __shared__ float g_at[GRAM_TOP_MAX];               // of each given token that takes part: its gradient, place and logit
  __shared__ int32_t place[GRAM_TOP_MAX];
  __shared__ float z_at[GRAM_TOP_MAX];
  const int64_t n = blockIdx.x;
  const T* z = logits + n * a.ld;
  T* dz = dlogits + n * a.ld_out;
  for (int i = threadIdx.x; i < a.C; i += LP_THREADS) {
    int32_t t = a.targets[n * a.C + i];
    if (t < -1 || t >= a.V) { gram_device_fail(a.status, GRAM_ERR_ID_RANGE); t = -1; }
    const float x = t >= 0 ? row_load(z + t) : ROW_NEG_INF;
    place[i] = x == ROW_NEG_INF ? -1 : t;
    z_at[i] = x;
    g_at[i] = x == ROW_NEG_INF ? 0.f : a.dlogp[n * a.C + i];
  }
  __syncthreads();
  float G = 0.f;
  for (int i = 0; i < a.C; ++i) G += g_at[i];
  const float m = row_base(a.stats[2 * n]), log_s = a.stats[2 * n + 1], h = a.dentropy ? a.dentropy[n] : 0.f, H = a.dentropy ? a.entropy[n] : 0.f;
  const bool none = G == 0.f && h == 0.f;
  auto dense = [&](float x) {
    if (none || x == ROW_NEG_INF) return 0.f;
    const float lp = (x - m) * a.scale - log_s;
    return -a.scale * (row_ex2(lp * kLog2e) * (G + h * row_hold(lp + H)));
  };
  for (int v = threadIdx.x; v < a.V; v += LP_THREADS) dz[v] = row_round<T>(dense(row_load(z + v)));
  __syncthreads();
  for (int i = threadIdx.x; i < a.C; i += LP_THREADS) {
    if (place[i] < 0) continue;
    float g = 0.f;
    bool first = true;
    for (int j = 0; j < a.C; ++j)
      if (place[j] == place[i]) {
        first = first && j >= i;
        g += g_at[j];
      }
    if (first) dz[place[i]] = row_round<T>(dense(z_at[i]) + a.scale * g);
  }
}

struct DistillArgs {
  const int32_t* ids;
  const float* teacher;
  float* loss;
  const float* weight;
  int64_t ld, ld_out;
  int32_t V, k;
  float scale;
  int32_t* status;
};

template <typename T>
__global__ void __launch_bounds__(LP_THREADS) distill_kernel(const T* logits, T* dlogits, DistillArgs a) {
  if (!chain_begin()) return;
  __shared__ RowStat part[LP_WARPS];
  __shared__ float q_at[GRAM_TOP_MAX], z_at[GRAM_TOP_MAX];
  __shared__ int32_t place[GRAM_TOP_MAX];
  const int64_t n = blockIdx.x;
  const T* z = logits + n * a.ld;
  for (int i = threadIdx.x; i < a.k; i += LP_THREADS) {
    int32_t t = a.ids[n * a.k + i];
    if (t < -1 || t >= a.V) { gram_device_fail(a.status, GRAM_ERR_ID_RANGE); t = -1; }
    const float x = t >= 0 ? row_load(z + t) : ROW_NEG_INF, b = a.teacher[n * a.k + i];
    place[i] = x == ROW_NEG_INF || b == ROW_NEG_INF ? -1 : t;
    z_at[i] = x;
    q_at[i] = b;
  }
  const RowStat r = row_statistics(z, a.V, a.scale * kLog2e, part);
  const float log_s = row_log_sum(r), m = row_base(r.m);
  RowStat q = row_empty();
  for (int i = 0; i < a.k; ++i)
    if (place[i] >= 0) row_add(q, q_at[i], a.scale * kLog2e);
  const bool some = q.s != 0.f;
  const float log_q = row_log_sum(q);
  __syncthreads();
  if (threadIdx.x == 0) {
    float sum = 0.f;
    for (int i = 0; i < a.k; ++i) {
      if (place[i] < 0) continue;
      const float lq = (q_at[i] - q.m) * a.scale - log_q, e = expf(lq);
      if (!(e == 0.f)) sum += e * (lq - row_logp(z_at[i], r.m, log_s, a.scale));
    }
    a.loss[n] = sum;
  }
  if (!dlogits) return;
  const float w = (a.weight ? a.weight[n] : 1.f) * a.scale;
  const bool none = w == 0.f || !some;
  T* dz = dlogits + n * a.ld_out;
  auto p = [&](float x) { return none ? 0.f : w * row_ex2(row_hold((x - m) * a.scale * kLog2e - log_s * kLog2e)); };
  for (int v = threadIdx.x; v < a.V; v += LP_THREADS) dz[v] = row_round<T>(p(row_load(z + v)));
  __syncthreads();
  if (none) return;
  for (int i = threadIdx.x; i < a.k; i += LP_THREADS) {
    if (place[i] < 0) continue;
    float sum = 0.f;
    bool first = true;
    for (int j = 0; j < a.k; ++j)
      if (place[j] == place[i]) {
        first = first && j >= i;
        sum += expf((q_at[j] - q.m) * a.scale - log_q);
      }
    if (first) dz[place[i]] = row_round<T>(p(z_at[i]) - w * sum);
  }
}

}  // namespace

gram_status logprobs_launch(gram_ctx* ctx, const void* logits, int dtype, int64_t ld, int64_t N, int32_t V, float scale,
                            const RowAnswers& ask, cudaStream_t st) {
  if (N == 0) return GRAM_OK;
  ProfScope prof(ctx, GRAM_K_OTHER, (double)N * V * (dtype == GRAM_F32 ? 4 : 2), 1, st, "logprobs");
  int32_t* status = gram_status_word(ctx);
  if (dtype == GRAM_F32)
    launch_chain(logprobs_kernel<float>, dim3((unsigned)N), LP_THREADS, 0, st, (const float*)logits, ld, V, scale, ask, status);
  else
    launch_chain(logprobs_kernel<bf16>, dim3((unsigned)N), LP_THREADS, 0, st, (const bf16*)logits, ld, V, scale, ask, status);
  GRAM_LAUNCH_CHECK(ctx);
  return GRAM_OK;
}

gram_status logprobs_backward_launch(gram_ctx* ctx, const void* logits, int dtype, int64_t ld, int64_t N, int32_t V, float scale,
                                     const int32_t* targets, int32_t C, const float* stats, const float* entropy, const float* dlogp,
                                     const float* dentropy, void* dlogits, int64_t ld_out, cudaStream_t st) {
  if (N == 0) return GRAM_OK;
  ProfScope prof(ctx, GRAM_K_OTHER, 2.0 * N * V * (dtype == GRAM_F32 ? 4 : 2), 1, st, "logprobs_backward");
  const BackwardArgs a{targets, stats, entropy, dlogp, dentropy, ld, ld_out, V, C, scale, gram_status_word(ctx)};
  if (dtype == GRAM_F32)
    launch_chain(logprobs_backward_kernel<float>, dim3((unsigned)N), LP_THREADS, 0, st, (const float*)logits, (float*)dlogits, a);
  else
    launch_chain(logprobs_backward_kernel<bf16>, dim3((unsigned)N), LP_THREADS, 0, st, (const bf16*)logits, (bf16*)dlogits, a);
  GRAM_LAUNCH_CHECK(ctx);
  return GRAM_OK;
}

gram_status distill_launch(gram_ctx* ctx, const void* logits, int dtype, int64_t ld, int64_t N, int32_t V, float scale,
                           const int32_t* teacher_ids, const float* teacher_logits, int32_t k, float* loss, const float* weight,
                           void* dlogits, int64_t ld_out, cudaStream_t st) {
  if (N == 0) return GRAM_OK;
  ProfScope prof(ctx, GRAM_K_OTHER, (dlogits ? 2.0 : 1.0) * N * V * (dtype == GRAM_F32 ? 4 : 2), 1, st, "distill");
  const DistillArgs a{teacher_ids, teacher_logits, loss, weight, ld, ld_out, V, k, scale, gram_status_word(ctx)};
  if (dtype == GRAM_F32)
    launch_chain(distill_kernel<float>, dim3((unsigned)N), LP_THREADS, 0, st, (const float*)logits, (float*)dlogits, a);
  else
    launch_chain(distill_kernel<bf16>, dim3((unsigned)N), LP_THREADS, 0, st, (const bf16*)logits, (bf16*)dlogits, a);
  GRAM_LAUNCH_CHECK(ctx);
  return GRAM_OK;
}
