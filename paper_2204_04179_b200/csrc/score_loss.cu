// Softmax cross entropy of users against an item table, from the vectors themselves, with its gradients (gram_score_loss).
//
// With z = U I^T + b, p the softmax of scale z and t the rows' targets, loss_n = log sum_v exp(scale z_nv) - scale z_n,t, and the
// gradient of sum_n w_n loss_n with respect to z is g_nv = w_n scale (p_nv - [v = t_n]); then dU = g I, dI = g^T U, db_v = sum_n g_nv.
//
// g has as many entries as the logits, which are never kept: it is formed for a piece of the items at a time.
//   1. The statistics of the rows (m and log s) come from the kernels of gram_score_logprobs: one product.
//   2. loss_rows_kernel: the loss, and what a row's g needs, in one float4.
//   3. Of each piece: loss_grad_kernel forms its logits again on the tensor cores and writes g to the workspace in bf16 (for fp32
//      gradients as the sum of two bf16: 2^-16 of each entry); loss_products_kernel takes both products of it, dU += g I and dI = g^T U,
//      in one launch of tiles of either kind.
//   4. loss_finish_kernel: dU from its parts.
// Bounded by the tensor cores where users are many: 8 N V d flops (12 with fp32 gradients), of which the products that cannot be done
// without are 6; by the table's bytes, read three times and written once, where they are few.
#include "score_loss.h"

#include "logits.h"
#include "pair_pipe.cuh"
#include "row_softmax.cuh"

namespace {
using namespace tc;

constexpr int kPairs = kNumSMs / 2;
constexpr int LOSS_FEW = 256;                           // users whose logits are kept where 32 MB hold them

// ============================================================================================
// rows: loss, and the constants of g
// ============================================================================================
// What g needs of a row: p = 2^(c (z - m) - l), g = f (p - [v = t]).  t = -1: the row takes no part.  p is held at 1: of rows of huge
// logits m is a sum in another order than z.  f is NaN in a row whose loss is.
struct RowConst {
  float m, l, f;
  int32_t t;
};
static_assert(sizeof(RowConst) == 16, "read as one float4");

// A row's statistics, log p of its target and weight.
__device__ __forceinline__ RowConst loss_row(const ScoreLoss& a, const float* logp, const float2* stats, int64_t n) {
  const int32_t t = a.targets[n];
  const float lp = logp[n], w = a.weight ? a.weight[n] : 1.f;
  const float2 s = stats[n];
  const bool part = t >= 0 && t < a.V && w != 0.f && lp != ROW_NEG_INF;
  return RowConst{s.x, s.y * kLog2e, lp != lp ? lp : w * a.scale, part ? t : -1};
}
__device__ __forceinline__ float loss_of(const ScoreLoss& a, const float* logp, int64_t n, int32_t* status) {
  const int32_t t = a.targets[n];
  if (t >= 0 && t < a.V) return 0.f - logp[n];
  if (t != -1) gram_device_fail(status, GRAM_ERR_ID_RANGE);
  return 0.f;
}
// The user's vector, by a warp: zeros for a row that takes no part, so that whatever a padded row holds does not reach dI (0 times NaN).
__device__ __forceinline__ void loss_clean(const ScoreLoss& a, int64_t n, bool part, bf16* clean) {
  const uint4* from = reinterpret_cast<const uint4*>(reinterpret_cast<const bf16*>(a.users) + n * a.ld_users);
  uint4* to = reinterpret_cast<uint4*>(clean + n * a.d);
  for (int i = threadIdx.x & 31; i < a.d / 8; i += 32) to[i] = part ? __ldg(from + i) : make_uint4(0u, 0u, 0u, 0u);
}

// A warp a user.  rows, clean: null where they are not needed.
__global__ void __launch_bounds__(256) loss_rows_kernel(const ScoreLoss a, const float* logp, const float2* stats, RowConst* rows, bf16* clean,
                                                        int32_t* status) {
  if (!chain_begin()) return;
  const int64_t n = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (n >= a.N) return;
  const RowConst r = loss_row(a, logp, stats, n);
  if ((threadIdx.x & 31) == 0) {
    a.loss[n] = loss_of(a, logp, n, status);
    if (rows) rows[n] = r;
  }
  if (clean) loss_clean(a, n, r.t >= 0, clean);
}

// p, and g of a row's entry
__device__ __forceinline__ float loss_p(const RowConst& r, float z, float c) { return row_ex2(fminf(fmaf(z - r.m, c, -r.l), 0.f)); }

// Few users: g from logits that lie in L2, with the loss, the users' vectors and db, in one launch.  A block takes 128 columns, four a lane,
// its warps the rows in turn; of the first piece it also takes the rows of its own number's residue.
struct FewArgs {
  const float* z;                // [N, ldz]
  int64_t ldz;
  const float* logp;
  const float2* stats;
  int32_t first, cols;
  bf16* g;                       // [planes, N, ldg]
  int64_t ldg, plane;
  bf16* clean;                   // or null
  int32_t* status;
};
template <int PLANES> __global__ void __launch_bounds__(256) loss_few_kernel(const ScoreLoss a, const FewArgs f) {
  if (!chain_begin()) return;
  __shared__ float4 sums[8][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * 128 + 4 * lane;
  if (f.first == 0)
    for (int64_t n = blockIdx.x + (int64_t)warp * gridDim.x; n < a.N; n += 8 * (int64_t)gridDim.x) {
      if (lane == 0) a.loss[n] = loss_of(a, f.logp, n, f.status);
      if (f.clean) loss_clean(a, n, loss_row(a, f.logp, f.stats, n).t >= 0, f.clean);
    }
  const float c = a.scale * kLog2e;
  float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
  if (col < f.cols) {
#pragma unroll 4
    for (int64_t n = warp; n < a.N; n += 8) {
      const float4 z = *reinterpret_cast<const float4*>(f.z + n * f.ldz + f.first + col);
      const RowConst r = loss_row(a, f.logp, f.stats, n);
      float g[4] = {loss_p(r, z.x, c), loss_p(r, z.y, c), loss_p(r, z.z, c), loss_p(r, z.w, c)};
      const int hot = r.t - f.first - col;
#pragma unroll
      for (int j = 0; j < 4; ++j) g[j] = r.t < 0 ? 0.f : r.f * (j == hot ? g[j] - 1.f : g[j]);
      const uint2 h = make_uint2(pack_bf16x2(g[0], g[1]), pack_bf16x2(g[2], g[3]));
      bf16* to = f.g + n * f.ldg + col;
      *reinterpret_cast<uint2*>(to) = h;
      if constexpr (PLANES == 2) {
        const float2 u = unpack_bf16x2(h.x), v = unpack_bf16x2(h.y);
        *reinterpret_cast<uint2*>(to + f.plane) = make_uint2(pack_bf16x2(g[0] - u.x, g[1] - u.y), pack_bf16x2(g[2] - v.x, g[3] - v.y));
      }
      sum.x += g[0]; sum.y += g[1]; sum.z += g[2]; sum.w += g[3];
    }
  }
  if (!a.dbias) return;
  sums[warp][lane] = sum;
  __syncthreads();
  if (warp != 0) return;
#pragma unroll
  for (int i = 1; i < 8; ++i) {
    const float4 x = sums[i][lane];
    sum.x += x.x; sum.y += x.y; sum.z += x.z; sum.w += x.w;
  }
  float* to = a.dbias + f.first + col;
  if (col < f.cols) to[0] = sum.x;
  if (col + 1 < f.cols) to[1] = sum.y;
  if (col + 2 < f.cols) to[2] = sum.z;
  if (col + 3 < f.cols) to[3] = sum.w;
}

// ============================================================================================
// g of a piece
// ============================================================================================
constexpr int LG_STAGES = 6, LG_EPI_WARPS = 16, LG_PARTS = LG_EPI_WARPS / 4;
constexpr int LG_BIAS_BYTES = LG_EPI_WARPS * 64 * 4;    // a warp's columns
using GradPipe = PairPipe<LG_STAGES, LG_EPI_WARPS, LG_BIAS_BYTES>;

struct GradArgs {
  const RowConst* rows;
  const float* bias;             // [V] or null
  int64_t N;
  int32_t V, first, cols;        // of the table; the piece's first item and its columns (a multiple of 256, or up to the table's end)
  int32_t num_kb, tiles_m, total, width;
  int32_t box_rows;              // users of a copy
  float c;
  bf16* g;                       // [planes, N, ldg]
  int64_t ldg, plane;            // elements between rows (a multiple of 256) and between planes
  float* bias_part;              // [32-row blocks, ldg] or null
  int32_t give_up;
  int32_t* status;
};

// the sum of column l of a 32 x 32 block whose rows the lanes hold, in lane l: halves of the columns are exchanged in turn
__device__ __forceinline__ float column_sums(float (&v)[32]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const bool high = lane & o;
#pragma unroll
    for (int i = 0; i < o; ++i) {
      const float keep = high ? v[i + o] : v[i], give = high ? v[i] : v[i + o];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
    }
  }
  return v[0];
}
__device__ __forceinline__ void st32(void* p, const uint32_t* v) {        // 32 bytes, 32-byte aligned
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]),
               "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}

template <int PLANES>
__global__ void __launch_bounds__(GradPipe::THREADS, 1) loss_grad_kernel(const __grid_constant__ CUtensorMap users, const __grid_constant__ CUtensorMap items,
                                                                         const __grid_constant__ GradArgs a) {
  extern __shared__ uint8_t smem_raw[];
  GradPipe pipe;
  const bool go = pipe.open(smem_raw);
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  bool failed = false;
  if (pipe.warp == 0 && go) {
    // ------------------------------ copies (both blocks) ------------------------------
    int s = 0, tile = 0;
    uint32_t ph = 0;
    for (int t = pair; t < a.total && !failed; t += pairs, ++tile) {
      if (tile == a.give_up) { failed = true; break; }
      const int m0 = (t % a.tiles_m) * 2 * PAIR_ROWS + (int)pipe.rank * PAIR_ROWS;
      const int n0 = a.first + (t / a.tiles_m) * a.width + (int)pipe.rank * (a.width / 2);
      const bool some = m0 < a.N;                       // what the rows of users past the last hold is not looked at
      const uint32_t bytes = (some ? (uint32_t)a.box_rows * 128u : 0u) + (uint32_t)a.width * 64u;
      for (int kb = 0; kb < a.num_kb; ++kb) {
        if (!mbar_wait_warp(pipe.empty(s), ph ^ 1u, pipe.abort_flag)) { failed = true; break; }
        const uint32_t bar = pipe.lead_full(s);
        if (elect_one()) {
          mbar_arrive_expect_tx_remote(bar, bytes);
          if (some) tma_load_2d_pair(pipe.a_of(s), &users, kb * 64, m0, bar);
          tma_load_2d_pair(pipe.b_of(s), &items, kb * 64, n0, bar);
          if (a.width == PAIR_COLS) tma_load_2d_pair(pipe.b_of(s) + PAIR_BOX, &items, kb * 64, n0 + 64, bar);
        }
        __syncwarp();
        if (++s == LG_STAGES) { s = 0; ph ^= 1u; }
      }
    }
  } else if (pipe.warp == 1 && go) {
    // ------------------------------ products (leader) ------------------------------
    if (pipe.rank == 0) {
      const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(a.width >> 3) << 17) | ((uint32_t)(2 * PAIR_ROWS >> 4) << 24);
      const uint64_t da0 = make_desc(pipe.a_of(0), 16, 1024), db0 = make_desc(pipe.b_of(0), 16, 1024);
      int s = 0;
      uint32_t ph = 0, it = 0;
      for (int t = pair; t < a.total && !failed; t += pairs, ++it) {
        const int buf = (int)(it & 1);
        if (!mbar_wait_warp(pipe.tempty(buf), ((it >> 1) & 1) ^ 1u, pipe.abort_flag)) { failed = true; break; }
        tc_fence_after();
        const uint32_t tmem_d = pipe.tmem + (uint32_t)(buf * PAIR_COLS);
        for (int kb = 0; kb < a.num_kb; ++kb) {
          if (!mbar_wait_warp(pipe.full(s), ph, pipe.abort_flag)) { failed = true; break; }
          tc_fence_after();
          const uint32_t soff = (uint32_t)(s * (GradPipe::STAGE >> 4));
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
              tc_mma_pair(tmem_d, da0 + soff + (uint64_t)(k * 2), db0 + soff + (uint64_t)(k * 2), idesc, (kb > 0 || k > 0) ? 1u : 0u);
            tc_commit_pair(pipe.empty(s));
            if (kb == a.num_kb - 1) tc_commit_pair(pipe.tfull(buf));
          }
          __syncwarp();
          if (++s == LG_STAGES) { s = 0; ph ^= 1u; }
        }
      }
    }
  } else if (go) {
    // ------------------------------ g (both blocks) ------------------------------
    const int lane = pipe.lane, q = pipe.warp & 3, part = (pipe.warp - 2) >> 2;
    float* bias_w = reinterpret_cast<float*>(pipe.extra) + (pipe.warp - 2) * 64;
    const int blocks = a.width / PAIR_ROWS;             // of 32 columns of this warp
    uint32_t it = 0;
    for (int t = pair; t < a.total && !failed; t += pairs, ++it) {
      const int buf = (int)(it & 1);
      const int col_t = part * blocks * 32, col0 = (t / a.tiles_m) * a.width + col_t;      // of the tile, of the piece
      const int64_t n = (int64_t)(t % a.tiles_m) * 2 * PAIR_ROWS + (int)pipe.rank * PAIR_ROWS + q * 32 + lane;
      const bool active = n - lane < a.N;               // of the warp
      RowConst r{0.f, 0.f, 0.f, -1};
      const float* bias = nullptr;
      if (active) {
        if (n < a.N) {
          const float4 f = __ldg(reinterpret_cast<const float4*>(a.rows) + n);
          r = RowConst{f.x, f.y, f.z, __float_as_int(f.w)};
        }
        if (a.bias || a.first + col0 + blocks * 32 > a.V) {        // columns past the table count as masked out
          __syncwarp();
          for (int b = 0; b < blocks; ++b) {
            const int v = a.first + col0 + b * 32 + lane;
            bias_w[b * 32 + lane] = v >= a.V ? ROW_NEG_INF : a.bias ? __ldg(a.bias + v) : 0.f;
          }
          __syncwarp();
          bias = bias_w;
        }
      }
      const int hot = r.t - a.first - col0;             // the target's place among the warp's columns
      if (!mbar_wait_warp(pipe.tfull(buf), (it >> 1) & 1, pipe.abort_flag)) { failed = true; break; }
      tc_fence_after();
      if (active) {
        const uint32_t taddr = pipe.tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(buf * PAIR_COLS + col_t);
        for (int b = 0; b < blocks; ++b) {
          uint32_t v[32];
          tc_ld32_issue(taddr + b * 32, v);
          tc_ld32_wait(v);
          float g[32];
#pragma unroll
          for (int j = 0; j < 32; ++j) {
            float z = __uint_as_float(v[j]);
            if (bias) z += bias[b * 32 + j];
            g[j] = loss_p(r, z, a.c);
          }
          if (r.t >= 0 && (unsigned)(hot - b * 32) < 32u) {
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (j == hot - b * 32) g[j] -= 1.f;
          }
#pragma unroll
          for (int j = 0; j < 32; ++j) g[j] = r.t >= 0 ? g[j] * r.f : 0.f;
          if (n < a.N) {
            bf16* to = a.g + n * a.ldg + col0 + b * 32;
            uint32_t h[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) h[j] = pack_bf16x2(g[2 * j], g[2 * j + 1]);
            st32(to, h);
            st32(to + 16, h + 8);
            if constexpr (PLANES == 2) {
#pragma unroll
              for (int j = 0; j < 16; ++j) {
                const float2 f = unpack_bf16x2(h[j]);
                h[j] = pack_bf16x2(g[2 * j] - f.x, g[2 * j + 1] - f.y);
              }
              st32(to + a.plane, h);
              st32(to + a.plane + 16, h + 8);
            }
          }
          if (a.bias_part) a.bias_part[(n >> 5) * a.ldg + col0 + b * 32 + lane] = column_sums(g);
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_remote(pipe.lead_tempty(buf));
    }
  }
  pipe.close(failed, a.status);
}

// db of a piece: the sum of its 32-row blocks, eight groups of them side by side
__global__ void __launch_bounds__(256) loss_bias_kernel(const float* part, int64_t ldg, int32_t blocks, int32_t cols, float* dbias) {
  if (!chain_begin()) return;
  __shared__ float sums[8][32];
  const int lane = threadIdx.x & 31, group = threadIdx.x >> 5, v = blockIdx.x * 32 + lane;
  float s = 0.f;
  for (int i = group; i < blocks; i += 8) s += part[i * ldg + v];          // the rows reach past the last column
  sums[group][lane] = s;
  __syncthreads();
  if (group != 0 || v >= cols) return;
#pragma unroll
  for (int i = 1; i < 8; ++i) s += sums[i][lane];
  dbias[v] = s;
}

// ============================================================================================
// both products of a piece's g
// ============================================================================================
// PLANES: bf16 that g is the sum of; a stage holds all of them beside one piece of the vectors.  CHAINED: the sum of a unit comes as several
// accumulators, which eight warps add up in registers; else sixteen warps take one.
template <int PLANES, bool CHAINED> using ProdPipe = PairPipe<PLANES == 2 ? 4 : 6, CHAINED ? 8 : 16, 0, PLANES>;

// Blocks of 64 whose products (of both planes) are added up in one accumulator for fp32 gradients.  bf16 results hide the error of any length.
constexpr int LP_CHAIN = 24;

struct ProdArgs {
  int64_t N;
  int32_t cols, first, d;        // the piece's columns, its first item
  int32_t tiles_n;               // tiles of 256 columns of d
  int32_t items_m;               // tiles of 256 items (0: dI is not asked)
  int32_t users_m, splits;       // tiles of 256 users (0: dU is not asked); parts of the piece's items that a unit of dU sums over
  int32_t kb_users, kb_items, kb_split;      // blocks of 64 users, of 64 items, of a part's items
  int32_t units_u, total, users_first;       // units of dU, of both; whether those of dU are the heavier ones, which are dealt first
  int32_t extra;                 // lighter units that a pair gets for each heavier one that others have more
  int32_t chain;                 // blocks that are added up in one accumulator
  void* dI;                      // rows of the piece's items
  int64_t ld_dI;
  void* dU;                      // direct: the result; else fp32 [splits, N, d]
  int64_t ld_dU;
  int32_t direct, add;           // add: to what is there (not direct)
  int32_t wide_I, wide_U;        // rows begin on 32 bytes
  int32_t give_up;
  int32_t* status;
};

// Which units a pair takes, its i-th: the heavier ones are dealt first; pairs that get one less take `extra` lighter ones instead; the rest is dealt
// from the pairs with less on.  (The same in loss_span.)
struct ProdWalk {
  int pair, pairs, heavy, mine, extra, other, base, at, total;
  __device__ __forceinline__ explicit ProdWalk(const ProdArgs& a) : pair(blockIdx.x >> 1), pairs(gridDim.x >> 1), total(a.total) {
    heavy = a.users_first ? a.units_u : a.total - a.units_u;
    const int more = heavy % pairs;                     // pairs with one more
    mine = heavy / pairs + (pair < more);
    other = pairs - more;
    extra = pair < more ? 0 : a.extra;
    base = heavy + a.extra * other;
    at = pair < more ? pair + other : pair - more;
  }
  __device__ __forceinline__ int operator()(int i) const {
    if (i < mine) return pair + i * pairs;
    i -= mine;
    if (i < extra) return heavy + i * other + (pairs - other > pair ? 0 : pair - (pairs - other));
    return base + at + (i - extra) * pairs;
  }
};

// A unit: a tile of dI over all users, or a tile of dU over a part of the piece's items.
struct ProdUnit {
  bool users;
  int m0, n0, width, split, k0, blocks;      // first row and column; the sum's range in blocks of 64
  __device__ __forceinline__ ProdUnit(const ProdArgs& a, int t) {
    users = a.users_first ? t < a.units_u : t >= a.total - a.units_u;
    if (a.users_first ? !users : users) t -= a.users_first ? a.units_u : a.total - a.units_u;
    const int tn = t % a.tiles_n, r = t / a.tiles_n;
    n0 = tn * PAIR_COLS;
    width = a.d - n0 > PAIR_COLS / 2 ? PAIR_COLS : PAIR_COLS / 2;
    if (users) {
      split = r / a.users_m;
      m0 = (r - split * a.users_m) * 2 * PAIR_ROWS;
      k0 = split * a.kb_split;
      blocks = min(a.kb_split, a.kb_items - k0);
    } else {
      split = 0;
      m0 = r * 2 * PAIR_ROWS;
      k0 = 0;
      blocks = a.kb_users;
    }
  }
};

// 32 columns of one row, `some` of them there (a multiple of 8)
__device__ __forceinline__ void put_row(float* p, const float (&x)[32], int some, bool wide, bool add) {
#pragma unroll
  for (int j = 0; j < 32; j += 8) {
    if (j >= some) break;
    float4 u = make_float4(x[j], x[j + 1], x[j + 2], x[j + 3]), v = make_float4(x[j + 4], x[j + 5], x[j + 6], x[j + 7]);
    float4* q = reinterpret_cast<float4*>(p + j);
    if (add) {
      const float4 a = q[0], b = q[1];
      u.x += a.x; u.y += a.y; u.z += a.z; u.w += a.w;
      v.x += b.x; v.y += b.y; v.z += b.z; v.w += b.w;
    }
    if (wide) {
      const uint32_t h[8] = {__float_as_uint(u.x), __float_as_uint(u.y), __float_as_uint(u.z), __float_as_uint(u.w),
                             __float_as_uint(v.x), __float_as_uint(v.y), __float_as_uint(v.z), __float_as_uint(v.w)};
      st32(p + j, h);
    } else {
      q[0] = u;
      q[1] = v;
    }
  }
}
__device__ __forceinline__ void put_row(bf16* p, const float (&x)[32], int some, bool wide, bool) {
#pragma unroll
  for (int j = 0; j < 32; j += 16) {
    uint32_t h[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = pack_bf16x2(x[j + 2 * i], x[j + 2 * i + 1]);
    if (wide && j + 16 <= some) {
      st32(p + j, h);
    } else {
      uint4* q = reinterpret_cast<uint4*>(p + j);
      if (j < some) q[0] = make_uint4(h[0], h[1], h[2], h[3]);
      if (j + 8 < some) q[1] = make_uint4(h[4], h[5], h[6], h[7]);
    }
  }
}

template <typename GT, bool CHAINED>
__global__ void __launch_bounds__(ProdPipe<sizeof(GT) / 2, CHAINED>::THREADS, 1)
    loss_products_kernel(const __grid_constant__ CUtensorMap g0, const __grid_constant__ CUtensorMap g1, const __grid_constant__ CUtensorMap users,
                         const __grid_constant__ CUtensorMap items, const __grid_constant__ ProdArgs a) {
  constexpr int PLANES = sizeof(GT) / 2;
  using Pipe = ProdPipe<PLANES, CHAINED>;
  extern __shared__ uint8_t smem_raw[];
  Pipe pipe;
  const bool go = pipe.open(smem_raw);
  const ProdWalk walk(a);
  bool failed = false;
  if (pipe.warp == 0 && go) {
    // ------------------------------ copies (both blocks): two boxes of 64 x 64 of each plane of g, one or two of the vectors ------------------------------
    int s = 0;
    uint32_t ph = 0;
    for (int tile = 0, t; (t = walk(tile)) < a.total && !failed; ++tile) {
      if (tile == a.give_up) { failed = true; break; }
      const ProdUnit u(a, t);
      const int m0 = u.m0 + (int)pipe.rank * PAIR_ROWS, n0 = u.n0 + (int)pipe.rank * (u.width / 2);
      const uint32_t bytes = PLANES * 2 * PAIR_BOX + (uint32_t)(u.width / PAIR_ROWS) * PAIR_BOX;
      const CUtensorMap* vectors = u.users ? &items : &users;
      for (int kb = 0; kb < u.blocks; ++kb) {
        const int k = (u.k0 + kb) * 64, row = (u.users ? a.first : 0) + k;
        if (!mbar_wait_warp(pipe.empty(s), ph ^ 1u, pipe.abort_flag)) { failed = true; break; }
        const uint32_t bar = pipe.lead_full(s), sb = pipe.b_of(s);
        if (elect_one()) {
          mbar_arrive_expect_tx_remote(bar, bytes);
#pragma unroll
          for (int i = 0; i < PLANES; ++i) {
            const CUtensorMap* g = i ? &g1 : &g0;
            const uint32_t sa = pipe.a_of(s, i);
            tma_load_2d_pair(sa, g, u.users ? k : m0, u.users ? m0 : k, bar);
            tma_load_2d_pair(sa + PAIR_BOX, g, u.users ? k : m0 + 64, u.users ? m0 + 64 : k, bar);
          }
          tma_load_2d_pair(sb, vectors, n0, row, bar);
          if (u.width == PAIR_COLS) tma_load_2d_pair(sb + PAIR_BOX, vectors, n0 + 64, row, bar);
        }
        __syncwarp();
        if (++s == Pipe::STAGES) { s = 0; ph ^= 1u; }
      }
    }
  } else if (pipe.warp == 1 && go) {
    // ------------------------------ products (leader) ------------------------------
    if (pipe.rank == 0) {
      // the vectors lie with their columns side by side; so does g where items are the rows of the result
      constexpr uint32_t idesc0 = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(2 * PAIR_ROWS >> 4) << 24);
      const uint64_t da_k = make_desc(pipe.a_of(0), 16, 1024), da_mn = make_desc(pipe.a_of(0), PAIR_BOX, 1024);
      const uint64_t db0 = make_desc(pipe.b_of(0), PAIR_BOX, 1024);
      int s = 0;
      uint32_t ph = 0, it = 0;
      for (int tile = 0, t; (t = walk(tile)) < a.total && !failed; ++tile) {
        const ProdUnit u(a, t);
        const uint32_t idesc = idesc0 | (u.users ? 0u : 1u << 15) | ((uint32_t)(u.width >> 3) << 17);
        const uint64_t da0 = u.users ? da_k : da_mn;
        const uint32_t step_a = (u.users ? 32u : 2048u) >> 4;
        const int chain = CHAINED ? a.chain : u.blocks;
        for (int c0 = 0; c0 < u.blocks && !failed; c0 += chain, ++it) {            // an accumulator each
          const int c1 = min(c0 + chain, u.blocks), buf = (int)(it & 1);
          if (!mbar_wait_warp(pipe.tempty(buf), ((it >> 1) & 1) ^ 1u, pipe.abort_flag)) { failed = true; break; }
          tc_fence_after();
          const uint32_t tmem_d = pipe.tmem + (uint32_t)(buf * PAIR_COLS);
          for (int kb = c0; kb < c1; ++kb) {
            if (!mbar_wait_warp(pipe.full(s), ph, pipe.abort_flag)) { failed = true; break; }
            tc_fence_after();
            const uint32_t soff = (uint32_t)(s * (Pipe::STAGE >> 4));
            if (elect_one()) {
#pragma unroll
              for (uint32_t i = 0; i < PLANES; ++i)
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k)
                  tc_mma_pair(tmem_d, da0 + soff + i * (PAIR_OPERAND >> 4) + k * step_a, db0 + soff + k * (2048u >> 4), idesc,
                              (kb > c0 || k > 0 || i > 0) ? 1u : 0u);
              tc_commit_pair(pipe.empty(s));
              if (kb == c1 - 1) tc_commit_pair(pipe.tfull(buf));
            }
            __syncwarp();
            if (++s == Pipe::STAGES) { s = 0; ph ^= 1u; }
          }
        }
      }
    }
  } else if (go) {
    // ------------------------------ results (both blocks): a row and a part of the columns a thread ------------------------------
    constexpr int PARTS = Pipe::EPI_WARPS / 4;
    const int lane = pipe.lane, q = pipe.warp & 3, part = (pipe.warp - 2) >> 2;
    const uint32_t lane_addr = pipe.tmem + ((uint32_t)(q * 32) << 16);
    uint32_t it = 0;
    for (int tile = 0, t; (t = walk(tile)) < a.total && !failed; ++tile) {
      const ProdUnit u(a, t);
      const int64_t m = u.m0 + (int)pipe.rank * PAIR_ROWS + q * 32 + lane;
      const int blocks = u.width / 32 / PARTS, col = part * blocks * 32;                // of 32 columns
      const bool there = m < (u.users ? a.N : (int64_t)a.cols);
      auto put = [&](int b, const float (&x)[32]) {
        const int n = u.n0 + col + b * 32, some = a.d - n;
        if (!there || some <= 0) return;
        if (!u.users) put_row(reinterpret_cast<GT*>(a.dI) + m * a.ld_dI + n, x, some, a.wide_I, false);
        else if (a.direct) put_row(reinterpret_cast<GT*>(a.dU) + m * a.ld_dU + n, x, some, a.wide_U, false);
        else put_row(reinterpret_cast<float*>(a.dU) + ((int64_t)u.split * a.N + m) * a.d + n, x, some, a.wide_U, a.add);
      };
      if constexpr (CHAINED) {
        // The tensor cores cut off where this adds with rounding: a chain's length sets the sum's precision.
        float acc[4][32];
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
          for (int j = 0; j < 32; ++j) acc[b][j] = 0.f;
#pragma unroll 1
        for (int c0 = 0; c0 < u.blocks; c0 += a.chain, ++it) {
          const int buf = (int)(it & 1);
          if (!mbar_wait_warp(pipe.tfull(buf), (it >> 1) & 1, pipe.abort_flag)) { failed = true; break; }
          tc_fence_after();
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            if (b >= blocks) break;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              uint32_t v[16];
              tc_ld16(lane_addr + (uint32_t)(buf * PAIR_COLS + col + b * 32 + h * 16), v);
#pragma unroll
              for (int j = 0; j < 16; ++j) acc[b][h * 16 + j] += __uint_as_float(v[j]);
            }
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_remote(pipe.lead_tempty(buf));
        }
        if (failed) break;
#pragma unroll
        for (int b = 0; b < 4; ++b)
          if (b < blocks) put(b, acc[b]);
      } else {
        const int buf = (int)(it & 1);
        if (!mbar_wait_warp(pipe.tfull(buf), (it >> 1) & 1, pipe.abort_flag)) { failed = true; break; }
        tc_fence_after();
        for (int b = 0; b < blocks; ++b) {
          uint32_t v[32];
          tc_ld32_issue(lane_addr + (uint32_t)(buf * PAIR_COLS + col + b * 32), v);
          tc_ld32_wait(v);
          float x[32];
#pragma unroll
          for (int j = 0; j < 32; ++j) x[j] = __uint_as_float(v[j]);
          put(b, x);
          __syncwarp();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_remote(pipe.lead_tempty(buf));
        ++it;
      }
      __syncwarp();
    }
  }
  pipe.close(failed, a.status);
}

// dU as the sum of its parts
template <typename GT> __global__ void __launch_bounds__(256) loss_finish_kernel(const float* parts, int splits, int64_t N, int32_t d, GT* dU, int64_t ld) {
  if (!chain_begin()) return;
  const int64_t n4 = N * (d / 4);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n4; i += (int64_t)gridDim.x * 256) {
    float4 s = reinterpret_cast<const float4*>(parts)[i];
#pragma unroll 4
    for (int k = 1; k < splits; ++k) {
      const float4 x = reinterpret_cast<const float4*>(parts)[k * n4 + i];
      s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
    }
    const int64_t n = i / (d / 4);
    GT* to = dU + n * ld + 4 * (i - n * (d / 4));
    if constexpr (sizeof(GT) == 4) *reinterpret_cast<float4*>(to) = s;
    else *reinterpret_cast<uint2*>(to) = make_uint2(pack_bf16x2(s.x, s.y), pack_bf16x2(s.z, s.w));
  }
}

// ============================================================================================
// host side
// ============================================================================================
size_t up(size_t n) { return (n + 255) / 256 * 256; }

struct LossPlan {
  size_t logp, stats, rows, clean, parts, bias, g, bytes;       // places in the workspace
  int32_t cols, splits;                                         // of a piece; parts of dU
  int64_t ldg;
};

// How the units of a piece's products are dealt to the pairs (ProdWalk), and the blocks of 64 that the busiest one works through.
struct LossSpan {
  int64_t most;
  int32_t extra;
};
LossSpan loss_span(int64_t units_u, int64_t cost_u, int64_t units_i, int64_t cost_i) {
  const bool users_first = cost_u >= cost_i;
  const int64_t n1 = users_first ? units_u : units_i, c1 = users_first ? cost_u : cost_i, n2 = users_first ? units_i : units_u;
  const int64_t c2 = users_first ? cost_i : cost_u, pairs = n1 + n2 < kPairs ? n1 + n2 : kPairs;
  const int64_t more = n1 % pairs, other = pairs - more;
  int64_t extra = more ? c1 / c2 : 0;                   // rounded down: those pairs are dealt to first
  if (extra > n2 / other) extra = n2 / other;
  const int64_t rest = n2 - extra * other;
  const int64_t load_other = (n1 / pairs) * c1 + (extra + rest / pairs + (rest % pairs > 0)) * c2;
  const int64_t load_more = more ? (n1 / pairs + 1) * c1 + (rest / pairs + (rest % pairs > other)) * c2 : 0;
  return LossSpan{load_other > load_more ? load_other : load_more, (int32_t)extra};
}

// Parts that the sums of dU over a piece's items are cut into, so that the pairs are evenly busy.  A part costs its place in the sum: 8 N d
// bytes, in blocks of 64 of a pair (0.37 us for each bf16 of g).
int loss_splits(int64_t N, int32_t cols, int32_t d, int planes, bool users, bool items) {
  if (!users) return 0;
  const int64_t tiles_n = ceil_div(d, PAIR_COLS), kb_items = ceil_div(cols, 64), kb_users = ceil_div64(N, 64);
  const int64_t units_i = items ? ceil_div(cols, PAIR_COLS) * tiles_n : 0, tiles_u = ceil_div64(N, PAIR_COLS) * tiles_n;
  const double part = 8.0 * N * d / (5e6 * 0.37 * planes);
  int best = 1;
  double least = 1e300;
  for (int s = 1; s <= 32 && s * 4 <= (kb_items > 4 ? kb_items : 4); ++s) {
    const int64_t cost = ceil_div64(kb_items, s), parts = ceil_div64(kb_items, cost);
    const double time = (double)loss_span(tiles_u * parts, cost, units_i, kb_users).most + (parts > 1 ? parts * part : 0.0);
    if (time < least) { least = time; best = (int)parts; }
  }
  return best;
}

// Lays out a workspace of `room` bytes (0: of `cols` columns a piece).
LossPlan loss_plan(int64_t N, int32_t V, int32_t d, int planes, bool users, bool items, bool bias, int32_t cols, size_t room) {
  LossPlan p = {};
  const int32_t all = (int32_t)(((int64_t)V + 255) / 256 * 256 < INT32_MAX / 256 * 256 ? ((int64_t)V + 255) / 256 * 256 : INT32_MAX / 256 * 256);
  auto place = [&](int32_t c, int splits) {
    size_t at = 0;
    auto take = [&](size_t n) { const size_t was = at; at += up(n); return was; };
    p.logp = take((size_t)N * 4);
    p.stats = take((size_t)N * 8);
    p.rows = take((size_t)N * sizeof(RowConst));
    p.clean = take(items ? (size_t)N * d * 2 : 0);
    p.parts = take((size_t)splits * N * d * 4);
    p.bias = take(bias ? (size_t)ceil_div64(N, 32) * c * 4 : 0);
    p.g = take((size_t)planes * N * c * 2);
    p.bytes = at;
    p.cols = c;
    p.ldg = c;
    p.splits = splits;
  };
  auto with = [&](int32_t c) {
    const int32_t kb_items = ceil_div(c < V ? c : V, 64);
    int s = loss_splits(N, c < V ? c : V, d, planes, users, items);
    place(c, s);
    while (room && p.bytes > room && s > 1) place(c, s = ceil_div(kb_items, ceil_div(kb_items, s - 1)));      // as many as are not empty
  };
  if (!room) {
    with(cols < all ? cols : all);
    return p;
  }
  const size_t per = (size_t)planes * N * 2 + (bias ? (size_t)ceil_div64(N, 32) * 4 : 0);
  place(0, 0);
  int64_t c = room > p.bytes ? (int64_t)((room - p.bytes) / per) / 256 * 256 : 0;
  if (c > all) c = all;
  if (c < 256) c = 256;
  // pieces of about equal size
  const int64_t pieces = ceil_div64(V, c);
  c = ceil_div64(ceil_div64(V, pieces), 256) * 256;
  with((int32_t)c);
  while (p.bytes > room && p.cols > 256) with(p.cols - 256);
  return p;
}

constexpr int64_t kGoodG = (int64_t)192 << 20;            // bytes of a piece's g

}  // namespace

void score_loss_workspace(int64_t N, int32_t V, int32_t d, int grad_dtype, size_t* least, size_t* best) {
  const int planes = grad_dtype == GRAM_F32 ? 2 : 1;
  const int64_t n = N > 0 ? N : 1;
  LossPlan p = loss_plan(n, V, d, planes, true, true, true, 256, 0);
  // the least: one part of dU
  const size_t parts = up((size_t)p.splits * n * d * 4), one = up((size_t)n * d * 4);
  *least = p.bytes - parts + one;
  int64_t cols = kGoodG / (2 * planes * n) / 256 * 256;
  if (cols < 256) cols = 256;
  if (cols > INT32_MAX / 2) cols = INT32_MAX / 2 / 256 * 256;
  p = loss_plan(n, V, d, planes, true, true, true, (int32_t)cols, 0);
  *best = p.bytes > *least ? p.bytes : *least;
}

gram_status score_loss_launch(gram_ctx* ctx, const ScoreLoss& a, void* ws, size_t ws_bytes, void* score_ws, size_t score_ws_bytes, cudaStream_t st) {
  const bool grads = a.dusers || a.ditems || a.dbias;
  const int planes = a.grad_dtype == GRAM_F32 ? 2 : 1;
  LossPlan p = loss_plan(a.N, a.V, a.d, planes, a.dusers != nullptr, a.ditems != nullptr, a.dbias != nullptr, 0, ws_bytes ? ws_bytes : 1);
  const size_t need = grads ? p.bytes : p.rows;
  if (need > ws_bytes)
    return gram_set_error(ctx, "gram_score_loss: a workspace of %zu bytes is needed, not %zu", need, ws_bytes), GRAM_ERR_WORKSPACE;
  uint8_t* base = (uint8_t*)ws;
  float* logp = (float*)(base + p.logp);
  float2* stats = (float2*)(base + p.stats);
  RowAnswers ask;
  ask.targets = a.targets;
  ask.logp = logp;
  ask.stats = (float*)stats;
  ask.C = 1;
  RowConst* rows = grads ? (RowConst*)(base + p.rows) : nullptr;
  bf16* clean = a.ditems ? (bf16*)(base + p.clean) : nullptr;
  // Few logits stay in the context's workspace, out of L2, in place of a second product for each piece.
  const int64_t ldz = ((int64_t)a.V + 7) / 8 * 8;
  const bool few = grads && a.N <= LOSS_FEW && (size_t)a.N * ldz * sizeof(float) <= (score_ws_bytes < (32u << 20) ? score_ws_bytes : 32u << 20);
  if (few) {
    GRAM_TRY(score_logits_launch(ctx, a.users, a.ld_users, a.items, a.ld_items, a.bias, a.N, a.V, a.d, (float*)score_ws, ldz, st));
    GRAM_TRY(logprobs_launch(ctx, score_ws, GRAM_F32, ldz, a.N, a.V, a.scale, ask, st));
  } else {
    GRAM_TRY(score_logprobs_launch(ctx, a.users, a.ld_users, a.items, a.ld_items, a.bias, a.N, a.V, a.d, a.scale, ask, score_ws, score_ws_bytes, st));
    ProfScope prof(ctx, GRAM_K_OTHER, (double)a.N * (32 + (clean ? 4.0 * a.d : 0.0)), 1, st, "loss_rows");
    launch_chain(loss_rows_kernel, dim3((unsigned)ceil_div64(a.N, 8)), 256, 0, st, a, (const float*)logp, (const float2*)stats, rows, clean,
                 gram_status_word(ctx));
    GRAM_LAUNCH_CHECK(ctx);
  }
  if (!grads) return GRAM_OK;

  const char* what = "gram_score_loss: cannot describe the vectors";
  CUtensorMap map_u, map_i, map_clean, map_items, map_g[2];
  int box_rows = PAIR_ROWS;                              // copies are no larger than the users
  while (box_rows > 8 && box_rows / 2 >= a.N) box_rows /= 2;
  if (!make_map(&map_u, a.users, (uint64_t)a.d, (uint64_t)a.N, (uint64_t)a.ld_users, 64, (uint32_t)box_rows) ||
      !make_map(&map_i, a.items, (uint64_t)a.d, (uint64_t)a.V, (uint64_t)a.ld_items, 64, 64))
    return gram_set_error(ctx, what), GRAM_ERR_UNSUPPORTED;
  map_items = map_i;
  map_clean = map_i;
  if (clean && !make_map(&map_clean, clean, (uint64_t)a.d, (uint64_t)a.N, (uint64_t)a.d, 64, 64)) return gram_set_error(ctx, what), GRAM_ERR_UNSUPPORTED;

  bf16* g = (bf16*)(base + p.g);
  const int64_t plane = a.N * p.ldg;
  const int32_t pieces = ceil_div(a.V, p.cols);
  for (int32_t piece = 0; piece < pieces; ++piece) {
    const int32_t first = piece * p.cols, cols = a.V - first < p.cols ? a.V - first : p.cols;
    if (few) {
      const FewArgs e{(const float*)score_ws, ldz, logp, stats, first, cols, g, p.ldg, plane, clean, gram_status_word(ctx)};
      ProfScope prof(ctx, GRAM_K_OTHER, (4.0 + 2 * planes) * a.N * cols, 1, st, "loss_few");
      launch_chain(planes == 2 ? loss_few_kernel<2> : loss_few_kernel<1>, dim3((unsigned)ceil_div(cols, 128)), 256, 0, st, a, e);
      GRAM_LAUNCH_CHECK(ctx);
    } else {
      GradArgs e = {};
      e.rows = rows;
      e.bias = a.bias;
      e.N = a.N;
      e.V = a.V;
      e.first = first;
      e.cols = cols;
      e.num_kb = ceil_div(a.d, 64);
      e.tiles_m = (int32_t)ceil_div64(a.N, 2 * PAIR_ROWS);
      e.width = (int64_t)e.tiles_m * ceil_div(cols, PAIR_COLS) < kPairs ? PAIR_COLS / 2 : PAIR_COLS;      // tiles of half the width where they leave pairs idle
      e.total = e.tiles_m * ceil_div(cols, e.width);
      e.box_rows = box_rows;
      e.c = a.scale * kLog2e;
      e.g = g;
      e.ldg = p.ldg;
      e.plane = plane;
      e.bias_part = a.dbias ? (float*)(base + p.bias) : nullptr;
      e.give_up = gram_ring_rows(ctx);
      e.status = gram_status_word(ctx);
      {
        ProfScope prof(ctx, GRAM_K_GEMM, 2.0 * a.N * cols * a.d, 1, st, "loss_grad");
        const int pairs = e.total < kPairs ? e.total : kPairs;
        auto kern = planes == 2 ? loss_grad_kernel<2> : loss_grad_kernel<1>;
        GRAM_CUDA(ctx, launch_pairs(kern, pairs, GradPipe::THREADS, GradPipe::SMEM, st, map_u, map_i, e));
      }
      if (a.dbias) {
        ProfScope prof(ctx, GRAM_K_COLSUM, (double)a.N / 8 * cols, 1, st, "loss_bias");
        launch_chain(loss_bias_kernel, dim3((unsigned)ceil_div(cols, 32)), 256, 0, st, (const float*)e.bias_part, p.ldg, (int32_t)ceil_div64(a.N, 32), cols,
                     a.dbias + first);
        GRAM_LAUNCH_CHECK(ctx);
      }
    }
    if (!a.dusers && !a.ditems) continue;
    for (int i = 0; i < 2; ++i)
      if (!make_map(&map_g[i], g + (i < planes ? i : 0) * plane, (uint64_t)cols, (uint64_t)a.N, (uint64_t)p.ldg, 64, 64))
        return gram_set_error(ctx, what), GRAM_ERR_UNSUPPORTED;
    ProdArgs w = {};
    const size_t size = planes == 2 ? 4 : 2;
    w.N = a.N;
    w.cols = cols;
    w.first = first;
    w.d = a.d;
    w.tiles_n = ceil_div(a.d, PAIR_COLS);
    w.items_m = a.ditems ? ceil_div(cols, 2 * PAIR_ROWS) : 0;
    w.users_m = a.dusers ? (int32_t)ceil_div64(a.N, 2 * PAIR_ROWS) : 0;
    w.kb_users = (int32_t)ceil_div64(a.N, 64);
    w.kb_items = ceil_div(cols, 64);
    w.direct = p.splits == 1 && pieces == 1;
    // the last piece may have fewer parts; the sums of the others stay
    w.kb_split = p.splits ? ceil_div(w.kb_items, p.splits) : 0;
    w.splits = p.splits ? ceil_div(w.kb_items, w.kb_split) : 0;
    w.units_u = w.users_m * w.tiles_n * w.splits;
    w.total = w.units_u + w.items_m * w.tiles_n;
    w.users_first = w.kb_split >= w.kb_users;
    w.extra = loss_span(w.units_u, w.kb_split ? w.kb_split : 1, w.total - w.units_u, w.kb_users).extra;
    w.chain = LP_CHAIN;
    w.dI = a.ditems ? (uint8_t*)a.ditems + (size_t)first * a.ld_ditems * size : nullptr;
    w.ld_dI = a.ld_ditems;
    w.dU = w.direct ? a.dusers : (void*)(base + p.parts);
    w.ld_dU = a.ld_dusers;
    w.add = piece > 0;
    w.wide_I = (uintptr_t)a.ditems % 32 == 0 && a.ld_ditems * size % 32 == 0;
    w.wide_U = w.direct ? (uintptr_t)a.dusers % 32 == 0 && a.ld_dusers * size % 32 == 0 : 1;
    w.give_up = gram_ring_rows(ctx);
    w.status = gram_status_word(ctx);
    ProfScope prof(ctx, GRAM_K_GEMM, 2.0 * planes * a.N * cols * a.d * ((a.dusers != nullptr) + (a.ditems != nullptr)), 1, st, "loss_products");
    const int pairs = w.total < kPairs ? w.total : kPairs;
    const int longest = w.units_u && w.kb_split > w.kb_users ? w.kb_split : w.kb_users;
    auto launch = [&](auto kern, auto pipe) {
      using Pipe = decltype(pipe);
      return launch_pairs(kern, pairs, Pipe::THREADS, Pipe::SMEM, st, map_g[0], map_g[1], map_clean, map_items, w);
    };
    if (planes == 1) GRAM_CUDA(ctx, launch(loss_products_kernel<bf16, false>, ProdPipe<1, false>()));
    else if (longest <= LP_CHAIN) GRAM_CUDA(ctx, launch(loss_products_kernel<float, false>, ProdPipe<2, false>()));
    else GRAM_CUDA(ctx, launch(loss_products_kernel<float, true>, ProdPipe<2, true>()));
  }
  if (a.dusers && !(p.splits == 1 && pieces == 1)) {
    ProfScope prof(ctx, GRAM_K_OTHER, (double)a.N * a.d * 4 * (p.splits + 1), 1, st, "loss_finish");
    const float* parts = (const float*)(base + p.parts);
    int64_t blocks = ceil_div64(a.N * (a.d / 4), 256);
    if (blocks > kNumSMs * 8) blocks = kNumSMs * 8;
    if (planes == 2) launch_chain(loss_finish_kernel<float>, dim3((unsigned)blocks), 256, 0, st, parts, (int)p.splits, a.N, a.d, (float*)a.dusers, a.ld_dusers);
    else launch_chain(loss_finish_kernel<bf16>, dim3((unsigned)blocks), 256, 0, st, parts, (int)p.splits, a.N, a.d, (bf16*)a.dusers, a.ld_dusers);
    GRAM_LAUNCH_CHECK(ctx);
  }
  return GRAM_OK;
}
