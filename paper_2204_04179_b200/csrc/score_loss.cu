// Softmax cross entropy of users against an item table, from the vectors themselves, with its gradients (gram_score_loss).
//
// With z = U I^T + b, p the softmax of scale z and t the rows' targets, loss_n = log sum_v exp(scale z_nv) - scale z_n,t, and the
// gradient of sum_n w_n loss_n with respect to z is g_nv = w_n scale (p_nv - [v = t_n]); then dU = g I, dI = g^T U, db_v = sum_n g_nv.
//
// g has as many entries as the logits, which are not kept but for few users: it is formed for a piece at a time, some of the items and all users, or some of
// the users and all items where users are more.
//   1. The statistics of the rows (m and log s) come from the kernels of gram_score_logprobs: one product.
//   2. loss_rows_kernel: the loss, and what a row's g needs, in one float4.
//   3. Of each piece: loss_grad_kernel forms its logits again on the tensor cores and writes g to the workspace in bf16 (for fp32
//      gradients as the sum of two bf16: 2^-16 of each entry); loss_products_kernel takes both products of it, g I and g^T U, in one launch of tiles
//      of either kind.  Where pieces are of items, those of g^T U are done with the piece and g I is summed over all; else the other way round.
//   4. loss_finish_kernel: the summed gradient from its parts.
// Where users are few and their logits fit 32 MB they are kept in L2 after all, and a kernel of elementwise work takes the place of the second product; up to
// four users' products are taken by lanes, with g in 32 bits.
// Bounded by the tensor cores where users are many: 8 N V d flops (12 with fp32 gradients), of which the products that cannot be done
// without are 6; by the table's bytes, read twice and written once, where they are few.  Measured, vectors of 768: 4096 users against 100 000 items
// 1700 us in a call by itself (1480 TFLOP/s of the 8 N V d) and 2070 in a loop of calls under the power cap (1220); against 30 522 with bias 548 and 675;
// 25 600 users against 10 000 items, fp32 gradients, 1750 and 2070 (12 N V d: 1350 TFLOP/s by itself); 64 users against 100 000 120 in a graph of calls
// (three passes over the table's 154 MB at 3.8 TB/s), one user against 10 000 21.
#include "score_loss.h"

#include "logits.h"
#include "pair_pipe.cuh"
#include "row_softmax.cuh"

namespace {
using namespace tc;

constexpr int kPairs = kNumSMs / 2;
// Users whose logits are kept where 32 MB hold them.  us so and with a second product: 64 users, 100 000 items of 768 128 and 160, 260 and 30 000
// 89 and 94, 512 and 15 000 60 and 69, 600 and 13 000 65 and 67, but 1000 and 8000 68 and 61, 2000 and 4000 of 128 62 and 37: the logits' way out
// and back costs more there than their product.
constexpr int LOSS_FEW = 512, LOSS_FEW_ROWS = 64;
constexpr int LOSS_SHORT = 8 * kPairs;                  // blocks of 64 items x 256 columns whose products take the pairs 2 us for each plane

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

// The entry of a row's target is about -f where all others are small, so that its rounding to bf16 would be that of the whole row of dU (up to 2^-8 of
// it, one way for all columns).  What the rounding left is kept, and that much of the item is added to the row in 32 bits when its parts are joined
// (not where pieces are of users, more than the items).  One user against 10 000 items: up to 0.0039 and now 0.0017 of dU, the result's own rounding; 64 users
// against 100 000 items 118.6 -> 119.6 us, 4096 against 30 522 549 -> 558.
struct RowRest {
  float rest;
  int32_t t;                     // -1: none
};

// Whether a row's target takes part: not where the bias takes it out, or nothing is left.  Its log p alone does not tell: one that leaves 32 bits (a mask of
// the type's lowest value at a scale above 1) is -inf too.
__device__ __forceinline__ bool loss_target(const ScoreLoss& a, int32_t t, float lp, float m) {
  return lp != ROW_NEG_INF || (m != ROW_NEG_INF && !(a.bias && a.bias[t] == ROW_NEG_INF));
}
// A row's statistics, log p of its target and weight.
__device__ __forceinline__ RowConst loss_row(const ScoreLoss& a, const float* logp, const float2* stats, int64_t n) {
  const int32_t t = a.targets[n];
  const float lp = logp[n], w = a.weight ? a.weight[n] : 1.f;
  const float2 s = stats[n];
  const bool part = t >= 0 && t < a.V && w != 0.f && loss_target(a, t, lp, s.x);
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

// A warp a user.  rows, rest, clean: null where they are not needed.
__global__ void __launch_bounds__(256) loss_rows_kernel(const ScoreLoss a, const float* logp, const float2* stats, RowConst* rows, RowRest* rest, bf16* clean,
                                                        int32_t* status) {
  chain_next();
  if (!chain_begin()) return;
  const int64_t n = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (n >= a.N) return;
  const RowConst r = loss_row(a, logp, stats, n);
  if ((threadIdx.x & 31) == 0) {
    a.loss[n] = loss_of(a, logp, n, status);
    if (rows) rows[n] = r;
    if (rest) rest[n] = RowRest{0.f, r.t};
  }
  if (clean) loss_clean(a, n, r.t >= 0, clean);
}

// p, and g of a row's entry
__device__ __forceinline__ float loss_p(const RowConst& r, float z, float c) { return row_ex2(fminf(fmaf(z - r.m, c, -r.l), 0.f)); }

// A piece: users [n0, n0 + rows) and items [first, first + cols), all of them or all of the others.
struct Piece {
  int64_t n0, rows;
  int32_t first, cols;
  bf16* g;                       // [planes, rows, ldg]; none where db alone is asked
  int64_t ldg, plane;            // elements between rows (a multiple of 256) and between planes
};

// PLANES of the kernels that form g: bf16 that it leaves as the sum of; 0: only db's sums leave.
// Few users: g from logits that lie in L2, with the loss, the users' vectors and db, in one launch.  A block takes 128 columns, four a lane,
// and 64 rows, its warps in turn; where the piece is the rows' first, the block also takes those of its own number's residue.
struct FewArgs {
  Piece at;
  const float* z;                // [N, ldz]
  int64_t ldz;
  const float* logp;
  const float2* stats;
  bf16* clean;                   // or null
  RowRest* rest;                 // or null
  float* bias_part;              // [groups of rows, ldg]
  int32_t* status;
};
template <int PLANES> __global__ void __launch_bounds__(256) loss_few_kernel(const ScoreLoss a, const FewArgs f) {
  chain_next();
  if (!chain_begin()) return;
  __shared__ float4 sums[8][32];
  __shared__ RowConst row[LOSS_FEW_ROWS];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * 128 + 4 * lane;
  const Piece& at = f.at;
  const int i0 = (int)blockIdx.y * LOSS_FEW_ROWS, rows = min((int)at.rows, i0 + LOSS_FEW_ROWS);       // of this block
  if (i0 + (int)threadIdx.x < rows) row[threadIdx.x] = loss_row(a, f.logp, f.stats, at.n0 + i0 + threadIdx.x);
  __syncthreads();
  if (at.first == 0)
    for (int i = i0 + blockIdx.x + warp * (int)gridDim.x; i < rows; i += 8 * (int)gridDim.x) {
      if (lane == 0) a.loss[at.n0 + i] = loss_of(a, f.logp, at.n0 + i, f.status);
      if (f.clean) loss_clean(a, at.n0 + i, row[i - i0].t >= 0, f.clean);
      if (f.rest && lane == 0 && row[i - i0].t < 0) f.rest[at.n0 + i] = RowRest{0.f, -1};
    }
  const float c = a.scale * kLog2e;
  float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
  if (col < at.cols) {
    const float* z_at = f.z + at.n0 * f.ldz + at.first + col;
#pragma unroll 8
    for (int i = i0 + warp; i < rows; i += 8) {
      const float4 z = *reinterpret_cast<const float4*>(z_at + i * f.ldz);
      const RowConst r = row[i - i0];
      float g[4] = {loss_p(r, z.x, c), loss_p(r, z.y, c), loss_p(r, z.z, c), loss_p(r, z.w, c)};
      const int hot = r.t - at.first - col;
#pragma unroll
      for (int j = 0; j < 4; ++j) g[j] = r.t < 0 ? 0.f : r.f * (j == hot ? g[j] - 1.f : g[j]);
      sum.x += g[0]; sum.y += g[1]; sum.z += g[2]; sum.w += g[3];
      if constexpr (PLANES == 0) continue;
      bf16* to = at.g + i * at.ldg + col;
#pragma unroll
      for (int k = 0; k < PLANES; ++k) {
        const uint2 h = make_uint2(pack_bf16x2(g[0], g[1]), pack_bf16x2(g[2], g[3]));
        *reinterpret_cast<uint2*>(to + k * at.plane) = h;
        const float2 u = unpack_bf16x2(h.x), v = unpack_bf16x2(h.y);
        g[0] -= u.x; g[1] -= u.y; g[2] -= v.x; g[3] -= v.y;
      }
      if (f.rest && r.t >= 0 && (unsigned)hot < 4u) f.rest[at.n0 + i] = RowRest{hot & 2 ? (hot & 1 ? g[3] : g[2]) : (hot & 1 ? g[1] : g[0]), r.t};
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
  const bool part = gridDim.y > 1;                      // joined by loss_bias_kernel
  float* to = part ? f.bias_part + blockIdx.y * at.ldg + col : a.dbias + at.first + col;
  const float all[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (col + j < at.cols) to[j] = !part && at.n0 > 0 ? to[j] + all[j] : all[j];
}

// Few users and few items, all of g in one piece and db not asked: a block takes a row of logits into registers, with its statistics, the loss,
// the user's vector and g, in place of gram_logprobs' kernel and the one above.
constexpr int LR_THREADS = 512, LR_EACH = 32;           // logits of a thread: rows of up to 16 384
template <int PLANES> __global__ void __launch_bounds__(LR_THREADS) loss_row_kernel(const ScoreLoss a, const FewArgs f) {
  chain_next();
  if (!chain_begin()) return;
  __shared__ float part[2][LR_THREADS / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t n = blockIdx.x;
  const float c = a.scale * kLog2e;
  const float* row = f.z + n * f.ldz;
  const int32_t t = a.targets[n];
  const bool in = t >= 0 && t < a.V;
  const float w = a.weight ? a.weight[n] : 1.f, zt = in ? row[t] : 0.f;
  float4 z[LR_EACH / 4];
  float m = ROW_NEG_INF;
#pragma unroll
  for (int i = 0; i < LR_EACH / 4; ++i) {
    const int v = 4 * (i * LR_THREADS + (int)threadIdx.x);
    z[i] = make_float4(ROW_NEG_INF, ROW_NEG_INF, ROW_NEG_INF, ROW_NEG_INF);
    if (v < a.V) {                                      // the row reaches to the next multiple of 8
      z[i] = *reinterpret_cast<const float4*>(row + v);
      if (v + 1 >= a.V) z[i].y = ROW_NEG_INF;
      if (v + 2 >= a.V) z[i].z = ROW_NEG_INF;
      if (v + 3 >= a.V) z[i].w = ROW_NEG_INF;
    }
    m = fmaxf(m, fmaxf(fmaxf(z[i].x, z[i].y), fmaxf(z[i].z, z[i].w)));
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (lane == 0) part[0][warp] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < LR_THREADS / 32; ++i) m = fmaxf(m, part[0][i]);
  const float ref = m == ROW_NEG_INF ? 0.f : m;         // a row with nothing left has a sum of 0
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < LR_EACH / 4; ++i) {
    z[i].x = row_ex2((z[i].x - ref) * c);
    z[i].y = row_ex2((z[i].y - ref) * c);
    z[i].z = row_ex2((z[i].z - ref) * c);
    z[i].w = row_ex2((z[i].w - ref) * c);
    s += (z[i].x + z[i].y) + (z[i].z + z[i].w);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (lane == 0) part[1][warp] = s;
  __syncthreads();
  s = 0.f;
#pragma unroll
  for (int i = 0; i < LR_THREADS / 32; ++i) s += part[1][i];
  const float lp = in ? row_logp(zt, m, logf(s), a.scale) : 0.f;
  const bool takes_part = in && w != 0.f && loss_target(a, t, lp, m);
  if (threadIdx.x == 0) {
    if (!in && t != -1) gram_device_fail(f.status, GRAM_ERR_ID_RANGE);
    a.loss[n] = 0.f - lp;
  }
  if (f.clean && warp == 0) loss_clean(a, n, takes_part, f.clean);
  if (f.rest && threadIdx.x == 0 && !takes_part) f.rest[n] = RowRest{0.f, -1};
  const float factor = lp != lp ? lp : w * a.scale, each = takes_part ? factor / s : 0.f;
#pragma unroll
  for (int i = 0; i < LR_EACH / 4; ++i) {
    const int v = 4 * (i * LR_THREADS + (int)threadIdx.x);
    if (v >= a.V) break;
    // of the target p - 1, in one rounding of the difference
    float g[4] = {z[i].x, z[i].y, z[i].z, z[i].w};
#pragma unroll
    for (int j = 0; j < 4; ++j) g[j] = !takes_part ? 0.f : v + j == t ? factor * (g[j] / s - 1.f) : g[j] * each;
    bf16* to = f.at.g + n * f.at.ldg + v;
#pragma unroll
    for (int k = 0; k < PLANES; ++k) {
      const uint2 h = make_uint2(pack_bf16x2(g[0], g[1]), pack_bf16x2(g[2], g[3]));
      *reinterpret_cast<uint2*>(to + k * f.at.plane) = h;
      const float2 u = unpack_bf16x2(h.x), x = unpack_bf16x2(h.y);
      g[0] -= u.x; g[1] -= u.y; g[2] -= x.x; g[3] -= x.y;
    }
    if (f.rest && takes_part && (unsigned)(t - v) < 4u) f.rest[n] = RowRest{(t - v) & 2 ? ((t - v) & 1 ? g[3] : g[2]) : ((t - v) & 1 ? g[1] : g[0]), t};
  }
}

// Up to four users: both products by lanes.  What they cost is the table's bytes, read and written once; a tile of the tensor cores would be 256 users, with
// bf16 entries.  A block takes `chunk` items and 256 columns: g of its items in 32 bits from logits in L2, then a warp an item at a time, a lane eight columns of
// it: dI leaves, dU and db are summed on the way.  us of a call in a graph, by tensor cores and so: 1 x 10 000 x 768 25.6 and 20.6, 1 x 148 184 x 728
// with fp32 gradients 226 and 187, 4 x 2000 x 768 fp32 21.6 and 16.2, 4 x 100 000 x 768 111 and 113.  Eight items ahead for four took 22.4 for 20.6.
constexpr int LO_USERS = 4, LO_CHUNK = 512;             // most items of a block
constexpr int LO_AHEAD = 4;                             // items of a warp whose loads are on their way together
struct OneArgs {
  const float* z;                // [N, ldz]
  int64_t ldz;
  const float* logp;
  const float2* stats;
  int32_t chunk, wide;           // wide: rows of dI begin on 32 bytes
  float* parts;                  // [chunks, N, d]: dU
  int32_t* status;
};
__device__ __forceinline__ void st32(void* p, const uint32_t* v) {        // 32 bytes, 32-byte aligned
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]),
               "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}
template <typename GT> __device__ __forceinline__ void put8(GT* to, const f32x2 (&x)[4], bool wide) {        // wide: 32-byte aligned (fp32: whole sectors)
  uint32_t h[8];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 f = x2_unpack(x[j]);
    if constexpr (sizeof(GT) == 4) {
      h[2 * j] = __float_as_uint(f.x);
      h[2 * j + 1] = __float_as_uint(f.y);
    } else {
      h[j] = pack_bf16x2(f.x, f.y);
    }
  }
  uint4* q = reinterpret_cast<uint4*>(to);
  if (sizeof(GT) == 4 && wide) {
    st32(to, h);
  } else {
    q[0] = make_uint4(h[0], h[1], h[2], h[3]);
    if constexpr (sizeof(GT) == 4) q[1] = make_uint4(h[4], h[5], h[6], h[7]);
  }
}
__device__ __forceinline__ void get8(uint4 w, f32x2 (&x)[4]) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] = x2_pack(__uint_as_float(u[j] << 16), __uint_as_float(u[j] & 0xffff0000u));
}
template <typename GT, int USERS> __global__ void __launch_bounds__(256) loss_one_kernel(const ScoreLoss a, const OneArgs f) {
  chain_next();
  if (!chain_begin()) return;
  __shared__ float g[USERS][LO_CHUNK];
  __shared__ __align__(16) float sums[8][USERS][256];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, N = (int)a.N;
  const int v0 = blockIdx.x * f.chunk, rows = min(f.chunk, a.V - v0), col = blockIdx.y * 256 + 8 * lane;
  const float c = a.scale * kLog2e;
  RowConst r[USERS];
#pragma unroll
  for (int n = 0; n < USERS; ++n) r[n] = n < N ? loss_row(a, f.logp, f.stats, n) : RowConst{0.f, 0.f, 0.f, -1};
  if (blockIdx.x == 0 && blockIdx.y == 0 && (int)threadIdx.x < N) a.loss[threadIdx.x] = loss_of(a, f.logp, threadIdx.x, f.status);
  for (int i = threadIdx.x; i < rows; i += 256) {
    float sum = 0.f;
#pragma unroll
    for (int n = 0; n < USERS; ++n) {
      float x = 0.f;
      if (r[n].t >= 0) {
        const float p = loss_p(r[n], f.z[n * f.ldz + v0 + i], c);
        x = r[n].f * (v0 + i == r[n].t ? p - 1.f : p);
      }
      g[n][i] = x;
      sum += x;
    }
    if (a.dbias && blockIdx.y == 0) a.dbias[v0 + i] = sum;
  }
  __syncthreads();
  f32x2 u[USERS][4], acc[USERS][4];
#pragma unroll
  for (int n = 0; n < USERS; ++n) {
#pragma unroll
    for (int j = 0; j < 4; ++j) u[n][j] = acc[n][j] = x2_pack(0.f, 0.f);
    if (r[n].t >= 0 && col < a.d) get8(__ldg(reinterpret_cast<const uint4*>(reinterpret_cast<const bf16*>(a.users) + n * a.ld_users + col)), u[n]);
  }
  if (col < a.d) {
    const bf16* items = reinterpret_cast<const bf16*>(a.items) + (int64_t)v0 * a.ld_items + col;
    GT* out = reinterpret_cast<GT*>(a.ditems) + (int64_t)v0 * a.ld_ditems + col;
    for (int i0 = warp; i0 < rows; i0 += 8 * LO_AHEAD) {
      uint4 raw[LO_AHEAD];                              // all loads on their way before the first store
#pragma unroll
      for (int k = 0; k < LO_AHEAD; ++k)
        if (a.dusers && i0 + 8 * k < rows) raw[k] = __ldg(reinterpret_cast<const uint4*>(items + (i0 + 8 * k) * a.ld_items));
#pragma unroll
      for (int k = 0; k < LO_AHEAD; ++k) {
        const int i = i0 + 8 * k;
        if (i >= rows) break;
        f32x2 x[4], w[4];
        get8(raw[k], w);
#pragma unroll
        for (int n = 0; n < USERS; ++n) {
          const f32x2 gn = x2_pack(g[n][i], g[n][i]);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            x[j] = n == 0 ? x2_mul(gn, u[n][j]) : x2_fma(gn, u[n][j], x[j]);
            acc[n][j] = x2_fma(gn, w[j], acc[n][j]);    // not looked at where dU is not asked
          }
        }
        if (a.ditems) put8(out + i * a.ld_ditems, x, f.wide);
      }
    }
  }
  if (!a.dusers) return;
#pragma unroll
  for (int n = 0; n < USERS; ++n)
#pragma unroll
    for (int j = 0; j < 4; ++j) *reinterpret_cast<float2*>(&sums[warp][n][8 * lane + 2 * j]) = x2_unpack(acc[n][j]);
  __syncthreads();
  const int at = blockIdx.y * 256 + (int)threadIdx.x;
  if (at >= a.d) return;
#pragma unroll
  for (int n = 0; n < USERS; ++n) {
    float x = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) x += sums[w][n][threadIdx.x];
    if (n < N) f.parts[((int64_t)blockIdx.x * N + n) * a.d + at] = x;
  }
}
// their dU: a block takes 32 columns of a user, its warps the parts in turn
template <typename GT> __global__ void __launch_bounds__(1024) loss_one_finish_kernel(const float* parts, int32_t chunks, int32_t d, int64_t stride, GT* dU, int64_t ld) {
  if (!chain_begin()) return;
  __shared__ float sums[32][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
  float s = 0.f;
  if (col < d) {
#pragma unroll 8
    for (int k = warp; k < chunks; k += 32) s += parts[k * stride + (int64_t)blockIdx.y * d + col];
  }
  sums[warp][lane] = s;
  __syncthreads();
  s = sums[lane][warp];                                 // of column `warp` now, a part a lane
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (lane == 0 && blockIdx.x * 32 + warp < d) dU[blockIdx.y * ld + blockIdx.x * 32 + warp] = row_round<GT>(s);
}

// ============================================================================================
// g of a piece
// ============================================================================================
constexpr int LG_STAGES = 6, LG_EPI_WARPS = 16, LG_PARTS = LG_EPI_WARPS / 4;
constexpr int LG_BIAS_BYTES = LG_EPI_WARPS * 64 * 4;    // a warp's columns
using GradPipe = PairPipe<LG_STAGES, LG_EPI_WARPS, LG_BIAS_BYTES>;

struct GradArgs {
  Piece at;
  const RowConst* rows;          // [N]
  RowRest* rest;                 // [N] or null
  const float* bias;             // [V] or null
  int32_t V;
  int32_t num_kb, tiles_m, width;
  int32_t whole, total;          // tiles before those at the end that are dealt as two of half the width; of all, halves counted twice
  int32_t box_rows;              // users of a copy
  float c;
  float* bias_part;              // [32-row blocks of the piece, ldg] or null
  int32_t give_up;
  int32_t* status;
};

// first user and item of the piece, and width, of the t-th tile
struct GradTile {
  int m0, n0, width;
  __device__ __forceinline__ GradTile(const GradArgs& a, int t) {
    int half = -1;
    if (t >= a.whole) {
      half = (t - a.whole) & 1;
      t = a.whole + ((t - a.whole) >> 1);
    }
    const int n = t / a.tiles_m;
    m0 = (t - n * a.tiles_m) * 2 * PAIR_ROWS;
    n0 = n * a.width;
    width = a.width;
    if (half >= 0) {
      width = PAIR_COLS / 2;
      n0 += half * width;
    }
  }
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
      const GradTile u(a, t);
      const int m0 = u.m0 + (int)pipe.rank * PAIR_ROWS, n0 = a.at.first + u.n0 + (int)pipe.rank * (u.width / 2);
      const bool some = m0 < a.at.rows;                 // what the rows of users past the last hold is not looked at
      const uint32_t bytes = (some ? (uint32_t)a.box_rows * 128u : 0u) + (uint32_t)u.width * 64u;
      for (int kb = 0; kb < a.num_kb; ++kb) {
        if (!mbar_wait_warp(pipe.empty(s), ph ^ 1u, pipe.abort_flag)) { failed = true; break; }
        const uint32_t bar = pipe.lead_full(s);
        if (elect_one()) {
          mbar_arrive_expect_tx_remote(bar, bytes);
          if (some) tma_load_2d_pair(pipe.a_of(s), &users, kb * 64, (int)a.at.n0 + m0, bar);
          tma_load_2d_pair(pipe.b_of(s), &items, kb * 64, n0, bar);
          if (u.width == PAIR_COLS) tma_load_2d_pair(pipe.b_of(s) + PAIR_BOX, &items, kb * 64, n0 + 64, bar);
        }
        __syncwarp();
        if (++s == LG_STAGES) { s = 0; ph ^= 1u; }
      }
    }
  } else if (pipe.warp == 1 && go) {
    // ------------------------------ products (leader) ------------------------------
    if (pipe.rank == 0) {
      constexpr uint32_t idesc0 = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(2 * PAIR_ROWS >> 4) << 24);
      const uint64_t da0 = make_desc(pipe.a_of(0), 16, 1024), db0 = make_desc(pipe.b_of(0), 16, 1024);
      int s = 0;
      uint32_t ph = 0, it = 0;
      for (int t = pair; t < a.total && !failed; t += pairs, ++it) {
        const uint32_t idesc = idesc0 | ((uint32_t)(GradTile(a, t).width >> 3) << 17);
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
    const f32x2 cc = x2_pack(a.c, a.c);
    uint32_t it = 0;
    for (int t = pair; t < a.total && !failed; t += pairs, ++it) {
      const int buf = (int)(it & 1);
      const GradTile u(a, t);
      const int blocks = u.width / PAIR_ROWS;           // of 32 columns of this warp
      const int col_t = part * blocks * 32, col0 = u.n0 + col_t;                // of the tile, of the piece
      const int64_t n = (int64_t)u.m0 + (int)pipe.rank * PAIR_ROWS + q * 32 + lane;        // of the piece
      const bool active = n - lane < a.at.rows;         // of the warp
      RowConst r{0.f, 0.f, 0.f, -1};
      const float* bias = nullptr;
      if (active) {
        if (n < a.at.rows) {
          const float4 f = __ldg(reinterpret_cast<const float4*>(a.rows) + a.at.n0 + n);
          r = RowConst{f.x, f.y, f.z, __float_as_int(f.w)};
        }
        if (a.bias || a.at.first + col0 + blocks * 32 > a.V) {     // columns past the table count as masked out
          __syncwarp();
          for (int b = 0; b < blocks; ++b) {
            const int v = a.at.first + col0 + b * 32 + lane;
            bias_w[b * 32 + lane] = v >= a.V ? ROW_NEG_INF : a.bias ? __ldg(a.bias + v) : 0.f;
          }
          __syncwarp();
          bias = bias_w;
        }
      }
      const int hot = r.t - a.at.first - col0;          // the target's place among the warp's columns
      const f32x2 m2 = x2_pack(-r.m, -r.m), l2 = x2_pack(-r.l, -r.l), f2 = x2_pack(r.f, r.f);
      const bool hold = __any_sync(0xffffffffu, row_is_huge(r.m, a.c));
      if (!mbar_wait_warp(pipe.tfull(buf), (it >> 1) & 1, pipe.abort_flag)) { failed = true; break; }
      tc_fence_after();
      if (active) {
        const uint32_t taddr = pipe.tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(buf * PAIR_COLS + col_t);
        for (int b = 0; b < blocks; ++b) {
          uint32_t v[32];
          tc_ld32_issue(taddr + b * 32, v);
          tc_ld32_wait(v);
          if (bias) {
#pragma unroll
            for (int j = 0; j < 32; j += 4) {
              const float4 f = *reinterpret_cast<const float4*>(bias + b * 32 + j);
              v[j] = __float_as_uint(__uint_as_float(v[j]) + f.x);
              v[j + 1] = __float_as_uint(__uint_as_float(v[j + 1]) + f.y);
              v[j + 2] = __float_as_uint(__uint_as_float(v[j + 2]) + f.z);
              v[j + 3] = __float_as_uint(__uint_as_float(v[j + 3]) + f.w);
            }
          }
          float g[32];
#pragma unroll
          for (int j = 0; j < 32; j += 2) {
            const float2 y = x2_unpack(x2_fma(x2_add(x2_pack(__uint_as_float(v[j]), __uint_as_float(v[j + 1])), m2), cc, l2));
            g[j] = y.x;
            g[j + 1] = y.y;
          }
          if (hold) {
#pragma unroll
            for (int j = 0; j < 32; ++j) g[j] = fminf(g[j], 0.f);
          }
#pragma unroll
          for (int j = 0; j < 32; ++j) g[j] = row_ex2(g[j]);
          if (r.t >= 0 && (unsigned)(hot - b * 32) < 32u) {
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (j == hot - b * 32) g[j] -= 1.f;
          }
#pragma unroll
          for (int j = 0; j < 32; j += 2) {
            const float2 x = x2_unpack(x2_mul(x2_pack(g[j], g[j + 1]), f2));
            g[j] = x.x;
            g[j + 1] = x.y;
          }
          if (__any_sync(0xffffffffu, r.t < 0)) {       // rows that take no part
#pragma unroll
            for (int j = 0; j < 32; ++j) g[j] = r.t < 0 ? 0.f : g[j];
          }
          if (PLANES > 0 && n < a.at.rows) {
            bf16* to = a.at.g + n * a.at.ldg + col0 + b * 32;
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
              st32(to + a.at.plane, h);
              st32(to + a.at.plane + 16, h + 8);
            }
            if (a.rest && r.t >= 0 && (unsigned)(hot - b * 32) < 32u) {
              float rest = 0.f;
#pragma unroll
              for (int j = 0; j < 32; ++j)
                if (j == hot - b * 32) rest = g[j];
              float left = rest - __bfloat162float(__float2bfloat16_rn(rest));
              if (PLANES == 2) left -= __bfloat162float(__float2bfloat16_rn(left));
              a.rest[a.at.n0 + n].rest = left;
            }
          }
          if (a.bias_part) a.bias_part[(n >> 5) * a.at.ldg + col0 + b * 32 + lane] = column_sums(g);
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_remote(pipe.lead_tempty(buf));
    }
  }
  pipe.close(failed, a.status);
}

// db of a piece: the sum of its blocks of rows, eight groups of them side by side
__global__ void __launch_bounds__(256) loss_bias_kernel(const float* part, int64_t ldg, int64_t blocks, int32_t cols, int32_t add, float* dbias) {
  chain_next();
  if (!chain_begin()) return;
  __shared__ float sums[8][32];
  const int lane = threadIdx.x & 31, group = threadIdx.x >> 5, v = blockIdx.x * 32 + lane;
  float s = 0.f;
#pragma unroll 8
  for (int64_t i = group; i < blocks; i += 8) s += part[i * ldg + v];      // the rows reach past the last column
  sums[group][lane] = s;
  __syncthreads();
  if (group != 0 || v >= cols) return;
#pragma unroll
  for (int i = 1; i < 8; ++i) s += sums[i][lane];
  dbias[v] = add ? dbias[v] + s : s;
}

// ============================================================================================
// both products of a piece's g
// ============================================================================================
// PLANES: bf16 that g is the sum of; a stage holds all of them beside one piece of the vectors.  CHAINED: eight warps take the results, 128 columns
// each, which can add up several accumulators in registers; else sixteen with 64.  A warp has a box of 32 rows x 128 bytes for its results,
// two in turn where there are eight (46 users, 5545 items of 440, fp32 gradients 26.9 -> 24.3 us; sums of many users the same with a stage less).
template <int PLANES, bool CHAINED> using ProdPipe = PairPipe<PLANES == 1 ? 5 : 5 - PLANES, CHAINED ? 8 : 16, 16 * 4096, PLANES>;

// Blocks of 64 (of all planes) that are added up in one accumulator.  The tensor cores cut off, four times a block and plane, where other sums are
// rounded: up to 2^-23 of the sum each time, half of that on average.  fp32 gradients of 25 600 users and 10 000 items of 768 against 64 bits: 4.2e-6 from
// chains of 24 blocks, 2.65e-6 from 8 (of which g's rounding is 2.3e-6), 2.4e-6 from 4; 1767, 1770 and 1778 us.  bf16: 1024 blocks, 2.4e-4 on average, hidden by
// the result's rounding of 2^-8.
constexpr int LP_CHAIN = 8, LP_CHAIN_BF16 = 1024;

// One gradient's share in a piece.
struct ProdSide {
  int32_t tiles_m, rows;         // tiles of 256 of the piece's rows (0: not asked)
  int32_t kb, kb_split;          // blocks of 64 that the sums run over, and those of a part
  int32_t vec0;                  // the first of the vectors that they run over
  int32_t units, cost;           // tiles of all parts; what one costs, in blocks
  int32_t partial;               // fp32 sums that are joined later, in place of the result
  int32_t add;                   // to what is there (partial)
  int32_t part;                  // rows from one part to the next, a multiple of 256
};
struct ProdArgs {
  ProdSide of[2];                // users' and items' gradient
  int32_t d, tiles_n;            // tiles of 256 columns of d
  int32_t total, heavy;          // units of both; whose are the heavier ones, which are dealt first
  int32_t extra;                 // lighter units that a pair gets for each heavier one that others have more
  int32_t halves;                // units at the end that are dealt as two of half the columns each
  int32_t chain;                 // blocks that are added up in one accumulator
  int32_t give_up;
  int32_t* status;
};

// Which units a pair takes, its i-th: the heavier ones are dealt first; pairs that get one less take `extra` lighter ones instead; the rest is dealt
// from the pairs with less on, the last round as halves where twice as many are no more than the pairs.  (The same in loss_span.)
struct ProdWalk {
  int pair, pairs, heavy, mine, extra, other, base, at, total;       // total: halves count as units
  __device__ __forceinline__ explicit ProdWalk(const ProdArgs& a) : pair(blockIdx.x >> 1), pairs(gridDim.x >> 1), total(a.total + a.halves) {
    heavy = a.of[a.heavy].units;
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

// A unit: a tile of one of the gradients over a part of its sums.
struct ProdUnit {
  int side, m0, n0, width, split, k0, blocks;           // first row and column; the sum's range in blocks of 64
  __device__ __forceinline__ ProdUnit(const ProdArgs& a, int t) {
    int half = -1;
    const int whole = a.total - a.halves;
    if (t >= whole) {
      half = (t - whole) & 1;
      t = whole + ((t - whole) >> 1);
    }
    side = a.heavy;
    if (t >= a.of[side].units) {
      t -= a.of[side].units;
      side ^= 1;
    }
    const ProdSide& o = a.of[side];
    const int r = t / a.tiles_n;
    n0 = (t - r * a.tiles_n) * PAIR_COLS;
    width = a.d - n0 > PAIR_COLS / 2 && half < 0 ? PAIR_COLS : PAIR_COLS / 2;
    if (half > 0) n0 += PAIR_COLS / 2;                  // perhaps past the last column
    split = r / o.tiles_m;
    m0 = (r - split * o.tiles_m) * 2 * PAIR_ROWS;
    k0 = split * o.kb_split;
    blocks = min(o.kb_split, o.kb - k0);
  }
};

// 32 fp32 columns of a row to its place in a box of 32 rows x 128 bytes (128-byte swizzle); 32 of 64 bf16 columns
__device__ __forceinline__ void box_row(uint32_t box, const float (&x)[32]) {
  const uint32_t lane = threadIdx.x & 31, row = box + lane * 128u;
#pragma unroll
  for (uint32_t j = 0; j < 8; ++j)
    sts128(row + ((j ^ (lane & 7)) << 4), __float_as_uint(x[4 * j]), __float_as_uint(x[4 * j + 1]), __float_as_uint(x[4 * j + 2]), __float_as_uint(x[4 * j + 3]));
}
__device__ __forceinline__ void box_row(uint32_t box, const float (&x)[32], uint32_t half) {
  const uint32_t lane = threadIdx.x & 31, row = box + lane * 128u;
#pragma unroll
  for (uint32_t j = 0; j < 4; ++j)
    sts128(row + (((half * 4 + j) ^ (lane & 7)) << 4), pack_bf16x2(x[8 * j], x[8 * j + 1]), pack_bf16x2(x[8 * j + 2], x[8 * j + 3]),
           pack_bf16x2(x[8 * j + 4], x[8 * j + 5]), pack_bf16x2(x[8 * j + 6], x[8 * j + 7]));
}

template <typename GT, int PLANES, bool CHAINED>
__global__ void __launch_bounds__(ProdPipe<PLANES, CHAINED>::THREADS, 1)
    loss_products_kernel(const __grid_constant__ CUtensorMap g0, const __grid_constant__ CUtensorMap g1, const __grid_constant__ CUtensorMap g2,
                         const __grid_constant__ CUtensorMap users, const __grid_constant__ CUtensorMap items, const __grid_constant__ CUtensorMap out_u,
                         const __grid_constant__ CUtensorMap out_i, const __grid_constant__ ProdArgs a) {
  using Pipe = ProdPipe<PLANES, CHAINED>;
  extern __shared__ uint8_t smem_raw[];
  Pipe pipe;
  const bool go = pipe.open(smem_raw);
  chain_next();
  const ProdWalk walk(a);
  bool failed = false;
  if (pipe.warp == 0 && go) {
    // ------------------------------ copies (both blocks): two boxes of 64 x 64 of each plane of g, one or two of the vectors ------------------------------
    int s = 0;
    uint32_t ph = 0;
    for (int tile = 0, t; (t = walk(tile)) < walk.total && !failed; ++tile) {
      if (tile == a.give_up) { failed = true; break; }
      const ProdUnit u(a, t);
      const int m0 = u.m0 + (int)pipe.rank * PAIR_ROWS, n0 = u.n0 + (int)pipe.rank * (u.width / 2);
      const uint32_t bytes = PLANES * 2 * PAIR_BOX + (uint32_t)(u.width / PAIR_ROWS) * PAIR_BOX;
      const bool of_users = u.side == 0;                 // its rows are g's rows
      const CUtensorMap* vectors = of_users ? &items : &users;
      const int vec0 = a.of[u.side].vec0;
      for (int kb = 0; kb < u.blocks; ++kb) {
        const int k = (u.k0 + kb) * 64, row = vec0 + k;
        if (!mbar_wait_warp(pipe.empty(s), ph ^ 1u, pipe.abort_flag)) { failed = true; break; }
        const uint32_t bar = pipe.lead_full(s), sb = pipe.b_of(s);
        if (elect_one()) {
          mbar_arrive_expect_tx_remote(bar, bytes);
#pragma unroll
          for (int i = 0; i < PLANES; ++i) {
            const CUtensorMap* g = i == 0 ? &g0 : i == 1 ? &g1 : &g2;
            const uint32_t sa = pipe.a_of(s, i);
            tma_load_2d_pair(sa, g, of_users ? k : m0, of_users ? m0 : k, bar);
            tma_load_2d_pair(sa + PAIR_BOX, g, of_users ? k : m0 + 64, of_users ? m0 + 64 : k, bar);
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
      for (int tile = 0, t; (t = walk(tile)) < walk.total && !failed; ++tile) {
        const ProdUnit u(a, t);
        const uint32_t idesc = idesc0 | (u.side == 0 ? 0u : 1u << 15) | ((uint32_t)(u.width >> 3) << 17);
        const uint64_t da0 = u.side == 0 ? da_k : da_mn;
        const uint32_t step_a = (u.side == 0 ? 32u : 2048u) >> 4;
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
    // ------------------------------ results (both blocks): a row and 64 or 128 columns a thread ------------------------------
    constexpr int BLOCKS = CHAINED ? 4 : 2;             // of 32 columns
    const int lane = pipe.lane, q = pipe.warp & 3, part = (pipe.warp - 2) >> 2;
    const uint32_t lane_addr = pipe.tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(part * BLOCKS * 32);
    constexpr bool TWO = CHAINED;                       // boxes, in turn
    const uint32_t box0 = pipe.tiles + Pipe::STAGES * Pipe::STAGE + (uint32_t)(pipe.warp - 2) * (TWO ? 8192u : 4096u);
    uint32_t it = 0, box = box0;
    for (int tile = 0, t; (t = walk(tile)) < walk.total && !failed; ++tile) {
      const ProdUnit u(a, t);
      const ProdSide& o = a.of[u.side];
      const CUtensorMap* out = u.side == 0 ? &out_u : &out_i;
      const int m = u.m0 + (int)pipe.rank * PAIR_ROWS + q * 32, n = u.n0 + part * BLOCKS * 32;        // of the warp
      const bool there = m < o.rows && n < a.d && part * BLOCKS * 32 < u.width;
      const int row = m + u.split * o.part;
      auto free_box = [&]() {                           // its last store has read it
        if (lane == 0) {
          if (TWO) bulk_wait_read_but_one();
          else bulk_wait_read_all();
        }
        __syncwarp();
      };
      auto send = [&](int col, bool add) {
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          if (col < a.d) {
            if (add) tma_reduce_add_2d(out, box, col, row);
            else tma_store_2d(out, box, col, row);
          }
          bulk_commit();
        }
        if (TWO) box = box == box0 ? box0 + 4096u : box0;
      };
      auto put = [&](int b, const float (&x)[32]) {     // block b of the warp's columns
        if (sizeof(GT) == 4 || o.partial) {
          free_box();
          box_row(box, x);
          send(n + b * 32, o.partial && o.add);
        } else {
          if (b % 2 == 0) free_box();
          box_row(box, x, (uint32_t)b % 2);
          if (b % 2 == 1) send(n + (b - 1) * 32, false);
        }
      };
      if constexpr (CHAINED) {
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
          if (there) {
#pragma unroll
            for (int b = 0; b < 4; ++b)
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                uint32_t v[16];
                tc_ld16(lane_addr + (uint32_t)(buf * PAIR_COLS + b * 32 + h * 16), v);
#pragma unroll
                for (int j = 0; j < 16; ++j) acc[b][h * 16 + j] += __uint_as_float(v[j]);
              }
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_remote(pipe.lead_tempty(buf));
        }
        if (failed) break;
        if (there) {
#pragma unroll
          for (int b = 0; b < 4; ++b) put(b, acc[b]);
        }
      } else {
        const int buf = (int)(it & 1);
        if (!mbar_wait_warp(pipe.tfull(buf), (it >> 1) & 1, pipe.abort_flag)) { failed = true; break; }
        tc_fence_after();
        if (there) {
#pragma unroll
          for (int b = 0; b < BLOCKS; ++b) {
            uint32_t v[32];
            tc_ld32_issue(lane_addr + (uint32_t)(buf * PAIR_COLS + b * 32), v);
            tc_ld32_wait(v);
            float x[32];
#pragma unroll
            for (int j = 0; j < 32; ++j) x[j] = __uint_as_float(v[j]);
            put(b, x);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_remote(pipe.lead_tempty(buf));
        ++it;
      }
    }
    if (lane == 0) bulk_wait_all();                     // its stores are complete before the block may exit
  }
  pipe.close(failed, a.status);
}

// A gradient [N, d] as the sum of its parts, `part` elements from one to the next; the users' with what is left of their targets (rest).
template <typename GT> __global__ void __launch_bounds__(256) loss_finish_kernel(const float* parts, int splits, int64_t part, int64_t N, int32_t d, const RowRest* rest,
                                                                                 const bf16* items, int64_t ld_items, GT* grad, int64_t ld) {
  if (!chain_begin()) return;
  const int64_t n4 = N * (d / 4);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n4; i += (int64_t)gridDim.x * 256) {
    const int64_t n = i / (d / 4);
    const int c = 4 * (int)(i - n * (d / 4));
    uint2 item = make_uint2(0u, 0u);
    float left = 0.f;
    if (rest) {
      const RowRest r = rest[n];
      if (r.t >= 0) {
        item = __ldg(reinterpret_cast<const uint2*>(items + r.t * ld_items + c));
        left = r.rest;
      }
    }
    float4 s = reinterpret_cast<const float4*>(parts)[i];
#pragma unroll 8
    for (int k = 1; k < splits; ++k) {
      const float4 x = reinterpret_cast<const float4*>(parts + k * part)[i];
      s.x += x.x; s.y += x.y; s.z += x.z; s.w += x.w;
    }
    const float2 u = unpack_bf16x2(item.x), v = unpack_bf16x2(item.y);
    s = make_float4(fmaf(left, u.x, s.x), fmaf(left, u.y, s.y), fmaf(left, v.x, s.z), fmaf(left, v.y, s.w));
    GT* to = grad + n * ld + c;
    if constexpr (sizeof(GT) == 4) *reinterpret_cast<float4*>(to) = s;
    else *reinterpret_cast<uint2*>(to) = make_uint2(pack_bf16x2(s.x, s.y), pack_bf16x2(s.z, s.w));
  }
}

// ============================================================================================
// host side
// ============================================================================================
size_t up(size_t n) { return (n + 255) / 256 * 256; }

struct LossPlan {
  size_t logp, stats, rows, rest, clean, parts, bias, g, bytes; // places in the workspace
  bool cut_users;                                               // pieces are of users, else of items
  int32_t step, splits;                                         // users or items of a piece; parts of the summed gradient
  int64_t ldg;
};

// What a unit over `kb` blocks costs, in blocks of a pair (0.37 us): the products of all planes, or the way of 256 x 256 results out where that takes longer.
int64_t loss_cost(int64_t kb, int planes, bool f32) {
  const int64_t out = f32 ? 6 : 3;
  return kb * planes > out ? kb * planes : out;
}

// How the units of a piece's products are dealt to the pairs (ProdWalk), and the blocks that the busiest one works through.
struct LossSpan {
  int64_t most;
  int32_t heavy, extra, halves;  // heavy: whether the second kind is the heavier one
};
LossSpan loss_span(int64_t units_a, int64_t cost_a, int64_t units_b, int64_t cost_b) {
  const bool second = units_a == 0 || (units_b > 0 && cost_b > cost_a);
  const int64_t n1 = second ? units_b : units_a, c1 = second ? cost_b : cost_a, n2 = second ? units_a : units_b;
  const int64_t c2 = second ? cost_a : cost_b, pairs = n1 + n2 < kPairs ? n1 + n2 : kPairs;
  const int64_t more = n1 % pairs, other = pairs - more;
  int64_t extra = more ? c1 / c2 : 0;                   // rounded down: those pairs are dealt to first
  if (extra > n2 / other) extra = n2 / other;
  const int64_t rest = n2 - extra * other, last = rest % pairs;
  const bool half = last > 0 && 2 * last <= pairs && n1 + n2 > pairs;
  const int64_t round = half ? 2 * last : last, cost = half ? (c2 + 1) / 2 : c2;         // the last round
  const int64_t load_other = (n1 / pairs) * c1 + (extra + rest / pairs) * c2 + (round > 0 ? cost : 0);
  const int64_t load_more = more ? (n1 / pairs + 1) * c1 + (rest / pairs) * c2 + (round > other ? cost : 0) : 0;
  return LossSpan{load_other > load_more ? load_other : load_more, (int32_t)second, (int32_t)extra, (int32_t)(half ? last : 0)};
}

// Parts that the summed gradient's sums over a piece are cut into, so that the pairs are evenly busy.  `step` rows of the piece's own
// gradient, `all` of the summed one.  A part costs its place in the sum: 8 `all` d bytes, in blocks.
struct LossSplits {
  int parts;
  double time;                   // of the piece, in blocks
};
LossSplits loss_splits(int64_t step, int64_t all, int32_t d, int planes, bool f32, bool own, bool summed, bool joined) {
  const int64_t tiles_n = ceil_div(d, PAIR_COLS), kb = ceil_div64(step, 64);
  const int64_t units_own = own ? ceil_div64(step, PAIR_COLS) * tiles_n : 0, tiles = ceil_div64(all, PAIR_COLS) * tiles_n;
  const int64_t cost_own = loss_cost(ceil_div64(all, 64), planes, f32);
  if (!summed) return LossSplits{0, units_own ? (double)loss_span(units_own, cost_own, 0, 1).most : 0.0};
  const double part = 8.0 * all * d / (5e6 * 0.37);
  LossSplits best{1, 1e300};
  for (int s = 1; s <= 32 && s * 4 <= (kb > 4 ? kb : 4) && s * all < (1 << 30); ++s) {
    const int64_t of = ceil_div64(kb, s), parts = ceil_div64(kb, of);
    const double time = (double)loss_span(tiles * parts, loss_cost(of, planes, true), units_own, cost_own).most + (parts > 1 || joined ? parts * part : 0.0);
    if (time < best.time) best = LossSplits{(int)parts, time};
  }
  return best;
}

// Lays out a workspace of `room` bytes, or the one of pieces of `step`.  planes 0: no product takes g, which is not kept.
LossPlan loss_plan(int64_t N, int32_t V, int32_t d, int planes, bool f32, bool users, bool items, bool bias, int64_t step, size_t room) {
  LossPlan p = {};
  p.cut_users = N > V;
  const int64_t axis = p.cut_users ? N : V, all = p.cut_users ? V : N, all_up = (all + 255) / 256 * 256;
  const bool own = p.cut_users ? users : items, summed = p.cut_users ? items : users;
  const int64_t most = (axis + 255) / 256 * 256 < INT32_MAX / 256 * 256 ? (axis + 255) / 256 * 256 : INT32_MAX / 256 * 256;
  auto place = [&](int64_t c, int splits) {
    size_t at = 0;
    auto take = [&](size_t n) { const size_t was = at; at += up(n); return was; };
    const int64_t rows = p.cut_users ? c : N;
    p.ldg = p.cut_users ? all_up : c;
    p.logp = take((size_t)N * 4);
    p.stats = take((size_t)N * 8);
    p.rows = take((size_t)N * sizeof(RowConst));
    p.rest = take(users ? (size_t)N * sizeof(RowRest) : 0);
    p.clean = take(items ? (size_t)N * d * 2 : 0);
    p.parts = take((size_t)splits * all_up * d * 4);
    p.bias = take(bias ? (size_t)ceil_div64(rows, 32) * p.ldg * 4 : 0);
    p.g = take((size_t)planes * rows * p.ldg * 2);
    p.bytes = at;
    p.step = (int32_t)c;
    p.splits = splits;
  };
  auto with = [&](int64_t c) {
    const int64_t real = c < axis ? c : axis;
    const int kb = (int)ceil_div64(real, 64);
    int s = loss_splits(real, all, d, planes, f32, own, summed, !p.cut_users).parts;
    place(c, s);
    while (room && p.bytes > room && s > 1) place(c, s = ceil_div(kb, ceil_div(kb, s - 1)));      // as many as are not empty
  };
  if (!room) {
    with(step < most ? step : most);
    return p;
  }
  place(0, summed ? 1 : 0);
  const size_t per = (size_t)planes * (p.cut_users ? all_up : N) * 2 * 256 + (bias ? (p.cut_users ? (size_t)all_up * 32 : (size_t)ceil_div64(N, 32) * 1024) : 0);
  int64_t c = room > p.bytes && per ? (int64_t)((room - p.bytes) / per) * 256 : 0;      // per 0: the loss alone
  if (c > most) c = most;
  if (c < 256) c = 256;
  // Pieces of about equal size: as few as fit or up to half as many again, whichever count deals their units out most evenly (a piece costs
  // its launches, some 16 blocks).  4096 users, 100 000 items of 768: four pieces leave the pairs 3 % idle, three 6 %, five 9 %.
  const int64_t few = ceil_div64(axis, c);
  double least = 1e300;
  for (int64_t pieces = few; pieces <= few + few / 2 && pieces <= few + 4; ++pieces) {
    const int64_t size = ceil_div64(ceil_div64(axis, pieces), 256) * 256, whole = axis / size, rest = axis - whole * size;
    double time = few == 1 ? 0.0 : whole * (loss_splits(size, all, d, planes, f32, own, summed, !p.cut_users).time + 16);
    if (few > 1 && rest) time += loss_splits(rest, all, d, planes, f32, own, summed, !p.cut_users).time + 16;
    if (time < least) { least = time; c = size; }
  }
  with(c);
  while (p.bytes > room && p.step > 256) with(p.step - 256);
  return p;
}

constexpr int64_t kGoodG = (int64_t)256 << 20;            // bytes of a piece's g

// Few users' logits stay in the context's workspace (32 MB of it at most: they stay in L2), in place of a second product for each piece.
bool loss_few(int64_t N, int32_t V) { return N <= LOSS_FEW && N * (((int64_t)V + 7) / 8 * 8) * (int64_t)sizeof(float) <= (32 << 20); }
// bf16 that g is the sum of: fp32 gradients take one more where users are few and the products short, so that it costs little.
int loss_planes(int64_t N, int32_t V, int32_t d, int grad_dtype) {
  if (grad_dtype == GRAM_BF16) return 1;
  return loss_few(N, V) && ceil_div64(V, 64) * ceil_div(d, PAIR_COLS) <= LOSS_SHORT ? 3 : 2;
}

}  // namespace

void score_loss_workspace(int64_t N, int32_t V, int32_t d, int grad_dtype, size_t* least, size_t* best) {
  const bool f32 = grad_dtype == GRAM_F32;
  const int planes = loss_planes(N, V, d, grad_dtype);
  const int64_t n = N > 0 ? N : 1, all_up = ((n > V ? (int64_t)V : n) + 255) / 256 * 256;
  LossPlan p = loss_plan(n, V, d, planes, f32, true, true, true, 256, 0);
  *least = p.bytes - up((size_t)p.splits * all_up * d * 4) + up((size_t)all_up * d * 4);      // with one part of the summed gradient
  int64_t step = kGoodG / (2 * planes * all_up) / 256 * 256;
  if (step < 256) step = 256;
  p = loss_plan(n, V, d, planes, f32, true, true, true, step, 0);
  *best = p.bytes > *least ? p.bytes : *least;
}

gram_status score_loss_launch(gram_ctx* ctx, const ScoreLoss& a, void* ws, size_t ws_bytes, void* score_ws, size_t score_ws_bytes, cudaStream_t st) {
  const bool grads = a.dusers || a.ditems || a.dbias;
  const bool f32 = a.grad_dtype == GRAM_F32;
  const int planes = a.dusers || a.ditems ? loss_planes(a.N, a.V, a.d, a.grad_dtype) : 0;
  const LossPlan p = loss_plan(a.N, a.V, a.d, planes, f32, a.dusers != nullptr, a.ditems != nullptr, a.dbias != nullptr, 0, ws_bytes ? ws_bytes : 1);
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
  RowRest* rest = a.dusers && !p.cut_users ? (RowRest*)(base + p.rest) : nullptr;
  bf16* clean = a.ditems ? (bf16*)(base + p.clean) : nullptr;
  const int64_t ldz = ((int64_t)a.V + 7) / 8 * 8;
  const bool few = grads && loss_few(a.N, a.V);
  const bool by_lanes = few && (a.dusers || a.ditems) && a.N <= LO_USERS && a.d <= 65535 * 256;      // columns that a grid's second dimension counts
  const bool by_rows = few && !by_lanes && !a.dbias && a.V <= LR_THREADS * LR_EACH && p.step >= (p.cut_users ? a.N : (int64_t)a.V);
  if (few) {
    GRAM_TRY(score_logits_launch(ctx, a.users, a.ld_users, a.items, a.ld_items, a.bias, a.N, a.V, a.d, (float*)score_ws, ldz, st));
    if (!by_rows) GRAM_TRY(logprobs_launch(ctx, score_ws, GRAM_F32, ldz, a.N, a.V, a.scale, ask, st));
  } else {
    GRAM_TRY(score_logprobs_launch(ctx, a.users, a.ld_users, a.items, a.ld_items, a.bias, a.N, a.V, a.d, a.scale, ask, score_ws, score_ws_bytes, st));
    ProfScope prof(ctx, GRAM_K_OTHER, (double)a.N * (32 + (clean ? 4.0 * a.d : 0.0)), 1, st, "loss_rows");
    launch_chain(loss_rows_kernel, dim3((unsigned)ceil_div64(a.N, 8)), 256, 0, st, a, (const float*)logp, (const float2*)stats, rows, rest, clean,
                 gram_status_word(ctx));
    GRAM_LAUNCH_CHECK(ctx);
  }
  if (!grads) return GRAM_OK;
  if (by_lanes) {
    // chunks of items: eight blocks an SM or more, no more parts of dU than have room
    const int32_t columns = ceil_div(a.d, 256);
    const int64_t most = a.dusers ? (int64_t)((p.bias - p.parts) / ((size_t)a.N * a.d * 4)) : INT32_MAX;
    int64_t chunks = ceil_div64(8 * kNumSMs, columns);
    if (chunks < ceil_div64(a.V, LO_CHUNK)) chunks = ceil_div64(a.V, LO_CHUNK);
    if (chunks > ceil_div64(a.V, 32)) chunks = ceil_div64(a.V, 32);
    if (chunks > most) chunks = most;
    if (chunks >= ceil_div64(a.V, LO_CHUNK)) {
      const int32_t chunk = (int32_t)ceil_div64(a.V, chunks);
      chunks = ceil_div64(a.V, chunk);
      const int32_t wide = (uintptr_t)a.ditems % 32 == 0 && a.ld_ditems % 8 == 0;
      const OneArgs f{(const float*)score_ws, ldz, logp, stats, chunk, wide, (float*)(base + p.parts), gram_status_word(ctx)};
      const dim3 grid((unsigned)chunks, (unsigned)columns);
      {
        ProfScope prof(ctx, GRAM_K_OTHER, (double)a.V * a.d * (2 + (f32 ? 4 : 2)), 1, st, "loss_one");
        auto kern = f32 ? (a.N == 1 ? loss_one_kernel<float, 1> : a.N == 2 ? loss_one_kernel<float, 2> : loss_one_kernel<float, 4>)
                        : (a.N == 1 ? loss_one_kernel<bf16, 1> : a.N == 2 ? loss_one_kernel<bf16, 2> : loss_one_kernel<bf16, 4>);
        launch_chain(kern, grid, 256, 0, st, a, f);
        GRAM_LAUNCH_CHECK(ctx);
      }
      if (a.dusers) {
        ProfScope prof(ctx, GRAM_K_OTHER, (double)chunks * a.N * a.d * 4, 1, st, "loss_finish");
        const dim3 all((unsigned)ceil_div(a.d, 32), (unsigned)a.N);
        if (f32) launch_chain(loss_one_finish_kernel<float>, all, 1024, 0, st, (const float*)f.parts, (int32_t)chunks, a.d, a.N * a.d, (float*)a.dusers, a.ld_dusers);
        else launch_chain(loss_one_finish_kernel<bf16>, all, 1024, 0, st, (const float*)f.parts, (int32_t)chunks, a.d, a.N * a.d, (bf16*)a.dusers, a.ld_dusers);
        GRAM_LAUNCH_CHECK(ctx);
      }
      return GRAM_OK;
    }
  }

  const char* what = "gram_score_loss: cannot describe the vectors";
  CUtensorMap map_u, map_i, map_clean, map_g[3], map_out[2];
  int box_rows = PAIR_ROWS;                              // copies are no larger than the users
  while (box_rows > 8 && box_rows / 2 >= a.N) box_rows /= 2;
  if ((!few && !make_map(&map_u, a.users, (uint64_t)a.d, (uint64_t)a.N, (uint64_t)a.ld_users, 64, (uint32_t)box_rows)) ||
      !make_map(&map_i, a.items, (uint64_t)a.d, (uint64_t)a.V, (uint64_t)a.ld_items, 64, 64))
    return gram_set_error(ctx, what), GRAM_ERR_UNSUPPORTED;
  map_clean = map_i;
  if (clean && !make_map(&map_clean, clean, (uint64_t)a.d, (uint64_t)a.N, (uint64_t)a.d, 64, 64)) return gram_set_error(ctx, what), GRAM_ERR_UNSUPPORTED;

  const int64_t axis = p.cut_users ? a.N : a.V, pieces = ceil_div64(axis, p.step);
  const int own = p.cut_users ? 0 : 1;                   // whose gradient is done with the piece
  const bool joined = p.splits > 0 && (p.splits > 1 || pieces > 1 || own == 1);      // the users' always: what is left of their targets is added there
  auto join_bias = [&](const Piece& e, int64_t blocks) -> gram_status {
    ProfScope prof(ctx, GRAM_K_COLSUM, 4.0 * blocks * e.cols, 1, st, "loss_bias");
    launch_chain(loss_bias_kernel, dim3((unsigned)ceil_div(e.cols, 32)), 256, 0, st, (const float*)(base + p.bias), p.ldg, blocks, e.cols, (int32_t)(e.n0 > 0),
                 a.dbias + e.first);
    GRAM_LAUNCH_CHECK(ctx);
    return GRAM_OK;
  };
  for (int64_t i = 0; i < pieces; ++i) {
    const int64_t at = i * p.step, now = axis - at < p.step ? axis - at : p.step;
    Piece e;
    e.n0 = p.cut_users ? at : 0;
    e.rows = p.cut_users ? now : a.N;
    e.first = p.cut_users ? 0 : (int32_t)at;
    e.cols = p.cut_users ? a.V : (int32_t)now;
    e.g = (bf16*)(base + p.g);
    e.ldg = p.ldg;
    e.plane = e.rows * p.ldg;
    if (few) {
      const FewArgs f{e, (const float*)score_ws, ldz, logp, stats, clean, rest, (float*)(base + p.bias), gram_status_word(ctx)};
      ProfScope prof(ctx, GRAM_K_OTHER, (4.0 + 2 * planes) * e.rows * e.cols, 1, st, "loss_few");
      if (by_rows)
        launch_chain(planes == 3 ? loss_row_kernel<3> : planes == 2 ? loss_row_kernel<2> : loss_row_kernel<1>, dim3((unsigned)a.N), LR_THREADS, 0, st, a, f);
      else
        launch_chain(planes == 3 ? loss_few_kernel<3> : planes == 2 ? loss_few_kernel<2> : planes == 1 ? loss_few_kernel<1> : loss_few_kernel<0>, dim3((unsigned)ceil_div(e.cols, 128), (unsigned)ceil_div64(e.rows, LOSS_FEW_ROWS)), 256, 0, st, a, f);
      GRAM_LAUNCH_CHECK(ctx);
      if (a.dbias && e.rows > LOSS_FEW_ROWS) GRAM_TRY(join_bias(e, ceil_div64(e.rows, LOSS_FEW_ROWS)));
    } else {
      GradArgs f = {};
      f.at = e;
      f.rows = rows;
      f.rest = rest;
      f.bias = a.bias;
      f.V = a.V;
      f.num_kb = ceil_div(a.d, 64);
      f.tiles_m = (int32_t)ceil_div64(e.rows, 2 * PAIR_ROWS);
      f.width = (int64_t)f.tiles_m * ceil_div(e.cols, PAIR_COLS) < kPairs ? PAIR_COLS / 2 : PAIR_COLS;    // tiles of half the width where they leave pairs idle
      const int32_t tiles = f.tiles_m * ceil_div(e.cols, f.width), last = tiles % kPairs;
      f.whole = f.width == PAIR_COLS && last > 0 && 2 * last <= kPairs ? tiles - last : tiles;
      f.total = f.whole + 2 * (tiles - f.whole);
      f.box_rows = box_rows;
      f.c = a.scale * kLog2e;
      f.bias_part = a.dbias ? (float*)(base + p.bias) : nullptr;
      f.give_up = gram_ring_rows(ctx);
      f.status = gram_status_word(ctx);
      {
        ProfScope prof(ctx, GRAM_K_GEMM, 2.0 * e.rows * e.cols * a.d, 1, st, "loss_grad");
        const int pairs = f.total < kPairs ? f.total : kPairs;
        if (planes == 2) GRAM_CUDA(ctx, launch_pairs<loss_grad_kernel<2>>(pairs, GradPipe::THREADS, GradPipe::SMEM, st, map_u, map_i, f));
        else if (planes == 0) GRAM_CUDA(ctx, launch_pairs<loss_grad_kernel<0>>(pairs, GradPipe::THREADS, GradPipe::SMEM, st, map_u, map_i, f));
        else GRAM_CUDA(ctx, launch_pairs<loss_grad_kernel<1>>(pairs, GradPipe::THREADS, GradPipe::SMEM, st, map_u, map_i, f));
      }
      if (a.dbias) GRAM_TRY(join_bias(e, ceil_div64(e.rows, 32)));
    }
    if (!a.dusers && !a.ditems) continue;
    for (int k = 0; k < planes; ++k)
      if (!make_map(&map_g[k], e.g + k * e.plane, (uint64_t)e.cols, (uint64_t)e.rows, (uint64_t)p.ldg, 64, 64))
        return gram_set_error(ctx, what), GRAM_ERR_UNSUPPORTED;
    for (int k = planes; k < 3; ++k) map_g[k] = map_g[0];
    ProdArgs w = {};
    const size_t size = f32 ? 4 : 2;
    w.d = a.d;
    w.tiles_n = ceil_div(a.d, PAIR_COLS);
    for (int k = 0; k < 2; ++k) {
      ProdSide& o = w.of[k];
      void* grad = k ? a.ditems : a.dusers;
      const int64_t ld = k ? a.ld_ditems : a.ld_dusers;
      o.rows = (int32_t)(k ? e.cols : e.rows);
      o.tiles_m = grad ? ceil_div(o.rows, 2 * PAIR_ROWS) : 0;
      o.kb = (int32_t)ceil_div64(k ? e.rows : e.cols, 64);
      // the last piece may have fewer parts; the sums of the others stay
      o.kb_split = k == own || p.splits == 0 ? o.kb : ceil_div(o.kb, p.splits);
      o.vec0 = (int32_t)(k ? e.n0 : e.first);
      o.units = o.tiles_m * w.tiles_n * ceil_div(o.kb, o.kb_split);
      o.partial = k != own && joined;
      o.add = i > 0;
      o.part = (o.rows + 255) / 256 * 256;
      if (grad) {                                        // boxes of 32 rows x 128 bytes; those of a part end with the part's last tile
        uint8_t* to = o.partial ? base + p.parts : (uint8_t*)grad + (size_t)(k ? e.first : e.n0) * ld * size;
        const uint64_t out_rows = o.partial ? (uint64_t)p.splits * o.part : (uint64_t)o.rows, out_ld = o.partial ? (uint64_t)a.d : (uint64_t)ld;
        if (!(o.partial || f32 ? make_map_f32(&map_out[k], to, (uint64_t)a.d, out_rows, out_ld, 32, 32)
                                       : make_map(&map_out[k], to, (uint64_t)a.d, out_rows, out_ld, 64, 32)))
          return gram_set_error(ctx, "gram_score_loss: cannot describe the gradients"), GRAM_ERR_UNSUPPORTED;
      } else {
        map_out[k] = map_i;
      }
      o.cost = (int32_t)loss_cost(o.kb_split, planes, o.partial || f32);
    }
    const LossSpan span = loss_span(w.of[0].units, w.of[0].cost, w.of[1].units, w.of[1].cost);
    w.heavy = span.heavy;
    w.extra = span.extra;
    w.halves = span.halves;
    w.total = w.of[0].units + w.of[1].units;
    w.chain = f32 ? LP_CHAIN : LP_CHAIN_BF16;
    w.give_up = gram_ring_rows(ctx);
    w.status = gram_status_word(ctx);
    ProfScope prof(ctx, GRAM_K_GEMM, 2.0 * planes * e.rows * e.cols * a.d * ((a.dusers != nullptr) + (a.ditems != nullptr)), 1, st, "loss_products");
    const int pairs = w.total < kPairs ? w.total : kPairs;
#define LOSS_PRODUCTS(GT, PLANES, CHAINED)                                                                                                            \
  launch_pairs<loss_products_kernel<GT, PLANES, CHAINED>>(pairs, ProdPipe<PLANES, CHAINED>::THREADS, ProdPipe<PLANES, CHAINED>::SMEM, st, map_g[0], map_g[1], \
                                                          map_g[2], map_clean, map_i, map_out[0], map_out[1], w)
    const bool chained = (w.of[0].units && w.of[0].kb_split > LP_CHAIN_BF16) || (w.of[1].units && w.of[1].kb_split > LP_CHAIN_BF16);
    if (planes == 1 && !chained) GRAM_CUDA(ctx, LOSS_PRODUCTS(bf16, 1, false));
    else if (planes == 1) GRAM_CUDA(ctx, LOSS_PRODUCTS(bf16, 1, true));
    else if (planes == 2) GRAM_CUDA(ctx, LOSS_PRODUCTS(float, 2, true));
    else GRAM_CUDA(ctx, LOSS_PRODUCTS(float, 3, true));
#undef LOSS_PRODUCTS
  }
  if (joined) {
    void* grad = own ? a.dusers : a.ditems;
    const int64_t n = own ? a.N : a.V, ld = own ? a.ld_dusers : a.ld_ditems, part = (n + 255) / 256 * 256 * a.d;
    ProfScope prof(ctx, GRAM_K_OTHER, (double)n * a.d * 4 * (p.splits + 1), 1, st, "loss_finish");
    const float* parts = (const float*)(base + p.parts);
    int64_t blocks = ceil_div64(n * (a.d / 4), 256);
    if (blocks > kNumSMs * 8) blocks = kNumSMs * 8;
    const RowRest* left = own ? rest : nullptr;
    if (f32) launch_chain(loss_finish_kernel<float>, dim3((unsigned)blocks), 256, 0, st, parts, (int)p.splits, part, n, a.d, left, (const bf16*)a.items, a.ld_items, (float*)grad, ld);
    else launch_chain(loss_finish_kernel<bf16>, dim3((unsigned)blocks), 256, 0, st, parts, (int)p.splits, part, n, a.d, left, (const bf16*)a.items, a.ld_items, (bf16*)grad, ld);
    GRAM_LAUNCH_CHECK(ctx);
  }
  return GRAM_OK;
}
