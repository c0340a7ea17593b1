// Answers over an item table from the vectors themselves (gram_score_logprobs).
//
// The product users x items^T runs on pairs of SMs (tcgen05 cta_group::2) as in gemm.cu: a cluster of two blocks owns a tile
// of 256 users x 256 items, each stages its own 128 users and its own half of the items by TMA, the leader issues the MMAs,
// and each block's tensor memory receives 128 users' logits, two tiles in turn.  The logits never leave it: an epilogue
// thread owns one user (a lane of tensor memory) and a quarter of a tile's columns and keeps the softmax statistics of what it
// has seen in registers.
//
// Alternatives take a first pass over a part of the items (score_kernel<SAMPLE>), units of 128 spread over the table, which
// writes the maxima of groups of 8 or 32 columns; score_bar_kernel takes from them a bar that at least k entries of a user
// reach, and in the main pass a thread puts entries that reach its user's bar on a list of its own.  With a sample of S items
// about k V / S entries of a user do.  A sum of products is the same to the bit in both passes: it is formed in the order of d
// whatever the tile's width and the item's place in it.
//
// Work is cut evenly: the units of 128 items of all row tiles, one row tile after another, are divided into contiguous
// runs, one for each pair.  A run touches at most two row tiles, so a user's statistics and lists lie with a few pairs;
// score_join_kernel joins them.
//
// Where logits are few they are written after all (score_kernel<LOGITS>) and gram_logprobs' kernel reads them.
//
// Bounded by the products where users are many, by the table's bytes where they are few.  Measured against 100 000 items of 768 (8-bit
// codes; calls in a chain, on two tables in turn): 4096 users 373 us (1690 TFLOP/s), with 10 alternatives 475 to 500, on the same
// inputs 454, among calls whose inputs all differ 520; 1024 users 105 and 149; 64 users with 10 alternatives 46, one user 40 (the
// table's 154 MB at 6458 GB/s: 24).  Vectors of normal values take more power: 4096 users 400 and 515.  Where all scores are equal, so
// that lists are cut again and again, 4096 users with 10 alternatives take 1320, with 50 2350.
#include "logits.h"
#include "row_softmax.cuh"
#include "row_top.cuh"
#include "tc_common.cuh"

namespace {
using namespace tc;

constexpr int SM_ROWS = 128, SC_ROWS = 2 * SM_ROWS;     // users of a block and of a pair
constexpr int SC_BK = 64, SC_UNIT = 128, SC_COLS = 256; // k of a stage, items of a unit and of the widest tile
constexpr int SC_A_BYTES = SM_ROWS * SC_BK * 2, SC_B_BYTES = SC_COLS / 2 * SC_BK * 2, SC_STAGE = SC_A_BYTES + SC_B_BYTES;
constexpr int SC_STAGES = 6, SC_EPI_WARPS = 16, SC_THREADS = 64 + 32 * SC_EPI_WARPS;
constexpr int SC_PARTS = SC_EPI_WARPS / 4;              // parts of a tile's columns, each with its warps
constexpr int SC_BIAS_BYTES = SC_EPI_WARPS * 64 * 4;    // a warp's columns
constexpr int SC_SMEM = SC_STAGES * SC_STAGE + SC_BIAS_BYTES + 1024 + 256;
constexpr int SC_LIST_MAX = 256;                        // most entries of a thread's list
constexpr int SC_PAIR_THREADS = SC_PARTS * SC_ROWS;     // epilogue threads of a pair, one for each user and part
constexpr int SB_ROWS = 8, SB_GROUPS = 1024;            // score_bar_kernel: rows of a block, most groups of a row

enum ScoreMode { STATISTICS = 0, LISTS = 1, SAMPLE = 2, LOGITS = 3 };   // LISTS: statistics too

struct ScoreArgs {
  const float* bias;
  int64_t N;
  int32_t V, num_kb, k, cap;     // V: items of this pass; cap: entries that a list holds
  int32_t units, total, per_run; // units of a row tile, of all, of a pair's run
  int32_t box_rows;              // users of a copy
  float c;
  const float* bars;             // [N]
  uint64_t* lists;               // [pair, part, row of the tile, cap]
  uint64_t* early;               // [row tile, part, row, early_cap]: of the run that goes on with the next row tile
  int32_t early_cap;
  float4* stats;                 // [pair, row tile of the run (0, 1), part, row]: m, s, t, entries of the list
  float* logits;                 // LOGITS: [N, ld_logits], a multiple of 8
  int64_t ld_logits;
  float* sample;                 // maxima: [block of 32 columns, row] float4 of groups of 8, or one float
  int64_t sample_rows;
  int32_t fine;                  // groups of 8
  int32_t stride;                // the pass takes every stride-th two units of the table
  int32_t give_up;               // tile of a run at which its copies stop (gram_selftest_ring_rows)
  int32_t* status;
};

// The tiles of a run, as all roles walk over them.  A run is as long as all others, so it holds every residue of the unit's number
// modulo that length once; it begins with residue 0 and turns to its start at its end.  All pairs are then at units of about the
// same residue at any time, and the row tiles' reads of the table meet in L2: 1024 users against 100 000 items of 768 with 10
// alternatives 165 us from end to end of the run and 149 so, 4096 users 490 and 454 (calls one after another on the same inputs).
struct ScoreRun {
  int units, stride, per_run, begin, at, end;    // at: what lies ahead of the current row tile's part
  int lo, turn, stop;            // the part's first unit, where it begins, where its current piece ends
  int tm, unit, width;           // row tile, first unit and width in units of the current tile
  bool first, last, turned;      // of the run's part of this row tile; turned: the places are below those seen before
  __device__ __forceinline__ ScoreRun(const ScoreArgs& a, int pair)
      : units(a.units), stride(a.stride), per_run(a.per_run), begin(pair * a.per_run), at(begin), end(min(begin + a.per_run, a.total)), lo(0), turn(0),
        stop(0), tm(0), unit(0), width(0), first(false), last(false), turned(false) {}
  __device__ __forceinline__ bool next() {
    unit += width;
    if (unit == stop) {
      turned = !turned && turn > lo;
      if (turned) {
        unit = lo;
        stop = turn;
      } else {
        if (at >= end) return false;
        tm = at / units;
        lo = at - tm * units;
        stop = min(units, lo + end - at);
        at += stop - lo;
        turn = (lo + per_run - 1) / per_run * per_run;
        if (turn >= stop) turn = lo;
        unit = turn;
      }
    }
    const int left = stop - unit;
    width = min(left, stride > 1 && (unit & 1) ? 1 : SC_COLS / SC_UNIT);
    first = unit == turn;
    last = left == width && (turned || turn == lo);
    return true;
  }
  __device__ __forceinline__ int column() const { return ((unit >> 1) * stride * 2 + (unit & 1)) * SC_UNIT; }   // first item
  __device__ __forceinline__ int part() const { return tm - begin / units; }             // 0, or 1 for the second row tile
  __device__ __forceinline__ bool leaves() const { return (end - 1) / units != tm; }     // the run goes on with another row tile
};

// a list cut to its best k by the whole warp; returns (in every lane) the bar of the entries that follow, at places of `from` on
__device__ __noinline__ float score_cut(uint64_t* list, int have, int k, uint32_t from) { return warp_cut(list, have, k, from); }

// a block of 32 columns of this thread's row as it left tensor memory, plus the bias (the warp's 32 values in shared memory)
__device__ __forceinline__ void score_bias(uint32_t (&v)[32], const float* b) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float4 f = reinterpret_cast<const float4*>(b)[j];
    v[4 * j] = __float_as_uint(__uint_as_float(v[4 * j]) + f.x);
    v[4 * j + 1] = __float_as_uint(__uint_as_float(v[4 * j + 1]) + f.y);
    v[4 * j + 2] = __float_as_uint(__uint_as_float(v[4 * j + 2]) + f.z);
    v[4 * j + 3] = __float_as_uint(__uint_as_float(v[4 * j + 3]) + f.w);
  }
}
// the maxima of its four groups of 8 columns
__device__ __forceinline__ void score_tops(const uint32_t (&v)[32], float (&t)[4]) {
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = __uint_as_float(v[8 * g + j]);
    t[g] = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
  }
}
__device__ __forceinline__ void score_add(RowSums& r, const uint32_t (&v)[32], float top, float c) {
  r.see(top, c);
  f32x2 s = x2_pack(0.f, 0.f), t = s;                    // sums of their own: small terms would be lost in the row's so far
  const f32x2 cc = x2_pack(c, c), ref = x2_pack(-r.ref, -r.ref);
#pragma unroll
  for (int j = 0; j < 32; j += 2) {
    const f32x2 y = x2_fma(row_held(__uint_as_float(v[j]), __uint_as_float(v[j + 1])), cc, ref);
    const float2 y2 = x2_unpack(y);
    const f32x2 e = x2_pack(row_ex2(y2.x), row_ex2(y2.y));
    s = x2_add(s, e);
    t = x2_fma(e, y, t);
  }
  const float2 s2 = x2_unpack(s), t2 = x2_unpack(t);
  r.s += s2.x + s2.y;
  r.t += t2.x + t2.y;
}
// The entries of a block that reach the bar, to the lanes' lists (those of a warp `cap` apart): a bit for each of a group of 8, then
// one entry of each lane at a time.  A list without room for another group is cut to its best k first.
__device__ __forceinline__ void score_list(const uint32_t (&v)[32], const float (&t)[4], float& bar, uint32_t col, uint64_t* warp_lists, int cap, int k,
                                           int& have) {
  const int lane = threadIdx.x & 31;
  uint64_t* list = warp_lists + (int64_t)lane * cap;
  const uint32_t groups = __reduce_or_sync(0xffffffffu, (t[0] >= bar ? 1u : 0u) | (t[1] >= bar ? 2u : 0u) | (t[2] >= bar ? 4u : 0u) | (t[3] >= bar ? 8u : 0u));
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    if (!(groups & (1u << g))) continue;
    uint32_t full = __ballot_sync(0xffffffffu, have > cap - 8);
    while (full) {
      const int of = __ffs(full) - 1;
      full &= full - 1;
      __syncwarp();
      const float up = score_cut(warp_lists + (int64_t)of * cap, __shfl_sync(0xffffffffu, have, of), k, col + 8 * g);
      if (lane == of) { have = k; bar = up; }
    }
    uint32_t bits = 0u;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (__uint_as_float(v[8 * g + j]) >= bar) bits |= 1u << j;
    do {
      if (bits) {
        const int j = __ffs(bits) - 1;
        bits &= bits - 1u;
        const uint32_t a = j & 1 ? v[8 * g + 1] : v[8 * g], b = j & 1 ? v[8 * g + 3] : v[8 * g + 2];
        const uint32_t c = j & 1 ? v[8 * g + 5] : v[8 * g + 4], d = j & 1 ? v[8 * g + 7] : v[8 * g + 6];
        const uint32_t ab = j & 2 ? b : a, cd = j & 2 ? d : c;
        list[have++] = row_key(__uint_as_float(j & 4 ? cd : ab), col + 8 * g + j);
      }
    } while (__any_sync(0xffffffffu, bits != 0u));
  }
}

template <int MODE>
__global__ void __launch_bounds__(SC_THREADS, 1) score_kernel(const __grid_constant__ CUtensorMap users, const __grid_constant__ CUtensorMap items,
                                                              const __grid_constant__ ScoreArgs a) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t tiles = (raw + 1023u) & ~1023u;        // the same offset in both blocks of the pair
  float* bias_s = reinterpret_cast<float*>(smem_raw + (tiles - raw) + SC_STAGES * SC_STAGE);
  const uint32_t bar0 = tiles + SC_STAGES * SC_STAGE + SC_BIAS_BYTES;
  auto full_bar = [&](int s) { return bar0 + 8u * s; };                            // used in the leader
  auto empty_bar = [&](int s) { return bar0 + 8u * (SC_STAGES + s); };             // one per block
  auto tfull_bar = [&](int b) { return bar0 + 8u * (2 * SC_STAGES + b); };         // one per block
  auto tempty_bar = [&](int b) { return bar0 + 8u * (2 * SC_STAGES + 2 + b); };    // used in the leader
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem_raw + (bar0 - raw) + 8 * (2 * SC_STAGES + 4));
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  if (threadIdx.x == 0) {
    for (int s = 0; s < SC_STAGES; ++s) {
      mbar_init(full_bar(s), 2);                        // the two blocks' copies, each with its byte count
      mbar_init(empty_bar(s), 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(tfull_bar(b), 1);
      mbar_init(tempty_bar(b), 2 * SC_EPI_WARPS);
    }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  gram_cluster_sync();                                  // both blocks' barriers exist before anyone signals them
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  const bool go = chain_begin();
  const int pair = blockIdx.x >> 1;
  bool failed = false;
  ScoreRun run(a, pair);

  if (warp == 0 && go) {
    // ------------------------------ copies (both blocks) ------------------------------
    int s = 0;
    uint32_t ph = 0;
    const uint32_t lead_bar0 = map_to_cta(bar0, 0);
    for (int tile = 0; !failed && run.next(); ++tile) {
      if (tile == a.give_up) { failed = true; break; }
      const int m0 = run.tm * SC_ROWS + (int)rank * SM_ROWS;
      const int n0 = run.column() + (int)rank * (run.width * SC_UNIT / 2);     // this block's half of the items: boxes of 64
      // a block whose users are all past the last fetches none; what its rows of the product hold is not looked at
      const bool some = m0 < a.N;
      const uint32_t bytes = (some ? (uint32_t)a.box_rows * (SC_BK * 2) : 0u) + (uint32_t)run.width * (SC_UNIT / 2 * SC_BK * 2);
      for (int kb = 0; kb < a.num_kb; ++kb) {
        if (!mbar_wait_warp(empty_bar(s), ph ^ 1u, abort_flag)) { failed = true; break; }
        const uint32_t lead_full = lead_bar0 + 8u * s;
        const uint32_t sa = tiles + s * SC_STAGE, sb = sa + SC_A_BYTES;
        if (elect_one()) {
          mbar_arrive_expect_tx_remote(lead_full, bytes);
          if (some) tma_load_2d_pair(sa, &users, kb * SC_BK, m0, lead_full);
          tma_load_2d_pair(sb, &items, kb * SC_BK, n0, lead_full);
          if (run.width == 2) tma_load_2d_pair(sb + 8192, &items, kb * SC_BK, n0 + 64, lead_full);
        }
        __syncwarp();
        if (++s == SC_STAGES) { s = 0; ph ^= 1u; }
      }
    }
  } else if (warp == 1 && go) {
    // ------------------------------ products (leader) ------------------------------
    if (rank == 0) {
      constexpr uint32_t idesc0 = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(SC_ROWS >> 4) << 24);
      int s = 0;
      uint32_t ph = 0, it = 0;
      const uint64_t da0 = make_desc(tiles, 16, 1024), db0 = make_desc(tiles + SC_A_BYTES, 16, 1024);
      while (!failed && run.next()) {
        const uint32_t idesc = idesc0 | ((uint32_t)(run.width * SC_UNIT >> 3) << 17);
        const int buf = (int)(it & 1);
        if (!mbar_wait_warp(tempty_bar(buf), ((it >> 1) & 1) ^ 1u, abort_flag)) { failed = true; break; }
        tc_fence_after();
        const uint32_t tmem_d = tmem_base + (uint32_t)(buf * SC_COLS);
        for (int kb = 0; kb < a.num_kb; ++kb) {
          if (!mbar_wait_warp(full_bar(s), ph, abort_flag)) { failed = true; break; }
          tc_fence_after();
          const uint32_t soff = (uint32_t)(s * (SC_STAGE >> 4));
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < SC_BK / 16; ++k)
              tc_mma_pair(tmem_d, da0 + soff + (uint64_t)(k * 2), db0 + soff + (uint64_t)(k * 2), idesc, (kb > 0 || k > 0) ? 1u : 0u);
            tc_commit_pair(empty_bar(s));
            if (kb == a.num_kb - 1) tc_commit_pair(tfull_bar(buf));
          }
          __syncwarp();
          if (++s == SC_STAGES) { s = 0; ph ^= 1u; }
        }
        ++it;
      }
    }
  } else if (go) {
    // ------------------------------ statistics and lists (both blocks) ------------------------------
    const int q = warp & 3, part = (warp - 2) >> 2;
    const int row = (int)rank * SM_ROWS + q * 32 + lane;          // of the pair's tile
    float* bias_w = bias_s + (warp - 2) * 64;
    uint64_t* warp_lists = a.lists + ((int64_t)(pair * SC_PARTS + part) * SC_ROWS + (row - lane)) * a.cap;
    const uint32_t lane_addr = tmem_base + ((uint32_t)(q * 32) << 16);
    RowSums sums;
    int have = 0;
    float bar = 0.f;
    uint32_t it = 0;
    const uint32_t lead_tempty = map_to_cta(tempty_bar(0), 0);
    for (; !failed && run.next(); ++it) {
      const int buf = (int)(it & 1), blocks = run.width;          // blocks of 32 columns of this part
      const int col_t = part * blocks * 32, col0 = run.column() + col_t;
      const int64_t n = (int64_t)run.tm * SC_ROWS + row;
      const bool active = n - lane < a.N;                         // of the warp
      // columns past the table count as masked out
      const float* bias = nullptr;
      if (active && (a.bias || col0 + blocks * 32 > a.V)) {
        for (int b = 0; b < blocks; ++b) {
          const int v = col0 + b * 32 + lane;
          bias_w[b * 32 + lane] = v >= a.V ? ROW_NEG_INF : a.bias ? __ldg(a.bias + v) : 0.f;
        }
        __syncwarp();
        bias = bias_w;
      }
      if (!mbar_wait_warp(tfull_bar(buf), (it >> 1) & 1, abort_flag)) { failed = true; break; }
      tc_fence_after();
      if (active) {
        const uint32_t taddr = lane_addr + (uint32_t)(buf * SC_COLS + col_t);
        if (MODE <= LISTS && run.first) {
          sums = RowSums();
          have = 0;
          if (MODE == LISTS) bar = n < a.N ? a.bars[n] : __int_as_float(0x7fffffff);     // nothing reaches a NaN
        }
        // Behind the turn places are lower than those of the list, and of equal logits the lower place is the better one: a cut list's bar,
        // the next value above its least logit, goes back to that logit.
        if (MODE == LISTS && run.turned && run.unit == run.lo && n < a.N) bar = fmaxf(a.bars[n], row_order_logit(row_order(bar) - 1u));
        for (int b = 0; b < blocks; ++b) {
          uint32_t v[32];
          tc_ld32_issue(taddr + b * 32, v);
          tc_ld32_wait(v);
          if (bias) score_bias(v, bias + b * 32);
          if constexpr (MODE == LOGITS) {
            const int col = col0 + b * 32;
            if (n < a.N) {
              float* to = a.logits + n * a.ld_logits + col;
#pragma unroll
              for (int j = 0; j < 32; j += 8)                      // whole 32-byte sectors; a row's last may reach past the table
                if (col + j < a.V)
                  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to + j), "r"(v[j]), "r"(v[j + 1]), "r"(v[j + 2]),
                               "r"(v[j + 3]), "r"(v[j + 4]), "r"(v[j + 5]), "r"(v[j + 6]), "r"(v[j + 7])
                               : "memory");
            }
          } else {
            float t[4];
            score_tops(v, t);
            const float top = fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]));
            if constexpr (MODE == SAMPLE) {
              const int64_t at = (int64_t)((run.unit * SC_UNIT + col_t + b * 32) / 32) * a.sample_rows + n;
              if (a.fine) reinterpret_cast<float4*>(a.sample)[at] = make_float4(t[0], t[1], t[2], t[3]);
              else a.sample[at] = top;
            } else {
              score_add(sums, v, top, a.c);
              if (MODE == LISTS && __any_sync(0xffffffffu, top >= bar))
                score_list(v, t, bar, (uint32_t)(col0 + b * 32), warp_lists, a.cap, a.k, have);
            }
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_remote(lead_tempty + 8u * buf);
      if (MODE <= LISTS && active && run.last) {
        const RowStat r = sums.stat(a.c);
        if constexpr (MODE == LISTS) {
          if (run.leaves()) {                                     // the lists are needed again: these go elsewhere
            uint64_t* to = a.early + ((int64_t)(run.tm * SC_PARTS + part) * SC_ROWS + (row - lane)) * a.early_cap;
            __syncwarp();
            for (int of = 0; of < 32; ++of) {
              uint64_t* from = warp_lists + (int64_t)of * a.cap;
              int n_of = __shfl_sync(0xffffffffu, have, of);
              if (n_of > a.early_cap) {
                (void)score_cut(from, n_of, a.k, 0u);
                n_of = a.k;
                if (lane == of) have = n_of;
              }
              for (int i = lane; i < n_of; i += 32) to[(int64_t)of * a.early_cap + i] = from[i];
            }
            __syncwarp();
          }
        }
        a.stats[((int64_t)(pair * 2 + run.part()) * SC_PARTS + part) * SC_ROWS + row] = make_float4(r.m, r.s, r.t, __int_as_float(have));
      }
    }
  }
  if (failed && lane == 0) {
    *abort_flag = 1;
    gram_device_fail(a.status, GRAM_ERR_TIMEOUT);
  }
  // ------------------------------ teardown ------------------------------
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    if (warp == 1 && lane == 0) {                       // let copies and MMAs already issued drain (bounded)
      const uint64_t t0 = clock64();
      while (clock64() - t0 < WAIT_LIMIT_CYCLES / 64) {}
    }
    __syncthreads();
  }
  gram_cluster_sync();                                  // the peer no longer reads this block's memory or signals its barriers
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
  }
}

// The bar of each user: a value that k of its groups' maxima reach, or a little less; the lowest finite value if they are fewer.
// A block takes 8 rows, a warp each.
__global__ void __launch_bounds__(32 * SB_ROWS) score_bar_kernel(const float* sample, int64_t rows, int32_t blocks, int32_t fine, int64_t N, int32_t k,
                                                                 float* bars) {
  if (!chain_begin()) return;
  __shared__ __align__(16) float value[SB_ROWS][SB_GROUPS + 4];
  const int64_t n0 = (int64_t)blockIdx.x * SB_ROWS;
  const int groups = fine ? 4 * blocks : blocks;
  for (int i = threadIdx.x; i < blocks * SB_ROWS; i += 32 * SB_ROWS) {
    const int r = i % SB_ROWS, b = i / SB_ROWS;
    const int64_t at = (int64_t)b * rows + n0 + r;      // the rows are padded to whole tiles
    if (fine) *reinterpret_cast<float4*>(&value[r][4 * b]) = reinterpret_cast<const float4*>(sample)[at];
    else value[r][b] = sample[at];
  }
  __syncthreads();
  const int lane = threadIdx.x & 31, r = threadIdx.x >> 5;
  if (n0 + r >= N) return;
  uint32_t o[SB_GROUPS / 32], lo = ~0u, hi = 0u;
  int some = 0;
#pragma unroll
  for (int i = 0; i < SB_GROUPS / 32; ++i) {
    o[i] = 0u;
    if (i * 32 < groups) {
      const float x = i * 32 + lane < groups ? value[r][i * 32 + lane] : ROW_NEG_INF;
      if (x > ROW_NEG_INF) {
        o[i] = row_order(x);
        lo = min(lo, o[i]);
        hi = max(hi, o[i]);
        ++some;
      }
    }
  }
  // k of 32 lanes' maxima are above the least of them
  const uint32_t lane_hi = hi;
  lo = __reduce_min_sync(0xffffffffu, lo);
  if (k <= 32) lo = max(lo, __reduce_min_sync(0xffffffffu, lane_hi));
  hi = __reduce_max_sync(0xffffffffu, hi);
  float bar = -FLT_MAX;
  if ((int)__reduce_add_sync(0xffffffffu, some) >= k) {
    for (int step = 0; lo < hi && step < 16; ++step) {
      const uint32_t mid = hi - (hi - lo) / 2;
      int n = 0;
#pragma unroll
      for (int i = 0; i < SB_GROUPS / 32; ++i)
        if (i * 32 < groups) n += o[i] >= mid;
      n = __reduce_add_sync(0xffffffffu, n);
      if (n < k) hi = mid - 1;
      else {
        lo = mid;
        if (n <= k + k / 8) break;
      }
    }
    bar = row_order_logit(lo);
  }
  if (lane == 0) bars[n0 + r] = bar;
}

// users[n] . items[v], by a warp: of M items at once, `apart` elements from one to the next
template <int M> __device__ __forceinline__ void score_dots(const bf16* u, const bf16* w, int64_t apart, int d, float (&sum)[M]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int m = 0; m < M; ++m) sum[m] = 0.f;
  for (int i = lane; i < d / 8; i += 32) {
    const uint4 a = __ldg(reinterpret_cast<const uint4*>(u) + i);
    uint4 b[M];
#pragma unroll
    for (int m = 0; m < M; ++m) b[m] = __ldg(reinterpret_cast<const uint4*>(w + m * apart) + i);
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 x = RowVec<bf16>::pair(a, j), y = RowVec<bf16>::pair(b[m], j);
        sum[m] = fmaf(x.x, y.x, sum[m]);
        sum[m] = fmaf(x.y, y.y, sum[m]);
      }
  }
  if (lane < d % 8) {
    const int i = d / 8 * 8 + lane;
#pragma unroll
    for (int m = 0; m < M; ++m) sum[m] = fmaf(__bfloat162float(u[i]), __bfloat162float(w[m * apart + i]), sum[m]);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
#pragma unroll
    for (int m = 0; m < M; ++m) sum[m] += __shfl_xor_sync(0xffffffffu, sum[m], o);
}

// A user's logits as score_dots sums them, for rows of huge ones (out of line: with this in place the joining took 15 registers more).
// They are taken four at a time, once: of 4096 rows against 100 000 items of 768 in 109 ms (one at a time, once for the largest and once
// for the sums: 255; a call on other rows: 0.5), of 300 rows, a block each, in 10.
struct ScoreRow {
  const bf16 *user, *items;
  const float* bias;
  int64_t ld_i;
  int32_t V, d;
  __device__ __forceinline__ float operator()(int v) const {
    float z[1];
    score_dots<1>(user, items + (int64_t)v * ld_i, 0, d, z);
    return z[0] + (bias ? bias[v] : 0.f);
  }
  // f(logit) of every step-th item of [v, end)
  template <typename F> __device__ __forceinline__ void each(int v, int end, int step, F f) const {
    for (; end - v > 3 * step; v += 4 * step) {
      float z[4];
      score_dots<4>(user, items + (int64_t)v * ld_i, step * ld_i, d, z);
#pragma unroll
      for (int j = 0; j < 4; ++j) f(z[j] + (bias ? bias[v + j * step] : 0.f));
    }
    for (; v < end; v += step) f((*this)(v));
  }
};
__device__ __noinline__ float score_again(const ScoreRow& z, int v) { return z(v); }
// sums of e = 2^y and e y as they are when every y moves by d <= 0
__device__ __forceinline__ void score_raise(float& s, float& t, float d) {
  d = fmaxf(d, -200.f);
  const float f = row_ex2(d);
  t = f * fmaf(s, d, t);
  s *= f;
}
// The statistics of every step-th item from `first` on, relative to their largest logit.  The reference lags behind it as in RowSums: it
// is raised by 2^4 at least, so that the roundings of these steps fade.  Sums are of 64 items, and of these: short chains of additions.
__device__ __noinline__ RowStat score_sums(const ScoreRow& z, float c, int first, int step) {
  RowStat r = row_empty();
  float ref = ROW_NEG_INF;
  for (int v0 = first; v0 < z.V; v0 += 64 * step) {
    float s = 0.f, t = 0.f;
    z.each(v0, min(z.V, v0 + 64 * step), step, [&](float x) {
      if (x == ROW_NEG_INF) return;
      r.m = fmaxf(r.m, x);
      if ((x - ref) * c > 4.f) {
        score_raise(r.s, r.t, (ref - x) * c);
        score_raise(s, t, (ref - x) * c);
        ref = x;
      }
      const float y = (x - ref) * c, e = row_ex2(y);
      s += e;
      t = fmaf(e, fmaxf(y, -200.f), t);
    });
    r.s += s;
    r.t += t;
  }
  if (r.m > ROW_NEG_INF) score_raise(r.s, r.t, (ref - r.m) * c);
  return r;
}

// Joins the statistics of the runs that crossed a user's row tile, and their lists.  A warp takes a user, four users a block; where
// users are few a block takes one (ALONE): its eight warps share the given tokens and the reading of the lists.
// About 256 keys come in; more than fit are taken in turns, the best k of each going into the next.
// Where a wait of the main pass ran out (the call's answers are not defined then) parts of the statistics and lists were never written: how
// many entries a list holds, and which item one names, are held within their arrays, and a turn that has no room ends the reading.
// A row of huge logits (row_is_huge) is summed again, relative to its largest logit itself.  A last place of such logits is worth many
// units of an exponent, so that all its answers are taken from one set of them: the products as score_dots sums them, not those of the
// tensor cores, which add in another order.
constexpr int SJ_PARTS = (kNumSMs / 2 + 1) * SC_PARTS, SJ_KEYS = 512;          // parts of a user at most; keys of a turn
constexpr int SJ_WARPS = 4, SJ_ALONE_WARPS = 8;
template <bool ALONE>
__global__ void __launch_bounds__(32 * (ALONE ? SJ_ALONE_WARPS : SJ_WARPS)) score_join_kernel(const ScoreArgs a, const bf16* users, int64_t ld_u, const bf16* items, int64_t ld_i,
                                                                int32_t d, float scale, RowAnswers ask) {
  if (!chain_begin()) return;
  constexpr int ROWS = ALONE ? 1 : SJ_WARPS;
  __shared__ __align__(16) uint64_t keys_of[ROWS][SJ_KEYS];
  __shared__ const uint64_t* lists_of[ROWS][SJ_PARTS];
  __shared__ int starts_of[ROWS][SJ_PARTS + 1], kept;
  __shared__ RowStat huge_part[ALONE ? SJ_ALONE_WARPS : 1];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, slot = ALONE ? 0 : warp;
  const int64_t n = ALONE ? blockIdx.x : (int64_t)blockIdx.x * SJ_WARPS + warp;
  if (n >= a.N) return;                                 // whole warps; the block's barriers are in the other form only
  auto sync = [&]() {
    if (ALONE) __syncthreads();
    else __syncwarp();
  };
  uint64_t* keys = keys_of[slot];
  int* starts = starts_of[slot];                        // of each part's list among all of the user's keys
  const int tm = (int)(n / SC_ROWS), row = (int)(n % SC_ROWS);
  const int p0 = tm * a.units / a.per_run, p1 = ((tm + 1) * a.units - 1) / a.per_run, parts = (p1 - p0 + 1) * SC_PARTS;
  RowStat r = row_empty();
  int all = 0;
  for (int i0 = 0; i0 < parts; i0 += 32) {              // part i % SC_PARTS of pair p0 + i / SC_PARTS; every warp of a block does the same
    const int i = i0 + lane, p = p0 + i / SC_PARTS, part = i % SC_PARTS;
    int have = 0;
    if (i < parts) {
      const float4 f = a.stats[((int64_t)(p * 2 + (p == p0 && p * a.per_run < tm * a.units ? 1 : 0)) * SC_PARTS + part) * SC_ROWS + row];
      RowStat x{f.x, f.y, f.z};
      const float m = fmaxf(r.m, x.m);
      if (m > r.m) row_raise(r, m, a.c);
      if (m > x.m) row_raise(x, m, a.c);
      r.s += x.s;
      r.t += x.t;
      const bool early = p == p1 && min((p + 1) * a.per_run, a.total) > (tm + 1) * a.units;      // the run goes on with the next row tile
      have = max(0, min(__float_as_int(f.w), early ? a.early_cap : a.cap));
      lists_of[slot][i] = early ? a.early + ((int64_t)(tm * SC_PARTS + part) * SC_ROWS + row) * a.early_cap
                                : a.lists + ((int64_t)(p * SC_PARTS + part) * SC_ROWS + row) * a.cap;
    }
    int before = have;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, before, o);
      if (lane >= o) before += x;
    }
    if (i < parts) starts[i] = all + before - have;
    all += __shfl_sync(0xffffffffu, before, 31);
  }
  if (lane == 0) starts[parts] = all;
  r = row_join_lanes<32>(r, a.c);
  sync();                                               // (the warps of a block have written the same)
  const int k = ask.k;
  // keys [from, from + count) of all lists to keys[at ..)
  auto take = [&](int from, int count, int at) {
#pragma unroll 4
    for (int i = ALONE ? (int)threadIdx.x : lane; i < count; i += ALONE ? 32 * SJ_ALONE_WARPS : 32) {
      int lo = 0, hi = parts - 1;                       // the last part that starts at or before this key
      while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (starts[mid] <= from + i) lo = mid;
        else hi = mid - 1;
      }
      keys[at + i] = lists_of[slot][lo][from + i - starts[lo]];
    }
  };
  int have = 0;
  if (k > 0) {
    have = min(all, SJ_KEYS);
    take(0, have, 0);
  }
  float log_s = row_log_sum(r, a.c), entropy = row_entropy(r);
  const ScoreRow row_z{users + n * ld_u, items, a.bias, ld_i, a.V, d};
  const bool huge = row_is_huge(r.m, a.c);
  if (huge) {                                           // in all warps of a block or in none: each takes every eighth item
    r = score_sums(row_z, a.c, ALONE ? warp : 0, ALONE ? SJ_ALONE_WARPS : 1);
    if (ALONE) {
      if (lane == 0) huge_part[warp] = r;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < SJ_ALONE_WARPS; ++i) r.m = fmaxf(r.m, huge_part[i].m);
      r.s = r.t = 0.f;
#pragma unroll
      for (int i = 0; i < SJ_ALONE_WARPS; ++i) {
        RowStat x = huge_part[i];
        if (x.m > ROW_NEG_INF) score_raise(x.s, x.t, (x.m - r.m) * a.c);
        r.s += x.s;
        r.t += x.t;
      }
    }
    log_s = logf(r.s);
    entropy = log_s - kLn2 * (r.t / r.s);
  }
  for (int i = ALONE ? warp : 0; i < ask.C; i += ALONE ? SJ_ALONE_WARPS : 1) {
    const int32_t t = ask.targets[n * ask.C + i];
    float lp = 0.f;
    if (t >= 0 && t < a.V) {
      lp = row_logp(row_z(t), r.m, log_s, scale);
    } else if (t != -1) {
      gram_device_fail(a.status, GRAM_ERR_ID_RANGE);
    }
    if (lane == 0) ask.logp[n * ask.C + i] = lp;
  }
  if (lane == 0 && (!ALONE || warp == 0)) {
    if (ask.stats) { ask.stats[2 * n] = row_largest(r.m, log_s); ask.stats[2 * n + 1] = log_s; }
    if (ask.entropy) ask.entropy[n] = entropy;
  }
  if (k == 0) return;
  for (int from = have;;) {
    sync();
    if (!ALONE || warp == 0) {
      if (have > k + 16) have = warp_keep(keys, have, k);
      if (ALONE && lane == 0) kept = have;
    }
    sync();
    if (ALONE) have = kept;
    if (from == all || have == SJ_KEYS) break;
    const int count = min(all - from, SJ_KEYS - have);
    take(from, count, have);
    from += count;
    have += count;
  }
  if (ALONE && warp != 0) return;
  top_sort<32>(keys, have);
  const int64_t o = n * k;
  for (int i0 = 0; i0 < have; i0 += 32) {
    const int i = i0 + lane;
    const uint64_t key = i < have ? keys[i] : 0;
    float z = row_key_logit(key);
    if (huge)
      for (int j = 0; j < 32 && i0 + j < have; ++j) {
        const float x = score_again(row_z, (int)min((uint32_t)row_key_place(keys[i0 + j]), (uint32_t)a.V - 1u));
        if (lane == j) z = x;
      }
    const int above = i < have ? top_above<32>(keys, have, i) : k;
    if (above < k) {
      ask.top_ids[o + above] = row_key_place(key);
      ask.top_logp[o + above] = row_logp(z, r.m, log_s, scale);
    }
  }
  for (int i = have + lane; i < k; i += 32) {
    ask.top_ids[o + i] = -1;
    ask.top_logp[o + i] = ROW_NEG_INF;
  }
}

template <int MODE> cudaError_t launch_score(const CUtensorMap& users, const CUtensorMap& items, const ScoreArgs& a, int pairs, cudaStream_t st) {
  auto kern = score_kernel<MODE>;
  const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, SC_SMEM);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(2 * pairs));
  cfg.blockDim = dim3(SC_THREADS);
  cfg.dynamicSmemBytes = SC_SMEM;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1] = chain_attribute();
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kern, users, items, a);
}

// what is asked of the rows from the n-th on
RowAnswers from(RowAnswers ask, int64_t n) {
  if (ask.C) { ask.targets += n * ask.C; ask.logp += n * ask.C; }
  if (ask.stats) ask.stats += 2 * n;
  if (ask.entropy) ask.entropy += n;
  if (ask.k) { ask.top_logp += n * ask.k; ask.top_ids += n * ask.k; }
  return ask;
}

}  // namespace

// copies are no larger than the users (rows past the last are filled with zeros, which takes time: one user against 100 000
// items of 768 46 us with boxes of 128 rows, 35 with boxes of 8)
static int score_box_rows(int64_t N) {
  int rows = SM_ROWS;
  while (rows > 8 && rows / 2 >= N) rows /= 2;
  return rows;
}

gram_status score_logits_launch(gram_ctx* ctx, const void* users, int64_t ld_users, const void* items, int64_t ld_items, const float* bias, int64_t N,
                                int32_t V, int32_t d, float* logits, int64_t ld_logits, cudaStream_t st) {
  CUtensorMap map_u, map_i;
  const int box_rows = score_box_rows(N);
  if (!make_map(&map_u, users, (uint64_t)d, (uint64_t)N, (uint64_t)ld_users, SC_BK, (uint32_t)box_rows) ||
      !make_map(&map_i, items, (uint64_t)d, (uint64_t)V, (uint64_t)ld_items, SC_BK, 64))
    return gram_set_error(ctx, "scores: cannot describe the vectors"), GRAM_ERR_UNSUPPORTED;
  ScoreArgs a = {};
  a.bias = bias;
  a.N = N;
  a.V = V;
  a.box_rows = box_rows;
  a.num_kb = ceil_div(d, SC_BK);
  a.stride = 1;
  a.units = ceil_div(V, SC_UNIT);
  a.total = (int32_t)ceil_div64(N, SC_ROWS) * a.units;
  a.per_run = ceil_div(a.total, kNumSMs / 2);
  a.logits = logits;
  a.ld_logits = ld_logits;
  a.give_up = gram_ring_rows(ctx);
  a.status = gram_status_word(ctx);
  ProfScope prof(ctx, GRAM_K_GEMM, 2.0 * N * V * d, 1, st, "score");
  GRAM_CUDA(ctx, launch_score<LOGITS>(map_u, map_i, a, ceil_div(a.total, a.per_run), st));
  return GRAM_OK;
}

gram_status score_logprobs_launch(gram_ctx* ctx, const void* users, int64_t ld_users, const void* items, int64_t ld_items,
                                  const float* bias, int64_t N, int32_t V, int32_t d, float scale, const RowAnswers& ask, void* ws,
                                  size_t ws_bytes, cudaStream_t st) {
  if (V > (1 << 30) / (kNumSMs / 2) * SC_UNIT) return gram_set_error(ctx, "gram_score_logprobs: %d items", V), GRAM_ERR_UNSUPPORTED;   // units of all row tiles, in 32 bits
  const int32_t all_units = ceil_div(V, SC_UNIT);
  CUtensorMap map_u, map_i;
  const int box_rows = score_box_rows(N);
  if (!make_map(&map_i, items, (uint64_t)d, (uint64_t)V, (uint64_t)ld_items, SC_BK, 64))
    return gram_set_error(ctx, "gram_score_logprobs: cannot describe the items"), GRAM_ERR_UNSUPPORTED;
  const int64_t ld_logits = ((int64_t)V + 7) / 8 * 8;
  ScoreArgs a = {};
  a.bias = bias;
  a.box_rows = box_rows;
  a.num_kb = ceil_div(d, SC_BK);
  a.k = ask.k;
  a.c = scale * kLog2e;
  a.stride = 1;
  a.give_up = gram_ring_rows(ctx);
  a.status = gram_status_word(ctx);
  // Logits that the workspace holds (32 MB of it at most: they stay in L2) are written and read once more, in place of the sample,
  // the bars and the joining.  This way and the other, in us, items of 768:
  //   10 alternatives, 100 000 items, 1 user 41 and 53, 64 users 46 and 58; 30 522 items, 256 users 29 and 37; 128 alternatives of
  //   800 users, 10 000 items 33 and 91
  //   in several turns where the table is small: 10 alternatives, 1000 items, 20 000 users 78 and 156, 3000 items, 8192 users 87 and
  //   87, 10 000 items, 4096 users 141 and 87, but with 128 alternatives 180 and 300
  //   without alternatives the other way has no sample to take: 64 users, 30 522 items 17 and 21, 100 000 items 42 and 38
  const int64_t room = (int64_t)(ws_bytes < (32u << 20) ? ws_bytes : 32u << 20) / (int64_t)sizeof(float) / ld_logits;
  const int64_t at_once = room < SC_ROWS ? room : room / SC_ROWS * SC_ROWS;       // users of a turn
  if (ask.k > 0 ? at_once > 0 && (N <= at_once || at_once >= (ask.k > 64 ? 768 : 2048)) : N <= at_once && N * V <= (2 << 20)) {
    for (int64_t n = 0; n < N; n += at_once) {
      const int64_t now = N - n < at_once ? N - n : at_once;
      GRAM_TRY(score_logits_launch(ctx, (const bf16*)users + n * ld_users, ld_users, items, ld_items, bias, now, V, d, (float*)ws, ld_logits, st));
      GRAM_TRY(logprobs_launch(ctx, ws, GRAM_F32, ld_logits, now, V, scale, from(ask, n), st));
    }
    return GRAM_OK;
  }
  // The sample: so many items that about 256 entries of a user reach the bar, but 4096 at least and a third of the table at
  // most; its maxima by groups of 8 columns, by 32 where that is more than score_bar_kernel holds.
  int32_t sample = 0, fine = 1;
  if (ask.k) {
    int64_t want = (int64_t)ask.k * V / 256;
    if (want > V / 3) want = V / 3;
    if (want < 4096) want = 4096;
    if (want > SB_GROUPS * 32) want = SB_GROUPS * 32;
    sample = (int32_t)(want < V ? ceil_div64(want, SC_UNIT) * SC_UNIT : V);
    if (sample > V) sample = V;
    fine = sample <= SB_GROUPS * 8;
  }
  const int32_t sample_units = ceil_div(sample, SC_UNIT);
  // Row tiles of a launch: half the pairs at most, so that a run touches two row tiles at most and several threads share a
  // user's list; and no more than the sample's maxima have room for.
  const int64_t tiles = ceil_div64(N, SC_ROWS);
  int64_t most = kNumSMs / 4;
  const size_t sample_tile = (size_t)sample_units * (SC_UNIT / 32) * SC_ROWS * (fine ? 16 : 4);
  const size_t stats_bytes = (size_t)(kNumSMs / 2) * 2 * SC_PAIR_THREADS * sizeof(float4), bars_tile = SC_ROWS * sizeof(float);
  if (ask.k && most > (int64_t)((ws_bytes - stats_bytes) / (sample_tile + bars_tile))) most = (int64_t)((ws_bytes - stats_bytes) / (sample_tile + bars_tile));
  // Lists share the sample's place, 16 entries more than k at least in each.  Where the workspace is too small for those of all pairs and the
  // early ones of all row tiles, a launch takes fewer row tiles, and fewer pairs run.
  const int early_cap = ask.k > 32 ? ask.k : 32;
  int64_t per_launch, cap;
  int pairs;
  for (;; most /= 2) {
    per_launch = ceil_div64(tiles, ceil_div64(tiles, most));
    pairs = kNumSMs / 2;
    cap = 0;
    if (!ask.k) break;
    const int64_t room = ((int64_t)ws_bytes - (int64_t)stats_bytes - per_launch * (int64_t)bars_tile) / (SC_PAIR_THREADS * 8) - per_launch * early_cap;
    cap = room / pairs < SC_LIST_MAX ? room / pairs : SC_LIST_MAX;
    if (cap >= ask.k + 16) break;
    cap = ask.k + 16;
    pairs = (int)(room / cap);
    if (pairs >= 2 * per_launch) break;
    if (most == 1) return gram_set_error(ctx, "gram_score_logprobs: the workspace is too small for %d alternatives", ask.k), GRAM_ERR_WORKSPACE;
  }
  const size_t early_bytes = ask.k ? (size_t)per_launch * SC_PAIR_THREADS * early_cap * 8 : 0;
  ProfScope prof(ctx, GRAM_K_GEMM, 2.0 * N * V * d, (ask.k ? 4 : 2) * (int)ceil_div64(tiles, per_launch), st, "score");
  for (int64_t n = 0; n < N; n += per_launch * SC_ROWS) {
    const int64_t now = N - n < per_launch * SC_ROWS ? N - n : per_launch * SC_ROWS, now_tiles = ceil_div64(now, SC_ROWS);
    const bf16* u = (const bf16*)users + n * ld_users;
    if (!make_map(&map_u, u, (uint64_t)d, (uint64_t)now, (uint64_t)ld_users, SC_BK, (uint32_t)box_rows))
      return gram_set_error(ctx, "gram_score_logprobs: cannot describe the users"), GRAM_ERR_UNSUPPORTED;
    a.N = now;
    a.cap = (int32_t)cap;
    a.early_cap = early_cap;
    a.stats = (float4*)ws;
    float* bars = (float*)((uint8_t*)ws + stats_bytes);
    a.bars = bars;
    a.early = (uint64_t*)((uint8_t*)bars + per_launch * bars_tile);
    a.lists = a.early + early_bytes / 8;
    a.sample = (float*)a.early;
    a.sample_rows = now_tiles * SC_ROWS;
    a.fine = fine;
    auto cut = [&](int32_t units, int stride, int over) {        // the units of a pass in runs; returns their number
      a.V = V;
      a.units = units;
      a.stride = stride;
      a.total = (int32_t)(now_tiles * a.units);
      a.per_run = ceil_div(a.total, over);
      return ceil_div(a.total, a.per_run);
    };
    if (ask.k) {
      const int used = cut(sample_units, sample_units < all_units ? all_units / 2 / ceil_div(sample_units, 2) : 1, kNumSMs / 2);
      GRAM_CUDA(ctx, launch_score<SAMPLE>(map_u, map_i, a, used, st));
      launch_chain(score_bar_kernel, dim3((unsigned)ceil_div64(now, SB_ROWS)), 32 * SB_ROWS, 0, st, a.sample, a.sample_rows,
                   a.units * (SC_UNIT / 32), fine, now, ask.k, bars);
    }
    const RowAnswers part = from(ask, n);
    const int used = cut(all_units, 1, pairs);
    GRAM_CUDA(ctx, ask.k ? launch_score<LISTS>(map_u, map_i, a, used, st) : launch_score<STATISTICS>(map_u, map_i, a, used, st));
    if (now >= 4 * kNumSMs)
      launch_chain(score_join_kernel<false>, dim3((unsigned)ceil_div64(now, SJ_WARPS)), 32 * SJ_WARPS, 0, st, a, u, ld_users, (const bf16*)items, ld_items,
                   d, scale, part);
    else
      launch_chain(score_join_kernel<true>, dim3((unsigned)now), 32 * SJ_ALONE_WARPS, 0, st, a, u, ld_users, (const bf16*)items, ld_items, d, scale, part);
    GRAM_LAUNCH_CHECK(ctx);
  }
  return GRAM_OK;
}
