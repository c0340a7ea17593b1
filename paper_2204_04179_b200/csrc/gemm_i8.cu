// Tables in 8 bits: rows of codes with a scale each (gram_quantize_rows) and their products (gram_gemm_i8).
#include "gemm_i8.h"

#include "pair_pipe.cuh"

namespace {
using namespace tc;

constexpr int kPairs = kNumSMs / 2;

// ============================================================================================
// codes = x (127 / max |x|) to the nearest whole number, scale = max |x| / 127
// ============================================================================================
// A warp a row.  Rows of up to QR_HELD elements a lane are read once, longer ones twice (the second time out of L1 or L2).
// Bounded by HBM: 100 000 rows of 768 fp32 59 us in a loop of calls (6.5 TB/s), bf16 51; 64 rows of bf16 2.3 us in a graph of calls.
constexpr int QR_HELD = 32, QR_ROWS = 8;

template <typename T> struct QuantVec;                  // 16 bytes of a row, and their codes
template <> struct QuantVec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void load(const float* p, float* x) {
    const float4 v = __ldg(reinterpret_cast<const float4*>(p));
    x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
  }
};
template <> struct QuantVec<bf16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void load(const bf16* p, float* x) {
    const uint4 v = __ldg(reinterpret_cast<const uint4*>(p));
    const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = unpack_bf16x2(u[i]);
      x[2 * i] = f.x;
      x[2 * i + 1] = f.y;
    }
  }
};
__device__ __forceinline__ float quant_value(const float* p) { return __ldg(p); }
__device__ __forceinline__ float quant_value(const bf16* p) { return __bfloat162float(*p); }

// A maximum that NaN stays in: of bits without the sign, which order like whole numbers (NaN above infinity).
__device__ __forceinline__ uint32_t quant_size(float x) { return __float_as_uint(x) & 0x7fffffffu; }
__device__ __forceinline__ uint32_t quant_code(float x, float inv) { return (uint32_t)__float2int_rn(fminf(fmaxf(x * inv, -127.f), 127.f)) & 0xffu; }
struct QuantScale {
  float inv, scale;
};
// Rows below 1e-30 count as zeros (127 / max would leave 32 bits); in a row with infinity or NaN the scale is NaN and says so.
__device__ __forceinline__ QuantScale quant_scale(uint32_t top) {
  const float m = __uint_as_float(top);
  if (top >= 0x7f800000u) return QuantScale{0.f, __int_as_float(0x7fffffff)};
  if (m < 1e-30f) return QuantScale{0.f, 0.f};
  return QuantScale{__fdiv_rn(127.f, m), __fdiv_rn(m, 127.f)};
}

// VEC: rows and codes allow 16-byte loads and stores of as many codes
template <typename T, bool VEC>
__global__ void __launch_bounds__(32 * QR_ROWS) quantize_rows_kernel(const T* x, int64_t ld, int64_t rows, int32_t cols, int8_t* codes, int64_t ld_codes,
                                                                     float* scale) {
  if (!chain_begin()) return;
  constexpr int W = VEC ? QuantVec<T>::N : 1, HELD = QR_HELD / W;          // elements of a piece; pieces that a lane holds
  const uint32_t lane = threadIdx.x & 31, n = (uint32_t)cols;              // a step past the longest row leaves 31 bits, not 32
  const int64_t r = (int64_t)blockIdx.x * QR_ROWS + (threadIdx.x >> 5);
  if (r >= rows) return;
  const T* row = x + r * ld;
  int8_t* out = codes + r * ld_codes;
  const uint32_t pieces = n / W;                        // VEC: the rest is taken one by one
  float v[HELD][W];
  uint32_t top = 0u;
  auto load = [&](uint32_t i, float* to) {
    if constexpr (VEC) QuantVec<T>::load(row + i * W, to);
    else to[0] = quant_value(row + i);
  };
#pragma unroll
  for (int h = 0; h < HELD; ++h)
    if (h * 32 + lane < pieces) load(h * 32 + lane, v[h]);
#pragma unroll
  for (int h = 0; h < HELD; ++h)
    if (h * 32 + lane < pieces) {
#pragma unroll
      for (int j = 0; j < W; ++j) top = max(top, quant_size(v[h][j]));
    }
  for (uint32_t i = HELD * 32 + lane; i < pieces; i += 32) {
    float y[W];
    load(i, y);
#pragma unroll
    for (int j = 0; j < W; ++j) top = max(top, quant_size(y[j]));
  }
  for (uint32_t i = pieces * W + lane; i < n; i += 32) top = max(top, quant_size(quant_value(row + i)));
  const QuantScale s = quant_scale(__reduce_max_sync(0xffffffffu, top));
  // a row of infinities or NaN has codes 0 (0 times them would be NaN)
  const bool none = s.inv == 0.f;
  auto store = [&](uint32_t i, const float* y) {
    if constexpr (VEC) {
      uint32_t c[W / 4];
#pragma unroll
      for (int j = 0; j < W / 4; ++j)
        c[j] = none ? 0u : quant_code(y[4 * j], s.inv) | quant_code(y[4 * j + 1], s.inv) << 8 | quant_code(y[4 * j + 2], s.inv) << 16 |
                           quant_code(y[4 * j + 3], s.inv) << 24;
      if constexpr (W == 4) *reinterpret_cast<uint32_t*>(out + i * 4) = c[0];
      else *reinterpret_cast<uint2*>(out + i * 8) = make_uint2(c[0], c[1]);
    } else {
      out[i] = none ? (int8_t)0 : (int8_t)quant_code(y[0], s.inv);
    }
  };
#pragma unroll
  for (int h = 0; h < HELD; ++h)
    if (h * 32 + lane < pieces) store(h * 32 + lane, v[h]);
  for (uint32_t i = HELD * 32 + lane; i < pieces; i += 32) {
    float y[W];
    load(i, y);
    store(i, y);
  }
  for (uint32_t i = pieces * W + lane; i < n; i += 32) out[i] = none ? (int8_t)0 : (int8_t)quant_code(quant_value(row + i), s.inv);
  if (lane == 0) scale[r] = s.scale;
}

template <typename T>
void launch_quantize(const void* x, int64_t ld, int64_t rows, int32_t cols, int8_t* codes, int64_t ld_codes, float* scale, cudaStream_t st) {
  constexpr int W = QuantVec<T>::N;
  const bool vec = (uintptr_t)x % 16 == 0 && (ld % W == 0 || rows == 1) && (uintptr_t)codes % W == 0 && (ld_codes % W == 0 || rows == 1);
  auto kern = vec ? quantize_rows_kernel<T, true> : quantize_rows_kernel<T, false>;
  launch_chain(kern, dim3((unsigned)ceil_div64(rows, QR_ROWS)), 32 * QR_ROWS, 0, st, (const T*)x, ld, rows, cols, codes, ld_codes, scale);
}

// ============================================================================================
// the product
// ============================================================================================
// C's rows are tokens, its columns channels (rows of A and of B).  Sums are whole numbers of 32 bits, exact up to K = 131 071.  Two forms:
//   ROWS      a pair of SMs owns 256 tokens x 256 channels, tokens are the MMA's rows: a thread holds 32 neighbouring results of a row, which
//             leave by bulk stores.  Many tokens, C aligned to 16 bytes, rows of 16 bytes or more.
//   CHANNELS  256 channels x `width` tokens, channels are the MMA's rows: a warp's lanes run along C's rows, whatever its address and stride,
//             and a few tokens are a narrow tile.
// us of ROWS and of CHANNELS, K = 768, fp32 results, 2304, 16 384 and 100 000 channels: 96 tokens 8.2 and 5.8, 9.0 and 6.4, 25.7 and 22.9; 129 tokens 8.3 and 7.6,
// 9.4 and 8.8, 28.5 and 28.7; 512 tokens 8.6 and 8.3, 12.2 and 12.6, 56 and 58.5; bf16 results, 129 tokens 7.2 and 7.7, 8.5 and 9.0, 26.0 and 27.4; 512 7.6 and
// 8.4, 10.3 and 12.9, 43 and 53.
// The tiles of the operand with fewer rows vary fastest: it stays in L2 while the other is read once.
// Measured with K = 768: one token against 100 000 channels 16.9 us and 64 tokens 21.7 (the table's 77 MB at 4.6 TB/s, on tables in turn); many tokens with
// both operands of each tile fetched 2.5 to 3.0 POP/s at K = 2048.  Results that leave by single stores in place of bulk stores: 4096 x 16 384 x 768 65 us
// for 52; C at odd addresses takes that form.
constexpr int I8_BK = 128, I8_EPI_WARPS = 16;
using I8Rows = PairPipe<4, I8_EPI_WARPS, I8_EPI_WARPS * (4096 + 512)>;      // a warp's box of results, and its channels' scales and biases
using I8Channels = PairPipe<6, I8_EPI_WARPS, I8_EPI_WARPS * 64 * 4>;        // a warp's tokens' scales

struct I8Args {
  const float *scale_a, *scale_b, *bias;
  void* C;
  int64_t ldc, M;
  int32_t N, num_kb, width;      // width: columns of the MMA's tile
  int32_t fast, total;           // tiles that vary fastest
  int32_t rows_fast;             // those of the MMA's rows
  int32_t give_up;
  int32_t* status;
};
// first row of tile t's MMA rows and of its columns
__device__ __forceinline__ int i8_row(const I8Args& a, int t) { return (a.rows_fast ? t % a.fast : t / a.fast) * 2 * PAIR_ROWS; }
__device__ __forceinline__ int i8_col(const I8Args& a, int t) { return (a.rows_fast ? t / a.fast : t % a.fast) * a.width; }

__device__ __forceinline__ void i8_mma_pair(uint32_t tmem_d, uint64_t da, uint64_t db, uint32_t idesc, uint32_t accum) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}" ::"r"(tmem_d),
      "l"(da), "l"(db), "r"(idesc), "r"(accum)
      : "memory");
}

// the copies and products of all of a pair's tiles: both blocks' first warp and the leader's second
template <typename Pipe>
__device__ __forceinline__ bool i8_copies(const Pipe& pipe, const I8Args& a, const CUtensorMap& rows, const CUtensorMap& cols) {
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  const uint32_t bytes = PAIR_OPERAND + (uint32_t)a.width * (I8_BK / 2);
  int s = 0, tile = 0;
  uint32_t ph = 0;
  for (int t = pair; t < a.total; t += pairs, ++tile) {
    if (tile == a.give_up) return false;
    const int r0 = i8_row(a, t) + (int)pipe.rank * PAIR_ROWS, c0 = i8_col(a, t) + (int)pipe.rank * (a.width / 2);
    for (int kb = 0; kb < a.num_kb; ++kb) {
      if (!mbar_wait_warp(pipe.empty(s), ph ^ 1u, pipe.abort_flag)) return false;
      const uint32_t bar = pipe.lead_full(s);
      if (elect_one()) {
        mbar_arrive_expect_tx_remote(bar, bytes);
        tma_load_2d_pair(pipe.a_of(s), &rows, kb * I8_BK, r0, bar);
        tma_load_2d_pair(pipe.b_of(s), &cols, kb * I8_BK, c0, bar);
      }
      __syncwarp();
      if (++s == Pipe::STAGES) { s = 0; ph ^= 1u; }
    }
  }
  return true;
}
template <typename Pipe> __device__ __forceinline__ bool i8_products(const Pipe& pipe, const I8Args& a) {
  // signed 8-bit operands, sums in 32-bit whole numbers
  const uint32_t idesc = (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(a.width >> 3) << 17) | ((uint32_t)(2 * PAIR_ROWS >> 4) << 24);
  const uint64_t da0 = make_desc(pipe.a_of(0), 16, 1024), db0 = make_desc(pipe.b_of(0), 16, 1024);
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  int s = 0;
  uint32_t ph = 0, it = 0;
  for (int t = pair; t < a.total; t += pairs, ++it) {
    const int buf = (int)(it & 1);
    if (!mbar_wait_warp(pipe.tempty(buf), ((it >> 1) & 1) ^ 1u, pipe.abort_flag)) return false;
    tc_fence_after();
    const uint32_t tmem_d = pipe.tmem + (uint32_t)(buf * PAIR_COLS);
    for (int kb = 0; kb < a.num_kb; ++kb) {
      if (!mbar_wait_warp(pipe.full(s), ph, pipe.abort_flag)) return false;
      tc_fence_after();
      const uint32_t soff = (uint32_t)(s * (Pipe::STAGE >> 4));
      if (elect_one()) {
#pragma unroll
        for (int k = 0; k < 4; ++k)                     // 32 bytes of the rows each
          i8_mma_pair(tmem_d, da0 + soff + (uint64_t)(k * 2), db0 + soff + (uint64_t)(k * 2), idesc, (kb > 0 || k > 0) ? 1u : 0u);
        tc_commit_pair(pipe.empty(s));
        if (kb == a.num_kb - 1) tc_commit_pair(pipe.tfull(buf));
      }
      __syncwarp();
      if (++s == Pipe::STAGES) { s = 0; ph ^= 1u; }
    }
  }
  return true;
}

// 32 sums of a token with its scale and the channels' scales and biases, to its row of a box (128-byte swizzle): 32 fp32, or 32 of 64 bf16
template <typename CT> __device__ __forceinline__ void i8_put(uint32_t (&v)[32], float sa, const float* scale, const float* bias, uint32_t row_at, int half) {
  const uint32_t turn = threadIdx.x & 7;
#pragma unroll
  for (int j = 0; j < 32; j += 4) {
    const float4 s = *reinterpret_cast<const float4*>(scale + j), b = *reinterpret_cast<const float4*>(bias + j);
    v[j] = __float_as_uint(fmaf((float)(int32_t)v[j] * sa, s.x, b.x));
    v[j + 1] = __float_as_uint(fmaf((float)(int32_t)v[j + 1] * sa, s.y, b.y));
    v[j + 2] = __float_as_uint(fmaf((float)(int32_t)v[j + 2] * sa, s.z, b.z));
    v[j + 3] = __float_as_uint(fmaf((float)(int32_t)v[j + 3] * sa, s.w, b.w));
  }
  if constexpr (sizeof(CT) == 4) {
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j) sts128(row_at + ((j ^ turn) << 4), v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
  } else {
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j) {
      uint32_t h[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) h[i] = pack_bf16x2(__uint_as_float(v[8 * j + 2 * i]), __uint_as_float(v[8 * j + 2 * i + 1]));
      sts128(row_at + (((half * 4 + j) ^ turn) << 4), h[0], h[1], h[2], h[3]);
    }
  }
}

// Bulk stores write whole pieces of 16 bytes, with zeros over what is beside a row that ends within one: their map ends with the last whole piece, and what is
// left of a row is stored by its thread (kernels with LEFT: the code costs the others 1 %).  v: the 32 results from channel `first` on.  25 600 x 2303 x 768 in bf16, 7 left of each row: 45.5 us, 2304 43.1.
template <typename CT> __host__ __device__ __forceinline__ int32_t i8_whole(int32_t N) { return N / (16 / (int)sizeof(CT)) * (16 / (int)sizeof(CT)); }
template <typename CT> __device__ __forceinline__ void i8_left(const uint32_t (&v)[32], const I8Args& a, int64_t row, int first) {
  const int whole = i8_whole<CT>(a.N), left = a.N - whole;
  if ((unsigned)(whole - first) >= 32u || row >= a.M) return;
  CT* to = reinterpret_cast<CT*>(a.C) + row * a.ldc + whole;
  constexpr int P = 16 / sizeof(CT);
#pragma unroll
  for (int k = 0; k < 32; k += P) {
    if (k != whole - first) continue;
    if constexpr (sizeof(CT) == 4) {
      if (left & 2) *reinterpret_cast<uint2*>(to) = make_uint2(v[k], v[k + 1]);
      if (left & 1) to[left & 2] = __uint_as_float(left & 2 ? v[k + 2] : v[k]);
    } else {
      uint32_t h[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) h[i] = pack_bf16x2(__uint_as_float(v[k + 2 * i]), __uint_as_float(v[k + 2 * i + 1]));
      if (left & 4) *reinterpret_cast<uint2*>(to) = make_uint2(h[0], h[1]);
      if (left & 2) *reinterpret_cast<uint32_t*>(to + (left & 4)) = left & 4 ? h[2] : h[0];
      if (left & 1) to[left & 6] = __ushort_as_bfloat16((unsigned short)(left & 4 ? (left & 2 ? h[3] : h[2]) : left & 2 ? h[1] : h[0]));
    }
  }
}

template <typename CT, bool LEFT>
__global__ void __launch_bounds__(I8Rows::THREADS, 1) gemm_i8_rows_kernel(const __grid_constant__ CUtensorMap tokens, const __grid_constant__ CUtensorMap channels,
                                                                          const __grid_constant__ CUtensorMap result, const __grid_constant__ I8Args a) {
  extern __shared__ uint8_t smem_raw[];
  I8Rows pipe;
  const bool go = pipe.open(smem_raw);
  bool failed = false;
  if (pipe.warp == 0 && go) {
    failed = !i8_copies(pipe, a, tokens, channels);
  } else if (pipe.warp == 1 && go) {
    if (pipe.rank == 0) failed = !i8_products(pipe, a);
  } else if (go) {
    // ------------------------------ results (both blocks): a token and 64 channels a thread ------------------------------
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const int lane = pipe.lane, q = pipe.warp & 3, part = (pipe.warp - 2) >> 2, w = pipe.warp - 2;
    const uint32_t box = pipe.tiles + I8Rows::STAGES * I8Rows::STAGE + (uint32_t)w * 4096u, row_at = box + (uint32_t)lane * 128u;
    float* of = reinterpret_cast<float*>(pipe.extra + I8_EPI_WARPS * 4096) + w * 128;        // 64 scales, 64 biases
    uint32_t it = 0;
    for (int t = pair; t < a.total; t += pairs, ++it) {
      const int buf = (int)(it & 1), col0 = i8_col(a, t) + part * 64;
      const int row0 = i8_row(a, t) + (int)pipe.rank * PAIR_ROWS + q * 32;
      const bool active = row0 < a.M && col0 < a.N;     // of the warp
      float sa = 0.f;
      if (active) {
        if (row0 + lane < a.M) sa = __ldg(a.scale_a + row0 + lane);
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int n = col0 + i * 32 + lane;
          of[i * 32 + lane] = n < a.N ? __ldg(a.scale_b + n) : 0.f;
          of[64 + i * 32 + lane] = n < a.N && a.bias ? __ldg(a.bias + n) : 0.f;
        }
        __syncwarp();
      }
      if (!mbar_wait_warp(pipe.tfull(buf), (it >> 1) & 1, pipe.abort_flag)) { failed = true; break; }
      tc_fence_after();
      if (active) {
        const uint32_t taddr = pipe.tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(buf * PAIR_COLS + part * 64);
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          uint32_t v[32];
          tc_ld32_issue(taddr + b * 32, v);
          tc_ld32_wait(v);
          if (b == 0 || sizeof(CT) == 4) {              // the box's last store has read it
            if (lane == 0) bulk_wait_read_all();
            __syncwarp();
          }
          i8_put<CT>(v, sa, of + b * 32, of + 64 + b * 32, row_at, b);
          if (LEFT) i8_left<CT>(v, a, row0 + lane, col0 + b * 32);
          if (b == 1 || sizeof(CT) == 4) {
            fence_proxy_async_smem();
            __syncwarp();
            const int n = col0 + (sizeof(CT) == 4 ? b * 32 : 0);
            if (lane == 0 && n < i8_whole<CT>(a.N)) {
              tma_store_2d(&result, box, n, row0);
              bulk_commit();
            }
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_remote(pipe.lead_tempty(buf));
    }
    if (lane == 0) bulk_wait_all();                     // its stores are complete before the block may exit
  }
  pipe.close(failed, a.status);
}

// ROWS where a tile's channels fit beside the stages (K of up to 768): they stay in shared memory while tile after tile of tokens passes, so that
// what comes from L2 for a tile is half (4096 x 100 000 x 768, bf16 out, a call by itself: 290 us with both operands of each tile fetched, 244 so; 25 600 x 2304 x 768:
// 46 and 43.5; 4096 x 16 384 at K = 128 33.0 and 30.1, 512 39.9 and 34.8, 768 51.5 and 42; 25 600 x 2304 at K = 256 28.7 and 30.5, 512 34.3 and 34.1).  What bounds it now is shared memory, which operands, results and scales all pass through: the tensor cores are busy 67 % of the
// time, and neither more warps nor a cheaper conversion of the sums changed it.  A pair takes whole columns of tiles, neighbouring pairs neighbouring ones; what is left after the last full round is cut evenly
// over all pairs.
constexpr int I8_HELD = 6, I8_HELD_WARPS = 8;           // k-blocks of channels that are held
constexpr int I8_HELD_BYTES = I8_HELD * PAIR_OPERAND;
using I8Resident = PairPipe<5, I8_HELD_WARPS, I8_HELD_BYTES + I8_HELD_WARPS * 4096 + 2 * 2 * PAIR_COLS * 4 + 2 * I8_HELD * 8, 0>;

// A segment: tiles of tokens [from, to) against one tile of channels.
struct I8Segments {
  int channel, from, to;
  int pair, pairs, tokens, full, at, end, round;
  __device__ __forceinline__ explicit I8Segments(const I8Args& a) : pair(blockIdx.x >> 1), pairs(gridDim.x >> 1), tokens(a.fast), round(0) {
    const int channels = a.total / a.fast;
    full = channels / pairs;
    const int64_t rest = (int64_t)(channels - full * pairs) * tokens;
    at = (int)(rest * pair / pairs);
    end = (int)(rest * (pair + 1) / pairs);
  }
  __device__ __forceinline__ bool next() {
    if (round < full) {
      channel = round++ * pairs + pair;
      from = 0;
      to = tokens;
      return true;
    }
    if (at >= end) return false;
    channel = full * pairs + at / tokens;
    from = at % tokens;
    to = min(tokens, from + end - at);
    at += to - from;
    return true;
  }
};

template <typename CT, bool LEFT>
__global__ void __launch_bounds__(I8Resident::THREADS, 1) gemm_i8_resident_kernel(const __grid_constant__ CUtensorMap tokens, const __grid_constant__ CUtensorMap channels,
                                                                                  const __grid_constant__ CUtensorMap result, const __grid_constant__ I8Args a) {
  extern __shared__ uint8_t smem_raw[];
  I8Resident pipe;
  const bool go = pipe.open(smem_raw, [&]() {
    const uint32_t bars = smem_u32(pipe.extra) + I8_HELD_BYTES + I8_HELD_WARPS * 4096 + 2 * 2 * PAIR_COLS * 4;
    for (int kb = 0; kb < I8_HELD; ++kb) {
      mbar_init(bars + 8 * kb, 2);                      // the two blocks' copies of a k-block of channels; used in the leader
      mbar_init(bars + 8 * (I8_HELD + kb), 1);          // its place is free; one per block
    }
  });
  const uint32_t held = smem_u32(pipe.extra), boxes = held + I8_HELD_BYTES, bars = boxes + I8_HELD_WARPS * 4096 + 2 * 2 * PAIR_COLS * 4;
  auto held_full = [&](int kb) { return bars + 8u * kb; };
  auto held_empty = [&](int kb) { return bars + 8u * (I8_HELD + kb); };
  bool failed = false;
  I8Segments seg(a);
  if (pipe.warp == 0 && go) {
    // ------------------------------ copies (both blocks) ------------------------------
    const uint32_t lead_bars = map_to_cta(bars, 0);
    int s = 0, tile = 0;
    uint32_t ph = 0;
    for (uint32_t n = 0; !failed && seg.next(); ++n) {
      const int c0 = seg.channel * PAIR_COLS + (int)pipe.rank * PAIR_ROWS;
      for (int m = seg.from; m < seg.to && !failed; ++m, ++tile) {
        if (tile == a.give_up) { failed = true; break; }
        const int r0 = m * 2 * PAIR_ROWS + (int)pipe.rank * PAIR_ROWS;
        for (int kb = 0; kb < a.num_kb; ++kb) {
          if (m == seg.from && !mbar_wait_warp(held_empty(kb), (n & 1u) ^ 1u, pipe.abort_flag)) { failed = true; break; }
          if (!mbar_wait_warp(pipe.empty(s), ph ^ 1u, pipe.abort_flag)) { failed = true; break; }
          if (elect_one()) {
            if (m == seg.from) {
              mbar_arrive_expect_tx_remote(lead_bars + 8u * kb, PAIR_OPERAND);
              tma_load_2d_pair(held + kb * PAIR_OPERAND, &channels, kb * I8_BK, c0, lead_bars + 8u * kb);
            }
            mbar_arrive_expect_tx_remote(pipe.lead_full(s), PAIR_OPERAND);
            tma_load_2d_pair(pipe.a_of(s), &tokens, kb * I8_BK, r0, pipe.lead_full(s));
          }
          __syncwarp();
          if (++s == I8Resident::STAGES) { s = 0; ph ^= 1u; }
        }
      }
    }
  } else if (pipe.warp == 1 && go) {
    // ------------------------------ products (leader) ------------------------------
    if (pipe.rank == 0) {
      constexpr uint32_t idesc = (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(PAIR_COLS >> 3) << 17) | ((uint32_t)(2 * PAIR_ROWS >> 4) << 24);
      const uint64_t da0 = make_desc(pipe.a_of(0), 16, 1024), db0 = make_desc(held, 16, 1024);
      int s = 0;
      uint32_t ph = 0, it = 0;
      for (uint32_t n = 0; !failed && seg.next(); ++n) {
        for (int m = seg.from; m < seg.to && !failed; ++m, ++it) {
          const int buf = (int)(it & 1);
          if (!mbar_wait_warp(pipe.tempty(buf), ((it >> 1) & 1) ^ 1u, pipe.abort_flag)) { failed = true; break; }
          tc_fence_after();
          const uint32_t tmem_d = pipe.tmem + (uint32_t)(buf * PAIR_COLS);
          for (int kb = 0; kb < a.num_kb; ++kb) {
            if (m == seg.from && !mbar_wait_warp(held_full(kb), n & 1u, pipe.abort_flag)) { failed = true; break; }
            if (!mbar_wait_warp(pipe.full(s), ph, pipe.abort_flag)) { failed = true; break; }
            tc_fence_after();
            const uint64_t da = da0 + (uint32_t)(s * (I8Resident::STAGE >> 4)), db = db0 + (uint32_t)(kb * (PAIR_OPERAND >> 4));
            if (elect_one()) {
#pragma unroll
              for (int k = 0; k < 4; ++k) i8_mma_pair(tmem_d, da + (uint64_t)(k * 2), db + (uint64_t)(k * 2), idesc, (kb > 0 || k > 0) ? 1u : 0u);
              tc_commit_pair(pipe.empty(s));
              if (m == seg.to - 1) tc_commit_pair(held_empty(kb));
              if (kb == a.num_kb - 1) tc_commit_pair(pipe.tfull(buf));
            }
            __syncwarp();
            if (++s == I8Resident::STAGES) { s = 0; ph ^= 1u; }
          }
        }
      }
    }
  } else if (go) {
    // ------------------------------ results (both blocks): a token and 128 channels a thread ------------------------------
    const int lane = pipe.lane, q = pipe.warp & 3, half = (pipe.warp - 2) >> 2;
    const uint32_t box = boxes + (uint32_t)(pipe.warp - 2) * 4096u, row_at = box + (uint32_t)lane * 128u;
    uint32_t it = 0;
    for (uint32_t n = 0; !failed && seg.next(); ++n) {
      // The segment's scales and biases, in two places in turn: a warp that is ahead has seen all others leave the segment before the last.
      float* of = reinterpret_cast<float*>(pipe.extra + I8_HELD_BYTES + I8_HELD_WARPS * 4096) + (n & 1) * 2 * PAIR_COLS + half * 128;
      const int col0 = seg.channel * PAIR_COLS + half * 128;
      float scale[4], bias[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int c = col0 + k * 32 + lane;
        scale[k] = c < a.N ? __ldg(a.scale_b + c) : 0.f;
        bias[k] = c < a.N && a.bias ? __ldg(a.bias + c) : 0.f;
      }
      for (int m = seg.from; m < seg.to; ++m, ++it) {
        const int buf = (int)(it & 1), row0 = m * 2 * PAIR_ROWS + (int)pipe.rank * PAIR_ROWS + q * 32;
        const bool active = row0 < a.M && col0 < a.N;   // of the warp
        const float sa = row0 + lane < a.M ? __ldg(a.scale_a + row0 + lane) : 0.f;
        if (!mbar_wait_warp(pipe.tfull(buf), (it >> 1) & 1, pipe.abort_flag)) { failed = true; break; }
        tc_fence_after();
        if (m == seg.from) {                            // (the four warps of these columns write the same)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            of[k * 32 + lane] = scale[k];
            of[PAIR_COLS + k * 32 + lane] = bias[k];
          }
          __syncwarp();
        }
        if (active) {
          const uint32_t taddr = pipe.tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(buf * PAIR_COLS + half * 128);
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            uint32_t v[32];
            tc_ld32_issue(taddr + b * 32, v);
            tc_ld32_wait(v);
            if (b % 2 == 0 || sizeof(CT) == 4) {        // the box's last store has read it
              if (lane == 0) bulk_wait_read_all();
              __syncwarp();
            }
            i8_put<CT>(v, sa, of + b * 32, of + PAIR_COLS + b * 32, row_at, b % 2);
            if (LEFT) i8_left<CT>(v, a, row0 + lane, col0 + b * 32);
            if (b % 2 == 1 || sizeof(CT) == 4) {
              fence_proxy_async_smem();
              __syncwarp();
              const int c = col0 + (sizeof(CT) == 4 ? b : b - 1) * 32;
              if (lane == 0 && c < i8_whole<CT>(a.N)) {
                tma_store_2d(&result, box, c, row0);
                bulk_commit();
              }
            }
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_remote(pipe.lead_tempty(buf));
      }
    }
    if (lane == 0) bulk_wait_all();                     // its stores are complete before the block may exit
  }
  pipe.close(failed, a.status);
}

template <typename CT>
__global__ void __launch_bounds__(I8Channels::THREADS, 1) gemm_i8_channels_kernel(const __grid_constant__ CUtensorMap channels,
                                                                                  const __grid_constant__ CUtensorMap tokens, const __grid_constant__ I8Args a) {
  extern __shared__ uint8_t smem_raw[];
  I8Channels pipe;
  const bool go = pipe.open(smem_raw);
  bool failed = false;
  if (pipe.warp == 0 && go) {
    failed = !i8_copies(pipe, a, channels, tokens);
  } else if (pipe.warp == 1 && go) {
    if (pipe.rank == 0) failed = !i8_products(pipe, a);
  } else if (go) {
    // ------------------------------ results (both blocks): a channel a thread ------------------------------
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const int lane = pipe.lane, q = pipe.warp & 3, part = (pipe.warp - 2) >> 2;
    float* scale_w = reinterpret_cast<float*>(pipe.extra) + (pipe.warp - 2) * 64;
    const int blocks = (a.width + 127) / 128;           // of 32 tokens of this warp, one where the tile is narrow
    const int tok0 = part * blocks * 32;
    uint32_t it = 0;
    for (int t = pair; t < a.total && !failed; t += pairs, ++it) {
      const int buf = (int)(it & 1);
      const int64_t n = (int64_t)i8_row(a, t) + (int)pipe.rank * PAIR_ROWS + q * 32 + lane;
      const int64_t m0 = (int64_t)i8_col(a, t) + tok0;
      const bool active = n - lane < a.N && tok0 < a.width && m0 < a.M;         // of the warp
      float sb = 0.f, bias = 0.f;
      if (active) {
        if (n < a.N) {
          sb = __ldg(a.scale_b + n);
          if (a.bias) bias = __ldg(a.bias + n);
        }
        __syncwarp();
        for (int b = 0; b < blocks; ++b) scale_w[b * 32 + lane] = m0 + b * 32 + lane < a.M ? __ldg(a.scale_a + m0 + b * 32 + lane) : 0.f;
        __syncwarp();
      }
      if (!mbar_wait_warp(pipe.tfull(buf), (it >> 1) & 1, pipe.abort_flag)) { failed = true; break; }
      tc_fence_after();
      if (active) {
        const uint32_t taddr = pipe.tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(buf * PAIR_COLS + tok0);
        for (int b = 0; b < blocks; ++b) {
          uint32_t v[32];
          tc_ld32_issue(taddr + b * 32, v);
          tc_ld32_wait(v);
          CT* to = reinterpret_cast<CT*>(a.C) + (m0 + b * 32) * a.ldc + n;
          const int left = n < a.N ? (int)min((int64_t)32, a.M - m0 - b * 32) : 0;
#pragma unroll
          for (int j = 0; j < 32; ++j) {
            const float x = fmaf((float)(int32_t)v[j] * scale_w[b * 32 + j], sb, bias);
            if (j < left) {
              if constexpr (sizeof(CT) == 4) to[j * a.ldc] = x;
              else to[j * a.ldc] = __float2bfloat16_rn(x);
            }
          }
          __syncwarp();
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_remote(pipe.lead_tempty(buf));
    }
  }
  pipe.close(failed, a.status);
}

// 2-D map of 8-bit elements: `inner` contiguous ones per row, rows `ld` apart; boxes of 128 of them x `rows`
bool make_map_i8(CUtensorMap* map, const void* base, uint64_t inner, uint64_t outer, uint64_t ld, uint32_t rows) {
  EncodeTiledFn fn = get_encode_fn();
  if (!fn) return false;
  cuuint64_t dims[2] = {inner, outer};
  cuuint64_t strides[1] = {ld};
  cuuint32_t box[2] = {I8_BK, rows};
  cuuint32_t es[2] = {1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

gram_status quantize_rows_launch(gram_ctx* ctx, const void* x, int dtype, int64_t ld, int64_t rows, int32_t cols, int8_t* codes, int64_t ld_codes,
                                 float* scale, cudaStream_t st) {
  ProfScope prof(ctx, GRAM_K_OTHER, (double)rows * cols * (dtype == GRAM_F32 ? 5 : 3), 1, st, "quantize_rows");
  if (dtype == GRAM_F32) launch_quantize<float>(x, ld, rows, cols, codes, ld_codes, scale, st);
  else launch_quantize<bf16>(x, ld, rows, cols, codes, ld_codes, scale, st);
  GRAM_LAUNCH_CHECK(ctx);
  return GRAM_OK;
}

gram_status gemm_i8_launch(gram_ctx* ctx, const int8_t* A, int64_t lda, const float* scale_a, const int8_t* B, int64_t ldb, const float* scale_b,
                           const float* bias, void* C, int c_dtype, int64_t ldc, int64_t M, int32_t N, int32_t K, cudaStream_t st) {
  I8Args a = {};
  a.scale_a = scale_a;
  a.scale_b = scale_b;
  a.bias = bias;
  a.C = C;
  a.ldc = ldc;
  a.M = M;
  a.N = N;
  a.num_kb = ceil_div(K, I8_BK);
  const size_t size = c_dtype == GRAM_F32 ? 4 : 2;
  const bool rows = M > PAIR_ROWS && (uintptr_t)C % 16 == 0 && ldc * size % 16 == 0 && N * size >= 16;
  a.width = rows || M > 128 ? 256 : M > 64 ? 128 : M > 32 ? 64 : 32;
  const int64_t tiles_r = ceil_div64(rows ? M : N, 2 * PAIR_ROWS), tiles_c = ceil_div64(rows ? N : M, a.width);
  if (tiles_r * tiles_c > INT32_MAX - kPairs) return gram_set_error(ctx, "gram_gemm_i8: %lld x %d are too many results", (long long)M, N), GRAM_ERR_UNSUPPORTED;
  a.total = (int32_t)(tiles_r * tiles_c);
  const bool resident = rows && a.num_kb <= I8_HELD;
  a.rows_fast = resident || tiles_r < tiles_c;
  a.fast = (int32_t)(a.rows_fast ? tiles_r : tiles_c);
  a.give_up = gram_ring_rows(ctx);
  a.status = gram_status_word(ctx);
  const uint32_t rows_a = rows ? PAIR_ROWS : (uint32_t)a.width / 2, rows_b = rows ? (uint32_t)a.width / 2 : PAIR_ROWS;
  CUtensorMap channels, tokens, result = {};
  if (!make_map_i8(&channels, B, (uint64_t)K, (uint64_t)N, (uint64_t)ldb, rows_b) || !make_map_i8(&tokens, A, (uint64_t)K, (uint64_t)M, (uint64_t)lda, rows_a) ||
      (rows && !(c_dtype == GRAM_F32 ? make_map_f32(&result, C, (uint64_t)i8_whole<float>(N), (uint64_t)M, (uint64_t)ldc, 32, 32)
                                     : make_map(&result, C, (uint64_t)i8_whole<bf16>(N), (uint64_t)M, (uint64_t)ldc, 64, 32))))
    return gram_set_error(ctx, "gram_gemm_i8: cannot describe the matrices"), GRAM_ERR_UNSUPPORTED;
  ProfScope prof(ctx, GRAM_K_GEMM, 2.0 * M * N * K, 1, st, "gemm_i8");
  const int pairs = a.total < kPairs ? a.total : kPairs;
#define I8_ROWS(KERN, PIPE)                                                                                                            \
  (c_dtype == GRAM_F32 ? (left ? launch_pairs<KERN<float, true>>(pairs, PIPE::THREADS, PIPE::SMEM, st, tokens, channels, result, a)      \
                               : launch_pairs<KERN<float, false>>(pairs, PIPE::THREADS, PIPE::SMEM, st, tokens, channels, result, a))    \
                       : (left ? launch_pairs<KERN<bf16, true>>(pairs, PIPE::THREADS, PIPE::SMEM, st, tokens, channels, result, a)       \
                               : launch_pairs<KERN<bf16, false>>(pairs, PIPE::THREADS, PIPE::SMEM, st, tokens, channels, result, a)))
  const bool left = N * size % 16 != 0;
  if (resident) {
    GRAM_CUDA(ctx, I8_ROWS(gemm_i8_resident_kernel, I8Resident));
  } else if (rows) {
    GRAM_CUDA(ctx, I8_ROWS(gemm_i8_rows_kernel, I8Rows));
#undef I8_ROWS
  } else {
    if (c_dtype == GRAM_F32) GRAM_CUDA(ctx, launch_pairs<gemm_i8_channels_kernel<float>>(pairs, I8Channels::THREADS, I8Channels::SMEM, st, channels, tokens, a));
    else GRAM_CUDA(ctx, launch_pairs<gemm_i8_channels_kernel<bf16>>(pairs, I8Channels::THREADS, I8Channels::SMEM, st, channels, tokens, a));
  }
  return GRAM_OK;
}
