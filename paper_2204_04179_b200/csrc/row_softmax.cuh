// Softmax statistics of a row that is read once, and the order of its entries, shared by the kernels on logits.
//
// A row's statistics are (m, s, t): m the largest logit, s = sum of e, t = sum of e y over e = 2^y, y = c (z - m),
// c = scale log2(e).  The difference z - m is taken before the product, so that logits of the type's lowest value stay what
// they are: scale z alone could overflow.  Then log p(z) = scale (z - m) - ln s and the entropy is ln 2 (log2 s - t / s).
// A masked place (-inf) has y = -inf; y is held at -200, where 2^y is 0 in 32 bits, so that e y is 0 there and not NaN.  The
// hold passes a NaN on, so a NaN (or +inf, whose z - m is one) reaches s and everything computed from it.
#pragma once
#include "gram_internal.h"

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
#define ROW_NEG_INF __int_as_float(0xff800000)

struct RowStat {
  float m, s, t;
};
__device__ __forceinline__ float row_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float row_hold(float y) {   // at least -200; NaN stays NaN
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(y), "f"(-200.f));
  return r;
}
// what differences are taken to: a row with nothing in it has m = -inf
__device__ __forceinline__ float row_base(float m) { return m == ROW_NEG_INF ? 0.f : m; }
__device__ __forceinline__ RowStat row_empty() { return RowStat{ROW_NEG_INF, 0.f, 0.f}; }
__device__ __forceinline__ RowStat row_join(const RowStat& a, const RowStat& b, float c) {
  RowStat r;
  r.m = fmaxf(a.m, b.m);
  const float base = row_base(r.m);
  const float da = row_hold((a.m - base) * c), db = row_hold((b.m - base) * c);
  const float fa = row_ex2(da), fb = row_ex2(db);
  r.s = a.s * fa + b.s * fb;
  r.t = fa * (a.t + a.s * da) + fb * (b.t + b.s * db);
  return r;
}
__device__ __forceinline__ void row_add(RowStat& r, float z, float c) {
  if (z > r.m) {
    const float d = row_hold((r.m - z) * c), f = row_ex2(d);
    r.t = f * (r.t + r.s * d);
    r.s *= f;
    r.m = z;
  }
  const float y = row_hold((z - row_base(r.m)) * c), e = row_ex2(y);
  r.s += e;
  r.t += e * y;
}
__device__ __forceinline__ RowStat row_join_warp(RowStat r, float c) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    RowStat x;
    x.m = __shfl_xor_sync(0xffffffffu, r.m, o);
    x.s = __shfl_xor_sync(0xffffffffu, r.s, o);
    x.t = __shfl_xor_sync(0xffffffffu, r.t, o);
    // the lower lane's statistics come first on both sides, so that both get the same bits
    r = (threadIdx.x & o) ? row_join(x, r, c) : row_join(r, x, c);
  }
  return r;
}
__device__ __forceinline__ float row_log_sum(const RowStat& r) { return logf(r.s); }
__device__ __forceinline__ float row_entropy(const RowStat& r) { return r.s == 0.f ? 0.f : logf(r.s) - kLn2 * (r.t / r.s); }
__device__ __forceinline__ float row_logp(float z, float m, float log_s, float scale) {
  if (z == ROW_NEG_INF) return log_s != log_s ? log_s : z;
  float y = (z - m) * scale;
  if (y == ROW_NEG_INF) y = z * scale - m * scale;   // only the difference may have left 32 bits (the two are of opposite signs then)
  return y - log_s;
}

// The order of alternatives: larger logits first, then lower places.  -0 counts as 0.
__device__ __forceinline__ uint64_t row_key(float z, uint32_t place) {
  const uint32_t u = __float_as_uint(z + 0.f);
  return ((uint64_t)(u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u)) << 32) | (uint32_t)~place;
}
__device__ __forceinline__ float row_key_logit(uint64_t key) {
  const uint32_t u = (uint32_t)(key >> 32);
  return __uint_as_float(u ^ ((u >> 31) ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ int32_t row_key_place(uint64_t key) { return (int32_t)~(uint32_t)key; }

template <typename T> __device__ __forceinline__ float row_load(const T* p);
template <> __device__ __forceinline__ float row_load<float>(const float* p) { return *p; }
template <> __device__ __forceinline__ float row_load<bf16>(const bf16* p) { return __bfloat162float(*p); }
template <typename T> __device__ __forceinline__ T row_round(float v);
template <> __device__ __forceinline__ float row_round<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16 row_round<bf16>(float v) { return __float2bfloat16_rn(v); }
