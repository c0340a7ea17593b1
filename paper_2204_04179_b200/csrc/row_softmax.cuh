// Softmax statistics of a row that is read once, and the order of its entries, shared by the kernels on logits.
//
// A row's statistics are (m, s, t): m the largest logit, s = sum of e, t = sum of e y over e = 2^y, y = c z - R(m),
// c = scale log2(e).  R(m) is c m rounded to a whole number: c z - R is one fused multiply-add with a single rounding, and
// statistics of different m differ by exact powers of two.  Then ln sum exp(scale (z - m)) = ln s + ln 2 (R - c m), and the
// entropy is ln 2 (log2 s - t / s).
// A masked place (-inf) has e = 0; in t its y is held at -200, so that e y is 0 and not NaN.  A NaN (or +inf, whose c z - R is
// one) reaches s and everything computed from it.
// Logits so large that c m has no place left for a fraction (all places of a row at the type's lowest value) are the exception,
// row_is_huge: their rows are summed again with the difference z - m taken first.  So are rows at a scale so far from 1 that c times
// the value at which masked places are held (row_held) is no longer a finite number far below all others.
#pragma once
#include <float.h>

#include "gram_internal.h"

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
#define ROW_NEG_INF (-__builtin_inff())

struct RowStat {
  float m, s, t;
};
__device__ __forceinline__ float row_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// R(m), held at -2^23: a thread that has seen nothing, or only logits of the type's lowest value, keeps sums of 0
__device__ __forceinline__ float row_ref(float m, float c) { return fmaxf(rintf(m * c), -8388608.f); }
__device__ __forceinline__ bool row_is_huge(float m, float c) {
  return fabsf(m) <= FLT_MAX && !(fabsf(m * c) <= 4194304.f && c >= 1e-20f && c <= 1e8f);
}
__device__ __forceinline__ RowStat row_empty() { return RowStat{ROW_NEG_INF, 0.f, 0.f}; }
// r's statistics as they are with a larger m
__device__ __forceinline__ void row_raise(RowStat& r, float m, float c) {
  const float d = fmaxf(row_ref(r.m, c) - row_ref(m, c), -200.f), f = row_ex2(d);
  r.t = f * fmaf(r.s, d, r.t);
  r.s *= f;
  r.m = m;
}
// A thread's own sums while it reads.  Their reference lags behind m: it is raised when an entry lies 2^4 above it, so that
// most chunks leave it alone (further behind, the entropy's two parts would grow large against their difference).
struct RowSums {
  float m, ref, s, t;
  __device__ __forceinline__ RowSums() : m(ROW_NEG_INF), ref(-8388608.f), s(0.f), t(0.f) {}
  __device__ __forceinline__ void see(float top, float c) {            // before entries of at most `top` are added
    m = fmaxf(m, top);
    if (fmaf(top, c, -ref) > 4.f) {
      const float up = row_ref(top, c), d = fmaxf(ref - up, -200.f), f = row_ex2(d);
      t = f * fmaf(s, d, t);
      s *= f;
      ref = up;
    }
  }
  __device__ __forceinline__ void add(float z, float c) {
    see(z, c);
    const float y = fmaf(z, c, -ref), e = row_ex2(y);
    s += e;
    t = fmaf(e, fmaxf(y, -200.f), t);
  }
  __device__ __forceinline__ RowStat stat(float c) const {
    const float d = fmaxf(ref - row_ref(m, c), -200.f), f = row_ex2(d);
    return RowStat{m, s * f, f * fmaf(s, d, t)};
  }
};
// the statistics of L neighbouring lanes, in all of them
template <int L> __device__ __forceinline__ RowStat row_join_lanes(RowStat r, float c) {
  float m = r.m;
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (m > r.m) row_raise(r, m, c);
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) {
    r.s += __shfl_xor_sync(0xffffffffu, r.s, o);
    r.t += __shfl_xor_sync(0xffffffffu, r.t, o);
  }
  return r;
}
// the sum of a row with nothing left (m = -inf): 0 at any scale, or NaN where the row holds one
__device__ __forceinline__ float row_none(const RowStat& r) { return r.s != r.s ? r.s : 0.f; }
__device__ __forceinline__ float row_log_sum(const RowStat& r, float c) {
  return r.m == ROW_NEG_INF ? logf(row_none(r)) : fmaf(fmaf(-r.m, c, row_ref(r.m, c)), kLn2, logf(r.s));
}
__device__ __forceinline__ float row_entropy(const RowStat& r) { return r.m == ROW_NEG_INF ? row_none(r) : logf(r.s) - kLn2 * (r.t / r.s); }
// the largest logit as it is answered: a maximum passes over NaN
__device__ __forceinline__ float row_largest(float m, float log_s) { return log_s != log_s ? log_s : m; }
__device__ __forceinline__ float row_logp(float z, float m, float log_s, float scale) {
  if (z == ROW_NEG_INF) return log_s != log_s ? log_s : z;
  const float d = z - m;
  // where only the difference has left 32 bits the two are of opposite signs, and the difference of their products is no NaN
  return (d == ROW_NEG_INF ? z * scale - m * scale : d * scale) - log_s;
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

__device__ __forceinline__ uint32_t row_order(float z) { return (uint32_t)(row_key(z, 0) >> 32); }
__device__ __forceinline__ float row_order_logit(uint32_t o) { return __uint_as_float(o ^ ((o >> 31) ? 0x80000000u : 0xffffffffu)); }

template <typename T> __device__ __forceinline__ float row_load(const T* p);
template <> __device__ __forceinline__ float row_load<float>(const float* p) { return *p; }
template <> __device__ __forceinline__ float row_load<bf16>(const bf16* p) { return __bfloat162float(*p); }
template <typename T> __device__ __forceinline__ T row_round(float v);
template <> __device__ __forceinline__ float row_round<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16 row_round<bf16>(float v) { return __float2bfloat16_rn(v); }

// A row belongs to TPR threads: a warp, or a block of that many.  All threads of a group call these together.
template <int TPR> struct Group {
  static constexpr int WARPS = TPR / 32;
  static __device__ __forceinline__ int tid() { return threadIdx.x % TPR; }
  static __device__ __forceinline__ int row() { return threadIdx.x / TPR; }
  static __device__ __forceinline__ void sync() {
    if constexpr (TPR == 32) __syncwarp();
    else __syncthreads();
  }
  static __device__ __forceinline__ int count(bool p) {        // of a block: also a barrier
    if constexpr (TPR == 32) return __popc(__ballot_sync(0xffffffffu, p));
    else return __syncthreads_count(p);
  }
  static __device__ __forceinline__ int sum(int v, int* part) {
    v = __reduce_add_sync(0xffffffffu, v);
    if constexpr (TPR > 32) {
      __syncthreads();
      if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
      __syncthreads();
      v = 0;
#pragma unroll
      for (int w = 0; w < WARPS; ++w) v += part[w];
    }
    return v;
  }
  static __device__ __forceinline__ float sum(float v, float* part) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if constexpr (TPR > 32) {
      __syncthreads();
      if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
      __syncthreads();
      v = 0.f;
#pragma unroll
      for (int w = 0; w < WARPS; ++w) v += part[w];
    }
    return v;
  }
  // the group's statistics in all its threads, joined in the same order everywhere
  static __device__ __forceinline__ RowStat join(RowStat r, float c, RowStat* part) {
    r = row_join_lanes<32>(r, c);
    if constexpr (TPR > 32) {
      __syncthreads();
      if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = r;
      __syncthreads();
      r = row_join_lanes<WARPS>(part[threadIdx.x & (WARPS - 1)], c);
    }
    return r;
  }
  // two at once
  static __device__ __forceinline__ void join(RowStat& r, RowStat& q, float c, RowStat (*part)[2]) {
    r = row_join_lanes<32>(r, c);
    q = row_join_lanes<32>(q, c);
    if constexpr (TPR > 32) {
      __syncthreads();
      if ((threadIdx.x & 31) == 0) { part[threadIdx.x >> 5][0] = r; part[threadIdx.x >> 5][1] = q; }
      __syncthreads();
      r = row_join_lanes<WARPS>(part[threadIdx.x & (WARPS - 1)][0], c);
      q = row_join_lanes<WARPS>(part[threadIdx.x & (WARPS - 1)][1], c);
    }
  }
};

// Pairs of fp32 values in one register pair, one instruction for the two.
typedef uint64_t f32x2;
__device__ __forceinline__ f32x2 x2_pack(float a, float b) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 x2_unpack(f32x2 v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ f32x2 x2_add(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 x2_mul(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 x2_fma(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

// a pair held above -inf (NaN stays): c z is then finite, and e y of a masked place 0
__device__ __forceinline__ f32x2 row_held(float a, float b) {
  asm("max.NaN.f32 %0, %0, %1;" : "+f"(a) : "f"(-1e30f));
  asm("max.NaN.f32 %0, %0, %1;" : "+f"(b) : "f"(-1e30f));
  return x2_pack(a, b);
}

template <typename T> struct RowVec;                 // 16 bytes of logits
template <> struct RowVec<float> {
  static constexpr int N = 4;
  static constexpr uint32_t NONE = 0xff800000u;      // a word of masked places
  static __device__ __forceinline__ float top(const uint4& q) {
    return fmaxf(fmaxf(__uint_as_float(q.x), __uint_as_float(q.y)), fmaxf(__uint_as_float(q.z), __uint_as_float(q.w)));
  }
  static __device__ __forceinline__ float2 pair(const uint4& q, int i) {
    return i == 0 ? make_float2(__uint_as_float(q.x), __uint_as_float(q.y)) : make_float2(__uint_as_float(q.z), __uint_as_float(q.w));
  }
  static __device__ __forceinline__ f32x2 held(const uint4& q, int i) {
    const float2 x = pair(q, i);
    return row_held(x.x, x.y);
  }
  static __device__ __forceinline__ void put(uint4& q, int i, float2 v) {
    if (i == 0) { q.x = __float_as_uint(v.x); q.y = __float_as_uint(v.y); }
    else { q.z = __float_as_uint(v.x); q.w = __float_as_uint(v.y); }
  }
};
template <> struct RowVec<bf16> {
  static constexpr int N = 8;
  static constexpr uint32_t NONE = 0xff80ff80u;
  static __device__ __forceinline__ float top(const uint4& q) {
    const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&q);
    const __nv_bfloat162 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
    return fmaxf(__low2float(m), __high2float(m));
  }
  static __device__ __forceinline__ float2 pair(const uint4& q, int i) {
    const uint32_t w = i == 0 ? q.x : i == 1 ? q.y : i == 2 ? q.z : q.w;
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  }
  static __device__ __forceinline__ f32x2 held(const uint4& q, int i) {
    uint32_t w = i == 0 ? q.x : i == 1 ? q.y : i == 2 ? q.z : q.w;
    asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(w) : "r"(0xf149f149u));     // -1e30
    return x2_pack(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  }
  static __device__ __forceinline__ void put(uint4& q, int i, float2 v) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(v.x, v.y);
    const uint32_t w = *reinterpret_cast<const uint32_t*>(&h);
    if (i == 0) q.x = w; else if (i == 1) q.y = w; else if (i == 2) q.z = w; else q.w = w;
  }
};

// NV vectors' worth of logits, of at most `top`; ENTROPY: the sum of e y too
template <typename T, bool ENTROPY, int NV>
__device__ __forceinline__ void row_add_vectors(RowSums& r, const uint4 (&q)[NV], float top, float c) {
  r.see(top, c);
  f32x2 s = x2_pack(0.f, 0.f), t = s;                    // sums of their own: small terms would be lost in the row's so far
  const f32x2 cc = x2_pack(c, c), ref = x2_pack(-r.ref, -r.ref);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
#pragma unroll
    for (int j = 0; j < RowVec<T>::N / 2; ++j) {
      const float2 x = RowVec<T>::pair(q[i], j);
      const f32x2 y = x2_fma(ENTROPY ? RowVec<T>::held(q[i], j) : x2_pack(x.x, x.y), cc, ref);
      const float2 y2 = x2_unpack(y);
      const f32x2 e = x2_pack(row_ex2(y2.x), row_ex2(y2.y));
      s = x2_add(s, e);
      if (ENTROPY) t = x2_fma(e, y, t);
    }
  }
  const float2 s2 = x2_unpack(s), t2 = x2_unpack(t);
  r.s += s2.x + s2.y;
  if (ENTROPY) r.t += t2.x + t2.y;
}
