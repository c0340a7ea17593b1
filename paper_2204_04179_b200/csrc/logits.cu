// Answers read from rows of logits, and their gradients (gram_logprobs, gram_logprobs_backward, gram_distill).
//
// All three are bound by the bytes of the logits: each is read from HBM once, and a gradient is written once.  A row belongs
// to a group of threads, a warp for short rows (four rows a block) or a block of 128, and where a row is long or rows are
// few, to a cluster of up to 8 blocks with a contiguous slice each, whose statistics meet in distributed shared memory.
// Rows begin anywhere (a stride of 30 522 bf16 leaves them on 4-byte boundaries): the places up to the first 16-byte
// boundary and after the last are single elements of the slice's first threads, all others move 16 bytes at a time, four
// vectors a thread and chunk, the next chunk's on their way while one is added up.
// Measured (bytes of the logits, read once and a gradient written once, over the time of a call among others whose inputs L2 does not
// hold; the copy rate is 6458 GB/s):
//   log probabilities  25 600 x 10 000 fp32 159 us (6440 GB/s), 4096 x 30 522 bf16 47.5 (5260); with 64 alternatives 73 (3430: issue
//                      slots, 14 instructions an element, 8 without alternatives)
//   gradient           4096 x 30 522 bf16 86 us (5800)
//   distillation       8192 x 30 522 bf16 228 us (4390: a fifth of the second walk's reads miss L2), 256 x 100 000 fp32 51 (4020)
#include "logits.h"
#include "row_softmax.cuh"
#include "row_top.cuh"

namespace {

constexpr int LP_NV = 4, LP_PER_SM = 8;                           // vectors of a thread's chunk; blocks that an SM holds
constexpr int LP_THREADS = 128, LP_WARPS = LP_THREADS / 32;      // of a block

// ------------------------------ a slice of a row ----------------------------------------------------------------------
// Places [0, head) and [tail, V) are single elements, of the first and the last slice; the vectors between them are split
// evenly: a slice holds vectors [v0, v1), vector v the places head + v N ..
template <typename T> struct Slice {
  static constexpr int N = RowVec<T>::N;
  const T* z;                    // the row
  int head, tail, V, v0, v1;
  bool first, last;
  __device__ __forceinline__ Slice(const T* row, int V_, int rank, int shift) : z(row), V(V_), first(rank == 0), last(rank == (1 << shift) - 1) {
    const int past = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
    head = min(past ? N - past : 0, V);
    const int nv = (V - head) / N;
    tail = head + nv * N;
    const int per = (nv + (1 << shift) - 1) >> shift;     // 2^shift slices
    v0 = min(rank * per, nv);
    v1 = min(v0 + per, nv);
  }
  // A thread's single element: threads 0 .. 7 those at the row's start, 8 .. 15 those at its end.  -1: none
  __device__ __forceinline__ int edge(int tid) const {
    if (tid < 8) return first && tid < head ? tid : -1;
    return last && tid < 16 && tid - 8 < V - tail ? tail + (tid - 8) : -1;        // (tail + tid may leave 32 bits)
  }
  __device__ __forceinline__ int place(int v) const { return head + v * N; }
  __device__ __forceinline__ const uint4* vectors() const { return reinterpret_cast<const uint4*>(z + head); }
  template <bool LAST> __device__ __forceinline__ uint4 load(int v) const {        // LAST: nobody reads it again
    return LAST ? __ldcs(vectors() + v) : vectors()[v];
  }
  __device__ __forceinline__ bool has(int p) const {
    if (p < head) return first;
    if (p >= tail) return last;
    return p >= place(v0) && p < place(v1);
  }
  template <int TPR, int NV> __device__ __forceinline__ int chunks() const { return max(1, (v1 - v0 + TPR * NV - 1) / (TPR * NV)); }
  template <int TPR, int NV, bool LAST> __device__ __forceinline__ void load_chunk(int ch, int tid, uint4 (&q)[NV]) const {
    const int v = v0 + ch * (TPR * NV) + tid;
    if (v - tid + TPR * NV <= v1) {
#pragma unroll
      for (int i = 0; i < NV; ++i) q[i] = load<LAST>(v + i * TPR);
    } else {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        constexpr uint32_t none = RowVec<T>::NONE;
        q[i] = make_uint4(none, none, none, none);
        if (v + i * TPR < v1) q[i] = load<LAST>(v + i * TPR);
      }
    }
  }
};
// the largest of a chunk's entries of a thread
template <typename T, int NV> __device__ __forceinline__ float chunk_top(const uint4 (&q)[NV]) {
  float top = RowVec<T>::top(q[0]);
#pragma unroll
  for (int i = 1; i < NV; ++i) top = fmaxf(top, RowVec<T>::top(q[i]));
  return top;
}

// the same address in another block of the cluster
__device__ __forceinline__ uint32_t in_block(const void* p, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
  return r;
}
__device__ __forceinline__ void put_stat(RowStat* p, uint32_t rank, const RowStat& r) {
  asm volatile("st.shared::cluster.f32 [%0], %1;\n\tst.shared::cluster.f32 [%0+4], %2;\n\tst.shared::cluster.f32 [%0+8], %3;" ::"r"(in_block(p, rank)),
               "f"(r.m), "f"(r.s), "f"(r.t)
               : "memory");
}
__device__ __forceinline__ void put_key(uint64_t* p, uint32_t rank, uint64_t key) {
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(in_block(p, rank)), "l"(key) : "memory");
}
constexpr int MAX_SLICES = 8;
// the slices' statistics, joined in the same order everywhere
__device__ __forceinline__ RowStat join_slices(const RowStat* of, int slices, float c) {
  const int i = threadIdx.x & (MAX_SLICES - 1);
  return row_join_lanes<MAX_SLICES>(i < slices ? of[i] : row_empty(), c);
}

// The statistics of a row whose largest logit m is huge (row_is_huge), by one group: relative to m itself, R = c m is not used.
template <typename T, int TPR> __device__ __noinline__ float2 huge_sums(const T* z, int V, float m, float c, float* part) {
  using G = Group<TPR>;
  float s = 0.f, t = 0.f;
  for (uint32_t v = G::tid(); v < (uint32_t)V; v += TPR) {          // V + TPR may leave 31 bits
    const float y = (row_load(z + v) - m) * c, e = row_ex2(y);
    s += e;
    t = fmaf(e, fmaxf(y, -200.f), t);
  }
  s = G::sum(s, part);
  t = G::sum(t, part);
  return make_float2(s, t);
}
// of a row: ln of the sum of exp(scale (z - m)), the entropy
struct RowLogs { float log_s, entropy; };
template <typename T, int TPR> __device__ __forceinline__ RowLogs row_logs(const RowStat& r, const T* z, int V, float c, float* part) {
  if (row_is_huge(r.m, c)) {
    const float2 h = huge_sums<T, TPR>(z, V, r.m, c, part);
    return RowLogs{logf(h.x), logf(h.x) - kLn2 * (h.y / h.x)};
  }
  return RowLogs{row_log_sum(r, c), row_entropy(r)};
}

// ------------------------------ log probabilities ---------------------------------------------------------------------
template <typename T, int TPR, bool TOP>
__global__ void __launch_bounds__(LP_THREADS, TOP && TPR == 32 ? 7 : LP_PER_SM) logprobs_kernel(const T* logits, int64_t ld, int64_t N, int32_t V, float scale, int32_t shift,
                                                                 RowAnswers ask, int32_t* status) {
  using G = Group<TPR>;
  constexpr int NV = LP_NV;
  if (!chain_begin()) return;
  __shared__ RowStat part[LP_WARPS], of_slice[MAX_SLICES];
  __shared__ float fpart[LP_WARPS];
  __shared__ __align__(16) uint8_t scratch[TOP ? sizeof(TopScratch<TPR>) * (LP_THREADS / TPR) : 16];
  extern __shared__ uint64_t merged[];                  // [slices, k]: every slice's best, sorted, zeros behind them
  __shared__ uint64_t of_have[MAX_SLICES];
  const int slices = TPR == 32 ? 1 : 1 << shift, tid = G::tid(), rank = blockIdx.x & (slices - 1);
  const int64_t n = TPR == 32 ? (int64_t)blockIdx.x * LP_WARPS + G::row() : blockIdx.x >> shift;
  if (TPR > 32 && slices > 1) gram_cluster_sync();      // every block of the cluster runs before another writes to it
  if (n >= N) return;                                   // whole warps, in the form that has no barrier over the block
  TopScratch<TPR>& sc = reinterpret_cast<TopScratch<TPR>*>(scratch)[TOP ? G::row() : 0];
  const float c = scale * kLog2e;
  uint4 q[NV], next[NV];
  const Slice<T> s(logits + n * ld, V, rank, shift);
  s.template load_chunk<TPR, NV, !TOP>(0, tid, q);
  const int edge_place = s.edge(tid);
  const float edge = edge_place >= 0 ? row_load(s.z + edge_place) : ROW_NEG_INF;
  const int chunks = s.template chunks<TPR, NV>();
  RowSums sums;
  float tops[NV], top_group = ROW_NEG_INF;               // the largest of the thread's i-th vectors so far, and of a group's entries
  int group_shift = 0, group = 0;
  if constexpr (TOP) {
#pragma unroll
    for (int i = 0; i < NV; ++i) tops[i] = ROW_NEG_INF;
    while (((chunks - 1) >> group_shift) >= TopScratch<TPR>::GROUPS) ++group_shift;
    if (tid == 0) sc.entries = sc.found = 0;             // the statistics' barriers come before their use
  }
#pragma unroll 2
  for (int ch = 0; ch < chunks; ++ch) {
    if (ch + 1 < chunks) s.template load_chunk<TPR, NV, !TOP>(ch + 1, tid, next);
    float top = ROW_NEG_INF;
    if constexpr (TOP) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const float x = RowVec<T>::top(q[i]);
        tops[i] = fmaxf(tops[i], x);
        top = fmaxf(top, x);
      }
      top_group = fmaxf(top_group, top);
    } else {
      top = chunk_top<T>(q);
    }
    row_add_vectors<T, true>(sums, q, top, c);
    if constexpr (TOP) {
      if (((ch + 1) & ((1 << group_shift) - 1)) == 0 || ch == chunks - 1) {
        sc.group[group * TPR + tid] = top_group;
        top_group = ROW_NEG_INF;
        ++group;
      }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) q[i] = next[i];
  }
  if (edge_place >= 0) sums.add(edge, c);
  RowStat r = G::join(sums.stat(c), c, part);
  int have = 0;
  const uint64_t* list = sc.keys;
  if constexpr (TOP) {
    if (TPR == 32) G::sync();
    if (edge_place >= 0) tops[0] = fmaxf(tops[0], edge);
    const float bar = top_bar<TPR>(tops, ask.k, sc);
    have = top_collect<T, TPR, NV>(sc, TopSource{s.vectors(), s.head, s.v0, s.v1, edge, edge_place}, group, group_shift, bar, ask.k);
    top_sort<TPR>(sc.keys, have);
  }
  if (TPR > 32 && slices > 1) {
    if (TOP ? tid < slices : tid == 0) put_stat(&of_slice[rank], tid, r);
    if constexpr (TOP) {                                // this slice's best to every block, whose places each block then finds for its own
      if (tid < slices) put_key(&of_have[rank], tid, min(have, ask.k));
      for (int i = tid; i < max(have, ask.k); i += TPR) {
        const int at = i < have ? top_above<TPR>(list, have, i) : i;
        if (at < ask.k)
          for (int b = 0; b < slices; ++b) put_key(&merged[rank * ask.k + at], b, i < have ? list[i] : 0);
      }
    }
    gram_cluster_sync();
    if (!TOP && rank != 0) return;
    r = join_slices(of_slice, slices, c);
  }
  const RowLogs logs = row_logs<T, TPR>(r, s.z, V, c, fpart);
  const float log_s = logs.log_s;
  if (tid == 0 && rank == 0) {
    if (ask.stats) { ask.stats[2 * n] = row_largest(r.m, log_s); ask.stats[2 * n + 1] = log_s; }
    if (ask.entropy) ask.entropy[n] = logs.entropy;
  }
  for (int i = tid; rank == 0 && i < ask.C; i += TPR) {
    const int32_t t = ask.targets[n * ask.C + i];
    if (t < -1 || t >= V) gram_device_fail(status, GRAM_ERR_ID_RANGE);
    ask.logp[n * ask.C + i] = t >= 0 && t < V ? row_logp(row_load(s.z + t), r.m, log_s, scale) : 0.f;
  }
  if constexpr (TOP) {
    const int64_t o = n * ask.k;
    auto answer = [&](int at, uint64_t key) {
      ask.top_ids[o + at] = key ? row_key_place(key) : -1;
      ask.top_logp[o + at] = key ? row_logp(row_key_logit(key), r.m, log_s, scale) : ROW_NEG_INF;
    };
    if (TPR == 32 || slices == 1) {
      for (int i = tid; i < have; i += TPR) {
        const int above = top_above<TPR>(list, have, i);
        if (above < ask.k) answer(above, list[i]);
      }
      for (int i = have + tid; i < ask.k; i += TPR) answer(i, 0);
    } else {
      const int first_step = 1 << (31 - __clz(ask.k));
      int found = 0;
      for (int b = 0; b < slices; ++b) found += (int)of_have[b];
      for (int i = tid; i < (int)of_have[rank]; i += TPR) {
        const uint64_t key = merged[rank * ask.k + i];
        int at = 0;
        for (int b = 0; b < slices; b += 2) {           // there are two slices at least; keys of both lists above this one
          int lo0 = 0, lo1 = 0;
          const uint64_t *l0 = merged + b * ask.k, *l1 = l0 + ask.k;
          for (int step = first_step; step > 0; step >>= 1) {
            if (lo0 + step <= ask.k && l0[lo0 + step - 1] > key) lo0 += step;
            if (lo1 + step <= ask.k && l1[lo1 + step - 1] > key) lo1 += step;
          }
          at += lo0 + lo1;
        }
        if (at < ask.k) answer(at, key);
      }
      if (rank == 0)
        for (int i = found + tid; i < ask.k; i += TPR) answer(i, 0);
    }
  }
}

// ------------------------------ gradients -----------------------------------------------------------------------------
// Rows of the gradient may begin elsewhere within 16 bytes than the logits': a vector is then stored in pieces of the size that
// its address allows (bytes: 16, 8, 4 or, for bf16, 2; the same for all vectors of a row).
template <typename T> __device__ __forceinline__ int store_bytes(const T* first) {
  const uint32_t a = (uint32_t)reinterpret_cast<uintptr_t>(first);
  return a % 16 == 0 ? 16 : a % 8 == 0 ? 8 : a % 4 == 0 ? 4 : 2;
}
template <typename T> __device__ __forceinline__ void store_vector(T* at, const uint4& q, int bytes) {
  if (bytes == 16) {
    __stcs(reinterpret_cast<uint4*>(at), q);
  } else if (bytes == 8) {
    __stcs(reinterpret_cast<uint2*>(at), make_uint2(q.x, q.y));
    __stcs(reinterpret_cast<uint2*>(at) + 1, make_uint2(q.z, q.w));
  } else if (bytes == 4) {
    __stcs(reinterpret_cast<uint32_t*>(at), q.x);
    __stcs(reinterpret_cast<uint32_t*>(at) + 1, q.y);
    __stcs(reinterpret_cast<uint32_t*>(at) + 2, q.z);
    __stcs(reinterpret_cast<uint32_t*>(at) + 3, q.w);
  } else {
    const uint16_t* e = reinterpret_cast<const uint16_t*>(&q);
#pragma unroll
    for (int j = 0; j < 8; ++j) reinterpret_cast<uint16_t*>(at)[j] = e[j];
  }
}
// pairs of logits -> pairs of results, over a chunk that is in registers: `plain` for whole chunks of rows that lie alike within 16
// bytes, where `fast` says that it holds, and `any` otherwise (one straight line each: with the tests at every vector a gradient
// took 10 instructions an element instead of 8)
template <typename T, int TPR, int NV, typename F, typename A>
__device__ __forceinline__ void store_chunk(const Slice<T>& s, int ch, int tid, const uint4 (&q)[NV], T* dz, int bytes, bool fast, F plain, A any) {
  const int v = s.v0 + ch * (TPR * NV) + tid;
  T* at = dz + ((uint32_t)s.head + (uint32_t)v * RowVec<T>::N);       // v may lie past the slice, and its place past 31 bits
  if (fast && v - tid + TPR * NV <= s.v1) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      uint4 o;
#pragma unroll
      for (int j = 0; j < RowVec<T>::N / 2; ++j) RowVec<T>::put(o, j, plain(RowVec<T>::pair(q[i], j)));
      __stcs(reinterpret_cast<uint4*>(at + i * (TPR * RowVec<T>::N)), o);
    }
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (v + i * TPR < s.v1) {
        uint4 o;
#pragma unroll
        for (int j = 0; j < RowVec<T>::N / 2; ++j) RowVec<T>::put(o, j, any(RowVec<T>::pair(q[i], j)));
        store_vector(at + i * (TPR * RowVec<T>::N), o, bytes);
      }
    }
  }
}

// p of a logit x, given its row's statistics: 2^y / s, y = c x - R(m) as in row_softmax.cuh, or c (x - m) in a row of huge logits.
struct RowPower {
  float m, c, ref, log2_s;           // log2_s: of the sum that belongs to y
  bool is_huge;
  __device__ __forceinline__ RowPower(float m_, float log_s, float c_) : m(m_), c(c_), ref(row_ref(m_, c_)), is_huge(row_is_huge(m_, c_)) {
    log2_s = log_s * kLog2e + (is_huge ? 0.f : fmaf(m, c, -ref));
  }
  __device__ __forceinline__ float2 plain(float2 x) const { return x2_unpack(x2_fma(x2_pack(x.x, x.y), x2_pack(c, c), x2_pack(-ref, -ref))); }
  __device__ __forceinline__ float2 huge(float2 x) const { return make_float2((x.x - m) * c, (x.y - m) * c); }
};

struct BackwardArgs {
  const int32_t* targets;
  const float* stats;
  const float* entropy;
  const float* dlogp;
  const float* dentropy;
  int64_t ld, ld_out, N;
  int32_t V, C, shift;
  float scale;
  int32_t* status;
};

// What a row has at given places (the given tokens with their gradients, the teacher's entries with their logits): each thread
// holds EPT of them.
template <int TPR> struct AtPlaces {
  static constexpr int EPT = GRAM_TOP_MAX / TPR;
  int32_t id[EPT];
  float given[EPT], z[EPT];
  __device__ __forceinline__ void load_ids(const int32_t* ids, const float* values, int64_t n, int count, int V, int tid, int32_t* status) {
#pragma unroll
    for (int e = 0; e < EPT; ++e) {
      const int i = tid + e * TPR;
      id[e] = -1;
      given[e] = 0.f;
      if (i < count) {
        id[e] = ids[n * count + i];
        given[e] = values[n * count + i];
        if (id[e] < -1 || id[e] >= V) { gram_device_fail(status, GRAM_ERR_ID_RANGE); id[e] = -1; }
      }
    }
  }
  template <typename T> __device__ __forceinline__ void load_logits(const T* row) {
#pragma unroll
    for (int e = 0; e < EPT; ++e) z[e] = id[e] >= 0 ? row_load(row + id[e]) : ROW_NEG_INF;
  }
};
// The entries that take part, as all threads see them.
struct alignas(16) PlacesShared {
  int32_t place[GRAM_TOP_MAX];   // -1: takes no part
  float value[GRAM_TOP_MAX];
  // whether entry i is the first at its place, and the sum of all values there
  __device__ __forceinline__ bool sum_at(int i, int count, float& sum) const {
    const int p = place[i];
    int same = 0, before = 0;
#pragma unroll 4
    for (int j = 0; j < count; j += 4) {               // what lies behind `count` is -1
      const int4 q = *reinterpret_cast<const int4*>(place + j);
      const int n = (q.x == p) + (q.y == p) + (q.z == p) + (q.w == p);
      same += n;
      if (j + 3 < i) before += n;
    }
    sum = value[i];
    if (same == 1) return true;                         // as good as always
    for (int j = i & ~3; j < i; ++j) before += place[j] == p;
    if (before > 0) return false;
    sum = 0.f;
    for (int j = i; j < count; ++j)
      if (place[j] == p) sum += value[j];
    return true;
  }
};

// dz = scale (sum of g at the given places - p (sum of all g + h (log p + H))), 0 at masked places.  With l = log2 p the
// dense part is 2^l (A + B l), A = -scale (G + h H), B = -scale h ln 2, or in y = l + log2 s, which takes one rounding less per
// element, 2^y (A - B log2 s + B y) / s; y is held at -200 as in row_softmax.cuh.
template <typename T, int TPR>
__global__ void __launch_bounds__(LP_THREADS, LP_PER_SM) logprobs_backward_kernel(const T* logits, T* dlogits, BackwardArgs a) {
  using G = Group<TPR>;
  using At = AtPlaces<TPR>;
  constexpr int NV = LP_NV;
  if (!chain_begin()) return;
  __shared__ PlacesShared places[LP_THREADS / TPR];
  const int slices = TPR == 32 ? 1 : 1 << a.shift, tid = G::tid(), rank = blockIdx.x & (slices - 1);
  const int64_t n = TPR == 32 ? (int64_t)blockIdx.x * LP_WARPS + G::row() : blockIdx.x >> a.shift;
  if (n >= a.N) return;
  const float c = a.scale * kLog2e;
  uint4 q[NV], next[NV];
  const Slice<T> s(logits + n * a.ld, a.V, rank, a.shift);
  At at;
  s.template load_chunk<TPR, NV, true>(0, tid, q);
  at.load_ids(a.targets, a.dlogp, n, a.C, a.V, tid, a.status);
  at.load_logits(s.z);
  PlacesShared& here = places[G::row()];
  const float m = a.stats[2 * n], log_s = a.stats[2 * n + 1], h = a.dentropy ? a.dentropy[n] : 0.f, H = a.dentropy ? a.entropy[n] : 0.f;
  T* dz = dlogits + n * a.ld_out;
  const int bytes = store_bytes(dz + s.head);
  const int edge_place = s.edge(tid);
  const float edge = edge_place >= 0 ? row_load(s.z + edge_place) : ROW_NEG_INF;
  float sum = 0.f;
  if (a.C > 0) {
#pragma unroll
    for (int e = 0; e < At::EPT; ++e)
      if (tid + e * TPR < ((a.C + 3) & ~3)) {
        const bool use = at.z[e] != ROW_NEG_INF;      // "none" and masked places take no part
        here.place[tid + e * TPR] = use ? at.id[e] : -1;
        here.value[tid + e * TPR] = use ? at.given[e] : 0.f;
      }
    // in place, no slice may be overwritten before all have read the given tokens' logits
    if (TPR > 32 && slices > 1) gram_cluster_sync();
    else G::sync();
    for (int i = 0; i < a.C; ++i) sum += here.value[i];
  }
  const float A = -a.scale * fmaf(h, H, sum), B = -a.scale * h * kLn2;
  // nothing asked of a row without NaN, or nothing left in the row
  const bool none = (sum == 0.f && h == 0.f && log_s == log_s) || log_s == ROW_NEG_INF;
  const RowPower l(m, log_s, c);
  const float inv = exp2f(-l.log2_s), Ay = inv * fmaf(-B, l.log2_s, A), By = inv * B;
  auto value = [&](float2 y) {
    return make_float2(row_ex2(y.x) * fmaf(fmaxf(y.x, -200.f), By, Ay), row_ex2(y.y) * fmaf(fmaxf(y.y, -200.f), By, Ay));
  };
  auto plain = [&](float2 x) { return value(l.plain(x)); };
  auto any = [&](float2 x) { return none ? make_float2(0.f, 0.f) : value(l.is_huge ? l.huge(x) : l.plain(x)); };
  auto one = [&](float x) { return any(make_float2(x, x)).x; };
  const int chunks = s.template chunks<TPR, NV>();
  const bool fast = bytes == 16 && !none && !l.is_huge;
#pragma unroll 2
  for (int ch = 0; ch < chunks; ++ch) {
    if (ch + 1 < chunks && !none) s.template load_chunk<TPR, NV, true>(ch + 1, tid, next);
    store_chunk<T, TPR, NV>(s, ch, tid, q, dz, bytes, fast, plain, any);
#pragma unroll
    for (int i = 0; i < NV; ++i) q[i] = next[i];
  }
  if (edge_place >= 0) dz[edge_place] = row_round<T>(one(edge));
  if (a.C > 0) {
    G::sync();                                        // the given places are written again, by one thread each
#pragma unroll
    for (int e = 0; e < At::EPT; ++e) {
      const int i = tid + e * TPR;
      float g;
      if (i < a.C && here.place[i] >= 0 && s.has(here.place[i]) && here.sum_at(i, a.C, g))
        dz[here.place[i]] = row_round<T>(fmaf(a.scale, g, one(at.z[e])));
    }
  }
}

struct DistillArgs {
  const int32_t* ids;
  const float* teacher;
  float* loss;
  const float* weight;
  int64_t ld, ld_out, N;
  int32_t V, k, shift;
  float scale;
  int32_t* status;
};

// A slice is walked over twice: forwards for the statistics, backwards for the gradient, whose reads find it in L2 (the last
// chunk is still in registers).  The plan keeps the slices of the blocks that run together well below L2's size.
template <typename T, int TPR>
__global__ void __launch_bounds__(LP_THREADS, TPR == 32 ? 6 : LP_PER_SM) distill_kernel(const T* logits, T* dlogits, DistillArgs a) {
  using G = Group<TPR>;
  using At = AtPlaces<TPR>;
  constexpr int NV = LP_NV;
  if (!chain_begin()) return;
  __shared__ RowStat part[LP_WARPS][2], of_slice[MAX_SLICES];
  __shared__ float fpart[LP_WARPS];
  __shared__ PlacesShared places[LP_THREADS / TPR];
  const int slices = TPR == 32 ? 1 : 1 << a.shift, tid = G::tid(), rank = blockIdx.x & (slices - 1);
  const int64_t n = TPR == 32 ? (int64_t)blockIdx.x * LP_WARPS + G::row() : blockIdx.x >> a.shift;
  if (n >= a.N) return;
  const float c = a.scale * kLog2e;
  uint4 q[NV], next[NV];
  const Slice<T> s(logits + n * a.ld, a.V, rank, a.shift);
  At at;
  s.template load_chunk<TPR, NV, false>(0, tid, q);
  at.load_ids(a.ids, a.teacher, n, a.k, a.V, tid, a.status);
  at.load_logits(s.z);
  if (TPR > 32 && slices > 1) gram_cluster_sync();       // every block of the cluster runs before another writes to it
  PlacesShared& here = places[G::row()];
  const float w = (a.weight ? a.weight[n] : 1.f) * a.scale;
  const int edge_place = s.edge(tid);
  const float edge = edge_place >= 0 ? row_load(s.z + edge_place) : ROW_NEG_INF;
  const int chunks = s.template chunks<TPR, NV>();
  RowSums sums, teacher;
#pragma unroll 2
  for (int ch = 0; ch < chunks; ++ch) {
    const int then = ch + 1 < chunks ? ch + 1 : chunks - 2;    // the second walk begins with the last chunk, which stays in q
    if (then >= 0) s.template load_chunk<TPR, NV, false>(then, tid, next);
    row_add_vectors<T, false>(sums, q, chunk_top<T>(q), c);
    if (ch + 1 < chunks) {
#pragma unroll
      for (int i = 0; i < NV; ++i) q[i] = next[i];
    }
  }
  if (edge_place >= 0) sums.add(edge, c);
  bool use[At::EPT];
#pragma unroll
  for (int e = 0; e < At::EPT; ++e) {
    use[e] = at.z[e] != ROW_NEG_INF && at.given[e] != ROW_NEG_INF;
    if (use[e]) teacher.add(at.given[e], c);
  }
  RowStat r = sums.stat(c), t = teacher.stat(c);
  G::join(r, t, c, part);
  if (TPR > 32 && slices > 1) {
    if (tid < slices) put_stat(&of_slice[rank], tid, r);
    gram_cluster_sync();                               // all have read the teacher's places by now, too
    r = join_slices(of_slice, slices, c);
  }
  const float log_s = row_logs<T, TPR>(r, s.z, a.V, c, fpart).log_s;
  float log_t = row_log_sum(t, c);
  if (row_is_huge(t.m, c)) {
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < At::EPT; ++e)
      if (use[e]) sum += row_ex2((at.given[e] - t.m) * c);
    log_t = logf(G::sum(sum, fpart));
  }
  // such a row was read again as a whole: in place, no slice may be overwritten before all have done so
  if (TPR > 32 && slices > 1 && row_is_huge(r.m, c)) gram_cluster_sync();
  float loss = 0.f;
#pragma unroll
  for (int e = 0; e < At::EPT; ++e) {
    float qi = 0.f;
    if (use[e]) {
      const float lq = (at.given[e] - t.m) * a.scale - log_t;
      qi = expf(lq);
      if (!(qi == 0.f)) loss += qi * (lq - row_logp(at.z[e], r.m, log_s, a.scale));
    }
    if (tid + e * TPR < ((a.k + 3) & ~3)) {
      here.place[tid + e * TPR] = use[e] ? at.id[e] : -1;
      here.value[tid + e * TPR] = qi;
    }
  }
  if (rank == 0) {
    loss = G::sum(loss, fpart);
    if (tid == 0) a.loss[n] = loss;
  }
  if (!dlogits) return;
  // no teacher entry takes part: no largest one, and no NaN among them (the sum alone is 0 for large entries too, which were summed
  // again above)
  const bool none = w == 0.f || (t.m == ROW_NEG_INF && t.s == 0.f);
  T* dz = dlogits + n * a.ld_out;
  const int bytes = store_bytes(dz + s.head);
  const RowPower l(r.m, log_s, c);
  const float w_s = w * exp2f(-l.log2_s);
  const f32x2 ww = x2_pack(w_s, w_s);
  auto value = [&](float2 y) { return x2_unpack(x2_mul(x2_pack(row_ex2(y.x), row_ex2(y.y)), ww)); };
  auto plain = [&](float2 x) { return value(l.plain(x)); };
  auto any = [&](float2 x) { return none ? make_float2(0.f, 0.f) : value(l.is_huge ? l.huge(x) : l.plain(x)); };
  auto one = [&](float x) { return any(make_float2(x, x)).x; };
  const bool fast = bytes == 16 && !none && !l.is_huge;
#pragma unroll 2
  for (int ch = chunks - 1; ch >= 0; --ch) {
    store_chunk<T, TPR, NV>(s, ch, tid, q, dz, bytes, fast, plain, any);
#pragma unroll
    for (int i = 0; i < NV; ++i) q[i] = next[i];
    if (ch > 1) s.template load_chunk<TPR, NV, true>(ch - 2, tid, next);
  }
  if (edge_place >= 0) dz[edge_place] = row_round<T>(one(edge));
  G::sync();                                         // the teacher's places are written again, by one thread each
  if (!none) {
#pragma unroll
    for (int e = 0; e < At::EPT; ++e) {
      const int i = tid + e * TPR;
      float sum;
      if (i < a.k && here.place[i] >= 0 && s.has(here.place[i]) && here.sum_at(i, a.k, sum))
        dz[here.place[i]] = row_round<T>(fmaf(-w, sum, one(at.z[e])));
    }
  }
}

// ------------------------------ host side -----------------------------------------------------------------------------
// Where rows are many a warp takes one: no barrier, and a quarter of the work per row that does not depend on its length.
//   700 x 900 fp32 and more rows: 10 alternatives 6.2 us by blocks, 5.6 by warps; 20 000 x 900 93 and 35
//   longer rows need more of them: 600 x 1800 3.0 and 3.4, 1500 x 1800 5.0 and 4.1 (no alternatives)
//   gradients up to 12 KB: 8192 x 2500 fp32 31.9 and 27.9, 20 000 x 4000 100 and 106
//   distillation up to 20 KB: 8192 x 2500 fp32 55 and 40, 20 000 x 5000 191 and 169, 3000 x 10 000 bf16 37 and 30; 32 KB 150 and 159
//   rows that are only read, up to 40 KB: 10 000 x 5000 fp32 40 and 36, 25 600 x 10 000 157 and 152, with 10 alternatives 207 and
//   193; rows of 64 KB 55 and 64
//   with 32 alternatives up to 32 KB: 10 000 x 16 000 bf16 96 and 88, 40 KB 94 and 111
//   with 64 alternatives up to 20 KB: 10 000 x 5000 fp32 84 and 79, 40 KB 108 and 146; with 128 up to 2 KB: 20 000 x 400 293 and 233,
//   20 000 x 900 195 and 402 (a warp's lists run over)
// Other rows go to a block, or to a cluster: slices of at most `most_bytes`, and more of them while the GPU has room for their
// blocks and each thread still has a vector.
struct RowPlan {
  bool warps;
  int shift;                     // 2^shift slices
};
RowPlan row_plan(gram_ctx* ctx, int64_t N, int64_t row_bytes, int64_t most_bytes, int64_t warp_bytes) {
  RowPlan p{row_bytes <= warp_bytes && N >= (row_bytes <= 4096 ? 4 : row_bytes <= 8192 ? 8 : 16) * kNumSMs, 0};
  if (p.warps) return p;
  const int64_t vectors = row_bytes / 16;
  const int most = gram_cluster_blocks(ctx) < MAX_SLICES ? gram_cluster_blocks(ctx) : MAX_SLICES;
  while ((1 << p.shift) < most && (row_bytes >> p.shift) > most_bytes) ++p.shift;
  while ((1 << p.shift) < most && (N << (p.shift + 1)) <= LP_PER_SM * kNumSMs && (vectors >> (p.shift + 1)) >= LP_THREADS) ++p.shift;
  return p;
}
template <typename... P, typename... A>
gram_status launch_rows(gram_ctx* ctx, void (*kern)(P...), const RowPlan& plan, int64_t N, size_t smem, cudaStream_t st, A... args) {
  const int64_t blocks = plan.warps ? ceil_div64(N, LP_WARPS) : N << plan.shift;
  if (blocks > INT32_MAX) return gram_set_error(ctx, "%lld rows of %d slices", (long long)N, 1 << plan.shift), GRAM_ERR_UNSUPPORTED;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3(LP_THREADS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0] = chain_attribute();
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = 1u << plan.shift;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = plan.shift > 0 ? 2 : 1;
  GRAM_CUDA(ctx, cudaLaunchKernelEx(&cfg, kern, static_cast<P>(args)...));
  return GRAM_OK;
}

template <typename T>
gram_status logprobs_typed(gram_ctx* ctx, const T* z, int64_t ld, int64_t N, int32_t V, float scale, const RowAnswers& ask, cudaStream_t st) {
  const RowPlan plan = row_plan(ctx, N, (int64_t)V * sizeof(T), INT64_MAX, ask.k <= 16 ? 40 << 10 : ask.k <= 32 ? 32 << 10 : ask.k <= 64 ? 20 << 10 : 2 << 10);
  ProfScope prof(ctx, GRAM_K_OTHER, (double)N * V * sizeof(T), 1, st, "logprobs");
  int32_t* status = gram_status_word(ctx);
  const size_t smem = plan.shift > 0 ? (sizeof(uint64_t) * ask.k) << plan.shift : 0;
  auto run = [&](auto kern) { return launch_rows(ctx, kern, plan, N, smem, st, z, ld, N, V, scale, plan.shift, ask, status); };
  if (plan.warps) return ask.k ? run(logprobs_kernel<T, 32, true>) : run(logprobs_kernel<T, 32, false>);
  return ask.k ? run(logprobs_kernel<T, LP_THREADS, true>) : run(logprobs_kernel<T, LP_THREADS, false>);
}
template <typename T> gram_status backward_typed(gram_ctx* ctx, const T* z, T* dz, BackwardArgs a, cudaStream_t st) {
  const RowPlan plan = row_plan(ctx, a.N, (int64_t)a.V * sizeof(T), INT64_MAX, 12 << 10);
  ProfScope prof(ctx, GRAM_K_OTHER, 2.0 * a.N * a.V * sizeof(T), 1, st, "logprobs_backward");
  a.shift = plan.shift;
  if (plan.warps) return launch_rows(ctx, logprobs_backward_kernel<T, 32>, plan, a.N, 0, st, z, dz, a);
  return launch_rows(ctx, logprobs_backward_kernel<T, LP_THREADS>, plan, a.N, 0, st, z, dz, a);
}
template <typename T> gram_status distill_typed(gram_ctx* ctx, const T* z, T* dz, DistillArgs a, cudaStream_t st) {
  const RowPlan plan = row_plan(ctx, a.N, (int64_t)a.V * sizeof(T), 64 << 10, 20 << 10);
  ProfScope prof(ctx, GRAM_K_OTHER, (dz ? 2.0 : 1.0) * a.N * a.V * sizeof(T), 1, st, "distill");
  a.shift = plan.shift;
  if (plan.warps) return launch_rows(ctx, distill_kernel<T, 32>, plan, a.N, 0, st, z, dz, a);
  return launch_rows(ctx, distill_kernel<T, LP_THREADS>, plan, a.N, 0, st, z, dz, a);
}

}  // namespace

gram_status logprobs_launch(gram_ctx* ctx, const void* logits, int dtype, int64_t ld, int64_t N, int32_t V, float scale,
                            const RowAnswers& ask, cudaStream_t st) {
  if (N == 0) return GRAM_OK;
  if (dtype == GRAM_F32) return logprobs_typed(ctx, (const float*)logits, ld, N, V, scale, ask, st);
  return logprobs_typed(ctx, (const bf16*)logits, ld, N, V, scale, ask, st);
}

gram_status logprobs_backward_launch(gram_ctx* ctx, const void* logits, int dtype, int64_t ld, int64_t N, int32_t V, float scale,
                                     const int32_t* targets, int32_t C, const float* stats, const float* entropy, const float* dlogp,
                                     const float* dentropy, void* dlogits, int64_t ld_out, cudaStream_t st) {
  if (N == 0) return GRAM_OK;
  const BackwardArgs a{targets, stats, entropy, dlogp, dentropy, ld, ld_out, N, V, C, 0, scale, gram_status_word(ctx)};
  if (dtype == GRAM_F32) return backward_typed(ctx, (const float*)logits, (float*)dlogits, a, st);
  return backward_typed(ctx, (const bf16*)logits, (bf16*)dlogits, a, st);
}

gram_status distill_launch(gram_ctx* ctx, const void* logits, int dtype, int64_t ld, int64_t N, int32_t V, float scale,
                           const int32_t* teacher_ids, const float* teacher_logits, int32_t k, float* loss, const float* weight,
                           void* dlogits, int64_t ld_out, cudaStream_t st) {
  if (N == 0) return GRAM_OK;
  const DistillArgs a{teacher_ids, teacher_logits, loss, weight, ld, ld_out, N, V, k, 0, scale, gram_status_word(ctx)};
  if (dtype == GRAM_F32) return distill_typed(ctx, (const float*)logits, (float*)dlogits, a, st);
  return distill_typed(ctx, (const bf16*)logits, (bf16*)dlogits, a, st);
}
