// The best k places of a row or a slice of one.
//
// Candidates are kept as keys (row_key: larger logit first, then lower place) in shared memory, in no order.  The first
// chunk sets a bar: the k-th largest of the threads' maxima, or a little below; k entries at least reach it.  An entry below
// the bar is not among the best k, and once k entries have reached it neither is a later one that equals it, since slices
// are read in ascending order.  So of a chunk only a few entries are looked at twice.  Where more than half the list fills,
// it is cut to its best k, the last of which sets the new bar; a chunk that would overflow the list (equal logits, ascending
// rows) gives its own best k, found by bisection over the keys.
#pragma once
#include "row_softmax.cuh"

template <int TPR> struct TopList {
  static constexpr int CAP = TPR == 32 ? 384 : 1024;
  static_assert(CAP >= 4 * GRAM_TOP_MAX || TPR == 32 && CAP >= 3 * GRAM_TOP_MAX, "a list past its half holds more than k");
  uint64_t keys[CAP];
  int added[3];                  // entries of a chunk; three in turn, so that one is cleared while none looks at it
  int slow;
  int part[LP_WARPS];
  uint32_t lowest[LP_WARPS], highest[LP_WARPS];
};

template <typename T, int TPR, int NV> struct TopChunk {
  const uint4 (&q)[NV];
  int place0;                    // of this thread's first vector
  float edge;                    // this thread's single element, -inf without one
  int edge_place;
  // f(logit, place) of each entry of this thread's part of the chunk
  template <typename F> __device__ __forceinline__ void each(F f) const {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < RowVec<T>::N / 2; ++j) {
        const float2 x = RowVec<T>::pair(q[i], j);
        const int p = place0 + i * (TPR * RowVec<T>::N) + 2 * j;
        f(x.x, p);
        f(x.y, p + 1);
      }
    f(edge, edge_place);
  }
};

// the largest t of [lo, hi] such that at least k keys are >= t; there are k of at least lo, and none above hi; at_least(t) counts them
template <typename F> __device__ __forceinline__ uint64_t kth_key(int k, F at_least, uint64_t lo = 1, uint64_t hi = ~0ull) {
  while (lo < hi) {
    const uint64_t mid = hi - (hi - lo) / 2;
    const int n = at_least(mid);
    if (n == k) return mid;
    if (n > k) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}
// the first `have` keys of the list (k at least) cut to the best k; returns a bar that only better logits than theirs reach
template <int TPR> __device__ __noinline__ float top_cut(TopList<TPR>& l, int have, int k) {
  using G = Group<TPR>;
  constexpr int PER = TopList<TPR>::CAP / TPR;
  const int tid = G::tid();
  uint64_t key[PER], last = ~0ull;
#pragma unroll
  for (int i = 0; i < PER; ++i) key[i] = tid + i * TPR < have ? l.keys[tid + i * TPR] : 0;
  const uint64_t kth = kth_key(k, [&](uint64_t t) {
    int c = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) c += key[i] >= t;
    return G::sum(c, l.part);
  });
  if (tid == 0) l.slow = 0;
  G::sync();
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (key[i] >= kth) {
      l.keys[atomicAdd(&l.slow, 1)] = key[i];
      last = min(last, key[i]);
    }
  uint32_t low = __reduce_min_sync(0xffffffffu, (uint32_t)(last >> 32));
  if constexpr (TPR > 32) {
    if ((threadIdx.x & 31) == 0) l.lowest[threadIdx.x >> 5] = low;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < LP_WARPS; ++w) low = min(low, l.lowest[w]);
  }
  G::sync();
  return row_order_logit(low + 1u);
}
// the best k of a chunk's entries of at least `bar` (more than k) behind the list's first `have`
template <typename T, int TPR, int NV>
__device__ __noinline__ void top_take_best(TopList<TPR>& l, const TopChunk<T, TPR, NV>& ch, int have, int k, float bar) {
  using G = Group<TPR>;
  const uint64_t kth = kth_key(k, [&](uint64_t t) {
    int c = 0;
    ch.each([&](float x, int p) { c += x >= bar && row_key(x, p) >= t; });
    return G::sum(c, l.part);
  });
  if (G::tid() == 0) l.slow = have;
  G::sync();
  ch.each([&](float x, int p) {
    if (x >= bar && row_key(x, p) >= kth) l.keys[atomicAdd(&l.slow, 1)] = row_key(x, p);
  });
  G::sync();
}

// the first chunk's bar, from the threads' largest entries
template <int TPR> __device__ __forceinline__ float top_first_bar(TopList<TPR>& l, float top, int k) {
  using G = Group<TPR>;
  const bool some = top > ROW_NEG_INF;
  const uint32_t o = row_order(top);
  uint32_t lo = __reduce_min_sync(0xffffffffu, some ? o : 0xffffffffu), hi = __reduce_max_sync(0xffffffffu, some ? o : 0u);
  if constexpr (TPR > 32) {
    if ((threadIdx.x & 31) == 0) { l.lowest[threadIdx.x >> 5] = lo; l.highest[threadIdx.x >> 5] = hi; }
  }
  if (G::count(some) < k) return -FLT_MAX;              // a barrier, for the two arrays too
  if constexpr (TPR > 32) {
#pragma unroll
    for (int w = 0; w < LP_WARPS; ++w) { lo = min(lo, l.lowest[w]); hi = max(hi, l.highest[w]); }
  }
  for (int step = 0; lo < hi && step < 12; ++step) {
    const uint32_t mid = hi - (hi - lo) / 2;
    const int n = G::count(some && o >= mid);
    if (n < k) hi = mid - 1;
    else {
      lo = mid;
      if (n <= k + k / 8) break;
    }
  }
  return row_order_logit(lo);
}

struct TopState {
  int have;                      // keys in the list
  float bar;
  bool reached;                  // k entries have reached the bar: later ones must pass it
};
// one chunk's entries into the list; top: the thread's largest
template <typename T, int TPR, int NV>
__device__ __forceinline__ void top_chunk(TopList<TPR>& l, TopState& st, const TopChunk<T, TPR, NV>& ch, float top, int k, int number, bool last) {
  using G = Group<TPR>;
  constexpr int CAP = TopList<TPR>::CAP;
  if (number == 0) st.bar = top_first_bar(l, top, k);
  int* added = &l.added[number % 3];
  if (top >= st.bar)
    ch.each([&](float x, int p) {
      if (x >= st.bar) {
        const int at = st.have + atomicAdd(added, 1);
        if (at < CAP) l.keys[at] = row_key(x, p);
      }
    });
  if (G::tid() == 0) l.added[(number + 1) % 3] = 0;
  G::sync();
  const int n = *added;
  if (st.have + n > CAP) {
    if (st.have > k) (void)top_cut(l, st.have, k);
    st.have = min(st.have, k);
    if (n > k) top_take_best(l, ch, st.have, k, st.bar);
    else top_take_best(l, ch, st.have, n, st.bar);
    st.have += min(n, k);
    if (st.have >= k) { st.bar = top_cut(l, st.have, k); st.have = k; st.reached = true; }
    return;
  }
  st.have += n;
  if (st.have >= k && !st.reached) {
    st.bar = row_order_logit(row_order(st.bar) + 1u);
    st.reached = true;
  }
  if (st.have > CAP / 2 && !last) {
    st.bar = top_cut(l, st.have, k);
    st.have = k;
    st.reached = true;
  }
}
