// The best k places of a row or a slice of one.
//
// Candidates are kept as keys (row_key: larger logit first, then lower place) in shared memory, in no order.  The first
// chunk sets a bar that at least k of its entries reach: in each warp the value that k / warps of its lanes' maxima (two a
// lane) reach, or a little less, and the smallest of the warps'.  An entry below the bar is not among the best k, and once k
// entries have reached it neither is a later one that equals it, since slices are read in ascending order.  So of a chunk
// only a few entries are looked at twice.  Where more than half the list fills, it is cut to its best k, the last of which
// sets the new bar; a chunk that would overflow the list (equal logits, ascending rows) gives its own best k, found by
// bisection over the keys.
#pragma once
#include "row_softmax.cuh"

template <int TPR> struct TopList {
  static constexpr int CAP = TPR == 32 ? 384 : 1024;
  static_assert(CAP >= 3 * GRAM_TOP_MAX, "half a list holds k, and a cut one k more");
  uint64_t keys[CAP];
  int added[3];                  // entries of a chunk; three in turn, so that one is cleared while none looks at it
  int slow;
  int part[Group<TPR>::WARPS];
  uint32_t low[Group<TPR>::WARPS];
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
// `have` keys (k at least) cut to the best k by a warp; returns a bar that only better logits than theirs reach.  The keys are read
// again in each step of the bisection (shared memory, or L1): no array of them lives in registers.
__device__ __forceinline__ float warp_cut(uint64_t* keys, int have, int k) {
  const int lane = threadIdx.x & 31;
  uint32_t low = 0xffffffffu, high = 0u;
  for (int i = lane; i < have; i += 32) {
    const uint32_t o = (uint32_t)(keys[i] >> 32);
    low = min(low, o);
    high = max(high, o);
  }
  low = __reduce_min_sync(0xffffffffu, low);
  high = __reduce_max_sync(0xffffffffu, high);
  const uint64_t kth = kth_key(k, [&](uint64_t t) {
    int c = 0;
#pragma unroll 4
    for (int i = lane; i < have; i += 32) c += keys[i] >= t;
    return (int)__reduce_add_sync(0xffffffffu, c);
  }, (uint64_t)low << 32, (uint64_t)high << 32 | 0xffffffffu);
  int at = 0;
  low = 0xffffffffu;
  for (int i = 0; i < have; i += 32) {                   // what is kept moves down, behind what has been read
    const uint64_t key = i + lane < have ? keys[i + lane] : 0;
    const bool keep = key >= kth;                        // kth > 0
    const uint32_t who = __ballot_sync(0xffffffffu, keep);
    if (keep) {
      keys[at + __popc(who & ((1u << lane) - 1u))] = key;
      low = min(low, (uint32_t)(key >> 32));
    }
    at += __popc(who);
    __syncwarp();
  }
  return row_order_logit(__reduce_min_sync(0xffffffffu, low) + 1u);
}
// the same of a group's list, by its first warp; the list is complete behind a barrier, and so is what this leaves
template <int TPR> __device__ __noinline__ float top_cut(TopList<TPR>& l, int have, int k) {
  using G = Group<TPR>;
  if (G::tid() < 32) {
    const float bar = warp_cut(l.keys, have, k);
    if (G::tid() == 0) l.low[0] = __float_as_uint(bar);
  }
  G::sync();
  const float bar = __uint_as_float(l.low[0]);
  G::sync();
  return bar;
}
// the best k of a chunk's entries of at least `bar` (k at least) behind the list's first `have`
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

// the first chunk's bar, from two of each thread's entries, the largest of either half
template <int TPR> __device__ __forceinline__ float top_first_bar(TopList<TPR>& l, float a, float b, int k) {
  using G = Group<TPR>;
  const int want = (k + G::WARPS - 1) / G::WARPS;        // of each warp's 64
  const uint32_t oa = a > ROW_NEG_INF ? row_order(a) : 0u, ob = b > ROW_NEG_INF ? row_order(b) : 0u;
  uint32_t lo = 0u;
  if (__popc(__ballot_sync(0xffffffffu, oa != 0u)) + __popc(__ballot_sync(0xffffffffu, ob != 0u)) >= want) {
    lo = __reduce_min_sync(0xffffffffu, min(oa ? oa : ~0u, ob ? ob : ~0u));
    uint32_t hi = __reduce_max_sync(0xffffffffu, max(oa, ob));
    for (int step = 0; lo < hi && step < 12; ++step) {
      const uint32_t mid = hi - (hi - lo) / 2;
      const int n = __popc(__ballot_sync(0xffffffffu, oa >= mid)) + __popc(__ballot_sync(0xffffffffu, ob >= mid));
      if (n < want) hi = mid - 1;
      else {
        lo = mid;
        if (n <= want + want / 8) break;
      }
    }
  }
  if constexpr (TPR > 32) {
    if ((threadIdx.x & 31) == 0) l.low[threadIdx.x >> 5] = lo;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < G::WARPS; ++w) lo = min(lo, l.low[w]);
  }
  return lo ? row_order_logit(lo) : -FLT_MAX;
}

struct TopState {
  int have;                      // keys in the list
  float bar;
  bool reached;                  // k entries have reached the bar: later ones must pass it
};
// one chunk's entries into the list; a, b: the largest of either half of the thread's
template <typename T, int TPR, int NV>
__device__ __forceinline__ void top_chunk(TopList<TPR>& l, TopState& st, const TopChunk<T, TPR, NV>& ch, float a, float b, int k, int number, bool last) {
  using G = Group<TPR>;
  constexpr int CAP = TopList<TPR>::CAP;
  if (number == 0) st.bar = top_first_bar(l, a, b, k);
  int* added = &l.added[number % 3];
  if (fmaxf(a, b) >= st.bar)
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
    top_take_best(l, ch, st.have, min(n, k), st.bar);
    st.have += min(n, k);
    if (st.have >= k) {
      st.bar = top_cut(l, st.have, k);
      st.have = k;
      st.reached = true;
    }
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
