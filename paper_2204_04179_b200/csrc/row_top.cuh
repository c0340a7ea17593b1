// The best k places of a row or a slice of one.
//
// Candidates have keys (row_key: larger logit first, then lower place).  The first chunk sets a bar that at least k of the
// group's entries reach: the value that k of its threads' maxima reach, or a little less.  An entry below the bar is not among
// the best k, and behind the first chunk neither is one that equals it, since a thread reads in ascending order.  Of a chunk, a
// thread makes a bit mask of the entries that reach the bar, and the few places go to a list of its warp in shared memory;
// their logits are read again at the end, all at once.  No barrier is needed until the lists are brought together.  A list
// that would overflow (equal logits, ascending rows, large k) is cut to its best k, the last of which sets the warp's new bar.
#pragma once
#include "row_softmax.cuh"

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

constexpr int TOP_CAP = 3 * GRAM_TOP_MAX;              // entries of a warp's list: places while a row is read, keys then

// the first chunk's bar, from two of each thread's entries, the largest of either half; part: a word for each warp and bound
template <int TPR> __device__ __forceinline__ float top_first_bar(float a, float b, int k, uint32_t (*part)[2]) {
  using G = Group<TPR>;
  const bool two = k > TPR / 4;                          // 128 maxima are few for a larger k
  if (!two) a = fmaxf(a, b);
  const uint32_t oa = a > ROW_NEG_INF ? row_order(a) : 0u, ob = two && b > ROW_NEG_INF ? row_order(b) : 0u;
  uint32_t lo = __reduce_min_sync(0xffffffffu, min(oa ? oa : ~0u, ob ? ob : ~0u)), hi = __reduce_max_sync(0xffffffffu, max(oa, ob));
  if constexpr (TPR > 32) {
    if ((threadIdx.x & 31) == 0) { part[threadIdx.x >> 5][0] = lo; part[threadIdx.x >> 5][1] = hi; }
  }
  auto reach = [&](uint32_t o) {
    int n = G::count(oa >= o);
    if (two) n += G::count(ob >= o);
    return n;
  };
  if (reach(1u) < k) return -FLT_MAX;                    // a barrier, for `part` too
  if constexpr (TPR > 32) {
#pragma unroll
    for (int w = 0; w < G::WARPS; ++w) { lo = min(lo, part[w][0]); hi = max(hi, part[w][1]); }
  }
  for (int step = 0; lo < hi && step < 12; ++step) {
    const uint32_t mid = hi - (hi - lo) / 2;
    const int n = reach(mid);
    if (n < k) hi = mid - 1;
    else {
      lo = mid;
      if (n <= k + k / 8) break;
    }
  }
  return row_order_logit(lo);
}

struct TopState {
  int have;                      // places on the warp's list
  float bar;                     // entries must reach it
};
// What the overflow needs to read a thread's part of a chunk again: `count` vectors, `stride` apart, and its single element.
template <typename T> struct TopChunk {
  const T* z;                    // the row
  const uint4* from;             // the first vector, the place of its first element, vectors of the slice from it on
  int place0, left, stride, count;
  int edge;                      // place of the single element, -1: none
  template <typename F> __device__ __forceinline__ void each(F f) const {
    for (int i = 0; i < count; ++i) {
      constexpr uint32_t none = RowVec<T>::NONE;
      const uint4 q = i * stride < left ? from[i * stride] : make_uint4(none, none, none, none);
#pragma unroll
      for (int j = 0; j < RowVec<T>::N / 2; ++j) {
        const float2 x = RowVec<T>::pair(q, j);
        f(x.x, place0 + i * stride * RowVec<T>::N + 2 * j);
        f(x.y, place0 + i * stride * RowVec<T>::N + 2 * j + 1);
      }
    }
    f(edge >= 0 ? row_load(z + edge) : ROW_NEG_INF, edge);
  }
};
// A chunk whose entries overflow the list: the list and then the chunk's own best k, found by bisection, cut to the best k.
template <typename T> __device__ __noinline__ TopState top_overflow(uint64_t* list, TopState st, TopChunk<T> ch, int k) {
  const int lane = threadIdx.x & 31;
  constexpr int PER = TOP_CAP / 32;
  uint32_t* places = reinterpret_cast<uint32_t*>(list);
  {
    uint32_t p[PER];
    for (int i = 0; i < PER; ++i) p[i] = i * 32 + lane < st.have ? places[i * 32 + lane] : 0;
    __syncwarp();
    for (int i = 0; i < PER; ++i)
      if (i * 32 + lane < st.have) list[i * 32 + lane] = row_key(row_load(ch.z + p[i]), p[i]);
    __syncwarp();
  }
  auto cut = [&]() {
    st.bar = fmaxf(st.bar, warp_cut(list, st.have, k));
    st.have = k;
  };
  if (st.have > k) cut();
  auto at_least = [&](uint64_t t) {
    int c = 0;
    ch.each([&](float x, int p) { c += x >= st.bar && row_key(x, p) >= t; });
    return (int)__reduce_add_sync(0xffffffffu, c);
  };
  const int n = min(at_least(1), k);
  if (n > 0) {
    const uint64_t kth = kth_key(n, at_least);
    ch.each([&](float x, int p) {
      const bool keep = x >= st.bar && row_key(x, p) >= kth;
      const uint32_t who = __ballot_sync(0xffffffffu, keep);
      if (keep) list[st.have + __popc(who & ((1u << lane) - 1u))] = row_key(x, p);
      st.have += __popc(who);
    });
    __syncwarp();
    if (st.have >= k) cut();
  }
  {
    uint64_t key[PER];
    for (int i = 0; i < PER; ++i) key[i] = i * 32 + lane < st.have ? list[i * 32 + lane] : 0;
    __syncwarp();
    for (int i = 0; i < PER; ++i)
      if (i * 32 + lane < st.have) places[i * 32 + lane] = (uint32_t)row_key_place(key[i]);
    __syncwarp();
  }
  return st;
}
// A chunk's entries to the warp's list; top: the thread's largest; on_edge: its single element counts to this chunk.
template <typename T, int NV>
__device__ __forceinline__ void top_chunk(uint64_t* list, TopState& st, const TopChunk<T>& ch, const uint4 (&q)[NV], float top, bool on_edge, int k) {
  if (!__any_sync(0xffffffffu, top >= st.bar)) return;
  constexpr int N = RowVec<T>::N;
  static_assert(N * NV <= 32, "a bit for each entry");
  const uint32_t below = (1u << (threadIdx.x & 31)) - 1u;
  uint32_t* places = reinterpret_cast<uint32_t*>(list);
  uint32_t bits = 0u;
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < N / 2; ++j) {
      const float2 x = RowVec<T>::pair(q[i], j);
      if (x.x >= st.bar) bits |= 1u << (i * N + 2 * j);
      if (x.y >= st.bar) bits |= 1u << (i * N + 2 * j + 1);
    }
  bool edge = on_edge && row_load(ch.z + ch.edge) >= st.bar;
  int at = st.have;
  for (;;) {
    const bool in = bits != 0u || edge;
    const uint32_t who = __ballot_sync(0xffffffffu, in);
    if (!who) break;
    if (in) {
      const int j = __ffs(bits) - 1, slot = at + __popc(who & below);
      if (slot < TOP_CAP) places[slot] = bits ? (uint32_t)(ch.place0 + (j / N) * ch.stride * N + j % N) : (uint32_t)ch.edge;
      if (bits) bits &= bits - 1u;
      else edge = false;
    }
    at += __popc(who);
  }
  if (at <= TOP_CAP) {
    st.have = at;
  } else {
    __syncwarp();
    TopChunk<T> again = ch;
    if (!on_edge) again.edge = -1;
    st = top_overflow<T>(list, st, again, k);
  }
}

// The warps' lists (TOP_CAP entries apart) brought together as keys at the front of the first, and cut if they are long.  Returns
// the keys left, k or a few more, or all there are.  Called by the whole group, with a barrier behind it.
template <typename T, int TPR> __device__ __forceinline__ int top_gather(const T* z, uint64_t* list, int* count, int mine, int k) {
  using G = Group<TPR>;
  constexpr int PER = TOP_CAP / 32;
  const int lane = threadIdx.x & 31, warp = TPR == 32 ? 0 : threadIdx.x >> 5;
  const uint32_t* places = reinterpret_cast<const uint32_t*>(list + warp * TOP_CAP);
  uint64_t key[PER];
  __syncwarp();
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (i * 32 < mine) {
      const uint32_t p = i * 32 + lane < mine ? places[i * 32 + lane] : 0;
      key[i] = row_key(row_load(z + p), p);
    }
  int at = 0, all = mine;
  if constexpr (TPR > 32) {
    if (lane == 0) count[warp] = mine;
    __syncthreads();
    all = 0;
#pragma unroll
    for (int w = 0; w < G::WARPS; ++w) {
      if (w < warp) at += count[w];
      all += count[w];
    }
  } else {
    __syncwarp();
  }
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (i * 32 + lane < mine) list[at + i * 32 + lane] = key[i];
  G::sync();
  if (all > 128 && all > k + k / 4) {
    if (G::tid() < 32) (void)warp_cut(list, all, k);
    all = k;
    G::sync();
  }
  return all;
}
