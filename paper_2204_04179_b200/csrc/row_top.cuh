// The best k places of a row or a slice of one.
//
// While a row is read each thread only notes the largest entry of every group of chunks (one to a few).  At the end, a bar is
// set that at least k entries reach: the value that k of the threads' maxima reach, or a little less.  The best k lie in the
// groups whose maximum reaches the bar, hardly more than k of all threads' groups; these few are read again, and the entries
// that reach the bar become keys (row_key: larger logit first, then lower place), whose order is found by counting (top_sort).  Where
// more groups or entries reach the bar than the lists hold (equal logits), the k-th key is found by bisection over the row, which reads
// it up to 64 times: of rows whose logits are all equal 64 x 100 000 fp32 with 10 alternatives take 600 us (13 where they differ),
// 4096 x 30 522 bf16 with 64 5.2 ms (0.07).
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
// `have` keys (k at least) cut to the best k by a warp; returns a bar that all later entries reach which could still be among the
// best, given that these have places of `from` on: the least of the logits kept where such an entry may have the lower place of two
// equal ones, else the next value above it.  The keys are read again in each step of the bisection (shared memory, or L1): no array
// of them lives in registers.
__device__ __forceinline__ float warp_cut(uint64_t* keys, int have, int k, uint32_t from) {
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
  uint64_t least = ~0ull;                                // of a lane's keys that are kept: of equal logits the one with the highest place
  for (int i = 0; i < have; i += 32) {                   // what is kept moves down, behind what has been read
    const uint64_t key = i + lane < have ? keys[i + lane] : 0;
    const bool keep = key >= kth;                        // kth > 0
    const uint32_t who = __ballot_sync(0xffffffffu, keep);
    if (keep) {
      keys[at + __popc(who & ((1u << lane) - 1u))] = key;
      least = key < least ? key : least;
    }
    at += __popc(who);
    __syncwarp();
  }
  low = __reduce_min_sync(0xffffffffu, (uint32_t)(least >> 32));
  const uint32_t last = __reduce_max_sync(0xffffffffu, (uint32_t)(least >> 32) == low ? ~(uint32_t)least : 0u);
  return row_order_logit(last >= from ? low : low + 1u);
}

// of up to 512 keys (k at least) a warp keeps the best k or a few more, in no order; returns how many
__device__ __forceinline__ int warp_keep(uint64_t* keys, int have, int k) {
  const int lane = threadIdx.x & 31;
  uint64_t key[16];
  uint32_t lo = ~0u, hi = 0u;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    key[i] = 0;
    if (i * 32 < have && i * 32 + lane < have) {
      key[i] = keys[i * 32 + lane];
      lo = min(lo, (uint32_t)(key[i] >> 32));
      hi = max(hi, (uint32_t)(key[i] >> 32));
    }
  }
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_max_sync(0xffffffffu, hi);
  uint64_t a = (uint64_t)lo << 32, b = (uint64_t)hi << 32 | 0xffffffffu;
  int left = have;
  while (a < b && left > k + 16) {
    const uint64_t mid = b - (b - a) / 2;
    int n = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (i * 32 < have) n += key[i] >= mid;
    n = __reduce_add_sync(0xffffffffu, n);
    if (n < k) b = mid - 1;
    else {
      a = mid;
      left = n;
    }
  }
  int at = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (i * 32 < have) {
      const bool keep = key[i] >= a && key[i] != 0;
      const uint32_t who = __ballot_sync(0xffffffffu, keep);
      if (keep) keys[at + __popc(who & ((1u << lane) - 1u))] = key[i];
      at += __popc(who);
    }
  __syncwarp();
  return at;
}

// (20 KB a block: what eight of them leave of an SM's memory is L1, where loads in flight have their place.  With 26 KB rows of
// 100 000 fp32 were read at 5100 GB/s instead of 6200; with half the groups, whose entries are then twice as long, 64 alternatives
// of 2368 such rows take 189 us instead of 174.)
template <int TPR> struct alignas(16) TopScratch {
  static constexpr int GROUPS = TPR == 32 ? 16 : 32;    // of a thread
  static constexpr int KEYS = 384, ENTRIES = TPR == 32 ? 128 : 256;
  static_assert(KEYS >= GRAM_TOP_MAX, "an exact list fits");
  uint64_t keys[KEYS];
  float group[GROUPS * TPR];
  uint16_t entry[ENTRIES];       // groups whose maximum reaches the bar: group * TPR + thread
  int entries, found;
  int part[Group<TPR>::WARPS];
  int count[2][Group<TPR>::WARPS];
  uint32_t bound[Group<TPR>::WARPS][2];
};

// a bar, from the largest entry of each thread's i-th vectors (top[i])
template <int TPR> __device__ __forceinline__ float top_bar(const float (&top)[4], int k, TopScratch<TPR>& sc) {
  using G = Group<TPR>;
  // k of 2 k or more values: four a thread where k is large, else fewer, since each costs a count (in a block a barrier) a step
  const int values = TPR == 32 ? 4 : k > TPR / 2 ? 4 : k > TPR / 4 ? 2 : 1;
  uint32_t o[4], lo = ~0u, hi = 0u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float x = values == 4 ? top[i] : i == 0 ? (values == 2 ? fmaxf(top[0], top[1]) : fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])))
                                                  : i == 1 && values == 2 ? fmaxf(top[2], top[3]) : ROW_NEG_INF;
    o[i] = x > ROW_NEG_INF ? row_order(x) : 0u;
    lo = min(lo, o[i] ? o[i] : ~0u);
    hi = max(hi, o[i]);
  }
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_max_sync(0xffffffffu, hi);
  if constexpr (TPR > 32) {
    if ((threadIdx.x & 31) == 0) { sc.bound[threadIdx.x >> 5][0] = lo; sc.bound[threadIdx.x >> 5][1] = hi; }
  }
  auto reach = [&](uint32_t b) {
    int n = G::count(o[0] >= b);
    if (values > 1) n += G::count(o[1] >= b);
    if (values > 2) n += G::count(o[2] >= b) + G::count(o[3] >= b);
    return n;
  };
  if (reach(1u) < k) return -FLT_MAX;                    // a barrier, for the bounds too
  if constexpr (TPR > 32) {
#pragma unroll
    for (int w = 0; w < G::WARPS; ++w) { lo = min(lo, sc.bound[w][0]); hi = max(hi, sc.bound[w][1]); }
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

// f(logit, place) of each entry of a vector at `place`
template <typename T, typename F> __device__ __forceinline__ void each_of(const uint4& q, int place, F f) {
#pragma unroll
  for (int j = 0; j < RowVec<T>::N / 2; ++j) {
    const float2 x = RowVec<T>::pair(q, j);
    f(x.x, place + 2 * j);
    f(x.y, place + 2 * j + 1);
  }
}
// What is read again: vectors [v0, v1) from `from` on, the first at place `place0`, and this thread's single element (-1: none).
struct TopSource {
  const uint4* from;
  int place0, v0, v1;
  float edge;
  int edge_place;
};
// the best k of all entries by bisection; returns how many there are
template <typename T, int TPR> __device__ __noinline__ int top_exact(TopScratch<TPR>& sc, TopSource src, int k) {
  using G = Group<TPR>;
  const int tid = G::tid();
  auto each = [&](auto f) {
    for (int v = src.v0 + tid; v < src.v1; v += TPR) each_of<T>(src.from[v], src.place0 + v * RowVec<T>::N, f);
    if (src.edge_place >= 0) f(src.edge, src.edge_place);
  };
  auto at_least = [&](uint64_t t) {
    int c = 0;
    each([&](float x, int p) { c += x > ROW_NEG_INF && row_key(x, p) >= t; });
    return G::sum(c, sc.part);
  };
  const int n = min(at_least(1), k);
  if (n == 0) return 0;
  const uint64_t kth = kth_key(n, at_least);
  G::sync();
  if (tid == 0) sc.found = 0;
  G::sync();
  each([&](float x, int p) {
    if (x > ROW_NEG_INF && row_key(x, p) >= kth) sc.keys[atomicAdd(&sc.found, 1)] = row_key(x, p);
  });
  G::sync();
  return n;
}
// of many keys a group keeps the best k or a few more; returns how many, with a barrier behind it
template <int TPR> __device__ __noinline__ int top_keep(TopScratch<TPR>& sc, int have, int k) {
  using G = Group<TPR>;
  if constexpr (TPR == 32) return warp_keep(sc.keys, have, k);
  constexpr int PER = TopScratch<TPR>::KEYS / TPR;
  const int tid = G::tid(), lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint64_t key[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) key[i] = i * TPR + tid < have ? sc.keys[i * TPR + tid] : 0;
  int turn = 0;
  auto at_least = [&](uint64_t t) {                      // one barrier: the counts of two calls lie apart
    int c = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (i * TPR < have) c += key[i] >= t;
    c = __reduce_add_sync(0xffffffffu, c);
    if (lane == 0) sc.count[turn][warp] = c;
    __syncthreads();
    int n = 0;
#pragma unroll
    for (int w = 0; w < G::WARPS; ++w) n += sc.count[turn][w];
    turn ^= 1;
    return n;
  };
  uint64_t lo = 1, hi = ~0ull;
  int left = have;
  while (lo < hi && left > k + 16) {
    const uint64_t mid = hi - (hi - lo) / 2;
    const int n = at_least(mid);
    if (n < k) hi = mid - 1;
    else {
      lo = mid;
      left = n;
    }
  }
  left = at_least(lo);
  int at = 0;
#pragma unroll
  for (int w = 0; w < G::WARPS; ++w) at += w < warp ? sc.count[turn ^ 1][w] : 0;
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (i * TPR < have) {
      const bool in = key[i] >= lo;
      const uint32_t who = __ballot_sync(0xffffffffu, in);
      if (in) sc.keys[at + __popc(who & ((1u << lane) - 1u))] = key[i];
      at += __popc(who);
    }
  __syncthreads();
  return left;
}
// The candidates of a row or slice, as keys in sc.keys: at least its best k, or all there are.
// Group g holds the thread's vectors of chunks [g << shift, (g + 1) << shift), NV a chunk, TPR apart.  sc.entries and sc.found
// are 0 before, behind a barrier; a barrier is behind what this leaves.
template <typename T, int TPR, int NV>
__device__ __forceinline__ int top_collect(TopScratch<TPR>& sc, const TopSource& src, int groups, int shift, float bar, int k) {
  using G = Group<TPR>;
  using Sc = TopScratch<TPR>;
  const int tid = G::tid(), lane = threadIdx.x & 31;
  for (int g = 0; g < groups; ++g) {
    const bool in = sc.group[g * TPR + tid] >= bar;
    const uint32_t who = __ballot_sync(0xffffffffu, in);
    if (who) {
      int at = 0;
      if (lane == 0) at = atomicAdd(&sc.entries, __popc(who));
      at = __shfl_sync(0xffffffffu, at, 0) + __popc(who & ((1u << lane) - 1u));
      if (in && at < Sc::ENTRIES) sc.entry[at] = (uint16_t)(g * TPR + tid);
    }
  }
  auto put = [&](float x, int p) {
    if (x >= bar) {
      const int at = atomicAdd(&sc.found, 1);
      if (at < Sc::KEYS) sc.keys[at] = row_key(x, p);
    }
  };
  if (src.edge_place >= 0) put(src.edge, src.edge_place);
  G::sync();
  const int entries = sc.entries;
  if (entries <= Sc::ENTRIES) {
    static_assert(NV == 4, "the vectors of a group are a power of two");
    const int per = 2 + shift;                           // 2^per of them
    constexpr int NL = TPR == 32 ? 2 : NV;               // vectors of a thread on their way before the first is looked at
    for (int i0 = tid; i0 < entries << per; i0 += NL * TPR) {
      uint4 q[NL];
      int v[NL];
#pragma unroll
      for (int l = 0; l < NL; ++l) {
        const int i = i0 + l * TPR;
        constexpr uint32_t none = RowVec<T>::NONE;
        q[l] = make_uint4(none, none, none, none);
        v[l] = src.v1;
        if (i < entries << per) {
          const int e = sc.entry[i >> per];
          v[l] = src.v0 + (((e / TPR) << per) + (i & ((1 << per) - 1))) * TPR + e % TPR;
        }
        if (v[l] < src.v1) q[l] = src.from[v[l]];
      }
#pragma unroll
      for (int l = 0; l < NL; ++l) {
        if (l > 0 && i0 - tid + l * TPR >= entries << per) break;
        uint32_t in = 0;                                 // its entries that reach the bar (-FLT_MAX at least)
        int bit = 0;
        each_of<T>(q[l], 0, [&](float x, int) { in |= (x >= bar ? 1u : 0u) << bit++; });
        if (!in) continue;
        int at = atomicAdd(&sc.found, __popc(in));
        const T* z = reinterpret_cast<const T*>(src.from + v[l]);
        for (; in; in &= in - 1, ++at) {
          const int j = __ffs(in) - 1;
          if (at < Sc::KEYS) sc.keys[at] = row_key(row_load(z + j), src.place0 + v[l] * RowVec<T>::N + j);
        }
      }
    }
  }
  G::sync();
  int have = sc.found;
  if (entries > Sc::ENTRIES || have > Sc::KEYS) have = top_exact<T, TPR>(sc, src, k);
  else if (have > 2 * k + 96) have = top_keep<TPR>(sc, have, k);     // counting takes have^2 comparisons
  return have;
}
// The order of keys by counting, of few against all others.  A block's longer lists are sorted in segments of 32 first, a warp
// each; a key's place is then its own in its segment plus those of the other segments' above it, found by bisection: 128
// alternatives of 25 600 rows of 10 000 fp32 take 330 us so, 371 by counting alone.  A warp's lists are short (10 alternatives of
// those rows 193 us by counting, 200 with the choice).  The keys' array holds a whole number of segments; barriers are ahead of
// top_sort and behind it.
constexpr int TOP_COUNTED = 64;
template <int TPR> __device__ __forceinline__ void top_sort(uint64_t* keys, int have) {
  const int lane = threadIdx.x & 31;
  if (TPR == 32 || have <= TOP_COUNTED) {
    if (!(have & 1)) return;
    if (Group<TPR>::tid() == 0) keys[have] = 0;          // they are read in pairs
  } else {
    for (int base = Group<TPR>::tid() - lane; base < have; base += TPR) {
      const uint64_t key = base + lane < have ? keys[base + lane] : 0;
      if (!key) keys[base + lane] = 0;
      __syncwarp();
      int above = 0;
#pragma unroll 4
      for (int j = 0; j < 32; j += 2) {
        const ulonglong2 v = *reinterpret_cast<const ulonglong2*>(keys + base + j);
        above += (v.x > key) + (v.y > key);
      }
      __syncwarp();
      if (key) keys[base + above] = key;
    }
  }
  Group<TPR>::sync();
}
// how many keys are above the i-th
template <int TPR> __device__ __forceinline__ int top_above(const uint64_t* keys, int have, int i) {
  const uint64_t key = keys[i];
  if (TPR == 32 || have <= TOP_COUNTED) {
    int above = 0;
#pragma unroll 4
    for (int j = 0; j < have; j += 2) {
      const ulonglong2 v = *reinterpret_cast<const ulonglong2*>(keys + j);
      above += (v.x > key) + (v.y > key);
    }
    return above;
  }
  int above = i & 31;
  for (int base = 0; base < have; base += 32) {
    if (base == (i & ~31)) continue;
    int lo = 0;
#pragma unroll
    for (int step = 16; step > 0; step >>= 1)
      if (keys[base + lo + step - 1] > key) lo += step;
    above += lo + (keys[base + lo] > key);
  }
  return above;
}
