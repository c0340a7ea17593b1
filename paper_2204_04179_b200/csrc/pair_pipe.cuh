// What the persistent kernels on pairs of SMs share (the loss over a pool, products in 8 bits): a cluster of two blocks owns tiles of
// 256 x 256, each block stages its 128 rows of either operand by TMA, the leader issues the MMAs of both, and each block's tensor
// memory receives 128 rows of the result, two tiles in turn.  Warp 0 issues copies, warp 1 the MMAs, the others take results.
// All waits are bounded; a role that gives up sets the block's flag and the context's status, and all end.
#pragma once
#include <atomic>

#include "tc_common.cuh"

namespace tc {

constexpr int PAIR_ROWS = 128;                          // rows of a block; a pair has twice as many
constexpr int PAIR_COLS = 256;                          // columns of the widest tile, and of an accumulator
constexpr int PAIR_OPERAND = PAIR_ROWS * 128;           // bytes of 128 rows of 128, the swizzle's width
constexpr int PAIR_BOX = 64 * 128;                      // bytes of a copy's box: 64 rows of 128

// A stage holds `A` operands of the MMA's rows and one of its columns (none of its rows: a single operand, whichever it is).  EXTRA: bytes of the kernel's own, behind the stages.
template <int STAGES_, int EPI_WARPS_, int EXTRA = 0, int A = 1> struct PairPipe {
  static constexpr int STAGES = STAGES_, EPI_WARPS = EPI_WARPS_, THREADS = 64 + 32 * EPI_WARPS_, STAGE = (A + 1) * PAIR_OPERAND;
  static constexpr int SMEM = STAGES * STAGE + EXTRA + 1024 + 256;
  static_assert(SMEM <= 232448 && EXTRA % 16 == 0 && 8 * (2 * STAGES + 4) + 8 <= 256, "shared memory of a block");
  uint32_t tiles, bar0, tmem, rank, lead_bar0;
  uint8_t* extra;
  volatile int* abort_flag;
  int warp, lane;

  __device__ __forceinline__ uint32_t full(int s) const { return bar0 + 8u * s; }                          // used in the leader
  __device__ __forceinline__ uint32_t empty(int s) const { return bar0 + 8u * (STAGES + s); }              // one per block
  __device__ __forceinline__ uint32_t tfull(int b) const { return bar0 + 8u * (2 * STAGES + b); }          // one per block
  __device__ __forceinline__ uint32_t tempty(int b) const { return bar0 + 8u * (2 * STAGES + 2 + b); }     // used in the leader
  // the leader's, as seen from either block
  __device__ __forceinline__ uint32_t lead_full(int s) const { return lead_bar0 + 8u * s; }
  __device__ __forceinline__ uint32_t lead_tempty(int b) const { return lead_bar0 + 8u * (2 * STAGES + 2 + b); }
  __device__ __forceinline__ uint32_t a_of(int s, int i = 0) const { return tiles + s * STAGE + i * PAIR_OPERAND; }
  __device__ __forceinline__ uint32_t b_of(int s) const { return tiles + s * STAGE + A * PAIR_OPERAND; }

  // All threads; memory of the kernels before may be touched after it.  more(): further barriers, initialised by one thread.
  struct NoMore {
    __device__ void operator()() const {}
  };
  template <typename F = NoMore> __device__ __forceinline__ bool open(uint8_t* smem_raw, F more = F()) {
    const uint32_t raw = smem_u32(smem_raw);
    tiles = (raw + 1023u) & ~1023u;                     // the same offset in both blocks of the pair
    extra = smem_raw + (tiles - raw) + STAGES * STAGE;
    bar0 = tiles + STAGES * STAGE + EXTRA;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(extra + EXTRA + 8 * (2 * STAGES + 4));
    abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    warp = threadIdx.x >> 5;
    lane = threadIdx.x & 31;
    rank = cluster_ctarank();
    if (threadIdx.x == 0) {
      for (int s = 0; s < STAGES; ++s) {
        mbar_init(full(s), 2);                          // the two blocks' copies, each with its byte count
        mbar_init(empty(s), 1);
      }
      for (int b = 0; b < 2; ++b) {
        mbar_init(tfull(b), 1);
        mbar_init(tempty(b), 2 * EPI_WARPS);
      }
      more();
      *abort_flag = 0;
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512u) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    gram_cluster_sync();                                // both blocks' barriers exist before anyone signals them
    tc_fence_after();
    tmem = *tmem_slot;
    lead_bar0 = map_to_cta(bar0, 0);
    return chain_begin();
  }
  // All threads, each warp's lanes together.
  __device__ __forceinline__ void close(bool failed, int32_t* status) {
    if (failed && lane == 0) {
      *abort_flag = 1;
      gram_device_fail(status, GRAM_ERR_TIMEOUT);
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (*abort_flag) {
      if (warp == 1 && lane == 0) {                     // let copies and MMAs already issued drain (bounded)
        const uint64_t t0 = clock64();
        while (clock64() - t0 < WAIT_LIMIT_CYCLES / 64) {}
      }
      __syncthreads();
    }
    gram_cluster_sync();                                // the peer no longer reads this block's memory or signals its barriers
    if (warp == 1) {
      tc_fence_after();
      asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
  }
};

// The kernel's shared memory is asked for once on each device (of the first 64; then every time): the call takes as long as a launch.
template <auto KERN> inline cudaError_t allow_smem(int smem) {
  static std::atomic<uint64_t> done{0};
  int device = 0;
  cudaError_t e = cudaGetDevice(&device);
  if (e != cudaSuccess) return e;
  const uint64_t bit = device < 64 ? (uint64_t)1 << device : 0;
  if (bit && (done.load(std::memory_order_relaxed) & bit)) return cudaSuccess;
  e = cudaFuncSetAttribute(KERN, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
  return e;
}
// a launch of `pairs` clusters of two blocks
template <auto KERN, typename... A> inline cudaError_t launch_pairs(int pairs, int threads, int smem, cudaStream_t st, const A&... args) {
  const cudaError_t e = allow_smem<KERN>(smem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(2 * pairs));
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1] = chain_attribute();
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, KERN, args...);
}

}  // namespace tc
