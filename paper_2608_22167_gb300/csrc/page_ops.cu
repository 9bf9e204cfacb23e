// Shared pages of a paged cache: forking rows, releasing pages, copying whole
// pages, and moving the accepted path of a token tree to the front
// (mcpu_fork_block_tables, mcpu_shrink_block_tables, mcpu_copy_pages,
// mcpu_compact_kv). Integer bookkeeping and bit copies; every result is the
// same on every run: pages return to the stack in ascending order and are
// popped in the order of the forks, whatever order the blocks ran in.
//
// Every kernel is launched programmatically: its blocks may be placed while the
// grid before it still runs, and wait for that grid's end before they read or
// write anything (begin()), by ordinary loads: the non-coherent ones are for
// what stays constant as long as the kernel is there. These calls are short and come in rows, so the
// launches would otherwise be a good part of their time (384 forks released,
// made again and copied in 24 pools: 50 -> 41 us).
#include "tree_round.cuh"

namespace mcpu {

namespace {

constexpr int kForkThreads = 128, kForkEarly = 4;
constexpr int kReleaseThreads = 128, kReleasePer = 4, kReleaseSpan = kReleaseThreads * kReleasePer;
constexpr int kCollectThreads = 1024, kCollectPer = 4;
constexpr int kCopyThreads = 256;
constexpr int kCompactThreads = 256, kCompactMoves = 128, kCompactPools = 4, kCompactBatch = 8;

__device__ __forceinline__ void begin() {
  grid_dep_launch();
  grid_dep_wait();
}

template <typename... KArgs, typename... Args>
cudaError_t launch(void (*kernel)(KArgs...), dim3 grid, int threads, cudaStream_t stream, const Args&... args) {
  LaunchCfg lc(grid, dim3(threads), 0, stream, true);
  return cudaLaunchKernelEx(&lc.cfg, kernel, args...);
}

// Last block to arrive at `ticket` (of n): everything the other blocks did
// before is visible to it. Call with the whole block.
__device__ __forceinline__ bool last_block(int32_t* ticket, int n) {
  __shared__ int s_last;
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) s_last = atomicAdd(ticket, 1) == n - 1;
  __syncthreads();
  if (s_last) __threadfence();
  return s_last != 0;
}

// A fork whose rows and length are valid; *len its source's length.
__device__ __forceinline__ bool fork_valid(const PageParams& p, int f, int* len) {
  const int src = p.src_rows[f], dst = p.dst_rows[f];
  if (src < 0 || src >= p.num_seqs || dst < 0 || dst >= p.num_seqs || src == dst) return false;
  *len = __ldcg(p.seq_lens + src);
  return *len >= 0 && *len <= p.max_pages * kPage;
}

// One block per fork: latency bound (384 forks 9 us). The rank of a fork among those with a partial last page
// (counted over the forks before it) says which page of the stack it takes;
// the last block to finish lowers free_count.
__global__ void __launch_bounds__(kForkThreads) fork_kernel(const PageParams p) {
  begin();
  const int f = blockIdx.x;
  __shared__ int s_page, s_rank;
  if (threadIdx.x == 0) s_rank = 0;
  int S = 0;
  const bool ok = fork_valid(p, f, &S);
  const bool partial = ok && S % kPage != 0;
  const int avail = min(max(__ldcg(p.free_count), 0), p.num_pages);
  // the first entries of the source's table, and of the row's own, are on their way while the rank is counted
  int early[kForkEarly];
  bool held = false;  // the row holds a page, which is about to be lost
#pragma unroll
  for (int i = 0; i < kForkEarly; ++i) {
    const int j = threadIdx.x + i * kForkThreads;
    early[i] = ok && j < S / kPage ? p.block_table[(size_t)p.src_rows[f] * p.max_pages + j] : -1;
    held |= ok && j < p.max_pages && p.block_table[(size_t)p.dst_rows[f] * p.max_pages + j] >= 0;
  }
  int before = 0;
  if (partial) {
#pragma unroll 4
    for (int e = threadIdx.x; e < f; e += kForkThreads) {
      int len = 0;
      if (fork_valid(p, e, &len) && len % kPage != 0) ++before;
    }
  }
  __syncthreads();
  before = __reduce_add_sync(0xffffffffu, before);
  if (threadIdx.x % 32 == 0 && before > 0) atomicAdd(&s_rank, before);
  __syncthreads();
  const int rank = s_rank;
  if (ok) {
    const int src = p.src_rows[f], dst = p.dst_rows[f];
    const int full = S / kPage;
    const int32_t* from = p.block_table + (size_t)src * p.max_pages;
    int32_t* to = p.block_table + (size_t)dst * p.max_pages;
    if (threadIdx.x == 0) {
      int page = -1, tail = -1;
      if (partial) {
        if (rank < avail) {
          atomicAdd(p.scratch + kScratchForkPages, 1);
          page = p.free_pages[avail - 1 - rank];
          tail = from[full];
          if (page < 0 || page >= p.num_pages) page = -1;
          if (tail < 0 || tail >= p.num_pages || page < 0) {
            atomicOr(p.status, kStatusBadPage);
            tail = -1;
          }
        } else {
          atomicOr(p.status, kStatusPoolExhausted);
        }
      }
      p.copy_src[f] = tail;
      p.copy_dst[f] = tail < 0 ? -1 : page;
      p.seq_lens[dst] = S;
      s_page = page;
    }
    __syncthreads();
    for (int j = threadIdx.x, i = 0; j < p.max_pages; j += kForkThreads, ++i) {
      int e = -1;
      if (j < full) {
        e = i == 0 ? early[0] : i == 1 ? early[1] : i == 2 ? early[2] : i == 3 ? early[3] : from[j];
        if (e >= p.num_pages) {
          atomicOr(p.status, kStatusBadPage);
          e = -1;
        }
        if (e >= 0) atomicAdd(p.refs + e, 1);
      } else if (j == full) {
        e = s_page;
      }
      if (i >= kForkEarly) held |= to[j] >= 0;
      to[j] = e;
    }
    if (held) atomicOr(p.status, kStatusBadPage);
  } else if (threadIdx.x == 0) {
    atomicOr(p.status, kStatusBadLengths);
    p.copy_src[f] = p.copy_dst[f] = -1;
  }
  if (last_block(p.scratch + kScratchForkTicket, gridDim.x) && threadIdx.x == 0) {
    const int taken = __ldcg(p.scratch + kScratchForkPages);
    if (taken > 0) *p.free_count = avail - taken;
    p.scratch[kScratchForkPages] = 0;
    p.scratch[kScratchForkTicket] = 0;
  }
}

__host__ __device__ inline int segment_pages(int num_pages) {
  const int per = (num_pages + kPageSegments - 1) / kPageSegments;
  return per > 0 ? per : 1;
}

// Blocks (row, y): releases the entries y * kReleaseSpan .. of the row that lie
// outside its kept pages, kReleasePer a thread with their loads and counts in
// flight together. The holder that takes a page's count below zero is its
// last one: the page keeps the count -1 as its mark until collect_kernel has
// pushed it.
__global__ void __launch_bounds__(kReleaseThreads) release_kernel(const PageParams p) {
  begin();
  const int r = blockIdx.x;
  int32_t* row = p.block_table + (size_t)r * p.max_pages;
  for (int j0 = blockIdx.y * kReleaseSpan + threadIdx.x; j0 < p.max_pages; j0 += gridDim.y * kReleaseSpan) {
    int e[kReleasePer], old[kReleasePer];
#pragma unroll
    for (int i = 0; i < kReleasePer; ++i) {
      const int j = j0 + i * kReleaseThreads;
      e[i] = j < p.max_pages ? row[j] : -1;
    }
    const int S = p.seq_lens[r];
    if (S < 0 || S > p.max_pages * kPage) {
      if (j0 == 0) atomicOr(p.status, kStatusBadLengths);
      return;
    }
    const int end = (S + kPage - 1) / kPage;
    const int begin = p.window > 0 && S >= p.window ? (S - p.window + 1) / kPage : 0;
    const int seg = segment_pages(p.num_pages);
#pragma unroll
    for (int i = 0; i < kReleasePer; ++i) {
      const int j = j0 + i * kReleaseThreads;
      old[i] = 1;
      if (e[i] < 0 || (j >= begin && j < end)) continue;
      row[j] = -1;
      if (e[i] >= p.num_pages)
        atomicOr(p.status, kStatusBadPage);
      else
        old[i] = atomicSub(p.refs + e[i], 1);
    }
#pragma unroll
    for (int i = 0; i < kReleasePer; ++i) {
      if (old[i] == 0) {
        atomicAdd(p.scratch + e[i] / seg, 1);
      } else if (old[i] < 0) {  // released more often than held
        atomicAdd(p.refs + e[i], 1);
        atomicOr(p.status, kStatusBadPage);
      }
    }
  }
}

// Latency bound (about 8 us with the segments' scan). Block b pushes the marked pages of segment b, after those of the segments
// before it, and clears their marks.
__global__ void __launch_bounds__(kCollectThreads) collect_kernel(const PageParams p) {
  begin();
  __shared__ int s_warp[32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int count = __ldcg(p.free_count);
  const int n0 = __ldcg(p.scratch + lane), n1 = lane + 32 < kPageSegments ? __ldcg(p.scratch + lane + 32) : 0;
  const int total = __reduce_add_sync(0xffffffffu, n0 + n1);
  int base = max(count, 0) + __reduce_add_sync(0xffffffffu, (lane < (int)blockIdx.x ? n0 : 0) +
                                                                (lane + 32 < (int)blockIdx.x ? n1 : 0));
  const int seg = segment_pages(p.num_pages);
  const int begin = min((int64_t)blockIdx.x * seg, (int64_t)p.num_pages);
  const int end = min((int64_t)begin + seg, (int64_t)p.num_pages);
  if (__ldcg(p.scratch + blockIdx.x) > 0) {
    for (int64_t p0 = begin; p0 < end; p0 += kCollectThreads * kCollectPer) {
      const int64_t mine = p0 + (int64_t)threadIdx.x * kCollectPer;
      uint32_t marks = 0;
#pragma unroll
      for (int i = 0; i < kCollectPer; ++i)
        if (mine + i < end && p.refs[mine + i] < 0) marks |= 1u << i;
      const int n = __popc(marks);
      int incl = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
      }
      if (lane == 31) s_warp[warp] = incl;
      __syncthreads();
      int before = incl - n, all = 0;
      for (int w = 0; w < kCollectThreads / 32; ++w) {
        const int v = s_warp[w];
        before += w < warp ? v : 0;
        all += v;
      }
      for (int i = 0, k = base + before; i < kCollectPer; ++i) {
        if (!(marks >> i & 1u)) continue;
        p.refs[mine + i] = 0;
        if (k < p.num_pages)
          p.free_pages[k] = (int32_t)(mine + i);
        else
          atomicOr(p.status, kStatusBadPage);  // more pages than the pool has
        ++k;
      }
      base += all;
      __syncthreads();
    }
  }
  if (last_block(p.scratch + kScratchShrinkTicket, gridDim.x) && threadIdx.x <= kPageSegments) {
    if (threadIdx.x == 0) *p.free_count = min(max(count, 0) + total, p.num_pages);
    p.scratch[threadIdx.x] = 0;  // the segments' counts and the ticket after them
  }
}

// One block per (copy, pool): page_bytes in 16-byte vectors, four in flight.
// Bound by writing: 384 pages of 16 KiB in 24 pools, 139 MB, in 25 us.
__global__ void __launch_bounds__(kCopyThreads) copy_pages_kernel(const PoolPtrs pools, int num_pools,
                                                                  int64_t page_bytes, int32_t num_pages,
                                                                  const int32_t* copy_src, const int32_t* copy_dst,
                                                                  int32_t* status) {
  begin();
  const int f = blockIdx.x / num_pools, pool = blockIdx.x % num_pools;
  const int src = copy_src[f], dst = copy_dst[f];
  if (src < 0 || dst < 0 || src == dst) return;
  if (src >= num_pages || dst >= num_pages) {
    if (threadIdx.x == 0) atomicOr(status, kStatusBadPage);
    return;
  }
  const uint4* from = reinterpret_cast<const uint4*>(pools.p[pool] + src * page_bytes);
  uint4* to = reinterpret_cast<uint4*>(pools.p[pool] + dst * page_bytes);
  const int n = (int)(page_bytes / 16);
  for (int i0 = threadIdx.x; i0 < n; i0 += 4 * kCopyThreads) {
    uint4 v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (i0 + u * kCopyThreads < n) v[u] = from[i0 + u * kCopyThreads];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (i0 + u * kCopyThreads < n) to[i0 + u * kCopyThreads] = v[u];
  }
}

// One block per (row, group of kCompactPools pools). A thread owns one 16-byte
// vector of the row's K/V rows in one pool and makes all of its moves in
// order, kCompactBatch reads before as many writes: sources never lie before
// the destinations written so far (node numbers increase and are at least
// their rank), so no move overwrites what a later one reads. 256 rows, up to
// six moves, 24 pools: 38 MB in 7.6 us.
__global__ void __launch_bounds__(kCompactThreads) compact_kernel(const CompactParams p, const PoolPtrs pools) {
  begin();
  const int r = blockIdx.x;
  __shared__ int s_src[kCompactMoves], s_dst[kCompactMoves];  // page * 16 + slot
  const int q0 = p.qsl[r], q1 = p.qsl[r + 1];
  const int L = q1 - q0, S = p.seq_lens[r], n = p.taken[r];
  const int C = S - L;
  const int32_t* path = p.path + (size_t)r * p.max_accept;
  const int32_t* bt = p.block_table + (size_t)r * p.max_pages;
  int bad = 0;
  if (L < 0 || S < L || S > p.max_pages * kPage || n < 0 || n > L ||
      n > p.max_accept) {
    bad = kStatusBadLengths;
  } else {
    for (int i = threadIdx.x; i < n; i += kCompactThreads) {
      const int a = path[i], prev = i > 0 ? path[i - 1] : -1;
      if (a <= prev || a < i || a >= L) {
        bad |= kStatusBadLengths;
      } else if (a != i && p.num_pools > 0) {
        const int from = bt[(C + a) / kPage], to = bt[(C + i) / kPage];
        if (from < 0 || from >= p.num_pages || to < 0 || to >= p.num_pages) bad |= kStatusBadPage;
      }
    }
  }
  const bool any = __syncthreads_or(bad);
  if (bad) atomicOr(p.status, bad);
  if (blockIdx.y == 0 && threadIdx.x == 0) p.new_seq_lens[r] = any ? S : C + n;
  if (any) return;
  const int vecs = p.num_kv_heads * (kRowBytes / 16);  // 16-byte vectors of one token in one pool
  const int pool0 = blockIdx.y * kCompactPools;
  const int np = min(kCompactPools, p.num_pools - pool0);
  for (int i0 = 0; i0 < n; i0 += kCompactMoves) {
    const int m = min(kCompactMoves, n - i0);
    __syncthreads();
    for (int i = threadIdx.x; i < m; i += kCompactThreads) {
      const int a = path[i0 + i], from = C + a, to = C + i0 + i;
      s_src[i] = a == i0 + i ? -1 : bt[from / kPage] * kPage + from % kPage;
      s_dst[i] = bt[to / kPage] * kPage + to % kPage;
    }
    __syncthreads();
    for (int w = threadIdx.x; w < np * vecs; w += kCompactThreads) {
      uint4* pool = reinterpret_cast<uint4*>(pools.p[pool0 + w / vecs]);
      const int h = (w % vecs) >> 3, c = w & 7;
      auto at = [&](int d) { return pool + (((size_t)(d / kPage) * p.num_kv_heads + h) * kPage + d % kPage) * 8 + c; };
      for (int i = 0; i < m; i += kCompactBatch) {
        uint4 v[kCompactBatch];
#pragma unroll
        for (int u = 0; u < kCompactBatch; ++u)
          if (i + u < m && s_src[i + u] >= 0) v[u] = *at(s_src[i + u]);
#pragma unroll
        for (int u = 0; u < kCompactBatch; ++u)
          if (i + u < m && s_src[i + u] >= 0) *at(s_dst[i + u]) = v[u];
      }
    }
  }
}

}  // namespace

cudaError_t launch_fork(const PageParams& p, cudaStream_t stream) {
  return launch(fork_kernel, dim3(p.num_forks), kForkThreads, stream, p);
}

cudaError_t launch_shrink(const PageParams& p, cudaStream_t stream) {
  const dim3 grid(p.num_seqs, min((p.max_pages + kReleaseSpan - 1) / kReleaseSpan, 65535));
  const cudaError_t e = launch(release_kernel, grid, kReleaseThreads, stream, p);
  if (e != cudaSuccess) return e;
  return launch(collect_kernel, dim3(kPageSegments), kCollectThreads, stream, p);
}

cudaError_t launch_copy_pages(const PoolPtrs& pools, int32_t num_pools, int64_t page_bytes, int32_t num_pages,
                              const int32_t* copy_src, const int32_t* copy_dst, int32_t num_copies, int32_t* status,
                              cudaStream_t stream) {
  return launch(copy_pages_kernel, dim3(num_copies * num_pools), kCopyThreads, stream, pools, num_pools, page_bytes,
                num_pages, copy_src, copy_dst, status);
}

cudaError_t launch_compact(const CompactParams& p, const PoolPtrs& pools, cudaStream_t stream) {
  const int groups = (p.num_pools + kCompactPools - 1) / kCompactPools;
  return launch(compact_kernel, dim3(p.num_seqs, groups > 0 ? groups : 1), kCompactThreads, stream, p, pools);
}

}  // namespace mcpu
