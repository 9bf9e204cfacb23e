// Eviction by accumulated attention weight (mcpu_evict_kv).
//
// One block per (layer, row, kv head). Of the N = n - first - last middle slots
// the K = budget - first - last with the highest weight stay: the K-th largest
// is found by a radix select over the weights' bits (11, 11 and 10 of them, one
// histogram each, no more once all of a bin stay), and among the slots that equal
// it the lowest are taken. Kept slots below inner = budget - last stay where they
// are; there are as many holes below it as kept slots past it, and the i-th of
// these moves into the i-th hole. The last ones follow as one shift towards the
// front. Both regions are walked in step, a block of slots at a time, and only as
// much of the two lists is held as the next moves need.
//
// Bound by the moves (K and V rows read and written, scattered 128-byte rows:
// 6144 items of 2112 to 2560 keys cut to 2048 move 1.2 GB in 243 us, 78 % of the
// copy rate); for rows just past their budget by the chain lengths -> weights ->
// three histograms -> ranks -> pages -> rows (512 items: 19 us).
#include <type_traits>

#include "keep.cuh"

namespace mcpu {

namespace {

constexpr int kPer = 4;                       // slots a thread ranks at a time
constexpr int kRowVecs = kRowBytes / 16;  // 16-byte pieces of a slot's K, or V
constexpr int kBins = 2048;

// Unsigned order of the weights: NaN lowest, the two zeros equal.
__device__ __forceinline__ uint32_t order(float w) {
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// kThreads threads, kResident blocks of them on an SM; the orders of kKeys middle
// slots and kTable pages are held; a thread has kFlight rows on their way.
template <int kThreads_, int kResident_, int kKeys_, int kTable_, int kFlight_>
struct EvictSmem {
  static constexpr int kResident = kResident_, kFlight = kFlight_;
  static constexpr int kThreads = kThreads_, kWarps = kThreads / 32, kKeys = kKeys_, kTable = kTable_;
  static constexpr int kBlock = kPer * kThreads;  // slots ranked at a time
  static constexpr int kQueue = 2 * kBlock;       // slots waiting for their partners
  static constexpr int kMoves = kThreads;         // pairs moved at a time
  static_assert(kMoves + kBlock <= kQueue && kBins % kThreads == 0, "sizes");
  uint32_t keys[kKeys];
  union {
    uint32_t hist[kBins];
    struct {  // (once the cutoff is known)
      int32_t src[kQueue], dst[kQueue];
    };
  };
  uint32_t table[kTable];  // first row of a page's tile (a pool's rows are fewer than 2^32: 128 bytes each)
  int32_t scan[2][kWarps];
  uint32_t cutoff;
  int32_t want;
  bool whole;  // all of the cutoff's bin stay
};

// Sum of the warps' values before this one's, and of all. `turn` alternates between calls.
template <typename S>
__device__ __forceinline__ int warps_scan(int x, S& s, int turn, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (lane == 0) s.scan[turn][warp] = x;
  __syncthreads();
  const int v = lane < S::kWarps ? s.scan[turn][lane] : 0;
  *total = __reduce_add_sync(0xffffffffu, v);
  return __reduce_add_sync(0xffffffffu, lane < warp ? v : 0);
}

struct Walk {  // of a region: next slot, slots at the cutoff so far, slots queued so far
  int at, seen, have;
};
struct Ranks {
  const float* w;
  int first;
  uint32_t cutoff;
  int ties;
  bool cached;
};

// Ranks the next kBlock slots of a region, a warp 32 neighbours at a time: those
// kept (or the holes) go to the queue.
template <typename S>
__device__ __noinline__ Walk walk(S& s, const Ranks r, Walk region, int stop, bool holes, int turn) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int j = region.at + kPer * 32 * warp + lane, inside = min(region.at + S::kBlock, stop) - region.at;
  const uint32_t below = (1u << lane) - 1u;
  uint32_t u[kPer], above[kPer], same[kPer];  // the warp's slots above the cutoff, and at it
  if (r.cached) {
#pragma unroll
    for (int e = 0; e < kPer; ++e) u[e] = j + 32 * e < stop ? s.keys[j + 32 * e - r.first] : 0u;
  } else {
    float v[kPer];
#pragma unroll
    for (int e = 0; e < kPer; ++e) v[e] = j + 32 * e < stop ? __ldcg(r.w + j + 32 * e) : 0.f;
#pragma unroll
    for (int e = 0; e < kPer; ++e) u[e] = order(v[e]);
  }
  int counts = 0, all;  // above, and at << 16
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    const bool in = j + 32 * e < stop;
    above[e] = __ballot_sync(0xffffffffu, in && u[e] > r.cutoff);
    same[e] = r.ties > 0 ? __ballot_sync(0xffffffffu, in && u[e] == r.cutoff) : 0u;
    counts += __popc(above[e]) + (__popc(same[e]) << 16);
  }
  const int before = warps_scan(counts, s, turn, &all);
  // of the slots at the cutoff as many are kept as are left of the ties
  const int left = max(r.ties - region.seen, 0);
  int equal = before >> 16, run = (before & 0xffff) + min(equal, left);  // kept before this warp's
  if (holes) run = min(kPer * 32 * warp, inside) - run;
  int32_t* queue = holes ? s.dst : s.src;
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    uint32_t take = above[e];
    if (same[e]) {  // (the same for the warp)
      take |= __ballot_sync(0xffffffffu, (same[e] >> lane & 1u) && equal + __popc(same[e] & below) < left);
      equal += __popc(same[e]);
    }
    if (holes) take = ~take & __ballot_sync(0xffffffffu, j + 32 * e < stop);
    if (take >> lane & 1u) queue[(region.have + run + __popc(take & below)) % S::kQueue] = j + 32 * e;
    run += __popc(take);
  }
  const int kept = (all & 0xffff) + min(all >> 16, left);
  return Walk{region.at + S::kBlock, region.seen + (all >> 16), region.have + (holes ? inside - kept : kept)};
}

template <typename S>
__global__ void __launch_bounds__(S::kThreads, S::kResident)
    evict_kernel(const EvictParams p, const __grid_constant__ PoolPtrs pools) {
  constexpr int kThreads = S::kThreads, kWarps = S::kWarps, kBlock = S::kBlock, kQueue = S::kQueue, kMoves = S::kMoves,
                kFlight = S::kFlight;
  extern __shared__ __align__(16) uint8_t smem[];
  S& s = *reinterpret_cast<S*>(smem);
  grid_dep_launch();
  grid_dep_wait();
  const int h = blockIdx.x, r = blockIdx.y, m = blockIdx.z, Hkv = p.num_kv_heads;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int n = p.seq_lens[r];
  const bool speaks = h == 0 && m == 0 && threadIdx.x == 0;
  const uint32_t rows = (uint32_t)Hkv * kPage;  // of a page
  const int32_t* table = p.block_table + (size_t)r * p.max_pages;
  bool cut = n > p.limit;
  int32_t bits = 0;
  const int page0 = p.first / kPage, pages = (n + kPage - 1) / kPage;
  if (n < 0 || n > p.max_pages * kPage || n > p.max_slots) {
    bits = kStatusBadLengths;
  } else if (cut) {
    const int mine = p.first < p.budget ? (p.budget + kPage - 1) / kPage : 0;
    int32_t bad = 0;
    for (int j = page0 + threadIdx.x; j < pages; j += kThreads) {
      const int page = table[j];
      if (j - page0 < S::kTable) s.table[j - page0] = (uint32_t)page * rows;
      if (page < 0 || page >= p.num_pages) bad |= kStatusBadPage;
      else if (p.refs && j < mine && p.refs[page] > 0) bad |= kStatusUnsupportedRow;
    }
    bits = (__syncthreads_or(bad & kStatusBadPage) ? kStatusBadPage : 0) |
           (__syncthreads_or(bad & kStatusUnsupportedRow) ? kStatusUnsupportedRow : 0);
  }
  if (bits) cut = false;
  if (speaks) {
    if (bits) atomicOr(p.status, bits);
    p.new_seq_lens[r] = cut ? p.budget : n;
  }
  if (p.num_layers == 0 || (bits & kStatusBadLengths)) return;
  const size_t at = (((size_t)m * p.num_seqs + r) * Hkv + h) * p.max_slots;
  const float* w = p.weights + at;
  float* nw = p.new_weights + at;
  const int inner = p.budget - p.last;
  const int first = p.first, end = n - p.last, K = inner - first;
  // the weights that stay where they are, if they go elsewhere (those of the middle with the first histogram)
  if (nw != w)
    for (int j = threadIdx.x; j < (cut ? first : n); j += kThreads) nw[j] = w[j];
  if (!cut) return;

  const bool held = pages - page0 <= S::kTable;
  auto first_row = [&](int slot) { return held ? s.table[slot / kPage - page0] : (uint32_t)table[slot / kPage] * rows; };
  // a thread moves one 16-byte piece of K and of V, of every kThreads / 8-th slot
  constexpr int kLanes = kThreads / kRowVecs;
  const int mine = threadIdx.x / kRowVecs;
  const size_t head = (size_t)h * kTileBytes + threadIdx.x % kRowVecs * 16;
  uint8_t *base_k = pools.p[m] + head, *base_v = pools.p[p.num_layers + m] + head;
  auto offset = [&](int slot) { return (uint64_t)(first_row(slot) + (uint32_t)slot % kPage) * kRowBytes; };
  auto load = [&](int slot, uint4 (&v)[2]) {
    const uint64_t at = offset(slot);
    v[0] = __ldcs(reinterpret_cast<const uint4*>(base_k + at));
    v[1] = __ldcs(reinterpret_cast<const uint4*>(base_v + at));
  };
  auto store = [&](int slot, const uint4 (&v)[2]) {
    const uint64_t at = offset(slot);
    *reinterpret_cast<uint4*>(base_k + at) = v[0];
    *reinterpret_cast<uint4*>(base_v + at) = v[1];
  };

  // ---- the K-th largest weight of the middle: its order, and how many that equal it stay
  uint32_t cutoff = 0xffffffffu;
  int ties = 0, turn = 0;
  const bool cached = end - first <= S::kKeys;
  auto key = [&](int j) { return cached ? s.keys[j - first] : order(__ldcg(w + j)); };
  if (K > 0) {
    int want = K;
    uint32_t prefix = 0;
    constexpr int kLoads = 8;
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, width = pass == 2 ? 10 : 11;
      for (int i = threadIdx.x; i < kBins; i += kThreads) s.hist[i] = 0;
      __syncthreads();
      auto count = [&](uint32_t u) {
        if (pass == 0 || (u >> (shift + width)) == (prefix >> (shift + width)))
          atomicAdd(&s.hist[(u >> shift) & ((1u << width) - 1u)], 1u);
      };
      if (cached && pass > 0) {
#pragma unroll 4
        for (int j = threadIdx.x; j < end - first; j += kThreads) count(s.keys[j]);
      } else {
        for (int j0 = first + threadIdx.x; j0 < end; j0 += kLoads * kThreads) {
          float v[kLoads];
#pragma unroll
          for (int e = 0; e < kLoads; ++e) v[e] = j0 + e * kThreads < end ? __ldcg(w + j0 + e * kThreads) : 0.f;
#pragma unroll
          for (int e = 0; e < kLoads; ++e) {
            const int j = j0 + e * kThreads;
            if (j >= end) continue;
            const uint32_t u = order(v[e]);
            if (cached) s.keys[j - first] = u;
            if (pass == 0 && nw != w && j < inner) nw[j] = v[e];
            count(u);
          }
        }
      }
      __syncthreads();
      // bins from the highest down: each warp has a range of them, and the one
      // that holds the want-th key finds its bin, 32 at a time
      constexpr int kRows = kBins / kThreads;
      int c[kRows], sum = 0, total;
#pragma unroll
      for (int e = 0; e < kRows; ++e) {
        c[e] = s.hist[kBins - 1 - 32 * (kRows * warp + e) - lane];
        sum += c[e];
      }
      sum = __reduce_add_sync(0xffffffffu, sum);
      int before = warps_scan(sum, s, turn, &total);
      turn ^= 1;
      if (before < want && before + sum >= want) {
#pragma unroll
        for (int e = 0; e < kRows; ++e) {
          const int row = __reduce_add_sync(0xffffffffu, c[e]);
          if (before < want && before + row >= want) {
            int incl = c[e];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
              const int v = __shfl_up_sync(0xffffffffu, incl, o);
              if (lane >= o) incl += v;
            }
            if (before + incl - c[e] < want && before + incl >= want) {
              s.cutoff = prefix | (uint32_t)(kBins - 1 - 32 * (kRows * warp + e) - lane) << shift;
              s.want = want - (before + incl - c[e]);
              s.whole = before + incl == want;
            }
          }
          before += row;
        }
      }
      __syncthreads();
      prefix = s.cutoff;
      want = s.want;
      if (s.whole) {  // (of distinct weights mostly after two passes; prefix is not 0, as not all stay)
        --prefix;
        want = 0;
        break;
      }
    }
    cutoff = prefix;
    ties = want;
  }

  // ---- kept slots at or past inner fill the holes before it, in order
  int ties_before = 0;  // slots equal to the cutoff before inner
  if (ties > 0) {
    int same = 0;
#pragma unroll 4
    for (int j = first + threadIdx.x; j < inner; j += kThreads) same += key(j) == cutoff;
    warps_scan(__reduce_add_sync(0xffffffffu, same), s, turn, &ties_before);
    turn ^= 1;
  }
  Walk a{first, 0, 0}, b{inner, ties_before, 0};
  const Ranks ranks{w, first, cutoff, ties, cached};
  int done = 0;
#pragma unroll 1
  while (K > 0) {
    while (true) {  // kept slots for the next moves, then as many holes
      const bool holes = b.have - done >= kMoves || b.at >= end;
      if (holes && (a.have >= min(done + kMoves, b.have) || a.at >= inner)) break;
      if (holes) a = walk(s, ranks, a, inner, true, turn);
      else b = walk(s, ranks, b, end, false, turn);
      turn ^= 1;
    }
    __syncthreads();
    const int count = min(min(a.have, b.have) - done, kMoves);
    if (count <= 0) break;
#pragma unroll 1
    for (int i0 = mine; i0 < count; i0 += kFlight * kLanes) {
      uint4 v[kFlight][2];
#pragma unroll
      for (int k = 0; k < kFlight; ++k)
        if (i0 + k * kLanes < count) load(s.src[(done + i0 + k * kLanes) % kQueue], v[k]);
#pragma unroll
      for (int k = 0; k < kFlight; ++k)
        if (i0 + k * kLanes < count) store(s.dst[(done + i0 + k * kLanes) % kQueue], v[k]);
    }
    for (int e = threadIdx.x; e < count; e += kThreads) nw[s.dst[(done + e) % kQueue]] = w[s.src[(done + e) % kQueue]];
    done += count;
    __syncthreads();
  }

  // ---- the last ones, towards the front: a piece of them at a time, read before it is written
  __syncthreads();
  constexpr int kPiece = kFlight * kLanes;
  const bool apart = n - p.budget >= p.last;  // they do not overlap their new places
#pragma unroll 1
  for (int i0 = 0; i0 < p.last; i0 += kPiece) {
    const int count = min(p.last - i0, kPiece);
    uint4 v[kFlight][2];
    float weight = 0.f;
#pragma unroll
    for (int k = 0; k < kFlight; ++k)
      if (mine + k * kLanes < count) load(end + i0 + mine + k * kLanes, v[k]);
    if (threadIdx.x < count) weight = w[end + i0 + threadIdx.x];
    if (!apart) __syncthreads();
#pragma unroll
    for (int k = 0; k < kFlight; ++k)
      if (mine + k * kLanes < count) store(inner + i0 + mine + k * kLanes, v[k]);
    if (threadIdx.x < count) nw[inner + i0 + threadIdx.x] = weight;
    if (!apart) __syncthreads();
  }

  // ---- slots that are free now: keys that take them start without weight
  if (p.new_weights == p.weights) {
    __syncthreads();
    float* row = p.new_weights + (((size_t)blockIdx.z * p.num_seqs + blockIdx.y) * gridDim.x + blockIdx.x) * p.max_slots;
    for (int j = p.budget + threadIdx.x; j < n; j += kThreads) row[j] = 0.f;
  }
}

}  // namespace

using Middle = EvictSmem<256, 5, 4096, 1024, 2>;
using Large = EvictSmem<512, 2, 8192, 4096, 4>;

cudaError_t launch_evict(const EvictParams& p, const PoolPtrs& pools, int sms, cudaStream_t stream) {
  const dim3 grid(p.num_kv_heads, p.num_seqs, p.num_layers > 0 ? p.num_layers : 1);
  const int64_t items = (int64_t)grid.x * grid.y * grid.z;
  auto launch = [&](auto kernel, auto* smem) {
    using S = std::remove_pointer_t<decltype(smem)>;
    LaunchCfg lc(grid, dim3(S::kThreads), sizeof(S), stream, true);
    return cudaLaunchKernelEx(&lc.cfg, kernel, p, pools);
  };
  // Large blocks as long as all are on the SMs at once (256 items of 8192 to 32768
  // keys: 123 us, by small ones 199), then small ones, with more of them at
  // different steps (512 items of 2032 to 2128 keys, from HBM: 25 us, by large
  // ones 31; 6144 of 2112 to 2560: 247 and 302).
  if (items > 2 * sms) return launch(evict_kernel<Middle>, (Middle*)nullptr);
  return launch(evict_kernel<Large>, (Large*)nullptr);
}

cudaError_t prepare_evict_kernels() {
  constexpr auto kSmem = cudaFuncAttributeMaxDynamicSharedMemorySize;
  cudaError_t e = cudaFuncSetAttribute(evict_kernel<Middle>, kSmem, (int)sizeof(Middle));
  if (e == cudaSuccess) e = cudaFuncSetAttribute(evict_kernel<Large>, kSmem, (int)sizeof(Large));
  return e;
}

}  // namespace mcpu
