// Verification of drafted tokens (mcpu_verify_tree).
//
// At each node of the walk, with p = softmax(l / T) and (if given) q of the
// draft, the residual after rejecting k children of masses m_0 = 1, m_1 .. is
//   rest(y) = max(p(y) - M q(y), 0),  M = m_0 + .. + m_{k-1},  m_k = sum_y rest(y)
// because max(max(a, 0) - b, 0) = max(a - b, 0) for b >= 0: only M is carried,
// no vector. Without a draft a rejected token's p goes to 0, and m is what is
// left of the sum: a difference down to a quarter of it, then summed anew over the
// other tokens (1 - p loses the digits of a peaked distribution's tail). The next
// token is argmax_y rest(y) / e_y, which for exponential e is y with probability
// rest(y) / m.
//
// A cluster of blocks walks a row's tree, a slice of the vocabulary each; only
// the nodes that the walk visits are read. A node costs one pass over its
// logits (maximum, its place and the sum together), a rejection with draft
// probabilities one more (without, where little is left), the row's end one with
// the exponentials; what was read before comes from L2 then. After a pass every
// warp hands its result to all blocks of the cluster (distributed shared memory),
// and behind one cluster barrier every warp joins them all in the same order: all
// take the same decisions, and nothing is sent back.
//
// A pass streams the rows through shared memory: every warp copies its part
// ahead (cp.async) and takes it out again, with no block barrier, so that the
// loop that is executed stays small (unrolled over as many loads as a slice needs
// in flight, its instructions came from L2: 14000 cycles for one group of eight).
//
// Bound by the chain of a row's nodes where rows are few (64 rows, up to 7 nodes on
// a path, 131072 bf16 logits: 34 to 50 us from process to process; a node's first
// loads, two steps, the exchange), with SMs that hold no block for 36 % of the time
// (512 blocks in places for 456: rows that come late begin as others end); by HBM
// where they are many (384 rows of fp32 logits: 595 MB in 131 us, 67 % of the copy
// rate; SMs hold a block for 83 % of the time).
//
// Everything is fp32. Sums are pairs: 8 terms at a time, added by an exact two-sum
// (a plain chain of additions loses 1e-6 of a peaked distribution's tail).
// Exponentials by ex2.approx (2^-22).
#include <type_traits>

#include "keep.cuh"

namespace mcpu {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32, kMaxCluster = 8;
constexpr int kMaxNodes = MCPU_MAX_TREE_NODES;
constexpr float kLowest = -3.402823466e38f;  // a finite maximum to begin with: -inf logits weigh nothing against it
constexpr float kLog2e = 1.4426950408889634f, kLog2eLow = 1.925963033500e-08f;  // log2(e) = the sum of both

struct Stats {  // of a distribution: maximum, the lowest token that has it, sum of e^((l - max) / T)
  float max;
  int32_t at;
  float sum, low;  // the sum of both
};

struct VerifySmem {
  Stats stats[2][2][kMaxCluster * kWarps];  // [turn][target, draft][warp of the cluster]
  float2 sums[2][kMaxCluster * kWarps];
  uint64_t best[2][kMaxCluster * kWarps];
  int32_t gone[kMaxNodes];  // tokens of the rejected children of the node
  int32_t path[kMaxNodes];
  int32_t out[kMaxNodes];    // what was emitted after each node of the path,
  Stats node[kMaxNodes];     // and that node's distribution
};

// ----------------------------------------------------------- the cluster
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_sync() {
  cluster_arrive();
  cluster_wait();
}
// Stores to a shared-memory object in block `rank` of the cluster.
__device__ __forceinline__ uint32_t peer_addr(const void* p, uint32_t rank) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_addr(p)), "r"(rank));
  return a;
}
__device__ __forceinline__ void peer_store(uint32_t addr, uint32_t a, uint32_t b) {
  asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(addr), "r"(a), "r"(b) : "memory");
}

// ----------------------------------------------------- eight values of a row
template <typename T>
struct Raw {  // as they are loaded
  static constexpr int kWords = 8 * sizeof(T) / 4;
  uint32_t w[kWords];
  __device__ __forceinline__ float get(int i) const {
    if (sizeof(T) == 4) return __uint_as_float(w[i]);
    return __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);
  }
};
template <typename T>
constexpr uint32_t kNegInf = sizeof(T) == 4 ? 0xff800000u : 0xff80u;

// The slice of the vocabulary that a block has. Its threads take groups of eight
// values, kGroups of them a step; `shift` moves the groups to where the row has
// its 16-byte vectors, so that the first one may begin before the slice.
struct Slice {
  int begin, end, shift;
  // first value of the block's step k, of a thread's group e of it
  __device__ __forceinline__ int step(int k, int groups) const { return begin - shift + 8 * groups * k * kThreads; }
  static __device__ __forceinline__ int group(int step, int e) {
    return step + 8 * (e * kThreads + (int)threadIdx.x);
  }
  __device__ __forceinline__ int steps(int groups) const {
    const int per = 8 * groups * kThreads;
    return begin < end ? (end - begin + shift + per - 1) / per : 0;
  }
};

template <typename T>
__device__ __forceinline__ uint32_t offset16(const T* p) {
  return (uint32_t)(reinterpret_cast<uintptr_t>(p) & 15);
}

// Every warp has a ring of its own (warps may be at different passes). A slot
// holds, for every row and group of a step, 256 values as they lie in the row, a
// 16-byte vector a lane and copy: 512 bytes in one piece (a lane's own 32 bytes
// as two copies cost twice the traffic from L2: 384 fp32 rows 208 us, so 129).
// A row that need not have its vectors where the groups begin has one more
// (kExtra). Vectors of fp32 rows are swapped in pairs, so that lanes that take
// every other one meet no bank twice.
template <typename T>
constexpr int kVectors = 8 * sizeof(T) / 16;  // of a group, per thread
template <typename T, bool kExtra>
constexpr int kPartBytes = 16 * (32 * kVectors<T> + kExtra);

template <typename T>
__device__ __forceinline__ uint8_t* vector_at(uint8_t* part, int i) {
  return part + 16 * (sizeof(T) == 4 ? i ^ (i >> 3 & 1) : i);
}
__device__ __forceinline__ void copy16(uint8_t* dst, const uint8_t* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_addr(dst)), "l"(src) : "memory");
}

// A vector that may leave the row or the slice, whose first value is the row's at-th.
template <typename T>
__device__ __noinline__ void fetch_edge(uint8_t* dst, const T* row, int at, int begin, int end, int n) {
  constexpr int kValues = 16 / sizeof(T);
  if (at >= end || at + kValues <= begin) return;
  if (at >= 0 && at + kValues <= n) return copy16(dst, reinterpret_cast<const uint8_t*>(row + at));
#pragma unroll 1
  for (int i = 0; i < kValues; ++i)
    if (at + i >= 0 && at + i < n) reinterpret_cast<T*>(dst)[i] = row[at + i];
}

// Starts the copies of step k of a row of n values (kExtra: with the extra vectors).
template <int kGroups, bool kExtra, typename T>
__device__ __forceinline__ void fetch(uint8_t* slot, const T* row, const Slice& s, int k, int n) {
  const int lane = threadIdx.x & 31, first = s.group(s.step(k, kGroups), 0) - 8 * lane;  // of the warp
  const uint32_t off = kExtra ? offset16(row + first) : 0u;
  const int at = first - (int)off / (int)sizeof(T);
  const uint8_t* src = reinterpret_cast<const uint8_t*>(row + at) + 16 * lane;
#pragma unroll
  for (int e = 0; e < kGroups; ++e) {
    uint8_t* part = slot + e * kPartBytes<T, kExtra>;
    const int j = at + 8 * e * kThreads;
    if (j >= s.begin && j + kPartBytes<T, kExtra> / (int)sizeof(T) <= s.end) {
#pragma unroll
      for (int v = 0; v < kVectors<T>; ++v)
        copy16(vector_at<T>(part, 32 * v + lane), src + e * (kThreads * 8 * (int)sizeof(T)) + 512 * v);
      if (kExtra && off && lane == 0)
        copy16(vector_at<T>(part, 32 * kVectors<T>), src + e * (kThreads * 8 * (int)sizeof(T)) + 512 * kVectors<T>);
    } else {
#pragma unroll 1
      for (int i = lane; i < 32 * kVectors<T> + (off ? 1 : 0); i += 32)
        fetch_edge(vector_at<T>(part, i), row, j + i * (16 / (int)sizeof(T)), s.begin, s.end, n);
    }
  }
}

// Takes group e of step k out again; values outside the slice become `fill` (as bits of one).
template <int kGroups, bool kExtra, typename T>
__device__ __forceinline__ void take(uint8_t* slot, const T* row, const Slice& s, int k, int e, uint32_t fill, Raw<T>& r) {
  constexpr int kWords = Raw<T>::kWords;
  const int first = s.step(k, kGroups), per = 8 * kGroups * kThreads, lane = threadIdx.x & 31;
  const uint32_t off = kExtra ? offset16(row + first) : 0u;
  uint8_t* part = slot + e * kPartBytes<T, kExtra>;
#pragma unroll
  for (int v = 0; v < kVectors<T>; ++v) {
    const uint4 x = *reinterpret_cast<const uint4*>(vector_at<T>(part, lane * kVectors<T> + v));
    r.w[4 * v] = x.x, r.w[4 * v + 1] = x.y, r.w[4 * v + 2] = x.z, r.w[4 * v + 3] = x.w;
  }
  if (kExtra && off) {
    const uint4 x = *reinterpret_cast<const uint4*>(vector_at<T>(part, (lane + 1) * kVectors<T>));
    uint32_t w[kWords + 4];
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = r.w[i];
    w[kWords] = x.x, w[kWords + 1] = x.y, w[kWords + 2] = x.z, w[kWords + 3] = x.w;
    const uint32_t bits = (off & 3) * 8;
    // by two words, by one, by half of one
#pragma unroll
    for (int i = 0; i < kWords + 2; ++i) w[i] = off & 8 ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < kWords + 1; ++i) w[i] = off & 4 ? w[i + 1] : w[i];
#pragma unroll
    for (int i = 0; i < kWords; ++i) r.w[i] = sizeof(T) == 2 ? __funnelshift_r(w[i], w[i + 1], bits) : w[i];
  }
  if (first >= s.begin && first + per <= s.end) return;
  const int j = s.group(first, e);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (j + i >= s.begin && j + i < s.end) continue;
    if (sizeof(T) == 4) r.w[i] = fill;
    else if (i & 1) r.w[i >> 1] = (r.w[i >> 1] & 0xffffu) | fill << 16;
    else r.w[i >> 1] = (r.w[i >> 1] & 0xffff0000u) | fill;
  }
}

// Streams: issue(k, slot) for the steps k < n runs up to Pass::kDepth ahead of
// use(k, slot), every warp by itself. prime() sets the first copies on their way,
// once those of an earlier stream have landed.
template <typename Pass, typename Issue>
__device__ __forceinline__ void prime(uint8_t* ring, int n, Issue issue) {
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  __syncwarp();
#pragma unroll 1
  for (int k = 0; k < Pass::kDepth - 1; ++k) {
    if (k < n) issue(k, ring + k * Pass::kBytes);
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
}
template <typename Pass, typename Issue, typename Use>
__device__ __forceinline__ void stream(uint8_t* ring, int n, Issue issue, Use use) {
  int at = Pass::kDepth - 1;
#pragma unroll 1
  for (int k = 0; k < n; ++k) {
    // step k + kDepth - 1 goes where step k - 1 was
    uint8_t* slot = ring + at * Pass::kBytes;
    if (++at == Pass::kDepth) at = 0;
    __syncwarp();
    if (k + Pass::kDepth - 1 < n) issue(k + Pass::kDepth - 1, slot);
    asm volatile("cp.async.commit_group;" ::: "memory");
    asm volatile("cp.async.wait_group %0;" ::"n"(Pass::kDepth - 1) : "memory");
    __syncwarp();
    use(k, ring + at * Pass::kBytes);
  }
}

__device__ __forceinline__ float at_token(const __nv_bfloat16* x, int i) { return __bfloat162float(x[i]); }
__device__ __forceinline__ float at_token(const float* x, int i) { return x[i]; }

// hi + lo += x exactly (up to the rounding of lo)
__device__ __forceinline__ void add_exact(float& hi, float& lo, float x) {
  const float s = hi + x, b = s - hi;
  lo += (hi - (s - b)) + (x - b);
  hi = s;
}
__device__ __forceinline__ void warp_add_exact(float& hi, float& lo) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float oh = __shfl_xor_sync(0xffffffffu, hi, o), ol = __shfl_xor_sync(0xffffffffu, lo, o);
    lo += ol;
    add_exact(hi, lo, oh);  // (the error is exact: both sides of a pair get the same bits)
  }
}
// Largest value of the warp, and the lowest `at` of those that have it (no NaN).
__device__ __forceinline__ float warp_max(float m) {
  const uint32_t u = __float_as_uint(m);
  const uint32_t top = __reduce_max_sync(0xffffffffu, u & 0x80000000u ? ~u : u | 0x80000000u);
  return __uint_as_float(top & 0x80000000u ? top & 0x7fffffffu : ~top);
}
__device__ __forceinline__ void warp_max(float& m, int& at) {
  const float most = warp_max(m);
  at = __reduce_min_sync(0xffffffffu, m == most ? at : 0x7fffffff);
  m = most;
}
__device__ __forceinline__ uint64_t warp_best(uint64_t key) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const uint64_t other = __shfl_xor_sync(0xffffffffu, (unsigned long long)key, o);
    if (other > key) key = other;
  }
  return key;
}

// Packed: e^((v - m) / T) of the values 2 i, 2 i + 1 of a group, from -m and c = log2(e) / T twice each.
template <typename T>
__device__ __forceinline__ uint64_t weights2(const Raw<T>& v, int i, uint64_t neg_m, uint64_t c) {
  uint64_t x = add2(pack_f32x2(v.get(2 * i), v.get(2 * i + 1)), neg_m);
  asm("mul.rn.f32x2 %0, %0, %1;" : "+l"(x) : "l"(c));
  return pack_f32x2(ex2_approx(lo_f32(x)), ex2_approx(hi_f32(x)));
}

__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

template <typename T>
__device__ __forceinline__ float top_of(const Raw<T>& v) {
  float top = fmaxf(v.get(0), v.get(1));
#pragma unroll
  for (int i = 2; i < 8; i += 2) top = fmax3(top, v.get(i), v.get(i + 1));
  return top;
}

// What all warps of the cluster have of a distribution, joined in their order.
__device__ __forceinline__ Stats join_stats(const Stats* part, int parts, float c) {
  const int lane = threadIdx.x & 31;
  float m = kLowest, z = 0.f, zl = 0.f;
  int at = 0x7fffffff;
  for (int i = lane; i < parts; i += 32) {
    const Stats o = part[i];
    if (o.max > m || (o.max == m && o.at < at)) m = o.max, at = o.at;
  }
  warp_max(m, at);
  for (int i = lane; i < parts; i += 32) {
    const Stats o = part[i];
    const float f = ex2_approx((o.max - m) * c);
    add_exact(z, zl, o.sum * f);
    zl += o.low * f;
  }
  warp_add_exact(z, zl);
  return Stats{m, at, z, zl};
}

// Adds kN groups of a row to its running maximum and sum relative to it.
template <typename T, int kN>
__device__ __forceinline__ bool add_groups(const Raw<T> (&v)[kN], float c, float& m, float& z, float& zl, float* scaled) {
  float top = top_of(v[0]);
#pragma unroll
  for (int e = 1; e < kN; ++e) top = fmaxf(top, top_of(v[e]));
  const bool rises = top > m;
  if (rises) {
    const float f = ex2_approx((m - top) * c);
    z *= f;
    zl *= f;
    *scaled *= f;
    m = top;
  }
  const uint64_t neg = pack_f32x2(-m, -m), cc = pack_f32x2(c, c);
  uint64_t sum[2] = {0, 0};
#pragma unroll
  for (int e = 0; e < kN; ++e)
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i & 1] = add2(sum[i & 1], weights2(v[e], i, neg, cc));
  sum[0] = add2(sum[0], sum[1]);
  add_exact(z, zl, lo_f32(sum[0]) + hi_f32(sum[0]));
  return rises;
}

// Lets the eight tokens from j on into the race: rest / e > best where
// rest - best e > 0, so no division but for what comes to lead. Tokens of the
// `lost` rejected children do not take part.
__device__ __forceinline__ void race8(const uint64_t (&rest)[4], const Raw<float>& e, int j, const VerifySmem& s, int lost,
                                      float& best, int& best_at) {
  const uint64_t neg_best = pack_f32x2(-best, -best);
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint64_t lead = fma2(pack_f32x2(e.get(2 * i), e.get(2 * i + 1)), neg_best, rest[i]);
    top = fmax3(top, lo_f32(lead), hi_f32(lead));
  }
  if (!(top > 0.f)) return;
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float w = i & 1 ? hi_f32(rest[i >> 1]) : lo_f32(rest[i >> 1]);
    v[i] = w > 0.f ? __fdividef(w, e.get(i)) : 0.f;
  }
  for (int g = 0; g < lost; ++g) {
    const int i = s.gone[g] - j;
    if (i >= 0 && i < 8) {
#pragma unroll
      for (int d = 0; d < 8; ++d) v[d] = d == i ? 0.f : v[d];
    }
  }
  top = 0.f;
#pragma unroll
  for (int i = 0; i < 8; i += 2) top = fmax3(top, v[i], v[i + 1]);
  if (top > best) {
    best = top;
#pragma unroll
    for (int i = 7; i >= 0; --i) best_at = v[i] == top ? j + i : best_at;
  }
}

// The ring, and what a pass makes of it: groups a step, bytes, steps in flight.
// 60 KiB leave room for three blocks on an SM.
constexpr int kRingBytes = 60 * 1024, kWarpRing = kRingBytes / kWarps;
template <typename T>
struct PassOne {  // one row
  static constexpr int kGroups = 8 / sizeof(T), kBytes = kGroups * kPartBytes<T, false>, kDepth = kWarpRing / kBytes;
};
template <typename T>
struct PassTwo {  // target and draft
  static constexpr int kGroups = 4 / sizeof(T), kDraft = kGroups * kPartBytes<T, false>,
                       kBytes = kDraft + kGroups * kPartBytes<T, true>, kDepth = kWarpRing / kBytes;
};
template <typename T, bool kWithDraft>
struct PassRace {  // target, exponentials, draft
  static constexpr int kNoise = kPartBytes<T, false>, kDraft = kNoise + kPartBytes<float, true>,
                       kBytes = kDraft + (kWithDraft ? kPartBytes<T, true> : 0), kDepth = kWarpRing / kBytes;
};
static_assert(PassRace<float, true>::kDepth >= 2, "the deepest step");

template <typename T>
__global__ void __launch_bounds__(kThreads, 3) verify_kernel(const VerifyParams p) {
  __shared__ VerifySmem s;
  extern __shared__ __align__(16) uint8_t rings[];
  cluster_arrive();  // (every block of the cluster is there before the first store into its memory)
  grid_dep_launch();
  grid_dep_wait();
  const uint32_t rank = cluster_rank(), size = cluster_size();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint8_t* ring = rings + warp * kWarpRing;
  const int parts = (int)size * kWarps, mine = (int)rank * kWarps + warp;
  const int r = blockIdx.x / size, V = p.vocab;
  const int q0 = p.qsl[r], L = p.qsl[r + 1] - q0;
  const float heat = p.temperature ? p.temperature[r] : 0.f;
  int32_t bits = 0;
  if (p.qsl[0] != 0 || p.qsl[p.num_seqs] != p.total_q || q0 < 0 || L < 0 || L > p.total_q - q0) bits = kStatusBadLengths;
  else if (L > kMaxNodes) bits = kStatusUnsupportedRow;
  const bool greedy = heat == 0.f, walks = !bits && L > 0;
  bool bad = !greedy && !(heat >= 1e-20f && heat <= 1e20f);
  int cur = 0, len = walks ? 1 : 0, next = -1;
  const float div = greedy ? 1.f : heat;
  float c = __fdividef(kLog2e, div);
  c += __fdividef(fmaf(-c, div, kLog2e) + kLog2eLow, div);  // log2(e) / T, rounded once
  const uint64_t cc = pack_f32x2(c, c);
  const int per = (V + 8 * (int)size - 1) / (8 * (int)size) * 8;
  Slice slice;
  slice.shift = 0;
  slice.begin = min(V, (int)rank * per);
  slice.end = min(V, slice.begin + per);
  const float* noise = greedy ? nullptr : p.noise + (size_t)r * p.noise_stride;
  uint32_t turn = 0;  // of the exchange buffers
  int primed = -1;    // node whose first logits are on their way into the ring,
  bool primed_race = false;  // for the race
  cluster_wait();

  while (walks && !bad) {
    const T* x = static_cast<const T*>(p.logits) + (size_t)(q0 + cur) * p.logits_stride;
    const T* y = p.draft && !greedy ? static_cast<const T*>(p.draft) + (size_t)(q0 + cur) * p.draft_stride : nullptr;
    // the nodes after this one, up to 32: their loads are on their way during the pass
    const int w1 = (cur + 1) & ~31;
    int up = -1, token = -1;
    float u = 0.f;
    if (w1 + lane < L) {
      up = p.parents[q0 + w1 + lane];
      token = p.tokens[q0 + w1 + lane];
      if (!greedy) u = p.uniforms[q0 + w1 + lane];
    }
    const bool more = len < p.max_accept, token_ok = token >= 0 && token < V;
    bool kid = more && up == cur && w1 + lane > cur && token_ok;
    auto row_of = [&](const void* base, int64_t stride, int node) {
      return static_cast<const T*>(base) + (size_t)(q0 + node) * stride;
    };

    // ---- a sampled node without children: its sums and the race in one pass
    bool leaf = !greedy && !__any_sync(0xffffffffu, kid);
    for (int w0 = w1 + 32; w0 < L && leaf && more; w0 += 32) {
      const int t = w0 + lane < L && p.parents[q0 + w0 + lane] == cur ? p.tokens[q0 + w0 + lane] : -1;
      leaf = !__any_sync(0xffffffffu, t >= 0 && t < V);
    }
    if (leaf) {
      using Pass = PassRace<T, false>;
      constexpr int off_e = Pass::kNoise;
      float m = kLowest, z = 0.f, zl = 0.f, best = 0.f;
      int best_at = 0x7fffffff;
      slice.shift = offset16(x + slice.begin) / (int)sizeof(T);
      auto issue = [&](int k, uint8_t* slot) {
        fetch<1, false>(slot, x, slice, k, V);
        fetch<1, true>(slot + off_e, noise, slice, k, V);
      };
      if (primed != cur || !primed_race) prime<Pass>(ring, slice.steps(1), issue);
      stream<Pass>(ring, slice.steps(1), issue, [&](int k, uint8_t* slot) {
        Raw<T> v[1];
        Raw<float> e;
        take<1, false>(slot, x, slice, k, 0, kNegInf<T>, v[0]);
        take<1, true>(slot + off_e, noise, slice, k, 0, 0x3f800000u, e);
        add_groups(v, c, m, z, zl, &best);
        const uint64_t neg = pack_f32x2(-m, -m);
        uint64_t rest[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) rest[i] = weights2(v[0], i, neg, cc);
        race8(rest, e, slice.group(slice.step(k, 1), 0), s, 0, best, best_at);
      });
      const float wm = warp_max(m), f = ex2_approx((m - wm) * c);
      z *= f;
      zl *= f;
      warp_add_exact(z, zl);
      const uint64_t lead = warp_best((uint64_t)__float_as_uint(best * f) << 32 | (uint32_t)~best_at);
      if (lane < (int)size) {
        const uint32_t to = peer_addr(&s.stats[turn][0][mine], lane);
        peer_store(to, __float_as_uint(wm), 0x7fffffffu);
        peer_store(to + 8, __float_as_uint(z), __float_as_uint(zl));
        peer_store(peer_addr(&s.best[turn][mine], lane), (uint32_t)lead, (uint32_t)(lead >> 32));
      }
      cluster_sync();
      const Stats st = join_stats(s.stats[turn][0], parts, c);
      uint64_t key = 0;
      for (int i = lane; i < parts; i += 32) {
        const uint64_t o = s.best[turn][i];
        const float v = __uint_as_float((uint32_t)(o >> 32)) * ex2_approx((s.stats[turn][0][i].max - st.max) * c);
        key = max(key, (uint64_t)__float_as_uint(v) << 32 | (uint32_t)o);
      }
      key = warp_best(key);
      bad = !(st.sum > 0.f && st.sum < 3e38f) || !(key >> 32);
      if (!bad) next = (int)~(uint32_t)key;
      if (threadIdx.x == 0) {
        s.out[len - 1] = max(next, 0);
        s.node[len - 1] = st;
      }
      break;
    }

    // ---- maximum and sum of the node's distributions
    Stats st[2];
    using One = PassOne<T>;
    using Two = PassTwo<T>;
    float m[2] = {kLowest, kLowest}, z[2] = {0.f, 0.f}, zl[2] = {0.f, 0.f}, none = 0.f;
    int best_step = 0;  // that holds the thread's maximum
    slice.shift = offset16(x + slice.begin) / (int)sizeof(T);
    const bool ready = primed == cur && !primed_race;
    if (!y) {
      auto issue = [&](int k, uint8_t* slot) { fetch<One::kGroups, false>(slot, x, slice, k, V); };
      if (!ready) prime<One>(ring, slice.steps(One::kGroups), issue);
      stream<One>(ring, slice.steps(One::kGroups), issue, [&](int k, uint8_t* slot) {
        Raw<T> v[One::kGroups];
#pragma unroll
        for (int e = 0; e < One::kGroups; ++e) take<One::kGroups, false>(slot, x, slice, k, e, kNegInf<T>, v[e]);
        if (add_groups(v, c, m[0], z[0], zl[0], &none)) best_step = k;
      });
    } else {
      auto issue = [&](int k, uint8_t* slot) {
        fetch<Two::kGroups, false>(slot, x, slice, k, V);
        fetch<Two::kGroups, true>(slot + Two::kDraft, y, slice, k, V);
      };
      if (!ready) prime<Two>(ring, slice.steps(Two::kGroups), issue);
      stream<Two>(ring, slice.steps(Two::kGroups), issue, [&](int k, uint8_t* slot) {
        Raw<T> v[Two::kGroups];
#pragma unroll
        for (int e = 0; e < Two::kGroups; ++e) take<Two::kGroups, false>(slot, x, slice, k, e, kNegInf<T>, v[e]);
        add_groups(v, c, m[0], z[0], zl[0], &none);
#pragma unroll
        for (int e = 0; e < Two::kGroups; ++e)
          take<Two::kGroups, true>(slot + Two::kDraft, y, slice, k, e, kNegInf<T>, v[e]);
        add_groups(v, c, m[1], z[1], zl[1], &none);
      });
    }
    float lx = 0.f, ly = 0.f;  // the child's own logits
    if (kid) {
      lx = at_token(x, token);
      if (y) ly = at_token(y, token);
    }
#pragma unroll
    for (int d = 0; d < 2; ++d) {
      if (d == 1 && !y) break;
      const float wm = warp_max(m[d]);
      int at = 0x7fffffff;
      if (greedy) {
        if (sizeof(T) == 4 && wm == kLowest) {
          // the value that maxima begin with: no step has raised it, so the first
          // of the thread's tokens that has it, if any has (else the sum is 0)
          const int n = z[d] > 0.f ? slice.steps(One::kGroups) * One::kGroups * 8 : 0;
#pragma unroll 1
          for (int i = 0; i < n && at == 0x7fffffff; ++i) {
            const int e = i >> 3, j = slice.group(slice.step(e / One::kGroups, One::kGroups), e % One::kGroups) + (i & 7);
            if (j >= slice.begin && j < slice.end && at_token(x, j) == wm) at = j;
          }
        } else if (m[d] == wm) {  // the lowest token that has it, among this thread's of that step
          const bool held = best_step >= slice.steps(One::kGroups) - One::kDepth;  // it is in the ring still
          uint8_t* slot = ring + best_step % One::kDepth * One::kBytes;
#pragma unroll 1
          for (int e = One::kGroups - 1; e >= 0; --e) {
            const int j = slice.group(slice.step(best_step, One::kGroups), e);
            Raw<T> v;
            if (held) {
              take<One::kGroups, false>(slot, x, slice, best_step, e, kNegInf<T>, v);
            } else {
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const float l = j + i >= slice.begin && j + i < slice.end ? at_token(x, j + i) : -INFINITY;
                if (sizeof(T) == 4) v.w[i] = __float_as_uint(l);
                else if (i & 1) v.w[i >> 1] |= __float_as_uint(l) & 0xffff0000u;
                else v.w[i >> 1] = __float_as_uint(l) >> 16;
              }
            }
#pragma unroll
            for (int i = 7; i >= 0; --i) at = v.get(i) == wm ? j + i : at;
          }
        }
        at = __reduce_min_sync(0xffffffffu, at);
      }
      const float f = ex2_approx((m[d] - wm) * c);
      z[d] *= f;
      zl[d] *= f;
      warp_add_exact(z[d], zl[d]);
      if (lane < (int)size) {
        const uint32_t to = peer_addr(&s.stats[turn][d][mine], lane);
        peer_store(to, __float_as_uint(wm), (uint32_t)at);
        peer_store(to + 8, __float_as_uint(z[d]), __float_as_uint(zl[d]));
      }
    }
    cluster_arrive();
    {  // meanwhile the likeliest node to come: its logits (and, if it is known to have no children, the exponentials)
      const uint32_t kids = __ballot_sync(0xffffffffu, kid);
      primed = kids ? w1 + __ffs(kids) - 1 : -1;
      const bool known = L <= w1 + 32 || len + 1 >= p.max_accept;
      primed_race = !greedy && known &&
                    (len + 1 >= p.max_accept || !__any_sync(0xffffffffu, up == primed && w1 + lane > primed && token_ok));
      if (primed >= 0) {
        const T* cx = row_of(p.logits, p.logits_stride, primed);
        const T* cy = row_of(p.draft, p.draft_stride, primed);
        slice.shift = offset16(cx + slice.begin) / (int)sizeof(T);
        if (primed_race) {
          using Pass = PassRace<T, false>;
          prime<Pass>(ring, slice.steps(1), [&](int k, uint8_t* slot) {
            fetch<1, false>(slot, cx, slice, k, V);
            fetch<1, true>(slot + Pass::kNoise, noise, slice, k, V);
          });
        } else if (y) {
          prime<Two>(ring, slice.steps(Two::kGroups), [&](int k, uint8_t* slot) {
            fetch<Two::kGroups, false>(slot, cx, slice, k, V);
            fetch<Two::kGroups, true>(slot + Two::kDraft, cy, slice, k, V);
          });
        } else {
          prime<One>(ring, slice.steps(One::kGroups), [&](int k, uint8_t* slot) {
            fetch<One::kGroups, false>(slot, cx, slice, k, V);
          });
        }
      }
    }
    cluster_wait();
#pragma unroll
    for (int d = 0; d < 2; ++d) {
      if (d == 1 && !y) break;
      st[d] = join_stats(s.stats[turn][d], parts, c);
      bad |= !(st[d].sum > 0.f && st[d].sum < 3e38f);  // no token, NaN or +inf
    }
    turn ^= 1;
    if (bad) break;

    // ---- the children, in ascending order (every warp alike)
    const float ip = 1.f / (st[0].sum + st[0].low), iq = y ? 1.f / (st[1].sum + st[1].low) : 1.f;
    int went = -1, rejected = 0;
    // The residual's mass is a pair. Without a draft weights are relative to the
    // maximum, so that the likeliest token's is 1 and goes exactly; `whole` is the
    // last mass that was formed by adding.
    float mass = y ? 1.f : st[0].sum, mass_low = y ? 0.f : st[0].low, whole = mass + mass_low, gone = 0.f;
#pragma unroll 1
    for (int w0 = w1; w0 < L && went < 0 && len < p.max_accept; w0 += 32) {
      if (w0 > w1) {  // trees of more than 32 nodes
        up = token = -1;
        if (w0 + lane < L) {
          up = p.parents[q0 + w0 + lane];
          token = p.tokens[q0 + w0 + lane];
          if (!greedy) u = p.uniforms[q0 + w0 + lane];
        }
        kid = up == cur && token >= 0 && token < V;
        if (kid) {
          lx = at_token(x, token);
          if (y) ly = at_token(y, token);
        }
      }
      uint32_t kids = __ballot_sync(0xffffffffu, kid);
      if (greedy) {
        const uint32_t hit = __ballot_sync(0xffffffffu, kid && token == st[0].at);
        if (hit) went = w0 + __ffs(hit) - 1;
        continue;
      }
      const float px = ex2_approx((lx - st[0].max) * c) * (y ? ip : 1.f),
                  qx = y ? ex2_approx((ly - st[1].max) * c) * iq : 1.f;
#pragma unroll 1
      for (; kids && went < 0; kids &= kids - 1) {
        const int l = __ffs(kids) - 1;
        const int kt = __shfl_sync(0xffffffffu, token, l);
        const float kp = __shfl_sync(0xffffffffu, px, l), kq = __shfl_sync(0xffffffffu, qx, l);
        const float ku = __shfl_sync(0xffffffffu, u, l);
        float rest = kp;
        if (y) {
          rest = fmaxf(kp - gone * kq, 0.f);
        } else {
          bool again = false;
          for (int e = lane; e < rejected; e += 32) again |= s.gone[e] == kt;
          if (__any_sync(0xffffffffu, again)) rest = 0.f;
        }
        if (ku * (mass + mass_low) * kq < rest) {
          went = w0 + l;
          break;
        }
        ++rejected;
        if (!y) {
          __syncwarp();
          s.gone[rejected - 1] = kt;  // (every thread of the block writes the same)
          __syncwarp();
          add_exact(mass, mass_low, -rest);
          // A difference is good as long as little has gone. A quarter is left of
          // what was added up last with the probability of a quarter.
          if (4.f * (mass + mass_low) >= whole) continue;
        } else {
          gone += mass + mass_low;
        }
        // the residual's mass, if another child is to be tried
        bool more = (kids & (kids - 1)) != 0;
        for (int v0 = w0 + 32; v0 < L && !more; v0 += 32) {
          const int i = v0 + lane;
          const int t = i < L && p.parents[q0 + i] == cur ? p.tokens[q0 + i] : -1;
          more = __any_sync(0xffffffffu, t >= 0 && t < V);
        }
        if (!more) break;
        const float fq = gone * iq;
        float z = 0.f, zl = 0.f;
        const uint64_t neg_x = pack_f32x2(-st[0].max, -st[0].max), neg_y = pack_f32x2(-st[1].max, -st[1].max);
        const uint64_t ipp = pack_f32x2(ip, ip), fqq = pack_f32x2(-fq, -fq);
        slice.shift = offset16(x + slice.begin) / (int)sizeof(T);
        using Pass = PassTwo<T>;
        auto issue = [&](int k, uint8_t* slot) {
          fetch<Pass::kGroups, false>(slot, x, slice, k, V);
          if (y) fetch<Pass::kGroups, true>(slot + Pass::kDraft, y, slice, k, V);
        };
        prime<Pass>(ring, slice.steps(Pass::kGroups), issue);
        stream<Pass>(ring, slice.steps(Pass::kGroups), issue, [&](int k, uint8_t* slot) {
#pragma unroll
          for (int e = 0; e < Pass::kGroups; ++e) {
            Raw<T> a;
            uint64_t w[4];
            take<Pass::kGroups, false>(slot, x, slice, k, e, kNegInf<T>, a);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = weights2(a, i, neg_x, cc);
            uint32_t out = 0;  // which of the eight are tokens of rejected children
            if (y) {
              take<Pass::kGroups, true>(slot + Pass::kDraft, y, slice, k, e, kNegInf<T>, a);
#pragma unroll
              for (int i = 0; i < 4; ++i) w[i] = fma2(w[i], ipp, mul2(weights2(a, i, neg_y, cc), fqq));
            } else {
              const int j = slice.group(slice.step(k, Pass::kGroups), e);
#pragma unroll 1
              for (int i = 0; i < rejected; ++i) {
                const uint32_t at = (uint32_t)(s.gone[i] - j);
                out |= at < 8u ? 1u << at : 0u;
              }
            }
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i)
              sum += (out >> (2 * i) & 1u ? 0.f : fmaxf(lo_f32(w[i]), 0.f)) +
                     (out >> (2 * i + 1) & 1u ? 0.f : fmaxf(hi_f32(w[i]), 0.f));
            add_exact(z, zl, sum);
          }
        });
        warp_add_exact(z, zl);
        if (lane < (int)size) peer_store(peer_addr(&s.sums[turn][mine], lane), __float_as_uint(z), __float_as_uint(zl));
        cluster_sync();
        z = zl = 0.f;
        for (int e = lane; e < parts; e += 32) {
          add_exact(z, zl, s.sums[turn][e].x);
          zl += s.sums[turn][e].y;
        }
        warp_add_exact(z, zl);
        mass = z;
        mass_low = zl;
        whole = z + zl;
        turn ^= 1;
      }
    }

    // ---- no child: the race for the next token
    int out = went >= 0 ? p.tokens[q0 + went] : st[0].at;
    if (went < 0 && !greedy) {
      float fq = gone * iq;
      int lost = y ? 0 : rejected;
      out = 0x7fffffff;
#pragma unroll 1
      for (int tries = 0; tries < 2 && out == 0x7fffffff; ++tries, fq = 0.f, lost = 0) {
        float best = 0.f;
        int best_at = 0x7fffffff;
        const uint64_t neg_x = pack_f32x2(-st[0].max, -st[0].max), neg_y = y ? pack_f32x2(-st[1].max, -st[1].max) : 0;
        const uint64_t ipp = pack_f32x2(ip, ip), fqq = pack_f32x2(-fq, -fq);
        slice.shift = offset16(x + slice.begin) / (int)sizeof(T);
        constexpr int off_e = PassRace<T, true>::kNoise, off_y = PassRace<T, true>::kDraft;
        auto issue = [&](int k, uint8_t* slot) {
          fetch<1, false>(slot, x, slice, k, V);
          fetch<1, true>(slot + off_e, noise, slice, k, V);
          if (fq > 0.f) fetch<1, true>(slot + off_y, y, slice, k, V);
        };
        auto use = [&](int k, uint8_t* slot) {
          const int j = slice.group(slice.step(k, 1), 0);
          Raw<T> a;
          Raw<float> e;
          take<1, false>(slot, x, slice, k, 0, kNegInf<T>, a);
          take<1, true>(slot + off_e, noise, slice, k, 0, 0x3f800000u, e);
          uint64_t rest[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) rest[i] = weights2(a, i, neg_x, cc);
          if (fq > 0.f) {
            take<1, true>(slot + off_y, y, slice, k, 0, kNegInf<T>, a);
#pragma unroll
            for (int i = 0; i < 4; ++i) rest[i] = fma2(weights2(a, i, neg_y, cc), fqq, mul2(rest[i], ipp));
          }
          race8(rest, e, j, s, lost, best, best_at);
        };
        auto run = [&](auto with_draft) {
          using Pass = PassRace<T, decltype(with_draft)::value>;
          prime<Pass>(ring, slice.steps(1), issue);
          stream<Pass>(ring, slice.steps(1), issue, use);
        };
        if (fq > 0.f) run(std::true_type());
        else run(std::false_type());
        uint64_t key = warp_best((uint64_t)__float_as_uint(best) << 32 | (uint32_t)~best_at);
        if (lane < (int)size) peer_store(peer_addr(&s.best[turn][mine], lane), (uint32_t)key, (uint32_t)(key >> 32));
        cluster_sync();
        key = 0;
        for (int e = lane; e < parts; e += 32) key = max(key, s.best[turn][e]);
        key = warp_best(key);
        turn ^= 1;
        if (key >> 32) out = (int)~(uint32_t)key;
      }
    }
    if (threadIdx.x == 0) {
      s.out[len - 1] = out;
      s.node[len - 1] = st[0];
      if (went >= 0) s.path[len] = went;
    }
    if (went < 0) {
      next = out < V ? out : -1;
      bad = next < 0;
      break;
    }
    cur = went;
    ++len;
  }
  asm volatile("cp.async.wait_all;" ::: "memory");  // none in flight when the block ends
  if (rank != 0) return;
  __syncthreads();
  for (int i = threadIdx.x; i < p.max_accept; i += kThreads) {
    const int at = i > 0 && i < len ? s.path[i] : 0;
    p.path[(size_t)r * p.max_accept + i] = i < len ? at : -1;
    if (p.logprobs) {
      float v = 0.f;
      if (i < len && bad && i == len - 1) {
        v = __int_as_float(0x7fffffff);
      } else if (i < len) {
        const Stats o = s.node[i];
        const float l = at_token(static_cast<const T*>(p.logits) + (size_t)(q0 + at) * p.logits_stride, s.out[i]);
        v = (l - o.max) / div - (logf(o.sum) + o.low / o.sum);
      }
      p.logprobs[(size_t)r * p.max_accept + i] = v;
    }
  }
  if (threadIdx.x == 0) {
    if (bad && walks) bits |= kStatusBadValues;
    if (bits) atomicOr(p.status, bits);
    p.path_len[r] = len;
    p.next[r] = next;
  }
}

}  // namespace

cudaError_t launch_verify(const VerifyParams& p, bool fp32, int sms, cudaStream_t stream) {
  // blocks a row: as many as make four per SM, of which three fit at once and the
  // others begin as rows end (64 greedy rows of 131072 logits: 8 blocks a row 42 us,
  // 4 50, 2 62, 1 89), four at least (384 sampled fp32 rows: 2 blocks a row 152 us,
  // 4 144, 8 166), but half a group of logits for every thread (2 rows of 16000: 8
  // blocks a row 17 us, 4 19, 2 21; of 4000: 2 17, 1 19)
  int size = 1;
  while (size < kMaxCluster && (size < 4 || 2 * size * p.num_seqs <= 4 * sms) && size * 8 * kThreads <= p.vocab) size *= 2;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(size * p.num_seqs);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kRingBytes;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = size;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, fp32 ? verify_kernel<float> : verify_kernel<__nv_bfloat16>, p);
}

cudaError_t prepare_verify_kernels() {
  const cudaError_t e = cudaFuncSetAttribute(verify_kernel<float>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                             kRingBytes);
  if (e != cudaSuccess) return e;
  return cudaFuncSetAttribute(verify_kernel<__nv_bfloat16>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              kRingBytes);
}

}  // namespace mcpu
