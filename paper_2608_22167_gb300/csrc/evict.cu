// Eviction by accumulated attention weight (mcpu_evict_kv).
//
// One block per (layer, row, kv head). Of the N = n - first - last middle slots
// the K = budget - first - last with the highest weight stay: the K-th largest
// is found by a radix select over the weights' bits (8 at a time), and among
// the slots that equal it the lowest are taken. Kept slots below
// inner = budget - last stay where they are; there are as many holes below it
// as kept slots past it, and the i-th of these moves into the i-th hole. The
// last ones follow as one shift towards the front. No list of slots is ever
// stored: both regions are walked in step, a block of slots at a time.
#include "keep.cuh"

namespace mcpu {

namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kQueue = 2 * kThreads;
constexpr int kRowVecs = 2 * kRowBytes / 16;  // 16-byte pieces of a slot's K and V

// Unsigned order of the weights: NaN lowest, the two zeros equal.
__device__ __forceinline__ uint32_t order(float w) {
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

struct EvictSmem {
  uint32_t hist[256];
  int32_t scan[kWarps];
  int32_t total;
  uint32_t prefix;
  int32_t want;
  int32_t bad;
  int32_t src[kQueue], dst[kQueue];
};

// Exclusive prefix sum of a 0/1 flag over the block, and its total.
__device__ __forceinline__ int block_rank(bool flag, EvictSmem& s, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t vote = __ballot_sync(0xffffffffu, flag);
  if (lane == 0) s.scan[warp] = __popc(vote);
  __syncthreads();
  int before = 0, all = 0;
  for (int w = 0; w < kWarps; ++w) {
    const int n = s.scan[w];
    before += w < warp ? n : 0;
    all += n;
  }
  __syncthreads();
  *total = all;
  return before + __popc(vote & ((1u << lane) - 1u));
}

__global__ void __launch_bounds__(kThreads) evict_kernel(const EvictParams p, const __grid_constant__ PoolPtrs pools) {
  __shared__ EvictSmem s;
  const int h = blockIdx.x, r = blockIdx.y, m = blockIdx.z, Hkv = p.num_kv_heads;
  const int n = p.seq_lens[r];
  const bool speaks = h == 0 && m == 0 && threadIdx.x == 0;
  const int32_t* table = p.block_table + (size_t)r * p.max_pages;
  bool cut = n > p.limit;
  int32_t bits = 0;
  if (n < 0 || n > p.max_pages * kPage || n > p.max_slots) {
    bits = kStatusBadLengths;
  } else if (cut) {
    if (threadIdx.x == 0) s.bad = 0;
    __syncthreads();
    const int end = (n + kPage - 1) / kPage, mine = p.first < p.budget ? (p.budget + kPage - 1) / kPage : 0;
    int32_t bad = 0;
    for (int j = p.first / kPage + threadIdx.x; j < end; j += kThreads) {
      const int page = table[j];
      if (page < 0 || page >= p.num_pages) bad |= kStatusBadPage;
      else if (p.refs && j < mine && p.refs[page] > 0) bad |= kStatusUnsupportedRow;
    }
    if (bad) atomicOr(&s.bad, bad);
    __syncthreads();
    bits = s.bad;
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
  if (nw != w)
    for (int j = threadIdx.x; j < (cut ? inner : n); j += kThreads) nw[j] = w[j];
  if (!cut) return;
  const int first = p.first, end = n - p.last, K = inner - first;

  // ---- the K-th largest weight of the middle: its order, and how many that equal it stay
  if (threadIdx.x == 0) {
    s.prefix = 0;
    s.want = K;
  }
  __syncthreads();
  if (K > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = threadIdx.x; i < 256; i += kThreads) s.hist[i] = 0;
      __syncthreads();
      const uint32_t prefix = s.prefix;
      for (int j = first + threadIdx.x; j < end; j += kThreads) {
        const uint32_t u = order(w[j]);
        if (shift == 24 || (u >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&s.hist[(u >> shift) & 255], 1u);
      }
      __syncthreads();
      if (threadIdx.x == 0) {
        int want = s.want, b = 255;
        for (; b > 0 && (int)s.hist[b] < want; --b) want -= s.hist[b];
        s.prefix = prefix | ((uint32_t)b << shift);
        s.want = want;
      }
      __syncthreads();
    }
  }
  const uint32_t cutoff = s.prefix;
  const int ties = s.want;  // of the slots equal to the cutoff so many stay, the lowest
  __syncthreads();

  // ---- kept slots at or past inner fill the holes before it, in order
  int eq_a = 0;  // slots equal to the cutoff before inner
  {
    int mine = 0;
    for (int j = first + threadIdx.x; j < inner; j += kThreads) mine += order(w[j]) == cutoff;
    for (int o = 16; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
    if ((threadIdx.x & 31) == 0) s.scan[threadIdx.x >> 5] = mine;
    __syncthreads();
    for (int i = 0; i < kWarps; ++i) eq_a += s.scan[i];
    __syncthreads();
  }
  const uint8_t* row_pools[2] = {pools.p[m], pools.p[p.num_layers + m]};
  auto vec = [&](int slot, int e) {  // 16-byte piece e of a slot's K and V
    const size_t row = ((size_t)table[slot / kPage] * Hkv + h) * kPage + slot % kPage;
    return reinterpret_cast<uint4*>(const_cast<uint8_t*>(row_pools[e >> 3]) + row * kRowBytes) + (e & 7);
  };
  int ja = first, jb = inner, seen_a = 0, seen_b = eq_a, have_a = 0, have_b = 0, done = 0;
  while (true) {
    // the queues hold less than kThreads entries each here, or their region is at its end
    while (have_b - done < kThreads && jb < end) {
      const int j = jb + threadIdx.x;
      const uint32_t u = j < end ? order(w[j]) : 0u;
      const bool eq = K > 0 && j < end && u == cutoff;
      int all;
      const int rank = seen_b + block_rank(eq, s, &all);
      seen_b += all;
      const bool keep = K > 0 && j < end && (u > cutoff || (eq && rank < ties));
      const int slot = have_b + block_rank(keep, s, &all);
      if (keep) s.src[slot % kQueue] = j;
      have_b += all;
      jb += kThreads;
    }
    while (have_a - done < kThreads && ja < inner) {
      const int j = ja + threadIdx.x;
      const uint32_t u = j < inner ? order(w[j]) : 0u;
      const bool eq = j < inner && u == cutoff;
      int all;
      const int rank = seen_a + block_rank(eq, s, &all);
      seen_a += all;
      const bool hole = j < inner && !(u > cutoff || (eq && rank < ties));
      const int slot = have_a + block_rank(hole, s, &all);
      if (hole) s.dst[slot % kQueue] = j;
      have_a += all;
      ja += kThreads;
    }
    __syncthreads();
    const int count = min(min(have_a, have_b) - done, kThreads);
    if (count <= 0) break;
    for (int e = threadIdx.x; e < count * kRowVecs; e += kThreads) {
      const int i = (done + e / kRowVecs) % kQueue;
      *vec(s.dst[i], e % kRowVecs) = *vec(s.src[i], e % kRowVecs);
    }
    for (int e = threadIdx.x; e < count; e += kThreads) nw[s.dst[(done + e) % kQueue]] = w[s.src[(done + e) % kQueue]];
    done += count;
    __syncthreads();
  }
  // ---- the last ones: towards the front, so a piece of them at a time, read before it is written
  constexpr int kHeld = 4;
  for (int i0 = 0; i0 < p.last; i0 += kHeld * kThreads / kRowVecs) {
    const int count = min(p.last - i0, kHeld * kThreads / kRowVecs);
    uint4 held[kHeld];
    float held_w = 0.f;
#pragma unroll
    for (int k = 0; k < kHeld; ++k) {
      const int e = threadIdx.x + k * kThreads;
      if (e < count * kRowVecs) held[k] = *vec(end + i0 + e / kRowVecs, e % kRowVecs);
    }
    if (threadIdx.x < count) held_w = w[end + i0 + threadIdx.x];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kHeld; ++k) {
      const int e = threadIdx.x + k * kThreads;
      if (e < count * kRowVecs) *vec(inner + i0 + e / kRowVecs, e % kRowVecs) = held[k];
    }
    if (threadIdx.x < count) nw[inner + i0 + threadIdx.x] = held_w;
    __syncthreads();
  }
}

}  // namespace

cudaError_t launch_evict(const EvictParams& p, const PoolPtrs& pools, int sms, cudaStream_t stream) {
  (void)sms;
  LaunchCfg lc(dim3(p.num_kv_heads, p.num_seqs, p.num_layers > 0 ? p.num_layers : 1), dim3(kThreads), 0, stream, false);
  return cudaLaunchKernelEx(&lc.cfg, evict_kernel, p, pools);
}

}  // namespace mcpu
