// Verification of drafted tokens (mcpu_verify_tree).
//
// At each node of the walk, with p = softmax(l / T) and (if given) q of the
// draft, the residual after rejecting k children of masses m_0 = 1, m_1 .. is
//   rest(y) = max(p(y) - M q(y), 0),  M = m_0 + .. + m_{k-1},  m_k = sum_y rest(y)
// because max(max(a, 0) - b, 0) = max(a - b, 0) for b >= 0: only M is carried,
// no vector. The next token is argmax_y rest(y) / e_y, which for exponential e
// is y with probability rest(y) / m.
//
// A cluster of blocks walks a row's tree, a slice of the vocabulary each; only
// the nodes that the walk visits are read. A node costs one pass over its
// logits (maximum, its place and the sum together), a rejection with draft
// probabilities one more, the row's end one with the exponentials; what was
// read before comes from L2 then. After a pass every warp hands its result to
// all blocks of the cluster (distributed shared memory), and behind one cluster
// barrier every warp joins them all in the same order: all take the same
// decisions, and nothing is sent back.
//
// Everything is fp32. Sums are pairs: 8 terms at a time, each group added by an
// exact two-sum (a plain chain of additions loses 1e-6 of a peaked
// distribution's tail; so does a maximum times log2(e) taken out of the
// difference). Exponentials by ex2.approx (2^-22).
#include "keep.cuh"

namespace mcpu {

namespace {

constexpr int kMaxThreads = 512, kMinThreads = 256, kMaxWarps = kMaxThreads / 32, kMaxCluster = 8;
constexpr int kMaxNodes = MCPU_MAX_TREE_NODES;
constexpr float kLowest = -3.402823466e38f;  // a finite maximum to begin with: -inf logits weigh nothing against it
constexpr float kLog2e = 1.4426950408889634f, kLog2eLow = 1.925963033500e-08f;  // log2(e) = the sum of both

struct Stats {  // of a distribution: maximum, the lowest token that has it, sum of e^((l - max) / T)
  float max;
  int32_t at;
  float sum, low;  // the sum of both
};

struct VerifySmem {
  Stats stats[2][2][kMaxCluster * kMaxWarps];  // [turn][target, draft][warp of the cluster]
  float2 sums[2][kMaxCluster * kMaxWarps];
  uint64_t best[2][kMaxCluster * kMaxWarps];
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

// The slice of the vocabulary that a block has; thread t's group k is the eight
// values from begin + 8 (k threads + t) on.
struct Slice {
  int begin, end, vocab;
  __device__ __forceinline__ int first(int k) const { return begin + 8 * (k * (int)blockDim.x + (int)threadIdx.x); }
  __device__ __forceinline__ int groups() const {
    return (end - begin + 8 * (int)blockDim.x - 1) / (8 * (int)blockDim.x);
  }
};

// The eight values of a row from `at` on; `fill` (as bits of one) past the end.
// kWhole: every row starts at 16 bytes and its length is a multiple of 8. Else
// the row starts anywhere: one more vector, and shifts by the row's offset (the
// same for all threads); where that vector would leave the row, one by one.
template <bool kWhole, typename T>
__device__ __forceinline__ void load8(const T* row, int at, const Slice& s, uint32_t fill, Raw<T>& r) {
  constexpr int kWords = Raw<T>::kWords;
  const uint32_t two = sizeof(T) == 4 ? fill : fill << 16 | fill;
  if (kWhole) {
#pragma unroll
    for (int k = 0; k < kWords / 4; ++k) {
      uint4 x = make_uint4(two, two, two, two);
      if (at < s.end) x = __ldcg(reinterpret_cast<const uint4*>(row + at) + k);
      r.w[4 * k] = x.x, r.w[4 * k + 1] = x.y, r.w[4 * k + 2] = x.z, r.w[4 * k + 3] = x.w;
    }
    return;
  }
  const uint32_t off = (uint32_t)(reinterpret_cast<uintptr_t>(row + at) & 15);
  const bool inside = at + 8 + (off ? (int)((16 - off) / sizeof(T)) : 0) <= s.vocab && (off == 0 || at > 0);
  if (at < s.end && inside) {
    const uint4* v = reinterpret_cast<const uint4*>(reinterpret_cast<const uint8_t*>(row + at) - off);
    uint32_t w[kWords + 4];
#pragma unroll
    for (int k = 0; k <= kWords / 4; ++k) {
      if (k == kWords / 4 && off == 0) continue;
      const uint4 x = v[k];  // (through L1: the neighbour's vector too)
      w[4 * k] = x.x, w[4 * k + 1] = x.y, w[4 * k + 2] = x.z, w[4 * k + 3] = x.w;
    }
    // words first, then the half word
#pragma unroll
    for (int k = 0; k < kWords + 2; ++k) w[k] = off & 8 ? w[k + 2] : w[k];
#pragma unroll
    for (int k = 0; k < kWords + 1; ++k) w[k] = off & 4 ? w[k + 1] : w[k];
#pragma unroll
    for (int k = 0; k < kWords; ++k) r.w[k] = sizeof(T) == 2 && off & 2 ? __funnelshift_r(w[k], w[k + 1], 16) : w[k];
    return;
  }
#pragma unroll
  for (int k = 0; k < kWords; ++k) r.w[k] = two;
  if (at >= s.end) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (at + i >= s.vocab) break;
    if (sizeof(T) == 4) r.w[i] = reinterpret_cast<const uint32_t*>(row)[at + i];
    else if (i & 1) r.w[i >> 1] = (r.w[i >> 1] & 0xffffu) | (uint32_t)reinterpret_cast<const uint16_t*>(row)[at + i] << 16;
    else r.w[i >> 1] = (r.w[i >> 1] & 0xffff0000u) | reinterpret_cast<const uint16_t*>(row)[at + i];
  }
}

// A slice of a row into L2, ahead of its use.
template <typename T>
__device__ __forceinline__ void prefetch_slice(const T* row, const Slice& s) {
  for (int i = s.begin + threadIdx.x * (128 / (int)sizeof(T)); i < s.end; i += blockDim.x * (128 / (int)sizeof(T)))
    asm volatile("prefetch.global.L2 [%0];" ::"l"(row + i));
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
__device__ __forceinline__ void warp_max(float& m, int& at) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float om = __shfl_xor_sync(0xffffffffu, m, o);
    const int oat = __shfl_xor_sync(0xffffffffu, at, o);
    if (om > m || (om == m && oat < at)) m = om, at = oat;
  }
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

template <typename T, bool kWhole>
__global__ void __launch_bounds__(kMaxThreads, 1) verify_kernel(const VerifyParams p, int ahead) {
  constexpr int kFlight = 8 / sizeof(T);               // groups of a row loaded together
  constexpr int kRace = (kWhole ? 8 : 4) / sizeof(T);  // and of the two or three rows of the last passes
  __shared__ VerifySmem s;
  cluster_arrive();  // (every block of the cluster is there before the first store into its memory)
  grid_dep_launch();
  grid_dep_wait();
  const uint32_t rank = cluster_rank(), size = cluster_size();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  const int parts = (int)size * warps, mine = (int)rank * warps + warp;
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
  slice.vocab = V;
  slice.begin = min(V, (int)rank * per);
  slice.end = min(V, slice.begin + per);
  const int n = slice.groups();
  const float* noise = greedy ? nullptr : p.noise + (size_t)r * p.noise_stride;
  uint32_t turn = 0;  // of the exchange buffers
  cluster_wait();
  if (walks && !bad && !greedy && ahead) prefetch_slice(noise, slice);

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
    // ---- maximum and sum of the node's distributions
    Stats st[2];
    float lx = 0.f, ly = 0.f;  // the child's own logits
    bool kid = false;
#pragma unroll 1
    for (int d = 0; d < (y ? 2 : 1); ++d) {
      const T* row = d ? y : x;
      float m = kLowest, z = 0.f, zl = 0.f;
      int at = 0x7fffffff;
      auto load = [&](Raw<T>(&v)[kFlight], int k0) {
#pragma unroll
        for (int e = 0; e < kFlight; ++e) load8<kWhole>(row, slice.first(k0 + e), slice, kNegInf<T>, v[e]);
      };
      auto add = [&](const Raw<T>(&v)[kFlight], int k0) {
        float tops[kFlight], top = -INFINITY;
#pragma unroll
        for (int e = 0; e < kFlight; ++e) {
          tops[e] = fmaxf(v[e].get(0), v[e].get(1));
#pragma unroll
          for (int i = 2; i < 8; i += 2) tops[e] = fmax3(tops[e], v[e].get(i), v[e].get(i + 1));
          top = fmaxf(top, tops[e]);
        }
        if (top > m) {
          const float f = ex2_approx((m - top) * c);
          z *= f;
          zl *= f;
          m = top;
          if (greedy) {  // the lowest token that has it
#pragma unroll
            for (int e = kFlight - 1; e >= 0; --e)
              if (tops[e] == top) {
#pragma unroll
                for (int i = 7; i >= 0; --i)
                  if (v[e].get(i) == top) at = slice.first(k0 + e) + i;
              }
          }
        }
        const uint64_t neg = pack_f32x2(-m, -m);
#pragma unroll
        for (int e = 0; e < kFlight; ++e) {
          uint64_t sum = weights2(v[e], 0, neg, cc);
#pragma unroll
          for (int i = 1; i < 4; ++i) sum = add2(sum, weights2(v[e], i, neg, cc));
          add_exact(z, zl, lo_f32(sum) + hi_f32(sum));
        }
      };
      // one flight's arithmetic while the next one's loads are on their way
      Raw<T> va[kFlight], vb[kFlight];
      load(va, 0);
#pragma unroll 1
      for (int k0 = 0; k0 < n; k0 += 2 * kFlight) {
        load(vb, k0 + kFlight);
        add(va, k0);
        if (k0 + kFlight >= n) break;
        load(va, k0 + 2 * kFlight);
        add(vb, k0 + kFlight);
      }
      if (d == 0) {
        kid = up == cur && w1 + lane > cur && token >= 0 && token < V && len < p.max_accept;
        const uint32_t kids = __ballot_sync(0xffffffffu, kid);
        if (kid) {
          lx = at_token(x, token);
          if (y) ly = at_token(y, token);
        }
        if (ahead && kids) {  // the likeliest node to come
          const size_t child = q0 + w1 + __ffs(kids) - 1;
          prefetch_slice(static_cast<const T*>(p.logits) + child * p.logits_stride, slice);
          if (y) prefetch_slice(static_cast<const T*>(p.draft) + child * p.draft_stride, slice);
        }
      }
      float wm = m;
      warp_max(wm, at);
      const float f = ex2_approx((m - wm) * c);
      z *= f;
      zl *= f;
      warp_add_exact(z, zl);
      if (lane < (int)size) {
        const uint32_t to = peer_addr(&s.stats[turn][d][mine], lane);
        peer_store(to, __float_as_uint(wm), (uint32_t)at);
        peer_store(to + 8, __float_as_uint(z), __float_as_uint(zl));
      }
    }
    cluster_sync();
#pragma unroll
    for (int d = 0; d < 2; ++d) {
      if (d == 1 && !y) break;
      float m = kLowest, z = 0.f, zl = 0.f;
      int at = 0x7fffffff;
      for (int i = lane; i < parts; i += 32) {
        const Stats o = s.stats[turn][d][i];
        if (o.max > m || (o.max == m && o.at < at)) m = o.max, at = o.at;
      }
      warp_max(m, at);
      for (int i = lane; i < parts; i += 32) {
        const Stats o = s.stats[turn][d][i];
        const float f = ex2_approx((o.max - m) * c);
        add_exact(z, zl, o.sum * f);
        zl += o.low * f;
      }
      warp_add_exact(z, zl);
      st[d] = Stats{m, at, z, zl};
      bad |= !(z > 0.f && z < 3e38f);  // no token, NaN or +inf
    }
    turn ^= 1;
    if (bad) break;

    // ---- the children, in ascending order (every warp alike)
    const float ip = 1.f / (st[0].sum + st[0].low), iq = y ? 1.f / (st[1].sum + st[1].low) : 1.f;
    int went = -1, rejected = 0;
    float mass = 1.f, gone = 0.f;
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
      const float px = ex2_approx((lx - st[0].max) * c) * ip, qx = y ? ex2_approx((ly - st[1].max) * c) * iq : 1.f;
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
        if (ku * mass * kq < rest) {
          went = w0 + l;
          break;
        }
        ++rejected;
        if (!y) {
          mass = fmaxf(mass - rest, 0.f);
          __syncwarp();
          s.gone[rejected - 1] = kt;  // (every thread of the block writes the same)
          __syncwarp();
          continue;
        }
        gone += mass;
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
#pragma unroll 1
        for (int k0 = 0; k0 < n; k0 += kRace) {
          Raw<T> a[kRace], b[kRace];
#pragma unroll
          for (int e = 0; e < kRace; ++e) {
            load8<kWhole>(x, slice.first(k0 + e), slice, kNegInf<T>, a[e]);
            load8<kWhole>(y, slice.first(k0 + e), slice, kNegInf<T>, b[e]);
          }
#pragma unroll
          for (int e = 0; e < kRace; ++e) {
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint64_t w = fma2(weights2(a[e], i, neg_x, cc), ipp, mul2(weights2(b[e], i, neg_y, cc), fqq));
              sum += fmaxf(lo_f32(w), 0.f) + fmaxf(hi_f32(w), 0.f);
            }
            add_exact(z, zl, sum);
          }
        }
        warp_add_exact(z, zl);
        if (lane < (int)size) peer_store(peer_addr(&s.sums[turn][mine], lane), __float_as_uint(z), __float_as_uint(zl));
        cluster_sync();
        z = zl = 0.f;
        for (int e = lane; e < parts; e += 32) {
          add_exact(z, zl, s.sums[turn][e].x);
          zl += s.sums[turn][e].y;
        }
        warp_add_exact(z, zl);
        mass = z + zl;
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
#pragma unroll 1
        for (int k0 = 0; k0 < n; k0 += kRace) {
          Raw<T> a[kRace], b[kRace];
          Raw<float> e[kRace];
#pragma unroll
          for (int k = 0; k < kRace; ++k) {
            load8<kWhole>(noise, slice.first(k0 + k), slice, 0x3f800000u, e[k]);
            load8<kWhole>(x, slice.first(k0 + k), slice, kNegInf<T>, a[k]);
            if (fq > 0.f) load8<kWhole>(y, slice.first(k0 + k), slice, kNegInf<T>, b[k]);
          }
#pragma unroll
          for (int k = 0; k < kRace; ++k) {
            float v[8], top = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              uint64_t w = mul2(weights2(a[k], i, neg_x, cc), ipp);
              if (fq > 0.f) w = fma2(weights2(b[k], i, neg_y, cc), fqq, w);
              v[2 * i] = __fdividef(lo_f32(w), e[k].get(2 * i));
              v[2 * i + 1] = __fdividef(hi_f32(w), e[k].get(2 * i + 1));
            }
            const int at = slice.first(k0 + k);
            for (int j = 0; j < lost; ++j) {  // tokens of rejected children do not take part
              const int i = s.gone[j] - at;
              if (i >= 0 && i < 8) {
#pragma unroll
                for (int d = 0; d < 8; ++d) v[d] = d == i ? 0.f : v[d];
              }
            }
#pragma unroll
            for (int i = 0; i < 8; i += 2) top = fmax3(top, v[i], v[i + 1]);
            if (top > best) {
              best = top;
#pragma unroll
              for (int i = 7; i >= 0; --i) best_at = v[i] == top ? at + i : best_at;
            }
          }
        }
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
  if (rank != 0) return;
  __syncthreads();
  for (int i = threadIdx.x; i < p.max_accept; i += blockDim.x) {
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
  // up to one block per SM large ones, several a row; more rows share the SMs in smaller ones
  int size = 1, threads = p.num_seqs <= sms ? kMaxThreads : p.num_seqs <= 2 * sms ? kMaxThreads / 2 : kMinThreads;
  while (size < kMaxCluster && 2 * size * p.num_seqs <= sms && 2 * size * kMinThreads * 8 <= p.vocab) size *= 2;
  while (threads > kMinThreads && size * threads * 4 > p.vocab) threads /= 2;
  const size_t bytes = fp32 ? 4 : 2;
  auto whole = [&](const void* q, int64_t stride, size_t b) {
    return !q || (reinterpret_cast<uintptr_t>(q) % 16 == 0 && stride * b % 16 == 0);
  };
  const bool aligned = p.vocab % 8 == 0 && whole(p.logits, p.logits_stride, bytes) &&
                   whole(p.draft, p.draft_stride, bytes) && whole(p.noise, p.noise_stride, 4);
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(size * p.num_seqs);
  cfg.blockDim = dim3(threads);
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = size;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  const int ahead = p.num_seqs <= sms;
  if (fp32)
    return cudaLaunchKernelEx(&cfg, aligned ? verify_kernel<float, true> : verify_kernel<float, false>, p, ahead);
  return cudaLaunchKernelEx(&cfg, aligned ? verify_kernel<__nv_bfloat16, true> : verify_kernel<__nv_bfloat16, false>, p, ahead);
}

}  // namespace mcpu
