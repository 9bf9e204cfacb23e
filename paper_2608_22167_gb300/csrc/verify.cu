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
// Sums: 8 terms at a time in fp32, each group added to an fp32 pair by an exact
// two-sum, joined in fp64 (a plain chain of fp32 additions loses 1e-6 of a peaked
// distribution's tail). Exponentials by ex2.approx (2^-22).
#include "keep.cuh"

namespace mcpu {

namespace {

constexpr int kMaxThreads = 512, kMaxWarps = kMaxThreads / 32, kMaxCluster = 8;
constexpr int kMaxNodes = MCPU_MAX_TREE_NODES;
constexpr float kLowest = -3.402823466e38f;  // a finite maximum to begin with: -inf logits weigh nothing against it

struct Stats {  // of a distribution: maximum, the lowest token that has it, sum of e^((l - max) / T)
  float max;
  int32_t at;
  double sum;
};

struct VerifySmem {
  Stats stats[2][2][kMaxCluster * kMaxWarps];  // [turn][target, draft][warp of the cluster]
  double sums[2][kMaxCluster * kMaxWarps];
  uint64_t best[2][kMaxCluster * kMaxWarps];
  int32_t parents[kMaxNodes], tokens[kMaxNodes];
  float uniforms[kMaxNodes];
  int32_t gone[kMaxNodes];                            // tokens of the rejected children of the node
  int32_t path[kMaxNodes];
  double log_arg[kMaxNodes], log_sum[kMaxNodes];      // log p of what was emitted: the difference of arg and log sum
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
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Address of a shared-memory object in block `rank` of the cluster.
__device__ __forceinline__ uint32_t peer_addr(const void* p, uint32_t rank) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_addr(p)), "r"(rank));
  return a;
}
__device__ __forceinline__ void peer_store(uint32_t addr, uint64_t v) {
  asm volatile("st.shared::cluster.b64 [%0], %1;" ::"r"(addr), "l"(v) : "memory");
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

// The slice of the vocabulary that a block has, and how its threads share it:
// eight neighbouring values a thread where all rows in use start at 16 bytes
// (step 1), else eight a block apart, one coalesced load each (rows of an odd
// number of tokens start anywhere).
struct Slice {
  int begin, end, step;
  __device__ __forceinline__ int first(int k) const {  // first value of the thread's group k
    return begin + (step == 1 ? 8 * (k * (int)blockDim.x + (int)threadIdx.x) : 8 * k * (int)blockDim.x + (int)threadIdx.x);
  }
  __device__ __forceinline__ int groups() const {
    return (end - begin + 8 * (int)blockDim.x - 1) / (8 * (int)blockDim.x);
  }
};

// Values at, at + step, .. of a row, `fill` (as bits of one) from `end` on.
template <typename T>
__device__ __forceinline__ void load8(const T* row, int at, const Slice& s, uint32_t fill, Raw<T>& r) {
  if (s.step == 1 && at + 8 <= s.end) {
#pragma unroll
    for (int k = 0; k < Raw<T>::kWords / 4; ++k) {
      const uint4 x = __ldcg(reinterpret_cast<const uint4*>(row + at) + k);
      r.w[4 * k] = x.x, r.w[4 * k + 1] = x.y, r.w[4 * k + 2] = x.z, r.w[4 * k + 3] = x.w;
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int j = at + i * s.step;
    uint32_t v = fill;
    if (j < s.end) v = sizeof(T) == 4 ? __ldcg(reinterpret_cast<const uint32_t*>(row) + j)
                                      : __ldcg(reinterpret_cast<const uint16_t*>(row) + j);
    if (sizeof(T) == 4) r.w[i] = v;
    else if (i & 1) r.w[i >> 1] |= v << 16;
    else r.w[i >> 1] = v;
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

// Calls f(first value, values of a) for this thread's groups of eight, as many
// as 64 bytes loaded together.
template <typename T, typename F>
__device__ __forceinline__ void for_groups(const T* a, const Slice& s, F f) {
  constexpr int kFlight = 8 / sizeof(T);
  const int n = s.groups();
  for (int k0 = 0; k0 < n; k0 += kFlight) {
    Raw<T> r[kFlight];
#pragma unroll
    for (int e = 0; e < kFlight; ++e) load8(a, k0 + e < n ? s.first(k0 + e) : s.end, s, kNegInf<T>, r[e]);
#pragma unroll
    for (int e = 0; e < kFlight; ++e)
      if (k0 + e < n) f(s.first(k0 + e), r[e]);
  }
}

template <typename T>
__global__ void __launch_bounds__(kMaxThreads, 2) verify_kernel(const VerifyParams p) {
  __shared__ VerifySmem s;
  grid_dep_launch();
  grid_dep_wait();
  const uint32_t rank = cluster_rank(), size = cluster_size();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  const int parts = (int)size * warps, mine = (int)rank * warps + warp;
  const int r = blockIdx.x / size, V = p.vocab;
  const int q0 = p.qsl[r], L = p.qsl[r + 1] - q0;
  int32_t bits = 0;
  if (p.qsl[0] != 0 || p.qsl[p.num_seqs] != p.total_q || q0 < 0 || L < 0 || L > p.total_q - q0) bits = kStatusBadLengths;
  else if (L > kMaxNodes) bits = kStatusUnsupportedRow;
  const float heat = p.temperature ? p.temperature[r] : 0.f;
  const bool greedy = heat == 0.f;
  bool bad = !greedy && !(heat >= 1e-20f && heat <= 1e20f);
  const bool walks = !bits && L > 0;
  int cur = 0, len = walks ? 1 : 0, next = -1;
  if (walks && !bad) {  // the same in all blocks of the cluster
    for (int i = threadIdx.x; i < L; i += blockDim.x) {
      s.parents[i] = p.parents[q0 + i];
      s.tokens[i] = p.tokens[q0 + i];
      s.uniforms[i] = greedy ? 0.f : p.uniforms[q0 + i];
    }
    if (threadIdx.x == 0) s.path[0] = 0;
    // before the first store into another block's memory all have to be there
    cluster_sync();
  }
  const double T_inv = greedy ? 1.0 : 1.0 / (double)heat;
  const float c = (float)(1.4426950408889634 * T_inv);
  const int per = (V + 8 * (int)size - 1) / (8 * (int)size) * 8;
  Slice slice;
  slice.begin = min(V, (int)rank * per);
  slice.end = min(V, slice.begin + per);
  uint32_t turn = 0;  // of the exchange buffers
  const float* noise = greedy ? nullptr : p.noise + (size_t)r * p.noise_stride;
  auto whole = [](const void* row) { return (reinterpret_cast<uintptr_t>(row) & 15) == 0; };

  // e^((l - max) / T) relative to 2 ulp, for single tokens
  auto weight = [&](const T* row, const Stats& st, int token) -> double {
    const double x = ((double)at_token(row, token) - (double)st.max) * T_inv;
    const float hi = (float)fmax(x, -200.0);
    return (double)expf(hi) * (1.0 + (fmax(x, -200.0) - (double)hi));
  };

  while (walks && !bad) {
    const T* x = static_cast<const T*>(p.logits) + (size_t)(q0 + cur) * p.logits_stride;
    const T* y = p.draft && !greedy ? static_cast<const T*>(p.draft) + (size_t)(q0 + cur) * p.draft_stride : nullptr;
    slice.step = whole(x) && whole(y) && whole(noise) ? 1 : (int)blockDim.x;
    // ---- maximum and sum of the node's distributions
    Stats st[2];
    const int dists = y ? 2 : 1;
#pragma unroll 1
    for (int d = 0; d < dists; ++d) {
      float m = kLowest, z = 0.f, zl = 0.f;
      int at = 0x7fffffff;
      for_groups(d ? y : x, slice, [&](int j, const Raw<T>& v) {
        float top = v.get(0);
#pragma unroll
        for (int i = 1; i < 8; ++i) top = fmaxf(top, v.get(i));
        if (top > m || (top == m && at == 0x7fffffff)) {
          const float f = exp2f((m - top) * c);
          z *= f;
          zl *= f;
          m = top;
#pragma unroll
          for (int i = 7; i >= 0; --i)
            if (v.get(i) == top) at = j + i * slice.step;
        }
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += ex2_approx((v.get(i) - m) * c);
        add_exact(z, zl, sum);
      });
      float wm = m;
      int wat = at;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        const float om = __shfl_xor_sync(0xffffffffu, wm, o);
        const int oat = __shfl_xor_sync(0xffffffffu, wat, o);
        if (om > wm || (om == wm && oat < wat)) wm = om, wat = oat;
      }
      double wz = ((double)z + (double)zl) * (double)exp2f((m - wm) * c);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) wz += __shfl_xor_sync(0xffffffffu, wz, o);
      if (lane < (int)size) {
        const uint32_t to = peer_addr(&s.stats[turn][d][mine], lane);
        peer_store(to, (uint64_t)__float_as_uint(wm) | (uint64_t)(uint32_t)wat << 32);
        peer_store(to + 8, (uint64_t)__double_as_longlong(wz));
      }
    }
    cluster_sync();
#pragma unroll 1
    for (int d = 0; d < dists; ++d) {
      Stats b{kLowest, 0x7fffffff, 0.0};
      for (int i = lane; i < parts; i += 32) {
        const Stats o = s.stats[turn][d][i];
        if (o.max > b.max || (o.max == b.max && o.at < b.at)) b.max = o.max, b.at = o.at;
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        const float om = __shfl_xor_sync(0xffffffffu, b.max, o);
        const int oat = __shfl_xor_sync(0xffffffffu, b.at, o);
        if (om > b.max || (om == b.max && oat < b.at)) b.max = om, b.at = oat;
      }
      for (int i = lane; i < parts; i += 32) {
        const Stats o = s.stats[turn][d][i];
        b.sum += o.sum * (double)exp2f((o.max - b.max) * c);
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) b.sum += __shfl_xor_sync(0xffffffffu, b.sum, o);
      st[d] = b;
      bad |= !(b.sum > 0.0 && b.sum < 1e300);
    }
    turn ^= 1;
    if (bad) break;

    // ---- the children, in ascending order (every warp alike)
    int went = -1, rejected = 0;
    double mass = 1.0, gone = 0.0;
    if (len < p.max_accept) {
      for (int w0 = cur + 1 & ~31; w0 < L && went < 0; w0 += 32) {
        const int i = w0 + lane;
        const int token = i < L ? s.tokens[i] : -1;
        const bool kid = i > cur && i < L && s.parents[i] == cur && token >= 0 && token < V;
        uint32_t kids = __ballot_sync(0xffffffffu, kid);
        if (greedy) {
          const uint32_t hit = __ballot_sync(0xffffffffu, kid && token == st[0].at);
          if (hit) went = w0 + __ffs(hit) - 1;
          continue;
        }
        const double px = kid ? weight(x, st[0], token) / st[0].sum : 0.0;
        const double qx = kid && y ? weight(y, st[1], token) / st[1].sum : 1.0;
        for (; kids && went < 0; kids &= kids - 1) {
          const int l = __ffs(kids) - 1;
          const int kt = __shfl_sync(0xffffffffu, token, l);
          const double kp = __shfl_sync(0xffffffffu, px, l), kq = __shfl_sync(0xffffffffu, qx, l);
          const double u = (double)s.uniforms[w0 + l];
          if (!y) {
            bool again = false;
            for (int e = lane; e < rejected; e += 32) again |= s.gone[e] == kt;
            const double rest = __any_sync(0xffffffffu, again) ? 0.0 : kp;
            if (u * mass < rest) {
              went = w0 + l;
            } else {
              mass = fmax(mass - rest, 0.0);
              __syncwarp();
              s.gone[rejected++] = kt;  // (every thread of the block writes the same)
              __syncwarp();
            }
            continue;
          }
          if (u * mass * kq < fmax(kp - gone * kq, 0.0)) {
            went = w0 + l;
            break;
          }
          gone += mass;
          ++rejected;
          // the residual's mass, if another child is to be tried
          bool more = (kids & (kids - 1)) != 0;
          for (int v0 = w0 + 32; v0 < L && !more; v0 += 32) {
            const int j = v0 + lane;
            more = __any_sync(0xffffffffu, j < L && s.parents[j] == cur && s.tokens[j] >= 0 && s.tokens[j] < V);
          }
          if (!more) break;
          const float ip = (float)(1.0 / st[0].sum), iq = (float)(gone / st[1].sum);
          float z = 0.f, zl = 0.f;
          for_groups(x, slice, [&](int j, const Raw<T>& v) {
            Raw<T> d;
            load8(y, j, slice, kNegInf<T>, d);
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e)
              sum += fmaxf(ex2_approx((v.get(e) - st[0].max) * c) * ip - ex2_approx((d.get(e) - st[1].max) * c) * iq, 0.f);
            add_exact(z, zl, sum);
          });
          double wz = (double)z + (double)zl;
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) wz += __shfl_xor_sync(0xffffffffu, wz, o);
          if (lane < (int)size) peer_store(peer_addr(&s.sums[turn][mine], lane), (uint64_t)__double_as_longlong(wz));
          cluster_sync();
          mass = 0.0;
          for (int e = lane; e < parts; e += 32) mass += s.sums[turn][e];
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) mass += __shfl_xor_sync(0xffffffffu, mass, o);
          turn ^= 1;
        }
      }
    }

    // ---- no child: the race for the next token
    int out = went >= 0 ? s.tokens[went] : st[0].at;
    if (went < 0 && !greedy) {
      const float ip = (float)(1.0 / st[0].sum), iq = y ? (float)(gone / st[1].sum) : 0.f;
      out = 0x7fffffff;
#pragma unroll 1
      for (int tries = 0; tries < 2 && out == 0x7fffffff; ++tries) {
        float best = 0.f;
        int best_at = 0x7fffffff;
        for_groups(x, slice, [&](int j, const Raw<T>& v) {
          Raw<float> e;
          load8(noise, j, slice, 0x3f800000u, e);
          float rest[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) rest[i] = ex2_approx((v.get(i) - st[0].max) * c) * ip;
          if (iq > 0.f && tries == 0) {
            Raw<T> d;
            load8(y, j, slice, kNegInf<T>, d);
#pragma unroll
            for (int i = 0; i < 8; ++i) rest[i] -= ex2_approx((d.get(i) - st[1].max) * c) * iq;
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float a = rest[i] > 0.f ? __fdiv_rn(rest[i], e.get(i)) : 0.f;
            if (a > best) {
              bool lost = false;
              if (!y && tries == 0)
                for (int k = 0; k < rejected; ++k) lost |= s.gone[k] == j + i * slice.step;
              if (!lost) best = a, best_at = j + i * slice.step;
            }
          }
        });
        uint64_t key = (uint64_t)__float_as_uint(best) << 32 | (uint32_t)~best_at;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
          const uint64_t other = __shfl_xor_sync(0xffffffffu, (unsigned long long)key, o);
          if (other > key) key = other;
        }
        if (lane < (int)size) peer_store(peer_addr(&s.best[turn][mine], lane), key);
        cluster_sync();
        key = 0;
        for (int e = lane; e < parts; e += 32) key = max(key, s.best[turn][e]);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
          const uint64_t other = __shfl_xor_sync(0xffffffffu, (unsigned long long)key, o);
          if (other > key) key = other;
        }
        turn ^= 1;
        if (key >> 32) out = (int)~(uint32_t)key;
      }
    }
    if (threadIdx.x == 0 && rank == 0) {
      if (out < V) s.log_arg[len - 1] = ((double)at_token(x, out) - (double)st[0].max) * T_inv;
      s.log_sum[len - 1] = st[0].sum;
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
    p.path[(size_t)r * p.max_accept + i] = i < len ? (i == 0 ? 0 : s.path[i]) : -1;
    if (p.logprobs) {
      float v = 0.f;
      if (i < len) v = bad && i == len - 1 ? __int_as_float(0x7fffffff) : (float)(s.log_arg[i] - log(s.log_sum[i]));
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
  // blocks a row: as many as two per SM give, and a group of eight logits for each thread
  int size = 1;
  while (size < kMaxCluster && 2 * size * p.num_seqs <= 2 * sms && 2 * size * kMaxThreads * 8 <= p.vocab) size *= 2;
  const int threads = p.num_seqs > 2 * sms ? kMaxThreads / 2 : kMaxThreads;
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
  return cudaLaunchKernelEx(&cfg, fp32 ? verify_kernel<float> : verify_kernel<__nv_bfloat16>, p);
}

}  // namespace mcpu
