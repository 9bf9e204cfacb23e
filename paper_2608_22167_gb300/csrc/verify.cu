// Verification of drafted tokens (mcpu_verify_tree).
//
// At each node of the walk, with p = softmax(l / T) and (if given) q of the
// draft, the residual after rejecting k children of masses m_0 = 1, m_1 .. is
//   rest(y) = max(p(y) - M q(y), 0),  M = m_0 + .. + m_{k-1},  m_k = sum_y rest(y)
// because max(max(a, 0) - b, 0) = max(a - b, 0) for b >= 0: only M is carried,
// no vector. The next token is argmax_y rest(y) / e_y, which for exponential e
// is y with probability rest(y) / m.
//
// One block per row walks its tree; a node costs one pass over its logits
// (maximum and sum together), a rejection with draft probabilities one more,
// the row's end one with the exponentials.
#include "keep.cuh"

namespace mcpu {

namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMaxNodes = MCPU_MAX_TREE_NODES;
constexpr float kLowest = -3.402823466e38f;  // a finite maximum to begin with: -inf logits weigh nothing against it

__device__ __forceinline__ float value(const __nv_bfloat16* x, int i) { return __bfloat162float(x[i]); }
__device__ __forceinline__ float value(const float* x, int i) { return x[i]; }

struct Stats {  // of a distribution: maximum, sum of e^((l - max) / T)
  float max;
  double sum;
};
struct Best {
  float v;
  int32_t i;
};

struct VerifySmem {
  float part_max[kWarps];
  double part_sum[kWarps];
  Best part_best[kWarps];
  Stats stats;
  double sum;
  Best best;
  int32_t parents[kMaxNodes], tokens[kMaxNodes];
  int32_t kids[kMaxNodes];
  double p_kid[kMaxNodes];
  int32_t num_kids, accepted;
};

__device__ __forceinline__ bool better(Best a, Best b) { return a.v > b.v || (a.v == b.v && a.i < b.i); }

// Maximum and scaled sum over the whole row of logits.
template <typename T>
__device__ Stats row_stats(const T* x, int vocab, float c, VerifySmem& s) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float m = kLowest, z = 0.f;
  for (int i = threadIdx.x; i < vocab; i += kThreads) {
    const float v = value(x, i);
    if (v > m) {
      z *= exp2f((m - v) * c);
      m = v;
    }
    z += exp2f((v - m) * c);
  }
  float wm = m;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) wm = fmaxf(wm, __shfl_xor_sync(0xffffffffu, wm, o));
  double wz = (double)(z * exp2f((m - wm) * c));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) wz += __shfl_xor_sync(0xffffffffu, wz, o);
  if (lane == 0) {
    s.part_max[warp] = wm;
    s.part_sum[warp] = wz;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    float bm = kLowest;
    for (int w = 0; w < kWarps; ++w) bm = fmaxf(bm, s.part_max[w]);
    double bz = 0;
    for (int w = 0; w < kWarps; ++w) bz += s.part_sum[w] * (double)exp2f((s.part_max[w] - bm) * c);
    s.stats = Stats{bm, bz};
  }
  __syncthreads();
  const Stats r = s.stats;
  __syncthreads();
  return r;
}

__device__ double block_sum(float x, VerifySmem& s) {
  double v = x;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if ((threadIdx.x & 31) == 0) s.part_sum[threadIdx.x >> 5] = v;
  __syncthreads();
  if (threadIdx.x == 0) {
    double t = 0;
    for (int w = 0; w < kWarps; ++w) t += s.part_sum[w];
    s.sum = t;
  }
  __syncthreads();
  const double r = s.sum;
  __syncthreads();
  return r;
}

__device__ Best block_best(Best b, VerifySmem& s) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const Best a{__shfl_xor_sync(0xffffffffu, b.v, o), __shfl_xor_sync(0xffffffffu, b.i, o)};
    if (better(a, b)) b = a;
  }
  if ((threadIdx.x & 31) == 0) s.part_best[threadIdx.x >> 5] = b;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kWarps; ++w)
      if (better(s.part_best[w], b)) b = s.part_best[w];
    s.best = b;
  }
  __syncthreads();
  const Best r = s.best;
  __syncthreads();
  return r;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) verify_kernel(const VerifyParams p) {
  __shared__ VerifySmem s;
  const int r = blockIdx.x, V = p.vocab;
  const int q0 = p.qsl[r], L = p.qsl[r + 1] - q0;
  int32_t* path = p.path + (size_t)r * p.max_accept;
  float* logprobs = p.logprobs ? p.logprobs + (size_t)r * p.max_accept : nullptr;
  int32_t bits = 0;
  if (p.qsl[0] != 0 || p.qsl[p.num_seqs] != p.total_q || q0 < 0 || L < 0 || L > p.total_q - q0) bits = kStatusBadLengths;
  else if (L > kMaxNodes) bits = kStatusUnsupportedRow;
  for (int i = threadIdx.x; i < p.max_accept; i += kThreads) {
    path[i] = -1;
    if (logprobs) logprobs[i] = 0.f;
  }
  const float heat = p.temperature ? p.temperature[r] : 0.f;
  const bool greedy = heat == 0.f;
  if (bits || L == 0) {
    if (threadIdx.x == 0) {
      if (bits) atomicOr(p.status, bits);
      p.path_len[r] = 0;
      p.next[r] = -1;
    }
    return;
  }
  for (int i = threadIdx.x; i < L; i += kThreads) {
    s.parents[i] = p.parents[q0 + i];
    s.tokens[i] = p.tokens[q0 + i];
  }
  __syncthreads();  // also: the outputs are cleared before they are written
  const double T_inv = greedy ? 1.0 : 1.0 / (double)heat;
  const float c = (float)(1.4426950408889634 * T_inv);
  int cur = 0, len = 1, next = -1;
  bool bad = !greedy && !(heat >= 1e-20f && heat <= 1e20f);
  float last = __int_as_float(0x7fffffff);
  if (threadIdx.x == 0) path[0] = 0;
  while (!bad) {
    const T* x = static_cast<const T*>(p.logits) + (size_t)(q0 + cur) * p.logits_stride;
    const T* y = p.draft && !greedy ? static_cast<const T*>(p.draft) + (size_t)(q0 + cur) * p.draft_stride : nullptr;
    const Stats sp = row_stats(x, V, c, s);
    bad = !(sp.sum > 0.0 && sp.sum < 1e300);
    if (bad) break;
    Stats sq{0.f, 1.0};
    if (y) {
      sq = row_stats(y, V, c, s);
      bad = !(sq.sum > 0.0 && sq.sum < 1e300);
      if (bad) break;
    }
    auto prob = [&](const T* row, const Stats& st, int token) {
      return exp(((double)value(row, token) - (double)st.max) * T_inv) / st.sum;
    };
    // children, in ascending order
    if (threadIdx.x == 0) {
      int n = 0;
      if (len < p.max_accept)
        for (int i = cur + 1; i < L; ++i)
          if (s.parents[i] == cur && s.tokens[i] >= 0 && s.tokens[i] < V) s.kids[n++] = i;
      s.num_kids = n;
      s.accepted = -1;
    }
    __syncthreads();
    const int nk = s.num_kids;
    Best pick{-1.f, 0x7fffffff};
    if (greedy) {
      Best b{-INFINITY, 0x7fffffff};
      for (int i = threadIdx.x; i < V; i += kThreads) {
        const float v = value(x, i);
        if (v > b.v) b = Best{v, i};
      }
      pick = block_best(b, s);
      if (threadIdx.x == 0)
        for (int k = 0; k < nk; ++k)
          if (s.tokens[s.kids[k]] == pick.i) {
            s.accepted = s.kids[k];
            break;
          }
      __syncthreads();
    } else {
      double mass = 1.0, gone = 0.0;
      if (!y) {
        for (int k = threadIdx.x; k < nk; k += kThreads) s.p_kid[k] = prob(x, sp, s.tokens[s.kids[k]]);
        __syncthreads();
        if (threadIdx.x == 0) {
          for (int k = 0; k < nk; ++k) {
            const int i = s.kids[k];
            double rest = s.p_kid[k];
            for (int e = 0; e < k; ++e)
              if (s.tokens[s.kids[e]] == s.tokens[i]) rest = 0.0;
            if ((double)p.uniforms[q0 + i] * mass < rest) {
              s.accepted = i;
              break;
            }
            mass = fmax(mass - rest, 0.0);
          }
        }
        __syncthreads();
      } else {
        for (int k = 0; k < nk; ++k) {
          const int i = s.kids[k];
          if (threadIdx.x == 0) {
            const double qx = prob(y, sq, s.tokens[i]);
            const double rest = fmax(prob(x, sp, s.tokens[i]) - gone * qx, 0.0);
            if ((double)p.uniforms[q0 + i] * mass * qx < rest) s.accepted = i;
          }
          __syncthreads();
          if (s.accepted >= 0) break;
          gone += mass;
          if (k + 1 == nk) break;
          const float ip = (float)(1.0 / sp.sum), iq = (float)(gone / sq.sum);
          float sum = 0.f;
          for (int e = threadIdx.x; e < V; e += kThreads)
            sum += fmaxf(exp2f((value(x, e) - sp.max) * c) * ip - exp2f((value(y, e) - sq.max) * c) * iq, 0.f);
          mass = block_sum(sum, s);
        }
      }
      if (s.accepted < 0) {
        const float* noise = p.noise + (size_t)r * p.noise_stride;
        const float ip = (float)(1.0 / sp.sum), iq = y && nk ? (float)(gone / sq.sum) : 0.f;
        for (int tries = 0; tries < 2 && !(pick.v > 0.f); ++tries) {
          Best b{0.f, 0x7fffffff};
          for (int e = threadIdx.x; e < V; e += kThreads) {
            float rest = exp2f((value(x, e) - sp.max) * c) * ip;
            if (iq > 0.f && tries == 0) rest -= exp2f((value(y, e) - sq.max) * c) * iq;
            if (!(rest > 0.f)) continue;
            const float v = rest / noise[e];
            if (v > b.v) {
              bool out = false;
              if (!y && tries == 0)
                for (int k = 0; k < nk; ++k) out |= s.tokens[s.kids[k]] == e;
              if (!out) b = Best{v, e};
            }
          }
          pick = block_best(b, s);
        }
      }
    }
    const int went = s.accepted;
    const int token = went >= 0 ? s.tokens[went] : pick.i;
    if (threadIdx.x == 0 && logprobs && token < V)
      logprobs[len - 1] = (float)(((double)value(x, token) - (double)sp.max) * T_inv - log(sp.sum));
    if (went < 0) {
      next = token < V ? token : -1;
      bad = next < 0;
      break;
    }
    cur = went;
    if (threadIdx.x == 0) path[len] = cur;
    ++len;
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    if (bad) {
      atomicOr(p.status, kStatusBadValues);
      if (logprobs) logprobs[len - 1] = last;
    }
    p.path_len[r] = len;
    p.next[r] = next;
  }
}

}  // namespace

cudaError_t launch_verify(const VerifyParams& p, bool fp32, int sms, cudaStream_t stream) {
  (void)sms;
  LaunchCfg lc(dim3(p.num_seqs), dim3(kThreads), 0, stream, false);
  return cudaLaunchKernelEx(&lc.cfg, fp32 ? verify_kernel<float> : verify_kernel<__nv_bfloat16>, p);
}

}  // namespace mcpu
