// Attention weights per cached key (mcpu_accumulate_weights):
//   w_j = decay w_j [j < C] + sum_{i: j <= p_i, p_i - j < W} sum_u exp(scale q_iu . k_j - lse_iu)
// One thread per key, its 64 values in registers; the queries come through
// shared memory, 16 rows at a time.
#include "keep.cuh"

namespace mcpu {

namespace {

constexpr int kThreads = 128, kRows = 16;

__global__ void __launch_bounds__(kThreads) weights_kernel(const WeightParams p) {
  __shared__ float q[kRows][kHeadDim];
  __shared__ float lse2[kRows];
  __shared__ int bad_path;
  const int h = blockIdx.y, r = blockIdx.z, g = p.group;
  const int q0 = p.qsl[r], L = p.qsl[r + 1] - q0, S = p.seq_lens[r];
  const bool first = blockIdx.x == 0 && h == 0 && threadIdx.x == 0;
  const int n = p.path ? p.path_len[r] : L;
  if (threadIdx.x == 0) bad_path = 0;
  __syncthreads();
  if (p.qsl[0] != 0 || p.qsl[p.num_seqs] != p.total_q || q0 < 0 || L < 0 || L > p.total_q - q0 || n < 0 || n > S ||
      (p.path && n > p.max_path) || S > p.max_pages * kPage || S > p.max_slots) {
    if (first) atomicOr(p.status, kStatusBadLengths);
    return;
  }
  if (n == 0) return;
  const int32_t* path = p.path ? p.path + (size_t)r * p.max_path : nullptr;
  if (path) {
    for (int i = threadIdx.x; i < n; i += kThreads)
      if (path[i] < 0 || path[i] >= L) bad_path = 1;
    __syncthreads();
    if (bad_path) {
      if (first) atomicOr(p.status, kStatusBadLengths);
      return;
    }
  }
  const int C = S - n;
  for (int64_t j0 = (int64_t)blockIdx.x * kThreads; j0 < S; j0 += (int64_t)gridDim.x * kThreads) {
    const int j = (int)j0 + threadIdx.x;
    // queries that see a key of this block: i >= j - C, i < j + W - C
    const int i0 = max(0, (int)j0 - C);
    const int last = min((int)j0 + kThreads, S) - 1;
    const int i1 = p.window > 0 ? (int)min((int64_t)n, (int64_t)last + p.window - C) : n;
    float k[kHeadDim];
    const bool live = j < S;
    bool page_ok = false;
    if (live && i0 < i1) {
      const int page = p.block_table[(size_t)r * p.max_pages + j / kPage];
      page_ok = page >= 0 && page < p.num_pages;
      if (page_ok) {
        const uint4* src = reinterpret_cast<const uint4*>(
            p.k_cache + (((size_t)page * p.num_kv_heads + h) * kPage + j % kPage) * kHeadDim);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint4 v = src[e];
          const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            const float2 f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w[d]));
            k[8 * e + 2 * d] = f.x;
            k[8 * e + 2 * d + 1] = f.y;
          }
        }
      } else if (j >= C || p.window <= 0 || j > C - p.window) {
        atomicOr(p.status, kStatusBadPage);
      }
    }
    float sum = 0.f;
    for (int64_t row0 = (int64_t)i0 * g; row0 < (int64_t)i1 * g; row0 += kRows) {
      __syncthreads();
      for (int e = threadIdx.x; e < kRows * kHeadDim; e += kThreads) {
        const int64_t row = row0 + e / kHeadDim;
        const int i = (int)(row / g), u = (int)(row % g);
        if (i < i1) {
          const size_t t = q0 + (path ? path[i] : i);
          const size_t at = t * p.num_q_heads + (size_t)h * g + u;
          q[e / kHeadDim][e % kHeadDim] = __bfloat162float(p.q[at * kHeadDim + e % kHeadDim]);
          if (e % kHeadDim == 0) lse2[e / kHeadDim] = p.lse[at] == -INFINITY ? INFINITY : p.lse[at] * 1.4426950408889634f;
        }
      }
      __syncthreads();
      if (!page_ok) continue;
      for (int e = 0; e < kRows && row0 + e < (int64_t)i1 * g; ++e) {
        const int i = (int)((row0 + e) / g);
        if (j > C + i || (p.window > 0 && C + i - j >= p.window)) continue;
        float s = 0.f;
#pragma unroll
        for (int d = 0; d < kHeadDim; ++d) s = fmaf(q[e][d], k[d], s);
        sum += lse2[e] == INFINITY ? 0.f : exp2f(s * p.scale_log2 - lse2[e]);
      }
    }
    if (!live) continue;
    float* w = p.weights + ((size_t)r * p.num_kv_heads + h) * p.max_slots + j;
    const bool seen = j >= C || (p.window <= 0 || (int64_t)j + p.window > C);  // by the first query, or its own
    if (seen && !page_ok) continue;
    const float old = j < C && p.decay != 0.f ? p.decay * *w : 0.f;
    *w = old + sum;
  }
}

}  // namespace

cudaError_t launch_weights(const WeightParams& p, int sms, cudaStream_t stream) {
  (void)sms;
  const int64_t slots = (int64_t)p.max_pages * kPage < p.max_slots ? (int64_t)p.max_pages * kPage : p.max_slots;
  const int64_t blocks = (slots + kThreads - 1) / kThreads;
  LaunchCfg lc(dim3((unsigned)(blocks < 4096 ? blocks : 4096), p.num_kv_heads, p.num_seqs), dim3(kThreads), 0, stream,
               false);
  return cudaLaunchKernelEx(&lc.cfg, weights_kernel, p);
}

}  // namespace mcpu
