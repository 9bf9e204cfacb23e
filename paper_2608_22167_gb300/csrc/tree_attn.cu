// Paged attention of drafted-token trees (mcpu_tree_attention_forward).
//
// o_t = sum_{j in V(t)} e^{s_j - m} v_j / sum_{j in V(t)} e^{s_j - m},  s_j = scale q_t . k_j
// where V(t) holds the row's context keys (inside the window of t's position)
// and the nodes whose bit is set in t's mask. First form: one warp per (node,
// q head), 32 keys at a time, online softmax in fp32.
#include "tree_round.cuh"

namespace mcpu {

namespace {

constexpr int kTreeWarps = 4;

__global__ void __launch_bounds__(kTreeWarps * 32) tree_kernel(const TreeParams p) {
  const int t = blockIdx.x, h = blockIdx.y * kTreeWarps + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (h >= p.num_q_heads) return;
  if (p.qsl[0] != 0 || p.qsl[p.num_seqs] != p.total_q) {
    if (lane == 0) atomicOr(p.status, kStatusBadLengths);
    return;
  }
  int lo = 0, hi = p.num_seqs;  // qsl[lo] <= t < qsl[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (__ldg(p.qsl + mid) <= t) lo = mid; else hi = mid;
  }
  const int q0 = __ldg(p.qsl + lo), L = __ldg(p.qsl + lo + 1) - q0, S = __ldg(p.seq_lens + lo);
  if (L < 1 || S < L || S > p.max_pages * kPage || t < q0 || t >= q0 + L) {
    if (lane == 0) atomicOr(p.status, kStatusBadLengths);
    return;
  }
  if (L > 32 * p.words) {
    if (lane == 0) atomicOr(p.status, kStatusUnsupportedRow);
    return;
  }
  const int C = S - L, kvh = h / p.group;
  int begin = 0;
  if (p.window > 0) begin = max(0, min(max(__ldg(p.positions + t), C), S - 1) - p.window + 1);
  const int32_t* bt = p.block_table + (size_t)lo * p.max_pages;
  const __nv_bfloat16* q = p.q + ((size_t)t * p.num_q_heads + h) * kHeadDim;
  float m = -INFINITY, l = 0.f, o0 = 0.f, o1 = 0.f;
  for (int k0 = min(begin, C) / 32 * 32; k0 < S; k0 += 32) {
    const int j = k0 + lane, n = j - C;
    const bool sees = j < C ? j >= begin
                            : j < S && (__ldg(p.mask + (size_t)t * p.words + (n >> 5)) >> (n & 31) & 1u) != 0;
    int page = -1;
    if (sees) {
      page = __ldg(bt + j / kPage);
      if (page < 0 || page >= p.num_pages) {
        atomicOr(p.status, kStatusBadPage);
        page = -1;
      }
    }
    const size_t at = (((size_t)max(page, 0) * p.num_kv_heads + kvh) * kPage + j % kPage) * kHeadDim;
    float s = -INFINITY;
    if (sees) {
      s = 0.f;
      if (page >= 0)
        for (int d = 0; d < kHeadDim; ++d) s += __bfloat162float(q[d]) * __bfloat162float(p.k_cache[at + d]);
      s *= p.scale_log2;
    }
    float top = s;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (top == -INFINITY) continue;
    const float mn = fmaxf(m, top), a = exp2f(m - mn), w = exp2f(s - mn);
    m = mn;
    l = l * a + w;
    o0 *= a;
    o1 *= a;
    for (int i = 0; i < 32; ++i) {
      const float wi = __shfl_sync(0xffffffffu, w, i);
      const int pi = __shfl_sync(0xffffffffu, page, i);
      const size_t ai = __shfl_sync(0xffffffffu, (unsigned long long)at, i);
      if (wi == 0.f || pi < 0) continue;
      o0 += wi * __bfloat162float(p.v_cache[ai + 2 * lane]);
      o1 += wi * __bfloat162float(p.v_cache[ai + 2 * lane + 1]);
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
  float inv = l > 0.f ? 1.f / l : 0.f, lse2 = l > 0.f ? m + __log2f(l) : -INFINITY;
  if (p.sinks) inv = finish_with_sink(m, l, p.sinks[h] * 1.4426950408889634f, &lse2);
  const size_t row = (size_t)t * p.num_q_heads + h;
  reinterpret_cast<uint32_t*>(p.out + row * kHeadDim)[lane] = pack_bf16x2(o0 * inv, o1 * inv);
  if (lane == 0) p.lse[row] = lse2 * 0.69314718055994531f;
}

}  // namespace

cudaError_t launch_tree(const TreeParams& p, cudaStream_t stream) {
  tree_kernel<<<dim3(p.total_q, (p.num_q_heads + kTreeWarps - 1) / kTreeWarps), kTreeWarps * 32, 0, stream>>>(p);
  return cudaGetLastError();
}

}  // namespace mcpu
