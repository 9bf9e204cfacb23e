// Per-head RMS norm of q and k, rotary embedding and KV append in one pass
// (mcpu_norm_rope_kv_append).
//
// For a 64-dim head row x of query token t:
//   n = x * w / sqrt(mean(x^2) + eps)
//   y_i = n_i c_i - n_{i+32} s_i,  y_{i+32} = n_{i+32} c_i + n_i s_i   (i < 32)
// in fp32, rounded once to bf16; (c, s) is the angle row of the token's
// position. q rows go to q_out, k rows to the token's page slot, v rows there
// bit for bit.
#include "tree_round.cuh"

namespace mcpu {

constexpr int kNormWarps = 8;

// one CTA per query token; a warp per head row, lane l owns dims l and l + 32
__global__ void __launch_bounds__(kNormWarps * 32) norm_rope_kernel(const NormRopeParams p) {
  const int t = blockIdx.x;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  __shared__ int s_pos, s_dst;  // angle row (-1: skip the token), page * 16 + slot (-1: no K/V write)
  if (threadIdx.x == 0) {
    int pos = -1, dst = -1;
    if (p.qsl[0] != 0 || p.qsl[p.num_seqs] != p.total_q) {
      atomicOr(p.status, kStatusBadLengths);
    } else {
      int lo = 0, hi = p.num_seqs;  // qsl[lo] <= t < qsl[hi]
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (__ldg(p.qsl + mid) <= t) lo = mid; else hi = mid;
      }
      const int q0 = __ldg(p.qsl + lo), q1 = __ldg(p.qsl + lo + 1);
      const int L = q1 - q0, S = __ldg(p.seq_lens + lo);
      if (L < 1 || S < L || S > p.max_pages * kPage || t < q0 || t >= q1) {
        atomicOr(p.status, kStatusBadLengths);
      } else {
        const int slot = S - L + (t - q0);
        pos = p.positions ? __ldg(p.positions + t) : slot;
        if (pos < 0 || pos >= p.max_position) {
          atomicOr(p.status, kStatusBadLengths);
          pos = -1;
        } else {
          const int page = __ldg(p.block_table + (size_t)lo * p.max_pages + slot / kPage);
          if (page < 0 || page >= p.num_pages)
            atomicOr(p.status, kStatusBadPage);
          else
            dst = page * kPage + slot % kPage;
        }
      }
    }
    s_pos = pos;
    s_dst = dst;
  }
  __syncthreads();
  const int pos = s_pos, dst = s_dst;
  if (pos < 0) return;
  const float c = __ldg(p.cos_sin + (size_t)pos * kHeadDim + lane);
  const float s = __ldg(p.cos_sin + (size_t)pos * kHeadDim + 32 + lane);
  const int Hq = p.num_q_heads, Hkv = p.num_kv_heads;
  for (int row = warp; row < Hq + 2 * Hkv; row += kNormWarps) {
    const bool is_q = row < Hq, is_v = row >= Hq + Hkv;
    if (!is_q && dst < 0) continue;
    const int h = is_q ? row : is_v ? row - Hq - Hkv : row - Hq;
    const __nv_bfloat16* x = is_q   ? p.q + t * p.q_stride + h * kHeadDim
                             : is_v ? p.v + t * p.v_stride + h * kHeadDim
                                    : p.k + t * p.k_stride + h * kHeadDim;
    __nv_bfloat16* out =
        is_q ? p.q_out + ((size_t)t * Hq + h) * kHeadDim
             : (is_v ? p.v_cache : p.k_cache) + (((size_t)(dst / kPage) * Hkv + h) * kPage + dst % kPage) * kHeadDim;
    if (is_v) {
      out[lane] = x[lane];
      out[lane + 32] = x[lane + 32];
      continue;
    }
    float a = __bfloat162float(x[lane]), b = __bfloat162float(x[lane + 32]);
    float ss = a * a + b * b;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    const float mean = ss * (1.f / kHeadDim) + p.eps;
    const float r = mean > 0.f ? 1.f / sqrtf(mean) : 0.f;
    const float* w = is_q ? p.wq : p.wk;
    a *= r * __ldg(w + lane);
    b *= r * __ldg(w + lane + 32);
    out[lane] = __float2bfloat16_rn(a * c - b * s);
    out[lane + 32] = __float2bfloat16_rn(b * c + a * s);
  }
}

cudaError_t launch_norm_rope(const NormRopeParams& p, cudaStream_t stream) {
  norm_rope_kernel<<<p.total_q, kNormWarps * 32, 0, stream>>>(p);
  return cudaGetLastError();
}

}  // namespace mcpu
