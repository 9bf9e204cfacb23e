// Per-head RMS norm of q and k, rotary embedding and KV append in one pass
// (mcpu_norm_rope_kv_append).
//
// For a 64-dim head row x of query token t:
//   n = x * w / sqrt(mean(x^2) + eps)
//   y_i = n_i c_i - n_{i+32} s_i,  y_{i+32} = n_{i+32} c_i + n_i s_i   (i < 32)
// in fp32, rounded once to bf16; (c, s) is the angle row of the token's
// position. q rows go to q_out, k rows to the token's page slot, v rows there
// bit for bit.
//
// Bound by memory (every row read once and written once). Eight lanes share a
// head row; lane j holds dims 4j .. 4j + 3 and the four 32 further on, so the
// rotation needs no exchange, the mean takes three shuffles, and the weights
// and angles stay in registers: a warp walks the rows of one token, four at a
// time and kRowBatch batches in flight. With few tokens a token's rows are
// spread over up to eight warps, so that a decode step fills the GPU.
#include "tree_round.cuh"

namespace mcpu {

namespace {

constexpr int kNormThreads = 256;
constexpr int kNormWarps = kNormThreads / 32;
constexpr int kRowBatch = 4;  // head rows (of 4 per warp) whose loads are in flight together

// The row r with qsl[r] <= t < qsl[r + 1] of a non-decreasing qsl, by 32-way
// search over the whole warp (any row if there is none: the caller checks).
__device__ __forceinline__ int find_row(const int32_t* qsl, int num_seqs, int t, int lane) {
  int lo = 0, n = num_seqs;
  while (n > 1) {
    const int step = (n + 31) >> 5, at = lane * step;
    const uint32_t le = __ballot_sync(0xffffffffu, at < n && __ldg(qsl + lo + min(at, n - 1)) <= t);
    const int k = max(__popc(le) - 1, 0) * step;
    lo += k;
    n = min(step, n - k);
  }
  return lo;
}

__device__ __forceinline__ float2 unpack2(uint32_t v) {
  return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&v));
}

// Norm and rotation of a token's `rows` head rows, from x (dense) to rows
// out_step elements apart; the warp takes rows first, first + 4 kSplit, ...
template <int kSplit>
__device__ __forceinline__ void turn_rows(const __nv_bfloat16* x, __nv_bfloat16* out, int out_step, const float* weight,
                                          float eps, const float (&c)[4], const float (&s)[4], int rows, int first,
                                          int j) {
  float w[8];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    w[e] = __ldg(weight + 4 * j + e);
    w[4 + e] = __ldg(weight + 32 + 4 * j + e);
  }
  constexpr int kStep = 4 * kSplit;
  // (first & 3 differs by lane group: the bound keeps the warp together for the shuffles)
  for (int r0 = first; r0 < rows + (first & 3); r0 += kStep * kRowBatch) {
    uint2 lo[kRowBatch], hi[kRowBatch];
#pragma unroll
    for (int b = 0; b < kRowBatch; ++b) {
      const int row = r0 + b * kStep;
      lo[b] = hi[b] = make_uint2(0u, 0u);
      if (row < rows) {
        const uint2* in = reinterpret_cast<const uint2*>(x + row * kHeadDim);
        lo[b] = __ldcs(in + j);
        hi[b] = __ldcs(in + 8 + j);
      }
    }
#pragma unroll
    for (int b = 0; b < kRowBatch; ++b) {
      const int row = r0 + b * kStep;
      const float2 x0 = unpack2(lo[b].x), x1 = unpack2(lo[b].y), x2 = unpack2(hi[b].x), x3 = unpack2(hi[b].y);
      const float a[4] = {x0.x, x0.y, x1.x, x1.y}, d[4] = {x2.x, x2.y, x3.x, x3.y};
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) ss = fmaf(a[e], a[e], fmaf(d[e], d[e], ss));
#pragma unroll
      for (int o = 1; o < 8; o <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      const float mean = ss * (1.f / kHeadDim) + eps;
      const float inv = mean > 0.f ? 1.f / sqrtf(mean) : 0.f;
      float y[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float u = a[e] * inv * w[e], v = d[e] * inv * w[4 + e];
        y[e] = u * c[e] - v * s[e];
        y[4 + e] = v * c[e] + u * s[e];
      }
      if (row < rows) {
        uint2* to = reinterpret_cast<uint2*>(out + (size_t)row * out_step);
        to[j] = make_uint2(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]));
        to[8 + j] = make_uint2(pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7]));
      }
    }
  }
}

// kSplit warps share a token
template <int kSplit>
__global__ void __launch_bounds__(kNormThreads, 4) norm_rope_kernel(const NormRopeParams p) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane >> 3, j = lane & 7;
  const int t = blockIdx.x * (kNormWarps / kSplit) + warp / kSplit;
  if (t >= p.total_q) return;
  if (p.qsl[0] != 0 || p.qsl[p.num_seqs] != p.total_q) {
    if (lane == 0) atomicOr(p.status, kStatusBadLengths);
    return;
  }
  const int r = find_row(p.qsl, p.num_seqs, t, lane);
  const int q0 = __ldg(p.qsl + r), q1 = __ldg(p.qsl + r + 1), S = __ldg(p.seq_lens + r);
  const int L = q1 - q0, slot = S - L + (t - q0);
  const bool fits = L >= 1 && S >= L && S <= p.max_pages * kPage && t >= q0 && t < q1;
  const int pos = !fits ? -1 : p.positions ? __ldg(p.positions + t) : slot;
  if (pos < 0 || pos >= p.max_position) {
    if (lane == 0) atomicOr(p.status, kStatusBadLengths);
    return;
  }
  const int page = __ldg(p.block_table + (size_t)r * p.max_pages + slot / kPage);
  const bool page_ok = page >= 0 && page < p.num_pages;
  if (!page_ok && lane == 0) atomicOr(p.status, kStatusBadPage);
  const float* ang = p.cos_sin + (size_t)pos * kHeadDim + 4 * j;
  float c[4], s[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {  // scalar loads: the table is 4-byte aligned
    c[e] = __ldg(ang + e);
    s[e] = __ldg(ang + 32 + e);
  }
  const int Hq = p.num_q_heads, Hkv = p.num_kv_heads, first = (warp % kSplit) * 4 + sub;
  turn_rows<kSplit>(p.q + t * p.q_stride, p.q_out + (size_t)t * Hq * kHeadDim, kHeadDim, p.wq, p.eps, c, s, Hq, first, j);
  if (!page_ok) return;
  const size_t cache = ((size_t)page * Hkv * kPage + slot % kPage) * kHeadDim;
  turn_rows<kSplit>(p.k + t * p.k_stride, p.k_cache + cache, kPage * kHeadDim, p.wk, p.eps, c, s, Hkv, first, j);
  const __nv_bfloat16* vt = p.v + t * p.v_stride;
  for (int row = first; row < Hkv; row += 4 * kSplit) {
    const uint4 v = __ldcs(reinterpret_cast<const uint4*>(vt + row * kHeadDim) + j);
    reinterpret_cast<uint4*>(p.v_cache + cache + (size_t)row * kPage * kHeadDim)[j] = v;
  }
}

}  // namespace

cudaError_t launch_norm_rope(const NormRopeParams& p, int sms, cudaStream_t stream) {
  // warps per token: a warp each once that makes several waves of blocks, else
  // as many as keep the SMs full
  if (p.total_q > 64 * sms)
    norm_rope_kernel<1><<<(p.total_q + 7) / 8, kNormThreads, 0, stream>>>(p);
  else if (p.total_q > 4 * sms)
    norm_rope_kernel<4><<<(p.total_q + 1) / 2, kNormThreads, 0, stream>>>(p);
  else
    norm_rope_kernel<8><<<p.total_q, kNormThreads, 0, stream>>>(p);
  return cudaGetLastError();
}

}  // namespace mcpu
