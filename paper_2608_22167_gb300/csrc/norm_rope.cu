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
// Measured (64 q / 8 kv heads): 33.8k tokens 115 us, 6.1 TB/s read and
// written, 90 % of the copy rate; 4096 tokens in 256 rows 20 us; 64 tokens
// 3.7 us in a graph. A warp per token against two or four at 4096 tokens: 22,
// 26 and 29 us (each warp pays for the lookups); rows streamed through shared
// memory by bulk copies instead, seven warps an SM: 167 us for the 33.8k.
#include "tree_round.cuh"

namespace mcpu {

namespace {

constexpr int kNormThreads = 256;
constexpr int kNormWarps = kNormThreads / 32;
constexpr int kRowBatch = 5;  // head rows (of 4 per warp) whose loads are in flight together

// The row r with qsl[r] <= t < qsl[r + 1] of a non-decreasing qsl, by 32-way
// search over the whole warp (any row if there is none: the caller checks).
__device__ __forceinline__ int find_row(const int32_t* qsl, int num_seqs, int t, int lane) {
  int lo = 0, n = num_seqs;
  while (n > 1) {
    const int step = (n + 31) >> 5, at = lane * step;
    const uint32_t le = __ballot_sync(0xffffffffu, at < n && qsl[lo + min(at, n - 1)] <= t);
    const int k = max(__popc(le) - 1, 0) * step;
    lo += k;
    n = min(step, n - k);
  }
  return lo;
}

// Four floats at a 4-byte aligned address, in one load where `vec` says that
// it is 16-byte aligned. For weights and angles only: no kernel of this library
// writes them, so they are constant from before this grid is placed, as the
// non-coherent path asks; positions, lengths and tables need not be.
__device__ __forceinline__ void load4(const float* p, bool vec, float* out) {
  if (vec) {
    const float4 v = __ldg(reinterpret_cast<const float4*>(p));
    out[0] = v.x, out[1] = v.y, out[2] = v.z, out[3] = v.w;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) out[e] = __ldg(p + e);
  }
}

__device__ __forceinline__ float2 unpack2(uint32_t v) {
  return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&v));
}

// kSplit warps share a token. Its head rows are numbered q, then k, then v; a
// warp takes rows first, first + kStep, ... The first batch of loads needs the
// token's number only and is on its way while its row, position and page are
// looked up.
template <int kSplit>
__global__ void __launch_bounds__(kNormThreads, 4) norm_rope_kernel(const NormRopeParams p) {
  grid_dep_launch();  // the next grid's blocks may be placed as this one's leave (they wait for its end)
  grid_dep_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane >> 3, j = lane & 7;
  const int t = blockIdx.x * (kNormWarps / kSplit) + warp / kSplit;
  if (t >= p.total_q) return;
  const int Hq = p.num_q_heads, Hkv = p.num_kv_heads, all = Hq + 2 * Hkv;
  constexpr int kStep = 4 * kSplit;
  const int first = (warp % kSplit) * 4 + sub;
  uint2 lo[kRowBatch], hi[kRowBatch];
  auto load = [&](int r0) {
#pragma unroll
    for (int b = 0; b < kRowBatch; ++b) {
      const int row = r0 + b * kStep;
      lo[b] = hi[b] = make_uint2(0u, 0u);
      if (row < all) {
        const __nv_bfloat16* x = row < Hq         ? p.q + t * p.q_stride + row * kHeadDim
                                 : row < Hq + Hkv ? p.k + t * p.k_stride + (row - Hq) * kHeadDim
                                                  : p.v + t * p.v_stride + (row - Hq - Hkv) * kHeadDim;
        lo[b] = __ldcs(reinterpret_cast<const uint2*>(x) + j);
        hi[b] = __ldcs(reinterpret_cast<const uint2*>(x) + 8 + j);
      }
    }
  };
  load(first);
  if (p.qsl[0] != 0 || p.qsl[p.num_seqs] != p.total_q) {
    if (lane == 0) atomicOr(p.status, kStatusBadLengths);
    return;
  }
  const bool vec = ((reinterpret_cast<uintptr_t>(p.wq) | reinterpret_cast<uintptr_t>(p.wk) |
                     reinterpret_cast<uintptr_t>(p.cos_sin)) & 15) == 0;
  float w[8];
  load4(p.wq + 4 * j, vec, w);
  load4(p.wq + 32 + 4 * j, vec, w + 4);
  // the angles come by a given position, or by the slot once the row is known
  int pos = p.positions ? p.positions[t] : -1;
  float c[4], s[4];
  auto load_angles = [&]() {
    const float* ang = p.cos_sin + (size_t)pos * kHeadDim + 4 * j;
    load4(ang, vec, c);
    load4(ang + 32, vec, s);
  };
  if (pos >= 0 && pos < p.max_position) load_angles();
  const int r = find_row(p.qsl, p.num_seqs, t, lane);
  const int q0 = p.qsl[r], q1 = p.qsl[r + 1], S = p.seq_lens[r];
  const int L = q1 - q0, slot = S - L + (t - q0);
  const bool fits = L >= 1 && S >= L && S <= p.max_pages * kPage && t >= q0 && t < q1;
  if (!p.positions) pos = slot;
  if (!fits || pos < 0 || pos >= p.max_position) {
    if (lane == 0) atomicOr(p.status, kStatusBadLengths);
    return;
  }
  const int page = p.block_table[(size_t)r * p.max_pages + slot / kPage];
  const bool page_ok = page >= 0 && page < p.num_pages;
  if (!page_ok && lane == 0) atomicOr(p.status, kStatusBadPage);
  if (!p.positions) load_angles();
  const int rows = page_ok ? all : Hq;  // rows that are written
  const size_t cache = ((size_t)max(page, 0) * Hkv * kPage + slot % kPage) * kHeadDim;
  for (int r0 = first;;) {
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
      if (row >= Hq) {  // from here on: k (the rows of v ignore it)
        load4(p.wk + 4 * j, vec, w);
        load4(p.wk + 32 + 4 * j, vec, w + 4);
      }
      const float mean = ss * (1.f / kHeadDim) + p.eps;
      const float inv = mean == 0.f ? 0.f : rsqrtf(mean);  // 2 ulp; a NaN of the row reaches all of it
      if (row < Hq + Hkv) {
        float y[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float u = a[e] * inv * w[e], v = d[e] * inv * w[4 + e];
          y[e] = u * c[e] - v * s[e];
          y[4 + e] = v * c[e] + u * s[e];
        }
        lo[b] = make_uint2(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]));
        hi[b] = make_uint2(pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7]));
      }
      if (row < rows) {
        __nv_bfloat16* out = row < Hq         ? p.q_out + ((size_t)t * Hq + row) * kHeadDim
                             : row < Hq + Hkv ? p.k_cache + cache + (size_t)(row - Hq) * kPage * kHeadDim
                                              : p.v_cache + cache + (size_t)(row - Hq - Hkv) * kPage * kHeadDim;
        reinterpret_cast<uint2*>(out)[j] = lo[b];
        reinterpret_cast<uint2*>(out)[8 + j] = hi[b];
      }
    }
    r0 += kStep * kRowBatch;
    if (r0 - sub >= rows) break;  // the whole warp
    load(r0);
  }
}

}  // namespace

cudaError_t launch_norm_rope(const NormRopeParams& p, int sms, cudaStream_t stream) {
  // warps per token: one once that fills the SMs' warps about twice over, else
  // as many as fill them
  const int split = p.total_q > 16 * sms ? 1 : p.total_q > 4 * sms ? 4 : kNormWarps;
  LaunchCfg lc(dim3((p.total_q + kNormWarps / split - 1) / (kNormWarps / split)), dim3(kNormThreads), 0, stream, true);
  return cudaLaunchKernelEx(&lc.cfg, split == 1 ? norm_rope_kernel<1> : split == 4 ? norm_rope_kernel<4> : norm_rope_kernel<8>, p);
}

}  // namespace mcpu
