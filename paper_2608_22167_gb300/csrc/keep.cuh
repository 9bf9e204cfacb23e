// Launch interfaces of the kernels that decide what stays after a round
// (api_keep.cu checks the arguments and calls them): verification of drafted
// tokens, accumulated attention weights, eviction.
#pragma once

#include "../../include/mcpu.h"
#include "api_internal.h"
#include "common.cuh"
#include "tree_round.cuh"

namespace mcpu {

struct VerifyParams {
  const void *logits, *draft;  // draft: null if the children were chosen, not drawn
  int64_t logits_stride, draft_stride, noise_stride;
  const int32_t *tokens, *parents, *qsl;
  const float *temperature, *uniforms, *noise;
  int32_t *path, *path_len, *next;
  float* logprobs;
  int32_t* status;
  int32_t num_seqs, total_q, vocab, max_accept;
};
cudaError_t launch_verify(const VerifyParams& p, bool fp32, int sms, cudaStream_t stream);

struct WeightParams {
  const __nv_bfloat16 *q, *k_cache;
  const float* lse;
  const int32_t *block_table, *seq_lens, *qsl, *path, *path_len;
  float* weights;  // [B, Hkv, max_slots]
  int32_t* status;
  int4* cuts;    // [kWeightCtas] the cut unit that begins in each piece: last piece (-1: none), row, kv head, first key
  float* parts;  // [2 * kWeightCtas][256] sums of cut units' parts
  int32_t max_path, max_slots, window, num_seqs, total_q, max_pages, num_pages, num_q_heads, num_kv_heads, group;
  int32_t oob_row;  // a pool row past the end: read as zeros
  float decay, scale_log2, inv_scale;
};
constexpr int kWeightCtas = 160;  // CTAs the workspace has room for (one per SM)
cudaError_t launch_weights(const CUtensorMap& kmap, const CUtensorMap& qmap, const WeightParams& p, int sms,
                           cudaStream_t stream);

struct EvictParams {
  const float* weights;  // [layers, B, Hkv, max_slots]
  float* new_weights;    // the same, or weights itself
  const int32_t *block_table, *seq_lens, *refs;
  int32_t *new_seq_lens, *status;
  int32_t num_layers, max_slots, limit, budget, first, last, num_seqs, max_pages, num_pages, num_kv_heads;
};
cudaError_t launch_evict(const EvictParams& p, const PoolPtrs& pools, int sms, cudaStream_t stream);

}  // namespace mcpu
