// Launch interfaces of the kernels of one tree-drafted decoding round
// (api_tree.cu checks the arguments and calls them): norm + rotation + KV
// append, tree attention, path compaction, and the life cycle of shared pages.
#pragma once

#include "../../include/mcpu.h"
#include "common.cuh"

namespace mcpu {

struct NormRopeParams {
  const __nv_bfloat16 *q, *k, *v;
  int64_t q_stride, k_stride, v_stride;  // elements from one token to the next
  const float *wq, *wk;                  // [64]
  float eps;
  const int32_t* positions;  // [T] or null
  const float* cos_sin;      // [max_position, 64]: cos then sin
  __nv_bfloat16 *q_out, *k_cache, *v_cache;
  const int32_t *block_table, *seq_lens, *qsl;
  int32_t* status;
  int32_t num_seqs, total_q, max_pages, num_pages, num_q_heads, num_kv_heads, max_position;
};

cudaError_t launch_norm_rope(const NormRopeParams& p, int sms, cudaStream_t stream);

struct TreeParams {
  const int32_t *block_table, *seq_lens, *qsl;
  const uint32_t* mask;      // [T, words]
  const int32_t* positions;  // [T], read with a window only
  const float* sinks;        // [Hq] or null
  __nv_bfloat16* out;
  float* lse;
  int32_t* status;
  int4* cuts;       // [4 * kTreeMaxCtas] the cut tile that begins in each piece: last piece (-1: none), token, tokens, kv head
  float* lse_part;  // [kTreeSlots][128] base-2 normalisers of cut tiles' parts
  float* o_part;    // [kTreeSlots][128][64], normalised
  int32_t words, window, num_seqs, total_q, max_pages, num_pages, num_q_heads, num_kv_heads, group;
  int32_t oob_row;   // a pool row past the end: read as zeros
  float scale_log2;  // softmax scale * log2(e)
};
constexpr int kTreeMaxCtas = 160;  // CTAs the workspace has room for (one per SM)
constexpr int kTreeTileRows = 128;
// partial slots: two for each lane's piece of the solo line, two per tile of
// the pair for each CTA's piece of the joint line
constexpr int kTreeSoloSlots = 4 * kTreeMaxCtas, kTreeSlots = 8 * kTreeMaxCtas;
cudaError_t launch_tree(const CUtensorMap& kmap, const CUtensorMap& vmap, const CUtensorMap& qmap,
                        const TreeParams& p, int sms, cudaStream_t stream);

struct PoolPtrs {
  uint8_t* p[MCPU_MAX_POOLS];
};

struct CompactParams {
  const int32_t *block_table, *seq_lens, *qsl, *path, *taken;
  int32_t *new_seq_lens, *status;
  int32_t num_pools, max_accept, num_seqs, max_pages, num_pages, num_kv_heads;
};
cudaError_t launch_compact(const CompactParams& p, const PoolPtrs& pools, cudaStream_t stream);

// words of page_scratch: pages returned per segment of page_refs, then tickets
constexpr int kPageSegments = 48;
constexpr int kScratchShrinkTicket = 48, kScratchForkTicket = 49, kScratchForkPages = 50;
static_assert(kScratchShrinkTicket == kPageSegments && kPageSegments > 32 && kPageSegments <= 64 &&
                  kScratchForkPages < MCPU_PAGE_SCRATCH,
              "collect_kernel reads two counts a lane and clears the ticket with them");

struct PageParams {
  int32_t *block_table, *seq_lens;
  const int32_t *src_rows, *dst_rows;
  int32_t *refs, *free_pages, *free_count, *copy_src, *copy_dst, *scratch, *status;
  int32_t num_forks, window, num_seqs, max_pages, num_pages;
};
cudaError_t launch_fork(const PageParams& p, cudaStream_t stream);
cudaError_t launch_shrink(const PageParams& p, cudaStream_t stream);
cudaError_t launch_copy_pages(const PoolPtrs& pools, int32_t num_pools, int64_t page_bytes, int32_t num_pages,
                              const int32_t* copy_src, const int32_t* copy_dst, int32_t num_copies, int32_t* status,
                              cudaStream_t stream);

}  // namespace mcpu
