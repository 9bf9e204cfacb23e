// C ABI of one round of tree-drafted decoding (declared in include/mcpu.h):
// host-side argument checks and launches. Nothing here allocates or
// synchronises.
#include "../../include/mcpu.h"
#include "api_internal.h"
#include "tree_round.cuh"

namespace {

using namespace mcpu;

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// non-null and 4-byte aligned
template <typename... T>
bool words_ok(const T*... p) {
  return ((p != nullptr && aligned(p, 4)) && ...);
}

// null, an unaligned pool, or more pools than one call takes
mcpu_status check_pools(void* const* pools, int32_t num_pools, PoolPtrs* out) {
  if (num_pools < 0 || num_pools > MCPU_MAX_POOLS || (num_pools > 0 && !pools)) return MCPU_ERR_INVALID_ARG;
  for (int i = 0; i < num_pools; ++i) {
    if (!pools[i] || !aligned(pools[i], 16)) return MCPU_ERR_INVALID_ARG;
    out->p[i] = static_cast<uint8_t*>(pools[i]);
  }
  return MCPU_OK;
}

mcpu_status check_page_dims(const mcpu_dims* d) {
  if (!d || d->num_seqs < 0 || d->max_pages_per_seq < 0 || d->num_pages < 0) return MCPU_ERR_INVALID_ARG;
  // token positions and rounded-up page counts stay within 32 bits
  if ((int64_t)d->max_pages_per_seq * kPage >= (int64_t)0x7fff0000 || d->num_pages >= 0x7fff0000)
    return MCPU_ERR_UNSUPPORTED;
  return MCPU_OK;
}

// Workspace: the status word, the cut tiles, their parts. Returns its size;
// with `p`, sets p's pointers into `ws`.
size_t tree_layout(uint8_t* ws, TreeParams* p) {
  constexpr size_t cuts = 256, lse = cuts + sizeof(int4) * 4 * kTreeMaxCtas;
  constexpr size_t o = lse + sizeof(float) * kTreeSlots * kTreeTileRows;
  static_assert(lse % 256 == 0 && o % 256 == 0, "alignment");
  if (p) {
    p->status = reinterpret_cast<int32_t*>(ws);
    p->cuts = reinterpret_cast<int4*>(ws + cuts);
    p->lse_part = reinterpret_cast<float*>(ws + lse);
    p->o_part = reinterpret_cast<float*>(ws + o);
  }
  return o + sizeof(float) * kTreeSlots * kTreeTileRows * kHeadDim;
}

}  // namespace

extern "C" {

mcpu_status mcpu_norm_rope_kv_append(const void* q, int64_t q_stride, const void* k_new, int64_t k_stride,
                                     const void* v_new, int64_t v_stride, const float* q_weight,
                                     const float* k_weight, float eps, const int32_t* positions,
                                     const float* cos_sin, int32_t max_position, void* q_out, void* k_cache,
                                     void* v_cache, const int32_t* block_table, const int32_t* seq_lens,
                                     const int32_t* query_start_loc, const mcpu_dims* dims, int32_t* status_word,
                                     mcpu_stream_t stream) {
  mcpu_status st = check_dims(dims);
  if (st != MCPU_OK) return st;
  if (!(eps >= 0.f) || eps > 3.0e38f) return MCPU_ERR_INVALID_ARG;
  if (dims->total_q == 0 || dims->num_seqs == 0) return MCPU_OK;
  if (!q || !k_new || !v_new || !q_out || !k_cache || !v_cache || max_position < 1) return MCPU_ERR_INVALID_ARG;
  if (!words_ok(q_weight, k_weight, cos_sin, block_table, seq_lens, query_start_loc, status_word) ||
      !aligned(positions, 4))
    return MCPU_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(q_out, 16) || !aligned(k_cache, 16) ||
      !aligned(v_cache, 16))
    return MCPU_ERR_INVALID_ARG;
  const int64_t qd = (int64_t)dims->num_q_heads * kHeadDim, kd = (int64_t)dims->num_kv_heads * kHeadDim;
  if (q_stride < qd || k_stride < kd || v_stride < kd || q_stride % 8 || k_stride % 8 || v_stride % 8)
    return MCPU_ERR_INVALID_ARG;
  if (q_out == q && q_stride != qd) return MCPU_ERR_INVALID_ARG;
  if (dims->num_pages < 1 || dims->max_pages_per_seq < 1) return MCPU_ERR_INVALID_ARG;
  int sms = 0;
  st = device_sms(&sms);
  if (st != MCPU_OK) return st;
  NormRopeParams p;
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.k = static_cast<const __nv_bfloat16*>(k_new);
  p.v = static_cast<const __nv_bfloat16*>(v_new);
  p.q_stride = q_stride;
  p.k_stride = k_stride;
  p.v_stride = v_stride;
  p.wq = q_weight;
  p.wk = k_weight;
  p.eps = eps;
  p.positions = positions;
  p.cos_sin = cos_sin;
  p.q_out = static_cast<__nv_bfloat16*>(q_out);
  p.k_cache = static_cast<__nv_bfloat16*>(k_cache);
  p.v_cache = static_cast<__nv_bfloat16*>(v_cache);
  p.block_table = block_table;
  p.seq_lens = seq_lens;
  p.qsl = query_start_loc;
  p.status = status_word;
  p.num_seqs = dims->num_seqs;
  p.total_q = dims->total_q;
  p.max_pages = dims->max_pages_per_seq;
  p.num_pages = dims->num_pages;
  p.num_q_heads = dims->num_q_heads;
  p.num_kv_heads = dims->num_kv_heads;
  p.max_position = max_position;
  return from_cuda(launch_norm_rope(p, sms, reinterpret_cast<cudaStream_t>(stream)));
}

size_t mcpu_tree_workspace_size(const mcpu_dims* dims) {
  if (check_dims(dims) != MCPU_OK) return 0;
  return tree_layout(nullptr, nullptr);
}

mcpu_status mcpu_tree_attention_forward(const void* q, const void* k_cache, const void* v_cache,
                                        const int32_t* block_table, const int32_t* seq_lens,
                                        const int32_t* query_start_loc, const uint32_t* tree_mask,
                                        int32_t mask_words, const int32_t* positions, int32_t sliding_window,
                                        float softmax_scale, const float* sinks, const mcpu_dims* dims, void* out,
                                        float* lse, void* workspace, size_t workspace_bytes, mcpu_stream_t stream) {
  mcpu_status st = check_dims(dims);
  if (st != MCPU_OK) return st;
  if (!(softmax_scale > 0.f) || softmax_scale > 3.0e38f) return MCPU_ERR_INVALID_ARG;
  if (mask_words < 1 || mask_words > MCPU_MAX_TREE_WORDS) return MCPU_ERR_INVALID_ARG;
  if (!workspace || !aligned(workspace, 256)) return MCPU_ERR_INVALID_ARG;
  if (workspace_bytes < mcpu_tree_workspace_size(dims)) return MCPU_ERR_WORKSPACE_TOO_SMALL;
  if (dims->total_q == 0 || dims->num_seqs == 0) return MCPU_OK;
  if (!q || !k_cache || !v_cache || !out) return MCPU_ERR_INVALID_ARG;
  if (!words_ok(block_table, seq_lens, query_start_loc, lse) || !words_ok(tree_mask) || !aligned(positions, 4) ||
      !aligned(sinks, 4))
    return MCPU_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(out, 16))
    return MCPU_ERR_INVALID_ARG;
  if (sliding_window > 0 && !positions) return MCPU_ERR_INVALID_ARG;
  if (dims->num_pages < 1 || dims->max_pages_per_seq < 1) return MCPU_ERR_INVALID_ARG;
  int sms = 0;
  st = device_sms(&sms);
  if (st != MCPU_OK) return st;
  const int group = dims->num_q_heads / dims->num_kv_heads;
  const int64_t rows = (int64_t)dims->num_pages * dims->num_kv_heads * kPage;
  CUtensorMap kmap, vmap, qmap;
  if (!encode_pool(&kmap, k_cache, rows) || !encode_pool(&vmap, v_cache, rows) ||
      !encode_query(&qmap, q, dims->total_q, dims->num_q_heads, group, 128))
    return MCPU_ERR_INVALID_ARG;
  TreeParams p;
  tree_layout(static_cast<uint8_t*>(workspace), &p);
  p.block_table = block_table;
  p.seq_lens = seq_lens;
  p.qsl = query_start_loc;
  p.mask = tree_mask;
  p.positions = positions;
  p.sinks = sinks;
  p.out = static_cast<__nv_bfloat16*>(out);
  p.lse = lse;
  p.words = mask_words;
  p.window = sliding_window > 0 ? sliding_window : 0;
  p.num_seqs = dims->num_seqs;
  p.total_q = dims->total_q;
  p.max_pages = dims->max_pages_per_seq;
  p.num_pages = dims->num_pages;
  p.num_q_heads = dims->num_q_heads;
  p.num_kv_heads = dims->num_kv_heads;
  p.group = group;
  p.oob_row = (int32_t)rows;
  p.scale_log2 = softmax_scale * 1.4426950408889634f;
  return from_cuda(launch_tree(kmap, vmap, qmap, p, sms, reinterpret_cast<cudaStream_t>(stream)));
}

mcpu_status mcpu_compact_kv(void* const* pools, int32_t num_pools, const int32_t* block_table,
                            const int32_t* seq_lens, const int32_t* query_start_loc, const int32_t* accept_path,
                            int32_t max_accept, const int32_t* accept_len, const mcpu_dims* dims,
                            int32_t* new_seq_lens, int32_t* status_word, mcpu_stream_t stream) {
  mcpu_status st = check_dims(dims);
  if (st != MCPU_OK) return st;
  PoolPtrs pp;
  st = check_pools(pools, num_pools, &pp);
  if (st != MCPU_OK) return st;
  if (max_accept < 0) return MCPU_ERR_INVALID_ARG;
  if (dims->num_seqs == 0) return MCPU_OK;
  if (!words_ok(block_table, seq_lens, query_start_loc, accept_len, new_seq_lens, status_word) ||
      (max_accept > 0 && !words_ok(accept_path)))
    return MCPU_ERR_INVALID_ARG;
  if (new_seq_lens == seq_lens) return MCPU_ERR_INVALID_ARG;
  if (num_pools > 0 && (dims->num_pages < 1 || dims->max_pages_per_seq < 1)) return MCPU_ERR_INVALID_ARG;
  CompactParams p;
  p.block_table = block_table;
  p.seq_lens = seq_lens;
  p.qsl = query_start_loc;
  p.path = accept_path;
  p.taken = accept_len;
  p.new_seq_lens = new_seq_lens;
  p.status = status_word;
  p.num_pools = num_pools;
  p.max_accept = max_accept;
  p.num_seqs = dims->num_seqs;
  p.max_pages = dims->max_pages_per_seq;
  p.num_pages = dims->num_pages;
  p.num_kv_heads = dims->num_kv_heads;
  return from_cuda(launch_compact(p, pp, reinterpret_cast<cudaStream_t>(stream)));
}

mcpu_status mcpu_fork_block_tables(int32_t* block_table, int32_t* seq_lens, const int32_t* src_rows,
                                   const int32_t* dst_rows, int32_t num_forks, const mcpu_dims* dims,
                                   int32_t* page_refs, const int32_t* free_pages, int32_t* free_count,
                                   int32_t* copy_src, int32_t* copy_dst, int32_t* page_scratch, int32_t* status_word,
                                   mcpu_stream_t stream) {
  mcpu_status st = check_page_dims(dims);
  if (st != MCPU_OK) return st;
  if (num_forks < 0) return MCPU_ERR_INVALID_ARG;
  if (num_forks > MCPU_MAX_FORKS) return MCPU_ERR_UNSUPPORTED;
  if (num_forks == 0) return MCPU_OK;
  if (!words_ok(block_table, seq_lens, src_rows, dst_rows, page_refs, free_pages, free_count, copy_src, copy_dst,
                page_scratch, status_word))
    return MCPU_ERR_INVALID_ARG;
  PageParams p{};
  p.block_table = block_table;
  p.seq_lens = seq_lens;
  p.src_rows = src_rows;
  p.dst_rows = dst_rows;
  p.refs = page_refs;
  p.free_pages = const_cast<int32_t*>(free_pages);
  p.free_count = free_count;
  p.copy_src = copy_src;
  p.copy_dst = copy_dst;
  p.scratch = page_scratch;
  p.status = status_word;
  p.num_forks = num_forks;
  p.num_seqs = dims->num_seqs;
  p.max_pages = dims->max_pages_per_seq;
  p.num_pages = dims->num_pages;
  return from_cuda(launch_fork(p, reinterpret_cast<cudaStream_t>(stream)));
}

mcpu_status mcpu_shrink_block_tables(int32_t* block_table, const int32_t* seq_lens, int32_t sliding_window,
                                     const mcpu_dims* dims, int32_t* page_refs, int32_t* free_pages,
                                     int32_t* free_count, int32_t* page_scratch, int32_t* status_word,
                                     mcpu_stream_t stream) {
  mcpu_status st = check_page_dims(dims);
  if (st != MCPU_OK) return st;
  if (dims->num_seqs == 0 || dims->max_pages_per_seq == 0) return MCPU_OK;
  if (!words_ok(block_table, seq_lens, page_refs, free_pages, free_count, page_scratch, status_word))
    return MCPU_ERR_INVALID_ARG;
  PageParams p{};
  p.block_table = block_table;
  p.seq_lens = const_cast<int32_t*>(seq_lens);
  p.refs = page_refs;
  p.free_pages = free_pages;
  p.free_count = free_count;
  p.scratch = page_scratch;
  p.status = status_word;
  p.window = sliding_window > 0 ? sliding_window : 0;
  p.num_seqs = dims->num_seqs;
  p.max_pages = dims->max_pages_per_seq;
  p.num_pages = dims->num_pages;
  return from_cuda(launch_shrink(p, reinterpret_cast<cudaStream_t>(stream)));
}

mcpu_status mcpu_copy_pages(void* const* pools, int32_t num_pools, int64_t page_bytes, int32_t num_pages,
                            const int32_t* copy_src, const int32_t* copy_dst, int32_t num_copies,
                            int32_t* status_word, mcpu_stream_t stream) {
  PoolPtrs pp;
  const mcpu_status st = check_pools(pools, num_pools, &pp);
  if (st != MCPU_OK) return st;
  if (page_bytes < 16 || page_bytes % 16 || num_pages < 0 || num_copies < 0) return MCPU_ERR_INVALID_ARG;
  if (page_bytes > (1 << 30) || (int64_t)num_copies * num_pools >= (int64_t)0x7fff0000) return MCPU_ERR_UNSUPPORTED;
  if (num_copies == 0 || num_pools == 0) return MCPU_OK;
  if (!words_ok(copy_src, copy_dst, status_word)) return MCPU_ERR_INVALID_ARG;
  return from_cuda(launch_copy_pages(pp, num_pools, page_bytes, num_pages, copy_src, copy_dst, num_copies,
                                     status_word, reinterpret_cast<cudaStream_t>(stream)));
}

}  // extern "C"
