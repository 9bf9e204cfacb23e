// C ABI of what stays after a round (declared in include/mcpu.h): verification
// of drafted tokens, attention weights per key, eviction. Host-side argument
// checks and launches; nothing here allocates or synchronises.
#include "keep.cuh"

namespace {

using namespace mcpu;

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// non-null and 4-byte aligned
template <typename... T>
bool words_ok(const T*... p) {
  return ((p != nullptr && aligned(p, 4)) && ...);
}

// The workspace of mcpu_accumulate_weights: the status word, the cut units, their parts.
constexpr size_t kWeightsCuts = 256, kWeightsParts = kWeightsCuts + sizeof(int4) * kWeightCtas;
constexpr size_t kWeightsWorkspace = kWeightsParts + sizeof(float) * 2 * kWeightCtas * 256;
static_assert(kWeightsParts % 256 == 0, "alignment");

}  // namespace

extern "C" {

mcpu_status mcpu_verify_tree(const void* logits, int64_t logits_stride, const void* draft_logits,
                             int64_t draft_stride, int32_t logits_type, int32_t vocab, const int32_t* tokens,
                             const int32_t* parents, const int32_t* query_start_loc, const float* temperature,
                             const float* uniforms, const float* exponentials, int64_t exponentials_stride,
                             int32_t num_seqs, int32_t total_q, int32_t max_accept, int32_t* accept_path,
                             int32_t* accept_len, int32_t* next_token, float* logprobs, int32_t* status_word,
                             mcpu_stream_t stream) {
  if (num_seqs < 0 || total_q < 0 || vocab < 1 || max_accept < 1) return MCPU_ERR_INVALID_ARG;
  if (logits_type != MCPU_BF16 && logits_type != MCPU_FP32) return MCPU_ERR_INVALID_ARG;
  if (num_seqs > kMaxSeqs || vocab > (1 << 30) || max_accept > (1 << 30)) return MCPU_ERR_UNSUPPORTED;
  if (num_seqs == 0) return MCPU_OK;
  const size_t size = logits_type == MCPU_FP32 ? 4 : 2;
  if (!words_ok(query_start_loc, accept_path, accept_len, next_token, status_word) || !aligned(logprobs, 4) ||
      !aligned(temperature, 4) || !aligned(uniforms, 4) || !aligned(exponentials, 4))
    return MCPU_ERR_INVALID_ARG;
  if (total_q > 0) {
    if (!words_ok(tokens, parents) || !logits || !aligned(logits, size) || !aligned(draft_logits, size))
      return MCPU_ERR_INVALID_ARG;
    if (logits_stride < vocab || (draft_logits && draft_stride < vocab)) return MCPU_ERR_INVALID_ARG;
    if (temperature && (!uniforms || !exponentials || exponentials_stride < vocab)) return MCPU_ERR_INVALID_ARG;
  }
  int sms = 0;
  const mcpu_status st = device_sms(&sms);
  if (st != MCPU_OK) return st;
  VerifyParams p;
  p.logits = logits;
  p.draft = draft_logits;
  p.logits_stride = logits_stride;
  p.draft_stride = draft_stride;
  p.noise_stride = exponentials_stride;
  p.tokens = tokens;
  p.parents = parents;
  p.qsl = query_start_loc;
  p.temperature = temperature;
  p.uniforms = uniforms;
  p.noise = exponentials;
  p.path = accept_path;
  p.path_len = accept_len;
  p.next = next_token;
  p.logprobs = logprobs;
  p.status = status_word;
  p.num_seqs = num_seqs;
  p.total_q = total_q;
  p.vocab = vocab;
  p.max_accept = max_accept;
  return from_cuda(launch_verify(p, logits_type == MCPU_FP32, sms, reinterpret_cast<cudaStream_t>(stream)));
}

size_t mcpu_weights_workspace_size(const mcpu_dims* dims) {
  return check_dims(dims) == MCPU_OK ? kWeightsWorkspace : 0;
}

mcpu_status mcpu_accumulate_weights(const void* q, const float* lse, const void* k_cache,
                                    const int32_t* block_table, const int32_t* seq_lens,
                                    const int32_t* query_start_loc, const int32_t* query_path, int32_t max_path,
                                    const int32_t* path_len, int32_t sliding_window, float softmax_scale,
                                    float decay, const mcpu_dims* dims, float* key_weights, int32_t max_slots,
                                    void* workspace, size_t workspace_bytes, mcpu_stream_t stream) {
  mcpu_status st = check_dims(dims);
  if (st != MCPU_OK) return st;
  if (!(softmax_scale >= 1e-30f && softmax_scale <= 1e30f)) return MCPU_ERR_INVALID_ARG;
  if (!(decay >= 0.f && decay <= 1.f) || max_slots < 1) return MCPU_ERR_INVALID_ARG;
  if (query_path ? !path_len || max_path < 0 : path_len != nullptr) return MCPU_ERR_INVALID_ARG;
  if (!workspace || !aligned(workspace, 256)) return MCPU_ERR_INVALID_ARG;
  if (workspace_bytes < kWeightsWorkspace) return MCPU_ERR_WORKSPACE_TOO_SMALL;
  if (dims->total_q == 0 || dims->num_seqs == 0) return MCPU_OK;
  if (!words_ok(lse, block_table, seq_lens, query_start_loc, key_weights) || !aligned(query_path, 4) ||
      !aligned(path_len, 4) || !q || !k_cache || !aligned(q, 16) || !aligned(k_cache, 16))
    return MCPU_ERR_INVALID_ARG;
  if (dims->num_pages < 1 || dims->max_pages_per_seq < 1) return MCPU_ERR_INVALID_ARG;
  int sms = 0;
  st = device_sms(&sms);
  if (st != MCPU_OK) return st;
  const int64_t rows = (int64_t)dims->num_pages * dims->num_kv_heads * kPage;
  const int group = dims->num_q_heads / dims->num_kv_heads;
  CUtensorMap kmap, qmap;
  if (!encode_pool(&kmap, k_cache, rows) || !encode_query(&qmap, q, dims->total_q, dims->num_q_heads, group, 128))
    return MCPU_ERR_INVALID_ARG;
  WeightParams p;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  p.cuts = reinterpret_cast<int4*>(ws + kWeightsCuts);
  p.parts = reinterpret_cast<float*>(ws + kWeightsParts);
  p.oob_row = (int32_t)rows;
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.k_cache = static_cast<const __nv_bfloat16*>(k_cache);
  p.lse = lse;
  p.block_table = block_table;
  p.seq_lens = seq_lens;
  p.qsl = query_start_loc;
  p.path = query_path;
  p.path_len = path_len;
  p.weights = key_weights;
  p.status = static_cast<int32_t*>(workspace);
  p.max_path = max_path;
  p.max_slots = max_slots;
  p.window = sliding_window > 0 ? sliding_window : 0;
  p.num_seqs = dims->num_seqs;
  p.total_q = dims->total_q;
  p.max_pages = dims->max_pages_per_seq;
  p.num_pages = dims->num_pages;
  p.num_q_heads = dims->num_q_heads;
  p.num_kv_heads = dims->num_kv_heads;
  p.group = group;
  p.decay = decay;
  p.scale_log2 = softmax_scale * 1.4426950408889634f;
  p.inv_scale = 1.f / softmax_scale;
  return from_cuda(launch_weights(kmap, qmap, p, sms, reinterpret_cast<cudaStream_t>(stream)));
}

mcpu_status mcpu_evict_kv(void* const* pools, int32_t num_layers, const float* key_weights, int32_t max_slots,
                          const int32_t* block_table, const int32_t* seq_lens, int32_t limit, int32_t budget,
                          int32_t keep_first, int32_t keep_last, const int32_t* page_refs, const mcpu_dims* dims,
                          float* new_key_weights, int32_t* new_seq_lens, int32_t* status_word, mcpu_stream_t stream) {
  mcpu_status st = check_dims(dims);
  if (st != MCPU_OK) return st;
  if (num_layers < 0 || num_layers > MCPU_MAX_POOLS / 2 || (num_layers > 0 && !pools)) return MCPU_ERR_INVALID_ARG;
  PoolPtrs pp;
  for (int i = 0; i < 2 * num_layers; ++i) {
    if (!pools[i] || !aligned(pools[i], 16)) return MCPU_ERR_INVALID_ARG;
    pp.p[i] = static_cast<uint8_t*>(pools[i]);
  }
  if (budget < 1 || limit < budget || keep_first < 0 || keep_last < 0 || max_slots < 1 ||
      (int64_t)keep_first + keep_last > budget)
    return MCPU_ERR_INVALID_ARG;
  if (dims->num_seqs == 0) return MCPU_OK;
  if (!words_ok(block_table, seq_lens, new_seq_lens, status_word) || !aligned(page_refs, 4)) return MCPU_ERR_INVALID_ARG;
  if (num_layers > 0 && !words_ok(key_weights, new_key_weights)) return MCPU_ERR_INVALID_ARG;
  if (new_seq_lens == seq_lens) return MCPU_ERR_INVALID_ARG;
  int sms = 0;
  st = device_sms(&sms);
  if (st != MCPU_OK) return st;
  EvictParams p;
  p.weights = key_weights;
  p.new_weights = new_key_weights;
  p.block_table = block_table;
  p.seq_lens = seq_lens;
  p.refs = page_refs;
  p.new_seq_lens = new_seq_lens;
  p.status = status_word;
  p.num_layers = num_layers;
  p.max_slots = max_slots;
  p.limit = limit;
  p.budget = budget;
  p.first = keep_first;
  p.last = keep_last;
  p.num_seqs = dims->num_seqs;
  p.max_pages = dims->max_pages_per_seq;
  p.num_pages = dims->num_pages;
  p.num_kv_heads = dims->num_kv_heads;
  return from_cuda(launch_evict(p, pp, sms, reinterpret_cast<cudaStream_t>(stream)));
}

}  // extern "C"
