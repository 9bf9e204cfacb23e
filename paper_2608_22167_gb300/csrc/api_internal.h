// Host-side pieces shared by the translation units of the C ABI (api.cu,
// api_noalloc.cu, api_tree.cu): the dimension checks every forward entry point
// applies, the tensor maps of pools and queries, and the recording of the failed CUDA call behind an MCPU_ERR_CUDA (read
// back with mcpu_last_cuda_error).
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include "../../include/mcpu.h"

namespace mcpu {

// Status bit of MCPU_ERR_BAD_VALUES (the others are in common.cuh).
constexpr int32_t kStatusBadValues = 64;

// MCPU_OK, or the error for dims the kernels cannot serve: null, negative
// or inconsistent sizes (MCPU_ERR_INVALID_ARG); head_dim != 64,
// page_size != 16, H_q / H_kv outside {1, 2, 4, 8}, more than 2048 rows, or
// pools / tables too large for 32-bit TMA row coordinates
// (MCPU_ERR_UNSUPPORTED).
mcpu_status check_dims(const mcpu_dims* d);

// Records e as the calling thread's last failed CUDA call; MCPU_ERR_CUDA.
mcpu_status cuda_fail(cudaError_t e);

// MCPU_OK for cudaSuccess, else cuda_fail(e).
mcpu_status from_cuda(cudaError_t e);

// One-time setup of the current device (kernel attributes, tensor-map entry
// point); its SM count. Needed before the encoders below.
mcpu_status device_sms(int* sms);

// Growing block tables (rope_append.cu). context_lens: null for all of a row's
// entries; refs, copy_src and copy_dst: null where no page is shared.
struct GrowParams {
  int32_t* block_table;
  const int32_t *seq_lens, *context_lens, *free_pages;
  int32_t *refs, *free_count, *copy_src, *copy_dst, *status;
  int32_t num_seqs, max_pages, num_pages;
};
cudaError_t launch_grow_tables(const GrowParams& p, cudaStream_t stream);

// Tensor map of a bf16 pool as `rows` rows of 64 values, one box per (page,
// kv head) block; and of q [T, H_q, D], one box per `rows` query rows (rows /
// group tokens x the group's heads). False if the map cannot be made.
bool encode_pool(CUtensorMap* map, const void* pool, int64_t rows);
bool encode_query(CUtensorMap* map, const void* q, int32_t total_q, int32_t num_q_heads, int32_t group, int32_t rows);

}  // namespace mcpu
