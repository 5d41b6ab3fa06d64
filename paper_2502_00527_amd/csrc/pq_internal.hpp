// Internal declarations shared by the host-side entry points of libpolarquant.
// Nothing here is part of the public ABI (that is include/polarquant.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pq_plan.hpp"

namespace pq {

// Remembers the hipError_t of a failed call for pq_last_hip_error().
int record_hip_error(hipError_t e);

// True when this build has kernels for the layout.
bool layout_supported(const pq_layout* l);

// Checks of the arguments that the calls of single-token attention have in common.
int check_attention(const pq_layout* layout, const void* q, pq_dtype q_dtype, int32_t n_seqs, int32_t n_q_heads, const void* codes_pool,
                    const void* params_pool, const void* v_pool, int32_t v_bits, const void* v_params_pool, int64_t n_pool_pages,
                    const int32_t* block_table, int32_t max_pages_per_seq, const int32_t* seq_lens, int32_t max_seq_len, float sm_scale,
                    const void* residual_keys);

// Attention of sequences that are nearly all as long as max_seq_len lets them be (pq_decode.hip), of arguments that check_attention() has
// passed; the workspace is of as many bytes or more (0: there is no such launch), 256-byte aligned.  A workspace that the launch's plan does not fit into is refused.
size_t alike_workspace_bytes(const pq_layout* layout, int32_t n_seqs, int32_t n_q_heads, int32_t max_seq_len);
int attend_alike(const pq_layout* layout, const void* q, pq_dtype q_dtype, int32_t n_seqs, int32_t n_q_heads, const void* codes_pool,
                 const void* params_pool, const void* v_pool, int32_t v_bits, const void* v_params_pool, int64_t n_pool_pages,
                 const int32_t* block_table, int32_t max_pages_per_seq, const int32_t* seq_lens, int32_t max_seq_len, float sm_scale, float* out,
                 const void* residual_keys, void* workspace, size_t workspace_bytes, hipStream_t stream);

// An encoder's work-groups (256 threads) are one a (token group, KV head) in a one-dimensional grid, which HIP limits to
// 2^32 - 1 threads: launch(first group, groups) is called for as many ranges of token groups as that takes.
template <typename F>
hipError_t for_group_ranges(int64_t n_groups, int32_t n_kv_heads, F launch) {
  const int64_t most = ((int64_t{1} << 24) - 1) / n_kv_heads;            // 256 and more: n_kv_heads < 2^16
  hipError_t e = hipSuccess;
  for (int64_t first = 0; first < n_groups && e == hipSuccess; first += most)
    e = launch(first, n_groups - first < most ? n_groups - first : most);
  return e;
}

}  // namespace pq
