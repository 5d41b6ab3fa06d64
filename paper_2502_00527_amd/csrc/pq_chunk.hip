// Host side of pq_chunk_attention: checks, how a launch is shared out, and the kernel that joins the parts of rows whose pages
// were cut into parts.  The attention kernels are in pq_chunk_kernels.hpp.
#include <algorithm>

#include "pq_chunk_kernels.hpp"

namespace pq {
namespace {

constexpr int kJoinRows = 16;                     // of a work-group, 16 lanes each

// out = sum over parts of 2^(m_c - M) acc_c / sum of 2^(m_c - M) l_c, eight dims a lane.
__global__ __launch_bounds__(16 * kJoinRows) void pq_chunk_join_kernel(const ChunkAttentionArgs a, int rows) {
  const int kvh = blockIdx.x % a.n_kv_heads, unit = blockIdx.x / a.n_kv_heads;
  const chunk::i32x4 noted = *reinterpret_cast<const chunk::i32x4*>(a.ws_units + static_cast<int64_t>(unit) * 4);
  const int row0 = uni(noted.x), count = uni(noted.y), parts = uni(noted.z);
  const int row = blockIdx.y * kJoinRows + (threadIdx.x >> 4), slice = threadIdx.x & 15;
  const int token = row / a.group, head = row - token * a.group;
  if (parts == 0 || token >= count) return;
  const int64_t stride = static_cast<int64_t>(a.n_kv_heads) * rows, first = (static_cast<int64_t>(unit) * a.n_kv_heads + kvh) * rows + row;
  const f32x2* const ml = reinterpret_cast<const f32x2*>(a.ws_ml) + first;
  const f32x4* const acc = reinterpret_cast<const f32x4*>(a.ws_acc + first * kHeadDim) + 2 * slice;
  // the weights: parts `slice`, slice + 16, ..
  float m[chunk::kMaxParts / 16], w[chunk::kMaxParts / 16], top = kNegInf, l = 0.f;
#pragma unroll
  for (int i = 0; i < chunk::kMaxParts / 16; ++i) {
    const f32x2 part = slice + 16 * i < parts ? ml[(slice + 16 * i) * stride] : f32x2{kNegInf, 0.f};
    m[i] = part.x;
    w[i] = part.y;
    top = fmaxf(top, m[i]);
  }
#pragma unroll
  for (int d = 8; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
#pragma unroll
  for (int i = 0; i < chunk::kMaxParts / 16; ++i) {
    m[i] = top > kNegInf ? __builtin_amdgcn_exp2f(m[i] - top) : 0.f;
    l = fmaf(m[i], w[i], l);
  }
#pragma unroll
  for (int d = 8; d >= 1; d >>= 1) l += __shfl_xor(l, d);
  f32x4 sum[2] = {};
#pragma unroll
  for (int i = 0; i < chunk::kMaxParts / 16; ++i)
    for (int c0 = 16 * i; c0 < min(parts, 16 * i + 16); c0 += 4) {
#pragma unroll
      for (int c = c0; c < c0 + 4; ++c) {          // (past the last part: weight 0, and the last one's row)
        const float weight = __shfl(m[i], (threadIdx.x & 48) | (c & 15));
        const f32x4 *const v = acc + min(c, parts - 1) * stride * (kHeadDim / 4), v0 = v[0], v1 = v[1];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          sum[0][k] = fmaf(weight, v0[k], sum[0][k]);
          sum[1][k] = fmaf(weight, v1[k], sum[1][k]);
        }
      }
    }
  const float inv = l > 0.f ? 1.f / l : 0.f;
  u32x4 out;
#pragma unroll
  for (int i = 0; i < 4; ++i) out[i] = h2u(to_half2(sum[i >> 1][2 * (i & 1)] * inv, sum[i >> 1][2 * (i & 1) + 1] * inv));
  reinterpret_cast<u32x4*>(a.out + ((static_cast<int64_t>(row0) + token) * a.n_q_heads + kvh * a.group + head) * kHeadDim)[slice] = out;
}

int check_chunk_shape(const pq_layout* l, int32_t n_seqs, int32_t n_q_heads, int64_t n_tokens, int32_t max_seq_len) {
  if (!l || n_seqs <= 0 || n_q_heads <= 0 || n_tokens < 0 || max_seq_len <= 0) return PQ_ERR_INVALID_ARG;
  if (l->n_kv_heads <= 0 || n_q_heads % l->n_kv_heads != 0) return PQ_ERR_INVALID_ARG;
  if (!layout_supported(l)) return PQ_ERR_UNSUPPORTED;
  if (n_q_heads / l->n_kv_heads > 16) return PQ_ERR_UNSUPPORTED;
  // (launch_fits() has the last word)
  if (n_seqs > (1 << 20) || n_tokens >= (int64_t{1} << 31) || (n_tokens + n_seqs) * l->n_kv_heads >= (int64_t{1} << 24)) return PQ_ERR_UNSUPPORTED;
  return PQ_OK;
}

}  // namespace
}  // namespace pq

using namespace pq;

extern "C" size_t pq_chunk_workspace_bytes(const pq_layout* layout, int32_t n_seqs, int32_t n_q_heads, int64_t n_tokens, int32_t max_seq_len) {
  if (check_chunk_shape(layout, n_seqs, n_q_heads, n_tokens, max_seq_len) != PQ_OK) return 0;
  const ChunkLaunch p = plan_launch(layout, n_seqs, n_q_heads, n_tokens, (static_cast<int64_t>(max_seq_len) + kGroup - 1) / kGroup, false);
  return launch_fits(layout, p) ? p.bytes : 0;
}

extern "C" int pq_chunk_attention(const pq_layout* layout, const void* q, pq_dtype q_dtype, int64_t n_tokens, int32_t n_seqs,
                                  int32_t n_q_heads, const int32_t* starts, const void* codes_pool, const void* params_pool,
                                  const void* v_pool, int32_t v_bits, const void* v_params_pool, int64_t n_pool_pages,
                                  const int32_t* block_table, int32_t max_pages_per_seq, const int32_t* seq_lens,
                                  int32_t max_seq_len, int32_t window, int32_t n_sinks, float sm_scale, void* out,
                                  const void* residual_keys, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const int st = check_chunk_shape(layout, n_seqs, n_q_heads, n_tokens, max_seq_len);
  if (st != PQ_OK) return st;
  if (q_dtype != PQ_F16 && q_dtype != PQ_F32) return PQ_ERR_INVALID_ARG;
  if (q_dtype != PQ_F16 || (v_bits != 16 && v_bits != 4 && v_bits != 2)) return PQ_ERR_UNSUPPORTED;
  if (window < 0 || n_sinks < 0 || !isfinite(sm_scale) || n_pool_pages <= 0 || max_pages_per_seq <= 0) return PQ_ERR_INVALID_ARG;
  const int64_t seq_pages = (static_cast<int64_t>(max_seq_len) + kGroup - 1) / kGroup;
  if (seq_pages > max_pages_per_seq) return PQ_ERR_INVALID_ARG;
  if (n_tokens == 0) return PQ_OK;
  if (!q || !starts || !codes_pool || !params_pool || !v_pool || !block_table || !seq_lens || !out || (v_bits != 16 && !v_params_pool)) return PQ_ERR_INVALID_ARG;
  // 128-bit loads and stores
  if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out) | reinterpret_cast<uintptr_t>(codes_pool) | reinterpret_cast<uintptr_t>(params_pool) |
       reinterpret_cast<uintptr_t>(v_pool) | reinterpret_cast<uintptr_t>(residual_keys)) & 15u)
    return PQ_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(v_bits != 16 ? v_params_pool : nullptr) | reinterpret_cast<uintptr_t>(starts) | reinterpret_cast<uintptr_t>(block_table) |
       reinterpret_cast<uintptr_t>(seq_lens)) & 3u)
    return PQ_ERR_INVALID_ARG;
  // a window as long as the longest sequence hides nothing
  if (window >= max_seq_len) window = 0;
  n_sinks = window > 0 ? std::min(n_sinks, max_seq_len) : 0;
  const ChunkLaunch most = plan_launch(layout, n_seqs, n_q_heads, n_tokens, seq_pages, false);
  if (!launch_fits(layout, most)) return PQ_ERR_UNSUPPORTED;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) || workspace_bytes < most.bytes) return PQ_ERR_WORKSPACE;
  const ChunkLaunch p = plan_launch(layout, n_seqs, n_q_heads, n_tokens, pages_of_item(seq_pages, window, n_sinks, most.tile_tokens), window > 0);

  ChunkAttentionArgs a = {};
  a.q = static_cast<const __half*>(q);
  a.codes = static_cast<const uint8_t*>(codes_pool);
  a.params = static_cast<const uint32_t*>(params_pool);
  a.values = v_pool;
  a.v_params = static_cast<const uint32_t*>(v_params_pool);
  a.residual = static_cast<const __half*>(residual_keys);
  a.block_table = block_table;
  a.starts = starts;
  a.seq_lens = seq_lens;
  a.out = static_cast<__half*>(out);
  a.ws_acc = static_cast<float*>(workspace);
  a.ws_ml = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + p.acc_bytes);
  a.ws_units = reinterpret_cast<int32_t*>(static_cast<uint8_t*>(workspace) + p.acc_bytes + p.ml_bytes);
  a.n_tokens = n_tokens;
  a.n_pool_pages = n_pool_pages;
  a.n_seqs = n_seqs;
  a.n_kv_heads = layout->n_kv_heads;
  a.n_q_heads = n_q_heads;
  a.group = n_q_heads / layout->n_kv_heads;
  a.max_pages_per_seq = max_pages_per_seq;
  a.max_seq_len = max_seq_len;
  a.window = window;
  a.n_sinks = n_sinks;
  a.tile_tokens = p.tile_tokens;
  a.n_units = static_cast<int32_t>(p.n_units);
  a.cuts = p.cuts;
  a.parts = p.parts;
  a.longest_first = longest_first(p, n_seqs) ? 1 : 0;
  a.table_index = key_table_index(layout);
  // (above zero, so that masked scores stay -inf whatever the scale is)
  a.scale_log2 = std::max(static_cast<float>(std::fabs(static_cast<double>(sm_scale)) * 1.4426950408889634074), 1.17549435e-38f);
  a.negate = sm_scale < 0.f ? 1 : 0;
  const dim3 grid(static_cast<uint32_t>(p.n_units * layout->n_kv_heads));
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const auto launch = v_bits == 16 ? launch_chunk_v16 : (v_bits == 4 ? launch_chunk_v4 : launch_chunk_v2);
  if (!launch(layout, p.rows_of_16, a, grid, stream)) return PQ_ERR_UNSUPPORTED;
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && p.cuts) {
    const int rows = 16 * p.rows_of_16;
    hipLaunchKernelGGL(pq_chunk_join_kernel, dim3(grid.x, rows / kJoinRows), dim3(16 * kJoinRows), 0, stream, a, rows);
    e = hipGetLastError();
  }
  return e == hipSuccess ? PQ_OK : record_hip_error(e);
}
