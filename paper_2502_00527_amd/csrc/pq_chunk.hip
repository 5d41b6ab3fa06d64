// Host side of pq_chunk_attention: checks, how a launch is shared out, and the kernel that joins the parts of rows whose pages
// were split.  The attention kernels are in pq_chunk_kernels.hpp.
#include <algorithm>

#include "pq_chunk_kernels.hpp"

namespace pq {
namespace {

constexpr int kJoinThreads = 256;
constexpr int kMaxSplits = 64;                    // a lane each

// out = sum over splits of 2^(m_c - M) acc_c / sum of 2^(m_c - M) l_c: a wavefront a row, two dims a lane.
__global__ __launch_bounds__(kJoinThreads) void pq_chunk_join_kernel(const ChunkAttentionArgs a, int rows) {
  const int lane = threadIdx.x & 63;
  const int kvh = blockIdx.x % a.n_kv_heads, index = blockIdx.x / a.n_kv_heads;
  chunk::Item item;
  if (!chunk::find_item(a, index, lane, item)) return;
  const int first_position = item.len - item.n + item.first;
  const int pages = chunk::visible_pages(a, first_position, first_position + item.count - 1).count();
  const int splits = max(1, (pages + a.pages_per_split - 1) / a.pages_per_split);
  const int64_t slot = (static_cast<int64_t>(index) * a.n_kv_heads + kvh) * a.n_splits;
  for (int row = uni(blockIdx.y * (kJoinThreads / 64) + (threadIdx.x >> 6)); row < rows; row += gridDim.y * (kJoinThreads / 64)) {
    const int token = row / a.group, head = row - token * a.group;
    if (token >= item.count) return;
    // a split a lane: its weight
    const int64_t first = slot * rows + row;
    const f32x2 ml = lane < splits ? reinterpret_cast<const f32x2*>(a.ws_ml)[first + static_cast<int64_t>(lane) * rows] : f32x2{kNegInf, 0.f};
    float top = ml.x;
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    const float weight = top > kNegInf ? __builtin_amdgcn_exp2f(ml.x - top) : 0.f;
    float l = weight * ml.y;
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) l += __shfl_xor(l, d);
    f32x2 sum = {0.f, 0.f};
#pragma unroll 8
    for (int c = 0; c < splits; ++c) {
      const float w = u2f(static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(f2u(weight)), c)));
      const f32x2 v = reinterpret_cast<const f32x2*>(a.ws_acc + (first + static_cast<int64_t>(c) * rows) * kHeadDim)[lane];
      sum.x = fmaf(w, v.x, sum.x);
      sum.y = fmaf(w, v.y, sum.y);
    }
    const float inv = l > 0.f ? 1.f / l : 0.f;
    reinterpret_cast<uint32_t*>(a.out + ((item.row0 + item.first + token) * a.n_q_heads + kvh * a.group + head) * kHeadDim)[lane] = h2u(to_half2(sum.x * inv, sum.y * inv));
  }
}

// How a launch is shared out: items of 16 rows_of_16 query rows of a KV head, each one's pages in up to n_splits parts.
struct ChunkLaunch {
  int rows_of_16, tile_tokens, n_splits, pages_per_split;
  int64_t n_items;
  size_t acc_bytes, bytes;     // of the workspace
};

// Threads of a grid dimension: HIP takes 2^32 - 1.
bool launch_fits(const pq_layout* l, const ChunkLaunch& p) {
  return p.n_items * l->n_kv_heads < (int64_t{1} << 32) / (p.rows_of_16 <= 2 ? 256 : 1024);
}

size_t round256(size_t n) { return (n + 255) & ~static_cast<size_t>(255); }

ChunkLaunch plan_launch(const pq_layout* l, int32_t n_seqs, int32_t n_q_heads, int64_t n_tokens, int64_t max_pages) {
  ChunkLaunch p;
  const int64_t group = n_q_heads / l->n_kv_heads;
  const int64_t rows_16 = (n_tokens * group + 16 * static_cast<int64_t>(n_seqs) - 1) / (16 * static_cast<int64_t>(n_seqs));   // of a sequence, in the mean
  p.rows_of_16 = rows_16 <= 2 ? static_cast<int>(std::max<int64_t>(1, rows_16)) : chunk::kTileRows / 16;
  p.tile_tokens = static_cast<int>(16 * p.rows_of_16 / group);
  p.n_items = std::min<int64_t>(n_tokens, n_tokens / p.tile_tokens + n_seqs);
  // splits for what the items come to if chunks are alike
  const int64_t of_seq = (n_tokens + n_seqs - 1) / n_seqs, units = n_seqs * ((of_seq + p.tile_tokens - 1) / p.tile_tokens) * l->n_kv_heads;
  const int64_t pages = std::max<int64_t>(max_pages, 1);
  // At most this many splits, a number that only grows with the pages: the workspace has room for it, whatever a window leaves of them.
  // (The number taken is no such bound: 10 splits of 21 pages come to 7 of 3, of 20 pages to 10 of 2.)  Eight rounds of work-groups
  // need 270 MB.
  int64_t most;
  if (p.rows_of_16 <= 2) most = std::min((3 * kComputeUnits + units - 1) / units, (pages + 1) / 2);
  else most = std::min(8 * kComputeUnits / units, (pages + kWaveRound - 1) / kWaveRound);
  most = std::max<int64_t>(1, std::min<int64_t>(most, kMaxSplits));
  int64_t splits = most;
  if (p.rows_of_16 > 2) {
    // A compute unit has one work-group: rounds of them, in pages of time.  Starting and ending a work-group takes as long as three
    // pages, writing and joining the parts of 256 work-groups as 3.3
    double best = 0.;
    for (int64_t k = 1; k <= most; ++k) {
      const double rounds = static_cast<double>((units * k + kComputeUnits - 1) / kComputeUnits);
      const double cost = rounds * (static_cast<double>((pages + k - 1) / k) + 3.) + (k > 1 ? 2. + 3.3 * static_cast<double>(units * k) / kComputeUnits : 0.);
      if (k == 1 || cost < best) {
        best = cost;
        splits = k;
      }
    }
  }
  p.pages_per_split = static_cast<int>((pages + splits - 1) / splits);
  p.n_splits = static_cast<int>((pages + p.pages_per_split - 1) / p.pages_per_split);
  const size_t rows = most > 1 ? static_cast<size_t>(p.n_items) * l->n_kv_heads * most * 16 * p.rows_of_16 : 0;
  p.acc_bytes = round256(rows * kHeadDim * sizeof(float));
  p.bytes = std::max<size_t>(256, p.acc_bytes + round256(rows * 2 * sizeof(float)));
  return p;
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
  const ChunkLaunch p = plan_launch(layout, n_seqs, n_q_heads, n_tokens, (static_cast<int64_t>(max_seq_len) + kGroup - 1) / kGroup);
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
  const ChunkLaunch most = plan_launch(layout, n_seqs, n_q_heads, n_tokens, seq_pages);
  if (!launch_fits(layout, most)) return PQ_ERR_UNSUPPORTED;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) || workspace_bytes < most.bytes) return PQ_ERR_WORKSPACE;
  int64_t pages = seq_pages;
  if (window > 0) pages = std::min<int64_t>(pages, (static_cast<int64_t>(n_sinks) + kGroup - 1) / kGroup + (static_cast<int64_t>(window) + most.tile_tokens) / kGroup + 2);
  const ChunkLaunch p = plan_launch(layout, n_seqs, n_q_heads, n_tokens, pages);

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
  a.n_items = static_cast<int32_t>(p.n_items);
  a.n_splits = p.n_splits;
  a.pages_per_split = p.pages_per_split;
  a.table_index = key_table_index(layout);
  // (above zero, so that masked scores stay -inf whatever the scale is)
  a.scale_log2 = std::max(static_cast<float>(std::fabs(static_cast<double>(sm_scale)) * 1.4426950408889634074), 1.17549435e-38f);
  a.negate = sm_scale < 0.f ? 1 : 0;
  const dim3 grid(static_cast<uint32_t>(p.n_items * layout->n_kv_heads), p.n_splits);
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  if (v_bits == 16) launch_chunk_v16(layout, p.rows_of_16, a, grid, stream);
  else if (v_bits == 4) launch_chunk_v4(layout, p.rows_of_16, a, grid, stream);
  else launch_chunk_v2(layout, p.rows_of_16, a, grid, stream);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && p.n_splits > 1) {
    const int rows = 16 * p.rows_of_16;
    hipLaunchKernelGGL(pq_chunk_join_kernel, dim3(grid.x, rows / (kJoinThreads / 64)), dim3(kJoinThreads), 0, stream, a, rows);
    e = hipGetLastError();
  }
  return e == hipSuccess ? PQ_OK : record_hip_error(e);
}
