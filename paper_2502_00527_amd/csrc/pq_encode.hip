// Prefill-time encoder of the polar-quantized key cache (gfx950).
//
// Per pair (x, y) = (K[j], K[j + d/2]) (Section 3.2; pairing of footnote 2 in
// Section 3.1):   rho = sqrt(x^2 + y^2),  theta = atan2(y, x),
//   angle code  a = floor((theta + pi) 2^t / 2 pi)    uniform grid over [-pi, pi)
//   radius code c = Clamp(floor((rho - z) / s), 0, 2^r - 1)
// with z = min, s = (max - min) / 2^r of rho over the tokens of the group,
// both rounded to fp16 and used as rounded.  Codes are integer decisions, so
// the arithmetic that leads to them is pinned:
//   * rho, (rho - z) / s: as IEEE fp32 with one rounding per operation and no fused
//     multiply-add gives them (this file is compiled with floating-point contraction off).
//   * the angle bin is decided by exact sign/magnitude comparisons (octant)
//     and slope comparisons against the bin edges inside the octant that are as good as
//     exact (float64, or fp32 where fp16 keys make it enough), so it equals the floor of the real-number quotient; a point exactly on
//     an edge (only possible on an axis or a diagonal) belongs to the upper
//     bin, theta = +pi is clamped into the last bin, and x = y = 0 goes to
//     bin 2^(t-1).
// With the grouped angle quantizer (Section 3.2 as printed) the angle is instead
//   theta = atan2(y, x) in float64,  a = Clamp(floor((theta - z_t) / s_t), 0, 2^t - 1)
// with z_t = min, s_t = (max - min) / 2^t of theta over the group, rounded once from
// float64 to fp16 and used as rounded (a = 0 when s_t == 0); the page's parameter block
// then holds the 64 radius entries followed by the 64 angle entries.
//
// One work-group encodes one page (128 tokens) of one KV head: thread =
// (pair octet o = tid % 8, token slot tid / 8), four tokens per thread.
#pragma clang fp contract(off)

#include "pq_encode_group.hpp"

namespace pq {
namespace {

struct EncodeArgs {
  const void* keys;
  const int32_t* page_ids;
  uint8_t* codes;
  uint32_t* params;
  int64_t token_stride;
  int64_t head_stride;
  int64_t n_tokens;
  int64_t n_pool_pages;
  int32_t n_kv_heads;
  double tan_edge[kMaxAngleBins / 8];    // tan(k * 2 pi / 2^t) for the edges inside an octant
  float tan_edge_f[kMaxAngleBins / 8];   // ... rounded to fp32
};

template <int RB, int TB, typename KT, bool GA>
__global__ __launch_bounds__(kEncThreads) void pq_encode_kernel(const EncodeArgs a) {
  __shared__ EncodeShared<GA> stats;
  // the KV heads of a page are neighbours in memory and run together
  const int kvh = blockIdx.x % a.n_kv_heads, grp = blockIdx.x / a.n_kv_heads;
  const int64_t page = a.page_ids[grp];
  if (page < 0 || page >= a.n_pool_pages) return;
  const int64_t tok0 = static_cast<int64_t>(grp) * kGroup;
  const int nv = static_cast<int>(min<int64_t>(kGroup, a.n_tokens - tok0));
  const int64_t ph = page * a.n_kv_heads + kvh;
  encode_group<RB, TB, KT, GA>(StridedRows<KT>{static_cast<const KT*>(a.keys) + tok0 * a.token_stride + kvh * a.head_stride,
                                               a.token_stride}, nv, a.codes + ph * (kBlocks * kGroup * 2 * (RB + TB)),
                               a.params + ph * (kPairs * (GA ? 2 : 1)), a.tan_edge, a.tan_edge_f, stats);
}

// Appends one decode step's key per sequence to the fp16 residual buffer and, when that fills a
// group of 128 tokens, encodes the group into its page (the residual mechanism the paper's
// Appendix B.1 refers to: recent keys stay un-quantized until a full group exists).
struct AppendArgs {
  const void* new_keys;        // [seq][kv_head][d]
  __half* residual;            // [seq][kv_head][g][d]
  const int32_t* seq_lens;     // lengths BEFORE the append
  const int32_t* block_table;
  uint8_t* codes;
  uint32_t* params;
  int64_t n_pool_pages;
  int32_t n_kv_heads;
  int32_t max_pages_per_seq;
  double tan_edge[kMaxAngleBins / 8];
  float tan_edge_f[kMaxAngleBins / 8];
};

template <int RB, int TB, typename KT, bool GA>
__global__ __launch_bounds__(kEncThreads) void pq_append_kernel(const AppendArgs a) {
  __shared__ EncodeShared<GA> stats;
  const int kvh = blockIdx.x, seq = blockIdx.y, tid = threadIdx.x;
  const int L = a.seq_lens[seq];
  if (L < 0) return;
  const int slot = L % kGroup, grp = L / kGroup;
  const int64_t sh = static_cast<int64_t>(seq) * a.n_kv_heads + kvh;
  __half* const res = a.residual + sh * (kGroup * kHeadDim);
  if (tid < kHeadDim / 8) {
    float v[8];
    load8(static_cast<const KT*>(a.new_keys) + sh * kHeadDim + tid * 8, v);
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      w[e] = static_cast<uint32_t>(__half_as_ushort(__float2half_rn(v[2 * e]))) |
             (static_cast<uint32_t>(__half_as_ushort(__float2half_rn(v[2 * e + 1]))) << 16);
    *reinterpret_cast<uint4*>(res + slot * kHeadDim + tid * 8) = make_uint4(w[0], w[1], w[2], w[3]);
  }
  if (slot != kGroup - 1) return;                 // the group is not complete yet (uniform)
  if (grp >= a.max_pages_per_seq) return;
  const int64_t page = a.block_table[static_cast<int64_t>(seq) * a.max_pages_per_seq + grp];
  if (page < 0 || page >= a.n_pool_pages) return;
  __syncthreads();                                // the new row is visible to the whole work-group
  const int64_t ph = page * a.n_kv_heads + kvh;
  encode_group<RB, TB, __half, GA>(StridedRows<__half>{res, kHeadDim}, kGroup, a.codes + ph * (kBlocks * kGroup * 2 * (RB + TB)),
                                   a.params + ph * (kPairs * (GA ? 2 : 1)), a.tan_edge, a.tan_edge_f, stats);
}

template <int RB, int TB, bool GA = false>
hipError_t launch_encode(const EncodeArgs& a, pq_dtype dt, dim3 grid, hipStream_t st) {
  if (dt == PQ_F16) hipLaunchKernelGGL((pq_encode_kernel<RB, TB, __half, GA>), grid, dim3(kEncThreads), 0, st, a);
  else              hipLaunchKernelGGL((pq_encode_kernel<RB, TB, float, GA>), grid, dim3(kEncThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace
}  // namespace pq

using namespace pq;

extern "C" int pq_encode_keys(const pq_layout* layout, const void* keys, pq_dtype key_dtype,
                              int64_t token_stride, int64_t head_stride, int64_t n_tokens,
                              const int32_t* page_ids, void* codes_pool, void* params_pool,
                              int64_t n_pool_pages, void* hip_stream) {
  if (!layout) return PQ_ERR_INVALID_ARG;
  if (!layout_supported(layout)) return PQ_ERR_UNSUPPORTED;
  if (n_tokens < 0 || n_pool_pages <= 0) return PQ_ERR_INVALID_ARG;
  if (key_dtype != PQ_F16 && key_dtype != PQ_F32) return PQ_ERR_INVALID_ARG;
  if (n_tokens == 0) return PQ_OK;
  if (!keys || !page_ids || !codes_pool || !params_pool) return PQ_ERR_INVALID_ARG;
  // 128-bit loads: rows of a head must start on 16-byte boundaries
  const int64_t vec = key_dtype == PQ_F16 ? 8 : 4;
  if ((reinterpret_cast<uintptr_t>(keys) & 15u) || token_stride % vec || head_stride % vec ||
      token_stride < kHeadDim || head_stride < 0)
    return PQ_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(codes_pool) & 15u) || (reinterpret_cast<uintptr_t>(params_pool) & 15u))
    return PQ_ERR_INVALID_ARG;
  const int64_t n_groups = (n_tokens + kGroup - 1) / kGroup;
  if (n_groups >= (int64_t{1} << 24) || layout->n_kv_heads > 65535) return PQ_ERR_UNSUPPORTED;

  EncodeArgs a;
  a.keys = keys;
  a.page_ids = page_ids;
  a.codes = static_cast<uint8_t*>(codes_pool);
  a.params = static_cast<uint32_t*>(params_pool);
  a.token_stride = token_stride;
  a.head_stride = head_stride;
  a.n_tokens = n_tokens;
  a.n_pool_pages = n_pool_pages;
  a.n_kv_heads = layout->n_kv_heads;
  fill_edges(a, layout->t_bits);

  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  const int kind = layout->r_bits * 10 + layout->t_bits + (layout->angle_quantizer == PQ_ANGLE_GROUPED ? 100 : 0);
  const hipError_t e = for_group_ranges(n_groups, layout->n_kv_heads, [&](int64_t first, int64_t groups) {
    EncodeArgs part = a;
    part.keys = static_cast<const char*>(keys) + first * kGroup * token_stride * (key_dtype == PQ_F16 ? 2 : 4);
    part.page_ids += first;
    part.n_tokens -= first * kGroup;
    const dim3 grid(static_cast<uint32_t>(groups * layout->n_kv_heads));
    switch (kind) {
      case 144: return launch_encode<4, 4, true>(part, key_dtype, grid, st);
      case 133: return launch_encode<3, 3, true>(part, key_dtype, grid, st);
      case 153: return launch_encode<5, 3, true>(part, key_dtype, grid, st);
      case 135: return launch_encode<3, 5, true>(part, key_dtype, grid, st);
      case 142: return launch_encode<4, 2, true>(part, key_dtype, grid, st);
      case 124: return launch_encode<2, 4, true>(part, key_dtype, grid, st);
      case 44: return launch_encode<4, 4>(part, key_dtype, grid, st);
      case 33: return launch_encode<3, 3>(part, key_dtype, grid, st);
      case 53: return launch_encode<5, 3>(part, key_dtype, grid, st);
      case 35: return launch_encode<3, 5>(part, key_dtype, grid, st);
      case 42: return launch_encode<4, 2>(part, key_dtype, grid, st);
      default: return launch_encode<2, 4>(part, key_dtype, grid, st);     // layout_supported() admits no other
    }
  });
  if (e != hipSuccess) return record_hip_error(e);
  return PQ_OK;
}

namespace pq {
namespace {
template <int RB, int TB, bool GA = false>
hipError_t launch_append(const AppendArgs& a, pq_dtype dt, dim3 grid, hipStream_t st) {
  if (dt == PQ_F16) hipLaunchKernelGGL((pq_append_kernel<RB, TB, __half, GA>), grid, dim3(kEncThreads), 0, st, a);
  else              hipLaunchKernelGGL((pq_append_kernel<RB, TB, float, GA>), grid, dim3(kEncThreads), 0, st, a);
  return hipGetLastError();
}
}  // namespace
}  // namespace pq

extern "C" int pq_append_keys(const pq_layout* layout, const void* new_keys, pq_dtype key_dtype, int32_t n_seqs,
                              void* residual, const int32_t* seq_lens, const int32_t* block_table,
                              int32_t max_pages_per_seq, void* codes_pool, void* params_pool,
                              int64_t n_pool_pages, void* hip_stream) {
  if (!layout) return PQ_ERR_INVALID_ARG;
  if (!layout_supported(layout)) return PQ_ERR_UNSUPPORTED;
  if (n_seqs < 0 || n_pool_pages <= 0 || max_pages_per_seq <= 0) return PQ_ERR_INVALID_ARG;
  if (key_dtype != PQ_F16 && key_dtype != PQ_F32) return PQ_ERR_INVALID_ARG;
  if (n_seqs == 0) return PQ_OK;
  if (!new_keys || !residual || !seq_lens || !block_table || !codes_pool || !params_pool) return PQ_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(new_keys) & 15u) || (reinterpret_cast<uintptr_t>(residual) & 15u) ||
      (reinterpret_cast<uintptr_t>(codes_pool) & 15u) || (reinterpret_cast<uintptr_t>(params_pool) & 15u))
    return PQ_ERR_INVALID_ARG;
  if (n_seqs > 65535) return PQ_ERR_UNSUPPORTED;
  AppendArgs a;
  a.new_keys = new_keys;
  a.residual = static_cast<__half*>(residual);
  a.seq_lens = seq_lens;
  a.block_table = block_table;
  a.codes = static_cast<uint8_t*>(codes_pool);
  a.params = static_cast<uint32_t*>(params_pool);
  a.n_pool_pages = n_pool_pages;
  a.n_kv_heads = layout->n_kv_heads;
  a.max_pages_per_seq = max_pages_per_seq;
  fill_edges(a, layout->t_bits);
  const dim3 grid(layout->n_kv_heads, n_seqs);
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  hipError_t e = hipSuccess;
  switch (layout->r_bits * 10 + layout->t_bits + (layout->angle_quantizer == PQ_ANGLE_GROUPED ? 100 : 0)) {
    case 144: e = launch_append<4, 4, true>(a, key_dtype, grid, st); break;
    case 133: e = launch_append<3, 3, true>(a, key_dtype, grid, st); break;
    case 153: e = launch_append<5, 3, true>(a, key_dtype, grid, st); break;
    case 135: e = launch_append<3, 5, true>(a, key_dtype, grid, st); break;
    case 142: e = launch_append<4, 2, true>(a, key_dtype, grid, st); break;
    case 124: e = launch_append<2, 4, true>(a, key_dtype, grid, st); break;
    case 44: e = launch_append<4, 4>(a, key_dtype, grid, st); break;
    case 33: e = launch_append<3, 3>(a, key_dtype, grid, st); break;
    case 53: e = launch_append<5, 3>(a, key_dtype, grid, st); break;
    case 35: e = launch_append<3, 5>(a, key_dtype, grid, st); break;
    case 42: e = launch_append<4, 2>(a, key_dtype, grid, st); break;
    case 24: e = launch_append<2, 4>(a, key_dtype, grid, st); break;
    default: return PQ_ERR_UNSUPPORTED;
  }
  if (e != hipSuccess) return record_hip_error(e);
  return PQ_OK;
}
