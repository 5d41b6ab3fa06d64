// Choice of pages by a cheap score of the queries against the pages' bounds (pq_select_pages), and attention over the chosen
// ones (pq_sparse_attention).
//
// The score of a page is, block of 32 channels by block, q8 . c + |q8| . w in whole numbers -- one matrix instruction of 64 products
// per 16 pages and 16 query heads, {c, w} of a block being 64 bytes in the order the instruction reads them -- times the block's
// scales in fp32; whole numbers below 2^24 and fp32 operations that are rounded one by one make it the same for whoever computes it.
//
// A choice is a row of a block table: page and KV head are one index into the pools taken head by head, so that attention over the
// chosen pages is decode attention of n_seqs * n_kv_heads sequences with one KV head each.
#include <hip/hip_runtime.h>

#include "pq_internal.hpp"
#include "pq_rank.hpp"

#pragma clang fp contract(off)

namespace pq {
namespace {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

constexpr int kBoundBytes = 4 * kPairs;                      // of a page and head
constexpr int kBlockBytes = kBoundBytes / kBlocks;
constexpr float kTiny = 0x1p-100f;
constexpr int kMostKeys = 4096;                              // pages whose keys stay in LDS
constexpr int kTilePages = 16;                               // of a matrix instruction

struct SelectArgs {
  const void* q;
  const int8_t* bounds;
  const float* scales;
  const int32_t* block_table;
  const int32_t* seq_lens;
  int32_t* selected;
  int32_t* selected_lens;
  uint32_t* keys;                                            // [sequence][KV head][max_pages], if they do not stay in LDS
  int64_t n_pool_pages;
  int32_t n_kv_heads, group, max_pages_per_seq, max_seq_len, max_pages;
  int32_t n_selected, n_first, n_last;
  int32_t q_is_f32;
};

__device__ __forceinline__ int clamped(const SelectArgs& a, int seq) { return max(0, min(a.seq_lens[seq], a.max_seq_len)); }
__device__ __forceinline__ int pages_up(int tokens) { return (tokens + kGroup - 1) / kGroup; }

// The queries of a KV head as the matrix instruction's operand: lane (head l % 16, part l / 16) has 16 bytes a block, parts x, y, |x|, |y|
// of the block's 16 pairs.  Heads past the last are that one again.
struct QueryOperand {
  i32x4 code[kBlocks][64];
  float largest[kBlocks];
};
__device__ __forceinline__ void make_operand(QueryOperand& o, const SelectArgs& a, int64_t head0, int b, int lane) {
  const int64_t at = (head0 + min(lane & 15, a.group - 1)) * kHeadDim + ((lane >> 4) & 1) * kPairs + b * 16;
  float v[16];
  if (a.q_is_f32) {
    __builtin_memcpy(v, static_cast<const float*>(a.q) + at, sizeof(v));
  } else {
    _Float16 h[16];
    __builtin_memcpy(h, static_cast<const _Float16*>(a.q) + at, sizeof(h));
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = static_cast<float>(h[i]);
  }
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) m = fmaxf(m, fabsf(v[i]));
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
  const float up = m >= kTiny ? 127.0f / m : 0.f;
  i32x4 code;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    uint32_t word = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float r = rintf(v[4 * w + i] * up);
      word |= (static_cast<uint32_t>(static_cast<int>(lane < 32 ? r : fabsf(r))) & 255u) << (8 * i);
    }
    code[w] = static_cast<int>(word);
  }
  o.code[b][lane] = code;
  if (lane == 0) o.largest[b] = m;
}

// Keys of the scores of pages first .. first + 15, page l % 16 in every lane.
__device__ __forceinline__ uint32_t tile_keys(const QueryOperand& o, const SelectArgs& a, const int32_t* row, int kvh, int first, int pages, int lane) {
  const int p = first + (lane & 15);
  const int64_t page = p < pages ? row[p] : -1;
  const bool there = page >= 0 && page < a.n_pool_pages;
  const int64_t ph = there ? page * a.n_kv_heads + kvh : 0;
  const int8_t* const bound = a.bounds + ph * kBoundBytes + (lane >> 4) * 16;
  i32x4 b[kBlocks];
#pragma unroll
  for (int i = 0; i < kBlocks; ++i) b[i] = *reinterpret_cast<const i32x4*>(bound + i * kBlockBytes);
  const float4 scale = *reinterpret_cast<const float4*>(a.scales + ph * kBlocks);
  const float u[kBlocks] = {o.largest[0] * scale.x, o.largest[1] * scale.y, o.largest[2] * scale.z, o.largest[3] * scale.w};
  i32x4 n[kBlocks];
#pragma unroll
  for (int i = 0; i < kBlocks; ++i) n[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(o.code[i][lane], b[i], i32x4{0, 0, 0, 0}, 0, 0, 0);
  float best = -INFINITY;
#pragma unroll
  for (int i = 0; i < 4; ++i) {                              // heads 4 (l / 16) + i
    float t[kBlocks];
#pragma unroll
    for (int j = 0; j < kBlocks; ++j) t[j] = static_cast<float>(n[j][i]) * u[j];
    best = fmaxf(best, (t[0] + t[1]) + (t[2] + t[3]));
  }
  best = fmaxf(best, __shfl_xor(best, 16));
  best = fmaxf(best, __shfl_xor(best, 32));
  return key_of(there ? best : -INFINITY);
}

// Scores alone, of long sequences: one work-group 64 tiles of a (sequence, KV head).
constexpr int kScoreThreads = 256;
constexpr int kScorePages = 64 * kTilePages;
__global__ __launch_bounds__(kScoreThreads) void pq_page_scores_kernel(const SelectArgs a) {
  __shared__ __attribute__((aligned(16))) QueryOperand o;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, kvh = blockIdx.y, seq = blockIdx.z;
  const int pages = pages_up(clamped(a, seq)), first = blockIdx.x * kScorePages;
  if (first >= pages || pages <= a.n_selected) return;
  make_operand(o, a, (static_cast<int64_t>(seq) * a.n_kv_heads + kvh) * a.group, wave, lane);
  __syncthreads();
  const int32_t* const row = a.block_table + static_cast<int64_t>(seq) * a.max_pages_per_seq;
  uint32_t* const keys = a.keys + (static_cast<int64_t>(seq) * a.n_kv_heads + kvh) * a.max_pages;
  for (int p = first + wave * kTilePages; p < min(pages, first + kScorePages); p += kScoreThreads / 64 * kTilePages) {
    const uint32_t key = tile_keys(o, a, row, kvh, p, pages, lane);
    if (lane < kTilePages && p + lane < pages) keys[p + lane] = key;
  }
}

// kScored: pq_page_scores_kernel has left the keys in memory.
template <int kThreads, bool kScored>
__global__ __launch_bounds__(kThreads) void pq_select_kernel(const SelectArgs a) {
  __shared__ RankShared<kThreads> rank;
  __shared__ __attribute__((aligned(16))) QueryOperand o;
  __shared__ uint32_t in_lds[kScored ? 1 : kMostKeys];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, kvh = blockIdx.x, seq = blockIdx.y;
  const int len = clamped(a, seq), pages = pages_up(len);
  const int64_t unit = static_cast<int64_t>(seq) * a.n_kv_heads + kvh;
  const int32_t* const row = a.block_table + static_cast<int64_t>(seq) * a.max_pages_per_seq;
  int32_t* const out = a.selected + unit * a.n_selected;
  auto name = [&](int p) {                                   // the page's row in the pools taken head by head
    const int64_t page = row[p];
    return page >= 0 && page < a.n_pool_pages ? static_cast<int32_t>(page * a.n_kv_heads + kvh) : -1;
  };
  if (pages <= a.n_selected) {
    for (int p = tid; p < a.n_selected; p += kThreads) out[p] = p < pages ? name(p) : -1;
    if (tid == 0) a.selected_lens[unit] = len;
    return;
  }
  const uint32_t* const stored = kScored ? a.keys + unit * a.max_pages : nullptr;
  auto key = [&](int p) { return kScored ? stored[p] : in_lds[p]; };
  const int begin = a.n_first, end = pages - a.n_last, n_free = a.n_selected - a.n_first - a.n_last;
  if constexpr (!kScored) {
    if (wave < kBlocks) make_operand(o, a, unit * a.group, wave, lane);
    __syncthreads();
    for (int p = wave * kTilePages; p < pages; p += kThreads / 64 * kTilePages) {
      const uint32_t k = tile_keys(o, a, row, kvh, p, pages, lane);
      if (lane < kTilePages && p + lane < pages) in_lds[p + lane] = k;
    }
    __syncthreads();
  }
  const Threshold t = find_threshold<kThreads>(rank, begin, end, static_cast<uint32_t>(n_free), key, tid);
  Places places;
  for (int base = begin; base < end; base += kThreads) {
    const int p = base + tid;
    bool chosen;
    const uint32_t at = place<kThreads>(rank, places, t, p < end, p < end ? key(p) : 0, tid, chosen);
    if (chosen) out[a.n_first + at] = name(p);
  }
  for (int p = tid; p < a.n_first; p += kThreads) out[p] = name(p);
  for (int p = tid; p < a.n_last; p += kThreads) out[a.n_selected - a.n_last + p] = name(end + p);
  if (tid == 0) a.selected_lens[unit] = len - (pages - a.n_selected) * kGroup;
}

int64_t most_pages(int32_t max_seq_len) { return (static_cast<int64_t>(max_seq_len) + kGroup - 1) / kGroup; }

// Whether the scores take a launch of their own.
bool scores_apart(int32_t max_seq_len) { return most_pages(max_seq_len) > kMostKeys; }

int check_selection(const pq_layout* l, int32_t n_seqs, int32_t n_q_heads, int32_t max_seq_len, int32_t n_selected, int32_t n_first, int32_t n_last) {
  if (!l || n_seqs <= 0 || n_q_heads <= 0 || max_seq_len <= 0) return PQ_ERR_INVALID_ARG;
  if (l->n_kv_heads <= 0 || n_q_heads % l->n_kv_heads != 0) return PQ_ERR_INVALID_ARG;
  if (n_first < 0 || n_last < 1 || static_cast<int64_t>(n_first) + n_last > n_selected) return PQ_ERR_INVALID_ARG;
  if (!layout_supported(l)) return PQ_ERR_UNSUPPORTED;
  if (n_q_heads / l->n_kv_heads > 16 || static_cast<int64_t>(n_seqs) * l->n_kv_heads > 65535) return PQ_ERR_UNSUPPORTED;
  return PQ_OK;
}

size_t select_bytes(const pq_layout* l, int32_t n_seqs, int32_t max_seq_len) {
  const size_t keys = scores_apart(max_seq_len) ? static_cast<size_t>(n_seqs) * l->n_kv_heads * most_pages(max_seq_len) * sizeof(uint32_t) : 0;
  return std::max<size_t>(256, (keys + 255) & ~static_cast<size_t>(255));
}

// The arguments that the selection reads or writes, beyond check_selection().
int check_selection_pointers(const pq_layout* l, const void* q, pq_dtype q_dtype, const void* bounds, const void* bound_scales, int64_t n_pool_pages,
                             const int32_t* block_table, int32_t max_pages_per_seq, const int32_t* seq_lens, int32_t max_seq_len,
                             const int32_t* selected, const int32_t* selected_lens) {
  if (!q || !bounds || !bound_scales || !block_table || !seq_lens || !selected || !selected_lens) return PQ_ERR_INVALID_ARG;
  if (q_dtype != PQ_F16 && q_dtype != PQ_F32) return PQ_ERR_INVALID_ARG;
  if (n_pool_pages <= 0 || max_pages_per_seq <= 0 || most_pages(max_seq_len) > max_pages_per_seq) return PQ_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(bounds) | reinterpret_cast<uintptr_t>(bound_scales)) & 15u) return PQ_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(block_table) | reinterpret_cast<uintptr_t>(seq_lens) | reinterpret_cast<uintptr_t>(selected) |
       reinterpret_cast<uintptr_t>(selected_lens)) & 3u)
    return PQ_ERR_INVALID_ARG;
  if (n_pool_pages * l->n_kv_heads > INT32_MAX) return PQ_ERR_UNSUPPORTED;
  return PQ_OK;
}

int launch_selection(const pq_layout* l, const void* q, pq_dtype q_dtype, int32_t n_seqs, int32_t n_q_heads, const void* bounds, const void* bound_scales,
                     int64_t n_pool_pages, const int32_t* block_table, int32_t max_pages_per_seq, const int32_t* seq_lens, int32_t max_seq_len,
                     int32_t n_selected, int32_t n_first, int32_t n_last, int32_t* selected, int32_t* selected_lens, void* workspace, hipStream_t st) {
  SelectArgs a;
  a.q = q;
  a.bounds = static_cast<const int8_t*>(bounds);
  a.scales = static_cast<const float*>(bound_scales);
  a.block_table = block_table;
  a.seq_lens = seq_lens;
  a.selected = selected;
  a.selected_lens = selected_lens;
  a.keys = static_cast<uint32_t*>(workspace);
  a.n_pool_pages = n_pool_pages;
  a.n_kv_heads = l->n_kv_heads;
  a.group = n_q_heads / l->n_kv_heads;
  a.max_pages_per_seq = max_pages_per_seq;
  a.max_seq_len = max_seq_len;
  a.max_pages = static_cast<int32_t>(most_pages(max_seq_len));
  a.n_selected = n_selected;
  a.n_first = n_first;
  a.n_last = n_last;
  a.q_is_f32 = q_dtype == PQ_F32 ? 1 : 0;
  const dim3 grid(l->n_kv_heads, n_seqs);
  if (scores_apart(max_seq_len)) {
    hipLaunchKernelGGL(pq_page_scores_kernel, dim3((a.max_pages + kScorePages - 1) / kScorePages, l->n_kv_heads, n_seqs), dim3(kScoreThreads), 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return record_hip_error(e);
    hipLaunchKernelGGL((pq_select_kernel<1024, true>), grid, dim3(1024), 0, st, a);
  } else if (a.max_pages > 256) {
    hipLaunchKernelGGL((pq_select_kernel<1024, false>), grid, dim3(1024), 0, st, a);
  } else {
    hipLaunchKernelGGL((pq_select_kernel<256, false>), grid, dim3(256), 0, st, a);
  }
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? PQ_OK : record_hip_error(e);
}

// What decode attention over the chosen pages is: every (sequence, KV head) a sequence of its own, of as many tokens at most.
pq_layout one_head(const pq_layout* l) {
  pq_layout one = *l;
  one.n_kv_heads = 1;
  return one;
}
int32_t chosen_tokens(int32_t max_seq_len, int32_t n_selected) {
  return static_cast<int32_t>(std::min<int64_t>(max_seq_len, static_cast<int64_t>(n_selected) * kGroup));
}

}  // namespace
}  // namespace pq

using namespace pq;

extern "C" size_t pq_select_workspace_bytes(const pq_layout* layout, int32_t n_seqs, int32_t max_seq_len) {
  if (!layout || check_selection(layout, n_seqs, layout->n_kv_heads, max_seq_len, 1, 0, 1) != PQ_OK) return 0;
  return select_bytes(layout, n_seqs, max_seq_len);
}

extern "C" int pq_select_pages(const pq_layout* layout, const void* q, pq_dtype q_dtype, int32_t n_seqs, int32_t n_q_heads, const void* bounds,
                               const void* bound_scales, int64_t n_pool_pages, const int32_t* block_table, int32_t max_pages_per_seq,
                               const int32_t* seq_lens, int32_t max_seq_len, int32_t n_selected, int32_t n_first, int32_t n_last,
                               int32_t* selected, int32_t* selected_lens, void* workspace, size_t workspace_bytes, void* hip_stream) {
  int st = check_selection(layout, n_seqs, n_q_heads, max_seq_len, n_selected, n_first, n_last);
  if (st == PQ_OK)
    st = check_selection_pointers(layout, q, q_dtype, bounds, bound_scales, n_pool_pages, block_table, max_pages_per_seq, seq_lens, max_seq_len, selected,
                                  selected_lens);
  if (st != PQ_OK) return st;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) || workspace_bytes < select_bytes(layout, n_seqs, max_seq_len)) return PQ_ERR_WORKSPACE;
  return launch_selection(layout, q, q_dtype, n_seqs, n_q_heads, bounds, bound_scales, n_pool_pages, block_table, max_pages_per_seq, seq_lens, max_seq_len,
                          n_selected, n_first, n_last, selected, selected_lens, workspace, static_cast<hipStream_t>(hip_stream));
}

extern "C" size_t pq_sparse_workspace_bytes(const pq_layout* layout, int32_t n_seqs, int32_t n_q_heads, int32_t max_seq_len, int32_t n_selected) {
  if (check_selection(layout, n_seqs, n_q_heads, max_seq_len, n_selected, 0, 1) != PQ_OK) return 0;
  const pq_layout one = one_head(layout);
  const size_t attention = pq_decode_workspace_bytes(&one, n_seqs * layout->n_kv_heads, n_q_heads / layout->n_kv_heads, chosen_tokens(max_seq_len, n_selected));
  return attention == 0 ? 0 : select_bytes(layout, n_seqs, max_seq_len) + attention;
}

extern "C" int pq_sparse_attention(const pq_layout* layout, const void* q, pq_dtype q_dtype, int32_t n_seqs, int32_t n_q_heads, const void* codes_pool,
                                   const void* params_pool, const void* v_pool, int32_t v_bits, const void* v_params_pool, const void* bounds,
                                   const void* bound_scales, int64_t n_pool_pages, const int32_t* block_table, int32_t max_pages_per_seq,
                                   const int32_t* seq_lens, int32_t max_seq_len, int32_t n_selected, int32_t n_first, int32_t n_last, float sm_scale,
                                   int32_t* selected, int32_t* selected_lens, float* out, const void* residual_keys, void* workspace,
                                   size_t workspace_bytes, void* hip_stream) {
  if (!out || (reinterpret_cast<uintptr_t>(out) & 15u)) return PQ_ERR_INVALID_ARG;
  int st = check_selection(layout, n_seqs, n_q_heads, max_seq_len, n_selected, n_first, n_last);
  const bool given = !bounds && !bound_scales;
  if (st == PQ_OK)                                           // (a choice that is given needs neither bounds nor the table, lengths are its own)
    st = check_selection_pointers(layout, q, q_dtype, given ? q : bounds, given ? q : bound_scales, n_pool_pages, given ? selected : block_table,
                                  given ? INT32_MAX : max_pages_per_seq, given ? selected_lens : seq_lens, max_seq_len, selected, selected_lens);
  if (st != PQ_OK) return st;
  const pq_layout one = one_head(layout);
  const int32_t rows = n_seqs * layout->n_kv_heads, heads = n_q_heads / layout->n_kv_heads, tokens = chosen_tokens(max_seq_len, n_selected);
  const int64_t row_pages = n_pool_pages * layout->n_kv_heads;
  st = check_attention(&one, q, q_dtype, rows, heads, codes_pool, params_pool, v_pool, v_bits, v_params_pool, row_pages, selected, n_selected, selected_lens,
                       tokens, sm_scale, residual_keys);
  if (st != PQ_OK) return st;
  const size_t before = select_bytes(layout, n_seqs, max_seq_len);
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) || workspace_bytes < before + pq_decode_workspace_bytes(&one, rows, heads, tokens))
    return PQ_ERR_WORKSPACE;
  if (!given) {
    st = launch_selection(layout, q, q_dtype, n_seqs, n_q_heads, bounds, bound_scales, n_pool_pages, block_table, max_pages_per_seq, seq_lens, max_seq_len,
                          n_selected, n_first, n_last, selected, selected_lens, workspace, static_cast<hipStream_t>(hip_stream));
    if (st != PQ_OK) return st;
  }
  return pq_decode_attention(&one, q, q_dtype, rows, heads, codes_pool, params_pool, v_pool, v_bits, v_params_pool, row_pages, selected, n_selected,
                             selected_lens, tokens, sm_scale, out, nullptr, 0, residual_keys, static_cast<uint8_t*>(workspace) + before,
                             workspace_bytes - before, hip_stream);
}
