// pq_plan_pages: pages and slots of a batch's new tokens, from the request lengths.
//
// With have = ceil(len / g) and after = ceil((len + new) / g) pages before and after, sequence s takes the free pages
// from sum over t < s of (after_t - have_t) on, and token i of its chunk, at position len + i, has the slot
// page(position / g) * g + position % g.  A page is begun by the one new token with position % g == 0,
// which writes the block-table entry: nobody reads an entry that somebody writes.
//
// One launch: each work-group owns a range of tokens and finds the sequences they belong to by itself, a tile of
// kTile sequences at a time (prefix sums of tokens and pages, then a binary search a token in LDS), up to the
// tile that holds its last token.  Few tokens a thread, searched side by side: 200 sequences with
// 400K tokens take 5.8 us, with eight a thread one after the other they took 9.3 (a launch by itself: 3.7 - 4.2).  The last work-group goes through all of them and writes what belongs to sequences.
#include <hip/hip_runtime.h>

#include "pq_internal.hpp"

namespace pq {
namespace {

constexpr int kPlanThreads = 256;
constexpr int kSeqsPerThread = 4;
constexpr int kTile = kPlanThreads * kSeqsPerThread;         // sequences
constexpr int kTokensPerThread = 2;
constexpr int kTokensPerGroup = kPlanThreads * kTokensPerThread;

struct PlanArgs {
  const int32_t* seq_lens;
  const int32_t* new_lens;
  const int32_t* free_pages;
  int32_t* block_table;
  int32_t* starts;
  int64_t* slots;
  int32_t* lens_after;
  int32_t* counts;
  int64_t max_new_tokens;
  int32_t n_seqs;
  int32_t n_free;
  int32_t max_pages_per_seq;
};

__device__ __forceinline__ uint32_t pages_up(uint32_t tokens) { return (tokens + kGroup - 1) / kGroup; }

__global__ __launch_bounds__(kPlanThreads) void pq_plan_pages_kernel(const PlanArgs a) {
  __shared__ uint32_t first_token[kTile + 1];                // of the tile's sequences, and of what follows
  __shared__ uint32_t first_page[kTile];                     // place in free_pages
  __shared__ uint32_t wave_tokens[kPlanThreads / 64], wave_pages[kPlanThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const bool last = blockIdx.x == gridDim.x - 1;
  const uint32_t begin = blockIdx.x * kTokensPerGroup;
  const uint32_t end = static_cast<uint32_t>(min(a.max_new_tokens, static_cast<int64_t>(begin) + kTokensPerGroup));
  uint32_t tokens = 0, pages = 0;                            // of the sequences before the tile
  int search_from = kTile / 2;                               // half of a power of two that no tile has more sequences than
  while (search_from >= a.n_seqs && search_from > 0) search_from >>= 1;
  for (int s0 = 0; s0 < a.n_seqs && (last || tokens < end); s0 += kTile) {
    uint32_t fresh[kSeqsPerThread], need[kSeqsPerThread], my_tokens = 0, my_pages = 0;
#pragma unroll
    for (int k = 0; k < kSeqsPerThread; ++k) {
      const int s = s0 + tid * kSeqsPerThread + k;
      const uint32_t len = s < a.n_seqs ? max(0, a.seq_lens[s]) : 0;
      fresh[k] = s < a.n_seqs ? max(0, a.new_lens[s]) : 0;
      need[k] = pages_up(len + fresh[k]) - pages_up(len);
      my_tokens += fresh[k];
      my_pages += need[k];
    }
    uint32_t t = my_tokens, p = my_pages;                    // sums up to this thread
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t t2 = __shfl_up(t, d), p2 = __shfl_up(p, d);
      t += lane >= d ? t2 : 0;
      p += lane >= d ? p2 : 0;
    }
    if (lane == 63) {
      wave_tokens[wave] = t;
      wave_pages[wave] = p;
    }
    __syncthreads();
    uint32_t tile_tokens = 0, tile_pages = 0;
#pragma unroll
    for (int w = 0; w < kPlanThreads / 64; ++w) {
      t += w < wave ? wave_tokens[w] : 0;
      p += w < wave ? wave_pages[w] : 0;
      tile_tokens += wave_tokens[w];
      tile_pages += wave_pages[w];
    }
    t += tokens - my_tokens;
    p += pages - my_pages;
#pragma unroll
    for (int k = 0; k < kSeqsPerThread; ++k) {
      const int at = tid * kSeqsPerThread + k, s = s0 + at;
      first_token[at] = t;
      first_page[at] = p;
      if (last && s < a.n_seqs) {
        a.starts[s] = static_cast<int32_t>(t);
        a.lens_after[s] = static_cast<int32_t>(max(0, a.seq_lens[s]) + fresh[k]);
      }
      t += fresh[k];
      p += need[k];
    }
    tokens += tile_tokens;
    pages += tile_pages;
    if (tid == 0) first_token[kTile] = tokens;
    __syncthreads();
    const uint32_t tile_first = first_token[0];
    // the last sequence that starts at or before a token (empty ones before it start there too)
    int low_of[kTokensPerThread] = {};
    for (int step = search_from; step > 0; step >>= 1)
#pragma unroll
      for (int k = 0; k < kTokensPerThread; ++k)
        if (first_token[low_of[k] + step] <= begin + k * kPlanThreads + tid) low_of[k] += step;
#pragma unroll
    for (int k = 0; k < kTokensPerThread; ++k) {
      const uint32_t token = begin + k * kPlanThreads + tid;
      if (token >= end || token < tile_first || token >= tokens) continue;
      const int low = low_of[k], s = min(s0 + low, a.n_seqs - 1);     // (sums past 2^32 are not in order)
      const uint32_t len = max(0, a.seq_lens[s]);
      const uint32_t position = len + (token - first_token[low]), page = position / kGroup, have = pages_up(len);
      int32_t* const row = a.block_table + static_cast<int64_t>(s) * a.max_pages_per_seq;
      const bool in_row = page < static_cast<uint32_t>(a.max_pages_per_seq);
      int32_t id = -1;
      if (page >= have) {
        const uint32_t place = first_page[low] + (page - have);
        if (in_row && place < static_cast<uint32_t>(a.n_free)) id = a.free_pages[place];
        if (in_row && position % kGroup == 0) row[page] = id;
      } else if (in_row) {
        id = row[page];
      }
      a.slots[token] = id >= 0 ? static_cast<int64_t>(id) * kGroup + position % kGroup : -1;
    }
    __syncthreads();                                         // the next tile writes what was searched
  }
  for (int k = 0; k < kTokensPerThread; ++k) {               // behind the last token
    const uint32_t token = begin + k * kPlanThreads + tid;
    if (token < end && token >= tokens) a.slots[token] = -1;
  }
  if (last && tid == 0) {
    a.starts[a.n_seqs] = static_cast<int32_t>(tokens);
    a.counts[0] = static_cast<int32_t>(pages);
    a.counts[1] = static_cast<int32_t>(tokens);
  }
}

}  // namespace
}  // namespace pq

using namespace pq;

extern "C" int pq_plan_pages(const pq_layout* layout, const int32_t* seq_lens, const int32_t* new_lens, int32_t n_seqs,
                             const int32_t* free_pages, int32_t n_free, int32_t* block_table, int32_t max_pages_per_seq,
                             int32_t* starts, int64_t* slots, int64_t max_new_tokens, int32_t* lens_after, int32_t* counts,
                             void* hip_stream) {
  if (!layout) return PQ_ERR_INVALID_ARG;
  if (!layout_supported(layout)) return PQ_ERR_UNSUPPORTED;
  if (n_seqs < 0 || n_free < 0 || max_pages_per_seq <= 0 || max_new_tokens < 0) return PQ_ERR_INVALID_ARG;
  if (!starts || !counts || (n_seqs > 0 && (!seq_lens || !new_lens || !block_table || !lens_after)) || (n_free > 0 && !free_pages) ||
      (max_new_tokens > 0 && !slots))
    return PQ_ERR_INVALID_ARG;
  if (((reinterpret_cast<uintptr_t>(seq_lens) | reinterpret_cast<uintptr_t>(new_lens) | reinterpret_cast<uintptr_t>(free_pages) |
        reinterpret_cast<uintptr_t>(block_table) | reinterpret_cast<uintptr_t>(starts) | reinterpret_cast<uintptr_t>(lens_after) |
        reinterpret_cast<uintptr_t>(counts)) & 3u) || (reinterpret_cast<uintptr_t>(slots) & 7u))
    return PQ_ERR_INVALID_ARG;
  // (other work-groups still read what the last one would write)
  if (n_seqs > 0 && (lens_after == seq_lens || lens_after == new_lens || starts == seq_lens || starts == new_lens)) return PQ_ERR_INVALID_ARG;
  if (n_seqs > (1 << 20) || max_new_tokens >= (int64_t{1} << 31)) return PQ_ERR_UNSUPPORTED;
  PlanArgs a;
  a.seq_lens = seq_lens;
  a.new_lens = new_lens;
  a.free_pages = free_pages;
  a.block_table = block_table;
  a.starts = starts;
  a.slots = slots;
  a.lens_after = lens_after;
  a.counts = counts;
  a.max_new_tokens = max_new_tokens;
  a.n_seqs = n_seqs;
  a.n_free = n_free;
  a.max_pages_per_seq = max_pages_per_seq;
  const uint32_t groups = static_cast<uint32_t>(std::max<int64_t>(1, (max_new_tokens + kTokensPerGroup - 1) / kTokensPerGroup));
  hipLaunchKernelGGL(pq_plan_pages_kernel, dim3(groups), dim3(kPlanThreads), 0, static_cast<hipStream_t>(hip_stream), a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? PQ_OK : record_hip_error(e);
}
