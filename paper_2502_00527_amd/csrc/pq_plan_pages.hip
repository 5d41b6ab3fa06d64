// pq_plan_pages: pages and slots of a batch's new tokens, from the request lengths.
//
// With have = ceil(len / g) and after = ceil((len + new) / g) pages before and after, sequence s takes the free pages
// from sum over t < s of (after_t - have_t) on, and token i of its chunk, at position len + i, has the slot
// page(position / g) * g + position % g.  A page is begun by the one new token with position % g == 0,
// which writes the block-table entry: nobody reads an entry that somebody writes.
//
// Free pages are the entries of free_pages that are not negative.  Each work-group looks for negative ones among as many entries as the sequences of its tiles
// need, while the entries that it takes are on their way, and only where there are some goes through the list in order (find_pages()).  The look takes 0.1 us of a step
// and 0.7 of the prompts below, 13 KB of the list in each work-group; 1.0 of twice as many tokens, and 1.9 with a search for the end of what a work-group's own tokens need.
//
// One launch: each work-group owns a range of tokens and finds the sequences they belong to by itself, a tile of
// kTile sequences at a time (prefix sums of tokens and pages, then a binary search a token in LDS), up to the
// tile that holds its last token.  Few tokens a thread, searched side by side: 200 sequences with
// 400K tokens take 6.4 us (5.8 before free_pages was looked through), with eight a thread one after the other they took 9.3 (a launch by itself: 3.7 - 4.2).  The last work-group goes through all of them and writes what belongs to sequences.
#include <hip/hip_runtime.h>

#include "pq_decode_kernels.hpp"
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

constexpr int kScan = 2;                                     // loads of four entries of free_pages that a thread has under way together
constexpr uint32_t kHeld = 0xffffffffu;                      // the token's page is there already

__device__ __forceinline__ uint32_t pages_up(uint32_t tokens) { return (tokens + kGroup - 1) / kGroup; }

// The ids of places among the entries of free_pages that are not negative, -1 from the last of them on, and the entries of the list that `pages` of them
// take, those that are passed over with them (the list's length and as many as there are too few, if it runs out).  All threads of the work-group call it; `ids` and `counts` are LDS
// that nobody reads any more.
__device__ __forceinline__ uint32_t find_pages(const PlanArgs& a, uint32_t pages, const uint32_t (&place)[kTokensPerThread], int32_t (&id)[kTokensPerThread], int32_t* ids,
                                               uint32_t* counts, int tid) {
  const int lane = tid & 63, wave = tid >> 6;
#pragma unroll
  for (int k = 0; k < kTokensPerThread; ++k)
    if (place[k] != kHeld) id[k] = -1;
  uint32_t found = 0, used = 0;                              // ids in the entries so far, entries up to the last one that is needed
  for (int64_t first = 0; first < a.n_free && found < pages; first += kPlanThreads) {
    const int32_t v = first + tid < a.n_free ? a.free_pages[first + tid] : -1;
    const uint64_t mask = __builtin_amdgcn_ballot_w64(v >= 0);
    __syncthreads();                                         // everybody has read what the round before wrote
    if (lane == 0) counts[wave] = __builtin_popcountll(mask);
    __syncthreads();
    uint32_t at = __builtin_popcountll(mask & ((uint64_t{1} << lane) - 1)), all = 0;
#pragma unroll
    for (int w = 0; w < kPlanThreads / 64; ++w) {
      at += w < wave ? counts[w] : 0;
      all += counts[w];
    }
    if (v >= 0) ids[at] = v;
    if (v >= 0 && found + at == pages - 1) ids[kPlanThreads] = static_cast<int32_t>(first) + tid + 1;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kTokensPerThread; ++k)
      if (place[k] != kHeld && place[k] >= found && place[k] - found < all) id[k] = ids[place[k] - found];
    found += all;
    if (found >= pages) used = static_cast<uint32_t>(ids[kPlanThreads]);
  }
  return found >= pages ? used : static_cast<uint32_t>(a.n_free) + (pages - found);
}

__global__ __launch_bounds__(kPlanThreads) void pq_plan_pages_kernel(const PlanArgs a) {
  __shared__ uint32_t first_token[kTile + 1];                // of the tile's sequences, and of what follows
  __shared__ uint32_t first_page[kTile];                     // place in free_pages
  __shared__ uint32_t wave_tokens[kPlanThreads / 64], wave_pages[kPlanThreads / 64], gaps[kPlanThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const bool last = blockIdx.x == gridDim.x - 1;
  const uint32_t begin = blockIdx.x * kTokensPerGroup;
  const uint32_t end = static_cast<uint32_t>(min(a.max_new_tokens, static_cast<int64_t>(begin) + kTokensPerGroup));
  uint32_t tokens = 0, pages = 0;                            // of the sequences before the tile
  // of this thread's tokens: place among the free pages, entry of the block table (-1: past the row), place in the page (-1: no such token)
  uint32_t place[kTokensPerThread];
  int64_t entry[kTokensPerThread];
  int within[kTokensPerThread];
  int32_t id[kTokensPerThread];
#pragma unroll
  for (int k = 0; k < kTokensPerThread; ++k) {
    place[k] = kHeld;
    entry[k] = within[k] = id[k] = -1;
  }
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
      entry[k] = page < static_cast<uint32_t>(a.max_pages_per_seq) ? static_cast<int64_t>(s) * a.max_pages_per_seq + page : -1;
      place[k] = page >= have ? first_page[low] + (page - have) : kHeld;
      within[k] = position % kGroup;
      if (entry[k] >= 0 && place[k] == kHeld) id[k] = a.block_table[entry[k]];
      else if (entry[k] >= 0 && place[k] < static_cast<uint32_t>(a.n_free)) id[k] = a.free_pages[place[k]];
    }
    // (the next tile writes what was searched)
    if (s0 + kTile < a.n_seqs && (last || tokens < end)) __syncthreads();
  }
  uint32_t used = pages;
  const uint32_t needed = min(pages, static_cast<uint32_t>(a.n_free));
  if (needed > 0) {                                          // a negative one among them?  (Zeros behind them)
    const __amdgpu_buffer_rsrc_t r = make_rsrc(a.free_pages, needed * 4u);
    auto four = [&](uint32_t first) {
      const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(r, first * 4u, 0, 0);
      return (v.x | v.y) | (v.z | v.w);
    };
    bool gap;
    if (needed <= 4 * 64) {                                  // every wavefront for itself
      gap = __builtin_amdgcn_ballot_w64(static_cast<int32_t>(four(4 * lane)) < 0) != 0;
    } else {
      uint32_t all = 0;
      for (uint32_t first = 4 * tid; first < needed; first += kScan * 4 * kPlanThreads) {
        uint32_t some[kScan];
#pragma unroll
        for (int i = 0; i < kScan; ++i) some[i] = four(first + i * 4 * kPlanThreads);
#pragma unroll
        for (int i = 0; i < kScan; ++i) all |= some[i];
      }
      const bool mine = __builtin_amdgcn_ballot_w64(static_cast<int32_t>(all) < 0) != 0;
      if (lane == 0) gaps[wave] = mine;
      __syncthreads();
      gap = (gaps[0] | gaps[1] | gaps[2] | gaps[3]) != 0;
    }
    if (gap) used = find_pages(a, pages, place, id, reinterpret_cast<int32_t*>(first_page), wave_pages, tid);
  }
#pragma unroll
  for (int k = 0; k < kTokensPerThread; ++k) {
    if (within[k] < 0) continue;
    if (place[k] != kHeld && entry[k] >= 0 && within[k] == 0) a.block_table[entry[k]] = id[k];
    a.slots[begin + k * kPlanThreads + tid] = entry[k] >= 0 && id[k] >= 0 ? static_cast<int64_t>(id[k]) * kGroup + within[k] : -1;
  }
  for (int k = 0; k < kTokensPerThread; ++k) {               // behind the last token
    const uint32_t token = begin + k * kPlanThreads + tid;
    if (token < end && token >= tokens) a.slots[token] = -1;
  }
  if (last && tid == 0) {
    a.starts[a.n_seqs] = static_cast<int32_t>(tokens);
    a.counts[0] = static_cast<int32_t>(used);
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
