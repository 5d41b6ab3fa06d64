// pq_evict_pages: the pages of the smallest weights leave a block table, the others move together, weights with them.
//
// How many pages a sequence gives up follows from its length alone, so that each work-group finds its place in the list of freed
// pages by summing over the sequences before it: one launch, nobody waits for anybody.  Which ones is a choice of the k largest keys
// (pq_rank.hpp), the keys being the weights' upside down.
//
// One work-group a sequence.  Bound: a launch's own time, 3.6 us, and four waits of the work-group; 16 bytes a page are read and written.  64 sequences of 100
// pages 5.6 us, 48 of up to 1024 5.8; one of 8192 pages, which read their weights again each time, 25 (one by one 30).
#include <hip/hip_runtime.h>

#include "pq_decode_sched.hpp"
#include "pq_internal.hpp"
#include "pq_rank.hpp"

namespace pq {
namespace {

constexpr int kKeysPerThread = 4;
constexpr int kRankRound = kRankThreads * kKeysPerThread;    // pages whose weights stay in registers; of others they are read again

struct EvictArgs {
  const int32_t* block_table;
  const int32_t* seq_lens;
  const float* weights;
  int32_t* table_after;
  int32_t* lens_after;
  float* weights_after;
  int32_t* freed;
  int32_t* counts;
  int64_t weights_stride;
  int32_t n_seqs, max_pages_per_seq, n_kept, n_first, n_last, n_freed;
};

struct Kept {
  int pages, last, gone;                                     // of the sequence; kept at its end; given up
};
__device__ __forceinline__ Kept kept_of(const EvictArgs& a, int seq) {
  const int len = max(0, a.seq_lens[seq]);
  Kept k;
  k.pages = len / kGroup + (len % kGroup != 0);
  if (k.pages > a.max_pages_per_seq) return {a.max_pages_per_seq, 0, 0};          // no such sequence: left as it is
  k.last = max(a.n_last, len % kGroup != 0 ? 1 : 0);
  const int sure = static_cast<int>(min(static_cast<int64_t>(k.pages), static_cast<int64_t>(a.n_first) + k.last));
  k.gone = max(0, k.pages - max(a.n_kept, sure));
  return k;
}

__global__ __launch_bounds__(kRankThreads) void pq_evict_kernel(const EvictArgs a) {
  __shared__ RankShared rank;
  __shared__ uint32_t sums[kRankWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), seq = blockIdx.x;
  const int64_t table_row = static_cast<int64_t>(seq) * a.max_pages_per_seq, weight_row = seq * a.weights_stride;
  // a first round of the rows, which exist whatever the sequence's length, is asked for before the lengths
  int32_t id[kKeysPerThread];
  float weight[kKeysPerThread];
  auto load_round = [&](int p0, int most) {
#pragma unroll
    for (int j = 0; j < kKeysPerThread; ++j) {
      const bool there = p0 + j < most && seq < a.n_seqs;
      id[j] = there ? a.block_table[table_row + p0 + j] : 0;
      weight[j] = there ? a.weights[weight_row + p0 + j] : 0.f;
    }
  };
  load_round(tid * kKeysPerThread, a.max_pages_per_seq);
  uint32_t before = 0;
  for (int s = tid; s < min(seq, a.n_seqs); s += kRankThreads) before += kept_of(a, s).gone;
  const Kept k = seq < a.n_seqs ? kept_of(a, seq) : Kept{0, 0, 0};
  before = wave_sum(before);
  if (lane == 0) sums[wave] = before;
  const int begin = min(a.n_first, k.pages), end = max(begin, k.pages - k.last);  // pages there is a choice of
  // the smallest weight has the largest key; a NaN counts as the largest weight
  auto key_of_weight = [](float w) { return ~(w == w ? key_of(w) : 0xffffffffu); };
  uint32_t first_key[kKeysPerThread];
#pragma unroll
  for (int j = 0; j < kKeysPerThread; ++j) first_key[j] = key_of_weight(weight[j]);
  auto each = [&](auto f) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < kKeysPerThread; ++j) {
      const int p = tid * kKeysPerThread + j;
      if (p >= begin && p < end) f(first_key[j]);
    }
    constexpr int kAtOnce = 8;                               // loads that are under way together
    for (int p0 = max(begin, kRankRound) + tid; p0 < end; p0 += kAtOnce * kRankThreads) {
      float w[kAtOnce];
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) w[j] = p0 + j * kRankThreads < end ? a.weights[weight_row + p0 + j * kRankThreads] : 0.f;
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j)
        if (p0 + j * kRankThreads < end) f(key_of_weight(w[j]));
    }
  };
  const Threshold t = find_threshold(rank, end - begin, static_cast<uint32_t>(k.gone), each, tid);
  before = (sums[0] + sums[1]) + (sums[2] + sums[3]);
  if (seq >= a.n_seqs - 1 && tid == 0) a.counts[0] = static_cast<int32_t>(before + k.gone);
  if (seq >= a.n_seqs) return;
  if (tid == 0) a.lens_after[seq] = max(0, a.seq_lens[seq]) - k.gone * kGroup;
  if (k.gone == 0 && a.table_after == a.block_table && a.weights_after == a.weights) return;
  Places places;
  for (int base = 0; base < k.pages; base += kRankRound) {
    const int p0 = base + tid * kKeysPerThread;
    if (base > 0) load_round(p0, k.pages);
    bool in[kKeysPerThread], chosen[kKeysPerThread];
    uint32_t v[kKeysPerThread], at[kKeysPerThread];
#pragma unroll
    for (int j = 0; j < kKeysPerThread; ++j) {
      in[j] = p0 + j >= begin && p0 + j < end && k.gone > 0;
      v[j] = in[j] ? key_of_weight(weight[j]) : 0;
    }
    // everybody has read before anybody writes, to where others have read before: what was asked for has come, and all wait for one another in
    // place_keys()
    stores_done();
    place_keys<kKeysPerThread>(rank, places, t, in, v, tid, chosen, at);
#pragma unroll
    for (int j = 0; j < kKeysPerThread; ++j) {
      const int p = p0 + j;
      if (chosen[j]) {
        if (before + at[j] < static_cast<uint32_t>(a.n_freed)) a.freed[before + at[j]] = id[j];
      } else if (p < k.pages) {
        a.table_after[table_row + p - at[j]] = id[j];
        a.weights_after[weight_row + p - at[j]] = weight[j];
      }
    }
  }
  for (int p = k.pages - k.gone + tid; p < k.pages; p += kRankThreads) {
    a.table_after[table_row + p] = -1;
    a.weights_after[weight_row + p] = 0.f;
  }
}

}  // namespace
}  // namespace pq

using namespace pq;

extern "C" int pq_evict_pages(const pq_layout* layout, const int32_t* block_table, int32_t max_pages_per_seq, const int32_t* seq_lens, int32_t n_seqs,
                              const float* weights, int64_t weights_stride, int32_t n_kept, int32_t n_first, int32_t n_last, int32_t* table_after,
                              int32_t* lens_after, float* weights_after, int32_t* freed, int32_t n_freed, int32_t* counts, void* hip_stream) {
  if (!layout) return PQ_ERR_INVALID_ARG;
  if (!layout_supported(layout)) return PQ_ERR_UNSUPPORTED;
  if (n_seqs < 0 || max_pages_per_seq <= 0 || weights_stride < max_pages_per_seq || n_kept < 0 || n_first < 0 || n_last < 0 || n_freed < 0)
    return PQ_ERR_INVALID_ARG;
  if (!counts || (n_seqs > 0 && (!block_table || !seq_lens || !weights || !table_after || !lens_after || !weights_after)) || (n_freed > 0 && !freed))
    return PQ_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(block_table) | reinterpret_cast<uintptr_t>(seq_lens) | reinterpret_cast<uintptr_t>(weights) |
       reinterpret_cast<uintptr_t>(table_after) | reinterpret_cast<uintptr_t>(lens_after) | reinterpret_cast<uintptr_t>(weights_after) |
       reinterpret_cast<uintptr_t>(freed) | reinterpret_cast<uintptr_t>(counts)) & 3u)
    return PQ_ERR_INVALID_ARG;
  if (n_seqs > 0 && lens_after == seq_lens) return PQ_ERR_INVALID_ARG;        // (other work-groups still read what one would write)
  if (n_seqs > 65535) return PQ_ERR_UNSUPPORTED;
  EvictArgs a;
  a.block_table = block_table;
  a.seq_lens = seq_lens;
  a.weights = weights;
  a.table_after = table_after;
  a.lens_after = lens_after;
  a.weights_after = weights_after;
  a.freed = freed;
  a.counts = counts;
  a.weights_stride = weights_stride;
  a.n_seqs = n_seqs;
  a.max_pages_per_seq = max_pages_per_seq;
  a.n_kept = n_kept;
  a.n_first = n_first;
  a.n_last = n_last;
  a.n_freed = n_freed;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  const dim3 grid(static_cast<uint32_t>(std::max(n_seqs, 1)));
  hipLaunchKernelGGL(pq_evict_kernel, grid, dim3(kRankThreads), 0, st, a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? PQ_OK : record_hip_error(e);
}
