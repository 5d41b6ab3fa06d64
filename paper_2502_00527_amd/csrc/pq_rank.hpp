// The k largest of a list of 32-bit keys, ties to the first ones, by one work-group: where the choice lies, and each key's place in it.
//
// A threshold T and a number n of ties say it: key i is chosen if it is above T, or is T and fewer than n keys before it are.  T is found
// by counting keys in 256 bins of equal width between the smallest and the largest key, then within the bin where
// the count crosses k, and so on: scores of one call share their high bits, so that bins by bits would hold nearly all keys at first
// (and their counters would be one word of LDS).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace pq {
namespace {

constexpr int kBins = 256;

// A float as a key that grows with it; -0 is 0.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.f);
  return u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}

template <int kThreads>
struct RankShared {
  uint32_t hist[kBins];
  uint32_t low[kThreads / 64], high[kThreads / 64];
  uint32_t bin, above, inside;
  uint32_t counts[2][kThreads / 64][2];       // chosen surely, ties: of a wavefront's keys
};

struct Threshold {
  uint32_t key, ties;
};

// key(i), i in [begin, end), is read several times; 0 <= k <= end - begin.  All threads of the work-group call it and get the result.
template <int kThreads, typename Key>
__device__ __forceinline__ Threshold find_threshold(RankShared<kThreads>& sh, int begin, int end, uint32_t k, Key key, int tid) {
  if (k == 0) return {0xffffffffu, 0};
  if (k >= static_cast<uint32_t>(end - begin)) return {0, 0xffffffffu};
  const int lane = tid & 63, wave = tid >> 6;
  uint32_t low = 0xffffffffu, high = 0;
  for (int i = begin + tid; i < end; i += kThreads) {
    const uint32_t v = key(i);
    low = min(low, v);
    high = max(high, v);
  }
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) {
    low = min(low, __shfl_xor(low, d));
    high = max(high, __shfl_xor(high, d));
  }
  if (lane == 0) {
    sh.low[wave] = low;
    sh.high[wave] = high;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    low = min(low, sh.low[w]);
    high = max(high, sh.high[w]);
  }
  uint32_t base = low, limit = high - low;                   // keys base .. base + limit are in question
  while (limit > 0) {
    const int shift = max(0, 24 - __builtin_clz(limit));
    for (int i = tid; i < kBins; i += kThreads) sh.hist[i] = 0;
    __syncthreads();
    for (int i = begin + tid; i < end; i += kThreads) {
      const uint32_t v = key(i), off = v - base;
      if (v >= base && off <= limit) atomicAdd(&sh.hist[off >> shift], 1u);
    }
    __syncthreads();
    if (wave == 0) {
      uint32_t h[kBins / 64], sum = 0;
#pragma unroll
      for (int j = 0; j < kBins / 64; ++j) {
        h[j] = sh.hist[lane * (kBins / 64) + j];
        sum += h[j];
      }
      uint32_t from = sum;                                   // keys of this lane's bins and all above
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const uint32_t other = __shfl_down(from, d);
        from += lane + d < 64 ? other : 0;
      }
      uint32_t above = from - sum;
      if (above < k && from >= k) {                          // in one lane
#pragma unroll
        for (int j = kBins / 64 - 1; j >= 0; --j) {
          if (above < k && above + h[j] >= k) {
            sh.bin = lane * (kBins / 64) + j;
            sh.above = above;
            sh.inside = h[j];
          }
          above += h[j];
        }
      }
    }
    __syncthreads();
    k -= sh.above;
    base += sh.bin << shift;
    if (sh.inside == k) return {base, 0xffffffffu};          // all of the bin: those above its first key, and that one
    limit = (1u << shift) - 1;
  }
  return {base, k};
}

// How many keys before this thread's are chosen, and whether its own is; keys come kThreads at a time in order, thread after thread.
struct Places {
  uint32_t sure = 0, ties = 0;
  int turn = 0;
};
template <int kThreads>
__device__ __forceinline__ uint32_t place(RankShared<kThreads>& sh, Places& p, const Threshold& t, bool in, uint32_t key, int tid, bool& chosen) {
  const int lane = tid & 63, wave = tid >> 6;
  const bool above = in && key > t.key, tie = in && key == t.key;
  const uint64_t a = __builtin_amdgcn_ballot_w64(above), b = __builtin_amdgcn_ballot_w64(tie), before = (uint64_t{1} << lane) - 1;
  if (lane == 0) {
    sh.counts[p.turn][wave][0] = __builtin_popcountll(a);
    sh.counts[p.turn][wave][1] = __builtin_popcountll(b);
  }
  __syncthreads();
  uint32_t sure = p.sure + __builtin_popcountll(a & before), ties = p.ties + __builtin_popcountll(b & before);
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    const uint32_t s = sh.counts[p.turn][w][0], n = sh.counts[p.turn][w][1];
    sure += w < wave ? s : 0;
    ties += w < wave ? n : 0;
    p.sure += s;
    p.ties += n;
  }
  p.turn ^= 1;
  chosen = above || (tie && ties < t.ties);
  return sure + min(ties, t.ties);
}

}  // namespace
}  // namespace pq
