// The k largest of a list of 32-bit keys, ties to the first ones, by one work-group: where the choice lies, and each key's place in it.
//
// A threshold T and a number n of ties say it: key i is chosen if it is above T, or is T and fewer than n keys before it are.  T is found
// by counting keys in 1024 bins of equal width between the smallest and the largest key, and where the count crosses k, each of that bin's keys against
// each, or, if they are more than 64, in 1024 bins again.  (Scores of one call share their high bits: bins by bits would hold nearly all of them at
// first, and their counters would be one word of LDS.  Weights spread over 30 powers of two put 80 of 900 keys into one of 256 bins: a second
// count.)  A wait of the work-group costs as much as all its arithmetic on a thousand keys:
// there are three, and one more for the places.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace pq {
namespace {

constexpr int kRankThreads = 256;
constexpr int kRankWaves = kRankThreads / 64;
constexpr int kBins = 1024;

// A float as a key that grows with it; -0 is 0.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.f);
  return u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}

// op over the wavefront, in every lane: rotations within the rows of 16 lanes, then rows with rows.
template <int CTRL>
__device__ __forceinline__ uint32_t moved(uint32_t x) {
  return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), CTRL, 0xf, 0xf, true));
}
template <typename Op>
__device__ __forceinline__ uint32_t over_rows(uint32_t x, Op op) {
  auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = op(r[0], r[1]);
  r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return op(r[0], r[1]);
}
template <typename Op>
__device__ __forceinline__ uint32_t over_wave(uint32_t x, Op op) {
  x = op(x, moved<0x128>(x));                                // row_ror 8, 4, 2, 1
  x = op(x, moved<0x124>(x));
  x = op(x, moved<0x122>(x));
  x = op(x, moved<0x121>(x));
  return over_rows(x, op);
}
__device__ __forceinline__ uint32_t wave_min(uint32_t x) { return over_wave(x, [](uint32_t a, uint32_t b) { return min(a, b); }); }
__device__ __forceinline__ uint32_t wave_max(uint32_t x) { return over_wave(x, [](uint32_t a, uint32_t b) { return max(a, b); }); }
__device__ __forceinline__ uint32_t wave_sum(uint32_t x) { return over_wave(x, [](uint32_t a, uint32_t b) { return a + b; }); }
// Sum over this lane and those above it.
__device__ __forceinline__ uint32_t sum_from(uint32_t x, int lane) {
  x += moved<0x101>(x);                                      // row_shl 1, 2, 4, 8: zeros come in
  x += moved<0x102>(x);
  x += moved<0x104>(x);
  x += moved<0x108>(x);
  const uint32_t r1 = __builtin_amdgcn_readlane(x, 16), r2 = __builtin_amdgcn_readlane(x, 32), r3 = __builtin_amdgcn_readlane(x, 48);
  return x + (lane < 16 ? r1 : 0) + (lane < 32 ? r2 : 0) + (lane < 48 ? r3 : 0);
}

struct RankShared {
  __attribute__((aligned(16))) uint32_t hist[kBins];
  __attribute__((aligned(16))) uint32_t low[kRankWaves], high[kRankWaves];
  uint32_t listed;
  uint32_t list[64];
  __attribute__((aligned(16))) uint2 counts[2][kRankWaves];  // chosen surely, ties: of a wavefront's keys
};
static_assert(kBins == 4 * kRankThreads && kRankWaves == 4, "four words together");

struct Threshold {
  uint32_t key, ties;
};

// each(f): f(key) for this thread's share of the `count` keys; called several times.  0 <= k <= count.  All threads of the work-group call it and get the
// result; what they have stored in LDS is there for everybody after the wait that it begins with.
template <typename Each>
__device__ __forceinline__ Threshold find_threshold(RankShared& sh, int count, uint32_t k, Each each, int tid) {
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  uint32_t low = 0xffffffffu, high = 0;
  each([&](uint32_t v) {
    low = min(low, v);
    high = max(high, v);
  });
  low = wave_min(low);
  high = wave_max(high);
  if (lane == 0) {
    sh.low[wave] = low;
    sh.high[wave] = high;
  }
  reinterpret_cast<uint4*>(sh.hist)[tid] = make_uint4(0, 0, 0, 0);
  if (tid == 0) sh.listed = 0;
  __syncthreads();
  if (k == 0) return {0xffffffffu, 0};
  if (k >= static_cast<uint32_t>(count)) return {0, 0xffffffffu};
  const uint4 lows = *reinterpret_cast<const uint4*>(sh.low), highs = *reinterpret_cast<const uint4*>(sh.high);
  uint32_t base = __builtin_amdgcn_readfirstlane(min(min(lows.x, lows.y), min(lows.z, lows.w)));
  uint32_t limit = __builtin_amdgcn_readfirstlane(max(max(highs.x, highs.y), max(highs.z, highs.w))) - base;   // keys base .. base + limit are in question
  while (limit > 0) {
    const int shift = max(0, 22 - __builtin_clz(limit));
    each([&](uint32_t v) {
      const uint32_t off = v - base;
      if (v >= base && off <= limit) atomicAdd(&sh.hist[off >> shift], 1u);
    });
    __syncthreads();
    // every wavefront for itself: the bin where the count from above crosses k
    constexpr int kOwn = kBins / 64;
    uint32_t h[kOwn], sum = 0;
#pragma unroll
    for (int j = 0; j < kOwn; j += 4) {
      const uint4 h4 = *reinterpret_cast<const uint4*>(&sh.hist[lane * kOwn + j]);
      h[j] = h4.x;
      h[j + 1] = h4.y;
      h[j + 2] = h4.z;
      h[j + 3] = h4.w;
      sum += (h4.x + h4.y) + (h4.z + h4.w);
    }
    const uint32_t from = sum_from(sum, lane);
    const int at = __builtin_ctzll(__builtin_amdgcn_ballot_w64(from - sum < k && from >= k));
    // in that lane: how many of its bins are wholly above, which the last bin with k or more from it on tells
    uint32_t above = from - sum, bin = 0, taken = above, inside = 0;
#pragma unroll
    for (int j = kOwn - 1; j >= 0; --j) {
      const bool crossed = above + h[j] >= k;
      bin = max(bin, crossed ? j : 0u);
      inside = crossed ? inside : h[j];
      above += h[j];
      taken = crossed ? taken : above;
    }
    bin = __builtin_amdgcn_readlane(bin, at);
    k -= __builtin_amdgcn_readlane(taken, at);
    inside = sh.hist[at * kOwn + bin];
    inside = __builtin_amdgcn_readfirstlane(inside);
    base += (at * kOwn + bin) << shift;
    if (inside == k) return {base, 0xffffffffu};             // all of the bin: those above its first key, and that one
    limit = (1u << shift) - 1;
    if (limit == 0) break;
    if (inside <= 64) {                                      // few: each against each, in every wavefront
      each([&](uint32_t v) {
        if (v >= base && v - base <= limit) sh.list[atomicAdd(&sh.listed, 1u)] = v;
      });
      __syncthreads();
      const uint32_t mine = static_cast<uint32_t>(lane) < inside ? sh.list[lane] : 0;
      uint32_t larger = 0, equal = 0;
      for (uint32_t j = 0; j < inside; ++j) {
        const uint32_t v = __builtin_amdgcn_readlane(mine, j);
        larger += v > mine;
        equal += v == mine;
      }
      const int here = __builtin_ctzll(__builtin_amdgcn_ballot_w64(static_cast<uint32_t>(lane) < inside && larger < k && larger + equal >= k));
      return {static_cast<uint32_t>(__builtin_amdgcn_readlane(mine, here)), k - __builtin_amdgcn_readlane(larger, here)};
    }
    __syncthreads();                                           // everybody has read the bins
    reinterpret_cast<uint4*>(sh.hist)[tid] = make_uint4(0, 0, 0, 0);
    __syncthreads();
  }
  return {base, k};
}

// Rounds of kRankThreads * kKeys keys in order, thread t's being kKeys t .. of a round: which are chosen, and how many chosen ones are before each.
struct Places {
  uint32_t sure = 0, ties = 0;
  int turn = 0;
};
template <int kKeys>
__device__ __forceinline__ void place_keys(RankShared& sh, Places& p, const Threshold& t, const bool (&in)[kKeys], const uint32_t (&key)[kKeys], int tid,
                                           bool (&chosen)[kKeys], uint32_t (&at)[kKeys]) {
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  bool above[kKeys], tie[kKeys];
  uint32_t sure = 0, ties = 0, all_sure = 0, all_ties = 0;   // before this thread's first key, and of the wavefront
  auto below = [](uint64_t mask, uint32_t add) {             // of the lanes below this one
    return __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(mask >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(mask), add));
  };
#pragma unroll
  for (int j = 0; j < kKeys; ++j) {
    above[j] = in[j] && key[j] > t.key;
    tie[j] = in[j] && key[j] == t.key;
    const uint64_t a = __builtin_amdgcn_ballot_w64(above[j]), b = __builtin_amdgcn_ballot_w64(tie[j]);
    sure = below(a, sure);
    ties = below(b, ties);
    all_sure += __builtin_popcountll(a);
    all_ties += __builtin_popcountll(b);
  }
  if (lane == 0) sh.counts[p.turn][wave] = make_uint2(all_sure, all_ties);
  __syncthreads();
  sure += p.sure;
  ties += p.ties;
#pragma unroll
  for (int w = 0; w < kRankWaves; ++w) {
    const uint2 c = sh.counts[p.turn][w];
    sure += w < wave ? c.x : 0;
    ties += w < wave ? c.y : 0;
    p.sure += c.x;
    p.ties += c.y;
  }
  p.turn ^= 1;
#pragma unroll
  for (int j = 0; j < kKeys; ++j) {
    chosen[j] = above[j] || (tie[j] && ties < t.ties);
    at[j] = sure + min(ties, t.ties);
    sure += above[j];
    ties += tie[j];
  }
}

}  // namespace
}  // namespace pq
