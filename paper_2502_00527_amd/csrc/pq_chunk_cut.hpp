// How a launch of pq_chunk_attention is shared out, on the device and alike by every wavefront of it.  Only wavefront-wide
// operations and arithmetic: tests run it for 64 lanes on the CPU.  ChunkAttentionArgs and the device functions of
// pq_decode_cut.hpp are declared before it.
#pragma once
#include "pq_chunk_plan.hpp"

namespace pq {
namespace {
namespace chunk {

// Chunks are non-decreasing ranges of [0, n_tokens]; whatever `starts` holds, rows stay within.
__device__ __forceinline__ void chunk_range(const ChunkAttentionArgs& a, int s, int64_t& first, int64_t& end) {
  first = min(max(static_cast<int64_t>(a.starts[s]), int64_t{0}), a.n_tokens);
  end = min(max(static_cast<int64_t>(a.starts[s + 1]), first), a.n_tokens);
}

// ---- how a launch is shared out: by every wavefront alike, a sequence a lane, from what the sequences really hold --------------------
// Items are tiles of tile_tokens of a sequence's chunk; the pages that one sees are cut into parts of alike length, a work-group each, in
// launches that the host lets be cut (plan_launch: few items).  A sequence's tiles are taken to see the same pages, its chunk's last tile's, and have the same
// number of parts: a chunk with little before it sees half of that in the mean.  Lengths are known here only, and max_seq_len may be far
// above them: cut by what there is, and with many rows and up to 64 sequences the longest first, 12 chunks of 1 .. 700 tokens over up to 8192 take 403 us, cut
// by the host as if all were as long as the longest 483; 16 x 5 tokens over 500 .. 6000 41 against 46 (37 now).  Where all are alike
// that costs 1 .. 3 us a work-group (16 x 128 tokens over 4000 164 against 153).
struct Sequence {
  int index, first, n, len;    // its chunk's first row and tokens, its tokens
  int tiles, pages;            // pages: what a tile sees at most
};
__device__ __forceinline__ Sequence sequence_of(const ChunkAttentionArgs& a, int s) {
  Sequence x = {s, 0, 0, 0, 0, 0};
  if (s < a.n_seqs) {
    int64_t first, end;
    chunk_range(a, s, first, end);
    x.first = static_cast<int>(first);                                     // (rows are below 2^31)
    x.n = static_cast<int>(end - first);
    x.len = min(max(a.seq_lens[s], 0), a.max_seq_len);
    x.tiles = static_cast<int>((static_cast<uint32_t>(x.n) + a.tile_tokens - 1) / a.tile_tokens);
    x.pages = pages_of_len(x.len);
    // (the first query's window and the others' tokens: n tokens in a row lie in (n + 126) / 128 + 1 pages at most)
    if (a.window > 0)
      x.pages = min(x.pages, pages_of_len(min(a.n_sinks, x.len)) + static_cast<int>((static_cast<uint32_t>(a.window) + a.tile_tokens + 125u) / kGroup) + 1);
  }
  return x;
}
// Parts of a sequence's items for a longest part of 1 / `cut` pages; 0: one.  (Whatever the rounding, everybody has the same number.)
__device__ __forceinline__ int parts_of(int pages, float cut) { return max(1, static_cast<int>(ceilf(static_cast<float>(pages) * cut))); }
__device__ __forceinline__ float cut_to(int per) { return 0.99999f * __builtin_amdgcn_rcpf(static_cast<float>(per)); }

// Sums and extremes over the launch's sequences; lane sums are cut off at kMost, so that the wavefront's is an int.
constexpr int kMost = 1 << 24;
template <typename F>
__device__ __forceinline__ int total(const ChunkAttentionArgs& a, const Sequence& mine, int lane, F of) {
  int sum = of(mine);
  for (int s0 = 64; s0 < a.n_seqs; s0 += 64) sum = min(sum + of(sequence_of(a, s0 + lane)), kMost);
  return wave_sum(sum);
}
__device__ __forceinline__ int count_units(const ChunkAttentionArgs& a, const Sequence& mine, int lane, float cut) {
  return total(a, mine, lane, [&](const Sequence& x) { return min(x.tiles, kMost / kMaxParts) * parts_of(x.pages, cut); });
}
struct Load {
  int items, work, longest, shortest;              // work: pages of all items, of each 1024 at most (sums stay within 32 bits)
  __device__ __forceinline__ Load(const ChunkAttentionArgs& a, const Sequence& mine, int lane) {
    uint32_t high = mine.tiles > 0 ? mine.pages : 0, low = mine.tiles > 0 ? mine.pages : kMost;
    for (int s0 = 64; s0 < a.n_seqs; s0 += 64) {
      const Sequence x = sequence_of(a, s0 + lane);
      high = max(high, x.tiles > 0 ? static_cast<uint32_t>(x.pages) : 0u);
      low = min(low, x.tiles > 0 ? static_cast<uint32_t>(x.pages) : static_cast<uint32_t>(kMost));
    }
    longest = static_cast<int>(wave_max_u32(high));
    shortest = kMost - static_cast<int>(wave_max_u32(kMost - low));
    items = total(a, mine, lane, [](const Sequence& x) { return x.tiles; });
    work = total(a, mine, lane, [](const Sequence& x) { return min(x.tiles, kMost / 1024) * min(x.pages, 1024); });
  }
};

// Few rows: work-groups that run at once, with parts as alike as can be -- the shortest that fit.  0: no cuts.  Steps from the mean on find
// them where sequences are alike.  A few sequences far above the rest need parts far longer than the mean (one of 1024 pages and 49 of one
// page, 8 KV heads, have 64 places: parts of 69 pages, the mean is 17); those are searched by halves, longer parts never being more.
// 131072 tokens beside 47, 55 and 62 sequences of 120: 116, 198 and 811 us; where the steps found nothing and nothing was cut, 1600.
__device__ __forceinline__ float find_fitting_cut(const ChunkAttentionArgs& a, const Sequence& mine, int lane) {
  const Load load(a, mine, lane);
  const int least = max(kFewLeast, (load.longest + kMaxParts - 1) / kMaxParts);
  if (load.items == 0 || load.items >= a.n_units) return 0.f;
  int per = max(least, static_cast<int>(ceilf(static_cast<float>(load.work) * __builtin_amdgcn_rcpf(static_cast<float>(a.n_units)) * 0.99999f)));
  int fails = per;
  for (int i = 0; i < 16 && per < load.longest; ++i) {
    if (count_units(a, mine, lane, cut_to(per)) <= a.n_units) return cut_to(per);
    fails = per;
    per += 1 + (per >> 4);
  }
  int fits = load.longest;                                                    // (items are fewer than units)
  while (fits - fails > 1 + (fails >> 4)) {
    per = fails + (fits - fails) / 2;
    (count_units(a, mine, lane, cut_to(per)) <= a.n_units ? fits : fails) = per;
  }
  return fits < load.longest ? cut_to(fits) : 0.f;
}
__device__ __forceinline__ float few_cut(const ChunkAttentionArgs& a, const Sequence& mine, int lane) { return a.cuts ? find_fitting_cut(a, mine, lane) : 0.f; }

// Many rows, cut by the host: a.parts of lane 0's sequence, the only one.
__device__ __forceinline__ float cut_alike(const ChunkAttentionArgs& a, const Sequence& mine) {
  const uint32_t parts = static_cast<uint32_t>(a.parts);
  const float cut = cut_to(max(kSharedLeast, static_cast<int>((static_cast<uint32_t>(mine.pages) + parts - 1) / parts)));
  return u2f(static_cast<uint32_t>(uni(static_cast<int>(f2u(cut)))));
}
// Many rows: candidate `index` of 16, and what it takes.  A compute unit has one work-group, and the longest come first: they end together,
// as far as the length of the shortest ones allows.  In pages of time: starting and ending a work-group takes as long as three, writing
// and joining 256 parts as 3.3.
__device__ __forceinline__ float judge_cut(const ChunkAttentionArgs& a, const Sequence& mine, int index, int lane, uint32_t& time) {
  const Load load(a, mine, lane);
  const int least = max(kSharedLeast, (load.longest + kMaxParts - 1) / kMaxParts);
  const float heads = static_cast<float>(a.n_kv_heads) * (1.f / kComputeUnits), longest = static_cast<float>(load.longest), shortest = static_cast<float>(load.shortest);
  // 1 .. 16 parts of the longest items, or, with few items, up to 8 rounds' worth
  const float more = fmaxf(1.f, 0.5f * __builtin_amdgcn_rcpf(fmaxf(static_cast<float>(load.items), 1.f) * heads)), parts = floorf(static_cast<float>(index + 1) * more);
  const float cut = index == 0 ? 0.f : cut_to(max(least, static_cast<int>(ceilf(longest * __builtin_amdgcn_rcpf(parts) * 0.99999f))));
  const int n = count_units(a, mine, lane, cut), parts_long = parts_of(load.longest, cut);
  const float rounds = static_cast<float>(n) * heads;
  const float part_long = longest * __builtin_amdgcn_rcpf(static_cast<float>(parts_long)), part_short = shortest * __builtin_amdgcn_rcpf(static_cast<float>(parts_of(load.shortest, cut)));
  float t = fmaxf(part_long + 3.f, static_cast<float>(load.work) * heads + 3.f * rounds + (ceilf(rounds) - rounds) * (part_short + 3.f));
  if (parts_long > 1) t += 2.f + 3.3f * rounds;
  time = index > 0 && n > a.n_units ? 0x7f000000u : f2u(t);                   // (positive floats are in order as integers)
  return cut;
}
// Times in order, with the candidate they belong to.
__device__ __forceinline__ uint32_t judged(uint32_t time, int index) { return (time & ~15u) | static_cast<uint32_t>(index); }

// A work-group's part of the launch: part `part` of tokens [first, first + count) of a sequence's chunk.
struct Item {
  int seq, first, count;
  int64_t row0;                // of the chunk in q and out
  int len;                     // tokens of the sequence, the chunk with them
  int n;                       // tokens of the chunk
  int unit, part, parts;       // unit: the part's
};

// The sequences by their pages, the longest ones first (n_seqs <= 64): lane l gets the one of rank l.
__device__ __forceinline__ Sequence longest_first(const ChunkAttentionArgs& a, const Sequence& mine, int lane) {
  int rank = lane < a.n_seqs ? 0 : lane;
  for (int s = 0; s < a.n_seqs; ++s) {
    const int other = __builtin_amdgcn_readlane(mine.pages, s);
    if (lane < a.n_seqs) rank += other > mine.pages || (other == mine.pages && s > lane) ? 1 : 0;
  }
  auto to_rank = [&](int x) { return __builtin_amdgcn_ds_permute(4 * rank, x); };
  return {to_rank(mine.index), to_rank(mine.first), to_rank(mine.n), to_rank(mine.len), to_rank(mine.tiles), to_rank(mine.pages)};
}
// Finds part `unit` of the launch: sequences in order, `mine` the lane's of the first 64; the later tiles of one first.
__device__ __forceinline__ bool find_item(const ChunkAttentionArgs& a, const Sequence& mine, float cut, int unit, int lane, Item& item) {
  int before = 0;
  for (int s0 = 0; s0 < a.n_seqs; s0 += 64) {
    const Sequence x = s0 == 0 ? mine : sequence_of(a, s0 + lane);
    const int parts = parts_of(x.pages, cut), units = x.tiles * parts, upto = before + wave_prefix(units);
    const uint64_t past = __builtin_amdgcn_ballot_w64(upto > unit);
    if (past != 0) {
      const int at = __builtin_ctzll(past), place = unit - (__builtin_amdgcn_readlane(upto, at) - __builtin_amdgcn_readlane(units, at));
      item.seq = __builtin_amdgcn_readlane(x.index, at);
      item.unit = unit;
      item.parts = __builtin_amdgcn_readlane(parts, at);
      const int from_last = place / item.parts;
      item.part = place - from_last * item.parts;
      item.row0 = __builtin_amdgcn_readlane(x.first, at);
      item.n = __builtin_amdgcn_readlane(x.n, at);
      item.first = (__builtin_amdgcn_readlane(x.tiles, at) - 1 - from_last) * a.tile_tokens;
      item.count = min(a.tile_tokens, item.n - item.first);
      item.len = __builtin_amdgcn_readlane(x.len, at);
      return true;
    }
    before = __builtin_amdgcn_readlane(upto, 63);
  }
  return false;
}

// Pages that an item's rows see: the sinks' [0, n_first) and [from, from + n_rest).
struct VisiblePages {
  int n_first, from, n_rest;
  __device__ __forceinline__ VisiblePages(const ChunkAttentionArgs& a, const Item& item) : n_first(0), from(0) {
    const int first_position = item.len - item.n + item.first;
    n_rest = pages_of_len(first_position + item.count);
    if (a.window > 0) {
      const int sinks = min(pages_of_len(a.n_sinks), n_rest), begin = max(0, first_position - a.window + 1) / kGroup;
      if (begin > sinks) {
        n_first = sinks;
        from = begin;
        n_rest = max(0, n_rest - begin);
      }
    }
  }
  __device__ __forceinline__ int count() const { return n_first + n_rest; }
  // of the item's parts, the last of which may be shorter or missing
  __device__ __forceinline__ int part_len(const Item& item) const { return max(1, (count() + item.parts - 1) / item.parts); }
};

}  // namespace chunk
}  // namespace
}  // namespace pq
