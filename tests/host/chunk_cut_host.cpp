// CPU run of how a launch of pq_chunk_attention is shared out (csrc/pq_chunk_cut.hpp) with the host's plan (csrc/pq_chunk_plan.hpp),
// for tests: the 64 lanes of a wavefront of cut_host.cpp.
#include "cut_host.cpp"

#include <cmath>

// lane l's value goes to lane address / 4, each to one of its own
inline int amd_ds_permute(int address, int x) {
  int found = 0;
  for (int from = 0; from < lanes::kLanes; ++from) {
    const int to = amd_readlane(address, from) / 4, value = amd_readlane(x, from);
    if (to == lanes::current) found = value;
  }
  return found;
}
#define __builtin_amdgcn_ds_permute amd_ds_permute

#include "pq_chunk_plan.hpp"

namespace pq {
inline uint32_t f2u(float x) { uint32_t u; memcpy(&u, &x, 4); return u; }
inline float u2f(uint32_t u) { float x; memcpy(&x, &u, 4); return x; }
struct ChunkAttentionArgs {
  const int32_t *starts, *seq_lens;
  int64_t n_tokens;
  int32_t n_seqs, n_kv_heads, max_seq_len, window, n_sinks, tile_tokens, n_units, cuts, parts;
};
}  // namespace pq

#include "pq_chunk_cut.hpp"

// A launch's plan and the units of one KV head.
//   plan[0..7]: rows of an item / 16, tokens of one, whether items may be cut, into how many parts the host has cut, items, units,
//     bytes of the workspace, whether the longest sequences come first
//   units[8 u ..]: sequence (-1: unit u has nothing), first token of the chunk, tokens, part, parts, pages seen, first page of the part, pages
// Returns the number of units.
extern "C" int chunk_cut_host(int n_seqs, int n_kv_heads, int n_q_heads, int64_t n_tokens, const int32_t* starts, const int32_t* lens, int max_seq_len,
                              int window, int n_sinks, float error, int64_t* plan, int32_t* units) {
  using namespace pq;
  using namespace pq::chunk;
  reciprocal_error = error;
  pq_layout layout = {};
  layout.head_dim = kHeadDim;
  layout.r_bits = layout.t_bits = 4;
  layout.group_tokens = kGroup;
  layout.n_kv_heads = n_kv_heads;
  if (window >= max_seq_len) window = 0;
  n_sinks = window > 0 ? std::min(n_sinks, max_seq_len) : 0;
  const int64_t seq_pages = (static_cast<int64_t>(max_seq_len) + kGroup - 1) / kGroup;
  const ChunkLaunch most = plan_launch(&layout, n_seqs, n_q_heads, n_tokens, seq_pages, false);
  const ChunkLaunch p = plan_launch(&layout, n_seqs, n_q_heads, n_tokens, pages_of_item(seq_pages, window, n_sinks, most.tile_tokens), window > 0);
  if (p.bytes > most.bytes) lanes::fail("a window's workspace is larger than the whole sequences'");
  const bool sorted = longest_first(p, n_seqs);
  const int64_t values[8] = {p.rows_of_16, p.tile_tokens, p.cuts, p.parts, p.n_items, p.n_units, static_cast<int64_t>(most.bytes), sorted};
  std::copy(values, values + 8, plan);
  ChunkAttentionArgs a = {};
  a.starts = starts;
  a.seq_lens = lens;
  a.n_tokens = n_tokens;
  a.n_seqs = n_seqs;
  a.n_kv_heads = n_kv_heads;
  a.max_seq_len = max_seq_len;
  a.window = window;
  a.n_sinks = n_sinks;
  a.tile_tokens = p.tile_tokens;
  a.n_units = static_cast<int32_t>(p.n_units);
  a.cuts = p.cuts;
  a.parts = p.parts;
  lanes::run([&](int lane) {
    Sequence mine = sequence_of(a, lane);
    const float cut = p.rows_of_16 <= 2 ? few_cut(a, mine, lane) : (a.parts > 0 ? cut_alike(a, mine) : 0.f);
    float chosen = cut;
    if (p.rows_of_16 > 2 && a.parts == 0 && a.cuts) {
      uint32_t least = ~0u;
      for (int index = 0; index < kSharedWaves; ++index) {            // (a wavefront each, on the card)
        uint32_t time;
        const float candidate = judge_cut(a, mine, index, lane, time);
        if (judged(time, index) < least) least = judged(time, index), chosen = candidate;
      }
    }
    if (sorted) mine = longest_first(a, mine, lane);
    for (int u = 0; u < a.n_units; ++u) {
      Item item;
      const bool there = find_item(a, mine, chosen, u, lane, item);
      if (lane != 0) continue;
      int32_t* const to = units + 8 * u;
      to[0] = -1;
      if (!there) continue;
      const VisiblePages pages(a, item);
      const int part_len = pages.part_len(item), begin = item.part * part_len, end = min(begin + part_len, pages.count());
      const int32_t found[8] = {item.seq, item.first, item.count, item.part, item.parts, pages.count(), begin, max(0, end - begin)};
      std::copy(found, found + 8, to);
    }
  });
  return a.n_units;
}
