// What the host plans a launch of pq_chunk_attention with: which kernel, how many work-groups, and the workspace.  Plain C++: tests
// build it for the CPU.
#pragma once
#include <cmath>

#include "pq_plan.hpp"

namespace pq {
namespace {
namespace chunk {

constexpr int kSharedWaves = 16;                   // of a work-group of the kernel for many rows
constexpr int kSharedRows = 16;                    // of a wavefront
constexpr int kTileRows = kSharedWaves * kSharedRows;
constexpr int kMaxParts = 64;                      // of an item: four a lane when they are joined
constexpr int kFewLeast = 2, kSharedLeast = 4;     // pages of a part

}  // namespace chunk

// A launch: items of 16 rows_of_16 query rows of a KV head; the kernels cut the pages that they see into parts, if `cuts`.
//
// Up to 32 rows a sequence (in the mean) are the few-rows kernel's, which makes its operands for 16 or 32 rows itself; more are the
// shared one's, which unpacks a page once for 256.  16 sequences of 4000 tokens, 4 query heads per KV head, microseconds: 8 new tokens each
// (32 rows) 39, 16 (64 rows) 54, 64 102 -- a page costs the few-rows kernel twice as much for 32 rows as for 16 and would
// cost it again for each 32 more.
struct ChunkLaunch {
  int rows_of_16, tile_tokens, cuts, parts;
  int64_t n_items, n_units;    // of a KV head
  size_t acc_bytes, ml_bytes, bytes;   // of the workspace
};

// Threads of a grid dimension: HIP takes 2^32 - 1.
inline bool launch_fits(const pq_layout* l, const ChunkLaunch& p) {
  return p.n_units * l->n_kv_heads < (int64_t{1} << 32) / (p.rows_of_16 <= 2 ? 256 : 1024);
}

// Pages that an item sees at most, of sequences of seq_pages.
inline int64_t pages_of_item(int64_t seq_pages, int32_t window, int32_t n_sinks, int tile_tokens) {
  if (window == 0) return seq_pages;
  return std::min<int64_t>(seq_pages, (static_cast<int64_t>(n_sinks) + kGroup - 1) / kGroup + (static_cast<int64_t>(window) + tile_tokens) / kGroup + 2);
}

inline size_t round256(size_t n) { return (n + 255) & ~static_cast<size_t>(255); }

inline ChunkLaunch plan_launch(const pq_layout* l, int32_t n_seqs, int32_t n_q_heads, int64_t n_tokens, int64_t max_pages, bool windowed) {
  ChunkLaunch p;
  const int64_t group = n_q_heads / l->n_kv_heads;
  const int64_t rows_16 = (n_tokens * group + 16 * static_cast<int64_t>(n_seqs) - 1) / (16 * static_cast<int64_t>(n_seqs));   // of a sequence, in the mean
  p.rows_of_16 = rows_16 <= 2 ? static_cast<int>(std::max<int64_t>(1, rows_16)) : chunk::kTileRows / 16;
  p.tile_tokens = static_cast<int>(16 * p.rows_of_16 / group);
  p.n_items = std::min<int64_t>(n_tokens, (n_tokens + static_cast<int64_t>(n_seqs) * (p.tile_tokens - 1)) / p.tile_tokens);
  // what the items come to if chunks are alike
  const int64_t of_seq = (n_tokens + n_seqs - 1) / n_seqs, units = n_seqs * ((of_seq + p.tile_tokens - 1) / p.tile_tokens), heads = l->n_kv_heads;
  // Places for parts.  Many rows: empty places cost time, each a compute unit's for what it takes to see that it is empty
  const bool few = p.rows_of_16 <= 2;
  const int64_t rounds = few ? 2 : (n_seqs == 1 ? 8 : (units * heads <= kComputeUnits ? 2 : 4)), places = rounds * kComputeUnits / heads;
  const int64_t least = few ? chunk::kFewLeast : chunk::kSharedLeast;
  // (the workspace's size only grows with the pages, so that it is enough for whatever a window leaves of them)
  p.parts = 0;
  p.cuts = units < places && max_pages > least ? 1 : 0;
  p.n_units = p.cuts ? std::max(p.n_items, std::min(places, p.n_items * std::min<int64_t>((max_pages + least - 1) / least, chunk::kMaxParts))) : p.n_items;
  const size_t rows = p.cuts ? static_cast<size_t>(p.n_units * heads) * 16 * p.rows_of_16 : 0;
  p.acc_bytes = round256(rows * kHeadDim * sizeof(float));
  p.ml_bytes = round256(rows * 2 * sizeof(float));
  p.bytes = std::max<size_t>(256, p.acc_bytes + p.ml_bytes + (p.cuts ? round256(p.n_units * 4 * sizeof(int32_t)) : 0));
  if (few || !p.cuts) return p;
  // Where items are alike as far as the host can tell, no more places than the kernel's rule (judge_cut) would take, if it cuts at all
  if (n_seqs == 1 || windowed || units * heads >= 2 * kComputeUnits) {
    int64_t parts = 1;
    double best = 0.;
    for (int64_t k = 1; k <= std::min<int64_t>({p.n_units / units, (max_pages + least - 1) / least, chunk::kMaxParts}); ++k) {
      const double n = static_cast<double>(units * heads * k) / kComputeUnits;
      const double time = std::ceil(n) * (static_cast<double>(max_pages) / static_cast<double>(k) + 3.) + (k > 1 ? 2. + 3.3 * n : 0.);
      if (k == 1 || time < best) {
        best = time;
        parts = k;
      }
    }
    if (parts == 1) p.cuts = 0;
    else if (n_seqs == 1) p.parts = static_cast<int>(parts);
    p.n_units = std::max(p.n_items, std::min(p.n_units, units * parts));
  }
  return p;
}

// Whether the sequences are taken by their pages: what a wavefront can sort.
inline bool longest_first(const ChunkLaunch& p, int32_t n_seqs) { return p.rows_of_16 > 2 && n_seqs > 1 && n_seqs <= 64; }

}  // namespace
}  // namespace pq
