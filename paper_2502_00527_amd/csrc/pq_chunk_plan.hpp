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
// Least pages of a part: what a work-group's start, end and its share of the join cost is worth.  Microseconds with half, these and twice as many, 8 KV heads of
// 4 query heads.  Few rows: 1 token over 1000 11.5, 12.7, 15.6; 8 x 5 over 1000 17.5, 16.1, 20.4; 1 x 3 over 16000 20.9, 20.8, 18.4; 16 x 5 over 500 .. 6000
// 36.8, 37.1, 37.1.  Many rows: 256 tokens over 2000 35.4, 36.4, 39.2; 64 over 16000 62.2, 62.5, 59.9; 512 over 8000 98.7, 98.7, 99.7.
constexpr int kFewLeast = 2, kSharedLeast = 4;

}  // namespace chunk

// A launch: items of 16 rows_of_16 query rows of a KV head; the kernels cut the pages that they see into parts, if `cuts`.
//
// Up to 32 rows a sequence (in the mean) are the few-rows kernel's, which makes its operands for 16 or 32 rows itself; more are the
// shared one's, which unpacks a page once for 256.  16 sequences of 4000 tokens, 4 query heads per KV head, microseconds: 8 new tokens each
// (32 rows) 39, 16 (64 rows) 54, 64 102 -- a page costs the few-rows kernel twice as much for 32 rows as for 16 and would
// cost it again for each 32 more.  The mean decides for the whole batch: 63 single tokens and a chunk of 1024, all over 4000, take 251 (the kernel for
// many rows: a compute unit for 4 rows of each single token), 111 + 111 in two calls; 255 over 1000 and a chunk of 1024 over 4000 291 (the other one, which unpacks
// the chunk's pages 128 times), 121 + 111 in two.
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
  // Places for parts, in rounds of the compute units (few rows: two work-groups share one).  Many rows: empty places cost time, each a compute unit's
  // for what it takes to see that it is empty; one sequence's parts are counted below, and the rounds only bound the workspace.
  // Microseconds with half, these and twice as many rounds, 8 KV heads of 4 query heads:
  //   few rows, 2: 16 x 5 tokens over 500 .. 6000 53.3, 37.1, 44.7; 30 x 1 over 500 .. 3000 44.5, 33.4, 36.3; 4 x 1 over 8000 23.7, 23.0, 29.8; 48 x 5 over
  //     500 .. 16000, 4-bit values, 256, 196, 161
  //   many rows, one sequence, 8: 64 tokens over 16000 63.4, 62.5, 63.3; 512 over 8000 100.6, 98.7, 100.7; 2048 over 32768 1160 each
  //   a compute unit or less each, 2: 12 x 64 over 500 .. 8000, 4-bit values, 101.3, 95.0, 103.0; 8 x 64 over 500 .. 12000 88.2, 86.5, 90.0; 16 x 128 over 4000 156.7, 161.6, 169.1
  //   more, 4: 12 x 1 .. 700 over up to 8192, 3+3 bits, 4-bit values, 307, 308, 316; 40 x 64 over 500 .. 8000 283.6, 287.3, 289.2
  // Batches of as many units as places are not cut, whatever the lengths (few rows: 64 sequences with 8 KV heads).  One sequence of 131072 tokens beside 55 and
  // 63 of 120, a new token each: 201 and 1606; 63 and 64 x 5 tokens over 500 .. 32000 457 and 506.  The join would cost every one of them 5.
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
