// Choice of pages by a cheap score of the queries against the pages' bounds (pq_select_pages), and attention over the chosen
// ones (pq_sparse_attention).
//
// The score of a page is, block of 32 channels by block, q8 . c + |q8| . w in whole numbers -- {c, w} of a block being 64 bytes, the
// depth of one matrix instruction, in the order it reads them -- times the block's
// scales in fp32; whole numbers below 2^24 and fp32 operations that are rounded one by one make it the same for whoever computes it.
// The instruction takes 16 pages and 16 rows: four heads of block 0, of block 1, ..., with zeros in the rows of other blocks, so that one accumulator has
// the four blocks' sums of four heads, a block in each row of lanes.  Adding blocks up is then two swaps of rows, which serve four tiles of 16
// pages at once and leave each lane the score of one page: 80 instructions for 64 pages and four heads, where an accumulator a block took 300.
//
// Few (sequence, KV head) units with many pages share a unit's pages among work-groups: one compute unit has about 60 lines of 128 bytes
// under way, and 1024 pages of 272 bytes took one 9.5 us.  The keys go to the workspace past the caches, and whoever registers last at the unit's
// arrival word makes the choice (pq_decode_sched.hpp): one launch, nobody waits for anybody.
//
// Bound: waits for memory and for one another, one after the other -- table, bounds, keys of the other work-groups, counts.  One sequence of 1024 pages (8 KV
// heads) 8.0 us, 32 ragged ones of up to 256 6.7, a launch's own time being 3.6; 32 of 1024 pages, 72 MB, 22.
//
// The grid runs over sequences first: work-groups go round the 8 dies, so that those of one sequence tend to start on one die where n_seqs is a multiple of 8, on two or four of them where it
// has a factor of 4 or 2, and its cache keeps lines that heads share, the block table's and the scales' (16 bytes a head).  64 sequences of 256 pages 12.0 -> 10.3 us, 16 of 1024
// 14.5 -> 12.5, 32 ragged ones of up to 256 7.3 -> 6.7.  Other numbers of 256 pages: 60 10.0 us where 64 take 10.0, 20 6.7, 13 6.6 where 16 take 6.6.
//
// A choice is a row of a block table: page and KV head are one index into the pools taken head by head, so that attention over the
// chosen pages is decode attention of n_seqs * n_kv_heads sequences with one KV head each.
#include <hip/hip_runtime.h>

#include "pq_decode_sched.hpp"
#include "pq_internal.hpp"
#include "pq_rank.hpp"

#pragma clang fp contract(off)

namespace pq {
namespace {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

constexpr int kBoundBytes = 4 * kPairs;                      // of a page and head
constexpr int kBlockBytes = kBoundBytes / kBlocks;
constexpr float kTiny = 0x1p-100f;
constexpr int kMostKeys = 8192;                              // pages whose keys stay in LDS
constexpr int kTilePages = 16;                               // of a matrix instruction

struct SelectArgs {
  const void* q;
  const int8_t* bounds;
  const float* scales;
  const int32_t* block_table;
  const int32_t* seq_lens;
  int32_t* selected;
  int32_t* selected_lens;
  uint64_t* arrivals;                                        // one word a unit; of units shared among work-groups
  uint32_t* keys;                                            // [unit][key_stride], of the same
  int32_t n_pool_pages;
  int32_t n_kv_heads, group, max_pages_per_seq, max_seq_len, max_pages;
  int32_t n_selected, n_first, n_last;
  int32_t key_stride;                                        // a multiple of 4
  int32_t part_pages;                                        // pages of a work-group; max_pages at least: of all
  int32_t q_is_f32;
};

__device__ __forceinline__ int clamped(const SelectArgs& a, int seq) { return max(0, min(a.seq_lens[seq], a.max_seq_len)); }
__device__ __forceinline__ int pages_up(int tokens) { return tokens / kGroup + (tokens % kGroup != 0); }

// The queries of a KV head as operands.  Lane l has head 4 s + l % 4 of set s, block (l / 4) % 4, and of its 16 pairs part l / 16: x, y, |x| or |y|.
// Heads past the last are that one again.
template <int kSets>
struct Query {
  i32x4 code[kSets];
  float largest;                                             // of block l / 16, any head

  u32x4 w[kSets][4];                                         // as they lie in memory
  __device__ __forceinline__ void fetch(const SelectArgs& a, int64_t head0, int lane) {
    const int per_row = a.q_is_f32 ? kHeadDim * 4 : kHeadDim * 2, per_part = per_row / 8;
#pragma unroll
    for (int s = 0; s < kSets; ++s) {
      const int64_t head = head0 + min(4 * s + (lane & 3), a.group - 1);
      const u32x4* const src = reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(a.q) + head * per_row + ((lane >> 4) & 1) * (per_row / 2) + ((lane >> 2) & 3) * per_part);
      w[s][0] = src[0];
      w[s][1] = src[1];
      w[s][2] = src[a.q_is_f32 ? 2 : 0];                     // (fp16: not looked at)
      w[s][3] = src[a.q_is_f32 ? 3 : 0];
    }
  }
  template <bool kF32>
  __device__ __forceinline__ float value(int s, int i) const {
    if constexpr (kF32) return u2f(w[s][i / 4][i % 4]);
    else return static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(w[s][i / 8][i / 2 % 4] >> (16 * (i & 1)))));
  }
  template <bool kF32>
  __device__ __forceinline__ void make(int lane) {
    float m = 0.f;
#pragma unroll
    for (int s = 0; s < kSets; ++s)
#pragma unroll
      for (int i = 0; i < 16; ++i) m = fmaxf(m, fabsf(value<kF32>(s, i)));
    uint32_t bits = __builtin_bit_cast(uint32_t, m);         // (not negative: in the order of its bits)
    bits = max(bits, moved<0xb1>(bits));                     // over the block's heads (quad_perm) and parts
    bits = max(bits, moved<0x4e>(bits));
    bits = over_rows(bits, [](uint32_t x, uint32_t y) { return max(x, y); });
    m = __builtin_bit_cast(float, bits);
    const uint32_t m0 = __builtin_amdgcn_readlane(bits, 0), m1 = __builtin_amdgcn_readlane(bits, 4), m2 = __builtin_amdgcn_readlane(bits, 8),
                   m3 = __builtin_amdgcn_readlane(bits, 12);
    largest = u2f(lane & 32 ? (lane & 16 ? m3 : m2) : (lane & 16 ? m1 : m0));
    const float up = m >= kTiny ? 127.0f / m : 0.f;
    const uint32_t sign = lane < 32 ? 0xffffffffu : 0x7fffffffu;
#pragma unroll
    for (int s = 0; s < kSets; ++s)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t word = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float r = rintf(value<kF32>(s, 4 * i + j) * up);
          word |= (static_cast<uint32_t>(static_cast<int>(__builtin_bit_cast(float, __builtin_bit_cast(uint32_t, r) & sign))) & 255u) << (8 * j);
        }
        code[s][i] = static_cast<int>(word);
      }
  }
  __device__ __forceinline__ i32x4 operand(int s, int b, int lane) const {
    const bool here = ((lane >> 2) & 3) == b;
    return i32x4{here ? code[s].x : 0, here ? code[s].y : 0, here ? code[s].z : 0, here ? code[s].w : 0};
  }
};

// Pages first .. first + 15 of a sequence: lane l has page l % 16's block-table entry, part l / 16 of its bounds' blocks, and the scale of block l / 16.
struct Tile {
  int32_t id;
  i32x4 bound[kBlocks];
  float scale;
  __device__ __forceinline__ bool there(const SelectArgs& a) const { return id >= 0 && id < a.n_pool_pages; }
  // (p < a.max_pages is in the row whatever the sequence's length)
  __device__ __forceinline__ void load_id(const SelectArgs& a, const int32_t* row, int p) { id = p < a.max_pages ? row[p] : -1; }
  __device__ __forceinline__ void load(const SelectArgs& a, int kvh, int lane) {
    const int64_t ph = there(a) ? id * a.n_kv_heads + kvh : 0;                     // (below 2^31: checked on the host)
    const int8_t* const from = a.bounds + ph * kBoundBytes + (lane >> 4) * 16;
#pragma unroll
    for (int i = 0; i < kBlocks; ++i) bound[i] = *reinterpret_cast<const i32x4*>(from + i * kBlockBytes);
    scale = a.scales[ph * kBlocks + (lane >> 4)];
  }
};
// Tiles of a wavefront whose loads are under way together: a block-table entry and then the bounds are two waits for memory, for all of them.
constexpr int kTilesAtOnce = 4;
constexpr int kBatchPages = kRankWaves * kTilesAtOnce * kTilePages;                // of a work-group

// The key of page 16 (l / 16) + l % 16 of the tiles in lane l (l / 16 modulo kTiles).
template <int kTiles, int kSets>
__device__ __forceinline__ uint32_t tile_keys(const Tile (&tile)[kTiles], const Query<kSets>& q, const SelectArgs& a, int lane) {
  const int row = lane >> 4;
  float best = -INFINITY;
#pragma unroll
  for (int s = 0; s < kSets; ++s) {
    float t[kTiles][4];                                      // [tile][head 4 s + i], of block `row` and page l % 16
    i32x4 n[kTiles];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) {
      const i32x4 x = q.operand(s, b, lane);
#pragma unroll
      for (int j = 0; j < kTiles; ++j) n[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(x, tile[j].bound[b], b == 0 ? i32x4{0, 0, 0, 0} : n[j], 0, 0, 0);
    }
#pragma unroll
    for (int j = 0; j < kTiles; ++j) {
      const float u = q.largest * tile[j].scale;
#pragma unroll
      for (int i = 0; i < 4; ++i) t[j][i] = static_cast<float>(n[j][i]) * u;
    }
    // blocks 0 + 1 and 2 + 3, then those: row r keeps tile r's
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float first = tsum16(t[0][i], t[1 % kTiles][i]), second = kTiles == 4 ? tsum16(t[2 % kTiles][i], t[3 % kTiles][i]) : first;
      best = fmaxf(best, tsum32(first, second));
    }
  }
  bool there = tile[0].there(a);
  if constexpr (kTiles == 2) there = row & 1 ? tile[1].there(a) : there;
  if constexpr (kTiles == 4) there = row < 2 ? (row == 0 ? there : tile[1].there(a)) : (row == 2 ? tile[2].there(a) : tile[3].there(a));
  return key_of(there ? best : -INFINITY);
}

// kTiles: of a wavefront at once.  kSets: of four query heads.  kKeys: keys of a thread when the choice is made: 1, where a batch is all there is -- every
// thread has scored one page -- or 4.
template <int kTiles, int kSets, int kKeys>
__global__ __launch_bounds__(kRankThreads) void pq_select_kernel(const SelectArgs a) {
  constexpr int kPartPages = kRankWaves * kTiles * kTilePages, kRound = kRankThreads * kKeys;
  constexpr int kAtOnce = 4;                                 // reads of four keys that are under way together
  static_assert(kKeys == 1 || kKeys == 4, "one page a thread, or a 128-bit read");
  static_assert(kKeys != 1 || kTiles == kTilesAtOnce, "a page a thread");
  __shared__ RankShared rank;
  __shared__ __attribute__((aligned(16))) uint32_t in_lds[kKeys == 1 ? 4 : kMostKeys];
  __shared__ int stage;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), kvh = blockIdx.y, seq = blockIdx.x, part = blockIdx.z;
  const int64_t unit = static_cast<int64_t>(seq) * a.n_kv_heads + kvh;
  const int32_t* const row = a.block_table + static_cast<int64_t>(seq) * a.max_pages_per_seq;
  int32_t* const out = a.selected + unit * a.n_selected;
  // the page's row in the pools taken head by head
  auto name = [&](int32_t page) { return page >= 0 && page < a.n_pool_pages ? page * a.n_kv_heads + kvh : -1; };
  Tile tile[kTiles];
  const int part0 = part * a.part_pages, first = part0 + wave * (kTiles * kTilePages);
#pragma unroll
  for (int j = 0; j < kTiles; ++j) tile[j].load_id(a, row, first + j * kTilePages + (lane & 15));
  Query<kSets> q;
  q.fetch(a, unit * a.group, lane);
  const int len = clamped(a, seq), pages = pages_up(len);
  if (pages <= a.n_selected) {
    if (part != 0) return;
    for (int p = tid; p < a.n_selected; p += kRankThreads) out[p] = p < pages ? name(row[p]) : -1;
    if (tid == 0) a.selected_lens[unit] = len;
    return;
  }
  if (part0 >= pages) return;
  const int parts = (pages + a.part_pages - 1) / a.part_pages, part_end = min(pages, part0 + a.part_pages);
  const int begin = a.n_first, end = pages - a.n_last;       // pages there is a choice of
  const bool shared = kKeys != 1 && parts > 1, in_memory = shared && pages > kMostKeys;
  const __amdgpu_buffer_rsrc_t r_keys = make_rsrc(a.keys + (shared ? unit * a.key_stride : 0), shared ? static_cast<uint32_t>(pages) * 4u : 0u);
  auto stored = [&](int p0) { return __builtin_amdgcn_raw_buffer_load_b128(r_keys, p0 * 4, 0, kAuxDevice); };
  uint32_t own = 0;                                          // kKeys == 1: page tid's
  for (int done = 0; part0 + done < part_end; done += kPartPages) {
    if (done > 0) {
#pragma unroll
      for (int j = 0; j < kTiles; ++j) tile[j].load_id(a, row, done + first + j * kTilePages + (lane & 15));
    }
#pragma unroll
    for (int j = 0; j < kTiles; ++j) tile[j].load(a, kvh, lane);
    if (done == 0) {
      if (a.q_is_f32) q.template make<true>(lane);
      else q.template make<false>(lane);
    }
    const uint32_t k = tile_keys<kTiles, kSets>(tile, q, a, lane);
    const int p = done + first + lane;
    if constexpr (kKeys == 1) {
      own = k;
    } else if (lane < kTiles * kTilePages && p < part_end) {
      if (shared) __builtin_amdgcn_raw_buffer_store_b32(k, r_keys, p * 4, 0, kAuxDevice);
      else in_lds[p] = k;
    }
  }
  if (shared) {
    stores_done();
    __syncthreads();
    if (tid == 0) stage = arrive(a.arrivals + unit, parts) ? 1 : 0;
    __syncthreads();
    if (stage == 0) return;
    if (tid == 0) reset_arrivals(a.arrivals + unit);
    if (!in_memory) {
      for (int p0 = tid * 4; p0 < pages; p0 += kAtOnce * kRound) {                 // (zeros behind the last)
        u32x4 k[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) k[j] = stored(p0 + j * kRound);
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j)
          if (p0 + j * kRound < pages) *reinterpret_cast<u32x4*>(&in_lds[p0 + j * kRound]) = k[j];
      }
    }
  }
  int32_t id[kKeys];
#pragma unroll
  for (int j = 0; j < kKeys; ++j) id[j] = tid * kKeys + j < pages ? row[tid * kKeys + j] : -1;
  if constexpr (kKeys != 1) __syncthreads();
  auto four = [&](int p0) { return in_memory ? stored(p0) : *reinterpret_cast<const u32x4*>(&in_lds[p0]); };
  auto each = [&](auto f) __attribute__((always_inline)) {
    if constexpr (kKeys == 1) {
      if (tid >= begin && tid < end) f(own);
    } else {
#pragma unroll 2
      for (int p0 = tid * 4; p0 < end; p0 += kRound) {
        const u32x4 k = four(p0);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (p0 + j >= begin && p0 + j < end) f(k[j]);
      }
    }
  };
  const Threshold t = find_threshold(rank, end - begin, static_cast<uint32_t>(a.n_selected - a.n_first - a.n_last), each, tid);
  Places places;
  for (int base = 0; base < pages; base += kRound) {
    const int p0 = base + tid * kKeys;
    bool in[kKeys], chosen[kKeys];
    uint32_t k[kKeys], at[kKeys];
    u32x4 now = {0, 0, 0, 0};
    if constexpr (kKeys != 1) {
      if (p0 < pages) now = four(p0);
    }
#pragma unroll
    for (int j = 0; j < kKeys; ++j) {
      in[j] = p0 + j >= begin && p0 + j < end;
      k[j] = kKeys == 1 ? own : now[j];
      if (base > 0) id[j] = p0 + j < pages ? row[p0 + j] : -1;
    }
    place_keys<kKeys>(rank, places, t, in, k, tid, chosen, at);
#pragma unroll
    for (int j = 0; j < kKeys; ++j) {
      const int p = p0 + j, to = chosen[j] ? a.n_first + static_cast<int>(at[j]) : (p < begin ? p : (p >= end ? a.n_selected - pages + p : -1));
      if (to >= 0 && p < pages) out[to] = name(id[j]);
    }
  }
  if (tid == 0) a.selected_lens[unit] = len - (pages - a.n_selected) * kGroup;
}

template <int kTiles, int kKeys>
void launch_select(const SelectArgs& a, dim3 grid, hipStream_t st) {
  if (a.group <= 4) hipLaunchKernelGGL((pq_select_kernel<kTiles, 1, kKeys>), grid, dim3(kRankThreads), 0, st, a);
  else if (a.group <= 8) hipLaunchKernelGGL((pq_select_kernel<kTiles, 2, kKeys>), grid, dim3(kRankThreads), 0, st, a);
  else hipLaunchKernelGGL((pq_select_kernel<kTiles, 4, kKeys>), grid, dim3(kRankThreads), 0, st, a);
}

int64_t most_pages(int32_t max_seq_len) { return (static_cast<int64_t>(max_seq_len) + kGroup - 1) / kGroup; }

// Pages of a work-group: all of a unit's, if that is one batch of loads a wavefront or the units fill the compute units; otherwise as few as make
// no more than a work-group a compute unit, or a batch.  (8 units of 1024 pages 8.2 us, a work-group each 15.6; 128 of 512 10.5 and 11.5; 256 of 512 12.3 and 12.4, of 1024 21.7 and 22.0; 512 of 512 22.1
// and 20.7, 1024 of 312 29.0 and 25.8.
// With twice as many work-groups 32 units of 1024 pages 10.7 instead of 9.3.)
// All of these are of equal lengths, and the rule knows no others: it goes by max_seq_len.  256 units of which 8 have 4096 pages and the others 64 take 52 us, the 8 alone 16.
int32_t pages_of_part(const pq_layout* l, int32_t n_seqs, int32_t max_seq_len) {
  const int64_t pages = most_pages(max_seq_len), units = static_cast<int64_t>(n_seqs) * l->n_kv_heads;
  if (pages <= kBatchPages || (units >= kComputeUnits && pages <= kMostKeys)) return static_cast<int32_t>(std::min<int64_t>(pages, kMostKeys));
  for (int tiles = 1; tiles < kTilesAtOnce; tiles *= 2) {
    const int part = kRankWaves * tiles * kTilePages;
    if (units * ((pages + part - 1) / part) <= kComputeUnits) return part;
  }
  return kBatchPages;
}
bool shares_units(const pq_layout* l, int32_t n_seqs, int32_t max_seq_len) { return pages_of_part(l, n_seqs, max_seq_len) < most_pages(max_seq_len); }

int check_selection(const pq_layout* l, int32_t n_seqs, int32_t n_q_heads, int32_t max_seq_len, int32_t n_selected, int32_t n_first, int32_t n_last) {
  if (!l || n_seqs <= 0 || n_q_heads <= 0 || max_seq_len <= 0) return PQ_ERR_INVALID_ARG;
  if (l->n_kv_heads <= 0 || n_q_heads % l->n_kv_heads != 0) return PQ_ERR_INVALID_ARG;
  if (n_first < 0 || n_last < 1 || static_cast<int64_t>(n_first) + n_last > n_selected) return PQ_ERR_INVALID_ARG;
  if (!layout_supported(l)) return PQ_ERR_UNSUPPORTED;
  if (n_q_heads / l->n_kv_heads > 16 || static_cast<int64_t>(n_seqs) * l->n_kv_heads > 65535) return PQ_ERR_UNSUPPORTED;
  if (most_pages(max_seq_len) > 65535 * int64_t{kBatchPages}) return PQ_ERR_UNSUPPORTED;      // grid.z, and a count of 16 bits at an arrival word
  return PQ_OK;
}

int64_t key_stride(int32_t max_seq_len) { return (most_pages(max_seq_len) + 3) & ~int64_t{3}; }
size_t round256(size_t n) { return (n + 255) & ~static_cast<size_t>(255); }
size_t arrival_bytes(const pq_layout* l, int32_t n_seqs) { return round256(static_cast<size_t>(n_seqs) * l->n_kv_heads * sizeof(uint64_t)); }
// The arrival words, then the keys: as many bytes as a batch of no more sequences and pages may need.  Units of up to kMostKeys pages are shared in batches of fewer
// than kComputeUnits units only, so that a smaller batch may need more than this one.
size_t select_bytes(const pq_layout* l, int32_t n_seqs, int32_t max_seq_len) {
  const int64_t most_seqs = most_pages(max_seq_len) > kMostKeys ? n_seqs : std::min<int64_t>(n_seqs, (kComputeUnits - 1) / l->n_kv_heads);
  if (most_seqs == 0 || !shares_units(l, static_cast<int32_t>(most_seqs), max_seq_len)) return 256;
  return arrival_bytes(l, static_cast<int32_t>(most_seqs)) + round256(static_cast<size_t>(most_seqs) * l->n_kv_heads * key_stride(max_seq_len) * sizeof(uint32_t));
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
  a.arrivals = static_cast<uint64_t*>(workspace);
  a.keys = reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(workspace) + (shares_units(l, n_seqs, max_seq_len) ? arrival_bytes(l, n_seqs) : 0));
  a.n_pool_pages = static_cast<int32_t>(n_pool_pages);
  a.n_kv_heads = l->n_kv_heads;
  a.group = n_q_heads / l->n_kv_heads;
  a.max_pages_per_seq = max_pages_per_seq;
  a.max_seq_len = max_seq_len;
  a.max_pages = static_cast<int32_t>(most_pages(max_seq_len));
  a.n_selected = n_selected;
  a.n_first = n_first;
  a.n_last = n_last;
  a.q_is_f32 = q_dtype == PQ_F32 ? 1 : 0;
  a.key_stride = static_cast<int32_t>(key_stride(max_seq_len));
  a.part_pages = pages_of_part(l, n_seqs, max_seq_len);
  const dim3 grid(n_seqs, l->n_kv_heads, (a.max_pages + a.part_pages - 1) / a.part_pages);
  if (a.max_pages <= kBatchPages) launch_select<kTilesAtOnce, 1>(a, grid, st);
  else if (a.part_pages == kBatchPages / 4) launch_select<1, 4>(a, grid, st);
  else if (a.part_pages == kBatchPages / 2) launch_select<2, 4>(a, grid, st);
  else launch_select<kTilesAtOnce, 4>(a, grid, st);
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
  const size_t attention = alike_workspace_bytes(&one, n_seqs * layout->n_kv_heads, n_q_heads / layout->n_kv_heads, chosen_tokens(max_seq_len, n_selected));
  return attention == 0 ? 0 : select_bytes(layout, n_seqs, max_seq_len) + attention;
}

extern "C" int pq_sparse_attention(const pq_layout* layout, const void* q, pq_dtype q_dtype, int32_t n_seqs, int32_t n_q_heads, const void* codes_pool,
                                   const void* params_pool, const void* v_pool, int32_t v_bits, const void* v_params_pool, const void* bounds,
                                   const void* bound_scales, int64_t n_pool_pages, const int32_t* block_table, int32_t max_pages_per_seq,
                                   const int32_t* seq_lens, int32_t max_seq_len, int32_t n_selected, int32_t n_first, int32_t n_last, float sm_scale,
                                   int32_t* selected, int32_t* selected_lens, float* out, const void* residual_keys, void* workspace,
                                   size_t workspace_bytes, void* hip_stream) {
  if (!out || (reinterpret_cast<uintptr_t>(out) & 15u)) return PQ_ERR_INVALID_ARG;
  // a choice that is given needs neither bounds nor the table, lengths are its own, and which pages were sure to be in it is of no account
  const bool given = !bounds && !bound_scales;
  int st = check_selection(layout, n_seqs, n_q_heads, max_seq_len, n_selected, given ? 0 : n_first, given ? 1 : n_last);
  if (st == PQ_OK)
    st = check_selection_pointers(layout, q, q_dtype, given ? q : bounds, given ? q : bound_scales, n_pool_pages, given ? selected : block_table,
                                  given ? INT32_MAX : max_pages_per_seq, given ? selected_lens : seq_lens, max_seq_len, selected, selected_lens);
  if (st != PQ_OK) return st;
  const pq_layout one = one_head(layout);
  const int32_t rows = n_seqs * layout->n_kv_heads, heads = n_q_heads / layout->n_kv_heads, tokens = chosen_tokens(max_seq_len, n_selected);
  const int64_t row_pages = n_pool_pages * layout->n_kv_heads;
  st = check_attention(&one, q, q_dtype, rows, heads, codes_pool, params_pool, v_pool, v_bits, v_params_pool, row_pages, selected, n_selected, selected_lens,
                       tokens, sm_scale, residual_keys);
  if (st != PQ_OK) return st;
  const size_t before = select_bytes(layout, n_seqs, max_seq_len), attention = alike_workspace_bytes(&one, rows, heads, tokens);
  if (attention == 0) return PQ_ERR_UNSUPPORTED;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) || workspace_bytes < before + attention) return PQ_ERR_WORKSPACE;
  if (!given) {
    st = launch_selection(layout, q, q_dtype, n_seqs, n_q_heads, bounds, bound_scales, n_pool_pages, block_table, max_pages_per_seq, seq_lens, max_seq_len,
                          n_selected, n_first, n_last, selected, selected_lens, workspace, static_cast<hipStream_t>(hip_stream));
    if (st != PQ_OK) return st;
  }
  return attend_alike(&one, q, q_dtype, rows, heads, codes_pool, params_pool, v_pool, v_bits, v_params_pool, row_pages, selected, n_selected, selected_lens,
                      tokens, sm_scale, out, residual_keys, static_cast<uint8_t*>(workspace) + before, workspace_bytes - before, static_cast<hipStream_t>(hip_stream));
}
