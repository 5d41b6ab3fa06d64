// Attention of a batch's chunks of new tokens over the packed cache (pq_chunk_attention), on the matrix cores.
//
// For KV head k, token i of a sequence's chunk and query head h of the G that read k, row (i, h):
//     out = sum_t p_t V_t / sum_t p_t,   p_t = exp2(scale q . k~_t - m),   t over the tokens the row sees:
//     t <= position(i), and with a window t > position(i) - window or t < n_sinks
// One pass over the keys with a running m and l (online softmax).
//
// Operands.  Both products are v_mfma_f32_16x16x32_f16 with the query rows as columns: S^T = K~ Q^T, 16 tokens x 16 rows, then
// O^T = V^T P^T, 16 dims x 16 rows.  The accumulator of the first (lane = row l % 16, tokens 4 (l / 16) .. + 3) is, for two
// tiles of 16 tokens, the second one's operand as it lies, and a row's maximum and sum belong to four lanes; the order of
// the summed index is free, so keys come as they are packed -- lane (token l % 16, pair block l / 16) has the unit with its
// 16 pairs, four pairs (x, y) an instruction -- and values as whole rows, lane (slice of 8 dims l % 16, tokens 4 (l / 16) .. + 3 of
// both tiles): dim e of every slice is one instruction.
//
// Rounding.  Queries are fp16; reconstructed keys, probabilities and de-quantized values are rounded to fp16 for the
// matrix unit, like the output: each 2^-12 of itself in the mean, where the cache's own quantization is 2^-4.  Sums, m and l are
// fp32.  Probabilities are taken times 2^kLift, so that weights down to 2^-21 of the largest keep all their bits.
// m is raised only when a score is 2^(15 - kLift) above it (the product then still fits fp16), and then by all lanes of the row.
#pragma once
#include "pq_decode_matrix.hpp"

namespace pq {

struct ChunkAttentionArgs {
  const __half* q;             // [n_tokens][n_q_heads][d]
  const uint8_t* codes;
  const uint32_t* params;
  const void* values;
  const uint32_t* v_params;
  const __half* residual;
  const int32_t* block_table;
  const int32_t* starts;
  const int32_t* seq_lens;     // with the chunk
  __half* out;                 // [n_tokens][n_q_heads][d]
  float* ws_acc;               // [item][KV head][split][row][d], un-normalised
  float* ws_ml;                // [item][KV head][split][row][2]
  int64_t n_tokens;
  int64_t n_pool_pages;
  int32_t n_seqs;
  int32_t n_kv_heads;
  int32_t n_q_heads;
  int32_t group;               // query heads per KV head
  int32_t max_pages_per_seq;
  int32_t max_seq_len;
  int32_t window;              // 0: none
  int32_t n_sinks;
  int32_t tile_tokens;         // of an item
  int32_t n_items;             // at most
  int32_t n_splits;            // of an item's pages
  int32_t table_index;
  float scale_log2;            // > 0
  int32_t negate;              // the queries
};

// Launchers, one for each value width (pq_chunk_attention.hip): rows_of_16 is 1 or 4.  False: no such kernel.
bool launch_chunk_v16(const pq_layout* l, int rows_of_16, const ChunkAttentionArgs& a, dim3 grid, hipStream_t st);
bool launch_chunk_v4(const pq_layout* l, int rows_of_16, const ChunkAttentionArgs& a, dim3 grid, hipStream_t st);
bool launch_chunk_v2(const pq_layout* l, int rows_of_16, const ChunkAttentionArgs& a, dim3 grid, hipStream_t st);

namespace {
namespace chunk {

constexpr int kLift = 7;
constexpr float kSlack = 15.f - kLift;

// A work-group's part of the launch: tokens [first, first + count) of a sequence's chunk.
struct Item {
  int seq, first, count;
  int64_t row0;                // of the chunk in q and out
  int len;                     // tokens of the sequence, the chunk with them
  int n;                       // tokens of the chunk
};

// Chunks are non-decreasing ranges of [0, n_tokens]; whatever `starts` holds, rows stay within.
__device__ __forceinline__ void chunk_range(const ChunkAttentionArgs& a, int s, int64_t& first, int64_t& end) {
  first = min(max(static_cast<int64_t>(a.starts[s]), int64_t{0}), a.n_tokens);
  end = min(max(static_cast<int64_t>(a.starts[s + 1]), first), a.n_tokens);
}

// Finds item `index`: sequences in order, each one's tiles in order.  Every wavefront does it for itself, 64 sequences at a time.
__device__ __forceinline__ bool find_item(const ChunkAttentionArgs& a, int index, int lane, Item& item) {
  int before = 0;
  for (int s0 = 0; s0 < a.n_seqs; s0 += 64) {
    const int s = s0 + lane;
    int64_t first = 0, end = 0;
    if (s < a.n_seqs) chunk_range(a, s, first, end);
    const int tiles = static_cast<int>((static_cast<uint32_t>(end - first) + a.tile_tokens - 1) / a.tile_tokens);
    const int upto = before + wave_prefix(tiles);
    const uint64_t past = __builtin_amdgcn_ballot_w64(upto > index);
    if (past != 0) {
      const int at = __builtin_ctzll(past);
      item.seq = s0 + at;
      const int tile = index - (__builtin_amdgcn_readlane(upto, at) - __builtin_amdgcn_readlane(tiles, at));
      chunk_range(a, item.seq, first, end);
      item.row0 = first;
      item.n = static_cast<int>(end - first);
      item.first = tile * a.tile_tokens;
      item.count = min(a.tile_tokens, item.n - item.first);
      item.len = min(max(a.seq_lens[item.seq], 0), a.max_seq_len);
      return true;
    }
    before = __builtin_amdgcn_readlane(upto, 63);
  }
  return false;
}

// Pages that an item's rows see: the sinks' [0, n_first) and [from, from + n_rest).
struct VisiblePages {
  int n_first, from, n_rest;
  __device__ __forceinline__ int count() const { return n_first + n_rest; }
};
__device__ __forceinline__ VisiblePages visible_pages(const ChunkAttentionArgs& a, int first_position, int last_position) {
  VisiblePages v = {0, 0, pages_of_len(last_position + 1)};
  if (a.window > 0) {
    const int sinks = min(pages_of_len(a.n_sinks), v.n_rest);
    const int begin = max(0, first_position - a.window + 1) / kGroup;
    if (begin > sinks) v = {sinks, begin, max(0, v.n_rest - begin)};
  }
  return v;
}

// ---- keys: an operand of 16 tokens x 4 pairs of each block, from the packed units ------------------
__device__ __forceinline__ f16x2 low2(f16x2 v) { return f16x2{v.x, v.x}; }
__device__ __forceinline__ f16x2 high2(f16x2 v) { return f16x2{v.y, v.y}; }

// Uniform grid: k~ = s (c' cos, c' sin) + z (cos, sin), the two vectors a function of the packed symbol: an 8-byte table entry, kept 32
// times in LDS (row of a symbol 256 bytes), which lane l reads in column l % 32: no bank conflicts.  Two packed instructions a pair.
template <int W>
struct UniformKeys {
  static constexpr int kLdsBytes = (1 << W) * kTableRow;
  uint32_t lane_lut, table;
  __device__ __forceinline__ void init(const uint8_t* lds, int, int lane) {
    table = lds_addr(lds);
    lane_lut = (lane & 31) * 8;
  }
  // by the whole work-group of NT threads; a barrier must follow
  template <int NT>
  static __device__ __forceinline__ void fill(uint8_t* lds, int table_index, int tid) {
    constexpr int kCopies = 32 * (1 << W) / NT;
    const uint4 entry = fetch_key_entry<W>(key_table<W>(table_index), tid);
    const f16x2 unscale = {static_cast<_Float16>(1.f / (1 << kTableShift)), static_cast<_Float16>(1.f / (1 << kTableShift))};
    const u32x2 word = {h2u(u2h(entry.x) * unscale), h2u(u2h(entry.y) * unscale)};
    uint8_t* const row = lds + (tid & ((1 << W) - 1)) * kTableRow;
    const int first = tid + (tid >> W) * kCopies;
#pragma unroll
    for (int i = 0; i < kCopies; ++i) *reinterpret_cast<u32x2*>(row + ((first + i) & 31) * 8) = word;
  }
  __device__ __forceinline__ void page(uint32_t, int) {}
  // word e: (x, y) of pair 4 KS + e of the lane's block
  template <int KS>
  __device__ __forceinline__ f16x8 operand(const Unit<W / 2>& u, const uint32_t (&params)[16]) const {
    uint32_t w[4];
    auto one = [&](auto e_) {
      constexpr int e = decltype(e_)::value, K = 4 * KS + e;
      uint32_t addr;
      if constexpr (W == 8) {
        addr = __builtin_amdgcn_perm(u.d[K >> 2], lane_lut, 0x0c0c0000u | ((4u + (K & 3)) << 8)) + table;
      } else {
        addr = (symbol<W, K>(u) << 8) + (lane_lut + table);
      }
      const u32x2 t = *(const PQ_LDS u32x2*)static_cast<uintptr_t>(addr);
      const f16x2 sz = u2h(params[K]);
      w[e] = h2u(__builtin_elementwise_fma(u2h(t.x), low2(sz), u2h(t.y) * high2(sz)));
    };
    one(std::integral_constant<int, 0>{});
    one(std::integral_constant<int, 1>{});
    one(std::integral_constant<int, 2>{});
    one(std::integral_constant<int, 3>{});
    return as_operand(w[0], w[1], w[2], w[3]);
  }
};

// Grouped quantizer: the angle levels belong to the page, whose (cos, sin) each wavefront keeps as fp16 in a table of its own:
// row of pair j, 2^t states, 4 bytes each.
template <int RB, int TB>
struct GroupedKeys {
  static constexpr int W = RB + TB, NA = 1 << TB;
  static constexpr int kLdsBytes = kPairs * NA * 4;          // of a wavefront
  uint32_t table, row;
  __device__ __forceinline__ void init(const uint8_t* lds, int wave, int lane) {
    table = lds_addr(lds) + wave * kLdsBytes;
    row = table + (lane >> 4) * (16 * NA * 4);
  }
  template <int NT>
  static __device__ __forceinline__ void fill(uint8_t*, int, int) {}
  // angle: {fp16 s, fp16 z} of pair `lane`
  __device__ __forceinline__ void page(uint32_t angle, int lane) {
    wave_lds_sync();                                         // the page before has been read
    const float level = static_cast<float>(lane & (NA - 1)) + 0.5f;
    constexpr int kPairsAtOnce = 64 >> TB;
#pragma unroll
    for (int it = 0; it < NA; ++it) {
      const f16x2 sz = u2h(static_cast<uint32_t>(__shfl(static_cast<int>(angle), it * kPairsAtOnce + (lane >> TB))));
      const float turns = fmaf(level, static_cast<float>(sz.x), static_cast<float>(sz.y)) * 0.15915494309189535f;
      *(PQ_LDS uint32_t*)static_cast<uintptr_t>(table + it * 256 + lane * 4) = h2u(to_half2(__builtin_amdgcn_cosf(turns), __builtin_amdgcn_sinf(turns)));
    }
    wave_lds_sync();
  }
  template <int KS>
  __device__ __forceinline__ f16x8 operand(const Unit<W / 2>& u, const uint32_t (&params)[16]) const {
    uint32_t w[4];
    auto one = [&](auto e_) {
      constexpr int e = decltype(e_)::value, K = 4 * KS + e;
      const uint32_t sym = symbol<W, K>(u);
      const uint32_t trig = *(const PQ_LDS uint32_t*)static_cast<uintptr_t>(row + K * (NA * 4) + (sym >> RB) * 4);
      // c + 1/2 exactly: 1024 + c as fp16, less 1023.5
      const uint32_t c = sym & ((1u << RB) - 1u);
      const f16x2 sz = u2h(params[K]);
      const _Float16 level = __builtin_bit_cast(_Float16, static_cast<uint16_t>(c | 0x6400u)) - static_cast<_Float16>(1023.5f);
      const _Float16 rho = __builtin_fmaf16(level, sz.x, sz.y);
      w[e] = h2u(u2h(trig) * f16x2{rho, rho});
    };
    one(std::integral_constant<int, 0>{});
    one(std::integral_constant<int, 1>{});
    one(std::integral_constant<int, 2>{});
    one(std::integral_constant<int, 3>{});
    return as_operand(w[0], w[1], w[2], w[3]);
  }
};

// Un-quantized keys of the residual group, as operands: coordinates x, y of the same four pairs from two places of a row.
__device__ __forceinline__ f16x8 residual_operand(__amdgpu_buffer_rsrc_t rows, uint32_t offset) {
  const u32x2 x = __builtin_amdgcn_raw_buffer_load_b64(rows, offset, 0, kAuxCached), y = __builtin_amdgcn_raw_buffer_load_b64(rows, offset, kPairs * 2, kAuxCached);
  return as_operand(__builtin_amdgcn_perm(y.x, x.x, 0x05040100u), __builtin_amdgcn_perm(y.x, x.x, 0x07060302u),
                    __builtin_amdgcn_perm(y.y, x.y, 0x05040100u), __builtin_amdgcn_perm(y.y, x.y, 0x07060302u));
}

// ---- values: what a lane loads of 32 tokens (its tokens 4 (l / 16) .. + 3 of both tiles, its slice of 8 dims), and operand e of them ----
template <int VB>
struct Values;
template <>
struct Values<16> {
  static constexpr uint32_t kPageBytes = kGroup * kHeadDim * 2;
  uint4 row[8];
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t rv, __amdgpu_buffer_rsrc_t, int step, int lane) {
    const uint32_t voff = (lane >> 4) * 1024 + (lane & 15) * 16;
#pragma unroll
    for (int j = 0; j < 8; ++j) row[j] = buf_load16<kAuxCached>(rv, voff, (32 * step + 16 * (j >> 2) + (j & 3)) * 256);
  }
  template <int E>
  __device__ __forceinline__ f16x8 operand() const {
    auto word = [&](int j) { return E / 2 == 0 ? row[j].x : (E / 2 == 1 ? row[j].y : (E / 2 == 2 ? row[j].z : row[j].w)); };
    constexpr uint32_t kPick = E & 1 ? 0x07060302u : 0x05040100u;
    return as_operand(__builtin_amdgcn_perm(word(1), word(0), kPick), __builtin_amdgcn_perm(word(3), word(2), kPick),
                      __builtin_amdgcn_perm(word(5), word(4), kPick), __builtin_amdgcn_perm(word(7), word(6), kPick));
  }
};
// Quantized values: V~ = code s + z, two tokens a word.  A masked code with the exponent of 1024 is 1024 + code, exactly.
template <int VB>
struct Values {
  static constexpr uint32_t kPageBytes = kGroup * kHeadDim * VB / 8;
  uint32_t word[2][VB];                            // of a tile: VB = 4: [token pair][dims 0-3, 4-7]; VB = 2: [token pair]
  uint32_t par[2][4];                              // {s, z} of the four tokens; paired(): {s, s}, {z, z} of two tokens
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t rv, __amdgpu_buffer_rsrc_t rvp, int step, int lane) {
    const uint32_t quarter = lane >> 4, slice = lane & 15;
#pragma unroll
    for (int tile = 0; tile < 2; ++tile) {
      const u32x4 p = __builtin_amdgcn_raw_buffer_load_b128(rvp, quarter * 16, (32 * step + 16 * tile) * 4, kAuxCached);
      par[tile][0] = p.x; par[tile][1] = p.y; par[tile][2] = p.z; par[tile][3] = p.w;
      if constexpr (VB == 4) {
        const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(rv, quarter * 256 + slice * 16, (8 * step + 4 * tile) * 256, kAuxCached);
        word[tile][0] = v.x; word[tile][1] = v.y; word[tile][2] = v.z; word[tile][3] = v.w;
      } else {
        const u32x2 v = __builtin_amdgcn_raw_buffer_load_b64(rv, (quarter >> 1) * 256 + slice * 16 + (quarter & 1) * 8, (4 * step + 2 * tile) * 256, kAuxCached);
        word[tile][0] = v.x; word[tile][1] = v.y;
      }
    }
  }
  template <int E>
  __device__ __forceinline__ f16x8 operand() const {
    uint32_t w[4];
#pragma unroll
    for (int tile = 0; tile < 2; ++tile)
#pragma unroll
      for (int pair = 0; pair < 2; ++pair) {
        const uint32_t x = VB == 4 ? word[tile][2 * pair + E / 4] : word[tile][pair];
        constexpr int kShift = VB == 4 ? 4 * (E % 4) : 2 * E;
        constexpr uint32_t kMask = ((1u << VB) - 1u) * 0x10001u;
        const f16x2 code = u2h(((x >> kShift) & kMask) | 0x64006400u) - f16x2{static_cast<_Float16>(1024.f), static_cast<_Float16>(1024.f)};
        const f16x2 s = u2h(__builtin_amdgcn_perm(par[tile][2 * pair + 1], par[tile][2 * pair], 0x05040100u));
        const f16x2 z = u2h(__builtin_amdgcn_perm(par[tile][2 * pair + 1], par[tile][2 * pair], 0x07060302u));
        w[2 * tile + pair] = h2u(__builtin_elementwise_fma(code, s, z));
      }
    return as_operand(w[0], w[1], w[2], w[3]);
  }
};

template <int N, typename F>
__device__ __forceinline__ void unrolled(F f) {
  if constexpr (N > 0) {
    unrolled<N - 1>(f);
    f(std::integral_constant<int, N - 1>{});
  }
}

// ---- the kernel's body --------------------------------------------------------------------------------
// A work-group serves 16 RT rows of one KV head; its four wavefronts take the pages in turn and are folded at the end.
constexpr int kChunkWaves = 4;

template <typename Keys, int W, bool kGrouped, int VB, int RT>
__device__ __forceinline__ void attention_body(const ChunkAttentionArgs& a) {
  constexpr uint32_t kCodesBytes = kBlocks * kGroup * 2 * W;
  constexpr uint32_t kParamWords = kPairs * (kGrouped ? 2 : 1);
  constexpr int kTableBytes = Keys::kLdsBytes * (kGrouped ? kChunkWaves : 1);
  constexpr int kFoldBytes = 2 * RT * 8 * 64 * 16;
  __shared__ __attribute__((aligned(16))) uint8_t lds[kTableBytes > kFoldBytes ? kTableBytes : kFoldBytes];
  __shared__ float fold_m[kChunkWaves][RT * 16], fold_l[kChunkWaves][RT * 16];
  const int tid = threadIdx.x, wave = uni(tid >> 6), lane = tid & 63, quarter = lane >> 4, col = lane & 15;
  const int kvh = blockIdx.x % a.n_kv_heads, index = a.n_items - 1 - blockIdx.x / a.n_kv_heads;   // later tokens, which see more, first
  const int split = blockIdx.y;
  Item item;
  if (!find_item(a, index, lane, item)) return;
  const int first_position = item.len - item.n + item.first, last_position = first_position + item.count - 1;
  const VisiblePages pages = visible_pages(a, first_position, last_position);
  const int per = whole_rounds((pages.count() + a.n_splits - 1) / a.n_splits);
  const int begin = split * per, end = min(begin + per, pages.count());
  if (split > 0 && begin >= end) return;

  Keys::template fill<kChunkWaves * 64>(lds, a.table_index, tid);
  Keys keys;
  keys.init(lds, wave, lane);

  // the rows of this lane's columns, their positions, and their queries as operands
  int position[RT];
  f16x8 q[RT][4];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int row = 16 * rt + col, token = row / a.group, head = row - token * a.group;
    const bool there = token < item.count;
    position[rt] = there ? first_position + token : INT32_MAX;
    const __half* const at = a.q + ((item.row0 + item.first + (there ? token : 0)) * a.n_q_heads + kvh * a.group + (there ? head : 0)) * kHeadDim;
    const uint32_t sign = a.negate ? 0x80008000u : 0u;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      u32x2 x, y;
      __builtin_memcpy(&x, at + 16 * quarter + 4 * ks, 8);
      __builtin_memcpy(&y, at + kPairs + 16 * quarter + 4 * ks, 8);
      q[rt][ks] = as_operand(__builtin_amdgcn_perm(y.x, x.x, 0x05040100u) ^ sign, __builtin_amdgcn_perm(y.x, x.x, 0x07060302u) ^ sign,
                             __builtin_amdgcn_perm(y.y, x.y, 0x05040100u) ^ sign, __builtin_amdgcn_perm(y.y, x.y, 0x07060302u) ^ sign);
    }
  }
  const int tail_page = a.residual != nullptr && item.len % kGroup != 0 ? item.len / kGroup : -1;
  const __amdgpu_buffer_rsrc_t tail_rows = make_rsrc(a.residual + (static_cast<int64_t>(item.seq) * a.n_kv_heads + kvh) * (kGroup * kHeadDim),
                                                     tail_page >= 0 ? static_cast<uint32_t>(item.len % kGroup) * (kHeadDim * 2) : 0u);
  // a row's largest score so far (times the scale), as the lane's exponent offset kLift - m; -inf: nothing seen
  float m[RT], l[RT];
  f32x4 acc[8][RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    m[rt] = kNegInf;
    l[rt] = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e][rt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  __syncthreads();

  const int32_t* const table = a.block_table + static_cast<int64_t>(item.seq) * a.max_pages_per_seq;
  const uint32_t voff_codes = (quarter * kGroup + col) * (2 * W);
  for (int at = begin + wave; at < end; at += kChunkWaves) {
    const int page = uni(at < pages.n_first ? at : pages.from + at - pages.n_first);
    const int id = page < a.max_pages_per_seq ? uni(table[page]) : -1;
    if (id < 0 || id >= a.n_pool_pages) continue;                        // masked
    const int64_t ph = static_cast<int64_t>(id) * a.n_kv_heads + kvh;
    const bool packed = page != tail_page;
    const int nv = min(kGroup, item.len - page * kGroup);
    const __amdgpu_buffer_rsrc_t rc = make_rsrc(a.codes + ph * kCodesBytes, packed ? kCodesBytes : 0u);
    const __amdgpu_buffer_rsrc_t rp = make_rsrc(a.params + ph * kParamWords, packed ? kParamWords * 4u : 0u);
    const __amdgpu_buffer_rsrc_t rv = make_rsrc(static_cast<const uint8_t*>(a.values) + ph * Values<VB>::kPageBytes,
                                                VB == 16 ? static_cast<uint32_t>(nv) * (kHeadDim * 2) : Values<VB>::kPageBytes);
    const __amdgpu_buffer_rsrc_t rvp = make_rsrc(a.v_params + (VB == 16 ? 0 : ph * kGroup), VB == 16 ? 0u : static_cast<uint32_t>(nv) * 4u);
    uint32_t params[16];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint4 p = buf_load16<kAuxCached>(rp, quarter * 64, i * 16);
      params[4 * i] = p.x; params[4 * i + 1] = p.y; params[4 * i + 2] = p.z; params[4 * i + 3] = p.w;
    }
    if constexpr (kGrouped) keys.page(buf_load4<kAuxCached>(rp, lane * 4, kPairs * 4), lane);
    Unit<W / 2> units[8];
#pragma unroll
    for (int t = 0; t < 8; ++t) units[t] = load_unit<W>(rc, voff_codes, static_cast<uint32_t>(16 * t) * (2 * W));
    // whether some row does not see all of the page
    const int page_end = page * kGroup + kGroup - 1;
    const bool masks = page_end > first_position || (a.window > 0 && last_position - a.window >= page * kGroup && page_end >= a.n_sinks);
#pragma unroll
    for (int step = 0; step < 4; ++step) {
      Values<VB> v;
      v.load(rv, rvp, step, lane);
      f32x4 s[2][RT];
#pragma unroll
      for (int tile = 0; tile < 2; ++tile) {
        const int t = 2 * step + tile;
        f16x8 k_op[4];
        if (packed) {
          unrolled<4>([&](auto ks) { k_op[ks] = keys.template operand<decltype(ks)::value>(units[t], params); });
        } else {
#pragma unroll
          for (int ks = 0; ks < 4; ++ks) k_op[ks] = residual_operand(tail_rows, (16 * t + col) * (kHeadDim * 2) + quarter * 32 + ks * 8);
        }
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
            s[tile][rt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k_op[ks], q[rt][ks], ks == 0 ? zero : s[tile][rt], 0, 0, 0);
          }
      }
      if (masks) {
#pragma unroll
        for (int tile = 0; tile < 2; ++tile)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int token = page * kGroup + 32 * step + 16 * tile + 4 * quarter + i;
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
              bool seen = token <= position[rt];
              if (a.window > 0) seen = seen && (position[rt] - token < a.window || token < a.n_sinks);
              if (!seen) s[tile][rt][i] = kNegInf;
            }
          }
      }
      float top[RT];
      bool above = false;
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        float x = max3(s[0][rt][0], s[0][rt][1], s[0][rt][2]);
        x = max3(x, s[0][rt][3], s[1][rt][0]);
        x = max3(x, s[1][rt][1], s[1][rt][2]);
        top[rt] = max2(x, s[1][rt][3]) * a.scale_log2;
        above = above || top[rt] > m[rt] + kSlack;
      }
      if (__builtin_amdgcn_ballot_w64(above) != 0) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          float x = top[rt];
          auto r = __builtin_amdgcn_permlane16_swap(f2u(x), f2u(x), false, false);
          x = max2(u2f(r[0]), u2f(r[1]));
          auto r2 = __builtin_amdgcn_permlane32_swap(f2u(x), f2u(x), false, false);
          x = max3(u2f(r2[0]), u2f(r2[1]), m[rt]);
          const float keep = x > kNegInf ? __builtin_amdgcn_exp2f(m[rt] - x) : 1.f;
          m[rt] = x;
          l[rt] *= keep;
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[e][rt] *= keep;
        }
      }
      f16x8 p_op[RT];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const float off = m[rt] > kNegInf ? kLift - m[rt] : 0.f;
        uint32_t w[4];
#pragma unroll
        for (int tile = 0; tile < 2; ++tile)
#pragma unroll
          for (int pair = 0; pair < 2; ++pair) {
            const f16x2 p = to_half2(__builtin_amdgcn_exp2f(fmaf(s[tile][rt][2 * pair], a.scale_log2, off)),
                                     __builtin_amdgcn_exp2f(fmaf(s[tile][rt][2 * pair + 1], a.scale_log2, off)));
            w[2 * tile + pair] = h2u(p);
            l[rt] = __builtin_amdgcn_fdot2(p, f16x2{static_cast<_Float16>(1.f), static_cast<_Float16>(1.f)}, l[rt], false);
          }
        p_op[rt] = as_operand(w[0], w[1], w[2], w[3]);
      }
      unrolled<8>([&](auto e) {
        const f16x8 v_op = v.template operand<decltype(e)::value>();
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) acc[e][rt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v_op, p_op[rt], acc[e][rt], 0, 0, 0);
      });
    }
  }

  // ---- fold the wavefronts ----
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    l[rt] = sum_rows(l[rt]);
    if (quarter == 0) {
      fold_m[wave][16 * rt + col] = m[rt];
      fold_l[wave][16 * rt + col] = l[rt];
    }
  }
  __syncthreads();                                                       // (the keys' table is free, too)
  float top[RT], total[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    top[rt] = kNegInf;
    total[rt] = 0.f;
#pragma unroll
    for (int w = 0; w < kChunkWaves; ++w) top[rt] = fmaxf(top[rt], fold_m[w][16 * rt + col]);
#pragma unroll
    for (int w = 0; w < kChunkWaves; ++w)
      total[rt] += top[rt] > kNegInf ? fold_l[w][16 * rt + col] * __builtin_amdgcn_exp2f(fold_m[w][16 * rt + col] - top[rt]) : 0.f;
    const float weight = top[rt] > kNegInf ? __builtin_amdgcn_exp2f(m[rt] - top[rt]) : 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e][rt] *= weight;
  }
  f32x4* const part = reinterpret_cast<f32x4*>(lds);
#pragma unroll
  for (int half = 2; half >= 1; half >>= 1) {
    if (wave >= half && wave < 2 * half) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) part[((wave - half) * 8 * RT + e * RT + rt) * 64 + lane] = acc[e][rt];
    }
    __syncthreads();
    if (wave < half) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) acc[e][rt] += part[(wave * 8 * RT + e * RT + rt) * 64 + lane];
    }
    __syncthreads();
  }
  if (wave != 0) return;
  // lane: dims 32 quarter + 8 i + e of its rows
  if (a.n_splits > 1) {
    const int64_t slot = (static_cast<int64_t>(index) * a.n_kv_heads + kvh) * a.n_splits + split;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int64_t row = slot * (16 * RT) + 16 * rt + col;
      float* const to = a.ws_acc + row * kHeadDim + 32 * quarter;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        *reinterpret_cast<f32x4*>(to + 8 * i) = f32x4{acc[0][rt][i], acc[1][rt][i], acc[2][rt][i], acc[3][rt][i]};
        *reinterpret_cast<f32x4*>(to + 8 * i + 4) = f32x4{acc[4][rt][i], acc[5][rt][i], acc[6][rt][i], acc[7][rt][i]};
      }
      if (quarter == 0) {
        a.ws_ml[row * 2] = top[rt];
        a.ws_ml[row * 2 + 1] = total[rt];
      }
    }
    return;
  }
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int row = 16 * rt + col, token = row / a.group, head = row - token * a.group;
    if (token >= item.count) continue;
    const float inv = total[rt] > 0.f ? 1.f / total[rt] : 0.f;
    __half* const to = a.out + ((item.row0 + item.first + token) * a.n_q_heads + kvh * a.group + head) * kHeadDim + 32 * quarter;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<u32x4*>(to + 8 * i) = u32x4{h2u(to_half2(acc[0][rt][i] * inv, acc[1][rt][i] * inv)), h2u(to_half2(acc[2][rt][i] * inv, acc[3][rt][i] * inv)),
                                                    h2u(to_half2(acc[4][rt][i] * inv, acc[5][rt][i] * inv)), h2u(to_half2(acc[6][rt][i] * inv, acc[7][rt][i] * inv))};
  }
}

// ---- many rows: operands shared through LDS -------------------------------------------------------------------
// A work-group of 16 wavefronts serves up to 256 rows of one KV head.  Each page is unpacked once: wavefront w makes half of the key
// operands of tile w / 2 (16 tokens), and of the value operands of step w / 4 (32 tokens) half of the dims of one of the two tiles, and
// stores them as the matrix instructions read them, 16 bytes a lane, while everybody computes with the page before; one barrier a
// page.  A wavefront has 16 rows, or, where the work-group has fewer, shares them with others that take other tokens.
//
// The score product carries the scale (in the keys) and, as what its accumulators start from, kLift - m: what comes out is the
// exponent.  Sums of weights are a matrix product too, with ones.
//
// Four wavefronts a SIMD, 128 registers each: while one waits for its matrix instructions or its LDS reads the others' exponentials
// (16 cycles each, the largest part of the vector unit's work) run.
constexpr int kSharedWaves = 16;
constexpr int kSharedRows = 16;                    // of a wavefront
constexpr int kTileRows = kSharedWaves * kSharedRows;
constexpr int kImage = kGroup * kHeadDim * 2;      // bytes of a page's key or value operands

// Key coordinates are made in fp32 and rounded once.  trig<K>(): scale times (cos, sin) of the angle level of pair K (of the 8 that a
// lane has).
template <int RB, int TB>
struct SharedUniformKeys {
  static constexpr int W = RB + TB, NA = 1 << TB;
  static constexpr int kLdsBytes = NA * 256;       // 32 copies of an entry: no bank conflicts
  static constexpr bool kGrouped = false;
  uint32_t lane_at;
  __device__ __forceinline__ void init(const uint8_t* lds, float scale, int tid) {
    const uint32_t table = lds_addr(lds);
    lane_at = table + (tid & 31) * 8;
    for (int i = tid; i < NA * 32; i += kSharedWaves * 64) {
      const float angle = ((static_cast<float>(i >> 5) + 0.5f) * (1.f / NA) - 0.5f) * 6.283185307179586f;
      *(PQ_LDS f32x2*)static_cast<uintptr_t>(table + i * 8) = f32x2{cosf(angle) * scale, sinf(angle) * scale};
    }
  }
  __device__ __forceinline__ void build(uint32_t, int, int) {}
  template <int K>
  __device__ __forceinline__ f32x2 trig(uint32_t angle, int) const { return *(const PQ_LDS f32x2*)static_cast<uintptr_t>(lane_at + angle * 256); }
};
// Grouped quantizer: the page's levels, as fp16, made by the work-group for the page after the next (two tables).
template <int RB, int TB>
struct SharedGroupedKeys {
  static constexpr int W = RB + TB, NA = 1 << TB;
  static constexpr int kPageBytes = kPairs * NA * 4;
  static constexpr int kLdsBytes = 2 * kPageBytes;
  static constexpr bool kGrouped = true;
  uint32_t table, row;
  float scale;
  __device__ __forceinline__ void init(const uint8_t* lds, float scale_, int tid) {
    table = lds_addr(lds);
    row = table + (((tid & 63) >> 4) * 16 + ((tid >> 6) & 1) * 8) * (NA * 4);
    scale = scale_;
  }
  // angle: {fp16 s, fp16 z} of pair `lane`
  __device__ __forceinline__ void build(uint32_t angle, int parity, int tid) {
    const int lane = tid & 63, wave = uni(tid >> 6);
    const float level = static_cast<float>(lane & (NA - 1)) + 0.5f;
    constexpr int kPairsAtOnce = 64 >> TB;
    for (int it = wave; it < NA; it += kSharedWaves) {
      const f16x2 sz = u2h(static_cast<uint32_t>(__shfl(static_cast<int>(angle), it * kPairsAtOnce + (lane >> TB))));
      const float turns = fmaf(level, static_cast<float>(sz.x), static_cast<float>(sz.y)) * 0.15915494309189535f;
      *(PQ_LDS uint32_t*)static_cast<uintptr_t>(table + parity * kPageBytes + it * 256 + lane * 4) = h2u(to_half2(__builtin_amdgcn_cosf(turns), __builtin_amdgcn_sinf(turns)));
    }
  }
  template <int K>
  __device__ __forceinline__ f32x2 trig(uint32_t angle, int parity) const {
    const f16x2 t = u2h(*(const PQ_LDS uint32_t*)static_cast<uintptr_t>(row + parity * kPageBytes + K * (NA * 4) + angle * 4));
    return f32x2{static_cast<float>(t.x) * scale, static_cast<float>(t.y) * scale};
  }
};

// A wavefront's part of the value operands: words 2 tile, + 1 (the lane's tokens of one tile) of dims 4 half .. + 3 of each slice.
template <int VB>
struct PartValues {
  uint32_t word[2], par[4];                        // of the two token pairs; {s, z} of the four tokens
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t rv, __amdgpu_buffer_rsrc_t rvp, int step, int tile, int half, int lane) {
    const uint32_t quarter = lane >> 4, slice = lane & 15;
    const u32x4 p = __builtin_amdgcn_raw_buffer_load_b128(rvp, quarter * 16, (32 * step + 16 * tile) * 4, kAuxCached);
    par[0] = p.x; par[1] = p.y; par[2] = p.z; par[3] = p.w;
    if constexpr (VB == 4) {
      const uint32_t at = quarter * 256 + slice * 16 + half * 4, block = (8 * step + 4 * tile) * 256;
      word[0] = buf_load4<kAuxCached>(rv, at, block);
      word[1] = buf_load4<kAuxCached>(rv, at + 8, block);
    } else {
      const u32x2 v = __builtin_amdgcn_raw_buffer_load_b64(rv, (quarter >> 1) * 256 + slice * 16 + (quarter & 1) * 8, (4 * step + 2 * tile) * 256, kAuxCached);
      word[0] = v.x;
      word[1] = v.y;
    }
  }
  template <int E>
  __device__ __forceinline__ u32x2 operand(int half) const {
    constexpr uint32_t kMask = ((1u << VB) - 1u) * 0x10001u;
    const f16x2 base = {static_cast<_Float16>(1024.f), static_cast<_Float16>(1024.f)};
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t x = VB == 2 ? word[i] >> (8 * half) : word[i];
      w[i] = h2u(__builtin_elementwise_fma(u2h(((x >> (VB * E)) & kMask) | 0x64006400u) - base, u2h(__builtin_amdgcn_perm(par[2 * i + 1], par[2 * i], 0x05040100u)),
                                           u2h(__builtin_amdgcn_perm(par[2 * i + 1], par[2 * i], 0x07060302u))));
    }
    return u32x2{w[0], w[1]};
  }
};
template <>
struct PartValues<16> {
  u32x2 row[4];
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t rv, __amdgpu_buffer_rsrc_t, int step, int tile, int half, int lane) {
    const uint32_t voff = (lane >> 4) * 1024 + (lane & 15) * 16 + half * 8;
#pragma unroll
    for (int j = 0; j < 4; ++j) row[j] = __builtin_amdgcn_raw_buffer_load_b64(rv, voff, (32 * step + 16 * tile + j) * 256, kAuxCached);
  }
  template <int E>
  __device__ __forceinline__ u32x2 operand(int) const {
    auto word = [&](int j) { return E < 2 ? row[j].x : row[j].y; };
    constexpr uint32_t kPick = E & 1 ? 0x07060302u : 0x05040100u;
    return u32x2{__builtin_amdgcn_perm(word(1), word(0), kPick), __builtin_amdgcn_perm(word(3), word(2), kPick)};
  }
};

// One page on its way from memory to the operands in LDS: a wavefront's part of it.
template <typename Keys, int RB, int VB>
struct PageProducer {
  static constexpr int W = Keys::W;
  static constexpr uint32_t kCodesBytes = kBlocks * kGroup * 2 * W;
  static constexpr uint32_t kParamWords = kPairs * (Keys::kGrouped ? 2 : 1);
  uint32_t codes[2];                               // 8 symbols
  uint32_t params[8];                              // {s, z} of their pairs; in the tail page un-quantized keys, x and y of four pairs twice
  PartValues<VB> values;
  bool is_tail;

  // id < 0: masked, zeros everywhere
  __device__ __forceinline__ void load(const ChunkAttentionArgs& a, int kvh, int id, bool tail, __amdgpu_buffer_rsrc_t tail_rows, int nv, int wave, int lane) {
    const int quarter = lane >> 4, col = lane & 15, half = wave & 1;
    const int64_t ph = static_cast<int64_t>(max(id, 0)) * a.n_kv_heads + kvh;
    is_tail = tail;
    const bool packed = id >= 0 && !is_tail;
    const __amdgpu_buffer_rsrc_t rc = make_rsrc(a.codes + ph * kCodesBytes, packed ? kCodesBytes : 0u);
    const __amdgpu_buffer_rsrc_t rp = make_rsrc(a.params + ph * kParamWords, packed ? kParamWords * 4u : 0u);
    const uint32_t unit = (quarter * kGroup + col) * (2 * W), tile = static_cast<uint32_t>(16 * (wave >> 1)) * (2 * W);
    if constexpr (W == 8) {
      const u32x2 c = __builtin_amdgcn_raw_buffer_load_b64(rc, unit + half * 8, tile, kAuxCached);
      codes[0] = c.x;
      codes[1] = c.y;
    } else {
      const u32x2 c = __builtin_amdgcn_raw_buffer_load_b64(rc, unit + half * 4, tile, kAuxCached);       // 48 bits from bit 0, or from bit 16
      codes[0] = half ? __builtin_amdgcn_alignbit(c.y, c.x, 16) : c.x;
      codes[1] = half ? c.y >> 16 : c.y;
    }
    if (!is_tail) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint4 p = buf_load16<kAuxCached>(rp, quarter * 64 + half * 32, i * 16);
        params[4 * i] = p.x; params[4 * i + 1] = p.y; params[4 * i + 2] = p.z; params[4 * i + 3] = p.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t at = (16 * (wave >> 1) + col) * (kHeadDim * 2) + quarter * 32 + half * 16 + i * 8;
        const u32x2 x = __builtin_amdgcn_raw_buffer_load_b64(tail_rows, at, 0, kAuxCached), y = __builtin_amdgcn_raw_buffer_load_b64(tail_rows, at, kPairs * 2, kAuxCached);
        params[4 * i] = x.x; params[4 * i + 1] = x.y; params[4 * i + 2] = y.x; params[4 * i + 3] = y.y;
      }
    }
    const __amdgpu_buffer_rsrc_t rv = make_rsrc(static_cast<const uint8_t*>(a.values) + ph * Values<VB>::kPageBytes,
                                                id < 0 ? 0u : (VB == 16 ? static_cast<uint32_t>(nv) * (kHeadDim * 2) : Values<VB>::kPageBytes));
    values.load(rv, make_rsrc(VB == 16 ? a.v_params : a.v_params + ph * kGroup, VB == 16 || id < 0 ? 0u : static_cast<uint32_t>(nv) * 4u), wave >> 2, (wave >> 1) & 1, half, lane);
  }
  // angle parameters, asked for a page earlier than the rest
  static __device__ __forceinline__ uint32_t load_angle(const ChunkAttentionArgs& a, int kvh, int id, int lane) {
    const int64_t ph = static_cast<int64_t>(max(id, 0)) * a.n_kv_heads + kvh;
    return buf_load4<kAuxCached>(make_rsrc(a.params + ph * kParamWords, id < 0 ? 0u : kParamWords * 4u), lane * 4, kPairs * 4);
  }

  __device__ __forceinline__ void store(const Keys& keys, int parity, float scale, uint8_t* key_image, uint8_t* value_image, int wave, int lane) const {
    f16x8* const k_to = reinterpret_cast<f16x8*>(key_image) + ((wave >> 1) * 4 + (wave & 1) * 2) * 64 + lane;
    if (is_tail) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const f16x2 x = u2h(params[4 * i + (e >> 1)]), y = u2h(params[4 * i + 2 + (e >> 1)]);
          w[e] = h2u(to_half2(static_cast<float>(x[e & 1]) * scale, static_cast<float>(y[e & 1]) * scale));
        }
        k_to[i * 64] = as_operand(w[0], w[1], w[2], w[3]);
      }
    } else {
      Unit<W / 2> unit;
      unit.d[0] = codes[0];
      unit.d[1] = codes[1];
      unrolled<2>([&](auto i_) {
        constexpr int i = decltype(i_)::value;
        uint32_t w[4];
        unrolled<4>([&](auto e_) {
          constexpr int e = decltype(e_)::value, K = 4 * i + e;
          const uint32_t sym = symbol<W, K>(unit);
          const f32x2 t = keys.template trig<K>(sym >> RB, parity);
          const f16x2 sz = u2h(params[K]);
          const float s = static_cast<float>(sz.x), rho = fmaf(static_cast<float>(sym & ((1u << RB) - 1u)), s, fmaf(0.5f, s, static_cast<float>(sz.y)));
          w[e] = h2u(to_half2(rho * t.x, rho * t.y));
        });
        k_to[i * 64] = as_operand(w[0], w[1], w[2], w[3]);
      });
    }
    u32x2* const v_to = reinterpret_cast<u32x2*>(value_image) + (((wave >> 2) * 8 + (wave & 1) * 4) * 64 + lane) * 2 + ((wave >> 1) & 1);
    unrolled<4>([&](auto e) { v_to[decltype(e)::value * 128] = values.template operand<decltype(e)::value>(wave & 1); });
  }
};

template <typename Keys, int RB, int VB>
__device__ __forceinline__ void shared_body(const ChunkAttentionArgs& a) {
  __shared__ __attribute__((aligned(16))) uint8_t image[2][2][kImage];       // [page parity][keys, values]
  __shared__ __attribute__((aligned(16))) uint8_t trig[Keys::kLdsBytes];
  __shared__ float fold_m[kSharedWaves][kSharedRows], fold_l[kSharedWaves][kSharedRows];
  const int tid = threadIdx.x, wave = uni(tid >> 6), lane = tid & 63, quarter = lane >> 4, col = lane & 15;
  const int kvh = blockIdx.x % a.n_kv_heads, index = a.n_items - 1 - blockIdx.x / a.n_kv_heads;   // later tokens, which see more, first
  const int split = blockIdx.y;
  Item item;
  if (!find_item(a, index, lane, item)) return;
  const int first_position = item.len - item.n + item.first, last_position = first_position + item.count - 1;
  const VisiblePages pages = visible_pages(a, first_position, last_position);
  const int per = whole_rounds((pages.count() + a.n_splits - 1) / a.n_splits);
  const int begin = uni(split * per), end = uni(min(begin + per, pages.count()));
  if (split > 0 && begin >= end) return;

  // wavefront = (rows 16 row_group .., part): `groups` row groups, a power of two; a part is 4 / parts steps of 32 tokens of each page, or,
  // from eight parts on, one step of every (parts / 4)-th page
  const int n_rows = item.count * a.group, needed = (n_rows + kSharedRows - 1) / kSharedRows;
  const int groups = needed > 8 ? 16 : (needed > 4 ? 8 : (needed > 2 ? 4 : needed)), parts = kSharedWaves / groups;
  const int row_group = uni(wave & (groups - 1)), part = uni(wave / groups);
  const bool computes = uni(row_group * kSharedRows < n_rows ? 1 : 0);
  const int step0 = uni(parts >= 4 ? part & 3 : part * (4 / parts)), step1 = uni(parts >= 4 ? step0 + 1 : step0 + 4 / parts);
  const int phase = part >> 2, phases = parts >= 4 ? parts / 4 : 1;          // a power of two

  const int row = row_group * kSharedRows + col, row_token = row / a.group, row_head = row - row_token * a.group;
  const bool row_there = row_token < item.count;
  const int position = row_there ? first_position + row_token : INT32_MAX;
  const int64_t row_at = ((item.row0 + item.first + (row_there ? row_token : 0)) * a.n_q_heads + kvh * a.group + (row_there ? row_head : 0)) * kHeadDim;
  f16x8 q[4];
  {
    const uint32_t sign = a.negate ? 0x80008000u : 0u;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      u32x2 x, y;
      __builtin_memcpy(&x, a.q + row_at + 16 * quarter + 4 * ks, 8);
      __builtin_memcpy(&y, a.q + row_at + kPairs + 16 * quarter + 4 * ks, 8);
      q[ks] = as_operand(__builtin_amdgcn_perm(y.x, x.x, 0x05040100u) ^ sign, __builtin_amdgcn_perm(y.x, x.x, 0x07060302u) ^ sign,
                         __builtin_amdgcn_perm(y.y, x.y, 0x05040100u) ^ sign, __builtin_amdgcn_perm(y.y, x.y, 0x07060302u) ^ sign);
    }
  }
  // positions of the wavefront's rows
  const int wave_first = uni(first_position + row_group * kSharedRows / a.group);
  const int wave_last = uni(min(last_position, first_position + (row_group * kSharedRows + kSharedRows - 1) / a.group));

  const int tail_page = a.residual != nullptr && item.len % kGroup != 0 ? item.len / kGroup : -1;
  const __amdgpu_buffer_rsrc_t tail_rows = make_rsrc(a.residual + (static_cast<int64_t>(item.seq) * a.n_kv_heads + kvh) * (kGroup * kHeadDim),
                                                     tail_page >= 0 ? static_cast<uint32_t>(item.len % kGroup) * (kHeadDim * 2) : 0u);
  const int32_t* const table = a.block_table + static_cast<int64_t>(item.seq) * a.max_pages_per_seq;
  auto page_of = [&](int at) { return uni(at < pages.n_first ? at : pages.from + at - pages.n_first); };
  auto id_of = [&](int at) {                                               // -1: masked, or past the end
    if (at >= end) return -1;
    const int page = page_of(at);
    const int id = page < a.max_pages_per_seq ? uni(table[page]) : -1;
    return id < 0 || id >= a.n_pool_pages ? -1 : id;
  };

  // off = kLift - m (0 as long as the row has seen nothing); a score above `limit` makes the row's m rise
  float off = 0.f, limit = kNegInf;
  f32x4 acc[8], sums = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = f32x4{0.f, 0.f, 0.f, 0.f};
  Keys keys;
  keys.init(trig, a.scale_log2, tid);
  PageProducer<Keys, RB, VB> producer;
  auto load_page = [&](int at, int id) {
    const int page = page_of(at);
    producer.load(a, kvh, id, page == tail_page, tail_rows, min(kGroup, item.len - page * kGroup), wave, lane);
  };
  // page `begin` into image[0]; page begin + 1 on its way
  int id = id_of(begin), id1 = id_of(begin + 1);
  if (begin < end) load_page(begin, id);
  if constexpr (Keys::kGrouped) {
    keys.build(producer.load_angle(a, kvh, id, lane), 0, tid);
    keys.build(producer.load_angle(a, kvh, id1, lane), 1, tid);
  }
  __syncthreads();
  if (begin < end) producer.store(keys, 0, a.scale_log2, image[0][0], image[0][1], wave, lane);
  if (begin + 1 < end) load_page(begin + 1, id1);
  __syncthreads();

  for (int at = begin; at < end; ++at) {
    const int parity = (at - begin) & 1, page = page_of(at);
    const bool masked_page = id < 0;
    id = id1;
    if (at + 1 < end) {
      producer.store(keys, parity ^ 1, a.scale_log2, image[parity ^ 1][0], image[parity ^ 1][1], wave, lane);
      id1 = id_of(at + 2);
      if (at + 2 < end) load_page(at + 2, id1);
      // the table of this page's parity has been read (before the last barrier)
      if constexpr (Keys::kGrouped) keys.build(producer.load_angle(a, kvh, id1, lane), parity, tid);
    }
    if (computes && !masked_page && ((at - begin) & (phases - 1)) == phase) {
      const f16x8* const k_image = reinterpret_cast<const f16x8*>(image[parity][0]) + lane;
      const f16x8* const v_image = reinterpret_cast<const f16x8*>(image[parity][1]) + lane;
#pragma unroll 1
      for (int step = step0; step < step1; ++step) {
        const int token0 = page * kGroup + 32 * step;
        // nobody sees the step's tokens
        if (token0 > wave_last || (a.window > 0 && token0 >= a.n_sinks && token0 + 31 <= wave_first - a.window)) continue;
        const bool masks = token0 + 31 > wave_first || (a.window > 0 && token0 <= wave_last - a.window && token0 + 31 >= a.n_sinks);
        f32x4 s[2];
        s[0] = s[1] = f32x4{off, off, off, off};
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
#pragma unroll
          for (int tile = 0; tile < 2; ++tile) s[tile] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k_image[((2 * step + tile) * 4 + ks) * 64], q[ks], s[tile], 0, 0, 0);
        if (masks) {
#pragma unroll
          for (int tile = 0; tile < 2; ++tile)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int token = token0 + 16 * tile + 4 * quarter + i;
              bool seen = token <= position;
              if (a.window > 0) seen = seen && (position - token < a.window || token < a.n_sinks);
              if (!seen) s[tile][i] = kNegInf;
            }
        }
        float top = max3(s[0][0], s[0][1], s[0][2]);
        top = max3(top, s[0][3], s[1][0]);
        top = max3(top, s[1][1], s[1][2]);
        top = max2(top, s[1][3]);
        if (__builtin_amdgcn_ballot_w64(top > limit) != 0) {
          auto r = __builtin_amdgcn_permlane16_swap(f2u(top), f2u(top), false, false);
          top = max2(u2f(r[0]), u2f(r[1]));
          auto r2 = __builtin_amdgcn_permlane32_swap(f2u(top), f2u(top), false, false);
          top = max2(u2f(r2[0]), u2f(r2[1]));
          // the row's largest score goes to kLift, if it is above that or the row's first
          const bool first = limit == kNegInf;
          const float down = top > kNegInf && (first || top > kLift) ? kLift - top : 0.f;
          if (top > kNegInf) limit = 15.f;
          off += down;
          const float keep = first ? 1.f : __builtin_amdgcn_exp2f(down);
          sums *= keep;
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[e] *= keep;
          s[0] += down;
          s[1] += down;
        }
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          w[i] = h2u(to_half2(__builtin_amdgcn_exp2f(s[i >> 1][2 * (i & 1)]), __builtin_amdgcn_exp2f(s[i >> 1][2 * (i & 1) + 1])));
        const f16x8 p = as_operand(w[0], w[1], w[2], w[3]);
        constexpr uint32_t kOnes = 0x3c003c00u;
        sums = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_operand(kOnes, kOnes, kOnes, kOnes), p, sums, 0, 0, 0);
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v_image[(step * 8 + e) * 64], p, acc[e], 0, 0, 0);
      }
    }
    __syncthreads();
  }

  // ---- fold the parts of a row group ----
  float m = limit > kNegInf ? kLift - off : kNegInf, l = sums[0];
  if (parts > 1) {
    if (quarter == 0) {
      fold_m[wave][col] = m;
      fold_l[wave][col] = l;
    }
    __syncthreads();
    float top = kNegInf, total = 0.f;
    for (int p = 0; p < parts; ++p) top = fmaxf(top, fold_m[row_group + p * groups][col]);
    for (int p = 0; p < parts; ++p) total += top > kNegInf ? fold_l[row_group + p * groups][col] * __builtin_amdgcn_exp2f(fold_m[row_group + p * groups][col] - top) : 0.f;
    const float weight = top > kNegInf ? __builtin_amdgcn_exp2f(m - top) : 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] *= weight;
    m = top;
    l = total;
    f32x4* const room = reinterpret_cast<f32x4*>(&image[0][0][0]);           // 8 KB a wavefront
    if (part > 0) {
#pragma unroll
      for (int e = 0; e < 8; ++e) room[(wave * 8 + e) * 64 + lane] = acc[e];
    }
    __syncthreads();
    if (part > 0) return;
    for (int p = 1; p < parts; ++p) {
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += room[((row_group + p * groups) * 8 + e) * 64 + lane];
    }
  }
  if (!computes) return;
  // lane: dims 32 quarter + 8 i + e of its row
  if (a.n_splits > 1) {
    const int64_t slot_row = ((static_cast<int64_t>(index) * a.n_kv_heads + kvh) * a.n_splits + split) * kTileRows + row;
    float* const to = a.ws_acc + slot_row * kHeadDim + 32 * quarter;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      *reinterpret_cast<f32x4*>(to + 8 * i) = f32x4{acc[0][i], acc[1][i], acc[2][i], acc[3][i]};
      *reinterpret_cast<f32x4*>(to + 8 * i + 4) = f32x4{acc[4][i], acc[5][i], acc[6][i], acc[7][i]};
    }
    if (quarter == 0) {
      a.ws_ml[slot_row * 2] = m;
      a.ws_ml[slot_row * 2 + 1] = l;
    }
    return;
  }
  if (!row_there) return;
  const float inv = l > 0.f ? 1.f / l : 0.f;
  __half* const to = a.out + row_at + 32 * quarter;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    *reinterpret_cast<u32x4*>(to + 8 * i) = u32x4{h2u(to_half2(acc[0][i] * inv, acc[1][i] * inv)), h2u(to_half2(acc[2][i] * inv, acc[3][i] * inv)),
                                                  h2u(to_half2(acc[4][i] * inv, acc[5][i] * inv)), h2u(to_half2(acc[6][i] * inv, acc[7][i] * inv))};
}

}  // namespace chunk
}  // namespace
}  // namespace pq
