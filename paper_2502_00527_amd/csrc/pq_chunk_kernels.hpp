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
// Rounding.  Queries are fp16; reconstructed keys (made in fp32, the softmax's scale in them), probabilities and de-quantized values
// are rounded to fp16 for the matrix unit, like the output: each 2^-12 of itself in the mean, where the cache's own quantization is
// 2^-4.  Sums, m and l are fp32.  The score product starts from kLift - m, so that what comes out is the exponent of a weight times
// 2^kLift: weights down to 2^-21 of the largest keep all their bits, and m is raised only when a score is 2^(15 - kLift) above it (the
// weight then still fits fp16), and then by all lanes of the row.
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
  float* ws_acc;               // [unit][KV head][row][d], un-normalised
  float* ws_ml;                // [unit][KV head][row][2]
  int32_t* ws_units;           // [unit][4]: note_unit()
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
  int32_t n_units;             // places for parts of items, of a KV head
  int32_t cuts;                // whether items may be cut:
  int32_t parts;               // alike, into so many parts; 0: by what the sequences hold
  int32_t longest_first;
  int32_t table_index;
  float scale_log2;            // > 0
  int32_t negate;              // the queries
};

// Launchers, one for each value width (pq_chunk_attention.hip): rows_of_16 is 1, 2 or kTileRows / 16.  False: no such kernel.
bool launch_chunk_v16(const pq_layout* l, int rows_of_16, const ChunkAttentionArgs& a, dim3 grid, hipStream_t st);
bool launch_chunk_v4(const pq_layout* l, int rows_of_16, const ChunkAttentionArgs& a, dim3 grid, hipStream_t st);
bool launch_chunk_v2(const pq_layout* l, int rows_of_16, const ChunkAttentionArgs& a, dim3 grid, hipStream_t st);

}  // namespace pq

#include "pq_chunk_cut.hpp"

namespace pq {
namespace {
namespace chunk {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

constexpr int kLift = 7;

// What the parts' join has to know of a unit: rows from `row` on, the number of parts if it is the first of several, otherwise 0.
__device__ __forceinline__ void note_unit(const ChunkAttentionArgs& a, int kvh, int unit, int row, int count, int parts) {
  if (a.cuts && kvh == 0) *reinterpret_cast<i32x4*>(a.ws_units + static_cast<int64_t>(unit) * 4) = i32x4{row, count, parts, 0};
}
__device__ __forceinline__ void note_unit(const ChunkAttentionArgs& a, int kvh, const Item& item, const VisiblePages& pages) {
  const int part_len = pages.part_len(item);
  note_unit(a, kvh, item.unit, static_cast<int>(item.row0) + item.first, item.count,
            item.part == 0 && item.parts > 1 ? max(1, (pages.count() + part_len - 1) / part_len) : 0);
}

template <int N, typename F>
__device__ __forceinline__ void unrolled(F f) {
  if constexpr (N > 0) {
    unrolled<N - 1>(f);
    f(std::integral_constant<int, N - 1>{});
  }
}

// ---- keys -------------------------------------------------------------------------------------------
// A pair's coordinates rho~ (cos, sin), rho~ = (c + 1/2) s + z, in fp32, rounded once.  code: c; sz: {fp16 s, fp16 z}; trig: (cos, sin) of
// the angle level times the softmax's scale (in the exponent's units), which scores carry from here on.
__device__ __forceinline__ uint32_t key_pair(float code, uint32_t sz_, f32x2 trig) {
  const f16x2 sz = u2h(sz_);
  const float s = static_cast<float>(sz.x), rho = fmaf(code, s, fmaf(0.5f, s, static_cast<float>(sz.y)));
  return h2u(to_half2(rho * trig.x, rho * trig.y));
}
// Radius code of pair K of a unit as a float, and `base` + 2^kShift times its angle code.
template <int RB, int TB, int K, int kShift>
__device__ __forceinline__ void key_fields(const Unit<(RB + TB) / 2>& u, uint32_t base, float& code, uint32_t& addr) {
  if constexpr (RB == 4 && TB == 4 && kShift == 4) {
    pair_fields<RB, TB, K>(u, base, code, addr);
  } else {
    const uint32_t sym = symbol<RB + TB, K>(u);
    code = static_cast<float>(sym & ((1u << RB) - 1u));
    addr = base + ((sym >> RB) << kShift);
  }
}
// The same of four un-quantized pairs: x and y of them as they lie in a row of the residual.
__device__ __forceinline__ f16x8 plain_pairs(u32x2 x_, u32x2 y_, float scale) {
  uint32_t w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const f16x2 x = u2h(x_[e >> 1]), y = u2h(y_[e >> 1]);
    w[e] = h2u(to_half2(static_cast<float>(x[e & 1]) * scale, static_cast<float>(y[e & 1]) * scale));
  }
  return as_operand(w[0], w[1], w[2], w[3]);
}

// Uniform grid: one table of the levels for all pairs.  Its at most 32 entries lie in different banks: no conflicts.
template <int RB, int TB>
struct UniformTrig {
  static constexpr int NA = 1 << TB, kShift = TB == 5 ? 3 : 4, kTableBytes = NA << kShift;
  static constexpr bool kGrouped = false;
  uint32_t table;
  __device__ __forceinline__ void init(uint8_t* lds, float scale, int, int tid) {
    table = lds_addr(lds);
    if (tid < NA) {
      const float angle = ((static_cast<float>(tid) + 0.5f) * (1.f / NA) - 0.5f) * 6.283185307179586f;
      *reinterpret_cast<f32x2*>(lds + (tid << kShift)) = f32x2{cosf(angle) * scale, sinf(angle) * scale};
    }
  }
  __device__ __forceinline__ void build(uint32_t, int, int, int, int) {}
  // word of the lane's pair K
  template <int K>
  __device__ __forceinline__ uint32_t pair(const Unit<(RB + TB) / 2>& u, uint32_t sz, int) const {
    float code;
    uint32_t addr;
    key_fields<RB, TB, K, kShift>(u, table, code, addr);
    return key_pair(code, sz, *(const PQ_LDS f32x2*)static_cast<uintptr_t>(addr));
  }
};
// Grouped quantizer: the levels belong to the page; a table of its 64 x 2^t (cos, sin) as fp16.
template <int RB, int TB>
struct GroupedTrig {
  static constexpr int NA = 1 << TB, kTableBytes = kPairs * NA * 4;
  static constexpr bool kGrouped = true;
  uint32_t table, row;
  float scale;
  // first_pair: the lane's
  __device__ __forceinline__ void init(uint8_t* lds, float scale_, int first_pair, int) {
    table = lds_addr(lds);
    row = table + first_pair * (NA * 4);
    scale = scale_;
  }
  // rounds first, first + step, .. of table `which`; angle: {fp16 s, fp16 z} of pair `lane`
  __device__ __forceinline__ void build(uint32_t angle, int which, int first, int step, int lane) {
    const float level = static_cast<float>(lane & (NA - 1)) + 0.5f;
    constexpr int kPairsAtOnce = 64 >> TB;
    for (int it = first; it < NA; it += step) {
      const f16x2 sz = u2h(static_cast<uint32_t>(__shfl(static_cast<int>(angle), it * kPairsAtOnce + (lane >> TB))));
      const float turns = fmaf(level, static_cast<float>(sz.x), static_cast<float>(sz.y)) * 0.15915494309189535f;
      *(PQ_LDS uint32_t*)static_cast<uintptr_t>(table + which * kTableBytes + it * 256 + lane * 4) = h2u(to_half2(__builtin_amdgcn_cosf(turns), __builtin_amdgcn_sinf(turns)));
    }
  }
  template <int K>
  __device__ __forceinline__ uint32_t pair(const Unit<(RB + TB) / 2>& u, uint32_t sz, int which) const {
    float code;
    uint32_t addr;
    key_fields<RB, TB, K, 2>(u, row + which * kTableBytes, code, addr);
    const f16x2 t = u2h(*(const PQ_LDS uint32_t*)static_cast<uintptr_t>(addr + K * (NA * 4)));
    return key_pair(code, sz, f32x2{static_cast<float>(t.x) * scale, static_cast<float>(t.y) * scale});
  }
};

// ---- rows: 16 RT query rows of a wavefront, their scores of 32 tokens (two tiles), and what is summed over them ----------
template <int RT>
struct Rows {
  // Scores come out of the matrix unit as exponents, off = kLift - m added (0 as long as the row has seen nothing); one above `limit`
  // makes the row's m rise.
  float off[RT], limit[RT];
  f32x4 acc[8][RT], sums[RT];                      // sums of weights: like one more dim, all four alike
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      off[rt] = 0.f;
      limit[rt] = kNegInf;
      sums[rt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e][rt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
  __device__ __forceinline__ f32x4 start(int rt) const { return f32x4{off[rt], off[rt], off[rt], off[rt]}; }
  // tokens from token0 on that the rows at `position` do not see: later ones, and with a window those between the sinks and it
  __device__ __forceinline__ void mask(const ChunkAttentionArgs& a, f32x4 (&s)[2][RT], int token0, const int (&position)[RT], int quarter) const {
    const int sinks = a.window > 0 ? a.n_sinks : 0;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int first = token0 + 4 * quarter, last = position[rt] - first, hidden_to = a.window > 0 ? last - a.window : -1 - first, hidden_from = sinks - first;
#pragma unroll
      for (int tile = 0; tile < 2; ++tile)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int token = 16 * tile + i;         // from `first` on
          const bool hidden = static_cast<bool>(static_cast<int>(token > last) | (static_cast<int>(token <= hidden_to) & static_cast<int>(token >= hidden_from)));
          s[tile][rt][i] = hidden ? kNegInf : s[tile][rt][i];
        }
    }
  }
  // raises m where that is due
  __device__ __forceinline__ void settle(f32x4 (&s)[2][RT]) {
    float top[RT];
    bool above = false;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float x = max3(s[0][rt][0], s[0][rt][1], s[0][rt][2]);
      x = max3(x, s[0][rt][3], s[1][rt][0]);
      x = max3(x, s[1][rt][1], s[1][rt][2]);
      top[rt] = max2(x, s[1][rt][3]);
      above = above || top[rt] > limit[rt];
    }
    if (__builtin_amdgcn_ballot_w64(above) == 0) return;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float x = top[rt];
      auto r = __builtin_amdgcn_permlane16_swap(f2u(x), f2u(x), false, false);
      x = max2(u2f(r[0]), u2f(r[1]));
      auto r2 = __builtin_amdgcn_permlane32_swap(f2u(x), f2u(x), false, false);
      x = max2(u2f(r2[0]), u2f(r2[1]));
      // the row's largest score goes to kLift, if it is above that or the row's first
      const bool first = limit[rt] == kNegInf;
      const float down = x > kNegInf && (first || x > kLift) ? kLift - x : 0.f;
      if (x > kNegInf) limit[rt] = 15.f;           // 2^15 still is an fp16 number
      off[rt] += down;
      const float keep = first ? 1.f : __builtin_amdgcn_exp2f(down);
      sums[rt] *= keep;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e][rt] *= keep;
      s[0][rt] += down;
      s[1][rt] += down;
    }
  }
  __device__ __forceinline__ void weights(const f32x4 (&s)[2][RT], f16x8 (&p)[RT]) {
    constexpr uint32_t kOnes = 0x3c003c00u;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        w[i] = h2u(to_half2(__builtin_amdgcn_exp2f(s[i >> 1][rt][2 * (i & 1)]), __builtin_amdgcn_exp2f(s[i >> 1][rt][2 * (i & 1) + 1])));
      p[rt] = as_operand(w[0], w[1], w[2], w[3]);
      sums[rt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_operand(kOnes, kOnes, kOnes, kOnes), p[rt], sums[rt], 0, 0, 0);
    }
  }
  __device__ __forceinline__ void add(int e, f16x8 v_op, const f16x8 (&p)[RT]) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) acc[e][rt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v_op, p[rt], acc[e][rt], 0, 0, 0);
  }
  __device__ __forceinline__ float top(int rt) const { return limit[rt] > kNegInf ? kLift - off[rt] : kNegInf; }
  // The lane's 32 dims of a row, 32 (l / 16) + 8 i + e: a part of its pages, or the output.
  __device__ __forceinline__ void store_part(const ChunkAttentionArgs& a, int rt, int64_t row, float m, float l, int quarter) const {
    float* const to = a.ws_acc + row * kHeadDim + 32 * quarter;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      *reinterpret_cast<f32x4*>(to + 8 * i) = f32x4{acc[0][rt][i], acc[1][rt][i], acc[2][rt][i], acc[3][rt][i]};
      *reinterpret_cast<f32x4*>(to + 8 * i + 4) = f32x4{acc[4][rt][i], acc[5][rt][i], acc[6][rt][i], acc[7][rt][i]};
    }
    if (quarter == 0) {
      a.ws_ml[row * 2] = m;
      a.ws_ml[row * 2 + 1] = l;
    }
  }
  __device__ __forceinline__ void store_out(int rt, __half* to, float l, int quarter) const {
    const float inv = l > 0.f ? 1.f / l : 0.f;
    auto pair = [&](int e, int i) { return h2u(to_half2(acc[e][rt][i] * inv, acc[e + 1][rt][i] * inv)); };
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<u32x4*>(to + 32 * quarter + 8 * i) = u32x4{pair(0, i), pair(2, i), pair(4, i), pair(6, i)};
  }
};

// Element offset of a row's query and output, and its position; rows past the item's last one are its first one, at no position.
struct RowPlace {
  int64_t at;
  int position;
  bool there;
  __device__ __forceinline__ RowPlace(const ChunkAttentionArgs& a, const Item& item, int kvh, int row) {
    const int token = row / a.group, head = row - token * a.group;
    there = token < item.count;
    position = there ? item.len - item.n + item.first + token : INT32_MAX;
    at = ((item.row0 + item.first + (there ? token : 0)) * a.n_q_heads + kvh * a.group + (there ? head : 0)) * kHeadDim;
  }
};
// Operand KS of a row's query: pairs 16 (l / 16) + 4 KS .. + 3.
__device__ __forceinline__ f16x8 query_operand(const ChunkAttentionArgs& a, int64_t at, int quarter, int ks) {
  const uint32_t sign = a.negate ? 0x80008000u : 0u;
  u32x2 x, y;
  __builtin_memcpy(&x, a.q + at + 16 * quarter + 4 * ks, 8);
  __builtin_memcpy(&y, a.q + at + kPairs + 16 * quarter + 4 * ks, 8);
  return as_operand(__builtin_amdgcn_perm(y.x, x.x, 0x05040100u) ^ sign, __builtin_amdgcn_perm(y.x, x.x, 0x07060302u) ^ sign,
                    __builtin_amdgcn_perm(y.y, x.y, 0x05040100u) ^ sign, __builtin_amdgcn_perm(y.y, x.y, 0x07060302u) ^ sign);
}

// The pages of a work-group's part, and what is known of each.
struct PartPages {
  VisiblePages pages;
  const int32_t* table;
  int64_t n_pool_pages;
  int begin, end, width, tail_page, len;
  __device__ __forceinline__ PartPages(const ChunkAttentionArgs& a, const Item& item) : pages(a, item) {
    const int part_len = pages.part_len(item);
    begin = uni(item.part * part_len);
    end = uni(min(begin + part_len, pages.count()));
    table = a.block_table + static_cast<int64_t>(item.seq) * a.max_pages_per_seq;
    n_pool_pages = a.n_pool_pages;
    width = a.max_pages_per_seq;
    len = item.len;
    tail_page = a.residual != nullptr && item.len % kGroup != 0 ? item.len / kGroup : -1;
  }
  __device__ __forceinline__ int page(int at) const { return uni(at < pages.n_first ? at : pages.from + at - pages.n_first); }
  // pool page of page `at`; -1: masked, or past the end
  __device__ __forceinline__ int id(int at) const {
    if (at >= end) return -1;
    const int p = page(at);
    const int id = p < width ? uni(table[p]) : -1;
    return id < 0 || id >= n_pool_pages ? -1 : id;
  }
  // of the un-quantized keys of the last, incomplete group
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t tail_rows(const ChunkAttentionArgs& a, const Item& item, int kvh) const {
    return make_rsrc(a.residual + (static_cast<int64_t>(item.seq) * a.n_kv_heads + kvh) * (kGroup * kHeadDim),
                     tail_page >= 0 ? static_cast<uint32_t>(len % kGroup) * (kHeadDim * 2) : 0u);
  }
};
template <int W, bool kGrouped, int VB>
struct PageFormat {
  static constexpr uint32_t kCodesBytes = kBlocks * kGroup * 2 * W;
  static constexpr uint32_t kParamWords = kPairs * (kGrouped ? 2 : 1);
  static constexpr uint32_t kValueBytes = kGroup * kHeadDim * VB / 8;
};

// ---- values: what a lane loads of 32 tokens (its tokens 4 (l / 16) .. + 3 of both tiles, its slice of 8 dims), and operand e of them ----
template <int VB>
struct Values;
template <>
struct Values<16> {
  uint4 row[8];
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t rv, __amdgpu_buffer_rsrc_t, int step, int lane) {
    const uint32_t voff = (lane >> 4) * 1024 + (lane & 15) * 16;
#pragma unroll
    for (int j = 0; j < 8; ++j) row[j] = buf_load16<kAuxStream>(rv, voff, (32 * step + 16 * (j >> 2) + (j & 3)) * 256);
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

// ---- few rows: operands made in registers --------------------------------------------------------------------
// A work-group serves up to 16 RT rows of one KV head; its four wavefronts take 32 tokens of each page, making their operands in
// registers, and are folded at the end.  What bounds it is what is under way: keys and values of the page after the next are asked for
// as a page's are used.  The queries, the same for all four, are read from LDS for each tile: with them in registers
// there would be no room for that.
constexpr int kFewWaves = 4;

template <typename Trig, int RB, int W, int VB, int RT>
__device__ __forceinline__ void few_body(const ChunkAttentionArgs& a) {
  constexpr bool kGrouped = Trig::kGrouped;
  using Format = PageFormat<W, kGrouped, VB>;
  constexpr int kTableBytes = Trig::kTableBytes * (kGrouped ? kFewWaves : 1);
  constexpr int kFoldBytes = 2 * RT * 8 * 64 * 16;
  __shared__ __attribute__((aligned(16))) uint8_t lds[kTableBytes > kFoldBytes ? kTableBytes : kFoldBytes];
  __shared__ __attribute__((aligned(16))) uint32_t page_params[kFewWaves][kPairs];
  __shared__ __attribute__((aligned(16))) f16x8 query[RT][4][64];
  __shared__ float fold_m[kFewWaves][RT * 16], fold_l[kFewWaves][RT * 16];
  const int tid = threadIdx.x, wave = uni(tid >> 6), lane = tid & 63, quarter = lane >> 4, col = lane & 15;
  const int kvh = blockIdx.x % a.n_kv_heads;
  Item item;
  const Sequence mine = sequence_of(a, lane);
  if (!find_item(a, mine, few_cut(a, mine, lane), blockIdx.x / a.n_kv_heads, lane, item)) {
    if (tid == 0) note_unit(a, kvh, blockIdx.x / a.n_kv_heads, 0, 0, 0);
    return;
  }
  const PartPages pages(a, item);
  if (tid == 0) note_unit(a, kvh, item, pages.pages);
  if (item.part > 0 && pages.begin >= pages.end) return;
  const int first_position = item.len - item.n + item.first, last_position = first_position + item.count - 1;

  // A page on its way: the wavefront's two tiles of keys, the parameters of pair `lane`; and values, of the next page or the next two.  (32
  // rows and fp16 values: two pages of them need scratch, 38.7 us against 37.0 for 16 x 5 tokens over 500 .. 6000.)
  constexpr int kValuesAhead = VB == 16 && RT == 2 ? 1 : 2;
  struct Page {
    Unit<W / 2> units[2];
    uint32_t par, angle;
    int id;
  };
  const uint32_t voff_codes = (quarter * kGroup + col) * (2 * W);
  auto load = [&](int at, Page& p) {
    p.id = pages.id(at);
    const int64_t ph = static_cast<int64_t>(max(p.id, 0)) * a.n_kv_heads + kvh;
    const bool packed = p.id >= 0 && pages.page(at) != pages.tail_page;
    const __amdgpu_buffer_rsrc_t rc = make_rsrc(a.codes + ph * Format::kCodesBytes, packed ? Format::kCodesBytes : 0u);
    const __amdgpu_buffer_rsrc_t rp = make_rsrc(a.params + ph * Format::kParamWords, packed ? Format::kParamWords * 4u : 0u);
    p.par = buf_load4<kAuxCached>(rp, lane * 4, 0);
    if constexpr (kGrouped) p.angle = buf_load4<kAuxCached>(rp, lane * 4, kPairs * 4);
#pragma unroll
    for (int tile = 0; tile < 2; ++tile) p.units[tile] = load_unit<W>(rc, voff_codes, static_cast<uint32_t>(32 * wave + 16 * tile) * (2 * W));
  };
  Values<VB> values[kValuesAhead];
  auto load_values = [&](int at, int id, Values<VB>& v) {
    const int64_t ph = static_cast<int64_t>(max(id, 0)) * a.n_kv_heads + kvh;
    const int nv = min(kGroup, pages.len - pages.page(at) * kGroup);
    v.load(make_rsrc(static_cast<const uint8_t*>(a.values) + ph * Format::kValueBytes, id < 0 ? 0u : (VB == 16 ? static_cast<uint32_t>(nv) * (kHeadDim * 2) : Format::kValueBytes)),
           make_rsrc(VB == 16 ? a.v_params : a.v_params + ph * kGroup, VB == 16 || id < 0 ? 0u : static_cast<uint32_t>(nv) * 4u), wave, lane);
  };
  Page p[2];
  load(pages.begin, p[0]);
  load_values(pages.begin, p[0].id, values[0]);
  load(pages.begin + 1, p[1]);
  if constexpr (kValuesAhead == 2) load_values(pages.begin + 1, p[1].id, values[1]);

  int position[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const RowPlace place(a, item, kvh, 16 * rt + col);
    position[rt] = place.position;
    query[rt][wave][lane] = query_operand(a, place.at, quarter, wave);                       // one of four operands a wavefront
  }
  Trig trig;
  trig.init(lds + (kGrouped ? wave * Trig::kTableBytes : 0), a.scale_log2, 16 * quarter, tid);
  const __amdgpu_buffer_rsrc_t tail_rows = pages.tail_rows(a, item, kvh);
  Rows<RT> rows;
  rows.clear();
  __syncthreads();

  // One way through for pages that are seen and that are not: with a second copy of the loads the accumulators moved between registers
  // at its ends (41.0 us against 37.0).
  auto attend = [&](int at, Page& p, const Page& following, Values<VB>& v) {
    auto load_next = [&] {
      if constexpr (kValuesAhead == 1) load_values(at + 1, following.id, v);
      load(at + 2, p);
      if constexpr (kValuesAhead == 2) load_values(at + 2, p.id, v);
    };
    const int page = pages.page(at), token0 = page * kGroup + 32 * wave;
    // otherwise nobody sees these tokens
    if (p.id >= 0 && token0 <= last_position && (a.window == 0 || token0 < a.n_sinks || token0 + 31 > first_position - a.window)) {
      const bool masks = token0 + 31 > first_position || (a.window > 0 && token0 <= last_position - a.window && token0 + 31 >= a.n_sinks);
      f32x4 s[2][RT];
      auto scores = [&](int tile, const f16x8 (&k_op)[4]) {
        uint32_t query_at = lds_addr(&query[0][0][0]) + lane * 16;
        asm volatile("" : "+v"(query_at));                                    // (read for each tile, not kept)
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
#pragma unroll
          for (int rt = 0; rt < RT; ++rt)
            s[tile][rt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k_op[ks], *(const PQ_LDS f16x8*)static_cast<uintptr_t>(query_at + (rt * 4 + ks) * 1024),
                                                                 ks == 0 ? rows.start(rt) : s[tile][rt], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      };
      f16x8 k_op[4];
      if (page != pages.tail_page) {
        wave_lds_sync();                                                      // the page before has been read
        page_params[wave][lane] = p.par;
        if constexpr (kGrouped) trig.build(p.angle, 0, 0, 1, lane);
        wave_lds_sync();
        uint32_t params[16];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const u32x4 four = *reinterpret_cast<const u32x4*>(&page_params[wave][16 * quarter + 4 * i]);
          params[4 * i] = four.x; params[4 * i + 1] = four.y; params[4 * i + 2] = four.z; params[4 * i + 3] = four.w;
        }
#pragma unroll
        for (int tile = 0; tile < 2; ++tile) {
          unrolled<4>([&](auto ks_) {
            constexpr int ks = decltype(ks_)::value;
            uint32_t w[4];
            unrolled<4>([&](auto e_) {
              constexpr int K = 4 * ks + decltype(e_)::value;
              w[decltype(e_)::value] = trig.template pair<K>(p.units[tile], params[K], 0);
            });
            k_op[ks] = as_operand(w[0], w[1], w[2], w[3]);
          });
          scores(tile, k_op);
        }
      } else {
#pragma unroll
        for (int tile = 0; tile < 2; ++tile) {
#pragma unroll
          for (int ks = 0; ks < 4; ++ks) {
            const uint32_t offset = (32 * wave + 16 * tile + col) * (kHeadDim * 2) + quarter * 32 + ks * 8;
            k_op[ks] = plain_pairs(__builtin_amdgcn_raw_buffer_load_b64(tail_rows, offset, 0, kAuxCached),
                                   __builtin_amdgcn_raw_buffer_load_b64(tail_rows, offset, kPairs * 2, kAuxCached), a.scale_log2);
          }
          scores(tile, k_op);
        }
      }
      if (masks) rows.mask(a, s, token0, position, quarter);
      rows.settle(s);
      f16x8 weights[RT];
      rows.weights(s, weights);
      unrolled<8>([&](auto e) { rows.add(decltype(e)::value, v.template operand<decltype(e)::value>(), weights); });
      __builtin_amdgcn_sched_barrier(0);
    }
    load_next();
  };
  for (int at = pages.begin; at < pages.end; at += 2) {
    attend(at, p[0], p[1], values[0]);
    attend(at + 1, p[1], p[0], values[kValuesAhead - 1]);                   // (no page is past the last one, and seen by nobody)
  }

  // ---- fold the wavefronts ----
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    if (quarter == 0) {
      fold_m[wave][16 * rt + col] = rows.top(rt);
      fold_l[wave][16 * rt + col] = rows.sums[rt][0];
    }
  }
  __syncthreads();                                                          // (the table is free, too)
  float top[RT], total[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    top[rt] = kNegInf;
    total[rt] = 0.f;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) top[rt] = fmaxf(top[rt], fold_m[w][16 * rt + col]);
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w)
      total[rt] += top[rt] > kNegInf ? fold_l[w][16 * rt + col] * __builtin_amdgcn_exp2f(fold_m[w][16 * rt + col] - top[rt]) : 0.f;
    const float weight = top[rt] > kNegInf ? __builtin_amdgcn_exp2f(rows.top(rt) - top[rt]) : 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) rows.acc[e][rt] *= weight;
  }
  f32x4* const room = reinterpret_cast<f32x4*>(lds);
#pragma unroll
  for (int half = 2; half >= 1; half >>= 1) {
    if (wave >= half && wave < 2 * half) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) room[((wave - half) * 8 * RT + e * RT + rt) * 64 + lane] = rows.acc[e][rt];
    }
    __syncthreads();
    if (wave < half) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) rows.acc[e][rt] += room[(wave * 8 * RT + e * RT + rt) * 64 + lane];
    }
    __syncthreads();
  }
  if (wave != 0) return;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    if (item.parts > 1) {
      if (16 * rt + col < item.count * a.group)
        rows.store_part(a, rt, (static_cast<int64_t>(item.unit) * a.n_kv_heads + kvh) * (16 * RT) + 16 * rt + col, top[rt], total[rt], quarter);
    } else {
      const RowPlace place(a, item, kvh, 16 * rt + col);
      if (place.there) rows.store_out(rt, a.out + place.at, total[rt], quarter);
    }
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
constexpr int kImage = kGroup * kHeadDim * 2;      // bytes of a page's key or value operands

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
template <typename Trig, int RB, int W, int VB>
struct PageProducer {
  using Format = PageFormat<W, Trig::kGrouped, VB>;
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
    const __amdgpu_buffer_rsrc_t rc = make_rsrc(a.codes + ph * Format::kCodesBytes, packed ? Format::kCodesBytes : 0u);
    const __amdgpu_buffer_rsrc_t rp = make_rsrc(a.params + ph * Format::kParamWords, packed ? Format::kParamWords * 4u : 0u);
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
    const __amdgpu_buffer_rsrc_t rv = make_rsrc(static_cast<const uint8_t*>(a.values) + ph * Format::kValueBytes,
                                                id < 0 ? 0u : (VB == 16 ? static_cast<uint32_t>(nv) * (kHeadDim * 2) : Format::kValueBytes));
    values.load(rv, make_rsrc(VB == 16 ? a.v_params : a.v_params + ph * kGroup, VB == 16 || id < 0 ? 0u : static_cast<uint32_t>(nv) * 4u), wave >> 2, (wave >> 1) & 1, half, lane);
  }
  // angle parameters, asked for a page earlier than the rest
  static __device__ __forceinline__ uint32_t load_angle(const ChunkAttentionArgs& a, int kvh, int id, int lane) {
    const int64_t ph = static_cast<int64_t>(max(id, 0)) * a.n_kv_heads + kvh;
    return buf_load4<kAuxCached>(make_rsrc(a.params + ph * Format::kParamWords, id < 0 ? 0u : Format::kParamWords * 4u), lane * 4, kPairs * 4);
  }

  __device__ __forceinline__ void store(const Trig& trig, int parity, float scale, uint8_t* key_image, uint8_t* value_image, int wave, int lane) const {
    f16x8* const k_to = reinterpret_cast<f16x8*>(key_image) + ((wave >> 1) * 4 + (wave & 1) * 2) * 64 + lane;
    if (is_tail) {
#pragma unroll
      for (int i = 0; i < 2; ++i) k_to[i * 64] = plain_pairs(u32x2{params[4 * i], params[4 * i + 1]}, u32x2{params[4 * i + 2], params[4 * i + 3]}, scale);
    } else {
      Unit<W / 2> unit;
      unit.d[0] = codes[0];
      unit.d[1] = codes[1];
      unrolled<2>([&](auto i_) {
        constexpr int i = decltype(i_)::value;
        uint32_t w[4];
        unrolled<4>([&](auto e_) {
          constexpr int K = 4 * i + decltype(e_)::value;
          w[decltype(e_)::value] = trig.template pair<K>(unit, params[K], parity);
        });
        k_to[i * 64] = as_operand(w[0], w[1], w[2], w[3]);
      });
    }
    u32x2* const v_to = reinterpret_cast<u32x2*>(value_image) + (((wave >> 2) * 8 + (wave & 1) * 4) * 64 + lane) * 2 + ((wave >> 1) & 1);
    unrolled<4>([&](auto e) { v_to[decltype(e)::value * 128] = values.template operand<decltype(e)::value>(wave & 1); });
  }
};

template <typename Trig, int RB, int W, int VB>
__device__ __forceinline__ void shared_body(const ChunkAttentionArgs& a) {
  __shared__ __attribute__((aligned(16))) uint8_t image[2][2][kImage];       // [page parity][keys, values]
  __shared__ __attribute__((aligned(16))) uint8_t tables[Trig::kTableBytes * (Trig::kGrouped ? 2 : 1)];
  __shared__ float fold_m[kSharedWaves][kSharedRows], fold_l[kSharedWaves][kSharedRows];
  const int tid = threadIdx.x, wave = uni(tid >> 6), lane = tid & 63, quarter = lane >> 4, col = lane & 15;
  const int kvh = blockIdx.x % a.n_kv_heads;
  Item item;
  Sequence mine = sequence_of(a, lane);
  float cut = 0.f;
  if (a.parts > 0) {
    cut = cut_alike(a, mine);
  } else if (a.cuts) {
    // a candidate a wavefront
    uint32_t time;
    const float candidate = judge_cut(a, mine, wave, lane, time);
    if (lane == 0) {
      fold_m[0][wave] = candidate;
      fold_l[0][wave] = u2f(judged(time, wave));
    }
    __syncthreads();
    cut = fold_m[0][~wave_max_u32(~f2u(fold_l[0][col])) & 15u];
    __syncthreads();                                                          // (fold_m and fold_l are used again)
  }
  if (a.longest_first) mine = longest_first(a, mine, lane);
  if (!find_item(a, mine, cut, blockIdx.x / a.n_kv_heads, lane, item)) {
    if (tid == 0) note_unit(a, kvh, blockIdx.x / a.n_kv_heads, 0, 0, 0);
    return;
  }
  const PartPages pages(a, item);
  if (tid == 0) note_unit(a, kvh, item, pages.pages);
  const int begin = pages.begin, end = pages.end;
  if (item.part > 0 && begin >= end) return;
  const int first_position = item.len - item.n + item.first, last_position = first_position + item.count - 1;

  // wavefront = (rows 16 row_group .., part): `groups` row groups, a power of two; a part is 4 / parts steps of 32 tokens of each page, or,
  // from eight parts on, one step of every (parts / 4)-th page
  const int n_rows = item.count * a.group, needed = (n_rows + kSharedRows - 1) / kSharedRows;
  const int groups = needed > 8 ? 16 : (needed > 4 ? 8 : (needed > 2 ? 4 : needed)), parts = kSharedWaves / groups;
  const int row_group = uni(wave & (groups - 1)), part = uni(wave / groups);
  const bool computes = uni(row_group * kSharedRows < n_rows ? 1 : 0);
  const int step0 = uni(parts >= 4 ? part & 3 : part * (4 / parts)), step1 = uni(parts >= 4 ? step0 + 1 : step0 + 4 / parts);
  const int phase = part >> 2, phases = parts >= 4 ? parts / 4 : 1;          // a power of two

  const int row = row_group * kSharedRows + col;
  const RowPlace place(a, item, kvh, row);
  const int position[1] = {place.position};
  f16x8 q[4];
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) q[ks] = query_operand(a, place.at, quarter, ks);
  // positions of the wavefront's rows
  const int wave_first = uni(first_position + row_group * kSharedRows / a.group);
  const int wave_last = uni(min(last_position, first_position + (row_group * kSharedRows + kSharedRows - 1) / a.group));

  const __amdgpu_buffer_rsrc_t tail_rows = pages.tail_rows(a, item, kvh);
  Rows<1> rows;
  rows.clear();
  Trig trig;
  trig.init(tables, a.scale_log2, 16 * quarter + 8 * (wave & 1), tid);
  PageProducer<Trig, RB, W, VB> producer;
  auto load_page = [&](int at, int id) {
    const int page = pages.page(at);
    producer.load(a, kvh, id, page == pages.tail_page, tail_rows, min(kGroup, pages.len - page * kGroup), wave, lane);
  };
  // page `begin` into image[0]; page begin + 1 on its way
  int id = pages.id(begin), id1 = pages.id(begin + 1);
  if (begin < end) load_page(begin, id);
  if constexpr (Trig::kGrouped) {
    trig.build(producer.load_angle(a, kvh, id, lane), 0, wave, kSharedWaves, lane);
    trig.build(producer.load_angle(a, kvh, id1, lane), 1, wave, kSharedWaves, lane);
  }
  __syncthreads();
  if (begin < end) producer.store(trig, 0, a.scale_log2, image[0][0], image[0][1], wave, lane);
  if (begin + 1 < end) load_page(begin + 1, id1);
  __syncthreads();

  for (int at = begin; at < end; ++at) {
    const int parity = (at - begin) & 1, page = pages.page(at);
    const bool masked_page = id < 0;
    id = id1;
    if (at + 1 < end) {
      producer.store(trig, parity ^ 1, a.scale_log2, image[parity ^ 1][0], image[parity ^ 1][1], wave, lane);
      id1 = pages.id(at + 2);
      if (at + 2 < end) load_page(at + 2, id1);
      // the table of this page's parity has been read (before the last barrier)
      if constexpr (Trig::kGrouped) trig.build(producer.load_angle(a, kvh, id1, lane), parity, wave, kSharedWaves, lane);
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
        f32x4 s[2][1];
        s[0][0] = s[1][0] = rows.start(0);
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
#pragma unroll
          for (int tile = 0; tile < 2; ++tile) s[tile][0] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k_image[((2 * step + tile) * 4 + ks) * 64], q[ks], s[tile][0], 0, 0, 0);
        if (masks) rows.mask(a, s, token0, position, quarter);
        rows.settle(s);
        f16x8 p[1];
        rows.weights(s, p);
#pragma unroll
        for (int e = 0; e < 8; ++e) rows.add(e, v_image[(step * 8 + e) * 64], p);
      }
    }
    __syncthreads();
  }

  // ---- fold the parts of a row group ----
  float m = rows.top(0), l = rows.sums[0][0];
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
    for (int e = 0; e < 8; ++e) rows.acc[e][0] *= weight;
    m = top;
    l = total;
    f32x4* const room = reinterpret_cast<f32x4*>(&image[0][0][0]);           // 8 KB a wavefront
    if (part > 0) {
#pragma unroll
      for (int e = 0; e < 8; ++e) room[(wave * 8 + e) * 64 + lane] = rows.acc[e][0];
    }
    __syncthreads();
    if (part > 0) return;
    for (int p = 1; p < parts; ++p) {
#pragma unroll
      for (int e = 0; e < 8; ++e) rows.acc[e][0] += room[((row_group + p * groups) * 8 + e) * 64 + lane];
    }
  }
  if (!computes) return;
  if (item.parts > 1 && row < n_rows) rows.store_part(a, 0, (static_cast<int64_t>(item.unit) * a.n_kv_heads + kvh) * kTileRows + row, m, l, quarter);
  else if (item.parts == 1 && place.there) rows.store_out(0, a.out + place.at, l, quarter);
}

}  // namespace chunk
}  // namespace
}  // namespace pq
