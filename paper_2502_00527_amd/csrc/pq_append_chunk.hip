// pq_append_chunk: new tokens of a batch into the cache, any number of them a sequence.
//
// Keys.  A sequence of `len` tokens has len % g fp16 rows in its residual buffer; its chunk of n new keys
// completes m = (len % g + n) / g groups.  Work is shared out in tasks, max(m, 1) for each sequence with new tokens and KV head:
// task k < m encodes group k (encode_group, as the encoder does; its rows are the residual's and then the chunk's), and task
// 0 afterwards writes the rows of the incomplete group to the residual buffer -- after, because these are the
// rows that group 0 was read from, and nobody else reads them.  The host knows the number of tokens, not the
// sequences': sum of max(m, 1) <= min(T, T / g + n_seqs), and each work-group finds its task from prefix sums of the tasks.
//
// Values.  A row goes to its slot: copied (fp16), or quantized (value_codes) and written to the halves of the words
// that are its token's.  Rows are independent; work-groups of the same launch behind those of the keys take 128 of one KV head each.
#pragma clang fp contract(off)

#include "pq_encode_group.hpp"
#include "pq_value_codes.hpp"

namespace pq {
namespace {

struct ChunkArgs {
  const void* keys;
  const __half* values;        // null: keys only
  int64_t key_token_stride, key_head_stride, value_token_stride, value_head_stride;
  int64_t n_tokens;
  const int32_t* starts;
  const int32_t* seq_lens;     // before the append
  const int64_t* slots;
  __half* residual;
  const int32_t* block_table;
  uint8_t* codes;
  uint32_t* params;
  void* v_pool;
  uint32_t* v_params;
  int64_t n_pool_pages;
  int32_t n_seqs;
  int32_t n_kv_heads;
  int32_t max_pages_per_seq;
  int32_t v_bits;
  uint32_t key_tasks;          // of a KV head; work-groups from key_tasks * n_kv_heads on are the values'
  double tan_edge[kMaxAngleBins / 8];
  float tan_edge_f[kMaxAngleBins / 8];
};

// Eight elements of a key as fp16, as the residual buffer holds them.
__device__ __forceinline__ u32x4 load_half8(const __half* p) { return *reinterpret_cast<const u32x4*>(p); }
__device__ __forceinline__ u32x4 load_half8(const float* p) {
  float v[8];
  load8(p, v);
  return u32x4{pack_half2(v[0], v[1]), pack_half2(v[2], v[3]), pack_half2(v[4], v[5]), pack_half2(v[6], v[7])};
}

// Rows of a group: the first n_held from the residual buffer, the others from the chunk, where `fresh` is token 0's (also where
// there is none: token t's row is fresh + t * stride).
template <typename KT>
struct ChunkRows {
  const __half* held;
  int n_held;
  const KT* fresh;
  int64_t stride;
  __device__ __forceinline__ void load(RawPairs<__half>& raw, int token, int element) const {
    if (token < n_held) {
      raw.load(held + token * kHeadDim + element);
    } else {
      const KT* const p = fresh + token * stride + element;
      raw.x[0] = load_half8(p);
      raw.y[0] = load_half8(p + kPairs);
    }
  }
};

// A sequence's chunk, as far as it is one.
struct Chunk {
  int64_t first;               // row of its first token
  int len, n;                  // tokens before, new tokens
  __device__ __forceinline__ int held() const { return len % kGroup; }
  __device__ __forceinline__ int complete() const { return static_cast<int>((static_cast<int64_t>(held()) + n) / kGroup); }
  __device__ __forceinline__ int tasks() const { return n > 0 ? max(1, complete()) : 0; }
};
__device__ __forceinline__ Chunk chunk_of(const ChunkArgs& a, int s) {
  Chunk c;
  c.first = min(max(static_cast<int64_t>(a.starts[s]), int64_t{0}), a.n_tokens);
  const int64_t end = min(max(static_cast<int64_t>(a.starts[s + 1]), c.first), a.n_tokens);
  const int len = a.seq_lens[s];
  c.len = max(len, 0);
  c.n = len < 0 ? 0 : static_cast<int>(end - c.first);
  return c;
}

// The sequence and the group of a task; false past the last one.
__device__ __forceinline__ bool find_task(const ChunkArgs& a, uint32_t task, int& seq, int& group) {
  __shared__ uint32_t wave_tasks[kEncThreads / 64];
  __shared__ int found[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (tid == 0) found[0] = -1;
  uint32_t before = 0;
  for (int s0 = 0; s0 < a.n_seqs && before <= task; s0 += kEncThreads) {
    const int s = s0 + tid;
    const uint32_t mine = s < a.n_seqs ? chunk_of(a, s).tasks() : 0;
    uint32_t sum = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t o = __shfl_up(sum, d);
      sum += lane >= d ? o : 0;
    }
    if (lane == 63) wave_tasks[wave] = sum;
    __syncthreads();
    uint32_t all = 0;
#pragma unroll
    for (int w = 0; w < kEncThreads / 64; ++w) {
      sum += w < wave ? wave_tasks[w] : 0;
      all += wave_tasks[w];
    }
    sum += before;
    if (task < sum && task >= sum - mine) {
      found[0] = s;
      found[1] = static_cast<int>(task - (sum - mine));
    }
    before += all;
    __syncthreads();
  }
  seq = __builtin_amdgcn_readfirstlane(found[0]);
  group = __builtin_amdgcn_readfirstlane(found[1]);
  return seq >= 0;
}

template <int RB, int TB, typename KT, bool GA>
__device__ __forceinline__ void append_keys(const ChunkArgs& a, uint32_t task, int kvh, EncodeShared<GA>& stats) {
  int seq, group;
  if (!find_task(a, task, seq, group)) return;
  const Chunk c = chunk_of(a, seq);
  const int held = c.held(), complete = c.complete();
  __half* const res = a.residual + (static_cast<int64_t>(seq) * a.n_kv_heads + kvh) * (kGroup * kHeadDim);
  // row of the token at place 0 of group 0, whether or not it is the chunk's
  const KT* const base = static_cast<const KT*>(a.keys) + (c.first - held) * a.key_token_stride + kvh * a.key_head_stride;
  if (group < complete) {
    const int64_t index = static_cast<int64_t>(c.len / kGroup) + group;
    const int64_t page = index < a.max_pages_per_seq ? a.block_table[static_cast<int64_t>(seq) * a.max_pages_per_seq + index] : -1;
    if (page >= 0 && page < a.n_pool_pages) {
      const int64_t ph = page * a.n_kv_heads + kvh;
      encode_group<RB, TB, __half, GA>(ChunkRows<KT>{res, group == 0 ? held : 0, base + group * kGroup * a.key_token_stride, a.key_token_stride},
                                       kGroup, a.codes + ph * (kBlocks * kGroup * 2 * (RB + TB)), a.params + ph * (kPairs * (GA ? 2 : 1)),
                                       a.tan_edge, a.tan_edge_f, stats);
    }
  }
  if (group != 0) return;
  __syncthreads();                               // group 0 has been read by the whole work-group
  const int from = complete > 0 ? 0 : held, to = static_cast<int>((static_cast<int64_t>(held) + c.n) % kGroup);
  const KT* const tail = base + static_cast<int64_t>(complete) * kGroup * a.key_token_stride;
  for (int i = threadIdx.x; i < (to - from) * (kHeadDim / 8); i += kEncThreads) {
    const int row = from + i / (kHeadDim / 8), element = i % (kHeadDim / 8) * 8;
    *reinterpret_cast<u32x4*>(res + row * kHeadDim + element) = load_half8(tail + row * a.key_token_stride + element);
  }
}

constexpr int kValueRows = 128;                  // of a work-group

template <int VB>
__device__ __forceinline__ void append_quantized(const ChunkArgs& a, int64_t row0, int kvh) {
  using namespace value_codes;
  constexpr int kRows = 4;
  const int sl = threadIdx.x & 7;                // slices sl and sl + 8
  u32x4 raw[kRows][2];
  int64_t slot[kRows];
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    const int64_t row = row0 + (threadIdx.x >> 3) + 32 * k;
    const u32x4* const p = reinterpret_cast<const u32x4*>(a.values + min(row, a.n_tokens - 1) * a.value_token_stride + kvh * a.value_head_stride) + sl;
    raw[k][0] = p[0];
    raw[k][1] = p[8];
    slot[k] = row < a.n_tokens ? a.slots[row] : -1;
  }
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    const uint32_t w[2][4] = {{raw[k][0].x, raw[k][0].y, raw[k][0].z, raw[k][0].w}, {raw[k][1].x, raw[k][1].y, raw[k][1].z, raw[k][1].w}};
    const TokenScale<VB> token(min_and_negated_max({w[0][0], w[0][1], w[0][2], w[0][3], w[1][0], w[1][1], w[1][2], w[1][3]}));
    const uint32_t field[2] = {token.codes(w[0]), token.codes(w[1])};
    const int64_t page = slot[k] / kGroup;
    if (slot[k] < 0 || page >= a.n_pool_pages) continue;
    const int place = static_cast<int>(slot[k] % kGroup);
    const int64_t ph = page * a.n_kv_heads + kvh;
    constexpr int kUnit = 16 / VB;               // tokens
    uint8_t* const block = static_cast<uint8_t*>(a.v_pool) + ph * (kGroup * kHeadDim * VB / 8) + (place / kUnit) * 256;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      uint16_t* const half = reinterpret_cast<uint16_t*>(block + (sl + 8 * p) * 16);
      if constexpr (VB == 4) {
        const int at = (place % 4 / 2) * 4 + place % 2;
        half[at] = static_cast<uint16_t>(field[p]);
        half[at + 2] = static_cast<uint16_t>(field[p] >> 16);
      } else {
        half[place % 8] = static_cast<uint16_t>(field[p]);
      }
    }
    if (sl == 0) a.v_params[ph * kGroup + place] = token.stored;
  }
}

__device__ __forceinline__ void append_rows(const ChunkArgs& a, int64_t row0, int kvh) {
  constexpr int kRows = 8;
  const int quad = threadIdx.x & 15;
  u32x4 raw[kRows];
  int64_t slot[kRows];
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    const int64_t row = row0 + (threadIdx.x >> 4) + 16 * k;
    raw[k] = reinterpret_cast<const u32x4*>(a.values + min(row, a.n_tokens - 1) * a.value_token_stride + kvh * a.value_head_stride)[quad];
    slot[k] = row < a.n_tokens ? a.slots[row] : -1;
  }
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    const int64_t page = slot[k] / kGroup;
    if (slot[k] < 0 || page >= a.n_pool_pages) continue;
    const int64_t at = (page * a.n_kv_heads + kvh) * kGroup + slot[k] % kGroup;
    reinterpret_cast<u32x4*>(static_cast<__half*>(a.v_pool) + at * kHeadDim)[quad] = raw[k];
  }
}

template <int RB, int TB, typename KT, bool GA>
__global__ __launch_bounds__(kEncThreads) void pq_append_chunk_kernel(const ChunkArgs a) {
  __shared__ EncodeShared<GA> stats;
  // the KV heads of a page are neighbours in memory and run together
  const uint32_t unit = blockIdx.x / a.n_kv_heads;
  const int kvh = blockIdx.x % a.n_kv_heads;
  if (unit < a.key_tasks) {
    append_keys<RB, TB, KT, GA>(a, unit, kvh, stats);
    return;
  }
  const int64_t row0 = static_cast<int64_t>(unit - a.key_tasks) * kValueRows;
  if (a.v_bits == 16) append_rows(a, row0, kvh);
  else if (a.v_bits == 4) append_quantized<4>(a, row0, kvh);
  else append_quantized<2>(a, row0, kvh);
}

template <int RB, int TB, bool GA = false>
hipError_t launch_chunk(const ChunkArgs& a, pq_dtype dt, dim3 grid, hipStream_t st) {
  if (dt == PQ_F16) hipLaunchKernelGGL((pq_append_chunk_kernel<RB, TB, __half, GA>), grid, dim3(kEncThreads), 0, st, a);
  else              hipLaunchKernelGGL((pq_append_chunk_kernel<RB, TB, float, GA>), grid, dim3(kEncThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace
}  // namespace pq

using namespace pq;

extern "C" int pq_append_chunk(const pq_layout* layout, const void* keys, pq_dtype key_dtype, int64_t key_token_stride,
                               int64_t key_head_stride, const void* values, int64_t value_token_stride, int64_t value_head_stride,
                               int64_t n_tokens, int32_t n_seqs, const int32_t* starts, const int32_t* seq_lens,
                               const int64_t* slots, void* residual, const int32_t* block_table, int32_t max_pages_per_seq,
                               void* codes_pool, void* params_pool, void* v_pool, int32_t v_bits, void* v_params_pool,
                               int64_t n_pool_pages, void* hip_stream) {
  if (!layout) return PQ_ERR_INVALID_ARG;
  if (!layout_supported(layout)) return PQ_ERR_UNSUPPORTED;
  if (n_tokens < 0 || n_seqs < 0 || n_pool_pages <= 0 || max_pages_per_seq <= 0) return PQ_ERR_INVALID_ARG;
  if (key_dtype != PQ_F16 && key_dtype != PQ_F32) return PQ_ERR_INVALID_ARG;
  if (values && v_bits != 16 && v_bits != 4 && v_bits != 2) return PQ_ERR_UNSUPPORTED;
  if (n_tokens == 0 || n_seqs == 0) return PQ_OK;
  if (!keys || !starts || !seq_lens || !residual || !block_table || !codes_pool || !params_pool) return PQ_ERR_INVALID_ARG;
  if (values && (!slots || !v_pool || (v_bits != 16 && !v_params_pool))) return PQ_ERR_INVALID_ARG;
  // 128-bit loads and stores
  const int64_t vec = key_dtype == PQ_F16 ? 8 : 4;
  if ((reinterpret_cast<uintptr_t>(keys) & 15u) || key_token_stride % vec || key_head_stride % vec || key_token_stride < 0 || key_head_stride < 0)
    return PQ_ERR_INVALID_ARG;
  if (values && ((reinterpret_cast<uintptr_t>(values) & 15u) || value_token_stride % 8 || value_head_stride % 8 || value_token_stride < 0 ||
                 value_head_stride < 0 || (reinterpret_cast<uintptr_t>(v_pool) & 15u) || (reinterpret_cast<uintptr_t>(slots) & 7u) ||
                 (v_bits != 16 && (reinterpret_cast<uintptr_t>(v_params_pool) & 3u))))
    return PQ_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(residual) | reinterpret_cast<uintptr_t>(codes_pool) | reinterpret_cast<uintptr_t>(params_pool)) & 15u)
    return PQ_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(starts) | reinterpret_cast<uintptr_t>(seq_lens) | reinterpret_cast<uintptr_t>(block_table)) & 3u)
    return PQ_ERR_INVALID_ARG;
  const int64_t key_tasks = std::min<int64_t>(n_tokens, n_tokens / kGroup + n_seqs);
  const int64_t value_tasks = values ? (n_tokens + kValueRows - 1) / kValueRows : 0;
  // work-groups of 256 threads in one grid dimension of HIP, which takes 2^32 - 1 threads; rows are int32 in `starts`
  if (n_tokens >= (int64_t{1} << 31) || (key_tasks + value_tasks) * layout->n_kv_heads >= (int64_t{1} << 24)) return PQ_ERR_UNSUPPORTED;
  ChunkArgs a;
  a.keys = keys;
  a.values = static_cast<const __half*>(values);
  a.key_token_stride = key_token_stride;
  a.key_head_stride = key_head_stride;
  a.value_token_stride = value_token_stride;
  a.value_head_stride = value_head_stride;
  a.n_tokens = n_tokens;
  a.starts = starts;
  a.seq_lens = seq_lens;
  a.slots = slots;
  a.residual = static_cast<__half*>(residual);
  a.block_table = block_table;
  a.codes = static_cast<uint8_t*>(codes_pool);
  a.params = static_cast<uint32_t*>(params_pool);
  a.v_pool = v_pool;
  a.v_params = static_cast<uint32_t*>(v_params_pool);
  a.n_pool_pages = n_pool_pages;
  a.n_seqs = n_seqs;
  a.n_kv_heads = layout->n_kv_heads;
  a.max_pages_per_seq = max_pages_per_seq;
  a.v_bits = v_bits;
  a.key_tasks = static_cast<uint32_t>(key_tasks);
  fill_edges(a, layout->t_bits);
  const dim3 grid(static_cast<uint32_t>((key_tasks + value_tasks) * layout->n_kv_heads));
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  hipError_t e = hipSuccess;
  switch (layout->r_bits * 10 + layout->t_bits + (layout->angle_quantizer == PQ_ANGLE_GROUPED ? 100 : 0)) {
    case 144: e = launch_chunk<4, 4, true>(a, key_dtype, grid, st); break;
    case 133: e = launch_chunk<3, 3, true>(a, key_dtype, grid, st); break;
    case 153: e = launch_chunk<5, 3, true>(a, key_dtype, grid, st); break;
    case 135: e = launch_chunk<3, 5, true>(a, key_dtype, grid, st); break;
    case 142: e = launch_chunk<4, 2, true>(a, key_dtype, grid, st); break;
    case 124: e = launch_chunk<2, 4, true>(a, key_dtype, grid, st); break;
    case 44: e = launch_chunk<4, 4>(a, key_dtype, grid, st); break;
    case 33: e = launch_chunk<3, 3>(a, key_dtype, grid, st); break;
    case 53: e = launch_chunk<5, 3>(a, key_dtype, grid, st); break;
    case 35: e = launch_chunk<3, 5>(a, key_dtype, grid, st); break;
    case 42: e = launch_chunk<4, 2>(a, key_dtype, grid, st); break;
    default: e = launch_chunk<2, 4>(a, key_dtype, grid, st); break;       // layout_supported() admits no other
  }
  return e == hipSuccess ? PQ_OK : record_hip_error(e);
}
