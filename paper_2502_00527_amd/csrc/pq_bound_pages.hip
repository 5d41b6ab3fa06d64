// pq_bound_pages: bounds of the key elements of complete pages, in 8 bits, from the packed codes.
//
// A channel's bounds are the smallest and largest of rho~ cos theta~ (or sin) over 128 tokens.  For one pair and angle code a,
// rho~ grows with the radius code, so that only the smallest and largest radius code seen with a count: the tokens
// leave one bit each, 1 << c in word (a, pair), and 2^t words a pair are evaluated instead of 128 tokens.  A token costs
// the reading of its byte, a shift and an OR in LDS; the words of 64 pairs lie in 64 banks.
// Rounding is monotonic, so that the result is that of all tokens bit for bit.
//
// One work-group a page and KV head: wavefront = 32 tokens, lane = pair.
#include <hip/hip_runtime.h>

#include <cmath>

#include "pq_internal.hpp"

#pragma clang fp contract(off)

namespace pq {
namespace {

constexpr int kBoundThreads = 256;
constexpr int kBoundBytes = 4 * kPairs;                      // of a page and head: centres and half-widths of 128 channels
constexpr float kTiny = 0x1p-100f;                           // below it a block's bounds are zeros

struct BoundArgs {
  const uint8_t* codes;
  const uint32_t* params;
  const int32_t* block_table;
  const int32_t* lens_before;
  const int32_t* lens_after;
  int8_t* bounds;
  float* scales;
  int64_t n_pool_pages;
  int32_t n_kv_heads;
  int32_t max_pages_per_seq;
};

// cos and sin of the centres of the uniform grid's bins, rounded once from float64.
struct BinTable {
  float cs[kMaxAngleBins], sn[kMaxAngleBins];
};

__device__ __forceinline__ float half_of(uint32_t word, int high) {
  return static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(word >> (16 * high))));
}

template <int RB, int TB, bool kGroupedAngles>
__global__ __launch_bounds__(kBoundThreads, 8) void pq_bound_pages_kernel(const BoundArgs a, const BinTable bins) {
  constexpr int W = RB + TB, UB = 2 * W;
  constexpr int kBlockBytes = kGroup * UB, kBlockStride = kBlockBytes + 16;       // (the four pair blocks in different banks)
  constexpr int kStates = 1 << TB;
  __shared__ union {
    __attribute__((aligned(16))) uint8_t codes[kBlocks * kBlockStride + 16];
    __attribute__((aligned(16))) float part[kBoundThreads / 64][kPairs][4];      // when the codes have been read
  } sh;
  __shared__ uint32_t seen[kStates][kPairs];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int kvh = blockIdx.x % a.n_kv_heads, nth = blockIdx.x / a.n_kv_heads, seq = blockIdx.y;
  const int first = a.lens_before ? max(0, a.lens_before[seq]) / kGroup : 0, last = max(0, a.lens_after[seq]) / kGroup;
  const int64_t page_of = static_cast<int64_t>(first) + nth;
  if (page_of >= last || page_of >= a.max_pages_per_seq) return;
  const int64_t page = a.block_table[static_cast<int64_t>(seq) * a.max_pages_per_seq + page_of];
  if (page < 0 || page >= a.n_pool_pages) return;
  const int64_t ph = page * a.n_kv_heads + kvh;

  const uint4* const src = reinterpret_cast<const uint4*>(a.codes + ph * (kBlocks * kBlockBytes));
  constexpr int kQuads = kBlocks * kBlockBytes / 16, kPerThread = (kQuads + kBoundThreads - 1) / kBoundThreads;
  uint4 raw[kPerThread];
#pragma unroll
  for (int i = 0; i < kPerThread; ++i)
    if (i * kBoundThreads + tid < kQuads) raw[i] = src[i * kBoundThreads + tid];
  const uint32_t* const par = a.params + ph * (kPairs * (kGroupedAngles ? 2 : 1));
  const uint32_t radius_par = par[lane], angle_par = kGroupedAngles ? par[kPairs + lane] : 0;
  for (int i = tid; i < kStates * kPairs; i += kBoundThreads) (&seen[0][0])[i] = 0;
#pragma unroll
  for (int i = 0; i < kPerThread; ++i) {
    const int at = (i * kBoundThreads + tid) * 16;
    if (at < kQuads * 16) *reinterpret_cast<uint4*>(sh.codes + at / kBlockBytes * kBlockStride + at % kBlockBytes) = raw[i];
  }
  __syncthreads();

  const int k = lane & 15;
  const uint8_t* const unit = sh.codes + (lane >> 4) * kBlockStride + wave * 32 * UB;
#pragma unroll
  for (int t = 0; t < 32; ++t) {
    uint32_t symbol;
    if constexpr (W == 8) {
      symbol = unit[t * UB + k];
    } else {                                                 // bits 6 k .. 6 k + 5 of the unit
      const uint32_t* const words = reinterpret_cast<const uint32_t*>(unit + t * UB) + 6 * k / 32;
      symbol = __builtin_amdgcn_alignbit(words[1], words[0], 6 * k % 32) & 63u;
    }
    atomicOr(&seen[symbol >> RB][lane], 1u << (symbol & ((1u << RB) - 1)));
  }
  __syncthreads();

  const float rs = half_of(radius_par, 0), rz = half_of(radius_par, 1);
  float low_x = INFINITY, high_x = -INFINITY, low_y = INFINITY, high_y = -INFINITY;
#pragma unroll
  for (int i = 0; i < kStates / 4; ++i) {
    const int state = 4 * i + wave;
    const uint32_t radii = seen[state][lane];
    if (radii == 0) continue;
    float cs, sn;
    if constexpr (kGroupedAngles) {
      const double theta = (state + 0.5) * static_cast<double>(half_of(angle_par, 0)) + static_cast<double>(half_of(angle_par, 1));
      double s, c;
      sincos(theta, &s, &c);
      cs = static_cast<float>(c);
      sn = static_cast<float>(s);
    } else {
      cs = bins.cs[state];
      sn = bins.sn[state];
    }
    // (c + 1/2) s is exact
    const float near = (__builtin_ctz(radii) + 0.5f) * rs + rz, far = (31 - __builtin_clz(radii) + 0.5f) * rs + rz;
    low_x = fminf(low_x, fminf(near * cs, far * cs));
    high_x = fmaxf(high_x, fmaxf(near * cs, far * cs));
    low_y = fminf(low_y, fminf(near * sn, far * sn));
    high_y = fmaxf(high_y, fmaxf(near * sn, far * sn));
  }
  *reinterpret_cast<float4*>(sh.part[wave][lane]) = make_float4(low_x, high_x, low_y, high_y);
  __syncthreads();
  if (wave != 0) return;
#pragma unroll
  for (int w = 1; w < kBoundThreads / 64; ++w) {
    const float4 p = *reinterpret_cast<const float4*>(sh.part[w][lane]);
    low_x = fminf(low_x, p.x);
    high_x = fmaxf(high_x, p.y);
    low_y = fminf(low_y, p.z);
    high_y = fmaxf(high_y, p.w);
  }
  float largest = fmaxf(fmaxf(fabsf(low_x), fabsf(high_x)), fmaxf(fabsf(low_y), fabsf(high_y)));
#pragma unroll
  for (int d = 1; d < 16; d <<= 1) largest = fmaxf(largest, __shfl_xor(largest, d));         // of the block's 16 pairs
  const float up = largest >= kTiny ? 127.0f / largest : 0.f;
  auto code = [&](float v) { return static_cast<int8_t>(static_cast<int>(rintf(v * 0.5f * up))); };
  int8_t* const dst = a.bounds + ph * kBoundBytes + (lane >> 4) * (kBoundBytes / kBlocks) + k;
  dst[0] = code(low_x + high_x);
  dst[16] = code(low_y + high_y);
  dst[32] = code(high_x - low_x);
  dst[48] = code(high_y - low_y);
  if (k == 0) a.scales[ph * kBlocks + (lane >> 4)] = largest / 127.0f;
}

template <int RB, int TB>
void launch_bound(const pq_layout* l, const BoundArgs& a, dim3 grid, hipStream_t st) {
  BinTable bins = {};
  if (l->angle_quantizer == PQ_ANGLE_GROUPED) {
    hipLaunchKernelGGL((pq_bound_pages_kernel<RB, TB, true>), grid, dim3(kBoundThreads), 0, st, a, bins);
    return;
  }
  for (int s = 0; s < (1 << TB); ++s) {
    const double theta = -M_PI + (s + 0.5) * (2.0 * M_PI / (1 << TB));
    bins.cs[s] = static_cast<float>(cos(theta));
    bins.sn[s] = static_cast<float>(sin(theta));
  }
  hipLaunchKernelGGL((pq_bound_pages_kernel<RB, TB, false>), grid, dim3(kBoundThreads), 0, st, a, bins);
}

}  // namespace
}  // namespace pq

using namespace pq;

extern "C" size_t pq_bounds_bytes_per_page(const pq_layout* l) {
  return layout_supported(l) ? static_cast<size_t>(l->n_kv_heads) * kBoundBytes : 0;
}
extern "C" size_t pq_bound_scales_bytes_per_page(const pq_layout* l) {
  return layout_supported(l) ? static_cast<size_t>(l->n_kv_heads) * kBlocks * sizeof(float) : 0;
}

extern "C" int pq_bound_pages(const pq_layout* layout, const void* codes_pool, const void* params_pool, int64_t n_pool_pages,
                              const int32_t* block_table, int32_t max_pages_per_seq, const int32_t* lens_before,
                              const int32_t* lens_after, int32_t n_seqs, int32_t max_new_tokens, void* bounds, void* bound_scales,
                              void* hip_stream) {
  if (!layout) return PQ_ERR_INVALID_ARG;
  if (!layout_supported(layout)) return PQ_ERR_UNSUPPORTED;
  if (n_seqs < 0 || max_new_tokens < 0 || max_pages_per_seq <= 0 || n_pool_pages <= 0) return PQ_ERR_INVALID_ARG;
  if (n_seqs == 0 || max_new_tokens == 0) return PQ_OK;
  if (!codes_pool || !params_pool || !block_table || !lens_after || !bounds || !bound_scales) return PQ_ERR_INVALID_ARG;
  if (((reinterpret_cast<uintptr_t>(codes_pool) | reinterpret_cast<uintptr_t>(params_pool) | reinterpret_cast<uintptr_t>(bounds) |
        reinterpret_cast<uintptr_t>(bound_scales)) & 15u) ||
      ((reinterpret_cast<uintptr_t>(block_table) | reinterpret_cast<uintptr_t>(lens_before) | reinterpret_cast<uintptr_t>(lens_after)) & 3u))
    return PQ_ERR_INVALID_ARG;
  // multiples of g that so many tokens can reach
  const int64_t groups = std::min<int64_t>(max_pages_per_seq, (static_cast<int64_t>(max_new_tokens) + kGroup - 1) / kGroup);
  if (n_seqs > 65535 || groups * layout->n_kv_heads >= (int64_t{1} << 24)) return PQ_ERR_UNSUPPORTED;   // grid
  BoundArgs a;
  a.codes = static_cast<const uint8_t*>(codes_pool);
  a.params = static_cast<const uint32_t*>(params_pool);
  a.block_table = block_table;
  a.lens_before = lens_before;
  a.lens_after = lens_after;
  a.bounds = static_cast<int8_t*>(bounds);
  a.scales = static_cast<float*>(bound_scales);
  a.n_pool_pages = n_pool_pages;
  a.n_kv_heads = layout->n_kv_heads;
  a.max_pages_per_seq = max_pages_per_seq;
  const dim3 grid(static_cast<uint32_t>(groups * layout->n_kv_heads), static_cast<uint32_t>(n_seqs));
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  switch (layout->r_bits * 10 + layout->t_bits) {
    case 44: launch_bound<4, 4>(layout, a, grid, st); break;
    case 33: launch_bound<3, 3>(layout, a, grid, st); break;
    case 53: launch_bound<5, 3>(layout, a, grid, st); break;
    case 35: launch_bound<3, 5>(layout, a, grid, st); break;
    case 42: launch_bound<4, 2>(layout, a, grid, st); break;
    default: launch_bound<2, 4>(layout, a, grid, st); break;     // layout_supported() admits no other
  }
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? PQ_OK : record_hip_error(e);
}
