// pq_bound_pages: bounds of the key elements of complete pages, in 8 bits, from the packed codes.
//
// A channel's bounds are the smallest and largest of rho~ cos theta~ (or sin) over 128 tokens.  For one pair and angle code a,
// rho~ grows with the radius code, so that only the smallest and largest radius code seen with a count: the tokens
// leave one bit each, of 2^(r + t) a pair, and 2^t states a pair are evaluated instead of 128 tokens.
// Rounding is monotonic, so that the result is that of all tokens bit for bit.
//
// A bit is set by an OR in LDS (lane = pair: its words lie in its own bank).  An instruction brings address and data of 64 lanes to LDS in
// about 8 cycles, whatever the SIMD, a byte's reading in 4: with the symbols read from LDS one by one that path was busy for 83 % of 50 us
// (8 x 20K .. 32K tokens x 8 heads).  So a wavefront loads a token's unit of 16 symbols a lane and transposes bytes between the 16 lanes of a
// block of pairs in registers, 20 instructions for 16 symbols: 29 us.  What bounds it then is vector issue, busy for 72 % of that with launch and
// tail; 114 MB at 7 TB/s are 16 us.
//
// One work-group a page and KV head; wavefront = 32 tokens.  16384 pages and heads of 8-bit symbols: 35.9 us, 4096: 11.3, 512: 3.7.  With four
// heads one after the other, the next one's codes on their way meanwhile: 39.1, 13.9, 7.2.
#include <hip/hip_runtime.h>

#include <cmath>

#include "pq_decode_kernels.hpp"
#include "pq_internal.hpp"
#include "pq_rank.hpp"

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

__device__ __forceinline__ float min3(float a, float b, float c) {
  float r;
  asm("v_min3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
__device__ __forceinline__ float max_rows(float x) {         // over the 4 rows of 16 lanes; not negative: in the order of its bits
  return __builtin_bit_cast(float, over_rows(__builtin_bit_cast(uint32_t, x), [](uint32_t a, uint32_t b) { return max(a, b); }));
}

// Lanes and symbols.  Lane l loads the unit of block (l >> 2) & 3 and token {l & 3, bits 4 and 5 of l}; afterwards it has the symbols of 16 tokens
// of pair 16 block + {l & 3, bits 4 and 5 of l} of them.
__device__ __forceinline__ int lane_block(int lane) { return (lane >> 2) & 3; }
__device__ __forceinline__ int lane_place(int lane) { return (lane & 3) | ((lane >> 2) & 12); }
template <int CTRL>
__device__ __forceinline__ void swap_bytes(uint32_t (&d)[4], uint32_t select) {
#pragma unroll
  for (int i = 0; i < 4; ++i) d[i] = __builtin_amdgcn_perm(moved<CTRL>(d[i]), d[i], select);
}
__device__ __forceinline__ void transpose_bytes(uint32_t (&d)[4], uint32_t select2, uint32_t select1) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {                              // bit 3 of the place against lane bit 5: words i and i + 2
    const auto r = __builtin_amdgcn_permlane32_swap(d[i], d[i + 2], false, false);
    d[i] = r[0];
    d[i + 2] = r[1];
  }
#pragma unroll
  for (int i = 0; i < 4; i += 2) {                           // bit 2 against lane bit 4: words i and i + 1
    const auto r = __builtin_amdgcn_permlane16_swap(d[i], d[i + 1], false, false);
    d[i] = r[0];
    d[i + 1] = r[1];
  }
  swap_bytes<0x4e>(d, select2);                              // bit 1 against lane bit 1 (quad_perm 2, 3, 0, 1), bit 0 against lane bit 0 (1, 0, 3, 2)
  swap_bytes<0xb1>(d, select1);
}
// A unit as it lies in memory, and as one symbol a byte (6-bit symbols: with two bits of the next one above them).
template <int W>
struct TokenUnit {
  uint32_t w[W / 2];
  __device__ __forceinline__ void load(const uint8_t* from) {
    if constexpr (W == 8) {
      const uint4 v = *reinterpret_cast<const uint4*>(from);
      w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    } else {
      const uint32_t* const src = reinterpret_cast<const uint32_t*>(from);
      w[0] = src[0]; w[1] = src[1]; w[2] = src[2];
    }
  }
  __device__ __forceinline__ void symbols(uint32_t (&d)[4]) const {
    if constexpr (W == 8) {
#pragma unroll
      for (int i = 0; i < 4; ++i) d[i] = w[i];
    } else {
      const uint32_t four[4] = {w[0], __builtin_amdgcn_alignbit(w[1], w[0], 24), __builtin_amdgcn_alignbit(w[2], w[1], 16), w[2] >> 8};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t x = four[i];
        d[i] = (x & 0xffu) | ((x << 2) & 0xff00u) | ((x << 4) & 0xff0000u) | ((x << 6) & 0xff000000u);
      }
    }
  }
};

// 1 << (byte `kByte` of x, its low five bits)
template <int kByte>
__device__ __forceinline__ uint32_t bit_of_byte(uint32_t x, uint32_t one) {
  if constexpr (kByte == 0) return one << (x & 31);
  uint32_t r;
  if constexpr (kByte == 1) asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_1 src1_sel:DWORD" : "=v"(r) : "v"(x), "v"(one));
  if constexpr (kByte == 2) asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_2 src1_sel:DWORD" : "=v"(r) : "v"(x), "v"(one));
  if constexpr (kByte == 3) asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_3 src1_sel:DWORD" : "=v"(r) : "v"(x), "v"(one));
  return r;
}

// cos and sin of |theta| < 4, good to a few units of 2^-53: Cody and Waite's reduction by quarter turns with pi / 2 in two parts, then the Taylor
// series on [-pi / 4, pi / 4], whose first omitted terms are below 2^-54.
__device__ __forceinline__ void cos_sin(double theta, float& cs, float& sn) {
  constexpr double kHigh = 0x1.921fb54442d18p+0, kLow = 0x1.1a62633145c07p-54;             // pi / 2
  const double turns = rint(theta * 0x1.45f306dc9c883p-1);                                 // 2 / pi
  const double x = fma(-turns, kLow, fma(-turns, kHigh, theta)), y = x * x;
  double s = -1.0 / 1307674368000.0, c = 1.0 / 20922789888000.0;                           // 15!, 16!
  s = fma(s, y, 1.0 / 6227020800.0);
  s = fma(s, y, -1.0 / 39916800.0);
  s = fma(s, y, 1.0 / 362880.0);
  s = fma(s, y, -1.0 / 5040.0);
  s = fma(s, y, 1.0 / 120.0);
  s = fma(s, y, -1.0 / 6.0);
  s = fma(s * y, x, x);
  c = fma(c, y, -1.0 / 87178291200.0);
  c = fma(c, y, 1.0 / 479001600.0);
  c = fma(c, y, -1.0 / 3628800.0);
  c = fma(c, y, 1.0 / 40320.0);
  c = fma(c, y, -1.0 / 720.0);
  c = fma(c, y, 1.0 / 24.0);
  c = fma(c, y, -0.5);
  c = fma(c, y, 1.0);
  const int quarter = static_cast<int>(turns);
  const float fs = static_cast<float>(s), fc = static_cast<float>(c);
  const float a = quarter & 1 ? fs : fc, b = quarter & 1 ? fc : fs;
  cs = (quarter + 1) & 2 ? -a : a;
  sn = quarter & 2 ? -b : b;
}

template <int RB, int TB, bool kGroupedAngles>
__global__ __launch_bounds__(kBoundThreads, kGroupedAngles ? 5 : 8) void pq_bound_pages_kernel(const BoundArgs a, const BinTable bins) {
  constexpr int W = RB + TB, UB = 2 * W;
  constexpr int kWords = (1 << W) / 32, kOfWord = 32 >> RB;                       // of a pair's bits; angle codes of a word
  static_assert(kPairs * 4 == 256, "a word's number is the second byte of an address, the lane its first");
  __shared__ struct {
    __attribute__((aligned(16))) uint32_t seen[kWords][kPairs];
    __attribute__((aligned(16))) float part[kBoundThreads / 64][kPairs][4];
  } sh;
  auto& seen = sh.seen;
  auto& part = sh.part;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kvh = blockIdx.x % a.n_kv_heads, nth = blockIdx.x / a.n_kv_heads, seq = blockIdx.y;
  const int first = a.lens_before ? max(0, a.lens_before[seq]) / kGroup : 0, last = max(0, a.lens_after[seq]) / kGroup;
  const int64_t page_of = static_cast<int64_t>(first) + nth;
  if (page_of >= last || page_of >= a.max_pages_per_seq) return;
  const int64_t page = a.block_table[static_cast<int64_t>(seq) * a.max_pages_per_seq + page_of];
  if (page < 0 || page >= a.n_pool_pages) return;
  const int64_t ph = page * a.n_kv_heads + kvh;
  const int block = lane_block(lane), k = lane_place(lane), pair = block * 16 + k;
  // bytes {0, 1} of the own word and of the other lane's in the lane below, {2, 3} in the one above; then the even ones and the odd ones
  const uint32_t select2 = lane & 2 ? 0x03020706u : 0x05040100u, select1 = lane & 1 ? 0x03070105u : 0x06020400u;

  const uint32_t lane4 = lane * 4, seen_at = lds_addr(&seen[0][0]);
  uint32_t one = 1;
  asm("" : "+v"(one));
  TokenUnit<W> raw[2];
  const uint8_t* const from = a.codes + ph * (kBlocks * kGroup * UB) + (block * kGroup + wave * 32 + k) * UB;
  raw[0].load(from);
  raw[1].load(from + 16 * UB);
  const uint32_t* const par = a.params + ph * (kPairs * (kGroupedAngles ? 2 : 1));
  const uint32_t radius_par = par[pair], angle_par = kGroupedAngles ? par[kPairs + pair] : 0;
  for (int i = tid; i < kWords * kPairs; i += kBoundThreads) (&seen[0][0])[i] = 0;
  __syncthreads();
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    uint32_t d[4];
    raw[u].symbols(d);
    transpose_bytes(d, select2, select1);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t four = d[i], words = (four >> 5) & (0x01010101u * (kWords - 1));            // (bits above a symbol's are another's)
      auto set = [&](uint32_t at, uint32_t bit) {
        __hip_atomic_fetch_or((PQ_LDS uint32_t*)static_cast<uintptr_t>(seen_at + at), bit, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
      };
      set(__builtin_amdgcn_perm(words, lane4, 0x0c0c0400u), bit_of_byte<0>(four, one));
      set(__builtin_amdgcn_perm(words, lane4, 0x0c0c0500u), bit_of_byte<1>(four, one));
      set(__builtin_amdgcn_perm(words, lane4, 0x0c0c0600u), bit_of_byte<2>(four, one));
      set(__builtin_amdgcn_perm(words, lane4, 0x0c0c0700u), bit_of_byte<3>(four, one));
    }
  }
  __syncthreads();

  const float rs = half_of(radius_par, 0), rz = half_of(radius_par, 1), ts = half_of(angle_par, 0), tz = half_of(angle_par, 1);
  float low_x = INFINITY, high_x = -INFINITY, low_y = INFINITY, high_y = -INFINITY;
#pragma unroll kGroupedAngles ? 1 : (1 << TB) / 4
  for (int i = 0; i < (1 << TB) / 4; ++i) {
    const int state = 4 * i + wave;                        // angle code
    const uint32_t radii = (seen[state / kOfWord][lane] >> ((state % kOfWord) << RB)) & static_cast<uint32_t>((uint64_t{1} << (1 << RB)) - 1);
    float cs, sn;
    if constexpr (kGroupedAngles) {
      cos_sin((state + 0.5) * static_cast<double>(ts) + static_cast<double>(tz), cs, sn);
    } else {
      cs = bins.cs[state];
      sn = bins.sn[state];
    }
    // (c + 1/2) s is exact, so that one rounding is what its sum with z has.  A state that nobody has is no number, which minima and maxima pass over
    float near = fmaf(__builtin_ctz(radii) + 0.5f, rs, rz), far = fmaf(31.5f - __builtin_clz(radii), rs, rz);
    near = radii == 0 ? NAN : near;
    far = radii == 0 ? NAN : far;
    low_x = min3(low_x, near * cs, far * cs);
    high_x = max3(high_x, near * cs, far * cs);
    low_y = min3(low_y, near * sn, far * sn);
    high_y = max3(high_y, near * sn, far * sn);
  }
  *reinterpret_cast<float4*>(part[wave][lane]) = make_float4(low_x, high_x, low_y, high_y);
  __syncthreads();
  if (wave != 0) return;
#pragma unroll
  for (int w = 1; w < kBoundThreads / 64; ++w) {
    const float4 p = *reinterpret_cast<const float4*>(part[w][lane]);
    low_x = fminf(low_x, p.x);
    high_x = fmaxf(high_x, p.y);
    low_y = fminf(low_y, p.z);
    high_y = fmaxf(high_y, p.w);
  }
  float largest = fmaxf(fmaxf(fabsf(low_x), fabsf(high_x)), fmaxf(fabsf(low_y), fabsf(high_y)));
  largest = fmaxf(largest, __builtin_bit_cast(float, moved<0x4e>(__builtin_bit_cast(uint32_t, largest))));   // of the block's 16 pairs
  largest = fmaxf(largest, __builtin_bit_cast(float, moved<0xb1>(__builtin_bit_cast(uint32_t, largest))));
  largest = max_rows(largest);
  const float up = largest >= kTiny ? 127.0f / largest : 0.f;
  auto code = [&](float v) { return static_cast<int8_t>(static_cast<int>(rintf(v * 0.5f * up))); };
  int8_t* const dst = a.bounds + ph * kBoundBytes + block * (kBoundBytes / kBlocks) + k;
  dst[0] = code(low_x + high_x);
  dst[16] = code(low_y + high_y);
  dst[32] = code(high_x - low_x);
  dst[48] = code(high_y - low_y);
  if (k == 0) a.scales[ph * kBlocks + block] = largest / 127.0f;
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
