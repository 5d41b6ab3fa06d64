// Kernels of pq_chunk_attention (pq_chunk_kernels.hpp) and their launch ladder.
//
// This file is the fp16-value kernels; pq_chunk_attention_v4.hip and pq_chunk_attention_v2.hip compile it again for 4-bit and
// 2-bit values.
#include "pq_chunk_kernels.hpp"

#ifndef PQ_CHUNK_VB
#define PQ_CHUNK_VB 16
#define PQ_CHUNK_LAUNCH launch_chunk_v16
#endif

namespace pq {
namespace {
namespace chunk {

#define PQ_CHUNK_ATTR(waves, per_simd) __launch_bounds__((waves) * 64) __attribute__((amdgpu_waves_per_eu(per_simd, per_simd)))
template <int RB, int TB, bool kGrouped>
using TrigOf = std::conditional_t<kGrouped, GroupedTrig<RB, TB>, UniformTrig<RB, TB>>;

template <int RB, int TB, int VB, int RT, bool kGrouped>
__global__ PQ_CHUNK_ATTR(kFewWaves, 2) void pq_chunk_few_kernel(const ChunkAttentionArgs a) { few_body<TrigOf<RB, TB, kGrouped>, RB, RB + TB, VB, RT>(a); }
template <int RB, int TB, int VB, bool kGrouped>
__global__ PQ_CHUNK_ATTR(kSharedWaves, kSharedWaves / 4) void pq_chunk_shared_kernel(const ChunkAttentionArgs a) { shared_body<TrigOf<RB, TB, kGrouped>, RB, RB + TB, VB>(a); }

template <int RB, int TB, bool kGrouped>
bool launch(int rows_of_16, const ChunkAttentionArgs& a, dim3 grid, hipStream_t st) {
  if (rows_of_16 == 1) hipLaunchKernelGGL((pq_chunk_few_kernel<RB, TB, PQ_CHUNK_VB, 1, kGrouped>), grid, dim3(kFewWaves * 64), 0, st, a);
  else if (rows_of_16 == 2) hipLaunchKernelGGL((pq_chunk_few_kernel<RB, TB, PQ_CHUNK_VB, 2, kGrouped>), grid, dim3(kFewWaves * 64), 0, st, a);
  else hipLaunchKernelGGL((pq_chunk_shared_kernel<RB, TB, PQ_CHUNK_VB, kGrouped>), grid, dim3(kSharedWaves * 64), 0, st, a);
  return true;
}

}  // namespace chunk
}  // namespace

bool PQ_CHUNK_LAUNCH(const pq_layout* l, int rows_of_16, const ChunkAttentionArgs& a, dim3 grid, hipStream_t st) {
  switch (l->r_bits * 10 + l->t_bits + (l->angle_quantizer == PQ_ANGLE_GROUPED ? 100 : 0)) {
    case 44: return chunk::launch<4, 4, false>(rows_of_16, a, grid, st);
    case 33: return chunk::launch<3, 3, false>(rows_of_16, a, grid, st);
    case 53: return chunk::launch<5, 3, false>(rows_of_16, a, grid, st);
    case 35: return chunk::launch<3, 5, false>(rows_of_16, a, grid, st);
    case 42: return chunk::launch<4, 2, false>(rows_of_16, a, grid, st);
    case 24: return chunk::launch<2, 4, false>(rows_of_16, a, grid, st);
    case 144: return chunk::launch<4, 4, true>(rows_of_16, a, grid, st);
    case 133: return chunk::launch<3, 3, true>(rows_of_16, a, grid, st);
    case 153: return chunk::launch<5, 3, true>(rows_of_16, a, grid, st);
    case 135: return chunk::launch<3, 5, true>(rows_of_16, a, grid, st);
    case 142: return chunk::launch<4, 2, true>(rows_of_16, a, grid, st);
    case 124: return chunk::launch<2, 4, true>(rows_of_16, a, grid, st);
    default: return false;
  }
}

}  // namespace pq
