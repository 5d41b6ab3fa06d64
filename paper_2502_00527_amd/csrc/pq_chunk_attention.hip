// Kernels of pq_chunk_attention (pq_chunk_kernels.hpp) and their launch ladder.
//
// This file is the fp16-value kernels, the merge of splits and the entry points; pq_chunk_attention_v4.hip and
// pq_chunk_attention_v2.hip compile the kernels again for 4-bit and 2-bit values.
#include "pq_chunk_kernels.hpp"

#ifndef PQ_CHUNK_VB
#define PQ_CHUNK_VB 16
#define PQ_CHUNK_LAUNCH launch_chunk_v16
#endif

namespace pq {
namespace {
namespace chunk {

#define PQ_CHUNK_ATTR(rt) __launch_bounds__(kChunkWaves * 64) __attribute__((amdgpu_waves_per_eu(rt == 1 ? 2 : 1, rt == 1 ? 2 : 1)))
#define PQ_SHARED_ATTR __launch_bounds__(kSharedWaves * 64) __attribute__((amdgpu_waves_per_eu(kSharedWaves / 4, kSharedWaves / 4)))

template <int RB, int TB, int VB, bool kGrouped>
__global__ PQ_SHARED_ATTR void pq_chunk_shared_kernel(const ChunkAttentionArgs a) {
  shared_body<std::conditional_t<kGrouped, SharedGroupedKeys<RB, TB>, SharedUniformKeys<RB, TB>>, RB, VB>(a);
}
template <int RB, int TB, int VB>
bool launch_shared(bool grouped, const ChunkAttentionArgs& a, dim3 grid, hipStream_t st) {
  if (grouped) hipLaunchKernelGGL((pq_chunk_shared_kernel<RB, TB, VB, true>), grid, dim3(kSharedWaves * 64), 0, st, a);
  else hipLaunchKernelGGL((pq_chunk_shared_kernel<RB, TB, VB, false>), grid, dim3(kSharedWaves * 64), 0, st, a);
  return true;
}
template <int VB>
bool launch_shared(const pq_layout* l, const ChunkAttentionArgs& a, dim3 grid, hipStream_t st) {
  const bool grouped = l->angle_quantizer == PQ_ANGLE_GROUPED;
  switch (l->r_bits * 10 + l->t_bits) {
    case 44: return launch_shared<4, 4, VB>(grouped, a, grid, st);
    case 33: return launch_shared<3, 3, VB>(grouped, a, grid, st);
    case 53: return launch_shared<5, 3, VB>(grouped, a, grid, st);
    case 35: return launch_shared<3, 5, VB>(grouped, a, grid, st);
    case 42: return launch_shared<4, 2, VB>(grouped, a, grid, st);
    case 24: return launch_shared<2, 4, VB>(grouped, a, grid, st);
    default: return false;
  }
}

template <int W, int VB, int RT>
__global__ PQ_CHUNK_ATTR(RT) void pq_chunk_attention_kernel(const ChunkAttentionArgs a) { attention_body<UniformKeys<W>, W, false, VB, RT>(a); }
template <int RB, int TB, int VB, int RT>
__global__ PQ_CHUNK_ATTR(RT) void pq_chunk_grouped_kernel(const ChunkAttentionArgs a) { attention_body<GroupedKeys<RB, TB>, RB + TB, true, VB, RT>(a); }

template <int VB, int RT>
bool launch(const pq_layout* l, const ChunkAttentionArgs& a, dim3 grid, hipStream_t st) {
  const dim3 block(kChunkWaves * 64);
  switch (l->r_bits * 10 + l->t_bits + (l->angle_quantizer == PQ_ANGLE_GROUPED ? 100 : 0)) {
    case 44: case 53: case 35: hipLaunchKernelGGL((pq_chunk_attention_kernel<8, VB, RT>), grid, block, 0, st, a); return true;
    case 33: case 42: case 24: hipLaunchKernelGGL((pq_chunk_attention_kernel<6, VB, RT>), grid, block, 0, st, a); return true;
    case 144: hipLaunchKernelGGL((pq_chunk_grouped_kernel<4, 4, VB, RT>), grid, block, 0, st, a); return true;
    case 133: hipLaunchKernelGGL((pq_chunk_grouped_kernel<3, 3, VB, RT>), grid, block, 0, st, a); return true;
    case 153: hipLaunchKernelGGL((pq_chunk_grouped_kernel<5, 3, VB, RT>), grid, block, 0, st, a); return true;
    case 135: hipLaunchKernelGGL((pq_chunk_grouped_kernel<3, 5, VB, RT>), grid, block, 0, st, a); return true;
    case 142: hipLaunchKernelGGL((pq_chunk_grouped_kernel<4, 2, VB, RT>), grid, block, 0, st, a); return true;
    case 124: hipLaunchKernelGGL((pq_chunk_grouped_kernel<2, 4, VB, RT>), grid, block, 0, st, a); return true;
    default: return false;
  }
}

}  // namespace chunk
}  // namespace

bool PQ_CHUNK_LAUNCH(const pq_layout* l, int rows_of_16, const ChunkAttentionArgs& a, dim3 grid, hipStream_t st) {
  return rows_of_16 == 1 ? chunk::launch<PQ_CHUNK_VB, 1>(l, a, grid, st) : chunk::launch_shared<PQ_CHUNK_VB>(l, a, grid, st);
}

}  // namespace pq
