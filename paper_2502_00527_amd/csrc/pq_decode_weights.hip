// Decode attention that leaves each page's sum of exponentials beside its output (pq_decode_attention_weights): the kernels of
// pq_decode_matrix.hpp with kWeights, and their launch ladder.  The grouped quantizer's walk serves one and two query heads per KV head, too.  Attention over chosen pages
// with quantized values goes through them without the sums.
//
// This file is the fp16-value kernels; pq_decode_weights_v4.hip and pq_decode_weights_v2.hip compile it again for 4-bit and
// 2-bit values.
#include "pq_decode_matrix.hpp"

#ifndef PQ_WEIGHTS_VB
#define PQ_WEIGHTS_VB 16
#define PQ_WEIGHTS_LAUNCH launch_weights_v16
#endif

namespace pq {
namespace {
namespace weights {

#define PQ_WEIGHTS_ATTR(waves) __launch_bounds__(waves * 64) __attribute__((amdgpu_waves_per_eu(2, 2)))

template <int W, int VB, int NH, bool Q32, bool kCut, int kWaves>
__global__ PQ_WEIGHTS_ATTR(kWaves) void pq_decode_weights_kernel(const DecodeArgs a) { attention_body<W, VB, NH, Q32, kCut, kWaves, 0, false, true>(a); }
template <int RB, int TB, int VB, int NH, bool kCut>
__global__ PQ_WEIGHTS_ATTR(4) void pq_decode_weights_grouped_kernel(const DecodeArgs a) { attention_body<RB + TB, VB, NH, true, kCut, 4, RB, false, true>(a); }

template <int W, int NH, bool Q32>
void launch_uniform(const DecodeArgs& a, dim3 grid, hipStream_t st) {
  if (a.cut_places > 0) hipLaunchKernelGGL((pq_decode_weights_kernel<W, PQ_WEIGHTS_VB, NH, Q32, true, 4>), grid, dim3(256), 0, st, a);
  else if (a.wide_groups) hipLaunchKernelGGL((pq_decode_weights_kernel<W, PQ_WEIGHTS_VB, NH, Q32, false, 8>), grid, dim3(512), 0, st, a);
  else hipLaunchKernelGGL((pq_decode_weights_kernel<W, PQ_WEIGHTS_VB, NH, Q32, false, 4>), grid, dim3(256), 0, st, a);
}
template <int W>
bool launch_q(const DecodeArgs& a, dim3 grid, hipStream_t st) {
  if (a.n_heads <= 4) a.q_is_f32 ? launch_uniform<W, 4, true>(a, grid, st) : launch_uniform<W, 4, false>(a, grid, st);
  else a.q_is_f32 ? launch_uniform<W, 8, true>(a, grid, st) : launch_uniform<W, 8, false>(a, grid, st);
  return true;
}
template <int RB, int TB, int NH>
void launch_heads(const DecodeArgs& a, dim3 grid, hipStream_t st) {
  if (a.cut_places > 0) hipLaunchKernelGGL((pq_decode_weights_grouped_kernel<RB, TB, PQ_WEIGHTS_VB, NH, true>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((pq_decode_weights_grouped_kernel<RB, TB, PQ_WEIGHTS_VB, NH, false>), grid, dim3(256), 0, st, a);
}
template <int RB, int TB>
bool launch_grouped(const DecodeArgs& a, dim3 grid, hipStream_t st) {
  if (a.n_heads <= 4) launch_heads<RB, TB, 4>(a, grid, st);
  else launch_heads<RB, TB, 8>(a, grid, st);
  return true;
}

}  // namespace weights
}  // namespace

bool PQ_WEIGHTS_LAUNCH(const pq_layout* l, const DecodeArgs& a, dim3 grid, hipStream_t st) {
  switch (l->r_bits * 10 + l->t_bits + (l->angle_quantizer == PQ_ANGLE_GROUPED ? 100 : 0)) {
    case 44: case 53: case 35: return weights::launch_q<8>(a, grid, st);
    case 33: case 42: case 24: return weights::launch_q<6>(a, grid, st);
    case 144: return weights::launch_grouped<4, 4>(a, grid, st);
    case 133: return weights::launch_grouped<3, 3>(a, grid, st);
    case 153: return weights::launch_grouped<5, 3>(a, grid, st);
    case 135: return weights::launch_grouped<3, 5>(a, grid, st);
    case 142: return weights::launch_grouped<4, 2>(a, grid, st);
    case 124: return weights::launch_grouped<2, 4>(a, grid, st);
    default: return false;
  }
}

}  // namespace pq
