// Attention through a sliding window with sinks: the kernels of pq_decode_matrix.hpp with the pages between sinks and window left
// out (WindowView), and their launch ladder.  The grouped quantizer's walk serves one and two query heads per KV head, too:
// its kernel on the vector unit knows of no window.
//
// This file is the fp16-value kernels; pq_decode_window_v4.hip and pq_decode_window_v2.hip compile it again for 4-bit and
// 2-bit values.
#include "pq_decode_matrix.hpp"

#ifndef PQ_WINDOW_VB
#define PQ_WINDOW_VB 16
#define PQ_WINDOW_LAUNCH launch_window_v16
#endif

namespace pq {
namespace {
namespace window {

#define PQ_WINDOW_ATTR(waves) __launch_bounds__(waves * 64) __attribute__((amdgpu_waves_per_eu(2, 2)))

template <int W, int VB, int NH, bool Q32, int kWaves>
__global__ PQ_WINDOW_ATTR(kWaves) void pq_window_attention_kernel(const DecodeArgs a) { attention_body<W, VB, NH, Q32, false, kWaves, 0, true>(a); }
template <int RB, int TB, int VB, int NH>
__global__ PQ_WINDOW_ATTR(4) void pq_window_grouped_kernel(const DecodeArgs a) { attention_body<RB + TB, VB, NH, true, false, 4, RB, true>(a); }

template <int W, int VB, int NH, bool Q32>
void launch_uniform(const DecodeArgs& a, dim3 grid, hipStream_t st) {
  if (a.wide_groups) hipLaunchKernelGGL((pq_window_attention_kernel<W, VB, NH, Q32, 8>), grid, dim3(512), 0, st, a);
  else hipLaunchKernelGGL((pq_window_attention_kernel<W, VB, NH, Q32, 4>), grid, dim3(256), 0, st, a);
}
template <int W>
bool launch_q(const DecodeArgs& a, dim3 grid, hipStream_t st) {
  if (a.n_heads <= 4) a.q_is_f32 ? launch_uniform<W, PQ_WINDOW_VB, 4, true>(a, grid, st) : launch_uniform<W, PQ_WINDOW_VB, 4, false>(a, grid, st);
  else a.q_is_f32 ? launch_uniform<W, PQ_WINDOW_VB, 8, true>(a, grid, st) : launch_uniform<W, PQ_WINDOW_VB, 8, false>(a, grid, st);
  return true;
}
template <int RB, int TB>
bool launch_grouped(const DecodeArgs& a, dim3 grid, hipStream_t st) {
  if (a.n_heads <= 4) hipLaunchKernelGGL((pq_window_grouped_kernel<RB, TB, PQ_WINDOW_VB, 4>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((pq_window_grouped_kernel<RB, TB, PQ_WINDOW_VB, 8>), grid, dim3(256), 0, st, a);
  return true;
}

}  // namespace window
}  // namespace

bool PQ_WINDOW_LAUNCH(const pq_layout* l, const DecodeArgs& a, dim3 grid, hipStream_t st) {
  switch (l->r_bits * 10 + l->t_bits + (l->angle_quantizer == PQ_ANGLE_GROUPED ? 100 : 0)) {
    case 44: case 53: case 35: return window::launch_q<8>(a, grid, st);
    case 33: case 42: case 24: return window::launch_q<6>(a, grid, st);
    case 144: return window::launch_grouped<4, 4>(a, grid, st);
    case 133: return window::launch_grouped<3, 3>(a, grid, st);
    case 153: return window::launch_grouped<5, 3>(a, grid, st);
    case 135: return window::launch_grouped<3, 5>(a, grid, st);
    case 142: return window::launch_grouped<4, 2>(a, grid, st);
    case 124: return window::launch_grouped<2, 4>(a, grid, st);
    default: return false;
  }
}

}  // namespace pq
