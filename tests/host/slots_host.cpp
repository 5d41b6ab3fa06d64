// Partials that launches leave in their workspaces, and the bounds their sizes go by (pq_plan.hpp), for a range of shapes: how many shapes have more than the bounds of their own
// or of the larger shape before them say.
#define __host__
#define __device__
#include "pq_plan.hpp"

extern "C" int slots_host(int n_kv_heads, int group, int angles, const int32_t* seqs, int n_seqs, const int32_t* lens, int n_lens) {
  const pq_layout l = {pq::kHeadDim, 4, 4, pq::kGroup, n_kv_heads, angles};
  const int heads = n_kv_heads * group;
  int wrong = 0;
  for (int i = 0; i < n_seqs; ++i)
    for (int j = 0; j < n_lens; ++j) {
      const int s = seqs[i], most = lens[j];
      const int64_t pages = (static_cast<int64_t>(most) + pq::kGroup - 1) / pq::kGroup, units = static_cast<int64_t>(s) * n_kv_heads;
      const size_t decode = pq::workspace_slots_up_to(&l, s, heads, most), window = pq::window_partials_up_to(units, pages);
      wrong += pq::workspace_slots(&l, s, heads, most) > decode;
      wrong += static_cast<size_t>(units) * pq::plan_window(&l, s, most).n_chunks > window;
      for (int v_bits : {16, 4, 2}) wrong += static_cast<size_t>(s) * heads * pq::plan_attention(&l, v_bits, s, heads, most).n_chunks > decode;
      if (i > 0) {
        wrong += pq::workspace_slots_up_to(&l, seqs[i - 1], heads, most) > decode;
        wrong += pq::window_partials_up_to(static_cast<int64_t>(seqs[i - 1]) * n_kv_heads, pages) > window;
      }
      if (j > 0) {
        wrong += pq::workspace_slots_up_to(&l, s, heads, lens[j - 1]) > decode;
        wrong += pq::window_partials_up_to(units, (static_cast<int64_t>(lens[j - 1]) + pq::kGroup - 1) / pq::kGroup) > window;
      }
    }
  return wrong;
}
