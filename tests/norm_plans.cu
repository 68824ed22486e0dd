// How the group norm shares out a call among blocks (graph_plan), for a test to look at: linked with the library's own object
// files and the runtime without a GPU (fake_cudart.cpp).
#include "dg_norm.cuh"

extern "C" {
int norm_tile_groups() { return dg::kTileGroups; }
int norm_graph_threads() { return dg::kGraphThreads; }

// out: blocks (0: the call is not one for the kernels of short graphs), blocks of long graphs, log2 of a cluster's blocks, then of
// the two shapes: channels of a vector, threads across, threads down, tiles.
void norm_graph_plan(dg_graph_t g, int F, int groups, int x_type, int y_type, int backward, int rows_kept, long long* out) {
  dg::NormArgs a{};
  a.F = F, a.groups = groups, a.width = F / groups;
  a.rows = g->batch_rows < 0 ? g->n : g->batch_rows;
  a.graphs = g->batch_count;
  const int vec = dg::norm_vector(a, (dg_type_t)x_type, (dg_type_t)y_type);
  const bool shared = !backward && vec > 1 && a.width % vec == 0;
  const dg::GraphPlan p = dg::graph_plan(g, a, vec, x_type == DG_F32 ? 4 : 2, rows_kept, shared);
  *out++ = p.blocks, *out++ = p.long_blocks, *out++ = p.cluster_log;
  for (const dg::GraphShape& s : p.shape) *out++ = s.vec, *out++ = s.across, *out++ = s.down, *out++ = s.tiles;
}
}
