// Gradients of the group norm with an activation: dg_norm.cuh has the formulas.
//
// As forward: pieces of rows leave the sums of d and of d hat of their channels, a small kernel makes A and B of every
// group and the gradients of weight and bias of them, and the last launch goes through the pieces backwards.
#include "dg_norm.cuh"

namespace dg {
namespace {

// Rows in flight per thread, of each matrix, and blocks of an SM that walk through pieces: 233 k x 256, fp32, ReLU, from a cold L2:
// 199 us; with three blocks 215, with two rows and three blocks 205, with four 211.
constexpr int kRows = 4, kPieceBlocks = 2;
// Rows of a thread in shared memory: six blocks of short graphs on an SM.
constexpr int kStep = 2, kRing = 4, kSlots = kStep * kRing;

// A thread's sums of d and of d hat over rows.
template <int ACT, int VEC>
struct Sums {
  Two d[kPairs<VEC>], dh[kPairs<VEC>];
  __device__ __forceinline__ void add(const Channels<VEC>& x, const Channels<VEC>& dy, const Fixed<VEC>& f) {
#pragma unroll
    for (int k = 0; k < kPairs<VEC>; ++k) {
      Two hat, q;
      backward_terms<ACT, VEC>(pair_of(x, k), pair_of(dy, k), f, k, &hat, &q);
      d[k] = d[k] + q;
      dh[k] = fma2(q, hat, dh[k]);
    }
  }
  __device__ __forceinline__ void add(const Sums& o) {
#pragma unroll
    for (int k = 0; k < kPairs<VEC>; ++k) d[k] = d[k] + o.d[k], dh[k] = dh[k] + o.dh[k];
  }
  __device__ __forceinline__ void put(float2 (&total)[VEC]) const {
    Channels<VEC> s, t;
#pragma unroll
    for (int k = 0; k < kPairs<VEC>; ++k) set_pair(s, k, d[k]), set_pair(t, k, dh[k]);
#pragma unroll
    for (int c = 0; c < VEC; ++c) total[c] = make_float2(s.v[c], t.v[c]);
  }
};

// means(c): (A, B) of the vector's channel c
template <int VEC, typename Means>
__device__ __forceinline__ void means_of(Two (&A)[kPairs<VEC>], Two (&B)[kPairs<VEC>], Means means) {
  Channels<VEC> p, q;
#pragma unroll
  for (int c = 0; c < VEC; ++c) {
    const float2 m = means(c);
    p.v[c] = m.x, q.v[c] = m.y;
  }
#pragma unroll
  for (int k = 0; k < kPairs<VEC>; ++k) A[k] = pair_of(p, k), B[k] = pair_of(q, k);
}

// dx = rstd (d w - A - hat B) of a vector
template <int ACT, int VEC>
__device__ __forceinline__ Channels<VEC> gradient_of(const Channels<VEC>& x, const Channels<VEC>& dy, const Fixed<VEC>& f,
                                                     const Two (&A)[kPairs<VEC>], const Two (&B)[kPairs<VEC>]) {
  Channels<VEC> r;
#pragma unroll
  for (int k = 0; k < kPairs<VEC>; ++k) {
    Two hat, q;
    backward_terms<ACT, VEC>(pair_of(x, k), pair_of(dy, k), f, k, &hat, &q);
    set_pair(r, k, (fma2(q, f.w[k], both(-1.f) * A[k]) - hat * B[k]) * f.rstd[k]);
  }
  return r;
}

// partial[piece][channel] = (sum of d, sum of d hat).  The sums of every kRows rows are added to the thread's in 32 bits, those
// of kStretch times as many to its place in shared memory in 64: what is lost does not grow with the rows.
template <typename X, typename Y, int ACT, int VEC>
__global__ void __launch_bounds__(kNormThreads, kPieceBlocks)
    norm_sums_kernel(NormArgs a, NormShape sh, const Piece* pieces, float2* partial) {
  constexpr int kStretch = 16;
  __shared__ double2 parts[kNormThreads * VEC];
  const Place at = place_of(a, sh, pieces, blockIdx.x);
#pragma unroll
  for (int c = 0; c < VEC; ++c) parts[c * kNormThreads + threadIdx.x] = make_double2(0.0, 0.0);
  if (at.channel < a.F && at.y < at.piece.rows) {
    const Fixed<VEC> f = fixed_of<VEC>(a, at.piece.graph, at.channel);
    int32_t rows = (at.piece.rows - at.y + at.down - 1) / at.down;
    const int64_t pace = (int64_t)at.down * a.F, base = ((int64_t)at.piece.row + at.y) * a.F + at.channel;
    const X* x = static_cast<const X*>(a.X) + base;
    const Y* dy = static_cast<const Y*>(a.dY) + base;
    Sums<ACT, VEC> all = {};
    auto close = [&]() {
      float2 total[VEC];
      all.put(total);
#pragma unroll
      for (int c = 0; c < VEC; ++c) {
        double2* const so_far = parts + c * kNormThreads + threadIdx.x;
        *so_far = make_double2(so_far->x + total[c].x, so_far->y + total[c].y);
      }
      all = Sums<ACT, VEC>{};
    };
    auto step = [&](auto once) {
      constexpr bool kOnce = decltype(once)::value;
      Channels<VEC> v[kRows], d[kRows];
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        v[u] = load_channels<X, VEC, kOnce>(x + u * pace);
        d[u] = load_channels<Y, VEC, kOnce>(dy + u * pace);
      }
      Sums<ACT, VEC> some = {};
#pragma unroll
      for (int u = 0; u < kRows; ++u) some.add(v[u], d[u], f);
      all.add(some);
      rows -= kRows, x += kRows * pace, dy += kRows * pace;
    };
    while (rows >= kRows + sh.kept) {
#pragma unroll 1
      for (int q = 0; q < kStretch && rows >= kRows + sh.kept; ++q) step(std::true_type());
      close();
    }
    while (rows >= kRows) {
#pragma unroll 1
      for (int q = 0; q < kStretch && rows >= kRows; ++q) step(std::false_type());
      close();
    }
    for (; rows > 0; --rows, x += pace, dy += pace) all.add(load_channels<X, VEC, false>(x), load_channels<Y, VEC, false>(dy), f);
    close();
  }
  int half = 1;
  while (half < sh.down) half *= 2;
  for (half /= 2; half > 0; half /= 2) {
    __syncthreads();
    const int other = threadIdx.x + half * sh.across;
    if (at.y < half && at.y + half < sh.down) {
#pragma unroll
      for (int c = 0; c < VEC; ++c) {
        double2* const mine = parts + c * kNormThreads + threadIdx.x;
        const double2 o = parts[c * kNormThreads + other];
        *mine = make_double2(mine->x + o.x, mine->y + o.y);
      }
    }
  }
  if (at.y == 0 && at.channel < a.F) {
    float2* out = partial + (int64_t)blockIdx.x * a.F + at.channel;
#pragma unroll
    for (int c = 0; c < VEC; ++c) {
      const double2 total = parts[c * kNormThreads + threadIdx.x];
      out[c] = make_float2((float)total.x, (float)total.y);
    }
  }
}

constexpr int kJoinThreads = 512, kTile = 4;

// totals[graph][channel] = the sums of a graph's pieces, in 64 bits: blocks of 4 channels x 128 threads along the pieces where
// there is one graph (their totals are the gradients of bias and weight too).
__device__ __forceinline__ void join_channels(int32_t F, const float2* partial, int64_t lo, int64_t hi, float2* total, float* dweight,
                                              float* dbias, int32_t tile) {
  __shared__ double2 sums[kJoinThreads];
  const int32_t c = tile * kTile + threadIdx.x % kTile;
  double s1 = 0.0, s2 = 0.0;
  if (c < F) {
#pragma unroll 8
    for (int64_t p = lo + threadIdx.x / kTile; p < hi; p += kJoinThreads / kTile) {
      const float2 v = partial[p * F + c];
      s1 += v.x;
      s2 += v.y;
    }
  }
  sums[threadIdx.x] = make_double2(s1, s2);
  for (int half = kJoinThreads / 2; half >= kTile; half /= 2) {
    __syncthreads();
    if (threadIdx.x < half) {
      sums[threadIdx.x].x += sums[threadIdx.x + half].x;
      sums[threadIdx.x].y += sums[threadIdx.x + half].y;
    }
  }
  if (threadIdx.x >= kTile || c >= F) return;
  const float2 r = make_float2((float)sums[threadIdx.x].x, (float)sums[threadIdx.x].y);
  if (total) total[c] = r;
  if (dbias) dbias[c] = r.x;
  if (dweight) dweight[c] = r.y;
}
__global__ void __launch_bounds__(kJoinThreads)
    norm_join_sums_kernel(int32_t F, const float2* partial, int64_t rows, float2* total, float* dweight, float* dbias) {
  cudaGridDependencySynchronize();
  join_channels(F, partial, 0, rows, total, dweight, dbias, blockIdx.x);
}
// Many graphs: a warp for a graph and 8 channels, 4 threads along the pieces.
__global__ void __launch_bounds__(kNormThreads)
    norm_join_graphs_kernel(int32_t F, int64_t graphs, const int32_t* first, const float2* partial, float2* totals) {
  cudaGridDependencySynchronize();
  const int32_t tiles = (F + 7) / 8, lane = threadIdx.x & 31;
  const int64_t item = (int64_t)blockIdx.x * (kNormThreads / 32) + threadIdx.x / 32, graph = item / tiles;
  if (graph >= graphs) return;
  const int32_t c = (int32_t)(item - graph * tiles) * 8 + lane % 8, hi = first[graph + 1];
  double s1 = 0.0, s2 = 0.0;
  if (c < F) {
#pragma unroll 4
    for (int32_t p = first[graph] + lane / 8; p < hi; p += 4) {
      const float2 v = partial[(int64_t)p * F + c];
      s1 += v.x;
      s2 += v.y;
    }
  }
#pragma unroll
  for (int o = 16; o >= 8; o /= 2) {
    s1 += __shfl_xor_sync(0xffffffffu, s1, o);
    s2 += __shfl_xor_sync(0xffffffffu, s2, o);
  }
  if (lane < 8 && c < F) totals[graph * F + c] = make_float2((float)s1, (float)s2);
}

// Short graphs: sums, A and B and the results in one launch.  graph_sums[graph][channel] = (sum of d, sum of d hat), or, for
// one graph, the gradients themselves.
template <typename X, typename Y, int ACT, int VEC>
__global__ void __launch_bounds__(kGraphThreads, VEC == 8 ? 4 : 6)
    norm_graph_bwd_kernel(const __grid_constant__ NormArgs a, const __grid_constant__ GraphPlan plan, float2* graph_sums, float* dweight, float* dbias) {
  __shared__ float2 parts[kGraphThreads * VEC], group_sums[kTileGroups], group_means[kTileGroups];
  const bool is_long = blockIdx.x < plan.long_blocks;
  const GraphShape sh = is_long ? plan.shape[0] : plan.shape[1];
  const GraphPlace at = graph_place(a, plan, sh, is_long);
  const int32_t first_group = at.tile_first / a.width;
  const X* x = static_cast<const X*>(a.X) + at.base;
  const Y* dy = static_cast<const Y*>(a.dY) + at.base;
  X* dx = static_cast<X*>(a.out) + at.base;
  const bool mine = at.channel < a.F;
  Fixed<VEC> f;
  if (mine) {
    fix_weights<VEC>(f, a, at.channel);
    fix_stats<VEC>(f, [&](int c) {
      return a.stats[(int64_t)at.graph * a.groups + first_group + group_of(plan, at.channel - at.tile_first + c)];
    });
  }
  extern __shared__ uint4 slots[];
  RawChannels<X, VEC>* const v = reinterpret_cast<RawChannels<X, VEC>*>(slots) + threadIdx.x;
  RawChannels<Y, VEC>* const d = reinterpret_cast<RawChannels<Y, VEC>*>(reinterpret_cast<RawChannels<X, VEC>*>(slots) + kSlots * kGraphThreads) + threadIdx.x;
  const int64_t pace = (int64_t)at.step * a.F;
  // the thread's rows, and in groups of kStep
  const int32_t count = mine && at.row < at.rows ? (at.rows - at.row + at.step - 1) / at.step : 0;
  const int32_t steps = (count + kStep - 1) / kStep;
  auto fetch_rows = [&](int32_t q, int place) {
    int64_t from = q * kStep * pace;
#pragma unroll
    for (int u = 0; u < kStep; ++u, from += pace) {
      if (q * kStep + u >= count) break;
      fetch<X, VEC>(v + (place * kStep + u) * kGraphThreads, x + from);
      fetch<Y, VEC>(d + (place * kStep + u) * kGraphThreads, dy + from);
    }
  };
  Sums<ACT, VEC> all = {};
  ring_forward<kRing>(steps, fetch_rows, [&](int32_t q, int place) {
#pragma unroll
    for (int u = 0; u < kStep; ++u) {
      if (q * kStep + u >= count) break;
      const int at_slot = (place * kStep + u) * kGraphThreads;
      all.add(numbers_of(v[at_slot]), numbers_of(d[at_slot]), f);
    }
  });
  float2 total[VEC];
  all.put(total);
  // parts[y][channel of the tile]
  const int32_t stride = sh.across * VEC;
  if (at.y < sh.down) {
#pragma unroll
    for (int k = 0; k < VEC; ++k) parts[threadIdx.x * VEC + k] = total[k];
  }
  __syncthreads();
  // a channel's sum over the block's rows, in parts[0][channel]
  for (int32_t k = threadIdx.x; k < at.tile_channels; k += kGraphThreads) {
    float2 s = parts[k];
    for (int32_t yy = 1; yy < sh.down; ++yy) {
      s.x += parts[yy * stride + k].x;
      s.y += parts[yy * stride + k].y;
    }
    parts[k] = s;
  }
  __syncthreads();
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
  const int32_t groups = group_of(plan, at.tile_channels - 1) + 1, lanes = 1 << sh.lanes_log;
  // several groups a warp: `lanes` threads along the channels of each
  for (int32_t g0 = warp * (32 >> sh.lanes_log); g0 < groups; g0 += (kGraphThreads / 32) * (32 >> sh.lanes_log)) {
    const int32_t g = g0 + (lane >> sh.lanes_log);
    float s1 = 0.f, s2 = 0.f;
    if (g < groups) {
      for (int32_t k = lane & (lanes - 1); k < a.width; k += lanes) {
        const float2 p = parts[g * a.width + k];
        const float w = a.weight ? a.weight[at.tile_first + g * a.width + k] : 1.f;
        s1 = fmaf(w, p.x, s1);
        s2 = fmaf(w, p.y, s2);
      }
    }
    for (int o = lanes / 2; o > 0; o /= 2) {
      s1 += __shfl_xor_sync(0xffffffffu, s1, o);
      s2 += __shfl_xor_sync(0xffffffffu, s2, o);
    }
    if (g < groups && (lane & (lanes - 1)) == 0) group_sums[g] = make_float2(s1, s2);
  }
  const int32_t cluster = 1 << plan.cluster_log;
  if (cluster > 1) {
    cluster_arrive();
    cluster_wait();
  }
  __syncthreads();
  for (int32_t g = threadIdx.x; g < groups; g += kGraphThreads) {
    const float n = at.rows > 0 ? (float)at.rows * a.width : 1.f;
    float2 s = group_sums[g];
    if (cluster > 1) {
      s = make_float2(0.f, 0.f);
      for (int32_t r = 0; r < cluster; ++r) {
        const float2 o = of_rank(group_sums + g, r);
        s.x += o.x;
        s.y += o.y;
      }
    }
    group_means[g] = make_float2(s.x / n, s.y / n);
  }
  if (at.rank == 0 && (dweight || dbias)) {
    for (int32_t k = threadIdx.x; k < at.tile_channels; k += kGraphThreads) {
      float2 s = parts[k];
      for (int32_t r = 1; r < cluster; ++r) {
        const float2 o = of_rank(parts + k, r);
        s.x += o.x;
        s.y += o.y;
      }
      const int32_t channel = at.tile_first + k;
      if (graph_sums) {
        graph_sums[(int64_t)at.graph * a.F + channel] = s;
      } else {
        if (dbias) dbias[channel] = s.x;
        if (dweight) dweight[channel] = s.y;
      }
    }
  }
  if (cluster > 1) cluster_arrive();  // the others' shared memory has been read
  __syncthreads();
  if (mine && a.out) {
    Two A[kPairs<VEC>], B[kPairs<VEC>];
    means_of<VEC>(A, B, [&](int c) { return group_means[group_of(plan, at.channel - at.tile_first + c)]; });
    ring_back<kRing>(steps, fetch_rows, [&](int32_t q, int place) {
      X* to = dx + q * kStep * pace;
#pragma unroll
      for (int u = 0; u < kStep; ++u, to += pace) {
        if (q * kStep + u >= count) break;
        const int at_slot = (place * kStep + u) * kGraphThreads;
        store_channels<X, VEC>(to, gradient_of<ACT, VEC>(numbers_of(v[at_slot]), numbers_of(d[at_slot]), f, A, B));
      }
    });
  }
  if (cluster > 1) cluster_wait();
}

// As forward, from the last rows back.  A and B of the tile's groups come from the channels' totals, summed anew by every
// block: a few hundred numbers from the L2, where a launch between would cost more.
template <typename X, typename Y, int ACT, int VEC>
__global__ void __launch_bounds__(kNormThreads, kPieceBlocks)
    norm_apply_bwd_kernel(NormArgs a, NormShape sh, const Piece* pieces, const float2* totals) {
  __shared__ float2 means[kNormThreads * VEC];  // of the groups that the tile touches: no more than its channels
  cudaGridDependencySynchronize();
  const Place at = place_of(a, sh, pieces, blockIdx.x);
  const int32_t tile_first = blockIdx.y * sh.across * VEC, tile_end = min(tile_first + sh.across * VEC, a.F);
  const int32_t first_group = tile_first / a.width, groups = (tile_end - 1) / a.width - first_group + 1;
  const Rows graph_rows = rows_of(a, at.piece.graph);
  const double n = (double)(graph_rows.hi - graph_rows.lo) * a.width;
  const float2* mine = totals + (int64_t)at.piece.graph * a.F;
  int32_t lanes = 1;
  while (lanes < a.width && lanes < 32) lanes *= 2;
  for (int32_t g0 = 0; g0 < groups; g0 += kNormThreads / lanes) {
    const int32_t g = g0 + threadIdx.x / lanes;
    double s1 = 0.0, s2 = 0.0;
    if (g < groups) {
      for (int32_t k = threadIdx.x % lanes; k < a.width; k += lanes) {
        const int32_t channel = (first_group + g) * a.width + k;
        const float2 t = mine[channel];
        const double w = a.weight ? a.weight[channel] : 1.f;
        s1 += w * t.x;
        s2 += w * t.y;
      }
    }
    for (int o = lanes / 2; o > 0; o /= 2) {
      s1 += __shfl_xor_sync(0xffffffffu, s1, o);
      s2 += __shfl_xor_sync(0xffffffffu, s2, o);
    }
    if (g < groups && threadIdx.x % lanes == 0) means[g] = make_float2((float)(s1 / n), (float)(s2 / n));
  }
  __syncthreads();
  if (at.channel >= a.F || at.y >= at.piece.rows) return;
  const Fixed<VEC> f = fixed_of<VEC>(a, at.piece.graph, at.channel);
  Two A[kPairs<VEC>], B[kPairs<VEC>];
  means_of<VEC>(A, B, [&](int c) { return means[(at.channel + c) / a.width - first_group]; });
  int32_t rows = (at.piece.rows - at.y + at.down - 1) / at.down;
  const int64_t pace = (int64_t)at.down * a.F;
  const int64_t base = ((int64_t)at.piece.row + at.y) * a.F + at.channel + (rows - 1) * pace;
  const X* x = static_cast<const X*>(a.X) + base;
  const Y* dy = static_cast<const Y*>(a.dY) + base;
  X* dx = static_cast<X*>(a.out) + base;
  for (; rows >= kRows; rows -= kRows, x -= kRows * pace, dy -= kRows * pace, dx -= kRows * pace) {
    Channels<VEC> v[kRows], d[kRows];
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      v[u] = load_channels<X, VEC, true>(x - u * pace);
      d[u] = load_channels<Y, VEC, true>(dy - u * pace);
    }
#pragma unroll
    for (int u = 0; u < kRows; ++u) store_channels<X, VEC>(dx - u * pace, gradient_of<ACT, VEC>(v[u], d[u], f, A, B));
  }
  for (; rows > 0; --rows, x -= pace, dy -= pace, dx -= pace)
    store_channels<X, VEC>(dx, gradient_of<ACT, VEC>(load_channels<X, VEC, true>(x), load_channels<Y, VEC, true>(dy), f, A, B));
}

template <typename X, typename Y, int ACT>
__global__ void __launch_bounds__(kNormThreads) norm_bwd_direct_kernel(NormArgs a, int across) {
  const X* x = static_cast<const X*>(a.X);
  const Y* dy = static_cast<const Y*>(a.dY);
  X* dx = static_cast<X*>(a.out);
  const int64_t graph = blockIdx.x / a.groups;
  const int32_t channel = (int32_t)(blockIdx.x % a.groups) * a.width;
  const Rows r = rows_of(a, graph);
  if (r.hi <= r.lo) return;
  const double cells = (double)(r.hi - r.lo) * a.width;
  const float2 st = a.stats[blockIdx.x];
  double s1 = 0.0, s2 = 0.0;
  auto terms = [&](int64_t i, int32_t c, float* hat) {
    const float v = as_float(x[i]), w = a.weight ? a.weight[c] : 1.f;
    *hat = (v - st.x) * st.y;
    return before_activation<ACT>(as_float(dy[i]), v, st.x, st.y, w, a.bias ? a.bias[c] : 0.f) * w;
  };
  for_cells(a, r, channel, across, [&](int64_t i, int32_t c) {
    float hat;
    const double q = terms(i, c, &hat);
    s1 += q;
    s2 += q * hat;
  });
  const float A = (float)(block_sum(s1) / cells), B = (float)(block_sum(s2) / cells);
  for_cells(a, r, channel, across, [&](int64_t i, int32_t c) {
    float hat;
    const float q = terms(i, c, &hat);
    dx[i] = as<X>((q - A - hat * B) * st.y);
  });
}

// dw and db: 32 channels x 32 threads along the rows.
template <typename X, typename Y, int ACT>
__global__ void __launch_bounds__(1024) norm_weights_direct_kernel(NormArgs a, float* dweight, float* dbias) {
  __shared__ double sums[2][32][33];
  const X* x = static_cast<const X*>(a.X);
  const Y* dy = static_cast<const Y*>(a.dY);
  const int32_t c = blockIdx.x * 32 + threadIdx.x;
  double s1 = 0.0, s2 = 0.0;
  if (c < a.F) {
    const float w = a.weight ? a.weight[c] : 1.f, b = a.bias ? a.bias[c] : 0.f;
    for (int64_t graph = 0; graph < a.graphs; ++graph) {
      const Rows r = rows_of(a, graph);
      const float2 st = a.stats[graph * a.groups + c / a.width];
      for (int64_t row = r.lo + threadIdx.y; row < r.hi; row += 32) {
        const float v = as_float(x[row * a.F + c]);
        const double d = before_activation<ACT>(as_float(dy[row * a.F + c]), v, st.x, st.y, w, b);
        s1 += d;
        s2 += d * ((v - st.x) * st.y);
      }
    }
  }
  sums[0][threadIdx.y][threadIdx.x] = s1;
  sums[1][threadIdx.y][threadIdx.x] = s2;
  __syncthreads();
  s1 = sums[0][threadIdx.x][threadIdx.y];
  s2 = sums[1][threadIdx.x][threadIdx.y];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    s1 += __shfl_xor_sync(0xffffffffu, s1, o);
    s2 += __shfl_xor_sync(0xffffffffu, s2, o);
  }
  const int32_t channel = blockIdx.x * 32 + threadIdx.y;
  if (threadIdx.x == 0 && channel < a.F) {
    if (dbias) dbias[channel] = (float)s1;
    if (dweight) dweight[channel] = (float)s2;
  }
}

template <typename X, typename Y, int ACT>
dg_status_t backward(const Graph* g, const NormArgs& a, dg_type_t x, dg_type_t y, float* dweight, float* dbias, cudaStream_t s) {
  constexpr bool kWide = sizeof(X) == 2 && sizeof(Y) == 2;
  const bool weights = dweight || dbias;
  if (!weights && !a.out) return DG_OK;
  const int vec = norm_vector(a, x, y);
  const unsigned channel_blocks = (unsigned)((a.F + kTile - 1) / kTile);
  void* memory = nullptr;
  const GraphPlan plan = graph_plan(g, a, vec, sizeof(X), kSlots, false);
  const size_t graph_bytes = a.graphs > 1 ? (size_t)a.graphs * a.F * sizeof(float2) : 0;
  if (plan.blocks > 0 && (!weights || !graph_bytes || scratch_alloc(g, graph_bytes, s, &memory) == cudaSuccess)) {
    float2* sums = static_cast<float2*>(memory);
    cudaError_t e = by_vector<kWide>(vec, [&](auto v) {
      constexpr int VEC = decltype(v)::value;
      constexpr size_t kBytes = (size_t)kSlots * kGraphThreads * VEC * (sizeof(X) + sizeof(Y));
      static_assert(kBytes <= kMostPlaces, "ask for more shared memory");
      return launch_graphs(plan, norm_graph_bwd_kernel<X, Y, ACT, VEC>, kBytes, s, a, sums, dweight, dbias);
    });
    if (e == cudaSuccess && sums)
      e = launch_kernel(norm_join_sums_kernel, dim3(channel_blocks), kJoinThreads, s, true, a.F, (const float2*)sums, a.graphs,
                        (float2*)nullptr, dweight, dbias);
    pool_free(memory, s);
    DG_CUDA(e);
    count_launches(1 + (sums != nullptr));
    return DG_OK;
  }
  const NormShape sh = norm_shape(g, a, vec, sizeof(X) + sizeof(Y), kPieceBlocks);
  const size_t partial_bytes = (size_t)sh.pieces * a.F * sizeof(float2), total_bytes = (size_t)a.graphs * a.F * sizeof(float2);
  if (plan.blocks > 0 || scratch_alloc(g, partial_bytes + total_bytes, s, &memory) != cudaSuccess) {
    int across = 1;
    while (across < a.width && across < kNormThreads) across *= 2;
    if (weights)
      norm_weights_direct_kernel<X, Y, ACT><<<(unsigned)((a.F + 31) / 32), dim3(32, 32), 0, s>>>(a, dweight, dbias);
    if (a.out) norm_bwd_direct_kernel<X, Y, ACT><<<(unsigned)(a.graphs * a.groups), kNormThreads, 0, s>>>(a, across);
    DG_CUDA(cudaGetLastError());
    count_launches(weights + (a.out != nullptr));
    return DG_OK;
  }
  float2* partial = static_cast<float2*>(memory);
  float2* totals = reinterpret_cast<float2*>(static_cast<char*>(memory) + partial_bytes);
  const dim3 grid((unsigned)sh.pieces, (unsigned)sh.tiles);
  const Piece* pieces = g->batch_pieces;
  const int64_t items = a.graphs * ((a.F + 7) / 8);  // of the join of many graphs: a warp each
  if (sh.pieces > 0)
    by_vector<kWide>(vec, [&](auto v) {
      norm_sums_kernel<X, Y, ACT, decltype(v)::value><<<grid, kNormThreads, 0, s>>>(a, sh, pieces, partial);
    });
  cudaError_t e = cudaGetLastError();
  if (e == cudaSuccess && pieces)
    e = launch_kernel(norm_join_graphs_kernel, dim3((unsigned)((items + 7) / 8)), kNormThreads, s, true, a.F, a.graphs,
                      g->batch_first, (const float2*)partial, totals);
  // the gradients of weight and bias, and the totals where one graph has all pieces
  if (e == cudaSuccess && (weights || !pieces))
    e = launch_kernel(norm_join_sums_kernel, dim3(channel_blocks), kJoinThreads, s, true, a.F,
                      (const float2*)(pieces ? totals : partial), pieces ? a.graphs : (int64_t)sh.pieces, pieces ? nullptr : totals,
                      dweight, dbias);
  if (e == cudaSuccess && a.out && sh.pieces > 0)
    e = by_vector<kWide>(vec, [&](auto v) {
      return launch_kernel(norm_apply_bwd_kernel<X, Y, ACT, decltype(v)::value>, grid, kNormThreads, s, true, a, sh, pieces,
                           (const float2*)totals);
    });
  pool_free(memory, s);
  DG_CUDA(e);
  count_launches((sh.pieces > 0) + (pieces != nullptr) + (weights || !pieces) + (a.out && sh.pieces > 0));
  return DG_OK;
}

}  // namespace

dg_status_t group_norm_bwd(const Graph* g, const NormArgs& a, dg_type_t x, dg_type_t y, dg_act_t act, float* dweight,
                           float* dbias, cudaStream_t s) {
  return by_type(x, y, act, [&](auto xs, auto ys, auto kind) {
    return backward<decltype(xs), decltype(ys), decltype(kind)::value>(g, a, x, y, dweight, dbias, s);
  });
}

}  // namespace dg
