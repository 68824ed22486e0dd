// Gradients of the group norm with an activation: dg_norm.cuh has the formulas.
//
// As forward: pieces of rows leave the sums of d and of d hat of their channels, a small kernel makes A and B of every
// group and the gradients of weight and bias of them, and the last launch goes through the pieces backwards.
#include "dg_norm.cuh"

namespace dg {
namespace {

constexpr int kRows = 4;   // in flight per thread, of each matrix
// Rows of a thread in shared memory: six blocks of short graphs on an SM.
constexpr int kStep = 2, kRing = 4, kSlots = kStep * kRing;

// partial[piece][channel] = (sum of d, sum of d hat).  The sums of every kRows rows are added to the thread's.
template <typename X, typename Y, int ACT, int VEC>
__global__ void __launch_bounds__(kNormThreads) norm_sums_kernel(NormArgs a, NormShape sh, const Piece* pieces, float2* partial) {
  __shared__ float2 parts[kNormThreads * VEC];
  const Place at = place_of(a, sh, pieces, blockIdx.x);
  float2 total[VEC] = {};
  if (at.channel < a.F) {
    const Fixed<VEC> f = fixed_of<VEC>(a, at.piece.graph, at.channel);
    const int64_t base = (int64_t)at.piece.row * a.F + at.channel;
    const X* x = static_cast<const X*>(a.X) + base;
    const Y* dy = static_cast<const Y*>(a.dY) + base;
    for (int32_t r0 = at.y; r0 < at.piece.rows; r0 += at.down * kRows) {
      Channels<VEC> v[kRows], d[kRows];
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        const int32_t r = r0 + u * at.down;
        if (r < at.piece.rows) {
          v[u] = load_channels<X, VEC>(x + (int64_t)r * a.F);
          d[u] = load_channels<Y, VEC>(dy + (int64_t)r * a.F);
        }
      }
#pragma unroll
      for (int c = 0; c < VEC; ++c) {
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
          if (r0 + u * at.down < at.piece.rows) {
            const float q = before_activation<ACT>(d[u].v[c], v[u].v[c], f.mean[c], f.rstd[c], f.w[c], f.b[c]);
            s1 += q;
            s2 = fmaf(q, (v[u].v[c] - f.mean[c]) * f.rstd[c], s2);
          }
        }
        total[c].x += s1;
        total[c].y += s2;
      }
    }
  }
#pragma unroll
  for (int c = 0; c < VEC; ++c) parts[c * kNormThreads + threadIdx.x] = total[c];
  int half = 1;
  while (half < sh.down) half *= 2;
  for (half /= 2; half > 0; half /= 2) {
    __syncthreads();
    const int other = threadIdx.x + half * sh.across;
    if (at.y < half && at.y + half < sh.down) {
#pragma unroll
      for (int c = 0; c < VEC; ++c) {
        const float2 o = parts[c * kNormThreads + other];
        total[c].x += o.x;
        total[c].y += o.y;
        parts[c * kNormThreads + threadIdx.x] = total[c];
      }
    }
  }
  if (at.y == 0 && at.channel < a.F) {
    float2* out = partial + (int64_t)blockIdx.x * a.F + at.channel;
#pragma unroll
    for (int c = 0; c < VEC; ++c) out[c] = total[c];
  }
}

constexpr int kJoinThreads = 512;

// (A, B) of a group from its pieces' sums, in 64 bits: `lanes` threads (a power of two) along its channels, the others along
// the pieces.
__device__ __forceinline__ void join_means(const NormArgs& a, const NormShape& sh, const int32_t* first, const float2* partial,
                                           float2* means, int32_t lanes, int64_t pair, int32_t thread, int32_t threads, bool warp) {
  const int64_t graph = pair / a.groups;
  const int32_t group = (int32_t)(pair % a.groups);
  const Rows r = rows_of(a, graph);
  const int32_t lo = first ? first[graph] : 0, hi = first ? first[graph + 1] : sh.pieces;
  const int32_t down = threads / lanes;
  double s1 = 0.0, s2 = 0.0;
  for (int32_t k = thread % lanes; k < a.width; k += lanes) {
    const int32_t channel = group * a.width + k;
    const double w = a.weight ? a.weight[channel] : 1.f;
    double t1 = 0.0, t2 = 0.0;
#pragma unroll 4
    for (int32_t p = lo + thread / lanes; p < hi; p += down) {
      const float2 v = partial[(int64_t)p * a.F + channel];
      t1 += v.x;
      t2 += v.y;
    }
    s1 += w * t1;
    s2 += w * t2;
  }
  s1 = warp ? warp_sum(s1) : block_sum(s1);
  s2 = warp ? warp_sum(s2) : block_sum(s2);
  const double n = r.hi > r.lo ? (double)(r.hi - r.lo) * a.width : 1.0;
  if (thread == 0) means[pair] = make_float2((float)(s1 / n), (float)(s2 / n));
}

// The gradients of weight and bias of 8 channels: 64 threads along the `rows` rows of sums.  In 64 bits.
__device__ __forceinline__ void join_weights(int32_t F, const float2* partial, int64_t rows, float* dweight, float* dbias, int32_t tile) {
  __shared__ double2 sums[kJoinThreads];
  const int32_t c = tile * 8 + threadIdx.x % 8;
  double s1 = 0.0, s2 = 0.0;
  if (c < F) {
#pragma unroll 8
    for (int64_t p = threadIdx.x / 8; p < rows; p += kJoinThreads / 8) {
      const float2 v = partial[p * F + c];
      s1 += v.x;
      s2 += v.y;
    }
  }
  sums[threadIdx.x] = make_double2(s1, s2);
  for (int half = kJoinThreads / 2; half >= 8; half /= 2) {
    __syncthreads();
    if (threadIdx.x < half) {
      sums[threadIdx.x].x += sums[threadIdx.x + half].x;
      sums[threadIdx.x].y += sums[threadIdx.x + half].y;
    }
  }
  if (threadIdx.x >= 8 || c >= F) return;
  if (dbias) dbias[c] = (float)sums[threadIdx.x].x;
  if (dweight) dweight[c] = (float)sums[threadIdx.x].y;
}

// One graph: a block for a group, then the blocks of the weights.
__global__ void __launch_bounds__(kJoinThreads)
    norm_join_sums_kernel(NormArgs a, NormShape sh, const float2* partial, float2* means, float* dweight, float* dbias, int32_t lanes) {
  cudaGridDependencySynchronize();
  const int32_t pairs = means ? a.groups : 0;
  if (blockIdx.x < pairs)
    join_means(a, sh, nullptr, partial, means, lanes, blockIdx.x, threadIdx.x, kJoinThreads, false);
  else
    join_weights(a.F, partial, sh.pieces, dweight, dbias, blockIdx.x - pairs);
}
// Many graphs: a warp for a group.
__global__ void __launch_bounds__(kNormThreads)
    norm_join_means_kernel(NormArgs a, NormShape sh, const int32_t* first, const float2* partial, float2* means, int32_t lanes) {
  cudaGridDependencySynchronize();
  const int64_t pair = (int64_t)blockIdx.x * (kNormThreads / 32) + threadIdx.x / 32;
  if (pair < a.graphs * a.groups) join_means(a, sh, first, partial, means, lanes, pair, threadIdx.x % 32, 32, true);
}
__global__ void __launch_bounds__(kJoinThreads)
    norm_weight_sums_kernel(int32_t F, const float2* partial, int64_t rows, float* dweight, float* dbias) {
  cudaGridDependencySynchronize();
  join_weights(F, partial, rows, dweight, dbias, blockIdx.x);
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
  int32_t group[VEC];
  Fixed<VEC> f = {};
  if (mine) {
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
      group[k] = group_of(plan, at.channel - at.tile_first + k);
      const float2 st = a.stats[(int64_t)at.graph * a.groups + first_group + group[k]];
      f.mean[k] = st.x, f.rstd[k] = st.y;
      f.w[k] = a.weight ? a.weight[at.channel + k] : 1.f;
      f.b[k] = a.bias ? a.bias[at.channel + k] : 0.f;
    }
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
  float2 total[VEC] = {};
  ring_forward<kRing>(steps, fetch_rows, [&](int32_t q, int place) {
#pragma unroll
    for (int u = 0; u < kStep; ++u) {
      if (q * kStep + u >= count) break;
      const int at_slot = (place * kStep + u) * kGraphThreads;
      const Channels<VEC> vx = numbers_of(v[at_slot]), vd = numbers_of(d[at_slot]);
#pragma unroll
      for (int k = 0; k < VEC; ++k) {
        const float q = before_activation<ACT>(vd.v[k], vx.v[k], f.mean[k], f.rstd[k], f.w[k], f.b[k]);
        total[k].x += q;
        total[k].y = fmaf(q, (vx.v[k] - f.mean[k]) * f.rstd[k], total[k].y);
      }
    }
  });
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
    float A[VEC], B[VEC];
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
      const float2 m = group_means[group[k]];
      A[k] = m.x, B[k] = m.y;
    }
    ring_back<kRing>(steps, fetch_rows, [&](int32_t q, int place) {
      X* to = dx + q * kStep * pace;
#pragma unroll
      for (int u = 0; u < kStep; ++u, to += pace) {
        if (q * kStep + u >= count) break;
        const int at_slot = (place * kStep + u) * kGraphThreads;
        const Channels<VEC> vx = numbers_of(v[at_slot]), vd = numbers_of(d[at_slot]);
        Channels<VEC> r;
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
          const float q = before_activation<ACT>(vd.v[k], vx.v[k], f.mean[k], f.rstd[k], f.w[k], f.b[k]) * f.w[k];
          const float hat = (vx.v[k] - f.mean[k]) * f.rstd[k];
          r.v[k] = (q - A[k] - hat * B[k]) * f.rstd[k];
        }
        store_channels<X, VEC>(to, r);
      }
    });
  }
  if (cluster > 1) cluster_wait();
}

template <typename X, typename Y, int ACT, int VEC>
__global__ void __launch_bounds__(kNormThreads) norm_apply_bwd_kernel(NormArgs a, NormShape sh, const Piece* pieces, const float2* means) {
  cudaGridDependencySynchronize();
  const Place at = place_of(a, sh, pieces, gridDim.x - 1 - blockIdx.x);
  if (at.channel >= a.F) return;
  const Fixed<VEC> f = fixed_of<VEC>(a, at.piece.graph, at.channel);
  float A[VEC], B[VEC];
#pragma unroll
  for (int c = 0; c < VEC; ++c) {
    const float2 m = means[(int64_t)at.piece.graph * a.groups + (at.channel + c) / a.width];
    A[c] = m.x, B[c] = m.y;
  }
  const int64_t base = (int64_t)at.piece.row * a.F + at.channel;
  const X* x = static_cast<const X*>(a.X) + base;
  const Y* dy = static_cast<const Y*>(a.dY) + base;
  X* dx = static_cast<X*>(a.out) + base;
  for (int32_t r0 = at.y; r0 < at.piece.rows; r0 += at.down * kRows) {
    Channels<VEC> v[kRows], d[kRows];
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      const int32_t r = r0 + u * at.down;
      if (r < at.piece.rows) {
        v[u] = load_channels<X, VEC>(x + (int64_t)r * a.F);
        d[u] = load_channels<Y, VEC>(dy + (int64_t)r * a.F);
      }
    }
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      if (r0 + u * at.down >= at.piece.rows) break;
#pragma unroll
      for (int c = 0; c < VEC; ++c) {
        const float q = before_activation<ACT>(d[u].v[c], v[u].v[c], f.mean[c], f.rstd[c], f.w[c], f.b[c]) * f.w[c];
        const float hat = (v[u].v[c] - f.mean[c]) * f.rstd[c];
        v[u].v[c] = (q - A[c] - hat * B[c]) * f.rstd[c];
      }
      store_channels<X, VEC>(dx + (int64_t)(r0 + u * at.down) * a.F, v[u]);
    }
  }
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
  const unsigned weight_blocks = (unsigned)((a.F + 7) / 8);
  void* memory = nullptr;
  const GraphPlan plan = graph_plan(g, a, vec, sizeof(X), kSlots, false);
  const size_t graph_bytes = weights && a.graphs > 1 ? (size_t)a.graphs * a.F * sizeof(float2) : 0;
  if (plan.blocks > 0 && (!graph_bytes || scratch_alloc(g, graph_bytes, s, &memory) == cudaSuccess)) {
    float2* sums = static_cast<float2*>(memory);
    cudaError_t e = by_vector<kWide>(vec, [&](auto v) {
      constexpr int VEC = decltype(v)::value;
      constexpr size_t kBytes = (size_t)kSlots * kGraphThreads * VEC * (sizeof(X) + sizeof(Y));
      return launch_graphs(plan, norm_graph_bwd_kernel<X, Y, ACT, VEC>, kBytes, s, a, sums, dweight, dbias);
    });
    if (e == cudaSuccess && sums)
      e = launch_kernel(norm_weight_sums_kernel, dim3(weight_blocks), kJoinThreads, s, true, a.F, (const float2*)sums, a.graphs,
                        dweight, dbias);
    pool_free(memory, s);
    DG_CUDA(e);
    count_launches(1 + (sums != nullptr));
    return DG_OK;
  }
  const NormShape sh = norm_shape(g, a, vec);
  const size_t partial_bytes = (size_t)sh.pieces * a.F * sizeof(float2);
  const int64_t pairs = a.out ? a.graphs * a.groups : 0;
  if (plan.blocks > 0 || scratch_alloc(g, partial_bytes + (size_t)pairs * sizeof(float2), s, &memory) != cudaSuccess) {
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
  float2* means = reinterpret_cast<float2*>(static_cast<char*>(memory) + partial_bytes);
  const dim3 grid((unsigned)sh.pieces, (unsigned)sh.tiles);
  const Piece* pieces = g->batch_pieces;
  if (sh.pieces > 0)
    by_vector<kWide>(vec, [&](auto v) {
      norm_sums_kernel<X, Y, ACT, decltype(v)::value><<<grid, kNormThreads, 0, s>>>(a, sh, pieces, partial);
    });
  cudaError_t e = cudaGetLastError();
  int32_t lanes = 1;
  while (lanes < a.width && lanes < 32) lanes *= 2;
  const bool together = !pieces;  // one graph: the weights' blocks ride along
  if (e == cudaSuccess && together)
    e = launch_kernel(norm_join_sums_kernel, dim3((unsigned)pairs + (weights ? weight_blocks : 0)), kJoinThreads, s, true, a, sh,
                      (const float2*)partial, a.out ? means : (float2*)nullptr, dweight, dbias, lanes);
  if (e == cudaSuccess && !together && a.out)
    e = launch_kernel(norm_join_means_kernel, dim3((unsigned)((pairs + 7) / 8)), kNormThreads, s, true, a, sh, g->batch_first,
                      (const float2*)partial, means, lanes);
  if (e == cudaSuccess && a.out && sh.pieces > 0)
    e = by_vector<kWide>(vec, [&](auto v) {
      return launch_kernel(norm_apply_bwd_kernel<X, Y, ACT, decltype(v)::value>, grid, kNormThreads, s, true, a, sh, pieces,
                           (const float2*)means);
    });
  if (e == cudaSuccess && !together && weights)
    e = launch_kernel(norm_weight_sums_kernel, dim3(weight_blocks), kJoinThreads, s, true, a.F, (const float2*)partial,
                      (int64_t)sh.pieces, dweight, dbias);
  pool_free(memory, s);
  DG_CUDA(e);
  count_launches((sh.pieces > 0) + (together ? 1 : weights + (a.out != nullptr)) + (a.out && sh.pieces > 0));
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
