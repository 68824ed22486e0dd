// Group norm with an activation over the rows of an n x F matrix, channels last, forward: dg_norm.cuh has the formulas.
//
// Statistics need every row before the first result, so a matrix is read twice: pieces of rows leave the mean and the sum
// of squares about it of their channels, a small kernel joins them, and the last launch goes through the pieces backwards,
// those first that the L2 still holds.
#include "dg_norm.cuh"

namespace dg {
namespace {

// Rows a thread has in flight, and most rows of a stretch: sums in 32 bits go over no more.  (All of a thread's rows in one, with
// 1690 a thread and the first at 10^4 standard deviations: 1 / sqrt(var) 2e-4 off.)
constexpr int kStatRows = 8, kStretch = 64;
// Rows of a thread in shared memory: eight blocks on an SM.
constexpr int kStep = 4, kRing = 3, kSlots = kStep * kRing;

// Count, mean and sum of squares about the mean; joined they lose nothing to large means, as sums of x and x^2 would.
struct Moments {
  float mean, m2;
};
__device__ __forceinline__ void join(float& n, Moments& a, float nb, Moments b) {
  if (nb == 0.f) return;
  const float total = n + nb, share = nb / total, d = b.mean - a.mean;
  a.mean = fmaf(d, share, a.mean);
  a.m2 = a.m2 + b.m2 + d * d * (n * share);
  n = total;
}

// Adds `rows` of kStep rows (the rest are zeros) to a thread's moments: of a channel, or, with SHARED, of a vector of
// channels of one group.  n: cells so far.
template <int VEC, bool SHARED>
constexpr int kUnits = SHARED ? 1 : VEC;
template <int VEC, bool SHARED>
__device__ __forceinline__ void add_rows(const Channels<VEC>* v, int rows, float& n, Moments (&m)[kUnits<VEC, SHARED>]) {
  constexpr int kCells = SHARED ? VEC : 1;
  const bool full = rows >= kStep;
  const float cells = (float)(full ? kStep * kCells : rows * kCells), inverse = full ? 1.f / (kStep * kCells) : 1.f / cells;
  const float total = n + cells, share = __fdividef(cells, total);
#pragma unroll
  for (int k = 0; k < kUnits<VEC, SHARED>; ++k) {
    float sum = 0.f;
#pragma unroll
    for (int u = 0; u < kStep; ++u) {
      if constexpr (SHARED) {
#pragma unroll
        for (int c = 0; c < VEC; ++c) sum += v[u].v[c];
      } else {
        sum += v[u].v[k];
      }
    }
    const float mean = sum * inverse;
    float m2 = 0.f;
#pragma unroll
    for (int u = 0; u < kStep; ++u) {
      float part = 0.f;
      if constexpr (SHARED) {
#pragma unroll
        for (int c = 0; c < VEC; ++c) part = fmaf(v[u].v[c] - mean, v[u].v[c] - mean, part);
      } else {
        part = (v[u].v[k] - mean) * (v[u].v[k] - mean);
      }
      m2 += u < rows ? part : 0.f;
    }
    const float d = mean - m[k].mean;
    m[k].mean = fmaf(d, share, m[k].mean);
    m[k].m2 += fmaf(d * d, n * share, m2);
  }
  n = total;
}

// Joins the moments of a block's rows in pairs, always in the same order: those of all rows are in the first `across`
// threads, and in parts[unit * kNormThreads + thread] of them.
template <int UNITS>
__device__ __forceinline__ void join_block(float& n, Moments (&m)[UNITS], Moments* parts, float* counts, int32_t across, int32_t down) {
  counts[threadIdx.x] = n;
#pragma unroll
  for (int k = 0; k < UNITS; ++k) parts[k * kNormThreads + threadIdx.x] = m[k];
  const int32_t y = threadIdx.x / across;
  int half = 1;
  while (half < down) half *= 2;
  for (half /= 2; half > 0; half /= 2) {
    __syncthreads();
    const int other = threadIdx.x + half * across;
    if (y < half && y + half < down) {
      const float nb = counts[other];
      float total = n;
#pragma unroll
      for (int k = 0; k < UNITS; ++k) {
        total = n;
        join(total, m[k], nb, parts[k * kNormThreads + other]);
        parts[k * kNormThreads + threadIdx.x] = m[k];
      }
      n = total;
      counts[threadIdx.x] = n;
    }
  }
}

// partial[piece][unit]: the moments of a piece's rows.  A thread sums differences from a number near by, and their squares, over
// stretches of rows, and joins the stretches' moments in 64 bits.  What is lost when a stretch's own mean is taken off is of
// the order of its rows' distance from that number: the mean of the first rows, then that of the stretch before.  The first
// two stretches are short, so that rows far from all others in front (a hub's) do not count for many.
template <typename X, int VEC, bool SHARED>
__global__ void __launch_bounds__(kNormThreads, VEC == 8 ? 3 : 4)
    norm_stats_kernel(NormArgs a, NormShape sh, const Piece* pieces, float2* partial) {
  constexpr int kEach = kUnits<VEC, SHARED>, kP = kPairs<VEC>;
  __shared__ double2 stretches[kNormThreads * kEach];  // (mean, sum of squares about it) of the thread's stretches so far
  __shared__ float counts[kNormThreads];
  const Place at = place_of(a, sh, pieces, blockIdx.x);
  Moments m[kEach] = {};
  float n = 0.f;
  if (at.channel < a.F && at.y < at.piece.rows) {
    const X* x = static_cast<const X*>(a.X) + (int64_t)at.piece.row * a.F + at.channel;
    const int32_t rows = (at.piece.rows - at.y + at.down - 1) / at.down;
    const int64_t pace = (int64_t)at.down * a.F;
    Two from[kP], sum[kP] = {}, squares[kP] = {};
    x += at.y * a.F;
    auto add = [&](const Channels<VEC>& v) {
#pragma unroll
      for (int k = 0; k < kP; ++k) {
        const Two d = pair_of(v, k) - from[k];
        sum[k] = sum[k] + d;
        squares[k] = fma2(d, d, squares[k]);
      }
    };
    {
      Channels<VEC> mean = {};
      const int32_t few = min(rows, kStep);
#pragma unroll
      for (int u = 0; u < kStep; ++u) {
        if (u >= few) break;
        const Channels<VEC> v = load_channels<X, VEC, false>(x + u * pace);
#pragma unroll
        for (int c = 0; c < VEC; ++c) mean.v[c] += v.v[c];
      }
      const float inverse = 1.f / few;
      if constexpr (SHARED) {
        float all = 0.f;
#pragma unroll
        for (int c = 0; c < VEC; ++c) all += mean.v[c];
#pragma unroll
        for (int c = 0; c < VEC; ++c) mean.v[c] = all * (1.f / VEC);
      }
#pragma unroll
      for (int k = 0; k < kP; ++k) from[k] = pair_of(mean, k) * both(inverse);
    }
    // Joins the sums of the last `some` rows to the stretches before, which have `before`; the next begins.
    auto close = [&](int32_t before, int32_t some) {
      const float inverse = 1.f / (some * (SHARED ? VEC : 1));
      const double share = (double)some / (before + some), weight = (double)before * (SHARED ? VEC : 1) * share;
      Channels<VEC> s, q, f;
#pragma unroll
      for (int k = 0; k < kP; ++k) set_pair(s, k, sum[k]), set_pair(q, k, squares[k]), set_pair(f, k, from[k]);
#pragma unroll
      for (int c = 0; c < kEach; ++c) {
        float total = s.v[c], all = q.v[c];
        if constexpr (SHARED) {
#pragma unroll
          for (int o = 1; o < VEC; ++o) total += s.v[o], all += q.v[o];
        }
        const float off = total * inverse, m2 = fmaf(-off, total, all), mean = f.v[c] + off;
        double2* const so_far = stretches + c * kNormThreads + threadIdx.x;
        double2 r = before > 0 ? *so_far : make_double2(0.0, 0.0);
        const double d = mean - r.x;
        r.x += d * share;
        r.y += (m2 < 0.f ? 0.f : m2) + d * d * weight;  // NaN stays NaN
        *so_far = r;
        f.v[c] = mean;
      }
#pragma unroll
      for (int k = 0; k < kP; ++k) {
        from[k] = SHARED ? both(f.v[0]) : pair_of(f, k);
        sum[k] = squares[k] = both(0.f);
      }
    };
    int32_t r = 0, begin = 0;
    while (r + kStatRows <= rows) {
      Channels<VEC> v[kStatRows];
      if (r + kStatRows <= rows - sh.kept) {
#pragma unroll
        for (int u = 0; u < kStatRows; ++u) v[u] = load_channels<X, VEC, true>(x + u * pace);
      } else {
#pragma unroll
        for (int u = 0; u < kStatRows; ++u) v[u] = load_channels<X, VEC, false>(x + u * pace);
      }
#pragma unroll
      for (int u = 0; u < kStatRows; ++u) add(v[u]);
      r += kStatRows, x += kStatRows * pace;
      if (r % kStretch == 0 || r <= 2 * kStatRows) {
        close(begin, r - begin);
        begin = r;
      }
    }
    for (; r < rows; ++r, x += pace) add(load_channels<X, VEC, false>(x));
    if (r > begin) close(begin, r - begin);
    n = (float)rows * (SHARED ? VEC : 1);
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const double2 all = stretches[k * kNormThreads + threadIdx.x];
      m[k] = Moments{(float)all.x, (float)all.y};
    }
  }
  __syncthreads();  // the places are used anew
  join_block<kEach>(n, m, reinterpret_cast<Moments*>(stretches), counts, sh.across, sh.down);
  if (at.y == 0 && at.channel < a.F) {
    const int32_t units = a.F / VEC * kEach;
    float2* out = partial + (int64_t)blockIdx.x * units + at.channel / VEC * kEach;
#pragma unroll
    for (int k = 0; k < kEach; ++k) out[k] = make_float2(m[k].mean, m[k].m2);
  }
}

// Short graphs: statistics and results in one launch.  What every block costs beside its cells counts here: sums over the
// block are plain ones (the mean, then the squares about it), one warp for a group.
template <typename X, typename Y, int ACT, int VEC, bool SHARED>
__global__ void __launch_bounds__(kGraphThreads, VEC == 8 ? 6 : 8) norm_graph_kernel(const __grid_constant__ NormArgs a, const __grid_constant__ GraphPlan plan) {
  constexpr int kEach = kUnits<VEC, SHARED>;
  __shared__ Moments parts[kGraphThreads * kEach];
  __shared__ float counts[kGraphThreads];
  __shared__ float2 group_parts[kTileGroups], group_stats[kTileGroups], block_cells;
  const bool is_long = blockIdx.x < plan.long_blocks;
  const GraphShape sh = is_long ? plan.shape[0] : plan.shape[1];
  const GraphPlace at = graph_place(a, plan, sh, is_long);
  const X* x = static_cast<const X*>(a.X) + at.base;
  Y* y = static_cast<Y*>(a.out) + at.base;
  const bool mine = at.channel < a.F;
  extern __shared__ uint4 slots[];
  RawChannels<X, VEC>* const slot = reinterpret_cast<RawChannels<X, VEC>*>(slots) + threadIdx.x;
  const int64_t pace = (int64_t)at.step * a.F;
  // the thread's rows, and in groups of kStep
  const int32_t count = mine && at.row < at.rows ? (at.rows - at.row + at.step - 1) / at.step : 0;
  const int32_t steps = (count + kStep - 1) / kStep;
  auto fetch_rows = [&](int32_t q, int place) {
    const X* from = x + q * kStep * pace;
#pragma unroll
    for (int u = 0; u < kStep; ++u, from += pace)
      if (q * kStep + u < count) fetch<X, VEC>(slot + (place * kStep + u) * kGraphThreads, from);
  };
  Moments m[kEach] = {};
  float n = 0.f;
  Fixed<VEC> f;
  if (mine) fix_weights<VEC>(f, a, at.channel);
  ring_forward<kRing>(steps, fetch_rows, [&](int32_t q, int place) {
    Channels<VEC> v[kStep];
    const int32_t rows = min(count - q * kStep, kStep);
#pragma unroll
    for (int u = 0; u < kStep; ++u) {
      v[u] = Channels<VEC>{};
      if (u < rows) v[u] = numbers_of(slot[(place * kStep + u) * kGraphThreads]);
    }
    add_rows<VEC, SHARED>(v, rows, n, m);
  });
  // parts[y][unit of the tile], and the cells of each in counts[y]
  if (at.y < sh.down) {
#pragma unroll
    for (int k = 0; k < kEach; ++k) parts[threadIdx.x * kEach + k] = m[k];
    if (at.x == 0) counts[at.y] = n;
  }
  __syncthreads();
  // a team of threads for a group
  const int32_t groups = group_of(plan, at.tile_channels - 1) + 1, units = SHARED ? a.width / VEC : a.width;
  const int32_t team = 1 << sh.team_log, lanes = 1 << sh.lanes_log, stride = sh.across * kEach;
  const int32_t k0 = threadIdx.x & (lanes - 1), y0 = (threadIdx.x & (team - 1)) >> sh.lanes_log, down = team >> sh.lanes_log;
  for (int32_t g0 = 0; g0 < groups; g0 += kGraphThreads >> sh.team_log) {
    const int32_t g = g0 + (threadIdx.x >> sh.team_log);
    const bool some = g < groups;
    const Moments* of_group = parts + g * units;
    float sum = 0.f, total = 0.f;
    if (some) {
      for (int32_t yy = y0; yy < sh.down; yy += down) {
        const float c = counts[yy];
        for (int32_t k = k0; k < units; k += lanes) {
          sum = fmaf(c, of_group[yy * stride + k].mean, sum);
          total += c;
        }
      }
    }
    for (int o = team / 2; o > 0; o /= 2) {
      sum += __shfl_xor_sync(0xffffffffu, sum, o);
      total += __shfl_xor_sync(0xffffffffu, total, o);
    }
    const float mean = total > 0.f ? sum / total : 0.f;
    float squares = 0.f;
    if (some) {
      for (int32_t yy = y0; yy < sh.down; yy += down) {
        const float c = counts[yy];
        for (int32_t k = k0; k < units; k += lanes) {
          const Moments u = of_group[yy * stride + k];
          const float d = u.mean - mean;
          squares += c > 0.f ? fmaf(c * d, d, u.m2) : 0.f;
        }
      }
    }
    for (int o = team / 2; o > 0; o /= 2) squares += __shfl_xor_sync(0xffffffffu, squares, o);
    if (some && (threadIdx.x & (team - 1)) == 0) {
      group_parts[g] = make_float2(mean, squares);
      if (g == 0) block_cells = make_float2(total, 0.f);  // of any group
    }
  }
  if (plan.cluster_log > 0) {
    cluster_arrive();
    cluster_wait();
  }
  __syncthreads();
  for (int32_t g = threadIdx.x; g < groups; g += kGraphThreads) {
    float2 p = group_parts[g];
    if (plan.cluster_log > 0) {
      // the blocks' parts, in the order of their ranks
      float cells = 0.f;
      Moments all = {0.f, 0.f};
      for (int32_t r = 0; r < 1 << plan.cluster_log; ++r) {
        const float2 o = of_rank(group_parts + g, r);
        join(cells, all, of_rank(&block_cells, r).x, Moments{o.x, o.y});
      }
      p = make_float2(all.mean, all.m2);
    }
    const float cells = at.rows > 0 ? (float)at.rows * a.width : 1.f;
    const float2 st = make_float2(p.x, 1.f / sqrtf(p.y / cells + a.eps));
    group_stats[g] = st;
    if (at.rank == 0) a.stats[(int64_t)at.graph * a.groups + at.tile_first / a.width + g] = st;
  }
  if (plan.cluster_log > 0) cluster_arrive();  // the others' shared memory has been read
  __syncthreads();
  if (mine) {
    const int32_t first = at.channel - at.tile_first, shared_group = SHARED ? group_of(plan, first) : 0;
    fix_stats<VEC>(f, [&](int c) { return group_stats[SHARED ? shared_group : group_of(plan, first + c)]; });
    ring_back<kRing>(steps, fetch_rows, [&](int32_t q, int place) {
      Y* to = y + q * kStep * pace;
#pragma unroll
      for (int u = 0; u < kStep; ++u, to += pace) {
        if (q * kStep + u >= count) break;
        Channels<VEC> v = numbers_of(slot[(place * kStep + u) * kGraphThreads]);
        normalise<ACT, VEC>(v, f);
        store_channels<Y, VEC>(to, v);
      }
    });
  }
  if (plan.cluster_log > 0) cluster_wait();
}

// stats of a group from its pieces' moments, in 64 bits; `units` moments of `cells` channels each for a group.  A block, or
// with PER_WARP a warp, for a group: `lanes` threads (a power of two) along the units, the others along the
// pieces.  Means are taken from the first one on, so that one pass is enough: the differences' squares are exact.
template <bool PER_WARP>
__global__ void norm_join_kernel(NormArgs a, NormShape sh, const Piece* pieces, const int32_t* first, const float2* partial,
                                 int32_t units, int32_t cells, int32_t lanes) {
  cudaGridDependencySynchronize();
  const int32_t thread = PER_WARP ? threadIdx.x & 31 : threadIdx.x;
  const int64_t pair = PER_WARP ? (int64_t)blockIdx.x * (blockDim.x / 32) + threadIdx.x / 32 : blockIdx.x;
  if (pair >= a.graphs * a.groups) return;
  const int64_t graph = pair / a.groups;
  const int32_t group = (int32_t)(pair % a.groups);
  const Rows r = rows_of(a, graph);
  const int32_t lo = first ? first[graph] : 0, hi = first ? first[graph + 1] : sh.pieces;
  const double n = r.hi > r.lo ? (double)(r.hi - r.lo) * a.width : 1.0;
  const float2* mine = partial + (int64_t)group * units;
  const int64_t stride = (int64_t)a.groups * units;
  const int32_t down = (PER_WARP ? 32 : blockDim.x) / lanes;
  const double from = hi > lo ? mine[lo * stride].x : 0.f;
  double sum = 0.0, squares = 0.0;
#pragma unroll 4
  for (int32_t p = lo + thread / lanes; p < hi; p += down) {
    const double rows = pieces ? pieces[p].rows : p + 1 < sh.pieces ? sh.rows : (int32_t)(a.rows - (int64_t)p * sh.rows);
    double s1 = 0.0, s2 = 0.0;
    for (int32_t k = thread % lanes; k < units; k += lanes) {
      const float2 m = mine[p * stride + k];
      const double d = m.x - from;
      s1 += d;
      s2 += m.y + rows * cells * d * d;
    }
    sum += rows * cells * s1;
    squares += s2;
  }
  const double2 both_sums = PER_WARP ? make_double2(warp_sum(sum), warp_sum(squares)) : block_sums(sum, squares);
  sum = both_sums.x;
  squares = both_sums.y;
  const double off = sum / n, var = squares / n - off * off;
  // from and the moments of no rows are 0; a variance below 0 is one of rounding (NaN stays NaN)
  if (thread == 0)
    a.stats[pair] = make_float2((float)(from + off), (float)(1.0 / sqrt((var < 0.0 ? 0.0 : var) + (double)a.eps)));
}

// Every block takes the rows of its piece from the last one back: all pieces are read at the same time, and the L2 holds
// their ends.
template <typename X, typename Y, int ACT, int VEC>
__global__ void __launch_bounds__(kNormThreads, VEC == 8 ? 3 : 4) norm_apply_kernel(NormArgs a, NormShape sh, const Piece* pieces) {
  constexpr int kRows = sizeof(X) * VEC == 16 ? 4 : 8;  // in flight
  cudaGridDependencySynchronize();
  const Place at = place_of(a, sh, pieces, blockIdx.x);
  if (at.channel >= a.F || at.y >= at.piece.rows) return;
  const Fixed<VEC> f = fixed_of<VEC>(a, at.piece.graph, at.channel);
  int32_t rows = (at.piece.rows - at.y + at.down - 1) / at.down;
  const int64_t pace = (int64_t)at.down * a.F;
  const int64_t base = ((int64_t)at.piece.row + at.y) * a.F + at.channel + (rows - 1) * pace;
  const X* x = static_cast<const X*>(a.X) + base;
  Y* y = static_cast<Y*>(a.out) + base;
  for (; rows >= kRows; rows -= kRows, x -= kRows * pace, y -= kRows * pace) {
    Channels<VEC> v[kRows];
#pragma unroll
    for (int u = 0; u < kRows; ++u) v[u] = load_channels<X, VEC, true>(x - u * pace);
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      normalise<ACT, VEC>(v[u], f);
      store_channels<Y, VEC>(y - u * pace, v[u]);
    }
  }
  for (; rows > 0; --rows, x -= pace, y -= pace) {
    Channels<VEC> v = load_channels<X, VEC, true>(x);
    normalise<ACT, VEC>(v, f);
    store_channels<Y, VEC>(y, v);
  }
}

// One block for each group of each graph, which goes through its cells three times; sums in 64 bits.
template <typename X, typename Y, int ACT>
__global__ void __launch_bounds__(kNormThreads) norm_fwd_direct_kernel(NormArgs a, int across) {
  const X* x = static_cast<const X*>(a.X);
  Y* y = static_cast<Y*>(a.out);
  const int64_t graph = blockIdx.x / a.groups;
  const int32_t channel = (int32_t)(blockIdx.x % a.groups) * a.width;
  const Rows r = rows_of(a, graph);
  const double cells = r.hi > r.lo ? (double)(r.hi - r.lo) * a.width : 1.0;
  double sum = 0.0;
  for_cells(a, r, channel, across, [&](int64_t i, int32_t) { sum += as_float(x[i]); });
  const double mean = block_sum(sum) / cells;
  sum = 0.0;
  for_cells(a, r, channel, across, [&](int64_t i, int32_t) {
    const double d = as_float(x[i]) - mean;
    sum += d * d;
  });
  const float2 st = make_float2((float)mean, (float)(1.0 / sqrt(block_sum(sum) / cells + (double)a.eps)));
  if (threadIdx.x == 0) a.stats[blockIdx.x] = st;
  for_cells(a, r, channel, across, [&](int64_t i, int32_t c) {
    const float hat = (as_float(x[i]) - st.x) * st.y;
    y[i] = as<Y>(activated<ACT>(fmaf(hat, a.weight ? a.weight[c] : 1.f, a.bias ? a.bias[c] : 0.f)));
  });
}

template <typename X, typename Y, int ACT>
dg_status_t forward(const Graph* g, const NormArgs& a, dg_type_t x, dg_type_t y, cudaStream_t s) {
  const int vec = norm_vector(a, x, y);
  const bool shared = vec > 1 && a.width % vec == 0;
  if (const GraphPlan plan = graph_plan(g, a, vec, sizeof(X), kSlots, shared); plan.blocks > 0) {
    DG_CUDA((by_vector<sizeof(X) == 2 && sizeof(Y) == 2>(vec, [&](auto v) {
      constexpr int VEC = decltype(v)::value;
      constexpr size_t kBytes = (size_t)kSlots * kGraphThreads * VEC * sizeof(X);
      static_assert(kBytes <= kMostPlaces, "ask for more shared memory");
      return shared ? launch_graphs(plan, norm_graph_kernel<X, Y, ACT, VEC, true>, kBytes, s, a)
                    : launch_graphs(plan, norm_graph_kernel<X, Y, ACT, VEC, false>, kBytes, s, a);
    })));
    count_launches(1);
    return DG_OK;
  }
  const NormShape sh = norm_shape(g, a, vec, sizeof(X), vec == 8 ? 3 : 4);
  const int32_t units = shared ? a.F / vec : a.F;
  void* memory = nullptr;
  if (sh.pieces > 0 && scratch_alloc(g, (size_t)sh.pieces * units * sizeof(float2), s, &memory) != cudaSuccess) {
    int across = 1;
    while (across < a.width && across < kNormThreads) across *= 2;
    norm_fwd_direct_kernel<X, Y, ACT><<<(unsigned)(a.graphs * a.groups), kNormThreads, 0, s>>>(a, across);
    DG_CUDA(cudaGetLastError());
    count_launches(1);
    return DG_OK;
  }
  float2* partial = static_cast<float2*>(memory);
  const dim3 grid((unsigned)sh.pieces, (unsigned)sh.tiles);
  const Piece* pieces = g->batch_pieces;
  if (sh.pieces > 0)
    by_vector<sizeof(X) == 2>(vec, [&](auto v) {
      constexpr int VEC = decltype(v)::value;
      if (shared)
        norm_stats_kernel<X, VEC, true><<<grid, kNormThreads, 0, s>>>(a, sh, pieces, partial);
      else
        norm_stats_kernel<X, VEC, false><<<grid, kNormThreads, 0, s>>>(a, sh, pieces, partial);
    });
  cudaError_t e = cudaGetLastError();
  // a warp joins a few pieces, a block many
  const int32_t of_group = units / a.groups;
  int32_t lanes = 1;
  while (lanes < of_group && lanes < 32) lanes *= 2;
  const int32_t cells = shared ? vec : 1;
  const int64_t pairs = a.graphs * a.groups;
  if (e == cudaSuccess)
    e = pieces ? launch_kernel(norm_join_kernel<true>, dim3((unsigned)((pairs + 7) / 8)), kNormThreads, s, true, a, sh, pieces,
                               g->batch_first, (const float2*)partial, of_group, cells, lanes)
               : launch_kernel(norm_join_kernel<false>, dim3((unsigned)pairs), 512, s, true, a, sh, pieces, g->batch_first,
                               (const float2*)partial, of_group, cells, lanes);
  if (e == cudaSuccess && sh.pieces > 0)
    e = by_vector<sizeof(X) == 2 && sizeof(Y) == 2>(vec, [&](auto v) {
      return launch_kernel(norm_apply_kernel<X, Y, ACT, decltype(v)::value>, grid, kNormThreads, s, true, a, sh, pieces);
    });
  pool_free(memory, s);
  DG_CUDA(e);
  count_launches(sh.pieces > 0 ? 3 : 1);
  return DG_OK;
}

}  // namespace

int norm_vector(const NormArgs& a, dg_type_t x, dg_type_t y) {
  int vec = x == DG_BF16 && y == DG_BF16 ? 8 : 4;
  auto fits = [&](const void* p, dg_type_t type) { return (uintptr_t)p % (vec * (type == DG_F32 ? 4 : 2)) == 0; };
  // forward: Y has the type y; backward: dX has the type x
  while (vec > 1 && !(a.F % vec == 0 && fits(a.X, x) && fits(a.dY, y) && fits(a.out, a.dY ? x : y))) vec /= 2;
  return vec;
}

GraphPlan graph_plan(const Graph* g, const NormArgs& a, int vec, int x_bytes, int rows_kept, bool shared) {
  GraphPlan plan{}, none{};
  const int64_t longest = g->batch_longest < 0 ? g->n : g->batch_longest;
  const int32_t vectors = a.F / vec;
  // the fewest vectors that whole groups fill
  int32_t least = a.width;
  while (least % vec) least += a.width;
  least /= vec;
  if (least > kGraphThreads) return none;
  // The most: threads of a block, and groups that its arrays hold.  (The fewest hold no more groups than a vector channels.)
  int32_t most = vectors < kGraphThreads ? vectors : kGraphThreads;
  if (most > kTileGroups * a.width / vec) most = kTileGroups * a.width / vec;
  plan.by_width = 1.f / a.width;
  plan.order = g->batch_order;
  auto shape = [&](int32_t across) {
    GraphShape sh{};
    sh.vec = vec;
    const int32_t parts = vectors / least, tiles = (vectors + across - 1) / across;  // of even width
    sh.across = (parts + tiles - 1) / tiles * least;
    sh.by_across = (65536 + sh.across - 1) / sh.across;
    sh.down = kGraphThreads / sh.across;
    sh.tiles = (vectors + sh.across - 1) / sh.across;
    const int32_t units = shared ? a.width / vec : a.width;
    while (sh.lanes_log < 5 && (1 << sh.lanes_log) < units) ++sh.lanes_log;
    const int32_t groups = sh.across * vec / a.width;
    sh.team_log = 5;
    while (sh.team_log > sh.lanes_log && (kGraphThreads >> sh.team_log) < groups) --sh.team_log;
    return sh;
  };
  auto narrow = [&](int bytes) {
    int32_t across = least;
    while (across * vec * x_bytes < bytes && across + least <= most) across += least;
    return across;
  };
  auto kept = [&](const GraphShape& sh) { return (int64_t)sh.down * rows_kept; };  // rows in a block's shared memory
  // Few graphs: clusters, in tiles of whole lines, or of sectors where that leaves SMs without a block.
  int32_t across = narrow(128);
  if (a.graphs * (vectors / across) < g->sm_count) across = narrow(32);
  GraphShape& first = plan.shape[0];
  first = shape(across);
  if (a.graphs * first.tiles < 2 * (int64_t)g->sm_count) {
    if (longest > (kept(first) << kClusterLog) * 2) return none;
    plan.cluster_log = kClusterLog;
    plan.long_graphs = (int32_t)a.graphs;
    plan.blocks = plan.long_blocks = (int32_t)(a.graphs * first.tiles << kClusterLog);
    return plan;
  }
  // Many: those of more than eight times what a block keeps in narrow tiles, the others as wide as an average graph leaves
  // threads with rows.  2048 graphs of 1 to 2500 rows of 128, forward / backward, from a cold L2: 39 / 52 us; narrow from twice what
  // a block keeps on 39 / 64, from once 49 / 76; in pieces as the long graphs' kernels take them 64 / 123.  (The long ones by
  // clusters, when this was chosen: 43 / 74 where it was 33 / 58.)
  first = shape(narrow(64));
  if (longest > 16 * kept(first)) return none;
  across = first.across;
  while (across + least <= most && 4 * (int64_t)(kGraphThreads / (across + least)) * rows_kept * a.graphs >= a.rows)
    across += least;
  plan.shape[1] = shape(across);
  if (g->batch_lengths) {
    const int64_t most = 8 * kept(plan.shape[1]);
    int64_t lo = 0, hi = a.graphs;
    while (lo < hi) {
      const int64_t mid = (lo + hi) / 2;
      if (g->batch_lengths[mid] > most) lo = mid + 1; else hi = mid;
    }
    plan.long_graphs = (int32_t)lo;
  }
  plan.blocks = plan.long_graphs * (int64_t)first.tiles + (a.graphs - plan.long_graphs) * plan.shape[1].tiles;
  if (plan.blocks >= (int64_t)1 << 31) return none;
  plan.long_blocks = plan.long_graphs * first.tiles;
  return plan;
}

NormShape norm_shape(const Graph* g, const NormArgs& a, int vec, int cell_bytes, int blocks_per_sm) {
  NormShape sh{};
  sh.vec = vec;
  const int32_t vectors = a.F / vec;
  // the tiles that leave the fewest threads idle, none narrower than 16 vectors
  int64_t best = -1;
  for (int32_t tiles = (vectors + kNormThreads - 1) / kNormThreads; tiles == 1 || vectors / tiles >= 16; ++tiles) {
    const int32_t across = (vectors + tiles - 1) / tiles, down = kNormThreads / across;
    if (across == 0) break;
    const int64_t used = (int64_t)vectors * down * 65536 / tiles;  // threads with work, times a constant
    if (used > best) {
      best = used;
      sh.across = across, sh.down = down, sh.tiles = (vectors + across - 1) / across;
    }
    if (tiles >= 4 + (vectors + kNormThreads - 1) / kNormThreads) break;
  }
  if (g->batch_pieces) {
    sh.pieces = g->batch_piece_count;
    sh.kept = INT32_MAX / 2;  // the graphs' pieces come in several waves
    return sh;
  }
  // one wave: then every block reads its piece forward and back, and the L2 holds the end of each
  const int64_t blocks = (int64_t)g->sm_count * blocks_per_sm / sh.tiles;
  int64_t rows = (a.rows + blocks - 1) / (blocks > 0 ? blocks : 1);
  const int64_t least = (int64_t)sh.down * 8;
  if (rows < least) rows = least;
  sh.rows = (int32_t)rows;
  sh.pieces = (int32_t)((a.rows + rows - 1) / rows);
  const int64_t kept = (int64_t)(g->l2_bytes / 2) / ((int64_t)a.F * cell_bytes * (sh.pieces > 0 ? sh.pieces : 1)) / sh.down;
  sh.kept = (int32_t)(kept < rows ? kept : rows);
  return sh;
}

dg_status_t group_norm_fwd(const Graph* g, const NormArgs& a, dg_type_t x, dg_type_t y, dg_act_t act, cudaStream_t s) {
  return by_type(x, y, act, [&](auto xs, auto ys, auto kind) {
    return forward<decltype(xs), decltype(ys), decltype(kind)::value>(g, a, x, y, s);
  });
}

}  // namespace dg
