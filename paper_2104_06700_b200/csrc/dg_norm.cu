// Group norm with an activation over the rows of an n x F matrix, channels last, forward: dg_norm.cuh has the formulas.
//
// Statistics need every row before the first result, so a matrix is read twice: pieces of rows leave the mean and the sum
// of squares about it of their channels, a small kernel joins them, and the last launch goes through the pieces backwards,
// those first that the L2 still holds.
#include "dg_norm.cuh"

namespace dg {
namespace {

// Rows a thread has in flight, and takes the mean of before it joins that to what it has.
constexpr int kStatRows = 8;

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

// partial[piece][unit]: the moments of a channel, or, with SHARED, of a vector of channels of one group.
template <typename X, int VEC, bool SHARED>
__global__ void __launch_bounds__(kNormThreads) norm_stats_kernel(NormArgs a, NormShape sh, const Piece* pieces, float2* partial) {
  constexpr int kUnits = SHARED ? 1 : VEC;
  constexpr float kCells = SHARED ? VEC : 1;
  __shared__ Moments parts[kNormThreads * kUnits];
  __shared__ float counts[kNormThreads];
  const Place at = place_of(a, sh, pieces, blockIdx.x);
  Moments m[kUnits] = {};
  float n = 0.f;
  if (at.channel < a.F) {
    const X* x = static_cast<const X*>(a.X) + (int64_t)at.piece.row * a.F + at.channel;
    for (int32_t r0 = at.y; r0 < at.piece.rows; r0 += at.down * kStatRows) {
      Channels<VEC> v[kStatRows];
      int rows = 0;
#pragma unroll
      for (int u = 0; u < kStatRows; ++u) {
        const int32_t r = r0 + u * at.down;
        if (r < at.piece.rows) {
          v[u] = load_channels<X, VEC>(x + (int64_t)r * a.F);
          ++rows;
        } else {
#pragma unroll
          for (int c = 0; c < VEC; ++c) v[u].v[c] = 0.f;
        }
      }
      const float cells = rows * kCells, inverse = 1.f / cells;
      const float total = n + cells, share = cells / total;
#pragma unroll
      for (int k = 0; k < kUnits; ++k) {
        float sum = 0.f;
#pragma unroll
        for (int u = 0; u < kStatRows; ++u) {
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
        for (int u = 0; u < kStatRows; ++u) {
          if (u < rows) {
            if constexpr (SHARED) {
#pragma unroll
              for (int c = 0; c < VEC; ++c) m2 = fmaf(v[u].v[c] - mean, v[u].v[c] - mean, m2);
            } else {
              m2 = fmaf(v[u].v[k] - mean, v[u].v[k] - mean, m2);
            }
          }
        }
        const float d = mean - m[k].mean;
        m[k].mean = fmaf(d, share, m[k].mean);
        m[k].m2 += m2 + d * d * (n * share);
      }
      n = total;
    }
  }
  counts[threadIdx.x] = n;
#pragma unroll
  for (int k = 0; k < kUnits; ++k) parts[k * kNormThreads + threadIdx.x] = m[k];
  // the rows' threads in pairs, always in the same order
  int half = 1;
  while (half < sh.down) half *= 2;
  for (half /= 2; half > 0; half /= 2) {
    __syncthreads();
    const int other = threadIdx.x + half * sh.across;
    if (at.y < half && at.y + half < sh.down) {
      const float nb = counts[other];
      float total = n;
#pragma unroll
      for (int k = 0; k < kUnits; ++k) {
        total = n;
        join(total, m[k], nb, parts[k * kNormThreads + other]);
        parts[k * kNormThreads + threadIdx.x] = m[k];
      }
      n = total;
      counts[threadIdx.x] = n;
    }
  }
  if (at.y == 0 && at.channel < a.F) {
    const int32_t units = a.F / VEC * kUnits;
    float2* out = partial + (int64_t)blockIdx.x * units + at.channel / VEC * kUnits;
#pragma unroll
    for (int k = 0; k < kUnits; ++k) out[k] = make_float2(m[k].mean, m[k].m2);
  }
}

// stats of a group from its pieces' moments, in 64 bits; `units` moments of `cells` channels each for a group.
__global__ void __launch_bounds__(kNormThreads) norm_join_kernel(NormArgs a, NormShape sh, const Piece* pieces, const int32_t* first,
                                                                  const float2* partial, int32_t units, int32_t cells) {
  cudaGridDependencySynchronize();
  const int64_t graph = blockIdx.x / a.groups;
  const int32_t group = (int32_t)(blockIdx.x % a.groups);
  const Rows r = rows_of(a, graph);
  const int32_t lo = first ? first[graph] : 0, hi = first ? first[graph + 1] : sh.pieces;
  const int64_t entries = (int64_t)(hi - lo) * units;
  const double n = r.hi > r.lo ? (double)(r.hi - r.lo) * a.width : 1.0;
  auto rows = [&](int32_t p) {
    if (pieces) return pieces[p].rows;
    const int64_t left = a.rows - (int64_t)p * sh.rows;
    return (int32_t)(left < sh.rows ? left : sh.rows);
  };
  auto moments = [&](int64_t e, double* count) {
    const int32_t p = lo + (int32_t)(e / units);
    *count = (double)rows(p) * cells;
    return partial[((int64_t)p * a.groups + group) * units + e % units];
  };
  double sum = 0.0, count;
  for (int64_t e = threadIdx.x; e < entries; e += blockDim.x) {
    const float2 m = moments(e, &count);
    sum += count * m.x;
  }
  const double mean = block_sum(sum) / n;
  sum = 0.0;
  for (int64_t e = threadIdx.x; e < entries; e += blockDim.x) {
    const float2 m = moments(e, &count);
    const double d = m.x - mean;
    sum += m.y + count * d * d;
  }
  sum = block_sum(sum);
  if (threadIdx.x == 0) a.stats[blockIdx.x] = make_float2((float)mean, (float)(1.0 / sqrt(sum / n + (double)a.eps)));
}

template <typename X, typename Y, int ACT, int VEC>
__global__ void __launch_bounds__(kNormThreads) norm_apply_kernel(NormArgs a, NormShape sh, const Piece* pieces) {
  constexpr int kRows = 4;
  cudaGridDependencySynchronize();
  const Place at = place_of(a, sh, pieces, gridDim.x - 1 - blockIdx.x);
  if (at.channel >= a.F) return;
  float mean[VEC], rstd[VEC], w[VEC], b[VEC];
#pragma unroll
  for (int c = 0; c < VEC; ++c) {
    const float2 st = a.stats[(int64_t)at.piece.graph * a.groups + (at.channel + c) / a.width];
    mean[c] = st.x, rstd[c] = st.y;
    w[c] = a.weight ? a.weight[at.channel + c] : 1.f;
    b[c] = a.bias ? a.bias[at.channel + c] : 0.f;
  }
  const int64_t base = (int64_t)at.piece.row * a.F + at.channel;
  const X* x = static_cast<const X*>(a.X) + base;
  Y* y = static_cast<Y*>(a.out) + base;
  for (int32_t r0 = at.y; r0 < at.piece.rows; r0 += at.down * kRows) {
    Channels<VEC> v[kRows];
#pragma unroll
    for (int u = 0; u < kRows; ++u)
      if (r0 + u * at.down < at.piece.rows) v[u] = load_channels<X, VEC>(x + (int64_t)(r0 + u * at.down) * a.F);
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      if (r0 + u * at.down >= at.piece.rows) break;
#pragma unroll
      for (int c = 0; c < VEC; ++c) v[u].v[c] = activated<ACT>(fmaf((v[u].v[c] - mean[c]) * rstd[c], w[c], b[c]));
      store_channels<Y, VEC>(y + (int64_t)(r0 + u * at.down) * a.F, v[u]);
    }
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
  const NormShape sh = norm_shape(g, a, vec);
  const bool shared = vec > 1 && a.width % vec == 0;
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
  const int threads = sh.pieces / a.graphs * (units / a.groups) > 64 ? kNormThreads : 32;
  if (e == cudaSuccess)
    e = launch_kernel(norm_join_kernel, dim3((unsigned)(a.graphs * a.groups)), threads, s, true, a, sh, pieces, g->batch_first,
                      (const float2*)partial, units / a.groups, shared ? (int32_t)vec : (int32_t)1);
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

NormShape norm_shape(const Graph* g, const NormArgs& a, int vec) {
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
  if (g->batch_pieces || a.offsets) {
    sh.pieces = g->batch_piece_count;
    return sh;
  }
  const int64_t blocks = (int64_t)g->sm_count * 6 / sh.tiles;
  int64_t rows = (a.rows + blocks - 1) / (blocks > 0 ? blocks : 1);
  const int64_t least = (int64_t)sh.down * 8;
  if (rows < least) rows = least;
  sh.rows = (int32_t)rows;
  sh.pieces = (int32_t)((a.rows + rows - 1) / rows);
  return sh;
}

dg_status_t group_norm_fwd(const Graph* g, const NormArgs& a, dg_type_t x, dg_type_t y, dg_act_t act, cudaStream_t s) {
  return by_type(x, y, act, [&](auto xs, auto ys, auto kind) {
    return forward<decltype(xs), decltype(ys), decltype(kind)::value>(g, a, x, y, s);
  });
}

}  // namespace dg
