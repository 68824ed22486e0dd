// Gradients of the group norm with an activation: dg_norm.cuh has the formulas.
//
// As forward: pieces of rows leave the sums of d and of d hat of their channels, a small kernel makes A and B of every
// group and the gradients of weight and bias of them, and the last launch goes through the pieces backwards.
#include "dg_norm.cuh"

namespace dg {
namespace {

constexpr int kRows = 4;  // in flight per thread, of each matrix

// A thread's channels: what does not change along its rows.
template <int VEC>
struct Fixed {
  float mean[VEC], rstd[VEC], w[VEC], b[VEC];
};
template <int VEC>
__device__ __forceinline__ Fixed<VEC> fixed_of(const NormArgs& a, int32_t graph, int32_t channel) {
  Fixed<VEC> f;
#pragma unroll
  for (int c = 0; c < VEC; ++c) {
    const float2 st = a.stats[(int64_t)graph * a.groups + (channel + c) / a.width];
    f.mean[c] = st.x, f.rstd[c] = st.y;
    f.w[c] = a.weight ? a.weight[channel + c] : 1.f;
    f.b[c] = a.bias ? a.bias[channel + c] : 0.f;
  }
  return f;
}

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

// The first graphs x groups blocks: (A, B) of a group.  The others: the gradients of weight and bias of 8 channels each,
// a warp along the pieces for a channel.  Sums in 64 bits.
__global__ void __launch_bounds__(kNormThreads)
    norm_join_sums_kernel(NormArgs a, NormShape sh, const int32_t* first, const float2* partial, float2* means, float* dweight,
                          float* dbias) {
  cudaGridDependencySynchronize();
  const int64_t pairs = means ? a.graphs * a.groups : 0;
  if (blockIdx.x < pairs) {
    const int64_t graph = blockIdx.x / a.groups;
    const int32_t group = (int32_t)(blockIdx.x % a.groups);
    const Rows r = rows_of(a, graph);
    const int32_t lo = first ? first[graph] : 0, hi = first ? first[graph + 1] : sh.pieces;
    const int64_t entries = (int64_t)(hi - lo) * a.width;
    double s1 = 0.0, s2 = 0.0;
    for (int64_t e = threadIdx.x; e < entries; e += blockDim.x) {
      const int32_t channel = group * a.width + (int32_t)(e % a.width);
      const float2 p = partial[(lo + e / a.width) * a.F + channel];
      const double w = a.weight ? a.weight[channel] : 1.f;
      s1 += w * p.x;
      s2 += w * p.y;
    }
    s1 = block_sum(s1);
    s2 = block_sum(s2);
    const double n = r.hi > r.lo ? (double)(r.hi - r.lo) * a.width : 1.0;
    if (threadIdx.x == 0) means[blockIdx.x] = make_float2((float)(s1 / n), (float)(s2 / n));
    return;
  }
  const int lane = threadIdx.x & 31, warps = blockDim.x / 32;
  const int64_t c = (blockIdx.x - pairs) * warps + threadIdx.x / 32;
  if (c >= a.F) return;
  double s1 = 0.0, s2 = 0.0;
  for (int32_t p = lane; p < sh.pieces; p += 32) {
    const float2 v = partial[(int64_t)p * a.F + c];
    s1 += v.x;
    s2 += v.y;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    s1 += __shfl_xor_sync(0xffffffffu, s1, o);
    s2 += __shfl_xor_sync(0xffffffffu, s2, o);
  }
  if (lane == 0) {
    if (dbias) dbias[c] = (float)s1;
    if (dweight) dweight[c] = (float)s2;
  }
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
  const NormShape sh = norm_shape(g, a, vec);
  const size_t partial_bytes = (size_t)sh.pieces * a.F * sizeof(float2);
  const int64_t pairs = a.out ? a.graphs * a.groups : 0;
  void* memory = nullptr;
  if (scratch_alloc(g, partial_bytes + (size_t)pairs * sizeof(float2), s, &memory) != cudaSuccess) {
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
  const int threads = a.graphs == 1 || sh.pieces / a.graphs * a.width > 64 ? kNormThreads : 32;
  const int64_t blocks = pairs + (weights ? (a.F + threads / 32 - 1) / (threads / 32) : 0);
  if (e == cudaSuccess)
    e = launch_kernel(norm_join_sums_kernel, dim3((unsigned)blocks), threads, s, true, a, sh, g->batch_first,
                      (const float2*)partial, a.out ? means : (float2*)nullptr, dweight, dbias);
  if (e == cudaSuccess && a.out && sh.pieces > 0)
    e = by_vector<kWide>(vec, [&](auto v) {
      return launch_kernel(norm_apply_bwd_kernel<X, Y, ACT, decltype(v)::value>, grid, kNormThreads, s, true, a, sh, pieces,
                           (const float2*)means);
    });
  pool_free(memory, s);
  DG_CUDA(e);
  count_launches(1 + (sh.pieces > 0) + (a.out && sh.pieces > 0));
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
