// Group norm with an activation over the rows of an n x F matrix, channels last, and its gradients: dg_norm.cuh has
// the formulas.
#include "dg_norm.cuh"

namespace dg {
namespace {

constexpr int kBlock = 256;

// The sum of v over a block of kBlock threads, in every thread and always in the same order.
__device__ double block_sum(double v) {
  __shared__ double sums[kBlock / 32];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();  // the last call's sums have been read
  if (threadIdx.x % 32 == 0) sums[threadIdx.x / 32] = v;
  __syncthreads();
  v = 0.0;
#pragma unroll
  for (int i = 0; i < kBlock / 32; ++i) v += sums[i];
  return v;
}

// Calls f(index of the cell, its channel) for the thread's cells of a group.  Threads lie along the channels first.
template <typename Fn>
__device__ __forceinline__ void for_cells(const NormArgs& a, Rows r, int32_t channel, int across, Fn f) {
  const int x = threadIdx.x % across, y = threadIdx.x / across, down = kBlock / across;
  for (int64_t row = r.lo + y; row < r.hi; row += down)
    for (int32_t c = x; c < a.width; c += across) f(row * a.F + channel + c, channel + c);
}

// One block for each group of each graph, which goes through its cells three times; sums in 64 bits.
template <typename X, typename Y, int ACT>
__global__ void __launch_bounds__(kBlock) norm_fwd_direct_kernel(NormArgs a, int across) {
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
__global__ void __launch_bounds__(kBlock) norm_bwd_direct_kernel(NormArgs a, int across) {
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
dg_status_t forward(const Graph* g, const NormArgs& a, cudaStream_t s) {
  int across = 1;
  while (across < a.width && across < kBlock) across *= 2;
  norm_fwd_direct_kernel<X, Y, ACT><<<(unsigned)(a.graphs * a.groups), kBlock, 0, s>>>(a, across);
  DG_CUDA(cudaGetLastError());
  count_launches(1);
  return DG_OK;
}

template <typename X, typename Y, int ACT>
dg_status_t backward(const Graph* g, const NormArgs& a, float* dweight, float* dbias, cudaStream_t s) {
  int across = 1;
  while (across < a.width && across < kBlock) across *= 2;
  if (dweight || dbias)
    norm_weights_direct_kernel<X, Y, ACT><<<(unsigned)((a.F + 31) / 32), dim3(32, 32), 0, s>>>(a, dweight, dbias);
  if (a.out) norm_bwd_direct_kernel<X, Y, ACT><<<(unsigned)(a.graphs * a.groups), kBlock, 0, s>>>(a, across);
  DG_CUDA(cudaGetLastError());
  count_launches((dweight || dbias) + (a.out != nullptr));
  return DG_OK;
}

// f(X, Y, act) for the call's types and activation
template <typename Fn>
dg_status_t by_type(dg_type_t x, dg_type_t y, dg_act_t act, Fn f) {
  auto with_act = [&](auto xs, auto ys) {
    if (act == DG_ACT_RELU) return f(xs, ys, std::integral_constant<int, DG_ACT_RELU>());
    if (act == DG_ACT_SILU) return f(xs, ys, std::integral_constant<int, DG_ACT_SILU>());
    return f(xs, ys, std::integral_constant<int, DG_ACT_NONE>());
  };
  if (x == DG_F32) return y == DG_F32 ? with_act(float(), float()) : with_act(float(), __nv_bfloat16());
  return y == DG_F32 ? with_act(__nv_bfloat16(), float()) : with_act(__nv_bfloat16(), __nv_bfloat16());
}

}  // namespace

dg_status_t group_norm_fwd(const Graph* g, const NormArgs& a, dg_type_t x, dg_type_t y, dg_act_t act, cudaStream_t s) {
  return by_type(x, y, act, [&](auto xs, auto ys, auto kind) {
    return forward<decltype(xs), decltype(ys), decltype(kind)::value>(g, a, s);
  });
}

dg_status_t group_norm_bwd(const Graph* g, const NormArgs& a, dg_type_t x, dg_type_t y, dg_act_t act, float* dweight,
                           float* dbias, cudaStream_t s) {
  return by_type(x, y, act, [&](auto xs, auto ys, auto kind) {
    return backward<decltype(xs), decltype(ys), decltype(kind)::value>(g, a, dweight, dbias, s);
  });
}

}  // namespace dg
