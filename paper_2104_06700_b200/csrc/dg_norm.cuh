// Group norm with an activation, shared by its kernels (not part of the ABI).
//
// A group is the channels [c, c + F / groups) of the rows of one graph of the batch; N cells.
//   mean = sum x / N,  var = sum (x - mean)^2 / N,  rstd = 1 / sqrt(var + eps)
//   hat = (x - mean) rstd,  z = hat w + b,  y = act(z)
//   dz = dy act'(z),  db = sum dz,  dw = sum dz hat  (over all rows),
//   dx = rstd (dz w - A - hat B),  A = sum(dz w) / N,  B = sum(dz w hat) / N
#pragma once

#include <cuda_bf16.h>

#include "dg_internal.cuh"

namespace dg {

struct NormArgs {
  const void* X;         // rows x F
  const void* dY;        // backward
  void* out;             // Y, or backward dX (may be null)
  float2* stats;         // graphs x groups: (mean, rstd)
  const float* weight;   // null: 1
  const float* bias;     // null: 0
  const int64_t* offsets;  // device, graphs + 1; null: one graph of `rows` rows
  int64_t rows;          // behind the last graph's last row
  int64_t graphs;
  int32_t F, groups, width;  // width = F / groups
  float eps;
};

struct Rows {
  int64_t lo, hi;
};
__device__ __forceinline__ Rows rows_of(const NormArgs& a, int64_t graph) {
  return a.offsets ? Rows{a.offsets[graph], a.offsets[graph + 1]} : Rows{0, a.rows};
}

__device__ __forceinline__ float as_float(float v) { return v; }
__device__ __forceinline__ float as_float(__nv_bfloat16 v) { return __bfloat162float(v); }
// A result leaves in its own type, rounded once, to nearest.
template <typename T>
__device__ __forceinline__ T as(float v) {
  if constexpr (sizeof(T) == 4) {
    return v;
  } else {
    return __float2bfloat16_rn(v);
  }
}

// 1 / (1 + exp(-z)).  The fast exponential is off by 2 + |1.2 z| units of 2^-23 and the result by less than that: a
// cell costs 4 to 12 bytes of memory traffic, and the exact one with its division costs as much time.
__device__ __forceinline__ float sigmoid(float z) { return __fdividef(1.f, 1.f + __expf(-z)); }

template <int ACT>
__device__ __forceinline__ float activated(float z) {
  if constexpr (ACT == DG_ACT_RELU) return z <= 0.f ? 0.f : z;  // NaN stays NaN
  if constexpr (ACT == DG_ACT_SILU) return z * sigmoid(z);
  return z;
}

// dy act'(z).  The ReLU's border is where z changes its sign: near it (|hat w| is about |b| there and z is off by up to
// 2^-22 |b|) the sign is taken in 64 bits, so that no row's gradient is lost or added by rounding.
template <int ACT>
__device__ __forceinline__ float before_activation(float dy, float x, float mean, float rstd, float w, float b) {
  if constexpr (ACT == DG_ACT_NONE) return dy;
  const float z = fmaf((x - mean) * rstd, w, b);
  if constexpr (ACT == DG_ACT_RELU) {
    if (fabsf(z) >= fabsf(b) * 0x1p-20f) return z <= 0.f ? 0.f : dy;
    const double exact = ((double)x - mean) * rstd * w + b;
    return exact <= 0.0 ? 0.f : dy;
  }
  const float s = sigmoid(z);
  return dy * (s * fmaf(z, 1.f - s, 1.f));
}

// dg_norm.cu
dg_status_t group_norm_fwd(const Graph* g, const NormArgs& a, dg_type_t x, dg_type_t y, dg_act_t act, cudaStream_t s);
dg_status_t group_norm_bwd(const Graph* g, const NormArgs& a, dg_type_t x, dg_type_t y, dg_act_t act, float* dweight,
                           float* dbias, cudaStream_t s);

}  // namespace dg
