// AdamW over many tensors at once, its two states in 32 or in 8 bits, and the norm of all gradients.
//
//   g' = g factor,  m = m + (1 - b1)(g' - m),  v = b2 v + (1 - b2) g'^2,  t = steps taken + 1
//   p = p (1 - lr wd) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// A warp takes 256 numbers of a tensor, the block that shares a scale when the states are 8-bit: the largest |m| and
// sqrt(v) of the block are a warp's reduction away, and the new scales leave in the pass that reads the old ones.
#include <cuda_bf16.h>
#include <math.h>

#include "dg_internal.cuh"

namespace dg {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kBlocksPerSm = 3;                     // what 80 registers a thread leave room for
constexpr int kNumbers = 256;                       // of a warp's task: 8 a lane, and one scale
constexpr int kNormBlocks = 148 * 4;
constexpr float kLargest = 448.f;                   // of e4m3
constexpr float kLeastScale = 0x1p-126f;            // its inverse is finite

// What a launch is told of its tensors, by value: at most 32764 bytes of arguments.
constexpr int kMost = 400, kFew = 24;
enum { kParamBf16 = 1, kGradBf16 = 2, k8Bits = 4, kVectors = 8 };
template <int N>
struct Tensors {
  void* param[N];
  const void* grad[N];
  void* m[N];
  void* v[N];
  float2* scales[N];
  __nv_bfloat16* copy[N];
  int64_t* step[N];
  int64_t count[N];
  int64_t first[N + 1];  // tasks before tensor i's
  uint32_t id[N];
  uint8_t flags[N];
  int32_t n;
};

// The caller's workspace: zero before its first use.
struct Workspace {
  uint32_t step_ticket, norm_ticket;
  double partial[kNormBlocks];
};
static_assert(sizeof(Workspace) <= DG_ADAMW_WORKSPACE_BYTES, "dg.h promises less");

struct Hyper {
  double lr, log2_beta1, log2_beta2;
  float rest1, beta2, rest2, eps, decay;  // 1 - beta1, beta2, 1 - beta2, eps, 1 - lr wd
};

// A 32-bit hash: lowbias32 of Chris Wellons.
__device__ __forceinline__ uint32_t mix(uint32_t x) {
  x ^= x >> 16;
  x *= 0x7feb352du;
  x ^= x >> 15;
  x *= 0x846ca68bu;
  return x ^ (x >> 16);
}

template <int N>
__device__ __forceinline__ int tensor_of(const Tensors<N>& a, int64_t task, int from) {
  int lo = from, hi = a.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (a.first[mid] <= task) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// Four neighbouring numbers; `left` of them exist.
template <typename T, bool VEC>
__device__ __forceinline__ void load4(const T* p, int left, float* out) {
  if constexpr (VEC && sizeof(T) == 4) {
    const float4 q = *reinterpret_cast<const float4*>(p);
    out[0] = q.x, out[1] = q.y, out[2] = q.z, out[3] = q.w;
  } else if constexpr (VEC) {
    const uint2 q = *reinterpret_cast<const uint2*>(p);
    out[0] = __uint_as_float(q.x << 16), out[1] = __uint_as_float(q.x & 0xffff0000u);
    out[2] = __uint_as_float(q.y << 16), out[3] = __uint_as_float(q.y & 0xffff0000u);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      out[j] = 0.f;
      if (j < left) {
        if constexpr (sizeof(T) == 4) out[j] = p[j]; else out[j] = __bfloat162float(p[j]);
      }
    }
  }
}
template <bool VEC>
__device__ __forceinline__ void store4(float* p, int left, const float* in) {
  if constexpr (VEC) {
    *reinterpret_cast<float4*>(p) = make_float4(in[0], in[1], in[2], in[3]);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < left) p[j] = in[j];
  }
}
template <bool VEC>
__device__ __forceinline__ void store4(uint16_t* p, int left, const uint32_t* in) {
  if constexpr (VEC) {
    *reinterpret_cast<uint2*>(p) = make_uint2(in[0] | in[1] << 16, in[2] | in[3] << 16);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < left) p[j] = (uint16_t)in[j];
  }
}
template <bool VEC>
__device__ __forceinline__ uint32_t load_bytes(const uint8_t* p, int left) {
  if constexpr (VEC) return *reinterpret_cast<const uint32_t*>(p);
  uint32_t r = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (j < left) r |= (uint32_t)p[j] << (8 * j);
  return r;
}
template <bool VEC>
__device__ __forceinline__ void store_bytes(uint8_t* p, int left, uint32_t v) {
  if constexpr (VEC) {
    *reinterpret_cast<uint32_t*>(p) = v;
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < left) p[j] = (uint8_t)(v >> (8 * j));
  }
}

// The number an e4m3 code stands for: exponents from -6 on, steps of 2^-9 below 2^-6; 0x7f is NaN.
__device__ __forceinline__ float from_e4m3(uint32_t code) {
  const uint32_t rest = code & 0x7f;
  // the seven bits in fp32's place stand for the number times 2^-120
  float v = __uint_as_float(rest << 20) * 0x1p120f;
  if (rest == 0x7f) v = NAN;
  return code & 0x80 ? -v : v;
}

// An 8-bit state is rounded up with a probability that is its distance from the lower neighbour: the averages move by a
// thousandth of themselves a step, far less than half a step of 3 bits, and rounding to nearest would hold them where they
// are.  y >= 0 or NaN; r: 16 random bits.  In [2^-6, 448] the three mantissa bits to keep are followed by 20: adding the
// random ones there carries into them.  2^-6 more gives the smaller numbers, evenly 2^-9 apart, the same form.
__device__ __forceinline__ uint32_t to_e4m3(float y, uint32_t r) {
  if (y != y || y == INFINITY) return 0x7f;
  y = fminf(y, kLargest);
  const bool small = y < 0x1p-6f;
  if (small) y += 0x1p-6f;
  const uint32_t code = ((__float_as_uint(y) + (r << 4) + 8u) >> 20) - (small ? 968u : 960u);
  return code < 126u ? code : 126u;
}

// A bf16 parameter is rounded up or down by 16 random bits too: steps of a thousandth of it would all be lost to nearest.
__device__ __forceinline__ uint32_t to_bf16_random(float p, uint32_t r) {
  const uint32_t bits = __float_as_uint(p);
  if ((bits & 0x7f800000u) == 0x7f800000u) return __bfloat16_as_ushort(__float2bfloat16_rn(p));
  return (bits + (r & 0xffffu)) >> 16;
}

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
// off by at most 2^-23 of itself
__device__ __forceinline__ float fast_sqrt(float v) {
  float r;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
// the largest of the finite ones: a number that is not finite keeps to itself
__device__ __forceinline__ float finite_max(float m, float v) { return v < INFINITY ? fmaxf(m, v) : m; }

struct Step {
  float c1, c2;   // lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
  uint32_t key;
};

// One task: the numbers base .. base + 255 of a tensor, as far as it goes.  A lane has four at 4 lane, four 128 further.
template <int N, typename P, typename G, bool EIGHT, bool VEC>
__device__ __forceinline__ void update(const Tensors<N>& a, int i, int64_t base, const Hyper& h, const Step& st, float factor) {
  const int lane = threadIdx.x & 31;
  const int64_t at = base + 4 * lane, end = a.count[i];
  const uint32_t key = mix(st.key ^ (uint32_t)(base >> 32));
  float p[8], g[8], m[8], v[8];
  float2 scale = make_float2(0.f, 0.f);
  if (EIGHT) scale = a.scales[i][base / kNumbers];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int64_t q = at + 128 * k;
    const int left = VEC ? 4 : (int)(end - q < 0 ? 0 : end - q < 4 ? end - q : 4);
    load4<P, VEC>(static_cast<const P*>(a.param[i]) + q, left, p + 4 * k);
    load4<G, VEC>(static_cast<const G*>(a.grad[i]) + q, left, g + 4 * k);
    if constexpr (EIGHT) {
      const uint32_t mb = load_bytes<VEC>(static_cast<const uint8_t*>(a.m[i]) + q, left);
      const uint32_t ub = load_bytes<VEC>(static_cast<const uint8_t*>(a.v[i]) + q, left);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        m[4 * k + j] = from_e4m3(mb >> (8 * j) & 0xff) * scale.x;
        const float u = from_e4m3(ub >> (8 * j) & 0xff) * scale.y;
        v[4 * k + j] = u * u;
      }
    } else {
      load4<float, VEC>(static_cast<const float*>(a.m[i]) + q, left, m + 4 * k);
      load4<float, VEC>(static_cast<const float*>(a.v[i]) + q, left, v + 4 * k);
    }
  }
  float most_m = 0.f, most_u = 0.f;
  float u[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float gj = g[j] * factor;
    m[j] = fmaf(h.rest1, gj - m[j], m[j]);
    v[j] = fmaf(h.rest2 * gj, gj, h.beta2 * v[j]);
    u[j] = fast_sqrt(v[j]);
    p[j] = fmaf(p[j], h.decay, -st.c1 * __fdividef(m[j], fmaf(u[j], st.c2, h.eps)));
    if (EIGHT) {
      most_m = finite_max(most_m, fabsf(m[j]));
      most_u = finite_max(most_u, u[j]);
    }
  }
  float inv_m = 0.f, inv_u = 0.f;
  if (EIGHT) {
    const float sm = fmaxf(__fdiv_rn(warp_max(most_m), kLargest), kLeastScale);
    const float su = fmaxf(__fdiv_rn(warp_max(most_u), kLargest), kLeastScale);
    inv_m = __frcp_rn(sm);
    inv_u = __frcp_rn(su);
    if (lane == 0) a.scales[i][base / kNumbers] = make_float2(sm, su);
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int64_t q = at + 128 * k;
    const int left = VEC ? 4 : (int)(end - q < 0 ? 0 : end - q < 4 ? end - q : 4);
    uint32_t r[4] = {};
    if (EIGHT || sizeof(P) == 2) {
#pragma unroll
      for (int j = 0; j < 4; ++j) r[j] = mix((uint32_t)(q + j) + key);
    }
    if constexpr (sizeof(P) == 4) {
      store4<VEC>(static_cast<float*>(a.param[i]) + q, left, p + 4 * k);
      if (a.copy[i]) {  // the master weights keep what the copy loses: to nearest
        uint32_t c[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) c[j] = __bfloat16_as_ushort(__float2bfloat16_rn(p[4 * k + j]));
        store4<VEC>(reinterpret_cast<uint16_t*>(a.copy[i]) + q, left, c);
      }
    } else {
      uint32_t c[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) c[j] = to_bf16_random(p[4 * k + j], r[j]);
      store4<VEC>(static_cast<uint16_t*>(a.param[i]) + q, left, c);
    }
    if constexpr (EIGHT) {
      uint32_t mb = 0, ub = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float mj = m[4 * k + j], uj = u[4 * k + j];
        const uint32_t cm = to_e4m3(fabsf(mj) * inv_m, r[j] & 0xffff) | (mj < 0.f ? 0x80u : 0u);
        uint32_t cu = to_e4m3(uj * inv_u, r[j] >> 16);
        if (uj > 0.f && cu == 0) cu = 1;  // a denominator that was not 0 does not become 0
        mb |= cm << (8 * j);
        ub |= cu << (8 * j);
      }
      store_bytes<VEC>(static_cast<uint8_t*>(a.m[i]) + q, left, mb);
      store_bytes<VEC>(static_cast<uint8_t*>(a.v[i]) + q, left, ub);
    } else {
      store4<VEC>(static_cast<float*>(a.m[i]) + q, left, m + 4 * k);
      store4<VEC>(static_cast<float*>(a.v[i]) + q, left, v + 4 * k);
    }
  }
}

template <int N, typename P, typename G>
__device__ __forceinline__ void update_typed(const Tensors<N>& a, int i, int64_t base, const Hyper& h, const Step& st,
                                             float factor) {
  const bool vectors = a.flags[i] & kVectors && base + kNumbers <= a.count[i];
  if (a.flags[i] & k8Bits) {
    if (vectors)
      update<N, P, G, true, true>(a, i, base, h, st, factor);
    else
      update<N, P, G, true, false>(a, i, base, h, st, factor);
  } else {
    if (vectors)
      update<N, P, G, false, true>(a, i, base, h, st, factor);
    else
      update<N, P, G, false, false>(a, i, base, h, st, factor);
  }
}

template <int N>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm)
    adamw_kernel(const __grid_constant__ Tensors<N> a, Hyper h, const float* factor_at, uint64_t seed, Workspace* ws) {
  const int lane = threadIdx.x & 31;
  cudaGridDependencySynchronize();
  const float factor = factor_at ? *factor_at : 1.f;
  const int64_t tasks = a.first[a.n];
  int i = -1;
  Step st{};
  for (int64_t task = (int64_t)blockIdx.x * kWarps + threadIdx.x / 32; task < tasks; task += (int64_t)gridDim.x * kWarps) {
    const int now = tensor_of(a, task, i < 0 ? 0 : i);
    if (now != i) {
      i = now;
      const int64_t taken = *a.step[i];
      const double t = (double)(taken + 1);
      // 1 - beta^t: one lane each
      const double rest = 1.0 - exp2(t * (lane == 0 ? h.log2_beta1 : h.log2_beta2));
      const float c = (float)(lane == 0 ? h.lr / rest : 1.0 / sqrt(rest));
      st.c1 = __shfl_sync(0xffffffffu, c, 0);
      st.c2 = __shfl_sync(0xffffffffu, c, 1);
      uint32_t k = mix((uint32_t)seed + 0x9e3779b9u);
      k = mix(k ^ (uint32_t)(seed >> 32));
      k = mix(k + (uint32_t)taken);
      st.key = mix(k ^ a.id[i]);
    }
    const int64_t base = (task - a.first[i]) * kNumbers;
    switch (a.flags[i] & (kParamBf16 | kGradBf16)) {
      case 0: update_typed<N, float, float>(a, i, base, h, st, factor); break;
      case kParamBf16: update_typed<N, __nv_bfloat16, float>(a, i, base, h, st, factor); break;
      case kGradBf16: update_typed<N, float, __nv_bfloat16>(a, i, base, h, st, factor); break;
      default: update_typed<N, __nv_bfloat16, __nv_bfloat16>(a, i, base, h, st, factor);
    }
  }
  // the last block to come here counts the step: every other one has read the counts
  __shared__ bool last;
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    last = atomicInc(&ws->step_ticket, gridDim.x - 1) == gridDim.x - 1;  // 0 again behind the last one
  }
  __syncthreads();
  if (last)
    for (int k = threadIdx.x; k < a.n; k += kThreads) *a.step[k] += 1;
}

// result = (norm of all gradients, min(1, max_norm / (norm + 1e-6))).  Squares and sums in 64 bits: a gradient of 10^20 is no
// infinity, and the order is fixed: a block's tasks, then the blocks.
template <int N>
__global__ void __launch_bounds__(kThreads)
    grad_norm_kernel(const __grid_constant__ Tensors<N> a, bool first, bool last_launch, float max_norm, Workspace* ws,
                     float* result) {
  const int lane = threadIdx.x & 31;
  const int64_t tasks = a.first[a.n];
  double sum = 0.0;
  int i = 0;
  for (int64_t task = (int64_t)blockIdx.x * kWarps + threadIdx.x / 32; task < tasks; task += (int64_t)gridDim.x * kWarps) {
    i = tensor_of(a, task, i);
    const int64_t base = (task - a.first[i]) * kNumbers;
    for (int64_t q = base + lane; q < base + kNumbers && q < a.count[i]; q += 32) {
      const double g = a.flags[i] & kGradBf16 ? (double)__bfloat162float(static_cast<const __nv_bfloat16*>(a.grad[i])[q])
                                              : (double)static_cast<const float*>(a.grad[i])[q];
      sum += g * g;
    }
  }
  __shared__ double sums[kWarps];
  __shared__ bool last;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) sums[threadIdx.x / 32] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    sum = first ? 0.0 : ws->partial[blockIdx.x];
    for (int w = 0; w < kWarps; ++w) sum += sums[w];
    ws->partial[blockIdx.x] = sum;
    __threadfence();
    last = atomicInc(&ws->norm_ticket, gridDim.x - 1) == gridDim.x - 1;
    __threadfence();
  }
  __syncthreads();
  if (!last || !last_launch) return;
  sum = 0.0;
  for (int b = threadIdx.x; b < kNormBlocks; b += kThreads) sum += b < (int)gridDim.x ? __ldcg(&ws->partial[b]) : 0.0;
  __syncthreads();
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) sums[threadIdx.x / 32] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    sum = 0.0;
    for (int w = 0; w < kWarps; ++w) sum += sums[w];
    const float norm = (float)sqrt(sum);
    result[0] = norm;
    const float factor = max_norm / (norm + 1e-6f);
    result[1] = factor > 1.f ? 1.f : factor;  // NaN stays NaN
  }
}

dg_status_t invalid(const char* msg) {
  set_error("%s", msg);
  return DG_ERR_INVALID_ARG;
}

bool aligned(const void* p, size_t to) { return (uintptr_t)p % to == 0; }

// The list's tensors from `at` on, as many as fit; returns their tasks.
template <int N>
int64_t fill(const dg_adamw_list_t& t, int64_t at, bool gradients_only, Tensors<N>* a) {
  int64_t tasks = 0;
  const int n = t.tensors - at < N ? (int)(t.tensors - at) : N;
  for (int k = 0; k < n; ++k) {
    const int64_t i = at + k;
    int flags = t.grad_type[i] == DG_BF16 ? kGradBf16 : 0;
    bool vectors = aligned(t.grad[i], t.grad_type[i] == DG_BF16 ? 8 : 16);
    a->grad[k] = t.grad[i];
    a->count[k] = t.numbers[i];
    a->first[k] = tasks;
    tasks += (t.numbers[i] + kNumbers - 1) / kNumbers;
    if (!gradients_only) {
      const bool bf16 = t.param_type[i] == DG_BF16, eight = t.state_bits[i] == 8;
      a->param[k] = t.param[i];
      a->m[k] = t.exp_avg[i];
      a->v[k] = t.exp_avg_sq[i];
      a->scales[k] = eight ? reinterpret_cast<float2*>(t.scales[i]) : nullptr;
      a->copy[k] = t.copy ? static_cast<__nv_bfloat16*>(t.copy[i]) : nullptr;
      a->step[k] = t.step[i];
      a->id[k] = t.id ? t.id[i] : (uint32_t)i;
      flags |= (bf16 ? kParamBf16 : 0) | (eight ? k8Bits : 0);
      const size_t state = eight ? 4 : 16;
      vectors = vectors && aligned(t.param[i], bf16 ? 8 : 16) && aligned(t.exp_avg[i], state) &&
                aligned(t.exp_avg_sq[i], state) && aligned(a->copy[k], 8);
    }
    a->flags[k] = (uint8_t)(flags | (vectors ? kVectors : 0));
  }
  a->first[n] = tasks;
  a->n = n;
  return tasks;
}

dg_status_t device_sms(int* sms) {
  int device = 0;
  DG_CUDA(cudaGetDevice(&device));
  DG_CUDA(cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, device));
  return DG_OK;
}

template <int N>
dg_status_t step_launch(const dg_adamw_list_t& t, int64_t at, const Hyper& h, const float* factor, uint64_t seed, Workspace* ws,
                        int sms, cudaStream_t s) {
  Tensors<N> a;
  const int64_t tasks = fill(t, at, false, &a);
  int64_t blocks = (tasks + kWarps - 1) / kWarps;
  if (blocks > sms * kBlocksPerSm) blocks = sms * kBlocksPerSm;
  if (blocks < 1) blocks = 1;  // tensors without numbers count their steps too
  DG_CUDA(launch_kernel(adamw_kernel<N>, dim3((unsigned)blocks), kThreads, s, true, a, h, factor, seed, ws));
  count_launches(1);
  return DG_OK;
}

template <int N>
dg_status_t norm_launch(const dg_adamw_list_t& t, int64_t at, float max_norm, Workspace* ws, float* result, cudaStream_t s) {
  Tensors<N> a;
  fill(t, at, true, &a);
  grad_norm_kernel<N><<<kNormBlocks, kThreads, 0, s>>>(a, at == 0, at + a.n == t.tensors, max_norm, ws, result);
  DG_CUDA(cudaGetLastError());
  count_launches(1);
  return DG_OK;
}

dg_status_t check_list(const dg_adamw_list_t* list, const void* ws, bool gradients_only) {
  if (!list) return invalid("list is NULL");
  const dg_adamw_list_t& t = *list;
  if (t.tensors < 0 || t.tensors > ((int64_t)1 << 31)) return invalid("the number of tensors must be from 0 to 2^31");
  if (!ws || !aligned(ws, 256)) return invalid("workspace is NULL or not 256-byte aligned");
  if (t.tensors == 0) return DG_OK;
  if (!t.numbers || !t.grad || !t.grad_type) return invalid("an array of the list is NULL");
  if (!gradients_only && (!t.param || !t.exp_avg || !t.exp_avg_sq || !t.step || !t.param_type || !t.state_bits))
    return invalid("an array of the list is NULL");
  for (int64_t i = 0; i < t.tensors; ++i) {
    const bool some = t.numbers[i] > 0;
    if (t.numbers[i] < 0 || t.numbers[i] > ((int64_t)1 << 40)) return invalid("a tensor must have from 0 to 2^40 numbers");
    if (t.grad_type[i] != DG_F32 && t.grad_type[i] != DG_BF16) return invalid("a type must be DG_F32 or DG_BF16");
    if (some && !t.grad[i]) return invalid("a tensor's grad is NULL");
    if (!aligned(t.grad[i], t.grad_type[i] == DG_F32 ? 4 : 2)) return invalid("a gradient must be aligned to its type");
    if (gradients_only) continue;
    if (t.param_type[i] != DG_F32 && t.param_type[i] != DG_BF16) return invalid("a type must be DG_F32 or DG_BF16");
    if (t.state_bits[i] != 8 && t.state_bits[i] != 32) return invalid("state_bits must be 8 or 32");
    if (!t.step[i] || !aligned(t.step[i], 8)) return invalid("a tensor's step is NULL or misaligned");
    const void* copy = t.copy ? t.copy[i] : nullptr;
    if (copy && t.param_type[i] != DG_F32) return invalid("a copy needs an fp32 param");
    const size_t state = t.state_bits[i] == 32 ? 4 : 1;
    if (!aligned(t.param[i], t.param_type[i] == DG_F32 ? 4 : 2) || !aligned(copy, 2) || !aligned(t.exp_avg[i], state) ||
        !aligned(t.exp_avg_sq[i], state))
      return invalid("a tensor must be aligned to its type");
    if (some && (!t.param[i] || !t.exp_avg[i] || !t.exp_avg_sq[i])) return invalid("a tensor's pointer is NULL");
    if (t.state_bits[i] == 32) continue;
    if (!t.scales || (some && !t.scales[i])) return invalid("8-bit states need scales");
    if (!aligned(t.scales[i], 8)) return invalid("scales must be 8-byte aligned");
  }
  return DG_OK;
}

}  // namespace
}  // namespace dg

using namespace dg;

extern "C" dg_status_t dg_grad_norm(const dg_adamw_list_t* list, float max_norm, void* workspace, float* result, void* stream) {
  if (dg_status_t st = check_list(list, workspace, true)) return st;
  if (!(max_norm >= 0.f)) return invalid("max_norm must not be negative");
  if (!result) return invalid("result is NULL");
  Workspace* ws = static_cast<Workspace*>(workspace);
  cudaStream_t s = (cudaStream_t)stream;
  if (list->tensors <= kFew) return norm_launch<kFew>(*list, 0, max_norm, ws, result, s);
  for (int64_t i = 0; i < list->tensors; i += kMost)
    if (dg_status_t st = norm_launch<kMost>(*list, i, max_norm, ws, result, s)) return st;
  return DG_OK;
}

extern "C" dg_status_t dg_adamw_step(const dg_adamw_list_t* list, double lr, double beta1, double beta2, double eps,
                                     double weight_decay, const float* grad_factor, uint64_t seed, void* workspace,
                                     void* stream) {
  if (dg_status_t st = check_list(list, workspace, false)) return st;
  if (!(beta1 >= 0.0 && beta1 < 1.0 && beta2 >= 0.0 && beta2 < 1.0)) return invalid("beta1 and beta2 must be in [0, 1)");
  if (!(lr >= 0.0 && lr < INFINITY) || !(eps >= 0.0 && eps < INFINITY) || !(weight_decay >= 0.0 && weight_decay < INFINITY))
    return invalid("lr, eps and weight_decay must be finite and not negative");
  if (list->tensors == 0) return DG_OK;
  const Hyper h{lr, log2(beta1), log2(beta2), (float)(1.0 - beta1), (float)beta2, (float)(1.0 - beta2), (float)eps,
                (float)(1.0 - lr * weight_decay)};
  int sms = 0;
  if (dg_status_t st = device_sms(&sms)) return st;
  Workspace* ws = static_cast<Workspace*>(workspace);
  cudaStream_t s = (cudaStream_t)stream;
  if (list->tensors <= kFew) return step_launch<kFew>(*list, 0, h, grad_factor, seed, ws, sms, s);
  for (int64_t i = 0; i < list->tensors; i += kMost)
    if (dg_status_t st = step_launch<kMost>(*list, i, h, grad_factor, seed, ws, sms, s)) return st;
  return DG_OK;
}
