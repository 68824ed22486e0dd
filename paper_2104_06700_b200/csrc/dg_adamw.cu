// AdamW over many tensors at once, its two states in 32 or in 8 bits, and the norm of all gradients.
//
//   g' = g factor,  m = m + (1 - b1)(g' - m),  v = b2 v + (1 - b2) g'^2,  t = steps taken + 1
//   p = p (1 - lr wd) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// A warp takes 256 numbers of a tensor, the block that shares a scale when the states are 8-bit: the largest |m| and
// sqrt(v) of the block are a warp's reduction away, and the new scales leave in the pass that reads the old ones.
#include <cuda_bf16.h>
#include <math.h>

#include <type_traits>

#include "dg_internal.cuh"
#include "dg_pairs.cuh"

namespace dg {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
// Blocks of an SM.  Numbers in 32 bits: two, whose 128 registers a thread hold a task's first block while the powers of beta
// are on their way (245 M numbers, clipped: 1205 us, three blocks 1396).  In 8 bits arithmetic counts, and more warps hide it:
// four at 64 registers, of which up to 19 are spilled (245 M numbers, launches with pauses between them: 686 us, three blocks 744;
// without pauses, at the clocks that leaves, 711 - 752).
constexpr int blocks_per_sm(bool eight) { return eight ? 4 : 2; }
constexpr int kNumbers = 256;                       // of a warp's task: 8 a lane, and one scale
// 256 numbers each, of a warp's task.  8-bit states: see step_kind (245 M numbers, with pauses: 686 us, 706 with four; 120 tensors of
// 37 M 136, 140).
constexpr int kBlocksPerTask = 4, kMostBlocks = 16;
constexpr int kNormNumbers = 2048;                  // of a warp's task of the norm
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
  int32_t numbers;       // of a task: a multiple of 256
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

// Four neighbouring numbers as they are stored; `left` of them exist.
template <typename T>
struct Quad {
  std::conditional_t<sizeof(T) == 4, float4, uint2> raw;
};
template <typename T, bool VEC>
__device__ __forceinline__ Quad<T> load4(const T* p, int left) {
  Quad<T> r;
  if constexpr (VEC) {
    r.raw = *reinterpret_cast<const decltype(r.raw)*>(p);
  } else if constexpr (sizeof(T) == 4) {
    r.raw = make_float4(left > 0 ? p[0] : 0.f, left > 1 ? p[1] : 0.f, left > 2 ? p[2] : 0.f, left > 3 ? p[3] : 0.f);
  } else {
    const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
    r.raw = make_uint2((left > 0 ? h[0] : 0u) | (left > 1 ? (uint32_t)h[1] << 16 : 0u),
                       (left > 2 ? h[2] : 0u) | (left > 3 ? (uint32_t)h[3] << 16 : 0u));
  }
  return r;
}
template <typename T>
__device__ __forceinline__ void numbers_of(const Quad<T>& q, float* out) {
  if constexpr (sizeof(T) == 4) {
    out[0] = q.raw.x, out[1] = q.raw.y, out[2] = q.raw.z, out[3] = q.raw.w;
  } else {
    out[0] = __uint_as_float(q.raw.x << 16), out[1] = __uint_as_float(q.raw.x & 0xffff0000u);
    out[2] = __uint_as_float(q.raw.y << 16), out[3] = __uint_as_float(q.raw.y & 0xffff0000u);
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
// the upper halves of four words
template <bool VEC>
__device__ __forceinline__ void store_upper4(uint16_t* p, int left, const uint32_t* in) {
  if constexpr (VEC) {
    *reinterpret_cast<uint2*>(p) = make_uint2(__byte_perm(in[0], in[1], 0x7632), __byte_perm(in[2], in[3], 0x7632));
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < left) p[j] = (uint16_t)(in[j] >> 16);
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

// What two e4m3 codes stand for.
__device__ __forceinline__ Two from_e4m3(uint32_t codes) {
  float a, b;
  asm("{ .reg .b16 c, lo, hi; .reg .b32 h; cvt.u16.u32 c, %2; cvt.rn.f16x2.e4m3x2 h, c; mov.b32 {lo, hi}, h;"
      " cvt.f32.f16 %0, lo; cvt.f32.f16 %1, hi; }"
      : "=f"(a), "=f"(b)
      : "r"(codes));
  return two(a, b);
}

// An 8-bit state is rounded up with a probability that is its distance from the lower neighbour: the averages move by a
// thousandth of themselves a step, far less than half a step of 3 bits, and rounding to nearest would hold them where they
// are.  `in_front`: the number times 2^-120, at most 448 of them up to a rounding: behind its sign and four zeros it has e4m3's
// bits, denormal ones too, and 20 behind them; adding 16 random bits (and half of the last) there carries into them.  The
// code's seven bits come out in front of byte 3, over what is left of the sum: the shift by four drops the sign.
__device__ __forceinline__ uint32_t to_e4m3(float in_front, uint32_t random_over_128) {
  return min((__float_as_uint(in_front) << 4) + random_over_128, 0x7effffffu);
}
// bytes 3 of four words
__device__ __forceinline__ uint32_t first_bytes(const uint32_t (&w)[4]) {
  return __byte_perm(__byte_perm(w[0], w[1], 0x0073), __byte_perm(w[2], w[3], 0x0073), 0x5410);
}

// 1 / v, off by at most 2^-23 of itself
__device__ __forceinline__ float fast_inverse(float v) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
// The largest magnitude, NaN if one is.
__device__ __forceinline__ float most_of(float a, float b, float c) {
  float r;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float warp_most(float v) {
  float r;
  asm("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}
// The largest of a warp's finite ones: a number that is not finite keeps to itself.
__device__ float warp_most_finite(const float (&v)[8]) {
  float m = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) m = fabsf(v[j]) < INFINITY ? fmaxf(m, fabsf(v[j])) : m;
  return warp_most(m);
}

struct Step {
  float c1, c2;   // lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
  uint32_t key;
};

template <typename P, bool VEC, int N>
__device__ __forceinline__ void store_param(const Tensors<N>& a, int i, int64_t q, int left, const float* p, const uint32_t* r) {
  uint32_t c[4];
  if constexpr (sizeof(P) == 4) {
    store4<VEC>(static_cast<float*>(a.param[i]) + q, left, p);
    if (a.copy[i]) {  // the master weights keep what the copy loses: to nearest
#pragma unroll
      for (int j = 0; j < 4; ++j) c[j] = __bfloat16_as_ushort(__float2bfloat16_rn(p[j]));
      store4<VEC>(reinterpret_cast<uint16_t*>(a.copy[i]) + q, left, c);
    }
  } else {
    // Rounded up or down by 16 random bits too: steps of a thousandth of a parameter would all be lost to nearest.
#pragma unroll
    for (int j = 0; j < 4; ++j) c[j] = __float_as_uint(p[j]) + (r[j] & 0xffffu);
    if (!(most_of(most_of(p[0], p[1], p[2]), p[3], 0.f) < INFINITY)) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (!(fabsf(p[j]) < INFINITY)) c[j] = (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(p[j])) << 16;
    }
    store_upper4<VEC>(static_cast<uint16_t*>(a.param[i]) + q, left, c);
  }
}

// The numbers base .. base + 255 of a tensor, as far as it goes, as they are stored.  A lane has four at 4 lane, four 128
// further.
template <typename P, typename G, bool EIGHT>
struct Block {
  Quad<P> p[2];
  Quad<G> g[2];
  std::conditional_t<EIGHT, uint32_t, Quad<float>> m[2], v[2];
  float2 scale;
};
__device__ __forceinline__ int left_of(int64_t q, int64_t end) { return (int)(end - q < 0 ? 0 : end - q < 4 ? end - q : 4); }

template <typename P, typename G, bool EIGHT, bool VEC, int N>
__device__ __forceinline__ Block<P, G, EIGHT> load_block(const Tensors<N>& a, int i, int64_t base) {
  Block<P, G, EIGHT> r;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int64_t q = base + 4 * (threadIdx.x & 31) + 128 * k;
    const int left = VEC ? 4 : left_of(q, a.count[i]);
    r.p[k] = load4<P, VEC>(static_cast<const P*>(a.param[i]) + q, left);
    r.g[k] = load4<G, VEC>(static_cast<const G*>(a.grad[i]) + q, left);
    if constexpr (EIGHT) {
      r.m[k] = load_bytes<VEC>(static_cast<const uint8_t*>(a.m[i]) + q, left);
      r.v[k] = load_bytes<VEC>(static_cast<const uint8_t*>(a.v[i]) + q, left);
    } else {
      r.m[k] = load4<float, VEC>(static_cast<const float*>(a.m[i]) + q, left);
      r.v[k] = load4<float, VEC>(static_cast<const float*>(a.v[i]) + q, left);
    }
  }
  if constexpr (EIGHT) r.scale = a.scales[i][base / kNumbers];
  return r;
}

template <typename P, typename G, bool EIGHT, bool VEC, int N>
__device__ __forceinline__ void update(const Tensors<N>& a, int i, int64_t base, const Block<P, G, EIGHT>& in, const Hyper& h,
                                       const Step& st, float factor) {
  const int lane = threadIdx.x & 31;
  const int64_t at = base + 4 * lane, end = a.count[i];
  const uint32_t key = mix(st.key ^ (uint32_t)(base >> 32));
  float p[8], g[8], m[8], v[8];   // EIGHT: v is sqrt(v)
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    numbers_of(in.p[k], p + 4 * k);
    numbers_of(in.g[k], g + 4 * k);
    if constexpr (!EIGHT) {
      numbers_of(in.m[k], m + 4 * k);
      numbers_of(in.v[k], v + 4 * k);
    }
  }
  if constexpr (EIGHT) {
    // Operation by operation as the formulas have them, each rounded to nearest and none fused: which way an 8-bit number
    // is rounded hangs on the last bit, a few numbers in a million go the other way when an operation is left out, and what
    // they were is the next step's scale.  Any fp32 arithmetic that follows the formulas gets these codes.
    const Two scale_m = both(in.scale.x), scale_u = both(in.scale.y), rest1 = both(h.rest1), rest2 = both(h.rest2);
    const Two beta2 = both(h.beta2), factors = both(factor);
    float most_m = 0.f, most_u = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const Two gj = two(g[2 * j], g[2 * j + 1]) * factors;
      const Two old = from_e4m3(in.m[j / 2] >> (16 * (j % 2))) * scale_m, root = from_e4m3(in.v[j / 2] >> (16 * (j % 2))) * scale_u;
      // The sums are single additions: ptxas makes one operation of a product and a sum of pairs.
      const float2 mo = apart(old), step = apart(rest1 * (gj - old)), kept = apart(beta2 * (root * root)), taken = apart(rest2 * gj * gj);
      const float2 mj = make_float2(__fadd_rn(mo.x, step.x), __fadd_rn(mo.y, step.y));
      const float2 vj = make_float2(__fadd_rn(kept.x, taken.x), __fadd_rn(kept.y, taken.y));
      v[2 * j] = __fsqrt_rn(vj.x), v[2 * j + 1] = __fsqrt_rn(vj.y);
      const float2 under = apart(fma2(two(v[2 * j], v[2 * j + 1]), both(st.c2), both(h.eps)));
      const Two ratio = two(mj.x, mj.y) * two(fast_inverse(under.x), fast_inverse(under.y));
      const float2 pj = apart(fma2(ratio, both(-st.c1), two(p[2 * j], p[2 * j + 1]) * both(h.decay)));
      p[2 * j] = pj.x, p[2 * j + 1] = pj.y;
      m[2 * j] = mj.x, m[2 * j + 1] = mj.y;
      most_m = most_of(most_m, mj.x, mj.y);
      most_u = most_of(most_u, v[2 * j], v[2 * j + 1]);
    }
    most_m = warp_most(most_m);
    most_u = warp_most(most_u);
    const bool careful = !(most_m < INFINITY && most_u < INFINITY);  // of the whole warp
    if (careful) {
      most_m = warp_most_finite(m);
      most_u = warp_most_finite(v);
    }
    const float2 scale = make_float2(fmaxf(__fmul_rn(most_m, 1.f / kLargest), kLeastScale),
                                     fmaxf(__fmul_rn(most_u, 1.f / kLargest), kLeastScale));
    if (lane == 0) a.scales[i][base / kNumbers] = scale;
    const Two inv_m = both(__frcp_rn(scale.x)), inv_u = both(__frcp_rn(scale.y)), front = both(0x1p-120f);
    float ym[8], yu[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 a2 = apart(two(m[2 * j], m[2 * j + 1]) * inv_m * front), b2 = apart(two(v[2 * j], v[2 * j + 1]) * inv_u * front);
      ym[2 * j] = a2.x, ym[2 * j + 1] = a2.y;
      yu[2 * j] = b2.x, yu[2 * j + 1] = b2.y;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int64_t q = at + 128 * k;
      const int left = VEC ? 4 : left_of(q, end);
      uint32_t r[4], cm[4], cu[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        r[j] = mix((uint32_t)(q + j) + key);
        cm[j] = to_e4m3(ym[4 * k + j], __byte_perm(r[j], 0x80u, 0x5104));
        cu[j] = to_e4m3(yu[4 * k + j], __byte_perm(r[j], 0x80u, 0x5324));
        // a denominator that was not 0 does not become 0 (a root that is not 0 is above 2^-75)
        cu[j] = max(cu[j], min(__float_as_uint(v[4 * k + j]), 0x01000000u));
      }
      if (careful) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (!(fabsf(m[4 * k + j]) < INFINITY)) cm[j] = 0x7f000000u;
          if (!(v[4 * k + j] < INFINITY)) cu[j] = 0x7f000000u;
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) cm[j] |= __float_as_uint(m[4 * k + j]) & 0x80000000u;
      store_param<P, VEC>(a, i, q, left, p + 4 * k, r);
      store_bytes<VEC>(static_cast<uint8_t*>(a.m[i]) + q, left, first_bytes(cm));
      store_bytes<VEC>(static_cast<uint8_t*>(a.v[i]) + q, left, first_bytes(cu));
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float gj = g[j] * factor;
      m[j] = fmaf(h.rest1, gj - m[j], m[j]);
      v[j] = fmaf(h.rest2 * gj, gj, h.beta2 * v[j]);
      p[j] = fmaf(p[j], h.decay, -st.c1 * (m[j] * fast_inverse(fmaf(sqrtf(v[j]), st.c2, h.eps))));
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int64_t q = at + 128 * k;
      const int left = VEC ? 4 : left_of(q, end);
      uint32_t r[4] = {};
      if (sizeof(P) == 2) {
#pragma unroll
        for (int j = 0; j < 4; ++j) r[j] = mix((uint32_t)(q + j) + key);
      }
      store_param<P, VEC>(a, i, q, left, p + 4 * k, r);
      store4<VEC>(static_cast<float*>(a.m[i]) + q, left, m + 4 * k);
      store4<VEC>(static_cast<float*>(a.v[i]) + q, left, v + 4 * k);
    }
  }
}

template <int N, typename P, typename G, bool EIGHT>
__global__ void __launch_bounds__(kThreads, blocks_per_sm(EIGHT))
    adamw_kernel(const __grid_constant__ Tensors<N> a, Hyper h, const float* factor_at, uint64_t seed, Workspace* ws) {
  const int lane = threadIdx.x & 31;
  cudaGridDependencySynchronize();
  const float factor = factor_at ? *factor_at : 1.f;
  const int64_t tasks = a.first[a.n];
  int i = -1;
  Step st{};
  for (int64_t task = (int64_t)blockIdx.x * kWarps + threadIdx.x / 32; task < tasks; task += (int64_t)gridDim.x * kWarps) {
    const int now = tensor_of(a, task, i < 0 ? 0 : i);
    int64_t base = (task - a.first[now]) * a.numbers;
    const int64_t left = a.count[now] - base, end = base + (left < a.numbers ? left : a.numbers);
    const bool vectors = a.flags[now] & kVectors && base + kNumbers <= end;
    Block<P, G, EIGHT> first;
    if (!EIGHT && vectors) first = load_block<P, G, EIGHT, true>(a, now, base);
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
    if (vectors) {
      if (!EIGHT) {
        update<P, G, EIGHT, true>(a, i, base, first, h, st, factor);
        base += kNumbers;
      }
#pragma unroll 1
      for (; base + kNumbers <= end; base += kNumbers)
        update<P, G, EIGHT, true>(a, i, base, load_block<P, G, EIGHT, true>(a, i, base), h, st, factor);
    }
#pragma unroll 1
    for (; base < end; base += kNumbers)
      update<P, G, EIGHT, false>(a, i, base, load_block<P, G, EIGHT, false>(a, i, base), h, st, factor);
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

// Adds the squares of `count` numbers to a lane's four sums.
template <typename T>
__device__ __forceinline__ void add_squares(const T* g, int count, bool vectors, int lane, double (&part)[4]) {
  constexpr int kLoads = 4;
  if (vectors && count == kNormNumbers) {
#pragma unroll 1
    for (int q = 4 * lane; q < kNormNumbers; q += 128 * kLoads) {
      float v[kLoads][4];
#pragma unroll
      for (int u = 0; u < kLoads; ++u) numbers_of(load4<T, true>(g + q + 128 * u, 4), v[u]);
#pragma unroll
      for (int u = 0; u < kLoads; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j) part[j] = fma((double)v[u][j], (double)v[u][j], part[j]);
    }
    return;
  }
  for (int q = 4 * lane; q < count; q += 128) {
    float v[4];
    numbers_of(load4<T, false>(g + q, count - q), v);
#pragma unroll
    for (int j = 0; j < 4; ++j) part[j] = fma((double)v[j], (double)v[j], part[j]);
  }
}

// result = (norm of all gradients, min(1, max_norm / (norm + 1e-6))).  Squares and sums in 64 bits: a gradient of 10^20 is no
// infinity, and the order is fixed: a block's tasks, then the blocks.
template <int N>
__global__ void __launch_bounds__(kThreads)
    grad_norm_kernel(const __grid_constant__ Tensors<N> a, bool first, bool last_launch, float max_norm, Workspace* ws,
                     float* result) {
  const int lane = threadIdx.x & 31;
  const int64_t tasks = a.first[a.n];
  double part[4] = {};
  int i = 0;
  for (int64_t task = (int64_t)blockIdx.x * kWarps + threadIdx.x / 32; task < tasks; task += (int64_t)gridDim.x * kWarps) {
    i = tensor_of(a, task, i);
    const int64_t base = (task - a.first[i]) * kNormNumbers;
    const int64_t count = a.count[i] - base < kNormNumbers ? a.count[i] - base : kNormNumbers;
    if (a.flags[i] & kGradBf16)
      add_squares(static_cast<const __nv_bfloat16*>(a.grad[i]) + base, (int)count, a.flags[i] & kVectors, lane, part);
    else
      add_squares(static_cast<const float*>(a.grad[i]) + base, (int)count, a.flags[i] & kVectors, lane, part);
  }
  double sum = (part[0] + part[1]) + (part[2] + part[3]);
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

// Which kernel takes a tensor; the norm's takes all gradients.
int kind_of(const dg_adamw_list_t& t, int64_t i) {
  return (t.param_type[i] == DG_BF16 ? kParamBf16 : 0) | (t.grad_type[i] == DG_BF16 ? kGradBf16 : 0) | (t.state_bits[i] == 8 ? k8Bits : 0);
}

// The list's tensors from *at on, of one kind (-1: gradients alone, of any), as many as fit; *at goes behind them.  Returns
// their tasks of `each` numbers.
template <int N>
int64_t fill(const dg_adamw_list_t& t, int64_t* at, int kind, int32_t each, Tensors<N>* a) {
  int64_t tasks = 0;
  int k = 0;
  for (; *at < t.tensors && k < N; ++*at) {
    const int64_t i = *at;
    if (kind >= 0 && kind_of(t, i) != kind) continue;
    bool vectors = aligned(t.grad[i], t.grad_type[i] == DG_BF16 ? 8 : 16);
    a->grad[k] = t.grad[i];
    a->count[k] = t.numbers[i];
    a->first[k] = tasks;
    tasks += (t.numbers[i] + each - 1) / each;
    if (kind >= 0) {
      a->param[k] = t.param[i];
      a->m[k] = t.exp_avg[i];
      a->v[k] = t.exp_avg_sq[i];
      a->scales[k] = kind & k8Bits ? reinterpret_cast<float2*>(t.scales[i]) : nullptr;
      a->copy[k] = t.copy ? static_cast<__nv_bfloat16*>(t.copy[i]) : nullptr;
      a->step[k] = t.step[i];
      a->id[k] = t.id ? t.id[i] : (uint32_t)i;
      const size_t state = kind & k8Bits ? 4 : 16;
      vectors = vectors && aligned(t.param[i], kind & kParamBf16 ? 8 : 16) && aligned(t.exp_avg[i], state) &&
                aligned(t.exp_avg_sq[i], state) && aligned(a->copy[k], 8);
    }
    a->flags[k] = (uint8_t)((t.grad_type[i] == DG_BF16 ? kGradBf16 : 0) | (vectors ? kVectors : 0));
    ++k;
  }
  a->first[k] = tasks;
  a->numbers = each;
  a->n = k;
  return tasks;
}

dg_status_t device_sms(int* sms) {
  int device = 0;
  DG_CUDA(cudaGetDevice(&device));
  DG_CUDA(cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, device));
  return DG_OK;
}

struct StepCall {
  Hyper h;
  const float* factor;
  uint64_t seed;
  Workspace* ws;
  int sms;
  cudaStream_t s;
};

template <int N, typename P, typename G, bool EIGHT>
dg_status_t step_kind(const dg_adamw_list_t& t, int kind, const StepCall& c) {
  for (int64_t at = 0; at < t.tensors;) {
    Tensors<N> a;
    const int64_t from = at;
    int64_t tasks = fill(t, &at, kind, kNumbers, &a);
    if (a.n == 0) break;
    const int64_t warps = (int64_t)c.sms * blocks_per_sm(EIGHT) * kWarps;
    // Long tasks where every warp has some: what a warp finds out about its tensor serves more numbers.
    if (EIGHT && tasks > warps) {
      // of so many blocks that a few whole rounds of the warps take them all; a tensor's last task is half empty on average
      const int64_t rounds = (tasks + warps * kMostBlocks - 1) / (warps * kMostBlocks), half_empty = a.n / 2;
      const int64_t places = warps * rounds > 2 * half_empty ? warps * rounds - half_empty : half_empty + 1;
      const int64_t each = (tasks + places - 1) / places;
      tasks = fill(t, &(at = from), kind, kNumbers * (int32_t)each, &a);
    } else if (!EIGHT && tasks > warps * 2 * kBlocksPerTask) {
      tasks = fill(t, &(at = from), kind, kNumbers * kBlocksPerTask, &a);
    }
    int64_t blocks = (tasks + kWarps - 1) / kWarps;
    if (blocks > c.sms * blocks_per_sm(EIGHT)) blocks = c.sms * blocks_per_sm(EIGHT);
    if (blocks < 1) blocks = 1;  // tensors without numbers count their steps too
    DG_CUDA(launch_kernel(adamw_kernel<N, P, G, EIGHT>, dim3((unsigned)blocks), kThreads, c.s, true, a, c.h, c.factor, c.seed, c.ws));
    count_launches(1);
  }
  return DG_OK;
}

// One launch for each kind of tensor in the list: a kernel for all kinds keeps the registers of the dearest for every one.
template <int N>
dg_status_t step_all(const dg_adamw_list_t& t, const StepCall& c) {
  int kinds = 0;
  for (int64_t i = 0; i < t.tensors; ++i) kinds |= 1 << kind_of(t, i);
  for (int kind = 0; kind < 8; ++kind) {
    if (!(kinds >> kind & 1)) continue;
    auto typed = [&](auto p, auto g) {
      using P = decltype(p);
      using G = decltype(g);
      return kind & k8Bits ? step_kind<N, P, G, true>(t, kind, c) : step_kind<N, P, G, false>(t, kind, c);
    };
    const bool gb = kind & kGradBf16;
    const dg_status_t st = kind & kParamBf16 ? (gb ? typed(__nv_bfloat16(), __nv_bfloat16()) : typed(__nv_bfloat16(), 0.f))
                                             : (gb ? typed(0.f, __nv_bfloat16()) : typed(0.f, 0.f));
    if (st != DG_OK) return st;
  }
  return DG_OK;
}

template <int N>
dg_status_t norm_launch(const dg_adamw_list_t& t, int64_t* at, float max_norm, Workspace* ws, float* result, cudaStream_t s) {
  Tensors<N> a;
  const bool first = *at == 0;
  const int64_t tasks = fill(t, at, -1, kNormNumbers, &a);
  int64_t blocks = (tasks + kWarps - 1) / kWarps;
  if (blocks > kNormBlocks || t.tensors > N) blocks = kNormBlocks;  // the launches of one list add to the same sums
  if (blocks < 1) blocks = 1;
  grad_norm_kernel<N><<<(unsigned)blocks, kThreads, 0, s>>>(a, first, *at == t.tensors, max_norm, ws, result);
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
  if (!result || !aligned(result, 4)) return invalid("result is NULL or misaligned");
  Workspace* ws = static_cast<Workspace*>(workspace);
  cudaStream_t s = (cudaStream_t)stream;
  int64_t at = 0;
  if (list->tensors <= kFew) return norm_launch<kFew>(*list, &at, max_norm, ws, result, s);
  while (at < list->tensors)
    if (dg_status_t st = norm_launch<kMost>(*list, &at, max_norm, ws, result, s)) return st;
  return DG_OK;
}

extern "C" dg_status_t dg_adamw_step(const dg_adamw_list_t* list, double lr, double beta1, double beta2, double eps,
                                     double weight_decay, const float* grad_factor, uint64_t seed, void* workspace,
                                     void* stream) {
  if (dg_status_t st = check_list(list, workspace, false)) return st;
  if (!(beta1 >= 0.0 && beta1 < 1.0 && beta2 >= 0.0 && beta2 < 1.0)) return invalid("beta1 and beta2 must be in [0, 1)");
  if (!(lr >= 0.0 && lr < INFINITY) || !(eps >= 0.0 && eps < INFINITY) || !(weight_decay >= 0.0 && weight_decay < INFINITY))
    return invalid("lr, eps and weight_decay must be finite and not negative");
  if (!aligned(grad_factor, 4)) return invalid("grad_factor must be aligned to its type");
  if (list->tensors == 0) return DG_OK;
  // an eps below the least normal number is that: its inverse has to be finite
  const float least = eps > 0.0 && eps < (double)kLeastScale ? kLeastScale : (float)eps;
  const Hyper h{lr, log2(beta1), log2(beta2), (float)(1.0 - beta1), (float)beta2, (float)(1.0 - beta2), least,
                (float)(1.0 - lr * weight_decay)};
  int sms = 0;
  if (dg_status_t st = device_sms(&sms)) return st;
  const StepCall c{h, grad_factor, seed, static_cast<Workspace*>(workspace), sms, (cudaStream_t)stream};
  return list->tensors <= kFew ? step_all<kFew>(*list, c) : step_all<kMost>(*list, c);
}
