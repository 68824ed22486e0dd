// Group norm with an activation, shared by its kernels (not part of the ABI).
//
// A group is the channels [c, c + F / groups) of the rows of one graph of the batch; N cells.
//   mean = sum x / N,  var = sum (x - mean)^2 / N,  rstd = 1 / sqrt(var + eps)
//   hat = (x - mean) rstd,  z = hat w + b,  y = act(z)
//   dz = dy act'(z),  db = sum dz,  dw = sum dz hat  (over all rows),
//   dx = rstd (dz w - A - hat B),  A = sum(dz w) / N,  B = sum(dz w hat) / N
#pragma once

#include <cuda_bf16.h>

#include <type_traits>

#include "dg_internal.cuh"
#include "dg_pairs.cuh"

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

// 1 / (1 + exp(-z)), of hardware's 2^x and 1 / x: off by 2 + |1.5 z| units of 2^-23.  A cell costs 4 to 12 bytes of memory
// traffic, and the exact functions cost as much time.  *t: exp(-z).
__device__ __forceinline__ float sigmoid(float z, float* t) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(*t) : "f"(z * -1.4426950408889634f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + *t));
  return r;
}
// z, or -43 below that: SiLU and its derivative are under 10^-17 there, and the product of two 1 + exp(-z) is finite.  NaN stays.
__device__ __forceinline__ float above_floor(float z) {
  asm("max.NaN.f32 %0, %0, %1;" : "+f"(z) : "f"(-43.f));
  return z;
}
__device__ __forceinline__ Two above_floor(Two z) {
  const float2 q = apart(z);
  return two(above_floor(q.x), above_floor(q.y));
}

template <int ACT>
__device__ __forceinline__ float activated(float z) {
  if constexpr (ACT == DG_ACT_RELU) return z <= 0.f ? 0.f : z;  // NaN stays NaN
  if constexpr (ACT == DG_ACT_SILU) {
    float t;
    z = above_floor(z);
    return z * sigmoid(z, &t);
  }
  return z;
}
// Of a pair of numbers not below -43, with one reciprocal for both, that of the product: hardware's
// functions bound these kernels (2048 graphs of 1 to 2500 rows of 128, SiLU, backward: 52 us, 58 with two reciprocals; 2.4 M x 100
// bf16 forward 293 and 295, backward 566 and 584).  The pair may lie in two
// groups: NaN is taken for -43 here, so that it does not reach the other one through the product.  The caller's z is NaN still.
__device__ __forceinline__ Two sigmoid(Two z, Two* t) {
  const float2 q = apart(z * both(-1.4426950408889634f));
  float2 e;
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.x) : "f"(fminf(q.x, 63.f)));  // at most 62.04, or NaN
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.y) : "f"(fminf(q.y, 63.f)));
  *t = two(e.x, e.y);
  e = apart(*t + both(1.f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(e.x * e.y));
  return both(r) * two(e.y, e.x);
}

// dy act'(z).  SiLU' = s (1 + z (1 - s)), where 1 - s is t s with t = exp(-z): a difference would keep s's rounding, which a large z
// multiplies (z = 10^6 beside a moderate one: 6 % off).  The ReLU's border is where z changes its sign: near it (|hat w| is about |b| there and z is off by up to
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
  const float q = above_floor(z);
  float t;
  const float s = sigmoid(q, &t);
  return dy * (s * fmaf(q, t * s, 1.f));
}

// ---- rows in pieces: the kernels of long graphs ------------------------------------------------------------------

// A run of rows of one graph, for one block (and one tile of channels).
struct Piece {
  int32_t graph, row, rows, pad;
};

// How a matrix is shared out.  Threads lie along the vectors of a tile of channels first (`across`), then along the rows
// (`down`); a thread keeps to its channels.
struct NormShape {
  int32_t vec;       // channels of a vector
  int32_t across, down, tiles;
  int32_t rows;      // of a piece where one graph has all rows
  int32_t pieces;
  int32_t kept;      // of a thread's rows, the last ones: what the L2 still holds of the first pass in the second
};

constexpr int kNormThreads = 256;

// VEC neighbouring numbers as fp32.
template <int VEC>
struct Channels {
  float v[VEC];
};
// ONCE: the L2 need not keep them.
template <typename T, int VEC, bool ONCE>
__device__ __forceinline__ Channels<VEC> load_channels(const T* p) {
  auto get = [](const auto* q) {
    if constexpr (ONCE) return __ldcs(q);
    else return *q;
  };
  Channels<VEC> r;
  if constexpr (sizeof(T) == 4 && VEC == 4) {
    const float4 q = get(reinterpret_cast<const float4*>(p));
    r.v[0] = q.x, r.v[1] = q.y, r.v[2] = q.z, r.v[3] = q.w;
  } else if constexpr (sizeof(T) == 4 && VEC == 2) {
    const float2 q = get(reinterpret_cast<const float2*>(p));
    r.v[0] = q.x, r.v[1] = q.y;
  } else if constexpr (sizeof(T) == 2 && VEC >= 2) {
    uint32_t w[VEC / 2];
    if constexpr (VEC == 8) {
      const uint4 q = get(reinterpret_cast<const uint4*>(p));
      w[0] = q.x, w[1] = q.y, w[2] = q.z, w[3] = q.w;
    } else if constexpr (VEC == 4) {
      const uint2 q = get(reinterpret_cast<const uint2*>(p));
      w[0] = q.x, w[1] = q.y;
    } else {
      w[0] = get(reinterpret_cast<const uint32_t*>(p));
    }
#pragma unroll
    for (int i = 0; i < VEC / 2; ++i) {
      r.v[2 * i] = __uint_as_float(w[i] << 16);
      r.v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  } else {
    static_assert(VEC == 1, "one number");
    if constexpr (sizeof(T) == 4)
      r.v[0] = get(p);
    else
      r.v[0] = __uint_as_float((uint32_t)get(reinterpret_cast<const unsigned short*>(p)) << 16);
  }
  return r;
}
template <typename T, int VEC>
__device__ __forceinline__ void store_channels(T* p, const Channels<VEC>& r) {
  if constexpr (sizeof(T) == 4 && VEC == 4) {
    __stcs(reinterpret_cast<float4*>(p), make_float4(r.v[0], r.v[1], r.v[2], r.v[3]));
  } else if constexpr (sizeof(T) == 4 && VEC == 2) {
    __stcs(reinterpret_cast<float2*>(p), make_float2(r.v[0], r.v[1]));
  } else if constexpr (sizeof(T) == 2 && VEC >= 2) {
    uint32_t w[VEC / 2];
#pragma unroll
    for (int i = 0; i < VEC / 2; ++i) {
      const __nv_bfloat162 pair = __floats2bfloat162_rn(r.v[2 * i], r.v[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&pair);
    }
    if constexpr (VEC == 8)
      __stcs(reinterpret_cast<uint4*>(p), make_uint4(w[0], w[1], w[2], w[3]));
    else if constexpr (VEC == 4)
      __stcs(reinterpret_cast<uint2*>(p), make_uint2(w[0], w[1]));
    else
      __stcs(reinterpret_cast<unsigned int*>(p), w[0]);
  } else {
    static_assert(VEC == 1, "one number");
    *p = as<T>(r.v[0]);
  }
}

// What a kernel may have without asking the runtime for more (a microsecond of host time a call): 48 KiB, of which the
// arrays beside the places take no more than 11.
constexpr size_t kMostPlaces = (48 - 11) << 10;

// VEC numbers as they are stored, from shared memory.
template <typename T, int VEC>
struct RawChannels {
  std::conditional_t<sizeof(T) * VEC == 16, uint4,
                     std::conditional_t<sizeof(T) * VEC == 8, uint2, std::conditional_t<sizeof(T) * VEC == 4, uint32_t, uint16_t>>> v;
};
template <typename T, int VEC>
__device__ __forceinline__ Channels<VEC> numbers_of(const RawChannels<T, VEC>& q) {
  uint32_t w[4] = {};
  if constexpr (sizeof(T) * VEC == 16)
    w[0] = q.v.x, w[1] = q.v.y, w[2] = q.v.z, w[3] = q.v.w;
  else if constexpr (sizeof(T) * VEC == 8)
    w[0] = q.v.x, w[1] = q.v.y;
  else
    w[0] = q.v;
  Channels<VEC> r;
#pragma unroll
  for (int c = 0; c < VEC; ++c) {
    if constexpr (sizeof(T) == 4)
      r.v[c] = __uint_as_float(w[c]);
    else
      r.v[c] = __uint_as_float(c % 2 ? w[c / 2] & 0xffff0000u : w[c / 2] << 16);
  }
  return r;
}
// Copies a vector into the thread's own place in shared memory, behind its back where the hardware copies that many bytes.
template <typename T, int VEC>
__device__ __forceinline__ void fetch(RawChannels<T, VEC>* to, const T* from) {
  constexpr int kBytes = sizeof(T) * VEC;
  if constexpr (kBytes >= 4) {
    const uint32_t at = (uint32_t)__cvta_generic_to_shared(to);
    if constexpr (kBytes == 16)
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at), "l"(from) : "memory");
    else
      asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(at), "l"(from), "n"(kBytes) : "memory");
  } else {
    to->v = *reinterpret_cast<const uint16_t*>(from);
  }
}
__device__ __forceinline__ void fetch_group() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// All but the latest PENDING groups have arrived.
template <int PENDING>
__device__ __forceinline__ void fetched() {
  asm volatile("cp.async.wait_group %0;" ::"n"(PENDING) : "memory");
}

// A thread's rows, in groups of STEP, through a ring of RING groups of places in shared memory.  `fetch_rows(group, place)` begins
// the copies of a group (of those of its rows that exist), `use(group, place)` takes it from there; the places of a group are
// filled again when it has been used.  Forward: the last groups stay where they are.  Back: those first, then the others.
template <int RING, typename Fetch, typename Use>
__device__ __forceinline__ void ring_forward(int32_t groups, Fetch fetch_rows, Use use) {
#pragma unroll
  for (int q = 0; q < RING; ++q) {
    if (q < groups) fetch_rows(q, q);
    fetch_group();
  }
  int place = 0;
#pragma unroll 1
  for (int32_t q = 0; q < groups; ++q) {
    fetched<RING - 1>();
    use(q, place);
    if (q + RING < groups) fetch_rows(q + RING, place);
    fetch_group();
    place = place + 1 == RING ? 0 : place + 1;
  }
}
template <int RING, typename Fetch, typename Use>
__device__ __forceinline__ void ring_back(int32_t groups, Fetch fetch_rows, Use use) {
  int place = (groups - 1) % RING;  // of the last group
#pragma unroll 1
  for (int32_t q = groups - 1; q >= 0; --q) {
    fetched<RING - 1>();  // the last RING groups arrived long ago
    use(q, place);
    if (q >= RING) fetch_rows(q - RING, place);
    fetch_group();
    place = place == 0 ? RING - 1 : place - 1;
  }
}

// A thread's channels: what does not change along its rows, in pairs (of one channel twice where it has one).
template <int VEC>
constexpr int kPairs = (VEC + 1) / 2;
template <int VEC>
struct Fixed {
  Two mean[kPairs<VEC>], rstd[kPairs<VEC>], w[kPairs<VEC>], b[kPairs<VEC>];
};
template <int VEC>
__device__ __forceinline__ Two pair_of(const Channels<VEC>& v, int k) {
  return two(v.v[2 * k], v.v[VEC == 1 ? 0 : 2 * k + 1]);
}
template <int VEC>
__device__ __forceinline__ void set_pair(Channels<VEC>& v, int k, Two p) {
  const float2 q = apart(p);
  v.v[2 * k] = q.x;
  if constexpr (VEC > 1) v.v[2 * k + 1] = q.y;
}
template <int VEC>
__device__ __forceinline__ void fix_weights(Fixed<VEC>& f, const NormArgs& a, int32_t channel) {
  Channels<VEC> w, b;
#pragma unroll
  for (int c = 0; c < VEC; ++c) {
    w.v[c] = a.weight ? a.weight[channel + c] : 1.f;
    b.v[c] = a.bias ? a.bias[channel + c] : 0.f;
  }
#pragma unroll
  for (int k = 0; k < kPairs<VEC>; ++k) f.w[k] = pair_of(w, k), f.b[k] = pair_of(b, k);
}
// stats(c): (mean, rstd) of the vector's channel c
template <int VEC, typename Stats>
__device__ __forceinline__ void fix_stats(Fixed<VEC>& f, Stats stats) {
  Channels<VEC> mean, rstd;
#pragma unroll
  for (int c = 0; c < VEC; ++c) {
    const float2 st = stats(c);
    mean.v[c] = st.x, rstd.v[c] = st.y;
  }
#pragma unroll
  for (int k = 0; k < kPairs<VEC>; ++k) f.mean[k] = pair_of(mean, k), f.rstd[k] = pair_of(rstd, k);
}
template <int VEC>
__device__ __forceinline__ Fixed<VEC> fixed_of(const NormArgs& a, int32_t graph, int32_t channel) {
  Fixed<VEC> f;
  fix_weights<VEC>(f, a, channel);
  fix_stats<VEC>(f, [&](int c) { return a.stats[(int64_t)graph * a.groups + (channel + c) / a.width]; });
  return f;
}
// act(hat w + b)
template <int ACT, int VEC>
__device__ __forceinline__ void normalise(Channels<VEC>& v, const Fixed<VEC>& f) {
#pragma unroll
  for (int k = 0; k < kPairs<VEC>; ++k) {
    Two z = fma2((pair_of(v, k) - f.mean[k]) * f.rstd[k], f.w[k], f.b[k]);
    if constexpr (ACT == DG_ACT_SILU) {
      z = above_floor(z);
      Two t;
      z = z * sigmoid(z, &t);
    }
    if constexpr (ACT == DG_ACT_RELU) {
      const float2 q = apart(z);
      z = two(activated<ACT>(q.x), activated<ACT>(q.y));
    }
    set_pair(v, k, z);
  }
}
// Of a pair of cells: hat, and d = dy act'(z).
template <int ACT, int VEC>
__device__ __forceinline__ void backward_terms(Two x, Two dy, const Fixed<VEC>& f, int k, Two* hat, Two* d) {
  const Two off = x - f.mean[k];
  *hat = off * f.rstd[k];
  if constexpr (ACT == DG_ACT_NONE) {
    *d = dy;
  } else {
    Two z = fma2(*hat, f.w[k], f.b[k]);
    if constexpr (ACT == DG_ACT_SILU) {
      z = above_floor(z);
      Two t;
      const Two s = sigmoid(z, &t);
      *d = dy * (s * fma2(z, t * s, both(1.f)));
    } else {
      const float2 zs = apart(z), ds = apart(dy), bs = apart(f.b[k]);
      float2 r = make_float2(zs.x <= 0.f ? 0.f : ds.x, zs.y <= 0.f ? 0.f : ds.y);
      if (!(fabsf(zs.x) >= fabsf(bs.x) * 0x1p-20f) || !(fabsf(zs.y) >= fabsf(bs.y) * 0x1p-20f)) {
        const float2 xs = apart(x), m = apart(f.mean[k]), q = apart(f.rstd[k]), w = apart(f.w[k]);
        r.x = before_activation<ACT>(ds.x, xs.x, m.x, q.x, w.x, bs.x);
        r.y = before_activation<ACT>(ds.y, xs.y, m.y, q.y, w.y, bs.y);
      }
      *d = two(r.x, r.y);
    }
  }
}

// Where a thread works: its piece, its first channel, its place along the rows.
struct Place {
  Piece piece;
  int32_t channel;   // >= F: none
  int32_t y, down;
};
__device__ __forceinline__ Place place_of(const NormArgs& a, const NormShape& sh, const Piece* pieces, int32_t p) {
  Place r;
  if (pieces) {
    r.piece = pieces[p];
  } else {
    const int64_t row = (int64_t)p * sh.rows, left = a.rows - row;
    r.piece = Piece{0, (int32_t)row, (int32_t)(left < sh.rows ? left : sh.rows), 0};
  }
  r.y = threadIdx.x / sh.across;
  r.down = sh.down;
  const int32_t vector = blockIdx.y * sh.across + threadIdx.x % sh.across;
  r.channel = r.y < sh.down && vector < a.F / sh.vec ? vector * sh.vec : a.F;
  return r;
}

// How a call's matrices are shared out among blocks.
NormShape norm_shape(const Graph* g, const NormArgs& a, int vec, int cell_bytes, int blocks_per_sm);
// The widest vectors that rows of F numbers and these pointers allow.
int norm_vector(const NormArgs& a, dg_type_t x, dg_type_t y);

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
// f(VEC): 8 for two bf16 matrices alone
template <bool WIDE, typename Fn>
auto by_vector(int vec, Fn f) {
  if constexpr (WIDE)
    if (vec == 8) return f(std::integral_constant<int, 8>());
  if (vec == 4) return f(std::integral_constant<int, 4>());
  if (vec == 2) return f(std::integral_constant<int, 2>());
  return f(std::integral_constant<int, 1>());
}

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// The sums of a and b over a block of at most 1024 threads, in every thread and always in the same order.
__device__ __forceinline__ double2 block_sums(double a, double b) {
  __shared__ double2 sums[32];
  a = warp_sum(a);
  b = warp_sum(b);
  __syncthreads();  // the last call's sums have been read
  if (threadIdx.x % 32 == 0) sums[threadIdx.x / 32] = make_double2(a, b);
  __syncthreads();
  const double2 part = threadIdx.x % 32 < blockDim.x / 32 ? sums[threadIdx.x % 32] : make_double2(0.0, 0.0);
  return make_double2(warp_sum(part.x), warp_sum(part.y));
}
__device__ __forceinline__ double block_sum(double v) { return block_sums(v, 0.0).x; }

// ---- a cluster of blocks for a graph and a tile of channels: short graphs -------------------------------------------

// A cluster of blocks takes the rows of one graph in the channels of a tile, which holds whole groups: what it sums it
// needs nowhere else.  Every thread fetches its rows into places of its own in shared memory, all at once, and rows that fit
// there are read once.
constexpr int kClusterLog = 3;
// Of a block: with as few as 16 rows for a thread what a thread costs beside them counts (2048 graphs of 1 to 2500 rows of
// 128, forward, when it was chosen: 41 us with 256 threads, 38 with 128).
constexpr int kGraphThreads = 128;
constexpr int kTileGroups = 128;  // most groups of a tile
struct GraphShape {
  int32_t vec, across, down, tiles;
  uint32_t by_across;    // thread / across = thread * by_across >> 16
  int32_t lanes_log;     // log2 of the threads along a group's units, at most 5
  int32_t team_log;      // log2 of the threads of a group while a block's sums are joined, at most 5
};
// One launch: long graphs in narrow tiles first, then the others in wide ones; or, where the graphs are few, all of them in
// narrow ones by clusters.
struct GraphPlan {
  GraphShape shape[2];     // of long graphs, of the others
  const Piece* order;      // whole graphs, longest first; null: one graph
  int64_t blocks;          // 0: not a call for these kernels
  int32_t long_blocks, long_graphs;
  int32_t cluster_log;     // log2 of the blocks of a cluster
  float by_width;          // 1 / width: groups of a tile's channels
};
GraphPlan graph_plan(const Graph* g, const NormArgs& a, int vec, int x_bytes, int rows_kept, bool shared);

struct GraphPlace {
  int32_t graph, rank;
  int32_t channel, tile_channels;  // the thread's first channel (>= F: none), those of the tile
  int32_t tile_first;
  int32_t x, y;                    // its place in the block: along the tile's vectors, along the rows
  int32_t row, step;               // its first row of the graph, and the distance to its next
  int32_t rows;
  int64_t base;                    // of that row's first channel, in numbers
};
__device__ __forceinline__ GraphPlace graph_place(const NormArgs& a, const GraphPlan& plan, const GraphShape& sh, bool is_long) {
  GraphPlace r;
  const uint32_t item = (is_long ? blockIdx.x : blockIdx.x - plan.long_blocks) >> plan.cluster_log;
  r.rank = blockIdx.x & ((1 << plan.cluster_log) - 1);
  const int32_t at = item / (uint32_t)sh.tiles, tile = item - at * sh.tiles;
  Piece whole{0, 0, (int32_t)a.rows, 0};
  if (plan.order) whole = plan.order[is_long ? at : at + plan.long_graphs];
  r.graph = whole.graph;
  r.rows = whole.rows;
  r.tile_first = tile * sh.across * sh.vec;
  r.tile_channels = min(sh.across * sh.vec, a.F - r.tile_first);
  r.y = threadIdx.x * sh.by_across >> 16;
  r.x = threadIdx.x - r.y * sh.across;
  r.channel = r.y < sh.down && r.x * sh.vec < r.tile_channels ? r.tile_first + r.x * sh.vec : a.F;
  r.row = r.rank * sh.down + r.y;
  r.step = sh.down << plan.cluster_log;
  r.base = ((int64_t)whole.row + r.row) * a.F + r.channel;
  return r;
}
// The group of a channel of the tile: at most 2048 channels, so that the product is off by less than 1 / (2 width).
__device__ __forceinline__ int32_t group_of(const GraphPlan& plan, int32_t channel) {
  return (int32_t)((channel + 0.5f) * plan.by_width);
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// The pair of numbers at the same place in another block's shared memory.
__device__ __forceinline__ float2 of_rank(const float2* p, int32_t rank) {
  const uint32_t mine = (uint32_t)__cvta_generic_to_shared(p);
  uint32_t there;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(mine), "r"(rank));
  float2 r;
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(r.x), "=f"(r.y) : "r"(there));
  return r;
}
__device__ __forceinline__ float warp_total(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
template <typename... P, typename... A>
cudaError_t launch_graphs(const GraphPlan& plan, void (*kernel)(NormArgs, GraphPlan, P...), size_t shared, cudaStream_t s,
                          const NormArgs& a, const A&... args) {
  cudaLaunchAttribute attribute{};
  attribute.id = cudaLaunchAttributeClusterDimension;
  attribute.val.clusterDim.x = 1u << plan.cluster_log;
  attribute.val.clusterDim.y = attribute.val.clusterDim.z = 1;
  cudaLaunchConfig_t config{};
  config.gridDim = dim3((unsigned)plan.blocks);
  config.blockDim = dim3(kGraphThreads);
  config.dynamicSmemBytes = shared;
  config.stream = s;
  config.attrs = &attribute;
  config.numAttrs = plan.cluster_log > 0 ? 1 : 0;
  return cudaLaunchKernelEx(&config, kernel, a, plan, args...);
}

// ---- one block for a group, where a call has no scratch ---------------------------------------------------------

// Calls f(index of the cell, its channel) for the thread's cells of a group.  Threads lie along the channels first.
template <typename Fn>
__device__ __forceinline__ void for_cells(const NormArgs& a, Rows r, int32_t channel, int across, Fn f) {
  const int x = threadIdx.x % across, y = threadIdx.x / across, down = kNormThreads / across;
  for (int64_t row = r.lo + y; row < r.hi; row += down)
    for (int32_t c = x; c < a.width; c += across) f(row * a.F + channel + c, channel + c);
}

// dg_norm.cu, dg_norm_bwd.cu
dg_status_t group_norm_fwd(const Graph* g, const NormArgs& a, dg_type_t x, dg_type_t y, dg_act_t act, cudaStream_t s);
dg_status_t group_norm_bwd(const Graph* g, const NormArgs& a, dg_type_t x, dg_type_t y, dg_act_t act, float* dweight,
                           float* dbias, cudaStream_t s);

}  // namespace dg
