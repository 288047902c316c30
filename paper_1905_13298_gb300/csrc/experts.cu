// Tokens in order of their expert, and back.
//
// ds_expert_order is a counting sort that keeps the order of equal keys, in
// one launch: a cluster of up to eight CTAs, whose warps take consecutive
// ranges of the slots.  A warp counts its slots by expert in shared memory (32
// at a time, those of one expert found by a match over the warp), the counts
// are added up over warps, CTAs and experts, and a second pass over the ids
// gives each slot its row.
//
// The other operators move rows and are bound by memory: a token's row is read
// once and written to the rows of its slots; a token's sum reads its slots'
// rows, all on their way at once.
#include "experts.cuh"

namespace ds {
namespace {

// ---------------------------------------------------------------------------
// Order
// ---------------------------------------------------------------------------
constexpr int kOrderThreads = 1024, kOrderWarps = kOrderThreads / 32;

struct OrderParams {
  const void* ids;
  int32_t *offsets, *counts, *position, *slot;
  int64_t slots, rows, per_warp;  // per_warp: a multiple of 32
  int experts, align, wide;       // wide: ids have 64 bits
};

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ int load_of_rank(const int* p, uint32_t rank) {
  const uint32_t own = (uint32_t)__cvta_generic_to_shared(p);
  uint32_t at;
  int v;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(own), "r"(rank));
  asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(at));
  return v;
}

// The expert of a slot, -1 where there is none.
__device__ __forceinline__ int expert_of(const OrderParams& P, int64_t s, int64_t end) {
  if (s >= end) return -1;
  if (P.wide) {
    const int64_t id = static_cast<const int64_t*>(P.ids)[s];
    return id >= 0 && id < P.experts ? (int)id : -1;
  }
  const int id = static_cast<const int32_t*>(P.ids)[s];
  return id >= 0 && id < P.experts ? id : -1;
}

__global__ void __launch_bounds__(kOrderThreads) order_kernel(const OrderParams P) {
  extern __shared__ int order_smem[];
  const int E = P.experts;
  int* const hist = order_smem;                   // [warps][E]: counts, then rows of this warp's next slots
  int* const total = hist + kOrderWarps * E;      // [E] of this CTA
  int* const end_of = total + E;                  // [E] rows in use of each expert end here
  __shared__ int warp_sum[kOrderWarps];
  __shared__ int rows_used;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank(), ranks = cluster_size();
  int* const mine = hist + warp * E;
  for (int e = lane; e < E; e += 32) mine[e] = 0;
  __syncwarp();
  const int64_t from = ((int64_t)rank * kOrderWarps + warp) * P.per_warp;
  const int64_t to = from + P.per_warp < P.slots ? from + P.per_warp : P.slots;
  for (int64_t s = from; s < to; s += 32) {
    const int e = expert_of(P, s + lane, to);
    const uint32_t same = __match_any_sync(0xFFFFFFFFu, e);
    if (e >= 0 && lane == __ffs(same) - 1) mine[e] += __popc(same);
    __syncwarp();
  }
  __syncthreads();
  for (int e = threadIdx.x; e < E; e += kOrderThreads) {
    int sum = 0;
    for (int w = 0; w < kOrderWarps; ++w) {
      const int c = hist[w * E + e];
      hist[w * E + e] = sum;
      sum += c;
    }
    total[e] = sum;
  }
  cluster_barrier();
  // a thread per expert (there are at most as many): counts of the CTAs before this one, and of all
  int before = 0, count = 0;
  const int e = threadIdx.x;
  if (e < E) {
    for (uint32_t r = 0; r < ranks; ++r) {
      const int c = load_of_rank(&total[e], r);
      if (r < rank) before += c;
      count += c;
    }
  }
  const int room = (count + P.align - 1) / P.align * P.align;
  int sum = room;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int up = __shfl_up_sync(0xFFFFFFFFu, sum, d);
    if (lane >= d) sum += up;
  }
  if (lane == 31) warp_sum[warp] = sum;
  __syncthreads();
  int start = sum - room;
  for (int w = 0; w < warp; ++w) start += warp_sum[w];
  if (e < E) {
    for (int w = 0; w < kOrderWarps; ++w) hist[w * E + e] += start + before;
    end_of[e] = start + count;
    if (rank == 0) {
      P.counts[e] = count;
      P.offsets[e + 1] = start + room;
      if (e == 0) P.offsets[0] = 0;
    }
    if (e == E - 1) rows_used = start + room;
  }
  __syncthreads();
  for (int64_t s = from; s < to; s += 32) {
    const int id = expert_of(P, s + lane, to);
    const uint32_t same = __match_any_sync(0xFFFFFFFFu, id);
    int row = -1;
    if (id >= 0) row = mine[id] + __popc(same & ((1u << lane) - 1u));
    __syncwarp();
    if (id >= 0 && lane == __ffs(same) - 1) mine[id] += __popc(same);
    __syncwarp();
    if (s + lane < to) P.position[s + lane] = row;
    if (row >= 0 && row < P.rows) P.slot[row] = (int32_t)(s + lane);
  }
  // rows without a slot: behind each expert's, up to the next one's, and behind the last
  for (int x = (int)rank * kOrderWarps + warp; x < E; x += (int)ranks * kOrderWarps) {
    const int stop = (end_of[x] + P.align - 1) / P.align * P.align;  // segments start at multiples
    for (int64_t r = end_of[x] + lane; r < stop && r < P.rows; r += 32) P.slot[r] = -1;
  }
  for (int64_t r = rows_used + (int64_t)rank * kOrderThreads + threadIdx.x; r < P.rows; r += ranks * kOrderThreads)
    P.slot[r] = -1;
  cluster_barrier();  // the other CTAs read this one's counts until here
}

// ---------------------------------------------------------------------------
// Rows
// ---------------------------------------------------------------------------
constexpr int kThreads = 256, kWarps = kThreads / 32;

template <int UNIT>
struct UnitOf;
template <>
struct UnitOf<16> {
  using T = uint4;
};
template <>
struct UnitOf<8> {
  using T = uint2;
};
template <>
struct UnitOf<4> {
  using T = uint32_t;
};
template <>
struct UnitOf<2> {
  using T = uint16_t;
};

struct GatherParams {
  RowCopy a, b;
  const int32_t *position, *slot;
  int64_t tokens, rows;
  int top_k;
  int64_t units;  // of a row of a (whole ones)
  int rest;       // bytes of a row behind them
  int64_t parts;  // a warp copies a part of a row
  int64_t copies; // warps that copy; the others write zeros
};

constexpr int kPart = 4;        // units of a lane
constexpr int kZeroRows = 8;    // rows of a warp that looks for rows without a slot

template <int UNIT>
__device__ __forceinline__ void zero_row(const GatherParams& P, int64_t r, int lane) {
  using T = typename UnitOf<UNIT>::T;
  T* to = reinterpret_cast<T*>(static_cast<char*>(P.a.dst) + r * P.a.ld_dst);
  for (int64_t u = lane; u < P.units; u += 32) to[u] = T{};
  if (lane < P.rest) static_cast<uint8_t*>(P.a.dst)[r * P.a.ld_dst + P.units * UNIT + lane] = 0;
  if (P.b.src) {
    float* s = reinterpret_cast<float*>(static_cast<char*>(P.b.dst) + r * P.b.ld_dst);
    for (int64_t u = lane; u < P.b.bytes / 4; u += 32) s[u] = 0.f;
  }
}

// A warp reads a part of a token's row and writes it to the rows of the token's slots.
template <int UNIT>
__global__ void __launch_bounds__(kThreads) gather_kernel(const GatherParams P) {
  using T = typename UnitOf<UNIT>::T;
  const int lane = threadIdx.x & 31;
  const int64_t id = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
  if (id >= P.copies) {
    const int64_t r0 = (id - P.copies) * kZeroRows, r = r0 + lane;
    uint32_t todo = __ballot_sync(0xFFFFFFFFu, lane < kZeroRows && r < P.rows && P.slot[r < P.rows ? r : 0] < 0);
    while (todo) {
      zero_row<UNIT>(P, r0 + __ffs(todo) - 1, lane);
      todo &= todo - 1;
    }
    return;
  }
  const int64_t t = id / P.parts, u0 = (id - t * P.parts) * (32 * kPart) + lane;
  const char* from = static_cast<const char*>(P.a.src) + t * P.a.ld_src;
  T v[kPart];
#pragma unroll
  for (int i = 0; i < kPart; ++i)
    if (u0 + 32 * i < P.units) v[i] = reinterpret_cast<const T*>(from)[u0 + 32 * i];
  // the row's last bytes, and the second matrix, go with its first part
  const bool first = u0 == lane;
  uint8_t last = 0;
  if (first && lane < P.rest) last = reinterpret_cast<const uint8_t*>(from)[P.units * UNIT + lane];
  for (int j0 = 0; j0 < P.top_k; j0 += 32) {
    const int32_t mine = j0 + lane < P.top_k ? P.position[t * P.top_k + j0 + lane] : -1;
    const int n = P.top_k - j0 < 32 ? P.top_k - j0 : 32;
    for (int j = 0; j < n; ++j) {
      const int64_t row = __shfl_sync(0xFFFFFFFFu, mine, j);
      if (row < 0 || row >= P.rows) continue;
      char* to = static_cast<char*>(P.a.dst) + row * P.a.ld_dst;
#pragma unroll
      for (int i = 0; i < kPart; ++i)
        if (u0 + 32 * i < P.units) reinterpret_cast<T*>(to)[u0 + 32 * i] = v[i];
      if (first && lane < P.rest) reinterpret_cast<uint8_t*>(to)[P.units * UNIT + lane] = last;
      if (first && P.b.src) {
        const float* s = reinterpret_cast<const float*>(static_cast<const char*>(P.b.src) + t * P.b.ld_src);
        float* d = reinterpret_cast<float*>(static_cast<char*>(P.b.dst) + row * P.b.ld_dst);
        for (int64_t u = lane; u < P.b.bytes / 4; u += 32) d[u] = s[u];
      }
    }
  }
}

struct CombineParams {
  const void *y, *add;
  int64_t ldy, ld_add, ldo, cols, tokens, rows, parts;
  const int32_t *position, *slot;
  const float* weights;
  void* out;
  int top_k, vec;
};

constexpr int kRowsAtOnce = 8;  // rows of a token on their way at once

// A warp makes 256 values of a token's sum.
template <typename T>
__global__ void __launch_bounds__(kThreads) combine_kernel(const CombineParams P) {
  const int lane = threadIdx.x & 31;
  const int64_t id = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int64_t t = id / P.parts, c = (id - t * P.parts) * 256 + lane * 8;
  if (t >= P.tokens) return;
  const int n = left8(P.cols, c);
  const bool vec = P.vec;
  Raw8<T> more;
  if (P.add) more.template load<true>(static_cast<const T*>(P.add) + t * P.ld_add + c, n, vec);
  float acc[8] = {};
  for (int j0 = 0; j0 < P.top_k; j0 += kRowsAtOnce) {
    int32_t at = -1;
    float w = 1.f;
    if (lane < kRowsAtOnce && j0 + lane < P.top_k) {
      at = P.position[t * P.top_k + j0 + lane];
      if (P.weights) w = P.weights[t * P.top_k + j0 + lane];
    }
    Raw8<T> v[kRowsAtOnce];
    int32_t row[kRowsAtOnce];
#pragma unroll
    for (int j = 0; j < kRowsAtOnce; ++j) {
      row[j] = __shfl_sync(0xFFFFFFFFu, at, j);
      if (row[j] >= 0 && row[j] < P.rows)
        v[j].template load<true>(static_cast<const T*>(P.y) + row[j] * P.ldy + c, n, vec);
    }
#pragma unroll
    for (int j = 0; j < kRowsAtOnce; ++j) {
      const float wj = __shfl_sync(0xFFFFFFFFu, w, j);
      if (row[j] < 0 || row[j] >= P.rows) continue;
      float f[8];
      v[j].get(f);
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[i] = fmaf(wj, f[i], acc[i]);
    }
  }
  if (P.add) {
    float f[8];
    more.get(f);
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] += f[i];
  }
  store8<true>(static_cast<T*>(P.out) + t * P.ldo + c, n, vec, acc);
}

struct CombineBackwardParams {
  const void *d, *y;
  int64_t ldd, ldy, lddy, cols, tokens, rows;
  const int32_t *position, *slot;
  const float* weights;
  void* dy;
  float* dweights;
  int top_k, vec;
};

// A warp goes through a token's row; with slots in groups, the row of dout is read once for each group.
template <typename T>
__global__ void __launch_bounds__(kThreads) combine_backward_kernel(const CombineBackwardParams P) {
  const int lane = threadIdx.x & 31;
  const int64_t id = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const bool vec = P.vec;
  if (id >= P.tokens) {
    const int64_t r0 = (id - P.tokens) * kZeroRows, r = r0 + lane;
    uint32_t todo = __ballot_sync(0xFFFFFFFFu, lane < kZeroRows && r < P.rows && P.slot[r < P.rows ? r : 0] < 0);
    const float zero[8] = {};
    while (todo) {
      T* to = static_cast<T*>(P.dy) + (r0 + __ffs(todo) - 1) * P.lddy;
      for (int64_t c = lane * 8; c < P.cols; c += 256) store8<true>(to + c, left8(P.cols, c), vec, zero);
      todo &= todo - 1;
    }
    return;
  }
  const int64_t t = id;
  const T* const d = static_cast<const T*>(P.d) + t * P.ldd;
  for (int j0 = 0; j0 < P.top_k; j0 += kRowsAtOnce) {
    int32_t at = -1;
    float w = 1.f;
    if (lane < kRowsAtOnce && j0 + lane < P.top_k) {
      at = P.position[t * P.top_k + j0 + lane];
      if (P.weights) w = P.weights[t * P.top_k + j0 + lane];
    }
    int32_t row[kRowsAtOnce];
    float wj[kRowsAtOnce], dot[kRowsAtOnce];
#pragma unroll
    for (int j = 0; j < kRowsAtOnce; ++j) {
      row[j] = __shfl_sync(0xFFFFFFFFu, at, j);
      if (row[j] >= P.rows) row[j] = -1;
      wj[j] = __shfl_sync(0xFFFFFFFFu, w, j);
      dot[j] = 0.f;
    }
    for (int64_t c = lane * 8; c < P.cols; c += 256) {
      const int n = left8(P.cols, c);
      Raw8<T> rd, ry[kRowsAtOnce];
      rd.template load<true>(d + c, n, vec);
      if (P.dweights) {
#pragma unroll
        for (int j = 0; j < kRowsAtOnce; ++j)
          if (row[j] >= 0) ry[j].template load<true>(static_cast<const T*>(P.y) + row[j] * P.ldy + c, n, vec);
      }
      float f[8];
      rd.get(f);
#pragma unroll
      for (int j = 0; j < kRowsAtOnce; ++j) {
        if (row[j] < 0) continue;
        if (P.dweights) {
          float g[8];
          ry[j].get(g);
#pragma unroll
          for (int i = 0; i < 8; ++i) dot[j] = fmaf(f[i], g[i], dot[j]);
        }
        float o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = wj[j] * f[i];
        store8<true>(static_cast<T*>(P.dy) + row[j] * P.lddy + c, n, vec, o);
      }
    }
    if (P.dweights) {
#pragma unroll
      for (int j = 0; j < kRowsAtOnce; ++j) {
#pragma unroll
        for (int x = 16; x >= 1; x >>= 1) dot[j] += __shfl_xor_sync(0xFFFFFFFFu, dot[j], x);
        if (lane == j && j0 + j < P.top_k) P.dweights[t * P.top_k + j0 + j] = dot[j];
      }
    }
  }
}

int64_t over(int64_t n, int64_t d) { return (n + d - 1) / d; }

bool rows_aligned(const void* p, int64_t ld, int type) {
  return p == nullptr || (aligned(p, 16) && ld * type_size(type) % 16 == 0);
}

template <int UNIT>
cudaError_t launch_gather(GatherParams& p, cudaStream_t st) {
  p.units = p.a.bytes / UNIT;
  p.rest = (int)(p.a.bytes % UNIT);
  p.parts = over(p.units > 0 ? p.units : 1, 32 * kPart);
  p.copies = p.tokens * p.parts;
  const int64_t ctas = over(p.copies + over(p.rows, kZeroRows), kWarps);
  if (ctas > ((int64_t)1 << 31) - 1) return cudaErrorInvalidValue;
  if (ctas > 0) gather_kernel<UNIT><<<(unsigned)ctas, kThreads, 0, st>>>(p);
  return cudaGetLastError();
}

template <typename T>
cudaError_t launch_combine(const CombineParams& p, cudaStream_t st) {
  const int64_t ctas = over(p.tokens * p.parts, kWarps);
  if (ctas > ((int64_t)1 << 31) - 1) return cudaErrorInvalidValue;
  combine_kernel<T><<<(unsigned)ctas, kThreads, 0, st>>>(p);
  return cudaGetLastError();
}
template <typename T>
cudaError_t launch_combine_backward(const CombineBackwardParams& p, cudaStream_t st) {
  const int64_t ctas = over(p.tokens + over(p.rows, kZeroRows), kWarps);
  if (ctas > ((int64_t)1 << 31) - 1) return cudaErrorInvalidValue;
  combine_backward_kernel<T><<<(unsigned)ctas, kThreads, 0, st>>>(p);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_expert_order(const void* ids, int id_type, const ds_expert_slots& s, cudaStream_t st) {
  const size_t smem = sizeof(int) * (size_t)s.experts * (kOrderWarps + 2);
  static const cudaError_t attr = cudaFuncSetAttribute(
      order_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(sizeof(int) * DS_EXPERTS_MAX * (kOrderWarps + 2)));
  if (attr != cudaSuccess) return attr;
  OrderParams p;
  p.ids = ids;
  p.offsets = s.offsets, p.counts = s.counts, p.position = s.position, p.slot = s.slot;
  p.slots = s.tokens * s.top_k, p.rows = s.rows;
  p.experts = s.experts, p.align = s.align, p.wide = id_type == DS_INDEX_I64;
  int ctas = 1;
  while (ctas < 8 && p.slots > (int64_t)ctas * kOrderThreads) ctas *= 2;
  p.per_warp = over(over(p.slots, (int64_t)ctas * kOrderWarps), 32) * 32;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ctas);
  cfg.blockDim = dim3(kOrderThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned)ctas;
  at[0].val.clusterDim.y = 1;
  at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, order_kernel, p);
}

cudaError_t launch_expert_gather(const RowCopy& a, const RowCopy& b, const ds_expert_slots& s, cudaStream_t st) {
  GatherParams p = {};
  p.a = a, p.b = b;
  p.position = s.position, p.slot = s.slot;
  p.tokens = s.tokens, p.rows = s.rows, p.top_k = s.top_k;
  switch (a.unit) {
    case 16: return launch_gather<16>(p, st);
    case 8: return launch_gather<8>(p, st);
    case 4: return launch_gather<4>(p, st);
    default: return launch_gather<2>(p, st);
  }
}

cudaError_t launch_expert_combine(const void* y, int type, int64_t ldy, int64_t cols, const ds_expert_slots& s,
                                  const float* weights, const void* add, int64_t ld_add, void* out, int64_t ldo,
                                  cudaStream_t st) {
  CombineParams p = {};
  p.y = y, p.add = add, p.out = out, p.weights = weights;
  p.ldy = ldy, p.ld_add = ld_add, p.ldo = ldo, p.cols = cols;
  p.tokens = s.tokens, p.rows = s.rows, p.top_k = s.top_k;
  p.position = s.position, p.slot = s.slot;
  p.parts = over(cols, 256);
  p.vec = rows_aligned(y, ldy, type) && rows_aligned(add, ld_add, type) && rows_aligned(out, ldo, type);
  if (type == DS_TYPE_F32) return launch_combine<float>(p, st);
  if (type == DS_TYPE_BF16) return launch_combine<__nv_bfloat16>(p, st);
  return launch_combine<__half>(p, st);
}

cudaError_t launch_expert_combine_backward(const void* dout, int64_t ldd, const void* y, int64_t ldy, int type,
                                           int64_t cols, const ds_expert_slots& s, const float* weights, void* dy,
                                           int64_t lddy, float* dweights, cudaStream_t st) {
  CombineBackwardParams p = {};
  p.d = dout, p.y = y, p.dy = dy, p.weights = weights, p.dweights = dweights;
  p.ldd = ldd, p.ldy = ldy, p.lddy = lddy, p.cols = cols;
  p.tokens = s.tokens, p.rows = s.rows, p.top_k = s.top_k;
  p.position = s.position, p.slot = s.slot;
  p.vec = rows_aligned(dout, ldd, type) && rows_aligned(dweights ? y : nullptr, ldy, type) && rows_aligned(dy, lddy, type);
  if (type == DS_TYPE_F32) return launch_combine_backward<float>(p, st);
  if (type == DS_TYPE_BF16) return launch_combine_backward<__nv_bfloat16>(p, st);
  return launch_combine_backward<__half>(p, st);
}

}  // namespace ds
