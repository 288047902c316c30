// Tokens in order of their expert, and back.
//
// ds_expert_order is a counting sort that keeps the order of equal keys, in
// one launch: a cluster of up to 16 CTAs, whose warps take consecutive
// ranges of the slots.  A warp counts its slots by expert in shared memory (32
// at a time, those of one expert found by a match over the warp), the counts
// are added up over warps, CTAs and experts, and a second pass over the ids
// gives each slot its row.  It is bound by latency: 64 slots take 4.4 us, 32768
// of 32 experts 7.4 (9.4 with eight CTAs), of which launch and cluster barriers
// are 5.7.
//
// The other operators move rows and are bound by memory: a token's row is read
// once and written to the rows of its slots; a token's sum reads its slots'
// rows, all on their way at once.  8192 x 4 slots of 2048: 8-bit rows gathered
// in 15.7 us, 16-bit ones in 28.7 (0.89 and 0.93 of HBM).
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
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
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

// Ids of a lane on their way at once; the first ones are kept for the second pass.  With eight, 64 slots take 4.7 us (4.4
// with four), 32768 of 32 experts 8.4 (8.0), 131072 of 64 19.9 (20.5), 1.1 million 138 (132; 144 one at a time).
constexpr int kHeld = 4;
constexpr uint32_t kMostCtas = 16;  // CTAs of a cluster

// CLUSTER: more than one CTA.
template <bool CLUSTER>
__global__ void __launch_bounds__(kOrderThreads) order_kernel(const OrderParams P) {
  extern __shared__ int order_smem[];
  const int E = P.experts, warps = blockDim.x >> 5;
  int* const hist = order_smem;          // [warps][E]: counts, then rows of this warp's next slots
  int* const total = hist + warps * E;   // [E] of this CTA
  int* const end_of = total + E;         // [E] rows in use of each expert end here
  __shared__ int warp_sum[kOrderWarps];
  __shared__ int rows_used;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = CLUSTER ? cluster_rank() : 0, ranks = CLUSTER ? cluster_size() : 1;
  int* const mine = hist + warp * E;
  const int64_t from = ((int64_t)rank * warps + warp) * P.per_warp;
  const int64_t to = from + P.per_warp < P.slots ? from + P.per_warp : P.slots;
  int held[kHeld];
  auto load = [&](int64_t s, int (&ids)[kHeld]) {
#pragma unroll
    for (int k = 0; k < kHeld; ++k) ids[k] = expert_of(P, s + 32 * k + lane, to);
  };
  load(from, held);
  for (int e = lane; e < E; e += 32) mine[e] = 0;
  __syncwarp();
  auto count_32 = [&](int e) {
    const uint32_t same = __match_any_sync(0xFFFFFFFFu, e);
    if (e >= 0 && lane == __ffs(same) - 1) mine[e] += __popc(same);
    __syncwarp();
  };
  auto count = [&](int64_t s, const int (&ids)[kHeld]) {
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
      if (s + 32 * k < to) count_32(ids[k]);
  };
  count(from, held);
  for (int64_t s = from + 32 * kHeld; s < to; s += 32 * kHeld) {
    int ids[kHeld];
    load(s, ids);
    count(s, ids);
  }
  __syncthreads();
  // a thread per expert (there are at most as many)
  const int e = threadIdx.x;
  int here = 0;
  if (e < E) {
#pragma unroll 8
    for (int w = 0; w < warps; ++w) here += hist[w * E + e];
  }
  int before = 0, all = here;  // slots of the CTAs before this one, and of all
  if constexpr (CLUSTER) {
    if (e < E) total[e] = here;
    __syncwarp();  // a warp arrives together: the barrier is an aligned one
    cluster_arrive();
    cluster_wait();
    if (e < E) {
      int c[kMostCtas];
#pragma unroll
      for (uint32_t r = 0; r < kMostCtas; ++r) c[r] = r < ranks ? load_of_rank(&total[e], r) : 0;
      all = 0;
#pragma unroll
      for (uint32_t r = 0; r < kMostCtas; ++r) {
        if (r < rank) before += c[r];
        all += c[r];
      }
    }
    __syncwarp();
    cluster_arrive();  // the other CTAs' counts have been read
  }
  const int room = (int)(((uint32_t)all + P.align - 1) / P.align * P.align);
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
    int at = start + before;
#pragma unroll 8
    for (int w = 0; w < warps; ++w) {
      const int c = hist[w * E + e];
      hist[w * E + e] = at;
      at += c;
    }
    end_of[e] = start + all;
    if (rank == 0) {
      P.counts[e] = all;
      P.offsets[e + 1] = start + room;
      if (e == 0) P.offsets[0] = 0;
    }
    if (e == E - 1) rows_used = start + room;
  }
  __syncthreads();
  auto place_32 = [&](int64_t s, int id) {
    const uint32_t same = __match_any_sync(0xFFFFFFFFu, id);
    int row = -1;
    if (id >= 0) row = mine[id] + __popc(same & ((1u << lane) - 1u));
    __syncwarp();
    if (id >= 0 && lane == __ffs(same) - 1) mine[id] += __popc(same);
    __syncwarp();
    if (s + lane < to) P.position[s + lane] = row;
    if (row >= 0 && row < P.rows) P.slot[row] = (int32_t)(s + lane);
  };
  auto place = [&](int64_t s, const int (&ids)[kHeld]) {
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
      if (s + 32 * k < to) place_32(s + 32 * k, ids[k]);
  };
  place(from, held);
  for (int64_t s = from + 32 * kHeld; s < to; s += 32 * kHeld) {
    int ids[kHeld];
    load(s, ids);
    place(s, ids);
  }
  // rows without a slot: behind each expert's, up to the next one's, and behind the last
  for (int x = (int)rank * warps + warp; x < E; x += (int)ranks * warps) {
    const int64_t stop = ((uint32_t)end_of[x] + P.align - 1) / P.align * P.align;  // segments start at multiples
    for (int64_t r = end_of[x] + lane; r < stop && r < P.rows; r += 32) P.slot[r] = -1;
  }
  for (int64_t r = rows_used + (int64_t)rank * blockDim.x + threadIdx.x; r < P.rows; r += ranks * blockDim.x)
    P.slot[r] = -1;
  __syncwarp();
  if constexpr (CLUSTER) cluster_wait();  // this CTA's counts have been read by the others
}

// ---------------------------------------------------------------------------
// Rows
// ---------------------------------------------------------------------------
// CTAs of four warps, and one wide access of each row for a lane: loads that start later while others end (8192 x 4 slots,
// 2048 bf16: combine 33 us, 42 with 256 threads and two accesses; its gradient 49 and 53; gather 28.5 and 34).
constexpr int kThreads = 128, kWarps = kThreads / 32;

// An access of BYTES bytes and the values in it.
template <int BYTES>
struct UnitOf;
template <>
struct UnitOf<16> {
  using T = uint4;
};
template <>
struct UnitOf<4> {
  using T = uint32_t;
};
template <>
struct UnitOf<2> {
  using T = uint16_t;
};
template <typename T, int BYTES>
struct Unit {
  static constexpr int COUNT = BYTES / (int)sizeof(T);
  typename UnitOf<BYTES>::T u;
  __device__ __forceinline__ void get(float (&v)[COUNT]) const {
    const T* p = reinterpret_cast<const T*>(&u);
#pragma unroll
    for (int i = 0; i < COUNT; ++i) v[i] = to_float(p[i]);
  }
  __device__ __forceinline__ void set(const float (&v)[COUNT]) {
    T* p = reinterpret_cast<T*>(&u);
#pragma unroll
    for (int i = 0; i < COUNT; ++i) from_float(v[i], p[i]);
  }
};
// Unit i of row r.
template <typename U>
__device__ __forceinline__ U* unit_at(void* base, int64_t r, int64_t ld_bytes, int64_t i) {
  return reinterpret_cast<U*>(static_cast<char*>(base) + r * ld_bytes) + i;
}
template <typename U>
__device__ __forceinline__ const U* unit_at(const void* base, int64_t r, int64_t ld_bytes, int64_t i) {
  return reinterpret_cast<const U*>(static_cast<const char*>(base) + r * ld_bytes) + i;
}

// n / d for d of at most 2^31, without a division of 64 bits where n has 32: that costs more than a short row.
__device__ __forceinline__ int64_t quotient(int64_t n, int64_t d) {
  return n >> 32 == 0 ? (int64_t)((uint32_t)n / (uint32_t)d) : n / d;
}

// Which of the n rows from r0 on hold no slot, as bits; there are `rows` in all.
__device__ __forceinline__ uint32_t rows_without(const int32_t* slot, int64_t r0, int n, int64_t rows) {
  const int lane = threadIdx.x & 31;
  const int64_t r = r0 + lane;
  return __ballot_sync(0xFFFFFFFFu, lane < n && r < rows && slot[r < rows ? r : 0] < 0);
}
// Rows that a warp looks through for those without a slot: up to 8 KB, which it then may have to write.
int rows_to_zero(int64_t row_bytes) {
  const int64_t n = 8192 / (row_bytes > 0 ? row_bytes : 1);
  return n < 1 ? 1 : (n < 32 ? (int)n : 32);
}

struct GatherParams {
  RowCopy a, b;
  const int32_t *position, *slot;
  int64_t tokens, rows;
  int top_k;
  int64_t units;   // of a row of a (whole ones)
  int rest;        // bytes of a row behind them
  int64_t parts;   // a warp copies a part of a row
  int64_t copies;  // warps that copy; the others write zeros
  int zero_rows;   // that such a warp looks through
};

constexpr int kPart = 2;  // units of a lane

template <int BYTES>
__device__ __forceinline__ void zero_row(const GatherParams& P, int64_t r, int lane) {
  using T = typename UnitOf<BYTES>::T;
  for (int64_t u = lane; u < P.units; u += 32) *unit_at<T>(P.a.dst, r, P.a.ld_dst, u) = T{};
  if (lane < P.rest) unit_at<uint8_t>(P.a.dst, r, P.a.ld_dst, P.units * BYTES)[lane] = 0;
  if (P.b.dst)
    for (int64_t u = lane; u < P.b.bytes / 4; u += 32) *unit_at<float>(P.b.dst, r, P.b.ld_dst, u) = 0.f;
}

// A warp reads a part of a token's row and writes it to the rows of the token's slots.
template <int BYTES>
__global__ void __launch_bounds__(kThreads) gather_kernel(const GatherParams P) {
  using T = typename UnitOf<BYTES>::T;
  const int lane = threadIdx.x & 31;
  const int64_t id = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
  if (id >= P.copies) {
    const int64_t r0 = (id - P.copies) * P.zero_rows;
    for (uint32_t todo = rows_without(P.slot, r0, P.zero_rows, P.rows); todo; todo &= todo - 1)
      zero_row<BYTES>(P, r0 + __ffs(todo) - 1, lane);
    return;
  }
  const int64_t t = quotient(id, P.parts), u0 = (id - t * P.parts) * (32 * kPart) + lane;
  T v[kPart];
#pragma unroll
  for (int i = 0; i < kPart; ++i)
    if (u0 + 32 * i < P.units) v[i] = *unit_at<T>(P.a.src, t, P.a.ld_src, u0 + 32 * i);
  // the row's last bytes, and the second matrix, go with its first part
  const bool first = u0 == lane;
  uint8_t last = 0;
  if (first && lane < P.rest) last = unit_at<uint8_t>(P.a.src, t, P.a.ld_src, P.units * BYTES)[lane];
  for (int j0 = 0; j0 < P.top_k; j0 += 32) {
    const int32_t mine = j0 + lane < P.top_k ? P.position[t * P.top_k + j0 + lane] : -1;
    const int n = P.top_k - j0 < 32 ? P.top_k - j0 : 32;
    for (int j = 0; j < n; ++j) {
      const int64_t row = __shfl_sync(0xFFFFFFFFu, mine, j);
      if (row < 0 || row >= P.rows) continue;
#pragma unroll
      for (int i = 0; i < kPart; ++i)
        if (u0 + 32 * i < P.units) *unit_at<T>(P.a.dst, row, P.a.ld_dst, u0 + 32 * i) = v[i];
      if (first && lane < P.rest) unit_at<uint8_t>(P.a.dst, row, P.a.ld_dst, P.units * BYTES)[lane] = last;
      if (first && P.b.dst)
        for (int64_t u = lane; u < P.b.bytes / 4; u += 32)
          *unit_at<float>(P.b.dst, row, P.b.ld_dst, u) = *unit_at<float>(P.b.src, t, P.b.ld_src, u);
    }
  }
}

struct CombineParams {
  const void *y, *add;
  int64_t ldy, ld_add, ldo;  // in bytes
  int64_t units, tokens, rows, parts;
  const int32_t* position;
  const float* weights;
  void* out;
  int top_k;
};

// Units of a lane.
constexpr int units_of(int bytes) { return bytes == 16 ? 1 : 8; }

// A warp makes a part of a token's sum, from AT_ONCE rows at a time.
template <typename T, int BYTES, int AT_ONCE>
__global__ void __launch_bounds__(kThreads) combine_kernel(const CombineParams P) {
  using U = Unit<T, BYTES>;
  constexpr int N = units_of(BYTES);
  const int lane = threadIdx.x & 31;
  const int64_t id = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int64_t t = quotient(id, P.parts), u0 = (id - t * P.parts) * (32 * N) + lane;
  if (t >= P.tokens) return;
  float acc[N][U::COUNT] = {};
  U more[N];
  if (P.add) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (u0 + 32 * i < P.units) more[i] = *unit_at<U>(P.add, t, P.ld_add, u0 + 32 * i);
  }
  for (int j0 = 0; j0 < P.top_k; j0 += AT_ONCE) {
    int32_t at = -1;
    float w = 1.f;
    if (lane < AT_ONCE && j0 + lane < P.top_k) {
      at = P.position[t * P.top_k + j0 + lane];
      if (at >= P.rows) at = -1;
      if (P.weights) w = P.weights[t * P.top_k + j0 + lane];
    }
    U v[AT_ONCE][N];
    int32_t row[AT_ONCE];
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      row[j] = __shfl_sync(0xFFFFFFFFu, at, j);
      if (row[j] < 0) continue;
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (u0 + 32 * i < P.units) v[j][i] = *unit_at<U>(P.y, row[j], P.ldy, u0 + 32 * i);
    }
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      const float wj = __shfl_sync(0xFFFFFFFFu, w, j);
      if (row[j] < 0) continue;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        float f[U::COUNT];
        v[j][i].get(f);
#pragma unroll
        for (int k = 0; k < U::COUNT; ++k) acc[i][k] = fmaf(wj, f[k], acc[i][k]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (u0 + 32 * i >= P.units) continue;
    if (P.add) {
      float f[U::COUNT];
      more[i].get(f);
#pragma unroll
      for (int k = 0; k < U::COUNT; ++k) acc[i][k] += f[k];
    }
    U o;
    o.set(acc[i]);
    *unit_at<U>(P.out, t, P.ldo, u0 + 32 * i) = o;
  }
}

struct CombineBackwardParams {
  const void *d, *y;
  int64_t ldd, ldy, lddy;  // in bytes
  int64_t units, tokens, rows;
  const int32_t *position, *slot;
  const float* weights;
  void* dy;
  float* dweights;
  int top_k, zero_rows;
};

constexpr int kMostShare = 16;  // warps of a token

// A warp goes through a token's row, or (SHARED) all of a CTA's warps through parts of it in turn, where tokens are few;
// with slots in groups of AT_ONCE, the row of dout is read once for each group.
template <typename T, int BYTES, int AT_ONCE, bool SHARED>
__global__ void __launch_bounds__(SHARED ? 32 * kMostShare : kThreads)
    combine_backward_kernel(const CombineBackwardParams P) {
  using U = Unit<T, BYTES>;
  constexpr int N = units_of(BYTES);
  __shared__ float part[SHARED ? kMostShare : 1][AT_ONCE];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, share = SHARED ? (int)(blockDim.x >> 5) : 1;
  const int64_t t = SHARED ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * kWarps + warp;
  if (t >= P.tokens) {
    const int64_t r0 = (SHARED ? (t - P.tokens) * share + warp : t - P.tokens) * P.zero_rows;
    for (uint32_t todo = rows_without(P.slot, r0, P.zero_rows, P.rows); todo; todo &= todo - 1)
      for (int64_t u = lane; u < P.units; u += 32) *unit_at<U>(P.dy, r0 + __ffs(todo) - 1, P.lddy, u) = U{};
    return;
  }
  for (int j0 = 0; j0 < P.top_k; j0 += AT_ONCE) {
    int32_t at = -1;
    float w = 1.f;
    if (lane < AT_ONCE && j0 + lane < P.top_k) {
      at = P.position[t * P.top_k + j0 + lane];
      if (at >= P.rows) at = -1;
      if (P.weights) w = P.weights[t * P.top_k + j0 + lane];
    }
    int32_t row[AT_ONCE];
    float wj[AT_ONCE], dot[AT_ONCE];
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      row[j] = __shfl_sync(0xFFFFFFFFu, at, j);
      wj[j] = __shfl_sync(0xFFFFFFFFu, w, j);
      dot[j] = 0.f;
    }
    // N units of all rows are loaded before the first is stored, which may be where y lies
    for (int64_t u0 = (SHARED ? warp * (32 * N) : 0) + lane; u0 < P.units; u0 += share * (32 * N)) {
      U rd[N], ry[AT_ONCE][N];
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (u0 + 32 * i < P.units) rd[i] = *unit_at<U>(P.d, t, P.ldd, u0 + 32 * i);
      if (P.dweights) {
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j)
#pragma unroll
          for (int i = 0; i < N; ++i)
            if (row[j] >= 0 && u0 + 32 * i < P.units) ry[j][i] = *unit_at<U>(P.y, row[j], P.ldy, u0 + 32 * i);
      }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (u0 + 32 * i >= P.units) break;
        float f[U::COUNT];
        rd[i].get(f);
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
          if (row[j] < 0) continue;
          if (P.dweights) {
            float g[U::COUNT];
            ry[j][i].get(g);
#pragma unroll
            for (int k = 0; k < U::COUNT; ++k) dot[j] = fmaf(f[k], g[k], dot[j]);
          }
          float o[U::COUNT];
#pragma unroll
          for (int k = 0; k < U::COUNT; ++k) o[k] = wj[j] * f[k];
          U s;
          s.set(o);
          *unit_at<U>(P.dy, row[j], P.lddy, u0 + 32 * i) = s;
        }
      }
    }
    if (P.dweights) {
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j) {
#pragma unroll
        for (int x = 16; x >= 1; x >>= 1) dot[j] += __shfl_xor_sync(0xFFFFFFFFu, dot[j], x);
        if constexpr (SHARED) {
          if (lane == j) part[warp][j] = dot[j];
        } else {
          if (lane == j && j0 + j < P.top_k) P.dweights[t * P.top_k + j0 + j] = dot[j];
        }
      }
      if constexpr (SHARED) {  // the warps' parts in their order
        __syncthreads();
        if (threadIdx.x < AT_ONCE && j0 + (int)threadIdx.x < P.top_k) {
          float sum = 0.f;
          for (int w = 0; w < share; ++w) sum += part[w][threadIdx.x];
          P.dweights[t * P.top_k + j0 + threadIdx.x] = sum;
        }
        __syncthreads();
      }
    }
  }
}

int64_t over(int64_t n, int64_t d) { return (n + d - 1) / d; }

template <int BYTES>
cudaError_t launch_gather(GatherParams& p, cudaStream_t st) {
  p.units = p.a.bytes / BYTES;
  p.rest = (int)(p.a.bytes % BYTES);
  p.parts = over(p.units > 0 ? p.units : 1, 32 * kPart);
  p.copies = p.tokens * p.parts;
  p.zero_rows = rows_to_zero(p.a.bytes);
  const int64_t ctas = over(p.copies + over(p.rows, p.zero_rows), kWarps);
  if (ctas > ((int64_t)1 << 31) - 1) return cudaErrorInvalidValue;
  if (ctas > 0) gather_kernel<BYTES><<<(unsigned)ctas, kThreads, 0, st>>>(p);
  return cudaGetLastError();
}

template <typename T, int BYTES, int AT_ONCE>
cudaError_t launch_combine(CombineParams& p, cudaStream_t st) {
  p.parts = over(p.units, 32 * units_of(BYTES));
  const int64_t ctas = over(p.tokens * p.parts, kWarps);
  if (ctas > ((int64_t)1 << 31) - 1) return cudaErrorInvalidValue;
  combine_kernel<T, BYTES, AT_ONCE><<<(unsigned)ctas, kThreads, 0, st>>>(p);
  return cudaGetLastError();
}
template <typename T, int BYTES, int AT_ONCE>
cudaError_t launch_combine(CombineBackwardParams& p, cudaStream_t st) {
  // Warps of a token while the device is not full of tokens' warps, at least two rounds through the row for each (16 x 8
  // slots of 16384 bf16 8.8 us, 46 with one warp; 512 x 8 51, 130)
  const int64_t room = 32 * (int64_t)(sm_count() > 0 ? sm_count() : 1), rounds = over(p.units, 32 * units_of(BYTES));
  int share = 1;
  while (share < kMostShare && 2 * share * p.tokens <= room && 4 * share <= rounds) share *= 2;
  p.zero_rows = rows_to_zero(p.units * BYTES);
  const int64_t zeros = over(p.rows, p.zero_rows);
  const int64_t ctas = share > 1 ? p.tokens + over(zeros, share) : over(p.tokens + zeros, kWarps);
  if (ctas > ((int64_t)1 << 31) - 1) return cudaErrorInvalidValue;
  if (share > 1)
    combine_backward_kernel<T, BYTES, AT_ONCE, true><<<(unsigned)ctas, 32 * share, 0, st>>>(p);
  else
    combine_backward_kernel<T, BYTES, AT_ONCE, false><<<(unsigned)ctas, kThreads, 0, st>>>(p);
  return cudaGetLastError();
}
// As many rows at once as a token has, of 2, 4 or 8: registers and instructions for more cost a third of the time.
template <typename T, int BYTES, typename Params>
cudaError_t choose_rows(Params& p, int64_t bytes, cudaStream_t st) {
  p.units = bytes / BYTES;
  if (p.top_k <= 2) return launch_combine<T, BYTES, 2>(p, st);
  if (p.top_k <= 4) return launch_combine<T, BYTES, 4>(p, st);
  return launch_combine<T, BYTES, 8>(p, st);
}
// `unit`: the bytes of an access that all rows allow.
template <typename T, typename Params>
cudaError_t choose_unit(Params& p, int64_t bytes, int unit, cudaStream_t st) {
  if (unit == 16) return choose_rows<T, 16>(p, bytes, st);
  if constexpr (sizeof(T) == 2) {
    if (unit == 2) return choose_rows<T, 2>(p, bytes, st);
  }
  return choose_rows<T, 4>(p, bytes, st);
}
template <typename Params>
cudaError_t choose_type(Params& p, int type, int64_t cols, int unit, cudaStream_t st) {
  if (type == DS_TYPE_F32) return choose_unit<float>(p, cols * 4, unit, st);
  if (type == DS_TYPE_BF16) return choose_unit<__nv_bfloat16>(p, cols * 2, unit, st);
  return choose_unit<__half>(p, cols * 2, unit, st);
}

// 16 where the row's bytes and these rows' addresses are multiples of it, else 4, else 2.
struct Rows {
  const void* p;
  int64_t ld;
};
template <size_t N>
int unit_of(int64_t bytes, const Rows (&rows)[N]) {
  for (int u = 16; u > 2; u /= 4) {
    bool all = bytes % u == 0;
    for (const Rows& r : rows) all = all && (r.p == nullptr || (aligned(r.p, u) && r.ld % u == 0));
    if (all) return u;
  }
  return 2;
}

// A cluster of so many CTAs; `at` has to live as long as the configuration.
cudaLaunchConfig_t order_config(unsigned ctas, unsigned threads, size_t smem, cudaLaunchAttribute* at) {
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = ctas;
  at[0].val.clusterDim.y = 1;
  at[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ctas);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cfg;
}

}  // namespace

cudaError_t launch_expert_order(const void* ids, int id_type, const ds_expert_slots& s, cudaStream_t st) {
  static const cudaError_t attr = [] {
    const int most = (int)sizeof(int) * DS_EXPERTS_MAX * (kOrderWarps + 2);
    const cudaError_t e = cudaFuncSetAttribute(order_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
    return e != cudaSuccess ? e
                            : cudaFuncSetAttribute(order_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
  }();
  if (attr != cudaSuccess) return attr;
  // CTAs of a cluster: 16 where the device takes so many of the largest size at once, else the portable 8
  static const int most_ctas = [] {
    cudaLaunchAttribute at[1];
    cudaLaunchConfig_t cfg = order_config(kMostCtas, kOrderThreads, sizeof(int) * DS_EXPERTS_MAX * (kOrderWarps + 2), at);
    int n = 0;
    const bool takes =
        cudaFuncSetAttribute(order_kernel<true>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess &&
        cudaOccupancyMaxActiveClusters(&n, order_kernel<true>, &cfg) == cudaSuccess && n > 0;
    if (!takes) cudaGetLastError();
    return takes ? (int)kMostCtas : 8;
  }();
  OrderParams p;
  p.ids = ids;
  p.offsets = s.offsets, p.counts = s.counts, p.position = s.position, p.slot = s.slot;
  p.slots = s.tokens * s.top_k, p.rows = s.rows;
  p.experts = s.experts, p.align = s.align, p.wide = id_type == DS_INDEX_I64;
  // warps for 32 slots each, and a thread for each expert
  int64_t threads = over(p.slots > p.experts ? p.slots : p.experts, 32) * 32;
  if (threads > kOrderThreads) threads = kOrderThreads;
  int ctas = 1;
  while (ctas < most_ctas && p.slots > (int64_t)ctas * threads) ctas *= 2;
  p.per_warp = over(over(p.slots, ctas * threads / 32), 32) * 32;
  const size_t smem = sizeof(int) * (size_t)p.experts * (size_t)(threads / 32 + 2);
  if (ctas == 1) {
    order_kernel<false><<<1, (unsigned)threads, smem, st>>>(p);
    return cudaGetLastError();
  }
  cudaLaunchAttribute at[1];
  cudaLaunchConfig_t cfg = order_config((unsigned)ctas, (unsigned)threads, smem, at);
  cfg.stream = st;
  return cudaLaunchKernelEx(&cfg, order_kernel<true>, p);
}

cudaError_t launch_expert_gather(const RowCopy& a, const RowCopy& b, const ds_expert_slots& s, cudaStream_t st) {
  GatherParams p = {};
  p.a = a, p.b = b;
  p.position = s.position, p.slot = s.slot;
  p.tokens = s.tokens, p.rows = s.rows, p.top_k = s.top_k;
  // rows of 8-bit values start at multiples of 16 bytes, and may end anywhere
  const int unit = b.dst ? 16 : unit_of(a.bytes, {Rows{a.src, a.ld_src}, Rows{a.dst, a.ld_dst}});
  if (unit == 16) return launch_gather<16>(p, st);
  return unit == 4 ? launch_gather<4>(p, st) : launch_gather<2>(p, st);
}

cudaError_t launch_expert_combine(const void* y, int type, int64_t ldy, int64_t cols, const ds_expert_slots& s,
                                  const float* weights, const void* add, int64_t ld_add, void* out, int64_t ldo,
                                  cudaStream_t st) {
  const int64_t size = type_size(type);
  CombineParams p = {};
  p.y = y, p.add = add, p.out = out, p.weights = weights;
  p.ldy = ldy * size, p.ld_add = ld_add * size, p.ldo = ldo * size;
  p.tokens = s.tokens, p.rows = s.rows, p.top_k = s.top_k;
  p.position = s.position;
  return choose_type(p, type, cols, unit_of(cols * size, {Rows{y, p.ldy}, Rows{add, p.ld_add}, Rows{out, p.ldo}}), st);
}

cudaError_t launch_expert_combine_backward(const void* dout, int64_t ldd, const void* y, int64_t ldy, int type,
                                           int64_t cols, const ds_expert_slots& s, const float* weights, void* dy,
                                           int64_t lddy, float* dweights, cudaStream_t st) {
  const int64_t size = type_size(type);
  CombineBackwardParams p = {};
  p.d = dout, p.y = y, p.dy = dy, p.weights = weights, p.dweights = dweights;
  p.ldd = ldd * size, p.ldy = ldy * size, p.lddy = lddy * size;
  p.tokens = s.tokens, p.rows = s.rows, p.top_k = s.top_k;
  p.position = s.position, p.slot = s.slot;
  return choose_type(p, type, cols, unit_of(cols * size, {Rows{dout, p.ldd}, Rows{y, p.ldy}, Rows{dy, p.lddy}}), st);
}

}  // namespace ds
