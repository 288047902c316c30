// Products of the experts' parts with 8-bit operands: the persistent kernel of
// large products (f8_linear.cuh) over the tiles of all experts.  Which rows an
// expert has is known on the device only, so every CTA makes the list of the
// tiles from the segments' offsets when it starts; nothing waits for the host.
//
// What bounds them: as the dense product, the read-back and sums of a block
// beside its products; neither the tensor cores (34% of the time) nor issue
// slots (47%) are full, nor L2, which gives 3.2 GB of operands, 9.5 TB/s.
// 8192 x 4 rows of 32 experts, 2048 -> 4096: 338 us, 1.63 PFLOP/s (the dense
// product of as many rows 323); weight gradients of 32 x 2048 x 2048 added to
// others 280 us (223 without), of which the products take 144 and the sums' way
// out and in the rest.  With few
// rows an expert, its weights from memory: 16 x 4 rows of the same experts 35
// us, 5.3 TB/s of the weights met.
#include "experts.cuh"
#include "f8_linear.cuh"

namespace ds {
namespace {

// One expert's part of the output, for the stores, and a tile's place in it.
struct OutputPart {
  const float *bias, *add;
  void* y;
  int64_t M, N, ld_add, ldy;
  int type, vec, pairs;
  int m0, n0;
};

// y = x w_e^T by the kernel of small products: a CTA's tile among those of all experts.  Every warp finds it for itself,
// by the number of row tiles before each expert, so that no barrier is needed.
template <int BN>
struct SegmentPlace {
  const int32_t* offsets;
  int experts;
  uint32_t rows, cols, tiles_n;
  int m0, n0, e, end;  // of the tile: rows of x and w, the expert (`experts`: rows that none has), the segment's end

  __device__ __forceinline__ uint32_t first_row(int i) const {
    const uint32_t o = i <= experts ? (uint32_t)offsets[i] : rows;
    return o < rows ? o : rows;
  }
  __device__ __forceinline__ bool find(const Params&, uint32_t tile) {
    const uint32_t rt = tile / tiles_n, lane = threadIdx.x & 31;
    const int per = (experts + 1 + 31) / 32, from = (int)lane * per;
    const int to = from + per < experts + 1 ? from + per : experts + 1;
    auto row_tiles = [&](uint32_t a, uint32_t b) { return b > a ? (b - a + BN - 1) / BN : 0u; };
    uint32_t sum = 0, row = from < to ? first_row(from) : 0;
    for (int i = from; i < to; ++i) {
      const uint32_t next = first_row(i + 1);
      sum += row_tiles(row, next);
      row = next;
    }
    uint32_t upto = sum;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const uint32_t up = __shfl_up_sync(0xFFFFFFFFu, upto, d);
      if (lane >= d) upto += up;
    }
    const uint32_t here = __ballot_sync(0xFFFFFFFFu, rt < upto);
    if (here == 0) return false;
    const int src = __ffs(here) - 1;
    uint32_t left = rt - (upto - sum);
    if ((int)lane == src) {
      row = first_row(from);
      for (int i = from; i < to; ++i) {
        const uint32_t next = first_row(i + 1), n = row_tiles(row, next);
        if (left < n) {
          e = i, m0 = (int)(row + left * BN), end = (int)next;
          break;
        }
        left -= n;
        row = next;
      }
    }
    e = __shfl_sync(0xFFFFFFFFu, e, src);
    m0 = __shfl_sync(0xFFFFFFFFu, m0, src);
    end = __shfl_sync(0xFFFFFFFFu, end, src);
    n0 = (int)((uint32_t)e * cols + (tile - rt * tiles_n) * ROWS);
    return true;
  }
  __device__ __forceinline__ int blocks(const Params& P) const { return e < experts ? P.nk : 0; }
  __device__ __forceinline__ OutputPart output(const Params& P) const {
    return OutputPart{e < experts && P.bias ? P.bias + (int64_t)e * cols : nullptr,
                      nullptr, P.y, (int64_t)end, (int64_t)cols, 0, P.ldy, P.type, P.vec, P.pairs, m0, column(P)};
  }
  __device__ __forceinline__ int column(const Params&) const { return n0 - (int)((uint32_t)e * cols); }
};

// y = x w_e^T.  Tiles of expert after expert, and behind them those of the rows that no expert has (no blocks: zeros).
template <int COLS_OF_TILE>
struct SegmentTiles {
  static constexpr int N = COLS_OF_TILE;
  static constexpr bool WALKS = true;
  static constexpr bool ADDS = false;  // whether sums are added to others' that are asked for ahead
  static constexpr uint32_t GROUP = 16;  // row tiles that share columns, as TileOrder::G
  const int32_t* offsets;
  int experts;
  uint32_t rows, cols, tiles_n;
  uint32_t* start;  // shared memory: [experts + 2], first rows of the segments; the last two: rows in use, all rows
  uint32_t* first;  // [experts + 2], first tiles
  static size_t bytes(int experts) { return (size_t)(experts + 2) * 8; }

  __device__ __forceinline__ SegmentTiles ready(const Params&, void* at) const {
    SegmentTiles s = *this;
    s.start = static_cast<uint32_t*>(at);
    s.first = s.start + experts + 2;
    for (int e = threadIdx.x; e < experts + 2; e += blockDim.x) {
      const uint32_t o = e <= experts ? (uint32_t)offsets[e] : rows;
      s.start[e] = o < rows ? o : rows;
    }
    __syncthreads();
    if (threadIdx.x < 32) {  // a lane counts the tiles of some experts in a row
      const int per = (experts + 1 + 31) / 32, from = threadIdx.x * per;
      uint32_t sum = 0;
      for (int e = from; e < from + per && e <= experts; ++e) sum += s.tiles_m(e) * tiles_n;
      uint32_t upto = sum;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const uint32_t up = __shfl_up_sync(0xFFFFFFFFu, upto, d);
        if (threadIdx.x >= d) upto += up;
      }
      uint32_t at_tile = upto - sum;
      for (int e = from; e < from + per && e <= experts; ++e) {
        s.first[e] = at_tile;
        at_tile += s.tiles_m(e) * tiles_n;
      }
      if (threadIdx.x == 31) s.first[experts + 1] = upto;
    }
    return s;  // a barrier follows before it is used
  }
  __device__ __forceinline__ uint32_t tiles_m(int e) const {
    return start[e + 1] > start[e] ? (start[e + 1] - start[e] + ROWS - 1) / ROWS : 0u;
  }
  // Experts are met in order: a walk looks at the next ones' first tiles instead of searching, which took 2 us a tile.
  struct Walk {
    uint32_t t;
    int e;
    __device__ __forceinline__ void seek(const SegmentTiles& o) {
      while (e <= o.experts && t >= o.first[e + 1]) ++e;
    }
    __device__ __forceinline__ bool ended(const SegmentTiles& o) const { return e > o.experts; }
    __device__ __forceinline__ void next(const SegmentTiles& o) {
      t += gridDim.x;
      seek(o);
    }
    __device__ __forceinline__ int blocks(const Params& P, const SegmentTiles& o) const { return e < o.experts ? P.nk : 0; }
    __device__ __forceinline__ Tile tile(const Params& P, const SegmentTiles& o) const {
      int tm, tn;
      grouped(t - o.first[e], o.tiles_m(e), o.tiles_n, GROUP, tm, tn);
      return Tile{(int)o.start[e] + tm * ROWS, (int)((uint32_t)e * o.cols) + tn * N, 0, blocks(P, o)};
    }
    __device__ __forceinline__ OutputPart output(const Params& P, const SegmentTiles& o) const {
      const Tile at = tile(P, o);
      return OutputPart{e < o.experts && P.bias ? P.bias + (int64_t)e * o.cols : nullptr,
                        nullptr, P.y, (int64_t)o.start[e + 1], (int64_t)o.cols, 0, P.ldy, P.type, P.vec, P.pairs,
                        at.m0, at.n0 - (int)((uint32_t)e * o.cols)};
    }
  };
  __device__ __forceinline__ Walk walk() const {
    Walk w{blockIdx.x, 0};
    w.seek(*this);
    return w;
  }
  __device__ __forceinline__ int64_t blocks(const Params& P) const {
    const uint32_t n = first[experts], mine = blockIdx.x < n ? (n - blockIdx.x - 1) / gridDim.x + 1 : 0;
    return (int64_t)mine * P.nk;
  }
  __device__ __forceinline__ int aligned(const Params& P, const Tile&) const { return P.aligned; }
};

// dw_e = dy_t x_t^T over the blocks of each segment: P.x is dy_t, P.w is x_t.  An expert without rows has tiles without
// blocks.
template <int COLS_OF_TILE>
struct GradientTiles {
  static constexpr int N = COLS_OF_TILE;
  static constexpr bool WALKS = true, ADDS = true;
  const int32_t* offsets;
  int experts;
  uint32_t rows, tiles_m, tiles_n, G;
  uint32_t* start;  // shared memory: [experts + 1], first blocks of the segments
  static size_t bytes(int experts) { return (size_t)(experts + 1) * 4; }

  __device__ __forceinline__ GradientTiles ready(const Params&, void* at) const {
    GradientTiles s = *this;
    s.start = static_cast<uint32_t*>(at);
    for (int e = threadIdx.x; e <= experts; e += blockDim.x) {
      const uint32_t o = (uint32_t)offsets[e];
      s.start[e] = ((o < rows ? o : rows) + BK - 1) / BK;
    }
    __syncwarp();  // one warp allocates tensor memory next, all its lanes together
    return s;
  }
  __device__ __forceinline__ int blocks_of_expert(int e) const {
    return start[e + 1] > start[e] ? (int)(start[e + 1] - start[e]) : 0;
  }
  struct Walk {
    uint32_t r;  // of the expert's tiles
    int e;
    __device__ __forceinline__ void seek(const GradientTiles& o) {
      while (r >= o.tiles_m * o.tiles_n) {
        r -= o.tiles_m * o.tiles_n;
        ++e;
      }
    }
    __device__ __forceinline__ bool ended(const GradientTiles& o) const { return e >= o.experts; }
    __device__ __forceinline__ void next(const GradientTiles& o) {
      r += gridDim.x;
      seek(o);
    }
    __device__ __forceinline__ int blocks(const Params&, const GradientTiles& o) const { return o.blocks_of_expert(e); }
    __device__ __forceinline__ Tile tile(const Params& P, const GradientTiles& o) const {
      int tm, tn;
      grouped(r, o.tiles_m, o.tiles_n, o.G, tm, tn);
      return Tile{tm * ROWS, tn * N, (int)o.start[e], blocks(P, o)};
    }
    __device__ __forceinline__ OutputPart output(const Params& P, const GradientTiles& o) const {
      const int64_t row = (int64_t)e * P.M;
      const Tile at = tile(P, o);
      return OutputPart{nullptr, P.add ? P.add + row * P.ld_add : nullptr, static_cast<float*>(P.y) + row * P.ldy,
                        P.M, P.N, P.ld_add, P.ldy, DS_TYPE_F32, P.vec, P.pairs, at.m0, at.n0};
    }
  };
  __device__ __forceinline__ Walk walk() const {
    Walk w{blockIdx.x, 0};
    w.seek(*this);
    return w;
  }
  __device__ __forceinline__ int64_t blocks(const Params& P) const {
    int64_t n = 0;
    for (Walk w = walk(); !w.ended(*this); w.next(*this)) n += w.blocks(P, *this);
    return n;
  }
  __device__ __forceinline__ int aligned(const Params& P, const Tile& t) const {
    return P.aligned == 8 && t.kb0 % 8 == 0 ? 8 : (P.aligned >= 4 && t.kb0 % 4 == 0 ? 4 : 1);
  }
};

template <bool COLS, bool WIDE, typename Order>
cudaError_t launch(const CUtensorMap& mx, const CUtensorMap& mw, const Params& p, const Order& order, int64_t most,
                   cudaStream_t st) {
  using Cfg = BigCfg<COLS, Order::N>;
  static const cudaError_t attr =
      cudaFuncSetAttribute(linear_f8_big_kernel<COLS, WIDE, Order>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                           (int)(Cfg::SMEM + Order::bytes(DS_EXPERTS_MAX)));
  if (attr != cudaSuccess) return attr;
  static_assert(Cfg::SMEM + (DS_EXPERTS_MAX + 2) * 8 <= 232448, "shared memory of a CTA");
  const int64_t sms = sm_count() > 0 ? sm_count() : 1;
  linear_f8_big_kernel<COLS, WIDE, Order><<<(unsigned)(most < sms ? most : sms), Cfg::THREADS,
                                            Cfg::SMEM + Order::bytes(order.experts), st>>>(mx, mw, p, order);
  return cudaGetLastError();
}

template <typename Order>
cudaError_t start(const CUtensorMap& mx, const CUtensorMap& mw, const Params& p, const Order& order, int64_t most, bool wide,
                  cudaStream_t st) {
  if (p.w.shift)
    return wide ? launch<false, true>(mx, mw, p, order, most, st) : launch<false, false>(mx, mw, p, order, most, st);
  return wide ? launch<true, true>(mx, mw, p, order, most, st) : launch<true, false>(mx, mw, p, order, most, st);
}

// What both products' parameters have in common; wide: rows are aligned for stores of eight values.
Params params_of(const ExpertProduct& e, const ds_f8_matrix* x, const ds_f8_matrix* w, bool* wide) {
  Params p = {};
  p.x = scales_at(x);
  p.w = scales_at(w);
  p.bias = e.bias;
  p.add = e.add;
  p.y = e.y;
  p.M = x->rows;
  p.N = w->rows;
  p.ld_add = e.ld_add;
  p.ldy = e.ldy;
  p.nk = (int)((x->cols + BK - 1) / BK);
  p.idesc = idesc_of(x, w);
  p.type = e.type;
  const size_t size = e.type == DS_TYPE_F32 ? 4 : 2;
  auto rows = [&](int n) {
    return aligned(e.y, n * size) && e.ldy % n == 0;
  };
  p.vec = rows(4) && (e.add == nullptr || (aligned(e.add, 16) && e.ld_add % 4 == 0));
  p.pairs = rows(2) && (e.add == nullptr || (aligned(e.add, 8) && e.ld_add % 2 == 0));
  *wide = p.vec && rows(8);
  auto scales = [&](int n) {
    return aligned(p.x.s, 4 * n) && p.x.ld % n == 0 && aligned(p.w.s, 4 * n) && p.w.ld % n == 0;
  };
  p.aligned = scales(8) ? 8 : (scales(4) ? 4 : 1);
  p.wait_cycles = f8_wait_cycles();
  return p;
}

int64_t over(int64_t n, int64_t d) { return (n + d - 1) / d; }

// Whether tiles of 128 columns take less time than those of 256, by the estimate of the dense product's tiles (1.3 us and
// 0.6 a block, 0.7 and 0.4 for half the width, 0.013 a column where rows are not aligned) for experts of as many rows
// each: 512 x 4 slots, 32 experts of 2048 -> 512 18.7 us, 20.9 with 256; 600 tokens to 4 of 1024 -> 2048 10.2, 12.6;
// 4096 x 2, 8 of 1024 -> 512 14.5, 13.0; 3000 x 6, 60 of 700 -> 333 32.5, 40.6.
bool narrow_tiles(const ExpertProduct& e, int64_t slots, int64_t met) {
  bool wide;
  const Params p = params_of(e, e.x, e.w, &wide);
  const int64_t cols = e.w->rows / e.s->experts, rows = slots / ROWS + (met + 1) / 2, sms = sm_count() > 0 ? sm_count() : 1;
  auto time = [&](int n, double tile, double block) {
    return (double)over(rows * over(cols, n), sms) * (tile + block * p.nk + (wide ? 0.0 : 0.013 * n));
  };
  return time(128, 0.7, 0.4) < time(256, 1.3, 0.6);
}

template <int N>
cudaError_t linear(const ExpertProduct& e, cudaStream_t st) {
  bool wide;
  const Params p = params_of(e, e.x, e.w, &wide);
  const int64_t cols = e.w->rows / e.s->experts;
  CUtensorMap mx = {}, mw = {};
  if (p.nk > 0 && (!make_map(&mx, e.x, ROWS) || !make_map(&mw, e.w, N))) return cudaErrorInvalidValue;
  SegmentTiles<N> t = {};
  t.offsets = e.s->offsets;
  t.experts = e.s->experts;
  t.rows = (uint32_t)e.s->rows;
  t.cols = (uint32_t)cols;
  t.tiles_n = (uint32_t)over(cols, N);
  const int64_t most = (over(e.s->rows, ROWS) + e.s->experts) * t.tiles_n;
  return start(mx, mw, p, t, most, wide, st);
}

// `met`: experts that may have rows.
template <int BN>
cudaError_t linear_small(const ExpertProduct& e, int64_t met, cudaStream_t st) {
  using Place = SegmentPlace<BN>;
  constexpr size_t smem = smem_bytes<BN>();
  static const cudaError_t attr =
      cudaFuncSetAttribute(linear_f8_kernel<BN, Place>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (attr != cudaSuccess) return attr;
  bool wide;
  Params p = params_of(e, e.x, e.w, &wide);
  p.idesc = idesc_of(e.w, e.x);  // w along the lanes
  CUtensorMap mx = {}, mw = {};
  if (p.nk > 0 && (!make_map(&mx, e.x, BN) || !make_map(&mw, e.w, ROWS))) return cudaErrorInvalidValue;
  Place place = {};
  place.offsets = e.s->offsets;
  place.experts = e.s->experts;
  place.rows = (uint32_t)e.s->rows;
  place.cols = (uint32_t)(e.w->rows / e.s->experts);
  place.tiles_n = (uint32_t)over(place.cols, ROWS);
  // enough for any choice of experts; the reduction is split while the experts that are likely met leave SMs without work
  const int64_t most = over(e.s->rows, BN) + met + 1, likely = met * place.tiles_n;
  int split = 1;
  while (split < 8 && 2 * split <= p.nk && 2 * split * likely <= 2 * (int64_t)(sm_count() > 0 ? sm_count() : 1)) split *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(most * place.tiles_n * split));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned)split;
  at[0].val.clusterDim.y = 1;
  at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, linear_f8_kernel<BN, Place>, mw, mx, p, split, place);
}

template <int N, bool WIDE>
cudaError_t weight_grad(const ExpertProduct& e, cudaStream_t st) {
  bool wide;
  const Params p = params_of(e, e.w, e.x, &wide);
  CUtensorMap mx = {}, mw = {};
  if (p.nk > 0 && (!make_map(&mx, e.w, ROWS) || !make_map(&mw, e.x, N))) return cudaErrorInvalidValue;
  GradientTiles<N> t = {};
  t.offsets = e.s->offsets;
  t.experts = e.s->experts;
  t.rows = (uint32_t)e.s->rows;
  t.tiles_m = (uint32_t)over(p.M, ROWS);
  t.tiles_n = (uint32_t)over(p.N, N);
  t.G = t.tiles_m < 12 ? t.tiles_m : 12;  // about one wave of tiles is a square
  const int64_t tiles = (int64_t)t.experts * t.tiles_m * t.tiles_n;
  return p.w.shift ? launch<false, WIDE>(mx, mw, p, t, tiles, st) : launch<true, WIDE>(mx, mw, p, t, tiles, st);
}

}  // namespace

// The kernel of small products while an expert has few rows, its tile's rows of x above their mean (experts differ); us of
// 32 experts of 2048 x 4096, 4 of them for each of so many tokens, with 16, 32, 64 rows and by the large kernel:
//   1 token 9.3, 9.8, 12.3, 19.4;  16: 35, 36, 39, 45;  64: 48, 47, 52, 58;  128: 61, 52, 55, 59;  256: 88, 67, 61, 63;
//   512: 147, 97, 82, 63
// Over 11 shapes of 4 to 512 experts, K of 512 to 4096, N of 333 to 4096 and up to 160 rows an expert the choice is 2% above
// the best of these kernels in the mean.  12 of 165 products are more than 10% above it: those next to a border (4 experts of
// 8 rows 13.3, 10.1 with 32), tiles of 256 columns where 128 are better (256 experts of 1024 -> 512, 72 rows each 59, 52.5),
// and 60 to 160 rows an expert that are not aligned (60 experts of 700 -> 333: 19.4 to 27, 12.4 to 22.5 with 64 rows a tile).
cudaError_t launch_expert_linear_f8(const ExpertProduct& e, cudaStream_t st) {
  const int64_t slots = e.s->tokens * e.s->top_k, met = slots < e.s->experts ? slots : e.s->experts;
  const int64_t each = met > 0 ? over(over(slots, met), e.s->align) * e.s->align : 0;  // gaps are multiplied too
  if (each <= 10) return linear_small<16>(e, met, st);
  if (each <= 21) return linear_small<32>(e, met, st);
  if (each <= 42) return linear_small<64>(e, met, st);
  return narrow_tiles(e, slots, met) ? linear<128>(e, st) : linear<256>(e, st);
}

// Tiles of half the width where rows of dw are not aligned: 60 x 333 x 700 from 3000 x 6 slots 37 us, 46 with 256 columns;
// elsewhere they take 1 to 5% more or less.
cudaError_t launch_expert_weight_grad_f8(const ExpertProduct& e, cudaStream_t st) {
  bool wide;
  params_of(e, e.w, e.x, &wide);
  return wide ? weight_grad<256, true>(e, st) : weight_grad<128, false>(e, st);
}

int read_expert_f8_fault_flag() { return read_and_clear_fault(); }

}  // namespace ds
