// Product of two 8-bit floating-point matrices with a scale per block of 128
// values of the reduction, on the 5th-generation tensor cores (sm_103a).
//
//   y[m][n] = bias[n] + add[m][n] + sum_b sx[m][b] sw[n][b] sum_{k in block b} qx[m][k] qw[n][k]
//
// A block's inner sum is four tcgen05.mma of kind::f8f6f4 (K = 32 each) into
// an accumulator of its own in tensor memory; it is then read back and added,
// times its two scales, to float32 sums in registers.  So scales may be any
// float32 and differ per row (a sum times either scale has to stay within the
// normal numbers), and no sum is held in fewer than 32 bits.
//
// The kernels are in f8_linear.cuh, which the experts' products share.
//
// linear_f8_kernel lays 128 rows of w along the lanes of tensor memory and BN
// rows of x along its columns: with one token in flight the weights, which
// are all the traffic, still fill the tensor core's 128 lanes.  A
// thread-block cluster splits the reduction of one tile and its CTAs add
// their parts through distributed shared memory in rank order, so results do
// not depend on timing.  Measured: 1 x 4096 x 4096 7.7 us (2.2 TB/s; 6.5 with
// the weights in L2; an empty launch of clusters takes 3), 300 x 1000 x 2050
// 8.7 us, 128 x 8192 x 4096 15.7 us (2.1 TB/s).
#include <atomic>

#include "f8_linear.cuh"

namespace ds {

namespace {

std::atomic<long long> g_wait_cycles{kTimeoutCycles};

template <bool COLS, bool WIDE, int N>
cudaError_t launch_big(const CUtensorMap& mx, const CUtensorMap& mw, const Params& p, cudaStream_t st) {
  using Cfg = BigCfg<COLS, N>;
  static const cudaError_t attr = cudaFuncSetAttribute(
      linear_f8_big_kernel<COLS, WIDE, TileOrder<N>>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Cfg::SMEM);
  if (attr != cudaSuccess) return attr;
  TileOrder<N> t{(uint32_t)((p.M + ROWS - 1) / ROWS), (uint32_t)((p.N + N - 1) / N), 1};
  const uint32_t sms = sm_count() > 0 ? sm_count() : 1, count = t.tiles_m * t.tiles_n, grid = count < sms ? count : sms;
  t.G = (grid + t.tiles_n - 1) / t.tiles_n;  // about one wave of tiles per group
  if (t.G > t.tiles_m) t.G = t.tiles_m;
  linear_f8_big_kernel<COLS, WIDE, TileOrder<N>><<<grid, Cfg::THREADS, Cfg::SMEM, st>>>(mx, mw, p, t);
  return cudaGetLastError();
}

template <int N>
cudaError_t start_big(const CUtensorMap& mx, const CUtensorMap& mw, const Params& p, bool wide, cudaStream_t st) {
  if (p.w.shift) return wide ? launch_big<false, true, N>(mx, mw, p, st) : launch_big<false, false, N>(mx, mw, p, st);
  return wide ? launch_big<true, true, N>(mx, mw, p, st) : launch_big<true, false, N>(mx, mw, p, st);
}

template <int BN>
cudaError_t launch(const CUtensorMap& mw, const CUtensorMap& mx, const Params& p, int split, cudaStream_t st) {
  constexpr size_t smem = smem_bytes<BN>();
  static_assert(Cfg<BN>::CTAS * (smem + 1024) <= 233472, "CTAs of an SM");
  // once per process, thread-safe (function-local static)
  static const cudaError_t attr =
      cudaFuncSetAttribute(linear_f8_kernel<BN, OnePlace<BN>>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (attr != cudaSuccess) return attr;
  const int64_t tiles = (p.M + BN - 1) / BN * ((p.N + ROWS - 1) / ROWS);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * split));
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
  return cudaLaunchKernelEx(&cfg, linear_f8_kernel<BN, OnePlace<BN>>, mw, mx, p, split, OnePlace<BN>{});
}

// Which kernel: the time of each that could run is estimated, in microseconds, by a fit to its measured times on one
// GB300 (720 products of N 512 .. 8192, K 512 .. 5632, M 1 .. 3000 in a stream; bf16 results).  The large kernel takes
// 3.5 to start, and a wave of its tiles 1.3 and 0.60 a block of the reduction (0.79 with a scale per row of w), of half
// tiles 0.7 and 0.40 (0.53).  A wave of the small kernel takes 3.8, 4.0 or 4.2 and 0.23, 0.24 or 0.38 a block for BN =
// 16, 32, 64, 1.6 times the latter where two CTAs share an SM; to that come 0.6 for each CTA of an SM in turn, and 0.4
// (0.6) for a cluster (of 8).  Splitting a reduction divides the blocks of a CTA and multiplies the CTAs; a cluster of 8
// finds room for 27 / 32 of the CTAs that would fit one by one.  Stores of rows that are not aligned add 0.013 a column
// of a tile (0.02 in the small kernel; 4096 x 1024 x 4097 takes 44 us, 31 with 4096 columns).  The choice takes 0.5%
// more than the best of all on average, 24% at most.
struct Plan {
  int bn, split, big;  // big: rows of w per tile of the large kernel, or 0
};
Plan plan_of(const Params& p, bool wide) {
  const int64_t sms = sm_count() > 0 ? sm_count() : 1;
  auto over = [](int64_t n, int64_t d) { return (n + d - 1) / d; };
  Plan best{16, 1, 0};
  double least = 1e30;
  auto consider = [&](int bn, int split, int big, double time) {
    if (time < 0.99 * least) best = Plan{bn, split, big}, least = time;
  };
  const struct {
    int bn;
    double wave, block;
  } small[3] = {{16, 3.8, 0.23}, {32, 4.0, 0.24}, {64, 4.2, 0.38}};
  for (const auto& k : small) {
    for (int split = 1; split <= 8 && (split == 1 || split <= p.nk); split *= 2) {
      const int64_t ctas = over(p.M, k.bn) * over(p.N, ROWS) * split, room = split < 8 ? sms : sms * 27 / 32;
      const double wave = k.wave + k.block * (ctas > room ? 1.6 : 1.0) * (double)over(p.nk, split) +
                          (p.vec ? 0.0 : 0.02 * k.bn / split);
      consider(k.bn, split, 0,
               (double)over(ctas, 2 * room > 0 ? 2 * room : 1) * wave + 0.6 * (double)ctas / (double)sms +
                   (split == 1 ? 0.0 : (split < 8 ? 0.4 : 0.6)));
    }
  }
  if (p.nk > 0) {
    for (int big = 256; big >= 128; big /= 2) {
      const double block = big == 256 ? (p.w.shift ? 0.60 : 0.79) : (p.w.shift ? 0.40 : 0.53);
      const double wave = (big == 256 ? 1.3 : 0.7) + (wide ? 0.0 : 0.013 * big) + block * p.nk;
      consider(0, 1, big, 3.5 + (double)over(over(p.M, ROWS) * over(p.N, big), sms) * wave);
    }
  }
  return best;
}

Params params_of(const LinearF8Params& l) {
  Params p = {};
  p.x = scales_at(l.x);
  p.w = scales_at(l.w);
  p.bias = l.bias;
  p.add = l.add;
  p.y = l.y;
  p.M = l.x->rows;
  p.N = l.w->rows;
  p.ld_add = l.ld_add;
  p.ldy = l.ldy;
  p.nk = (int)((l.x->cols + BK - 1) / BK);
  p.idesc = idesc_of(l.w, l.x);
  p.type = l.type;
  const size_t size = l.type == DS_TYPE_F32 ? 4 : 2;
  p.vec = reinterpret_cast<uintptr_t>(l.y) % (4 * size) == 0 && l.ldy % 4 == 0 &&
          (l.add == nullptr || (reinterpret_cast<uintptr_t>(l.add) % 16 == 0 && l.ld_add % 4 == 0));
  p.pairs = reinterpret_cast<uintptr_t>(l.y) % (2 * size) == 0 && l.ldy % 2 == 0 &&
            (l.add == nullptr || (reinterpret_cast<uintptr_t>(l.add) % 8 == 0 && l.ld_add % 2 == 0));
  auto aligned = [&](int n) {
    return reinterpret_cast<uintptr_t>(p.x.s) % (4 * n) == 0 && p.x.ld % n == 0 &&
           reinterpret_cast<uintptr_t>(p.w.s) % (4 * n) == 0 && p.w.ld % n == 0;
  };
  p.aligned = aligned(8) ? 8 : (aligned(4) ? 4 : 1);
  p.wait_cycles = f8_wait_cycles();
  return p;
}
// Whether the large kernel's stores of eight values are aligned.
bool wide_of(const LinearF8Params& l, const Params& p) {
  const size_t size = l.type == DS_TYPE_F32 ? 4 : 2;
  return p.vec && reinterpret_cast<uintptr_t>(l.y) % (8 * size) == 0 && l.ldy % 8 == 0;
}

}  // namespace

int linear_f8_tile(const LinearF8Params& l) {
  const Params p = params_of(l);
  const Plan plan = plan_of(p, wide_of(l, p));
  return plan.big ? plan.big : plan.bn;
}

cudaError_t launch_linear_f8(const LinearF8Params& l, cudaStream_t st) {
  Params p = params_of(l);
  const bool wide = wide_of(l, p);
  const Plan plan = plan_of(p, wide);
  CUtensorMap mw = {}, mx = {};  // an empty reduction loads nothing
  if (p.nk > 0 && (!make_map(&mw, l.w, plan.big ? plan.big : ROWS) || !make_map(&mx, l.x, plan.big ? ROWS : plan.bn)))
    return cudaErrorInvalidValue;
  if (plan.big) p.idesc = idesc_of(l.x, l.w);  // x along the lanes
  if (plan.big == 256) return start_big<256>(mx, mw, p, wide, st);
  if (plan.big == 128) return start_big<128>(mx, mw, p, wide, st);
  switch (plan.bn) {
    case 16: return launch<16>(mw, mx, p, plan.split, st);
    case 32: return launch<32>(mw, mx, p, plan.split, st);
    default: return launch<64>(mw, mx, p, plan.split, st);
  }
}

void set_f8_wait_cycles(long long cycles) {
  g_wait_cycles.store(cycles > 0 ? cycles : kTimeoutCycles, std::memory_order_relaxed);
}

long long f8_wait_cycles() { return g_wait_cycles.load(std::memory_order_relaxed); }

int read_f8_fault_flag() { return read_and_clear_fault(); }

}  // namespace ds
