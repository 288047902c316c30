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

constexpr int kThreads = 256;
constexpr int kEpiWarps = 4;

// STAGES of the data ring, ACC accumulators in tensor memory, CTAs that share an SM.
template <int BN>
struct Cfg;
template <>
struct Cfg<16> {
  static constexpr int STAGES = 5, ACC = 4, CTAS = 2;
};
template <>
struct Cfg<32> {
  static constexpr int STAGES = 5, ACC = 4, CTAS = 2;
};
template <>
struct Cfg<64> {
  static constexpr int STAGES = 4, ACC = 4, CTAS = 2;
};

template <int BN>
struct __align__(16) Shared {
  static constexpr int SLOTS = Cfg<BN>::STAGES + Cfg<BN>::ACC + 1;  // of scales: see kScaleSlots
  float scale[SLOTS][ROWS + BN];                                    // rows of w, then rows of x
  uint64_t full[Cfg<BN>::STAGES];   // a stage's copies and scales have come
  uint64_t mult[Cfg<BN>::STAGES];   // its products are done
  uint64_t tempty[Cfg<BN>::ACC];    // an accumulator has been read
  uint64_t done;
  uint32_t tmem_base;
  int abort;
};

template <int BN>
constexpr size_t smem_bytes() {
  return (size_t)Cfg<BN>::STAGES * (ROWS + BN) * BK + sizeof(Shared<BN>) + 1024;
}

// One tile: 128 rows of w (n0 ..), BN rows of x (m0 ..).  blockIdx.x = tile * split + rank in the cluster; the rank
// takes the blocks [rank nk / split, (rank + 1) nk / split) of the reduction.  Warp 0 loads, warp 1 multiplies, warps 2
// and 3 bring scales (as in the large kernel below), warps 4-7 add.
template <int BN>
__global__ void __launch_bounds__(kThreads, Cfg<BN>::CTAS) linear_f8_kernel(const __grid_constant__ CUtensorMap tmap_w,
                                                             const __grid_constant__ CUtensorMap tmap_x,
                                                             const Params P, const int split) {
  constexpr int STAGES = Cfg<BN>::STAGES, ACC = Cfg<BN>::ACC;
  constexpr int A_BYTES = ROWS * BK, STAGE_BYTES = A_BYTES + BN * BK;
  constexpr int TMEM_COLS = ACC * BN;
  static_assert(TMEM_COLS >= 32 && TMEM_COLS <= 512, "tensor memory");
  static_assert(STAGES * STAGE_BYTES >= BN * ROWS * 4, "the ring holds the exchanged sums");
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  unsigned char* ring = reinterpret_cast<unsigned char*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  Shared<BN>* sh = reinterpret_cast<Shared<BN>*>(ring + STAGES * STAGE_BYTES);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t tiles_n = (uint32_t)((P.N + ROWS - 1) / ROWS);
  const uint32_t tile = blockIdx.x / split;
  const int rank = (int)(blockIdx.x - tile * split);
  const uint32_t tm = tile / tiles_n;
  const int n0 = (int)(tile - tm * tiles_n) * ROWS, m0 = (int)tm * BN;
  const int kb0 = (int)((int64_t)P.nk * rank / split);
  const int nk = (int)((int64_t)P.nk * (rank + 1) / split) - kb0;
  volatile int* abort = &sh->abort;

  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(&sh->full[s], 3);  // the copies, and two warps with scales
      mbar_init(&sh->mult[s], 1);
    }
    for (int b = 0; b < ACC; ++b) mbar_init(&sh->tempty[b], kEpiWarps);
    mbar_init(&sh->done, 1);
    sh->abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh->tmem_base)),
                 "r"(TMEM_COLS)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem_base = sh->tmem_base;

  uint64_t acc[BN / 2];
#pragma unroll
  for (int j = 0; j < BN / 2; ++j) acc[j] = 0;

  if (warp == 0) {
    if (lane == 0) {
      Ring<STAGES> st;
      int i = 0;
      for (; i < nk; ++i, st.next()) {
        if (!mbar_wait(&sh->mult[st.slot], st.parity ^ 1u, abort, P.wait_cycles, &g_f8_fault)) break;
        unsigned char* a = ring + st.slot * STAGE_BYTES;
        mbar_expect_tx(&sh->full[st.slot], STAGE_BYTES);
        tma_load_2d(a, &tmap_w, &sh->full[st.slot], (kb0 + i) * BK, n0);
        tma_load_2d(a + A_BYTES, &tmap_x, &sh->full[st.slot], (kb0 + i) * BK, m0);
      }
      // the last copies issued land before the CTA leaves
      for (int j = i > STAGES ? i - STAGES : 0; j < i; ++j)
        mbar_drain(&sh->full[j % STAGES], (uint32_t)(j / STAGES) & 1u, *abort ? kLandedCycles : kTimeoutCycles);
    }
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t idesc = P.idesc | ((uint32_t)(BN >> 3) << 17) | ((uint32_t)(ROWS >> 4) << 24);
      const uint64_t adesc = sw128_desc(smem_u32(ring)), bdesc = sw128_desc(smem_u32(ring) + A_BYTES);
      Ring<STAGES> st;
      Ring<ACC> ac;
      for (int i = 0; i < nk; ++i, st.next(), ac.next()) {
        if (!mbar_wait(&sh->full[st.slot], st.parity, abort, P.wait_cycles, &g_f8_fault) ||
            !mbar_wait(&sh->tempty[ac.slot], ac.parity ^ 1u, abort, P.wait_cycles, &g_f8_fault))
          break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint64_t at = (uint64_t)(st.slot * (STAGE_BYTES >> 4));
#pragma unroll
        for (int k = 0; k < BK / 32; ++k)
          umma_f8(tmem_base + ac.slot * BN, adesc + at + 2 * k, bdesc + at + 2 * k, idesc, k > 0);
        umma_commit(&sh->mult[st.slot]);
      }
      // every MMA issued by this CTA has completed before its memory is used again
      umma_commit(&sh->done);
      mbar_drain(&sh->done, 0u);
    }
  } else if (warp < 4) {
    constexpr int XROWS = (BN + 63) / 64, PER = 2 + XROWS, GROUP = 4;
    const int j = threadIdx.x - 64;
    ScaleFeed<PER, GROUP> feed;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int64_t n = n0 + j + 64 * i, m = m0 + j + 64 * (i - 2);
      feed.src[i] = nullptr;
      if (i < 2) {
        if (n < P.N) feed.src[i] = P.w.s + (n >> P.w.shift) * P.w.ld + kb0;
      } else if (j + 64 * (i - 2) < BN && m < P.M) {
        feed.src[i] = P.x.s + (m >> P.x.shift) * P.x.ld + kb0;
      }
    }
    const int vec = kb0 % 4 == 0 ? P.aligned : 1;
    feed.load(0, nk, vec);
    Ring<STAGES> st;
    Ring<Shared<BN>::SLOTS> sc;
    bool ok = true;
    for (int i0 = 0; i0 < nk && ok; i0 += GROUP) {
      float v[PER][GROUP];
#pragma unroll
      for (int i = 0; i < PER; ++i)
#pragma unroll
        for (int b = 0; b < GROUP; ++b) v[i][b] = feed.next[i][b];
      if (i0 + GROUP < nk) feed.load(i0 + GROUP, nk, vec);
#pragma unroll
      for (int b = 0; b < GROUP; ++b) {
        if (i0 + b >= nk) break;
        ok = __all_sync(0xFFFFFFFFu,
                        mbar_wait(&sh->mult[st.slot], st.parity ^ 1u, abort, P.wait_cycles, &g_f8_fault));
        if (!ok) break;
        float* to = sh->scale[sc.slot] + j;
#pragma unroll
        for (int i = 0; i < PER; ++i)
          if (i < 2 || j + 64 * (i - 2) < BN) to[64 * i] = v[i][b];
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh->full[st.slot]);
        st.next();
        sc.next();
      }
    }
  } else {
    const int q = warp & 3;
    Ring<STAGES> st;
    Ring<ACC> ac;
    Ring<Shared<BN>::SLOTS> sc;
    for (int i = 0; i < nk; ++i, st.next(), ac.next(), sc.next()) {
      const bool ok = mbar_wait(&sh->mult[st.slot], st.parity, abort, P.wait_cycles, &g_f8_fault);
      if (!__all_sync(0xFFFFFFFFu, ok)) break;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const uint32_t t = tmem_base + ((uint32_t)(32 * q) << 16) + ac.slot * BN;
      const float* scale = sh->scale[sc.slot];
      const float rs = scale[32 * q + lane];
      const uint64_t row2 = pair(rs, rs);
#pragma unroll
      for (int c = 0; c < BN; c += 16) {
        uint32_t r[16];
        tmem_ld16(t + c, r);
        tmem_wait_ld();
#pragma unroll
        for (int j = 0; j < 16; j += 4) {
          const ulonglong2 s2 = *reinterpret_cast<const ulonglong2*>(&scale[ROWS + c + j]);
          acc[(c + j) / 2] = fma2(mul2(pair(r[j], r[j + 1]), row2), s2.x, acc[(c + j) / 2]);
          acc[(c + j) / 2 + 1] = fma2(mul2(pair(r[j + 2], r[j + 3]), row2), s2.y, acc[(c + j) / 2 + 1]);
        }
      }
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh->tempty[ac.slot]);
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (warp == 1) {
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(TMEM_COLS)
                 : "memory");
  }
  // the ring is free: the CTA's sums, [x row][w row]
  float* part = reinterpret_cast<float*>(ring);
  if (warp >= 4) {
    const int at = 32 * (warp & 3) + lane;
#pragma unroll
    for (int j = 0; j < BN / 2; ++j) {
      part[(2 * j) * ROWS + at] = __uint_as_float((uint32_t)acc[j]);
      part[(2 * j + 1) * ROWS + at] = __uint_as_float((uint32_t)(acc[j] >> 32));
    }
  }
  __syncwarp();
  if (split > 1)
    cluster_sync();
  else
    __syncthreads();
  // rank r adds up and writes the r-th share of the tile
  const uint32_t part_addr = smem_u32(part);
  for (int i = rank * kThreads + threadIdx.x; i < BN * (ROWS / 4); i += split * kThreads) {
    const int c = i / (ROWS / 4), r4 = (i % (ROWS / 4)) * 4;
    if (m0 + c >= P.M || n0 + r4 >= P.N) continue;
    const uint32_t at = part_addr + (uint32_t)(c * ROWS + r4) * 4;
    float4 u[8];  // all on their way before the first is added
#pragma unroll
    for (int s = 0; s < 8; ++s)
      if (s < split)
        u[s] = split > 1 ? ld_cluster4(map_rank(at, s)) : *reinterpret_cast<const float4*>(&part[c * ROWS + r4]);
    float4 v = u[0];
#pragma unroll
    for (int s = 1; s < 8; ++s)
      if (s < split) v.x += u[s].x, v.y += u[s].y, v.z += u[s].z, v.w += u[s].w;
    finish4(P, m0 + c, n0 + r4, v);
  }
  __syncwarp();
  if (split > 1) cluster_sync();  // a CTA's sums are read by the others until here
}

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
      cudaFuncSetAttribute(linear_f8_kernel<BN>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
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
  return cudaLaunchKernelEx(&cfg, linear_f8_kernel<BN>, mw, mx, p, split);
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
