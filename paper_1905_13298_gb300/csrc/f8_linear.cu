// Product of two 8-bit floating-point matrices with a scale per block of 128
// values of the reduction, on the 5th-generation tensor cores (sm_103a).
//
//   y[m][n] = bias[n] + add[m][n] + sum_b sx[m][b] sw[n][b] sum_{k in block b} qx[m][k] qw[n][k]
//
// A block's inner sum is four tcgen05.mma of kind::f8f6f4 (K = 32 each) into
// an accumulator of its own in tensor memory; it is then read back and added,
// times its two scales, to float32 sums in registers.  So scales may be any
// float32 and differ per row, and no sum is held in fewer than 32 bits.
//
// linear_f8_kernel lays 128 rows of w along the lanes of tensor memory and BN
// rows of x along its columns: with one token in flight the weights, which
// are all the traffic, still fill the tensor core's 128 lanes.  A
// thread-block cluster splits the reduction of one tile and its CTAs add
// their parts through distributed shared memory in rank order, so results do
// not depend on timing.
#include <atomic>

#include "f8_common.cuh"
#include "tensor_core.cuh"

namespace ds {

__device__ int g_f8_fault;  // set when a bounded wait of the 8-bit product gives up

namespace {

std::atomic<long long> g_wait_cycles{kTimeoutCycles};

// An operand's scales: row r, block b at s[(r >> shift) * ld + b].
struct Scales {
  const float* s;
  int64_t ld;
  int shift;
};

struct Params {
  Scales x, w;
  const float *bias, *add;
  void* y;
  int64_t M, N, ld_add, ldy;
  int nk;         // blocks of the reduction
  uint32_t idesc;  // formats of the operands, without the tile's shape
  int type;       // of y
  int vec;        // y's rows are aligned for stores of four values, add's for loads of four
  long long wait_cycles;
};

__device__ __forceinline__ void umma_f8(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc,
                                        uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(tmem_d),
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}

__device__ __forceinline__ void tmem_ld16(uint32_t addr, uint32_t r[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, "
      "%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// Pairs of float32 in one 64-bit register: two multiplications per instruction.
__device__ __forceinline__ uint64_t pair(uint32_t lo, uint32_t hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(lo), "r"(hi));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t map_rank(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ float4 ld_cluster4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
               : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(addr)
               : "memory");
  return v;
}

__device__ __forceinline__ void store_one(void* y, int type, int64_t i, float v) {
  if (type == DS_TYPE_F32)
    static_cast<float*>(y)[i] = v;
  else if (type == DS_TYPE_BF16)
    static_cast<__nv_bfloat16*>(y)[i] = __float2bfloat16_rn(v);
  else
    static_cast<__half*>(y)[i] = __float2half_rn(v);
}

// Adds bias and `add` to four outputs (m, n .. n + 3), rounds them once to y's type and stores those that exist.
__device__ __forceinline__ void finish4(const Params& P, int64_t m, int64_t n, float4 v) {
  const int64_t left = P.N - n;
  float o[4] = {v.x, v.y, v.z, v.w};
  if (P.bias) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < left) o[i] += P.bias[n + i];
  }
  const bool vec = P.vec && left >= 4;
  if (P.add) {
    const float* a = P.add + m * P.ld_add + n;
    if (vec) {
      const float4 f = *reinterpret_cast<const float4*>(a);
      o[0] += f.x, o[1] += f.y, o[2] += f.z, o[3] += f.w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i < left) o[i] += a[i];
    }
  }
  const int64_t at = m * P.ldy + n;
  if (vec) {
    if (P.type == DS_TYPE_F32)
      *reinterpret_cast<float4*>(static_cast<float*>(P.y) + at) = make_float4(o[0], o[1], o[2], o[3]);
    else if (P.type == DS_TYPE_BF16)
      *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(P.y) + at) =
          make_uint2(pack2(o[0], o[1], (const __nv_bfloat16*)nullptr), pack2(o[2], o[3], (const __nv_bfloat16*)nullptr));
    else
      *reinterpret_cast<uint2*>(static_cast<__half*>(P.y) + at) =
          make_uint2(pack2(o[0], o[1], (const __half*)nullptr), pack2(o[2], o[3], (const __half*)nullptr));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < left) store_one(P.y, P.type, at + i, o[i]);
  }
}

constexpr int BK = 128;    // bytes of a row per stage: one block of the reduction
constexpr int ROWS = 128;  // rows of w per tile: the lanes of tensor memory
constexpr int kThreads = 192;
constexpr int kEpiWarps = 4;

template <int BN>
struct Cfg;
// STAGES: two CTAs per SM up to BN = 64; ACC: accumulators in tensor memory
template <>
struct Cfg<16> {
  static constexpr int STAGES = 6, ACC = 4;
};
template <>
struct Cfg<32> {
  static constexpr int STAGES = 5, ACC = 4;
};
template <>
struct Cfg<64> {
  static constexpr int STAGES = 4, ACC = 4;
};
template <>
struct Cfg<128> {
  static constexpr int STAGES = 6, ACC = 4;
};

template <int BN>
struct __align__(16) Shared {
  float col_scale[kEpiWarps][2][BN];
  uint64_t full[Cfg<BN>::STAGES];
  uint64_t empty[Cfg<BN>::STAGES];
  uint64_t tfull[Cfg<BN>::ACC];
  uint64_t tempty[Cfg<BN>::ACC];
  uint64_t done;
  uint32_t tmem_base;
  int abort;
};

template <int BN>
constexpr size_t smem_bytes() {
  return (size_t)Cfg<BN>::STAGES * (ROWS + BN) * BK + sizeof(Shared<BN>) + 1024;
}

// One tile: 128 rows of w (n0 ..), BN rows of x (m0 ..).  blockIdx.x = tile * split + rank in the cluster; the rank takes
// the blocks [rank nk / split, (rank + 1) nk / split) of the reduction.  Warp 0 loads, warp 1 multiplies, warps 2-5 scale.
template <int BN>
__global__ void __launch_bounds__(kThreads) linear_f8_kernel(const __grid_constant__ CUtensorMap tmap_w,
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
  const int64_t tiles_n = (P.N + ROWS - 1) / ROWS;
  const int64_t tile = blockIdx.x / split;
  const int rank = (int)(blockIdx.x - tile * split);
  const int64_t tm = tile / tiles_n;
  const int64_t n0 = (tile - tm * tiles_n) * ROWS, m0 = tm * BN;
  const int kb0 = (int)((int64_t)P.nk * rank / split);
  const int nk = (int)((int64_t)P.nk * (rank + 1) / split) - kb0;
  volatile int* abort = &sh->abort;

  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(&sh->full[s], 1);
      mbar_init(&sh->empty[s], 1);
    }
    for (int b = 0; b < ACC; ++b) {
      mbar_init(&sh->tfull[b], 1);
      mbar_init(&sh->tempty[b], kEpiWarps);
    }
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
      int i = 0;
      for (; i < nk; ++i) {
        const int s = i % STAGES;
        if (i >= STAGES &&
            !mbar_wait(&sh->empty[s], (uint32_t)((i / STAGES) & 1) ^ 1u, abort, P.wait_cycles, &g_f8_fault))
          break;
        unsigned char* a = ring + s * STAGE_BYTES;
        mbar_expect_tx(&sh->full[s], STAGE_BYTES);
        tma_load_2d(a, &tmap_w, &sh->full[s], (kb0 + i) * BK, (int)n0);
        tma_load_2d(a + A_BYTES, &tmap_x, &sh->full[s], (kb0 + i) * BK, (int)m0);
      }
      for (int j = (i > STAGES ? i - STAGES : 0); j < i; ++j)
        mbar_drain(&sh->full[j % STAGES], (uint32_t)(j / STAGES) & 1u);
    }
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t idesc = P.idesc | ((uint32_t)(BN >> 3) << 17) | ((uint32_t)(ROWS >> 4) << 24);
      for (int i = 0; i < nk; ++i) {
        const int s = i % STAGES, b = i % ACC;
        if (i >= ACC &&
            !mbar_wait(&sh->tempty[b], (uint32_t)((i / ACC) - 1) & 1u, abort, P.wait_cycles, &g_f8_fault))
          break;
        if (!mbar_wait(&sh->full[s], (uint32_t)(i / STAGES) & 1u, abort, P.wait_cycles, &g_f8_fault)) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint32_t a = smem_u32(ring + s * STAGE_BYTES), x = a + A_BYTES;
#pragma unroll
        for (int k = 0; k < BK / 32; ++k)
          umma_f8(tmem_base + (uint32_t)(b * BN), sw128_desc(a + 32 * k), sw128_desc(x + 32 * k), idesc, k > 0);
        umma_commit(&sh->empty[s]);
        umma_commit(&sh->tfull[b]);
      }
      // every MMA issued by this CTA has completed before its memory is used again
      umma_commit(&sh->done);
      mbar_drain(&sh->done, 0u);
    }
  } else {
    const int q = warp & 3, e = warp - 2;
    constexpr int PER = (BN + 31) / 32;
    const int64_t n = n0 + 32 * q + lane;
    const float* sw = P.w.s + (n >> P.w.shift) * P.w.ld + kb0;
    const float* sx[PER];
    bool has[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int64_t m = m0 + 32 * j + lane;
      has[j] = 32 * j + lane < BN && m < P.M;
      sx[j] = P.x.s + (m >> P.x.shift) * P.x.ld + kb0;
    }
    float rs = 0.f, cs[PER];
    auto fetch = [&](int i) {  // scales of block i (a row that does not exist has no scale, and zeros in its products)
      rs = n < P.N ? sw[i] : 0.f;
#pragma unroll
      for (int j = 0; j < PER; ++j) cs[j] = has[j] ? sx[j][i] : 0.f;
    };
    if (nk > 0) fetch(0);
    for (int i = 0; i < nk; ++i) {
      const int b = i % ACC;
      float* col = sh->col_scale[e][i & 1];
#pragma unroll
      for (int j = 0; j < PER; ++j)
        if (32 * j + lane < BN) col[32 * j + lane] = cs[j];
      const uint64_t row2 = pair(__float_as_uint(rs), __float_as_uint(rs));
      __syncwarp();
      if (i + 1 < nk) fetch(i + 1);
      const bool ok = mbar_wait(&sh->tfull[b], (uint32_t)(i / ACC) & 1u, abort, P.wait_cycles, &g_f8_fault);
      if (!__all_sync(0xFFFFFFFFu, ok)) break;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const uint32_t t = tmem_base + ((uint32_t)(32 * q) << 16) + (uint32_t)(b * BN);
#pragma unroll
      for (int c = 0; c < BN; c += 16) {
        uint32_t r[16];
        tmem_ld16(t + c, r);
        tmem_wait_ld();
#pragma unroll
        for (int j = 0; j < 16; j += 4) {
          const ulonglong2 s2 = *reinterpret_cast<const ulonglong2*>(&col[c + j]);
          acc[(c + j) / 2] = fma2(mul2(pair(r[j], r[j + 1]), row2), s2.x, acc[(c + j) / 2]);
          acc[(c + j) / 2 + 1] = fma2(mul2(pair(r[j + 2], r[j + 3]), row2), s2.y, acc[(c + j) / 2 + 1]);
        }
      }
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh->tempty[b]);
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
  if (warp >= 2) {
    const int at = 32 * (warp & 3) + lane;
#pragma unroll
    for (int j = 0; j < BN / 2; ++j) {
      part[(2 * j) * ROWS + at] = __uint_as_float((uint32_t)acc[j]);
      part[(2 * j + 1) * ROWS + at] = __uint_as_float((uint32_t)(acc[j] >> 32));
    }
  }
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
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s = 0; s < split; ++s) {
      const float4 u = split > 1 ? ld_cluster4(map_rank(at, s)) : *reinterpret_cast<const float4*>(&part[c * ROWS + r4]);
      v.x += u.x, v.y += u.y, v.z += u.z, v.w += u.w;
    }
    finish4(P, m0 + c, n0 + r4, v);
  }
  __syncwarp();
  if (split > 1) cluster_sync();  // a CTA's sums are read by the others until here
}

bool make_map(CUtensorMap* map, const ds_f8_matrix* m, uint32_t box_rows) {
  return make_map_2d(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, m->q, m->cols, m->rows, m->ld, BK, box_rows);
}

template <int BN>
cudaError_t launch(const CUtensorMap& mw, const CUtensorMap& mx, const Params& p, cudaStream_t st) {
  constexpr size_t smem = smem_bytes<BN>();
  // once per process, thread-safe (function-local static)
  static const cudaError_t attr =
      cudaFuncSetAttribute(linear_f8_kernel<BN>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (attr != cudaSuccess) return attr;
  const int64_t tiles = (p.M + BN - 1) / BN * ((p.N + ROWS - 1) / ROWS);
  // Split the reduction while that fills SMs that would idle and leaves each CTA a block.
  int split = 1;
  while (split < 8 && tiles * split * 2 <= 2 * (int64_t)sm_count() && split * 2 <= p.nk) split *= 2;
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

Scales scales_of(const ds_f8_matrix* m) {
  return Scales{m->scale, m->ld_scale, m->blocks == DS_F8_TILES ? 7 : 0};
}

}  // namespace

cudaError_t launch_linear_f8(const LinearF8Params& l, cudaStream_t st) {
  Params p = {};
  p.x = scales_of(l.x);
  p.w = scales_of(l.w);
  p.bias = l.bias;
  p.add = l.add;
  p.y = l.y;
  p.M = l.x->rows;
  p.N = l.w->rows;
  p.ld_add = l.ld_add;
  p.ldy = l.ldy;
  p.nk = (int)((l.x->cols + BK - 1) / BK);
  // kind::f8f6f4: float32 D, formats of A (w) and B (x), both K-major
  p.idesc = (1u << 4) | ((uint32_t)l.w->format << 7) | ((uint32_t)l.x->format << 10);
  p.type = l.type;
  const size_t size = l.type == DS_TYPE_F32 ? 4 : 2;
  p.vec = reinterpret_cast<uintptr_t>(l.y) % (4 * size) == 0 && l.ldy % 4 == 0 &&
          (l.add == nullptr || (reinterpret_cast<uintptr_t>(l.add) % 16 == 0 && l.ld_add % 4 == 0));
  p.wait_cycles = g_wait_cycles.load(std::memory_order_relaxed);
  const int bn = p.M <= 16 ? 16 : (p.M <= 32 ? 32 : (p.M <= 64 ? 64 : 128));
  CUtensorMap mw, mx;
  if (p.nk > 0) {
    if (!make_map(&mw, l.w, ROWS) || !make_map(&mx, l.x, (uint32_t)bn)) return cudaErrorInvalidValue;
  } else {  // an empty reduction loads nothing
    mw = mx = CUtensorMap{};
  }
  switch (bn) {
    case 16: return launch<16>(mw, mx, p, st);
    case 32: return launch<32>(mw, mx, p, st);
    case 64: return launch<64>(mw, mx, p, st);
    default: return launch<128>(mw, mx, p, st);
  }
}

void set_f8_wait_cycles(long long cycles) {
  g_wait_cycles.store(cycles > 0 ? cycles : kTimeoutCycles, std::memory_order_relaxed);
}

int read_f8_fault_flag() {
  int v = 0;
  if (cudaMemcpyFromSymbol(&v, g_f8_fault, sizeof(int)) != cudaSuccess) return -1;
  const int zero = 0;
  if (v != 0 && cudaMemcpyToSymbol(g_f8_fault, &zero, sizeof(int)) != cudaSuccess) return -1;
  return v;
}

}  // namespace ds
