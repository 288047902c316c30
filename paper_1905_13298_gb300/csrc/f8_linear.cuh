// The 8-bit product's device code that the dense products and the experts' share:
// scales, stores, and the kernels of small and of large products.
#pragma once

#include <type_traits>

#include "f8_common.cuh"
#include "tensor_core.cuh"

namespace ds {
namespace {

__device__ int g_f8_fault;  // set when a bounded wait of this file's products gives up

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
  int aligned;    // how many scales of a row a load may take: 8, 4 or 1
  int vec;        // y's rows are aligned for stores of four values, add's for loads of four
  int pairs;      // ... of two
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
// 16 lanes x 64 columns: of each 8 columns thread 4 a + b holds columns 2 b and 2 b + 1 of lane a, then of lane a + 8.
__device__ __forceinline__ void tmem_ld_fragment(uint32_t addr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, "
      "%14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

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
               : "r"(addr));  // stays behind the cluster's barrier, which is volatile too
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

// Where sums go: P is the product's parameters, or an OutputPart.  Adds bias and `add` to four outputs (m, n .. n + 3),
// rounds them once to y's type and stores those that exist.
template <typename To>
__device__ __forceinline__ void finish4(const To& P, int64_t m, int64_t n, float4 v) {
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
          make_uint2(pack2(o[0], o[1], (const __nv_bfloat16*)nullptr),
                     pack2(o[2], o[3], (const __nv_bfloat16*)nullptr));
    else
      *reinterpret_cast<uint2*>(static_cast<__half*>(P.y) + at) =
          make_uint2(pack2(o[0], o[1], (const __half*)nullptr), pack2(o[2], o[3], (const __half*)nullptr));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < left) store_one(P.y, P.type, at + i, o[i]);
  }
}

// 32 bytes of one row: a whole sector of the second-level cache.
__device__ __forceinline__ void store_sector(void* p, const uint32_t v[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]),
               "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}
// Four threads 4 a + b exchange the parts of their four units of N values: v[u] of thread b goes to v[b] of thread u.
template <int N>
__device__ __forceinline__ void turn_quad(float (&v)[4][N]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int bit = 1; bit <= 2; bit *= 2) {
    const bool up = lane & bit;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (u & bit) continue;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        float &lo = v[u][i], &hi = v[u | bit][i];
        const float got = __shfl_xor_sync(0xFFFFFFFFu, up ? lo : hi, bit);
        if (up)
          lo = got;
        else
          hi = got;
      }
    }
  }
}
// Columns 32 c .. of a warp's 32 rows of sums, turned so that thread 4 a + b has columns 8 b .. of four rows.  What a
// store costs is the rows that it touches: eight here, 32 where a thread has a row, which took 3 us of a tile.
// LANES: thread i holds row i, and gets rows 4 a .. 4 a + 3.  Otherwise the sums lie as tmem_ld_fragment spreads them,
// acc[64 c + 32 h + 4 g + 2 e + i] being row 16 h + 8 e + a, column 64 c + 8 g + 2 b + i, and it gets rows a, a + 8 ..
template <bool LANES>
__device__ __forceinline__ void turned_rows(const float* acc, int c, float (&o)[4][8]) {
  if constexpr (LANES) {
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int i = 0; i < 8; ++i) o[u][i] = acc[32 * c + 8 * u + i];
    turn_quad(o);
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float v[4][2];
#pragma unroll
      for (int j = 0; j < 8; ++j)
        v[j >> 1][j & 1] = acc[64 * (c >> 1) + 32 * (r >> 1) + 16 * (c & 1) + 4 * (j >> 1) + 2 * (r & 1) + (j & 1)];
      turn_quad(v);
#pragma unroll
      for (int j = 0; j < 8; ++j) o[r][j] = v[j >> 1][j & 1];
    }
  }
}
// Bias and `add` are added to the sums of 32 rows from m, NC columns from n; these are rounded once to y's type and
// stored.  For rows that are aligned for stores of eight values (and for loads of four from add).
template <bool LANES, typename To, int NC>
__device__ __forceinline__ void store_wide(const To& P, int64_t m, int64_t n, const float (&acc)[NC]) {
  constexpr int STEP = LANES ? 1 : 8;
  const int lane = threadIdx.x & 31;
  m += LANES ? lane & ~3 : lane >> 2;
  n += 8 * (lane & 3);
#pragma unroll
  for (int c = 0; c < NC / 32; ++c, n += 32) {
    float o[4][8];
    turned_rows<LANES>(acc, c, o);
    if (n + 8 > P.N) {
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < 8; j += 4)
          if (m + STEP * r < P.M && n + j < P.N)
            finish4(P, m + STEP * r, n + j, make_float4(o[r][j], o[r][j + 1], o[r][j + 2], o[r][j + 3]));
      continue;
    }
    if (P.bias) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float b = P.bias[n + j];
#pragma unroll
        for (int r = 0; r < 4; ++r) o[r][j] += b;
      }
    }
    if (P.add) {  // four rows are loaded before any of them is stored
      float4 f[4][2] = {};
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if (m + STEP * r >= P.M) continue;
        const float4* a = reinterpret_cast<const float4*>(P.add + (m + STEP * r) * P.ld_add + n);
        f[r][0] = a[0], f[r][1] = a[1];
      }
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < 8; j += 4) {
          const float4 u = f[r][j / 4];
          o[r][j] += u.x, o[r][j + 1] += u.y, o[r][j + 2] += u.z, o[r][j + 3] += u.w;
        }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      if (m + STEP * r >= P.M) continue;
      const int64_t at = (m + STEP * r) * P.ldy + n;
      if (P.type == DS_TYPE_F32) {
        uint32_t w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = __float_as_uint(o[r][j]);
        store_sector(static_cast<float*>(P.y) + at, w);
      } else {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          w[j] = P.type == DS_TYPE_BF16 ? pack2(o[r][2 * j], o[r][2 * j + 1], (const __nv_bfloat16*)nullptr)
                                        : pack2(o[r][2 * j], o[r][2 * j + 1], (const __half*)nullptr);
        *reinterpret_cast<uint4*>(static_cast<__half*>(P.y) + at) = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
  }
}
constexpr int kPatchPitch = 36;  // floats between the rows of a patch of 8 x 32: no bank conflicts
// The same for rows of any alignment: a patch of shared memory makes it 32 columns of one row per store (4096 x 4096 x
// 4097 into bf16 93 us, with add 114; 79 and 97 for 4096 columns; by fours of a row's columns 129 and 247).
// COUNT = 2: rows are aligned for pairs of values, and a store takes 32 columns of two rows.
template <bool LANES, typename T, int COUNT, typename To, int NC>
__device__ __forceinline__ void store_narrow_as(const To& P, int64_t m, int64_t n, const float (&acc)[NC],
                                                float* patch) {
  struct alignas(sizeof(T) * COUNT) Some {
    T v[COUNT];
  };
  struct alignas(4 * COUNT) Floats {
    float v[COUNT];
  };
  const int lane = threadIdx.x & 31, half = COUNT * lane / 32, mine = COUNT * lane % 32;
  const int rows = (int)(P.M - m < 32 ? P.M - m : 32);
  // of the i-th row of the r-th patch, as this thread stores it
  auto place = [&](int i) { return COUNT * i + half; };
  auto row = [&](int r, int i) { return LANES ? 4 * place(i) + r : 8 * r + place(i); };
#pragma unroll
  for (int c = 0; c < NC / 32; ++c) {
    const int64_t col = n + 32 * c + mine;
    const int left = (int)(P.N - col < COUNT ? P.N - col : COUNT);
    auto exists = [&](int r, int i) { return left > 0 && row(r, i) < rows; };
    Floats bias = {}, v[4][8 / COUNT] = {};  // v: of add, the values of 32 rows on their way at once
    if (P.bias) {
#pragma unroll
      for (int k = 0; k < COUNT; ++k)
        if (k < left) bias.v[k] = P.bias[col + k];
    }
    if (P.add) {
      const float* from = P.add + m * P.ld_add + col;
      asm volatile("" : "+l"(from));  // addresses are found here, not all of them before the first use
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int i = 0; i < 8 / COUNT; ++i) {
          if (!exists(r, i)) continue;
          const float* a = from + row(r, i) * P.ld_add;
          if (left == COUNT)
            v[r][i] = *reinterpret_cast<const Floats*>(a);
          else
            v[r][i].v[0] = a[0];
        }
    }
    float o[4][8];
    turned_rows<LANES>(acc, c, o);
    T* y = static_cast<T*>(P.y) + m * P.ldy + col;
    asm volatile("" : "+l"(y));
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      __syncwarp();
      float4* to = reinterpret_cast<float4*>(&patch[(lane >> 2) * kPatchPitch + 8 * (lane & 3)]);
      to[0] = make_float4(o[r][0], o[r][1], o[r][2], o[r][3]);
      to[1] = make_float4(o[r][4], o[r][5], o[r][6], o[r][7]);
      __syncwarp();
#pragma unroll
      for (int i = 0; i < 8 / COUNT; ++i) {
        if (!exists(r, i)) continue;
        const Floats f = *reinterpret_cast<const Floats*>(&patch[place(i) * kPatchPitch + mine]);
        Some out;
#pragma unroll
        for (int k = 0; k < COUNT; ++k) from_float(f.v[k] + bias.v[k] + v[r][i].v[k], out.v[k]);
        T* at = y + row(r, i) * P.ldy;
        if (left == COUNT)
          *reinterpret_cast<Some*>(at) = out;
        else
          at[0] = out.v[0];
      }
    }
  }
}
template <bool LANES, typename T, typename To, int NC>
__device__ __forceinline__ void store_narrow_of(const To& P, int64_t m, int64_t n, const float (&acc)[NC],
                                                float* patch) {
  if (P.pairs)
    store_narrow_as<LANES, T, 2>(P, m, n, acc, patch);
  else
    store_narrow_as<LANES, T, 1>(P, m, n, acc, patch);
}
// One branch by the type for all of them: one per value made the code of a tile miss in the instruction cache.
template <bool LANES, typename To, int NC>
__device__ __forceinline__ void store_narrow(const To& P, int64_t m, int64_t n, const float (&acc)[NC],
                                             float* patch) {
  if (P.type == DS_TYPE_F32)
    store_narrow_of<LANES, float>(P, m, n, acc, patch);
  else if (P.type == DS_TYPE_BF16)
    store_narrow_of<LANES, __nv_bfloat16>(P, m, n, acc, patch);
  else
    store_narrow_of<LANES, __half>(P, m, n, acc, patch);
}

constexpr int BK = 128;    // bytes of a row per stage: one block of the reduction
constexpr int ROWS = 128;  // rows of w per tile: the lanes of tensor memory
// A position in a ring of N barriers: the slot and the parity of its phase.
template <int N>
struct Ring {
  uint32_t slot = 0, parity = 0;
  __device__ __forceinline__ void next() {
    if (++slot == N) {
      slot = 0;
      parity ^= 1u;
    }
  }
};

// The scales of PER rows on their way to shared memory, GROUP blocks of the reduction at a time (4 or 8).
template <int PER, int GROUP>
struct ScaleFeed {
  const float* src[PER];  // at a row's first block; NULL: no such row, and zeros in its products
  float next[PER][GROUP];
  // aligned: how many scales a load may take, 8, 4 or 1
  __device__ __forceinline__ void load(int i0, int nk, int aligned) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
#pragma unroll
      for (int b = 0; b < GROUP; ++b) next[i][b] = 0.f;
      if (src[i] == nullptr) continue;
      if (GROUP == 8 && aligned == 8 && nk - i0 >= 8) {
        float* v = next[i];
        asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[GROUP - 4]), "=f"(v[GROUP - 3]),
                       "=f"(v[GROUP - 2]), "=f"(v[GROUP - 1])
                     : "l"(src[i] + i0));
        continue;
      }
#pragma unroll
      for (int h = 0; h < GROUP; h += 4) {
        if (aligned >= 4 && nk - i0 >= h + 4) {
          const float4 f = *reinterpret_cast<const float4*>(src[i] + i0 + h);
          next[i][h] = f.x, next[i][h + 1] = f.y, next[i][h + 2] = f.z, next[i][h + 3] = f.w;
        } else {
#pragma unroll
          for (int b = h; b < h + 4; ++b)
            if (i0 + b < nk) next[i][b] = src[i][i0 + b];
        }
      }
    }
  }
};

// After a wait gave up, a stage's barrier may miss the arrivals of warps that left; its copies land within
// microseconds, and this many cycles (8 ms) are waited for them.
constexpr long long kLandedCycles = 1 << 24;

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

// Where a CTA's tile of a single product lies: rows m0 .. of x and n0 .. of w; how many blocks its reduction has, and
// what its sums go to.
template <int BN>
struct OnePlace {
  int m0, n0;
  __device__ __forceinline__ bool find(const Params& P, uint32_t tile) {
    const uint32_t tiles_n = (uint32_t)((P.N + ROWS - 1) / ROWS), tm = tile / tiles_n;
    n0 = (int)(tile - tm * tiles_n) * ROWS, m0 = (int)tm * BN;
    return true;
  }
  __device__ __forceinline__ int blocks(const Params& P) const { return P.nk; }
  __device__ __forceinline__ const Params& output(const Params& P) const { return P; }
  __device__ __forceinline__ int column(const Params&) const { return n0; }
};

// One tile: 128 rows of w (n0 ..), BN rows of x (m0 ..).  blockIdx.x = tile * split + rank in the cluster; the rank
// takes the blocks [rank nk / split, (rank + 1) nk / split) of the reduction.  Warp 0 loads, warp 1 multiplies, warps 2
// and 3 bring scales (as in the large kernel below), warps 4-7 add.
template <int BN, typename Place>
__global__ void __launch_bounds__(kThreads, Cfg<BN>::CTAS) linear_f8_kernel(const __grid_constant__ CUtensorMap tmap_w,
                                                             const __grid_constant__ CUtensorMap tmap_x,
                                                             const Params P, const int split, Place place) {
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
  const uint32_t tile = blockIdx.x / split;
  const int rank = (int)(blockIdx.x - tile * split);
  if (!place.find(P, tile)) return;  // the same for a whole cluster
  const int n0 = place.n0, m0 = place.m0, blocks = place.blocks(P);
  const int kb0 = (int)((int64_t)blocks * rank / split);
  const int nk = (int)((int64_t)blocks * (rank + 1) / split) - kb0;
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
  const auto& to = place.output(P);
  const int col0 = place.column(P);
  for (int i = rank * kThreads + threadIdx.x; i < BN * (ROWS / 4); i += split * kThreads) {
    const int c = i / (ROWS / 4), r4 = (i % (ROWS / 4)) * 4;
    if (m0 + c >= to.M || col0 + r4 >= to.N) continue;
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
    finish4(to, m0 + c, col0 + r4, v);
  }
  __syncwarp();
  if (split > 1) cluster_sync();  // a CTA's sums are read by the others until here
}

// ---------------------------------------------------------------------------
// Large products: one persistent CTA per SM walks tiles of 128 rows of x (the
// lanes) by N = 256 or 128 rows of w (the columns).  Warp 0 loads, warp 1
// multiplies block after block into two (four) accumulators in turn, and eight
// warps read each block back and add it, scaled, to the tile's sums: N / 2
// float32 per thread.  Further warps write a block's scales to shared memory
// as part of its stage (the stage's barrier counts them with the copies), so
// the warps that add wait for one barrier per block.
//
// A block's products take 512 cycles; what the adding warps do for it has to
// fit there.  A wait that succeeds costs 85 cycles, an arrival 70, a load from
// shared memory 40: a second barrier per block for the scales made it 1100.
// Measured at 8192 x 4096 x 4096: 140 us (1.96 PFLOP/s) with a scale per 128
// rows of w, 175 us (1.57) with one per row, where the adding warps multiply
// twice and the scales' loads compete with them for the path to shared memory
// (169 us without these loads).
// Tiles of half the width take two thirds of the time: 512 x 2048 x 4096 with a
// scale per 128 rows, 128 of them, 11.0 us, 64 of the others 13.7.
// ---------------------------------------------------------------------------
constexpr int kBigEpiWarps = 8;
// N: rows of w per tile.  Tiles of 256 read less; of 128 they leave fewer SMs without work where there are few, and room
// for more stages and accumulators.
// Warps for scales: with a scale per row of w two of them kept up with a block per 2400 cycles only (239 us at 8192 x
// 4096 x 4096), six keep up with the adding warps; two suffice for the 130 scales of the other case and leave more
// registers.  All threads are launched with the mean of the registers that the adding warps and the others then take.
template <bool COLS, int N>
struct BigCfg {
  static constexpr int STAGES = N == 256 ? 4 : 6, ACC = 512 / N;
  static constexpr int EACH = N / (kBigEpiWarps / 4);  // columns of a tile that a warp adds up
  static constexpr int SCALE_WARPS = COLS ? 6 : 2, OTHERS = 2 + SCALE_WARPS;
  static constexpr int THREADS = 32 * (OTHERS + kBigEpiWarps);
  static constexpr int REGS = COLS ? 208 : 216, REGS_OTHERS = COLS ? 48 : 72;
  static_assert(OTHERS * REGS_OTHERS + kBigEpiWarps * REGS <= (65536 / THREADS / 8 * 8) * (THREADS / 32), "registers");
  // Slots of the scales' ring.  A slot of the data ring is free when the products of the block STAGES before are done,
  // which needed the accumulator of the block STAGES + ACC before, whose readers were done with the block before that:
  // so a slot of the scales' ring may be written again SLOTS blocks later without a wait of its own.
  static constexpr int SLOTS = N == 256 ? 8 : 16;
  static_assert(SLOTS > STAGES + ACC, "scales in use");
  static constexpr int SCALE_ROWS = ROWS + N, STAGE_BYTES = (ROWS + N) * BK;
  struct __align__(16) Shared {
    float patch[kBigEpiWarps][8 * kPatchPitch];
    float scale[SLOTS][SCALE_ROWS];  // rows of x, then rows of w
    uint64_t full[STAGES];   // a stage's copies and scales have come
    uint64_t mult[STAGES];   // its products are done: the sums may be read, the stage written again
    uint64_t tempty[ACC];    // an accumulator has been read
    uint64_t done;
    uint32_t tmem_base;
    int abort;
  };
  static constexpr size_t SMEM = (size_t)STAGES * STAGE_BYTES + sizeof(Shared) + 1024;
  static_assert(SMEM <= 232448, "shared memory of a CTA");
};

// A tile of the persistent kernel: 128 rows of x from m0, rows of w from n0, the blocks kb0 .. kb0 + nk - 1 of the
// reduction.
struct Tile {
  int m0, n0, kb0, nk;
};

// Tile r of a grid of tiles in grouped order: G row tiles, columns slowest inside a group, so that the tiles in flight
// share rows of both operands in L2.
__device__ __forceinline__ void grouped(uint32_t r, uint32_t tiles_m, uint32_t tiles_n, uint32_t G, int& tm, int& tn) {
  const uint32_t per_group = G * tiles_n, g = r / per_group, first = g * G;
  const uint32_t size = tiles_m - first < G ? tiles_m - first : G;
  const uint32_t q = r - g * per_group;
  tm = (int)(first + q % size);
  tn = (int)(q / size);
}

// The tiles of one product.  An order of several products' tiles WALKS: the kernel asks it for all blocks of the reduction
// that a CTA's tiles have, for walks over these tiles (each of a CTA's parts goes its own), and for where a tile's sums go.
// One product's tiles are counted by t: by walks it took 1% more (8192 x 4096 x 4096 140.4 us, 139.2).
template <int COLS_OF_TILE>
struct TileOrder {
  static constexpr int N = COLS_OF_TILE;
  static constexpr bool WALKS = false;  // tile t is at(t), and all have P.nk blocks
  uint32_t tiles_m, tiles_n, G;
  __device__ __forceinline__ const TileOrder& ready(const Params&, void*) const { return *this; }
  struct Walk {  // stands where other orders have one; nothing asks it
    __device__ __forceinline__ bool ended(const TileOrder&) const { return true; }
    __device__ __forceinline__ int blocks(const Params&, const TileOrder&) const { return 0; }
  };
  __device__ __forceinline__ Walk walk() const { return Walk{}; }
  __device__ __forceinline__ uint32_t count() const { return tiles_m * tiles_n; }
  __device__ __forceinline__ void at(uint32_t t, int& m0, int& n0) const {
    grouped(t, tiles_m, tiles_n, G, m0, n0);
    m0 *= ROWS, n0 *= N;
  }
  __device__ __forceinline__ int64_t blocks(const Params& P) const {
    const uint32_t n = count(), mine = blockIdx.x < n ? (n - blockIdx.x - 1) / gridDim.x + 1 : 0;
    return (int64_t)mine * P.nk;
  }
};

// COLS: w has a scale per row, so the columns of a tile differ; otherwise a warp's 128 columns share one.
template <bool COLS, bool WIDE, typename Order>
__global__ void __launch_bounds__(BigCfg<COLS, Order::N>::THREADS, 1)
    linear_f8_big_kernel(const __grid_constant__ CUtensorMap tmap_x, const __grid_constant__ CUtensorMap tmap_w,
                         const Params P, const Order order) {
  constexpr int N = Order::N;
  using Cfg = BigCfg<COLS, N>;
  using BigShared = typename Cfg::Shared;
  constexpr int BIG_STAGES = Cfg::STAGES, BIG_ACC = Cfg::ACC, kBigCols = Cfg::EACH;
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  unsigned char* ring = reinterpret_cast<unsigned char*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  BigShared* sh = reinterpret_cast<BigShared*>(ring + BIG_STAGES * Cfg::STAGE_BYTES);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  volatile int* abort = &sh->abort;
  const auto& tiles = order.ready(P, sh + 1);
  const int nk = P.nk;  // blocks of a tile, and tiles, of a single product
  uint32_t ntiles = 0;
  if constexpr (!Order::WALKS) ntiles = tiles.count();

  if (threadIdx.x == 0) {
    for (int s = 0; s < BIG_STAGES; ++s) {
      mbar_init(&sh->full[s], 1 + Cfg::SCALE_WARPS);  // the copies, and the warps with scales
      mbar_init(&sh->mult[s], 1);
    }
    for (int b = 0; b < BIG_ACC; ++b) mbar_init(&sh->tempty[b], kBigEpiWarps);
    mbar_init(&sh->done, 1);
    sh->abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh->tmem_base)),
                 "r"(BIG_ACC * N)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem_base = sh->tmem_base;

  if (warp < Cfg::OTHERS) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Cfg::REGS_OTHERS));
    if (warp == 0 && lane == 0) {
      // A slot's first use waits for the phase before the first one, which a fresh barrier reports as complete.
      Ring<BIG_STAGES> st;
      uint32_t issued = 0;
      bool ok = true;
      auto copy = [&](int m0, int n0, int kb0, int nk) {
        for (int i = 0; i < nk; ++i, ++issued, st.next()) {
          ok = mbar_wait(&sh->mult[st.slot], st.parity ^ 1u, abort, P.wait_cycles, &g_f8_fault);
          if (!ok) break;
          unsigned char* a = ring + st.slot * Cfg::STAGE_BYTES;
          mbar_expect_tx(&sh->full[st.slot], Cfg::STAGE_BYTES);
          tma_load_2d(a, &tmap_x, &sh->full[st.slot], (kb0 + i) * BK, m0);
          tma_load_2d(a + ROWS * BK, &tmap_w, &sh->full[st.slot], (kb0 + i) * BK, n0);
        }
      };
      if constexpr (Order::WALKS) {
        for (auto walk = tiles.walk(); !walk.ended(tiles) && ok; walk.next(tiles)) {
          const Tile tile = walk.tile(P, tiles);
          copy(tile.m0, tile.n0, tile.kb0, tile.nk);
        }
      } else {
        for (uint32_t t = blockIdx.x; t < ntiles && ok; t += gridDim.x) {
          int m0, n0;
          tiles.at(t, m0, n0);
          copy(m0, n0, 0, nk);
        }
      }
      // the last copies issued land before the CTA leaves
      for (uint32_t j = issued > BIG_STAGES ? issued - BIG_STAGES : 0; j < issued; ++j)
        mbar_drain(&sh->full[j % BIG_STAGES], (j / BIG_STAGES) & 1u, *abort ? kLandedCycles : kTimeoutCycles);
    } else if (warp == 1 && lane == 0) {
      const uint32_t idesc = P.idesc | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(ROWS >> 4) << 24);
      const uint64_t adesc = sw128_desc(smem_u32(ring)), bdesc = sw128_desc(smem_u32(ring) + ROWS * BK);
      const int64_t total = tiles.blocks(P);
      Ring<BIG_STAGES> st;
      Ring<BIG_ACC> ac;
      // The waits for the next block stand between this block's products, which keep the tensor core busy meanwhile.
      bool ok = total > 0 && mbar_wait(&sh->full[0], 0u, abort, P.wait_cycles, &g_f8_fault);
      for (int64_t n = 0; n < total && ok; ++n) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint64_t at = (uint64_t)(st.slot * (Cfg::STAGE_BYTES >> 4));
        const uint32_t d = tmem_base + ac.slot * N;
        uint64_t* const mult = &sh->mult[st.slot];
        umma_f8(d, adesc + at, bdesc + at, idesc, 0u);
        umma_f8(d, adesc + at + 2, bdesc + at + 2, idesc, 1u);
        st.next();
        ac.next();
        if (n + 1 < total) ok = mbar_wait(&sh->full[st.slot], st.parity, abort, P.wait_cycles, &g_f8_fault);
        umma_f8(d, adesc + at + 4, bdesc + at + 4, idesc, 1u);
        umma_f8(d, adesc + at + 6, bdesc + at + 6, idesc, 1u);
        umma_commit(mult);
        if (n + 1 < total)
          ok = ok && mbar_wait(&sh->tempty[ac.slot], ac.parity ^ 1u, abort, P.wait_cycles, &g_f8_fault);
      }
      umma_commit(&sh->done);
      mbar_drain(&sh->done, 0u);
    } else if (warp >= 2) {
      // Scales: thread j holds rows j, j + SPAN .. of the tile's 128 rows of x and N of w (or the scales that these
      // share), of four blocks at a time; the next four are on their way while these are written.  Where the rows of w
      // have their own, a load of eight costs the path to shared memory half as much; it is waited for, which the
      // blocks ahead in the ring hide (175 us at 8192 x 4096 x 4096, 182 with four).
      constexpr int SPAN = 32 * Cfg::SCALE_WARPS, USED = COLS ? Cfg::SCALE_ROWS : ROWS + N / 128, GROUP = COLS ? 8 : 4;
      constexpr int PER = (USED + SPAN - 1) / SPAN;
      const int j = threadIdx.x - 64;
      ScaleFeed<PER, GROUP> feed;
      auto point = [&](int m0, int n0, int kb0) {  // at the scales of a tile's rows
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          const int r = j + SPAN * i;
          const int64_t m = m0 + r, n = n0 + (COLS ? r - ROWS : (r - ROWS) * 128);
          feed.src[i] = nullptr;
          if (r < ROWS) {
            if (m < P.M) feed.src[i] = P.x.s + (m >> P.x.shift) * P.x.ld + kb0;
          } else if ((COLS || r < USED) && n < P.N) {
            feed.src[i] = P.w.s + (COLS ? n : n >> 7) * P.w.ld + kb0;
          }
        }
      };
      Ring<BIG_STAGES> st;
      uint32_t it = 0;
      bool ok = true;
      // a tile's blocks; `ahead` points at the next tile's scales and loads the first of them, where there is one
      auto feed_tile = [&](int blocks, int vec, auto ahead) {
        for (int i0 = 0; i0 < blocks && ok; i0 += GROUP) {
          float v[PER][GROUP];
          if constexpr (COLS) feed.load(i0, blocks, vec);
#pragma unroll
          for (int i = 0; i < PER; ++i)
#pragma unroll
            for (int b = 0; b < GROUP; ++b) v[i][b] = feed.next[i][b];
          if constexpr (!COLS) {
            if (i0 + GROUP < blocks)
              feed.load(i0 + GROUP, blocks, vec);
            else
              ahead();
          }
#pragma unroll
          for (int b = 0; b < GROUP; ++b) {
            if (i0 + b >= blocks) break;
            ok = __all_sync(0xFFFFFFFFu,
                            mbar_wait(&sh->mult[st.slot], st.parity ^ 1u, abort, P.wait_cycles, &g_f8_fault));
            if (!ok) break;
            float* to = sh->scale[it % Cfg::SLOTS] + j;
#pragma unroll
            for (int i = 0; i < PER; ++i)
              if (USED % SPAN == 0 || j + SPAN * i < USED) to[SPAN * i] = v[i][b];
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh->full[st.slot]);
            st.next();
            ++it;
          }
        }
      };
      if constexpr (Order::WALKS) {
        auto walk = tiles.walk();
        Tile tile = {};
        int vec = 1;
        auto take = [&] {  // the first tile from here on that has blocks
          while (!walk.ended(tiles) && walk.blocks(P, tiles) == 0) walk.next(tiles);
          if (walk.ended(tiles)) return false;
          tile = walk.tile(P, tiles);
          vec = tiles.aligned(P, tile);
          point(tile.m0, tile.n0, tile.kb0);
          return true;
        };
        bool more = take();
        if constexpr (!COLS)
          if (more) feed.load(0, tile.nk, vec);
        while (more && ok) {
          const int blocks = tile.nk, same = vec;
          walk.next(tiles);
          if constexpr (COLS) {
            feed_tile(blocks, same, [] {});
            more = take();
          } else {
            feed_tile(blocks, same, [&] {
              more = take();
              if (more) feed.load(0, tile.nk, vec);
            });
          }
        }
      } else {
        auto take = [&](uint32_t t) {
          int m0, n0;
          tiles.at(t, m0, n0);
          point(m0, n0, 0);
        };
        if constexpr (!COLS) {
          take(blockIdx.x);
          feed.load(0, nk, P.aligned);
        }
        for (uint32_t t = blockIdx.x; t < ntiles && ok; t += gridDim.x) {
          if constexpr (COLS) take(t);
          feed_tile(nk, P.aligned, [&] {
            if (t + gridDim.x < ntiles) {
              take(t + gridDim.x);
              feed.load(0, nk, P.aligned);
            }
          });
        }
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(Cfg::REGS));
    const int q = warp & 3, e = warp - Cfg::OTHERS, col0 = (e >> 2) * kBigCols;
    const uint32_t tmem = tmem_base + ((uint32_t)(32 * q) << 16) + (uint32_t)col0;
    Ring<BIG_STAGES> st;
    Ring<BIG_ACC> ac;
    uint32_t it = 0;
    bool ok = true;
    auto wait_block = [&] {
      ok = __all_sync(0xFFFFFFFFu, mbar_wait(&sh->mult[st.slot], st.parity, abort, P.wait_cycles, &g_f8_fault));
      st.next();
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      return ok;
    };
    auto release = [&] {  // the block is in registers: the accumulator may be written again
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh->tempty[ac.slot]);
      ac.next();
    };
    uint32_t t = blockIdx.x;
    auto walk = tiles.walk();
    while ((Order::WALKS ? !walk.ended(tiles) : t < ntiles) && ok) {
      float acc[kBigCols];
#pragma unroll
      for (int j = 0; j < kBigCols; ++j) acc[j] = 0.f;
      const int blocks = Order::WALKS ? walk.blocks(P, tiles) : nk;
      for (int i = 0; i < blocks; ++i, ++it) {
        if (!wait_block()) break;
        const uint32_t taddr = tmem + ac.slot * N;
        const float* scale = sh->scale[it % Cfg::SLOTS];
        if constexpr (COLS) {
          // Fragments of 16 rows x 64 columns: a thread has 32 of the warp's columns, so that a warp reads a quarter of
          // the scales that it would with all 128 (a read of shared memory returns 128 bytes a cycle, also where all
          // threads read the same; those of 128 columns took 1000 cycles of an SM).
          const float* row = scale + 32 * q + (lane >> 2);
          const float* col = scale + ROWS + col0 + 2 * (lane & 3);
          uint64_t row2[4], col2[8];
#pragma unroll
          for (int i = 0; i < 4; ++i) row2[i] = pair(row[8 * i], row[8 * i]);
#pragma unroll
          for (int c = 0; c < kBigCols / 64; ++c) {
#pragma unroll
            for (int g = 0; g < 8; ++g) col2[g] = *reinterpret_cast<const uint64_t*>(&col[64 * c + 8 * g]);
#pragma unroll
            for (int h = 0; h < 2; ++h) {  // rows 16 h ..
              uint32_t v[32];
              tmem_ld_fragment(taddr + 64 * c + ((uint32_t)h << 20), v);
              tmem_wait_ld();
              if (c == kBigCols / 64 - 1 && h == 1) release();
              // two multiplications per value: in pairs they take 20% less time (one per value does not gain from it)
#pragma unroll
              for (int j = 0; j < 32; j += 2) {
                float* o = &acc[64 * c + 32 * h + j];
                const uint64_t scaled = mul2(pair(v[j], v[j + 1]), row2[2 * h + (j / 2) % 2]);
                unpair(fma2(scaled, col2[j / 4], pair(o[0], o[1])), o[0], o[1]);
              }
            }
          }
        } else {
          // One multiplication per value, by the product of the scales; by one after the other where that leaves the
          // normal numbers (a sum times both may not), as the other kernels multiply.  The choice costs 2 us of 140.
          uint32_t v[2][16];
          tmem_ld16(taddr, v[0]);
          const float sx = scale[32 * q + lane], sw = scale[ROWS + col0 / 128], s = sx * sw;
          auto add_block = [&](auto apart) {
#pragma unroll
            for (int c = 0; c < kBigCols / 16; ++c) {
              tmem_wait_ld();
              if (c < kBigCols / 16 - 1)
                tmem_ld16(taddr + 16 * (c + 1), v[(c + 1) & 1]);
              else
                release();
#pragma unroll
              for (int j = 0; j < 16; ++j) {
                const float f = __uint_as_float(v[c & 1][j]);
                acc[16 * c + j] = decltype(apart)::value ? fmaf(f * sx, sw, acc[16 * c + j]) : fmaf(f, s, acc[16 * c + j]);
              }
            }
          };
          const uint32_t exponent = __float_as_uint(s) & 0x7F800000u;
          if (__all_sync(0xFFFFFFFFu, exponent - 0x00800000u < 0x7F000000u))
            add_block(std::false_type());
          else
            add_block(std::true_type());
        }
      }
      if constexpr (Order::WALKS) {
        const auto part = walk.output(P, tiles);
        if constexpr (Order::ADDS) {
          // All that the sums are added to is asked for at once, a row per thread: the loads that follow, of which registers
          // hold a quarter at a time, then wait for memory once and not four times (32 x 2048 x 2048 from 8192 x 4 slots 281
          // us, 321 without; asked for while the sums are made it slows the operands' copies, 293 us)
          if (part.add && part.m0 + 32 * q + lane < part.M) {
            const float* row = part.add + (part.m0 + 32 * q + lane) * part.ld_add;
#pragma unroll
            for (int c = part.n0 + col0; c < part.n0 + col0 + kBigCols; c += 32)
              if (c < part.N) asm volatile("prefetch.global.L2 [%0];" ::"l"(row + c));
          }
        }
        if constexpr (WIDE)
          store_wide<!COLS>(part, part.m0 + 32 * q, part.n0 + col0, acc);
        else
          store_narrow<!COLS>(part, part.m0 + 32 * q, part.n0 + col0, acc, sh->patch[e]);
        walk.next(tiles);
      } else {
        int m0, n0;
        tiles.at(t, m0, n0);
        if constexpr (WIDE)
          store_wide<!COLS>(P, m0 + 32 * q, n0 + col0, acc);
        else
          store_narrow<!COLS>(P, m0 + 32 * q, n0 + col0, acc, sh->patch[e]);
        t += gridDim.x;
      }
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (warp == 1) {
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(BIG_ACC * N)
                 : "memory");
  }
}

int read_and_clear_fault() {
  int v = 0;
  if (cudaMemcpyFromSymbol(&v, g_f8_fault, sizeof(int)) != cudaSuccess) return -1;
  const int zero = 0;
  if (v != 0 && cudaMemcpyToSymbol(g_f8_fault, &zero, sizeof(int)) != cudaSuccess) return -1;
  return v;
}

bool make_map(CUtensorMap* map, const ds_f8_matrix* m, uint32_t box_rows) {
  return make_map_2d(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, m->q, m->cols, m->rows, m->ld, BK, box_rows);
}

Scales scales_at(const ds_f8_matrix* m) {
  return Scales{m->scale, m->ld_scale, m->blocks == DS_F8_TILES ? 7 : 0};
}

// kind::f8f6f4: float32 D, the formats of A (along the lanes) and B, both K-major; the tile's shape is added later.
uint32_t idesc_of(const ds_f8_matrix* a, const ds_f8_matrix* b) {
  return (1u << 4) | ((uint32_t)a->format << 7) | ((uint32_t)b->format << 10);
}

}  // namespace
}  // namespace ds
