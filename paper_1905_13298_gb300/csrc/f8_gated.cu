// SiLU-gated activation whose inputs are kept in 8 bits for the backward pass.
//
//   forward   a = silu(g) u  -> 8 bits;  checkpoint: g and u -> 8 bits (both with a scale per row and 128 columns)
//   backward  du = da silu(g),  dg = da u sig(g) (1 + g (1 - sig(g))),  g and u read from the checkpoint;
//             written in 8 bits by rows (the operand of the input's gradient) and by columns (that of the
//             weight's), and a once more by columns (the operand of the next layer's weight gradient)
//
// g and u are two halves of one matrix; the up half starts at the next
// multiple of 128 columns so that no block holds values of both.  Nothing but
// the 8-bit checkpoint outlives the forward pass: 2 bytes per gate instead of
// the 4 of a bf16 pair, and a is made again rather than kept.
//
// The forward pass streams: 16 lanes hold a block of each of g, u and a.  The
// backward pass walks 128 x 128 tiles, one CTA per SM, 4 rows x 8 columns of a
// tile per thread, and writes its five 8-bit outputs from registers, so the
// checkpoint and da are read once.  Three results of 16384 float32 fill most of
// an SM's registers, so no second CTA can hide the first one's reads: TMA
// brings the next tile to shared memory while this one is rounded and stored.
//
// Measured in bf16: forward 4095 x 8200 with the checkpoint 54 us (4.4 TB/s;
// bound by instructions: the sigmoid, conversions, maxima and scales), 8192 x
// 4096 without it 44 us (3.8 TB/s); backward 8192 x 8192 160 us (3.9 TB/s: a
// tile's phases, sigmoid, maxima, scales, rounding and turning, are parted by
// barriers that nothing else on the SM fills).
#include <type_traits>

#include "f8_common.cuh"
#include "tensor_core.cuh"

namespace ds {

__device__ int g_gated_fault;  // set when a bounded wait of the backward pass gives up

namespace {

constexpr int kThreads = 128;
constexpr int kTileThreads = 512;
constexpr int kTileWarps = kTileThreads / 32;

__device__ __forceinline__ float rcp(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ uint64_t both(float v) { return pair(v, v); }
// sig(g) = z / (1 + z) or 1 / (1 + z) with z = e^-|g|, as exact as an exponential, a sum and a quotient in float32: 1 + z
// is 1 .. 2, and the quotient by its approximate reciprocal is corrected by the remainder.  2^x of the special-function
// unit alone would take 15% less time in all (gate 4095 x 8200 46 us), but the rounding of x = -|g| log2 e costs |g| 2^-24:
// g sig(g) in the mean square 1.7e-6 off at g = -86 .. -60, 5e-8 here.
__device__ __forceinline__ uint64_t sigmoid2(uint64_t g) {
  float g0, g1, d0, d1;
  unpair(g, g0, g1);
  const float z0 = expf(-fabsf(g0)), z1 = expf(-fabsf(g1));
  const uint64_t minus_d = fma2(pair(z0, z1), both(-1.f), both(-1.f));
  unpair(minus_d, d0, d1);
  const uint64_t n = pair(g0 < 0.f ? z0 : 1.f, g1 < 0.f ? z1 : 1.f), r = pair(rcp(-d0), rcp(-d1)), q = mul2(n, r);
  return fma2(fma2(minus_d, q, n), r, q);
}

// Two rows of a unit (a block of 128 features) at a time: with the checkpoint six blocks, whose scales six lanes make.
// Small CTAs of 64 registers keep 32 warps on an SM; the next unit's inputs held beside this one's (118 registers, 16
// warps) took 30% longer.
constexpr int R = 2;

template <typename T, bool E5M2>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? 8 : 6)
    gated_f8_kernel(const T* gu, int64_t ld, bool vec, int64_t rows, int64_t features, const F8Out out, const F8Out ckpt,
                    bool pow2) {
  const int64_t nb = (features + kF8Block - 1) / kF8Block, up = nb * kF8Block, groups = (rows + R - 1) / R;
  const int sub = threadIdx.x & 15;
  Units at(((int64_t)blockIdx.x * kThreads + threadIdx.x) >> 4, (int64_t)gridDim.x * (kThreads / 16), nb);
  for (; __any_sync(0xFFFFFFFFu, at.r < groups); at.next()) {
    const int64_t r0 = at.r * R, c = at.b * kF8Block + sub * 8;
    const bool in = at.r < groups;
    const int n = in ? left8(features, c) : 0;
    const int m = in ? (rows - r0 < R ? (int)(rows - r0) : R) : 0;
    Raw8<T> rg[R], ru[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const T* p = gu + (i < m ? r0 + i : 0) * ld + (n > 0 ? c : 0);
      rg[i].template load<true>(p, i < m ? n : 0, vec);
      ru[i].template load<true>(p + up, i < m ? n : 0, vec);
    }
    float a[R][8], mx[8];  // maxima of a, g and u of each row
    mx[6] = mx[7] = 0.f;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      float g[8], u[8];
      rg[i].get(g);
      ru[i].get(u);
#pragma unroll
      for (int j = 0; j < 8; j += 2) {
        const uint64_t gj = pair(g[j], g[j + 1]);
        unpair(mul2(mul2(gj, sigmoid2(gj)), pair(u[j], u[j + 1])), a[i][j], a[i][j + 1]);
      }
      mx[i] = amax8(a[i]);
      mx[2 + i] = ckpt.q ? amax8(g) : 0.f;
      mx[4 + i] = ckpt.q ? amax8(u) : 0.f;
    }
    float mine = lanes_max<8>(mx);
    const bool check = __any_sync(0xFFFFFFFFu, !(mine < kInf));
    if (check) {
#pragma unroll
      for (int i = 0; i < R; ++i) {
        float g[8], u[8];
        rg[i].get(g);
        ru[i].get(u);
        mx[i] = amax8_finite(a[i]);
        mx[2 + i] = amax8_finite(g);
        mx[4 + i] = amax8_finite(u);
      }
      mine = lanes_max<8>(mx);
    }
    const int which = sub & 7;  // the block whose scale this lane makes
    const F8Out& to = which < 2 ? out : ckpt;
    const F8Scale s = f8_scale<E5M2>(mine, pow2);
    if (sub < (ckpt.q ? 6 : 2) && (which & 1) < m)
      to.s[(r0 + (which & 1)) * to.lds + at.b + (which >= 4 ? nb : 0)] = s.s;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const float inv = of_lane(s.inv, i), inv_g = of_lane(s.inv, 2 + i), inv_u = of_lane(s.inv, 4 + i);
      const uint2 q = check ? f8x8<E5M2, true>(a[i], inv) : f8x8<E5M2, false>(a[i], inv);
      if (i < m && n > 0) store_q8(out.q + (r0 + i) * out.ld + c, n, q);
      if (ckpt.q && i < m) {
        float g[8], u[8];
        rg[i].get(g);
        ru[i].get(u);
        uint8_t* o = ckpt.q + (r0 + i) * ckpt.ld + c;
        // the columns between the halves are zeros
        *reinterpret_cast<uint2*>(o) = check ? f8x8<E5M2, true>(g, inv_g) : f8x8<E5M2, false>(g, inv_g);
        if (n > 0) store_q8(o + up, n, check ? f8x8<E5M2, true>(u, inv_u) : f8x8<E5M2, false>(u, inv_u));
      }
    }
  }
}

// The tile that TMA brings (rows as they lie in memory), its scales, and the results: each has its turned tile and
// column maxima, so that one pass of barriers serves all three.
template <typename T>
struct TileSmem {
  T da[128][128];
  uint8_t g[128][128], u[128][128];
  uint8_t turned[3][128 * 128];
  float col_max[3][kTileWarps][128];
  float col_inv[3][128];
  float scale[2][2][128];  // of g's and u's rows, of this tile and the next
  uint64_t full;
  int abort;
};

// A 4 x 8 patch of a result, its largest magnitudes by columns (the warp's 8 rows together) to shared memory.
template <bool CHECK>
__device__ __forceinline__ void column_maxima(float (*col_max)[128], const float v[4][8]) {
  const int tc = threadIdx.x & 15, warp = threadIdx.x >> 5;
  float cm[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if (CHECK) {
      cm[j] = fmaxf(fmaxf(finite_abs(v[0][j]), finite_abs(v[1][j])), fmaxf(finite_abs(v[2][j]), finite_abs(v[3][j])));
    } else {
      cm[j] = fmaxf(fmaxf(fabsf(v[0][j]), fabsf(v[1][j])), fmaxf(fabsf(v[2][j]), fabsf(v[3][j])));
    }
  }
  const bool up = threadIdx.x & 16;
  float c[4];
#pragma unroll
  for (int j = 0; j < 4; ++j)
    c[j] = fmaxf(up ? cm[j + 4] : cm[j], __shfl_xor_sync(0xFFFFFFFFu, up ? cm[j] : cm[j + 4], 16));
  *reinterpret_cast<float4*>(&col_max[warp][tc * 8 + (up ? 4 : 0)]) = make_float4(c[0], c[1], c[2], c[3]);
}

// The row form of a patch: m of its rows, n of its columns.  CHECK: the tile is not whole, or holds infinities.
template <bool E5M2, bool CHECK>
__device__ __forceinline__ void write_rows(const float v[4][8], const F8Out& out, int64_t r0, int64_t c0, int64_t block,
                                           int m, int n, bool pow2) {
  const int tc = threadIdx.x & 15;
  float rm[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) rm[i] = CHECK ? amax8_finite(v[i]) : amax8(v[i]);
  const float b = lanes_max<4>(rm);  // lane l of 16: row l & 3
  const F8Scale s = f8_scale<E5M2>(b, pow2);
  uint8_t* p = out.q + r0 * out.ld + c0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float inv = of_lane(s.inv, i);
    const uint2 q = f8x8<E5M2, CHECK>(v[i], inv);
    if (!CHECK)
      *reinterpret_cast<uint2*>(p) = q;
    else if (i < m && n > 0)
      store_q8(p, n, q);
    p += out.ld;
  }
  if (tc < m && tc < 4) out.s[(r0 + tc) * out.lds + block] = s.s;
}

// The patch by columns, as bytes, to the turned tile.
template <bool E5M2, bool CHECK>
__device__ __forceinline__ void turn_patch(uint8_t* turned, const float* col_inv, const float v[4][8]) {
  const int tr = threadIdx.x >> 4, tc = threadIdx.x & 15;
  const float4 lo = *reinterpret_cast<const float4*>(&col_inv[tc * 8]);
  const float4 hi = *reinterpret_cast<const float4*>(&col_inv[tc * 8 + 4]);
  const float inv[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
  uint32_t* to = reinterpret_cast<uint32_t*>(&turned[tc * 8 * 128 + (((tr >> 1) ^ tc) << 3) + ((tr & 1) << 2)]);
  uint32_t low[8], high[8];
  f8_columns<E5M2, CHECK>(v[0], v[1], inv, low);
  f8_columns<E5M2, CHECK>(v[2], v[3], inv, high);
#pragma unroll
  for (int j = 0; j < 8; ++j) to[j * 32] = low[j] | high[j] << 16;
}

template <typename T>
struct BackwardIn {
  const float* scale;  // of the checkpoint
  int64_t lds;
  const T* da;
  int64_t ld;
  bool vec;  // da's rows are aligned for TMA; otherwise a thread reads its own patch
  int64_t rows, features;
  long long wait_cycles;
};

// IN5, E5M2: the formats of the checkpoint and of what is written.
template <typename T, bool IN5, bool E5M2>
__global__ void __launch_bounds__(kTileThreads, 1)
    gated_f8_backward_kernel(const __grid_constant__ CUtensorMap map_ckpt, const __grid_constant__ CUtensorMap map_da,
                             const BackwardIn<T> B, const F8Out dgu, const F8Out dgu_t, const F8Out a_t, bool pow2) {
  extern __shared__ __align__(128) unsigned char smem_raw[];
  TileSmem<T>& sm = *reinterpret_cast<TileSmem<T>*>(smem_raw);
  const int tr = threadIdx.x >> 4, tc = threadIdx.x & 15;
  const int64_t rows = B.rows, features = B.features;
  const uint32_t nb = (uint32_t)((features + kF8Block - 1) / kF8Block);
  const uint32_t tiles = (uint32_t)((rows + kF8Block - 1) / kF8Block) * nb;
  const int64_t up = (int64_t)nb * kF8Block;
  // one thread: the copies of tile t
  auto bring = [&](uint32_t t) {
    const uint32_t r = t / nb, c = t - r * nb;
    mbar_expect_tx(&sm.full, sizeof(sm.g) + sizeof(sm.u) + (B.vec ? sizeof(sm.da) : 0));
    tma_load_2d(sm.g, &map_ckpt, &sm.full, (int)(c * kF8Block), (int)(r * kF8Block));
    tma_load_2d(sm.u, &map_ckpt, &sm.full, (int)(up + c * kF8Block), (int)(r * kF8Block));
    if (B.vec) tma_load_2d(sm.da, &map_da, &sm.full, (int)(c * kF8Block), (int)(r * kF8Block));
  };
  // threads 0 .. 255: the scale of row (thread % 128) of g or u in tile t
  auto scale_of = [&](uint32_t t) {
    const uint32_t tile_r = t / nb, tile_c = t - tile_r * nb;
    const int64_t r = (int64_t)tile_r * kF8Block + (threadIdx.x & 127);
    return r < rows ? B.scale[r * B.lds + tile_c + (threadIdx.x >= 128 ? nb : 0)] : 0.f;
  };
  if (threadIdx.x == 0) {
    mbar_init(&sm.full, 1);
    sm.abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    bring(blockIdx.x);
  }
  if (threadIdx.x < 256) sm.scale[0][threadIdx.x >> 7][threadIdx.x & 127] = scale_of(blockIdx.x);
  __syncthreads();
  uint32_t turn = 0;
  for (uint32_t tile = blockIdx.x; tile < tiles; tile += gridDim.x, turn ^= 1u) {
    const uint32_t tile_r = tile / nb, tile_c = tile - tile_r * nb;
    const int64_t r0 = (int64_t)tile_r * kF8Block + tr * 4, c_tile = (int64_t)tile_c * kF8Block, c0 = c_tile + tc * 8;
    const int n = left8(features, c0);
    const int m = rows - r0 >= 4 ? 4 : (rows - r0 < 0 ? 0 : (int)(rows - r0));
    const bool more = tile + gridDim.x < tiles;
    float next_scale = 0.f;
    if (more && threadIdx.x < 256) next_scale = scale_of(tile + gridDim.x);
    const bool ok = mbar_wait(&sm.full, turn, &sm.abort, B.wait_cycles, &g_gated_fault);
    float dg[4][8], du[4][8], a[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float d[8], g[8], u[8];
      const int row = tr * 4 + i;
      Raw8<T> rd;
      if (B.vec)
        rd.load(&sm.da[row][tc * 8], 8, true);
      else
        rd.load(B.da + (i < m ? r0 + i : 0) * B.ld + (n > 0 ? c0 : 0), i < m ? n : 0, false);
      rd.get(d);
      f8x8_value<IN5>(*reinterpret_cast<const uint2*>(&sm.g[row][tc * 8]), g);
      f8x8_value<IN5>(*reinterpret_cast<const uint2*>(&sm.u[row][tc * 8]), u);
      if (n < 8) {  // what lies between the halves is not read
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = j < n ? g[j] : 0.f;
      }
      const float sg = sm.scale[turn][0][row], su = sm.scale[turn][1][row];
#pragma unroll
      for (int j = 0; j < 8; j += 2) {  // two columns per instruction
        const uint64_t gj = mul2(pair(g[j], g[j + 1]), pair(sg, sg)), uj = mul2(pair(u[j], u[j + 1]), pair(su, su));
        const uint64_t dj = pair(d[j], d[j + 1]), sig = sigmoid2(gj), act = mul2(gj, sig);
        unpair(mul2(act, uj), a[i][j], a[i][j + 1]);
        unpair(mul2(dj, act), du[i][j], du[i][j + 1]);
        // sig (1 + g (1 - sig))
        const uint64_t slope = fma2(act, fma2(sig, pair(-1.f, -1.f), pair(1.f, 1.f)), sig);
        unpair(mul2(mul2(dj, uj), slope), dg[i][j], dg[i][j + 1]);
      }
    }
    const int cols = features - c_tile >= kF8Block ? kF8Block : (int)(features - c_tile);
    const bool full = cols == kF8Block && (int64_t)(tile_r + 1) * kF8Block <= rows;
    // a column's scale each: of dg, du and a; the gate half's columns go on to the up half with zeros
    const int which = threadIdx.x >> 7, c = threadIdx.x & 127;
    const F8Out& out = which < 2 ? dgu_t : a_t;
    auto column_scales = [&] {
      float mx = 0.f;
      if (which < 3) {
#pragma unroll
        for (int w = 0; w < kTileWarps; ++w) mx = fmaxf(mx, sm.col_max[which][w][c]);
        const F8Scale s = f8_scale<E5M2>(mx, pow2);
        sm.col_inv[which][c] = s.inv;
        if (out.q && mx < kInf && (which == 0 || c < cols))
          out.s[((which == 1 ? up : 0) + c_tile + c) * out.lds + tile_r] = s.s;
      }
      return mx;
    };
    auto maxima = [&](auto finite) {
      column_maxima<decltype(finite)::value>(sm.col_max[0], dg);
      column_maxima<decltype(finite)::value>(sm.col_max[1], du);
      column_maxima<decltype(finite)::value>(sm.col_max[2], a);
    };
    auto emit = [&](auto finite) {
      constexpr bool CHECK = decltype(finite)::value;
      if (dgu.q) {
        write_rows<E5M2, CHECK>(dg, dgu, r0, c0, tile_c, m, 8, pow2);
        write_rows<E5M2, CHECK>(du, dgu, r0, up + c0, nb + tile_c, m, n, pow2);
      }
      if (dgu_t.q) {
        turn_patch<E5M2, CHECK>(sm.turned[0], sm.col_inv[0], dg);
        turn_patch<E5M2, CHECK>(sm.turned[1], sm.col_inv[1], du);
      }
      if (a_t.q) turn_patch<E5M2, CHECK>(sm.turned[2], sm.col_inv[2], a);
    };
    maxima(std::false_type());
    if (__syncthreads_or(!ok)) {
      if (threadIdx.x == 0) mbar_drain(&sm.full, turn);  // the copies land before the CTA leaves
      break;
    }
    // the tile is in registers: the next one may come
    if (more && threadIdx.x == 0) bring(tile + gridDim.x);
    if (more && threadIdx.x < 256) sm.scale[turn ^ 1u][threadIdx.x >> 7][threadIdx.x & 127] = next_scale;
    // an infinity anywhere is some column's largest magnitude
    if (__syncthreads_or(!(column_scales() < kInf))) {
      maxima(std::true_type());
      __syncthreads();
      column_scales();
      __syncthreads();
      emit(std::true_type());
    } else if (!full) {
      emit(std::true_type());
    } else {
      emit(std::false_type());
    }
    __syncthreads();
    const int64_t first = (int64_t)tile_r * kF8Block;
    auto write = [&](auto whole) {
      constexpr bool FULL = decltype(whole)::value;
      if (dgu_t.q) {
        write_turned<kTileThreads, FULL>(sm.turned[0], dgu_t.q + c_tile * dgu_t.ld, dgu_t.ld, first, rows, kF8Block);
        write_turned<kTileThreads, FULL>(sm.turned[1], dgu_t.q + (up + c_tile) * dgu_t.ld, dgu_t.ld, first, rows, cols);
      }
      if (a_t.q) write_turned<kTileThreads, FULL>(sm.turned[2], a_t.q + c_tile * a_t.ld, a_t.ld, first, rows, cols);
    };
    if (full)
      write(std::true_type());
    else
      write(std::false_type());
    // the next tile's maxima are written before a barrier, its turned tiles after two: nobody still reads these
  }
}

template <typename T>
cudaError_t forward(const void* gu, int64_t ld, int64_t rows, int64_t features, const F8Out& out, const F8Out& ckpt,
                    bool e5m2, bool pow2, cudaStream_t st) {
  const int64_t nb = (features + kF8Block - 1) / kF8Block;
  const int64_t want = ((rows + R - 1) / R * nb + kThreads / 16 - 1) / (kThreads / 16);
  const int64_t cap = (int64_t)(sm_count() > 0 ? sm_count() : 1) * 32;
  const bool vec = (reinterpret_cast<uintptr_t>(gu) & 15) == 0 && ld * sizeof(T) % 16 == 0;
  auto* kernel = e5m2 ? gated_f8_kernel<T, true> : gated_f8_kernel<T, false>;
  kernel<<<(unsigned)(want < cap ? want : cap), kThreads, 0, st>>>(static_cast<const T*>(gu), ld, vec, rows, features,
                                                                   out, ckpt, pow2);
  return cudaGetLastError();
}

template <typename T, bool IN5, bool E5M2>
cudaError_t backward_as(const ds_f8_matrix* ckpt, const void* da, int64_t ld, int64_t features, const F8Out& dgu,
                        const F8Out& dgu_t, const F8Out& a_t, bool pow2, cudaStream_t st) {
  const int64_t tiles = (ckpt->rows + kF8Block - 1) / kF8Block * ((features + kF8Block - 1) / kF8Block);
  const bool vec = (reinterpret_cast<uintptr_t>(da) & 15) == 0 && ld * sizeof(T) % 16 == 0;
  // once per process, thread-safe (function-local static)
  static const cudaError_t attr =
      cudaFuncSetAttribute(gated_f8_backward_kernel<T, IN5, E5M2>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                           (int)sizeof(TileSmem<T>));
  if (attr != cudaSuccess) return attr;
  const CUtensorMapDataType type = std::is_same<T, float>::value    ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                   : std::is_same<T, __half>::value ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16
                                                                    : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
  CUtensorMap map_ckpt, map_da = {};
  if (!make_map_2d(&map_ckpt, CU_TENSOR_MAP_DATA_TYPE_UINT8, ckpt->q, ckpt->cols, ckpt->rows, ckpt->ld, kF8Block,
                   kF8Block, CU_TENSOR_MAP_SWIZZLE_NONE) ||
      (vec && !make_map_2d(&map_da, type, da, features, ckpt->rows, ld * (int64_t)sizeof(T), kF8Block, kF8Block,
                           CU_TENSOR_MAP_SWIZZLE_NONE)))
    return cudaErrorInvalidValue;
  const BackwardIn<T> in{ckpt->scale, ckpt->ld_scale, static_cast<const T*>(da), ld, vec, ckpt->rows, features,
                         f8_wait_cycles()};
  const int64_t sms = sm_count() > 0 ? sm_count() : 1;
  gated_f8_backward_kernel<T, IN5, E5M2><<<(unsigned)(tiles < sms ? tiles : sms), kTileThreads, sizeof(TileSmem<T>),
                                           st>>>(map_ckpt, map_da, in, dgu, dgu_t, a_t, pow2);
  return cudaGetLastError();
}

template <typename T>
cudaError_t backward(const ds_f8_matrix* ckpt, const void* da, int64_t ld, int64_t features, const F8Out& dgu,
                     const F8Out& dgu_t, const F8Out& a_t, bool e5m2, bool pow2, cudaStream_t st) {
  auto* run = ckpt->format == DS_F8_E5M2 ? (e5m2 ? backward_as<T, true, true> : backward_as<T, true, false>)
                                         : (e5m2 ? backward_as<T, false, true> : backward_as<T, false, false>);
  return run(ckpt, da, ld, features, dgu, dgu_t, a_t, pow2, st);
}

}  // namespace

cudaError_t launch_gated_f8(const void* gu, int type, int64_t ld, int64_t rows, int64_t features, const F8Out& out,
                            const F8Out& ckpt, bool e5m2, bool pow2, cudaStream_t st) {
  if (type == DS_TYPE_F32) return forward<float>(gu, ld, rows, features, out, ckpt, e5m2, pow2, st);
  if (type == DS_TYPE_BF16) return forward<__nv_bfloat16>(gu, ld, rows, features, out, ckpt, e5m2, pow2, st);
  return forward<__half>(gu, ld, rows, features, out, ckpt, e5m2, pow2, st);
}

cudaError_t launch_gated_f8_backward(const ds_f8_matrix* ckpt, const void* da, int type, int64_t ld, int64_t features,
                                     const F8Out& dgu, const F8Out& dgu_t, const F8Out& a_t, bool e5m2, bool pow2,
                                     cudaStream_t st) {
  if (type == DS_TYPE_F32) return backward<float>(ckpt, da, ld, features, dgu, dgu_t, a_t, e5m2, pow2, st);
  if (type == DS_TYPE_BF16) return backward<__nv_bfloat16>(ckpt, da, ld, features, dgu, dgu_t, a_t, e5m2, pow2, st);
  return backward<__half>(ckpt, da, ld, features, dgu, dgu_t, a_t, e5m2, pow2, st);
}

int read_gated_f8_fault_flag() {
  int v = 0;
  if (cudaMemcpyFromSymbol(&v, g_gated_fault, sizeof(int)) != cudaSuccess) return -1;
  const int zero = 0;
  if (v != 0 && cudaMemcpyToSymbol(g_gated_fault, &zero, sizeof(int)) != cudaSuccess) return -1;
  return v;
}

}  // namespace ds
