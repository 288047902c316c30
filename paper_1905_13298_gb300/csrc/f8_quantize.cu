// Conversion to 8-bit matrices with a scale per block of 128 values.
//
// Two kernels.  Rows alone (one scale per row and 128 columns): 16 lanes hold
// a block, 8 values each, and find its amax with four shuffles.  Tiles, and
// everything that is written transposed: a CTA holds a 128 x 128 tile in
// registers (an 8 x 8 patch per thread), takes row maxima by shuffles and
// column maxima through shared memory, and turns the tile around as bytes in
// shared memory, so that the source is read once whatever is written from it.
#include "f8_common.cuh"

namespace ds {
namespace {

constexpr int kThreads = 256;

// Sources: eight values (r, c .. c + 7) of which n exist.
template <typename T>
struct SourceFloat {
  const T* p;
  int64_t ld;
  bool vec;
  __device__ __forceinline__ void load(int64_t r, int64_t c, int n, float v[8]) const {
    Raw8<T> raw;
    raw.load(p + r * ld + c, n, vec);
    raw.get(v);
  }
};
struct SourceF8 {
  const uint8_t* q;
  const float* s;
  int64_t ld, lds;
  bool e5m2, tiles;
  __device__ __forceinline__ void load(int64_t r, int64_t c, int n, float v[8]) const {
    const uint8_t* p = q + r * ld + c;
    uint2 u = make_uint2(0u, 0u);
    if (n >= 8) {
      u = *reinterpret_cast<const uint2*>(p);
    } else {
      for (int i = 0; i < n; ++i) {
        const uint32_t b = p[i];
        if (i < 4)
          u.x |= b << (8 * i);
        else
          u.y |= b << (8 * (i - 4));
      }
    }
    f8x8_value(u, e5m2, v);
    const float sc = n > 0 ? s[(tiles ? r / kF8Block : r) * lds + c / kF8Block] : 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? v[i] * sc : 0.f;
  }
};

__device__ __forceinline__ int left8(int64_t cols, int64_t c) {
  const int64_t n = cols - c;
  return n >= 8 ? 8 : (n < 0 ? 0 : (int)n);
}

template <typename Source>
__global__ void __launch_bounds__(kThreads) quantize_rows_kernel(const Source src, int64_t rows, int64_t cols,
                                                                 const F8Out out, bool pow2) {
  const int64_t nb = (cols + kF8Block - 1) / kF8Block;
  const int64_t total = rows * nb;
  const int sub = threadIdx.x & 15;
  const int64_t first = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> 4;
  const int64_t step = (int64_t)gridDim.x * (kThreads / 16);
  // both halves of a warp take the same number of rounds: the shuffles are full
  for (int64_t base = first & ~(int64_t)1; base < total; base += step) {
    const int64_t i = base + (first & 1);
    const bool in = i < total;
    const int64_t r = in ? i / nb : 0, b = in ? i - r * nb : 0;
    const int64_t c = b * kF8Block + sub * 8;
    const int n = in ? left8(cols, c) : 0;
    float v[8];
    src.load(r, n > 0 ? c : 0, n, v);
    const F8Scale s = f8_scale(max16(amax8(v)), out.e5m2, pow2);
    if (n > 0) store_q8(out.q + r * out.ld + c, n, f8x8(v, s.inv, out.e5m2));
    if (in && sub == 0) out.s[r * out.lds + b] = s.s;
  }
}

struct TileSmem {
  uint8_t turned[128 * 128];  // [column][row], 8-byte chunks XOR-swizzled
  float col_max[kThreads / 32][128];
};

template <typename Source>
__global__ void __launch_bounds__(kThreads) quantize_tile_kernel(const Source src, int64_t rows, int64_t cols,
                                                                 const F8Out out, const F8Out out_t, bool pow2) {
  __shared__ __align__(16) TileSmem sm;
  const int tr = threadIdx.x >> 4, tc = threadIdx.x & 15, warp = threadIdx.x >> 5;
  const int64_t tiles_c = (cols + kF8Block - 1) / kF8Block;
  const int64_t tile_r = blockIdx.x / tiles_c, tile_c = blockIdx.x - tile_r * tiles_c;
  const int64_t r0 = tile_r * kF8Block + tr * 8, c0 = tile_c * kF8Block + tc * 8;
  const int n = left8(cols, c0), m = left8(rows, r0);
  float v[8][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) src.load(i < m ? r0 + i : 0, n > 0 ? c0 : 0, i < m ? n : 0, v[i]);

  float cm[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    cm[j] = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) cm[j] = fmaxf(cm[j], finite_abs(v[i][j]));
    cm[j] = fmaxf(cm[j], __shfl_xor_sync(0xFFFFFFFFu, cm[j], 16));
  }
  if ((threadIdx.x & 16) == 0) {
#pragma unroll
    for (int j = 0; j < 8; ++j) sm.col_max[warp][tc * 8 + j] = cm[j];
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    cm[j] = 0.f;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) cm[j] = fmaxf(cm[j], sm.col_max[w][tc * 8 + j]);
  }
  float tile_max = 0.f;
  if (out.tiles || out_t.tiles) {
#pragma unroll
    for (int j = 0; j < 8; ++j) tile_max = fmaxf(tile_max, cm[j]);
    tile_max = max16(tile_max);
  }

  if (out.q) {
    const F8Scale t = f8_scale(tile_max, out.e5m2, pow2);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const F8Scale s = out.tiles ? t : f8_scale(max16(amax8(v[i])), out.e5m2, pow2);
      if (i < m) {
        if (n > 0) store_q8(out.q + (r0 + i) * out.ld + c0, n, f8x8(v[i], s.inv, out.e5m2));
        if (!out.tiles && tc == 0) out.s[(r0 + i) * out.lds + tile_c] = s.s;
      }
    }
    if (out.tiles && threadIdx.x == 0) out.s[tile_r * out.lds + tile_c] = t.s;
  }
  if (out_t.q) {
    const F8Scale t = f8_scale(tile_max, out_t.e5m2, pow2);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const F8Scale s = out_t.tiles ? t : f8_scale(cm[j], out_t.e5m2, pow2);
      float u[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] = v[i][j];
      const uint2 q = f8x8(u, s.inv, out_t.e5m2);
      *reinterpret_cast<uint2*>(&sm.turned[(tc * 8 + j) * 128 + ((tr ^ tc) << 3)]) = q;
      if (!out_t.tiles && tr == 0 && j < n) out_t.s[(c0 + j) * out_t.lds + tile_r] = s.s;
    }
    if (out_t.tiles && threadIdx.x == 0) out_t.s[tile_c * out_t.lds + tile_r] = t.s;
    __syncthreads();
    // 16 lanes write one 128-byte row of the transposed matrix
    const int64_t rr = tile_r * kF8Block + tc * 8;
    const int nr = left8(rows, rr);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int col = tr + 16 * k;
      const int64_t c = tile_c * kF8Block + col;
      if (c < cols && nr > 0)
        store_q8(out_t.q + c * out_t.ld + rr, nr,
                 *reinterpret_cast<const uint2*>(&sm.turned[col * 128 + ((tc ^ (col >> 3)) << 3)]));
    }
  }
}

template <typename Source>
cudaError_t run(const Source& src, int64_t rows, int64_t cols, const F8Out& out, const F8Out& out_t, bool pow2,
                cudaStream_t st) {
  const int64_t nb = (cols + kF8Block - 1) / kF8Block;
  if (out_t.q == nullptr && !out.tiles) {
    const int64_t want = (rows * nb + kThreads / 16 - 1) / (kThreads / 16);
    const int64_t cap = (int64_t)(sm_count() > 0 ? sm_count() : 1) * 32;
    quantize_rows_kernel<<<(unsigned)(want < cap ? want : cap), kThreads, 0, st>>>(src, rows, cols, out, pow2);
  } else {
    const int64_t tiles = (rows + kF8Block - 1) / kF8Block * nb;
    quantize_tile_kernel<<<(unsigned)tiles, kThreads, 0, st>>>(src, rows, cols, out, out_t, pow2);
  }
  return cudaGetLastError();
}

template <typename T>
cudaError_t run_float(const void* x, int64_t rows, int64_t cols, int64_t ldx, const F8Out& out, const F8Out& out_t,
                      bool pow2, cudaStream_t st) {
  const bool vec = (reinterpret_cast<uintptr_t>(x) & 15) == 0 && ldx * sizeof(T) % 16 == 0;
  return run(SourceFloat<T>{static_cast<const T*>(x), ldx, vec}, rows, cols, out, out_t, pow2, st);
}

// Shift weights as 8-bit tiles: s * 2^p = (s * 2^(p + 8)) * 2^-8, exact in e4m3 (2^-7, its smallest magnitude here, is a
// subnormal that the format holds exactly).  One thread writes four codes.
__global__ void __launch_bounds__(kThreads) expand_f8_kernel(const uint8_t* __restrict__ blob, int64_t n_out,
                                                             int64_t k_red, const F8Out out) {
  const BlobLayout L = blob_layout(n_out, k_red);
  const int64_t quads = (k_red + 3) / 4, total = n_out * quads;
  for (int64_t e = blockIdx.x * (int64_t)blockDim.x + threadIdx.x; e < total; e += (int64_t)gridDim.x * blockDim.x) {
    const int64_t n = e / quads, k = (e - n * quads) * 4;
    const int64_t rec = (k >> 5) * n_out + n;
    const uint32_t nib = reinterpret_cast<const uint32_t*>(blob + L.nib + rec * 16)[(k >> 3) & 3] >> (4 * (k & 7));
    const uint2 b = reinterpret_cast<const uint2*>(blob + L.bits + rec * 8)[0];
    const int j = (int)(k & 31);
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float mag = __uint_as_float((135u - ((nib >> (4 * i)) & 15u)) << 23);  // 2^(8 + p)
      v[i] = ((b.y >> (j + i)) & 1u) ? (((b.x >> (j + i)) & 1u) ? -mag : mag) : 0.f;
    }
    const uint32_t q = f8x2(v[0], v[1], false) | (f8x2(v[2], v[3], false) << 16);
    uint8_t* o = out.q + n * out.ld + k;
    if (k + 4 <= k_red) {
      *reinterpret_cast<uint32_t*>(o) = q;
    } else {
      for (int i = 0; k + i < k_red; ++i) o[i] = (uint8_t)(q >> (8 * i));
    }
    if (n % kF8Block == 0 && k % kF8Block == 0) out.s[n / kF8Block * out.lds + k / kF8Block] = 0.00390625f;
  }
}

}  // namespace

cudaError_t launch_quantize_f8(const void* x, int type, int64_t rows, int64_t cols, int64_t ldx, const F8Out& out,
                               const F8Out& out_t, bool pow2, cudaStream_t st) {
  if (type == DS_TYPE_F32) return run_float<float>(x, rows, cols, ldx, out, out_t, pow2, st);
  if (type == DS_TYPE_BF16) return run_float<__nv_bfloat16>(x, rows, cols, ldx, out, out_t, pow2, st);
  return run_float<__half>(x, rows, cols, ldx, out, out_t, pow2, st);
}

cudaError_t launch_requantize_f8(const ds_f8_matrix* in, const F8Out& out, const F8Out& out_t, bool pow2,
                                 cudaStream_t st) {
  const SourceF8 src{static_cast<const uint8_t*>(in->q), in->scale, in->ld, in->ld_scale, in->format == DS_F8_E5M2,
                     in->blocks == DS_F8_TILES};
  return run(src, in->rows, in->cols, out, out_t, pow2, st);
}

cudaError_t launch_expand_f8(const uint8_t* blob, int64_t n_out, int64_t k_red, const F8Out& out, cudaStream_t st) {
  const int64_t want = (n_out * ((k_red + 3) / 4) + kThreads - 1) / kThreads;
  const int64_t cap = (int64_t)(sm_count() > 0 ? sm_count() : 1) * 32;
  expand_f8_kernel<<<(unsigned)(want < cap ? want : cap), kThreads, 0, st>>>(blob, n_out, k_red, out);
  return cudaGetLastError();
}

}  // namespace ds
