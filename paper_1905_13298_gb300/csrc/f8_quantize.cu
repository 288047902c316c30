// Conversion to 8-bit matrices with a scale per block of 128 values.
//
// Two kernels.  Rows alone (one scale per row and 128 columns): 16 lanes hold
// a block, 8 values each, and find its amax with four shuffles.  Tiles, and
// everything that is written transposed: a CTA holds a 128 x 128 tile in
// registers (an 8 x 8 patch per thread, 16-bit sources as they came), takes row
// maxima by shuffles and column maxima through shared memory, and turns the
// tile around as bytes in shared memory, so that the source is read once
// whatever is written from it.  Both are bound by HBM where their instructions
// fit beside it: a tile's are about 10 per value and direction, and infinities
// (the only values that need more) send the tile down a second path.
//
// Measured at 8192 x 4096: bf16 to rows 18.8 us (5.4 TB/s), to tiles 19.1
// (5.3), to rows and transposed rows 25.4 (5.4), float32 to rows 26.4 (6.4).
// 8-bit rows to transposed rows, 4096 x 8192: 24.4 us (2.8 TB/s), bound by
// instructions: each value is decoded twice, once for its column's maximum and
// once to be rounded, since decoded tiles would leave room for one CTA of an SM.
#include "f8_common.cuh"

namespace ds {
namespace {

constexpr int kThreads = 256;

// Sources: eight values (r, c .. c + 7), of which n exist, as a Raw that gives them in float32 and their largest
// magnitudes.
template <typename T>
struct SourceFloat {
  using Raw = Raw8<T>;
  static constexpr bool PACKED = sizeof(T) == 2;    // 16-bit values: maxima of their bits, two at a time
  static constexpr int CTAS = sizeof(T) == 2 ? 4 : 2;  // that the registers of a tile's patches let share an SM
  const T* p;
  int64_t ld;
  bool vec;
  __device__ __forceinline__ void load(int64_t r, int64_t c, int n, Raw& raw) const {
    raw.template load<true>(p + r * ld + c, n, vec);
  }
};
// Eight 8-bit values and their scale, decoded where they are used: an eighth of the registers of the values.
template <bool E5M2>
struct RawF8 {
  static constexpr bool PAIRS = false;  // in tiles they would not fit in the registers (24 us, 27 with pairs)
  uint2 u;
  float s;
  __device__ __forceinline__ void get(float v[8]) const {
    f8x8_value<E5M2>(u, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= s;
  }
};
template <bool E5M2>
struct SourceF8 {
  using Raw = RawF8<E5M2>;
  static constexpr bool PACKED = false;
  static constexpr int CTAS = 3;
  const uint8_t* q;
  const float* s;
  int64_t ld, lds;
  bool tiles;
  __device__ __forceinline__ void load(int64_t r, int64_t c, int n, Raw& raw) const {
    raw.u = load_q8(q + r * ld + c, n);
    raw.s = n > 0 ? s[(tiles ? r / kF8Block : r) * lds + c / kF8Block] : 0.f;
  }
};

// Rows alone: 16 lanes hold one block of each of R rows.
constexpr int R = 4;
template <typename Source, bool E5M2>
__global__ void __launch_bounds__(kThreads) quantize_rows_kernel(const Source src, int64_t rows, int64_t cols,
                                                                 const F8Out out, bool pow2) {
  const int64_t nb = (cols + kF8Block - 1) / kF8Block, groups = (rows + R - 1) / R;
  const int sub = threadIdx.x & 15;
  // both halves of a warp go on until the later one is done: the shuffles are full
  Units at(((int64_t)blockIdx.x * kThreads + threadIdx.x) >> 4, (int64_t)gridDim.x * (kThreads / 16), nb);
  for (; __any_sync(0xFFFFFFFFu, at.r < groups); at.next()) {
    const int64_t r0 = at.r * R, c = at.b * kF8Block + sub * 8;
    const int n = at.r < groups ? left8(cols, c) : 0;
    const int m = at.r < groups ? (rows - r0 < R ? (int)(rows - r0) : R) : 0;
    typename Source::Raw raw[R];
#pragma unroll
    for (int i = 0; i < R; ++i) src.load(i < m ? r0 + i : 0, n > 0 ? c : 0, i < m ? n : 0, raw[i]);
    float rm[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      float v[8];
      raw[i].get(v);
      rm[i] = amax8(v);
    }
    float mx = lanes_max<R>(rm);
    const bool check = __any_sync(0xFFFFFFFFu, !(mx < kInf));
    if (check) {
#pragma unroll
      for (int i = 0; i < R; ++i) {
        float v[8];
        raw[i].get(v);
        rm[i] = amax8_finite(v);
      }
      mx = lanes_max<R>(rm);
    }
    const F8Scale s = f8_scale<E5M2>(mx, pow2);
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const float inv = of_lane(s.inv, i);
      float v[8];
      raw[i].get(v);
      const uint2 q = check ? f8x8<E5M2, true>(v, inv) : f8x8<E5M2, false>(v, inv);
      if (i < m && n > 0) store_q8(out.q + (r0 + i) * out.ld + c, n, q);
    }
    if (sub < m) out.s[(r0 + sub) * out.lds + at.b] = s.s;
  }
}

struct TileSmem {
  uint8_t turned[128 * 128];  // [column][row], 8-byte chunks XOR-swizzled
  float col_max[kThreads / 32][128];
  float col_inv[128];
  float warp_max[kThreads / 32];
};

// Largest magnitudes of the patch's rows and columns; where a value is not finite its row's is not either.
template <typename Source>
__device__ __forceinline__ void patch_maxima(const typename Source::Raw (&raw)[8], float rm[8], float cm[8]) {
  if constexpr (Source::PACKED) {
    uint32_t col[4] = {0u, 0u, 0u, 0u};
    typename Source::Raw out;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t w[4] = {raw[i].u.x & 0x7FFF7FFFu, raw[i].u.y & 0x7FFF7FFFu, raw[i].u.z & 0x7FFF7FFFu,
                             raw[i].u.w & 0x7FFF7FFFu};
#pragma unroll
      for (int k = 0; k < 4; ++k) col[k] = __vmaxu2(col[k], w[k]);
      const uint32_t m = __vmaxu2(__vmaxu2(w[0], w[1]), __vmaxu2(w[2], w[3]));
      out.u = make_uint4(m, 0u, 0u, 0u);
      float v[8];
      out.get(v);
      // comparisons that keep a NaN: the bits of NaN are the largest
      rm[i] = (m & 0xFFFFu) > (m >> 16) ? v[0] : v[1];
    }
    out.u = make_uint4(col[0], col[1], col[2], col[3]);
    out.get(cm);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) cm[j] = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float v[8];
      raw[i].get(v);
      rm[i] = amax8(v);
#pragma unroll
      for (int j = 0; j < 8; ++j) cm[j] = fmaxf(cm[j], fabsf(v[j]));
    }
  }
}

struct TileAt {
  int64_t rows, cols, r0, c0, tile_r, tile_c;
  int m, n;  // rows and columns of the patch that exist
};

// CHECK: the tile is not whole, or holds infinities.
template <typename Raw, bool E5M2, bool CHECK>
__device__ __forceinline__ void write_rows(const Raw (&raw)[8], float row_max, const F8Out& out, const TileAt& t,
                                           float tile_max, bool pow2) {
  const int lane = threadIdx.x & 31, tc = lane & 15;
  const F8Scale s = f8_scale<E5M2>(out.tiles ? tile_max : row_max, pow2);  // lane i of 16: row i's
  uint8_t* p = out.q + t.r0 * out.ld + t.c0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float inv = of_lane(s.inv, i);
    float v[8];
    raw[i].get(v);
    const uint2 q = f8x8<E5M2, CHECK, Raw::PAIRS>(v, inv);
    if (!CHECK)
      *reinterpret_cast<uint2*>(p) = q;
    else if (i < t.m && t.n > 0)
      store_q8(p, t.n, q);
    p += out.ld;
  }
  if (!out.tiles) {
    if (tc < t.m && tc < 8) out.s[(t.r0 + tc) * out.lds + t.tile_c] = s.s;
  } else if (threadIdx.x == 0) {
    out.s[t.tile_r * out.lds + t.tile_c] = s.s;
  }
}

template <typename Raw, bool E5M2, bool CHECK>
__device__ __forceinline__ void turn_columns(const Raw (&raw)[8], TileSmem& sm) {
  const int tr = threadIdx.x >> 4, tc = threadIdx.x & 15;
  float inv[8];
#pragma unroll
  for (int j = 0; j < 8; j += 4) {
    const float4 f = *reinterpret_cast<const float4*>(&sm.col_inv[tc * 8 + j]);
    inv[j] = f.x, inv[j + 1] = f.y, inv[j + 2] = f.z, inv[j + 3] = f.w;
  }
  uint2 q[8];  // column j: rows 0 .. 7 of the patch
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    float a[8], b[8];
    raw[i].get(a);
    raw[i + 1].get(b);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t two = f8x2<E5M2>(f8_unit<CHECK>(a[j], inv[j]), f8_unit<CHECK>(b[j], inv[j]));
      uint32_t& w = i < 4 ? q[j].x : q[j].y;
      w = (i & 2) ? w | (two << 16) : two;
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j)
    *reinterpret_cast<uint2*>(&sm.turned[(tc * 8 + j) * 128 + ((tr ^ tc) << 3)]) = q[j];
}

template <typename Source, bool E5M2>
__global__ void __launch_bounds__(kThreads, Source::CTAS)
    quantize_tile_kernel(const Source src, int64_t rows, int64_t cols, const F8Out out, const F8Out out_t, bool pow2) {
  __shared__ __align__(16) TileSmem sm;
  const int tr = threadIdx.x >> 4, tc = threadIdx.x & 15, warp = threadIdx.x >> 5;
  TileAt t;
  const int64_t tiles_c = (cols + kF8Block - 1) / kF8Block;
  t.rows = rows;
  t.cols = cols;
  t.tile_r = blockIdx.x / tiles_c;
  t.tile_c = blockIdx.x - t.tile_r * tiles_c;
  t.r0 = t.tile_r * kF8Block + tr * 8;
  t.c0 = t.tile_c * kF8Block + tc * 8;
  t.m = left8(rows, t.r0);
  t.n = left8(cols, t.c0);
  typename Source::Raw raw[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) src.load(i < t.m ? t.r0 + i : 0, t.n > 0 ? t.c0 : 0, i < t.m ? t.n : 0, raw[i]);

  float rm[8], cm[8];
  patch_maxima<Source>(raw, rm, cm);
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 8; ++i) bad = bad || !(rm[i] < kInf);
  const bool check = __syncthreads_or(bad);
  if (check) {
#pragma unroll
    for (int j = 0; j < 8; ++j) cm[j] = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float v[8];
      raw[i].get(v);
      rm[i] = amax8_finite(v);
#pragma unroll
      for (int j = 0; j < 8; ++j) cm[j] = fmaxf(cm[j], finite_abs(v[j]));
    }
  }
  {
    float c[4];  // of the warp's 16 rows: its lower lanes columns 0 .. 3 of their 8, its upper lanes 4 .. 7
    const bool up = threadIdx.x & 16;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      c[j] = fmaxf(up ? cm[j + 4] : cm[j], __shfl_xor_sync(0xFFFFFFFFu, up ? cm[j] : cm[j + 4], 16));
    *reinterpret_cast<float4*>(&sm.col_max[warp][tc * 8 + (up ? 4 : 0)]) = make_float4(c[0], c[1], c[2], c[3]);
  }
  const float row_max = out.q || out_t.tiles ? lanes_max<8>(rm) : 0.f;  // lane l of 16: row l & 7
  float tile_max = 0.f;
  if (out.tiles || out_t.tiles) {
    float m = row_max;
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
    if ((threadIdx.x & 31) == 0) sm.warp_max[warp] = m;
  }
  __syncthreads();
  if (out.tiles || out_t.tiles) {
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) tile_max = fmaxf(tile_max, sm.warp_max[w]);
  }
  if (out_t.q && threadIdx.x < 128) {
    float m = 0.f;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) m = fmaxf(m, sm.col_max[w][threadIdx.x]);
    const F8Scale s = f8_scale<E5M2>(out_t.tiles ? tile_max : m, pow2);
    sm.col_inv[threadIdx.x] = s.inv;
    const int64_t c = t.tile_c * kF8Block + threadIdx.x;
    if (!out_t.tiles) {
      if (c < cols) out_t.s[c * out_t.lds + t.tile_r] = s.s;
    } else if (threadIdx.x == 0) {
      out_t.s[t.tile_c * out_t.lds + t.tile_r] = s.s;
    }
  }
  // most tiles are whole and hold no infinity: their stores need no conditions
  const bool full = (t.tile_r + 1) * kF8Block <= rows && (t.tile_c + 1) * kF8Block <= cols;
  if (out.q) {
    if (check || !full)
      write_rows<typename Source::Raw, E5M2, true>(raw, row_max, out, t, tile_max, pow2);
    else
      write_rows<typename Source::Raw, E5M2, false>(raw, row_max, out, t, tile_max, pow2);
  }
  if (out_t.q) {
    __syncthreads();
    if (check)
      turn_columns<typename Source::Raw, E5M2, true>(raw, sm);
    else
      turn_columns<typename Source::Raw, E5M2, false>(raw, sm);
    __syncthreads();
    // 8 lanes write one 128-byte row of the transposed matrix
    const int64_t left = cols - t.tile_c * kF8Block;
    uint8_t* to = out_t.q + t.tile_c * kF8Block * out_t.ld;
    if (full)
      write_turned<kThreads, true>(sm.turned, to, out_t.ld, t.tile_r * kF8Block, rows, kF8Block);
    else
      write_turned<kThreads, false>(sm.turned, to, out_t.ld, t.tile_r * kF8Block, rows,
                                    left < kF8Block ? (int)left : kF8Block);
  }
}

template <typename Source, bool E5M2>
cudaError_t run_as(const Source& src, int64_t rows, int64_t cols, const F8Out& out, const F8Out& out_t, bool pow2,
                   cudaStream_t st) {
  const int64_t nb = (cols + kF8Block - 1) / kF8Block;
  if (out_t.q == nullptr && !out.tiles) {
    const int64_t want = ((rows + R - 1) / R * nb + kThreads / 16 - 1) / (kThreads / 16);
    // 16-bit values are walked by the CTAs that fit at once (18.8 us at 8192 x 4096, 20.8 with one unit per CTA); of
    // float32, twice the bytes, more CTAs in turn keep more in flight (26.4 us, 27.1 walked)
    const int64_t cap = (int64_t)(sm_count() > 0 ? sm_count() : 1) * (Source::PACKED ? 4 : 32);
    quantize_rows_kernel<Source, E5M2>
        <<<(unsigned)(want < cap ? want : cap), kThreads, 0, st>>>(src, rows, cols, out, pow2);
  } else {
    const int64_t tiles = (rows + kF8Block - 1) / kF8Block * nb;
    quantize_tile_kernel<Source, E5M2><<<(unsigned)tiles, kThreads, 0, st>>>(src, rows, cols, out, out_t, pow2);
  }
  return cudaGetLastError();
}

template <typename Source>
cudaError_t run(const Source& src, int64_t rows, int64_t cols, const F8Out& out, const F8Out& out_t, bool e5m2,
                bool pow2, cudaStream_t st) {
  return e5m2 ? run_as<Source, true>(src, rows, cols, out, out_t, pow2, st)
              : run_as<Source, false>(src, rows, cols, out, out_t, pow2, st);
}

template <typename T>
cudaError_t run_float(const void* x, int64_t rows, int64_t cols, int64_t ldx, const F8Out& out, const F8Out& out_t,
                      bool e5m2, bool pow2, cudaStream_t st) {
  const bool vec = (reinterpret_cast<uintptr_t>(x) & 15) == 0 && ldx * sizeof(T) % 16 == 0;
  return run(SourceFloat<T>{static_cast<const T*>(x), ldx, vec}, rows, cols, out, out_t, e5m2, pow2, st);
}

template <bool E5M2>
cudaError_t run_f8(const ds_f8_matrix* in, const F8Out& out, const F8Out& out_t, bool e5m2, bool pow2,
                   cudaStream_t st) {
  return run(SourceF8<E5M2>{static_cast<const uint8_t*>(in->q), in->scale, in->ld, in->ld_scale,
                            in->blocks == DS_F8_TILES},
             in->rows, in->cols, out, out_t, e5m2, pow2, st);
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
    const uint32_t q = f8x2<false>(v[0], v[1]) | (f8x2<false>(v[2], v[3]) << 16);
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
                               const F8Out& out_t, bool e5m2, bool pow2, cudaStream_t st) {
  if (type == DS_TYPE_F32) return run_float<float>(x, rows, cols, ldx, out, out_t, e5m2, pow2, st);
  if (type == DS_TYPE_BF16) return run_float<__nv_bfloat16>(x, rows, cols, ldx, out, out_t, e5m2, pow2, st);
  return run_float<__half>(x, rows, cols, ldx, out, out_t, e5m2, pow2, st);
}

cudaError_t launch_requantize_f8(const ds_f8_matrix* in, const F8Out& out, const F8Out& out_t, bool e5m2, bool pow2,
                                 cudaStream_t st) {
  return in->format == DS_F8_E5M2 ? run_f8<true>(in, out, out_t, e5m2, pow2, st)
                                  : run_f8<false>(in, out, out_t, e5m2, pow2, st);
}

cudaError_t launch_expand_f8(const uint8_t* blob, int64_t n_out, int64_t k_red, const F8Out& out, cudaStream_t st) {
  const int64_t want = (n_out * ((k_red + 3) / 4) + kThreads - 1) / kThreads;
  const int64_t cap = (int64_t)(sm_count() > 0 ? sm_count() : 1) * 32;
  expand_f8_kernel<<<(unsigned)(want < cap ? want : cap), kThreads, 0, st>>>(blob, n_out, k_red, out);
  return cudaGetLastError();
}

}  // namespace ds
