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
// backward pass holds a 128 x 128 tile per CTA, 4 rows x 8 columns of it per
// thread, and writes its five 8-bit outputs from registers, so the checkpoint
// and da are read once.
#include "f8_common.cuh"

namespace ds {
namespace {

constexpr int kThreads = 256;
constexpr int kTileThreads = 512;
constexpr int kTileWarps = kTileThreads / 32;

__device__ __forceinline__ int left8(int64_t cols, int64_t c) {
  const int64_t n = cols - c;
  return n >= 8 ? 8 : (n < 0 ? 0 : (int)n);
}

// sig(g) = 1 / (1 + exp(-g)): exp(-g) overflows to inf below -88.7 and the quotient is then 0, as it should be.
__device__ __forceinline__ float sigmoid(float g) { return __fdividef(1.f, 1.f + __expf(-g)); }

template <typename T>
__global__ void __launch_bounds__(kThreads) gated_f8_kernel(const T* gu, int64_t ld, bool vec, int64_t rows,
                                                            int64_t features, const F8Out out, const F8Out ckpt,
                                                            bool pow2) {
  const int64_t nb = (features + kF8Block - 1) / kF8Block;
  const int64_t up = nb * kF8Block;
  const int64_t total = rows * nb;
  const int sub = threadIdx.x & 15;
  const int64_t first = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> 4;
  const int64_t step = (int64_t)gridDim.x * (kThreads / 16);
  for (int64_t base = first & ~(int64_t)1; base < total; base += step) {
    const int64_t i = base + (first & 1);
    const bool in = i < total;
    const int64_t r = in ? i / nb : 0, b = in ? i - r * nb : 0;
    const int64_t c = b * kF8Block + sub * 8;
    const int n = in ? left8(features, c) : 0;
    const int64_t cc = n > 0 ? c : 0;
    Raw8<T> rg, ru;
    rg.load(gu + r * ld + cc, n, vec);
    ru.load(gu + r * ld + up + cc, n, vec);
    float g[8], u[8], a[8];
    rg.get(g);
    ru.get(u);
#pragma unroll
    for (int j = 0; j < 8; ++j) a[j] = g[j] * sigmoid(g[j]) * u[j];
    const F8Scale sa = f8_scale(max16(amax8(a)), out.e5m2, pow2);
    if (n > 0) store_q8(out.q + r * out.ld + c, n, f8x8(a, sa.inv, out.e5m2));
    if (in && sub == 0) out.s[r * out.lds + b] = sa.s;
    if (ckpt.q) {
      const F8Scale sg = f8_scale(max16(amax8(g)), ckpt.e5m2, pow2);
      const F8Scale su = f8_scale(max16(amax8(u)), ckpt.e5m2, pow2);
      if (in) {
        uint8_t* q = ckpt.q + r * ckpt.ld + c;
        const int pad = left8(up, c);  // the columns between the halves are zeros (0 / s)
        store_q8(q, pad, f8x8(g, sg.inv, ckpt.e5m2));
        if (n > 0) store_q8(q + up, n, f8x8(u, su.inv, ckpt.e5m2));
        if (sub == 0) {
          ckpt.s[r * ckpt.lds + b] = sg.s;
          ckpt.s[r * ckpt.lds + nb + b] = su.s;
        }
      }
    }
  }
}

struct TileSmem {
  uint8_t turned[128 * 128];
  float col_max[kTileWarps][128];
  float col_inv[128];
};

// One 128 x 128 tile of a result: its rows to `rows_out` at column c0, its columns to `cols_out` at row c0.  v is the
// thread's 4 x 8 patch (zero beyond the matrix), m rows and n columns of it exist, n_rows columns of the row form are
// written (the zeros between the halves are part of it).
__device__ __forceinline__ void write_tile(TileSmem& sm, const float v[4][8], const F8Out& rows_out,
                                           const F8Out& cols_out, int64_t rows, int64_t r0, int64_t tile_r,
                                           int64_t c0, int64_t c_tile, int m, int n_rows, int n_cols, bool pow2) {
  const int tr = threadIdx.x >> 4, tc = threadIdx.x & 15, warp = threadIdx.x >> 5;
  if (rows_out.q) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const F8Scale s = f8_scale(max16(amax8(v[i])), rows_out.e5m2, pow2);
      if (i < m) {
        if (n_rows > 0) store_q8(rows_out.q + (r0 + i) * rows_out.ld + c0, n_rows, f8x8(v[i], s.inv, rows_out.e5m2));
        if (tc == 0) rows_out.s[(r0 + i) * rows_out.lds + c_tile / kF8Block] = s.s;
      }
    }
  }
  if (cols_out.q) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float m4 = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) m4 = fmaxf(m4, finite_abs(v[i][j]));
      m4 = fmaxf(m4, __shfl_xor_sync(0xFFFFFFFFu, m4, 16));
      if ((threadIdx.x & 16) == 0) sm.col_max[warp][tc * 8 + j] = m4;
    }
    __syncthreads();
    if (threadIdx.x < 128) {
      float mx = 0.f;
#pragma unroll
      for (int w = 0; w < kTileWarps; ++w) mx = fmaxf(mx, sm.col_max[w][threadIdx.x]);
      const F8Scale s = f8_scale(mx, cols_out.e5m2, pow2);
      sm.col_inv[threadIdx.x] = s.inv;
      if ((int64_t)threadIdx.x < n_cols) cols_out.s[(c_tile + threadIdx.x) * cols_out.lds + tile_r] = s.s;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float inv = sm.col_inv[tc * 8 + j];
      const uint32_t q = f8x2(f8_unit(v[0][j], inv), f8_unit(v[1][j], inv), cols_out.e5m2) |
                         (f8x2(f8_unit(v[2][j], inv), f8_unit(v[3][j], inv), cols_out.e5m2) << 16);
      *reinterpret_cast<uint32_t*>(&sm.turned[(tc * 8 + j) * 128 + (((tr >> 1) ^ tc) << 3) + ((tr & 1) << 2)]) = q;
    }
    __syncthreads();
    const int64_t rr = tile_r * kF8Block + tc * 8;
    const int nr = left8(rows, rr);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int col = tr + 32 * k;
      if (col < n_cols && nr > 0)
        store_q8(cols_out.q + (c_tile + col) * cols_out.ld + rr, nr,
                 *reinterpret_cast<const uint2*>(&sm.turned[col * 128 + ((tc ^ (col >> 3)) << 3)]));
    }
    __syncthreads();  // the next tile writes col_max and turned again
  }
}

struct GatedIn {
  const uint8_t* q;
  const float* s;
  int64_t ld, lds;
  bool e5m2;
};

__device__ __forceinline__ uint2 load_q8(const uint8_t* p, int n) {
  if (n >= 8) return *reinterpret_cast<const uint2*>(p);
  uint2 u = make_uint2(0u, 0u);
  for (int i = 0; i < n; ++i) {
    const uint32_t b = p[i];
    if (i < 4)
      u.x |= b << (8 * i);
    else
      u.y |= b << (8 * (i - 4));
  }
  return u;
}

template <typename T>
__global__ void __launch_bounds__(kTileThreads) gated_f8_backward_kernel(const GatedIn in, const T* da, int64_t ld,
                                                                         bool vec, int64_t rows, int64_t features,
                                                                         const F8Out dgu, const F8Out dgu_t,
                                                                         const F8Out a_t, bool pow2) {
  __shared__ __align__(16) TileSmem sm;
  const int tr = threadIdx.x >> 4, tc = threadIdx.x & 15;
  const int64_t nb = (features + kF8Block - 1) / kF8Block, up = nb * kF8Block;
  const int64_t tile_r = blockIdx.x / nb, tile_c = blockIdx.x - tile_r * nb;
  const int64_t r0 = tile_r * kF8Block + tr * 4, c_tile = tile_c * kF8Block, c0 = c_tile + tc * 8;
  const int n = left8(features, c0);
  const int m = rows - r0 >= 4 ? 4 : (rows - r0 < 0 ? 0 : (int)(rows - r0));
  const int64_t cc = n > 0 ? c0 : 0;

  float dg[4][8], du[4][8], a[4][8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t r = i < m ? r0 + i : 0;
    const int ni = i < m ? n : 0;
    Raw8<T> rd;
    rd.load(da + r * ld + cc, ni, vec);
    const uint2 qg = load_q8(in.q + r * in.ld + cc, ni), qu = load_q8(in.q + r * in.ld + up + cc, ni);
    const float sg = ni > 0 ? in.s[r * in.lds + tile_c] : 0.f, su = ni > 0 ? in.s[r * in.lds + nb + tile_c] : 0.f;
    float d[8], g[8], u[8];
    rd.get(d);
    f8x8_value(qg, in.e5m2, g);
    f8x8_value(qu, in.e5m2, u);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float gj = g[j] * sg, uj = u[j] * su;
      const float sig = sigmoid(gj), act = gj * sig;
      a[i][j] = act * uj;
      du[i][j] = d[j] * act;
      dg[i][j] = d[j] * uj * (sig * (1.f + gj * (1.f - sig)));
    }
  }
  const int cols = features - c_tile >= kF8Block ? kF8Block : (int)(features - c_tile);
  // the gate half's rows go on to the up half with zeros, and so do its columns in the transposed matrix
  write_tile(sm, dg, dgu, dgu_t, rows, r0, tile_r, c0, c_tile, m, 8, kF8Block, pow2);
  write_tile(sm, du, dgu, dgu_t, rows, r0, tile_r, up + c0, up + c_tile, m, n, cols, pow2);
  write_tile(sm, a, F8Out{}, a_t, rows, r0, tile_r, c0, c_tile, m, 0, cols, pow2);
}

template <typename T>
cudaError_t forward(const void* gu, int64_t ld, int64_t rows, int64_t features, const F8Out& out, const F8Out& ckpt,
                    bool pow2, cudaStream_t st) {
  const int64_t nb = (features + kF8Block - 1) / kF8Block;
  const int64_t want = (rows * nb + kThreads / 16 - 1) / (kThreads / 16);
  const int64_t cap = (int64_t)(sm_count() > 0 ? sm_count() : 1) * 32;
  const bool vec = (reinterpret_cast<uintptr_t>(gu) & 15) == 0 && ld * sizeof(T) % 16 == 0;
  gated_f8_kernel<T><<<(unsigned)(want < cap ? want : cap), kThreads, 0, st>>>(static_cast<const T*>(gu), ld, vec,
                                                                               rows, features, out, ckpt, pow2);
  return cudaGetLastError();
}

template <typename T>
cudaError_t backward(const ds_f8_matrix* ckpt, const void* da, int64_t ld, int64_t features, const F8Out& dgu,
                     const F8Out& dgu_t, const F8Out& a_t, bool pow2, cudaStream_t st) {
  const GatedIn in{static_cast<const uint8_t*>(ckpt->q), ckpt->scale, ckpt->ld, ckpt->ld_scale,
                   ckpt->format == DS_F8_E5M2};
  const int64_t tiles = (ckpt->rows + kF8Block - 1) / kF8Block * ((features + kF8Block - 1) / kF8Block);
  const bool vec = (reinterpret_cast<uintptr_t>(da) & 15) == 0 && ld * sizeof(T) % 16 == 0;
  gated_f8_backward_kernel<T><<<(unsigned)tiles, kTileThreads, 0, st>>>(in, static_cast<const T*>(da), ld, vec,
                                                                        ckpt->rows, features, dgu, dgu_t, a_t, pow2);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_gated_f8(const void* gu, int type, int64_t ld, int64_t rows, int64_t features, const F8Out& out,
                            const F8Out& ckpt, bool pow2, cudaStream_t st) {
  if (type == DS_TYPE_F32) return forward<float>(gu, ld, rows, features, out, ckpt, pow2, st);
  if (type == DS_TYPE_BF16) return forward<__nv_bfloat16>(gu, ld, rows, features, out, ckpt, pow2, st);
  return forward<__half>(gu, ld, rows, features, out, ckpt, pow2, st);
}

cudaError_t launch_gated_f8_backward(const ds_f8_matrix* ckpt, const void* da, int type, int64_t ld, int64_t features,
                                     const F8Out& dgu, const F8Out& dgu_t, const F8Out& a_t, bool pow2,
                                     cudaStream_t st) {
  if (type == DS_TYPE_F32) return backward<float>(ckpt, da, ld, features, dgu, dgu_t, a_t, pow2, st);
  if (type == DS_TYPE_BF16) return backward<__nv_bfloat16>(ckpt, da, ld, features, dgu, dgu_t, a_t, pow2, st);
  return backward<__half>(ckpt, da, ld, features, dgu, dgu_t, a_t, pow2, st);
}

}  // namespace ds
