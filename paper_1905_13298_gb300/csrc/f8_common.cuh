// Shared device code of the 8-bit floating-point operators: loads of eight
// consecutive values of any supported type, the block scale and the rounding
// to 8 bits.
//
// A block of 128 values (one row, or 128 x 128 for a tile) is held as
//     q = round8(v * min(MAX / amax, 2^126)),   s = max(amax / MAX, 2^-126),
// amax its largest finite magnitude and MAX the format's largest value (448
// for e4m3, 57344 for e5m2); with DS_F8_POW2 s is rounded up to a power of
// two and q = round8(v / s), so that a later change of blocks rounds nothing
// but values that leave the format's range.  A
// non-finite value becomes the 8-bit NaN, and does not enter the scale.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "ds_common.cuh"

namespace ds {

constexpr int kF8Block = 128;

template <int TYPE>
struct TypeOf;
template <>
struct TypeOf<DS_TYPE_F32> {
  using T = float;
};
template <>
struct TypeOf<DS_TYPE_BF16> {
  using T = __nv_bfloat16;
};
template <>
struct TypeOf<DS_TYPE_F16> {
  using T = __half;
};

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ void from_float(float v, float& o) { o = v; }
__device__ __forceinline__ void from_float(float v, __nv_bfloat16& o) { o = __float2bfloat16_rn(v); }
__device__ __forceinline__ void from_float(float v, __half& o) { o = __float2half_rn(v); }

__device__ __forceinline__ void unpack2(uint32_t u, float& a, float& b, const __nv_bfloat16*) {
  a = __uint_as_float(u << 16);
  b = __uint_as_float(u & 0xFFFF0000u);
}
__device__ __forceinline__ void unpack2(uint32_t u, float& a, float& b, const __half*) {
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u));
  a = f.x;
  b = f.y;
}
__device__ __forceinline__ uint32_t pack2(float a, float b, const __nv_bfloat16*) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t pack2(float a, float b, const __half*) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// Pairs of float32 in one 64-bit register: two multiplications per instruction.
__device__ __forceinline__ uint64_t pair(uint32_t lo, uint32_t hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(lo), "r"(hi));
  return r;
}
__device__ __forceinline__ uint64_t pair(float lo, float hi) { return pair(__float_as_uint(lo), __float_as_uint(hi)); }
__device__ __forceinline__ void unpair(uint64_t v, float& lo, float& hi) {
  lo = __uint_as_float((uint32_t)v);
  hi = __uint_as_float((uint32_t)(v >> 32));
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

// Eight 16-bit values at any address: by the widest accesses that it allows.  Rows an odd number of values apart start
// anywhere; the branches go the same way for a whole row.
__device__ __forceinline__ uint4 load16(const void* p) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p);
  if (a % 8 == 0) {
    const uint2 *w = static_cast<const uint2*>(p), lo = w[0], hi = w[1];
    return make_uint4(lo.x, lo.y, hi.x, hi.y);
  }
  if (a % 4 == 0) {
    const uint32_t* w = static_cast<const uint32_t*>(p);
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  const uint16_t* h = static_cast<const uint16_t*>(p);
  const uint32_t* w = reinterpret_cast<const uint32_t*>(h + 1);
  const uint32_t a0 = h[0], a1 = w[0], a2 = w[1], a3 = w[2], a4 = h[7];
  return make_uint4(a0 | a1 << 16, a1 >> 16 | a2 << 16, a2 >> 16 | a3 << 16, a3 >> 16 | a4 << 16);
}
__device__ __forceinline__ void store16(void* p, uint4 u) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p);
  if (a % 8 == 0) {
    uint2* w = static_cast<uint2*>(p);
    w[0] = make_uint2(u.x, u.y), w[1] = make_uint2(u.z, u.w);
  } else if (a % 4 == 0) {
    uint32_t* w = static_cast<uint32_t*>(p);
    w[0] = u.x, w[1] = u.y, w[2] = u.z, w[3] = u.w;
  } else {
    uint16_t* h = static_cast<uint16_t*>(p);
    uint32_t* w = reinterpret_cast<uint32_t*>(h + 1);
    h[0] = (uint16_t)u.x, w[0] = u.x >> 16 | u.y << 16, w[1] = u.y >> 16 | u.z << 16;
    w[2] = u.z >> 16 | u.w << 16, h[7] = (uint16_t)(u.w >> 16);
  }
}

// Eight consecutive values as they lie in memory; `vec` says that p is 16-byte aligned.  The `n` first exist, the
// others read as zero.  ODD: eight 16-bit values that are not aligned are loaded by load16; otherwise one by one, which
// is less code.
template <typename T>
struct Raw8 {
  static constexpr bool PAIRS = true;
  uint4 u;
  template <bool ODD = false>
  __device__ __forceinline__ void load(const T* p, int n, bool vec) {
    if (vec && n >= 8) {
      u = *reinterpret_cast<const uint4*>(p);
    } else if (ODD && n >= 8) {
      u = load16(p);
    } else {
      const uint16_t* s = reinterpret_cast<const uint16_t*>(p);
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        w[i] = (2 * i < n ? s[2 * i] : 0u) | ((2 * i + 1 < n ? (uint32_t)s[2 * i + 1] : 0u) << 16);
      u = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
  __device__ __forceinline__ void get(float v[8]) const {
    unpack2(u.x, v[0], v[1], (const T*)nullptr);
    unpack2(u.y, v[2], v[3], (const T*)nullptr);
    unpack2(u.z, v[4], v[5], (const T*)nullptr);
    unpack2(u.w, v[6], v[7], (const T*)nullptr);
  }
};
template <>
struct Raw8<float> {
  static constexpr bool PAIRS = true;
  float4 a, b;
  template <bool ODD = false>
  __device__ __forceinline__ void load(const float* p, int n, bool vec) {
    if (vec && n >= 8) {
      a = reinterpret_cast<const float4*>(p)[0];
      b = reinterpret_cast<const float4*>(p)[1];
    } else {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : 0.f;
      a = make_float4(v[0], v[1], v[2], v[3]);
      b = make_float4(v[4], v[5], v[6], v[7]);
    }
  }
  __device__ __forceinline__ void get(float v[8]) const {
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
    v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  }
};

template <bool ODD, typename T>
__device__ __forceinline__ void store8(T* p, int n, bool vec, const float v[8]) {
  if ((vec || ODD) && n >= 8) {
    const uint4 u = make_uint4(pack2(v[0], v[1], (const T*)nullptr), pack2(v[2], v[3], (const T*)nullptr),
                               pack2(v[4], v[5], (const T*)nullptr), pack2(v[6], v[7], (const T*)nullptr));
    if (vec)
      *reinterpret_cast<uint4*>(p) = u;
    else
      store16(p, u);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) from_float(v[i], p[i]);
  }
}
template <bool ODD>
__device__ __forceinline__ void store8(float* p, int n, bool vec, const float v[8]) {
  if (vec && n >= 8) {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = v[i];
  }
}

// ---------------------------------------------------------------------------
// 8-bit formats
// ---------------------------------------------------------------------------
// The format is a template argument throughout: as a value it would cost both conversions and a selection.
template <bool E5M2>
__device__ __forceinline__ uint32_t f8x2(float lo, float hi) {
  uint16_t r;
  if (E5M2)
    asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  else
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
template <bool E5M2>
__device__ __forceinline__ float2 f8x2_value(uint16_t q) {
  uint32_t h;
  if (E5M2)
    asm("cvt.rn.f16x2.e5m2x2 %0, %1;" : "=r"(h) : "h"(q));
  else
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(q));
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}
template <bool E5M2>
__device__ __forceinline__ void f8x8_value(uint2 q, float v[8]) {
  const uint32_t w[2] = {q.x, q.y};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float2 a = f8x2_value<E5M2>((uint16_t)(w[i] & 0xFFFFu));
    const float2 b = f8x2_value<E5M2>((uint16_t)(w[i] >> 16));
    v[4 * i] = a.x, v[4 * i + 1] = a.y, v[4 * i + 2] = b.x, v[4 * i + 3] = b.y;
  }
}

struct F8Scale {
  float s, inv;
};
template <bool E5M2>
__device__ __forceinline__ F8Scale f8_scale(float amax, bool pow2) {
  constexpr float kMax = E5M2 ? 57344.f : 448.f;
  // amax / kMax, correctly rounded, by a multiplication and the correction of its remainder (the division by a constant
  // of P. Markstein, IBM J. Res. Dev. 34 (1), 1990; exact remainders down to quotients of 2^-126, below which s is set)
  constexpr float kPart = 1.f / kMax;
  const float near = amax * kPart;
  float s = fmaxf(fmaf(fmaf(-near, kMax, amax), kPart, near), 1.17549435e-38f);
  if (pow2) {
    s = __uint_as_float((__float_as_uint(s) + 0x7FFFFFu) & 0xFF800000u);
    return F8Scale{s, __frcp_rn(s)};
  }
  // kMax / amax (not 1 / s: one rounding instead of two) from an approximate reciprocal and the quotient's remainder.
  // Quarters, so that the reciprocal of none is subnormal.  One correction gives the correctly rounded quotient for every
  // amax, or what fminf leaves out (compared with __fdiv_rn over all 2^23 mantissas of 255 exponents; the tests sample).
  const float a = 0.25f * amax;
  float near_inv;
  asm("rcp.approx.f32 %0, %1;" : "=f"(near_inv) : "f"(a));
  const float quot = 0.25f * kMax * near_inv;
  return F8Scale{s, fminf(fmaf(fmaf(-quot, a, 0.25f * kMax), near_inv, quot), 8.50705917e37f)};
}
// Values in units of the scale.  CHECK: the values may hold infinities, which have to become NaN and not the largest
// value (v * 0 is NaN for them and 0 otherwise); NaN stays NaN by itself.
template <bool CHECK>
__device__ __forceinline__ float f8_unit(float v, float inv) {
  return CHECK ? fmaf(v, 0.f, v * inv) : v * inv;
}
template <bool E5M2, bool CHECK>
__device__ __forceinline__ uint32_t f8x4(float a, float b, float c, float d, float inv) {
  return f8x2<E5M2>(f8_unit<CHECK>(a, inv), f8_unit<CHECK>(b, inv)) |
         (f8x2<E5M2>(f8_unit<CHECK>(c, inv), f8_unit<CHECK>(d, inv)) << 16);
}
// Two rows' 8-bit values of eight columns with a factor each, by columns: the low half of two[j] is column j.
template <bool E5M2, bool CHECK>
__device__ __forceinline__ void f8_columns(const float a[8], const float b[8], const float inv[8], uint32_t two[8]) {
#pragma unroll
  for (int j = 0; j < 8; j += 2) {
    if constexpr (CHECK) {
#pragma unroll
      for (int k = j; k < j + 2; ++k) two[k] = f8x2<E5M2>(f8_unit<true>(a[k], inv[k]), f8_unit<true>(b[k], inv[k]));
    } else {
      const uint64_t f = pair(inv[j], inv[j + 1]);
      float a0, a1, b0, b1;
      unpair(mul2(pair(a[j], a[j + 1]), f), a0, a1);
      unpair(mul2(pair(b[j], b[j + 1]), f), b0, b1);
      two[j] = f8x2<E5M2>(a0, b0);
      two[j + 1] = f8x2<E5M2>(a1, b1);
    }
  }
}
// PAIRS: two multiplications per instruction, for which values lie in pairs of registers.
template <bool E5M2, bool CHECK, bool PAIRS = true>
__device__ __forceinline__ uint2 f8x8(const float v[8], float inv) {
  if constexpr (!CHECK && PAIRS) {
    uint32_t q[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float lo, hi;
      unpair(mul2(pair(v[2 * j], v[2 * j + 1]), pair(inv, inv)), lo, hi);
      q[j] = f8x2<E5M2>(lo, hi);
    }
    return make_uint2(q[0] | q[1] << 16, q[2] | q[3] << 16);
  }
  return make_uint2(f8x4<E5M2, CHECK>(v[0], v[1], v[2], v[3], inv), f8x4<E5M2, CHECK>(v[4], v[5], v[6], v[7], inv));
}
// The address is 8-byte aligned: rows start 16 bytes apart or a multiple of it.
__device__ __forceinline__ void store_q8(uint8_t* p, int n, uint2 q) {
  if (n >= 8) {
    *reinterpret_cast<uint2*>(p) = q;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = (uint8_t)((i < 4 ? q.x >> (8 * i) : q.y >> (8 * (i - 4))) & 0xFFu);
  }
}

// Eight 8-bit values of which n exist (the others read as zero); 8-byte aligned.
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

constexpr float kInf = __builtin_huge_valf();

__device__ __forceinline__ float finite_abs(float v) {
  const float a = fabsf(v);
  return a < kInf ? a : 0.f;  // false for NaN as well
}
// The largest magnitude; NaN is passed over (fmaxf), an infinity is the result.
__device__ __forceinline__ float amax8(const float v[8]) {
  float m = fabsf(v[0]);
#pragma unroll
  for (int i = 1; i < 8; ++i) m = fmaxf(m, fabsf(v[i]));
  return fmaxf(m, 0.f);
}
__device__ __forceinline__ float amax8_finite(const float v[8]) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, finite_abs(v[i]));
  return m;
}
// The largest over the 16 lanes that hold one block of 128 columns.
__device__ __forceinline__ float max16(float m) {
#pragma unroll
  for (int d = 8; d >= 1; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
  return m;
}
// R maxima over the same 16 lanes at once: lane l gets that of value l & (R - 1).  Each exchange halves the values that
// a lane answers for (8 shuffles for 8 values instead of 32), and a lane then makes one scale, not R.
template <int R>
__device__ __forceinline__ float lanes_max(const float (&m)[R]) {
  float a[R];
#pragma unroll
  for (int i = 0; i < R; ++i) a[i] = m[i];
#pragma unroll
  for (int h = R / 2; h >= 1; h >>= 1) {
    const bool up = threadIdx.x & h;
#pragma unroll
    for (int i = 0; i < h; ++i)
      a[i] = fmaxf(up ? a[i + h] : a[i], __shfl_xor_sync(0xFFFFFFFFu, up ? a[i] : a[i + h], h));
  }
  float v = a[0];
#pragma unroll
  for (int d = R; d < 16; d <<= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, d));
  return v;
}
__device__ __forceinline__ float of_lane(float v, int l) { return __shfl_sync(0xFFFFFFFFu, v, l, 16); }

// The scale and the 8-bit values of a block that 16 lanes hold; all 32 lanes of the warp call it.  Infinities are
// rare: they are looked for by the largest magnitude, and the block is then gone over again.
template <bool E5M2>
__device__ __forceinline__ F8Scale f8_block(const float v[8], bool pow2, uint2& q) {
  float m = max16(amax8(v));
  const bool inf = __any_sync(0xFFFFFFFFu, !(m < kInf));
  if (inf) m = max16(amax8_finite(v));
  const F8Scale s = f8_scale<E5M2>(m, pow2);
  q = inf ? f8x8<E5M2, true>(v, s.inv) : f8x8<E5M2, false>(v, s.inv);
  return s;
}

// Steps of a half-warp through the (row, block) units of a matrix in row order, without a division per step.
struct Units {
  int64_t r;
  int64_t b, nb, step_r, step_b;
  __device__ __forceinline__ Units(int64_t first, int64_t step, int64_t blocks) : nb(blocks) {
    r = first / blocks;
    b = first - r * blocks;
    step_r = step / blocks;
    step_b = step - step_r * blocks;
  }
  __device__ __forceinline__ void next() {
    r += step_r;
    b += step_b;
    if (b >= nb) {
      b -= nb;
      ++r;
    }
  }
};

// 16 bytes of a turned tile: two 8-byte chunks of column `col` from chunk 2 k on (the chunks of a column are XORed with
// the number of its group of 8).
__device__ __forceinline__ uint4 turned16(const uint8_t* turned, int col, int k) {
  const int sw = (col >> 3) & 15;
  const uint4 v = *reinterpret_cast<const uint4*>(&turned[col * 128 + (((2 * k) ^ (sw & 14)) << 3)]);
  return (sw & 1) ? make_uint4(v.z, v.w, v.x, v.y) : v;
}
// ... written where they exist; the address is 16-byte aligned.
__device__ __forceinline__ void store_q16(uint8_t* p, int n, uint4 q) {
  if (n >= 16) {
    *reinterpret_cast<uint4*>(p) = q;
  } else {
    store_q8(p, n, make_uint2(q.x, q.y));
    if (n > 8) store_q8(p + 8, n - 8, make_uint2(q.z, q.w));
  }
}
// A turned tile to the transposed matrix: columns 0 .. cols - 1 from `to`, rows r0 .. of `rows`.  FULL: 128 of each.
template <int THREADS, bool FULL>
__device__ __forceinline__ void write_turned(const uint8_t* turned, uint8_t* to, int64_t ld, int64_t r0, int64_t rows,
                                             int cols) {
  const int k = threadIdx.x & 7, first = threadIdx.x >> 3;
  const int64_t left = rows - r0 - 16 * k;
  uint8_t* p = to + r0 + 16 * k + first * ld;
  if (FULL) {
#pragma unroll
    for (int i = 0; i < 1024 / THREADS; ++i, p += THREADS / 8 * ld)
      *reinterpret_cast<uint4*>(p) = turned16(turned, first + THREADS / 8 * i, k);
  } else if (left > 0) {
    const int n = left >= 16 ? 16 : (int)left;
    for (int col = first; col < cols; col += THREADS / 8, p += THREADS / 8 * ld)
      store_q16(p, n, turned16(turned, col, k));
  }
}

__device__ __forceinline__ int left8(int64_t cols, int64_t c) {
  const int64_t n = cols - c;
  return n >= 8 ? 8 : (n < 0 ? 0 : (int)n);
}

// ---------------------------------------------------------------------------
// Launch parameters
// ---------------------------------------------------------------------------
struct F8Out {  // an 8-bit matrix that a kernel writes (q == NULL: none); its format goes with the launch
  uint8_t* q;
  float* s;
  int64_t ld, lds;
  int tiles;
};
inline F8Out f8_out(const ds_f8_matrix* m) {
  if (m == nullptr) return F8Out{nullptr, nullptr, 0, 0, 0};
  return F8Out{static_cast<uint8_t*>(m->q), m->scale, m->ld, m->ld_scale, m->blocks == DS_F8_TILES};
}

struct RmsnormParams {
  const void *x, *residual;
  int64_t ldx, ldr;
  const float* weight;
  int64_t rows, cols;
  float eps;
  F8Out out;
  void* h;
  int64_t ldh;
  float* rstd;
  int e5m2, pow2;
};
struct RmsnormBackwardParams {
  const void *dy, *h, *dh;
  int64_t lddy, ldh, lddh;
  const float *rstd, *weight;
  int64_t rows, cols;
  void* dx;
  int64_t lddx;
  float *dw, *partial;
};
struct LinearF8Params {
  const ds_f8_matrix *x, *w;
  const float *bias, *add;
  int64_t ld_add;
  void* y;
  int type;
  int64_t ldy;
};

constexpr int64_t kF8NormPartials = 608;  // rows of partial weight gradients: 4 CTAs on each of 152 SMs

// e5m2: the format of every matrix that the call writes.
cudaError_t launch_quantize_f8(const void* x, int type, int64_t rows, int64_t cols, int64_t ldx, const F8Out& out,
                               const F8Out& out_t, bool e5m2, bool pow2, cudaStream_t st);
cudaError_t launch_requantize_f8(const ds_f8_matrix* in, const F8Out& out, const F8Out& out_t, bool e5m2, bool pow2,
                                 cudaStream_t st);
cudaError_t launch_expand_f8(const uint8_t* blob, int64_t n_out, int64_t k_red, const F8Out& out, cudaStream_t st);
cudaError_t launch_rmsnorm_f8(const RmsnormParams& p, int type, cudaStream_t st);
cudaError_t launch_rmsnorm_f8_backward(const RmsnormBackwardParams& p, int type, cudaStream_t st);
cudaError_t launch_gated_f8(const void* gu, int type, int64_t ld, int64_t rows, int64_t features, const F8Out& out,
                            const F8Out& ckpt, bool e5m2, bool pow2, cudaStream_t st);
cudaError_t launch_gated_f8_backward(const ds_f8_matrix* ckpt, const void* da, int type, int64_t ld, int64_t features,
                                     const F8Out& dgu, const F8Out& dgu_t, const F8Out& a_t, bool e5m2, bool pow2,
                                     cudaStream_t st);
cudaError_t launch_linear_f8(const LinearF8Params& p, cudaStream_t st);
int linear_f8_tile(const LinearF8Params& p);  // rows of the tile that the launch would take
int read_f8_fault_flag();
int read_gated_f8_fault_flag();
void set_f8_wait_cycles(long long cycles);
long long f8_wait_cycles();  // limit of a bounded wait of the next launches

}  // namespace ds
