// One step of Adam with decoupled weight decay over many tensors in one launch
// (the formulas and the 8-bit states' rounding are in the header).
//
// The work is one pass over memory: 28 bytes a value with float32 throughout
// and 16-bit gradients and copies, 16 with 8-bit states.  With float32 states
// it runs at the rate of a copy (50 M values 203 us; 216 where tensors are not
// aligned, 133 and 192 with 8-bit states).  A CTA takes 1024 consecutive values
// of one tensor, a thread eight of them, all of whose loads
// are on their way before the first is used.  The tensors' addresses are in
// the kernel's parameters: nothing is copied to the device before a step, and
// a captured step is replayed with them.
#include <math.h>

#include <algorithm>
#include <exception>
#include <type_traits>
#include <vector>

#include "f8_checks.cuh"

namespace ds {
namespace {

constexpr int kThreads = 128, kEach = 8, kSpan = kThreads * kEach;
constexpr int kFew = 50, kMany = 400;  // tensors of a launch: parameters of up to 4 KB, or up to 32 KB

struct Tensor {
  void* p;
  const void* g;
  void *m, *v;
  float *m_scale, *v_scale;
  void* copy;
  int64_t n;
  uint32_t first;   // CTA of its first values
  float decay;      // 1 - lr * weight_decay, or weight_decay where lr is on the device
  uint32_t number;  // in the call
  int8_t p_type, g_type, copy_type;
  int8_t aligned;   // all its addresses are multiples of eight values
};

struct Factors {
  float beta1, rest1, beta2, rest2, eps;
  float rate, root;       // lr / (1 - beta1^t), (1 - beta2^t)^(-1/2)
  float lr;
  double log1, log2;      // of the betas, where t is on the device
  const int64_t* step_dev;
  const float *lr_dev, *grad_scale;
  uint32_t step, seed;
};

template <int N>
struct Params {
  Factors f;
  int count;
  Tensor t[N];
};
static_assert(sizeof(Params<kFew>) <= 4096 && sizeof(Params<kMany>) <= 32764, "kernel parameters");

// A thread's eight values as they lie in memory, of a type known at run time: the same branch for a whole CTA.  They are
// taken apart only after all arrays' loads have been issued.
struct Raw {
  uint32_t r[8];
};
// Where they lie: eight in a row from `first` (STEP = 1), all of them there and their addresses multiples of the access,
// or every 16th (STEP = 16) while they exist: 16 threads then read one value each of 16 in a row, at any address.  Either
// way these threads hold 128 in a row, a block of the 8-bit states.
template <int STEP>
struct Place {
  int64_t first, end;
  __device__ __forceinline__ bool has(int k) const { return STEP == 1 || first + STEP * k < end; }
};
template <int STEP>
__device__ __forceinline__ void load_raw(Raw& o, const void* base, int type, const Place<STEP>& at) {
  if (type == DS_TYPE_F32) {
    const float* p = static_cast<const float*>(base) + at.first;
    if constexpr (STEP == 1) {
      asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                   : "=r"(o.r[0]), "=r"(o.r[1]), "=r"(o.r[2]), "=r"(o.r[3]), "=r"(o.r[4]), "=r"(o.r[5]), "=r"(o.r[6]),
                     "=r"(o.r[7])
                   : "l"(p));
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) o.r[k] = at.has(k) ? __float_as_uint(p[STEP * k]) : 0u;
    }
  } else {
    const uint16_t* p = static_cast<const uint16_t*>(base) + at.first;
    if constexpr (STEP == 1) {
      const uint4 a = *reinterpret_cast<const uint4*>(p);
      o.r[0] = a.x, o.r[1] = a.y, o.r[2] = a.z, o.r[3] = a.w;
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        o.r[k] = (at.has(2 * k) ? p[STEP * 2 * k] : 0u) |
                 (at.has(2 * k + 1) ? (uint32_t)p[STEP * (2 * k + 1)] << 16 : 0u);
    }
  }
}
__device__ __forceinline__ void get_raw(const Raw& o, int type, float v[8]) {
  if (type == DS_TYPE_F32) {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = __uint_as_float(o.r[k]);
  } else if (type == DS_TYPE_BF16) {
#pragma unroll
    for (int k = 0; k < 4; ++k) unpack2(o.r[k], v[2 * k], v[2 * k + 1], (const __nv_bfloat16*)nullptr);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) unpack2(o.r[k], v[2 * k], v[2 * k + 1], (const __half*)nullptr);
  }
}
template <int STEP, typename T>
__device__ __forceinline__ void store_values_as(T* p, const Place<STEP>& at, const float v[8]) {
  p += at.first;
  if constexpr (STEP != 1) {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (at.has(k)) from_float(v[k], p[STEP * k]);
  } else if constexpr (sizeof(T) == 4) {
    asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(v[0]), "f"(v[1]), "f"(v[2]),
                 "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7])
                 : "memory");
  } else {
    store8<false>(p, 8, true, v);
  }
}
template <int STEP>
__device__ __forceinline__ void store_values(void* base, int type, const Place<STEP>& at, const float v[8]) {
  if (type == DS_TYPE_F32)
    store_values_as(static_cast<float*>(base), at, v);
  else if (type == DS_TYPE_BF16)
    store_values_as(static_cast<__nv_bfloat16*>(base), at, v);
  else
    store_values_as(static_cast<__half*>(base), at, v);
}

// Eight 8-bit values, the missing ones zero.
template <int STEP>
__device__ __forceinline__ uint2 load_bytes(const void* base, const Place<STEP>& at) {
  const uint8_t* p = static_cast<const uint8_t*>(base) + at.first;
  if constexpr (STEP == 1) return *reinterpret_cast<const uint2*>(p);
  uint32_t w[2] = {0u, 0u};
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (at.has(k)) w[k >> 2] |= (uint32_t)p[STEP * k] << (8 * (k & 3));
  return make_uint2(w[0], w[1]);
}
template <int STEP>
__device__ __forceinline__ void store_bytes(void* base, const Place<STEP>& at, uint2 q) {
  uint8_t* p = static_cast<uint8_t*>(base) + at.first;
  if constexpr (STEP == 1) {
    *reinterpret_cast<uint2*>(p) = q;
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (at.has(k)) p[STEP * k] = (uint8_t)((k < 4 ? q.x >> (8 * k) : q.y >> (8 * (k - 4))) & 0xFFu);
  }
}

__device__ __forceinline__ uint64_t both(float v) { return pair(v, v); }
__device__ __forceinline__ float lo_of(uint64_t v) { return __uint_as_float((uint32_t)v); }
__device__ __forceinline__ float hi_of(uint64_t v) { return __uint_as_float((uint32_t)(v >> 32)); }
// A product that a sum follows.  The definition rounds it, and a packed sum would be contracted with a packed product;
// as a fused one with zero it is not (the sign of a product of zero apart, it is the same).
__device__ __forceinline__ uint64_t product(uint64_t a, uint64_t b) { return fma2(a, b, 0); }
__device__ __forceinline__ uint64_t sum(uint64_t a, uint64_t b) { return fma2(a, both(1.f), b); }
__device__ __forceinline__ uint64_t difference(uint64_t a, uint64_t b) { return fma2(b, both(-1.f), a); }
// The largest magnitude of three; NaN where one is.
__device__ __forceinline__ float max3_abs(float a, float b, float c) {
  float r;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// Square roots of two values, correctly rounded, for 0 and from 2^-149 to 2^67; NaN above that.  With an approximate
// reciprocal root y of the values u in units of 2^-60, g = u y and one correction by the root's residual u - g^2, which is
// exact (P. Markstein, IBM J. Res. Dev. 34 (1), 1990).  Equal to __fsqrt_rn: compared for all of these numbers.
__device__ __forceinline__ uint64_t root2(uint64_t v) {
  const uint64_t from = fma2(v, both(0x1p60f), both(0x1p-126f));  // changes 0 only
  float y0, y1;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y0) : "f"(lo_of(from)));
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y1) : "f"(hi_of(from)));
  // the negatives of u and g, which the residual needs
  const uint64_t y = pair(y0, y1), u = mul2(v, both(-0x1p60f)), g = mul2(u, y);
  return mul2(fma2(fma2(g, g, u), mul2(y, both(0.5f)), g), both(-0x1p-30f));
}
// Quotients a / b, correctly rounded, for b from 2^-60 to 2^60 and a up to 2^60, where they are 0 or normal and a is not
// below 2^-102 (there the last place may be off): a quotient of one step by the correctly rounded reciprocal and its
// exact remainder, by the same paper.
__device__ __forceinline__ uint64_t quotient2(uint64_t a, uint64_t b) {
  float y0, y1;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y0) : "f"(lo_of(b)));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y1) : "f"(hi_of(b)));
  const uint64_t y = pair(y0, y1), minus = mul2(b, both(-1.f));
  const uint64_t r = fma2(fma2(minus, y, both(1.f)), y, y);
  const uint64_t q = mul2(a, r);
  return fma2(fma2(minus, q, a), r, q);
}

// Values in units of the scale to one of their e4m3 neighbours, with 16 random bits in `bits` (from bit 4 on): bits + 8
// fills what three bits of a mantissa leave of 23, and carries into the upper neighbour.  For magnitudes from 2^-6 on.
__device__ __forceinline__ uint32_t to_neighbour(float u, uint32_t bits) {
  return (__float_as_uint(u) + bits + 8u) & 0xFFF00000u;
}
// The same for all magnitudes: below 2^-6 the neighbours are 2^-9 apart, as they are from 2^-6 to 2^-5, where u is moved
// for it.
template <bool SIGNED>
__device__ __forceinline__ uint64_t to_neighbours(uint64_t u, uint32_t bits0, uint32_t bits1) {
  auto offset = [](float v) {
    const float off = SIGNED ? copysignf(0x1p-6f, v) : 0x1p-6f;
    return fabsf(v) < 0x1p-6f ? off : 0.f;
  };
  const uint64_t off = pair(offset(lo_of(u)), offset(hi_of(u))), w = sum(u, off);
  return difference(pair(to_neighbour(lo_of(w), bits0), to_neighbour(hi_of(w), bits1)), off);
}

// Two values of a block (in units of its scale) to 8 bits; `random`: the hash of each but for its last step, which
// changes the low half only.  LARGE: none of the warp's magnitudes is below 2^-6, or not finite.
template <bool ROOT, bool LARGE>
__device__ __forceinline__ uint32_t two_to_f8(uint64_t u, uint32_t random0, uint32_t random1) {
  auto bits = [](uint32_t x) { return (ROOT ? x >> 12 : (x << 4) ^ (x >> 12)) & 0xFFFF0u; };
  float lo, hi;
  if (LARGE) {
    lo = __uint_as_float(to_neighbour(lo_of(u), bits(random0)));
    hi = __uint_as_float(to_neighbour(hi_of(u), bits(random1)));
  } else {
    unpair(to_neighbours<!ROOT>(u, bits(random0), bits(random1)), lo, hi);
    if (ROOT) {  // u > 0 is above 2^-136
      const uint64_t large = mul2(u, both(0x1p127f));
      lo = fmaxf(lo, fminf(lo_of(large), 0x1p-9f));
      hi = fmaxf(hi, fminf(hi_of(large), 0x1p-9f));
    }
    if (!(fabsf(lo_of(u)) < kInf)) lo = __uint_as_float(0x7FC00000u);
    if (!(fabsf(hi_of(u)) < kInf)) hi = __uint_as_float(0x7FC00000u);
  }
  return f8x2<false>(lo, hi);
}

// The largest of the bit patterns of 16 lanes' magnitudes: NaN is above infinity, and that above all numbers.
__device__ __forceinline__ float top16(float v) {
  const uint32_t lanes = threadIdx.x & 16 ? 0xFFFF0000u : 0x0000FFFFu;
  return __uint_as_float(__reduce_max_sync(lanes, __float_as_uint(v) & 0x7FFFFFFFu));
}
__device__ __forceinline__ float top8(const uint64_t v[4]) {
  float t = max3_abs(lo_of(v[0]), hi_of(v[0]), lo_of(v[1]));
  t = max3_abs(t, hi_of(v[1]), lo_of(v[2]));
  t = max3_abs(t, hi_of(v[2]), lo_of(v[3]));
  return max3_abs(t, hi_of(v[3]), 0.f);
}
// The least magnitude of eight; NaN where one is.
__device__ __forceinline__ float least8(const uint64_t v[4]) {
  float t = __uint_as_float(0x7F800000u);
#pragma unroll
  for (int k = 0; k < 4; ++k) asm("min.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(t) : "f"(t), "f"(lo_of(v[k])), "f"(hi_of(v[k])));
  return t;
}
__device__ __forceinline__ float finite_top8(const uint64_t v[4]) {
  float t = 0.f;
#pragma unroll
  for (int k = 0; k < 4; ++k) t = fmaxf(t, fmaxf(finite_abs(lo_of(v[k])), finite_abs(hi_of(v[k]))));
  return t;
}

// 1 - beta^t from the logarithm of beta, for a t that only the device knows.
__device__ __forceinline__ float rest_of_power(double log_beta, int64_t t) {
  return -expm1f((float)((double)t * log_beta));
}

// With 8-bit states arithmetic takes as long as memory, 650 instructions for eight values of 32 threads: 48 warps of an SM
// hide its latency best, although 40 registers are a few too little (9 tensors of 50 M values, 16-bit gradients and
// copies: 133 us or 6.1 TB/s; 143 with 40 warps and 48 registers, 149 with 32 warps and 64).  Copies of the next values
// through shared memory meanwhile, and factors kept as pairs in the parameters, gained nothing.
template <bool F8, int N>
__global__ void __launch_bounds__(kThreads, F8 ? 12 : 8) adamw_kernel(const __grid_constant__ Params<N> P) {
  int lo = 0, hi = P.count - 1;  // the last tensor that starts at or before this CTA
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (P.t[mid].first <= blockIdx.x)
      lo = mid;
    else
      hi = mid - 1;
  }
  const Tensor& T = P.t[lo];
  const int64_t base = (int64_t)(blockIdx.x - T.first) * kSpan;
  // the same for a whole CTA: one branch around all the loads and one around all the stores
  const bool full = T.aligned && T.n - base >= kSpan;
  const Place<1> row{base + threadIdx.x * kEach, T.n};
  const Place<16> spread{base + (threadIdx.x & ~15) * kEach + (threadIdx.x & 15), T.n};
  const int64_t block = base / kF8Block + (threadIdx.x >> 4);
  const bool some = block * kF8Block < T.n;
  struct {
    Raw p, g, m, v;
    uint2 qm, qv;
    float sm, sv;
  } in;
  auto load = [&](const auto& at) {
    load_raw(in.g, T.g, T.g_type, at);
    if constexpr (F8) {
      in.qm = load_bytes(T.m, at);
      in.qv = load_bytes(T.v, at);
      in.sm = some ? T.m_scale[block] : 0.f;
      in.sv = some ? T.v_scale[block] : 0.f;
    } else {
      load_raw(in.m, T.m, DS_TYPE_F32, at);
      load_raw(in.v, T.v, DS_TYPE_F32, at);
    }
    load_raw(in.p, T.p, T.p_type, at);
  };
  if (full)
    load(row);
  else
    load(spread);

  const Factors& f = P.f;
  float rate = f.rate, root_factor = f.root, decay = T.decay;
  uint32_t step = f.step;
  if (f.lr_dev || f.step_dev) {
    const float lr = f.lr_dev ? *f.lr_dev : f.lr;
    float rest1 = f.rate, rest2 = f.root;  // where t is known: 1 - beta1^t, and the root's factor
    if (f.step_dev) {
      const int64_t t = *f.step_dev;
      step = (uint32_t)t;
      rest1 = rest_of_power(f.log1, t);
      rest2 = __frcp_rn(__fsqrt_rn(rest_of_power(f.log2, t)));
    }
    rate = __fdiv_rn(lr, rest1);
    root_factor = rest2;
    decay = 1.f - lr * T.decay;
  }

  // Pairs of values: two operations per instruction.  Every product and sum is rounded by itself, as defined.
  uint64_t p[4], g[4], m[4], v[4], root[4];
  auto pairs = [](const float (&x)[8], uint64_t (&o)[4]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) o[k] = pair(x[2 * k], x[2 * k + 1]);
  };
  auto values = [](const uint64_t (&x)[4], float (&o)[8]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) unpair(x[k], o[2 * k], o[2 * k + 1]);
  };
  float each[8];
  get_raw(in.g, T.g_type, each);
  pairs(each, g);
  if (f.grad_scale) {
    const uint64_t s = both(*f.grad_scale);
#pragma unroll
    for (int k = 0; k < 4; ++k) g[k] = mul2(g[k], s);
  }
  if constexpr (F8) {
    f8x8_value<false>(in.qm, each);
    pairs(each, m);
    f8x8_value<false>(in.qv, each);
    pairs(each, v);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      m[k] = mul2(m[k], both(in.sm));
      const uint64_t r = mul2(v[k], both(in.sv));
      v[k] = mul2(r, r);
    }
  } else {
    get_raw(in.m, DS_TYPE_F32, each);
    pairs(each, m);
    get_raw(in.v, DS_TYPE_F32, each);
    pairs(each, v);
  }
  get_raw(in.p, T.p_type, each);
  pairs(each, p);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    m[k] = sum(product(m[k], both(f.beta1)), product(g[k], both(f.rest1)));
    v[k] = sum(product(v[k], both(f.beta2)), product(mul2(g[k], g[k]), both(f.rest2)));
  }
  auto root_any = [&] {
#pragma unroll
    for (int k = 0; k < 4; ++k) root[k] = pair(__fsqrt_rn(lo_of(v[k])), __fsqrt_rn(hi_of(v[k])));
  };
  // FAST: by quotient2, within its range
  auto update = [&](auto fast) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint64_t up = mul2(m[k], both(rate)), under = sum(product(root[k], both(root_factor)), both(f.eps));
      uint64_t q;
      if constexpr (decltype(fast)::value)
        q = quotient2(up, under);
      else
        q = pair(__fdiv_rn(lo_of(up), lo_of(under)), __fdiv_rn(hi_of(up), hi_of(under)));
      p[k] = difference(product(p[k], both(decay)), q);
    }
    auto store = [&](const auto& at) {
      float each[8];
      values(p, each);
      store_values(T.p, T.p_type, at, each);
      if (T.copy) store_values(T.copy, T.copy_type, at, each);
    };
    if (full)
      store(row);
    else
      store(spread);
  };
  uint2 qm, qv;
  float sm = 0.f, sv = 0.f;
  if constexpr (F8) {
    const uint32_t key = step * 0xBB67AE85u + T.number * 0x6A09E667u + f.seed;
#pragma unroll
    for (int k = 0; k < 4; ++k) root[k] = root2(v[k]);
    if (!full) {  // values that do not exist add nothing to a block
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (!spread.has(k)) {
          const uint64_t keep = k & 1 ? 0xFFFFFFFFull : 0xFFFFFFFFull << 32;
          m[k / 2] &= keep, v[k / 2] &= keep, root[k / 2] &= keep;
        }
    }
    float top_m = top16(top8(m)), top_v = top16(top8(root));
    const bool fast = top_m * rate <= 0x1p60f && top_v < kInf && top_v * root_factor <= 0x1p59f && f.eps >= 0x1p-60f &&
                      f.eps <= 0x1p59f;
    auto states = [&] {
      const F8Scale s_m = f8_scale<false>(top_m, false), s_v = f8_scale<false>(top_v, false);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        m[k] = product(m[k], both(s_m.inv));  // a sum may follow, in to_neighbours
        root[k] = product(root[k], both(s_v.inv));
      }
      auto round = [&](auto large) {
        const uint32_t step = full ? 0x9E3779B1u : 16u * 0x9E3779B1u;
        uint32_t x0 = (uint32_t)(full ? row.first : spread.first) * 0x9E3779B1u + key, a[4], b[4];
        auto random = [&] {
          uint32_t x = (x0 ^ (x0 >> 16)) * 0x243F6A89u;
          x = (x ^ (x >> 15)) * 0xB7E15163u;
          x0 += step;
          return x;
        };
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t x = random(), y = random();
          a[k] = two_to_f8<false, decltype(large)::value>(m[k], x, y);
          b[k] = two_to_f8<true, decltype(large)::value>(root[k], x, y);
        }
        qm = make_uint2(a[0] | a[1] << 16, a[2] | a[3] << 16);
        qv = make_uint2(b[0] | b[1] << 16, b[2] | b[3] << 16);
      };
      // most warps hold no value below the format's smallest normal one
      if (__all_sync(0xFFFFFFFFu, fast && fminf(least8(m), least8(root)) >= 0x1p-6f))
        round(std::true_type());
      else
        round(std::false_type());
      sm = s_m.s;
      sv = s_v.s;
    };
    if (__all_sync(0xFFFFFFFFu, fast)) {
      update(std::true_type());
    } else {  // values that are not finite, or far from what training meets
      root_any();
      update(std::false_type());
      top_m = top16(finite_top8(m));
      top_v = top16(finite_top8(root));
    }
    states();
  } else {
    root_any();
    update(std::false_type());
  }
  auto store = [&](const auto& at) {
    if constexpr (F8) {
      store_bytes(T.m, at, qm);
      store_bytes(T.v, at, qv);
    } else {
      float each[8];
      values(m, each);
      store_values(T.m, DS_TYPE_F32, at, each);
      values(v, each);
      store_values(T.v, DS_TYPE_F32, at, each);
    }
  };
  if (full)
    store(row);
  else
    store(spread);
  if (F8 && (threadIdx.x & 15) == 0 && some) {
    T.m_scale[block] = sm;
    T.v_scale[block] = sv;
  }
}

template <int N>
cudaError_t launch(const std::vector<Tensor>& all, size_t from, int count, uint32_t ctas, const Factors& f, bool f8,
                   cudaStream_t st) {
  Params<N> p;
  p.f = f;
  p.count = count;
  for (int k = 0; k < count; ++k) p.t[k] = all[from + k];
  if (f8)
    adamw_kernel<true, N><<<ctas, kThreads, 0, st>>>(p);
  else
    adamw_kernel<false, N><<<ctas, kThreads, 0, st>>>(p);
  return cudaGetLastError();
}

cudaError_t launch_all(std::vector<Tensor>& all, const Factors& f, bool f8, cudaStream_t st) {

  size_t from = 0;
  while (from < all.size()) {
    uint64_t ctas = 0;
    size_t to = from;
    for (; to < all.size() && to - from < (size_t)kMany; ++to) {
      const uint64_t mine = (uint64_t)((all[to].n + kSpan - 1) / kSpan);
      if (to > from && ctas + mine > ((uint64_t)1 << 31) - 1) break;
      all[to].first = (uint32_t)ctas;
      ctas += mine;
    }
    const int count = (int)(to - from);
    const cudaError_t e = count <= kFew ? launch<kFew>(all, from, count, (uint32_t)ctas, f, f8, st)
                                        : launch<kMany>(all, from, count, (uint32_t)ctas, f, f8, st);
    if (e != cudaSuccess) return e;
    from = to;
  }
  return cudaSuccess;
}

// A tensor's memories: [at, end), and whether the call writes them.
struct Piece {
  uintptr_t at, end;
  int tensor;
  bool written;
};
constexpr int kKinds = 8;  // p, g, m, v, their scales, copy, and what the options point to

// Written memory is apart from everything else.  The pieces are gone through by address (those of one kind often lie in
// order already): one can only overlap those before it that reach past its start, of which the one that reaches furthest
// and the written one that does are kept.
ds_status check_pieces(std::vector<Piece> (&kinds)[kKinds]) {
  size_t next[kKinds] = {};
  auto before = [](const Piece& a, const Piece& b) { return a.at < b.at; };
  for (auto& pieces : kinds)
    if (!std::is_sorted(pieces.begin(), pieces.end(), before)) std::sort(pieces.begin(), pieces.end(), before);
  uintptr_t any = 0, written = 0;
  for (;;) {
    int first = -1;
    for (int k = 0; k < kKinds; ++k)
      if (next[k] < kinds[k].size() && (first < 0 || kinds[k][next[k]].at < kinds[first][next[first]].at)) first = k;
    if (first < 0) return DS_OK;
    const Piece& q = kinds[first][next[first]++];
    if (q.at < written || (q.written && q.at < any))
      return fail(DS_ERR_INVALID_ARG, "memory of tensor %d overlaps that of another tensor or of itself", q.tensor);
    if (q.end > any) any = q.end;
    if (q.written && q.end > written) written = q.end;
  }
}

ds_status adamw(const ds_adamw_tensor* tensors, int count, const ds_adamw_options* o, cudaStream_t st) {
  if (count < 0) return fail(DS_ERR_SHAPE, "count must not be negative");
  if (!o || (!tensors && count > 0)) return fail(DS_ERR_INVALID_ARG, "NULL pointer argument");
  if (!(o->beta1 >= 0 && o->beta1 < 1 && o->beta2 >= 0 && o->beta2 < 1))
    return fail(DS_ERR_INVALID_ARG, "beta1 and beta2 must be in [0, 1)");
  if (!(o->eps >= 0)) return fail(DS_ERR_INVALID_ARG, "eps must not be negative");
  if (!o->step_dev && o->step < 1) return fail(DS_ERR_INVALID_ARG, "the step must be at least 1");
  if (!o->lr_dev && !(o->lr >= 0)) return fail(DS_ERR_INVALID_ARG, "lr must not be negative");
  if (!aligned(o->step_dev, 8) || !aligned(o->lr_dev, 4) || !aligned(o->grad_scale, 4))
    return fail(DS_ERR_ALIGNMENT, "step_dev must be 8-byte aligned, lr_dev and grad_scale 4-byte aligned");
  std::vector<Tensor> all;
  std::vector<Piece> pieces[kKinds];
  all.reserve(count);
  for (auto& k : pieces) k.reserve(count + 3);
  bool f8 = false, known = false;
  for (int k = 0; k < count; ++k) {
    const ds_adamw_tensor& t = tensors[k];
    ds_status r;
    if (t.n < 0) return fail(DS_ERR_SHAPE, "tensor %d: n must not be negative", k);
    if (t.n > (int64_t)1 << 40) return fail(DS_ERR_UNSUPPORTED, "tensor %d: too large", k);
    if ((r = check_type(t.p_type)) != DS_OK || (r = check_type(t.g_type)) != DS_OK) return r;
    if (t.copy && (r = check_type(t.copy_type)) != DS_OK) return r;
    if (!(t.weight_decay >= 0)) return fail(DS_ERR_INVALID_ARG, "tensor %d: weight_decay must not be negative", k);
    if (t.n == 0) continue;
    if (!t.p || !t.g || !t.m || !t.v) return fail(DS_ERR_INVALID_ARG, "tensor %d: NULL pointer", k);
    if (!t.m_scale != !t.v_scale) return fail(DS_ERR_INVALID_ARG, "tensor %d: one scale of two is given", k);
    if (known && f8 != (t.m_scale != nullptr))
      return fail(DS_ERR_INVALID_ARG, "tensor %d: states of another kind than the others'", k);
    known = true;
    f8 = t.m_scale != nullptr;
    const int64_t ps = type_size(t.p_type), gs = type_size(t.g_type), cs = type_size(t.copy_type), ss = f8 ? 1 : 4;
    if (!aligned(t.p, ps) || !aligned(t.g, gs) || !aligned(t.m, ss) || !aligned(t.v, ss) || !aligned(t.copy, cs) ||
        !aligned(t.m_scale, 4) || !aligned(t.v_scale, 4))
      return fail(DS_ERR_ALIGNMENT, "tensor %d: memory is not aligned to its type", k);
    Tensor d = {};
    d.p = t.p, d.g = t.g, d.m = t.m, d.v = t.v, d.m_scale = t.m_scale, d.v_scale = t.v_scale, d.copy = t.copy, d.n = t.n;
    d.decay = o->lr_dev || o->step_dev ? t.weight_decay : (float)(1.0 - o->lr * (double)t.weight_decay);
    d.number = (uint32_t)k;
    d.p_type = (int8_t)t.p_type, d.g_type = (int8_t)t.g_type, d.copy_type = (int8_t)t.copy_type;
    d.aligned = aligned(t.p, 8 * ps) && aligned(t.g, 8 * gs) && aligned(t.m, 8 * ss) && aligned(t.v, 8 * ss) &&
                aligned(t.copy, 8 * cs);
    all.push_back(d);
    auto piece = [&](int kind, const void* p, int64_t bytes, bool written) {
      if (!p) return;
      const uintptr_t at = reinterpret_cast<uintptr_t>(p);
      pieces[kind].push_back(Piece{at, at + (uintptr_t)bytes, k, written});
    };
    piece(0, t.p, t.n * ps, true);
    piece(1, t.g, t.n * gs, false);
    piece(2, t.m, t.n * ss, true);
    piece(3, t.v, t.n * ss, true);
    piece(4, t.m_scale, blocks_of(t.n) * 4, true);
    piece(5, t.v_scale, blocks_of(t.n) * 4, true);
    piece(6, t.copy, t.n * cs, true);
  }
  if (all.empty()) return DS_OK;
  for (const void* p : {(const void*)o->step_dev, (const void*)o->lr_dev, (const void*)o->grad_scale})
    if (p) pieces[7].push_back(Piece{reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + (p == o->step_dev ? 8 : 4), -1, false});
  const ds_status r = check_pieces(pieces);
  if (r != DS_OK) return r;

  Factors f = {};
  f.beta1 = (float)o->beta1, f.rest1 = (float)(1.0 - o->beta1);
  f.beta2 = (float)o->beta2, f.rest2 = (float)(1.0 - o->beta2);
  f.eps = (float)o->eps;
  f.lr = (float)o->lr;
  f.step_dev = o->step_dev, f.lr_dev = o->lr_dev, f.grad_scale = o->grad_scale;
  f.seed = o->seed;
  f.step = (uint32_t)o->step;
  f.log1 = log(o->beta1), f.log2 = log(o->beta2);
  if (!o->step_dev) {
    const double rest1 = 1.0 - pow(o->beta1, (double)o->step), rest2 = 1.0 - pow(o->beta2, (double)o->step);
    f.rate = o->lr_dev ? (float)rest1 : (float)(o->lr / rest1);
    f.root = (float)(1.0 / sqrt(rest2));
  }
  return cuda_check(launch_all(all, f, f8, st), "adamw launch");
}

}  // namespace
}  // namespace ds

extern "C" ds_status ds_adamw(const ds_adamw_tensor* tensors, int count, const ds_adamw_options* options, void* stream) {
  ds::NvtxRange nvtx_range("ds_adamw");
  ds::clear_error();
  try {
    return ds::adamw(tensors, count, options, static_cast<cudaStream_t>(stream));
  } catch (const std::exception&) {
    return ds::fail(DS_ERR_UNSUPPORTED, "no host memory for the list of %d tensors", count);
  }
}
