// Root-mean-square norm of the residual stream with an 8-bit output, and its
// backward pass.
//
//   forward   h = x + r,  rstd = (mean(h^2) + eps)^-1/2,  n = h rstd w  -> 8 bits, a scale per 128 columns
//   backward  g = dy w,  c = mean(g h rstd),  dx = dh + rstd (g - h rstd c),  dw = sum over rows of dy h rstd
//
// The rounding to 8 bits passes gradients unchanged (the straight-through
// estimate that the paper uses for its own rounding, Eq. 8).  h and the sums
// are float32 in registers; h is rounded once, to the stream's type, where it
// is stored, and the norm itself is taken from the unrounded h.
//
// A CTA holds a row in registers (NV vectors of 8 columns per thread), so
// every input is read once and every output written once: both kernels are
// bound by HBM.  Rows too long for that (NV = 0) are read a second time.
// Measured at 8192 x 4096 bf16 with the residual: forward 38.5 us (6.1 TB/s),
// backward 47.7 us (5.6 TB/s, 5 of them the sum of dw's partial rows); without
// a residual the forward pass is bound by its instructions (30 us, 3.3 TB/s:
// about 30 per value, a third of them the blocks' maxima and scales).  4096 x
// 8192 43 us, 2048 x 16384 (read twice) 58 us.  Rows that are not aligned to
// 16 bytes have instances of their own (8192 x 4100 97 us; value by value 133;
// backward 159, 400).
#include <type_traits>

#include "f8_common.cuh"

namespace ds {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

// The sum over the CTA, the same value (and order of additions) in every thread.
template <int WARPS = kWarps>
__device__ __forceinline__ float cta_sum(float v, float* scratch) {
#pragma unroll
  for (int d = 16; d >= 1; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int w = 0; w < WARPS; ++w) s += scratch[w];
  return s;
}

struct Aligned {  // whether each array's rows start on 16-byte boundaries
  bool a, b, c, d;
};

template <typename T, bool ODD>
__device__ __forceinline__ void load_sum(const RmsnormParams& P, const Aligned& al, int64_t r, int64_t c, int n,
                                         float v[8]) {
  Raw8<T> x;
  x.template load<ODD>(static_cast<const T*>(P.x) + r * P.ldx + c, n, al.a);
  x.get(v);
  if (P.residual) {
    Raw8<T> res;
    float u[8];
    res.template load<ODD>(static_cast<const T*>(P.residual) + r * P.ldr + c, n, al.b);
    res.get(u);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += u[i];
  }
}

// Scales, rounds and stores eight columns; all 32 lanes call it.
template <typename T, bool E5M2, bool ODD>
__device__ __forceinline__ void emit(const RmsnormParams& P, const Aligned& al, int64_t r, int64_t c, int n,
                                     const float v[8], const float w[8], float rstd) {
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = v[i] * rstd * w[i];
  uint2 q;
  const F8Scale s = f8_block<E5M2>(y, P.pow2, q);
  if (n > 0) {
    store_q8(P.out.q + r * P.out.ld + c, n, q);
    if ((threadIdx.x & 15) == 0) P.out.s[r * P.out.lds + c / kF8Block] = s.s;
    if (P.h) store8<ODD>(static_cast<T*>(P.h) + r * P.ldh + c, n, al.c, v);
  }
}

__device__ __forceinline__ void load_weights(const RmsnormParams& P, int64_t c, int n, float w[8]) {
  Raw8<float> rw;
  rw.load(P.weight + c, n, true);
  rw.get(w);
}

// Groups of 256 threads that share an SM: what the registers allow.
template <typename T, int NV>
constexpr int kWalkers = sizeof(T) == 2 && NV == 1 ? 4 : 3;

// A CTA of THREADS walks rows with its share of the weights in registers; the next row is on its way while this one is
// worked on.  For rows whose registers leave room for that on a few CTAs of an SM.
template <typename T, int THREADS, int NV, bool E5M2, bool ODD>
__global__ void __launch_bounds__(THREADS, kWalkers<T, NV> * (kThreads / THREADS))
    rmsnorm_f8_walk_kernel(const RmsnormParams P, const Aligned al, float cols) {
  __shared__ float scratch[2][THREADS / 32];
  int64_t c[NV];
  int n[NV], turn = 0;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    c[k] = ((int64_t)k * THREADS + threadIdx.x) * 8;
    n[k] = left8(P.cols, c[k]);
    if (n[k] <= 0) c[k] = 0;
  }
  Raw8<T> x[NV], res[NV];
  auto load = [&](int64_t r) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      x[k].template load<ODD>(static_cast<const T*>(P.x) + r * P.ldx + c[k], n[k], al.a);
      if (P.residual) res[k].template load<ODD>(static_cast<const T*>(P.residual) + r * P.ldr + c[k], n[k], al.b);
    }
  };
  load(blockIdx.x);
  float w[NV][8];
#pragma unroll
  for (int k = 0; k < NV; ++k) load_weights(P, c[k], n[k], w[k]);
  for (int64_t r = blockIdx.x; r < P.rows; r += gridDim.x, turn ^= 1) {
    float v[NV][8], sum = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      x[k].get(v[k]);
      if (P.residual) {
        float u[8];
        res[k].get(u);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[k][i] += u[i];
      }
    }
    if (r + gridDim.x < P.rows) load(r + gridDim.x);
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fmaf(v[k][i], v[k][i], sum);
    const float rstd = 1.f / sqrtf(cta_sum<THREADS / 32>(sum, scratch[turn]) / cols + P.eps);
    if (P.rstd && threadIdx.x == 0) P.rstd[r] = rstd;
#pragma unroll
    for (int k = 0; k < NV; ++k) emit<T, E5M2, ODD>(P, al, r, c[k], n[k], v[k], w[k], rstd);
  }
}

// Longer rows: a CTA per row.
template <typename T, int NV, bool E5M2, bool ODD>
__global__ void __launch_bounds__(kThreads) rmsnorm_f8_kernel(const RmsnormParams P, const Aligned al,
                                                              float cols) {
  __shared__ float scratch[kWarps];
  const int64_t r = blockIdx.x;
  constexpr int kHeld = NV > 0 ? NV : 1;
  float v[kHeld][8];
  float sum = 0.f;
  if constexpr (NV > 0) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int64_t c = ((int64_t)k * kThreads + threadIdx.x) * 8;
      const int n = left8(P.cols, c);
      load_sum<T, ODD>(P, al, r, n > 0 ? c : 0, n, v[k]);
    }
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fmaf(v[k][i], v[k][i], sum);
  } else {
    for (int64_t c = threadIdx.x * 8; c < P.cols; c += kThreads * 8) {
      load_sum<T, ODD>(P, al, r, c, left8(P.cols, c), v[0]);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fmaf(v[0][i], v[0][i], sum);
    }
  }
  const float rstd = 1.f / sqrtf(cta_sum(sum, scratch) / cols + P.eps);
  if (P.rstd && threadIdx.x == 0) P.rstd[r] = rstd;
  if constexpr (NV > 0) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      int64_t c = ((int64_t)k * kThreads + threadIdx.x) * 8;
      const int n = left8(P.cols, c);
      if (n <= 0) c = 0;
      float w[8];
      load_weights(P, c, n, w);
      emit<T, E5M2, ODD>(P, al, r, c, n, v[k], w, rstd);
    }
  } else {
    // h may be stored over an input: a thread reads its columns again before it writes them
    for (int64_t base = 0; base < P.cols; base += kThreads * 8) {
      int64_t c = base + threadIdx.x * 8;
      const int n = left8(P.cols, c);
      if (n <= 0) c = 0;
      float w[8];
      load_sum<T, ODD>(P, al, r, c, n, v[0]);
      load_weights(P, c, n, w);
      emit<T, E5M2, ODD>(P, al, r, c, n, v[0], w, rstd);
    }
  }
}

// One row of the backward pass, as it lies in memory: dy, h and dh.
template <typename T, int NV, bool ODD>
struct RowIn {
  Raw8<T> dy[NV], h[NV], dh[NV];
  float rstd;
  __device__ __forceinline__ void load(const RmsnormBackwardParams& P, const Aligned& al, int64_t r) {
    rstd = P.rstd[r];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      int64_t c = ((int64_t)k * kThreads + threadIdx.x) * 8;
      const int n = left8(P.cols, c);
      c = n > 0 ? c : 0;
      dy[k].template load<ODD>(static_cast<const T*>(P.dy) + r * P.lddy + c, n, al.a);
      h[k].template load<ODD>(static_cast<const T*>(P.h) + r * P.ldh + c, n, al.b);
      if (P.dh) dh[k].template load<ODD>(static_cast<const T*>(P.dh) + r * P.lddh + c, n, al.c);
    }
  }
};

// A CTA walks rows with its share of the weights and of dw in registers; the next row is on its way while this one is
// worked on, so that the reads never stop for the row's sum (two CTAs of an SM keep 48 KB in flight at 4096 bf16
// columns).
template <typename T, int NV, bool ODD>
__global__ void __launch_bounds__(kThreads, NV == 1 ? (sizeof(T) == 2 ? 3 : 2) : (NV == 2 && sizeof(T) == 2 ? 2 : 1))
    rmsnorm_f8_backward_kernel(const RmsnormBackwardParams P, const Aligned al) {
  __shared__ float scratch[2][kWarps];
  // the next row, unless it would not fit in registers
  constexpr bool AHEAD = NV * sizeof(Raw8<T>) <= 64;
  float w[NV][8], dw[NV][8];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int64_t c = ((int64_t)k * kThreads + threadIdx.x) * 8;
    const int n = left8(P.cols, c);
    Raw8<float> rw;
    rw.load(P.weight + (n > 0 ? c : 0), n, true);
    rw.get(w[k]);
#pragma unroll
    for (int i = 0; i < 8; ++i) dw[k][i] = 0.f;
  }
  RowIn<T, NV, ODD> in, next;
  int turn = 0;
  if (AHEAD) next.load(P, al, blockIdx.x);
  for (int64_t r = blockIdx.x; r < P.rows; r += gridDim.x, turn ^= 1) {
    if (AHEAD) {
      in = next;
      if (r + gridDim.x < P.rows) next.load(P, al, r + gridDim.x);
    } else {
      in.load(P, al, r);
    }
    float dot = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      float dy[8], x[8];
      in.dy[k].get(dy);
      in.h[k].get(x);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] *= in.rstd;
        const float t = dy[i] * x[i];
        dot = fmaf(t, w[k][i], dot);
        dw[k][i] += t;
      }
    }
    const float mean = cta_sum(dot, scratch[turn]) / (float)P.cols;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int64_t c = ((int64_t)k * kThreads + threadIdx.x) * 8;
      const int n = left8(P.cols, c);
      float dy[8], x[8], d[8] = {};
      in.dy[k].get(dy);
      in.h[k].get(x);
      if (P.dh) in.dh[k].get(d);
#pragma unroll
      for (int i = 0; i < 8; ++i) d[i] = fmaf(in.rstd, dy[i] * w[k][i] - x[i] * in.rstd * mean, d[i]);
      if (n > 0) store8<ODD>(static_cast<T*>(P.dx) + r * P.lddx + c, n, al.d, d);
    }
  }
  float* partial = P.partial + (int64_t)blockIdx.x * P.cols;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int64_t c = ((int64_t)k * kThreads + threadIdx.x) * 8;
    const int n = left8(P.cols, c);
    if (n > 0) store8<false>(partial + c, n, P.cols % 4 == 0, dw[k]);
  }
}

// Rows too long for registers: read twice, dw summed in the CTA's partial row.
template <typename T>
__global__ void __launch_bounds__(kThreads) rmsnorm_f8_backward_long_kernel(const RmsnormBackwardParams P,
                                                                            const Aligned al) {
  __shared__ float scratch[2][kWarps];
  float* partial = P.partial + (int64_t)blockIdx.x * P.cols;
  int turn = 0;
  for (int64_t r = blockIdx.x; r < P.rows; r += gridDim.x, turn ^= 1) {
    const float rstd = P.rstd[r];
    auto read = [&](int64_t c, int n, float g[8], float x[8], float dy[8]) {
      Raw8<T> a, b;
      Raw8<float> w;
      a.load(static_cast<const T*>(P.dy) + r * P.lddy + c, n, al.a);
      b.load(static_cast<const T*>(P.h) + r * P.ldh + c, n, al.b);
      w.load(P.weight + c, n, true);
      a.get(dy);
      b.get(x);
      w.get(g);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] *= rstd;
        g[i] *= dy[i];
      }
    };
    float dot = 0.f;
    for (int64_t c = threadIdx.x * 8; c < P.cols; c += kThreads * 8) {
      const int n = left8(P.cols, c);
      float g[8], x[8], dy[8];
      read(c, n, g, x, dy);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        dot = fmaf(g[i], x[i], dot);
        if (i < n) partial[c + i] = fmaf(dy[i], x[i], r == blockIdx.x ? 0.f : partial[c + i]);
      }
    }
    const float mean = cta_sum(dot, scratch[turn]) / (float)P.cols;
    // dx may be one of the inputs: a thread reads its columns again before it writes them
    for (int64_t c = threadIdx.x * 8; c < P.cols; c += kThreads * 8) {
      const int n = left8(P.cols, c);
      float g[8], x[8], dy[8], d[8] = {};
      read(c, n, g, x, dy);
      if (P.dh) {
        Raw8<T> a;
        a.load(static_cast<const T*>(P.dh) + r * P.lddh + c, n, al.c);
        a.get(d);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) d[i] = fmaf(rstd, g[i] - x[i] * mean, d[i]);
      store8<false>(static_cast<T*>(P.dx) + r * P.lddx + c, n, al.d, d);
    }
  }
}

// dw[c] = sum of the partial rows, in a fixed order: 16 groups of rows, then the groups.
__global__ void __launch_bounds__(512) rmsnorm_dw_kernel(const float* partial, int64_t n, int64_t cols, float* dw) {
  __shared__ float part[16][33];
  const int lane = threadIdx.x & 31, group = threadIdx.x >> 5;
  const int64_t c = (int64_t)blockIdx.x * 32 + lane;
  float s = 0.f;
  if (c < cols) {
#pragma unroll 8
    for (int64_t i = group; i < n; i += 16) s += partial[i * cols + c];
  }
  part[group][lane] = s;
  __syncthreads();
  if (group == 0 && c < cols) {
    float t = 0.f;
#pragma unroll
    for (int g = 0; g < 16; ++g) t += part[g][lane];
    dw[c] = t;
  }
}

bool rows16(const void* p, int64_t ld, size_t size) {
  return p == nullptr || ((reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld * (int64_t)size % 16 == 0);
}

// Rows of up to 4096 16-bit values (2048 of float32) are walked: with residual 8192 x 2048 bf16 takes 21 us (a CTA per
// row 29), 8192 x 4096 39 (41); 4096 x 8192 would take 49 (43).  Rows of up to 1024 take smaller CTAs, whose threads all
// work (8192 x 1024 10 us, 23 with 256 threads).
template <typename T, bool E5M2, bool ODD>
cudaError_t forward_as(const RmsnormParams& p, const Aligned& al, cudaStream_t st) {
  const int64_t sms = sm_count() > 0 ? sm_count() : 1;
  const float cols = (float)p.cols;
  auto walk = [&](auto kernel, int threads, int groups) {
    const int64_t fit = sms * groups * (kThreads / threads);
    kernel<<<(unsigned)(p.rows < fit ? p.rows : fit), threads, 0, st>>>(p, al, cols);
  };
  const unsigned grid = (unsigned)p.rows;
  if (p.cols <= 1024)
    walk(rmsnorm_f8_walk_kernel<T, 128, 1, E5M2, ODD>, 128, kWalkers<T, 1>);
  else if (p.cols <= 2048)
    walk(rmsnorm_f8_walk_kernel<T, 256, 1, E5M2, ODD>, 256, kWalkers<T, 1>);
  else if (p.cols <= 4096) {
    if constexpr (sizeof(T) == 2)
      walk(rmsnorm_f8_walk_kernel<T, 256, 2, E5M2, ODD>, 256, kWalkers<T, 2>);
    else
      rmsnorm_f8_kernel<T, 2, E5M2, ODD><<<grid, kThreads, 0, st>>>(p, al, cols);
  } else if (p.cols <= 8192)
    rmsnorm_f8_kernel<T, 4, E5M2, ODD><<<grid, kThreads, 0, st>>>(p, al, cols);
  else
    rmsnorm_f8_kernel<T, 0, E5M2, ODD><<<grid, kThreads, 0, st>>>(p, al, cols);
  return cudaGetLastError();
}

// ODD: some rows of 16-bit values are not aligned, and their loads and stores are code that the others go without.
template <typename T, bool E5M2>
cudaError_t forward_of(const RmsnormParams& p, cudaStream_t st) {
  const Aligned al{rows16(p.x, p.ldx, sizeof(T)), rows16(p.residual, p.ldr, sizeof(T)), rows16(p.h, p.ldh, sizeof(T)),
                   true};
  if constexpr (sizeof(T) == 2) {
    if (!(al.a && al.b && al.c)) return forward_as<T, E5M2, true>(p, al, st);
  }
  return forward_as<T, E5M2, false>(p, al, st);
}

template <typename T>
cudaError_t forward(const RmsnormParams& p, cudaStream_t st) {
  return p.e5m2 ? forward_of<T, true>(p, st) : forward_of<T, false>(p, st);
}

template <typename T>
cudaError_t backward(const RmsnormBackwardParams& p, cudaStream_t st) {
  const Aligned al{rows16(p.dy, p.lddy, sizeof(T)), rows16(p.h, p.ldh, sizeof(T)), rows16(p.dh, p.lddh, sizeof(T)),
                   rows16(p.dx, p.lddx, sizeof(T))};
  const int nv = p.cols <= kThreads * 8 ? 1 : (p.cols <= 2 * kThreads * 8 ? 2 : (p.cols <= 4 * kThreads * 8 ? 4 : 0));
  // the CTAs that fit at once (of the 152 SMs; fewer SMs take them in turn), each with a partial row of dw
  const int of_sm = nv == 0 ? 4 : (nv == 1 ? (sizeof(T) == 2 ? 3 : 2) : (nv == 2 && sizeof(T) == 2 ? 2 : 1));
  const int64_t fit = kF8NormPartials / 4 * of_sm;
  const int64_t n = p.rows < fit ? p.rows : fit;
  if (n > 0) {
    const unsigned grid = (unsigned)n;
    auto run = [&](auto odd) {
      constexpr bool ODD = decltype(odd)::value;
      if (nv == 1)
        rmsnorm_f8_backward_kernel<T, 1, ODD><<<grid, kThreads, 0, st>>>(p, al);
      else if (nv == 2)
        rmsnorm_f8_backward_kernel<T, 2, ODD><<<grid, kThreads, 0, st>>>(p, al);
      else
        rmsnorm_f8_backward_kernel<T, 4, ODD><<<grid, kThreads, 0, st>>>(p, al);
    };
    if (nv == 0)
      rmsnorm_f8_backward_long_kernel<T><<<grid, kThreads, 0, st>>>(p, al);
    else if (sizeof(T) == 2 && !(al.a && al.b && al.c && al.d))
      run(std::integral_constant<bool, sizeof(T) == 2>{});
    else
      run(std::false_type{});
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  rmsnorm_dw_kernel<<<(unsigned)((p.cols + 31) / 32), 512, 0, st>>>(p.partial, n, p.cols, p.dw);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_rmsnorm_f8(const RmsnormParams& p, int type, cudaStream_t st) {
  if (type == DS_TYPE_F32) return forward<float>(p, st);
  if (type == DS_TYPE_BF16) return forward<__nv_bfloat16>(p, st);
  return forward<__half>(p, st);
}

cudaError_t launch_rmsnorm_f8_backward(const RmsnormBackwardParams& p, int type, cudaStream_t st) {
  if (type == DS_TYPE_F32) return backward<float>(p, st);
  if (type == DS_TYPE_BF16) return backward<__nv_bfloat16>(p, st);
  return backward<__half>(p, st);
}

}  // namespace ds
