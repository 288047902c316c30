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
#include "f8_common.cuh"

namespace ds {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

// The sum over the CTA, the same value (and order of additions) in every thread.
__device__ __forceinline__ float cta_sum(float v, float* scratch) {
#pragma unroll
  for (int d = 16; d >= 1; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) s += scratch[w];
  return s;
}

__device__ __forceinline__ int left8(int64_t cols, int64_t c) {
  const int64_t n = cols - c;
  return n >= 8 ? 8 : (n < 0 ? 0 : (int)n);
}

struct Aligned {  // whether each array's rows start on 16-byte boundaries
  bool a, b, c, d;
};

template <typename T>
__device__ __forceinline__ void load_sum(const RmsnormParams& P, const Aligned& al, int64_t r, int64_t c, int n,
                                         float v[8]) {
  Raw8<T> x;
  x.load(static_cast<const T*>(P.x) + r * P.ldx + c, n, al.a);
  x.get(v);
  if (P.residual) {
    Raw8<T> res;
    float u[8];
    res.load(static_cast<const T*>(P.residual) + r * P.ldr + c, n, al.b);
    res.get(u);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += u[i];
  }
}

// Scales, rounds and stores eight columns; all 32 lanes call it.
template <typename T>
__device__ __forceinline__ void emit(const RmsnormParams& P, const Aligned& al, int64_t r, int64_t c, int n,
                                     const float v[8], float rstd) {
  float w[8], y[8];
  Raw8<float> rw;
  rw.load(P.weight + c, n, al.d);
  rw.get(w);
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = v[i] * rstd * w[i];
  uint2 q;
  const F8Scale s = f8_block(y, P.out.e5m2, P.pow2, q);
  if (n > 0) {
    store_q8(P.out.q + r * P.out.ld + c, n, q);
    if ((threadIdx.x & 15) == 0) P.out.s[r * P.out.lds + c / kF8Block] = s.s;
    if (P.h) store8(static_cast<T*>(P.h) + r * P.ldh + c, n, al.c, v);
  }
}

template <typename T, int NV>
__global__ void __launch_bounds__(kThreads) rmsnorm_f8_kernel(const RmsnormParams P, const Aligned al) {
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
      load_sum<T>(P, al, r, n > 0 ? c : 0, n, v[k]);
    }
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fmaf(v[k][i], v[k][i], sum);
  } else {
    for (int64_t c = threadIdx.x * 8; c < P.cols; c += kThreads * 8) {
      load_sum<T>(P, al, r, c, left8(P.cols, c), v[0]);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fmaf(v[0][i], v[0][i], sum);
    }
  }
  const float rstd = 1.f / sqrtf(cta_sum(sum, scratch) / (float)P.cols + P.eps);
  if (P.rstd && threadIdx.x == 0) P.rstd[r] = rstd;
  if constexpr (NV > 0) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int64_t c = ((int64_t)k * kThreads + threadIdx.x) * 8;
      const int n = left8(P.cols, c);
      emit<T>(P, al, r, n > 0 ? c : 0, n, v[k], rstd);
    }
  } else {
    // h may be stored over an input: a thread reads its columns again before it writes them
    for (int64_t base = 0; base < P.cols; base += kThreads * 8) {
      const int64_t c = base + threadIdx.x * 8;
      const int n = left8(P.cols, c);
      load_sum<T>(P, al, r, n > 0 ? c : 0, n, v[0]);
      emit<T>(P, al, r, n > 0 ? c : 0, n, v[0], rstd);
    }
  }
}

template <typename T, int NV>
__global__ void __launch_bounds__(kThreads) rmsnorm_f8_backward_kernel(const RmsnormBackwardParams P,
                                                                       const Aligned al) {
  __shared__ float scratch[2][kWarps];
  constexpr int kHeld = NV > 0 ? NV : 1;
  float* partial = P.partial + (int64_t)blockIdx.x * P.cols;
  float dw[kHeld][8] = {};
  int turn = 0;
  for (int64_t r = blockIdx.x; r < P.rows; r += gridDim.x, turn ^= 1) {
    const float rstd = P.rstd[r];
    float g[kHeld][8], x[kHeld][8];  // dy w and h rstd
    float dot = 0.f;
    const T* dy_row = static_cast<const T*>(P.dy) + r * P.lddy;
    const T* h_row = static_cast<const T*>(P.h) + r * P.ldh;
    const T* dh_row = static_cast<const T*>(P.dh) + r * P.lddh;
    T* dx_row = static_cast<T*>(P.dx) + r * P.lddx;
    auto read = [&](int64_t c, int n, float gk[8], float xk[8], float dyk[8]) {
      Raw8<T> a, b;
      Raw8<float> w;
      a.load(dy_row + c, n, al.a);
      b.load(h_row + c, n, al.b);
      w.load(P.weight + c, n, true);
      a.get(dyk);
      b.get(xk);
      w.get(gk);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        xk[i] *= rstd;
        gk[i] *= dyk[i];
      }
    };
    auto write = [&](int64_t c, int n, const float gk[8], const float xk[8], float mean) {
      float d[8] = {};
      if (P.dh) {
        Raw8<T> a;
        a.load(dh_row + c, n, al.c);
        a.get(d);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) d[i] = fmaf(rstd, gk[i] - xk[i] * mean, d[i]);
      store8(dx_row + c, n, al.d, d);
    };
    if constexpr (NV > 0) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int64_t c = ((int64_t)k * kThreads + threadIdx.x) * 8;
        const int n = left8(P.cols, c);
        float dyk[8];
        read(n > 0 ? c : 0, n, g[k], x[k], dyk);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          dot = fmaf(g[k][i], x[k][i], dot);
          dw[k][i] = fmaf(dyk[i], x[k][i], dw[k][i]);
        }
      }
    } else {
      for (int64_t c = threadIdx.x * 8; c < P.cols; c += kThreads * 8) {
        const int n = left8(P.cols, c);
        float dyk[8];
        read(c, n, g[0], x[0], dyk);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          dot = fmaf(g[0][i], x[0][i], dot);
          if (i < n) partial[c + i] = fmaf(dyk[i], x[0][i], r == blockIdx.x ? 0.f : partial[c + i]);
        }
      }
    }
    const float mean = cta_sum(dot, scratch[turn]) / (float)P.cols;
    if constexpr (NV > 0) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int64_t c = ((int64_t)k * kThreads + threadIdx.x) * 8;
        const int n = left8(P.cols, c);
        if (n > 0) write(c, n, g[k], x[k], mean);
      }
    } else {
      for (int64_t c = threadIdx.x * 8; c < P.cols; c += kThreads * 8) {
        const int n = left8(P.cols, c);
        float dyk[8];
        read(c, n, g[0], x[0], dyk);
        write(c, n, g[0], x[0], mean);
      }
    }
  }
  if constexpr (NV > 0) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int64_t c = ((int64_t)k * kThreads + threadIdx.x) * 8;
      const int n = left8(P.cols, c);
      if (n > 0) store8(partial + c, n, P.cols % 4 == 0, dw[k]);
    }
  }
}

// dw[c] = sum of the partial rows, in a fixed order: 16 groups of rows, then the groups.
__global__ void __launch_bounds__(512) rmsnorm_dw_kernel(const float* partial, int64_t n, int64_t cols, float* dw) {
  __shared__ float part[16][33];
  const int lane = threadIdx.x & 31, group = threadIdx.x >> 5;
  const int64_t c = (int64_t)blockIdx.x * 32 + lane;
  float s = 0.f;
  if (c < cols)
    for (int64_t i = group; i < n; i += 16) s += partial[i * cols + c];
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
  return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld * (int64_t)size % 16 == 0;
}

template <typename T>
cudaError_t forward(const RmsnormParams& p, cudaStream_t st) {
  const Aligned al{rows16(p.x, p.ldx, sizeof(T)), rows16(p.residual, p.ldr, sizeof(T)), rows16(p.h, p.ldh, sizeof(T)),
                   rows16(p.weight, 0, 4)};
  const unsigned grid = (unsigned)p.rows;
  if (p.cols <= kThreads * 8)
    rmsnorm_f8_kernel<T, 1><<<grid, kThreads, 0, st>>>(p, al);
  else if (p.cols <= 2 * kThreads * 8)
    rmsnorm_f8_kernel<T, 2><<<grid, kThreads, 0, st>>>(p, al);
  else if (p.cols <= 4 * kThreads * 8)
    rmsnorm_f8_kernel<T, 4><<<grid, kThreads, 0, st>>>(p, al);
  else
    rmsnorm_f8_kernel<T, 0><<<grid, kThreads, 0, st>>>(p, al);
  return cudaGetLastError();
}

template <typename T>
cudaError_t backward(const RmsnormBackwardParams& p, cudaStream_t st) {
  const Aligned al{rows16(p.dy, p.lddy, sizeof(T)), rows16(p.h, p.ldh, sizeof(T)), rows16(p.dh, p.lddh, sizeof(T)),
                   rows16(p.dx, p.lddx, sizeof(T))};
  const int64_t n = p.rows < kF8NormPartials ? p.rows : kF8NormPartials;
  if (n > 0) {
    const unsigned grid = (unsigned)n;
    if (p.cols <= kThreads * 8)
      rmsnorm_f8_backward_kernel<T, 1><<<grid, kThreads, 0, st>>>(p, al);
    else if (p.cols <= 2 * kThreads * 8)
      rmsnorm_f8_backward_kernel<T, 2><<<grid, kThreads, 0, st>>>(p, al);
    else if (p.cols <= 4 * kThreads * 8)
      rmsnorm_f8_backward_kernel<T, 4><<<grid, kThreads, 0, st>>>(p, al);
    else
      rmsnorm_f8_backward_kernel<T, 0><<<grid, kThreads, 0, st>>>(p, al);
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
