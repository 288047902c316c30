// What the experts' operators share between their kernels and their entry points.
#pragma once

#include "f8_checks.cuh"

namespace ds {

struct ExpertProduct {  // y = x w_e^T for the rows of each segment, or (grad) dw_e = sum over its rows of dy_t x_t
  const ds_f8_matrix *x, *w;  // grad: x_t, dy_t
  const ds_expert_slots* s;
  const float* bias;
  const float* add;
  int64_t ld_add;
  void* y;
  int type;
  int64_t ldy;
};

cudaError_t launch_expert_order(const void* ids, int id_type, const ds_expert_slots& s, cudaStream_t st);
// Rows of `bytes` each, copied to the rows of their token's slots; with a second matrix of the same rows where its dst is
// given (a source without tokens has no memory).
struct RowCopy {
  const void* src;
  void* dst;
  int64_t ld_src, ld_dst, bytes;  // in bytes
};
cudaError_t launch_expert_gather(const RowCopy& a, const RowCopy& b, const ds_expert_slots& s, cudaStream_t st);
cudaError_t launch_expert_combine(const void* y, int type, int64_t ldy, int64_t cols, const ds_expert_slots& s,
                                  const float* weights, const void* add, int64_t ld_add, void* out, int64_t ldo,
                                  cudaStream_t st);
cudaError_t launch_expert_combine_backward(const void* dout, int64_t ldd, const void* y, int64_t ldy, int type,
                                           int64_t cols, const ds_expert_slots& s, const float* weights, void* dy,
                                           int64_t lddy, float* dweights, cudaStream_t st);
cudaError_t launch_expert_linear_f8(const ExpertProduct& p, cudaStream_t st);
cudaError_t launch_expert_weight_grad_f8(const ExpertProduct& p, cudaStream_t st);

}  // namespace ds
