// C ABI entry points of the 8-bit floating-point operators: argument
// validation, then stream-ordered launches.  Nothing is launched and no
// output is written when validation fails.
#include "f8_checks.cuh"

namespace ds {
namespace {

// The 8-bit matrices that a call writes have one format.
ds_status check_formats(const ds_f8_matrix* a, const ds_f8_matrix* b, const ds_f8_matrix* c, bool* e5m2) {
  const ds_f8_matrix* first = a ? a : (b ? b : c);
  for (const ds_f8_matrix* m : {a, b, c})
    if (m && m->format != first->format) return fail(DS_ERR_INVALID_ARG, "the outputs have different 8-bit formats");
  *e5m2 = first->format == DS_F8_E5M2;
  return DS_OK;
}

// The outputs of a quantiser: shapes, at least one, no overlap with each other or the source.
ds_status check_quantize(const Span (&src)[2], int64_t rows, int64_t cols, const ds_f8_matrix* out,
                         const ds_f8_matrix* out_t, uint32_t flags, bool* e5m2) {
  if (!out && !out_t) return fail(DS_ERR_INVALID_ARG, "neither out nor out_t is given");
  ds_status r = check_flags(flags);
  if (r != DS_OK) return r;
  if ((r = check_f8_out("out", out, rows, cols, false)) != DS_OK) return r;
  if ((r = check_f8_out("out_t", out_t, cols, rows, false)) != DS_OK) return r;
  if ((r = check_formats(out, out_t, nullptr, e5m2)) != DS_OK) return r;
  const Span outs[] = {values_of("out", out), scales_of("out's scales", out), values_of("out_t", out_t),
                       scales_of("out_t's scales", out_t)};
  if ((r = check_apart(outs, src)) != DS_OK) return r;
  if (blocks_of(rows) * blocks_of(cols) > ((int64_t)1 << 31) - 1) return fail(DS_ERR_UNSUPPORTED, "matrix too large");
  return DS_OK;
}

ds_status check_linear(const LinearF8Params& p) {
  if (!p.x || !p.w) return fail(DS_ERR_INVALID_ARG, "NULL x or w");
  ds_status r = check_type(p.type);
  if (r != DS_OK) return r;
  if ((r = check_f8("x", p.x)) != DS_OK) return r;
  if ((r = check_f8("w", p.w)) != DS_OK) return r;
  if (p.x->cols != p.w->cols)
    return fail(DS_ERR_SHAPE, "x has %lld columns, w %lld", (long long)p.x->cols, (long long)p.w->cols);
  const int64_t M = p.x->rows, N = p.w->rows, size = type_size(p.type);
  if (!p.y && M > 0 && N > 0) return fail(DS_ERR_INVALID_ARG, "NULL y");
  if ((r = check_tensor("y", p.y, M, N, p.ldy, size)) != DS_OK) return r;
  if ((r = check_tensor("add", p.add, M, N, p.ld_add, 4)) != DS_OK) return r;
  if ((r = check_tensor("bias", p.bias, 1, N, N, 4)) != DS_OK) return r;
  const bool in_place = p.type == DS_TYPE_F32 && same(p.y, p.ldy, p.add, p.ld_add);
  const Span outs[] = {span("y", p.y, strided(M, N, p.ldy, size))};
  const Span ins[] = {values_of("x", p.x), scales_of("x's scales", p.x), values_of("w", p.w),
                      scales_of("w's scales", p.w), span("bias", p.bias, 4 * N),
                      span("add", in_place ? nullptr : p.add, strided(M, N, p.ld_add, 4))};
  if ((r = check_apart(outs, ins)) != DS_OK) return r;
  // the finest tiling (16 x 128, split 8 ways) stays inside a grid's 2^31 - 1 CTAs
  if (blocks_of(N) * ((M + 15) / 16) > ((int64_t)1 << 28) - 1) return fail(DS_ERR_UNSUPPORTED, "M x N too large");
  return DS_OK;
}

}  // namespace
}  // namespace ds

using namespace ds;

extern "C" {

ds_status ds_quantize_f8(const void* x, int type, int64_t rows, int64_t cols, int64_t ldx, const ds_f8_matrix* out,
                         const ds_f8_matrix* out_t, uint32_t flags, void* stream) {
  NvtxRange nvtx_range("ds_quantize_f8");
  clear_error();
  ds_status r = check_type(type);
  if (r != DS_OK) return r;
  if ((r = check_dims("x", rows, cols)) != DS_OK) return r;
  if (!x && rows > 0 && cols > 0) return fail(DS_ERR_INVALID_ARG, "NULL x");
  if ((r = check_tensor("x", x, rows, cols, ldx, type_size(type))) != DS_OK) return r;
  const Span src[] = {span("x", x, strided(rows, cols, ldx, type_size(type))), span("x", nullptr, 0)};
  bool e5m2 = false;
  if ((r = check_quantize(src, rows, cols, out, out_t, flags, &e5m2)) != DS_OK) return r;
  if (rows == 0 || cols == 0) return DS_OK;
  return cuda_check(launch_quantize_f8(x, type, rows, cols, ldx, f8_out(out), f8_out(out_t), e5m2,
                                       (flags & DS_F8_POW2) != 0, static_cast<cudaStream_t>(stream)),
                    "quantize_f8 launch");
}

ds_status ds_requantize_f8(const ds_f8_matrix* x, const ds_f8_matrix* out, const ds_f8_matrix* out_t, uint32_t flags,
                           void* stream) {
  NvtxRange nvtx_range("ds_requantize_f8");
  clear_error();
  if (!x) return fail(DS_ERR_INVALID_ARG, "NULL x");
  ds_status r = check_f8("x", x);
  if (r != DS_OK) return r;
  const Span src[] = {values_of("x", x), scales_of("x's scales", x)};
  bool e5m2 = false;
  if ((r = check_quantize(src, x->rows, x->cols, out, out_t, flags, &e5m2)) != DS_OK) return r;
  if (x->rows == 0 || x->cols == 0) return DS_OK;
  return cuda_check(launch_requantize_f8(x, f8_out(out), f8_out(out_t), e5m2, (flags & DS_F8_POW2) != 0,
                                         static_cast<cudaStream_t>(stream)),
                    "requantize_f8 launch");
}

ds_status ds_expand_shift_weights_f8(const ds_weights* w, const ds_f8_matrix* out, void* stream) {
  NvtxRange nvtx_range("ds_expand_shift_weights_f8");
  clear_error();
  if (!w || !out) return fail(DS_ERR_INVALID_ARG, "NULL pointer argument");
  ds_status r = check_weights(w, w->n_out, w->k_red);
  if (r != DS_OK) return r;
  if ((r = check_f8_out("out", out, w->n_out, w->k_red, false)) != DS_OK) return r;
  if (out->format != DS_F8_E4M3 || out->blocks != DS_F8_TILES)
    return fail(DS_ERR_INVALID_ARG, "out must be e4m3 in tiles");
  return cuda_check(launch_expand_f8(static_cast<const uint8_t*>(w->packed), w->n_out, w->k_red, f8_out(out),
                                     static_cast<cudaStream_t>(stream)),
                    "8-bit expand launch");
}

ds_status ds_linear_f8(const ds_f8_matrix* x, const ds_f8_matrix* w, const float* bias, const float* add,
                       int64_t ld_add, void* y, int type, int64_t ldy, void* stream) {
  NvtxRange nvtx_range("ds_linear_f8");
  clear_error();
  const LinearF8Params p{x, w, bias, add, ld_add, y, type, ldy};
  const ds_status r = check_linear(p);
  if (r != DS_OK) return r;
  if (x->rows == 0 || w->rows == 0) return DS_OK;
  return cuda_check(launch_linear_f8(p, static_cast<cudaStream_t>(stream)), "linear_f8 launch");
}

int ds_linear_f8_tile(const ds_f8_matrix* x, const ds_f8_matrix* w, const float* add, int64_t ld_add, void* y, int type,
                      int64_t ldy) {
  clear_error();
  const LinearF8Params p{x, w, nullptr, add, ld_add, y, type, ldy};
  if (check_linear(p) != DS_OK || x->rows == 0 || w->rows == 0) return 0;
  return linear_f8_tile(p);
}

int ds_f8_fault_flag(void) {
  // all are read, and so cleared
  const int a = read_f8_fault_flag(), b = read_gated_f8_fault_flag(), c = read_expert_f8_fault_flag();
  return a < 0 || b < 0 || c < 0 ? -1 : (a | b | c);
}

void ds_f8_set_wait_limit(long long cycles) { set_f8_wait_cycles(cycles); }

ds_status ds_rmsnorm_f8(const void* x, int64_t ldx, const void* residual, int64_t ldr, const float* weight, int type,
                        int64_t rows, int64_t cols, float eps, const ds_f8_matrix* out, void* h, int64_t ldh,
                        float* rstd, uint32_t flags, void* stream) {
  NvtxRange nvtx_range("ds_rmsnorm_f8");
  clear_error();
  if (!out || !weight) return fail(DS_ERR_INVALID_ARG, "NULL out or weight");
  ds_status r = check_type(type);
  if (r != DS_OK) return r;
  if ((r = check_flags(flags)) != DS_OK) return r;
  if ((r = check_dims("x", rows, cols)) != DS_OK) return r;
  if (cols == 0) return fail(DS_ERR_SHAPE, "a norm needs columns");
  if (!(eps >= 0.f)) return fail(DS_ERR_INVALID_ARG, "eps must not be negative");
  if (!x && rows > 0) return fail(DS_ERR_INVALID_ARG, "NULL x");
  const int64_t size = type_size(type);
  if ((r = check_tensor("x", x, rows, cols, ldx, size)) != DS_OK) return r;
  if ((r = check_tensor("residual", residual, rows, cols, ldr, size)) != DS_OK) return r;
  if ((r = check_tensor("h", h, rows, cols, ldh, size)) != DS_OK) return r;
  if ((r = check_tensor("weight", weight, 1, cols, cols, 16)) != DS_OK) return r;
  if ((r = check_tensor("rstd", rstd, 1, rows, rows, 4)) != DS_OK) return r;
  if ((r = check_f8_out("out", out, rows, cols, true)) != DS_OK) return r;
  const Span outs[] = {values_of("out", out), scales_of("out's scales", out),
                       span("h", h, strided(rows, cols, ldh, size)), span("rstd", rstd, 4 * rows)};
  const Span ins[] = {span("x", same(h, ldh, x, ldx) ? nullptr : x, strided(rows, cols, ldx, size)),
                      span("residual", same(h, ldh, residual, ldr) ? nullptr : residual,
                           strided(rows, cols, ldr, size)),
                      span("weight", weight, 4 * cols)};
  if ((r = check_apart(outs, ins)) != DS_OK) return r;
  if (rows == 0) return DS_OK;
  const RmsnormParams p{x,  residual, ldx, ldr, weight, rows, cols, eps, f8_out(out),
                        h,  ldh,      rstd, out->format == DS_F8_E5M2, (flags & DS_F8_POW2) != 0};
  return cuda_check(launch_rmsnorm_f8(p, type, static_cast<cudaStream_t>(stream)), "rmsnorm_f8 launch");
}

size_t ds_rmsnorm_f8_backward_workspace_bytes(int64_t rows, int64_t cols) {
  if (rows < 0 || cols <= 0 || rows > kMaxDim || cols > kMaxDim) return 0;
  return (size_t)((rows < kF8NormPartials ? rows : kF8NormPartials) * cols * 4 + 255) / 256 * 256;
}

ds_status ds_rmsnorm_f8_backward(const void* dy, int64_t lddy, const void* h, int64_t ldh, const float* rstd,
                                 const float* weight, const void* dh, int64_t lddh, int type, int64_t rows,
                                 int64_t cols, void* dx, int64_t lddx, float* dw, void* ws, size_t ws_bytes,
                                 void* stream) {
  NvtxRange nvtx_range("ds_rmsnorm_f8_backward");
  clear_error();
  if (!weight || !dw) return fail(DS_ERR_INVALID_ARG, "NULL weight or dw");
  ds_status r = check_type(type);
  if (r != DS_OK) return r;
  if ((r = check_dims("dy", rows, cols)) != DS_OK) return r;
  if (cols == 0) return fail(DS_ERR_SHAPE, "a norm needs columns");
  if (rows > 0 && (!dy || !h || !rstd || !dx || !ws)) return fail(DS_ERR_INVALID_ARG, "NULL pointer argument");
  const int64_t size = type_size(type);
  if ((r = check_tensor("dy", dy, rows, cols, lddy, size)) != DS_OK) return r;
  if ((r = check_tensor("h", h, rows, cols, ldh, size)) != DS_OK) return r;
  if ((r = check_tensor("dh", dh, rows, cols, lddh, size)) != DS_OK) return r;
  if ((r = check_tensor("dx", dx, rows, cols, lddx, size)) != DS_OK) return r;
  if ((r = check_tensor("rstd", rstd, 1, rows, rows, 4)) != DS_OK) return r;
  if ((r = check_tensor("weight", weight, 1, cols, cols, 16)) != DS_OK) return r;
  if ((r = check_tensor("dw", dw, 1, cols, cols, 4)) != DS_OK) return r;
  const size_t need = ds_rmsnorm_f8_backward_workspace_bytes(rows, cols);
  if (ws_bytes < need) return fail(DS_ERR_BUFFER_TOO_SMALL, "workspace has %zu bytes, needs %zu", ws_bytes, need);
  if (!aligned(ws, 16)) return fail(DS_ERR_ALIGNMENT, "the workspace must be 16-byte aligned");
  const Span outs[] = {span("dx", dx, strided(rows, cols, lddx, size)), span("dw", dw, 4 * cols),
                       span("the workspace", ws, (int64_t)need)};
  const Span ins[] = {span("dy", same(dx, lddx, dy, lddy) ? nullptr : dy, strided(rows, cols, lddy, size)),
                      span("h", same(dx, lddx, h, ldh) ? nullptr : h, strided(rows, cols, ldh, size)),
                      span("dh", same(dx, lddx, dh, lddh) ? nullptr : dh, strided(rows, cols, lddh, size)),
                      span("rstd", rstd, 4 * rows), span("weight", weight, 4 * cols)};
  if ((r = check_apart(outs, ins)) != DS_OK) return r;
  const RmsnormBackwardParams p{dy,   h,    dh,   lddy, ldh,  lddh,
                                rstd, weight, rows, cols, dx, lddx, dw, static_cast<float*>(ws)};
  return cuda_check(launch_rmsnorm_f8_backward(p, type, static_cast<cudaStream_t>(stream)),
                    "rmsnorm_f8_backward launch");
}

ds_status ds_gated_f8(const void* gu, int type, int64_t ld, int64_t rows, int64_t features, const ds_f8_matrix* out,
                      const ds_f8_matrix* ckpt, uint32_t flags, void* stream) {
  NvtxRange nvtx_range("ds_gated_f8");
  clear_error();
  if (!out) return fail(DS_ERR_INVALID_ARG, "NULL out");
  ds_status r = check_type(type);
  if (r != DS_OK) return r;
  if ((r = check_flags(flags)) != DS_OK) return r;
  if ((r = check_dims("gu", rows, features)) != DS_OK) return r;
  if (features == 0) return fail(DS_ERR_SHAPE, "a gate needs features");
  if (!gu && rows > 0) return fail(DS_ERR_INVALID_ARG, "NULL gu");
  const int64_t width = blocks_of(features) * kF8Block + features, size = type_size(type);
  if ((r = check_tensor("gu", gu, rows, width, ld, size)) != DS_OK) return r;
  if ((r = check_f8_out("out", out, rows, features, true)) != DS_OK) return r;
  if ((r = check_f8_out("ckpt", ckpt, rows, width, true)) != DS_OK) return r;
  bool e5m2 = false;
  if ((r = check_formats(out, ckpt, nullptr, &e5m2)) != DS_OK) return r;
  const Span outs[] = {values_of("out", out), scales_of("out's scales", out), values_of("ckpt", ckpt),
                       scales_of("ckpt's scales", ckpt)};
  const Span ins[] = {span("gu", gu, strided(rows, width, ld, size))};
  if ((r = check_apart(outs, ins)) != DS_OK) return r;
  if (rows == 0) return DS_OK;
  return cuda_check(launch_gated_f8(gu, type, ld, rows, features, f8_out(out), f8_out(ckpt), e5m2,
                                    (flags & DS_F8_POW2) != 0, static_cast<cudaStream_t>(stream)),
                    "gated_f8 launch");
}

ds_status ds_gated_f8_backward(const ds_f8_matrix* ckpt, const void* da, int type, int64_t ld, int64_t features,
                               const ds_f8_matrix* dgu, const ds_f8_matrix* dgu_t, const ds_f8_matrix* a_t,
                               uint32_t flags, void* stream) {
  NvtxRange nvtx_range("ds_gated_f8_backward");
  clear_error();
  if (!ckpt) return fail(DS_ERR_INVALID_ARG, "NULL ckpt");
  if (!dgu && !dgu_t && !a_t) return fail(DS_ERR_INVALID_ARG, "no output is given");
  ds_status r = check_type(type);
  if (r != DS_OK) return r;
  if ((r = check_flags(flags)) != DS_OK) return r;
  if ((r = check_dims("da", ckpt->rows, features)) != DS_OK) return r;
  if (features == 0) return fail(DS_ERR_SHAPE, "a gate needs features");
  const int64_t rows = ckpt->rows, width = blocks_of(features) * kF8Block + features, size = type_size(type);
  if ((r = check_f8_out("ckpt", ckpt, rows, width, true)) != DS_OK) return r;
  if (!da && rows > 0) return fail(DS_ERR_INVALID_ARG, "NULL da");
  if ((r = check_tensor("da", da, rows, features, ld, size)) != DS_OK) return r;
  if ((r = check_f8_out("dgu", dgu, rows, width, true)) != DS_OK) return r;
  if ((r = check_f8_out("dgu_t", dgu_t, width, rows, true)) != DS_OK) return r;
  if ((r = check_f8_out("a_t", a_t, features, rows, true)) != DS_OK) return r;
  bool e5m2 = false;
  if ((r = check_formats(dgu, dgu_t, a_t, &e5m2)) != DS_OK) return r;
  const Span outs[] = {values_of("dgu", dgu),     scales_of("dgu's scales", dgu),
                       values_of("dgu_t", dgu_t), scales_of("dgu_t's scales", dgu_t),
                       values_of("a_t", a_t),     scales_of("a_t's scales", a_t)};
  const Span ins[] = {values_of("ckpt", ckpt), scales_of("ckpt's scales", ckpt),
                      span("da", da, strided(rows, features, ld, size))};
  if ((r = check_apart(outs, ins)) != DS_OK) return r;
  if (rows == 0) return DS_OK;
  if (blocks_of(rows) * blocks_of(features) > ((int64_t)1 << 31) - 1)
    return fail(DS_ERR_UNSUPPORTED, "matrix too large");
  return cuda_check(launch_gated_f8_backward(ckpt, da, type, ld, features, f8_out(dgu), f8_out(dgu_t), f8_out(a_t), e5m2,
                                             (flags & DS_F8_POW2) != 0, static_cast<cudaStream_t>(stream)),
                    "gated_f8_backward launch");
}

}  // extern "C"
