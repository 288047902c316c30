// C ABI entry points of the experts' operators: argument validation, then
// stream-ordered launches.  Nothing is launched and no output is written when
// validation fails.
#include "experts.cuh"

namespace ds {
namespace {

constexpr int kMaxAlign = 1 << 20;

int64_t rows_of(int64_t tokens, int32_t top_k, int32_t experts, int32_t align) {
  if (tokens < 0 || top_k < 1 || experts < 1 || experts > DS_EXPERTS_MAX || align < 1 || align > kMaxAlign) return -1;
  if (tokens > kMaxDim / top_k) return -1;
  const int64_t slots = tokens * top_k, some = slots < experts ? slots : experts;
  const int64_t rows = (slots + some * (align - 1)) / align * align;
  return rows > kMaxDim ? -1 : rows;
}

ds_status check_slots(const ds_expert_slots* s) {
  if (!s) return fail(DS_ERR_INVALID_ARG, "NULL slots");
  if (s->tokens < 0 || s->top_k < 1 || s->experts < 1 || s->align < 1 || s->rows < 0)
    return fail(DS_ERR_SHAPE, "tokens and rows must not be negative, top_k, experts and align at least 1");
  const int64_t need = rows_of(s->tokens, s->top_k, s->experts, s->align);
  if (need < 0 || s->rows > kMaxDim) return fail(DS_ERR_UNSUPPORTED, "too many experts, tokens or rows, or align too large");
  if (s->rows < need)
    return fail(DS_ERR_BUFFER_TOO_SMALL, "slots have %lld rows, %lld are needed", (long long)s->rows, (long long)need);
  if (!s->offsets || !s->counts || (s->tokens > 0 && !s->position) || (s->rows > 0 && !s->slot))
    return fail(DS_ERR_INVALID_ARG, "NULL pointer in the slots");
  if (!aligned(s->offsets, 4) || !aligned(s->counts, 4) || !aligned(s->position, 4) || !aligned(s->slot, 4))
    return fail(DS_ERR_ALIGNMENT, "the slots' memory must be 4-byte aligned");
  return DS_OK;
}

// What a call reads of the slots, or writes.
Span offsets_of(const ds_expert_slots* s) { return span("offsets", s->offsets, 4 * ((int64_t)s->experts + 1)); }
Span counts_of(const ds_expert_slots* s) { return span("counts", s->counts, 4 * (int64_t)s->experts); }
Span position_of(const ds_expert_slots* s) { return span("position", s->position, 4 * s->tokens * s->top_k); }
Span slot_of(const ds_expert_slots* s) { return span("slot", s->slot, 4 * s->rows); }

ds_status check_f8_rows(const char* name, const ds_f8_matrix* m, int64_t rows, int64_t cols) {
  if (!m) return fail(DS_ERR_INVALID_ARG, "NULL %s", name);
  return check_f8_out(name, m, rows, cols, true);
}

// Warps of a launch stay inside a grid's 2^31 - 1 CTAs.
ds_status check_size(const ds_expert_slots* s, int64_t cols) {
  if ((s->tokens + s->rows) > ((int64_t)1 << 34) / (cols / 64 + 1)) return fail(DS_ERR_UNSUPPORTED, "rows x cols too large");
  return DS_OK;
}

}  // namespace
}  // namespace ds

using namespace ds;

extern "C" {

int64_t ds_expert_rows(int64_t tokens, int32_t top_k, int32_t experts, int32_t align) {
  return rows_of(tokens, top_k, experts, align);
}

ds_status ds_expert_order(const void* ids, int id_type, const ds_expert_slots* s, void* stream) {
  NvtxRange nvtx_range("ds_expert_order");
  clear_error();
  ds_status r = check_slots(s);
  if (r != DS_OK) return r;
  if (id_type != DS_INDEX_I32 && id_type != DS_INDEX_I64) return fail(DS_ERR_INVALID_ARG, "unknown index type %d", id_type);
  if (!ids && s->tokens > 0) return fail(DS_ERR_INVALID_ARG, "NULL ids");
  const int64_t size = id_type == DS_INDEX_I64 ? 8 : 4;
  if (!aligned(ids, size)) return fail(DS_ERR_ALIGNMENT, "ids must be %d-byte aligned", (int)size);
  const Span outs[] = {offsets_of(s), counts_of(s), position_of(s), slot_of(s)};
  const Span ins[] = {span("ids", ids, size * s->tokens * s->top_k)};
  if ((r = check_apart(outs, ins)) != DS_OK) return r;
  return cuda_check(launch_expert_order(ids, id_type, *s, static_cast<cudaStream_t>(stream)), "expert_order launch");
}

ds_status ds_expert_gather(const void* x, int type, int64_t ldx, int64_t cols, const ds_expert_slots* s, void* out,
                           int64_t ldo, void* stream) {
  NvtxRange nvtx_range("ds_expert_gather");
  clear_error();
  ds_status r = check_slots(s);
  if (r != DS_OK) return r;
  if ((r = check_type(type)) != DS_OK) return r;
  if ((r = check_dims("x", s->tokens, cols)) != DS_OK) return r;
  if ((r = check_size(s, cols)) != DS_OK) return r;
  if (cols > 0 && ((!x && s->tokens > 0) || (!out && s->rows > 0))) return fail(DS_ERR_INVALID_ARG, "NULL x or out");
  const int64_t size = type_size(type);
  if ((r = check_tensor("x", x, s->tokens, cols, ldx, size)) != DS_OK) return r;
  if ((r = check_tensor("out", out, s->rows, cols, ldo, size)) != DS_OK) return r;
  const Span outs[] = {span("out", out, strided(s->rows, cols, ldo, size))};
  const Span ins[] = {span("x", x, strided(s->tokens, cols, ldx, size)), position_of(s), slot_of(s)};
  if ((r = check_apart(outs, ins)) != DS_OK) return r;
  if (cols == 0 || s->rows == 0) return DS_OK;
  const RowCopy a{x, out, ldx * size, ldo * size, cols * size};
  return cuda_check(launch_expert_gather(a, RowCopy{}, *s, static_cast<cudaStream_t>(stream)), "expert_gather launch");
}

ds_status ds_expert_gather_f8(const ds_f8_matrix* x, const ds_expert_slots* s, const ds_f8_matrix* out, void* stream) {
  NvtxRange nvtx_range("ds_expert_gather_f8");
  clear_error();
  ds_status r = check_slots(s);
  if (r != DS_OK) return r;
  if (!x || !out) return fail(DS_ERR_INVALID_ARG, "NULL x or out");
  if ((r = check_f8_rows("x", x, s->tokens, x->cols)) != DS_OK) return r;
  if ((r = check_f8_rows("out", out, s->rows, x->cols)) != DS_OK) return r;
  if (x->format != out->format) return fail(DS_ERR_INVALID_ARG, "x and out have different 8-bit formats");
  if ((r = check_size(s, x->cols)) != DS_OK) return r;
  const Span outs[] = {values_of("out", out), scales_of("out's scales", out)};
  const Span ins[] = {values_of("x", x), scales_of("x's scales", x), position_of(s), slot_of(s)};
  if ((r = check_apart(outs, ins)) != DS_OK) return r;
  if (x->cols == 0 || s->rows == 0) return DS_OK;
  const RowCopy a{x->q, out->q, x->ld, out->ld, x->cols};
  const RowCopy b{x->scale, out->scale, 4 * x->ld_scale, 4 * out->ld_scale, 4 * blocks_of(x->cols)};
  return cuda_check(launch_expert_gather(a, b, *s, static_cast<cudaStream_t>(stream)), "expert_gather_f8 launch");
}

ds_status ds_expert_combine(const void* y, int type, int64_t ldy, int64_t cols, const ds_expert_slots* s,
                            const float* weights, const void* add, int64_t ld_add, void* out, int64_t ldo,
                            void* stream) {
  NvtxRange nvtx_range("ds_expert_combine");
  clear_error();
  ds_status r = check_slots(s);
  if (r != DS_OK) return r;
  if ((r = check_type(type)) != DS_OK) return r;
  if ((r = check_dims("y", s->rows, cols)) != DS_OK) return r;
  if ((r = check_size(s, cols)) != DS_OK) return r;
  if (cols > 0 && s->tokens > 0 && (!y || !out)) return fail(DS_ERR_INVALID_ARG, "NULL y or out");
  const int64_t size = type_size(type), slots = s->tokens * s->top_k;
  if ((r = check_tensor("y", y, s->rows, cols, ldy, size)) != DS_OK) return r;
  if ((r = check_tensor("add", add, s->tokens, cols, ld_add, size)) != DS_OK) return r;
  if ((r = check_tensor("out", out, s->tokens, cols, ldo, size)) != DS_OK) return r;
  if ((r = check_tensor("weights", weights, 1, slots, slots, 4)) != DS_OK) return r;
  const Span outs[] = {span("out", out, strided(s->tokens, cols, ldo, size))};
  const Span ins[] = {span("y", y, strided(s->rows, cols, ldy, size)), span("weights", weights, 4 * slots),
                      span("add", same(out, ldo, add, ld_add) ? nullptr : add, strided(s->tokens, cols, ld_add, size)),
                      position_of(s)};
  if ((r = check_apart(outs, ins)) != DS_OK) return r;
  if (cols == 0 || s->tokens == 0) return DS_OK;
  return cuda_check(launch_expert_combine(y, type, ldy, cols, *s, weights, add, ld_add, out, ldo,
                                          static_cast<cudaStream_t>(stream)),
                    "expert_combine launch");
}

ds_status ds_expert_combine_backward(const void* dout, int64_t ldd, const void* y, int64_t ldy, int type, int64_t cols,
                                     const ds_expert_slots* s, const float* weights, void* dy, int64_t lddy,
                                     float* dweights, void* stream) {
  NvtxRange nvtx_range("ds_expert_combine_backward");
  clear_error();
  ds_status r = check_slots(s);
  if (r != DS_OK) return r;
  if ((r = check_type(type)) != DS_OK) return r;
  if ((r = check_dims("dy", s->rows, cols)) != DS_OK) return r;
  if (cols == 0) return fail(DS_ERR_SHAPE, "a gradient needs columns");
  if ((r = check_size(s, cols)) != DS_OK) return r;
  if ((!dout && s->tokens > 0) || (!dy && s->rows > 0) || (dweights && !y && s->rows > 0))
    return fail(DS_ERR_INVALID_ARG, "NULL dout, dy or y");
  const int64_t size = type_size(type), slots = s->tokens * s->top_k;
  if (!dweights) y = nullptr;
  if ((r = check_tensor("dout", dout, s->tokens, cols, ldd, size)) != DS_OK) return r;
  if ((r = check_tensor("y", y, s->rows, cols, ldy, size)) != DS_OK) return r;
  if ((r = check_tensor("dy", dy, s->rows, cols, lddy, size)) != DS_OK) return r;
  if ((r = check_tensor("weights", weights, 1, slots, slots, 4)) != DS_OK) return r;
  if ((r = check_tensor("dweights", dweights, 1, slots, slots, 4)) != DS_OK) return r;
  const Span outs[] = {span("dy", dy, strided(s->rows, cols, lddy, size)), span("dweights", dweights, 4 * slots)};
  const Span ins[] = {span("dout", dout, strided(s->tokens, cols, ldd, size)),
                      span("y", same(dy, lddy, y, ldy) ? nullptr : y, strided(s->rows, cols, ldy, size)),
                      span("weights", weights, 4 * slots), position_of(s), slot_of(s)};
  if ((r = check_apart(outs, ins)) != DS_OK) return r;
  if (s->tokens == 0 && s->rows == 0) return DS_OK;
  return cuda_check(launch_expert_combine_backward(dout, ldd, y, ldy, type, cols, *s, weights, dy, lddy, dweights,
                                                   static_cast<cudaStream_t>(stream)),
                    "expert_combine_backward launch");
}

ds_status ds_expert_linear_f8(const ds_f8_matrix* x, const ds_f8_matrix* w, const ds_expert_slots* s, const float* bias,
                              void* y, int type, int64_t ldy, void* stream) {
  NvtxRange nvtx_range("ds_expert_linear_f8");
  clear_error();
  ds_status r = check_slots(s);
  if (r != DS_OK) return r;
  if (!x || !w) return fail(DS_ERR_INVALID_ARG, "NULL x or w");
  if ((r = check_type(type)) != DS_OK) return r;
  if ((r = check_f8("x", x)) != DS_OK) return r;
  if ((r = check_f8("w", w)) != DS_OK) return r;
  if (x->rows != s->rows) return fail(DS_ERR_SHAPE, "x has %lld rows, the slots %lld", (long long)x->rows, (long long)s->rows);
  if (x->cols != w->cols) return fail(DS_ERR_SHAPE, "x has %lld columns, w %lld", (long long)x->cols, (long long)w->cols);
  if (w->rows % s->experts != 0)
    return fail(DS_ERR_SHAPE, "w has %lld rows, not a multiple of the %d experts", (long long)w->rows, s->experts);
  const int64_t n = w->rows / s->experts, size = type_size(type);
  if (w->blocks == DS_F8_TILES && n % kF8Block != 0)
    return fail(DS_ERR_SHAPE, "an expert has %lld rows of w, which has tiles: not a multiple of 128", (long long)n);
  if (x->blocks == DS_F8_TILES && s->align % kF8Block != 0)
    return fail(DS_ERR_SHAPE, "x has tiles, and align is not a multiple of 128");
  if (!y && s->rows > 0 && n > 0) return fail(DS_ERR_INVALID_ARG, "NULL y");
  if ((r = check_tensor("y", y, s->rows, n, ldy, size)) != DS_OK) return r;
  if ((r = check_tensor("bias", bias, s->experts, n, n, 4)) != DS_OK) return r;
  const Span outs[] = {span("y", y, strided(s->rows, n, ldy, size))};
  const Span ins[] = {values_of("x", x), scales_of("x's scales", x), values_of("w", w), scales_of("w's scales", w),
                      span("bias", bias, 4 * w->rows), offsets_of(s)};
  if ((r = check_apart(outs, ins)) != DS_OK) return r;
  if (blocks_of(n) * ((s->rows + 15) / 16 + s->experts) > ((int64_t)1 << 28) - 1)
    return fail(DS_ERR_UNSUPPORTED, "rows x N too large");
  if (s->rows == 0 || n == 0) return DS_OK;
  const ExpertProduct p{x, w, s, bias, nullptr, 0, y, type, ldy};
  return cuda_check(launch_expert_linear_f8(p, static_cast<cudaStream_t>(stream)), "expert_linear_f8 launch");
}

ds_status ds_expert_weight_grad_f8(const ds_f8_matrix* dy_t, const ds_f8_matrix* x_t, const ds_expert_slots* s,
                                   const float* add, int64_t ld_add, float* dw, int64_t lddw, void* stream) {
  NvtxRange nvtx_range("ds_expert_weight_grad_f8");
  clear_error();
  ds_status r = check_slots(s);
  if (r != DS_OK) return r;
  if (!dy_t || !x_t) return fail(DS_ERR_INVALID_ARG, "NULL dy_t or x_t");
  if ((r = check_f8("dy_t", dy_t)) != DS_OK) return r;
  if ((r = check_f8("x_t", x_t)) != DS_OK) return r;
  if (dy_t->cols != s->rows || x_t->cols != s->rows)
    return fail(DS_ERR_SHAPE, "dy_t has %lld columns, x_t %lld, the slots %lld rows", (long long)dy_t->cols,
                (long long)x_t->cols, (long long)s->rows);
  if (s->align % kF8Block != 0) return fail(DS_ERR_SHAPE, "align is not a multiple of 128");
  const int64_t n = dy_t->rows, k = x_t->rows, experts = s->experts;
  if (n > kMaxDim / experts) return fail(DS_ERR_UNSUPPORTED, "dw: too many rows");
  if (!dw && n > 0 && k > 0) return fail(DS_ERR_INVALID_ARG, "NULL dw");
  if ((r = check_tensor("dw", dw, experts * n, k, lddw, 4)) != DS_OK) return r;
  if ((r = check_tensor("add", add, experts * n, k, ld_add, 4)) != DS_OK) return r;
  const Span outs[] = {span("dw", dw, strided(experts * n, k, lddw, 4))};
  const Span ins[] = {values_of("dy_t", dy_t), scales_of("dy_t's scales", dy_t), values_of("x_t", x_t),
                      scales_of("x_t's scales", x_t),
                      span("add", same(dw, lddw, add, ld_add) ? nullptr : add, strided(experts * n, k, ld_add, 4)),
                      offsets_of(s)};
  if ((r = check_apart(outs, ins)) != DS_OK) return r;
  if (experts * blocks_of(n) * blocks_of(k) > ((int64_t)1 << 31) - 1) return fail(DS_ERR_UNSUPPORTED, "N x K too large");
  if (n == 0 || k == 0) return DS_OK;
  const ExpertProduct p{x_t, dy_t, s, nullptr, add, ld_add, dw, DS_TYPE_F32, lddw};
  return cuda_check(launch_expert_weight_grad_f8(p, static_cast<cudaStream_t>(stream)), "expert_weight_grad_f8 launch");
}

}  // extern "C"
