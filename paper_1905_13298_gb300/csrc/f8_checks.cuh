// Checks of arguments that the entry points of the 8-bit and the experts' operators share.
#pragma once

#include <initializer_list>

#include "f8_common.cuh"

namespace ds {

constexpr int64_t kMaxDim = ((int64_t)1 << 31) - 256;
constexpr int64_t kMaxBytes = (int64_t)1 << 48;

inline int64_t blocks_of(int64_t n) { return (n + kF8Block - 1) / kF8Block; }
inline int64_t type_size(int type) { return type == DS_TYPE_F32 ? 4 : 2; }
inline bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

inline ds_status check_type(int type) {
  if (type != DS_TYPE_F32 && type != DS_TYPE_BF16 && type != DS_TYPE_F16)
    return fail(DS_ERR_INVALID_ARG, "unknown type %d", type);
  return DS_OK;
}
inline ds_status check_flags(uint32_t flags) {
  if (flags & ~DS_F8_POW2) return fail(DS_ERR_INVALID_ARG, "only DS_F8_POW2 applies");
  return DS_OK;
}

// Device memory that a call reads or writes.
struct Span {
  const char* name;
  uintptr_t at;
  int64_t bytes;
};
inline Span span(const char* name, const void* p, int64_t bytes) {
  return Span{name, reinterpret_cast<uintptr_t>(p), p ? bytes : 0};
}
inline int64_t strided(int64_t rows, int64_t cols, int64_t ld, int64_t size) {
  return rows > 0 && cols > 0 ? ((rows - 1) * ld + cols) * size : 0;
}
inline Span values_of(const char* name, const ds_f8_matrix* m) {
  return m ? span(name, m->q, strided(m->rows, m->cols, m->ld, 1)) : span(name, nullptr, 0);
}
inline Span scales_of(const char* name, const ds_f8_matrix* m) {
  if (!m) return span(name, nullptr, 0);
  const int64_t r = m->blocks == DS_F8_TILES ? blocks_of(m->rows) : m->rows;
  return span(name, m->scale, strided(r, blocks_of(m->cols), m->ld_scale, 4));
}
inline bool overlap(const Span& a, const Span& b) {
  return a.bytes > 0 && b.bytes > 0 && a.at < b.at + (uintptr_t)b.bytes && b.at < a.at + (uintptr_t)a.bytes;
}
template <int NOUT, int NIN>
inline ds_status check_apart(const Span (&outs)[NOUT], const Span (&ins)[NIN]) {
  for (int i = 0; i < NOUT; ++i) {
    for (int j = 0; j < NIN; ++j)
      if (overlap(outs[i], ins[j])) return fail(DS_ERR_INVALID_ARG, "%s overlaps %s", outs[i].name, ins[j].name);
    for (int j = 0; j < i; ++j)
      if (overlap(outs[i], outs[j])) return fail(DS_ERR_INVALID_ARG, "%s overlaps %s", outs[i].name, outs[j].name);
  }
  return DS_OK;
}

inline ds_status check_dims(const char* name, int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 0) return fail(DS_ERR_SHAPE, "%s: rows and cols must not be negative", name);
  if (rows > kMaxDim || cols > kMaxDim) return fail(DS_ERR_UNSUPPORTED, "%s: rows or cols too large", name);
  return DS_OK;
}

inline ds_status check_f8(const char* name, const ds_f8_matrix* m) {
  ds_status r = check_dims(name, m->rows, m->cols);
  if (r != DS_OK) return r;
  if (m->format != DS_F8_E4M3 && m->format != DS_F8_E5M2)
    return fail(DS_ERR_INVALID_ARG, "%s: unknown 8-bit format %d", name, (int)m->format);
  if (m->blocks != DS_F8_ROWS && m->blocks != DS_F8_TILES)
    return fail(DS_ERR_INVALID_ARG, "%s: unknown blocks %d", name, (int)m->blocks);
  if (m->ld < m->cols || m->ld_scale < blocks_of(m->cols))
    return fail(DS_ERR_SHAPE, "%s: a row stride is shorter than a row", name);
  if (m->ld % 16 != 0) return fail(DS_ERR_ALIGNMENT, "%s: ld must be a multiple of 16", name);
  if (m->ld > ((int64_t)1 << 36) || m->ld_scale > ((int64_t)1 << 36) || m->rows * (m->ld / 16) > kMaxBytes / 16)
    return fail(DS_ERR_UNSUPPORTED, "%s: too large", name);
  if (m->rows > 0 && m->cols > 0) {
    if (!m->q || !m->scale) return fail(DS_ERR_INVALID_ARG, "%s: NULL pointer", name);
    if (!aligned(m->q, 16)) return fail(DS_ERR_ALIGNMENT, "%s: q must be 16-byte aligned", name);
    if (!aligned(m->scale, 4)) return fail(DS_ERR_ALIGNMENT, "%s: scale must be 4-byte aligned", name);
  }
  return DS_OK;
}

// An 8-bit output of the given shape (NULL: none).
inline ds_status check_f8_out(const char* name, const ds_f8_matrix* m, int64_t rows, int64_t cols, bool rows_only) {
  if (!m) return DS_OK;
  ds_status r = check_f8(name, m);
  if (r != DS_OK) return r;
  if (m->rows != rows || m->cols != cols)
    return fail(DS_ERR_SHAPE, "%s is %lld x %lld, not %lld x %lld", name, (long long)m->rows, (long long)m->cols,
                (long long)rows, (long long)cols);
  if (rows_only && m->blocks != DS_F8_ROWS) return fail(DS_ERR_INVALID_ARG, "%s must have DS_F8_ROWS blocks", name);
  return DS_OK;
}

// A [rows][cols] tensor aligned to `to` bytes with row stride ld (NULL passes; no elements: the pointer is not used).
inline ds_status check_tensor(const char* name, const void* p, int64_t rows, int64_t cols, int64_t ld, int64_t to) {
  if (!p) return DS_OK;
  if (ld < cols) return fail(DS_ERR_SHAPE, "%s: the row stride is shorter than a row", name);
  if (ld > ((int64_t)1 << 40) || (rows > 0 && ld > kMaxBytes / rows))
    return fail(DS_ERR_UNSUPPORTED, "%s: too large", name);
  if (!aligned(p, to)) return fail(DS_ERR_ALIGNMENT, "%s must be %d-byte aligned", name, (int)to);
  return DS_OK;
}

// An aliased output starts where its input does, with the same stride; anything else is an overlap.
inline bool same(const void* a, int64_t lda, const void* b, int64_t ldb) { return a != nullptr && a == b && lda == ldb; }

}  // namespace ds
