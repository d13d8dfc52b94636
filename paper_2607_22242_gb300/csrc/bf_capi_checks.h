// bf_capi_checks.h -- checks of arguments that the learning and the answering
// entry points share.  Each records its failure and returns BF_EINVAL, or BF_OK.
#pragma once

#include <cmath>

#include "bf_capi_internal.h"

namespace bfcapi {

constexpr uint64_t kMaxRows = 0x7FFFFFFFull;
constexpr uint64_t kMaxCols = 1ull << 30;

inline uint64_t align256(uint64_t x) { return (x + 255) / 256 * 256; }

inline uint32_t size_of(uint32_t dtype) { return dtype == BF_F32 ? 4u : 2u; }

inline bool aligned(const void* p, size_t to) { return (uintptr_t)p % to == 0; }

// A matrix argument; `rows` may be 0 with any data pointer.
inline int check_matrix(const bf_matrix* m, const char* name, const char* who) {
  if (!m) return fail(BF_EINVAL, "%s: %s is NULL", who, name);
  if (m->dtype > BF_F16) return fail(BF_EINVAL, "%s: %s has the unknown type %u", who, name, m->dtype);
  if (m->rows > kMaxRows) return fail(BF_EINVAL, "%s: %s has more than 2^31 - 1 rows", who, name);
  if (m->cols == 0 || m->cols > kMaxCols) return fail(BF_EINVAL, "%s: %s needs 1 to 2^30 columns", who, name);
  if (m->row_stride < m->cols || m->row_stride > (1ull << 40) / (m->rows ? m->rows : 1))
    return fail(BF_EINVAL, "%s: the row stride of %s is below its columns or beyond 2^40 elements in all", who, name);
  if (m->rows && !m->data) return fail(BF_EINVAL, "%s: %s has no data", who, name);
  if (!aligned(m->data, size_of(m->dtype))) return fail(BF_EINVAL, "%s: %s is not aligned to its type", who, name);
  return BF_OK;
}

// An array argument that calls with `count` elements read or write.
inline int check_array(const void* p, uint64_t count, size_t size, const char* name, const char* who) {
  if (count && !p) return fail(BF_EINVAL, "%s: %s is NULL", who, name);
  if (!aligned(p, size)) return fail(BF_EINVAL, "%s: %s is not aligned to its type", who, name);
  return BF_OK;
}

inline uint64_t extent(const bf_matrix* m) { return m->rows ? ((m->rows - 1) * m->row_stride + m->cols) * size_of(m->dtype) : 0; }

inline bool overlap(const bf_matrix* a, const bf_matrix* b) {
  const uintptr_t x = (uintptr_t)a->data, y = (uintptr_t)b->data;
  return x < y + extent(b) && y < x + extent(a);
}

inline int check_number(float v, bool ok, const char* name, const char* who) {
  return std::isfinite(v) && ok ? BF_OK : fail(BF_EINVAL, "%s: %s = %g is out of its range", who, name, (double)v);
}

// A temperature whose reciprocals, in two parts, are normal 32-bit numbers.
inline int check_temperature(float v, const char* who) { return check_number(v, v >= 1e-18f && v <= 1e18f, "temperature", who); }

#define BF_TRY(call)                         \
  do {                                       \
    if ((call) != BF_OK) return BF_EINVAL;   \
  } while (0)

inline int check_workspace(const void* workspace, uint64_t have, uint64_t need, const char* who) {
  if (!workspace || !aligned(workspace, 256))
    return fail(BF_EINVAL, "%s: the workspace is NULL or not aligned to 256 bytes", who);
  if (have < need)
    return fail(BF_EINVAL, "%s: the workspace has %llu bytes and %llu are needed", who, (unsigned long long)have,
                (unsigned long long)need);
  return BF_OK;
}

}  // namespace bfcapi
