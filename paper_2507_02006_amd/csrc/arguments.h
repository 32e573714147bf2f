// Checks of dense matrix arguments, shared by the entry points.
#pragma once
#include "status.h"
#include "train.h"

namespace aires {
namespace {

inline bool type_ok(int32_t t) { return t == AIRES_F32 || t == AIRES_BF16 || t == AIRES_F16; }

[[maybe_unused]] aires_status check_dense(const aires_dense* m, const char* name) {
  if (!m) return fail(AIRES_E_INVALID_ARG, "%s is NULL", name);
  if (!type_ok(m->dtype)) return fail(AIRES_E_INVALID_ARG, "%s: type %d invalid", name, (int)m->dtype);
  if (m->nrows < 0 || m->ncols < 0)
    return fail(AIRES_E_DIM, "%s is %lld x %lld", name, (long long)m->nrows, (long long)m->ncols);
  if (m->nrows > 0 && m->ncols > 0) {
    if (!m->data) return fail(AIRES_E_INVALID_ARG, "%s has no data", name);
    if (m->ld < m->ncols)
      return fail(AIRES_E_INVALID_ARG, "%s: ld %lld below %lld columns", name, (long long)m->ld, (long long)m->ncols);
  }
  return AIRES_OK;
}

[[maybe_unused]] aires_status check_same(const aires_dense* a, const char* an, const aires_dense* b, const char* bn) {
  if (a->nrows != b->nrows || a->ncols != b->ncols)
    return fail(AIRES_E_DIM, "%s is %lld x %lld, %s %lld x %lld", an, (long long)a->nrows, (long long)a->ncols, bn,
                (long long)b->nrows, (long long)b->ncols);
  return AIRES_OK;
}

[[maybe_unused]] kern::Mat mat(const aires_dense* m) {
  if (!m) return kern::Mat{nullptr, 0, 0, 0, 0};
  return kern::Mat{m->data, m->nrows, m->ncols, m->ld, m->dtype};
}

}  // namespace
}  // namespace aires
