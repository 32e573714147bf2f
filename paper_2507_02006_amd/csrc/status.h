// Status and last-error text shared by the entry points of this library.
#pragma once
#include "../../include/aires.h"

namespace aires {

// Stores the text of the calling thread's last error and returns s.
aires_status fail(aires_status s, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

}  // namespace aires

#define HIP_TRY(expr)                                                                 \
  do {                                                                                \
    hipError_t e_ = (expr);                                                           \
    if (e_ != hipSuccess)                                                             \
      return aires::fail(AIRES_E_HIP, "%s failed: %s", #expr, hipGetErrorString(e_)); \
  } while (0)

#define ST_TRY(expr)                       \
  do {                                     \
    aires_status s_ = (expr);              \
    if (s_ != AIRES_OK) return s_;         \
  } while (0)
