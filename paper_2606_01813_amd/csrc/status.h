// The host side's status and message of a call (caddtree_last_error), shared by its sources.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstdarg>
#include <cstdio>
#include <cstring>

#include "caddtree.h"

namespace caddtree {

inline thread_local char g_last_error[512];   // (a string could throw out of a C function)

caddtree_status_t fail(caddtree_status_t st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
inline caddtree_status_t fail(caddtree_status_t st, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_last_error, sizeof(g_last_error), fmt, ap);
  va_end(ap);
  return st;
}

inline caddtree_status_t ok() {
  g_last_error[0] = '\0';
  return CADDTREE_OK;
}

inline caddtree_status_t hip_fail(hipError_t e, const char* what) {
  return fail(CADDTREE_E_HIP, "%s: %s (%d)", what, hipGetErrorString(e), (int)e);
}

// The value a C caller stored in an enum-typed field or argument, read as the int it is: a C
// caller may pass any int there, which a C++ enum object must not hold.
template <typename E>
int enum_value(const E& e) {
  static_assert(sizeof(E) == sizeof(int), "the C enums of the interface are int-sized");
  int v;
  std::memcpy(&v, &e, sizeof v);
  return v;
}

}  // namespace caddtree
