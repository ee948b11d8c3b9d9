// The host side's check that what a call writes lies in no other array of it, shared by its sources.
#pragma once

#include <cstddef>
#include <cstdint>

#include "status.h"

namespace caddtree {

// An array of a call and whether the call writes it.  What is written must lie in no other array: the kernels of a call
// read and write in no fixed order.
struct Array {
  const char* name;
  const void* data;
  size_t bytes;              // (of sizes within the limits: below 2^64)
  bool written;
};
template <size_t n>
caddtree_status_t check_apart(const Array (&all)[n]) {
  for (size_t i = 0; i < n; ++i)
    for (size_t j = i + 1; j < n; ++j) {
      const Array &x = all[i], &y = all[j];
      const uintptr_t px = reinterpret_cast<uintptr_t>(x.data), py = reinterpret_cast<uintptr_t>(y.data);
      if ((x.written || y.written) && x.bytes > 0 && y.bytes > 0 && (px <= py ? py - px < x.bytes : px - py < y.bytes))
        return fail(CADDTREE_E_INVALID, "%s and %s overlap", x.name, y.name);
    }
  return CADDTREE_OK;
}

}  // namespace caddtree
