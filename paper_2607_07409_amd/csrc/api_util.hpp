// What the files of the C ABI share: the last-error message, argument helpers and the device check.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <cstring>

#include "../../include/dels.h"

namespace dls {
namespace abi {

void clear_error();
dls_status fail(dls_status s, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
dls_status hip_fail(hipError_t e, const char* what);
// a visible gfx950 device must be current; *cus: its CUs (0: no cooperative launch)
dls_status check_device(int* cus = nullptr);

inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }

// An enum from a C caller may hold any int; loading an out-of-range value as the C++ enum is
// undefined, so caller-supplied enums are read through their representation until validated.
template <typename E>
int enum_bits(const E& e) {
  static_assert(sizeof(E) == sizeof(int), "the C enums of the ABI are int-sized");
  int v;
  std::memcpy(&v, &e, sizeof v);
  return v;
}

inline bool valid_dtype(int t) { return t == DLS_F32 || t == DLS_BF16; }

}  // namespace abi
}  // namespace dls
