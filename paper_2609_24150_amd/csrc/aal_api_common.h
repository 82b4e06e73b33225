// Argument checks and error reporting shared by the files of the C-ABI layer.
#pragma once

#include "aal.h"
#include "aal_internal.h"

#include <stdarg.h>
#include <stdio.h>
#include <string.h>

namespace aal {

// The calling thread's error text behind aal_last_error() (defined in aal_api.hip).
char* error_text();
constexpr size_t kErrorTextBytes = 512;

}  // namespace aal

namespace {

inline void clear_error() { aal::error_text()[0] = '\0'; }

inline aal_status_t fail(aal_status_t s, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(aal::error_text(), aal::kErrorTextBytes, fmt, ap);
  va_end(ap);
  return s;
}

// Finite and > 0, checked on the bit pattern so that no floating-point
// compilation mode can fold the test away.
inline bool positive_finite(float x) {
  uint32_t u;
  memcpy(&u, &x, sizeof u);
  const bool sign = (u >> 31) != 0;
  const uint32_t expo = (u >> 23) & 0xffu;
  return !sign && expo != 0xffu && (u & 0x7fffffffu) != 0;
}

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// The integer held by an enum argument, read without loading it as the enum
// type: a C caller may pass any int, and values outside the enumerators are
// validated here rather than assumed away.
template <class E>
inline int raw(const E& e) {
  static_assert(sizeof(E) == sizeof(int), "enum arguments are int-sized");
  int v;
  memcpy(&v, &e, sizeof v);
  return v;
}

inline bool valid_dtype(int d) { return d == AAL_BF16 || d == AAL_F32; }

inline aal::DType to_dtype(int d) { return d == AAL_BF16 ? aal::DType::kBf16 : aal::DType::kF32; }

constexpr double kLog2e = 1.4426950408889634073599246810019;

// log2(e)/T as a finite positive float, or 0 if it is not representable.
inline float scale_for(float T) {
  const double s = kLog2e / double(T);
  if (!(s < 3.0e38)) return 0.f;
  const float f = float(s);
  return positive_finite(f) ? f : 0.f;
}

}  // namespace
