// Sizes of the machine and arithmetic that plans share; needs no GPU headers, so
// that a host compiler alone can check what is planned with it.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "nsc.h"

namespace nsc {

constexpr int kNumCU = 256;  // MI355X compute units (8 XCDs x 32)
constexpr int kNumXCD = 8;

inline int64_t gcd64(int64_t a, int64_t b) {
  while (b) {
    int64_t t = a % b;
    a = b;
    b = t;
  }
  return a;
}

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

// Bytes of an element of the single layers' tensors (NSC_T_*).
inline int64_t type_bytes(int32_t dtype) { return dtype == NSC_T_F32 ? 4 : 2; }

}  // namespace nsc
