// Arithmetic of group normalisation's work split that needs no GPU: the host
// plans with it, the kernels use it, and a host compiler alone can check it.
#pragma once

#include <stdint.h>

#ifdef __HIPCC__
#define NSC_HD __host__ __device__ __forceinline__
#else
#define NSC_HD inline
#endif

namespace nsc {

// Of the ve values at position pos of step p, those that lie inside an image of
// hw pixels of c channels (none or less: the vector lies behind it).  A step is
// s pixels, and only the last of an image's steps can be ragged; an image may
// hold more than 2^31 values.
NSC_HD int values_inside(int32_t hw, int32_t c, int32_t s, int32_t steps, int32_t p, int32_t pos,
                         int32_t ve) {
  if (p + 1 < steps) return ve;
  const int64_t left = (int64_t)hw * c - ((int64_t)p * s * c + pos);
  return left < ve ? (int)left : ve;
}

}  // namespace nsc
