// Element types of the single layers (NSC_T_*): loading, rounding, vectors.
#pragma once

#include "nsc_internal.h"

namespace nsc {

#define NSC_REQUIRE_L(cond, code, ...)                  \
  do {                                                  \
    if (!(cond)) return ::nsc::fail(code, __VA_ARGS__); \
  } while (0)

inline int64_t type_bytes(int32_t dtype) { return dtype == NSC_T_F32 ? 4 : 2; }

// VE consecutive elements as one load or store.
template <typename T, int VE>
struct alignas(sizeof(T) * VE) Vec {
  T e[VE];
};

template <typename T, int VE>
__device__ __forceinline__ void to_f32(const Vec<T, VE>& v, float (&f)[VE]) {
#pragma unroll
  for (int i = 0; i < VE; ++i) f[i] = (float)v.e[i];
}
// Rounded to nearest even.
template <typename T, int VE>
__device__ __forceinline__ Vec<T, VE> from_f32(const float (&f)[VE]) {
  Vec<T, VE> v;
#pragma unroll
  for (int i = 0; i < VE; ++i) v.e[i] = (T)f[i];
  return v;
}

// The sum over a wave's lanes, in every lane.
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

}  // namespace nsc
