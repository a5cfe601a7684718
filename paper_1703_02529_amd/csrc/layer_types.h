// Element types of the single layers (NSC_T_*): loading, rounding, vectors.
#pragma once

#include "nsc_internal.h"

#include <type_traits>

namespace nsc {

#define NSC_REQUIRE_L(cond, code, ...)                  \
  do {                                                  \
    if (!(cond)) return ::nsc::fail(code, __VA_ARGS__); \
  } while (0)

// VE consecutive elements as one load or store.
template <typename T, int VE>
struct alignas(sizeof(T) * VE) Vec {
  T e[VE];
};

// The same held as 32-bit words (of a 16-bit type's elements, two registers
// fewer of every four), or as the element where it is smaller.
template <typename T, int VE>
struct Pack {
  static constexpr int kBytes = sizeof(T) * VE, kWords = kBytes >= 4 ? kBytes / 4 : 1;
  typedef typename std::conditional<kBytes >= 4, uint32_t, uint16_t>::type Word;
  struct alignas(kBytes) Words {
    Word w[kWords];
  } v;
  static __device__ __forceinline__ Pack load(const T* p) {
    return Pack{*reinterpret_cast<const Words*>(p)};
  }
  __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<Words*>(p) = v; }
  __device__ __forceinline__ void to_f32(float (&f)[VE]) const {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < VE; ++i) f[i] = __uint_as_float(v.w[i]);
    } else if constexpr (kBytes == 2) {
      f[0] = (float)__builtin_bit_cast(T, v.w[0]);
    } else if constexpr (std::is_same<T, __bf16>::value) {
#pragma unroll
      for (int i = 0; i < VE; i += 2) {
        f[i] = __uint_as_float(v.w[i / 2] << 16);
        f[i + 1] = __uint_as_float(v.w[i / 2] & 0xFFFF0000u);
      }
    } else {
      typedef T T2 __attribute__((ext_vector_type(2)));
#pragma unroll
      for (int i = 0; i < VE; i += 2) {
        const T2 t = __builtin_bit_cast(T2, v.w[i / 2]);
        f[i] = (float)t[0];
        f[i + 1] = (float)t[1];
      }
    }
  }
  // Rounded to nearest even.
  static __device__ __forceinline__ Pack from_f32(const float (&f)[VE]) {
    Pack p;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < VE; ++i) p.v.w[i] = __float_as_uint(f[i]);
    } else if constexpr (kBytes == 2) {
      p.v.w[0] = __builtin_bit_cast(uint16_t, (T)f[0]);
    } else {
      typedef T T2 __attribute__((ext_vector_type(2)));
#pragma unroll
      for (int i = 0; i < VE; i += 2)
        p.v.w[i / 2] = __builtin_bit_cast(uint32_t, T2{(T)f[i], (T)f[i + 1]});
    }
    return p;
  }
  __device__ __forceinline__ void set(int i, T x) {
    if constexpr (sizeof(T) == 4) {
      v.w[i] = __builtin_bit_cast(uint32_t, x);
    } else if constexpr (kBytes == 2) {
      v.w[0] = __builtin_bit_cast(uint16_t, x);
    } else {
      const uint32_t b = __builtin_bit_cast(uint16_t, x);
      v.w[i / 2] = i & 1 ? (v.w[i / 2] & 0xFFFFu) | b << 16 : (v.w[i / 2] & 0xFFFF0000u) | b;
    }
  }
  // Makes the compiler take the values as new here, so that what was derived
  // from them before is derived again instead of being kept in registers, and
  // packs that are processed one after another stay so.
  __device__ __forceinline__ void renew() {
    if constexpr (kBytes >= 4) {
#pragma unroll
      for (int i = 0; i < kWords; ++i) asm volatile("" : "+v"(v.w[i]));
    }
  }
};

// Has loaded values arrive here.  (A store of a path that may or may not be
// taken lies between a load and a use otherwise, and the compiler waits for the
// store there: one by one.)
template <int N>
__device__ __forceinline__ void arrive(float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+v"(v[i]));
}

// The sum over a wave's lanes, in every lane.
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

}  // namespace nsc
