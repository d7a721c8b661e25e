// The two 16-bit float types of a KV pool and their 32-bit conversions
// (to nearest, ties to even), eight elements (16 B) at a time.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mori {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

struct F16 {
  typedef _Float16 scalar;
  typedef _Float16 x8 __attribute__((ext_vector_type(8)));
  typedef _Float16 x2 __attribute__((ext_vector_type(2)));
};
struct BF16 {
  typedef __bf16 scalar;
  typedef __bf16 x8 __attribute__((ext_vector_type(8)));
  typedef __bf16 x2 __attribute__((ext_vector_type(2)));
};

template <typename To, typename From>
__device__ inline To bits(From v) {
  static_assert(sizeof(To) == sizeof(From), "same size");
  return __builtin_bit_cast(To, v);
}

template <typename DT>
__device__ inline void widen(u32x4 v, float (&f)[8]) {
  const auto h = bits<typename DT::x8>(v);
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = (float)h[i];
}
template <typename DT>
__device__ inline u32x4 narrow(const float (&f)[8]) {
  typename DT::x8 h;
#pragma unroll
  for (int i = 0; i < 8; ++i) h[i] = (typename DT::scalar)f[i];
  return bits<u32x4>(h);
}

}  // namespace mori
