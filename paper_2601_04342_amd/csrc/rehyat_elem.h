// Element types of the operators that take more than bf16: storage, and conversion to and from fp32 (round to nearest,
// ties to even).
#pragma once
#include "rehyat_device.h"

namespace rehyat {

struct Bf16 {
  typedef uint16_t store;
  static __device__ __forceinline__ float get(store x) { return __builtin_bit_cast(float, (uint32_t)x << 16); }
  static __device__ __forceinline__ store put(float x) { return (store)pack_bf16(x, x); }
};
struct Fp16 {
  typedef uint16_t store;
  static __device__ __forceinline__ float get(store x) { return (float)__builtin_bit_cast(_Float16, x); }
  static __device__ __forceinline__ store put(float x) { return __builtin_bit_cast(store, (_Float16)x); }
};
struct Fp32 {
  typedef float store;
  static __device__ __forceinline__ float get(store x) { return x; }
  static __device__ __forceinline__ store put(float x) { return x; }
};

}  // namespace rehyat
