// Element types of the operators that take float32, float16 and bfloat16 alike.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ecc {

// codes of ecc_dtype (include/ecc.h)
constexpr int kF32 = 2, kF16 = 3, kBF16 = 6;

using half_t = _Float16;
using bf16_t = __bf16;

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(half_t v) { return (float)v; }
__device__ __forceinline__ float widen(bf16_t v) {
  return __uint_as_float((unsigned)__builtin_bit_cast(unsigned short, v) << 16);
}
template <typename T>
__device__ __forceinline__ T narrow(float v) { return (T)v; }  // to nearest even

}  // namespace ecc
