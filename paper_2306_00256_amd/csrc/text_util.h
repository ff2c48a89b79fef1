// Device-side helpers of the language-model operators: the element types of activations and logits, and workgroup
// reductions.
#pragma once
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include <cstdint>

#include "text.h"

namespace ceca {

struct bf16_t { uint16_t bits; };

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(bf16_t v) { return __uint_as_float((uint32_t)v.bits << 16); }
__device__ __forceinline__ float to_float(_Float16 v) { return (float)v; }
// The one rounding of a result that was computed in fp32: to nearest, ties to even.
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ _Float16 from_float<_Float16>(float v) { return (_Float16)v; }
template <> __device__ __forceinline__ bf16_t from_float<bf16_t>(float v) {
  const __bf16 b = (__bf16)v;
  return bf16_t{__builtin_bit_cast(uint16_t, b)};
}

}  // namespace ceca
