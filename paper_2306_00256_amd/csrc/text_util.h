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

// VEC neighbouring elements of a row.  Rows may begin at any element, so the access claims no more than an element's alignment
// (a 16-byte load or store of this chip needs no more).
template <typename T> struct RawOf { using R = T; };
template <> struct RawOf<bf16_t> { using R = uint16_t; };
template <typename T, int VEC> struct Pack {
  using R = typename RawOf<T>::R;
  typedef R Mem __attribute__((ext_vector_type(VEC), aligned(sizeof(T))));
  typedef R Reg __attribute__((ext_vector_type(VEC)));
  Reg v;
  __device__ __forceinline__ static Pack load(const T* p) { return Pack{*reinterpret_cast<const Mem*>(p)}; }
  __device__ __forceinline__ static Pack load_stream(const T* p) { return Pack{__builtin_nontemporal_load(reinterpret_cast<const Mem*>(p))}; }
  __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<Mem*>(p) = v; }
  __device__ __forceinline__ void store_stream(T* p) const { __builtin_nontemporal_store((Mem)v, reinterpret_cast<Mem*>(p)); }
  // The compiler must work out again what it made of these elements before: kept, the floats of a register tile would take up to twice
  // the tile's registers.
  __device__ __forceinline__ void again() {
    static_assert(sizeof(Reg) == 16, "one 16-byte register tuple");
    typedef uint32_t U __attribute__((ext_vector_type(4)));
    U u = __builtin_bit_cast(U, v);
    asm volatile("" : "+v"(u));
    v = __builtin_bit_cast(Reg, u);
  }
  __device__ __forceinline__ float get(int k) const { return to_float(__builtin_bit_cast(T, (R)v[k])); }
  __device__ __forceinline__ void set(int k, float x) { v[k] = __builtin_bit_cast(R, from_float<T>(x)); }
};

constexpr float kInf = __builtin_inff();

// Over a wavefront's rows of 16 lanes in four steps without LDS, then over the four rows: the same for every lane.
template <int CTRL> __device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(v), __float_as_int(v), CTRL, 0xf, 0xf, true));
}
template <typename F> __device__ __forceinline__ float row_all(float v, F f) {
  v = f(v, dpp<0xB1>(v));        // lanes 1 apart
  v = f(v, dpp<0x4E>(v));        // 2
  v = f(v, dpp<0x141>(v));       // the other four of eight
  return f(v, dpp<0x140>(v));    // the other eight of sixteen
}
__device__ __forceinline__ float lane_value(float v, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane)); }
template <typename F> __device__ __forceinline__ float wave_all(float v, F f) {
  v = row_all(v, f);
  return f(f(lane_value(v, 0), lane_value(v, 16)), f(lane_value(v, 32), lane_value(v, 48)));
}
struct Add { __device__ __forceinline__ float operator()(float a, float b) const { return a + b; } };
struct Max { __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); } };     // drops NaN

// Columns a thread reads at once: 16 bytes.
template <typename T> constexpr int kVec = 16 / (int)sizeof(T);

}  // namespace ceca
