// The largest logits of a row and their places.
#include "device_util.h"
#include "text_util.h"

namespace ceca {

namespace {

// Order of the logits as unsigned numbers: -inf < ... < -0 = +0 < ... < +inf < NaN.
__device__ __forceinline__ uint32_t order_key(float v) {
  if (v != v) return 0xffc00000u;
  const uint32_t b = __float_as_uint(v + 0.0f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
constexpr uint32_t kKeyMinusInf = 0x007fffffu;

// One workgroup per row picks the largest of what is left, K times.
template <typename T>
__global__ __launch_bounds__(256) void top_kernel(TopArgs a) {
  __shared__ uint64_t best[4];
  const int64_t row = blockIdx.x;
  const T* s = static_cast<const T*>(a.logits) + row * a.ld;
  uint64_t last = ~0ull;
  for (int k = 0; k < a.K; ++k) {
    uint64_t b = 0;
    for (int32_t v = threadIdx.x; v < a.V; v += 256) {
      const uint64_t key = (uint64_t)order_key(to_float(s[v])) << 32 | (uint32_t)~v;
      if (key < last && key > b) b = key;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const uint64_t c = __shfl_xor((unsigned long long)b, o, 64);
      b = c > b ? c : b;
    }
    __syncthreads();
    if (threadIdx.x % 64 == 0) best[threadIdx.x / 64] = b;
    __syncthreads();
    for (int w = 0; w < 4; ++w) b = best[w] > b ? best[w] : b;
    last = b;
    if (threadIdx.x == 0) {
      const bool is = (uint32_t)(b >> 32) > kKeyMinusInf;
      const int32_t at = (int32_t)~(uint32_t)b;
      a.top[row * a.K + k] = is ? to_float(s[at]) : -__builtin_inff();
      a.ids[row * a.K + k] = is ? at : -1;
    }
  }
}

}  // namespace

hipError_t launch_top(const TopArgs& a, hipStream_t st) {
  const dim3 grid((uint32_t)a.rows), block(256);
  if (a.type == TYPE_F32) top_kernel<float><<<grid, block, 0, st>>>(a);
  else if (a.type == TYPE_BF16) top_kernel<bf16_t><<<grid, block, 0, st>>>(a);
  else top_kernel<_Float16><<<grid, block, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace ceca
