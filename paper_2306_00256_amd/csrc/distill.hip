// Distillation from a teacher's top logits: loss and gradient.
#include "device_util.h"
#include "text_util.h"

namespace ceca {

namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kInf = __builtin_inff();

// Sum and maximum over the workgroup; `red`: one float per wavefront.  fmaxf drops NaN, sums keep it.
template <int THREADS> __device__ __forceinline__ float block_sum(float v, float* red) {
  v = wave_sum(v);
  __syncthreads();
  if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = v;
  __syncthreads();
  float s = 0.0f;
  for (int w = 0; w < THREADS / 64; ++w) s += red[w];
  return s;
}
template <int THREADS> __device__ __forceinline__ float block_max(float v, float* red) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  __syncthreads();
  if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = v;
  __syncthreads();
  float s = red[0];
  for (int w = 1; w < THREADS / 64; ++w) s = fmaxf(s, red[w]);
  return s;
}

// One workgroup per row; see ceca.h for the formulas.
template <typename T>
__global__ __launch_bounds__(256) void distill_kernel(DistillArgs a) {
  __shared__ float red[4], p[kTopMax];
  __shared__ int32_t id[kTopMax];
  const int64_t row = blockIdx.x;
  const int tid = threadIdx.x;
  const float w = a.weight ? a.weight[row] : 1.0f;
  T* grad = a.grad ? static_cast<T*>(a.grad) + row * a.ldg : nullptr;
  if (w == 0.0f) {
    if (a.loss && tid == 0) a.loss[row] = 0.0f;
    if (grad) for (int32_t v = tid; v < a.V; v += 256) grad[v] = from_float<T>(0.0f);
    return;
  }
  const T* s = static_cast<const T*>(a.logits) + row * a.ld;
  // the teacher's entries: shares p of those that are there, id -1 for the others
  int64_t trow = row;
  if (a.peer) trow = (int64_t)min(max(a.peer[row / a.T], 0), a.n - 1) * a.T + row % a.T;
  float u = -kInf;
  int32_t at = -1;
  if (tid < a.K) {
    at = a.ids[trow * a.K + tid];
    if (at >= 0 && at < a.V) u = a.top[trow * a.K + tid];
    if (u == -kInf) at = -1;
  }
  const float inv_tau = 1.0f / a.tau;
  float um = block_max<256>(u, red);
  if (um == -kInf) um = 0.0f;
  const float ux = (u - um) * inv_tau, ue = expf(ux), usum = block_sum<256>(ue, red);
  const bool soft = usum != 0.0f && a.hard < 1.0f;
  const float pk = at >= 0 ? ue / usum : 0.0f, logp = ux - logf(usum);
  id[tid] = at;
  p[tid] = pk;
  const int32_t label = a.labels ? a.labels[row] : -1;
  const bool hard = a.hard > 0.0f && label >= 0 && label < a.V;

  // the student's row
  float m = -kInf;
  for (int32_t v = tid; v < a.V; v += 256) m = fmaxf(m, to_float(s[v]));
  m = block_max<256>(m, red);
  if (m == -kInf) m = 0.0f;
  float q = 0.0f, r = 0.0f;
  for (int32_t v = tid; v < a.V; v += 256) {
    const float x = to_float(s[v]) - m;
    q += expf(x * inv_tau);
    r += expf(x);
  }
  q = block_sum<256>(q, red);
  r = block_sum<256>(r, red);
  const bool empty = r == 0.0f;
  const float cs = soft && !empty ? w * (1.0f - a.hard) : 0.0f, ch = hard && !empty ? w * a.hard : 0.0f;

  float x = 0.0f, term = 0.0f;
  if (at >= 0) {
    x = (to_float(s[at]) - m) * inv_tau;
    if (pk != 0.0f) term = pk * (logp + logf(q) - x);
  }
  if (a.loss) {
    const float sum = block_sum<256>(term, red);
    if (tid == 0) {
      float loss = 0.0f;
      if (cs != 0.0f) loss += cs * a.tau * a.tau * sum;
      if (ch != 0.0f) loss += ch * (logf(r) - (to_float(s[label]) - m));
      a.loss[row] = loss;
    }
  }
  if (!grad) return;
  const float gs = cs * a.tau, qs = cs != 0.0f ? gs / q : 0.0f, rs = ch != 0.0f ? ch / r : 0.0f;
  const bool zero = cs == 0.0f && ch == 0.0f;
  __syncthreads();
  float lx = hard ? to_float(s[label]) - m : 0.0f;        // read before the row is overwritten in place
  const float sx = at >= 0 ? to_float(s[at]) - m : 0.0f;
  __syncthreads();
  for (int32_t v = tid; v < a.V; v += 256) {
    const float y = to_float(s[v]) - m;
    grad[v] = from_float<T>(zero ? 0.0f : (cs != 0.0f ? qs * expf(y * inv_tau) : 0.0f) + (ch != 0.0f ? rs * expf(y) : 0.0f));
  }
  // the places of the teacher's entries and of the label once more, with their shares taken off; an id that comes
  // twice takes both
  __syncthreads();
  if (zero) return;
  if (cs != 0.0f && at >= 0) {
    float sum = 0.0f;
    for (int k = 0; k < a.K; ++k) if (id[k] == at) sum += p[k];
    float g = gs * (expf(sx * inv_tau) / q - sum);
    if (ch != 0.0f) g += ch * (expf(sx) / r - (at == label ? 1.0f : 0.0f));
    grad[at] = from_float<T>(g);
  }
  if (ch != 0.0f && tid == 0) {
    bool also = false;
    for (int k = 0; k < a.K; ++k) also |= cs != 0.0f && id[k] == label;
    if (!also) grad[label] = from_float<T>((cs != 0.0f ? qs * expf(lx * inv_tau) : 0.0f) + ch * (expf(lx) / r - 1.0f));
  }
}

}  // namespace

hipError_t launch_distill(const DistillArgs& a, hipStream_t st) {
  const dim3 grid((uint32_t)a.n * (uint32_t)a.T), block(256);
  if (a.type == TYPE_F32) distill_kernel<float><<<grid, block, 0, st>>>(a);
  else if (a.type == TYPE_BF16) distill_kernel<bf16_t><<<grid, block, 0, st>>>(a);
  else distill_kernel<_Float16><<<grid, block, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace ceca
