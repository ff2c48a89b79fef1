// Embedding lookup in the agents' tables, and its gradient.
#include "device_util.h"
#include "text_util.h"

namespace ceca {

namespace {

// out[i, t, :] = scale * E_i[token, :], one wavefront per position; zeros where the token is none of the vocabulary.
template <typename T>
__global__ __launch_bounds__(256) void embed_kernel(EmbedArgs a) {
  const int64_t row = (int64_t)blockIdx.x * 4 + threadIdx.x / 64;
  if (row >= (int64_t)a.n * a.T) return;
  const int32_t token = a.tokens[row];
  const bool real = token >= 0 && token < a.V;
  const float* e = a.E + row / a.T * a.lde + (real ? token : 0) * a.ldr;
  T* out = static_cast<T*>(a.rows) + row * a.ldo;
  for (int32_t c = threadIdx.x % 64; c < a.h; c += 64) out[c] = from_float<T>(real ? a.scale * e[c] : 0.0f);
}

// e_i[v, :] = scale * sum of the gradient's rows at v's positions, in their order: one wavefront per row of a table
// goes through the agent's tokens.
template <typename T>
__global__ __launch_bounds__(256) void embed_grad_kernel(EmbedArgs a) {
  const int64_t vrow = (int64_t)blockIdx.x * 4 + threadIdx.x / 64;
  if (vrow >= (int64_t)a.n * a.V) return;
  const int lane = threadIdx.x % 64;
  const int64_t i = vrow / a.V;
  const int32_t v = (int32_t)(vrow - i * a.V);
  const int32_t* tokens = a.tokens + i * a.T;
  const T* g = static_cast<const T*>(a.rows) + i * a.T * a.ldo;
  float* e = a.dE + i * a.lde + v * a.ldr;
  for (int32_t c0 = 0; c0 < a.h; c0 += 64) {
    const int32_t c = c0 + lane;
    float sum = 0.0f;
    bool some = false;
    for (int32_t t0 = 0; t0 < a.T; t0 += 64) {
      uint64_t hits = __ballot(t0 + lane < a.T && tokens[min(t0 + lane, a.T - 1)] == v);
      some |= hits != 0;
      for (; hits; hits &= hits - 1) {
        const int64_t t = t0 + __builtin_ctzll(hits);
        if (c < a.h) sum += to_float(g[t * a.ldo + c]);
      }
    }
    if (c < a.h) {
      if (!a.accumulate) e[c] = a.scale * sum;
      else if (some) e[c] += a.scale * sum;
    }
  }
}

template <template <typename> class Launch, typename... A> hipError_t by_type(int type, A... args) {
  if (type == TYPE_F32) return Launch<float>::go(args...);
  if (type == TYPE_BF16) return Launch<bf16_t>::go(args...);
  return Launch<_Float16>::go(args...);
}

template <typename T> struct Lookup {
  static hipError_t go(const EmbedArgs& a, hipStream_t st) {
    const int64_t blocks = ((int64_t)a.n * a.T + 3) / 4;
    embed_kernel<T><<<dim3((uint32_t)blocks), dim3(256), 0, st>>>(a);
    return hipGetLastError();
  }
};
template <typename T> struct Gradient {
  static hipError_t go(const EmbedArgs& a, hipStream_t st) {
    const int64_t blocks = ((int64_t)a.n * a.V + 3) / 4;
    embed_grad_kernel<T><<<dim3((uint32_t)blocks), dim3(256), 0, st>>>(a);
    return hipGetLastError();
  }
};

}  // namespace

hipError_t launch_embed(const EmbedArgs& a, hipStream_t st) { return by_type<Lookup>(a.type, a, st); }
hipError_t launch_embed_grad(const EmbedArgs& a, hipStream_t st) { return by_type<Gradient>(a.type, a, st); }

}  // namespace ceca
