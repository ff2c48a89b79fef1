// Internal interface between the C ABI (api.cpp) and the kernels of the language-model operators (embed.hip,
// distill.hip, top.hip).
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace ceca {

enum ElemType : int { TYPE_F32 = 0, TYPE_BF16 = 1, TYPE_F16 = 2 };

// Agent i's table: V rows of h floats at pitch ldr, from E + i lde on.
struct EmbedArgs {
  const float* E;
  float* dE;               // gradient rows, the same layout
  int64_t lde, ldr;
  const int32_t* tokens;   // n * T
  void* rows;              // out (lookup) or the gradient of out (read only)
  int64_t ldo;
  int32_t n, V, h, T;
  int32_t type;            // of rows
  float scale;
  int32_t accumulate;
};

struct DistillArgs {
  const void* logits;
  int64_t ld;
  void* grad;              // may be null; may be the logits
  int64_t ldg;
  float* loss;             // may be null
  const float* top;
  const int32_t* ids;
  const int32_t* peer;     // may be null
  const int32_t* labels;   // null: no hard term
  const float* weight;     // null: ones
  int32_t n, T, V, K;
  int32_t type;
  float tau, hard;
};

struct TopArgs {
  const void* logits;
  int64_t ld;
  float* top;
  int32_t* ids;
  int32_t rows, V, K;
  int32_t type;
};

constexpr int kTopMax = 256;         // most entries of a row's top logits

hipError_t launch_embed(const EmbedArgs& a, hipStream_t st);
hipError_t launch_embed_grad(const EmbedArgs& a, hipStream_t st);
hipError_t launch_distill(const DistillArgs& a, hipStream_t st);
hipError_t launch_top(const TopArgs& a, hipStream_t st);

}  // namespace ceca
