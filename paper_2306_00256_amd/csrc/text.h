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
  void* workspace;         // of embed_grad_workspace bytes
};

// How the gradient's positions are brought into the order of their tokens, and its workspace.
constexpr int kChunk = 16;             // sorted positions that one wavefront adds up
constexpr int kFewT = 256, kSomeT = 1024;   // positions per agent up to which nothing is sorted: always, with few positions in all
constexpr int kLdsT = 8192;            // ... up to which one workgroup sorts them in LDS
constexpr int64_t kSomePositions = 4096;
// Positions per workgroup where several sort together: 1024, one a thread, while few workgroups have to add up the others' counts.
constexpr int tile_of_sort(int64_t T) { return T <= (1 << 16) ? 1024 : 4096; }
constexpr int kDigitBits = 9, kDigits = 1 << kDigitBits;
// Up to this many tiles every one adds up the others' counts itself; beyond, a launch of its own does it for all, or the work would grow with
// the square of T (positions of 2 fp16, V = 32000: 2^18 of them, 65 tiles, 88.7 us either way; 2^20 292 -> 254; 2^25 32.5 -> 7.7 ms).
constexpr int kManyTiles = 64;
static_assert((1 << 16) / 1024 <= kManyTiles, "tiles of 1024 positions are not many");
struct EmbedGradPlan {
  bool small, lds;
  int32_t bits, pos_bits, chunks, tiles;
  int32_t hist_rows;                   // counts of an agent: one row per tile and, where a launch of its own sums them up, one for all
  int32_t passes, digit_bits;          // of the sort
  int64_t pitch;                       // floats per partial sum
  int64_t tok0, pos0, tok1, pos1, hist, partial, bytes;   // offsets in the workspace
};
inline int bits_of(uint32_t v) { return v ? 32 - __builtin_clz(v) : 0; }
inline EmbedGradPlan plan_embed_grad(int64_t n, int64_t V, int64_t h, int64_t T) {
  EmbedGradPlan p{};
  // unsorted, every position's wavefront looks through the agent's tokens
  p.small = T <= kFewT || (T <= kSomeT && n * T * ((h + 255) / 256) <= kSomePositions);
  if (p.small) return p;
  p.bits = bits_of((uint32_t)V);       // V itself stands for padding
  p.passes = (p.bits + kDigitBits - 1) / kDigitBits;
  p.digit_bits = (p.bits + p.passes - 1) / p.passes;
  p.pos_bits = bits_of((uint32_t)(T - 1));
  p.lds = T <= kLdsT && p.bits + p.pos_bits <= 32;
  p.chunks = (int32_t)((T + kChunk - 1) / kChunk);
  p.tiles = p.lds ? 1 : (int32_t)((T + tile_of_sort(T) - 1) / tile_of_sort(T));
  p.pitch = (h + 3) / 4 * 4;
  auto take = [&](int64_t bytes) { const int64_t at = p.bytes; p.bytes += (bytes + 255) / 256 * 256; return at; };
  p.tok0 = take(n * T * 4);
  p.pos0 = take(n * T * 4);
  if (!p.lds) {
    p.tok1 = take(n * T * 4);
    p.pos1 = take(n * T * 4);
    p.hist_rows = p.tiles + (p.tiles > kManyTiles);
    p.hist = take(n * p.hist_rows * (int64_t)kDigits * 4);
  }
  p.partial = take(n * p.chunks * 2 * p.pitch * 4);
  return p;
}

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
  void* workspace;         // of plan_distill(...).bytes
};

// Rows are split over `parts` workgroups of `cols` columns where there are too few to fill the device.
struct DistillPlan {
  int32_t parts, cols;
  int64_t stats, values, bytes;    // offsets in the workspace
};
DistillPlan plan_distill(int64_t rows, int32_t V, int32_t K, int type);

struct TopArgs {
  const void* logits;
  int64_t ld;
  float* top;
  int32_t* ids;
  int32_t rows, V, K;
  int32_t type;
  void* workspace;         // of plan_top(...).bytes
};

// Rows go through `parts` workgroups of `cols` columns (the last one may have fewer); with several, each leaves its K largest in the
// workspace, and further launches make one list of up to kMergeWords / K at a time, back and forth between two parts of it.
constexpr int kMergeWords = 4096;
struct TopPlan {
  int32_t parts, cols;
  int64_t second, bytes;   // offset of the workspace's second part
};
TopPlan plan_top(int64_t rows, int32_t V, int32_t K, int type);

constexpr int kTopMax = 256;         // most entries of a row's top logits

// What a call of these sizes launches (ceca_describe_text_launch): the pointers of `a` are not looked at.
void describe_embed(const EmbedArgs& a, int32_t* out);
void describe_embed_grad(const EmbedArgs& a, int32_t* out);
void describe_distill(int64_t rows, int32_t V, int32_t K, int type, bool grad, int32_t* out);
void describe_top(int64_t rows, int32_t V, int32_t K, int type, int32_t* out);

hipError_t launch_embed(const EmbedArgs& a, hipStream_t st);
hipError_t launch_embed_grad(const EmbedArgs& a, hipStream_t st);
hipError_t launch_distill(const DistillArgs& a, hipStream_t st);
hipError_t launch_top(const TopArgs& a, hipStream_t st);

}  // namespace ceca
