// Embedding lookup in the agents' tables, and its gradient by sorted tokens.
#include <algorithm>

#include "device_util.h"
#include "text_util.h"

namespace ceca {

namespace {

// A lane's columns of one row: VEC of them from column c on, the last VEC where fewer are left (it stores its own alone).
template <int VEC> struct Columns {
  int32_t c, at;              // first own column, first column read
  bool whole, some;
  __device__ __forceinline__ Columns(int32_t first, int32_t h) : c(first), at(min(first, h - VEC)), whole(first + VEC <= h), some(first < h) {}
  template <typename T> __device__ __forceinline__ void store(T* row, const float (&x)[VEC]) const {
    Pack<T, VEC> v;
#pragma unroll
    for (int k = 0; k < VEC; ++k) v.set(k, x[k]);
    if (whole) {
      v.store(row + at);
    } else if (some) {
#pragma unroll
      for (int k = 0; k < VEC; ++k)
        if (at + k >= c) row[at + k] = __builtin_bit_cast(T, (typename Pack<T, VEC>::R)v.v[k]);
    }
  }
};

// out[i, t, :] = scale * E_i[token, :], zeros where the token is none of the vocabulary.  Read and write once; a wavefront has
// 64 VEC columns of ROWS positions, all loads before the first store.
template <typename T, int VEC, int ROWS>
__global__ __launch_bounds__(256) void embed_kernel(EmbedArgs a, int32_t tiles) {
  const int64_t rows = (int64_t)a.n * a.T, groups = (rows + ROWS - 1) / ROWS, units = groups * tiles;
  for (int64_t unit = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / 64); unit < units; unit += (int64_t)gridDim.x * 4) {
    const int64_t group = unit / tiles, row0 = group * ROWS;
    const Columns<VEC> col((int32_t)(unit - group * tiles) * 64 * VEC + threadIdx.x % 64 * VEC, a.h);
    if (!col.some) continue;
    Pack<float, VEC> e[ROWS];
    bool real[ROWS];
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
      const int64_t row = min(row0 + k, rows - 1), i = row / a.T;
      const int32_t token = a.tokens[row];
      real[k] = token >= 0 && token < a.V;
      e[k] = Pack<float, VEC>::load(a.E + i * a.lde + (real[k] ? token : 0) * a.ldr + col.at);
    }
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
      if (row0 + k >= rows) break;
      float x[VEC];
#pragma unroll
      for (int c = 0; c < VEC; ++c) x[c] = real[k] ? a.scale * e[k].get(c) : 0.0f;
      col.store(static_cast<T*>(a.rows) + (row0 + k) * a.ldo, x);
    }
  }
}

// ---- the gradient ----
// e_i[v, :] = scale * sum of G's rows at v's positions.  A position's row is read once, a table's row is written once: what bounds
// it is the memory's rate, mostly for the zeros of rows whose tokens do not occur.  Four launches:
//   zeros  over the tables (not where the sums are added to what is there; few of them go with the sort)
//   sort   positions into the order of (token, position), in LDS
//   walk   a wavefront adds the rows of kChunk sorted positions up, in order; where a token's positions lie in one chunk its row
//          of the table is done, else the chunk's share goes to the workspace
//   join   the shares of tokens that lie in several chunks, in their order
// Which lane adds what follows from the tokens alone: no atomics on sums, the same bits every time.
// Zeros for the rows that no token names alone, by the walk's launch from a byte per row, were slower: 31 tables of 32000 x 512 575 us
// against 298 + 37 for all zeros and the walk.

// One 16-byte store per thread and short-lived workgroups in the order of memory are the fastest way to write zeros: 2 GB at 6.8
// TB/s, 6.0 with two stores, 5.6 to 6.1 with four and more or 1024 threads, 4.5 to 5.8 with long-lived workgroups that sweep
// memory together.  `all` workgroups' shares, `blocks` per piece of `count` floats, `pitch` apart.
struct ZeroArgs {
  float* p;
  int64_t count, pitch;
  uint32_t blocks, all;
};
template <int THREADS> __device__ __forceinline__ void write_zeros(const ZeroArgs& z, uint32_t b) {
  const uint32_t i = z.blocks == z.all ? 0 : b / z.blocks;
  const int64_t at = (int64_t)(b - i * z.blocks) * (4 * THREADS) + threadIdx.x * 4;
  float* q = z.p + i * z.pitch;
  if (at + 4 <= z.count) st_plain<vf4>(q + at, vf4{0.0f, 0.0f, 0.0f, 0.0f});
  else
    for (int64_t k = at; k < z.count; ++k) q[k] = 0.0f;
}
__global__ __launch_bounds__(256) void zeros_kernel(ZeroArgs z) {
  for (uint64_t b = blockIdx.x; b < z.all; b += gridDim.x) write_zeros<256>(z, (uint32_t)b);
}
// The same where something lies between the rows: a wavefront per row.
__global__ __launch_bounds__(256) void zero_rows_kernel(EmbedArgs a) {
  const int64_t rows = (int64_t)a.n * a.V;
  for (int64_t row = (int64_t)blockIdx.x * 4 + threadIdx.x / 64; row < rows; row += (int64_t)gridDim.x * 4) {
    const int64_t i = row / a.V;
    float* q = a.dE + i * a.lde + (row - i * a.V) * a.ldr;
    for (int32_t c = threadIdx.x % 64; c < a.h; c += 64) q[c] = 0.0f;
  }
}

// One stable pass over up to IPT * 1024 keys by `bits` bits from `shift` on: where every key of this thread goes.  A wavefront
// owns a block of 64 IPT keys, key j * 64 + lane of it is the lane's j-th; lanes with the same digit find each other by ballots,
// and a digit's count per wavefront is kept in `count` (16 x digits).
template <int IPT>
__device__ __forceinline__ void rank_keys(const uint32_t (&key)[IPT], uint32_t (&to)[IPT], int shift, int bits, uint32_t* count, uint32_t* totals) {
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, digits = 1 << bits;
  for (int k = tid; k < 16 * digits; k += 1024) count[k] = 0;
  __syncthreads();
  volatile uint32_t* mine = count + wave * digits;      // (lanes of the wavefront read what others of it wrote)
#pragma unroll
  for (int j = 0; j < IPT; ++j) {
    const uint32_t d = key[j] >> shift & (digits - 1);
    uint32_t lo = ~0u, hi = ~0u;               // lanes whose digit is the same, bit by bit
    for (int b = 0; b < bits; ++b) {
      const uint32_t off = (d >> b & 1) - 1;   // all ones where the bit is clear
      const uint64_t has = __ballot(off == 0);
      lo &= (uint32_t)has ^ off;
      hi &= (uint32_t)(has >> 32) ^ off;
    }
    const uint64_t same = (uint64_t)hi << 32 | lo;
    const uint32_t before = __builtin_amdgcn_mbcnt_hi(hi, __builtin_amdgcn_mbcnt_lo(lo, 0));
    const uint32_t seen = mine[d];
    __builtin_amdgcn_wave_barrier();
    if (before == 0) mine[d] = seen + (uint32_t)__builtin_popcountll(same);
    __builtin_amdgcn_wave_barrier();
    to[j] = seen + before;
  }
  __syncthreads();
  // exclusive sums in the order (digit, wavefront): 16 digits' counts a thread chunk, then over the threads
  const int per = 16 * digits / 1024 > 0 ? 16 * digits / 1024 : 1;
  const int first = tid * per;                         // entry e stands for digit e / 16 of wavefront e % 16
  uint32_t sum = 0;
  if (first < 16 * digits)
    for (int e = first; e < first + per; ++e) sum += count[(e % 16) * digits + e / 16];
  uint32_t upto = sum;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t x = __shfl_up(upto, o, 64);
    if (lane >= o) upto += x;
  }
  if (lane == 63) totals[wave] = upto;
  __syncthreads();
  uint32_t base = upto - sum;
  for (int w = 0; w < wave; ++w) base += totals[w];
  if (first < 16 * digits)
    for (int e = first; e < first + per; ++e) {
      const int at = (e % 16) * digits + e / 16;
      const uint32_t x = count[at];
      count[at] = base;
      base += x;
    }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < IPT; ++j) to[j] += mine[key[j] >> shift & (digits - 1)];
}

// Agents' positions sorted by one workgroup each, the keys (token, position) in one word.  (Up to 8192: 75 x 4524 positions of 32
// fp16 106 us, sorted by five workgroups each 124; 16384 would take 36 us alone, two passes of two launches 24.)
template <int IPT>
__global__ __launch_bounds__(1024) void sort_lds_kernel(EmbedArgs a, EmbedGradPlan p, ZeroArgs z, uint32_t sorts) {
  if (blockIdx.x >= sorts) {
    write_zeros<1024>(z, blockIdx.x - sorts);
    return;
  }
  extern __shared__ uint32_t lds[];
  uint32_t* count = lds;                               // 16 x digits
  uint32_t* totals = lds + 16 * kDigits;
  uint32_t* keys = totals + 16;                        // IPT * 1024
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  for (int64_t i = blockIdx.x; i < a.n; i += sorts) {
    const int32_t* tokens = a.tokens + i * a.T;
    uint32_t key[IPT], to[IPT];
    const uint32_t none = (uint32_t)((((uint64_t)1 << (p.bits + p.pos_bits)) - 1));
#pragma unroll
    for (int j = 0; j < IPT; ++j) {
      const int t = (wave * IPT + j) * 64 + lane;
      const int32_t v = t < a.T ? tokens[t] : -1;
      // places past the last position go last of all: the largest key, and behind the others of it
      const bool real = v >= 0 && v < a.V;
      key[j] = t < a.T ? (uint32_t)(real ? v : a.V) << p.pos_bits | (uint32_t)t : none;
    }
    for (int shift = 0; shift < p.bits; shift += p.digit_bits) {
      const int bits = min(p.digit_bits, p.bits - shift);
      rank_keys<IPT>(key, to, p.pos_bits + shift, bits, count, totals);
#pragma unroll
      for (int j = 0; j < IPT; ++j) keys[to[j]] = key[j];
      __syncthreads();
#pragma unroll
      for (int j = 0; j < IPT; ++j) key[j] = keys[(wave * IPT + j) * 64 + lane];
    }
    uint32_t* tok = reinterpret_cast<uint32_t*>(static_cast<char*>(a.workspace) + p.tok0) + i * a.T;
    uint32_t* pos = reinterpret_cast<uint32_t*>(static_cast<char*>(a.workspace) + p.pos0) + i * a.T;
#pragma unroll
    for (int j = 0; j < IPT; ++j) {
      const int t = (wave * IPT + j) * 64 + lane;
      if (t < a.T) {
        tok[t] = min(key[j] >> p.pos_bits, (uint32_t)a.V);
        pos[t] = key[j] & (((uint32_t)1 << p.pos_bits) - 1);
      }
    }
    __syncthreads();
  }
}

// Longer sequences: tiles of 1024 IPT positions, one pass of kDigitBits bits in two launches.  Counts of every tile first ...
struct PassArgs {
  const int32_t* tokens;       // first pass, else null
  const uint32_t *tok, *pos;   // later passes
  uint32_t *tok_out, *pos_out, *hist;
  int32_t n, V, T, tiles, hist_rows, shift, bits;
};
__device__ __forceinline__ uint32_t pass_key(const PassArgs& p, int64_t i, int64_t t) {
  if (!p.tokens) return p.tok[i * p.T + t];
  const int32_t v = p.tokens[i * p.T + t];
  return (uint32_t)(v >= 0 && v < p.V ? v : p.V);
}
template <int IPT> __global__ __launch_bounds__(1024) void count_digits_kernel(PassArgs p, ZeroArgs z, uint32_t counts) {
  if (blockIdx.x >= counts) {
    write_zeros<1024>(z, blockIdx.x - counts);
    return;
  }
  constexpr int kTile = 1024 * IPT;
  __shared__ uint32_t count[kDigits];
  const int64_t sorts = (int64_t)p.n * p.tiles;
  for (int64_t b = blockIdx.x; b < sorts; b += counts) {
    const int64_t i = b / p.tiles, tile = b - i * p.tiles, t0 = tile * kTile;
    if (threadIdx.x < kDigits) count[threadIdx.x] = 0;
    __syncthreads();
    for (int64_t t = t0 + threadIdx.x; t < min(t0 + kTile, (int64_t)p.T); t += 1024)
      atomicAdd(&count[pass_key(p, i, t) >> p.shift & ((1u << p.bits) - 1)], 1u);       // whole numbers: any order
    __syncthreads();
    if (threadIdx.x < kDigits) p.hist[(i * p.hist_rows + tile) * kDigits + threadIdx.x] = count[threadIdx.x];
    __syncthreads();
  }
}
// ... then, of many tiles, a digit's counts of earlier tiles and of all, by a wavefront per agent and digit ...
__global__ __launch_bounds__(256) void sum_counts_kernel(PassArgs p) {
  const int lane = threadIdx.x % 64;
  const int64_t units = (int64_t)p.n * kDigits;
  for (int64_t unit = (int64_t)blockIdx.x * 4 + threadIdx.x / 64; unit < units; unit += (int64_t)gridDim.x * 4) {
    uint32_t* hist = p.hist + unit / kDigits * p.hist_rows * kDigits + unit % kDigits;
    uint32_t before = 0;
    for (int64_t k0 = 0; k0 < p.tiles; k0 += 64) {
      const uint32_t mine = k0 + lane < p.tiles ? hist[(k0 + lane) * kDigits] : 0;
      uint32_t upto = mine;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const uint32_t x = __shfl_up(upto, o, 64);
        if (lane >= o) upto += x;
      }
      if (k0 + lane < p.tiles) hist[(k0 + lane) * kDigits] = before + upto - mine;
      before += __builtin_amdgcn_readlane(upto, 63);
    }
    if (lane == 0) hist[(int64_t)p.tiles * kDigits] = before;
  }
}
// ... then every tile's keys to their places: behind the smaller digits of all tiles and the same digit's of earlier tiles.
template <int IPT> __global__ __launch_bounds__(1024) void place_keys_kernel(PassArgs p) {
  constexpr int kTile = 1024 * IPT;
  __shared__ uint32_t count[16 * kDigits], totals[16], base[kDigits], sums[16];
  const int64_t sorts = (int64_t)p.n * p.tiles;
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  for (int64_t b = blockIdx.x; b < sorts; b += gridDim.x) {
    const int64_t i = b / p.tiles;
    const int32_t tile = (int32_t)(b - i * p.tiles);
    uint32_t before = 0, all = 0;
    if (tid < kDigits) {
      const uint32_t* hist = p.hist + i * p.hist_rows * kDigits + tid;
      if (p.hist_rows > p.tiles) {
        before = hist[(int64_t)tile * kDigits];
        all = hist[(int64_t)p.tiles * kDigits];
      } else {
#pragma unroll 8
        for (int32_t k = 0; k < p.tiles; ++k) {
          const uint32_t c = hist[k * kDigits];
          all += c;
          before += k < tile ? c : 0;
        }
      }
    }
    uint32_t upto = all;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t x = __shfl_up(upto, o, 64);
      if (lane >= o) upto += x;
    }
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    uint32_t start = upto - all + before;
    for (int w = 0; w < wave; ++w) start += sums[w];
    if (tid < kDigits) base[tid] = start;
    uint32_t key[IPT], pos[IPT], to[IPT];
    const uint32_t none = 0xffffffffu;
#pragma unroll
    for (int j = 0; j < IPT; ++j) {
      const int64_t t = (int64_t)tile * kTile + (wave * IPT + j) * 64 + lane;
      key[j] = t < p.T ? pass_key(p, i, t) : none;
      pos[j] = t < p.T ? (p.tokens ? (uint32_t)t : p.pos[i * p.T + t]) : none;
    }
    rank_keys<IPT>(key, to, p.shift, p.bits, count, totals);
    // to: the place among the tile's keys; `count` of wavefront 0 is now where a digit begins among them
#pragma unroll
    for (int j = 0; j < IPT; ++j) {
      const uint32_t d = key[j] >> p.shift & ((1u << p.bits) - 1);
      if (pos[j] != none) {
        const int64_t at = i * p.T + base[d] + (to[j] - count[d]);
        p.tok_out[at] = key[j];
        p.pos_out[at] = pos[j];
      }
    }
    __syncthreads();
  }
}

struct WalkArgs {
  EmbedArgs e;
  const uint32_t *tok, *pos;
  float* partial;
  int64_t pitch;
  int32_t chunks, tiles;      // chunks per agent, column tiles
};

// Rows whose loads are in flight: all of a chunk, or four where each may need the table's row too.  Measured, chunks of 16 (walk / join):
// 31 x 2048 positions of 512 bf16 28 us with 16 ahead, 35 with 8; 6 x 11469 of 1024 fp32 89 with 8 and 16, added to what is there
// 111 with 4, 120 with 8, 127 with 16.  Chunks of 32 with 8 ahead 45, 98 and 139, joins 5 us shorter; of 8 33, 87 and 112, joins 8
// longer.
constexpr int ahead(bool add) { return add ? 4 : kChunk; }

// One wavefront per chunk of sorted positions and tile of 64 VEC columns.
template <typename T, int VEC, bool ADD>
__global__ __launch_bounds__(256) void walk_kernel(WalkArgs w) {
  constexpr int kAhead = ahead(ADD);
  const EmbedArgs& a = w.e;
  const int lane = threadIdx.x % 64;
  const int64_t units = (int64_t)a.n * w.chunks * w.tiles;
  for (int64_t unit = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / 64); unit < units; unit += (int64_t)gridDim.x * 4) {
    const int64_t ic = unit / w.tiles, i = ic / w.chunks;
    const int32_t chunk = (int32_t)(ic - i * w.chunks);
    const Columns<VEC> col((int32_t)(unit - ic * w.tiles) * 64 * VEC + lane * VEC, a.h);
    const T* G = static_cast<const T*>(a.rows) + i * a.T * a.ldo + col.at;
    float* E = a.dE + i * a.lde;
    float* part = w.partial + ic * 2 * w.pitch;
    // lane l holds sorted place first - 1 + l: the one before the chunk, the chunk, the one behind it
    const int32_t first = chunk * kChunk, place = first - 1 + lane;
    const bool there = place >= 0 && place < a.T && lane <= kChunk + 1;
    const uint32_t tok = there ? w.tok[i * a.T + place] : 0xffffffffu;
    const uint32_t pos = there && tok < (uint32_t)a.V ? w.pos[i * a.T + place] : 0;
    uint32_t last = __builtin_amdgcn_readlane(tok, 0);          // the token before
    bool begun = false;                                          // whether the token at hand began in an earlier chunk
    float sum[VEC];
#pragma unroll
    for (int k = 0; k < VEC; ++k) sum[k] = 0.0f;
    for (int j0 = 0; j0 < kChunk; j0 += kAhead) {
      if (__builtin_amdgcn_readlane(tok, 1 + j0) >= (uint32_t)a.V) break;        // padding sorts last
      Pack<T, VEC> g[kAhead];
      Pack<float, VEC> old[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const uint32_t v = __builtin_amdgcn_readlane(tok, 1 + j0 + j);
        if (v < (uint32_t)a.V) {
          if (col.some) g[j] = Pack<T, VEC>::load_stream(G + (int64_t)__builtin_amdgcn_readlane(pos, 1 + j0 + j) * a.ldo);
          if (ADD && v != __builtin_amdgcn_readlane(tok, 2 + j0 + j)) {
            if (col.some) old[j] = Pack<float, VEC>::load(E + (int64_t)v * a.ldr + col.at);
          }
        }
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const uint32_t v = __builtin_amdgcn_readlane(tok, 1 + j0 + j), next = __builtin_amdgcn_readlane(tok, 2 + j0 + j);
        if (v < (uint32_t)a.V) {
          if (v != last || j0 + j == 0) {
            begun = v == last;
#pragma unroll
            for (int k = 0; k < VEC; ++k) sum[k] = 0.0f;
          }
          last = v;
#pragma unroll
          for (int k = 0; k < VEC; ++k) sum[k] += g[j].get(k);
          const bool ends = next != v;
          if (ends && !begun) {
            float x[VEC];
#pragma unroll
            for (int k = 0; k < VEC; ++k) x[k] = ADD ? __builtin_fmaf(a.scale, sum[k], old[j].get(k)) : a.scale * sum[k];
            col.store(E + (int64_t)v * a.ldr, x);
          } else if (ends || j0 + j == kChunk - 1) {
            col.store(part + (begun ? 0 : w.pitch), sum);       // (where one token fills the chunk from and to elsewhere: once)
          }
        }
      }
    }
  }
}

// One wavefront per chunk and tile of columns: the token that begins in the chunk and goes on behind it.  (Four
// wavefronts that share the chunks of a frequent token were slower: 14066 positions of 727 tokens 21 us, 14 this way.)
template <int VEC, bool ADD>
__global__ __launch_bounds__(256) void join_kernel(WalkArgs w) {
  const EmbedArgs& a = w.e;
  const int lane = threadIdx.x % 64;
  const int64_t units = (int64_t)a.n * (w.chunks - 1) * w.tiles;
  for (int64_t unit = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / 64); unit < units; unit += (int64_t)gridDim.x * 4) {
    const int64_t ic = unit / w.tiles, i = ic / (w.chunks - 1);
    const int32_t chunk = (int32_t)(ic - i * (w.chunks - 1));
    const uint32_t* tok = w.tok + i * a.T;
    const int32_t end = (chunk + 1) * kChunk;            // a place there is: this is not the last chunk
    const uint32_t v = tok[end - 1], next = tok[end], before = tok[max(chunk * kChunk - 1, 0)];       // (at once: a wait each would triple it)
    if (v >= (uint32_t)a.V || next != v || (chunk > 0 && before == v)) continue;     // no token, or done, or begun earlier
    const Columns<VEC> col((int32_t)(unit - ic * w.tiles) * 64 * VEC + lane * VEC, a.h);
    const float* part = w.partial + (i * w.chunks + chunk) * 2 * w.pitch;
    float sum[VEC];
    {
      const Pack<float, VEC> p = Pack<float, VEC>::load(part + w.pitch + (col.some ? col.at : 0));
#pragma unroll
      for (int k = 0; k < VEC; ++k) sum[k] = p.get(k);
    }
    for (int32_t c = chunk + 1; c < w.chunks; c += 64) {
      // chunks that begin with the token: a run of them, its end by ballot
      const uint64_t mine = __ballot(c + lane < w.chunks && tok[(int64_t)min(c + lane, w.chunks - 1) * kChunk] == v);
      const int32_t run = mine == ~0ull ? 64 : __builtin_ctzll(~mine);
      constexpr int kAhead = 16;
      for (int32_t k0 = 0; k0 < run; k0 += kAhead) {
        Pack<float, VEC> p[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
          p[j] = Pack<float, VEC>::load(part + (int64_t)(c - chunk + min(k0 + j, run - 1)) * 2 * w.pitch + (col.some ? col.at : 0));
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
          if (k0 + j < run) {
#pragma unroll
            for (int k = 0; k < VEC; ++k) sum[k] += p[j].get(k);
          }
      }
      if (run < 64) break;
    }
    float* row = a.dE + i * a.lde + (int64_t)v * a.ldr;
    if (col.some) {
      const Pack<float, VEC> old = ADD ? Pack<float, VEC>::load(row + col.at) : Pack<float, VEC>{};
#pragma unroll
      for (int k = 0; k < VEC; ++k) sum[k] = ADD ? __builtin_fmaf(a.scale, sum[k], old.get(k)) : a.scale * sum[k];
      col.store(row, sum);
    }
  }
}

// Up to 64 NT positions: a wavefront holds all of an agent's tokens, NT a lane.  The first position of each token adds up its
// rows; other wavefronts write the zeros of rows that none of the tokens names.  One launch.
template <typename T, int VEC, int NT, bool ADD>
__global__ __launch_bounds__(256) void few_positions_kernel(EmbedArgs a, int32_t tiles, int32_t run, int64_t runs) {
  const int lane = threadIdx.x % 64;
  const int64_t sums = (int64_t)a.n * a.T * tiles, units = sums + (ADD ? 0 : a.n * runs);
  for (int64_t unit = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / 64); unit < units; unit += (int64_t)gridDim.x * 4) {
    const bool adds = unit < sums;
    const int64_t i = adds ? unit / ((int64_t)a.T * tiles) : (unit - sums) / runs;
    int32_t tok[NT];
#pragma unroll
    for (int k = 0; k < NT; ++k) tok[k] = k * 64 + lane < a.T ? a.tokens[i * a.T + k * 64 + lane] : -1;
    if (adds) {
      const int32_t rest = (int32_t)(unit - i * ((int64_t)a.T * tiles)), t = rest / tiles;
      const int32_t v = a.tokens[i * a.T + t];
      if (v < 0 || v >= a.V) continue;
      uint64_t hits[NT];
      bool earlier = false;
#pragma unroll
      for (int k = 0; k < NT; ++k) {
        hits[k] = __ballot(tok[k] == v);
        earlier |= t > k * 64 && (hits[k] & (t - k * 64 >= 64 ? ~0ull : (1ull << (t - k * 64)) - 1)) != 0;
      }
      if (earlier) continue;
      const Columns<VEC> col((rest - t * tiles) * 64 * VEC + lane * VEC, a.h);
      if (!col.some) continue;
      const T* G = static_cast<const T*>(a.rows) + i * a.T * a.ldo + col.at;
      float* row = a.dE + i * a.lde + (int64_t)v * a.ldr;
      const Pack<float, VEC> old = ADD ? Pack<float, VEC>::load(row + col.at) : Pack<float, VEC>{};
      float sum[VEC];
#pragma unroll
      for (int c = 0; c < VEC; ++c) sum[c] = 0.0f;
#pragma unroll
      for (int k = 0; k < NT; ++k)
        for (uint64_t m = hits[k]; m;) {
          // up to eight rows at once (past the last one that row again)
          Pack<T, VEC> g[8];
          int some = 0, at = 0;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            if (m) {
              at = __builtin_ctzll(m);
              m &= m - 1;
              ++some;
            }
            g[j] = Pack<T, VEC>::load(G + (int64_t)(k * 64 + at) * a.ldo);
          }
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (j < some) {
#pragma unroll
              for (int c = 0; c < VEC; ++c) sum[c] += g[j].get(c);
            }
        }
#pragma unroll
      for (int c = 0; c < VEC; ++c) sum[c] = ADD ? __builtin_fmaf(a.scale, sum[c], old.get(c)) : a.scale * sum[c];
      col.store(row, sum);
    } else {
      const int32_t v0 = (int32_t)(unit - sums - i * runs) * run, v1 = (int32_t)min((int64_t)v0 + run, (int64_t)a.V);
      float* e = a.dE + i * a.lde;
      bool some = false;
#pragma unroll
      for (int k = 0; k < NT; ++k) some |= __ballot(tok[k] >= v0 && tok[k] < v1) != 0;
      const bool pieces = some || a.ldr != a.h;
      for (int32_t v = v0; v < v1; v = pieces ? v + 1 : v1) {
        bool named = false;
        if (some) {
#pragma unroll
          for (int k = 0; k < NT; ++k) named |= __ballot(tok[k] == v) != 0;
        }
        if (named) continue;
        float* p = e + v * a.ldr;
        const int64_t count = pieces ? a.h : (int64_t)(v1 - v0) * a.h, groups = count / 4;
        for (int64_t g = lane; g < groups; g += 64) st_stream<vf4>(p + 4 * g, vf4{0.0f, 0.0f, 0.0f, 0.0f});
        if (groups * 4 + lane < count) p[groups * 4 + lane] = 0.0f;
      }
    }
  }
}

constexpr int64_t kMostBlocks = 1 << 20, kMostZeros = 15 << 20;    // a launch has fewer than 2^32 threads

// Rows of about `floats` floats.
int32_t run_of(const EmbedArgs& a, int64_t floats) { return (int32_t)std::max<int64_t>(std::min<int64_t>(floats / a.h, a.V), 1); }
uint32_t four_a_block(int64_t units) { return (uint32_t)std::min((units + 3) / 4, kMostBlocks); }

// Columns a lane takes: short rows keep enough lanes with columns of their own.
int32_t columns_of(int32_t h) { return h > 128 ? 4 : h > 64 ? 2 : 1; }
int32_t tiles_of(int32_t h, int32_t vec) { return (h + 64 * vec - 1) / (64 * vec); }
// Four positions a wavefront once there are wavefronts enough (31 x 2048 positions of 512 bf16: 31.2 us, with two 33.5, eight 33.6).
int32_t positions_of(int64_t rows, int32_t tiles) { return rows * tiles >= 1 << 14 ? 4 : 1; }

template <typename T, int VEC> hipError_t lookup(const EmbedArgs& a, hipStream_t st) {
  const int32_t tiles = tiles_of(a.h, VEC);
  const int64_t rows = (int64_t)a.n * a.T;
  if (positions_of(rows, tiles) == 4) embed_kernel<T, VEC, 4><<<dim3(four_a_block((rows + 3) / 4 * tiles)), dim3(256), 0, st>>>(a, tiles);
  else embed_kernel<T, VEC, 1><<<dim3(four_a_block(rows * tiles)), dim3(256), 0, st>>>(a, tiles);
  return hipGetLastError();
}
template <typename T> struct Lookup {
  static hipError_t go(const EmbedArgs& a, hipStream_t st) {
    const int32_t vec = columns_of(a.h);
    return vec == 4 ? lookup<T, 4>(a, st) : vec == 2 ? lookup<T, 2>(a, st) : lookup<T, 1>(a, st);
  }
};

template <typename T, int VEC, int NT> hipError_t few_positions(const EmbedArgs& a, hipStream_t st) {
  const int32_t tiles = tiles_of(a.h, VEC), run = run_of(a, 1024);
  const int64_t runs = (a.V + (int64_t)run - 1) / run;
  const int64_t units = (int64_t)a.n * a.T * tiles + (a.accumulate ? 0 : a.n * runs);
  if (units == 0) return hipSuccess;
  if (a.accumulate) few_positions_kernel<T, VEC, NT, true><<<dim3(four_a_block(units)), dim3(256), 0, st>>>(a, tiles, run, runs);
  else few_positions_kernel<T, VEC, NT, false><<<dim3(four_a_block(units)), dim3(256), 0, st>>>(a, tiles, run, runs);
  return hipGetLastError();
}

// The zeros of all tables for workgroups of `floats` floats: one piece where nothing lies between the tables, else one per table
// (fewer than 2^43 bytes: workgroups fit 32 bits).
ZeroArgs zero_args(const EmbedArgs& a, int64_t floats) {
  const bool whole = a.n == 1 || a.lde == (int64_t)a.V * a.h;
  const int64_t count = (whole ? a.n : 1) * (int64_t)a.V * a.h, blocks = (count + floats - 1) / floats;
  return ZeroArgs{a.dE, count, a.lde, (uint32_t)blocks, (uint32_t)(blocks * (whole ? 1 : a.n))};
}
// Few zeros (up to 64 MB) go with the sort's launch: a launch less (5 x 9196 positions, V = 10705, h = 48 47 -> 37 us); more are faster on
// their own.
constexpr int64_t kFewZeros = 16 << 20;
bool zeros_ride(const EmbedArgs& a) {
  return a.ldr == a.h && (int64_t)a.n * a.V * a.h <= kFewZeros && zero_args(a, 4096).all <= 1u << 16;
}
// Who writes the zeros of sorted positions' tables.
enum ZeroForm : int { ZEROS_NONE = 0, ZEROS_WITH_SORT = 1, ZEROS_ALONE = 2, ZEROS_BY_ROW = 3 };
ZeroForm zero_form(const EmbedArgs& a) { return a.accumulate ? ZEROS_NONE : zeros_ride(a) ? ZEROS_WITH_SORT : a.ldr == a.h ? ZEROS_ALONE : ZEROS_BY_ROW; }
hipError_t zeros(const EmbedArgs& a, ZeroForm form, hipStream_t st) {
  if (form == ZEROS_BY_ROW) {
    zero_rows_kernel<<<dim3(four_a_block((int64_t)a.n * a.V)), dim3(256), 0, st>>>(a);
    return hipGetLastError();
  }
  const ZeroArgs z = zero_args(a, 1024);
  zeros_kernel<<<dim3((uint32_t)std::min<int64_t>(z.all, kMostZeros)), dim3(256), 0, st>>>(z);
  return hipGetLastError();
}

// Tokens a lane holds of positions that are not sorted, and positions a thread has of those that one workgroup sorts.
int32_t few_of(int64_t T) { return T <= 64 ? 1 : T <= 256 ? 4 : 16; }
int32_t keys_of(int64_t T) { return T <= 1024 ? 1 : T <= 2048 ? 2 : T <= 4096 ? 4 : 8; }

template <int IPT> hipError_t sort_lds(const EmbedArgs& a, const EmbedGradPlan& p, const ZeroArgs& z, hipStream_t st) {
  const size_t lds = (16 * kDigits + 16 + IPT * 1024) * sizeof(uint32_t);
  if (lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(&sort_lds_kernel<IPT>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  const uint32_t sorts = (uint32_t)std::min(a.n, 1 << 16);
  sort_lds_kernel<IPT><<<dim3(sorts + z.all), dim3(1024), lds, st>>>(a, p, z, sorts);
  return hipGetLastError();
}

template <typename T, int VEC> hipError_t gradient(const EmbedArgs& a, const EmbedGradPlan& p, hipStream_t st) {
  if (p.small) {
    const int32_t few = few_of(a.T);
    return few == 1 ? few_positions<T, VEC, 1>(a, st) : few == 4 ? few_positions<T, VEC, 4>(a, st) : few_positions<T, VEC, 16>(a, st);
  }
  char* ws = static_cast<char*>(a.workspace);
  auto words = [&](int64_t at) { return reinterpret_cast<uint32_t*>(ws + at); };
  uint32_t *tok = words(p.tok0), *pos = words(p.pos0);
  const ZeroForm form = zero_form(a);
  const ZeroArgs z = form == ZEROS_WITH_SORT ? zero_args(a, 4096) : ZeroArgs{};
  hipError_t e = form == ZEROS_ALONE || form == ZEROS_BY_ROW ? zeros(a, form, st) : hipSuccess;
  if (e != hipSuccess) return e;
  if (p.lds) {
    const int32_t keys = keys_of(a.T);
    e = keys == 1 ? sort_lds<1>(a, p, z, st) : keys == 2 ? sort_lds<2>(a, p, z, st) : keys == 4 ? sort_lds<4>(a, p, z, st) : sort_lds<8>(a, p, z, st);
  } else {
    uint32_t *tok2 = words(p.tok1), *pos2 = words(p.pos1);
    const dim3 grid((uint32_t)std::min((int64_t)a.n * p.tiles, kMostBlocks));
    for (int k = 0; k < p.passes && e == hipSuccess; ++k) {
      const PassArgs q{k ? nullptr : a.tokens, tok, pos, tok2, pos2, words(p.hist), a.n, a.V, a.T, p.tiles, p.hist_rows, k * p.digit_bits,
                       std::min(p.digit_bits, p.bits - k * p.digit_bits)};
      const ZeroArgs zk = k ? ZeroArgs{} : z;
      const dim3 counts(grid.x + zk.all);
      if (tile_of_sort(a.T) == 1024) {
        count_digits_kernel<1><<<counts, dim3(1024), 0, st>>>(q, zk, grid.x);
        place_keys_kernel<1><<<grid, dim3(1024), 0, st>>>(q);
      } else {
        count_digits_kernel<4><<<counts, dim3(1024), 0, st>>>(q, zk, grid.x);
        if (q.hist_rows > q.tiles) sum_counts_kernel<<<dim3(four_a_block((int64_t)a.n * kDigits)), dim3(256), 0, st>>>(q);
        place_keys_kernel<4><<<grid, dim3(1024), 0, st>>>(q);
      }
      e = hipGetLastError();
      std::swap(tok, tok2);
      std::swap(pos, pos2);
    }
  }
  if (e != hipSuccess) return e;
  WalkArgs w{a, tok, pos, reinterpret_cast<float*>(ws + p.partial), p.pitch, p.chunks, tiles_of(a.h, VEC)};
  const dim3 walk(four_a_block((int64_t)a.n * p.chunks * w.tiles)), join(four_a_block((int64_t)a.n * (p.chunks - 1) * w.tiles));
  if (a.accumulate) {
    walk_kernel<T, VEC, true><<<walk, dim3(256), 0, st>>>(w);
    join_kernel<VEC, true><<<join, dim3(256), 0, st>>>(w);
  } else {
    walk_kernel<T, VEC, false><<<walk, dim3(256), 0, st>>>(w);
    join_kernel<VEC, false><<<join, dim3(256), 0, st>>>(w);
  }
  return hipGetLastError();
}

template <typename T> struct Gradient {
  static hipError_t go(const EmbedArgs& a, hipStream_t st) {
    const EmbedGradPlan p = plan_embed_grad(a.n, a.V, a.h, a.T);
    const int32_t vec = columns_of(a.h);
    return vec == 4 ? gradient<T, 4>(a, p, st) : vec == 2 ? gradient<T, 2>(a, p, st) : gradient<T, 1>(a, p, st);
  }
};

template <template <typename> class Launch, typename... A> hipError_t by_type(int type, A... args) {
  if (type == TYPE_F32) return Launch<float>::go(args...);
  if (type == TYPE_BF16) return Launch<bf16_t>::go(args...);
  return Launch<_Float16>::go(args...);
}

}  // namespace

void describe_embed(const EmbedArgs& a, int32_t* out) {
  out[0] = columns_of(a.h);
  out[1] = positions_of((int64_t)a.n * a.T, tiles_of(a.h, out[0]));
}
void describe_embed_grad(const EmbedArgs& a, int32_t* out) {
  const EmbedGradPlan p = plan_embed_grad(a.n, a.V, a.h, a.T);
  out[0] = columns_of(a.h);
  out[1] = p.small ? few_of(a.T) : 0;
  out[2] = !p.small && p.lds ? keys_of(a.T) : 0;
  out[3] = !p.small && !p.lds ? tile_of_sort(a.T) : 0;
  out[4] = p.small ? ZEROS_NONE : zero_form(a);
  out[5] = !p.small && p.hist_rows > p.tiles;
}

hipError_t launch_embed(const EmbedArgs& a, hipStream_t st) { return by_type<Lookup>(a.type, a, st); }
hipError_t launch_embed_grad(const EmbedArgs& a, hipStream_t st) { return by_type<Gradient>(a.type, a, st); }

}  // namespace ceca
