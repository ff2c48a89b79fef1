// The largest logits of a row and their places.
//
// What bounds it: the row is read once.  A workgroup holds a row (or a part of it) in registers and looks for a threshold that at least
// K logits reach and few more: the K-th largest of the maxima of its threads' shares does, since every share that reaches it has
// such a logit.  What reaches the threshold goes to LDS, where a candidate's rank is the number of candidates before it.
// Where too many do (equal logits, few shares), the K-th largest logit itself is found bit by bit, and among its equals the
// last place that still belongs.  Candidates are ordered by one word of (value, place): the same result whatever the order in which
// they were put into LDS.
#include <algorithm>
#include <type_traits>

#include "device_util.h"
#include "text_util.h"

namespace ceca {

namespace {

// Order of the logits as whole numbers of kBits<T> bits: -inf < ... < -0 = +0 < ... < +inf < NaN.
template <typename T> constexpr int kBits = 8 * (int)sizeof(T);
template <typename T> struct Order;
template <> struct Order<float> {
  static constexpr uint32_t sign = 0x80000000u, all = 0xffffffffu, inf = 0x7f800000u;
  __device__ static __forceinline__ uint32_t raw(float x) { return __float_as_uint(x); }
  __device__ static __forceinline__ float value(uint32_t b) { return __uint_as_float(b); }
};
template <> struct Order<bf16_t> {
  static constexpr uint32_t sign = 0x8000u, all = 0xffffu, inf = 0x7f80u;
  __device__ static __forceinline__ uint32_t raw(float x) { return __float_as_uint(x) >> 16; }        // (x came from one: exact)
  __device__ static __forceinline__ float value(uint32_t b) { return __uint_as_float(b << 16); }
};
template <> struct Order<_Float16> {
  static constexpr uint32_t sign = 0x8000u, all = 0xffffu, inf = 0x7c00u;
  __device__ static __forceinline__ uint32_t raw(float x) { return __builtin_bit_cast(uint16_t, (_Float16)x); }
  __device__ static __forceinline__ float value(uint32_t b) { return (float)__builtin_bit_cast(_Float16, (uint16_t)b); }
};
template <typename T> __device__ __forceinline__ uint32_t key_of(float x) {
  using O = Order<T>;
  uint32_t b = O::raw(x + 0.0f);                              // -0 becomes +0
  if (x != x) b = O::inf | 1;                                 // one NaN for all
  return b & O::sign ? ~b & O::all : b | O::sign;
}
template <typename T> __device__ __forceinline__ float value_of(uint32_t key) {
  using O = Order<T>;
  return O::value(key & O::sign ? key ^ O::sign : ~key & O::all);
}
template <typename T> constexpr uint32_t kLeastKey = (~(Order<T>::inf | Order<T>::sign) & Order<T>::all) + 1;    // above -inf

// Candidates that a workgroup's LDS holds: fewer for single wavefronts, of which a compute unit has more.
constexpr int most_candidates(int threads) { return threads == 64 ? 512 : 1024; }

// Candidates in LDS to their ranks: the K first go out, as values and places or, from a part of a row, as they are.  A thread
// takes up to four at a time, which share what it reads.
template <typename T, int THREADS>
__device__ __forceinline__ void rank_and_store(const uint64_t* cand, int count, int K, float* top, int32_t* ids, uint64_t* words) {
  constexpr int AT_ONCE = 4;
  for (int c0 = threadIdx.x; c0 < count; c0 += THREADS * AT_ONCE) {
    uint64_t own[AT_ONCE];
    int rank[AT_ONCE];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      own[i] = c0 + i * THREADS < count ? cand[c0 + i * THREADS] : ~0ull;
      rank[i] = 0;
    }
    if (count <= THREADS) {
#pragma unroll 8
      for (int j = 0; j < count; ++j) rank[0] += cand[j] > own[0];
    } else {
#pragma unroll 4
      for (int j = 0; j < count; ++j) {
        const uint64_t other = cand[j];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) rank[i] += other > own[i];
      }
    }
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      if (c0 + i * THREADS >= count || rank[i] >= K) continue;
      if (words) {
        words[rank[i]] = own[i];
      } else {
        top[rank[i]] = value_of<T>((uint32_t)(own[i] >> 32));
        ids[rank[i]] = (int32_t)~(uint32_t)own[i];
      }
    }
  }
  for (int c = count + threadIdx.x; c < K; c += THREADS) {    // fewer than K that are not masked
    if (words) {
      words[c] = 0;
    } else {
      top[c] = -kInf;
      ids[c] = -1;
    }
  }
}

// Whole numbers over the workgroup (below 2^24: fp32 sums are exact).
template <int THREADS> __device__ __forceinline__ int count_all(int mine, float* slot) {
  const float w = wave_all((float)mine, Add());
  if (THREADS == 64) return (int)w;
  __syncthreads();
  if (threadIdx.x % 64 == 0) slot[threadIdx.x / 64] = w;
  __syncthreads();
  float sum = 0.0f;
#pragma unroll
  for (int k = 0; k < THREADS / 64; ++k) sum += slot[k];
  return (int)sum;
}

template <typename T, int THREADS, int NP>
__global__ __launch_bounds__(THREADS, NP == 16 ? 4 : 1) void top_kernel(TopArgs a, TopPlan plan) {
  constexpr int VEC = kVec<T>, WAVES = THREADS / 64;
  using P = Pack<T, VEC>;
  // shares of a thread, 512 in all where there are packs enough
  constexpr int SHARES = THREADS > 64 ? 2 : NP < 8 ? NP : 8, MOST = most_candidates(THREADS);
  __shared__ uint64_t cand[MOST];
  __shared__ uint32_t group[SHARES * THREADS], threshold;
  __shared__ float slot[WAVES];
  __shared__ int found;
  const int tid = threadIdx.x;
  for (int64_t unit = blockIdx.x; unit < (int64_t)a.rows * plan.parts; unit += gridDim.x) {
    const int64_t row = unit / plan.parts;
    const int32_t c0 = (int32_t)(unit - row * plan.parts) * plan.cols, cols = min(plan.cols, a.V - c0);
    const T* s = static_cast<const T*>(a.logits) + row * a.ld + c0;
    // packs as in the distillation's register tiles: by their distance from the beginning, the last one in place of those past it
    const int32_t packed = cols / VEC * VEC, tail = cols - packed;
    const uint32_t bytes = (uint32_t)packed * sizeof(T), last = bytes ? bytes - 16 : 0;
    uint32_t mine = tid * 16;
    auto at = [&](int j) { return mine + (uint32_t)(j * THREADS * 16); };
    auto there = [&](int j) { return at(j) < bytes; };
    P x[NP];
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      if (bytes) {
        x[j] = P::load_stream(reinterpret_cast<const T*>(reinterpret_cast<const char*>(s) + min(at(j), last)));
      } else {
#pragma unroll
        for (int c = 0; c < VEC; ++c) x[j].set(c, -kInf);
      }
    }
    float xt = tid < tail ? to_float(s[packed + tid]) : -kInf;
    __syncthreads();                                           // (LDS of the unit before)
    if (tid == 0) found = 0;

    const uint32_t key_t = key_of<T>(xt);
    auto put = [&](uint32_t key, int32_t place) {
      const int k = atomicAdd(&found, 1);
      if (k < MOST) cand[k] = (uint64_t)key << 32 | (uint32_t)~place;
    };

    // the largest of every share; a pack past the last one must not count twice
    uint32_t t = 0;
    {
      float g[SHARES];
#pragma unroll
      for (int e = 0; e < SHARES; ++e) g[e] = e ? -kInf : xt;
#pragma unroll
      for (int j = 0; j < NP; ++j) {
        float best = x[j].get(0);
#pragma unroll
        for (int c = 1; c < VEC; ++c) best = fmaxf(best, x[j].get(c));
        g[j % SHARES] = fmaxf(g[j % SHARES], there(j) ? best : -kInf);
        __builtin_amdgcn_sched_barrier(0);
      }
      // the K-th largest of them, from above, to 20 bits (what the others may add are few candidates more), by one wavefront
      auto search = [&](auto&& key, auto each) {
        for (int bit = kBits<T> - 1; bit >= std::max(kBits<T> - 20, 0); --bit) {
          const uint32_t t1 = t | 1u << bit;
          int n = 0;
#pragma unroll
          for (int e = 0; e < decltype(each)::value; ++e) n += __builtin_popcountll(__ballot(key[e] >= t1));
          if (n >= a.K) t = t1;
          if (n == a.K) break;
        }
      };
      if constexpr (WAVES == 1) {
        uint32_t key[SHARES];
#pragma unroll
        for (int e = 0; e < SHARES; ++e) key[e] = key_of<T>(g[e]);
        search(key, std::integral_constant<int, SHARES>());
        __syncthreads();
      } else {
#pragma unroll
        for (int e = 0; e < SHARES; ++e) group[e * THREADS + tid] = key_of<T>(g[e]);
        __syncthreads();
        if (tid < 64) {
          constexpr int EACH = SHARES * THREADS / 64;
          uint32_t key[EACH];
#pragma unroll
          for (int e = 0; e < EACH; ++e) key[e] = group[e * 64 + tid];
          search(key, std::integral_constant<int, EACH>());
          if (tid == 0) threshold = t;
        }
        __syncthreads();
        t = threshold;
      }
    }
    // (from a small tile the long way is shorter than ranking many: taken at once where fewer shares than K were found to hold any)
    constexpr bool KEPT = THREADS == 64 && NP <= 4;
    if (KEPT && t == 0 && cols > kTopMax) {
      if (tid == 0) found = kTopMax + 1;
      __syncthreads();
    } else {
      const float least = value_of<T>(max(t, kLeastKey<T>));
      asm volatile("" : "+v"(mine));
#pragma unroll
      for (int j = 0; j < NP; ++j) {
        x[j].again();
        bool some = false;
#pragma unroll
        for (int c = 0; c < VEC; ++c) some |= !(x[j].get(c) < least);           // (NaN too)
        if (there(j) && some) {
          x[j].again();
#pragma unroll
          for (int c = 0; c < VEC; ++c)
            if (!(x[j].get(c) < least)) put(key_of<T>(x[j].get(c)), c0 + (int32_t)(at(j) / sizeof(T)) + c);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      if (tid < tail && !(xt < least)) put(key_t, c0 + packed + tid);
      __syncthreads();
    }
    if (found > (KEPT ? kTopMax : MOST)) {
      // f(key, place) for every logit of this thread: from the keys of a small tile, else from memory once more (kept for the few rows
      // that come here, a large tile's logits would cost every row registers); 0 stands for none
      uint32_t key[KEPT ? NP * VEC : 1];
      if constexpr (KEPT) {
#pragma unroll
        for (int j = 0; j < NP; ++j)
#pragma unroll
          for (int c = 0; c < VEC; ++c) key[j * VEC + c] = there(j) ? key_of<T>(x[j].get(c)) : 0;
      }
      auto each = [&](auto&& f) {
        if constexpr (KEPT) {
#pragma unroll
          for (int j = 0; j < NP; ++j)
#pragma unroll
            for (int c = 0; c < VEC; ++c) f(key[j * VEC + c], c0 + (int32_t)(at(j) / sizeof(T)) + c);
        } else {
          for (int32_t c = tid * VEC; c < packed; c += THREADS * VEC) {
            const P y = P::load(s + c);
#pragma unroll
            for (int k = 0; k < VEC; ++k) f(key_of<T>(y.get(k)), c0 + c + k);
          }
        }
        f(key_t, c0 + packed + tid);
      };
      // the K-th largest key, bit by bit; masked logits are none
      auto count = [&](auto&& is) {
        int n = 0;
        each([&](uint32_t key, int32_t place) { n += is(key, place) ? 1 : 0; });
        return count_all<THREADS>(n, slot);
      };
      t = 0;
      int reach = 0;                                           // logits that reach it
      for (int bit = kBits<T> - 1; bit >= 0; --bit) {
        const uint32_t t1 = t | 1u << bit;
        const int n = count([&](uint32_t key, int32_t) { return key >= max(t1, kLeastKey<T>); });
        if (n >= a.K) {
          t = t1;
          reach = n;
        }
        if (n == a.K) break;                                   // just these
      }
      t = max(t, kLeastKey<T>);
      // more than K: how many of the K-th's equals belong, and the place of the last of them
      int32_t end = 0x7fffffff;
      if (reach > a.K) {
        const int need = a.K - count([&](uint32_t key, int32_t) { return key > t; });
        end = 0;
        for (int bit = 31 - __builtin_clz((uint32_t)a.V | 1); bit >= 0; --bit) {
          const int32_t end1 = end + (1 << bit);
          if (count([&](uint32_t key, int32_t place) { return key == t && place < end1; }) < need) end = end1;
        }
      }
      __syncthreads();
      if (tid == 0) found = 0;
      __syncthreads();
      each([&](uint32_t key, int32_t place) {
        if (key > t || (key == t && place <= end)) put(key, place);
      });
      __syncthreads();
    }
    float* top = a.top + row * a.K;
    int32_t* ids = a.ids + row * a.K;
    rank_and_store<T, THREADS>(cand, min(found, MOST), a.K, top, ids, plan.parts > 1 ? static_cast<uint64_t*>(a.workspace) + unit * a.K : nullptr);
  }
}

// One list of K from up to `per` of a row's `lists` lists of K (each from the largest down, zeros behind).  With m lists that have r
// words each no smaller than some word, m r >= K, at least K words reach it: the m-th largest of the lists' r-th words, with r
// about twice their share of K.  Where too many reach it, the K-th largest is found bit by bit (all words but zeros differ).
constexpr int kMergeThreads = 256, kMergeEach = kMergeWords / kMergeThreads;
struct MergeArgs {
  TopArgs a;
  const uint64_t* in;
  uint64_t* out;               // null: to top and ids
  int32_t lists, per, groups;  // per row: lists, lists per workgroup, workgroups
};
template <typename T>
__global__ __launch_bounds__(kMergeThreads) void top_merge_kernel(MergeArgs m) {
  constexpr int MOST = most_candidates(kMergeThreads);
  __shared__ uint64_t cand[MOST];
  __shared__ uint64_t least;
  __shared__ float slot[kMergeThreads / 64];
  __shared__ int found;
  const int tid = threadIdx.x, K = m.a.K;
  for (int64_t unit = blockIdx.x; unit < (int64_t)m.a.rows * m.groups; unit += gridDim.x) {
    const int64_t row = unit / m.groups;
    const int32_t first = (int32_t)(unit - row * m.groups) * m.per, lists = min(m.per, m.lists - first), all = lists * K;
    const uint64_t* words = m.in + (row * m.lists + first) * K;
    uint64_t w[kMergeEach];
#pragma unroll
    for (int e = 0; e < kMergeEach; ++e) w[e] = e * kMergeThreads + tid < all ? words[e * kMergeThreads + tid] : 0;
    const int some = min(lists, kMergeThreads), r = min((2 * K + some - 1) / some, K), at = (K + r - 1) / r - 1;
    const uint64_t rth = tid < some ? words[tid * K + r - 1] : 0;
    __syncthreads();
    cand[tid] = rth;
    if (tid == 0) {
      found = 0;
      least = 1;
    }
    __syncthreads();
    int rank = 0;
    for (int j = 0; j < some; ++j) rank += cand[j] > rth || (cand[j] == rth && j < tid);
    if (tid < some && rank == at && rth > 1) least = rth;
    __syncthreads();
    uint64_t t = least;
    auto collect = [&]() {               // (cand is read no more: a barrier lies between)
#pragma unroll
      for (int e = 0; e < kMergeEach; ++e)
        if (w[e] >= t) {
          const int k = atomicAdd(&found, 1);
          if (k < MOST) cand[k] = w[e];
        }
      __syncthreads();
    };
    collect();
    if (found > MOST) {
      t = 0;
      for (int bit = 31 + kBits<T>; bit >= 0; --bit) {
        const uint64_t t1 = t | 1ull << bit;
        int n = 0;
#pragma unroll
        for (int e = 0; e < kMergeEach; ++e) n += w[e] >= t1;
        if (count_all<kMergeThreads>(n, slot) >= K) t = t1;
      }
      t = max(t, (uint64_t)1);
      __syncthreads();
      if (tid == 0) found = 0;
      __syncthreads();
      collect();
    }
    rank_and_store<T, kMergeThreads>(cand, min(found, MOST), K, m.a.top + row * K, m.a.ids + row * K, m.out ? m.out + unit * K : nullptr);
  }
}

constexpr int64_t kMostTopBlocks = 1 << 22;

// A workgroup's threads and the packs that each holds.
struct TopTile { int32_t threads, packs; };
TopTile tile_of(const TopPlan& plan, int64_t rows, int type) {
  const int32_t packs = plan.cols / (type == TYPE_F32 ? 4 : 8);
  // 256 threads with up to 16 packs each: several rows on a compute unit, of which some load while others look for their threshold
  // (7936 rows of 32000 bf16, K = 64: 120 us; 512 threads with 8 packs 140, 128 with 32 212, 1024 with 4 376).  Longer rows
  // in parts: 1000 rows of 33216 fp32, K = 157, 67 us, in one tile of 512 threads 89.  Many short rows by a wavefront each, which
  // needs no barriers (87219 rows of 2304 bf16, K = 6: 143 us, by 256 threads 313); few of them are done sooner by more threads.
  if (packs <= 64) return {64, 1};
  if (packs <= 64 * 4) return {64, 4};
  if (packs <= 256 * 4 && rows * plan.parts <= 2048) return {256, 4};
  if (packs <= 64 * 8) return {64, 8};
  if (packs <= 64 * 16) return {64, 16};
  return {256, packs <= 256 * 8 ? 8 : 16};
}
MergeArgs merge_of(const TopArgs& a, const uint64_t* in, uint64_t* out, int32_t lists) {
  MergeArgs m{a, in, out, lists, kMergeWords / a.K, 0};
  m.groups = (lists + m.per - 1) / m.per;
  return m;
}

template <typename T> hipError_t launch(const TopArgs& a, hipStream_t st) {
  const TopPlan plan = plan_top(a.rows, a.V, a.K, a.type);
  const TopTile tile = tile_of(plan, a.rows, a.type);
  const dim3 grid((uint32_t)std::min((int64_t)a.rows * plan.parts, kMostTopBlocks)), block(tile.threads);
  if (tile.threads == 64) {
    if (tile.packs == 1) top_kernel<T, 64, 1><<<grid, block, 0, st>>>(a, plan);
    else if (tile.packs == 4) top_kernel<T, 64, 4><<<grid, block, 0, st>>>(a, plan);
    else if (tile.packs == 8) top_kernel<T, 64, 8><<<grid, block, 0, st>>>(a, plan);
    else top_kernel<T, 64, 16><<<grid, block, 0, st>>>(a, plan);
  } else {
    if (tile.packs == 4) top_kernel<T, 256, 4><<<grid, block, 0, st>>>(a, plan);
    else if (tile.packs == 8) top_kernel<T, 256, 8><<<grid, block, 0, st>>>(a, plan);
    else top_kernel<T, 256, 16><<<grid, block, 0, st>>>(a, plan);
  }
  uint64_t *in = static_cast<uint64_t*>(a.workspace), *out = in + plan.second / 8;
  for (int32_t lists = plan.parts; lists > 1;) {
    MergeArgs m = merge_of(a, in, out, lists);
    if (m.groups == 1) m.out = nullptr;
    top_merge_kernel<T><<<dim3((uint32_t)std::min((int64_t)a.rows * m.groups, kMostTopBlocks)), dim3(kMergeThreads), 0, st>>>(m);
    lists = m.groups;
    std::swap(in, out);
  }
  return hipGetLastError();
}

}  // namespace

TopPlan plan_top(int64_t rows, int32_t V, int32_t K, int type) {
  TopPlan p{};
  const int32_t vec = type == TYPE_F32 ? 4 : 8, most = 256 * 16 * vec;     // columns of the largest register tile
  // parts that registers hold; few rows of more than 32768 columns in parts of about 4096, up to 1024 workgroups and one merge
  // (64 rows of 84864 bf16: parts of 4096 17.0 us, of 32768 20.0; 286 rows of 28571: in one 12.2 us, in parts 14.8)
  int64_t parts = (V + (int64_t)most - 1) / most;
  if (rows > 0 && V > 32768) parts = std::max(parts, std::min<int64_t>({(V + 4095) / 4096, 1024 / rows, kMergeWords / K}));
  parts = std::max<int64_t>(parts, 1);
  p.cols = (int32_t)(((V + parts - 1) / parts + vec - 1) / vec * vec);
  p.parts = (V + p.cols - 1) / p.cols;
  if (p.parts > 1) {
    const int64_t groups = (p.parts + kMergeWords / K - 1) / (kMergeWords / K);
    p.second = (rows * p.parts * K * 8 + 255) / 256 * 256;
    p.bytes = p.second + (groups > 1 ? (rows * groups * K * 8 + 255) / 256 * 256 : 0);
  }
  return p;
}

void describe_top(int64_t rows, int32_t V, int32_t K, int type, int32_t* out) {
  const TopPlan plan = plan_top(rows, V, K, type);
  const TopTile tile = tile_of(plan, rows, type);
  TopArgs a{};
  a.K = K;
  out[0] = tile.threads;
  out[1] = tile.packs;
  out[2] = plan.parts;
  out[3] = 0;
  for (int32_t lists = plan.parts; lists > 1; lists = merge_of(a, nullptr, nullptr, lists).groups) ++out[3];
}

hipError_t launch_top(const TopArgs& a, hipStream_t st) {
  if (a.type == TYPE_F32) return launch<float>(a, st);
  return a.type == TYPE_BF16 ? launch<bf16_t>(a, st) : launch<_Float16>(a, st);
}

}  // namespace ceca
