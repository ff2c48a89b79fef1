// Distillation from a teacher's top logits: loss and gradient.
//
// A row of V student logits s against K teacher entries (u_k, id_k), with tau the temperature, a the share of the hard term and
// w the row's weight (p = softmax(u / tau), q = softmax(s / tau), r = softmax(s)):
//   loss = w [(1 - a) tau^2 sum_k p_k (log p_k - log q_id_k) - a log r_label]
//   dloss / ds_v = w [(1 - a) tau (q_v - sum_{id_k = v} p_k) + a (r_v - [v = label])]
// What bounds it: the row is read once and its gradient written once; two exponentials per logit (four with two softmaxes) take
// half as long as the memory at 16 bits per logit, so the loads of one row have to run beside the arithmetic of another.
#include <algorithm>

#include "device_util.h"
#include "text_util.h"

namespace ceca {

namespace {

constexpr float kLog2e = 1.44269504088896340736f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }       // zero below 2^-126

// What is known of a row before its logits are: every thread has its entries (EPT of them).
template <int EPT> struct Entries {
  float w;
  int32_t label;
  int32_t id[EPT];
  float u[EPT];
  template <int THREADS> __device__ __forceinline__ void load(const DistillArgs& a, int64_t row) {
    w = a.weight ? a.weight[row] : 1.0f;
    label = a.labels ? a.labels[row] : -1;
    int64_t from = row;
    if (a.peer) {
      const int64_t i = row / a.T;
      from = (int64_t)min(max(a.peer[i], 0), a.n - 1) * a.T + (row - i * a.T);
    }
#pragma unroll
    for (int e = 0; e < EPT; ++e) {
      const int k = e * THREADS + threadIdx.x;
      id[e] = -1;
      u[e] = -kInf;
      if (k < a.K) {
        id[e] = a.ids[from * a.K + k];
        u[e] = a.top[from * a.K + k];
      }
    }
  }
  // an id outside the vocabulary or a value of -inf is no entry
  __device__ __forceinline__ void settle(const DistillArgs& a) {
#pragma unroll
    for (int e = 0; e < EPT; ++e) {
      if (id[e] < 0 || id[e] >= a.V) u[e] = -kInf;
      if (u[e] == -kInf) id[e] = -1;
    }
    if (label >= a.V || !(a.hard > 0.0f)) label = -1;
  }
};

// A row's entries by their places, in LDS: open addressing in twice as many slots as there are entries at most.  Every entry keeps its
// share as the fp32 number it is.  Where entries share a place, the shares are summed as whole numbers, whose order does not matter,
// of 2^-46 of the power of two at or below the place's largest share: a unit of the row's own would leave small shares no bits.
constexpr int kSlots = 2 * kTopMax;
struct alignas(16) EntryTable {
  int32_t id[kSlots];          // -1: empty
  unsigned long long cell[kSlots];             // (exponent of the largest share) 2^56 + sum, where some entries share a place
  int32_t at[kTopMax];         // an entry's place, -1: none
  float p[kTopMax];            // its share, then all of its place's
  int32_t twice;               // whether entries share places
  template <int THREADS, int EPT> __device__ __forceinline__ void begin(const Entries<EPT>& own) {
    typedef int32_t I4 __attribute__((ext_vector_type(4)));
    for (int k = threadIdx.x; k < kSlots / 4; k += THREADS) reinterpret_cast<I4*>(id)[k] = I4{-1, -1, -1, -1};
#pragma unroll
    for (int e = 0; e < EPT; ++e)
      if (THREADS <= kTopMax || threadIdx.x < kTopMax) at[e * THREADS + threadIdx.x] = own.id[e];
    if (threadIdx.x == 0) twice = 0;
  }
  __device__ static __forceinline__ uint32_t first(int32_t v) { return ((uint32_t)v * 0x9e3779b1u) >> 23; }       // of 512
  // entry e's share at its place v (v >= 0; K <= 256 of 512 slots are taken, so the search ends)
  __device__ __forceinline__ void put(int e, int32_t v, float share) {
    p[e] = share;
    uint32_t k = first(v);
    for (;;) {
      const int32_t was = atomicCAS(&id[k], -1, v);
      if (was == v) twice = 1;
      if (was == -1 || was == v) break;
      k = (k + 1) % kSlots;
    }
  }
  // p[e]: what entry e's place got, for the thread that put it (behind a barrier, by all threads)
  template <int THREADS> __device__ __forceinline__ void join(int K) {
    if (!twice) return;
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));              // (addresses worked out here: few rows come this way)
#pragma unroll 1
    for (int k = tid; k < kSlots; k += THREADS) cell[k] = 0;
    __syncthreads();
    auto cell_of = [&](int32_t v) {
      uint32_t k = first(v);
      while (id[k] != v) k = (k + 1) % kSlots;
      return &cell[k];
    };
    auto each = [&](auto&& f) {
#pragma unroll 1
      for (int e = tid; e < K; e += THREADS)
        if (at[e] >= 0) f(p[e], cell_of(at[e]));
      __syncthreads();
    };
    each([&](float x, unsigned long long* c) { atomicMax(c, (unsigned long long)(__float_as_uint(x) >> 23 & 255) << 56); });
    each([&](float x, unsigned long long* c) { atomicAdd(c, (unsigned long long)__builtin_amdgcn_ldexpf(x == x ? x : 0.0f, 127 + 46 - (int)(*c >> 56))); });
    each([&](float& x, unsigned long long* c) { x = x == x ? __builtin_amdgcn_ldexpf((float)(*c & (1ull << 56) - 1), (int)(*c >> 56) - 127 - 46) : x; });
  }
  __device__ __forceinline__ bool has(int32_t v) const {
    for (uint32_t k = first(v); id[k] != -1; k = (k + 1) % kSlots)
      if (id[k] == v) return true;
    return false;
  }
};
static_assert(kSlots == 512, "EntryTable::first");

// The factors that a row's statistics give: m (the largest logit), q and r (the sums of the exponentials at tau and at 1).
struct Factors {
  float cs, ch;        // w (1 - a), w a; zero without the term
  float gs, qs, rs, both;    // tau cs, the factors of the two exponentials in the gradient, their sum
  bool zero;           // neither term, or no logit that is not masked
  __device__ __forceinline__ Factors(const DistillArgs& a, float w, bool soft, bool labelled, float q, float r) {
    const bool some = r != 0.0f;
    cs = soft && some && a.hard < 1.0f ? w * (1.0f - a.hard) : 0.0f;
    ch = labelled && some ? w * a.hard : 0.0f;
    zero = !(soft && a.hard < 1.0f) && !labelled;
    zero = zero || !some;
    gs = cs * a.tau;
    qs = cs != 0.0f ? gs / q : 0.0f;
    rs = ch != 0.0f ? ch / r : 0.0f;
    both = qs + rs;
    asm("" : "+v"(qs), "+v"(rs), "+v"(both));      // (plain arithmetic issues faster without scalar operands)
  }
};

// TWO: exponentials at tau and at 1, both terms being asked for at a temperature other than 1; else one factor `k` for all.
template <bool TWO> struct Scales {
  float kq, kr;        // log2 e / tau, log2 e
  __device__ __forceinline__ Scales(const DistillArgs& a) {
    const bool hard_alone = a.hard >= 1.0f || a.K == 0;
    kr = in_vgpr(kLog2e);
    kq = in_vgpr(!TWO && hard_alone ? kLog2e : kLog2e / a.tau);
  }
};

template <typename T, bool TWO> __device__ __forceinline__ float gradient_at(float x, const Scales<TWO>& k, const Factors& f) {
  if (TWO) return __builtin_fmaf(f.qs, exp2_fast(x * k.kq), f.rs * exp2_fast(x * k.kr));
  return f.both * exp2_fast(x * k.kq);
}

// One entry's part of the loss before its factors: tau p (log p - log q_id), with du and x the differences of its value and its logit from
// the largest, and lu, lq the logarithms of the sums.  (Times tau: x / tau alone may pass what fp32 holds where tau < 1 and the
// logit is the lowest finite one.)
__device__ __forceinline__ float entry_term(float p, float du, float lu, float lq, float x, float tau) {
  return p != 0.0f ? p * (du - x + tau * (lq - lu)) : 0.0f;
}

// The gradient at an entry's place or at the label, all of it.
template <bool TWO> __device__ __forceinline__ float gradient_there(float x, float p_sum, bool is_label, const Scales<TWO>& k, const Factors& f, float q, float r) {
  float g = 0.0f;
  if (f.cs != 0.0f) g = f.gs * (exp2_fast(x * k.kq) / q - p_sum);
  if (f.ch != 0.0f) g += f.ch * (exp2_fast(x * (TWO ? k.kr : k.kq)) / r - (is_label ? 1.0f : 0.0f));
  return g;
}

// Running statistics of one thread's logits: their maximum and the sums of the exponentials relative to it.  The lowest finite
// number stands for "none yet": nothing but masked logits leaves sums of zero behind.
constexpr float kLowest = -3.402823466e38f;
template <bool TWO> struct Running {
  float m = kLowest, q = 0.0f, r = 0.0f;
  __device__ __forceinline__ void rise(float to, const Scales<TWO>& k) {
    const float m1 = fmaxf(m, to);
    q *= exp2_fast((m - m1) * k.kq);
    if (TWO) r *= exp2_fast((m - m1) * k.kr);
    m = m1;
  }
  __device__ __forceinline__ void add(float x, const Scales<TWO>& k) {
    rise(x, k);
    q += exp2_fast((x - m) * k.kq);
    if (TWO) r += exp2_fast((x - m) * k.kr);
  }
  // a pack, counted where `there` (its maximum may count anyway); with `risen` the maximum is known to be no less than its own
  template <typename P, int VEC> __device__ __forceinline__ void add(const P& x, bool there, const Scales<TWO>& k, bool risen = false) {
    if (!risen) {
      float best = x.get(0);
#pragma unroll
      for (int c = 1; c < VEC; ++c) best = fmaxf(best, x.get(c));
      rise(best, k);
    }
    float qs = 0.0f, rs = 0.0f;
#pragma unroll
    for (int c = 0; c < VEC; ++c) {
      const float y = x.get(c) - m;
      qs += exp2_fast(y * k.kq);
      if (TWO) rs += exp2_fast(y * k.kr);
    }
    q += there ? qs : 0.0f;
    if (TWO) r += there ? rs : 0.0f;
    asm volatile("" : "+v"(q), "+v"(r));                 // here and now: put off, the sums would keep all differences
  }
  __device__ __forceinline__ void over_wave(const Scales<TWO>& k) {
    rise(wave_all(m, Max()), k);
    q = wave_all(q, Add());
    if (TWO) r = wave_all(r, Add());
  }
  // slot[0..2]: a float per wavefront each (put before a barrier)
  __device__ __forceinline__ void put(float (*slot)[16]) const {
    if (threadIdx.x % 64 == 0) {
      slot[0][threadIdx.x / 64] = m;
      slot[1][threadIdx.x / 64] = q;
      if (TWO) slot[2][threadIdx.x / 64] = r;
    }
  }
  template <int WAVES> __device__ __forceinline__ void take(const float (*slot)[16], const Scales<TWO>& k) {
    const int w = threadIdx.x % 16;
    const bool is = w < WAVES;
    m = is ? slot[0][w] : kLowest;
    q = is ? slot[1][w] : 0.0f;
    r = TWO && is ? slot[2][w] : 0.0f;
    rise(row_all(m, Max()), k);
    // lane 0's for all: a lane's own product may be fused into its first addition, which rounds differently
    m = lane_value(m, 0);
    q = lane_value(row_all(q, Add()), 0);
    r = TWO ? lane_value(row_all(r, Add()), 0) : q;
  }
};

// ---- rows that a workgroup holds in registers ----
// THREADS threads with NP packs of 16 bytes each (and one of the row's last, fewer than a pack's, elements).  LOOP: the workgroup goes
// on to other rows; while the gradient of one is computed and stored pack by pack, the next row's packs are loaded into the
// registers that become free and their statistics taken kLag packs later, so that memory is busy all the time.
constexpr int kLag = 4;
template <typename T, int THREADS, int NP, bool TWO, bool GRAD, bool LOOP>
__global__ __launch_bounds__(THREADS, NP == 1 ? 5 : THREADS < 1024 && NP == 16 ? 4 : 1) void distill_row_kernel(DistillArgs a, int64_t rows) {
  constexpr int VEC = kVec<T>, WAVES = THREADS / 64, EPT = THREADS >= kTopMax ? 1 : kTopMax / THREADS;
  using P = Pack<T, VEC>;
  constexpr int SETS = LOOP ? 2 : 1;                       // in turn: a row's are read behind its barriers
  __shared__ float red[SETS][6][16];
  __shared__ EntryTable table[GRAD ? SETS : 1];
  const int tid = threadIdx.x;
  const int32_t packed = a.V / VEC * VEC, tail = a.V - packed;
  const Scales<TWO> k(a);
  const float inv_tau = 1.0f / a.tau;
  // Packs by their 32-bit distance from the row's beginning (a scalar).  One past the row's last holds that one: all threads load,
  // and what is not there is left out of the sums.  (`mine` is hidden from the compiler in every phase: it would keep all
  // the distances in registers.)
  const uint32_t bytes = (uint32_t)packed * sizeof(T), last = bytes ? bytes - 16 : 0;
  uint32_t mine = tid * 16;
  auto at = [&](int j) { return mine + (uint32_t)(j * THREADS * 16); };
  auto there = [&](int j) { return at(j) < bytes; };
  auto some_there = [&](int j) { return (uint32_t)(j * THREADS * 16) < bytes; };      // of the workgroup's
  auto pack_of = [&](int j, const T* s, uint32_t limit) {
    return P::load_stream(reinterpret_cast<const T*>(reinterpret_cast<const char*>(s) + min(at(j), limit)));
  };
  auto logits_of = [&](int64_t row) { return static_cast<const T*>(a.logits) + row * a.ld; };
  auto grad_of = [&](int64_t row) { return static_cast<T*>(a.grad) + row * a.ldg; };
  auto blank = [&](int64_t row) {            // loss 0, gradient 0
    if (a.loss && tid == 0) a.loss[row] = 0.0f;
    if (!GRAD) return;
    T* grad = grad_of(row);
    P z;
    z.v = 0;
    for (uint32_t o = tid * 16; o < bytes; o += THREADS * 16) z.store_stream(reinterpret_cast<T*>(reinterpret_cast<char*>(grad) + o));
    if (tid < tail) grad[packed + tid] = from_float<T>(0.0f);
  };

  int64_t row = blockIdx.x;
  Entries<EPT> next;
  next.template load<THREADS>(a, row);
  int set = 0;
  while (row < rows) {
    if (next.w == 0.0f) {
      blank(row);
      row += gridDim.x;
      if (row < rows) next.template load<THREADS>(a, row);
      continue;
    }
    P x[NP];
    float xt = -kInf;
    {
      const T* s = logits_of(row);
#pragma unroll
      for (int j = 0; j < NP; ++j) {
        if (bytes) {
          x[j] = pack_of(j, s, last);
        } else {
#pragma unroll
          for (int c = 0; c < VEC; ++c) x[j].set(c, -kInf);
        }
      }
      if (tid < tail) xt = to_float(s[packed + tid]);
    }
    Running<TWO> st;
#pragma unroll
    for (int j = 0; j < NP; ++j) {
#pragma unroll
      for (int c = 0; c < VEC; ++c) st.m = fmaxf(st.m, x[j].get(c));
      __builtin_amdgcn_sched_barrier(0);     // pack by pack: all at once would take twice the registers
    }
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      x[j].again();
      if (some_there(j)) st.template add<P, VEC>(x[j], there(j), k, true);
      __builtin_amdgcn_sched_barrier(0);
    }
    bool run = true;
    while (run) {
      Entries<EPT> own = next;
      own.settle(a);
      const int64_t row1 = row + gridDim.x;
      const bool more = row1 < rows;
      const T* s = logits_of(row);
      // the logits at the entries' places and at the label, before anything is overwritten
      float se[EPT], sl;
#pragma unroll
      for (int e = 0; e < EPT; ++e) se[e] = to_float(s[max(own.id[e], 0)]);
      sl = to_float(s[max(own.label, 0)]);
      if (more) next.template load<THREADS>(a, row1);

      if (GRAD) table[set].template begin<THREADS>(own);

      float um = kLowest, usum = 0.0f, ue[EPT];
#pragma unroll
      for (int e = 0; e < EPT; ++e) um = fmaxf(um, own.u[e]);
      um = wave_all(um, Max());
#pragma unroll
      for (int e = 0; e < EPT; ++e) usum += exp2_fast((own.u[e] - um) * (inv_tau * kLog2e));
      usum = wave_all(usum, Add());
      if (tid < tail) st.add(xt, k);
      st.over_wave(k);
      st.put(red[set]);
      if (tid % 64 == 0) {
        red[set][3][tid / 64] = um;
        red[set][4][tid / 64] = usum;
      }
#pragma unroll
      for (int e = 0; e < EPT; ++e) asm volatile("" ::"v"(se[e]));        // here at the latest: others store behind the barrier
      asm volatile("" ::"v"(sl));
      __syncthreads();
      st.template take<WAVES>(red[set], k);
      const float m = in_vgpr(st.m), q = st.q, r = st.r;
      {
        const int w = tid % 16;
        const float mw = w < WAVES ? red[set][3][w] : kLowest, sw = w < WAVES ? red[set][4][w] : 0.0f;
        um = lane_value(row_all(mw, Max()), 0);
        usum = lane_value(row_all(sw * exp2_fast((mw - um) * (inv_tau * kLog2e)), Add()), 0);
      }
      const Factors f(a, own.w, usum != 0.0f, own.label >= 0, q, r);
      if (f.zero) {
        blank(row);
        break;
      }

      float term = 0.0f;
      const float lq = logf(q), lu = logf(usum);
#pragma unroll
      for (int e = 0; e < EPT; ++e) {
        if (own.id[e] >= 0) {
          ue[e] = exp2_fast((own.u[e] - um) * (inv_tau * kLog2e));
          const float p = ue[e] / usum;
          term += entry_term(p, own.u[e] - um, lu, lq, se[e] - m, a.tau);
          if (GRAD && f.cs != 0.0f) table[set].put(e * THREADS + tid, own.id[e], p);
        }
      }
      term = wave_all(term, Add());
      if (tid % 64 == 0) red[set][5][tid / 64] = term;
      run = LOOP && more && next.w != 0.0f;
      if (GRAD) {
        T* grad = grad_of(row);
        const T* s1 = logits_of(run ? row1 : row);
        const uint32_t limit = run ? last : 0;            // (else every thread loads the first pack once more)
        Running<TWO> st1;
        asm volatile("" : "+v"(mine));
#pragma unroll
        for (int j = 0; j < NP + (LOOP ? kLag : 0); ++j) {
          if (j < NP) {
            x[j].again();
            if (there(j)) {
              P g;
#pragma unroll
              for (int c = 0; c < VEC; ++c) g.set(c, gradient_at<T, TWO>(x[j].get(c) - m, k, f));
              g.store_stream(reinterpret_cast<T*>(reinterpret_cast<char*>(grad) + at(j)));
            }
            if (LOOP && bytes) x[j] = pack_of(j, s1, limit);
            __builtin_amdgcn_sched_barrier(0);
          }
          if (LOOP && j >= kLag) {
            x[j - kLag].again();
            if (some_there(j - kLag)) st1.template add<P, VEC>(x[j - kLag], there(j - kLag), k);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
        st = st1;
        if (tid < tail) {
          grad[packed + tid] = from_float<T>(gradient_at<T, TWO>(xt - m, k, f));
          if (LOOP) xt = to_float(s1[packed + tid]);
        }
      }
      __syncthreads();
      if (a.loss && tid == 0) {
        float sum = 0.0f, loss = 0.0f;
        for (int w = 0; w < WAVES; ++w) sum += red[set][5][w];
        if (f.cs != 0.0f) loss += f.cs * a.tau * sum;
        if (f.ch != 0.0f) loss += f.ch * (logf(r) - (sl - m));
        a.loss[row] = loss;
      }
      // the places of the entries and of the label once more, whole: an id that comes twice takes both shares
      if (GRAD) {
        T* grad = grad_of(row);
        if (f.cs != 0.0f) table[set].template join<THREADS>(a.K);
#pragma unroll
        for (int e = 0; e < EPT; ++e)
          if (f.cs != 0.0f && own.id[e] >= 0)
            grad[own.id[e]] = from_float<T>(gradient_there<TWO>(se[e] - m, table[set].p[e * THREADS + tid], own.id[e] == own.label, k, f, q, r));
        if (f.ch != 0.0f && tid == THREADS - 1 && !table[set].has(own.label))
          grad[own.label] = from_float<T>(gradient_there<TWO>(sl - m, 0.0f, true, k, f, q, r));
      }
      // (a set is written again in the row after the next one, behind a barrier that every reader has to reach)
      set = (set + 1) % SETS;
      if (run) row = row1;
    }
    __syncthreads();
    row += gridDim.x;
  }
}

// ---- rows that stream through ----
// Longer rows than registers hold: a workgroup reads the row twice, the second time mostly from the last-level cache.  The loss alone
// needs a row once and no registers to keep it in: more workgroups, more loads in flight (975 rows of 50021 fp16 25.2 us,
// from a register tile 32.8; four packs a thread at once: with more, or as a ring, the registers cost more than it gains; GRAD: without
// a gradient the kernel has neither its registers nor its table, 46 to 51 registers in place of 60 to 80: 28.5 us with them).  Few rows:
// `parts` workgroups take a row's columns; one launch leaves each part's maximum and sums in the workspace (and the logits at the
// entries' places, which the gradient may overwrite), a second one joins them and does the rest.
enum StreamMode : int { STREAM_ALL = 0, STREAM_STATS = 1, STREAM_REST = 2 };
struct StreamArgs {
  DistillArgs a;
  int64_t rows;
  int32_t parts, cols, mode;
  float* stats;        // 4 floats per part
  float* values;       // K + 1 per row
};

template <typename T, int THREADS, bool TWO, bool GRAD>
__global__ __launch_bounds__(THREADS, GRAD ? 6 : 8) void distill_stream_kernel(StreamArgs t) {
  constexpr int VEC = kVec<T>, WAVES = THREADS / 64, AHEAD = 4;
  using P = Pack<T, VEC>;
  __shared__ float red[6][16];
  __shared__ EntryTable table;                                // (none without uses)
  const DistillArgs& a = t.a;
  const int tid = threadIdx.x;
  const Scales<TWO> k(a);
  const float inv_tau = 1.0f / a.tau;
  for (int64_t unit = blockIdx.x; unit < t.rows * t.parts; unit += gridDim.x) {
    const int64_t row = unit / t.parts;
    const int32_t part = (int32_t)(unit - row * t.parts), c0 = part * t.cols, c1 = min(c0 + t.cols, a.V);
    const int32_t packed = c0 + (c1 - c0) / VEC * VEC;       // the rest, fewer than a pack, one by one
    const T* s = static_cast<const T*>(a.logits) + row * a.ld;
    T* grad = GRAD ? static_cast<T*>(a.grad) + row * a.ldg : nullptr;
    Entries<1> own;
    own.load<THREADS>(a, row);
    own.settle(a);
    __syncthreads();                                          // (shared arrays of the unit before)
    if (GRAD) table.template begin<THREADS>(own);
    if (own.w == 0.0f) {
      if (t.mode != STREAM_STATS) {
        if (a.loss && tid == 0 && part == 0) a.loss[row] = 0.0f;
        if (GRAD) {
          Pack<T, VEC> z;
          z.v = 0;
          for (int32_t c = c0 + tid * VEC; c < packed; c += THREADS * VEC) z.store_stream(grad + c);
          if (packed + tid < c1) grad[packed + tid] = from_float<T>(0.0f);
        }
      }
      continue;
    }
    Running<TWO> st;
    if (t.mode != STREAM_REST) {
      for (int32_t c = c0 + tid * VEC; c < packed; c += THREADS * VEC * AHEAD) {
        P x[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) x[j] = P::load(s + min(c + j * THREADS * VEC, packed - VEC));
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) st.template add<P, VEC>(x[j], c + j * THREADS * VEC < packed, k);
      }
      if (packed + tid < c1) st.add(to_float(s[packed + tid]), k);
    } else {
      // the parts' statistics: the same order in every workgroup
      const float* parts = t.stats + row * t.parts * 4;
      for (int32_t j = tid; j < t.parts; j += THREADS) {
        Running<TWO> one;
        one.m = parts[j * 4];
        one.q = parts[j * 4 + 1];
        one.r = parts[j * 4 + 2];
        const float m1 = fmaxf(st.m, one.m);
        one.rise(m1, k);
        st.rise(m1, k);
        st.q += one.q;
        if (TWO) st.r += one.r;
      }
    }
    st.over_wave(k);
    st.put(red);
    __syncthreads();
    st.template take<WAVES>(red, k);
    if (t.mode == STREAM_STATS) {
      if (tid == 0) {
        float* out = t.stats + unit * 4;
        out[0] = st.m;
        out[1] = st.q;
        out[2] = st.r;
      }
      // the logits that this part has for the entries and the label
      float* values = t.values + row * (a.K + 1);
      if (own.id[0] >= c0 && own.id[0] < c1) values[tid] = to_float(s[own.id[0]]);
      if (tid == 0 && own.label >= c0 && own.label < c1) values[a.K] = to_float(s[own.label]);
      continue;
    }
    const float m = in_vgpr(st.m), q = st.q, r = st.r;
    float se = 0.0f, sl = 0.0f;
    if (t.mode == STREAM_REST) {
      const float* values = t.values + row * (a.K + 1);
      if (own.id[0] >= 0) se = values[tid];
      if (own.label >= 0) sl = values[a.K];
    } else {
      if (own.id[0] >= 0) se = to_float(s[own.id[0]]);
      if (own.label >= 0) sl = to_float(s[own.label]);
      asm volatile("" ::"v"(se), "v"(sl));
    }
    float um = wave_all(fmaxf(own.u[0], kLowest), Max());
    if (tid % 64 == 0) red[3][tid / 64] = um;
    __syncthreads();
    um = red[3][0];
    for (int w = 1; w < WAVES; ++w) um = fmaxf(um, red[3][w]);
    const float ue = exp2_fast((own.u[0] - um) * (inv_tau * kLog2e));
    float usum = wave_all(ue, Add());
    if (tid % 64 == 0) red[4][tid / 64] = usum;
    __syncthreads();
    usum = 0.0f;
    for (int w = 0; w < WAVES; ++w) usum += red[4][w];
    const Factors f(a, own.w, usum != 0.0f, own.label >= 0, q, r);
    const float p = own.id[0] >= 0 ? ue / usum : 0.0f;
    float term = 0.0f;
    if (own.id[0] >= 0) {
      term = entry_term(p, own.u[0] - um, logf(usum), logf(q), se - m, a.tau);
      if (GRAD && f.cs != 0.0f) table.put(tid, own.id[0], p);
    }
    term = wave_all(term, Add());
    if (tid % 64 == 0) red[5][tid / 64] = term;
    if (GRAD) {
      for (int32_t c = c0 + tid * VEC; c < packed; c += THREADS * VEC * AHEAD) {
        Pack<T, VEC> x[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) x[j] = Pack<T, VEC>::load(s + min(c + j * THREADS * VEC, packed - VEC));
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
          if (c + j * THREADS * VEC >= packed) break;
          Pack<T, VEC> g;
#pragma unroll
          for (int e = 0; e < VEC; ++e) g.set(e, f.zero ? 0.0f : gradient_at<T, TWO>(x[j].get(e) - m, k, f));
          g.store_stream(grad + c + j * THREADS * VEC);
        }
      }
      if (packed + tid < c1) grad[packed + tid] = from_float<T>(f.zero ? 0.0f : gradient_at<T, TWO>(to_float(s[packed + tid]) - m, k, f));
    }
    __syncthreads();
    if (a.loss && tid == 0 && part == 0) {
      float loss = 0.0f;
      float sum = 0.0f;
      for (int w = 0; w < WAVES; ++w) sum += red[5][w];
      if (f.cs != 0.0f) loss += f.cs * a.tau * sum;
      if (f.ch != 0.0f) loss += f.ch * (logf(r) - (sl - m));
      a.loss[row] = loss;
    }
    if (GRAD && !f.zero) {
      if (f.cs != 0.0f) table.template join<THREADS>(a.K);
      if (f.cs != 0.0f && own.id[0] >= c0 && own.id[0] < c1)
        grad[own.id[0]] = from_float<T>(gradient_there<TWO>(se - m, table.p[tid], own.id[0] == own.label, k, f, q, r));
      if (f.ch != 0.0f && tid == THREADS - 1 && own.label >= c0 && own.label < c1 && !table.has(own.label))
        grad[own.label] = from_float<T>(gradient_there<TWO>(sl - m, 0.0f, true, k, f, q, r));
    }
  }
}

constexpr int64_t kMostRowBlocks = 1 << 21;       // (a launch has fewer than 2^32 threads)

// A workgroup's threads, and the packs of a row that each holds (0: the row streams).
struct DistillTile {
  int32_t threads, packs;
  bool loop;
};
// As many threads as the row needs with 12 or 16 packs each.  Rows of up to 512 threads leave room for several workgroups on a compute
// unit, of which some load while others compute: one row each (7936 rows of 32000 bf16, two softmaxes 201 us; looping, with the
// next row's loads in between, 242).  Rows of 1024 threads have the compute unit to themselves and loop (15872 rows of
// 128000 bf16 1507 us, 5.1 TB/s; with the loads between the rows it took 230 us more).
DistillTile tile_of(const DistillPlan& plan, int32_t V, int type, bool grad) {
  const int32_t vec = type == TYPE_F32 ? 4 : 8, packs = V / vec;
  // (the loss alone streams rows of more than 256 packs)
  if (plan.parts > 1 || packs > 1024 * 16 || (!grad && packs > 256)) return {plan.cols <= 256 * vec * 8 ? 256 : 512, 0, false};
  for (const DistillTile t : {DistillTile{64, 1, false}, {64, 4, false}, {256, 4, false}, {256, 8, false}, {256, 12, false}, {256, 16, false}, {512, 12, false}, {512, 16, false}, {1024, 12, true}})
    if (packs <= t.threads * t.packs) return t;
  return {1024, 16, true};
}

template <typename T, bool TWO, bool GRAD> void stream(const StreamArgs& t, int32_t threads, hipStream_t st) {
  const dim3 grid((uint32_t)std::min(t.rows * t.parts, kMostRowBlocks));
  if (threads == 256) distill_stream_kernel<T, 256, TWO, GRAD><<<grid, dim3(256), 0, st>>>(t);
  else distill_stream_kernel<T, 512, TWO, GRAD><<<grid, dim3(512), 0, st>>>(t);
}

template <typename T, bool TWO, bool GRAD> hipError_t launch(const DistillArgs& a, hipStream_t st) {
  const int64_t rows = (int64_t)a.n * a.T;
  const DistillPlan plan = plan_distill(rows, a.V, a.K, a.type);
  const DistillTile tile = tile_of(plan, a.V, a.type, GRAD);
  if (tile.packs == 0) {
    StreamArgs t{a, rows, plan.parts, plan.cols, STREAM_ALL, nullptr, nullptr};
    if (plan.parts > 1) {
      t.stats = reinterpret_cast<float*>(static_cast<char*>(a.workspace) + plan.stats);
      t.values = reinterpret_cast<float*>(static_cast<char*>(a.workspace) + plan.values);
      t.mode = STREAM_STATS;
      stream<T, TWO, false>(t, tile.threads, st);
      t.mode = STREAM_REST;
    }
    stream<T, TWO, GRAD>(t, tile.threads, st);
    return hipGetLastError();
  }
  const dim3 grid((uint32_t)std::min(rows, tile.loop ? (int64_t)256 : kMostRowBlocks)), block(tile.threads);
  const int32_t at_most = tile.threads * tile.packs;
  if (at_most == 64 * 1) distill_row_kernel<T, 64, 1, TWO, GRAD, false><<<grid, block, 0, st>>>(a, rows);
  else if (at_most == 64 * 4) distill_row_kernel<T, 64, 4, TWO, GRAD, false><<<grid, block, 0, st>>>(a, rows);
  else if constexpr (GRAD) {
    if (at_most == 256 * 4) distill_row_kernel<T, 256, 4, TWO, true, false><<<grid, block, 0, st>>>(a, rows);
    else if (at_most == 256 * 8) distill_row_kernel<T, 256, 8, TWO, true, false><<<grid, block, 0, st>>>(a, rows);
    else if (at_most == 256 * 12) distill_row_kernel<T, 256, 12, TWO, true, false><<<grid, block, 0, st>>>(a, rows);
    else if (at_most == 256 * 16) distill_row_kernel<T, 256, 16, TWO, true, false><<<grid, block, 0, st>>>(a, rows);
    else if (at_most == 512 * 12) distill_row_kernel<T, 512, 12, TWO, true, false><<<grid, block, 0, st>>>(a, rows);
    else if (at_most == 512 * 16) distill_row_kernel<T, 512, 16, TWO, true, false><<<grid, block, 0, st>>>(a, rows);
    else if (at_most == 1024 * 12) distill_row_kernel<T, 1024, 12, TWO, true, true><<<grid, block, 0, st>>>(a, rows);
    else distill_row_kernel<T, 1024, 16, TWO, true, true><<<grid, block, 0, st>>>(a, rows);
  }
  return hipGetLastError();
}

template <typename T> hipError_t by_terms(const DistillArgs& a, bool two, hipStream_t st) {
  if (two) return a.grad ? launch<T, true, true>(a, st) : launch<T, true, false>(a, st);
  return a.grad ? launch<T, false, true>(a, st) : launch<T, false, false>(a, st);
}

}  // namespace

DistillPlan plan_distill(int64_t rows, int32_t V, int32_t K, int type) {
  DistillPlan p{};
  p.parts = 1;
  p.cols = V;
  const int32_t vec = type == TYPE_F32 ? 4 : 8;
  // few rows of many columns, or not very many of more than registers hold: 4096 columns a part or more, up to 512 workgroups (with gradient, in
  // parts against whole: 65 rows of 128000 bf16 16 us against 26, 128 21 against 27, 192 34 against 28; but 100 rows of 65536 16 against 12.6, of 40000
  // fp32 14.6 against 13.2, and the losses alone 12.3 against 9.0 and 11.5 against 7.5)
  if (rows > 0 && ((rows <= 64 && V >= 32768) || (rows <= 256 && V / vec > 1024 * 16))) {
    const int32_t most = (int32_t)std::min<int64_t>(V / 4096, (512 + rows - 1) / rows);
    if (most > 1) {
      p.cols = ((V + most - 1) / most + vec - 1) / vec * vec;
      p.parts = (V + p.cols - 1) / p.cols;
    }
  }
  if (p.parts > 1) {
    p.values = (rows * p.parts * 16 + 255) / 256 * 256;
    p.bytes = p.values + (rows * (K + 1) * 4 + 255) / 256 * 256;
  }
  return p;
}

void describe_distill(int64_t rows, int32_t V, int32_t K, int type, bool grad, int32_t* out) {
  const DistillPlan plan = plan_distill(rows, V, K, type);
  const DistillTile tile = tile_of(plan, V, type, grad);
  out[0] = tile.threads;
  out[1] = tile.packs;
  out[2] = tile.loop;
  out[3] = plan.parts;
}

hipError_t launch_distill(const DistillArgs& a, hipStream_t st) {
  // both terms at a temperature other than 1: two softmaxes
  const bool two = a.K > 0 && a.hard > 0.0f && a.hard < 1.0f && a.tau != 1.0f;
  if (a.type == TYPE_F32) return by_terms<float>(a, two, st);
  return a.type == TYPE_BF16 ? by_terms<bf16_t>(a, two, st) : by_terms<_Float16>(a, two, st);
}

}  // namespace ceca
