// Sampling of one token per row of logits from given random numbers (dllm_sample).
//
// Temperature, top-k, top-p and min-p each keep a prefix of one ranking (logit
// descending, index ascending), so the kept set is a boundary in that ranking.
// It is found with one read of all logits and a second read of few:
//
//   sample_chunk_kernel    a workgroup per CHUNK logits of a row, held in
//     registers: their maximum, the sum of their weights exp((x - max) / T), and
//     counts and weights of BINS classes of x / T, eight to an octave of weight.
//     The classes lie on one grid for all chunks, so no chunk has to know the
//     row's maximum.
//   sample_edge_kernel     a workgroup per row: joins the classes and finds those
//     in which the boundary may fall.
//   sample_collect_kernel  a workgroup per chunk that has members of them: lists
//     their (logit, index).
//   sample_pick_kernel     a workgroup per row: the boundary among the listed
//     members, the kept mass of each chunk, and the chunk and then the token where
//     the running sum of kept weights, in index order, passes u times its total.
//
// Calls without top-k, top-p and min-p need the first and the last alone; few rows of
// one chunk run all of them in one launch (sample_row_kernel).
//
// Many rows: the first kernel is bound by the float64 weights and sums and the classes'
// LDS additions (256 rows x 152064 float32: 48 us, 3.2 TB/s), the collection by HBM (31
// us, 5 TB/s, where every chunk has members); few rows by the chain of dependent steps
// in and between the kernels (1 row x 126464: 29 us; 5.5, 6.4, 4.2 and 13.4.  It is not
// the launches: a row of 3001 logits in one of them takes 27).  A chunk is 8192 logits
// in 512 threads' registers: 19 chunks of a vocabulary of 152064 let one row use 19 CUs;
// a workgroup that kept its place over chunks had half the waves a CU (70 us against 52
// when it was tried).
//
// Which token wins must not depend on the order of execution, and not on rounding
// where shares are equal.  Weights are float64 (those behind conf, which no choice here
// depends on, float32, and their sum float64); where threads add
// concurrently they add whole numbers (a weight in units of 2^-40 of its class's), so
// every sum is the same in any order, but one taken over classes and one over members
// agree only to some 2e-12.  A share of the mass can fall exactly between two
// candidates only where it is that share of every level of equal logits, since weights
// of unlike ones have no rational relation.  So candidates that tie for the maximum are
// counted, and weigh exactly 1 in every sum, and of what is not theirs SLACK is taken
// off (top-p) or added (u) before a share of it is compared: equal shares then compare
// as equal, and top-p's among ties alone are exact.
#include <algorithm>
#include <type_traits>

#include "kernels.h"

namespace dllm {

namespace {

constexpr int CHUNK = 8192, NT = 512, E = CHUNK / NT, NW = NT / 64;
constexpr int BINS = 512;               // 64 octaves; the last class stands for everything without mass
constexpr double PER_NAT = 11.541560327111707;  // 8 / ln 2
constexpr double LEAST = 0x1p-63;       // weights below count as none
constexpr double SLACK = 0x1p-37;       // of masses that are compared
constexpr int LIST = 1 << 15;            // members listed of a row, at most
constexpr int INDEX_BITS = 22;          // of a listed member's second word; its class above
constexpr int MAX_CHUNKS = (1 << INDEX_BITS) / CHUNK;
static_assert(BINS == NT, "a thread per class");

// Global memory, said outright: pointers out of structures are else read as flat ones.
#if defined(__HIP_DEVICE_COMPILE__)
#define GLOBAL __attribute__((address_space(1)))
#else
#define GLOBAL
#endif

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(bf16_t x) { return bf2f(x); }

// Unsigned order of a float (-0 as +0).
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t u = __float_as_uint(x == 0.f ? 0.f : x);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) {
  return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}

// 2^(j / STEPS), j < STEPS, in LDS.
constexpr int STEPS = 512;
__device__ __forceinline__ void fill_powers(double* t) {
  static_assert(STEPS == NT, "an entry per thread");
  t[threadIdx.x] = exp2((double)threadIdx.x / STEPS);
}
// 2^(d / 8) for d in [-8000, 0]: whole steps of 1 / 512 octave by
// table and exponent, the rest (f, at most half a step, or 7e-4 nats) by the Taylor
// polynomial of degree 3, whose remainder is 1e-14.  Exactly 1 at 0.  Adding 1.5 x
// 2^46 leaves d in steps (units of 1 / 64) in the low word.
__device__ __forceinline__ double power_of(double d, const double* powers) {
  constexpr double L = 0.08664339756999316;  // ln 2 / 8
  const double t = d + 0x1.8p46, f = d - (t - 0x1.8p46);
  const int n = __double2loint(t);
  const double p = f * fma(fma(L * L * L / 6, f, L * L / 2), f, L);
  const double w = powers[n & (STEPS - 1)];
  const double r = fma(w, p, w);
  return __hiloint2double(__double2hiint(r) + ((n >> 9) << 20), __double2loint(r));
}
// The same for any d <= 0 (2^-1000 for what lies below, and for NaN: -inf at an
// infinite temperature).
__device__ __forceinline__ double weight_of(double d, const double* powers) { return power_of(fmax(d, -8000.0), powers); }
// What a class sums up, in one word.  A logit at a distance of f classes, |f| <= 1/2,
// from its class's centre weighs v = 2^(f / 8) of the centre's weight: by the Taylor
// polynomial of degree 6, whose remainder is 6e-14.  The count of the logits (at most
// CHUNK = 2^13) stands from bit 50 on, below it the sum of their v - 15/16 (each below
// 1/8) in whole numbers of 2^-40: the mantissa of 2^12 + 1/16 + (v - 1).
constexpr int COUNT_BIT = 50;
__device__ __forceinline__ uint64_t class_word(double f) {
  constexpr double L = 0.08664339756999316;  // ln 2 / 8
  double p = fma(L * L * L * L * L * L / 720, f, L * L * L * L * L / 120);
  p = fma(p, f, L * L * L * L / 24);
  p = fma(p, f, L * L * L / 6);
  p = fma(p, f, L * L / 2);
  p = fma(p, f, L);
  return __double_as_longlong(fma(p, f, 4096.0625)) - (0x40b0000000000000ull - (1ull << COUNT_BIT));
}
// The mass, of the centre's weight, of `count` logits whose words' lower parts sum up to `low`.
__device__ __forceinline__ double class_mass(uint64_t low, uint32_t count) { return (double)low * 0x1p-40 + count * 0.9375; }
__device__ __forceinline__ uint64_t low_of(uint64_t word) { return word & ((1ull << COUNT_BIT) - 1); }

// A lane's value moved within the wave by CTRL (a data-parallel primitive, a few
// cycles where a shuffle through LDS takes a hundred); `old` where none arrives.
template <int CTRL, int ROWS, typename V>
__device__ __forceinline__ V moved(V old, V x) {
  if constexpr (sizeof(V) == 4) {
    return __builtin_bit_cast(V, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, old), __builtin_bit_cast(int, x), CTRL, ROWS, 0xf, false));
  } else {
    typedef int v2i __attribute__((ext_vector_type(2)));
    const v2i o = __builtin_bit_cast(v2i, old), y = __builtin_bit_cast(v2i, x);
    return __builtin_bit_cast(V, v2i{__builtin_amdgcn_update_dpp(o.x, y.x, CTRL, ROWS, 0xf, false),
                                     __builtin_amdgcn_update_dpp(o.y, y.y, CTRL, ROWS, 0xf, false)});
  }
}
template <typename V>
__device__ __forceinline__ V from_lane(V x, int lane) {
  if constexpr (sizeof(V) == 4) {
    return __builtin_bit_cast(V, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), lane));
  } else {
    typedef int v2i __attribute__((ext_vector_type(2)));
    const v2i y = __builtin_bit_cast(v2i, x);
    return __builtin_bit_cast(V, v2i{__builtin_amdgcn_readlane(y.x, lane), __builtin_amdgcn_readlane(y.y, lane)});
  }
}
struct Max {
  template <typename V> __device__ __forceinline__ V operator()(V a, V b) const { return a > b ? a : b; }
};
struct Min {
  template <typename V> __device__ __forceinline__ V operator()(V a, V b) const { return a < b ? a : b; }
};
struct Sum {
  template <typename V> __device__ __forceinline__ V operator()(V a, V b) const { return a + b; }
};
// f over the lanes up to this one: within rows of 16 (by 1, 2, 4, 8), then the last
// lane of row 0 into row 1 and of row 2 into row 3, then of row 1 into rows 2 and 3.
template <typename V, typename F>
__device__ __forceinline__ V wave_upto(V x, F f) {
  auto none = [&] {  // what changes nothing
    if constexpr (std::is_same_v<F, Sum>)
      return (V)0;
    else
      return x;
  };
  x = f(x, moved<0x111, 0xf>(none(), x));
  x = f(x, moved<0x112, 0xf>(none(), x));
  x = f(x, moved<0x114, 0xf>(none(), x));
  x = f(x, moved<0x118, 0xf>(none(), x));
  x = f(x, moved<0x142, 0xa>(none(), x));
  return f(x, moved<0x143, 0xc>(none(), x));
}
template <typename V, typename F>
__device__ __forceinline__ V wave_all(V x, F f) { return from_lane(wave_upto(x, f), 63); }
typedef unsigned long long u64;

// What a chunk leaves: its largest logit, the lowest index of a NaN or +inf (or
// ~0), the lowest index of the maximum (greedy rows), how many candidates have it, and
// its sums at the row's temperature (where nothing is filtered) and at temperature 1,
// relative to the largest weight.
struct ChunkStat {
  float top;
  uint32_t bad, arg, ties;
  double sum, sum1;
};
// What sample_edge_kernel leaves: the boundary as far as the classes tell it.
// Under top-k the classes below `ek` stay, of class ek - 1 the first rk members
// only where rk > 0; [lo, hi] are the classes in which top-p's boundary can fall;
// class bm holds min-p's (-1: none).  Listed are the members of classes [p0, p1],
// k1 and m1 (-1: none).
struct RowState {
  int ek, rk, lo, hi, bm;
  int p0, p1, k1, m1;
  float least, most;  // every listed member lies within
  double base;        // class of the row's maximum
  __device__ __forceinline__ bool lists(int b) const { return (b >= p0 && b <= p1) || b == k1 || b == m1; }
};

struct SampleWs {
  ChunkStat* stat;   // [rows, chunks]
  u64* classes;      // [rows, chunks, BINS]: class_word sums
  double* prefix;    // [rows, BINS]: mass of the classes up to each
  RowState* state;   // [rows]
  uint2* list;       // [rows, list_len]: key, index | class << INDEX_BITS
  uint32_t* listed;  // [rows]
  uint8_t* holds;    // [rows, chunks]: 1 where a chunk has members of the listed classes
  int chunks, list_len;
};

// A row's controls.
struct Controls {
  bool greedy, filter;
  double inv_t, rate, top_p, min_p;  // rate: classes per unit of logit
  int top_k;
};
__device__ __forceinline__ Controls controls_of(const SampleArgs& a, int r) {
  Controls c;
  const float t = a.temperature ? a.temperature[r] : 1.f;
  c.greedy = !(t > 0.f);
  c.inv_t = c.greedy ? 1.0 : 1.0 / (double)t;
  c.rate = c.inv_t * PER_NAT;
  const int k = a.top_k ? a.top_k[r] : 0;
  c.top_k = k >= 1 && k < a.vocab ? k : 0;
  const float p = a.top_p ? a.top_p[r] : 1.f;
  c.top_p = p < 1.f ? (double)p : 1.0;
  const float m = a.min_p ? a.min_p[r] : 0.f;
  c.min_p = m > 0.f ? fmin((double)m, 1.0) : 0.0;
  c.filter = !c.greedy && (c.top_k > 0 || c.top_p < 1.0 || c.min_p > 0.0);
  return c;
}
// A logit in units of classes.  Never fused into a following subtraction: the
// largest logit then stands at a distance of exactly 0 from itself.
__device__ __forceinline__ double in_classes(float x, double rate) {
#pragma clang fp contract(off)
  return (double)x * rate;
}
// Class of a logit in a row whose maximum lies in class `base` of the grid.
__device__ __forceinline__ int class_of(float x, double rate, double base) {
  return (int)fmin(base - rint(in_classes(x, rate)), (double)(BINS - 1));
}

// N consecutive logits from v on (rows may start at any element: the loads are
// only as aligned as the type); -inf past the row and at the mask token.
template <typename T, int N>
__device__ __forceinline__ void load_logits(const T* x, int v, int V, int mask_id, float (&f)[N]) {
  struct __attribute__((packed, aligned(sizeof(T)))) Run {
    T e[N];
  };
  const GLOBAL T* g = (const GLOBAL T*)x + v;
  if (v + N <= V) {
    const Run r = *(const GLOBAL Run*)g;
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = to_f(r.e[i]);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = v + i < V ? to_f(g[i]) : -INFINITY;
  }
  if ((uint32_t)(mask_id - v) < (uint32_t)N) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (v + i == mask_id) f[i] = -INFINITY;
  }
}

// A thread's logits of a chunk: RUNS runs of 16 bytes, NT threads apart.
template <typename T>
struct Slice {
  static constexpr int N = 16 / (int)sizeof(T), RUNS = E / N;
  struct __attribute__((packed, aligned(sizeof(T)))) Run {
    T e[N];
  };
  Run r[RUNS];
  static __device__ __forceinline__ int at(int v0, int i) { return v0 + (i * NT + (int)threadIdx.x) * N; }
  // whole chunks only; the loads are left in flight
  __device__ __forceinline__ void fetch(const T* x, int v0) {
    const GLOBAL T* g = (const GLOBAL T*)x;
#pragma unroll
    for (int i = 0; i < RUNS; ++i) r[i] = *(const GLOBAL Run*)(g + at(v0, i));
  }
  // the logits of a chunk that was fetched (whole) or is read here
  __device__ __forceinline__ void take(const T* x, int v0, bool whole, int V, int mask_id, float (&f)[RUNS][N]) const {
    if (whole) {
#pragma unroll
      for (int i = 0; i < RUNS; ++i)
#pragma unroll
        for (int e = 0; e < N; ++e) f[i][e] = to_f(r[i].e[e]);
      if ((uint32_t)(mask_id - v0) < (uint32_t)CHUNK) {
#pragma unroll
        for (int i = 0; i < RUNS; ++i)
#pragma unroll
          for (int e = 0; e < N; ++e)
            if (at(v0, i) + e == mask_id) f[i][e] = -INFINITY;
      }
    } else {
#pragma unroll
      for (int i = 0; i < RUNS; ++i) load_logits<T, N>(x, at(v0, i), V, mask_id, f[i]);
    }
  }
};

struct ChunkShared {
  u64 classes[BINS + 64];  // 64 places for what has no class
  double powers[STEPS], sum[NW], sum1[NW];
  float top[NW];
  uint32_t bad[NW], arg[NW], ties[NW];
};
// Chunk `block % chunks` of row `block / chunks`.
template <typename T>
__device__ __forceinline__ void chunk_phase(const SampleArgs& a, const SampleWs& w, int block, ChunkShared& sh) {
  typedef Slice<T> SL;
  constexpr int N = SL::N, RUNS = SL::RUNS;
  u64* const classes = sh.classes;
  const double* const powers = sh.powers;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int row = block / w.chunks, v0 = block % w.chunks * CHUNK;
  const T* x = static_cast<const T*>(a.logits) + (long)row * a.row_stride;
  const bool whole = v0 + CHUNK <= a.vocab;
  SL slice;
  if (whole) slice.fetch(x, v0);
  const Controls c = controls_of(a, row);
  if (!c.filter) fill_powers(sh.powers);
  classes[tid] = 0;
  float f[RUNS][N];
  slice.take(x, v0, whole, a.vocab, a.mask_id, f);
  float top = -INFINITY;
  bool broken = false;  // a NaN or +inf among mine
#pragma unroll
  for (int i = 0; i < RUNS; ++i)
#pragma unroll
    for (int e = 0; e < N; ++e) {
      broken |= __builtin_amdgcn_classf(f[i][e], 0x203);
      top = fmaxf(top, f[i][e]);
    }
  uint32_t bad = ~0u;
  if (broken)
#pragma unroll
    for (int i = RUNS - 1; i >= 0; --i)
#pragma unroll
      for (int e = N - 1; e >= 0; --e)
        if (!(f[i][e] < INFINITY)) bad = SL::at(v0, i) + e;
  top = wave_all(top, Max{});
  bad = wave_all(bad, Min{});
  if (lane == 0) {
    sh.top[wave] = top;
    sh.bad[wave] = bad;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NW; ++i) {
    top = fmaxf(top, sh.top[i]);
    bad = min(bad, sh.bad[i]);
  }
  ChunkStat* out = w.stat + block;
  if (bad != ~0u || top == -INFINITY) {  // the row is decided, or no candidate here
    if (tid == 0) *out = ChunkStat{top, bad, ~0u, 0, 0.0, 0.0};
    return;
  }
  double sum1 = 0;  // at temperature 1, of float32 weights
#pragma unroll
  for (int i = 0; i < RUNS; ++i)
#pragma unroll
    for (int e = 0; e < N; ++e) sum1 += (double)__builtin_amdgcn_exp2f((f[i][e] - top) * 1.4426950408889634f);
  uint32_t ties = 0;  // of the wave
#pragma unroll
  for (int i = 0; i < RUNS; ++i)
#pragma unroll
    for (int e = 0; e < N; ++e) ties += __popcll(__ballot(f[i][e] == top));
  uint32_t arg = ~0u;
  double sum = 0;
  const double qtop = in_classes(top, c.rate);
  if (c.greedy) {
#pragma unroll
    for (int i = 0; i < RUNS; ++i)
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (f[i][e] == top) arg = min(arg, (uint32_t)(SL::at(v0, i) + e));
  } else if (!c.filter) {
#pragma unroll
    for (int i = 0; i < RUNS; ++i)
#pragma unroll
      for (int e = 0; e < N; ++e) sum += weight_of(in_classes(f[i][e], c.rate) - qtop, powers);
  } else {
    const double base = rint(qtop);
    if (fabs(qtop) < 0x1p30) {
      // the class: the nearest whole number to q, in the low word of q + 1.5 x 2^52;
      // logits far below (and -inf) stand 600 classes below the top.  No branch
      // per logit: what has no class goes to a place of the lane's own.
      const int base_i = (int)base;
      const double least = qtop - 600.0;
#pragma unroll
      for (int i = 0; i < RUNS; ++i) {
        double q[N], t[N];
        int b[N];
        u64 u[N];
#pragma unroll
        for (int e = 0; e < N; ++e) {
          q[e] = fmax(in_classes(f[i][e], c.rate), least);
          t[e] = q[e] + 0x1.8p52;
        }
#pragma unroll
        for (int e = 0; e < N; ++e) {
          b[e] = base_i - __double2loint(t[e]);
          b[e] = b[e] < BINS - 1 ? b[e] : BINS + lane;
        }
#pragma unroll
        for (int e = 0; e < N; ++e) u[e] = class_word(q[e] - (t[e] - 0x1.8p52));
#pragma unroll
        for (int e = 0; e < N; ++e) atomicAdd(classes + b[e], u[e]);
      }
    } else {
#pragma unroll 1
      for (int i = 0; i < E; ++i) {
        float y = 0.f;
#pragma unroll
        for (int j = 0; j < E; ++j) y = j == i ? f[j / N][j % N] : y;
        const double q = in_classes(y, c.rate);
        const int b = (int)fmin(base - rint(q), (double)BINS);
        if (b < BINS - 1) atomicAdd(classes + b, class_word(q - rint(q)));
      }
    }
  }
  if (c.greedy) arg = wave_all(arg, Min{});
  if (!c.filter) sum = wave_all(sum, Sum{});
  sum1 = wave_all(sum1, Sum{});
  if (lane == 0) {
    sh.arg[wave] = arg;
    sh.ties[wave] = ties;
    sh.sum[wave] = sum;
    sh.sum1[wave] = sum1;
  }
  __syncthreads();
  if (tid == 0) {
    ChunkStat s{top, bad, ~0u, 0, 0.0, 0.0};
    for (int i = 0; i < NW; ++i) {
      s.arg = min(s.arg, sh.arg[i]);
      s.ties += sh.ties[i];
      s.sum += sh.sum[i];
      s.sum1 += sh.sum1[i];
    }
    *out = s;
  }
  if (c.filter) w.classes[(size_t)block * BINS + tid] = classes[tid];
}
template <typename T>
__global__ void __launch_bounds__(NT) sample_chunk_kernel(SampleArgs a, SampleWs w) {
  __shared__ ChunkShared sh;
  chunk_phase<T>(a, w, blockIdx.x, sh);
}

// Inclusive scan over the workgroup's threads.
template <typename V>
__device__ __forceinline__ V block_scan(V x, V* buf) {
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  x = wave_upto(x, Sum{});
  if (lane == 63) buf[wave] = x;
  __syncthreads();
  V before = 0;
#pragma unroll
  for (int i = 0; i < NW - 1; ++i) before += i < wave ? buf[i] : (V)0;
  __syncthreads();
  return x + before;
}

// The chunks of a row, in LDS: the weight of each one's maximum (0: without
// mass), the classes between the row's maximum and its own (BINS: none), and its
// candidates that have the row's maximum.
struct Chunks {
  double fac[MAX_CHUNKS];
  int shift[MAX_CHUNKS];
  uint32_t ties[MAX_CHUNKS];
};
struct RowTop {
  float big;
  uint32_t bad, ties;
  double qtop, base;
  // Mass of class 0 of the row or of one of its chunks, in which `some` of the members
  // tie for the maximum: those weigh 1 each, the others are summed up without them.
  __device__ __forceinline__ double first_mass(uint64_t low, uint32_t count, uint32_t some, double centre) const {
    return class_mass(low - some * low_of(class_word(qtop - base)), count - some) * centre + some;
  }
};
// Fills `ch` (no barrier after it) and returns the row's maximum, to every thread.
__device__ __forceinline__ RowTop join_chunks(const ChunkStat* stat, int nch, const Controls& c, const double* powers,
                                              Chunks& ch) {
  RowTop r{-INFINITY, ~0u, 0, 0.0, 0.0};
  const int lane = threadIdx.x & 63;
  for (int i = lane; i < nch; i += 64) {  // every wave by itself
    const float top = stat[i].top;
    r.ties = (top > r.big ? 0 : r.ties) + (top >= r.big ? stat[i].ties : 0);
    r.big = fmaxf(r.big, top);
    r.bad = min(r.bad, stat[i].bad);
  }
  const float mine = r.big;
  r.big = wave_all(r.big, Max{});
  r.ties = wave_all(mine == r.big ? r.ties : 0u, Sum{});
  r.bad = wave_all(r.bad, Min{});
  if (r.big == -INFINITY) return r;
  r.qtop = in_classes(r.big, c.rate);
  r.base = rint(r.qtop);
  for (int i = threadIdx.x; i < nch; i += NT) {
    const float top = stat[i].top;
    // a chunk with mass has a token with mass: its maximum
    const double q = in_classes(top, c.rate), e = top > -INFINITY ? weight_of(q - r.qtop, powers) : 0.0;
    ch.fac[i] = e >= LEAST ? e : 0.0;
    ch.shift[i] = e >= LEAST ? (int)(r.base - rint(q)) : BINS;
    ch.ties[i] = top == r.big ? stat[i].ties : 0;
  }
  return r;
}

struct EdgeShared {
  Chunks ch;
  double powers[STEPS], binw[BINS], bufd[NW];
  uint32_t binc[BINS], bufu[NW];
  int k, lo, hi;
};
__device__ __forceinline__ void edge_phase(const SampleArgs& a, const SampleWs& w, int row, EdgeShared& sh) {
  Chunks& ch = sh.ch;
  double *const powers = sh.powers, *const binw = sh.binw, *const bufd = sh.bufd;
  uint32_t *const binc = sh.binc, *const bufu = sh.bufu;
  const int tid = threadIdx.x, nch = w.chunks;
  const Controls c = controls_of(a, row);
  if (!c.filter) return;
  fill_powers(powers);
  if (tid == 0) {
    sh.k = sh.lo = sh.hi = -1;
    w.listed[row] = 0;
  }
  __syncthreads();
  const RowTop top = join_chunks(w.stat + (size_t)row * nch, nch, c, powers, ch);
  if (top.bad != ~0u || top.big == -INFINITY) {  // decided without a boundary
    for (int i = tid; i < nch; i += NT) w.holds[(size_t)row * nch + i] = 0;
    return;
  }
  __syncthreads();
  const GLOBAL u64* hm = (const GLOBAL u64*)w.classes + (size_t)row * nch * BINS;
  u64 low = 0;
  uint32_t n = 0;
  constexpr int U = 8;
  for (int i0 = 0; i0 < nch; i0 += U) {
    u64 um[U];
    bool in[U];
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int i = min(i0 + j, nch - 1), k = tid - ch.shift[i];
      // what lies behind a chunk's classes has no mass in the row either
      in[j] = i0 + j < nch && k >= 0 && k < BINS - 1 && tid < BINS - 1;
      um[j] = hm[(size_t)i * BINS + (in[j] ? k : 0)];
    }
#pragma unroll
    for (int j = 0; j < U; ++j)
      if (in[j]) {
        low += low_of(um[j]);
        n += (uint32_t)(um[j] >> COUNT_BIT);
      }
  }
  const double centre = weight_of(top.base - top.qtop - tid, powers);
  double m = block_scan(tid == 0 ? top.first_mass(low, n, top.ties, centre) : class_mass(low, n) * centre, bufd);
  n = block_scan(n, bufu);
  binw[tid] = m;
  binc[tid] = n;
  w.prefix[(size_t)row * BINS + tid] = m;
  __syncthreads();
  RowState st{BINS, 0, 0, -1, -1, 0, -1, -1, -1, 0.f, 0.f, top.base};
  double least = binw[BINS - 2], most = least;  // bounds of the mass that top-p is a share of
  if (c.top_k) {
    if (tid < BINS - 1 && n >= (uint32_t)c.top_k && (tid == 0 || binc[tid - 1] < (uint32_t)c.top_k)) sh.k = tid;
    __syncthreads();
    const int b = sh.k;
    if (b >= 0) {
      most = least = binw[b];
      st.ek = b + 1;
      if ((uint32_t)c.top_k < binc[b]) {
        st.rk = c.top_k - (int)(b ? binc[b - 1] : 0u);
        least = b ? binw[b - 1] : 0.0;
      }
    }
  }
  int edge = st.ek;  // the classes below it may stay
  if (c.top_p < 1.0) {
    const double t0 = fmax(c.top_p * least * (1.0 - 1e-9), 0.0), t1 = fmax(c.top_p * most * (1.0 + 1e-9), 0.0);
    if (tid < BINS - 1) {
      const double before = tid ? binw[tid - 1] : -1.0;
      if (m >= t0 && before < t0) sh.lo = tid;
      if (m >= t1 && before < t1) sh.hi = tid;
    }
    __syncthreads();
    st.lo = max(sh.lo, 0);
    st.hi = min(sh.hi >= 0 ? sh.hi : BINS - 2, edge - 1);
    edge = min(edge, st.hi + 1);
  }
  if (c.min_p > 0.0) {
    // w >= min_p as a distance, which stays exact where every w rounds to 1
    st.bm = max((int)fmin(top.base - rint(top.qtop + log(c.min_p) * PER_NAT), (double)(BINS - 1)), 0);
    edge = min(edge, st.bm + 1);
  }
  // members are needed of the classes in which the boundary may fall, and of
  // top-k's where top-p is a share of what it keeps; listed are those that fit
  const bool by_p = c.top_p < 1.0 && st.lo < edge;  // top-p may decide
  uint32_t room = w.list_len;
  int first = BINS, final = 0;
  auto single = [&](int b) {
    const uint32_t members = binc[b] - (b ? binc[b - 1] : 0u);
    if (members > room) return -1;
    room -= members;
    first = min(first, b);
    final = max(final, b);
    return b;
  };
  if (st.rk > 0 && (by_p || st.ek == edge)) st.k1 = single(st.ek - 1);
  if (st.bm >= 0 && st.bm < BINS - 1 && st.bm + 1 == edge) st.m1 = single(st.bm);
  if (by_p) {
    const int end = min(min(st.hi, edge - 1), st.lo + 63);
    const uint32_t before = st.lo ? binc[st.lo - 1] : 0u;
    st.p0 = st.lo;
    st.p1 = st.lo - 1;
    while (st.p1 < end && binc[st.p1 + 1] - before <= room) ++st.p1;
    if (st.p1 >= st.p0) {
      first = min(first, st.p0);
      final = max(final, st.p1);
    }
  }
  // logits outside [least, most] lie in none of them (a margin covers float32)
  const double hi = (top.base - first + 1) / c.rate, lo = (top.base - final - 1) / c.rate;
  st.most = c.rate > 0 ? (float)(hi + fabs(hi) * 1e-6) : INFINITY;
  st.least = c.rate > 0 ? (float)(lo - fabs(lo) * 1e-6) : -INFINITY;
  if (tid == 0) w.state[row] = st;
  for (int i = tid; i < nch; i += NT) {
    u64 have = 0;
    auto look = [&](int b) {
      const int k = b - ch.shift[i];
      if (b >= 0 && k >= 0) have |= hm[(size_t)i * BINS + k];
    };
    look(st.k1);
    look(st.m1);
    for (int b = st.p0; b <= st.p1; ++b) look(b);
    w.holds[(size_t)row * nch + i] = have != 0;
  }
}

__global__ void __launch_bounds__(NT) sample_edge_kernel(SampleArgs a, SampleWs w) {
  __shared__ EdgeShared sh;
  edge_phase(a, w, blockIdx.x, sh);
}

struct CollectShared {
  uint32_t n[NW], at;
};
// Members of chunk `block % chunks` of row `block / chunks`.
template <typename T>
__device__ __forceinline__ void collect_phase(const SampleArgs& a, const SampleWs& w, int block, CollectShared& sh) {
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int row = block / w.chunks, chunk = block % w.chunks, v0 = chunk * CHUNK;
  const Controls c = controls_of(a, row);
  if (!c.filter || !w.holds[block]) return;
  const RowState st = w.state[row];
  const T* x = static_cast<const T*>(a.logits) + (long)row * a.row_stride;
  constexpr int N = 16 / sizeof(T), RUNS = E / N;
  float f[RUNS][N];
  Slice<T> slice;
  const bool whole = v0 + CHUNK <= a.vocab;
  if (whole) slice.fetch(x, v0);
  slice.take(x, v0, whole, a.vocab, a.mask_id, f);
  uint32_t hit = 0;
#pragma unroll
  for (int i = 0; i < RUNS; ++i)
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (f[i][e] >= st.least && f[i][e] <= st.most && f[i][e] > -INFINITY)
        hit |= (uint32_t)st.lists(class_of(f[i][e], c.rate, st.base)) << (i * N + e);
  // places in the row's list: one reservation per workgroup
  const uint32_t n = __popc(hit), incl = wave_upto(n, Sum{});
  if (lane == 63) sh.n[wave] = incl;
  __syncthreads();
  if (tid == 0) {
    uint32_t all = 0;
    for (int i = 0; i < NW; ++i) {
      const uint32_t k = sh.n[i];
      sh.n[i] = all;
      all += k;
    }
    if (w.chunks == 1) {  // (no other workgroup adds members)
      w.listed[row] = all;
      sh.at = 0;
    } else {
      sh.at = all ? atomicAdd(w.listed + row, all) : 0;
    }
  }
  __syncthreads();
  uint32_t at = sh.at + sh.n[wave] + incl - n;
#pragma unroll
  for (int i = 0; i < RUNS; ++i)
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (hit >> (i * N + e) & 1) {
        if (at < (uint32_t)w.list_len)
          w.list[(size_t)row * w.list_len + at] =
              make_uint2(key_of(f[i][e]), (uint32_t)(v0 + (i * NT + tid) * N + e) | (uint32_t)class_of(f[i][e], c.rate, st.base) << INDEX_BITS);
        ++at;
      }
}

template <typename T>
__global__ void __launch_bounds__(NT) sample_collect_kernel(SampleArgs a, SampleWs w) {
  __shared__ CollectShared sh;
  collect_phase<T>(a, w, blockIdx.x, sh);
}

// A class's members up to a boundary: those with a key above `key`, and those
// with it up to index `last`.
struct Cut {
  uint32_t key, last;
  double mass;  // of the members kept, where a limit was reached
};

template <typename T>
struct Picker {
  static constexpr int KEPT = 4096, FEW = 64;
  // LDS
  struct Shared {
    Chunks ch;
    double part[MAX_CHUNKS];  // kept mass of a chunk
    u64 extra[MAX_CHUNKS];
    double prefix[BINS], centre[BINS];  // mass up to a class; weight of its centre
    uint2 list[KEPT];  // the row's list, where it fits
    u64 sub_mass[NT];
    uint32_t sub_count[NT];
    uint4 few[FEW];
    double powers[STEPS], bufd[NW];
    uint32_t bufu[NW], first[NW], last[NW], a, b, n;
    int i;
    double m;
  };
  Shared& sh;
  const T* x;
  const GLOBAL uint2* list;
  RowTop top;
  double rate;
  int V, mask_id;
  uint32_t listed;
  RowState st;

  __device__ __forceinline__ double weight(float f) const {
    const double e = weight_of(in_classes(f, rate) - top.qtop, sh.powers);
    return e < LEAST ? 0.0 : e;
  }
  // f(key, index) for every member of class b: from the row's list, or where the
  // list does not hold them, from the logits.
  template <typename F>
  __device__ __forceinline__ void members(int b, F f) const {
    if (st.lists(b)) {
      for (uint32_t i = threadIdx.x; i < listed; i += NT) {
        uint2 m;
        if (listed <= KEPT) {
          m = sh.list[i];
        } else {
          m.x = list[i].x;
          m.y = list[i].y;
        }
        if ((int)(m.y >> INDEX_BITS) == b) f(m.x, m.y & ((1u << INDEX_BITS) - 1));
      }
      return;
    }
    constexpr int N = 16 / sizeof(T), U = 16 / N;
    float least, most;
    bounds(b, least, most);
    typedef float f16v __attribute__((ext_vector_type(16)));
    float ahead[U][N];
    auto fetch = [&](int v0) {
#pragma unroll
      for (int i = 0; i < U; ++i) load_logits<T, N>(x, v0 + (i * NT + (int)threadIdx.x) * N, V, mask_id, ahead[i]);
    };
    fetch(0);
    for (int v0 = 0; v0 < V; v0 += NT * N * U) {
      f16v y;
      uint32_t hit = 0;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        y[i] = ahead[i / N][i % N];
        hit |= (uint32_t)(y[i] >= least && y[i] <= most && y[i] > -INFINITY) << i;
      }
      if (v0 + NT * N * U < V) fetch(v0 + NT * N * U);
#pragma unroll 1
      for (int i = 0; i < 16; ++i) {  // (the same i in every lane: y[i] is one register)
        if (__ballot(hit >> i & 1) == 0) continue;
        const float f1 = y[i];
        if ((hit >> i & 1) && class_of(f1, rate, top.base) == b)
          f(key_of(f1), (uint32_t)(v0 + (i / N * NT + (int)threadIdx.x) * N + i % N));
      }
    }
  }
  // Logits that lie outside are not of class b (a margin covers float32).
  __device__ __forceinline__ void bounds(int b, float& least, float& most) const {
    const double lo = (top.base - b - 1) / rate, hi = (top.base - b + 1) / rate;
    least = rate > 0 ? (float)(lo - fabs(lo) * 1e-6) : -INFINITY;
    most = rate > 0 ? (float)(hi + fabs(hi) * 1e-6) : INFINITY;
  }
  // Class b's weights are at most 2^top_of(b); its sums are whole numbers of 2^(top_of(b) - 40).
  static __device__ __forceinline__ int top_of(int b) { return ((1 - b) >> 3) + 1; }

  // The members of class b that stay when at most `limit` of them may, and the mass
  // of the members before one must be less than `target`: the range of keys, then of
  // indices among equal keys, is narrowed NT parts at a time until few members are
  // left in it, which one wave then ranks.
  __device__ __forceinline__ Cut select(int b, uint32_t limit, double target) {
    const int tid = threadIdx.x, lane = tid & 63;
    const double unit = ldexp(1.0, top_of(b) - 40), units = ldexp(1.0, 40 - top_of(b));
    target = fmax(target, 1e-300);  // the first of all stays
    // the range: keys [lo, hi] from above, then indices [lo, hi] from below
    uint32_t lo = ~0u, hi = 0;
    uint32_t inside = st.lists(b) ? listed : ~0u;  // members in the range, at most
    if (inside > KEPT) {
      // the members' own range: one round of parts then mostly does, and equal ones show
      if (tid == 0) {
        sh.a = ~0u;
        sh.b = 0;
      }
      __syncthreads();
      members(b, [&](uint32_t key, uint32_t) {
        lo = min(lo, key);
        hi = max(hi, key);
      });
      lo = wave_all(lo, Min{});
      hi = wave_all(hi, Max{});
      if (lane == 0) {
        atomicMin(&sh.a, lo);
        atomicMax(&sh.b, hi);
      }
      __syncthreads();
      lo = sh.a;
      hi = sh.b;
      __syncthreads();
      if (lo > hi) return Cut{~0u, 0, 0.0};  // no members (rounding at a class's edge can lead here)
    } else {
      float least, most;
      bounds(b, least, most);
      lo = key_of(least);
      hi = key_of(most);
    }
    bool by_key = true;
    uint32_t n0 = 0, key0 = 0;  // members ranked before the range, and their mass; its key, once it is one
    double m0 = 0;
    auto in_range = [&](uint32_t key, uint32_t v) { return by_key ? key >= lo && key <= hi : key == key0 && v >= lo && v <= hi; };
    for (;;) {
      if (inside <= FEW) {
        __syncthreads();
        if (tid == 0) sh.n = 0;
        __syncthreads();
        members(b, [&](uint32_t key, uint32_t v) {
          if (!in_range(key, v)) return;
          const u64 fixed = (u64)(weight(value_of(key)) * units);
          sh.few[min(atomicAdd(&sh.n, 1u), (uint32_t)FEW - 1)] = make_uint4(key, v, (uint32_t)fixed, (uint32_t)(fixed >> 32));
        });
        __syncthreads();
        const int n = (int)sh.n;
        const uint4 mine = lane < n ? sh.few[lane] : make_uint4(0, ~0u, 0, 0);
        auto fixed_of = [](const uint4& m) { return (u64)m.w << 32 | m.z; };
        uint32_t rank = 0;
        u64 before = 0;
#pragma unroll 8
        for (int j = 0; j < n; ++j) {
          const uint4 o = sh.few[j];
          const bool first = o.x > mine.x || (o.x == mine.x && o.y < mine.y);
          rank += first;
          before += first ? fixed_of(o) : 0;
        }
        const double mass = m0 + (double)before * unit;
        const bool stays = lane < n && n0 + rank < limit && mass < target;
        // the last that stays: the one of the highest rank
        const uint32_t r = wave_all(stays ? rank + 1 : 0u, Max{});
        const u64 who = __ballot(stays && rank + 1 == r);
        if (who == 0) return Cut{~0u, 0, m0};  // no members
        const int l = __ffsll(who) - 1;
        return Cut{from_lane(mine.x, l), from_lane(mine.y, l), from_lane(mass + (double)fixed_of(mine) * unit, l)};
      }
      if (by_key && hi == lo) {
        // many equal members: those with the lowest indices
        const double each = weight(value_of(lo));
        const uint32_t ties = (uint32_t)fmax(fmin((double)(limit - n0), ceil((target - m0) / each)), 1.0);
        if (ties >= inside) return Cut{lo, ~0u, m0 + (double)inside * each};
        by_key = false;
        key0 = lo;
        limit = n0 + ties;
        target = INFINITY;
        lo = 0;
        hi = (uint32_t)V - 1;
      }
      const uint32_t span = hi - lo;
      const int down = span >= NT ? 32 - __clz(span) - 9 : 0;  // span >> down < NT = 2^9
      sh.sub_mass[tid] = 0;
      sh.sub_count[tid] = 0;
      if (tid == 0) sh.i = -1;
      __syncthreads();
      members(b, [&](uint32_t key, uint32_t v) {
        if (in_range(key, v)) {
          const uint32_t at = (by_key ? hi - key : v - lo) >> down;
          atomicAdd(sh.sub_mass + at, (u64)(weight(value_of(key)) * units));
          atomicAdd(sh.sub_count + at, 1u);
        }
      });
      __syncthreads();
      const uint32_t mine = sh.sub_count[tid];
      const double mass = (double)sh.sub_mass[tid] * unit;
      const uint32_t n1 = block_scan(mine, sh.bufu);
      const double m1 = block_scan(mass, sh.bufd);
      const bool reached = n0 + n1 >= limit || m0 + m1 >= target;
      const bool before = n0 + n1 - mine >= limit || m0 + (m1 - mass) >= target;
      if (reached && !before && mine > 0) {
        sh.i = tid;
        sh.a = n1 - mine;
        sh.b = mine;
        sh.m = m1 - mass;
      }
      __syncthreads();
      const int i = sh.i;
      if (i < 0) return Cut{0, ~0u, 0};  // no limit is reached: all stay
      n0 += sh.a;
      m0 += sh.m;
      inside = sh.b;
      const uint32_t p = (uint32_t)i << down, q = min(span, (((uint32_t)i + 1) << down) - 1);
      if (by_key) {
        lo = hi - q;
        hi = hi - p;
      } else {
        hi = lo + q;
        lo = lo + p;
      }
      __syncthreads();
    }
  }
};

template <typename T>
__device__ __forceinline__ void pick_phase(const SampleArgs& a, const SampleWs& w, int row, typename Picker<T>::Shared& sh) {
  typedef Picker<T> P;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int nch = w.chunks, V = a.vocab;
  const ChunkStat* stat = w.stat + (size_t)row * nch;
  const Controls c = controls_of(a, row);
  auto answer = [&](int token, float conf, float prob) {
    a.token[row] = token;
    if (a.conf) a.conf[row] = conf;
    if (a.prob) a.prob[row] = prob;
  };
  RowState st{};
  uint32_t listed = 0;
  if (c.filter) {  // (early: these loads pass beside the join of the chunks)
    st = w.state[row];
    listed = w.listed[row];
    sh.prefix[tid] = w.prefix[(size_t)row * BINS + tid];
  }
  fill_powers(sh.powers);
  sh.extra[tid] = 0;
  __syncthreads();
  P p{sh, static_cast<const T*>(a.logits) + (long)row * a.row_stride, (const GLOBAL uint2*)w.list + (size_t)row * w.list_len,
      join_chunks(stat, nch, c, sh.powers, sh.ch), c.rate, V, a.mask_id, listed, st};
  const RowTop& top = p.top;
  if (top.bad != ~0u || top.big == -INFINITY) {
    if (tid == 0) {
      if (top.bad != ~0u)
        answer((int)top.bad, NAN, NAN);
      else
        answer(-1, 0.f, 0.f);
    }
    return;
  }
  double all1 = 0;  // the row's sum at temperature 1
  uint32_t arg = ~0u;
  for (int i = lane; i < nch; i += 64) {
    const ChunkStat s = stat[i];
    if (s.top > -INFINITY) all1 += s.sum1 * weight_of(((double)s.top - top.big) * PER_NAT, sh.powers);
    if (s.top == top.big) arg = min(arg, s.arg);
  }
  all1 = wave_all(all1, Sum{});
  if (c.greedy) {
    arg = wave_all(arg, Min{});
    if (tid == 0) answer((int)arg, (float)(1.0 / all1), 1.f);
    return;
  }

  // ---- the boundary: classes below `edge` are kept whole, of class `edge` the members that stay
  int edge = BINS;
  Cut cut{~0u, 0, 0};  // of that class: none
  double reach = INFINITY;  // the largest (max - x) / T that min-p keeps in it
  auto stays = [&](float f, uint32_t key, uint32_t v) {
    return ((double)top.big - f) * c.inv_t <= reach && (key > cut.key || (key == cut.key && v <= cut.last));
  };
  if (c.filter) {
    const double* prefix = sh.prefix;
    sh.centre[tid] = weight_of(top.base - top.qtop - tid, sh.powers);
    if (p.listed <= P::KEPT)
      for (uint32_t i = tid; i < p.listed; i += NT) sh.list[i] = make_uint2(p.list[i].x, p.list[i].y);
    __syncthreads();
    auto mass_before = [&](int b) { return b > 0 ? prefix[b - 1] : 0.0; };
    const int bk = st.rk > 0 ? st.ek - 1 : -1;
    edge = bk >= 0 ? bk : st.ek;
    // the boundary by top-k and top-p: class `edge` holds it where limit or target say so
    uint32_t limit = bk >= 0 ? (uint32_t)st.rk : ~0u;
    double target = INFINITY;
    bool ranked = bk >= 0;
    // first pass: the mass that top-k keeps; second: the boundary itself
    const bool by_p = c.top_p < 1.0 && (st.bm < 0 || st.lo <= st.bm);
#pragma unroll 1
    for (int pass = by_p && bk >= 0 ? 0 : 1; pass < 2; ++pass) {
      if (pass == 1) {
        if (by_p) {
          const double all = bk >= 0 ? mass_before(bk) + cut.mass : prefix[min(st.ek, BINS - 1) - 1];
          const double share = c.top_p * (all - fmax(all - top.ties, 0.0) * SLACK);
          int b = st.lo;
          while (b < st.hi && prefix[b] < share) ++b;
          if (b < edge) {
            edge = b;
            limit = ~0u;
          }
          if (b == edge) {
            ranked = true;
            target = share - mass_before(b);
          }
        }
        if (st.bm >= 0 && st.bm <= edge) {
          if (st.bm < edge) ranked = false;
          edge = st.bm;
          reach = -log(c.min_p);
        }
        cut = edge < BINS - 1 && reach < INFINITY ? Cut{0, ~0u, 0} : Cut{~0u, 0, 0};
        if (edge >= BINS - 1 || !ranked) break;
      }
      cut = p.select(edge, limit, target);
    }
    // ---- kept mass of each chunk: its classes before the edge, then the edge's members
    const double unit = ldexp(1.0, P::top_of(edge) - 40), units = ldexp(1.0, 40 - P::top_of(edge));
    if (edge < BINS - 1 && cut.key != ~0u)
      p.members(edge, [&](uint32_t key, uint32_t v) {
        const float f = value_of(key);
        if (stays(f, key, v)) atomicAdd(sh.extra + v / CHUNK, (u64)(p.weight(f) * units));
      });
    const GLOBAL u64* h = (const GLOBAL u64*)w.classes + (size_t)row * nch * BINS;
    constexpr int U = 4;  // chunks of a wave at a time
    for (int i0 = wave; i0 < nch; i0 += NW * U) {
      double s[U];
#pragma unroll
      for (int j = 0; j < U; ++j) {
        const int i = i0 + j * NW;
        // classes of the chunk before the edge
        const int shift = sh.ch.shift[min(i, nch - 1)], end = i < nch ? min(edge, BINS - 1) - shift : 0;
        const uint32_t ties = lane == 0 ? sh.ch.ties[min(i, nch - 1)] : 0;
        s[j] = 0;
#pragma unroll
        for (int k = 0; k < BINS / 64; ++k) {
          const int at = k * 64 + lane;
          if (at < end) {
            const u64 word = h[(size_t)i * BINS + at];
            s[j] += k == 0 ? top.first_mass(low_of(word), (uint32_t)(word >> COUNT_BIT), ties, sh.centre[at + shift])
                           : class_mass(low_of(word), (uint32_t)(word >> COUNT_BIT)) * sh.centre[at + shift];
          }
        }
      }
#pragma unroll
      for (int j = 0; j < U; ++j) {
        s[j] = wave_all(s[j], Sum{});
        if (lane == 0 && i0 + j * NW < nch) sh.part[i0 + j * NW] = s[j];
      }
    }
    __syncthreads();
    if (tid < nch) sh.part[tid] += (double)sh.extra[tid] * unit;
  } else if (tid < nch) {
    sh.part[tid] = stat[tid].sum * sh.ch.fac[tid];
  }

  // ---- the chunk, then the token, where the running sum passes u times the whole
  __syncthreads();
  double total = 0;
  for (int i0 = 0; i0 < nch; i0 += 64) total += wave_all(i0 + lane < nch ? sh.part[i0 + lane] : 0.0, Sum{});
  float u = a.u[row];
  u = u > 0.f ? fminf(u, 1.f - 0x1p-24f) : 0.f;
  const double want = u * (total + fmax(total - top.ties, 0.0) * SLACK);
  // every wave by itself: the first chunk with mass whose running sum passes
  // `want`; if rounding leaves none, the last with mass
  int at = 0;
  double run = 0, sums = 0;
  for (int i0 = 0; i0 < nch; i0 += 64) {
    const double part = i0 + lane < nch ? sh.part[i0 + lane] : 0.0;
    const double upto = wave_upto(part, Sum{}) + sums;
    const u64 mass = __ballot(part > 0.0), past = __ballot(part > 0.0 && upto > want);
    if (past | mass) {
      const int l = past ? __ffsll(past) - 1 : 63 - __clzll(mass);
      at = i0 + l;
      run = from_lane(upto - part, l);
    }
    if (past) break;
    sums = from_lane(upto, 63);
  }
  const bool ranked_cut = c.filter && edge < BINS - 1 && cut.key != 0 && cut.key != ~0u && !(reach < INFINITY);
  const int v0 = at * CHUNK + tid * E;
  float y[E];
  load_logits<T, E>(p.x, v0, V, a.mask_id, y);
  double e[E], sum = 0;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const float f = y[i];
    bool keep = f > -INFINITY;
    if (ranked_cut) {  // the boundary is a member: the rest goes by the ranking
      const uint32_t key = key_of(f);
      keep = key > cut.key || (key == cut.key && (uint32_t)(v0 + i) <= cut.last);
    } else if (c.filter && keep) {
      const int b = class_of(f, c.rate, top.base);
      keep = b < edge ? b < BINS - 1 : b == edge && edge < BINS - 1 && stays(f, key_of(f), v0 + i);
    }
    e[i] = 0.0;
    if (keep) e[i] = p.weight(f);
    sum += e[i];
  }
  const double incl = block_scan(sum, sh.bufd);  // has barriers
  run += incl - sum;
  uint32_t mine = ~0u, last = 0;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    run += e[i];
    if (e[i] > 0.0) {
      last = v0 + i + 1;
      if (run > want && mine == ~0u) mine = v0 + i;
    }
  }
  mine = wave_all(mine, Min{});
  last = wave_all(last, Max{});
  if (lane == 0) {
    sh.first[wave] = mine;
    sh.last[wave] = last;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NW; ++i) {
    mine = min(mine, sh.first[i]);
    last = max(last, sh.last[i]);
  }
  // (rounding inside the chunk: its last kept token)
  const uint32_t token = mine != ~0u ? mine : last - 1;
  if ((int)token >= v0 && (int)token < v0 + E) {
    float f = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) f = v0 + i == (int)token ? y[i] : f;
    answer((int)token, (float)(weight_of(((double)f - top.big) * PER_NAT, sh.powers) / all1), (float)(p.weight(f) / total));
  }
}

template <typename T>
__global__ void __launch_bounds__(NT) sample_pick_kernel(SampleArgs a, SampleWs w) {
  __shared__ typename Picker<T>::Shared sh;
  pick_phase<T>(a, w, blockIdx.x, sh);
}

// All four for rows of one chunk: a workgroup's own stores are there after a barrier.
template <typename T>
__global__ void __launch_bounds__(NT) sample_row_kernel(SampleArgs a, SampleWs w) {
  __shared__ union Shared {
    ChunkShared chunk;
    EdgeShared edge;
    CollectShared collect;
    typename Picker<T>::Shared pick;
  } sh;
  chunk_phase<T>(a, w, blockIdx.x, sh.chunk);
  __syncthreads();
  if (a.top_k || a.top_p || a.min_p) {
    edge_phase(a, w, blockIdx.x, sh.edge);
    __syncthreads();
    collect_phase<T>(a, w, blockIdx.x, sh.collect);
    __syncthreads();
  }
  pick_phase<T>(a, w, blockIdx.x, sh.pick);
}

int chunks_of(int vocab) { return ceil_div(vocab, CHUNK); }

// Carves the workspace (null: sizes only); returns the bytes.
size_t carve(void* base, size_t rows, int vocab, SampleWs* w) {
  const size_t chunks = chunks_of(vocab);
  size_t off = 0;
  auto take = [&](size_t bytes) {
    char* at = static_cast<char*>(base) + off;
    off += (bytes + 255) / 256 * 256;
    return at;
  };
  w->chunks = (int)chunks;
  w->list_len = std::min(LIST, vocab);
  w->stat = reinterpret_cast<ChunkStat*>(take(rows * chunks * sizeof(ChunkStat)));
  w->classes = reinterpret_cast<u64*>(take(rows * chunks * BINS * sizeof(u64)));
  w->prefix = reinterpret_cast<double*>(take(rows * BINS * sizeof(double)));
  w->state = reinterpret_cast<RowState*>(take(rows * sizeof(RowState)));
  w->list = reinterpret_cast<uint2*>(take(rows * w->list_len * sizeof(uint2)));
  w->listed = reinterpret_cast<uint32_t*>(take(rows * sizeof(uint32_t)));
  w->holds = reinterpret_cast<uint8_t*>(take(rows * chunks));
  return off;
}

template <typename T>
void launch(const SampleArgs& a, const SampleWs& w, hipStream_t s) {
  // rows of one chunk in one launch while every CU has one at most (256 rows x 8192, all
  // controls: 34 us, four launches 38; 512 rows: 60 and 57; 1024 rows: 119 and 101, since
  // the other kernels leave room for more workgroups a CU than the last)
  if (w.chunks == 1 && a.rows <= device_cu_count()) {
    sample_row_kernel<T><<<a.rows, NT, 0, s>>>(a, w);
    DLLM_LAUNCH_CHECK("sample_row_kernel");
    return;
  }
  const unsigned n = (unsigned)a.rows * w.chunks;
  sample_chunk_kernel<T><<<n, NT, 0, s>>>(a, w);
  DLLM_LAUNCH_CHECK("sample_chunk_kernel");
  if (a.top_k || a.top_p || a.min_p) {
    sample_edge_kernel<<<a.rows, NT, 0, s>>>(a, w);
    DLLM_LAUNCH_CHECK("sample_edge_kernel");
    sample_collect_kernel<T><<<n, NT, 0, s>>>(a, w);
    DLLM_LAUNCH_CHECK("sample_collect_kernel");
  }
  sample_pick_kernel<T><<<a.rows, NT, 0, s>>>(a, w);
  DLLM_LAUNCH_CHECK("sample_pick_kernel");
}

}  // namespace

bool sample_fits(int rows, int vocab) { return (long)rows * chunks_of(vocab) < (1l << 22); }

size_t sample_bytes(int rows, int vocab) {
  SampleWs w;
  return carve(nullptr, rows, vocab, &w);
}

void launch_sample(const SampleArgs& a, void* ws, hipStream_t s) {
  SampleWs w;
  carve(ws, a.rows, a.vocab, &w);
  a.dtype == DLLM_F32 ? launch<float>(a, w, s) : launch<bf16_t>(a, w, s);
}

}  // namespace dllm
