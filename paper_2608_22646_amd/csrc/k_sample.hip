// Sampling of one token per row of logits from given random numbers (dllm_sample).
//
// Temperature, top-k, top-p and min-p each keep a prefix of one ranking (logit
// descending, index ascending), so the kept set is a boundary in that ranking.
// Two launches find it with one read of the logits and a part of a second:
//
//   sample_chunk_kernel  one workgroup per CHUNK logits of a row, held in
//     registers: their maximum, the sum of the weights exp((x - max) / T), and a
//     histogram of counts and weights over BINS classes of x / T, BINS_PER_NAT
//     to a unit.  The classes lie on one grid for all chunks, so no chunk has to
//     know the row's maximum.
//   sample_row_kernel    one workgroup per row: joins the histograms, finds the
//     class in which the boundary falls, orders that class's members alone by
//     (logit, index), then finds the chunk and the token where the running sum of
//     kept weights, in index order, passes u times its total.
//
// Which token wins must not depend on rounding or on the order of execution.
// Weights are float64 throughout; where threads add concurrently they add whole
// numbers (a weight in units of 2^-50 of its chunk's largest, 2^-40 of its
// class's), so every sum is the same in any order and good to about 1e-12.
#include <algorithm>

#include "kernels.h"

namespace dllm {

namespace {

constexpr int CHUNK = 8192, NT1 = 512, E1 = CHUNK / NT1;
constexpr int BINS = 512;               // the last one takes everything without mass
constexpr double BINS_PER_NAT = 11.0;   // 510 / 11 = 46.3 > 66 ln 2
constexpr double LEAST = 0x1p-66;       // weights below count as none
constexpr int NT2 = 512, LIST = 4096, MAX_CHUNKS = (1 << 22) / CHUNK;

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

// e^x for x <= 0 to 1e-14 relative: 2^k times the Taylor polynomial of degree 11
// over half a binade (its remainder is 6e-15); 0 below e^-700.
__device__ __forceinline__ double exp_neg(double x) {
  x = fmax(x, -700.0);
  const double k = rint(x * 1.4426950408889634);
  double r = fma(k, -0.693147180559945286, x);
  r = fma(k, -2.319046813846299558e-17, r);
  double p = 1.0 / 39916800;
  p = fma(p, r, 1.0 / 3628800);
  p = fma(p, r, 1.0 / 362880);
  p = fma(p, r, 1.0 / 40320);
  p = fma(p, r, 1.0 / 5040);
  p = fma(p, r, 1.0 / 720);
  p = fma(p, r, 1.0 / 120);
  p = fma(p, r, 1.0 / 24);
  p = fma(p, r, 1.0 / 6);
  p = fma(p, r, 0.5);
  p = fma(p, r, 1.0);
  p = fma(p, r, 1.0);
  return ldexp(p, (int)k);
}
// A weight w in [0, 1] as a whole number of 2^-50: the mantissa of 4 + w.
__device__ __forceinline__ uint64_t fixed50(double w) {
  return __double_as_longlong(4.0 + w) - 0x4010000000000000ull;
}

template <typename V, typename F>
__device__ __forceinline__ V wave_all(V x, F f) {
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) x = f(x, (V)__shfl_xor(x, s, 64));
  return x;
}

// What a chunk leaves: its largest logit, the lowest index of a NaN or +inf (or
// ~0), the lowest index of the maximum, and its sums at the row's temperature
// (in 2^-50 of the largest weight) and at temperature 1 (of the largest).
struct ChunkStat {
  float top;
  uint32_t bad, arg, pad;
  uint64_t sum;
  double sum1;
};

struct SampleWs {
  ChunkStat* stat;   // [rows, chunks]
  uint64_t* mass;    // [rows, chunks, BINS] in 2^-50
  uint32_t* count;   // [rows, chunks, BINS]
  int chunks;
};

// A row's controls.
struct Controls {
  bool greedy, filter;
  double inv_t, top_p, min_p;
  int top_k;
};
__device__ __forceinline__ Controls controls_of(const SampleArgs& a, int r) {
  Controls c;
  const float t = a.temperature ? a.temperature[r] : 1.f;
  c.greedy = !(t > 0.f);
  c.inv_t = c.greedy ? 1.0 : 1.0 / (double)t;
  const int k = a.top_k ? a.top_k[r] : 0;
  c.top_k = k >= 1 && k < a.vocab ? k : 0;
  const float p = a.top_p ? a.top_p[r] : 1.f;
  c.top_p = p < 1.f ? (double)p : 1.0;
  const float m = a.min_p ? a.min_p[r] : 0.f;
  c.min_p = m > 0.f ? fmin((double)m, 1.0) : 0.0;
  c.filter = !c.greedy && (c.top_k > 0 || c.top_p < 1.0 || c.min_p > 0.0);
  return c;
}
// Class of a logit on the grid that all rows of a temperature share.
__device__ __forceinline__ double class_of(float x, double rate) { return floor((double)x * rate); }

// N consecutive logits from v on (rows may start at any element: the loads are
// only as aligned as the type); -inf past the row and at the mask token.
template <typename T, int N>
__device__ __forceinline__ void load_logits(const T* x, int v, int V, int mask_id, float (&f)[N]) {
  struct __attribute__((packed, aligned(sizeof(T)))) Run {
    T e[N];
  };
  if (v + N <= V) {
    const Run r = *reinterpret_cast<const Run*>(x + v);
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = to_f(r.e[i]);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = v + i < V ? to_f(x[v + i]) : -INFINITY;
  }
  if ((uint32_t)(mask_id - v) < (uint32_t)N) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (v + i == mask_id) f[i] = -INFINITY;
  }
}

template <typename T>
__global__ void __launch_bounds__(NT1) sample_chunk_kernel(SampleArgs a, SampleWs w) {
  __shared__ uint64_t mass[BINS];
  __shared__ uint32_t count[BINS];
  __shared__ float s_top[NT1 / 64];
  __shared__ uint32_t s_bad[NT1 / 64], s_arg[NT1 / 64];
  __shared__ uint64_t s_sum[NT1 / 64];
  __shared__ double s_sum1[NT1 / 64];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int row = blockIdx.x / w.chunks, chunk = blockIdx.x % w.chunks, v0 = chunk * CHUNK;
  const T* x = static_cast<const T*>(a.logits) + (long)row * a.row_stride;
  const Controls c = controls_of(a, row);
  constexpr int N = 16 / sizeof(T), RUNS = E1 / N;  // 16-byte runs
  float f[RUNS][N];
#pragma unroll
  for (int i = 0; i < RUNS; ++i) load_logits<T, N>(x, v0 + (i * NT1 + tid) * N, a.vocab, a.mask_id, f[i]);
  if (c.filter) {
    mass[tid] = 0;
    count[tid] = 0;
  }
  float top = -INFINITY;
  uint32_t bad = ~0u;
#pragma unroll
  for (int i = 0; i < RUNS; ++i)
#pragma unroll
    for (int e = 0; e < N; ++e) {
      if (!(f[i][e] < INFINITY)) {
        bad = min(bad, (uint32_t)(v0 + (i * NT1 + tid) * N + e));
        f[i][e] = -INFINITY;
      }
      top = fmaxf(top, f[i][e]);
    }
  top = wave_all(top, [](float p, float q) { return fmaxf(p, q); });
  bad = wave_all(bad, [](uint32_t p, uint32_t q) { return min(p, q); });
  if (lane == 0) {
    s_top[wave] = top;
    s_bad[wave] = bad;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NT1 / 64; ++i) {
    top = fmaxf(top, s_top[i]);
    bad = min(bad, s_bad[i]);
  }
  ChunkStat* out = w.stat + blockIdx.x;
  if (top == -INFINITY) {  // no candidate here
    if (tid == 0) *out = ChunkStat{top, bad, ~0u, 0, 0, 0.0};
    return;
  }
  uint32_t arg = ~0u;
  uint64_t sum = 0;
  float sum1 = 0.f;
  const double rate = c.inv_t * BINS_PER_NAT, base = class_of(top, rate);
#pragma unroll
  for (int i = 0; i < RUNS; ++i)
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const float y = f[i][e];
      sum1 += __builtin_amdgcn_exp2f((y - top) * 1.4426950408889634f);
      if (c.greedy) {
        if (y == top) arg = min(arg, (uint32_t)(v0 + (i * NT1 + tid) * N + e));
      } else if (y > -INFINITY) {
        const uint64_t u = fixed50(exp_neg(((double)y - top) * c.inv_t));
        sum += u;
        if (c.filter) {
          const int b = (int)fmin(base - class_of(y, rate), (double)(BINS - 1));
          atomicAdd(reinterpret_cast<unsigned long long*>(mass + b), (unsigned long long)u);
          atomicAdd(count + b, 1u);
        }
      }
    }
  arg = wave_all(arg, [](uint32_t p, uint32_t q) { return min(p, q); });
  sum = wave_all((unsigned long long)sum, [](unsigned long long p, unsigned long long q) { return p + q; });
  const double d1 = wave_all((double)sum1, [](double p, double q) { return p + q; });
  if (lane == 0) {
    s_arg[wave] = arg;
    s_sum[wave] = sum;
    s_sum1[wave] = d1;
  }
  __syncthreads();
  if (tid == 0) {
    ChunkStat s{top, bad, ~0u, 0, 0, 0.0};
    for (int i = 0; i < NT1 / 64; ++i) {
      s.arg = min(s.arg, s_arg[i]);
      s.sum += s_sum[i];
      s.sum1 += s_sum1[i];
    }
    *out = s;
  }
  if (c.filter) {
    w.mass[(size_t)blockIdx.x * BINS + tid] = mass[tid];
    w.count[(size_t)blockIdx.x * BINS + tid] = count[tid];
  }
}

// Inclusive scan over the workgroup's threads.
template <typename V>
__device__ __forceinline__ V block_scan(V x, V* buf) {
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    const V y = __shfl_up(x, s, 64);
    if (lane >= s) x += y;
  }
  if (lane == 63) buf[wave] = x;
  __syncthreads();
  V before = 0;
  for (int i = 0; i < wave; ++i) before += buf[i];
  __syncthreads();
  return x + before;
}

// A class's members up to a boundary: those with a key above `cut`, and those
// with it up to index `last`.
struct Cut {
  uint32_t key, last;
  double mass;  // of the members kept
};

template <typename T>
__global__ void __launch_bounds__(NT2) sample_row_kernel(SampleArgs a, SampleWs w) {
  __shared__ double fac[MAX_CHUNKS];    // weight of a chunk's maximum
  __shared__ int shift[MAX_CHUNKS];     // classes between the row's maximum and the chunk's
  __shared__ double part[MAX_CHUNKS];   // kept mass of a chunk
  __shared__ uint64_t extra[MAX_CHUNKS];
  __shared__ uint2 list[LIST];          // (key, index) of a class's members
  __shared__ uint64_t sub_mass[NT2];
  __shared__ uint32_t sub_count[NT2];
  __shared__ double binw[BINS];         // inclusive prefix sums
  __shared__ uint32_t binc[BINS];
  __shared__ double bufd[NT2 / 64];
  __shared__ uint32_t bufu[NT2 / 64];
  __shared__ uint32_t s_a, s_b, s_n;
  __shared__ int s_i;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int row = blockIdx.x, nch = w.chunks, V = a.vocab;
  const T* x = static_cast<const T*>(a.logits) + (long)row * a.row_stride;
  const ChunkStat* stat = w.stat + (size_t)row * nch;
  const Controls c = controls_of(a, row);
  auto answer = [&](int token, float conf, float prob) {
    a.token[row] = token;
    if (a.conf) a.conf[row] = conf;
    if (a.prob) a.prob[row] = prob;
  };

  // ---- the row's maximum, and what ends the search at once
  float big = -INFINITY;
  uint32_t bad = ~0u;
  for (int i = lane; i < nch; i += 64) {  // every wave by itself
    big = fmaxf(big, stat[i].top);
    bad = min(bad, stat[i].bad);
  }
  big = wave_all(big, [](float p, float q) { return fmaxf(p, q); });
  bad = wave_all(bad, [](uint32_t p, uint32_t q) { return min(p, q); });
  if (bad != ~0u || big == -INFINITY) {
    if (tid == 0) {
      if (bad != ~0u)
        answer((int)bad, NAN, NAN);
      else
        answer(-1, 0.f, 0.f);
    }
    return;
  }
  double all1 = 0;
  uint32_t arg = ~0u;
  for (int i = lane; i < nch; i += 64) {
    const ChunkStat s = stat[i];
    if (s.top > -INFINITY) all1 += s.sum1 * exp_neg((double)s.top - big);
    if (s.top == big) arg = min(arg, s.arg);
  }
  all1 = wave_all(all1, [](double p, double q) { return p + q; });
  if (c.greedy) {
    arg = wave_all(arg, [](uint32_t p, uint32_t q) { return min(p, q); });
    if (tid == 0) answer((int)arg, (float)(1.0 / all1), 1.f);
    return;
  }
  const double rate = c.inv_t * BINS_PER_NAT, base = class_of(big, rate);
  for (int i = tid; i < nch; i += NT2) {
    const ChunkStat s = stat[i];
    // a chunk with mass has a token with mass: its maximum
    const double e = s.top > -INFINITY ? exp_neg(((double)s.top - big) * c.inv_t) : 0.0;
    const bool some = e >= LEAST;
    fac[i] = some ? e : 0.0;
    shift[i] = some ? (int)fmin(base - class_of(s.top, rate), (double)BINS) : BINS;
    part[i] = (double)s.sum * 0x1p-50 * fac[i];  // everything kept
    extra[i] = 0;
  }
  auto weight = [&](float f) {
    const double e = exp_neg(((double)f - big) * c.inv_t);
    return e < LEAST ? 0.0 : e;
  };
  auto bin_of = [&](float f) { return (int)fmin(base - class_of(f, rate), (double)(BINS - 1)); };
  __syncthreads();

  // ---- the boundary: classes below `edge` are kept whole, of class `edge` the members up to `cut`
  int edge = BINS;
  Cut cut{0, ~0u, 0};
  double scale = 1.0, reach = INFINITY;  // reach: the largest (max - x) / T that min-p keeps in class `edge`
  auto stays = [&](float f, uint32_t key, uint32_t v) {  // a member of class `edge`
    return ((double)big - f) * c.inv_t <= reach && (key > cut.key || (key == cut.key && v <= cut.last));
  };
  if (c.filter) {
    double m = 0;
    uint32_t n = 0;
    if (tid < BINS) {
      const uint64_t* hm = w.mass + (size_t)row * nch * BINS;
      const uint32_t* hc = w.count + (size_t)row * nch * BINS;
      for (int i = 0; i < nch; ++i) {
        const int k = tid - shift[i];
        // what a chunk's last class holds has no mass in the row either
        if (k >= 0 && shift[i] < BINS && tid < BINS - 1 && k < BINS - 1) {
          m += (double)hm[(size_t)i * BINS + k] * 0x1p-50 * fac[i];
          n += hc[(size_t)i * BINS + k];
        }
      }
    }
    const double cm = block_scan(m, bufd);
    const uint32_t cn = block_scan(n, bufu);
    if (tid < BINS) {
      binw[tid] = cm;
      binc[tid] = cn;
    }
    __syncthreads();
    auto mass_before = [&](int b) { return b > 0 ? binw[b - 1] : 0.0; };
    auto count_before = [&](int b) { return b > 0 ? binc[b - 1] : 0u; };

    // members of class b: into the list where they fit, else they are found in the row each time
    int listed = -1;
    auto scan_row = [&](int b, auto&& f) {
      // logits that can be in the class, with a margin that covers float32
      const double hi = (base - b + 1) / rate, lo = (base - b) / rate;
      const float fhi = rate > 0 ? (float)(hi + fabs(hi) * 1e-6) : INFINITY, flo = rate > 0 ? (float)(lo - fabs(lo) * 1e-6) : -INFINITY;
      constexpr int N = 16 / sizeof(T), U = 32 / N;
      for (int v0 = 0; v0 < V; v0 += NT2 * N * U) {
        float y[U][N];
#pragma unroll
        for (int i = 0; i < U; ++i) {
          const int v = v0 + (i * NT2 + tid) * N;
          load_logits<T, N>(x, v, V, a.mask_id, y[i]);
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
          const int v = v0 + (i * NT2 + tid) * N;
#pragma unroll
          for (int e = 0; e < N; ++e)
            if (y[i][e] >= flo && y[i][e] <= fhi && y[i][e] > -INFINITY && bin_of(y[i][e]) == b)
              f(key_of(y[i][e]), (uint32_t)(v + e));
        }
      }
    };
    auto members = [&](int b, auto&& f) {
      const uint32_t n = binc[b] - count_before(b);
      if (n > LIST) {
        scan_row(b, f);
        return;
      }
      if (listed != b) {
        __syncthreads();
        if (tid == 0) s_n = 0;
        __syncthreads();
        scan_row(b, [&](uint32_t key, uint32_t v) {
          const uint32_t at = atomicAdd(&s_n, 1u);
          if (at < LIST) list[at] = make_uint2(key, v);
        });
        __syncthreads();
        listed = b;
      }
      const int have = min((int)s_n, LIST);
      for (int i = tid; i < have; i += NT2) f(list[i].x, list[i].y);
    };
    // The members of class b that stay when at most `limit` of them may and, with
    // `mass` of them before it, one must have less than `target`: narrows the
    // range of keys, then of indices, by NT2 parts at a time.
    auto select = [&](int b, uint32_t limit, double target) {
      target = fmax(target, 1e-300);  // the first of all stays
      // whole numbers in 2^-40 of the class's largest possible weight
      scale = 0x1p40 / fmin(exp_neg(-(double)(b - 1) / BINS_PER_NAT), 1.0);
      auto fixed = [&](uint32_t key) { return (unsigned long long)(weight(value_of(key)) * scale); };
      __syncthreads();
      if (tid == 0) {
        s_a = ~0u;
        s_b = 0;
      }
      __syncthreads();
      uint32_t lo = ~0u, hi = 0;
      members(b, [&](uint32_t key, uint32_t) {
        lo = min(lo, key);
        hi = max(hi, key);
      });
      lo = wave_all(lo, [](uint32_t p, uint32_t q) { return min(p, q); });
      hi = wave_all(hi, [](uint32_t p, uint32_t q) { return max(p, q); });
      if (lane == 0) {
        atomicMin(&s_a, lo);
        atomicMax(&s_b, hi);
      }
      __syncthreads();
      lo = s_a;
      hi = s_b;
      uint32_t n0 = 0;   // members and mass ranked before the range
      double m0 = 0;
      // part i of the range, highest keys first; returns false if nothing reaches a limit
      auto narrow = [&](uint32_t span, auto&& each, uint32_t& from, uint32_t& to) {
        const int sh = span >= NT2 ? 32 - __clz(span) - 9 : 0;  // span >> sh < NT2 = 2^9
        sub_mass[tid] = 0;
        sub_count[tid] = 0;
        if (tid == 0) s_i = -1;
        __syncthreads();
        each([&](uint32_t at, uint32_t key) {
          atomicAdd(reinterpret_cast<unsigned long long*>(sub_mass + (at >> sh)), fixed(key));
          atomicAdd(sub_count + (at >> sh), 1u);
        });
        __syncthreads();
        const uint32_t n1 = block_scan(sub_count[tid], bufu);
        const double m1 = block_scan((double)sub_mass[tid] / scale, bufd);
        const double mb = m1 - (double)sub_mass[tid] / scale;
        const uint32_t nb = n1 - sub_count[tid];
        const bool reached = n0 + n1 >= limit || m0 + m1 >= target;
        const bool before = tid > 0 && (n0 + nb >= limit || m0 + mb >= target);
        if (reached && !before && sub_count[tid] > 0) s_i = tid;
        __syncthreads();
        const int i = s_i;
        if (i < 0) return false;
        if (tid == i) {
          s_a = nb;
          bufd[0] = mb;
        }
        __syncthreads();
        n0 += s_a;
        m0 += bufd[0];
        from = (uint32_t)i << sh;
        to = min(span, (((uint32_t)i + 1) << sh) - 1);
        __syncthreads();
        return true;
      };
      Cut r{0, ~0u, 0};
      while (hi > lo) {
        uint32_t p = 0, q = 0;
        const uint32_t top = hi, bottom = lo;
        if (!narrow(hi - lo, [&](auto&& add) { members(b, [&](uint32_t key, uint32_t) { if (key >= bottom && key <= top) add(top - key, key); }); }, p, q)) {
          r.mass = binw[b] - mass_before(b);
          return r;  // all of them
        }
        hi = top - p;
        lo = top - q;
      }
      // the members equal to lo: those with the lowest indices
      const double each = weight(value_of(lo));
      const uint32_t ties = (uint32_t)fmax(fmin((double)(limit - n0), ceil((target - m0) / each)), 1.0);
      r.key = lo;
      r.mass = m0;
      uint32_t first = 0, last = (uint32_t)V - 1;
      const uint32_t want = n0 + ties;
      limit = want;
      target = INFINITY;
      bool all = false;
      while (last > first && !all) {
        uint32_t p = 0, q = 0;
        const uint32_t f0 = first, l0 = last;
        all = !narrow(last - first, [&](auto&& add) { members(b, [&](uint32_t key, uint32_t v) { if (key == lo && v >= f0 && v <= l0) add(v - f0, key); }); }, p, q);
        if (!all) {
          first = f0 + p;
          last = f0 + q;
        }
      }
      r.last = all ? ~0u : last;
      r.mass += (double)ties * each;
      return r;
    };
    // first class whose inclusive prefix reaches the limit, or -1
    auto find = [&](auto&& reached) {
      __syncthreads();
      if (tid == 0) s_i = -1;
      __syncthreads();
      if (tid < BINS - 1 && reached(tid) && (tid == 0 || !reached(tid - 1))) s_i = tid;
      __syncthreads();
      return s_i;
    };
    int bk = -1, bp = -1;
    uint32_t rk = 0;
    double target = INFINITY, whole = binw[BINS - 2];
    if (c.top_k) {
      bk = find([&](int b) { return binc[b] >= (uint32_t)c.top_k; });
      if (bk >= 0) {
        rk = c.top_k - count_before(bk);
        whole = binw[bk];
        if (rk == binc[bk] - count_before(bk)) {
          edge = bk + 1;  // the class stays whole
          bk = -1;
        } else {
          edge = bk;
          if (c.top_p < 1.0) {
            cut = select(bk, rk, INFINITY);
            whole = mass_before(bk) + cut.mass;
          }
        }
      }
    }
    if (c.top_p < 1.0) {
      target = c.top_p * whole;
      bp = find([&](int b) { return binw[b] >= target; });
      if (bp >= 0 && (bp < edge || bp == bk)) edge = bp;
      if (bp > edge) bp = -1;
    }
    int bm = -1;
    if (c.min_p > 0.0) {
      // w >= min_p as a distance, which stays exact where every w rounds to 1
      const double d = -log(c.min_p);
      bm = max((int)fmin(base - floor(((double)big * c.inv_t - d) * BINS_PER_NAT), (double)(BINS - 1)), 0);
      if (bm <= edge) {
        edge = bm;
        reach = d;
      }
    }
    const bool ranked = edge == bk || edge == bp, split = edge < BINS - 1 && (ranked || reach < INFINITY);
    if (split && ranked)
      cut = select(edge, edge == bk ? rk : ~0u, edge == bp ? target - mass_before(edge) : INFINITY);
    else
      cut = Cut{split ? 0 : ~0u, 0, 0};  // every member that min-p leaves, or none

    // ---- kept mass of each chunk: its classes before the edge, then the edge's members
    scale = 0x1p40 / fmin(exp_neg(-(double)(edge - 1) / BINS_PER_NAT), 1.0);
    __syncthreads();
    if (split)
      members(edge, [&](uint32_t key, uint32_t v) {
        if (stays(value_of(key), key, v))
          atomicAdd(reinterpret_cast<unsigned long long*>(extra + v / CHUNK), (unsigned long long)(weight(value_of(key)) * scale));
      });
    __syncthreads();
    for (int i = wave; i < nch; i += NT2 / 64) {
      const uint64_t* h = w.mass + ((size_t)row * nch + i) * BINS;
      unsigned long long s = 0;
      const int end = min(edge, BINS - 1) - shift[i];  // classes of the chunk before the edge
      for (int k = lane; k < min(end, BINS - 1); k += 64) s += h[k];
      s = wave_all(s, [](unsigned long long p, unsigned long long q) { return p + q; });
      if (lane == 0) part[i] = (double)s * 0x1p-50 * fac[i] + (double)extra[i] / scale;
    }
    __syncthreads();
  }
  auto kept = [&](float f, uint32_t v) {
    if (!(f > -INFINITY)) return 0.0;
    const double e = weight(f);
    if (!c.filter) return e;
    const int b = bin_of(f);
    if (b > edge || b >= BINS - 1) return 0.0;
    if (b < edge) return e;
    const uint32_t key = key_of(f);
    return stays(f, key, v) ? e : 0.0;
  };

  // ---- the chunk, then the token, where the running sum passes u times the whole
  double total = 0;
  for (int i = 0; i < nch; ++i) total += part[i];
  float u = a.u[row];
  u = u > 0.f ? fminf(u, 1.f - 0x1p-24f) : 0.f;
  const double want = (double)u * total;
  double before = 0;
  int at = 0;  // the sums run as the total's did, and want is less than that
  for (; at < nch - 1 && before + part[at] <= want; ++at) before += part[at];
  constexpr int E = CHUNK / NT2;
  const int v0 = at * CHUNK + tid * E;
  float y[E];
  load_logits<T, E>(x, v0, V, a.mask_id, y);
  double e[E], sum = 0;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    e[i] = kept(y[i], v0 + i);
    sum += e[i];
  }
  __syncthreads();
  if (tid == 0) {
    s_a = ~0u;
    s_b = 0;
  }
  const double incl = block_scan(sum, bufd);  // has barriers
  double run = before + (incl - sum);
  uint32_t mine = ~0u, final = 0;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    run += e[i];
    if (e[i] > 0.0) {
      final = v0 + i + 1;
      if (run > want && mine == ~0u) mine = v0 + i;
    }
  }
  if (mine != ~0u) atomicMin(&s_a, mine);
  if (final) atomicMax(&s_b, final);
  __syncthreads();
  if (tid == 0) {
    // (rounding inside the chunk: its last kept token)
    const uint32_t token = min(s_a != ~0u ? s_a : s_b - 1, (uint32_t)V - 1);
    const float f = to_f(x[token]);
    answer((int)token, (float)(exp_neg((double)f - big) / all1), (float)(weight(f) / total));
  }
}

int chunks_of(int vocab) { return ceil_div(vocab, CHUNK); }

}  // namespace

size_t sample_bytes(int rows, int vocab) {
  return (size_t)rows * chunks_of(vocab) * (sizeof(ChunkStat) + BINS * 12) + 256;
}

void launch_sample(const SampleArgs& a, void* ws, hipStream_t s) {
  SampleWs w{};
  w.chunks = chunks_of(a.vocab);
  const size_t n = (size_t)a.rows * w.chunks;
  w.mass = static_cast<uint64_t*>(ws);
  w.stat = reinterpret_cast<ChunkStat*>(w.mass + n * BINS);
  w.count = reinterpret_cast<uint32_t*>(w.stat + n);
  auto go = [&](auto* chunk, auto* row) {
    chunk<<<(unsigned)n, NT1, 0, s>>>(a, w);
    DLLM_LAUNCH_CHECK("sample_chunk_kernel");
    row<<<a.rows, NT2, 0, s>>>(a, w);
    DLLM_LAUNCH_CHECK("sample_row_kernel");
  };
  if (a.dtype == DLLM_F32)
    go(sample_chunk_kernel<float>, sample_row_kernel<float>);
  else
    go(sample_chunk_kernel<bf16_t>, sample_row_kernel<bf16_t>);
}

}  // namespace dllm
