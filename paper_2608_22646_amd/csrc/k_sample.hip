// Sampling of one token per row of logits from given random numbers (dllm_sample).
//
// Temperature, top-k, top-p and min-p each keep a prefix of one ranking (logit
// descending, index ascending), so the kept set is described by a logit (as an
// ordered key), and how many of the candidates equal to it stay.
#include "kernels.h"

namespace dllm {

namespace {

constexpr int NT = 1024;

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

template <typename V>
__device__ V block_sum(V x, V* buf) {
  __syncthreads();
  buf[threadIdx.x] = x;
  __syncthreads();
  for (int s = NT / 2; s > 0; s >>= 1) {
    if (threadIdx.x < s) buf[threadIdx.x] += buf[threadIdx.x + s];
    __syncthreads();
  }
  const V r = buf[0];
  __syncthreads();
  return r;
}
__device__ uint32_t block_min(uint32_t x, uint32_t* buf) {
  __syncthreads();
  buf[threadIdx.x] = x;
  __syncthreads();
  for (int s = NT / 2; s > 0; s >>= 1) {
    if (threadIdx.x < s) buf[threadIdx.x] = min(buf[threadIdx.x], buf[threadIdx.x + s]);
    __syncthreads();
  }
  const uint32_t r = buf[0];
  __syncthreads();
  return r;
}

template <typename T>
__global__ void __launch_bounds__(NT) sample_kernel(SampleArgs a) {
  __shared__ double bufd[NT];
  uint32_t* bufu = reinterpret_cast<uint32_t*>(bufd);
  const int r = blockIdx.x, tid = threadIdx.x, V = a.vocab;
  const T* x = static_cast<const T*>(a.logits) + (long)r * a.row_stride;
  auto finish = [&](int token, float conf, float prob) {
    if (tid == 0) {
      a.token[r] = token;
      if (a.conf) a.conf[r] = conf;
      if (a.prob) a.prob[r] = prob;
    }
  };
  // the lowest index of NaN or +inf; the largest key; the lowest index that has it
  uint32_t bad = ~0u, top = 0;
  for (int v = tid; v < V; v += NT)
    if (v != a.mask_id) {
      const float f = to_f(x[v]);
      if (f != f || f == INFINITY)
        bad = min(bad, (uint32_t)v);
      else
        top = max(top, key_of(f));
    }
  bad = block_min(bad, bufu);
  if (bad != ~0u) return finish((int)bad, NAN, NAN);
  const uint32_t kmax = ~block_min(~top, bufu), kinf = key_of(-INFINITY);
  if (kmax <= kinf) return finish(-1, 0.f, 0.f);
  const double big = value_of(kmax);
  const float tf = a.temperature ? a.temperature[r] : 1.f;
  const bool greedy = !(tf > 0.f);
  const double inv_t = greedy ? 1.0 : 1.0 / (double)tf;
  auto weight = [&](float f) {
    const double w = exp((f - big) * inv_t);
    return w < 0x1p-64 ? 0.0 : w;
  };
  // sums over candidates with a key above (or: at least) k
  auto count = [&](uint32_t k) {
    uint32_t n = 0;
    for (int v = tid; v < V; v += NT)
      if (v != a.mask_id) n += key_of(to_f(x[v])) >= k;
    return (int)block_sum(n, bufu);
  };
  auto mass = [&](uint32_t k) {
    double m = 0;
    for (int v = tid; v < V; v += NT)
      if (v != a.mask_id) {
        const float f = to_f(x[v]);
        if (key_of(f) >= k && f > -INFINITY) m += weight(f);
      }
    return block_sum(m, bufd);
  };
  // kept: keys above `cut`, and the first `ties` of those equal to it
  uint32_t cut = kinf;
  int ties = 0;
  if (greedy) {
    cut = kmax;
    ties = 1;
  } else {
    const int tk = a.top_k ? a.top_k[r] : 0;
    if (tk >= 1 && tk < V && count(kinf + 1) > tk) {
      uint32_t lo = kinf + 1, hi = kmax;  // count(lo) >= tk; the largest such key
      while (lo < hi) {
        const uint32_t mid = lo + (hi - lo + 1) / 2;
        if (count(mid) >= tk)
          lo = mid;
        else
          hi = mid - 1;
      }
      cut = lo;
      ties = tk - count(lo + 1);
    }
    const float tp = a.top_p ? a.top_p[r] : 1.f;
    if (tp < 1.f) {
      const double wc = ties ? weight(value_of(cut)) : 0.0, above = mass(cut + 1);
      const double target = (double)tp * (above + ties * wc);
      // the lowest key whose mass above it is less than the target
      uint32_t lo = cut, hi = kmax;
      while (lo < hi) {
        const uint32_t mid = lo + (hi - lo) / 2;
        if (mass(mid + 1) < target)
          hi = mid;
        else
          lo = mid + 1;
      }
      const double w = weight(value_of(lo)), before = mass(lo + 1);
      if (lo > cut || ties) {
        const int all = lo == cut ? ties : count(lo) - count(lo + 1);
        int keep = all;
        if (w > 0) {
          const double need = ceil((target - before) / w);
          keep = need < 1 ? 1 : need < all ? (int)need : all;
        }
        cut = lo;
        ties = keep;
      }
    }
    const float mp = a.min_p ? a.min_p[r] : 0.f;
    if (mp > 0.f) {
      const double least = fmin((double)mp, 1.0);
      uint32_t lo = cut, hi = kmax;  // the lowest key with enough weight
      while (lo < hi) {
        const uint32_t mid = lo + (hi - lo) / 2;
        if (mid > kinf && weight(value_of(mid)) >= least)
          hi = mid;
        else
          lo = mid + 1;
      }
      if (lo > cut) {
        cut = lo - 1;
        ties = 0;
      }
    }
  }
  // the index up to which keys equal to cut are kept
  int last = -1;
  if (ties) {
    int lo = 0, hi = V - 1;
    while (lo < hi) {
      const int mid = lo + (hi - lo) / 2;
      uint32_t n = 0;
      for (int v = tid; v <= mid; v += NT) n += v != a.mask_id && key_of(to_f(x[v])) == cut;
      if ((int)block_sum(n, bufu) >= ties)
        hi = mid;
      else
        lo = mid + 1;
    }
    last = lo;
  }
  // prefix sums over contiguous segments, one per thread
  const int per = (V + NT - 1) / NT, v0 = min(tid * per, V), v1 = min(v0 + per, V);
  auto kept = [&](int v, float f) {
    if (v == a.mask_id || !(f > -INFINITY)) return 0.0;
    const uint32_t k = key_of(f);
    return k > cut || (k == cut && v <= last) ? (greedy ? 1.0 : weight(f)) : 0.0;
  };
  double seg = 0, all1 = 0;
  for (int v = v0; v < v1; ++v) {
    const float f = to_f(x[v]);
    seg += kept(v, f);
    if (v != a.mask_id) all1 += exp((double)f - big);
  }
  all1 = block_sum(all1, bufd);
  __syncthreads();
  bufd[tid] = seg;
  __syncthreads();
  double before = 0;
  for (int i = 0; i < tid; ++i) before += bufd[i];
  double total = 0;
  for (int i = 0; i < NT; ++i) total += bufd[i];
  float u = a.u[r];
  u = u > 0.f ? fminf(u, 1.f - 0x1p-24f) : 0.f;
  const double want = (double)u * total;
  __syncthreads();
  uint32_t mine = ~0u, final = 0;
  for (int v = v0; v < v1; ++v) {
    const double w = kept(v, to_f(x[v]));
    before += w;
    if (w > 0) {
      final = v + 1;
      if (before > want && mine == ~0u) mine = v;
    }
  }
  mine = block_min(mine, bufu);
  final = ~block_min(~final, bufu);
  const int token = mine != ~0u ? (int)mine : (int)final - 1;
  const float f = to_f(x[token]);
  finish(token, (float)(exp((double)f - big) / all1), (float)(kept(token, f) / total));
}

}  // namespace

size_t sample_bytes(int, int) { return 0; }

void launch_sample(const SampleArgs& a, void*, hipStream_t s) {
  if (a.dtype == DLLM_F32)
    sample_kernel<float><<<a.rows, NT, 0, s>>>(a);
  else
    sample_kernel<bf16_t><<<a.rows, NT, 0, s>>>(a);
  DLLM_LAUNCH_CHECK("sample_kernel");
}

}  // namespace dllm
