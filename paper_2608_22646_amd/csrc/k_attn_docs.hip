// Attention of documents of unlike lengths (dllm_attention): grouped heads,
// positional masks, capped scores and distance biases.
#include <algorithm>

#include "kernels.h"

namespace dllm {

namespace {

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(bf16_t x) { return bf2f(x); }
__device__ __forceinline__ void from_f(float& y, float x) { y = x; }
__device__ __forceinline__ void from_f(bf16_t& y, float x) { y = f2bf(x); }

// A document's ranges, cut to its slab and to the maxima.
struct Doc {
  int q0, nq, k0, nk, pos, prefix;
};
__device__ __forceinline__ Doc doc_of(const AttnArgs& a, int d) {
  auto cut = [](const int32_t* start, const int32_t* len, int d, int tokens, int most, int& s, int& n) {
    s = start ? min(max(start[d], 0), tokens) : 0;
    n = min(min(max(len ? len[d] : tokens, 0), tokens - s), most);
  };
  Doc r;
  cut(a.q_start, a.q_len, d, a.q_tokens, a.max_q, r.q0, r.nq);
  cut(a.kv_start, a.kv_len, d, a.kv_tokens, a.max_kv, r.k0, r.nk);
  r.pos = a.q_pos ? a.q_pos[d] : r.nk - r.nq;
  r.prefix = a.prefix ? a.prefix[d] : 0;
  return r;
}
// Keys 0 .. n - 1 that a query at position i sees.
__device__ __forceinline__ int sees(const AttnArgs& a, const Doc& d, long i) {
  if (a.block == 0) return d.nk;
  const long f = i >= 0 ? i / a.block : -((-i + a.block - 1) / a.block);  // floor
  return (int)min((long)d.nk, max(max((f + 1) * a.block, (long)d.prefix), 0l));
}

// One wave per (query, head): 64 keys at a time, one per lane, then the lanes
// take two dimensions each.
template <typename T, int HD>
__global__ void __launch_bounds__(64) attn_plain_kernel(AttnArgs a) {
  const int lane = threadIdx.x, h = blockIdx.y, dn = blockIdx.z;
  const Doc d = doc_of(a, dn);
  const int t = blockIdx.x;
  if (t >= d.nq) return;
  const int g = h / (a.Hq / a.Hkv);
  const T* q = static_cast<const T*>(a.q.data) + dn * a.q.stride_b + (long)(d.q0 + t) * a.q.stride_l + h * a.q.stride_h;
  const T* kb = static_cast<const T*>(a.k.data) + dn * a.k.stride_b + (long)d.k0 * a.k.stride_l + g * a.k.stride_h;
  const T* vb = static_cast<const T*>(a.v.data) + dn * a.v.stride_b + (long)d.k0 * a.v.stride_l + g * a.v.stride_h;
  T* o = static_cast<T*>(a.out.data) + dn * a.out.stride_b + (long)(d.q0 + t) * a.out.stride_l + h * a.out.stride_h;
  const long pos = (long)d.pos + t;
  const int n = sees(a, d, pos);
  const float slope = a.slopes ? a.slopes[h] : 0.f;
  __shared__ float ps[64];
  float m = -INFINITY, l = 0.f, acc[HD / 64] = {};
  for (int k0 = 0; k0 < n; k0 += 64) {
    const int j = k0 + lane;
    float s = -INFINITY;
    if (j < n) {
      s = 0.f;
      for (int e = 0; e < HD; ++e) s = fmaf(to_f(q[e]), to_f(kb[(long)j * a.k.stride_l + e]), s);
      s *= a.scale;
      if (a.cap > 0) s = a.cap * tanhf(s / a.cap);
      if (a.slopes) s -= slope * fabsf((float)(pos - j));
    }
    float top = s;
    for (int x = 32; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor(top, x, 64));
    const float m_new = fmaxf(m, top);
    const float ref = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = expf(m - ref), p = j < n ? expf(s - ref) : 0.f;
    m = m_new;
    l = l * alpha + warp_sum(p);
    __syncthreads();
    ps[lane] = p;
    __syncthreads();
    for (int e = 0; e < HD / 64; ++e) {
      acc[e] *= alpha;
      for (int x = 0; x < min(64, n - k0); ++x)
        acc[e] = fmaf(ps[x], to_f(vb[(long)(k0 + x) * a.v.stride_l + e * 64 + lane]), acc[e]);
    }
  }
  for (int e = 0; e < HD / 64; ++e) from_f(o[e * 64 + lane], l == 0.f ? 0.f : acc[e] / l);
}

}  // namespace

size_t attn_docs_bytes(const AttnArgs&) { return 0; }

void launch_attn_docs(const AttnArgs& a, void*, hipStream_t s) {
  const dim3 grid(a.max_q, a.Hq, a.docs);
  auto* f = a.dtype == DLLM_F32 ? (a.hd == 64 ? attn_plain_kernel<float, 64> : attn_plain_kernel<float, 128>)
                                : (a.hd == 64 ? attn_plain_kernel<bf16_t, 64> : attn_plain_kernel<bf16_t, 128>);
  f<<<grid, 64, 0, s>>>(a);
  DLLM_LAUNCH_CHECK("attn_plain_kernel");
}

}  // namespace dllm
