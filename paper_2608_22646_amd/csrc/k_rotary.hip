// Rotary positions of query and key heads: pairs (j, j + rot/2) or (2j, 2j + 1)
// of the first rot elements of each head turned by the angle p f_j.
//
// Every element is read and written once and costs three operations: HBM bounds
// it (5.1 .. 5.4 TB/s measured, a copy's rate).  What could cost more is the angle.  A token's rot/2 sines and cosines are
// the same for all its heads, so a workgroup takes a few whole tokens, forms
// their table once in LDS (one pair per thread) and then streams the heads'
// 16-byte pieces past it.  The angle p f_j is formed in float64 in quarter
// turns, where removing whole ones is exact; the remainder (at most half a
// quarter) goes to float32, so a position of any size costs no accuracy.
#include <algorithm>

#include "kernels.h"

namespace dllm {

namespace {

constexpr int NT = 256, MAX_TOKENS = 16;

template <typename T, int VEC>
struct alignas(VEC * sizeof(T)) Piece {
  T v[VEC];
};

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(bf16_t x) { return bf2f(x); }
__device__ __forceinline__ void from_f(float& y, float x) { y = x; }
__device__ __forceinline__ void from_f(bf16_t& y, float x) { y = f2bf(x); }

// Quarter turns per position of pair j.
__device__ double pair_rate(const RotaryArgs& a, int j) {
  double f = exp2(-2.0 * j / a.rot * a.log2_base);
  if (a.scaling == DLLM_ROPE_LINEAR) {
    f /= a.factor;
  } else if (a.scaling == DLLM_ROPE_PARTS) {
    const double g = fmin(fmax((a.orig_len * f / (2 * M_PI) - a.low) / (a.high - a.low), 0.0), 1.0);
    f = (1.0 - g) * f / a.factor + g * f;
  }
  return f * (2.0 / M_PI);
}

// Where a token's rows start, in elements.
struct TokenAt {
  int64_t q, q_out, k, k_out;
};

// VEC elements a piece (16 bytes), or single elements where sizes, strides or
// addresses do not allow pieces.  An item is what one thread turns at a time:
// two pieces of a half-layout head, one piece (or one pair) of an interleaved
// one, or a piece to pass through.  A thread walks its items (token, head, item
// of the head) by steps of the workgroup's size, without a division.
template <typename T, int VEC, bool INTER>
__global__ void __launch_bounds__(NT) rotary_kernel(RotaryArgs a) {
  extern __shared__ float table[];  // [tokens][2][rot / 2]: cos, sin
  __shared__ TokenAt start[MAX_TOKENS];
  const int half = a.rot / 2;
  const long total = (long)a.B * a.L;
  typedef Piece<T, VEC> P;
  constexpr int PAIRS = INTER ? (VEC > 1 ? VEC / 2 : 1) : VEC;  // pairs per item
  const int turned = half / PAIRS, per_head = turned + (a.hd - a.rot) / VEC;
  const int heads = a.n_q + a.n_k;
  // the step of NT items as (tokens, heads, items of a head), and the first item
  const int step_c = NT % per_head, step_r = NT / per_head, step_h = step_r % heads, step_t = step_r / heads;
  const int c0 = threadIdx.x % per_head, r0 = threadIdx.x / per_head, h0 = r0 % heads, ti0 = r0 / heads;
  for (long t0 = (long)blockIdx.x * a.tokens; t0 < total; t0 += (long)gridDim.x * a.tokens) {
    const int nt = (int)min((long)a.tokens, total - t0);
    for (int i = threadIdx.x; i < nt * half; i += NT) {
      const int j = i % half;
      const long t = t0 + i / half;
      const long p = a.pos ? (long)a.pos[t] : (long)a.pos0 + t % a.L;
      const double q = (double)p * pair_rate(a, j);
      const double k = rint(q);
      float s, c;
      sincospif(0.5f * (float)(q - k), &s, &c);  // |argument| <= 1/4
      const int quad = (int)(k - 4.0 * floor(k * 0.25));
      const float cs = quad & 1 ? s : c, sn = quad & 1 ? c : s;
      float* tok = table + (i / half) * 2 * half;
      tok[j] = (quad == 1 || quad == 2 ? -cs : cs) * a.gain;
      tok[half + j] = ((quad == 2 || quad == 3) != (a.inverse != 0) ? -sn : sn) * a.gain;
    }
    if ((int)threadIdx.x < nt) {
      const long t = t0 + threadIdx.x, b = t / a.L, l = t - b * a.L;
      start[threadIdx.x] = TokenAt{b * a.q.stride_b + l * a.q.stride_l, b * a.q_out.stride_b + l * a.q_out.stride_l,
                                   b * a.k.stride_b + l * a.k.stride_l, b * a.k_out.stride_b + l * a.k_out.stride_l};
    }
    __syncthreads();
    int c = c0, h = h0, ti = ti0;
    while (ti < nt) {
      const bool is_q = h < a.n_q;
      const TokenAt& at = start[ti];
      const T* x = is_q ? static_cast<const T*>(a.q.data) + at.q + h * a.q.stride_h
                        : static_cast<const T*>(a.k.data) + at.k + (h - a.n_q) * a.k.stride_h;
      T* y = is_q ? static_cast<T*>(a.q_out.data) + at.q_out + h * a.q_out.stride_h
                  : static_cast<T*>(a.k_out.data) + at.k_out + (h - a.n_q) * a.k_out.stride_h;
      const float* cs = table + ti * 2 * half + c * PAIRS;
      const float* sn = cs + half;
      if (c >= turned) {
        const int e = a.rot + (c - turned) * VEC;
        *reinterpret_cast<P*>(y + e) = *reinterpret_cast<const P*>(x + e);
      } else if constexpr (INTER && VEC > 1) {
        const P u = *reinterpret_cast<const P*>(x + c * VEC);
        P w;
#pragma unroll
        for (int e = 0; e < PAIRS; ++e) {
          const float p = to_f(u.v[2 * e]), q = to_f(u.v[2 * e + 1]);
          from_f(w.v[2 * e], p * cs[e] - q * sn[e]);
          from_f(w.v[2 * e + 1], q * cs[e] + p * sn[e]);
        }
        *reinterpret_cast<P*>(y + c * VEC) = w;
      } else {
        const int ia = INTER ? 2 * c : c * VEC, ib = INTER ? ia + 1 : ia + half;
        const P u = *reinterpret_cast<const P*>(x + ia), v = *reinterpret_cast<const P*>(x + ib);
        P wu, wv;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float p = to_f(u.v[e]), q = to_f(v.v[e]);
          from_f(wu.v[e], p * cs[e] - q * sn[e]);
          from_f(wv.v[e], q * cs[e] + p * sn[e]);
        }
        *reinterpret_cast<P*>(y + ia) = wu;
        *reinterpret_cast<P*>(y + ib) = wv;
      }
      c += step_c;
      h += step_h;
      ti += step_t;
      if (c >= per_head) {
        c -= per_head;
        ++h;
      }
      if (h >= heads) {
        h -= heads;
        ++ti;
      }
    }
    __syncthreads();  // the table is free for the next tokens
  }
}

bool in_pieces(const RotaryRows& r, int n, int bytes, int size) {
  if (n == 0) return true;
  const long m = (r.stride_b | r.stride_l | r.stride_h) * size;
  return ((uintptr_t)r.data | (uintptr_t)m) % bytes == 0;
}

template <typename T>
void launch(RotaryArgs a, hipStream_t s) {
  constexpr int V = 16 / sizeof(T);
  const bool pieces = (a.inter ? a.rot % V == 0 : a.rot / 2 % V == 0) && (a.hd - a.rot) % V == 0 &&
                      in_pieces(a.q, a.n_q, 16, sizeof(T)) && in_pieces(a.q_out, a.n_q, 16, sizeof(T)) &&
                      in_pieces(a.k, a.n_k, 16, sizeof(T)) && in_pieces(a.k_out, a.n_k, 16, sizeof(T));
  // Tokens a workgroup: four items a thread where tokens are many (28 + 4 bf16
  // heads x 8448 tokens: 25.8 us, 5.4 TB/s, against 29.7 at one token and 28.4 at
  // eight; 64 float32 heads x 4092 tokens, 2048 items each: one token 52.8 us,
  // 5.1 TB/s, two 61), fewer while that leaves less than four workgroups a CU.
  const int vec = pieces ? V : 1, pairs = a.inter ? std::max(vec / 2, 1) : vec;
  const long items = (long)(a.n_q + a.n_k) * (a.rot / 2 / pairs + (a.hd - a.rot) / vec), total = (long)a.B * a.L;
  a.tokens = (int)std::max(1l, std::min({4l * NT / items, (long)MAX_TOKENS, total / (4l * device_cu_count())}));
  const int grid = std::min(ceil_div((long)a.B * a.L, a.tokens), 1 << 20);
  const size_t lds = (size_t)a.tokens * a.rot * sizeof(float);
  auto* f = pieces ? (a.inter ? rotary_kernel<T, V, true> : rotary_kernel<T, V, false>)
                   : (a.inter ? rotary_kernel<T, 1, true> : rotary_kernel<T, 1, false>);
  f<<<grid, NT, lds, s>>>(a);
  DLLM_LAUNCH_CHECK("rotary_kernel");
}

}  // namespace

void launch_rotary(const RotaryArgs& a, hipStream_t s) {
  if (a.dtype == DLLM_F32)
    launch<float>(a, s);
  else
    launch<bf16_t>(a, s);
}

}  // namespace dllm
