// One row tile of attention: what the kernels that attend have in common.
//
// A row is one query of one head.  The G = n_heads / n_kv_heads query heads of a
// key/value head are rows of the same tile, so each key and value is read once for
// all of them.  A wave owns 32 rows and computes, per tile of KT keys,
//   S^T (keys x 32 rows) = K . Q^T      (Q held in registers)
// so that a lane holds scores of a single row, and the running maximum and sum of
// the softmax cost one exchange with lane ^ 32; then
//   O^T (hd x 32 rows) += V^T . P^T
// whose P^T operand is the score registers as they stand: the V^T operand takes
// its keys in the same order (bf16: LDS reads that transpose 4 x 16 blocks;
// float32: one key per lane half), so V is staged as it lies in memory.
//
// A workgroup has QG x KG waves: wave w takes the 32 rows w % QG of its row tile
// and the key tiles of group w / QG; the groups' states meet in LDS at the end.
// Each step brings KG tiles of K and V into an S-stage LDS ring by LDS-DMA.
#pragma once
#include <type_traits>

#include "kernels.h"
#include "lds_dma.h"

namespace dllm {

namespace {

typedef short v4s_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4s_t* lds_v4s_t;
typedef unsigned short v2us_t __attribute__((ext_vector_type(2)));

constexpr float LOG2E = 1.4426950408889634f;
// Sum of the lanes up to this one (within rows of 16 lanes, then over them).
__device__ __forceinline__ int lanes_upto(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
  return x;
}
typedef __bf16 bf2_t __attribute__((ext_vector_type(2)));
typedef float f2_t __attribute__((ext_vector_type(2)));
// Two floats to bf16 in one instruction, and acc + the sum of two bf16.
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2_t{lo, hi}, bf2_t));
}
__device__ __forceinline__ float add2(float acc, uint32_t w) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf2_t, w), __builtin_bit_cast(bf2_t, 0x3f803f80u), acc, false);
}
// 2^x by the hardware instruction alone: results below 2^-126 count as zero.
__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }
// max / sum over lanes l and l ^ 32, which hold the halves of one row's scores
__device__ __forceinline__ float max_pair32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_pair32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Two bf16, or a float, with NaN and infinities as zero.
template <typename T>
__device__ __forceinline__ uint32_t numbers(uint32_t w) {
  if constexpr (sizeof(T) == 2) {
    if ((w & 0x7f80u) == 0x7f80u) w &= 0xffff0000u;
    if ((w & 0x7f800000u) == 0x7f800000u) w &= 0xffffu;
  } else {
    if ((w & 0x7f800000u) == 0x7f800000u) w = 0;
  }
  return w;
}

// LDS tiles: rows of HD elements (one key each) in 16-byte chunks, chunk c of
// row r in slot c ^ swizzle(r), such that the lanes of one pass of a read meet
// all 64 banks: K is read in 16-byte chunks of 16 consecutive rows; V in four
// consecutive rows of 32 bf16 (the transposing read), or in 32 floats of rows r
// and r + 4.
template <typename T, int HD>
struct Tile {
  static constexpr int ROW = HD * (int)sizeof(T), CH = ROW / 16;  // bytes and chunks of a row
  static __device__ __forceinline__ int k_swz(int r) { return (CH >= 16 ? r : r >> 1) & (CH >= 16 ? 15 : 7); }
  static __device__ __forceinline__ int v_swz(int r) {
    if (sizeof(T) == 4) return ((r >> 2) & 1) << 3;
    return CH >= 16 ? (r & 3) << 2 : ((r >> 1) & 1) << 2;
  }
};

// LDS tiles hold what LDS-DMA brought and are read as several types; accesses that
// the compiler must not move past each other for their types' sake go through these.
typedef uint32_t __attribute__((may_alias)) word_t;
typedef uint32_t quad_t __attribute__((ext_vector_type(4), may_alias));
typedef float __attribute__((may_alias)) value_t;

// State of 32 rows: running maximum (log2 units) and what exponents are taken
// against (it, or 0 while it is -inf), sum and output; and what the lane's row is.
template <int HD>
struct Rows {
  f32x16_t o[HD / 32];
  float m, m_ref, l;
  int t, h, end;  // query, head, keys that it sees
  int at;         // position that its distances are taken from
  bool mine;      // there is such a row
  float slope;
};

// A document's ranges, cut to its slab and to the maxima.
struct Doc {
  int q0, nq, k0, nk, pos, prefix;
};
__device__ __forceinline__ Doc doc_of(const AttnArgs& a, int d) {
  Doc r;
  r.q0 = a.q_start ? min(max(a.q_start[d], 0), a.q_tokens) : 0;
  r.nq = min(min(max(a.q_len ? a.q_len[d] : a.q_tokens, 0), a.q_tokens - r.q0), a.max_q);
  r.k0 = a.kv_start ? min(max(a.kv_start[d], 0), a.kv_tokens) : 0;
  r.nk = min(min(max(a.kv_len ? a.kv_len[d] : a.kv_tokens, 0), a.kv_tokens - r.k0), a.max_kv);
  r.pos = a.q_pos ? a.q_pos[d] : r.nk - r.nq;
  r.prefix = a.prefix ? a.prefix[d] : 0;
  return r;
}
// Keys 0 .. n - 1 that query t of the document sees.
__device__ __forceinline__ int sees(const AttnArgs& a, const Doc& d, int t) {
  if (a.block == 0) return d.nk;
  const long i = (long)d.pos + t;
  int n = 0;  // a position before 0: its own block ends at or before position 0
  if (i >= d.nk)
    n = d.nk;
  else if (i >= 0)
    n = (int)min((long)d.nk, ((long)((uint32_t)i / (uint32_t)a.block) + 1) * a.block);
  return max(n, min(d.prefix, d.nk));
}

// Keys kb .. ke - 1 of a document (kp, vp: its first, as bytes; ksb, vsb: from one to
// the next); tile_first: keys that every row of the tile sees; see_first, see_last:
// those that the first and the last row of this wave see (rows in rising order).
struct Keys {
  const char *kp, *vp;
  uint32_t ksb, vsb;
  int kb, ke, tile_first, see_first, see_last;
  __device__ __forceinline__ int steps(int step) const { return ke > kb ? (ke - kb + step - 1) / step : 0; }
};
// The keys of head g from token k0 of slab b on.
template <typename T>
__device__ __forceinline__ Keys keys_at(const AttnView& k, const AttnView& v, long b, long k0, int g) {
  Keys r;
  r.kp = uniform(static_cast<const char*>(k.data) + (b * k.stride_b + k0 * k.stride_l + g * k.stride_h) * (long)sizeof(T));
  r.vp = uniform(static_cast<const char*>(v.data) + (b * v.stride_b + k0 * v.stride_l + g * v.stride_h) * (long)sizeof(T));
  r.ksb = (uint32_t)(k.stride_l * sizeof(T));
  r.vsb = (uint32_t)(v.stride_l * sizeof(T));
  return r;
}

// Bytes of LDS that a tile needs.
template <typename T, int HD, int QG, int KG, int KT, int S>
constexpr int attend_lds() {
  const int stages = S * KG * 2 * KT * Tile<T, HD>::ROW, merge = (QG * KG - QG) * (HD / 32 * 4 + 1) * 64 * 16;
  return stages > merge ? stages : merge;
}

// State R of a row tile over the keys k1, and with CHAIN over those and then k2's (of
// k1's, which stand before k2's, every row sees all).  rows_of(R) says what the lane's
// row is and returns its query (any row's where there is none); done(R) is called with
// the state of each row that there is.
template <typename T, int HD, int QG, int KG, int KT, int S, bool CHAIN, typename RowsOf, typename Done>
__device__ __forceinline__ void attend(const AttnArgs& a, char* lds, int tid, const Keys& k1, const Keys& k2, RowsOf rows_of, Done done) {
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int qg = wave % QG, kg = wave / QG, lq = lane & 31, half = lane >> 5;
#include "attn_tile_body.h"
  if (R.mine) done(R);
}

// The lane's row is finished: to its place in out.
template <typename T, int HD>
__device__ __forceinline__ void store_row(const Rows<HD>& R, T* to) {
  const int half = (threadIdx.x & 63) >> 5;
  const float inv = R.l == 0.f ? 0.f : 1.f / R.l;
#pragma unroll
  for (int ds = 0; ds < HD / 32; ++ds)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int e = ds * 32 + 8 * r + 4 * half;
      const float4 w = make_float4(R.o[ds][4 * r] * inv, R.o[ds][4 * r + 1] * inv, R.o[ds][4 * r + 2] * inv, R.o[ds][4 * r + 3] * inv);
      if constexpr (sizeof(T) == 2)
        *reinterpret_cast<uint2*>(to + e) = make_uint2(pack2(w.x, w.y), pack2(w.z, w.w));
      else
        *reinterpret_cast<float4*>(to + e) = w;
    }
}
// Or its state, to be joined: hd outputs, then (m, l).
template <int HD>
__device__ __forceinline__ void keep_state(const Rows<HD>& R, float* part, float2* part_ml, size_t at) {
  const int half = (threadIdx.x & 63) >> 5;
  float* to = part + at * HD;
#pragma unroll
  for (int ds = 0; ds < HD / 32; ++ds)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      *reinterpret_cast<float4*>(to + ds * 32 + 8 * r + 4 * half) =
          make_float4(R.o[ds][4 * r], R.o[ds][4 * r + 1], R.o[ds][4 * r + 2], R.o[ds][4 * r + 3]);
  if (half == 0) part_ml[at] = make_float2(R.m, R.l);
}

// Joins a row's n states, the i-th at index at(i), in their order: W waves per row,
// their lanes first a state's (maximum, sum) each, then 16 bytes of output each, in
// HD / 4 lanes per state, W 256 / HD states side by side.  (Workgroups of 256 threads;
// W > 1: one row each.)
template <typename T, int HD, int W, typename At>
__device__ __forceinline__ void join_row(T* to, int n, const float* part, const float2* part_ml, At at) {
  constexpr int LPC = HD / 4, SIDE = 64 / LPC * W;  // lanes per state, states side by side
  __shared__ float4 sums[W > 1 ? W - 1 : 1][LPC];
  const int lane = threadIdx.x & 63, wave = (threadIdx.x >> 6) % W;  // of the row
  const int e = lane % LPC * 4, side = wave * (64 / LPC) + lane / LPC;
  part += e;
  constexpr int EARLY = 4;  // outputs asked for beside the first maxima and sums
  float4 early[EARLY];
#pragma unroll
  for (int j = 0; j < EARLY; ++j)
    early[j] = j * SIDE + side < n ? *reinterpret_cast<const float4*>(part + at(j * SIDE + side) * HD) : make_float4(0.f, 0.f, 0.f, 0.f);
  float m = -INFINITY, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](const float4& w, float f) {
    o.x += w.x * f;
    o.y += w.y * f;
    o.z += w.z * f;
    o.w += w.w * f;
  };
  for (int c0 = 0; c0 < n; c0 += 64) {  // 64 chunks at a time, on the maximum so far
    float2 s = make_float2(-INFINITY, 0.f);
    if (c0 + lane < n) s = part_ml[at(c0 + lane)];
    float top = s.x;
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor(top, x, 64));
    const float m_new = fmaxf(m, top), ref = m_new == -INFINITY ? 0.f : m_new, f0 = exp2_hw(m - ref);
    m = m_new;
    const float f = exp2_hw(s.x - ref);
    l = l * f0 + warp_sum(s.y * f);
    o.x *= f0;
    o.y *= f0;
    o.z *= f0;
    o.w *= f0;
    const int here = min(64, n - c0);
    if (c0 == 0) {
#pragma unroll
      for (int j = 0; j < EARLY; ++j) {
        const float fc = __shfl(f, j * SIDE + side, 64);
        if (j * SIDE + side < here) add(early[j], fc);
      }
    }
#pragma unroll 4
    for (int i = c0 == 0 ? EARLY * SIDE : 0; i < here; i += SIDE) {
      const int c = min(i + side, here - 1);
      const float fc = __shfl(f, c, 64);
      const float4 w = *reinterpret_cast<const float4*>(part + at(c0 + c) * HD);
      if (i + side < here) add(w, fc);
    }
  }
#pragma unroll
  for (int x = LPC; x < 64; x <<= 1) {
    o.x += __shfl_xor(o.x, x, 64);
    o.y += __shfl_xor(o.y, x, 64);
    o.z += __shfl_xor(o.z, x, 64);
    o.w += __shfl_xor(o.w, x, 64);
  }
  if constexpr (W > 1) {
    if (wave > 0 && lane < LPC) sums[wave - 1][lane] = o;
    __syncthreads();
    if (side > 0) return;
#pragma unroll
    for (int i = 0; i < W - 1; ++i) add(sums[i][lane], 1.f);
  }
  if (side > 0) return;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  to += e;
  if constexpr (sizeof(T) == 2)
    *reinterpret_cast<uint2*>(to) = make_uint2(pack2(o.x * inv, o.y * inv), pack2(o.z * inv, o.w * inv));
  else
    *reinterpret_cast<float4*>(to) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
}

}  // namespace

}  // namespace dllm
