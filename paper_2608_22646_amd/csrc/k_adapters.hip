// Low-rank adapters of many requests beside a shared projection (dllm_adapters):
//   out = base + scale B (A x),  A and B those of the row's adapter.
//
// Both products run on tiles of up to 32 rows of one adapter.  Few rows: the rows of
// an adapter among 32 neighbours, found by the workgroup of the first of them.  Many
// rows: a first launch sorts the rows by adapter, so that a tile is full whatever
// their order.  Then
//   shrink: part[z][row][s, j] = the z-th share of sum_k A[s, j, k] x[row, k]; the
//     four waves of a workgroup take turns along k, operands straight from memory
//     (16 x 16 tiles, ranks by rows), and meet in LDS;
//   expand: the shares summed in their order and scaled, the sum in bf16 pieces that
//     hold 16 of its bits (24 for a float32 output) as the matrix unit's one operand,
//     B's rows as they lie in memory as the other; a wave computes 32 rows x 128
//     columns, column n = 8 c + i by lane c's i-th product, so that a lane reads and
//     writes 8 consecutive elements of base and out.
#include <algorithm>

#include "kernels.h"

namespace dllm {

namespace {

constexpr int TM = 32;           // rows of a tile
constexpr int COLS = 128;        // columns of a wave's block
constexpr int SORT_THREADS = 1024;

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int adapter_of(const AdaptersArgs& a, int row) {
  const int w = a.which[row];
  return w >= 0 && w < a.adapters ? w : -1;
}
__device__ __forceinline__ int rank_of(const AdaptersArgs& a, int adapter) {
  return a.ranks ? min(max(a.ranks[adapter], 0), a.rank) : a.rank;
}

// 16 bytes at p, of which the first n elements count (the rest give zeros and are
// not touched); whole: n is known to be all of them and p a multiple of 16.
template <typename T>
__device__ __forceinline__ u32x4_t piece(const T* p, int n, bool whole) {
  if (whole) return *reinterpret_cast<const u32x4_t*>(p);
  constexpr int E = 16 / sizeof(T);
  u32x4_t w = {0, 0, 0, 0};
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (e < n) {
      if constexpr (sizeof(T) == 2)
        w[e / 2] |= (uint32_t)p[e] << (16 * (e & 1));
      else
        w[e] = __float_as_uint(p[e]);
    }
  return w;
}

// A tile's rows in `rows` (LDS), how many, and their adapter (-1: none); count 0:
// there is no such tile.
struct Tile {
  int adapter, count;
};
__device__ __forceinline__ Tile tile_of(const AdaptersArgs& a, const AdaptersPlan& p, int i, int* rows) {
  const int lane = threadIdx.x & 63;
  Tile t;
  if (p.sorted) {
    const int4 d = p.tile[i];
    t = Tile{uniform(d.x), uniform(d.z)};
    if (threadIdx.x < TM && (int)threadIdx.x < t.count) rows[threadIdx.x] = p.order[d.y + threadIdx.x];
  } else {
    const int row = (i & ~(TM - 1)) + lane;
    const int w = lane < TM && row < a.rows ? adapter_of(a, row) : -2;
    t.adapter = __builtin_amdgcn_readlane(w, i & (TM - 1));
    const unsigned long long mine = __ballot(w == t.adapter);
    t.count = __ffsll(mine) - 1 == (i & (TM - 1)) ? __popcll(mine) : 0;
    if (threadIdx.x < 64 && w == t.adapter) rows[__popcll(mine & ((1ull << lane) - 1))] = row;
  }
  __syncthreads();
  return t;
}

// Sorts the rows by adapter (those without one last) and cuts them into tiles.  The
// order of an adapter's rows depends on the order of execution; no result does.
__global__ void __launch_bounds__(SORT_THREADS) adapters_sort_kernel(AdaptersArgs a, AdaptersPlan p) {
#if defined(__HIP_DEVICE_COMPILE__)
  extern __shared__ int sh[];
  const int bins = a.adapters + 1, tid = threadIdx.x, lane = tid & 63;
  int *const at = sh, *const tiles = sh + bins;  // rows' places, tiles' first ones
  __shared__ int2 sums[SORT_THREADS / 64];
  for (int i = tid; i < bins; i += SORT_THREADS) at[i] = 0;
  __syncthreads();
  // the place of each row among its bin's, by a wave at once where its rows share one
  auto add = [&](int row, bool there) {
    const int w = there ? adapter_of(a, row) : -1, bin = w < 0 ? a.adapters : w;
    const unsigned long long all = __ballot(there), same = __ballot(there && bin == uniform(bin));
    int pos = 0;
    if (same == all) {
      const int n = __popcll(all);
      if (lane == 0 && n) pos = atomicAdd(&at[bin], n);
      pos = uniform(pos) + __popcll(all & ((1ull << lane) - 1));
    } else if (there) {
      pos = atomicAdd(&at[bin], 1);
    }
    return pos;
  };
  for (int r0 = tid - lane; r0 < a.rows; r0 += SORT_THREADS) add(r0 + lane, r0 + lane < a.rows);
  __syncthreads();
  // sums of the bins before, `each` consecutive bins a thread
  const int each = (bins + SORT_THREADS - 1) / SORT_THREADS, b0 = min(tid * each, bins), b1 = min(b0 + each, bins);
  int2 mine = make_int2(0, 0);
  for (int b = b0; b < b1; ++b) {
    mine.x += at[b];
    mine.y += (at[b] + TM - 1) / TM;
  }
  int2 upto = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int x = __shfl_up(upto.x, o, 64), y = __shfl_up(upto.y, o, 64);
    if (lane >= o) {
      upto.x += x;
      upto.y += y;
    }
  }
  if (lane == 63) sums[tid >> 6] = upto;
  __syncthreads();
  int2 before = make_int2(upto.x - mine.x, upto.y - mine.y);
  int all_tiles = 0;
  for (int w = 0; w < SORT_THREADS / 64; ++w) {
    const int2 s = sums[w];
    if (w < (tid >> 6)) {
      before.x += s.x;
      before.y += s.y;
    }
    all_tiles += s.y;
  }
  for (int b = b0; b < b1; ++b) {
    const int n = at[b];
    at[b] = before.x;
    tiles[b] = before.y;
    before.x += n;
    before.y += (n + TM - 1) / TM;
  }
  __syncthreads();
  for (int i = tid; i < p.tiles; i += SORT_THREADS) {
    int4 d = make_int4(-1, 0, 0, 0);
    if (i < all_tiles) {
      int lo = 0, hi = bins - 1;  // the last bin whose first tile is at most i
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (tiles[mid] <= i)
          lo = mid;
        else
          hi = mid - 1;
      }
      const int first = at[lo] + (i - tiles[lo]) * TM, end = lo + 1 < bins ? at[lo + 1] : a.rows;
      d = make_int4(lo < a.adapters ? lo : -1, first, min(TM, end - first), 0);
    }
    p.tile[i] = d;
  }
  __syncthreads();
  for (int r0 = tid - lane; r0 < a.rows; r0 += SORT_THREADS) {
    const int row = r0 + lane, pos = add(row, row < a.rows);
    if (row < a.rows) p.order[pos] = row;
  }
#endif
}

template <typename T>
struct Kind {
  static constexpr int E = 16 / sizeof(T);  // elements of a piece
  static constexpr int STEP = 4 * E;        // along k: 64 bytes of a row, a piece for each 16 lanes
};

// c += the products of two fragments of a step
template <typename T>
__device__ __forceinline__ f32x4_t product(u32x4_t x, u32x4_t y, f32x4_t c) {
  if constexpr (sizeof(T) == 2)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, x), __builtin_bit_cast(bf16x8_t, y), c, 0, 0, 0);
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x[e]), __uint_as_float(y[e]), c, 0, 0, 0);
  return c;
}

// 16 MT rows by 16 J ranks (those of 16-blocks u0 .. of the adapter) over the steps
// of this share; acc[mt][j]: lane l holds row l % 16, ranks 4 (l / 16) ..
template <typename T, int MT, int J>
__device__ __forceinline__ void shrink_tile(const AdaptersArgs& a, const AdaptersPlan& p, const Tile& t, const int* rows, int u0, int n16,
                                            int s0, int s1, f32x4_t* red) {
  constexpr int E = Kind<T>::E, STEP = Kind<T>::STEP, U = J >= 8 ? 2 : J == 1 ? 8 : 4;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), l16 = lane & 15, g = lane >> 4;
  const T *x[MT], *w[J];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int i = m * 16 + l16;
    x[m] = static_cast<const T*>(a.x.data) + rows[i < t.count ? i : 0] * a.x.stride_l + g * E;
  }
  const int units = a.slices * n16, rank = rank_of(a, t.adapter);
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int u = min(u0 + j, units - 1), s = u / n16;
    w[j] = static_cast<const T*>(a.a.data) + t.adapter * a.a.stride_b + s * a.a.stride_h +
           min((u % n16) * 16 + l16, rank - 1) * a.a.stride_l + g * E;
  }
  f32x4_t acc[MT][J];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int j = 0; j < J; ++j) acc[m][j] = f32x4_t{0, 0, 0, 0};
  // steps whose pieces are whole, U at a time; then the rest, one at a time
  const int whole = p.vec_in ? min(s1, a.d_in / STEP) : s0;
  int b = s0 + wave * U;
  for (; b + U <= whole; b += 4 * U) {
    u32x4_t xf[U][MT], wf[U][J];
#pragma unroll
    for (int i = 0; i < U; ++i) {
#pragma unroll
      for (int m = 0; m < MT; ++m) xf[i][m] = *reinterpret_cast<const u32x4_t*>(x[m] + (long)(b + i) * STEP);
#pragma unroll
      for (int j = 0; j < J; ++j) wf[i][j] = *reinterpret_cast<const u32x4_t*>(w[j] + (long)(b + i) * STEP);
    }
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int j = 0; j < J; ++j) acc[m][j] = product<T>(wf[i][j], xf[i][m], acc[m][j]);
  }
  for (; b < s1; b += 4 * U)
    for (int i = b; i < min(b + U, s1); ++i) {
      const int n = a.d_in - i * STEP - g * E;
      const bool all = i < whole;
      u32x4_t xf[MT];
#pragma unroll
      for (int m = 0; m < MT; ++m) xf[m] = piece(x[m] + (long)i * STEP, n, all);
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const u32x4_t wf = piece(w[j] + (long)i * STEP, n, all);
#pragma unroll
        for (int m = 0; m < MT; ++m) acc[m][j] = product<T>(wf, xf[m], acc[m][j]);
      }
    }
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int j = 0; j < J; ++j) red[((wave * MT + m) * J + j) * 64 + lane] = acc[m][j];
  __syncthreads();
  const size_t width = (size_t)a.slices * p.r16;
  float* part = p.part + (size_t)blockIdx.y * a.rows * width;
  for (int i = threadIdx.x; i < MT * J * 64; i += 256) {
    const int l = i & 63, j = (i >> 6) % J, row = (i >> 6) / J * 16 + (l & 15), u = u0 + j;
    if (row >= t.count || u >= units) continue;
    f32x4_t v = red[i];
#pragma unroll
    for (int k = 1; k < 4; ++k) v += red[k * MT * J * 64 + i];
    *reinterpret_cast<f32x4_t*>(part + rows[row] * width + (u / n16) * p.r16 + (u % n16) * 16 + 4 * (l >> 4)) = v;
  }
}

template <typename T, int J>
__global__ void __launch_bounds__(256) adapters_shrink_kernel(AdaptersArgs a, AdaptersPlan p) {
#if defined(__HIP_DEVICE_COMPILE__)
  __shared__ f32x4_t red[4 * 2 * J * 64];
  __shared__ int rows[TM];
  const Tile t = tile_of(a, p, blockIdx.x, rows);
  if (t.count == 0 || t.adapter < 0) return;
  const int n16 = uniform((rank_of(a, t.adapter) + 15) >> 4), u0 = blockIdx.z * J, left = a.slices * n16 - u0;
  if (left <= 0) return;
  const int s0 = blockIdx.y * p.steps, s1 = min(s0 + p.steps, ceil_steps(a.d_in, Kind<T>::STEP));
  if (t.count > 16) {
    if (J > 4 && left > 4)
      shrink_tile<T, 2, J>(a, p, t, rows, u0, n16, s0, s1, red);
    else if (J > 2 && left > 2)
      shrink_tile<T, 2, J < 4 ? J : 4>(a, p, t, rows, u0, n16, s0, s1, red);
    else if (J > 1 && left > 1)
      shrink_tile<T, 2, J < 2 ? J : 2>(a, p, t, rows, u0, n16, s0, s1, red);
    else
      shrink_tile<T, 2, 1>(a, p, t, rows, u0, n16, s0, s1, red);
  } else {
    if (J > 4 && left > 4)
      shrink_tile<T, 1, J>(a, p, t, rows, u0, n16, s0, s1, red);
    else if (J > 2 && left > 2)
      shrink_tile<T, 1, J < 4 ? J : 4>(a, p, t, rows, u0, n16, s0, s1, red);
    else if (J > 1 && left > 1)
      shrink_tile<T, 1, J < 2 ? J : 2>(a, p, t, rows, u0, n16, s0, s1, red);
    else
      shrink_tile<T, 1, 1>(a, p, t, rows, u0, n16, s0, s1, red);
  }
#endif
}

// Eight consecutive elements of base or out as floats.
struct Eight {
  float v[8];
};
template <typename O>
__device__ __forceinline__ Eight load8(const O* p, int n, bool whole) {
  constexpr int W = sizeof(O) / 2;
  Eight r;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    const u32x4_t x = piece(p + w * (8 / W), n - w * (8 / W), whole);
#pragma unroll
    for (int e = 0; e < 8 / W; ++e) {
      if constexpr (W == 1)
        r.v[e] = __uint_as_float(e & 1 ? x[e / 2] & 0xffff0000u : x[e / 2] << 16);
      else
        r.v[w * 4 + e] = __uint_as_float(x[e]);
    }
  }
  return r;
}
template <typename O>
__device__ __forceinline__ void store8(O* p, const Eight& r, int n, bool whole) {
  if (whole) {
    if constexpr (sizeof(O) == 2) {
      *reinterpret_cast<u32x4_t*>(p) =
          u32x4_t{pack_bf16x2(r.v[0], r.v[1]), pack_bf16x2(r.v[2], r.v[3]), pack_bf16x2(r.v[4], r.v[5]), pack_bf16x2(r.v[6], r.v[7])};
    } else {
      *reinterpret_cast<f32x4_t*>(p) = f32x4_t{r.v[0], r.v[1], r.v[2], r.v[3]};
      *reinterpret_cast<f32x4_t*>(p + 4) = f32x4_t{r.v[4], r.v[5], r.v[6], r.v[7]};
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) Act<O>::store(p, e, r.v[e]);
  }
}

// A wave's block: rows of the tile by the columns n0 .. n0 + 127 below `end`.
// FAST: all of them are there, in whole pieces, and so are b's ranks.
template <typename T, typename O, int PARTS, int MT, bool FAST>
__device__ __forceinline__ void expand_block(const AdaptersArgs& a, const Tile& t, const int* rows, const u32x4_t* h, int rank, int steps,
                                             int n0, int end) {
  constexpr int E = Kind<T>::E;
  const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4;
  const int n = n0 + 8 * l16, left = end - n;
  Eight y[MT][4];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int i = m * 16 + 4 * g + r;
      if (a.base.data && i < t.count)
        y[m][r] = load8(static_cast<const O*>(a.base.data) + rows[i] * a.base.stride_l + n, left, FAST);
      else
        y[m][r] = Eight{};
    }
  f32x4_t acc[MT][8];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[m][i] = f32x4_t{0, 0, 0, 0};
  const T* b = static_cast<const T*>(a.b.data) + t.adapter * a.b.stride_b;
  for (int s = 0; s < steps; ++s) {
    const int c = (4 * s + g) / PARTS * E;  // the piece's first rank
    u32x4_t hf[MT], bf[8];
#pragma unroll
    for (int m = 0; m < MT; ++m) hf[m] = h[(s * MT + m) * 64 + lane];
    if constexpr (FAST) {
#pragma unroll
      for (int i = 0; i < 8; ++i) bf[i] = c < rank ? *reinterpret_cast<const u32x4_t*>(b + (n + i) * a.b.stride_l + c) : u32x4_t{0, 0, 0, 0};
      if (rank % E) {  // what lies behind the rank is not used, be it no number
        u32x4_t keep;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const int last = rank - c - w * (E / 4);  // elements of the word and behind it
          keep[w] = last <= 0 ? 0u : E == 8 && last == 1 ? 0xffffu : 0xffffffffu;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) bf[i] &= keep;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) bf[i] = piece(b + min(n + i, end - 1) * a.b.stride_l + c, rank - c, false);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int m = 0; m < MT; ++m) acc[m][i] = product<T>(hf[m], bf[i], acc[m][i]);
  }
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int i = m * 16 + 4 * g + r;
      if (i >= t.count) continue;
#pragma unroll
      for (int e = 0; e < 8; ++e) y[m][r].v[e] += acc[m][e][r];
      store8(static_cast<O*>(a.out.data) + rows[i] * a.out.stride_l + n, y[m][r], left, FAST);
    }
}

template <typename T, typename O, int PARTS, int MT>
__device__ __forceinline__ void expand_tile(const AdaptersArgs& a, const AdaptersPlan& p, const Tile& t, const int* rows, int slice, int n0,
                                            int end, bool vec, u32x4_t* h) {
  constexpr int E = Kind<T>::E;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int rank = t.adapter < 0 ? 0 : uniform(rank_of(a, t.adapter));
  const int pieces = (rank + E - 1) / E, steps = (pieces * PARTS + 3) >> 2;
  if (rank > 0) {
    // h[step][mt][lane]: row lane % 16, part v % PARTS of the ranks of piece v / PARTS, v = 4 step + lane / 16
    const float scale = a.scales ? a.scales[t.adapter] : 1.f;
    const size_t width = (size_t)a.slices * p.r16, next = (size_t)a.rows * width;
    for (int i = threadIdx.x; i < pieces * MT * 16; i += 256) {
      const int m = i % (MT * 16), c = i / (MT * 16);
      float v[E];
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = 0.f;
      if (m < t.count) {
        const float* from = p.part + rows[m] * width + slice * p.r16 + c * E;
#pragma unroll 4
        for (int z = 0; z < p.splits; ++z) {
#pragma unroll
          for (int q = 0; q < E / 4; ++q) {
            const f32x4_t w = *reinterpret_cast<const f32x4_t*>(from + z * next + 4 * q);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[4 * q + e] += w[e];
          }
        }
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = c * E + e < rank ? v[e] * scale : 0.f;
      }
#pragma unroll
      for (int q = 0; q < PARTS; ++q) {
        u32x4_t w;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] = __float_as_uint(v[e]);
        } else {
          // the value rounded to bf16, then what is left of it (nothing of an infinity)
#pragma unroll
          for (int e = 0; e < 8; e += 2) {
            w[e / 2] = pack_bf16x2(v[e], v[e + 1]);
#pragma unroll
            for (int d = 0; d < 2; ++d) {
              const float top = __uint_as_float(d ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
              v[e + d] = fabsf(top) < INFINITY ? v[e + d] - top : 0.f;
            }
          }
        }
        const int s = c * PARTS + q;
        h[((s >> 2) * MT + (m >> 4)) * 64 + (s & 3) * 16 + (m & 15)] = w;
      }
    }
    for (int i = threadIdx.x; i < (steps * 4 - pieces * PARTS) * MT * 16; i += 256) {
      const int m = i % (MT * 16), s = pieces * PARTS + i / (MT * 16);
      h[((s >> 2) * MT + (m >> 4)) * 64 + (s & 3) * 16 + (m & 15)] = u32x4_t{0, 0, 0, 0};
    }
    __syncthreads();
  }
  for (int n = n0 + wave * COLS; n < min(end, n0 + p.cols); n += 4 * COLS) {
    if (vec && n + COLS <= end)
      expand_block<T, O, PARTS, MT, true>(a, t, rows, h, rank, steps, n, end);
    else
      expand_block<T, O, PARTS, MT, false>(a, t, rows, h, rank, steps, n, end);
  }
}

template <typename T, typename O, int PARTS>
__global__ void __launch_bounds__(256) adapters_expand_kernel(AdaptersArgs a, AdaptersPlan p) {
#if defined(__HIP_DEVICE_COMPILE__)
  extern __shared__ u32x4_t frags[];
  __shared__ int rows[TM];
  const Tile t = tile_of(a, p, blockIdx.x, rows);
  if (t.count == 0 || (t.adapter < 0 && a.base.data == a.out.data)) return;
  int slice = 0, first = 0, block = blockIdx.y;
  for (; slice < a.slices - 1; ++slice) {
    const int n = (a.slice_end[slice] - first + p.cols - 1) / p.cols;
    if (block < n) break;
    block -= n;
    first = a.slice_end[slice];
  }
  const int n0 = first + block * p.cols, end = a.slice_end[slice];
  const bool vec = p.vec && n0 % (16 / (int)sizeof(O)) == 0;
  if (t.count > 16)
    expand_tile<T, O, PARTS, 2>(a, p, t, rows, slice, n0, end, vec, frags);
  else
    expand_tile<T, O, PARTS, 1>(a, p, t, rows, slice, n0, end, vec, frags);
#endif
}

AdaptersPlan plan_of(const AdaptersArgs& a) {
  AdaptersPlan p{};
  const int cus = device_cu_count(), size = a.dtype == DLLM_F32 ? 4 : 2;
  p.r16 = ceil_div(a.rank, 16) * 16;
  p.sorted = a.rows > 64;
  p.tiles = p.sorted ? std::min(a.rows, ceil_div(a.rows, TM) + a.adapters + 1) : a.rows;
  const int units = a.slices * p.r16 / 16;
  p.j = units >= 5 ? 8 : units >= 3 ? 4 : units;
  const int steps = ceil_steps(a.d_in, 64 / size), full = p.sorted ? ceil_div(a.rows, TM) : ceil_div(a.rows, 2);
  const int wanted = std::max(1, 2 * cus / (full * ceil_div(units, p.j)));
  p.splits = std::min({wanted, std::max(1, steps / 8), 16});
  p.steps = ceil_div(steps, p.splits);
  p.splits = ceil_div(steps, p.steps);
  p.cols = 4 * COLS;
  while (p.cols < 4096 && (long)full * (a.d_out / (2 * p.cols)) >= 4 * cus) p.cols *= 2;
  return p;
}

bool aligned(const AttnView& v, int size) {
  return ((uintptr_t)v.data & 15) == 0 && v.stride_l * size % 16 == 0 && v.stride_b * size % 16 == 0 && v.stride_h * size % 16 == 0;
}

template <typename T>
void shrink(const AdaptersArgs& a, const AdaptersPlan& p, hipStream_t s) {
  const dim3 grid(p.tiles, p.splits, ceil_div(a.slices * p.r16 / 16, p.j));
  if (p.j == 1)
    adapters_shrink_kernel<T, 1><<<grid, 256, 0, s>>>(a, p);
  else if (p.j == 2)
    adapters_shrink_kernel<T, 2><<<grid, 256, 0, s>>>(a, p);
  else if (p.j == 4)
    adapters_shrink_kernel<T, 4><<<grid, 256, 0, s>>>(a, p);
  else
    adapters_shrink_kernel<T, 8><<<grid, 256, 0, s>>>(a, p);
  DLLM_LAUNCH_CHECK("adapters_shrink_kernel");
}
template <typename T, typename O, int PARTS>
void expand(const AdaptersArgs& a, const AdaptersPlan& p, hipStream_t s) {
  int blocks = 0;
  for (int i = 0; i < a.slices; ++i) blocks += ceil_div(a.slice_end[i] - (i ? a.slice_end[i - 1] : 0), p.cols);
  const int steps = ceil_div((long)ceil_div(a.rank, Kind<T>::E) * PARTS, 4);
  adapters_expand_kernel<T, O, PARTS><<<dim3(p.tiles, blocks), 256, steps * 2 * 1024, s>>>(a, p);
  DLLM_LAUNCH_CHECK("adapters_expand_kernel");
}

size_t part_bytes(const AdaptersArgs& a, const AdaptersPlan& p) {
  return ((size_t)p.splits * a.rows * a.slices * p.r16 * 4 + 255) & ~(size_t)255;
}

}  // namespace

size_t adapters_bytes(const AdaptersArgs& a) {
  const AdaptersPlan p = plan_of(a);
  return part_bytes(a, p) + (p.sorted ? p.tiles * sizeof(int4) + a.rows * sizeof(int) : 0);
}

void launch_adapters(const AdaptersArgs& a, void* ws, hipStream_t s) {
  AdaptersPlan p = plan_of(a);
  const int size = a.dtype == DLLM_F32 ? 4 : 2, out = a.out_dtype == DLLM_F32 ? 4 : 2;
  p.part = static_cast<float*>(ws);
  p.tile = reinterpret_cast<int4*>(static_cast<char*>(ws) + part_bytes(a, p));
  p.order = reinterpret_cast<int*>(p.tile + p.tiles);
  p.vec_in = aligned(a.x, size) && aligned(a.a, size);
  p.vec = aligned(a.b, size) && a.rank * size % 16 == 0 && aligned(a.base, out) && aligned(a.out, out);
  if (p.sorted) {
    adapters_sort_kernel<<<1, SORT_THREADS, (a.adapters + 1) * 8, s>>>(a, p);
    DLLM_LAUNCH_CHECK("adapters_sort_kernel");
  }
  if (a.adapters > 0) {
    if (a.dtype == DLLM_F32)
      shrink<float>(a, p, s);
    else
      shrink<bf16_t>(a, p, s);
  }
  if (a.dtype == DLLM_F32)
    expand<float, float, 1>(a, p, s);
  else if (a.out_dtype == DLLM_F32)
    expand<bf16_t, float, 3>(a, p, s);
  else
    expand<bf16_t, bf16_t, 2>(a, p, s);
}

}  // namespace dllm
