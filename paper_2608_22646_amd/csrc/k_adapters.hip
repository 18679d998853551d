// Low-rank adapters of many requests beside a shared projection (dllm_adapters):
//   out = base + scale B (A x),  A and B those of the row's adapter.
//
// Both products run on tiles of up to 32 rows of one adapter.  Up to 64 rows: the rows of
// an adapter among 32 neighbours, found by the workgroup of the first of them.  More: a
// first launch of one workgroup sorts the rows by adapter, so that a tile is full whatever
// their order (512 rows found by neighbours: 46 to 49 us, sorted 27 to 35).  Then
//   shrink: part[z][row][s, j] = the z-th share of sum_k A[s, j, k] x[row, k]; rows of x
//     and of A to LDS, whose steps the eight waves of a workgroup share (16 x 16 tiles,
//     ranks by rows), and meet in LDS; 32 ranks a workgroup, which reads 64 rows of
//     operands; k is split where that leaves CUs without a workgroup;
//   join, where ranks are more than one step of the matrix unit and shares several: their
//     sum, once for all columns;
//   expand: the sum, scaled, in bf16 pieces that hold 16 of its bits (24 for a float32
//     output) as the matrix unit's one operand, B's rows as they lie in memory as the
//     other; a wave computes 32 rows x 128 columns, column n = 8 c + i by lane c's i-th
//     product, so that a lane reads and writes 8 consecutive elements of base and out (64
//     and 4 where there are few workgroups).
//
// What bounds them (kernel times, inputs not in a cache): 8448 rows of 4096 to 2 x 12288
// columns, rank 16: expand 148 to 153 us, HBM at 5.5 TB/s; shrink 32, with 84 MB to read; sort 10.
// 4223 rows, rank up to 128, 4096 to 4096: expand 39 and shrink 33 us, the L2s' answers to
// 32-row tiles that each read all of A and B (some 8 TB/s), sort 6.  By the element (4223 rows,
// 4096 to 4095, so that rows begin anywhere): expand of rank 16 51 us, in pieces to 4096
// columns 19; b too, rank 12, 102; rank 64 54 and 27, 60 115.  There the bf16 kernels of 8
// columns a lane spill: 12 and 196 bytes at ranks of one step, at more 36 with b.  Few rows: launches and
// the chain of dependent reads in them (256 rows, 12288 to 4096 float32, ranks up to 64:
// 3.8, 8.7, 4 and 7.5 us).
#include <algorithm>
#include <type_traits>

#include "kernels.h"
#include "lds_dma.h"

namespace dllm {

namespace {

constexpr int TM = 32;           // rows of a tile
constexpr int NW = 8;            // waves of a shrinking workgroup
constexpr int SORT_THREADS = 1024;

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t quad_t __attribute__((ext_vector_type(4), may_alias));  // of LDS that LDS-DMA wrote

__device__ __forceinline__ int adapter_of(const AdaptersArgs& a, int row) {
  const int w = a.which[row];
  return w >= 0 && w < a.adapters ? w : -1;
}
__device__ __forceinline__ int rank_of(const AdaptersArgs& a, int adapter) {
  return a.ranks ? min(max(a.ranks[adapter], 0), a.rank) : a.rank;
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
    if ((int)threadIdx.x < t.count) rows[threadIdx.x] = p.order[d.y + threadIdx.x];
  } else {
    // tile i: the i / groups-th of the 32 rows of group i % groups (rows that share an
    // adapter leave the first of them at work: those lie on consecutive XCDs).  w of a lane
    // without a row is -2, also where tile i's own row is not there: no tile, no rows.
    const int groups = (p.tiles + TM - 1) / TM, me = i / groups, row = i % groups * TM + lane;
    const int w = lane < TM && row < a.rows ? adapter_of(a, row) : -2;
    t.adapter = __builtin_amdgcn_readlane(w, me);
    const unsigned long long mine = __ballot(w == t.adapter);
    t.count = t.adapter >= -1 && __ffsll(mine) - 1 == me ? __popcll(mine) : 0;
    if (threadIdx.x < 64 && t.count && w == t.adapter) rows[__popcll(mine & ((1ull << lane) - 1))] = row;
  }
  __syncthreads();
  return t;
}

// Sorts the rows by adapter (those without one last) and cuts them into tiles.  The
// order of an adapter's rows depends on the order of execution; no result does.  ROWS rows of
// a thread are asked for at once, and once in all where there are no more (4223 rows: 6.2 us,
// one after the other 7.6; of up to 1024, one a thread: 3.8, eight 4.1).
template <int ROWS>
__global__ void __launch_bounds__(SORT_THREADS) adapters_sort_kernel(AdaptersArgs a, AdaptersPlan p) {
#if defined(__HIP_DEVICE_COMPILE__)
  extern __shared__ int sh[];
  const int bins = a.adapters + 1, tid = threadIdx.x, lane = tid & 63;
  int *const at = sh, *const tiles = sh + bins;  // rows' places, tiles' first ones
  __shared__ int2 sums[SORT_THREADS / 64];
  for (int i = tid; i < bins; i += SORT_THREADS) at[i] = 0;
  __syncthreads();
  // the place of each row among its bin's, by a wave at once where its rows share one
  auto add = [&](int w, bool there) {
    const int bin = w >= 0 && w < a.adapters ? w : a.adapters;
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
  int w[ROWS];
  auto ask = [&](int r0) {
#pragma unroll
    for (int k = 0; k < ROWS; ++k)
      if (r0 + k * SORT_THREADS < a.rows) w[k] = a.which[min(r0 + k * SORT_THREADS + tid, a.rows - 1)];
  };
  auto each_row = [&](int r0, auto f) {
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
      const int row = r0 + k * SORT_THREADS + tid;
      if (row - lane < a.rows) f(row, add(w[k], row < a.rows));
    }
  };
  constexpr int GO = ROWS * SORT_THREADS;
  for (int r0 = 0; r0 < a.rows; r0 += GO) {
    ask(r0);
    each_row(r0, [](int, int) {});
  }
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
  for (int r0 = 0; r0 < a.rows; r0 += GO) {
    if (a.rows > GO) ask(r0);
    each_row(r0, [&](int row, int pos) {
      if (row < a.rows) p.order[pos] = row;
    });
  }
#endif
}

template <typename T>
struct Kind {
  static constexpr int E = 16 / sizeof(T);  // elements of a piece
  static constexpr int STEP = 4 * E;        // along k: 64 bytes of a row, a piece for each 16 lanes
};

// N elements at p, of which the first n count (the rest give zeros; none but the first is
// touched behind them).
template <typename T, int N>
struct Words {
  uint32_t w[N * sizeof(T) / 4];
};
template <typename T, int N>
__device__ __forceinline__ Words<T, N> some(const T* p, int n) {
  T v[N];
#pragma unroll
  for (int e = 0; e < N; ++e) v[e] = p[e < n ? e : 0];
  Words<T, N> x{};
#pragma unroll
  for (int e = 0; e < N; ++e) {
    if constexpr (sizeof(T) == 2)
      x.w[e / 2] |= e < n ? (uint32_t)v[e] << (16 * (e & 1)) : 0u;
    else
      x.w[e] = e < n ? __float_as_uint(v[e]) : 0u;
  }
  return x;
}
template <typename T>
__device__ __forceinline__ u32x4_t piece(const T* p, int n) {
  return __builtin_bit_cast(u32x4_t, some<T, Kind<T>::E>(p, n));
}

// c + the products of two fragments of a step
template <typename T>
__device__ __forceinline__ f32x4_t product(u32x4_t x, u32x4_t y, f32x4_t c) {
  if constexpr (sizeof(T) == 2)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, x), __builtin_bit_cast(bf16x8_t, y), c, 0, 0, 0);
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x[e]), __uint_as_float(y[e]), c, 0, 0, 0);
  return c;
}

// Ranks c .. of a row's inner products, as the outer product's operand takes them: scaled,
// nothing from the adapter's rank on, in PARTS summands.  Piece c / E of slice s lies at
// h[s][c / E / 4][part][c / E % 4][row].
template <typename T, int PARTS>
__device__ __forceinline__ void summands(int c, int rank, float scale, float (&v)[Kind<T>::E], u32x4_t (&w)[PARTS]) {
  constexpr int E = Kind<T>::E;
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] = c + e < rank ? v[e] * scale : 0.f;
#pragma unroll
  for (int q = 0; q < PARTS; ++q) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int e = 0; e < 4; ++e) w[q][e] = __float_as_uint(v[e]);
    } else {
      // the value rounded to bf16, then what is left of it (nothing of an infinity)
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        w[q][e / 2] = pack_bf16x2(v[e], v[e + 1]);
#pragma unroll
        for (int d = 0; d < 2; ++d) {
          const float top = __uint_as_float(d ? w[q][e / 2] & 0xffff0000u : w[q][e / 2] << 16);
          v[e + d] = fabsf(top) < INFINITY ? v[e + d] - top : 0.f;
        }
      }
    }
  }
}
// Sum of the shares of E ranks of a row, in their order.
template <typename T>
__device__ __forceinline__ void sum_shares(const AdaptersArgs& a, const AdaptersPlan& p, int row, int s, int c, float (&v)[Kind<T>::E]) {
  constexpr int E = Kind<T>::E;
  const float* from = p.part + ((size_t)row * a.slices + s) * p.r16 + c;
  const size_t next = (size_t)a.rows * a.slices * p.r16;
  auto shares = [&](auto N, int z) {
    f32x4_t w[N][E / 4];
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int q = 0; q < E / 4; ++q) w[k][q] = *reinterpret_cast<const f32x4_t*>(from + (z + k) * next + 4 * q);
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] += w[k][e / 4][e % 4];
  };
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] = 0.f;
  int z = 0;
  for (; z + 8 <= p.splits; z += 8) shares(std::integral_constant<int, 8>{}, z);
  if (z + 4 <= p.splits) {
    shares(std::integral_constant<int, 4>{}, z);
    z += 4;
  }
  if (z + 2 <= p.splits) {
    shares(std::integral_constant<int, 2>{}, z);
    z += 2;
  }
  if (z < p.splits) shares(std::integral_constant<int, 1>{}, z);
}
template <typename T, int PARTS>
__device__ __forceinline__ void keep_piece(const AdaptersArgs& a, const AdaptersPlan& p, int row, int s, int c, int rank, float scale,
                                           float (&v)[Kind<T>::E]) {
  constexpr int E = Kind<T>::E;
  u32x4_t w[PARTS];
  summands<T, PARTS>(c, rank, scale, v, w);
#pragma unroll
  for (int q = 0; q < PARTS; ++q) p.h[(((size_t)s * p.hsteps + c / (4 * E)) * PARTS + q) * 4 * a.rows + (size_t)(c / E % 4) * a.rows + row] = w[q];
}

// What a shrinking workgroup computes: 16-blocks u0 .. u0 + J - 1 of its adapter's ranks
// (of `units`, n16 a slice).
struct Ranks {
  int rank, n16, units, u0;
};
// Row of A behind rank l of block u (the last one behind those that are not there).
template <typename T>
__device__ __forceinline__ const T* a_row(const AdaptersArgs& a, int adapter, const Ranks& k, int u, int l) {
  u = min(u, k.units - 1);
  return static_cast<const T*>(a.a.data) + adapter * a.a.stride_b + u / k.n16 * a.a.stride_h + min(u % k.n16 * 16 + l, k.rank - 1) * a.a.stride_l;
}

// The waves' sums of products, acc[mt][j] (lane l: row l % 16, ranks 4 (l / 16) ..), to
// the workspace.
template <typename T, int PARTS, int MT, int J>
__device__ __forceinline__ void gather(const AdaptersArgs& a, const AdaptersPlan& p, const Tile& t, const int* rows, const Ranks& k,
                                       const f32x4_t (&acc)[MT][J], f32x4_t* red) {
  constexpr int E = Kind<T>::E, Q = E / 4;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const float scale = a.scales ? a.scales[t.adapter] : 1.f;
  __syncthreads();
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int j = 0; j < J; ++j) red[((wave * MT + m) * J + j) * 64 + lane] = acc[m][j];
  __syncthreads();
  // a piece of E ranks of a row each
  for (int i = threadIdx.x; i < MT * J * 64 / Q; i += NW * 64) {
    const int l = i & 15, g4 = (i >> 4) % (4 / Q) * Q, mj = i / (64 / Q), m = mj / J, u = k.u0 + mj % J;
    if (m * 16 + l >= t.count || u >= k.units) continue;
    float v[E];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      f32x4_t sum = red[mj * 64 + (g4 + q) * 16 + l];
#pragma unroll
      for (int w = 1; w < NW; ++w) sum += red[(w * MT * J + mj) * 64 + (g4 + q) * 16 + l];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * q + e] = sum[e];
    }
    const int row = rows[m * 16 + l], s = u / k.n16, c = u % k.n16 * 16 + 4 * g4;
    if (p.keep) {
      keep_piece<T, PARTS>(a, p, row, s, c, k.rank, scale, v);
    } else {
      float* to = p.part + (((size_t)blockIdx.y * a.rows + row) * a.slices + s) * p.r16 + c;
#pragma unroll
      for (int q = 0; q < Q; ++q) *reinterpret_cast<f32x4_t*>(to + 4 * q) = f32x4_t{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
    }
  }
}

// Operands in whole pieces.  Rows of x, then of A, each CHUNK bytes along k a stage, by
// LDS-DMA: a load brings 1 KiB of one row (what neighbouring lanes read of 16 rows a few
// KiB apart would lie in few of the L2's channels); piece c of row r in slot c ^ (r % 16),
// so that 16 rows' pieces meet all banks.  Each wave multiplies two of a stage's 16 steps.
// One stage at a time and two workgroups a CU, one loading while the other multiplies (8448
// rows to 2 x 16 ranks, sort and expand included: 196 us; two stages of one workgroup 199).
constexpr int CHUNK = 1024;
template <typename T, int PARTS, int MT, int J>
__device__ __forceinline__ void shrink_tile(const AdaptersArgs& a, const AdaptersPlan& p, const Tile& t, const int* rows, const Ranks& k, char* lds) {
  constexpr int ROWS = 16 * (MT + J), PER = ROWS / NW;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), l16 = lane & 15, g = lane >> 4;
  const uint32_t bytes = (uint32_t)(a.d_in * sizeof(T));
  // this wave's rows
  const char* from[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int r = wave + NW * i;
    const T* q = r < 16 * MT ? static_cast<const T*>(a.x.data) + rows[min(r, t.count - 1)] * a.x.stride_l
                             : a_row<T>(a, t.adapter, k, k.u0 + (r - 16 * MT) / 16, (r - 16 * MT) % 16);
    from[i] = uniform(reinterpret_cast<const char*>(q));
  }
  const uint32_t to = lds_address(lds) + wave * CHUNK;
  f32x4_t acc[MT][J];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int j = 0; j < J; ++j) acc[m][j] = f32x4_t{0, 0, 0, 0};
  const int c0 = blockIdx.y * p.steps, n = min(p.steps, (int)((bytes + CHUNK - 1) / CHUNK) - c0);
  for (int u = 0; u < n; ++u) {
    if (u) barrier_nofence();
#pragma unroll
    for (int i = 0; i < PER; ++i)
      dma16(rsrc_of(from[i], bytes), (c0 + u) * CHUNK + (lane ^ ((wave + NW * i) & 15)) * 16, to + i * NW * CHUNK);
    wait_vmcnt<0>();
    barrier_nofence();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int slot = ((wave * 2 + i) * 4 + g) ^ l16;
      u32x4_t xf[MT], wf[J];
#pragma unroll
      for (int m = 0; m < MT; ++m) xf[m] = *reinterpret_cast<const quad_t*>(lds + (m * 16 + l16) * CHUNK + slot * 16);
#pragma unroll
      for (int j = 0; j < J; ++j) wf[j] = *reinterpret_cast<const quad_t*>(lds + ((MT + j) * 16 + l16) * CHUNK + slot * 16);
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int j = 0; j < J; ++j) acc[m][j] = product<T>(wf[j], xf[m], acc[m][j]);
    }
  }
  gather<T, PARTS>(a, p, t, rows, k, acc, reinterpret_cast<f32x4_t*>(lds));
}

// Operands that are read by the element: straight into registers, a step a wave.
template <typename T, int PARTS, int MT>
__device__ __forceinline__ void shrink_elements(const AdaptersArgs& a, const AdaptersPlan& p, const Tile& t, const int* rows, const Ranks& k,
                                                f32x4_t* red) {
  constexpr int E = Kind<T>::E, STEP = Kind<T>::STEP;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), l16 = lane & 15, g = lane >> 4;
  const T* x[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) x[m] = static_cast<const T*>(a.x.data) + rows[min(m * 16 + l16, t.count - 1)] * a.x.stride_l;
  const T* w = a_row<T>(a, t.adapter, k, k.u0, l16);
  f32x4_t acc[MT][1];
#pragma unroll
  for (int m = 0; m < MT; ++m) acc[m][0] = f32x4_t{0, 0, 0, 0};
  const int per = CHUNK / 64, s0 = blockIdx.y * p.steps * per, s1 = min(s0 + p.steps * per, (a.d_in + STEP - 1) / STEP);
  for (int b = s0 + wave; b < s1; b += NW) {
    // (a lane's first element may lie behind the last one: that is touched in its place)
    const int at = b * STEP + g * E, n = a.d_in - at;
    const u32x4_t wf = piece(w + min(at, a.d_in - 1), n);
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[m][0] = product<T>(wf, piece(x[m] + min(at, a.d_in - 1), n), acc[m][0]);
  }
  gather<T, PARTS>(a, p, t, rows, k, acc, red);
}

template <typename T, int PARTS, int J, bool VEC>
__global__ void __launch_bounds__(NW * 64) adapters_shrink_kernel(AdaptersArgs a, AdaptersPlan p) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int STAGES = VEC ? 16 * (2 + J) * CHUNK : 0, SUMS = NW * 2 * J * 1024;
  __shared__ __attribute__((aligned(1024))) char lds[STAGES > SUMS ? STAGES : SUMS];
  __shared__ int rows[TM];
  // workgroup i runs on XCD i % 8: those of a tile, which read the same rows of x, follow
  // each other on one
  const int blocks = gridDim.x / ((p.tiles + 7) & ~7), slot = blockIdx.x >> 3, tile = slot / blocks * 8 + (blockIdx.x & 7);
  if (tile >= p.tiles) return;
  const Tile t = tile_of(a, p, tile, rows);
  if (t.count == 0 || t.adapter < 0) return;
  Ranks k;
  k.rank = uniform(rank_of(a, t.adapter));
  k.n16 = (k.rank + 15) >> 4;
  k.units = a.slices * k.n16;
  k.u0 = slot % blocks * J;
  if (k.u0 >= k.units) return;
  if constexpr (!VEC) {
    if (t.count > 16)
      shrink_elements<T, PARTS, 2>(a, p, t, rows, k, reinterpret_cast<f32x4_t*>(lds));
    else
      shrink_elements<T, PARTS, 1>(a, p, t, rows, k, reinterpret_cast<f32x4_t*>(lds));
  } else if (t.count > 16) {
    if (J > 1 && k.units - k.u0 > 1)
      shrink_tile<T, PARTS, 2, J>(a, p, t, rows, k, lds);
    else
      shrink_tile<T, PARTS, 2, 1>(a, p, t, rows, k, lds);
  } else {
    if (J > 1 && k.units - k.u0 > 1)
      shrink_tile<T, PARTS, 1, J>(a, p, t, rows, k, lds);
    else
      shrink_tile<T, PARTS, 1, 1>(a, p, t, rows, k, lds);
  }
#endif
}

// Sums the shares of the inner products, in their order: a piece of a row each thread.
template <typename T, int PARTS>
__global__ void __launch_bounds__(64) adapters_join_kernel(AdaptersArgs a, AdaptersPlan p) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int E = Kind<T>::E;
  const int row = (int)blockIdx.x * 64 + threadIdx.x, s = blockIdx.y / (p.r16 / E), c = blockIdx.y % (p.r16 / E) * E;
  if (row >= a.rows) return;
  const int w = adapter_of(a, row);
  float v[E];
  sum_shares<T>(a, p, row, s, c, v);  // (beside the adapter; what an adapter does not have is not used)
  if (w < 0) return;
  const int rank = rank_of(a, w);
  if (c < rank) keep_piece<T, PARTS>(a, p, row, s, c, rank, a.scales ? a.scales[w] : 1.f, v);
#endif
}

// C consecutive elements of base, as they were read.
template <typename O, int C>
struct Some {
  static constexpr int W = C * sizeof(O) > 16 ? C * sizeof(O) / 16 : 1, WORDS = C * sizeof(O) / 4 / W;  // pieces of words
  typedef uint32_t piece_t __attribute__((ext_vector_type(WORDS)));
  piece_t w[W];
  __device__ __forceinline__ float at(int e) const {
    if constexpr (sizeof(O) == 2) return __uint_as_float(e & 1 ? w[0][e / 2] & 0xffff0000u : w[0][e / 2] << 16);
    return __uint_as_float(w[(e / 4) % W][e % 4]);
  }
};

// A wave's share of a tile: its rows by the columns n0, n0 + 4 COLS, .. below `last`,
// of a slice that ends at `end`; C columns a lane, COLS a wave.  VY, VB: base and out, b lie in whole 16-byte pieces.
// ONE: the ranks are those of one step.
template <typename T, typename O, int PARTS, bool VY, bool VB, bool ONE, int C>
__device__ __forceinline__ void expand_columns(const AdaptersArgs& a, const AdaptersPlan& p, const Tile& t, const int* rows, int rank,
                                               int steps, int slice, int n0, int last, int end) {
  constexpr int E = Kind<T>::E, COLS = 16 * C;
  typedef Some<O, C> Y;
  const int lane = threadIdx.x & 63, g = lane >> 4, MT = (t.count + 15) >> 4;
  const T* const b = static_cast<const T*>(a.b.data) + max(t.adapter, 0) * a.b.stride_b;
  // base NULL: what is read in its place counts as zero
  const O* const base = static_cast<const O*>(a.base.data ? a.base.data : a.out.data);
  const int64_t base_stride = a.base.data ? a.base.stride_l : a.out.stride_l;
  const uint32_t given = a.base.data ? 0xffffffffu : 0u;
  // the part q of step s of the rows 16 m ..
  const u32x4_t* const h = p.h + (size_t)slice * p.hsteps * PARTS * 4 * a.rows + (size_t)g * a.rows;
  auto load_h = [&](int s, int q, int m) {
    const int i = m * 16 + (lane & 15);
    u32x4_t w = {0, 0, 0, 0};
    if ((4 * s + g) * E < rank) w = h[(size_t)(s * PARTS + q) * 4 * a.rows + rows[i < t.count ? i : 0]];
    return w;
  };
  u32x4_t hf[ONE ? 2 : 1][PARTS];
  if constexpr (ONE) {
    const float scale = a.scales && rank ? a.scales[t.adapter] : 1.f;
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const int i = m * 16 + (lane & 15);
      float v[E];
      if (g * E < rank) {
        sum_shares<T>(a, p, rows[i < t.count ? i : 0], slice, g * E, v);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = 0.f;
      }
      summands<T, PARTS>(g * E, rank, scale, v, hf[m]);
    }
  }
  for (int nb = n0; nb < last; nb += 4 * COLS) {
    const int n = nb + C * (lane & 15), left = end - n;
    const int col = VY ? (left >= C ? n : nb) : n;  // columns that are not there: others' are read in their place
    // b's pieces of step s
    auto load_b = [&](int s, u32x4_t (&bf)[C]) {
      const int c = (4 * s + g) * E, c0 = c < rank ? c : 0;  // (ranks that are not there: h has zeros)
#pragma unroll
      for (int i = 0; i < C; ++i) {
        const T* from = b + min(col + i, end - 1) * a.b.stride_l + c0;
        if constexpr (VB)
          bf[i] = *reinterpret_cast<const u32x4_t*>(from);
        else
          bf[i] = piece(from, rank - c0);
      }
      if (VB && rank % E) {  // what lies behind the rank is not used, be it no number
        u32x4_t keep;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const int more = rank - c0 - w * (E / 4);  // elements of the word and behind it
          keep[w] = more <= 0 ? 0u : E == 8 && more == 1 ? 0xffffu : 0xffffffffu;
        }
#pragma unroll
        for (int i = 0; i < C; ++i) bf[i] &= keep;
      }
    };
    auto load_y = [&](int m, Y (&y)[4]) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int i = m * 16 + 4 * g + r;
        const O* from = base + rows[i < t.count ? i : 0] * base_stride + col;
        if constexpr (VY) {
#pragma unroll
          for (int k = 0; k < Y::W; ++k) y[r].w[k] = reinterpret_cast<const typename Y::piece_t*>(from)[k];
        } else {
#pragma unroll
          for (int k = 0; k < Y::W; ++k)
            y[r].w[k] = __builtin_bit_cast(typename Y::piece_t, some<O, C / Y::W>(from + min(k * C / Y::W, left - 1), left - k * C / Y::W));
        }
      }
    };
    auto finish = [&](int m, const Y (&y)[4], const f32x4_t (&acc)[C]) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int i = m * 16 + 4 * g + r;
        if (i >= t.count || left <= 0) continue;
        Y z = y[r];
#pragma unroll
        for (int k = 0; k < Y::W; ++k) z.w[k] &= given;
        float v[C];
#pragma unroll
        for (int e = 0; e < C; ++e) v[e] = z.at(e) + acc[e][r];
        O* to = static_cast<O*>(a.out.data) + rows[i] * a.out.stride_l + n;
        if constexpr (VY && sizeof(O) == 2) {
          typename Y::piece_t w;
#pragma unroll
          for (int e = 0; e < C; e += 2) w[e / 2] = pack_bf16x2(v[e], v[e + 1]);
          *reinterpret_cast<typename Y::piece_t*>(to) = w;
        } else if constexpr (VY) {
#pragma unroll
          for (int e = 0; e < C; e += 4) *reinterpret_cast<f32x4_t*>(to + e) = f32x4_t{v[e], v[e + 1], v[e + 2], v[e + 3]};
        } else {
#pragma unroll
          for (int e = 0; e < C; ++e)
            if (e < left) Act<O>::store(to, e, v[e]);
        }
      }
    };
    const f32x4_t zero = {0, 0, 0, 0};
    u32x4_t bf[1][C];
    Y y[2][4];
    if constexpr (ONE) {
      load_y(0, y[0]);
      if (MT > 1) load_y(1, y[1]);
      if (steps)
        load_b(0, bf[0]);
      else
#pragma unroll
        for (int i = 0; i < C; ++i) bf[0][i] = u32x4_t{0, 0, 0, 0};
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        if (m >= MT) break;
        f32x4_t acc[C];
#pragma unroll
        for (int q = 0; q < PARTS; ++q)
#pragma unroll
          for (int i = 0; i < C; ++i) acc[i] = product<T>(hf[m][q], bf[0][i], q ? acc[i] : zero);
        finish(m, y[m], acc);
      }
    } else {
      f32x4_t acc[2][C];
#pragma unroll
      for (int i = 0; i < C; ++i) acc[0][i] = acc[1][i] = zero;
      for (int s = 0; s < steps; ++s) {
        u32x4_t hs[2][PARTS];
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
          for (int q = 0; q < PARTS; ++q) hs[m][q] = load_h(s, q, m);
        load_b(s, bf[0]);
#pragma unroll
        for (int q = 0; q < PARTS; ++q)
#pragma unroll
          for (int i = 0; i < C; ++i) {
            acc[0][i] = product<T>(hs[0][q], bf[0][i], acc[0][i]);
            acc[1][i] = product<T>(hs[1][q], bf[0][i], acc[1][i]);
          }
      }
      // (base's rows of a bf16 output one half after the other: both at once spill registers, 36
      // us for 32 at 4223 rows of rank 128 into 4096 columns)
      constexpr bool BOTH = sizeof(O) == 4;
      load_y(0, y[0]);
      if (BOTH && MT > 1) load_y(1, y[1]);
      finish(0, y[0], acc[0]);
      if (MT > 1) {
        if (!BOTH) load_y(1, y[1]);
        finish(1, y[1], acc[1]);
      }
    }
  }
}

template <typename T, typename O, int PARTS, bool VY, bool VB, bool ONE, int C>
__global__ void __launch_bounds__(256, sizeof(O) == 2 ? 3 : 2) adapters_expand_kernel(AdaptersArgs a, AdaptersPlan p) {
#if defined(__HIP_DEVICE_COMPILE__)
  __shared__ int rows[TM];
  int slice = 0, first = 0, block = blockIdx.x % p.blocks;
  const Tile t = tile_of(a, p, blockIdx.x / p.blocks, rows);
  if (t.count == 0 || (t.adapter < 0 && a.base.data == a.out.data)) return;
  for (; slice < a.slices - 1; ++slice) {
    const int n = (a.slice_end[slice] - first + p.cols - 1) / p.cols;
    if (block < n) break;
    block -= n;
    first = a.slice_end[slice];
  }
  const int n0 = first + block * p.cols, end = a.slice_end[slice], last = min(end, n0 + p.cols), mine = n0 + uniform(threadIdx.x >> 6) * 16 * C;
  const int rank = t.adapter < 0 ? 0 : uniform(rank_of(a, t.adapter));
  const int steps = (rank + Kind<T>::STEP - 1) / Kind<T>::STEP;
  expand_columns<T, O, PARTS, VY, VB, ONE, C>(a, p, t, rows, rank, steps, slice, mine, last, end);
#endif
}

int parts_of(const AdaptersArgs& a) { return a.dtype == DLLM_F32 ? 1 : a.out_dtype == DLLM_F32 ? 3 : 2; }

AdaptersPlan plan_of(const AdaptersArgs& a) {
  AdaptersPlan p{};
  const int cus = device_cu_count(), size = a.dtype == DLLM_F32 ? 4 : 2;
  p.r16 = ceil_div(a.rank, 16) * 16;
  p.sorted = a.rows > 64;
  const int groups = ceil_div(a.rows, TM);
  p.tiles = p.sorted ? std::min(a.rows, groups + a.adapters + 1) : a.rows <= TM ? a.rows : groups * TM;
  const int units = a.slices * p.r16 / 16, full = p.sorted ? groups : std::min(a.rows, groups + a.adapters);
  // (blocks of 16 ranks a workgroup: two, with 64 KiB a stage and two workgroups a CU)
  p.j = std::min(units, 2);
  const int wgs = full * ceil_div(units, p.j), chunks = ceil_div((long)a.d_in * size, CHUNK);
  p.splits = std::max(1, std::min({cus / wgs, chunks, 16}));
  p.steps = ceil_div(chunks, p.splits);
  p.splits = ceil_div(chunks, p.steps);
  p.keep = a.rank > 64 / size && p.splits == 1;
  p.hsteps = ceil_div(a.rank, 64 / size);
  // columns of a workgroup: 512, or twice that where that leaves four for each CU, or half of it
  // where there would be fewer than CUs (8448 rows to 2 x 12288: 194 us, by 512 205; 4223 rows to
  // 4096: 80, by 1024 86; 777 rows to 201 + 77 float32: 18.9, by 512 21.7; 256 to 4096 float32:
  // 25.7 and 27; 2000 to 4096 of rank 64: 32, by 256 33.6)
  const long wide = (long)full * ceil_div(a.d_out, 512);
  p.narrow = wide < cus;
  p.cols = p.narrow ? 256 : wide < 8 * cus ? 512 : 1024;
  for (int i = 0; i < a.slices; ++i) p.blocks += ceil_div(a.slice_end[i] - (i ? a.slice_end[i - 1] : 0), p.cols);
  return p;
}

bool aligned(const AttnView& v, int size) {
  return ((uintptr_t)v.data & 15) == 0 && v.stride_l * size % 16 == 0 && v.stride_b * size % 16 == 0 && v.stride_h * size % 16 == 0;
}

template <typename T, typename O, int PARTS>
void run(const AdaptersArgs& a, const AdaptersPlan& p, hipStream_t s) {
  if (a.adapters > 0) {
    const dim3 grid(((p.tiles + 7) & ~7) * ceil_div(a.slices * p.r16 / 16, p.vec_in ? p.j : 1), p.splits);
    if (!p.vec_in)
      adapters_shrink_kernel<T, PARTS, 1, false><<<grid, NW * 64, 0, s>>>(a, p);
    else if (p.j == 1)
      adapters_shrink_kernel<T, PARTS, 1, true><<<grid, NW * 64, 0, s>>>(a, p);
    else
      adapters_shrink_kernel<T, PARTS, 2, true><<<grid, NW * 64, 0, s>>>(a, p);
    DLLM_LAUNCH_CHECK("adapters_shrink_kernel");
    if (a.rank > Kind<T>::STEP && !p.keep) {
      adapters_join_kernel<T, PARTS><<<dim3(ceil_div(a.rows, 64), a.slices * p.r16 / Kind<T>::E), 64, 0, s>>>(a, p);
      DLLM_LAUNCH_CHECK("adapters_join_kernel");
    }
  }
  auto launch = [&](auto vy, auto vb, auto one) {
    if (p.narrow)
      adapters_expand_kernel<T, O, PARTS, vy, vb, one, 4><<<p.tiles * p.blocks, 256, 0, s>>>(a, p);
    else
      adapters_expand_kernel<T, O, PARTS, vy, vb, one, 8><<<p.tiles * p.blocks, 256, 0, s>>>(a, p);
  };
  auto go = [&](auto vy, auto vb) {
    if (a.rank <= Kind<T>::STEP)
      launch(vy, vb, std::true_type{});
    else
      launch(vy, vb, std::false_type{});
  };
  if (!p.vec_b)
    go(std::false_type{}, std::false_type{});
  else if (!p.vec_y)
    go(std::false_type{}, std::true_type{});
  else
    go(std::true_type{}, std::true_type{});
  DLLM_LAUNCH_CHECK("adapters_expand_kernel");
}

size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }
// Bytes of the workspace's parts: inner products, their shares, tiles and order.
size_t h_bytes(const AdaptersArgs& a, const AdaptersPlan& p) { return p.hsteps == 1 ? 0 : up256((size_t)a.slices * p.hsteps * parts_of(a) * 4 * a.rows * 16); }
size_t part_bytes(const AdaptersArgs& a, const AdaptersPlan& p) {
  return p.keep ? 0 : up256((size_t)p.splits * a.rows * a.slices * p.r16 * 4);
}

}  // namespace

size_t adapters_bytes(const AdaptersArgs& a) {
  const AdaptersPlan p = plan_of(a);
  return h_bytes(a, p) + part_bytes(a, p) + (p.sorted ? p.tiles * sizeof(int4) + a.rows * sizeof(int) : 0);
}

// A launch's threads must be below 2^32.
bool adapters_fit(const AdaptersArgs& a) {
  const AdaptersPlan p = plan_of(a);
  return (long)p.tiles * p.blocks < (1l << 32) / 256 && ((long)p.tiles + 7) / 8 * 8 * a.slices * p.r16 / 16 < (1l << 32) / (NW * 64);
}

void launch_adapters(const AdaptersArgs& a, void* ws, hipStream_t s) {
  AdaptersPlan p = plan_of(a);
  const int size = a.dtype == DLLM_F32 ? 4 : 2, out = a.out_dtype == DLLM_F32 ? 4 : 2;
  char* at = static_cast<char*>(ws);
  p.h = reinterpret_cast<uint32_t __attribute__((ext_vector_type(4)))*>(at);
  p.part = reinterpret_cast<float*>(at += h_bytes(a, p));
  p.tile = reinterpret_cast<int4*>(at += part_bytes(a, p));
  p.order = reinterpret_cast<int*>(p.tile + p.tiles);
  p.vec_in = aligned(a.x, size) && aligned(a.a, size) && a.d_in * size % 16 == 0;
  p.vec_b = aligned(a.b, size) && a.rank * size % 16 == 0;
  p.vec_y = aligned(a.base, out) && aligned(a.out, out);
  for (int i = 0; i < a.slices; ++i) p.vec_y = p.vec_y && a.slice_end[i] % 8 == 0;
  if (p.sorted) {
    (a.rows > SORT_THREADS ? adapters_sort_kernel<8> : adapters_sort_kernel<1>)<<<1, SORT_THREADS, (a.adapters + 1) * 8, s>>>(a, p);
    DLLM_LAUNCH_CHECK("adapters_sort_kernel");
  }
  if (a.dtype == DLLM_F32)
    run<float, float, 1>(a, p, s);
  else if (a.out_dtype == DLLM_F32)
    run<bf16_t, float, 3>(a, p, s);
  else
    run<bf16_t, bf16_t, 2>(a, p, s);
}

}  // namespace dllm
