// Attention of documents of unlike lengths (dllm_attention): grouped heads,
// positional masks, capped scores and distance biases.
//
// A row is one query of one head.  The G = n_heads / n_kv_heads query heads of a
// key/value head are rows of the same tile (row r = query r / G, head r % G), so
// each key and value is read once for all of them.  A wave owns 32 rows and
// computes, per tile of KT keys,
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
// Where rows are few, the keys of a document are also split over workgroups
// (chunks of whole steps); each leaves its state in the workspace and
// attn_join_kernel joins them in chunk order.
//
// Many rows (bf16, 128-wide heads): the matrix unit and the softmax's instructions
// share a SIMD's issue, the exponentials being half of them; 8448 tokens, 28 + 4
// heads, visible up to the end of their block of 32: 517 us, 1.00 PFLOP/s (when it took
// 548, that was 499 without the softmax, 435 without the LDS reads as well and 389
// without the loads as well, at a clock that its power holds near 2 GHz).  Few rows: keys and values from HBM; one
// token of 16 documents of 2.6 to 8.4 thousand keys: 40 us and 5 for the join, 4.4
// TB/s; 32 queries x 1024 keys x 32 heads x 8: 31 us, 4.4 TB/s (a copy: 5.1).
// float32: the matrix unit's float32 rate, a sixteenth of bf16's.
#include <algorithm>
#include <type_traits>

#include "kernels.h"

namespace dllm {

namespace {

typedef short v4s_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4s_t* lds_v4s_t;
typedef unsigned short v2us_t __attribute__((ext_vector_type(2)));

constexpr float LOG2E = 1.4426950408889634f;
constexpr int MAX_SHARES = 256;

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

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ const char* uniform(const char* p) {
  const uint32_t lo = uniform((int)(uint64_t)p), hi = uniform((int)((uint64_t)p >> 32));
  return (const char*)((uint64_t)hi << 32 | lo);
}
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
// Where keys are split: the document's chunks are shares first .. first + count - 1
// of the call, of `steps` steps each, the last to the document's end.
struct Share {
  int doc, chunk, first, count, steps;
};
// Share i of the call (doc -1: there is none).  The longest chunk is made as short as
// p.shares shares allow when every document takes whole ones, at least p.least steps:
// found from all documents' lengths, so that unlike ones still keep the CUs equally busy.
__device__ Share share_of(const AttnArgs& a, const AttnPlan& p, int step, int i) {
  constexpr int R = MAX_SHARES / 64;  // documents lane, lane + 64, ..
  const int lane = threadIdx.x & 63;
  int n[R], all = 0;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    n[r] = 0;
    if (r * 64 + lane < a.docs) {
      const Doc d = doc_of(a, r * 64 + lane);
      if (d.nq > 0) n[r] = (sees(a, d, d.nq - 1) + step - 1) / step;
    }
    all += n[r];
  }
  all = __builtin_amdgcn_readlane(lanes_upto(all), 63);
  auto chunks = [&](int r, int len) { return r * 64 + lane < a.docs ? max(1, (int)((uint32_t)(n[r] + len - 1) / (uint32_t)len)) : 0; };
  // sum n / len <= chunks <= sum n / len + documents
  int lo = max(p.least, all / p.shares), hi = max(lo, all / (p.shares - a.docs) + 1);
  while (lo < hi) {
    const int len = (lo + hi) >> 1;
    int sum = 0;
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (r * 64 < a.docs) sum += chunks(r, len);
    if (__builtin_amdgcn_readlane(lanes_upto(sum), 63) <= p.shares)
      hi = len;
    else
      lo = len + 1;
  }
  Share s{-1, 0, 0, 0, 0};
  int before = 0;
#pragma unroll
  for (int r = 0; r < R; ++r)
    if (r * 64 < a.docs) {
      const int c = chunks(r, lo), upto = before + lanes_upto(c);
      const unsigned long long mine = __ballot(i < upto && i >= upto - c);
      if (mine) {
        const int l = __ffsll(mine) - 1;
        s.doc = r * 64 + l;
        s.count = __builtin_amdgcn_readlane(c, l);
        s.first = __builtin_amdgcn_readlane(upto - c, l);
        s.chunk = i - s.first;
        s.steps = (__builtin_amdgcn_readlane(n[r], l) + s.count - 1) / s.count;  // as equal as whole steps allow
      }
      before = __builtin_amdgcn_readlane(upto, 63);
    }
  return s;
}

template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (15 << 8) | ((N >> 4) << 14));
}
__device__ __forceinline__ void barrier_nofence() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
// Of a wave's LDS accesses, which run in order: the compiler moves none past this.
__device__ __forceinline__ void wave_order() { asm volatile("" ::: "memory"); }
typedef __bf16 bf2_t __attribute__((ext_vector_type(2)));
typedef float f2_t __attribute__((ext_vector_type(2)));
// Two floats to bf16 in one instruction, and acc + the sum of two bf16.
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2_t{lo, hi}, bf2_t));
}
__device__ __forceinline__ float add2(float acc, uint32_t w) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf2_t, w), __builtin_bit_cast(bf2_t, 0x3f803f80u), acc, false);
}
// Buffer descriptor of `bytes` bytes from p on (both the same in every lane):
// reads past its end give zeros.
typedef uint32_t rsrc_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ rsrc_t rsrc_of(const char* p, uint32_t bytes) {
  return rsrc_t{(uint32_t)uniform((int)(uint64_t)p), (uint32_t)uniform((int)((uint64_t)p >> 32)) & 0xffffu, (uint32_t)uniform((int)bytes), 0x00020000u};
}
__device__ __forceinline__ uint32_t lds_address(const char* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)p;
}
// 16 bytes per lane from the buffer to LDS at `to` + 16 lane.  Written out, since
// the compiler lets no transposing LDS read pass while an LDS-DMA load that it
// knows of is in flight; the waits for these loads are wait_vmcnt's alone.  m0, which
// the compiler cannot be told of, is left as it was.  (The idle cycles are what a
// descriptor fresh from readfirstlane needs before its use.)
__device__ __forceinline__ void dma16(rsrc_t rs, uint32_t off, uint32_t to) {
  uint32_t m0;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 4\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds\n\ts_mov_b32 m0, %0"
               : "=&s"(m0)
               : "s"(uniform((int)to)), "v"(off), "s"(rs)
               : "memory");
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

// One row tile against the keys kb .. ke - 1 of its document.
template <typename T, int HD, int QG, int KG, int KT, int S>
__global__ void __launch_bounds__(64 * QG * KG, KT == 64 ? 2 : 1) attn_docs_kernel(AttnArgs a, AttnPlan p) {
#if defined(__HIP_DEVICE_COMPILE__)
  typedef Tile<T, HD> TL;
  constexpr bool BF = sizeof(T) == 2;
  constexpr int NW = QG * KG, ND = HD / 32, TR = 32 * QG;  // TR: rows of the tile
  constexpr int K_BYTES = KT * TL::ROW, TILE = 2 * K_BYTES, STAGE = KG * TILE;
  constexpr int TP = TILE / 1024, PER = TP / QG;  // LDS-DMA instructions of 1 KiB: of a tile, of a wave
  static_assert(TP % (2 * QG) == 0, "the waves of a key group share a tile's loads evenly");
  constexpr int MERGE = (NW - QG) * (ND * 4 + 1) * 64 * 16;
  __shared__ __attribute__((aligned(1024))) char lds[S * STAGE > MERGE ? S * STAGE : MERGE];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int qg = wave % QG, kg = wave / QG;
  const int lq = lane & 31, half = lane >> 5;

  // Workgroup i runs on XCD i % 8.  A unit is (document, chunk, key/value head);
  // its row tiles, which read the same keys, go to one XCD (to `parts` of them
  // where units are too few for eight), the tiles with most keys first.
  const int i8 = (int)blockIdx.x >> 3, x8 = (int)blockIdx.x & 7;
  const int up = (i8 / p.part_tiles) * 8 + x8;  // unit and part
  const int unit = up / p.parts, tile = p.tiles - 1 - ((i8 % p.part_tiles) * p.parts + up % p.parts);
  if (unit >= p.units || tile < 0) return;
  const int g = unit % a.Hkv;
  int dn = unit / a.Hkv;
  Share sh{dn, 0, dn, 1, 0};
  if (p.shares > 0) {
    sh = share_of(a, p, KG * KT, dn);
    if (sh.doc < 0) return;
    dn = sh.doc;
  }
  Doc d = doc_of(a, dn);
  d = Doc{uniform(d.q0), uniform(d.nq), uniform(d.k0), uniform(d.nk), uniform(d.pos), uniform(d.prefix)};
  const int G = a.Hq / a.Hkv, rows = d.nq * G, r0 = tile * TR;
  // what the join needs of each document
  if (p.shares > 0 && sh.chunk == 0 && g == 0 && tile == 0 && tid == 0) p.table[dn] = make_int4(sh.first, sh.count, sh.steps * KG * KT, 0);
  if (r0 >= rows) return;
  const int t_last = (min(r0 + TR, rows) - 1) / G;
  const int chunk_keys = sh.steps * KG * KT, kb = uniform(sh.chunk * chunk_keys);
  const int ke = uniform(min(sees(a, d, t_last), sh.chunk + 1 < sh.count ? kb + chunk_keys : 0x7fffffff));
  if (sh.chunk > 0 && kb >= ke) return;
  const int tile_first = uniform(sees(a, d, r0 / G));  // keys that every row of the tile sees
  // this wave's rows
  const int w0 = r0 + 32 * qg, w1 = min(w0 + 32, rows);
  const int see_first = uniform(w0 < rows ? sees(a, d, w0 / G) : 0), see_last = uniform(w0 < rows ? sees(a, d, (w1 - 1) / G) : 0);
  const int seen = min(ke, see_last);  // keys that some row of this wave sees
  const bool neg = a.scale < 0.f;      // scores are formed with |scale| and, where it is negative, -q
  const float sc = fabsf(a.scale) * LOG2E;
  // capped scores: cap and 1 / cap in log2 units, 2 log2(e) / cap per unit of score,
  // and for small bf16 ones the coefficients of cap tanh(x / cap) / x in x^2 (in
  // numbers of any size that a float32 x^2 may meet)
  const bool capped = a.cap > 0.f;
  const float cap2 = a.cap * LOG2E, cap_in = capped ? fminf(2.f * sc / a.cap, 3e38f) : 0.f, cap_1 = capped ? fminf(1.f / cap2, 3e38f) : 0.f;
  const float th = sc * cap_1 * (sc * cap_1);
  const bool series = th <= 1e8f && sc <= 1e6f;
  const float th0 = 0.999999901f * sc, th1 = -0.333313563f * th * sc, th2 = 0.132708743f * th * th * sc;
  const float th3 = -0.0475493467f * th * th * th * sc;
  const bool direct = !capped && !a.slopes;

  // K and V of this head, as bytes; a tile's buffer starts at its first key
  const char* kp = uniform(static_cast<const char*>(a.k.data) +
                           (dn * a.k.stride_b + d.k0 * a.k.stride_l + g * a.k.stride_h) * (long)sizeof(T));
  const char* vp = uniform(static_cast<const char*>(a.v.data) +
                           (dn * a.v.stride_b + d.k0 * a.v.stride_l + g * a.v.stride_h) * (long)sizeof(T));
  const uint32_t ksb = (uint32_t)(a.k.stride_l * sizeof(T)), vsb = (uint32_t)(a.v.stride_l * sizeof(T));
  // The waves of a key group load its tile: wave qg the parts qg, qg + QG, ..,
  // K's before V's; a part is 1 KiB of whole rows, lane l filling slot l % CH
  // of row l / CH
  constexpr int RPP = 1024 / TL::ROW;  // rows of a part
  uint32_t off[PER];
#pragma unroll
  for (int x = 0; x < PER; ++x) {
    const bool isk = x < PER / 2;
    const int r = (qg + QG * (x % (PER / 2))) * RPP + lane / TL::CH;
    const int c = (lane % TL::CH) ^ (isk ? TL::k_swz(r) : TL::v_swz(r));
    off[x] = r * (isk ? ksb : vsb) + c * 16;
  }
  const uint32_t lds0 = lds_address(lds) + kg * TILE + qg * 1024;
  auto load = [&](int u, int slot) {  // step u into stage `slot`
    const int t0 = kb + (u * KG + kg) * KT;
    const int left = min(ke - t0, KT);  // reads past the last key give zeros
#pragma unroll
    for (const bool keys : {true, false}) {
      const uint32_t sb = keys ? ksb : vsb, bytes = left > 0 ? (uint32_t)(left - 1) * sb + TL::ROW : 0u;
      const rsrc_t rs = rsrc_of((keys ? kp : vp) + (left > 0 ? (long)t0 : 0l) * sb, bytes);
      const uint32_t to = lds0 + slot * STAGE + (keys ? 0 : K_BYTES);
#pragma unroll
      for (int x = 0; x < PER / 2; ++x) dma16(rs, off[keys ? x : PER / 2 + x], to + x * QG * 1024);
    }
  };
  const int nsteps = ke > kb ? (ke - kb + KG * KT - 1) / (KG * KT) : 0;
  constexpr int D = S - 1;  // stages in flight behind the one in use
  for (int u = 0; u < D && u < nsteps; ++u) load(u, u);

  // Q operand: the lane's rows, dims 16 ks + 8 half .. (bf16), 8 c + 4 half .. (float32)
  constexpr int NQ = BF ? HD / 16 : HD / 8;
  typedef float f32x4v __attribute__((ext_vector_type(4)));
  bf16x8_t qb[BF ? NQ : 1];
  f32x4v qf[BF ? 1 : NQ];
  Rows<HD> R;
  const int row = w0 + lq;
  R.mine = row < rows;
  R.t = row / G;
  R.h = g * G + row % G;
  R.end = R.mine ? sees(a, d, R.t) : 0;
  R.slope = 0.f;
  R.at = 0;
  if (a.slopes) {
    if (R.mine) R.slope = a.slopes[R.h] * LOG2E;
    // From the first or last visible key, where the position lies before or behind all
    // of them: the scores differ by one amount, which the softmax does not see, and
    // float32 need not hold it.  (One key further where the slope is infinite: a distance
    // of zero would be no number.)
    const int out = fabsf(R.slope) < INFINITY ? 0 : 1;
    R.at = (int)max(min((long)d.pos + R.t, (long)R.end - 1 + out), (long)-out);
  }
  R.m = -INFINITY;
  R.m_ref = 0.f;
  R.l = 0.f;
#pragma unroll
  for (int ds = 0; ds < ND; ++ds)
#pragma unroll
    for (int r = 0; r < 16; ++r) R.o[ds][r] = 0.f;
  const T* qrow = static_cast<const T*>(a.q.data) + dn * a.q.stride_b + (long)(d.q0 + (R.mine ? R.t : 0)) * a.q.stride_l +
                  (R.mine ? R.h : 0) * a.q.stride_h;
#pragma unroll
  for (int c = 0; c < NQ; ++c) {
    uint4 w = *reinterpret_cast<const uint4*>(qrow + c * (BF ? 16 : 8) + half * (BF ? 8 : 4));
    const uint32_t flip = neg ? (BF ? 0x80008000u : 0x80000000u) : 0u;
    w.x ^= flip;
    w.y ^= flip;
    w.z ^= flip;
    w.w ^= flip;
    if (!R.mine) w = make_uint4(0, 0, 0, 0);
    if constexpr (BF)
      qb[c] = __builtin_bit_cast(bf16x8_t, w);
    else
      qf[c] = __builtin_bit_cast(f32x4v, w);
  }

  constexpr int NS = KT / 32;  // 32-key score blocks of a tile
  // scores x of the keys at kt: register r of block b holds key 32 b + 8 (r / 4) + 4 half + r % 4
  auto scores = [&](const char* kt, f32x16_t (&x)[NS]) {
    const f32x16_t zero = {};
    if constexpr (BF) {
      bf16x8_t kf[NQ][NS];
#pragma unroll
      for (int c = 0; c < NQ; ++c)
#pragma unroll
        for (int b = 0; b < NS; ++b) {
          const int r = b * 32 + lq;
          kf[c][b] = *reinterpret_cast<const bf16x8_t*>(kt + r * TL::ROW + (((c * 2 + half) ^ TL::k_swz(r)) << 4));
        }
#pragma unroll
      for (int c = 0; c < NQ; ++c)
#pragma unroll
        for (int b = 0; b < NS; ++b) x[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[c][b], qb[c], c ? x[b] : zero, 0, 0, 0);
      // the K reads run six ahead of their MFMAs
      constexpr int KR = NQ * NS, AHEAD = 6;
      __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
      for (int n = 0; n < KR - AHEAD; ++n) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x008, AHEAD, 0);
    } else {
#pragma unroll
      for (int c = 0; c < NQ; ++c)
#pragma unroll
        for (int b = 0; b < NS; ++b) {
          const int r = b * 32 + lq;
          const f32x4v k4 = *reinterpret_cast<const f32x4v*>(kt + r * TL::ROW + (((c * 2 + half) ^ TL::k_swz(r)) << 4));
#pragma unroll
          for (int e = 0; e < 4; ++e) x[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(k4[e], qf[c][e], c + e ? x[b] : zero, 0, 0, 0);
        }
    }
  };
  // Raises the running maximum to mt (this lane's, in log2 units), but only when it
  // grows by more than 2^8: probabilities then stay below 2^8, at the same relative
  // precision.
  auto raise = [&](float mt) {
    mt = max_pair32(mt);
    if (__ballot(mt > R.m + 8.f) != 0ull) {
      const float m_new = fmaxf(R.m, mt);
      const float alpha = exp2_hw(R.m - (m_new == -INFINITY ? 0.f : m_new));
      R.m = m_new;
      R.m_ref = m_new == -INFINITY ? 0.f : m_new;
      R.l *= alpha;
#pragma unroll
      for (int ds = 0; ds < ND; ++ds)
#pragma unroll
        for (int r = 0; r < 16; ++r) R.o[ds][r] *= alpha;
    }
  };
  // Scores as they are in log2 units: scaled, capped, biased, masked (t0: the
  // tile's first key; whole: every row of the wave sees all of it), and their maximum.
  auto shape = [&](f32x16_t (&x)[NS], int t0, bool whole) {
    if (capped) {
      if constexpr (!BF) {
        // float32: tanh(y) = y + y z Q(z), z = y^2, Q of degree 4, for |y| <= 0.6, so
        // that small scores keep 1e-7 of themselves (the form by exponentials: of the
        // cap), and by exponentials above
#pragma unroll
        for (int b = 0; b < NS; ++b)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const float y = x[b][r] * sc, u = y * cap_1, z = u * u;
            const float q = fmaf(fmaf(fmaf(fmaf(-0.00589395f, z, 0.02079462f), z, -0.05378329f), z, 0.13331915f), z, -0.333333f);
            const float far = fmaf(-2.f * cap2, __builtin_amdgcn_rcpf(exp2_hw(fabsf(x[b][r]) * cap_in) + 1.f), cap2);
            x[b][r] = fabsf(u) <= 0.6f ? fmaf(y * z, q, y) : copysignf(far, y);
          }
      } else {
        float far = 0.f;
#pragma unroll
        for (int b = 0; b < NS; ++b)
#pragma unroll
          for (int r = 0; r < 16; ++r) far = fmaxf(far, fabsf(x[b][r]));
        if (series && __ballot(!(far * cap_in <= 0.8f)) == 0ull) {
          // |x / cap| <= 0.4 ln 2 = 0.277: tanh(y) = y P(y^2), P of degree 3 to 1e-7 of
          // itself (five instructions in place of two transcendental ones and three)
#pragma unroll
          for (int b = 0; b < NS; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const float z = x[b][r] * x[b][r];
              x[b][r] *= fmaf(fmaf(fmaf(th3, z, th2), z, th1), z, th0);
            }
        } else {
          // cap tanh(x / cap) = cap - 2 cap / (e^(2 x / cap) + 1), to 1e-7 of the cap
#pragma unroll
          for (int b = 0; b < NS; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) x[b][r] = fmaf(-2.f * cap2, __builtin_amdgcn_rcpf(exp2_hw(x[b][r] * cap_in) + 1.f), cap2);
        }
      }
    } else {
#pragma unroll
      for (int b = 0; b < NS; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) x[b][r] *= sc;
    }
    if (a.slopes) {
      const float at = (float)(R.at - t0 - 4 * half);
#pragma unroll
      for (int b = 0; b < NS; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) x[b][r] = fmaf(-R.slope, fabsf(at - (float)(32 * b + 8 * (r >> 2) + (r & 3))), x[b][r]);
    }
    const int end = min(R.end, ke) - t0 - 4 * half;
    float mt = -INFINITY;
#pragma unroll
    for (int b = 0; b < NS; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        if (!whole && 32 * b + 8 * (r >> 2) + (r & 3) >= end) x[b][r] = -INFINITY;
        mt = fmaxf(mt, x[b][r]);
      }
    return mt;
  };
  auto highest = [&](const f32x16_t (&x)[NS]) {
    float mt = -INFINITY;
#pragma unroll
    for (int b = 0; b < NS; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) mt = fmaxf(mt, x[b][r]);
    return mt;
  };
  // probabilities in place of scores x (which `fold` takes to log2 units), and in
  // pairs pw for bf16, the type that the matrix unit takes beside values of bf16's range
  // (IEEE half, eight times finer, ends at 65504, and values with it).  Each is off by
  // 2^-8 of itself at most; the sum is that of the rounded ones, which the products see.
  // Against 64 bits outputs are 0.0022 off in all, 0.0017 by their own rounding alone.
  auto exponentials = [&](f32x16_t (&x)[NS], uint32_t (&pw)[BF ? NS * 8 : 1], float fold) {
    float psum = 0.f;
#pragma unroll
    for (int b = 0; b < NS; ++b)
#pragma unroll
      for (int r = 0; r < 16; r += 2) {
        const float e0 = exp2_hw(fmaf(x[b][r], fold, -R.m_ref)), e1 = exp2_hw(fmaf(x[b][r + 1], fold, -R.m_ref));
        if constexpr (BF) {
          pw[b * 8 + r / 2] = pack2(e0, e1);
          psum = add2(psum, pw[b * 8 + r / 2]);
        } else {
          x[b][r] = e0;
          x[b][r + 1] = e1;
          psum += e0 + e1;
        }
      }
    R.l += psum;
  };
  // output += values at vt times probabilities: x, in bf16 the pairs pw
  auto products = [&](char* vt, const f32x16_t (&x)[NS], const uint32_t (&pw)[BF ? NS * 8 : 1]) {
    if constexpr (BF) {
      // slice jk: keys 16 jk + 4 half .. and 16 jk + 8 + 4 half ..; lane n of 16
      // gives the address of row n / 4, columns 4 (n % 4) .. of its 4 x 16 block
      // and receives column n
      const int n = lane & 15, c16 = (lane >> 4) & 1, vr = n >> 2;
      char* vb = vt + (4 * half + vr) * TL::ROW;
      char* va[ND];
#pragma unroll
      for (int ds = 0; ds < ND; ++ds) {
        const int e = ds * 32 + c16 * 16 + 4 * (n & 3);
        va[ds] = vb + ((((e >> 3) ^ TL::v_swz(vr)) << 4) | ((e & 7) * 2));
      }
#pragma unroll
      for (int jk = 0; jk < KT / 16; ++jk) {
        v4s_t lo[ND], hi[ND];
#pragma unroll
        for (int ds = 0; ds < ND; ++ds) {
          lo[ds] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_t)(va[ds] + jk * 16 * TL::ROW));
          hi[ds] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_t)(va[ds] + (jk * 16 + 8) * TL::ROW));
        }
        const bf16x8_t pf = __builtin_bit_cast(bf16x8_t, make_uint4(pw[jk * 4], pw[jk * 4 + 1], pw[jk * 4 + 2], pw[jk * 4 + 3]));
#pragma unroll
        for (int ds = 0; ds < ND; ++ds)
          R.o[ds] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_shufflevector(lo[ds], hi[ds], 0, 1, 2, 3, 4, 5, 6, 7), pf, R.o[ds], 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int b = 0; b < NS; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int key = 32 * b + 8 * (r >> 2) + (r & 3);
#pragma unroll
          for (int ds = 0; ds < ND; ++ds) {
            const int e = ds * 32 + lq;
            const float w =
                *reinterpret_cast<const value_t*>(vt + (key + 4 * half) * TL::ROW + ((((e >> 2) ^ (half << 3)) << 4) | ((e & 3) * 4)));
            R.o[ds] = __builtin_amdgcn_mfma_f32_32x32x2f32(w, x[b][r], R.o[ds], 0, 0, 0);
          }
        }
    }
  };
  // Before the products of a step in which some row does not see some key: a zero
  // probability still makes NaN of a value that is no number, so such values are
  // added here to the rows that see them, and zeroed.
  auto scrub = [&](int t0, char* vt) {
    constexpr uint32_t EXP = BF ? 0x7f807f80u : 0x7f800000u;  // exponents of a word
    uint32_t top = 0;
    for (int i = qg * 64 + lane; i < K_BYTES / 16; i += QG * 64) {
      const quad_t w = reinterpret_cast<const quad_t*>(vt)[i];
      for (const uint32_t x : {w.x & EXP, w.y & EXP, w.z & EXP, w.w & EXP})
        if constexpr (BF)
          top = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(v2us_t, top), __builtin_bit_cast(v2us_t, x)));
        else
          top = max(top, x);
    }
    bool broken = __ballot((top & 0xffffu) == 0x7f80u || (top >> 16) == 0x7f80u) != 0ull;
    if constexpr (QG > 1) broken = __syncthreads_or(broken);
    if (!broken) return;
    for (int key = 0; key < KT; ++key) {
      const char* vrow = vt + key * TL::ROW;
#pragma unroll
      for (int ds = 0; ds < ND; ++ds)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int e = ds * 32 + 8 * (r >> 2) + 4 * half + (r & 3), b = e * (int)sizeof(T);
          // (bf16: the word that holds the element, whose upper half is that of an odd one)
          const uint32_t w = *reinterpret_cast<const word_t*>(vrow + ((((b >> 4) ^ TL::v_swz(key)) << 4) | (b & 12)));
          const float f = __uint_as_float(BF ? (r & 1 ? w & 0xffff0000u : w << 16) : w);
          if (t0 + key < min(R.end, ke) && !(fabsf(f) < INFINITY)) R.o[ds][r] += f;
        }
    }
    // other lanes' reads lie before the stores, and the stores before other lanes' reads
    if constexpr (QG > 1)
      __syncthreads();
    else
      wave_order();
    for (int i = qg * 64 + lane; i < K_BYTES / 4; i += QG * 64) {
      word_t* w = reinterpret_cast<word_t*>(vt) + i;
      *w = numbers<T>(*w);
    }
    if constexpr (QG > 1)
      __syncthreads();
    else
      wave_order();
  };
  for (int u = 0; u < nsteps; ++u) {
    if (u + D <= nsteps)
      wait_vmcnt<PER*(D - 1)>();
    else
      wait_vmcnt<0>();
    // stage u is there; every wave is done with the one refilled next (with one
    // row group a wave reads only what it loaded itself)
    if constexpr (QG > 1)
      barrier_nofence();
    else
      wave_order();
    if (u + D < nsteps) load(u + D, (u + D) % S);
    const int t0 = kb + (u * KG + kg) * KT;
    char *const slot = lds + (u % S) * STAGE + kg * TILE, *const vt = slot + K_BYTES;
    if (kb + (u + 1) * KG * KT > tile_first) scrub(t0, vt);
    if (t0 >= seen) continue;  // nothing that this wave's rows see
    f32x16_t x[NS];
    uint32_t pw[BF ? NS * 8 : 1];
    scores(slot, x);
    const bool whole = t0 + KT <= min(ke, see_first);
    float mt, fold = 1.f;  // fold: factor still to be applied in the exponent
    if (direct && whole) {
      fold = sc;
      mt = highest(x) * sc;
    } else {
      mt = shape(x, t0, whole);
    }
    // softmax first: beside another wave's products, which then do not hold it up
    // (8448 tokens: 536 -> 519 us)
    __builtin_amdgcn_s_setprio(1);
    raise(mt);
    exponentials(x, pw, fold);
    __builtin_amdgcn_s_setprio(0);
    products(vt, x, pw);
  }
  R.l = sum_pair32(R.l);
  if constexpr (KG > 1) {
    // the key groups' states join in group order: group 0's wave takes the others'
    __syncthreads();
    float4* sh = reinterpret_cast<float4*>(lds);
    if (kg > 0) {
      float4* to = sh + (size_t)(wave - QG) * (ND * 4 + 1) * 64 + lane;
#pragma unroll
      for (int ds = 0; ds < ND; ++ds)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          to[(ds * 4 + r) * 64] = make_float4(R.o[ds][4 * r], R.o[ds][4 * r + 1], R.o[ds][4 * r + 2], R.o[ds][4 * r + 3]);
      to[ND * 4 * 64] = make_float4(R.m, R.l, 0.f, 0.f);
    }
    __syncthreads();
    if (kg > 0) return;
    for (int k2 = 1; k2 < KG; ++k2) {
      const float4* from = sh + (size_t)(k2 * QG + qg - QG) * (ND * 4 + 1) * 64 + lane;
      const float4 ml = from[ND * 4 * 64];
      const float m_new = fmaxf(R.m, ml.x), ref = m_new == -INFINITY ? 0.f : m_new;
      const float fa = exp2_hw(R.m - ref), fb = exp2_hw(ml.x - ref);
      R.m = m_new;
      R.l = R.l * fa + ml.y * fb;
#pragma unroll
      for (int ds = 0; ds < ND; ++ds)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float4 w = from[(ds * 4 + r) * 64];
          R.o[ds][4 * r] = R.o[ds][4 * r] * fa + w.x * fb;
          R.o[ds][4 * r + 1] = R.o[ds][4 * r + 1] * fa + w.y * fb;
          R.o[ds][4 * r + 2] = R.o[ds][4 * r + 2] * fa + w.z * fb;
          R.o[ds][4 * r + 3] = R.o[ds][4 * r + 3] * fa + w.w * fb;
        }
    }
  }
  if (!R.mine) return;
  if (p.shares > 0) {
    // state of (query, head) for this share: hd outputs, then (m, l)
    const size_t at = ((size_t)(sh.first + sh.chunk) * a.max_q + R.t) * a.Hq + R.h;
    float* to = p.part + at * HD;
#pragma unroll
    for (int ds = 0; ds < ND; ++ds)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        *reinterpret_cast<float4*>(to + ds * 32 + 8 * r + 4 * half) =
            make_float4(R.o[ds][4 * r], R.o[ds][4 * r + 1], R.o[ds][4 * r + 2], R.o[ds][4 * r + 3]);
    if (half == 0) p.part_ml[at] = make_float2(R.m, R.l);
    return;
  }
  const float inv = R.l == 0.f ? 0.f : 1.f / R.l;
  T* to = static_cast<T*>(a.out.data) + dn * a.out.stride_b + (long)(d.q0 + R.t) * a.out.stride_l + R.h * a.out.stride_h;
#pragma unroll
  for (int ds = 0; ds < ND; ++ds)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int e = ds * 32 + 8 * r + 4 * half;
      const float4 w = make_float4(R.o[ds][4 * r] * inv, R.o[ds][4 * r + 1] * inv, R.o[ds][4 * r + 2] * inv, R.o[ds][4 * r + 3] * inv);
      if constexpr (BF)
        *reinterpret_cast<uint2*>(to + e) = make_uint2(pack2(w.x, w.y), pack2(w.z, w.w));
      else
        *reinterpret_cast<float4*>(to + e) = w;
    }
#endif
}

// Joins a row's chunk states in a fixed order: W waves per row, their lanes first a
// chunk's (maximum, sum) each, then 16 bytes of output each, in HD / 4 lanes per
// chunk, W 256 / HD chunks side by side.
template <typename T, int HD, int W>
__global__ void __launch_bounds__(256) attn_join_kernel(AttnArgs a, AttnPlan p) {
  constexpr int LPC = HD / 4, SIDE = 64 / LPC * W;  // lanes per chunk, chunks side by side
  __shared__ float4 sums[W > 1 ? W - 1 : 1][LPC];
  const int lane = threadIdx.x & 63, wave = (threadIdx.x >> 6) % W;  // of the row
  const long row = ((long)blockIdx.x * 4 + (threadIdx.x >> 6)) / W;
  if (row >= (long)a.docs * a.max_q * a.Hq) return;
  const int h = (int)(row % a.Hq);
  const long dt = row / a.Hq;
  const int t = (int)(dt % a.max_q), dn = (int)(dt / a.max_q);
  const int4 w4 = p.table[dn];
  const Doc d = doc_of(a, dn);
  if (t >= d.nq) return;
  // its document's chunks of which it sees a key; its tile ran them all
  const int n = w4.z > 0 ? min(w4.y, (sees(a, d, t) + w4.z - 1) / w4.z) : 0;
  const size_t next = (size_t)a.max_q * a.Hq, at = w4.x * next + (size_t)t * a.Hq + h;
  const float2* ml = p.part_ml + at;
  const int e = lane % LPC * 4, side = wave * (64 / LPC) + lane / LPC;
  const float* part = p.part + at * HD + e;
  constexpr int EARLY = 4;  // outputs asked for beside the first maxima and sums
  float4 early[EARLY];
#pragma unroll
  for (int j = 0; j < EARLY; ++j)
    early[j] = j * SIDE + side < n ? *reinterpret_cast<const float4*>(part + (j * SIDE + side) * next * HD) : make_float4(0.f, 0.f, 0.f, 0.f);
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
    if (c0 + lane < n) s = ml[(c0 + lane) * next];
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
      const float4 w = *reinterpret_cast<const float4*>(part + (c0 + c) * next * HD);
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
  T* to = static_cast<T*>(a.out.data) + dn * a.out.stride_b + (long)(d.q0 + t) * a.out.stride_l + h * a.out.stride_h + e;
  if constexpr (sizeof(T) == 2)
    *reinterpret_cast<uint2*>(to) = make_uint2(pack2(o.x * inv, o.y * inv), pack2(o.z * inv, o.w * inv));
  else
    *reinterpret_cast<float4*>(to) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
}

// Keys of the chunks that a row tile's width is chosen for, and the least of one.
constexpr int CHUNK_MIN = 512, CHUNK_LEAST = 256;
// Which kernel a call takes and how its grid is laid out.  Sizes only, docs and max_q at least 1.
struct Choice {
  int qg, kg, kt;
  AttnPlan plan;
  long grid;
};
Choice choose(const AttnArgs& a) {
  Choice c{};
  const bool f32 = a.dtype == DLLM_F32, wide_row = f32 && a.hd == 128;
  const int rows = a.max_q * (a.Hq / a.Hkv);
  const long heads = (long)a.docs * a.Hkv, cus = device_cu_count();
  // The widest row tile with which row tiles and chunks of CHUNK_MIN keys can still
  // give every CU a workgroup, else the narrowest: a wide tile reads keys and values
  // for more rows, a narrow one leaves more waves to split the keys.  (64 queries x
  // 1024 keys, 4 documents, 28 + 4 heads: 16 us, the widest tile 28; with half the
  // workgroups too 28.  1024 queries and keys: 27 us; chunks of 256 keys 47, of 1024
  // keys 35.)
  const long chunks_max = std::max(1, a.max_kv / CHUNK_MIN);
  // bf16 with two workgroups of 128 rows for every CU: four waves that do not split the
  // keys, two workgroups a CU, so that one's softmax lies beside the other's products
  // (8 prompts of 358 .. 1023 tokens, 32 heads: 149 us; one of eight waves and 256 rows
  // a CU, which reads keys and values half as often: 166; 8448 tokens: 530 both)
  const bool dense = !f32 && rows > 128 && heads * ceil_div(rows, 128) * chunks_max >= 2 * cus;
  c.qg = 4;
  while (c.qg > 1 && (rows <= 16 * c.qg || heads * ceil_div(rows, 32 * c.qg) * chunks_max < cus)) c.qg /= 2;
  c.kg = dense ? 1 : c.qg == 4 ? (f32 ? 1 : 2) : wide_row ? 2 : 4;
  c.kt = dense ? 64 : 32;
  AttnPlan& p = c.plan;
  p.tiles = ceil_div(rows, 32 * c.qg);
  const int step = c.kg * c.kt;
  const long slots = dense ? 2 * cus : cus;
  // Where they leave CUs without a workgroup, shares for all of them (31 documents of
  // one token, one of 16384 keys among 500: 29 us; chunks as many for every document, by
  // the longest: 56).  Chunks of 256 keys at least (one token over 4000
  // float32 keys: 20 us, 128 keys 18, 512 keys 24; 32 queries x 768 keys twice, bf16:
  // 18, 18 and 15).
  p.least = ceil_div(CHUNK_LEAST, step);
  const long shares = std::min({slots / ((long)a.Hkv * p.tiles), (long)a.docs * (a.max_kv / CHUNK_LEAST), (long)MAX_SHARES});
  p.shares = shares > a.docs && (long)a.docs * (a.max_kv / step + 1) < (1l << 30) ? (int)shares : 0;
  const long units = (p.shares ? p.shares : a.docs) * (long)a.Hkv;
  p.units = (int)std::min(units, 0x7fffffffl);
  // units that leave XCDs unlike work are dealt in parts of their row tiles
  p.parts = 1;
  while (p.parts < (units >= 512 ? 1 : units >= 64 ? 2 : 8) && 2 * p.parts <= p.tiles && units * p.parts % 8) p.parts *= 2;
  p.part_tiles = ceil_div(p.tiles, p.parts);
  c.grid = (long)ceil_div(units * p.parts, 8) * 8 * p.part_tiles;
  return c;
}

template <typename T, int HD, int QG, int KG, int KT, int S>
void go(const AttnArgs& a, const Choice& c, hipStream_t s) {
  attn_docs_kernel<T, HD, QG, KG, KT, S><<<(unsigned)c.grid, 64 * QG * KG, 0, s>>>(a, c.plan);
  DLLM_LAUNCH_CHECK("attn_docs_kernel");
}
template <typename T, int HD>
void launch(const AttnArgs& a, const Choice& c, hipStream_t s) {
  constexpr bool F32 = sizeof(T) == 4, WIDE = F32 && HD == 128;  // WIDE: rows of 512 bytes, half the keys fit
  if (c.qg == 1)
    go<T, HD, 1, WIDE ? 2 : 4, 32, 2>(a, c, s);
  else if (c.qg == 2)
    go<T, HD, 2, WIDE ? 2 : 4, 32, 2>(a, c, s);
  else if (F32 || c.kg == 2)
    go<T, HD, 4, F32 ? 1 : 2, 32, 3>(a, c, s);
  else if constexpr (!F32)
    go<T, HD, 4, 1, 64, 2>(a, c, s);
  if (c.plan.shares > 0) {
    // four waves a row while that is at most sixteen a CU (28 heads' token over 8448 keys:
    // 17 us, one wave a row 21; 31 documents, one of them long: 24 and 28; 40: 45 and 44;
    // 32 queries of ten: 43 and 32)
    const long rows = (long)a.docs * a.max_q * a.Hq;
    if (rows <= 4l * device_cu_count())
      attn_join_kernel<T, HD, 4><<<(unsigned)rows, 256, 0, s>>>(a, c.plan);
    else
      attn_join_kernel<T, HD, 1><<<ceil_div(rows, 4), 256, 0, s>>>(a, c.plan);
    DLLM_LAUNCH_CHECK("attn_join_kernel");
  }
}

size_t part_values(const AttnArgs& a, const AttnPlan& p) { return (size_t)p.shares * a.max_q * a.Hq; }

}  // namespace

size_t attn_docs_bytes(const AttnArgs& a) {
  const Choice c = choose(a);
  return c.plan.shares > 0 ? part_values(a, c.plan) * (a.hd * 4 + 8) + (size_t)a.docs * sizeof(int4) : 0;
}

// A launch's threads must be below 2^32.
bool attn_docs_fits(const AttnArgs& a) {
  if (a.docs == 0 || a.max_q == 0) return true;
  const Choice c = choose(a);
  return c.grid * (64 * c.qg * c.kg) < (1l << 32);
}

void launch_attn_docs(const AttnArgs& a, void* ws, hipStream_t s) {
  Choice c = choose(a);
  if (c.plan.shares > 0) {
    c.plan.table = static_cast<int4*>(ws);
    c.plan.part = reinterpret_cast<float*>(c.plan.table + a.docs);
    c.plan.part_ml = reinterpret_cast<float2*>(c.plan.part + part_values(a, c.plan) * a.hd);
  }
  if (a.dtype == DLLM_F32)
    a.hd == 64 ? launch<float, 64>(a, c, s) : launch<float, 128>(a, c, s);
  else
    a.hd == 64 ? launch<bf16_t, 64>(a, c, s) : launch<bf16_t, 128>(a, c, s);
}

}  // namespace dllm
