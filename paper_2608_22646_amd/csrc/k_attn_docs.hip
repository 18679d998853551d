// Attention of documents of unlike lengths (dllm_attention): grouped heads,
// positional masks, capped scores and distance biases, on the row tiles of attn_tile.h.
//
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

#include "attn_tile.h"

namespace dllm {

namespace {

constexpr int MAX_SHARES = 256;

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

// One row tile against the keys kb .. ke - 1 of its document.
template <typename T, int HD, int QG, int KG, int KT, int S>
__global__ void __launch_bounds__(64 * QG * KG, KT == 64 ? 2 : 1) attn_docs_kernel(AttnArgs a, AttnPlan p) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int TR = 32 * QG;  // TR: rows of the tile
  __shared__ __attribute__((aligned(1024))) char lds[attend_lds<T, HD, QG, KG, KT, S>()];
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
  // this wave's rows
  const int w0 = r0 + 32 * qg, w1 = min(w0 + 32, rows), row = w0 + lq;
  Keys k1 = keys_at<T>(a.k, a.v, dn, d.k0, g);
  k1.kb = kb;
  k1.ke = ke;
  k1.tile_first = uniform(sees(a, d, r0 / G));
  k1.see_first = uniform(w0 < rows ? sees(a, d, w0 / G) : 0);
  k1.see_last = uniform(w0 < rows ? sees(a, d, (w1 - 1) / G) : 0);
  auto rows_of = [&](Rows<HD>& R) {
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
    return static_cast<const T*>(a.q.data) + dn * a.q.stride_b + (long)(d.q0 + (R.mine ? R.t : 0)) * a.q.stride_l +
           (R.mine ? R.h : 0) * a.q.stride_h;
  };
  constexpr bool CHAIN = false;
  const Keys& k2 = k1;
#include "attn_tile_body.h"
  if (!R.mine) return;
  if (p.shares > 0)  // state of (query, head) for this share
    keep_state(R, p.part, p.part_ml, ((size_t)(sh.first + sh.chunk) * a.max_q + R.t) * a.Hq + R.h);
  else
    store_row(R, static_cast<T*>(a.out.data) + dn * a.out.stride_b + (long)(d.q0 + R.t) * a.out.stride_l + R.h * a.out.stride_h);
#endif
}

template <typename T, int HD, int W>
__global__ void __launch_bounds__(256) attn_join_kernel(AttnArgs a, AttnPlan p) {
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
  join_row<T, HD, W>(static_cast<T*>(a.out.data) + dn * a.out.stride_b + (long)(d.q0 + t) * a.out.stride_l + h * a.out.stride_h, n,
                     p.part + at * HD, p.part_ml + at, [&](int i) { return i * next; });
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
