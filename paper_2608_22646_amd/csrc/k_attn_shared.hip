// Attention of documents behind prompts that they share (dllm_shared_attention), on the
// row tiles of attn_tile.h.
//
// Few rows of a document: the queries of consecutive documents of one prompt are stacked
// into row tiles, which read the prompt's keys once for all of them; each document's own
// keys are read by a tile of its own rows.  Both are split over workgroups by keys, leave
// their states in the workspace, and a join takes a row's states over its prompt's chunks
// and its document's.  What is stacked and split how is found on the device, from the
// lengths there (shared_plan_kernel): a list of units of like work, those of the prompts,
// the longer ones, first.
// Many rows: where every document's own rows fill the CUs with whole tiles, stacking would
// read no key less often and only add states; a tile then takes the prompt's keys and goes
// on with its document's, in one launch.
#include <algorithm>

#include "attn_tile.h"

namespace dllm {

namespace {

constexpr int PLAN_THREADS = 1024;
constexpr int UNIT_KEYS = 128, LEAST_KEYS = 256;  // chunks are multiples of this, and at least that
constexpr int STACK_ROWS = 128;                   // rows of a prompt's tile

// A prompt's range, cut to its slab and to the maximum.
struct Prompt {
  int k0, nk;
};
__device__ __forceinline__ Prompt prompt_at(const SharedArgs& s, int p) {
  Prompt r;
  r.k0 = s.p_start ? min(max(s.p_start[p], 0), s.p_tokens) : 0;
  r.nk = min(min(max(s.p_len ? s.p_len[p] : s.p_tokens, 0), s.p_tokens - r.k0), s.max_p);
  return r;
}
// The prompt that document d stands behind (-1: none).
__device__ __forceinline__ int prompt_of(const SharedArgs& s, int d) {
  const int p = s.prompt ? s.prompt[d] : 0;
  return p >= 0 && p < s.prompts ? p : -1;
}
// The position that a row's distances are taken from: its own, or the first or last
// visible key's where it lies before or behind all of them (one further where the slope
// is infinite): the scores differ by one amount, which the softmax does not see.
__device__ __forceinline__ int distances_from(long i, int before, int end, float slope) {
  const int out = fabsf(slope) < INFINITY ? 0 : 1;
  return (int)max(min(i, (long)end - 1 + out), (long)-before - out);
}

// ---- what is stacked and split how -------------------------------------------------
// Sum of the threads before this one, and of all of them.
__device__ __forceinline__ int before_of(int x, int* sums, int& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int upto = lanes_upto(x);
  __syncthreads();
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  int r = upto - x;
  all = 0;
  for (int w = 0; w < waves; ++w) {
    const int n = sums[w];
    if (w < wave) r += n;
    all += n;
  }
  return r;
}

// Per query in document order (p.tok): {document, token, own position, own keys that it
// sees}; per segment (p.seg: documents, then runs of documents behind one prompt):
// {state of its first chunk's first row, chunks, rows of a head, keys of a chunk}; per unit
// (p.unit): {document or ~prompt, first row, rows of its segment, first key}, {keys' end,
// state of its chunk, the run's first query}; per query (p.tok) what the join takes.
__global__ void __launch_bounds__(PLAN_THREADS) shared_plan_kernel(SharedArgs s, SharedPlan p) {
#if defined(__HIP_DEVICE_COMPILE__)
  const AttnArgs& a = s.own;
  __shared__ int sums[PLAN_THREADS / 64];
  __shared__ int first_l[PLAN_THREADS + 1], prompt_l[PLAN_THREADS], q0_l[PLAN_THREADS];
  __shared__ Doc doc_l[PLAN_THREADS];
  const int tid = threadIdx.x, N = blockDim.x, G = a.Hq / a.Hkv;
  // documents, and the runs among them
  int queries = 0, runs = 0, last_prompt = -1;
  for (int b0 = 0; b0 < a.docs; b0 += N) {
    const int d = b0 + tid, there = d < a.docs;
    Doc doc{0, 0, 0, 0, 0, 0};
    int pr = -1;
    if (there) {
      doc = doc_of(a, d);
      pr = prompt_of(s, d);
    }
    int all;
    const int first = min(queries + before_of(doc.nq, sums, all), p.cap);  // (documents that share queries: cut)
    doc.nq = min(doc.nq, p.cap - first);
    first_l[tid] = first;
    prompt_l[tid] = pr;
    doc_l[tid] = doc;
    const int total = min(queries + all, p.cap);
    if (tid == 0) first_l[min(N, a.docs - b0)] = total;
    __syncthreads();
    const int prev = tid ? prompt_l[tid - 1] : last_prompt;
    const int starts = there && pr >= 0 && pr != prev;
    int new_runs;
    const int run = runs + before_of(starts, sums, new_runs) + starts - 1;  // this or the last one
    if (there) {
      if (prev >= 0 && pr != prev) p.run[starts ? run - 1 : run].y = first;
      if (starts) {
        p.run[run].x = first;
        p.run[run].z = pr;
      }
      if (pr >= 0 && d == a.docs - 1) p.run[run].y = first + doc.nq;
      p.info[d] = make_int2(first, pr >= 0 ? run : -1);
      p.seg[d] = make_int4(0, 0, doc.nq * G, doc.nq > 0 ? sees(a, doc, doc.nq - 1) : 0);
    }
    const int here = min(N, a.docs - b0);
    for (int i = first_l[0] + tid; i < total; i += N) {
      int lo = 0, hi = here - 1;  // the last document whose first query is at most i
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (first_l[mid] <= i)
          lo = mid;
        else
          hi = mid - 1;
      }
      const Doc x = doc_l[lo];
      const int t = i - first_l[lo];
      p.tok[3 * (size_t)i] = make_int4(b0 + lo, x.q0 + t, (int)max(min((long)x.pos + t, 0x7fffffffl), -0x80000000l), sees(a, x, t));
    }
    last_prompt = prompt_l[here - 1];
    queries = total;
    runs += new_runs;
    __syncthreads();
  }
  // segments: the runs', then the documents'; rows, keys and row tiles of each
  const int segs = runs + a.docs;
  auto seg_at = [&](int i) { return i < runs ? a.docs + i : i - runs; };
  auto size_of = [&](int i, int& rows, int& keys) {
    if (i < runs) {
      const int4 r = p.run[i];
      rows = (r.y - r.x) * G;
      keys = prompt_at(s, r.z).nk;
    } else {
      const int4 r = p.seg[i - runs];
      rows = r.z;
      keys = r.w;
    }
    if (rows == 0) keys = 0;
  };
  auto tiles_of = [&](int i, int rows) { return (rows + (i < runs ? STACK_ROWS : p.own_rows) - 1) / (i < runs ? STACK_ROWS : p.own_rows); };
  // two segments a thread held, where there are no more
  const bool few = segs <= 2 * N;
  int rows_h[2] = {0, 0}, keys_h[2] = {0, 0}, tiles_h[2] = {0, 0};
  int units = 0, longest = 0;
  long work = 0;  // tiles times keys
  for (int i = tid, k = 0; i < segs; i += N, ++k) {
    int rows, keys;
    size_of(i, rows, keys);
    const int t = keys > 0 ? tiles_of(i, rows) : 0;
    if (few) {
      rows_h[k & 1] = rows;
      keys_h[k & 1] = keys;
      tiles_h[k & 1] = t;
    }
    units += t;
    work += (long)t * keys;
    longest = max(longest, keys);
  }
  int all_units, all_work, n;
  before_of(units, sums, all_units);
  before_of((int)min((work + UNIT_KEYS - 1) / UNIT_KEYS, 0x1fffffl), sums, all_work);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) longest = max(longest, __shfl_xor(longest, o, 64));
  __syncthreads();
  if ((tid & 63) == 0) sums[tid >> 6] = longest;
  __syncthreads();
  for (int w = 0; w < N >> 6; ++w) longest = max(longest, sums[w]);
  // The shortest chunks with which the units, at a key/value head each, are no more than
  // fit the rounds over the CUs that they take at least.
  const int heads = a.Hkv, rounds = (int)(((long)all_units * heads + p.slots - 1) / p.slots);
  const int most = (int)((long)rounds * p.slots / heads);
  int lo = LEAST_KEYS / UNIT_KEYS, hi = max(lo, (longest + UNIT_KEYS - 1) / UNIT_KEYS);
  if (few) {
    while (lo < hi) {
      const int len = (lo + hi) >> 1;
      int c = 0;
#pragma unroll
      for (int k = 0; k < 2; ++k) c += (keys_h[k] + len * UNIT_KEYS - 1) / (len * UNIT_KEYS) * tiles_h[k];
      before_of(c, sums, n);
      if (n <= most)
        hi = len;
      else
        lo = len + 1;
    }
  } else {
    lo = most > all_units ? min(hi, max(lo, all_work / (most - all_units) + 1)) : hi;
  }
  const int len = lo * UNIT_KEYS;
  // segments' units and states
  int entry = 0, state = 0;
  for (int i0 = 0; i0 < segs; i0 += N) {
    const int i = i0 + tid;
    int rows = 0, keys = 0, tiles = 0;
    if (i < segs) {
      size_of(i, rows, keys);
      tiles = keys > 0 ? tiles_of(i, rows) : 0;
    }
    const int chunks = (keys + len - 1) / len;
    const int each = chunks > 1 ? ((keys + chunks - 1) / chunks + UNIT_KEYS - 1) / UNIT_KEYS * UNIT_KEYS : keys;
    int all_e, all_s;
    const int e0 = entry + before_of(chunks * tiles, sums, all_e), s0 = state + before_of(chunks * rows * heads, sums, all_s);
    if (i < segs) {
      const int4 run = i < runs ? p.run[i] : make_int4(0, 0, 0, 0);
      p.seg[seg_at(i)] = make_int4(s0, chunks, rows, each);
      for (int e = 0; e < chunks * tiles && e0 + e < p.units; ++e) {
        const int c = e / tiles, t = e - c * tiles;
        p.unit[2 * (size_t)(e0 + e)] = make_int4(i < runs ? ~run.z : i - runs, t * (i < runs ? STACK_ROWS : p.own_rows), rows, c * each);
        p.unit[2 * (size_t)(e0 + e) + 1] = make_int4(min(keys, (c + 1) * each), s0 + c * rows * heads, run.x, 0);
      }
    }
    entry += all_e;
    state += all_s;
  }
  if (tid == 0) {
    p.count[0] = min(entry, p.units);
    p.count[1] = queries;
  }
  __syncthreads();
  for (int i = tid; i < queries; i += N) {
    const int4 t = p.tok[3 * (size_t)i];
    const int2 f = p.info[t.x];
    const int4 own = p.seg[t.x];
    int4 run = make_int4(0, 0, 0, 0);
    int at = 0;
    if (f.y >= 0) {
      run = p.seg[a.docs + f.y];
      at = (i - p.run[f.y].x) * G;
    }
    p.tok[3 * (size_t)i + 1] = make_int4(own.x + (i - f.x) * G, own.z, own.w > 0 ? min(own.y, (t.w + own.w - 1) / own.w) : 0, 0);
    p.tok[3 * (size_t)i + 2] = make_int4(run.x + at, run.z, run.y, 0);
  }
#endif
}

// ---- units ------------------------------------------------------------------------
template <typename T, int HD, int QG, int KG, int KT, int S>
struct Shape {
  static constexpr int qg = QG, kg = KG, kt = KT, s = S, lds = attend_lds<T, HD, QG, KG, KT, S>();
};
template <typename T, int HD>
struct Shapes {
  static constexpr bool WIDE = sizeof(T) == 4 && HD == 128;  // rows of 512 bytes, half the keys fit
  typedef Shape<T, HD, 4, 2, 32, WIDE ? 2 : 3> Stack;
  typedef Shape<T, HD, WIDE ? 4 : 2, WIDE ? 2 : 4, 32, 2> Own;
  static constexpr int lds = Stack::lds > Own::lds ? Stack::lds : Own::lds;
};
constexpr int own_rows(bool f32, int hd) { return f32 && hd == 128 ? 128 : 64; }

template <typename T, int HD>
__global__ void __launch_bounds__(512, 1) shared_units_kernel(SharedArgs s, SharedPlan p) {
#if defined(__HIP_DEVICE_COMPILE__)
  typedef typename Shapes<T, HD>::Stack Stack;
  typedef typename Shapes<T, HD>::Own Own;
  __shared__ __attribute__((aligned(1024))) char lds[Shapes<T, HD>::lds];
  const AttnArgs& a = s.own;
  const int G = a.Hq / a.Hkv, wave = uniform((int)threadIdx.x >> 6), lq = threadIdx.x & 31;
  const long n = (long)p.count[0] * a.Hkv;
  for (long u = blockIdx.x; u < n; u += gridDim.x) {
    if (u != (long)blockIdx.x) __syncthreads();  // the last unit's LDS is free
    const int e = (int)(u / a.Hkv), g = (int)(u % a.Hkv);
    const int4 u0 = p.unit[2 * (size_t)e], u1 = p.unit[2 * (size_t)e + 1];
    const int who = uniform(u0.x), r0 = uniform(u0.y), rows = uniform(u0.z);
    const size_t state = (size_t)uniform(u1.y) + (size_t)g * rows;
    auto keep = [&](const Rows<HD>& R) { keep_state(R, p.part, p.part_ml, state + (size_t)R.t * G + R.h % G); };
    if (who < 0) {
      const Prompt pr = prompt_at(s, ~who);
      Keys k = keys_at<T>(s.pk, s.pv, ~who, pr.k0, g);
      k.kb = uniform(u0.w);
      k.ke = k.tile_first = k.see_first = k.see_last = uniform(u1.x);
      const int before = uniform(pr.nk), row = r0 + 32 * (wave % Stack::qg) + lq, first = uniform(u1.z);
      if (r0 + 32 * (wave % Stack::qg) >= rows) k.see_first = k.see_last = 0;
      auto rows_of = [&](Rows<HD>& R) {
        R.mine = row < rows;
        R.t = R.mine ? row / G : 0;
        R.h = g * G + (R.mine ? row % G : 0);
        R.end = R.mine ? k.ke : 0;
        R.slope = 0.f;
        R.at = 0;
        const int4 q = p.tok[3 * (size_t)(first + R.t)];
        if (a.slopes) {
          if (R.mine) R.slope = a.slopes[R.h] * LOG2E;
          R.at = distances_from(q.z, before, q.w, R.slope) + before;
        }
        return static_cast<const T*>(a.q.data) + q.x * a.q.stride_b + q.y * a.q.stride_l + R.h * a.q.stride_h;
      };
      attend<T, HD, Stack::qg, Stack::kg, Stack::kt, Stack::s, false>(a, lds, k, k, rows_of, keep);
    } else {
      Doc d = doc_of(a, who);
      d = Doc{uniform(d.q0), uniform(d.nq), uniform(d.k0), uniform(d.nk), uniform(d.pos), uniform(d.prefix)};
      const int kb = uniform(u0.w), t_last = (min(r0 + 32 * Own::qg, rows) - 1) / G, ke = uniform(min(sees(a, d, t_last), u1.x));
      if (kb >= ke && kb > 0) continue;
      const int w0 = r0 + 32 * (wave % Own::qg), w1 = min(w0 + 32, rows), row = w0 + lq;
      Keys k = keys_at<T>(a.k, a.v, who, d.k0, g);
      k.kb = kb;
      k.ke = ke;
      k.tile_first = uniform(sees(a, d, r0 / G));
      k.see_first = uniform(w0 < rows ? sees(a, d, w0 / G) : 0);
      k.see_last = uniform(w0 < rows ? sees(a, d, (w1 - 1) / G) : 0);
      auto rows_of = [&](Rows<HD>& R) {
        R.mine = row < rows;
        R.t = R.mine ? row / G : 0;
        R.h = g * G + (R.mine ? row % G : 0);
        R.end = R.mine ? sees(a, d, R.t) : 0;
        R.slope = 0.f;
        R.at = 0;
        if (a.slopes) {
          if (R.mine) R.slope = a.slopes[R.h] * LOG2E;
          const int pr = prompt_of(s, who);
          R.at = distances_from((long)d.pos + R.t, pr >= 0 ? prompt_at(s, pr).nk : 0, R.end, R.slope);
        }
        return static_cast<const T*>(a.q.data) + who * a.q.stride_b + (long)(d.q0 + R.t) * a.q.stride_l + R.h * a.q.stride_h;
      };
      attend<T, HD, Own::qg, Own::kg, Own::kt, Own::s, false>(a, lds, k, k, rows_of, keep);
    }
  }
#endif
}

template <typename T, int HD, int W>
__global__ void __launch_bounds__(256) shared_join_kernel(SharedArgs s, SharedPlan p) {
#if defined(__HIP_DEVICE_COMPILE__)
  const AttnArgs& a = s.own;
  const long row = ((long)blockIdx.x * 4 + (threadIdx.x >> 6)) / W;
  const int h = (int)(row % a.Hq), G = a.Hq / a.Hkv;
  const long i = row / a.Hq;
  if (i >= p.count[1]) return;
  const int4 q = p.tok[3 * i], own = p.tok[3 * i + 1], run = p.tok[3 * i + 2];
  const int g = h / G, in = h % G;
  const size_t at_own = (size_t)own.x + (size_t)g * own.y + in, at_run = (size_t)run.x + (size_t)g * run.y + in;
  const size_t next_own = (size_t)own.y * a.Hkv, next_run = (size_t)run.y * a.Hkv;
  const int chunks = run.z;
  join_row<T, HD, W>(static_cast<T*>(a.out.data) + q.x * a.out.stride_b + q.y * a.out.stride_l + h * a.out.stride_h, chunks + own.z, p.part,
                     p.part_ml, [&](int c) { return c < chunks ? at_run + c * next_run : at_own + (c - chunks) * next_own; });
#endif
}

// ---- many rows --------------------------------------------------------------------
template <typename T, int HD, int QG, int KG, int KT, int S>
__global__ void __launch_bounds__(64 * QG * KG, KT == 64 ? 2 : 1) shared_chain_kernel(SharedArgs s, SharedPlan p) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int TR = 32 * QG;
  __shared__ __attribute__((aligned(1024))) char lds[attend_lds<T, HD, QG, KG, KT, S>()];
  const AttnArgs& a = s.own;
  const int G = a.Hq / a.Hkv, wave = uniform((int)threadIdx.x >> 6), qg = wave % QG, lq = threadIdx.x & 31;
  // Workgroup i runs on XCD i % 8: the row tiles of a (document, key/value head), which
  // read the same keys, go to one XCD, the tiles with most keys first
  const int i8 = (int)blockIdx.x >> 3, x8 = (int)blockIdx.x & 7;
  const int unit = (i8 / p.tiles) * 8 + x8, tile = p.tiles - 1 - i8 % p.tiles;
  if (unit >= a.docs * a.Hkv) return;
  const int g = unit % a.Hkv, dn = unit / a.Hkv;
  Doc d = doc_of(a, dn);
  d = Doc{uniform(d.q0), uniform(d.nq), uniform(d.k0), uniform(d.nk), uniform(d.pos), uniform(d.prefix)};
  const int rows = d.nq * G, r0 = tile * TR;
  if (r0 >= rows) return;
  const int pn = prompt_of(s, dn);
  const Prompt pr = pn >= 0 ? prompt_at(s, pn) : Prompt{0, 0};
  Keys k1 = keys_at<T>(s.pk, s.pv, max(pn, 0), pr.k0, g), k2 = keys_at<T>(a.k, a.v, dn, d.k0, g);
  k1.kb = k2.kb = 0;
  k1.ke = k1.tile_first = k1.see_first = k1.see_last = uniform(pr.nk);
  const int w0 = r0 + 32 * qg, w1 = min(w0 + 32, rows), row = w0 + lq;
  k2.ke = uniform(sees(a, d, (min(r0 + TR, rows) - 1) / G));
  k2.tile_first = uniform(sees(a, d, r0 / G));
  k2.see_first = uniform(w0 < rows ? sees(a, d, w0 / G) : 0);
  k2.see_last = uniform(w0 < rows ? sees(a, d, (w1 - 1) / G) : 0);
  if (w0 >= rows) k1.see_first = k1.see_last = 0;
  auto rows_of = [&](Rows<HD>& R) {
    R.mine = row < rows;
    R.t = R.mine ? row / G : 0;
    R.h = g * G + (R.mine ? row % G : 0);
    R.end = R.mine ? sees(a, d, R.t) : 0;
    R.slope = 0.f;
    R.at = 0;
    if (a.slopes) {
      if (R.mine) R.slope = a.slopes[R.h] * LOG2E;
      R.at = distances_from((long)d.pos + R.t, k1.ke, R.end, R.slope);
    }
    return static_cast<const T*>(a.q.data) + dn * a.q.stride_b + (long)(d.q0 + R.t) * a.q.stride_l + R.h * a.q.stride_h;
  };
  attend<T, HD, QG, KG, KT, S, true>(a, lds, k1, k2, rows_of, [&](const Rows<HD>& R) {
    store_row(R, static_cast<T*>(a.out.data) + dn * a.out.stride_b + (long)(d.q0 + R.t) * a.out.stride_l + R.h * a.out.stride_h);
  });
#endif
}

// ---- choice, from sizes only ------------------------------------------------------
SharedPlan choose(const SharedArgs& s) {
  const AttnArgs& a = s.own;
  SharedPlan p{};
  const int G = a.Hq / a.Hkv, rows = a.max_q * G, cus = device_cu_count();
  const bool f32 = a.dtype == DLLM_F32;
  p.slots = cus;
  p.own_rows = own_rows(f32, a.hd);
  p.tiles = ceil_div(rows, 128);
  p.chain = rows > 128 && (long)a.docs * a.Hkv * p.tiles >= 2 * cus;
  if (p.chain) {
    p.grid = ((long)a.docs * a.Hkv + 7) / 8 * 8 * p.tiles;
    return p;
  }
  const long packed = a.q.stride_b == 0 ? a.q_tokens : (long)a.docs * a.max_q;
  p.cap = (int)std::min(std::min((long)a.docs * a.max_q, packed), 0x7fffffffl);
  // units without a split: of the runs (as many as documents, but where prompts' documents
  // follow each other no more than those and one more for each without) and the documents
  const long stack = ((long)p.cap * G + STACK_ROWS - 1) / STACK_ROWS;
  const long own = std::min((long)a.docs * ceil_div(rows, p.own_rows), ((long)p.cap * G + p.own_rows - 1) / p.own_rows + a.docs);
  p.units = stack + (s.prompt ? a.docs : 1) + own + p.slots / a.Hkv + 1;
  const long expected = (stack + (s.prompt ? std::min(a.docs, s.prompts) : 1) + own) * a.Hkv;
  p.grid = std::min((expected + cus - 1) / cus * cus, 1l << 22);
  p.states = 2l * p.cap * a.Hq + (long)p.slots * STACK_ROWS;
  return p;
}

size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }
// The workspace's parts, one behind the other.
size_t lay_out(const SharedArgs& s, SharedPlan& p, char* ws) {
  char* at = ws;
  auto take = [&](size_t bytes) {
    char* r = at;
    at += up256(bytes);
    return r;
  };
  p.count = reinterpret_cast<int*>(take(2 * sizeof(int)));
  p.tok = reinterpret_cast<int4*>(take((size_t)p.cap * 3 * sizeof(int4)));
  p.seg = reinterpret_cast<int4*>(take((size_t)s.own.docs * 2 * sizeof(int4)));
  p.run = reinterpret_cast<int4*>(take((size_t)s.own.docs * sizeof(int4)));
  p.info = reinterpret_cast<int2*>(take((size_t)s.own.docs * sizeof(int2)));
  p.unit = reinterpret_cast<int4*>(take((size_t)p.units * 2 * sizeof(int4)));
  p.part_ml = reinterpret_cast<float2*>(take((size_t)p.states * sizeof(float2)));
  p.part = reinterpret_cast<float*>(take((size_t)p.states * s.own.hd * sizeof(float)));
  return at - ws;
}

template <typename T, int HD>
void launch(const SharedArgs& s, const SharedPlan& p, hipStream_t st) {
  constexpr bool F32 = sizeof(T) == 4;
  if (p.chain) {
    if constexpr (F32)
      shared_chain_kernel<T, HD, 4, 1, 32, 3><<<(unsigned)p.grid, 256, 0, st>>>(s, p);
    else
      shared_chain_kernel<T, HD, 4, 1, 64, 2><<<(unsigned)p.grid, 256, 0, st>>>(s, p);
    DLLM_LAUNCH_CHECK("shared_chain_kernel");
    return;
  }
  const int docs = s.own.docs;
  shared_plan_kernel<<<1, docs <= 64 ? 64 : docs <= 256 ? 256 : PLAN_THREADS, 0, st>>>(s, p);
  DLLM_LAUNCH_CHECK("shared_plan_kernel");
  shared_units_kernel<T, HD><<<(unsigned)p.grid, 512, 0, st>>>(s, p);
  DLLM_LAUNCH_CHECK("shared_units_kernel");
  const long rows = (long)p.cap * s.own.Hq;
  if (rows <= 4l * device_cu_count())
    shared_join_kernel<T, HD, 4><<<(unsigned)rows, 256, 0, st>>>(s, p);
  else
    shared_join_kernel<T, HD, 1><<<ceil_div(rows, 4), 256, 0, st>>>(s, p);
  DLLM_LAUNCH_CHECK("shared_join_kernel");
}

// Without a prompt's key it is attention of documents.
bool alone(const SharedArgs& s) { return s.prompts == 0 || s.max_p == 0; }

}  // namespace

size_t attn_shared_bytes(const SharedArgs& s) {
  if (alone(s)) return attn_docs_bytes(s.own);
  SharedPlan p = choose(s);
  return p.chain ? 0 : lay_out(s, p, nullptr);
}

// A launch's threads must be below 2^32, and states countable.
bool attn_shared_fits(const SharedArgs& s) {
  if (alone(s)) return attn_docs_fits(s.own);
  const SharedPlan p = choose(s);
  if (p.chain) return p.grid * 256 < (1l << 32);
  return p.states < (1l << 31) && p.units < (1l << 31) && (long)p.cap * s.own.Hq < (1l << 26);
}

void launch_attn_shared(const SharedArgs& s, void* ws, hipStream_t st) {
  if (alone(s)) return launch_attn_docs(s.own, ws, st);
  SharedPlan p = choose(s);
  if (!p.chain) lay_out(s, p, static_cast<char*>(ws));
  if (s.own.dtype == DLLM_F32)
    s.own.hd == 64 ? launch<float, 64>(s, p, st) : launch<float, 128>(s, p, st);
  else
    s.own.hd == 64 ? launch<bf16_t, 64>(s, p, st) : launch<bf16_t, 128>(s, p, st);
}

}  // namespace dllm
