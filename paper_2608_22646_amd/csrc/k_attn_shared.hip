// Attention of documents behind prompts that they share (dllm_shared_attention), on the
// row tiles of attn_tile.h, in one of two ways (chain_of):
//
// Chain, where keys are few or rows fill the CUs: a row tile of a document takes its prompt's
// keys and goes on with the document's own, in one launch without a workspace.
// Units, where few rows stand behind many keys: the queries of consecutive documents of one
// prompt are stacked into row tiles, which read the prompt's keys once for all of them; each
// document's own keys are read by a tile of its own rows.  Both are split over workgroups by
// keys, leave their states in the workspace, and a join takes a row's states over its
// prompt's chunks and its document's.  What is stacked and split how is found on the
// device, from the lengths there: a list of units of like work, those of the prompts, the
// longer ones, first: up to 64 documents by each workgroup for itself, 2.4 us; more by a
// launch before, of one workgroup, in which one thread writes all units of a segment: 65
// single tokens behind 8448 keys 19 us, 65 documents of 32 queries behind 1024 (32 heads)
// 23, 256 of them 74.
//
// What bounds them (kernel times, inputs not in a cache): 16 documents of 32 queries behind 8448
// keys, 32 heads: units 93 to 104 us, 0.7 to 0.8 PFLOP/s, of which two workgroups a CU reach 1.0
// while both have prompt keys; join 8.  Behind 1024: 37 to 40 and 7, where 67 MB of the
// documents' own keys come from HBM.  32 single tokens behind 8448 keys: 19 and 5; units are
// numbered heads fastest, so that of 4 heads the two row tiles of a chunk lie on different
// XCDs, and each prompt key passes through two L2s.  8 documents of up to 700 queries, chain:
// 125 in a row of calls, 138 to 143 traced, 0.7 PFLOP/s where long prompts in attention of
// documents reach 1.0: 2.3 rounds of workgroups, the last one not full, beside the issue of
// the softmax.  Small calls: launches, the plan and first tiles.
#include <algorithm>

#include "attn_tile.h"

namespace dllm {

namespace {

constexpr int PLAN_THREADS = 1024;
constexpr int MANY_ROWS = 128;                    // rows of a tile of many

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

// Rows of a segment's tiles (of up to 64 rows: few), and how many tiles.
__host__ __device__ __forceinline__ int tile_rows(const SharedPlan& p, int rows) { return rows > 64 ? MANY_ROWS : p.few_rows; }
__host__ __device__ __forceinline__ int tiles_of(const SharedPlan& p, int rows) {
  return rows > 64 ? (rows + MANY_ROWS - 1) / MANY_ROWS : (int)((uint32_t)(rows + p.few_rows - 1) / (uint32_t)p.few_rows);
}
__device__ __forceinline__ int units_of(const SharedPlan& p, int keys) { return (keys + p.unit_keys - 1) >> (31 - __clz(p.unit_keys)); }
// How far keys are split, of `all` units with `work` times p.unit_keys keys in all
// (without their heads): chunks no shorter than `least`, in p.unit_keys, and no more units
// than `most`.  Where there are fewer units than workgroups run at once, as many more as make
// them one round (half a round of float32, if they are few: two workgroups of a CU would only
// share its matrix units, and leave twice the states); else only what is longer than a
// workgroup's part of the whole, a unit's start and end counting as p.unit_cost.
struct Cut {
  int least, most;
};
__device__ __forceinline__ Cut cut_of(const SharedPlan& p, int all, int work, int heads) {
  const uint32_t busy = (uint32_t)p.busy / (uint32_t)heads, slots = 2 * (uint32_t)all <= busy ? busy : (uint32_t)p.slots / (uint32_t)heads;
  if ((uint32_t)all < slots) return Cut{max(1, (int)((uint32_t)work / slots)), (int)slots};
  const float part = ((float)work + (float)all * p.unit_cost) * (float)heads / (float)p.slots;
  return Cut{max(1, (int)fminf(part, (float)((1 << 30) / p.unit_keys))), 0x7fffffff};  // (no keys are as many)
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
  __shared__ int first_l[PLAN_THREADS + 1], prompt_l[PLAN_THREADS];
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
  // two segments a thread held, where there are no more
  const bool few = segs <= 2 * N;
  int rows_h[2] = {0, 0}, keys_h[2] = {0, 0}, tiles_h[2] = {0, 0};
  int units = 0, longest = 0, work = 0;  // work: tiles times keys, in unit_keys (the host sees to it that all fit)
  for (int i = tid, k = 0; i < segs; i += N, ++k) {
    int rows, keys;
    size_of(i, rows, keys);
    const int t = keys > 0 ? tiles_of(p, rows) : 0;
    if (few) {
      rows_h[k & 1] = rows;
      keys_h[k & 1] = keys;
      tiles_h[k & 1] = t;
    }
    units += t;
    work += t * units_of(p, keys);
    longest = max(longest, keys);
  }
  int all_units, all_work, n;
  before_of(units, sums, all_units);
  before_of(work, sums, all_work);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) longest = max(longest, __shfl_xor(longest, o, 64));
  __syncthreads();
  if ((tid & 63) == 0) sums[tid >> 6] = longest;
  __syncthreads();
  for (int w = 0; w < N >> 6; ++w) longest = max(longest, sums[w]);
  const int heads = a.Hkv;
  const Cut cut = cut_of(p, all_units, all_work, heads);
  int lo = cut.least, hi = max(lo, units_of(p, longest));
  if (few) {
    while (lo < hi) {
      const int len = (lo + hi) >> 1;
      int c = 0;
#pragma unroll
      for (int k = 0; k < 2; ++k) c += (keys_h[k] + len * p.unit_keys - 1) / (len * p.unit_keys) * tiles_h[k];
      before_of(c, sums, n);
      if (n <= cut.most)
        hi = len;
      else
        lo = len + 1;
    }
  } else if (cut.most < 0x7fffffff) {
    lo = cut.most > all_units ? min(hi, max(lo, all_work / (cut.most - all_units) + 1)) : hi;
  }
  const int len = lo * p.unit_keys;
  // segments' units and states
  int entry = 0, state = 0;
  for (int i0 = 0; i0 < segs; i0 += N) {
    const int i = i0 + tid;
    int rows = 0, keys = 0, tiles = 0;
    if (i < segs) {
      size_of(i, rows, keys);
      tiles = keys > 0 ? tiles_of(p, rows) : 0;
    }
    const int chunks = (keys + len - 1) / len;
    const int each = chunks > 1 ? units_of(p, (keys + chunks - 1) / chunks) * p.unit_keys : keys;
    int all_e, all_s;
    const int e0 = entry + before_of(chunks * tiles, sums, all_e), s0 = state + before_of(chunks * rows * heads, sums, all_s);
    if (i < segs) {
      const int4 run = i < runs ? p.run[i] : make_int4(0, 0, 0, 0);
      p.seg[seg_at(i)] = make_int4(s0, chunks, rows, each);
      for (int e = 0; e < chunks * tiles && e0 + e < p.units; ++e) {
        const int c = e / tiles, t = e - c * tiles;
        p.unit[2 * (size_t)(e0 + e)] = make_int4(i < runs ? ~run.z : i - runs, t * tile_rows(p, rows), rows, c * each);
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

// ---- the same, by each workgroup for itself ----------------------------------------
// At most 64 documents: lane d of the first wave holds document d, and the run of
// documents behind one prompt that starts with it.
struct Split {  // of a segment: its first unit, its first state, row tiles, rows of a head, chunks and their keys
  int unit, state, tiles, rows, chunks, each;
};
struct Segments {  // of a document, and of the run that starts with it
  Split stack, own;
  Doc doc;
  int first;                // the document's first query among all
  int prompt, p_k0, p_nk;   // its prompt (-1: none)
  int run;                  // the document that its run starts with (-1: behind no prompt)
};
struct Table {
  Segments of[64];
  int first[64];
  int units, queries;
  // The document that has query i of the call.
  __device__ __forceinline__ int holder(int i) const {
    int lo = 0;
#pragma unroll
    for (int k = 32; k > 0; k >>= 1) lo += first[lo + k] <= i ? k : 0;
    return lo;
  }
};
__device__ __forceinline__ int lane_of(int x, int lane) { return __builtin_amdgcn_readlane(x, lane); }

// By one wave.  The arrays are asked for at once: in the place of one that is not there,
// memory of the workspace, whose values are not looked at.
__device__ __forceinline__ void plan_docs(const SharedArgs& s, const SharedPlan& p, Table& t) {
  const AttnArgs& a = s.own;
  const int lane = threadIdx.x & 63, G = a.Hq / a.Hkv, heads = a.Hkv;
  const int* const none = reinterpret_cast<const int*>(p.seg);
  auto some = [&](const int* x) { return x ? x : none; };
  const int d = min(lane, a.docs - 1);
  const int q0 = some(a.q_start)[d], nq = some(a.q_len)[d], k0 = some(a.kv_start)[d], nk = some(a.kv_len)[d], pos = some(a.q_pos)[d],
            prefix = some(a.prefix)[d], pr = some(s.prompt)[d];
  const int pl = s.prompts > 64 ? 0 : min(lane, s.prompts - 1);  // up to 64 prompts: of prompt `lane`
  int pk0 = some(s.p_start)[s.p_start ? pl : 0], pn = some(s.p_len)[s.p_len ? pl : 0];
  Doc x;  // as doc_of
  x.q0 = a.q_start ? min(max(q0, 0), a.q_tokens) : 0;
  x.nq = min(min(max(a.q_len ? nq : a.q_tokens, 0), a.q_tokens - x.q0), a.max_q);
  x.k0 = a.kv_start ? min(max(k0, 0), a.kv_tokens) : 0;
  x.nk = min(min(max(a.kv_len ? nk : a.kv_tokens, 0), a.kv_tokens - x.k0), a.max_kv);
  x.pos = a.q_pos ? pos : x.nk - x.nq;
  x.prefix = a.prefix ? prefix : 0;
  const bool there = lane < a.docs;
  if (!there) x.nq = 0;
  const int prompt = there ? (s.prompt ? (pr >= 0 && pr < s.prompts ? pr : -1) : 0) : -1;
  const int pk = min(max(prompt, 0), s.prompts - 1);
  if (s.prompts > 64) {
    pk0 = some(s.p_start)[s.p_start ? pk : 0];
    pn = some(s.p_len)[s.p_len ? pk : 0];
  } else {
    pk0 = __shfl(pk0, pk, 64);
    pn = __shfl(pn, pk, 64);
  }
  Prompt y;  // as prompt_at
  y.k0 = s.p_start ? min(max(pk0, 0), s.p_tokens) : 0;
  y.nk = prompt < 0 ? 0 : min(min(max(s.p_len ? pn : s.p_tokens, 0), s.p_tokens - y.k0), s.max_p);
  const int upto = lanes_upto(x.nq), queries = min(lane_of(upto, 63), p.cap), first = min(upto - x.nq, p.cap);
  x.nq = min(x.nq, p.cap - first);  // (documents that share queries: cut)
  // runs: from a document whose prompt is not the last one's to the next such
  const int prev = __shfl_up(prompt, 1, 64);
  const bool border = there && prompt != (lane ? prev : -1);
  const unsigned long long borders = __ballot(border), starts = __ballot(border && prompt >= 0), mine = (2ull << lane) - 1;
  const int next = __ffsll(borders & ~mine) - 1, end = __shfl(first, max(next, 0), 64);
  Split st, ow;
  st.rows = border && prompt >= 0 ? ((next >= 0 ? end : queries) - first) * G : 0;
  ow.rows = x.nq * G;
  const int keys_s = st.rows > 0 ? y.nk : 0, keys_o = x.nq > 0 ? sees(a, x, x.nq - 1) : 0;
  st.tiles = keys_s > 0 ? tiles_of(p, st.rows) : 0;
  ow.tiles = keys_o > 0 ? tiles_of(p, ow.rows) : 0;
  const int ks = units_of(p, keys_s), ko = units_of(p, keys_o);
  const int all = lane_of(lanes_upto(st.tiles + ow.tiles), 63), work = lane_of(lanes_upto(st.tiles * ks + ow.tiles * ko), 63);
  const Cut cut = cut_of(p, all, work, heads);
  int longest = max(ks, ko);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) longest = max(longest, __shfl_xor(longest, o, 64));
  // the shortest chunks that give no more units; sum of keys / len <= units <= that and one more for each
  uint32_t lo = cut.least, hi = max(cut.least, longest);
  if (cut.most > all) hi = max(lo, min(hi, (uint32_t)work / (uint32_t)(cut.most - all) + 1));
  while (lo < hi) {
    const uint32_t len = (lo + hi) >> 1;
    const int c = (ks + len - 1) / len * st.tiles + (ko + len - 1) / len * ow.tiles;
    if (lane_of(lanes_upto(c), 63) <= cut.most)
      hi = len;
    else
      lo = len + 1;
  }
  int units = 0, states = 0;
  auto split = [&](Split& z, int keys, int k) {
    z.chunks = (k + lo - 1) / lo;
    z.each = z.chunks > 1 ? units_of(p, (uint32_t)(keys + z.chunks - 1) / (uint32_t)z.chunks) * p.unit_keys : keys;
    const int n = z.chunks * z.tiles, m = z.chunks * z.rows * heads, un = lanes_upto(n), um = lanes_upto(m);
    z.unit = units + un - n;
    z.state = states + um - m;
    units += lane_of(un, 63);
    states += lane_of(um, 63);
  };
  split(st, keys_s, ks);
  split(ow, keys_o, ko);
  t.of[lane] = Segments{st, ow, x, first, prompt, y.k0, y.nk, prompt >= 0 ? 63 - __clzll(starts & mine) : -1};
  t.first[lane] = there ? first : 0x7fffffff;
  if (lane == 0) {
    t.units = units;
    t.queries = queries;
  }
}
// What the join takes of query i (see shared_plan_kernel).
__device__ __forceinline__ void tell_query(const SharedArgs& s, const SharedPlan& p, const Table& t, int i) {
  const AttnArgs& a = s.own;
  const Segments& x = t.of[t.holder(i)];
  const Segments& y = t.of[max(x.run, 0)];
  const int G = a.Hq / a.Hkv, at = i - x.first, end = sees(a, x.doc, at), each = x.own.each;
  p.tok[3 * (size_t)i] = make_int4((int)(&x - t.of), x.doc.q0 + at, 0, 0);
  p.tok[3 * (size_t)i + 1] =
      make_int4(x.own.state + at * G, x.own.rows, each > 0 ? min(x.own.chunks, (int)((uint32_t)(end + each - 1) / (uint32_t)each)) : 0, 0);
  p.tok[3 * (size_t)i + 2] = make_int4(y.stack.state + (i - y.first) * G, y.stack.rows, x.run >= 0 ? y.stack.chunks : 0, 0);
}

// ---- units ------------------------------------------------------------------------
template <typename T, int HD, int QG, int KG, int KT, int S>
struct Shape {
  static constexpr int qg = QG, kg = KG, kt = KT, s = S, lds = attend_lds<T, HD, QG, KG, KT, S>();
  static_assert(QG * KG == 4 && lds <= 64 * 1024, "four waves, two workgroups a CU");
};
// Tiles of 128 rows; of few rows, where the waves split the keys, each with a stage of
// its own: beside the other workgroup's four waves their loads need no second one.  (Rows
// of 512 bytes: half the keys fit.)  Two workgroups a CU leave a lane 256 registers: float32
// of 128-wide heads spills 108 bytes of them, 112 where the plan is given (16 documents of 32
// queries behind 1024 keys, 32 heads: 135 us, the products 80; 32 tokens behind 2048, 28 + 4
// heads: 53), bf16 that plans for itself 8.
template <typename T, int HD>
struct Shapes {
  static constexpr bool F32 = sizeof(T) == 4, WIDE = F32 && HD == 128;
  typedef Shape<T, HD, 4, 1, F32 ? 32 : 64, F32 && !WIDE ? 4 : 2> Many;
  typedef Shape<T, HD, WIDE ? 2 : 1, WIDE ? 2 : 4, 32, F32 || HD == 128 ? 1 : 2> Few;
  static constexpr int lds = Many::lds > Few::lds ? Many::lds : Few::lds;
};

// SELF: every workgroup plans for itself; else shared_plan_kernel has.
template <typename T, int HD, bool SELF>
__global__ void __launch_bounds__(256, 2) shared_units_kernel(SharedArgs s, SharedPlan p) {
#if defined(__HIP_DEVICE_COMPILE__)
  __shared__ __attribute__((aligned(1024))) char lds[Shapes<T, HD>::lds];
  __shared__ std::conditional_t<SELF, Table, int> table;
  const AttnArgs& a = s.own;
  const int G = a.Hq / a.Hkv;
  const auto& t = table;
  if constexpr (SELF) {
    if (threadIdx.x < 64) plan_docs(s, p, table);
    __syncthreads();
  }
  const uint32_t n = (uint32_t)a.Hkv * (uint32_t)uniform([&] {
    if constexpr (SELF) return t.units;
    else return p.count[0];
  }());
  for (uint32_t u = blockIdx.x; u < n; u += gridDim.x) {
    if (u != blockIdx.x) __syncthreads();  // the last unit's LDS is free
    // (hidden from the compiler, which would keep what is the same for all units in registers)
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    const int wave = uniform(tid >> 6), lane = tid & 63, lq = lane & 31;
    const uint32_t e = u / (uint32_t)a.Hkv, g = u - e * (uint32_t)a.Hkv;
    int who, r0, rows, kb, kend, state0, first, before;  // (see shared_plan_kernel)
    Doc d;
    Keys k;
    if constexpr (SELF) {
      const Split &x = t.of[lane].stack, &y = t.of[lane].own;
      const int l0 = __ffsll(__ballot(e - x.unit < (uint32_t)(x.chunks * x.tiles))) - 1;
      const int l = l0 >= 0 ? l0 : __ffsll(__ballot(e - y.unit < (uint32_t)(y.chunks * y.tiles))) - 1;
      // its numbers, one a lane
      static_assert(sizeof(Segments) == 23 * 4, "Segments is 23 ints");
      const int rec = reinterpret_cast<const int*>(&t.of[l])[min(lane, 22)];
      const int z = l0 >= 0 ? 0 : 6;
      const int i = (int)e - lane_of(rec, z), tiles = lane_of(rec, z + 2), c = (uint32_t)i / (uint32_t)tiles, each = lane_of(rec, z + 5);
      rows = lane_of(rec, z + 3);
      d = Doc{lane_of(rec, 12), lane_of(rec, 13), lane_of(rec, 14), lane_of(rec, 15), lane_of(rec, 16), lane_of(rec, 17)};
      first = lane_of(rec, 18);
      before = lane_of(rec, 21);
      who = l0 >= 0 ? ~lane_of(rec, 19) : l;
      r0 = (i - c * tiles) * tile_rows(p, rows);
      kb = c * each;
      kend = c + 1 < lane_of(rec, z + 4) ? kb + each : l0 >= 0 ? before : 0x7fffffff;
      state0 = lane_of(rec, z + 1) + c * rows * a.Hkv;
      k = who < 0 ? keys_at<T>(s.pk, s.pv, ~who, lane_of(rec, 20), g) : keys_at<T>(a.k, a.v, who, d.k0, g);
    } else {
      const int4 u0 = p.unit[2 * (size_t)e], u1 = p.unit[2 * (size_t)e + 1];
      who = uniform(u0.x);
      r0 = uniform(u0.y);
      rows = uniform(u0.z);
      kb = uniform(u0.w);
      kend = uniform(u1.x);
      state0 = uniform(u1.y);
      first = uniform(u1.z);
      const int pn = who < 0 ? ~who : prompt_of(s, who);
      const Prompt pr = pn >= 0 ? prompt_at(s, pn) : Prompt{0, 0};
      before = uniform(pr.nk);
      if (who >= 0) {
        d = doc_of(a, who);
        d = Doc{uniform(d.q0), uniform(d.nq), uniform(d.k0), uniform(d.nk), uniform(d.pos), uniform(d.prefix)};
      }
      k = who < 0 ? keys_at<T>(s.pk, s.pv, ~who, uniform(pr.k0), g) : keys_at<T>(a.k, a.v, who, d.k0, g);
    }
    auto run = [&](auto shape) {
      typedef decltype(shape) X;
      const int w0 = r0 + 32 * (wave % X::qg), w1 = min(w0 + 32, rows), row = w0 + lq;
      k.kb = kb;
      if (who < 0) {
        k.ke = k.tile_first = kend;
        k.see_first = k.see_last = w0 < rows ? kend : 0;
      } else {
        k.ke = uniform(min(sees(a, d, (min(r0 + 32 * X::qg, rows) - 1) / G), kend));
        if (kb >= k.ke && kb > 0) return;
        k.tile_first = uniform(sees(a, d, r0 / G));
        k.see_first = uniform(w0 < rows ? sees(a, d, w0 / G) : 0);
        k.see_last = uniform(w0 < rows ? sees(a, d, (w1 - 1) / G) : 0);
      }
      auto rows_of = [&](Rows<HD>& R) {
        R.mine = row < rows;
        R.t = R.mine ? row / G : 0;
        R.h = (int)g * G + (R.mine ? row - R.t * G : 0);
        R.slope = 0.f;
        R.at = 0;
        int doc = who, token = d.q0 + R.t, end;
        long i = (long)d.pos + R.t;
        if (who >= 0) {
          end = sees(a, d, R.t);
        } else if constexpr (SELF) {
          doc = t.holder(first + R.t);
          const Doc q = t.of[doc].doc;
          const int x = first + R.t - t.first[doc];
          token = q.q0 + x;
          i = (long)q.pos + x;
          end = sees(a, q, x);
        } else {
          const int4 q = p.tok[3 * (size_t)(first + R.t)];
          doc = q.x;
          token = q.y;
          i = q.z;
          end = q.w;
        }
        R.end = R.mine ? (who < 0 ? k.ke : end) : 0;
        if (a.slopes) {
          if (R.mine) R.slope = a.slopes[R.h] * LOG2E;
          R.at = distances_from(i, before, end, R.slope) + (who < 0 ? before : 0);
        }
        return static_cast<const T*>(a.q.data) + doc * a.q.stride_b + token * a.q.stride_l + R.h * a.q.stride_h;
      };
      const size_t state = (size_t)state0 + (size_t)g * rows;
      attend<T, HD, X::qg, X::kg, X::kt, X::s, false>(
          a, lds, tid, k, k, rows_of, [&](const Rows<HD>& R) { keep_state(R, p.part, p.part_ml, state + (size_t)R.t * G + (R.h - (int)g * G)); });
    };
    if (tile_rows(p, rows) == MANY_ROWS)
      run(typename Shapes<T, HD>::Many{});
    else
      run(typename Shapes<T, HD>::Few{});
  }
  if constexpr (SELF) {
    if (blockIdx.x == 0 && threadIdx.x == 0) p.count[1] = t.queries;
    for (int i = blockIdx.x + threadIdx.x * gridDim.x; i < t.queries; i += 256 * gridDim.x) tell_query(s, p, t, i);
  }
#endif
}

// W > 0: W waves a row (join_row).  W = 0, many rows of few states: HD / 4 lanes a row,
// each 16 bytes of its output, so that twice as many rows are under way.
template <typename T, int HD, int W>
__global__ void __launch_bounds__(256) shared_join_kernel(SharedArgs s, SharedPlan p) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int LPR = HD / 4, SIDE = W ? 1 : 64 / LPR;  // lanes of a row, rows of a wave
  const AttnArgs& a = s.own;
  const int lane = threadIdx.x & 63, e = lane % LPR;
  const uint32_t row = W ? (blockIdx.x * 4u + (threadIdx.x >> 6)) / (W ? W : 1) : (blockIdx.x * 4u + (threadIdx.x >> 6)) * SIDE + lane / LPR;
  const int h = (int)(row % (uint32_t)a.Hq), G = a.Hq / a.Hkv;
  const uint32_t i = row / (uint32_t)a.Hq;
  const size_t i3 = 3 * (size_t)min(i, (uint32_t)p.cap - 1);
  const int4 q = p.tok[i3], own = p.tok[i3 + 1], run = p.tok[i3 + 2];  // (beside the count: of no query, not used)
  const bool there = i < (uint32_t)p.count[1];
  if (W && !there) return;
  const int g = h / G, in = h % G;
  const size_t at_own = (size_t)own.x + (size_t)g * own.y + in, at_run = (size_t)run.x + (size_t)g * run.y + in;
  const size_t next_own = (size_t)own.y * a.Hkv, next_run = (size_t)run.y * a.Hkv;
  const int chunks = run.z, n = there ? chunks + own.z : 0;
  auto at = [&](int c) { return c < chunks ? at_run + c * next_run : at_own + (c - chunks) * next_own; };
  T* const to = static_cast<T*>(a.out.data) + q.x * a.out.stride_b + q.y * a.out.stride_l + h * a.out.stride_h;
  if constexpr (W > 0) {
    join_row<T, HD, W>(to, n, p.part, p.part_ml, at);
  } else {
    constexpr int EARLY = 4;
    const float* part = p.part + e * 4;
    float4 early[EARLY];
#pragma unroll
    for (int c = 0; c < EARLY; ++c) early[c] = c < n ? *reinterpret_cast<const float4*>(part + at(c) * HD) : make_float4(0.f, 0.f, 0.f, 0.f);
    float m = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int c0 = 0; __any(c0 < n); c0 += LPR) {  // LPR states at a time, on the maximum so far
      float2 x = make_float2(-INFINITY, 0.f);
      if (c0 + e < n) x = p.part_ml[at(c0 + e)];
      float top = x.x;
#pragma unroll
      for (int k = LPR / 2; k > 0; k >>= 1) top = fmaxf(top, __shfl_xor(top, k, 64));
      const float m_new = fmaxf(m, top), ref = m_new == -INFINITY ? 0.f : m_new, f0 = exp2_hw(m - ref), f = exp2_hw(x.x - ref);
      m = m_new;
      float sum = x.y * f;
#pragma unroll
      for (int k = LPR / 2; k > 0; k >>= 1) sum += __shfl_xor(sum, k, 64);
      l = l * f0 + sum;
      o.x *= f0;
      o.y *= f0;
      o.z *= f0;
      o.w *= f0;
      auto add = [&](const float4& w, int c) {
        const float fc = __shfl(f, lane - e + c, 64);
        if (c0 + c >= n) return;  // (of a state that is not there, nothing: 0 times infinity)
        o.x += w.x * fc;
        o.y += w.y * fc;
        o.z += w.z * fc;
        o.w += w.w * fc;
      };
      if (c0 == 0) {
#pragma unroll
        for (int c = 0; c < EARLY; ++c) add(early[c], c);
      }
      for (int c = c0 ? 0 : EARLY; c < LPR && __any(c0 + c < n); ++c)
        add(c0 + c < n ? *reinterpret_cast<const float4*>(part + at(c0 + c) * HD) : make_float4(0.f, 0.f, 0.f, 0.f), c);
    }
    if (!there) return;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    if constexpr (sizeof(T) == 2)
      *reinterpret_cast<uint2*>(to + e * 4) = make_uint2(pack2(o.x * inv, o.y * inv), pack2(o.z * inv, o.w * inv));
    else
      *reinterpret_cast<float4*>(to + e * 4) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
  }
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
  // read the same keys, go to one XCD (to p.parts of them where there are too few for
  // eight), the tiles with most keys first
  const int i8 = (int)blockIdx.x >> 3, up = i8 / p.part_tiles * 8 + ((int)blockIdx.x & 7);  // unit and part
  const int unit = up / p.parts, tile = p.tiles - 1 - (i8 % p.part_tiles * p.parts + up % p.parts);
  if (unit >= a.docs * a.Hkv || tile < 0) return;
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
  attend<T, HD, QG, KG, KT, S, true>(a, lds, threadIdx.x, k1, k2, rows_of, [&](const Rows<HD>& R) {
    store_row(R, static_cast<T*>(a.out.data) + dn * a.out.stride_b + (long)(d.q0 + R.t) * a.out.stride_l + R.h * a.out.stride_h);
  });
#endif
}

// ---- choice, from sizes only ------------------------------------------------------
// What a call takes in microseconds, fitted to 288 calls of 1 to 64 rows a document, 1 to
// 48 documents and 64 to 1000 keys, timed in each form: alone on a CU a row tile takes `base`
// and `step` for each of its steps of `keys`, its steps over a prompt and its own keys one
// after the other; a unit takes a start beside its steps.  The form taken is 1 % off the
// best of four on average, units alone 25 %.  (bf16, 32 heads: 16 documents of 64 queries behind
// 60 keys: 13 us, units 47; 4 single tokens behind 800 and 200: units 16, chain 20.  28 + 4: 3 of
// 294 behind 64: 18, units 37.  float32, 28 + 4, 16 of 28 rows behind 400 and 100: units 29, chain 53.)
struct Shaped {
  int qg, keys;
  float base, step;
};
// Row tiles that take prompt and own keys in one go, of 32, 64 and 128 rows: however few
// there are, each takes its steps.
constexpr Shaped CHAINS[2][2][3] = {{{{1, 128, 5.8f, 0.93f}, {2, 128, 7.f, 0.95f}, {4, 64, 5.5f, 0.96f}},
                                     {{1, 128, 7.9f, 1.33f}, {2, 128, 9.7f, 1.33f}, {4, 64, 6.8f, 1.32f}}},
                                    {{{1, 128, 8.f, 2.6f}, {2, 128, 8.5f, 4.5f}, {4, 32, 10.f, 2.27f}},
                                     {{1, 64, 11.7f, 4.85f}, {2, 64, 11.7f, 4.75f}, {4, 32, 15.f, 4.1f}}}};  // [f32][hd 128]
// How a call's units, (document, key/value head), of `tiles` row tiles are dealt to XCDs.
struct Dealt {
  int tiles, parts, part_tiles;  // a unit's tiles, the parts that it is dealt in, tiles of one
  long per_xcd;
};
Dealt deal(const SharedArgs& s, int qg) {
  const long units = (long)s.own.docs * s.own.Hkv;
  Dealt d{ceil_div((long)s.own.max_q * (s.own.Hq / s.own.Hkv), 32 * qg), 1, 0, 0};
  while (d.parts < (units >= 512 ? 1 : units >= 64 ? 2 : 8) && 2 * d.parts <= d.tiles && units * d.parts % 8) d.parts *= 2;
  d.part_tiles = ceil_div(d.tiles, d.parts);
  d.per_xcd = (long)ceil_div(units * d.parts, 8) * d.part_tiles;
  return d;
}
float time_of_chain(const SharedArgs& s, const Shaped& x, bool f32) {
  const AttnArgs& a = s.own;
  const long tiles = deal(s, x.qg).per_xcd, cus = std::max(1, device_cu_count() / 8);
  const bool pairs = !f32 && x.qg == 4;  // two workgroups a CU, which then slow each other
  const int rounds = ceil_div(tiles, pairs ? 2 * cus : cus);
  float own = (float)ceil_div(a.max_kv, x.keys);
  if (a.block > 0 && a.max_q <= a.max_kv && rounds > 1) own *= 1.f - 0.5f * (float)a.max_q / (float)a.max_kv;  // what a mean row sees
  return 1.5f + (float)rounds * (x.base + (pairs && tiles > cus ? 1.27f : 1.f) * x.step * ((float)ceil_div(s.max_p, x.keys) + own));
}
// Units and their join.  (Stacks as if documents were told apart by prompt also where the array
// of them is not given and all stand behind prompt 0: the choice decides the workspace's size,
// which must not depend on the arrays.  Several prompts and no array: on the chain's side.)
float time_of_units(const SharedArgs& s, const SharedPlan& p, bool f32) {
  const AttnArgs& a = s.own;
  const bool wide = a.hd == 128;
  const int rows = a.max_q * (a.Hq / a.Hkv);
  const double all = (double)a.docs * rows, own = (double)a.docs * tiles_of(p, rows);
  const double stacks = std::max(all > 64 ? all / MANY_ROWS : all / p.few_rows, (double)std::min(a.docs, s.prompts));
  // a tile's p.unit_keys keys, of few and of many rows
  const float few = f32 ? wide ? 2.4f : 0.65f : wide ? 1.33f : 0.93f, many = f32 ? wide ? 4.1f : 2.27f : wide ? 4.3f : 2.4f;
  const float own_each = rows > 64 ? many : few, stack_each = all > 64 ? many : few;
  const double work = own * ceil_div(a.max_kv, p.unit_keys) * own_each + stacks * ceil_div(s.max_p, p.unit_keys) * stack_each;
  const float fixed = f32 ? wide ? 15.5f : 9.f : wide ? 9.5f : 7.5f, start = f32 ? 6.f : 4.5f, unit = f32 ? wide ? 16.f : 10.f : 9.f;
  const double share = a.Hkv * (work + unit * (own + stacks)) / ((f32 ? 1.0 : 1.67) * device_cu_count());
  return fixed + std::max(start + std::max(own_each, stack_each), (float)share) + 2e-4f * (float)(all * a.Hkv);
}
// The row groups of a tile that takes all keys of its rows, 0: units.
int chain_of(const SharedArgs& s, const SharedPlan& p) {
  const bool f32 = s.own.dtype == DLLM_F32;
  float best = time_of_units(s, p, f32);
  int qg = 0;
  for (const Shaped& x : CHAINS[f32][s.own.hd == 128]) {
    const float t = time_of_chain(s, x, f32);
    if (t <= best) {
      best = t;
      qg = x.qg;
    }
  }
  return qg;
}
SharedPlan choose(const SharedArgs& s) {
  const AttnArgs& a = s.own;
  SharedPlan p{};
  const int G = a.Hq / a.Hkv, rows = a.max_q * G, cus = device_cu_count();
  const bool f32 = a.dtype == DLLM_F32;
  p.slots = 2 * cus;
  p.busy = f32 ? cus : p.slots;
  // (bf16, 16 documents of 32 queries behind 1024 and 8448 keys, 32 heads: 43 and 105 us; a cost
  // of 1 to 3: 45 and 108; 64 keys and 8 are as fast there, but slower where keys are few: 4 documents
  // of 32 queries behind 656, 28 + 4 heads, 21.5 and 24.1.  float32, whose step takes five
  // times as long, 2 documents of 50 behind 143: 20.9 us, by 64 keys 25.7, by 128 35.1; 2 of 195
  // behind 85, 32 heads, which is more than half a round: 44.8, by a CU each 49.7)
  p.unit_keys = f32 ? 32 : 128;
  p.unit_cost = f32 ? 1 : 4;
  p.few_rows = f32 && a.hd == 128 ? 64 : 32;
  p.chain = chain_of(s, p);
  if (p.chain) {
    const Dealt d = deal(s, p.chain);
    p.tiles = d.tiles;
    p.parts = d.parts;
    p.part_tiles = d.part_tiles;
    p.grid = 8 * d.per_xcd;
    return p;
  }
  const long packed = a.out.stride_b == 0 ? a.q_tokens : (long)a.docs * a.max_q;
  p.cap = (int)std::min(std::min((long)a.docs * a.max_q, packed), 0x7fffffffl);
  // units without a split: of the runs (as many as documents, but where prompts' documents
  // follow each other no more than those) and of the documents
  const long whole = ((long)p.cap * G + MANY_ROWS - 1) / MANY_ROWS;
  const long own = std::min((long)a.docs * std::max(tiles_of(p, std::min(rows, 64)), tiles_of(p, rows)), whole + 2l * a.docs);
  const long base = whole + 2l * a.docs + own, keys = ceil_div(std::max(s.max_p, a.max_kv), p.unit_keys);
  // (cut_of: chunks beyond the first are fewer than 4/3 of the workgroups that run at once)
  const long more = std::min(2l * p.slots / a.Hkv + 1, base * (keys - 1));
  p.units = base + more;
  p.work = base * keys;
  const long expected = (whole + (s.prompt ? std::min(a.docs, s.prompts) : 1) + own) * a.Hkv;
  p.grid = std::min((expected + p.slots - 1) / p.slots * p.slots, 1l << 22);
  p.states = 2l * p.cap * a.Hq + more * a.Hkv * MANY_ROWS;
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
    constexpr int KG = F32 && HD == 128 ? 2 : 4;
    if (p.chain == 1)
      shared_chain_kernel<T, HD, 1, KG, 32, 2><<<(unsigned)p.grid, 64 * KG, 0, st>>>(s, p);
    else if (p.chain == 2)
      shared_chain_kernel<T, HD, 2, KG, 32, 2><<<(unsigned)p.grid, 128 * KG, 0, st>>>(s, p);
    else if constexpr (F32)
      shared_chain_kernel<T, HD, 4, 1, 32, 3><<<(unsigned)p.grid, 256, 0, st>>>(s, p);
    else
      shared_chain_kernel<T, HD, 4, 1, 64, 2><<<(unsigned)p.grid, 256, 0, st>>>(s, p);
    DLLM_LAUNCH_CHECK("shared_chain_kernel");
    return;
  }
  const int docs = s.own.docs;
  if (docs <= 64) {
    shared_units_kernel<T, HD, true><<<(unsigned)p.grid, 256, 0, st>>>(s, p);
  } else {
    shared_plan_kernel<<<1, docs <= 256 ? 256 : PLAN_THREADS, 0, st>>>(s, p);
    DLLM_LAUNCH_CHECK("shared_plan_kernel");
    shared_units_kernel<T, HD, false><<<(unsigned)p.grid, 256, 0, st>>>(s, p);
  }
  DLLM_LAUNCH_CHECK("shared_units_kernel");
  // Waves a row by how many rows there are (and the more rows, the fewer chunks each):
  // four up to four rows a CU, one up to 32 (1232 rows of up to 20 states: 3.9 us, HD / 4
  // lanes a row 10.2), above that HD / 4 lanes (16384 rows of 2 states: 6.3 us, a wave 8.8).
  const long rows = (long)p.cap * s.own.Hq, cus = device_cu_count();
  if (rows <= 4 * cus)
    shared_join_kernel<T, HD, 4><<<(unsigned)rows, 256, 0, st>>>(s, p);
  else if (rows <= 32 * cus)
    shared_join_kernel<T, HD, 1><<<ceil_div(rows, 4), 256, 0, st>>>(s, p);
  else
    shared_join_kernel<T, HD, 0><<<ceil_div(rows, 4 * (256 / HD)), 256, 0, st>>>(s, p);
  DLLM_LAUNCH_CHECK("shared_join_kernel");
}

// Without a prompt's key it is attention of documents.
bool alone(const SharedArgs& s) { return s.prompts == 0 || s.max_p == 0; }

}  // namespace

// (As without a block mask, which a query of the size may not know: with one a chain is never
// slower, so that a call that takes units takes them without it too, laid out alike.)
size_t attn_shared_bytes(const SharedArgs& of) {
  if (alone(of)) return attn_docs_bytes(of.own);
  SharedArgs s = of;
  s.own.block = 0;
  SharedPlan p = choose(s);
  return p.chain ? 0 : lay_out(s, p, nullptr);
}

// A launch's threads must be below 2^32, and states countable.
bool attn_shared_fits(const SharedArgs& s) {
  if (alone(s)) return attn_docs_fits(s.own);
  const SharedPlan p = choose(s);
  if (p.chain) return p.grid * 512 < (1l << 32);  // (at most eight waves)
  return p.states < (1l << 31) && p.units * s.own.Hkv < (1l << 31) && p.work < (1l << 30) && (long)p.cap * s.own.Hq < (1l << 26);
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
