// The statements of a row tile (attn_tile.h), for a function that has T, HD, QG, KG, KT, S, CHAIN,
// a, lds, lane, wave, qg, kg, lq, half, k1, k2 and rows_of under these names: attend, and
// attn_docs_kernel itself.  There they stand as statements because the compiler, which
// inlines either way, lays out the code of an inlined function otherwise, and that runs
// longer (captured calls, 32 queries x 1024 keys x 32 heads x 8: 26.5 us, as a function 27.6;
// one token of 16 documents: 38.6 and 39.2) and contracts other products into
// multiply-adds.  They leave in R the states of the rows, in the waves of key group 0; the
// others' have returned.
  typedef Tile<T, HD> TL;
  constexpr bool BF = sizeof(T) == 2;
  constexpr int ND = HD / 32;
  constexpr int K_BYTES = KT * TL::ROW, TILE = 2 * K_BYTES, STAGE = KG * TILE;
  constexpr int TP = TILE / 1024, PER = TP / QG;  // LDS-DMA instructions of 1 KiB: of a tile, of a wave
  static_assert(TP % (2 * QG) == 0, "the waves of a key group share a tile's loads evenly");
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

  // The waves of a key group load its tile: wave qg the parts qg, qg + QG, ..,
  // K's before V's; a part is 1 KiB of whole rows, lane l filling slot l % CH
  // of row l / CH
  constexpr int RPP = 1024 / TL::ROW;  // rows of a part
  uint32_t off[PER], off2[CHAIN ? PER : 1];
#pragma unroll
  for (int x = 0; x < PER; ++x) {
    const bool isk = x < PER / 2;
    const int r = (qg + QG * (x % (PER / 2))) * RPP + lane / TL::CH;
    const int c = (lane % TL::CH) ^ (isk ? TL::k_swz(r) : TL::v_swz(r));
    off[x] = r * (isk ? k1.ksb : k1.vsb) + c * 16;
    if constexpr (CHAIN) off2[x] = r * (isk ? k2.ksb : k2.vsb) + c * 16;
  }
  const uint32_t lds0 = lds_address(lds) + kg * TILE + qg * 1024;
  const int n1 = k1.steps(KG * KT), nsteps = CHAIN ? n1 + k2.steps(KG * KT) : n1;
  auto load = [&](int u, int slot) {  // step u into stage `slot`
    const bool next = CHAIN && u >= n1;
    const int t0 = next ? k2.kb + ((u - n1) * KG + kg) * KT : k1.kb + (u * KG + kg) * KT;
    const int left = min((next ? k2.ke : k1.ke) - t0, KT);  // reads past the last key give zeros
#pragma unroll
    for (const bool keys : {true, false}) {
      const uint32_t sb = next ? (keys ? k2.ksb : k2.vsb) : keys ? k1.ksb : k1.vsb, bytes = left > 0 ? (uint32_t)(left - 1) * sb + TL::ROW : 0u;
      const rsrc_t rs = rsrc_of((next ? (keys ? k2.kp : k2.vp) : keys ? k1.kp : k1.vp) + (left > 0 ? (long)t0 : 0l) * sb, bytes);
      const uint32_t to = lds0 + slot * STAGE + (keys ? 0 : K_BYTES);
#pragma unroll
      for (int x = 0; x < PER / 2; ++x) dma16(rs, CHAIN && next ? off2[keys ? x : PER / 2 + x] : off[keys ? x : PER / 2 + x], to + x * QG * 1024);
    }
  };
  constexpr int D = S > 1 ? S - 1 : 1;  // stages in flight behind the one in use (of a single stage, before it)
  for (int u = 0; u < D && u < nsteps; ++u) load(u, u);

  // Q operand: the lane's rows, dims 16 ks + 8 half .. (bf16), 8 c + 4 half .. (float32)
  constexpr int NQ = BF ? HD / 16 : HD / 8;
  typedef float f32x4v __attribute__((ext_vector_type(4)));
  bf16x8_t qb[BF ? NQ : 1];
  f32x4v qf[BF ? 1 : NQ];
  Rows<HD> R;
  const T* qrow = rows_of(R);
  R.m = -INFINITY;
  R.m_ref = 0.f;
  R.l = 0.f;
#pragma unroll
  for (int ds = 0; ds < ND; ++ds)
#pragma unroll
    for (int r = 0; r < 16; ++r) R.o[ds][r] = 0.f;
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

  // keys that the lane's row sees, of k1 where a chain is at its first keys
  auto limit = [&](bool first) { return CHAIN ? (first ? k1.ke : min(R.end, k2.ke)) : min(R.end, k1.ke); };
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
  auto shape = [&](f32x16_t (&x)[NS], int t0, bool first, bool whole) {
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
      const float at = (float)((CHAIN && first ? R.at + k1.ke : R.at) - t0 - 4 * half);
#pragma unroll
      for (int b = 0; b < NS; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) x[b][r] = fmaf(-R.slope, fabsf(at - (float)(32 * b + 8 * (r >> 2) + (r & 3))), x[b][r]);
    }
    const int end = limit(first) - t0 - 4 * half;
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
  auto scrub = [&](int t0, bool first, char* vt) {
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
          if (t0 + key < limit(first) && !(fabsf(f) < INFINITY)) R.o[ds][r] += f;
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
  for (int u = 0; __builtin_expect(u < nsteps, 1); ++u) {
    if constexpr (S == 1) {
      if (u > 0) {
        if constexpr (QG > 1) barrier_nofence();
        load(u, 0);
      }
    }
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
    if (S > 1 && u + D < nsteps) load(u + D, (u + D) % S);
    const bool next = CHAIN && u >= n1;
    const int kb = next ? k2.kb : k1.kb, ke = next ? k2.ke : k1.ke, tile_first = next ? k2.tile_first : k1.tile_first;
    const int see_first = next ? k2.see_first : k1.see_first, see_last = next ? k2.see_last : k1.see_last;
    const int t1 = kb + (u - (next ? n1 : 0)) * KG * KT, t0 = t1 + kg * KT;
    char *const slot = lds + (u % S) * STAGE + kg * TILE, *const vt = slot + K_BYTES;
    if (t1 + KG * KT > tile_first) scrub(t0, !next, vt);
    if (t0 >= min(ke, see_last)) continue;  // nothing that this wave's rows see
    f32x16_t x[NS];
    uint32_t pw[BF ? NS * 8 : 1];
    scores(slot, x);
    const bool whole = t0 + KT <= min(ke, see_first);
    float mt, fold = 1.f;  // fold: factor still to be applied in the exponent
    if (direct && whole) {
      fold = sc;
      mt = highest(x) * sc;
    } else {
      mt = shape(x, t0, !next, whole);
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
