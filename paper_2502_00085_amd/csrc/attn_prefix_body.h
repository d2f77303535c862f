// The body of a workgroup of the bf16 pass over the shared prefix: of the function prefix_wg (attn_prefix_wg.h, which says
// what its names are), and of k_attn_prefix itself where the launch has no other workgroups.  As an inlined function
// the compiler simplifies it before and after it has its place; the causal pass then takes 0.4 to 1 % longer
// (2,048 tokens from position 6,144, 2 layers: 487 us in the kernel, 490 as a function; the pass beside the tries' nodes 91.2 and
// 89.7).  Uses D, RW, KW, WGS, FOUR; s, a; kbuf0, vbuf0, kbuf1, vbuf1, wred, ml.
  using C = PrefixCfg<D, RW, KW>;
  static_assert(2 * C::LOADS < 64, "the wait counter holds a tile's loads");
  static_assert(KW == 1 || KW == 2, "one or two groups: the RW KW waves have a word each of wred");
  constexpr int NH = 2 / KW;  // 32-key halves of a tile per wave
  constexpr bool TRIES = WGS != Wgs::kPrefix;
  using T4 = Tile4<D, C::THREADS, 64>;
  PrefixHdr p = s.prefix[FOUR ? 1 : 0];
  const bool trie = WGS == Wgs::kTries || (WGS == Wgs::kBoth && blockIdx.x >= a.prefix_wgs);
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rw = wave % RW, kw = wave / RW;
  const int col = lane & 31, hh = lane >> 5;

  PrefixUnit u;
  PrefixRow q;
  TrieHdr th{};
  int t = 0, r0, share, shares;  // (of the keys)
  if (TRIES && trie) {
    int x = blockIdx.x - a.prefix_wgs;
    shares = a.trie_splits;
    share = x % shares;
    x /= shares;
    u.rb = x % a.trie_blocks;
    x /= a.trie_blocks;
    u.g = x % s.Hkv;
    x /= s.Hkv;
    t = x % a.tries;
    u.li = x / a.tries;
    u.split = a.splits + share;
    th = s.hdr[t];
    r0 = u.rb * RW * 32;
    const int G = s.Hq / s.Hkv, r = r0 + rw * 32 + col, i = r / G;
    q.in = i < a.per_trie;
    q.t = t;
    q.j = q.in ? i : 0;
    q.head = r % G;
    q.owner = t * a.per_trie + q.j;
    q.at = ((size_t)u.li * a.tries + t) * a.q_stride + q.j;
    q.lo = q.hi = 0;
  } else {
    u = prefix_unit(s, a);
    share = u.split;
    shares = a.splits;
    r0 = u.rb * RW * 32;
    q = prefix_row(s, a, u.li, r0 + rw * 32 + col);
  }
  const int lab = a.layer_begin + u.li;
  // the lane's query row as B operands of S^T: half hh of its d range (loaded before anything is known
  // of the row; a row that sees nothing has no say)
  bf16x8 qv[C::KSTEPS];
  {
    const uint4* qp = reinterpret_cast<const uint4*>(static_cast<const __bf16*>(a.q) +
                                                     (q.at * s.Hq + u.g * (s.Hq / s.Hkv) + q.head) * D + hh * (D / 2));
#pragma unroll
    for (int k = 0; k < C::KSTEPS; ++k) qv[k] = __builtin_bit_cast(bf16x8, qp[k]);
  }
  PrefixSpan span, all;  // (of the wave; of the WG)
  bool known = true;
  if (TRIES && trie) {
    const int lo = window_lo(s, t, th.base, th.n_nodes, th.leaf_depth, wred);  // (a word per wave)
    __syncthreads();
    const int shared = max(lo, min(th.n_shared, th.n_nodes));
    all = {lo, th.n_nodes, lo, shared};
  } else {
    known = prefix_range(s, a, p, r0, RW * 32, &all);
  }
  if (!known) {  // a window: from the rows' positions
    prefix_row_keys(s, a, p, q);
    span = prefix_span(q);
    all = prefix_range_of<RW>(span, rw, lane == 0 && kw == 0, wred);
  }
  const int lo = all.lo, hi = all.hi;
  // tiles of 64 keys, at multiples of 64: this split's share
  constexpr bool four = FOUR;
  static_assert(!FOUR || WGS == Wgs::kPrefix, "the tries' nodes are never in 4 bits");
  const int first = hi > 0 ? lo / 64 : 0, tiles = hi > 0 ? (hi + 63) / 64 - first : 0;
  const int per = (tiles + shares - 1) / shares;
  const int t0 = first + share * per, t1 = max(t0, min(first + tiles, t0 + per));
  // of it [m0, m1): tiles that every row sees whole; the cut ones before and after
  const int m0 = min(max(t0, (all.all_lo + 63) / 64), t1), m1 = max(m0, min(t1, all.all_hi / 64));
  const int before = m0 - t0, cut = before + t1 - m1;
  auto cut_tile = [&](int i) __attribute__((always_inline)) { return i < before ? t0 + i : m1 + i - before; };

  size_t head = ((size_t)lab * s.Hkv + u.g) << p.shift;  // rows before this (layer, KV head) in a page
  size_t page_rows = ((size_t)s.L * s.Hkv) << p.shift;
  const __bf16* kpages = static_cast<const __bf16*>(p.k);
  const __bf16* vpages = static_cast<const __bf16*>(p.v);
  if (TRIES && trie) {  // (one page)
    p.shift = 30;
    head = pool_row(s, t, lab, u.g, th.base) / D;
    page_rows = 0;
    kpages = static_cast<const __bf16*>(s.k_pool);
    vpages = static_cast<const __bf16*>(s.v_pool);
  }
  auto pages_of = [&](int tile) __attribute__((always_inline)) { return TRIES && trie ? TilePages{} : tile_pages(p, tile); };

  // Load j of this thread writes 16-byte LDS chunk c = j THREADS + tid of the tile's K (and V): tile
  // row c / CPR at physical chunk c % CPR; K rows rotated by one chunk per row, V rows by one 64-byte
  // block per row.  kofs / vofs: byte offset, in 64 consecutive rows, of the logical chunk it loads.
  uint32_t kofs[C::OFS], vofs[C::OFS];
#pragma unroll
  for (int j = 0; j < C::OFS; ++j) {
    const int c = j * C::THREADS + tid, row = c / C::CPR, pc = c % C::CPR;
    kofs[j] = row * (2 * D) + (pc + C::CPR - row % 32 % C::CPR) % C::CPR * 16;
    vofs[j] = row * (2 * D) + v_logical<C::CPR, C::NBLK, FOUR>(row % 32, pc) * 16;
  }
  auto issue = [&](int tile, const TilePages& pg, unsigned char* kdst, unsigned char* vdst) __attribute__((always_inline)) {
    const int tb = tile * 64;
    const bool one = p.shift >= 6, full = tb + 64 <= hi;  // (uniform) one page; no row past the end
    const size_t row0 = (size_t)pg.p[0] * page_rows + head + (one ? tb & ((1 << p.shift) - 1) : 0);
    const unsigned char* kt = reinterpret_cast<const unsigned char*>(kpages + row0 * D);
    const unsigned char* vt = reinterpret_cast<const unsigned char*>(vpages + row0 * D);
    const int last = hi - 1 - tb;  // (rows past the end: the last row)
#pragma unroll
    for (int j = 0; j < C::LOADS; ++j) {
      const uint32_t step = C::ONE_OFS ? j * (C::THREADS / C::CPR) * 2 * D : 0;
      uint32_t ko = kofs[C::ONE_OFS ? 0 : j], vo = vofs[C::ONE_OFS ? 0 : j];
      const unsigned char *ks = kt + step, *vs = vt + step;
      if (!one || !full) {
        const int row0j = (int)((ko + step) / (2 * D)), row = min(row0j, last);
        const uint32_t kc = ko + step - row0j * (2 * D), vc = vo + step - row0j * (2 * D);
        if (one) {
          ks = kt;
          vs = vt;
          ko = row * (2 * D) + kc;
          vo = row * (2 * D) + vc;
        } else {
          const int e = row >> p.shift;
          const int page = e == 0 ? pg.p[0] : e == 1 ? pg.p[1] : e == 2 ? pg.p[2] : pg.p[3];
          const size_t r = (size_t)page * page_rows + head + (row & ((1 << p.shift) - 1));
          ks = reinterpret_cast<const unsigned char*>(kpages + r * D);
          vs = reinterpret_cast<const unsigned char*>(vpages + r * D);
          ko = kc;
          vo = vc;
        }
      }
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(ks + ko),
                                       (__attribute__((address_space(3))) void*)(kdst + (j * C::THREADS + wave * 64) * 16), 16, 0, 0);
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(vs + vo),
                                       (__attribute__((address_space(3))) void*)(vdst + (j * C::THREADS + wave * 64) * 16), 16, 0, 0);
    }
  };

  // (4 bits) the tile's blocks of this thread, and the same unpacked into its rows in LDS
  auto fetch = [&](int tile, const TilePages& pg, T4& to) __attribute__((always_inline)) {
    fetch4<D, C::THREADS, 64>(p, pg, page_rows, head, tile * 64, hi - 1 - tile * 64, wave, to);
  };
  auto unpack = [&](const T4& from, unsigned char* kdst, unsigned char* vdst) __attribute__((always_inline)) {
    using B = Blocks4<D, C::THREADS, 64>;
#pragma unroll
    for (int j = 0; j < B::PER; ++j) {
      if (!B::some(j, wave)) continue;
      const bool v = B::is_v(j, wave);
      const int b = B::number(j, v), row = b / B::BPR, blk = b % B::BPR;
      const float unit = __uint_as_float(from.scale[j] << 23);
      unsigned char* const dst = (v ? vdst : kdst) + row * (2 * D);
      const int k0 = (4 * blk + row % 32) % C::CPR, v0 = (blk + row % 32 % C::NBLK) % C::NBLK * 4;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const uint32_t w = from.x[j][c];
        bf16x8 y;
#define CVT4(I) \
  { \
    const bf16x2 z = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, I); \
    y[2 * I] = z[0]; \
    y[2 * I + 1] = z[1]; \
  }
        CVT4(0) CVT4(1) CVT4(2) CVT4(3)
#undef CVT4
        const int at = v ? v0 + ((c + row) & 3) : k0 + c < C::CPR ? k0 + c : k0 + c - C::CPR;
        *reinterpret_cast<bf16x8*>(dst + at * 16) = y;
      }
    }
  };

  // the first two tiles go out before anything that waits for the tries
  TilePages next{};
  T4 ahead, ahead2;  // (4 bits) tiles under way
  if (t0 < t1) {
    const bool main = m0 < m1;
    const int x0 = main ? m0 : cut_tile(0), x1 = main ? m0 + 1 : cut_tile(1);
    const bool two = main ? m0 + 1 < m1 : cut > 1;
    const TilePages pg0 = pages_of(x0), pg1 = pages_of(two ? x1 : x0);
    if constexpr (four) {
      fetch(x0, pg0, ahead);
      fetch(two ? x1 : x0, pg1, ahead2);
    } else {
      issue(x0, pg0, kbuf0, vbuf0);
      if (two) issue(x1, pg1, kbuf1, vbuf1);
    }
    if (m0 + 2 < m1) next = pages_of(m0 + 2);
  }
  prefix_other_kind(s, p);
  if (TRIES && trie) {
    if (q.in && q.j < th.n_live) {
      q.lo = all.lo;
      q.hi = all.hi;
    }
    span = prefix_span(q);
    span.all_hi = min(span.all_hi, all.all_hi);
  } else if (known) {
    prefix_row_keys(s, a, p, q);
    span = prefix_span(q);
  }
  const int grp = lane >> 4, tm = (lane & 15) >> 2, tq = lane & 3;
  int kread[C::KSTEPS], vread[C::VROT][C::DT];
#pragma unroll
  for (int k = 0; k < C::KSTEPS; ++k) kread[k] = col * (2 * D) + (hh * (C::CPR / 2) + col + k) % C::CPR * 16;
#pragma unroll
  for (int x8 = 0; x8 < C::VROT; ++x8)
#pragma unroll
    for (int dt = 0; dt < C::DT; ++dt) {
      const int n = 8 * x8 + 4 * hh + tm;
      const int c = 4 * dt + 2 * (grp & 1) + (tq >> 1);
      vread[x8][dt] = (4 * hh + tm) * (2 * D) + v_chunk<C::CPR, C::NBLK, FOUR>(n, c) * 16 + 8 * (tq & 1);
    }

  const float scale = a.scale_log2;
  float m = kPrefixNegBig, lsum = 0.0f;
  f32x16 o[C::DT];
#pragma unroll
  for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[dt][v] = 0.0f;

  // (4 bits) no row of the WG is a query's: its records say so, and nothing is multiplied.  4 ragged prompts of up
  // to 512 tokens over 4,096 positions, 2 layers: 337 -> 326 us.
  if (four && known && a.rows == PrefixRows::kNodes) {
    if (lane == 0) wred[wave] = span.hi;
    __syncthreads();
    int most = 0;
#pragma unroll
    for (int i = 0; i < RW * KW; ++i) most = max(most, wred[i]);
    if (__builtin_amdgcn_readfirstlane(most) == 0) {
      unsigned char* const mine = rw == 0 ? kbuf0 : rw == 1 ? vbuf0 : rw == 2 ? kbuf1 : vbuf1;
      if (kw == 0) prefix_output<__bf16, D>(s, a, u, q, lane, m, lsum, o, reinterpret_cast<float*>(mine));
      return;
    }
  }

  // V^T of 16 keys and 32 elements of d: this lane's column of d = 32 dt + col
  auto vop = [&](const unsigned char* vh, int uu, int dt) __attribute__((always_inline)) {
    const unsigned char* vp = vh + 16 * uu * (2 * D);
    const i16x4 p0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(vp + vread[2 * uu % C::VROT][dt]));
    const i16x4 p1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(vp + 8 * (2 * D) + vread[(2 * uu + 1) % C::VROT][dt]));
    return __builtin_shufflevector(p0, p1, 0, 1, 2, 3, 4, 5, 6, 7);
  };

  const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
  // Probabilities of this lane's 16 keys relative to the row's shift m, rounded to bf16 (the operand
  // type of the second product; the sum takes the rounded ones, so that an error of a weight is in
  // numerator and denominator alike), and their sum.  Softmax does not depend on the shift: it moves
  // only when the probabilities leave their range, which their sum tells.
  auto weigh = [&](const f32x16& acc, bf16x8 (&pb)[2]) __attribute__((always_inline)) {
    float ps = 0.0f;
    auto weights = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int v = 0; v < 16; ++v) pb[v >> 3][v & 7] = (__bf16)__builtin_amdgcn_exp2f(__builtin_fmaf(acc[v], scale, -m));
      ps = 0.0f;
#pragma unroll
      for (int v = 0; v < 16; v += 2) {
        const bf16x2 pair = {pb[v >> 3][v & 7], pb[v >> 3][(v & 7) + 1]};
        ps = __builtin_amdgcn_fdot2_f32_bf16(pair, ones, ps, false);
      }
    };
    weights();
    if (__any(ps > kMost)) {
      float tmax = acc[0];
#pragma unroll
      for (int v = 1; v < 16; ++v) tmax = fmaxf(tmax, acc[v]);
      tmax = fmaxf(tmax, __shfl_xor(tmax, 32)) * scale;
      const float mn = tmax > m + kSlack ? tmax : m;
      const float alpha = __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      lsum *= alpha;
#pragma unroll
      for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[dt][v] *= alpha;
      weights();
    }
    lsum += ps;
  };
  auto add_values = [&](const unsigned char* vh, const bf16x8 (&pb)[2]) __attribute__((always_inline)) {
#pragma unroll
    for (int uu = 0; uu < 2; ++uu)
#pragma unroll
      for (int dt = 0; dt < C::DT; ++dt)
        o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vop(vh, uu, dt)), pb[uu], o[dt], 0, 0, 0);
  };
  auto step = [&](int tile, const unsigned char* kb, const unsigned char* vb, unsigned char* knext,
                  unsigned char* vnext) __attribute__((always_inline)) {
    if constexpr (four) {
      // the tile is unpacked, and the other buffer is free: the next one goes there
      __syncthreads();
      if (tile + 1 < m1) {
        unpack(ahead, knext, vnext);
        if (tile + 2 < m1) {
          fetch(tile + 2, next, ahead);
          if (tile + 3 < m1) next = pages_of(tile + 3);
        }
      }
    } else {
      // this thread's loads of the tile have landed, then every thread's, and the other buffer is free
      // (the second tile is on its way already)
      if (tile == m0 && m0 + 1 < m1) __builtin_amdgcn_s_waitcnt(wait_vm(2 * C::LOADS));
      else __builtin_amdgcn_s_waitcnt(kWaitVmAll);
      __syncthreads();
      if (tile > m0 && tile + 1 < m1) {
        issue(tile + 1, next, knext, vnext);
        if (tile + 2 < m1) next = pages_of(tile + 2);
      }
    }
    f32x16 acc[NH];
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[h][v] = 0.0f;
#pragma unroll
    for (int k = 0; k < C::KSTEPS; ++k)
#pragma unroll
      for (int h = 0; h < NH; ++h)
        acc[h] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            *reinterpret_cast<const bf16x8*>(kb + (KW == 2 ? kw : h) * C::HALF + kread[k]), qv[k], acc[h], 0, 0, 0);
#pragma unroll
    for (int h = 0; h < NH; ++h) {
      bf16x8 pb[2];
      weigh(acc[h], pb);
      add_values(vb + (KW == 2 ? kw : h) * C::HALF, pb);
    }
  };
  if constexpr (four) {
    // (the queries are there too: else the loop would wait for them, and with them for the tiles under way,
    // each time it multiplies)
    __builtin_amdgcn_s_waitcnt(kWaitVmAll);
    if (m0 < m1) {
      unpack(ahead, kbuf0, vbuf0);
      ahead = ahead2;
    }
  }
  for (int t = m0; t < m1; t += 2) {
    step(t, kbuf0, vbuf0, kbuf1, vbuf1);
    if (t + 1 < m1) step(t + 1, kbuf1, vbuf1, kbuf0, vbuf0);
  }

  // the cut tiles, two at a time: the ends of the rows' ranges
  for (int i = 0; i < cut; i += 2) {
    if (i > 0 || m0 < m1) {
      const bool two = i + 1 < cut;
      const TilePages pg0 = pages_of(cut_tile(i)), pg1 = pages_of(cut_tile(two ? i + 1 : i));
      __syncthreads();  // both buffers are free
      if constexpr (four) {
        fetch(cut_tile(i), pg0, ahead);
        fetch(cut_tile(two ? i + 1 : i), pg1, ahead2);
      } else {
        issue(cut_tile(i), pg0, kbuf0, vbuf0);
        if (two) issue(cut_tile(i + 1), pg1, kbuf1, vbuf1);
      }
    }
    if constexpr (four) {
      unpack(ahead, kbuf0, vbuf0);
      unpack(ahead2, kbuf1, vbuf1);
    }
    uint64_t masks[2] = {0, 0};  // (of a trie's nodes) of key `lane` of either tile
    if (TRIES && trie) {
      const uint64_t* mp = s.mask + (size_t)t * s.cap + th.base;
      masks[0] = mp[min(cut_tile(i) * 64 + lane, hi - 1)];
      masks[1] = mp[min(cut_tile(min(i + 1, cut - 1)) * 64 + lane, hi - 1)];
    }
    __builtin_amdgcn_s_waitcnt(kWaitVmAll);
    __syncthreads();
    const int halves = 2 * min(2, cut - i);
#pragma unroll 1
    for (int h = KW == 2 ? kw : 0; h < halves; h += KW) {
      const int hb = cut_tile(i + h / 2) * 64 + 32 * (h & 1);
      if (hb >= span.hi || hb + 32 <= span.lo) continue;  // (wave-uniform) no row sees them
      const unsigned char* kh = (h < 2 ? kbuf0 : kbuf1) + (h & 1) * C::HALF;
      const unsigned char* vh = (h < 2 ? vbuf0 : vbuf1) + (h & 1) * C::HALF;
      f32x16 acc;
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[v] = 0.0f;
#pragma unroll
      for (int k = 0; k < C::KSTEPS; ++k)
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(kh + kread[k]), qv[k], acc, 0, 0, 0);
      bf16x8 pb[2];
      const bool whole = hb >= span.all_lo && hb + 32 <= span.all_hi;  // (wave-uniform)
      const uint64_t mk = h < 2 ? masks[0] : masks[1];
      const int mlo = (int)(uint32_t)mk, mhi = (int)(uint32_t)(mk >> 32);
      if (!whole) {  // hidden scores become -inf
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int i32 = 8 * (v >> 2) + 4 * hh + (v & 3), n = hb + i32;
          bool ok = (n >= q.lo) & (n < q.hi);
          if (TRIES && trie) {
            const int at = (32 * (h & 1) + i32) << 2;
            const uint32_t w0 = (uint32_t)__builtin_amdgcn_ds_bpermute(at, mlo), w1 = (uint32_t)__builtin_amdgcn_ds_bpermute(at, mhi);
            ok &= (((q.j < 32 ? w0 : w1) >> (q.j & 31)) & 1u) != 0;
          }
          acc[v] = ok ? acc[v] : -INFINITY;
        }
      }
      weigh(acc, pb);
      // A hidden key weighs 0, but 0 times an infinite or NaN V is NaN: a tile that holds such a V
      // adds its products key by key, to the rows that see the key.
      bool odd = false;
      if (!whole) {
#pragma unroll
        for (int uu = 0; uu < 2; ++uu)
#pragma unroll
          for (int dt = 0; dt < C::DT; ++dt) {
            const i16x8 x = vop(vh, uu, dt);
#pragma unroll
            for (int e = 0; e < 8; ++e) odd |= (x[e] & 0x7f80) == 0x7f80;
          }
      }
      if (!__any(odd)) {
        add_values(vh, pb);
        continue;
      }
#pragma unroll 1
      for (int n = 0; n < 32; ++n) {  // key hb + n, held by half-wave (n / 4) % 2
        const int vi = (n >> 3) * 4 + (n & 3);
        float w = 0.0f;
#pragma unroll
        for (int v = 0; v < 16; ++v) w = v == vi ? (float)pb[v >> 3][v & 7] : w;
        w = __shfl(w, col + 32 * ((n >> 2) & 1));
        bool own = hb + n >= q.lo && hb + n < q.hi;
        if (TRIES && trie) {
          const int at = 32 * (h & 1) + n;
          const uint32_t w0 = (uint32_t)__builtin_amdgcn_readlane(mlo, at), w1 = (uint32_t)__builtin_amdgcn_readlane(mhi, at);
          own = own && (((q.j < 32 ? w0 : w1) >> (q.j & 31)) & 1u) != 0;
        }
#pragma unroll
        for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            // elements 32 dt + 8 q4 + 4 hh .. + 3 of the key's V row
            const bf16x4 x = *reinterpret_cast<const bf16x4*>(
                vh + n * (2 * D) + v_chunk<C::CPR, C::NBLK, FOUR>(n, 4 * dt + q4) * 16 + 8 * hh);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[dt][4 * q4 + e] += own ? w * (float)x[e] : 0.0f;
          }
      }
    }
  }

  if constexpr (KW == 2) {
    // the second group hands its state over through LDS, lane by lane: a quarter of O in each buffer
    static_assert(RW * 64 * (D / 8) * 4 <= 2 * C::HALF, "a quarter of O fits a buffer");
    __syncthreads();  // every wave has read its last tile
    float* const part[4] = {reinterpret_cast<float*>(kbuf0), reinterpret_cast<float*>(vbuf0), reinterpret_cast<float*>(kbuf1),
                            reinterpret_cast<float*>(vbuf1)};
    if (kw == 1) {
#pragma unroll
      for (int x = 0; x < D / 2; ++x) part[x / (D / 8)][(rw * (D / 8) + x % (D / 8)) * 64 + lane] = o[x / 16][x % 16];
      ml[rw * 128 + lane] = m;
      ml[rw * 128 + 64 + lane] = lsum;
    }
    __syncthreads();
    if (kw == 0) {
      const float m1 = ml[rw * 128 + lane], l1 = ml[rw * 128 + 64 + lane];
      const float mn = fmaxf(m, m1);
      const float f0 = __builtin_amdgcn_exp2f(m - mn), f1 = __builtin_amdgcn_exp2f(m1 - mn);
      m = mn;
      lsum = lsum * f0 + l1 * f1;
#pragma unroll
      for (int x = 0; x < D / 2; ++x)
        o[x / 16][x % 16] = o[x / 16][x % 16] * f0 + part[x / (D / 8)][(rw * (D / 8) + x % (D / 8)) * 64 + lane] * f1;
    }
    __syncthreads();
    if (kw == 1) return;
  } else {
    __syncthreads();  // every wave has read its last tile
  }

  lsum += __shfl_xor(lsum, 32);
  unsigned char* const mine = rw == 0 ? kbuf0 : rw == 1 ? vbuf0 : rw == 2 ? kbuf1 : vbuf1;
  prefix_output<__bf16, D>(s, a, u, q, lane, m, lsum, o, reinterpret_cast<float*>(mine));
