// Attention of many query rows over the shared prefix (gfx950 matrix cores, bf16 in, fp32 accumulate).
//
// softmax(scale q k^T) v over the prefix's positions, for the rows of every trie of the batch at
// once: a KV head's rows (owner, query head of its group) are packed into blocks, whichever trie they
// belong to, so that one pass over the prefix's keys serves them all.  Each row sees an interval of
// positions (all of the prefix, less what a sliding window cuts off; or, causal, up to its own).  A
// pass leaves each row's unnormalised output, shift and sum; they are merged with the trie's own.
//
//   S^T[key][row] = K_tile . Q^T,  O^T[d][row] += V_tile^T . P^T    on v_mfma_f32_32x32x16_bf16,
//
// operands and LDS layout as in the tree kernels: a wave holds 32 rows, one per lane pair, and reads
// K in MFMA layout and V transposed (ds_read_b64_tr_b16) from a tile of 64 keys in LDS.  The tile's
// rows come from the pages of a paged cache: a tile lies in one page of 64 keys or more, or in up to
// four smaller ones, whose numbers are loaded a tile ahead by scalar loads.
//
// What bounds it, by the rows that share a key (one MI355X, d = 128 unless stated; kernel trace, mean of
// passes once the clocks have settled, in brackets the least):
//   * few rows: HBM.  8 rows per KV head (32 KV heads, d = 96) over 50,001 keys: 112 (108) us, 5.5 (5.7)
//     TB/s of reads.  Below some 4,000 keys per KV head a launch is a chain of latencies: 128 rows over 4,096
//     keys of 8 KV heads, with the tries' own nodes, 16.5 (14.6) us (its 17 MB take 3.4).
//   * many rows: the clock under matrix load.  1,024 rows of 8 KV heads over 8,192 keys of 4 layers: 160 (154)
//     us, 859 (892) TFLOP/s; the causal pass of 2,048 tokens from position 6,144: 249 (246) us, 966 (976)
//     TFLOP/s, and 244 us, 984, without the trace (a library product of 8,192^3 makes 1,121 here).  There the
//     card runs at 2.0 to 2.1 of its 2.4 GHz, the matrix pipe busy for half of the CUs' clocks, the vector ALU
//     (the exponentials) as long, LDS a quarter.  Each of the two waves of a SIMD fills the other's gaps: a
//     loop that interleaves one half's weights with its neighbours' products by hand took the same time to 0.3 %.
// Tried and not kept: four tile buffers (16,384 keys in 8 splits: 60 us against 48); 8 waves, of two
// groups of keys, per 128 rows (8,192 keys, 1,024 rows: 55 us against 50); a fixed order of products and
// LDS reads (1.5 % slower); 64 rows per wave, one wave per SIMD (568 us against 480 for two causal layers).
#include <algorithm>

#include "attn_common.h"
#include "attn_prefix.h"

namespace td {

namespace {

constexpr float kMost = 8192.0f;  // a row's shift moves once 16 of its probabilities add up to more
constexpr float kSlack = 8.0f;    // ... to its largest score, if that is 2^8 above

// RW waves hold 32 rows each; KW groups of RW waves take the 32-key halves of each tile.
template <int D, int RW, int KW>
struct PrefixCfg {
  static constexpr int THREADS = 64 * RW * KW;
  static constexpr int KSTEPS = D / 16;    // 32x32x16 steps of S^T
  static constexpr int DT = D / 32;        // 32-wide d tiles of O^T
  static constexpr int CPR = D / 8;        // 16-byte chunks per key row
  static constexpr int NBLK = CPR / 4;     // 64-byte blocks per row
  static constexpr int HALF = 32 * D * 2;  // bytes of 32 K (or V) rows
  static constexpr int LOADS = 2 * HALF / 16 / THREADS;  // 16-byte loads per thread: K (or V) of a tile
  static_assert(2 * HALF % (16 * THREADS) == 0, "a tile is a whole number of WG loads");
  static constexpr bool ONE_OFS = THREADS % CPR == 0 && (THREADS / CPR) % CPR == 0;
  static constexpr int OFS = ONE_OFS ? 1 : LOADS;
  static constexpr int WAVES = 8 * HALF <= 80 * 1024 ? 2 : 1;  // per SIMD, as the LDS allows
  static constexpr int VROT = 8 % NBLK == 0 ? 1 : 4;  // rotations of V rows 8 apart
};

// TRIES: the launch's last WGs take the tries' own nodes (PrefixArgs::trie_splits), for calls so small
// that a launch of their own would run after this one instead of beside it.  A trie's rows in its
// pool are one page of nodes; every live row sees its shared prefix, and of the nodes after it those
// whose ancestor mask holds the row's beam.
template <int D, int RW, int KW, bool TRIES>
__global__ __launch_bounds__(64 * RW * KW, (PrefixCfg<D, RW, KW>::WAVES)) void k_attn_prefix(DevState s, PrefixArgs a) {
  using C = PrefixCfg<D, RW, KW>;
  static_assert(2 * C::LOADS < 64, "the wait counter holds a tile's loads");
  static_assert(KW == 1 || KW == 2, "one or two groups: the RW KW waves have a word each of wred");
  constexpr int NH = 2 / KW;  // 32-key halves of a tile per wave
  // (an array per buffer: the compiler can tell an operand read of one buffer from the direct loads
  // under way into the others)
  __shared__ __attribute__((aligned(16))) unsigned char kbuf0[2 * C::HALF], vbuf0[2 * C::HALF];
  __shared__ __attribute__((aligned(16))) unsigned char kbuf1[2 * C::HALF], vbuf1[2 * C::HALF];
  __shared__ int wred[4 * RW];
  __shared__ float ml[KW == 2 ? RW * 128 : 1];
  PrefixHdr p = *s.prefix;
  const bool trie = TRIES && blockIdx.x >= a.prefix_wgs;
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
    vofs[j] = row * (2 * D) + (pc + C::CPR - 4 * (row % 32 % C::NBLK)) % C::CPR * 16;
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

  // the first two tiles go out before anything that waits for the tries
  TilePages next{};
  if (t0 < t1) {
    const bool main = m0 < m1;
    const int x0 = main ? m0 : cut_tile(0), x1 = main ? m0 + 1 : cut_tile(1);
    const bool two = main ? m0 + 1 < m1 : cut > 1;
    const TilePages pg0 = pages_of(x0), pg1 = pages_of(two ? x1 : x0);
    issue(x0, pg0, kbuf0, vbuf0);
    if (two) issue(x1, pg1, kbuf1, vbuf1);
    if (m0 + 2 < m1) next = pages_of(m0 + 2);
  }
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
      vread[x8][dt] = (4 * hh + tm) * (2 * D) + phys_chunk<C::CPR, C::NBLK>(n, c) * 16 + 8 * (tq & 1);
    }

  const float scale = a.scale_log2;
  float m = kPrefixNegBig, lsum = 0.0f;
  f32x16 o[C::DT];
#pragma unroll
  for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[dt][v] = 0.0f;

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
    // this thread's loads of the tile have landed, then every thread's, and the other buffer is free
    // (the second tile is on its way already)
    if (tile == m0 && m0 + 1 < m1) __builtin_amdgcn_s_waitcnt(wait_vm(2 * C::LOADS));
    else __builtin_amdgcn_s_waitcnt(kWaitVmAll);
    __syncthreads();
    if (tile > m0 && tile + 1 < m1) {
      issue(tile + 1, next, knext, vnext);
      if (tile + 2 < m1) next = pages_of(tile + 2);
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
      issue(cut_tile(i), pg0, kbuf0, vbuf0);
      if (two) issue(cut_tile(i + 1), pg1, kbuf1, vbuf1);
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
                vh + n * (2 * D) + phys_chunk<C::CPR, C::NBLK>(n, 4 * dt + q4) * 16 + 8 * hh);
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
}

template <int D>
void launch_d(const DevState& s, const PrefixArgs& a, int rpb, hipStream_t st, hipEvent_t ev0, hipEvent_t ev1) {
  const dim3 grid(a.n_layers * s.Hkv * (a.splits * a.row_blocks + a.tries * a.trie_blocks * a.trie_splits));
#define LAUNCH_PREFIX(RW, KW, TRIES) \
  hipExtLaunchKernelGGL((k_attn_prefix<D, RW, KW, TRIES>), grid, dim3(64 * RW * KW), 0, st, ev0, ev1, 0, s, a)
  if constexpr (D == 64 || D == 96 || D == 128) {
    if (a.trie_splits > 0) {
      if (rpb == 32) LAUNCH_PREFIX(1, 2, true);
      else if (rpb == 64) LAUNCH_PREFIX(2, 2, true);
      else LAUNCH_PREFIX(4, 1, true);
      return;
    }
  }
  if (rpb == 32) LAUNCH_PREFIX(1, 2, false);
  else if (rpb == 64) LAUNCH_PREFIX(2, 2, false);
  else LAUNCH_PREFIX(4, 1, false);
#undef LAUNCH_PREFIX
}

// Each (row, 8-element chunk of d) is merged by TP adjacent lanes, lane j taking the groups of 8
// records j, j + TP, ...: every load of a group goes out before any is used; groups are merged with
// a running shift, the lanes' states pairwise, in one order.  A record with sum 0 weighs nothing
// (whatever its O); a NaN sum makes the row NaN.  Bound by the latency of its one or two loads in a
// row: 18 records each of 1,024 output rows, 4.7 to 5.1 us.
constexpr int kMergeThreads = 64;

template <typename T, int TP>
__global__ __launch_bounds__(kMergeThreads) void k_prefix_merge(DevState s, PrefixMergeArgs a, uint32_t items) {
  constexpr int GS = 8;
  const int D = s.D, G = s.Hq / s.Hkv, CH = D / 8;
  // (the host keeps items * TP below 2^31)
  const uint32_t item = (blockIdx.x * kMergeThreads + threadIdx.x) / TP;
  const int sub = threadIdx.x % TP;
  if (item >= items) return;  // (the lanes of an item leave together)
  const uint32_t row = item / CH;
  const int c = (int)(item % CH) * 8;
  const int head = row % s.Hq;
  const uint32_t o = row / s.Hq;  // (li tries + t) per_trie + j
  const int j = o % a.per_trie;
  const uint32_t tl = o / a.per_trie;
  const int t = tl % a.tries, li = tl / a.tries;
  const size_t prec = (size_t)row * a.prefix_splits;
  const int ts = a.trie != nullptr ? a.trie_splits : 0, n = ts + a.prefix_splits;
  const float* trec = nullptr;
  size_t tstep = 0;
  if (ts > 0) {
    const int r = j * G + head % G;
    const size_t unit = (((size_t)t * a.n_layers + li) * s.Hkv + head / G) * a.row_blocks + r / a.block_rows;
    trec = a.trie + (unit * ts * a.block_rows + r % a.block_rows) * (D + 2);
    tstep = (size_t)a.block_rows * (D + 2);
  }
  const bool live = a.rows != PrefixRows::kLeaves || j < s.hdr[t].n_live;
  float M = kPrefixNegBig, L = 0.0f, O[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) O[e] = 0.0f;
  for (int i0 = sub * GS; i0 < n; i0 += TP * GS) {
    float2 ml[GS];
    float2 ov[GS][4];
#pragma unroll
    for (int k = 0; k < GS; ++k) {
      const int i = i0 + k < n ? i0 + k : i0;  // (past the last: the group's first again, unused)
      // (the tries' records are D + 2 floats, 8-byte aligned)
      const float* rec = i < ts ? trec + i * tstep : a.prefix_o + (prec + i - ts) * D;
      ml[k] = i < ts ? *reinterpret_cast<const float2*>(rec + D) : a.prefix_ml[prec + i - ts];
#pragma unroll
      for (int e = 0; e < 4; ++e) ov[k][e] = *reinterpret_cast<const float2*>(rec + c + 2 * e);
    }
    float Mg = M;
#pragma unroll
    for (int k = 0; k < GS; ++k) Mg = i0 + k < n && ml[k].y != 0.0f ? fmaxf(Mg, ml[k].x) : Mg;
    const float fo = __builtin_amdgcn_exp2f(M - Mg);
    L *= fo;
#pragma unroll
    for (int e = 0; e < 8; ++e) O[e] *= fo;
#pragma unroll
    for (int k = 0; k < GS; ++k) {
      const bool use = i0 + k < n && ml[k].y != 0.0f;
      const float f = __builtin_amdgcn_exp2f(ml[k].x - Mg);
      L += use ? ml[k].y * f : 0.0f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        O[2 * e] += use ? ov[k][e].x * f : 0.0f;
        O[2 * e + 1] += use ? ov[k][e].y * f : 0.0f;
      }
    }
    M = Mg;
  }
#pragma unroll
  for (int w = 1; w < TP; w <<= 1) {
    const float M2 = __shfl_xor(M, w), L2 = __shfl_xor(L, w);
    float O2[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) O2[e] = __shfl_xor(O[e], w);
    const bool low = (sub & w) == 0;
    const float Mn = fmaxf(M, M2);
    const float f0 = __builtin_amdgcn_exp2f((low ? M : M2) - Mn), f1 = __builtin_amdgcn_exp2f((low ? M2 : M) - Mn);
    L = (low ? L : L2) * f0 + (low ? L2 : L) * f1;
#pragma unroll
    for (int e = 0; e < 8; ++e) O[e] = (low ? O[e] : O2[e]) * f0 + (low ? O2[e] : O[e]) * f1;
    M = Mn;
  }
  if (sub != 0) return;
  const float inv = live && L != 0.0f ? 1.0f / L : 0.0f;
  typedef T t8 __attribute__((ext_vector_type(8)));
  t8 y;
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = (T)(live && L != 0.0f ? O[e] * inv : 0.0f);
  *reinterpret_cast<t8*>(static_cast<T*>(a.out) + (size_t)row * D + c) = y;
}

}  // namespace

int prefix_rows_per_block(long rows) {
  return rows <= 32 ? 32 : rows <= 64 ? 64 : 128;
}

// A WG per CU, of at least 4 tiles of 64 keys; two per CU where each still has 16.  More splits make
// shorter chains of tiles and more records to merge.  Measured, 8 KV heads at d = 128, the pass and
// its merge, us: 128 rows over 4,096 keys, 8 / 16 / 32 splits: 22.6 / 20.9 / 24.6; over 16,384 keys, 16 /
// 32 / 64: 35.1 / 30.5 / 34.1; 1,024 rows (8 blocks) over 1,024 keys, 4 / 8: 25.5 / 27.7; over 8,192 keys,
// 4 / 8 / 16: 63 / 57 / 72; 32 rows over 4,096 keys, 16 / 32 / 64: 17.4 / 17.9 / 20.1.  In fp32 a tile takes
// ten times as long: one tile, and two per CU where each still has 2.
int prefix_splits(const DevState& s, long units, long keys, long most) {
  const long tiles = (keys + 63) / 64, few = s.dtype == TD_F32 ? 1 : 4, many = s.dtype == TD_F32 ? 2 : 16;
  const long one = std::min((256 + units - 1) / units, tiles / few), two = std::min((512 + units - 1) / units, tiles / many);
  return (int)std::max(1l, std::min(std::max(one, two), most));
}

hipError_t launch_prefix(const DevState& s, const PrefixArgs& a, hipStream_t st, hipEvent_t ev0, hipEvent_t ev1) {
  const int rpb = prefix_rows_per_block((long)a.tries * a.per_trie * (s.Hq / s.Hkv));
  if (a.trie_splits > 0 && (a.rows != PrefixRows::kLeaves || s.dtype != TD_BF16 || !mfma_head_dim(s.D))) return hipErrorInvalidValue;
  if (s.dtype == TD_F32) return launch_prefix32(s, a, rpb, st, ev0, ev1);
  switch (s.D) {
#define PREFIX_CASE(DD) case DD: launch_d<DD>(s, a, rpb, st, ev0, ev1); break;
    PREFIX_CASE(32) PREFIX_CASE(64) PREFIX_CASE(96) PREFIX_CASE(128)
    PREFIX_CASE(160) PREFIX_CASE(192) PREFIX_CASE(224) PREFIX_CASE(256)
#undef PREFIX_CASE
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

hipError_t launch_prefix_merge(const DevState& s, const PrefixMergeArgs& a, hipStream_t st, hipEvent_t ev1) {
  const long items = (long)a.n_layers * a.tries * a.per_trie * s.Hq * (s.D / 8);
  const int n = (a.trie ? a.trie_splits : 0) + a.prefix_splits;
  const int tp = n > 16 ? 4 : n > 8 ? 2 : 1;  // lanes per output chunk: 8 records each
  if (items * tp >= (1l << 31)) return hipErrorInvalidValue;  // (a workspace of records is far smaller)
  const dim3 grid((items * tp + kMergeThreads - 1) / kMergeThreads), block(kMergeThreads);
#define LAUNCH_MERGE(T, TP) \
  hipExtLaunchKernelGGL((k_prefix_merge<T, TP>), grid, block, 0, st, nullptr, ev1, 0, s, a, (uint32_t)items)
  if (s.dtype == TD_F32) tp == 4 ? LAUNCH_MERGE(float, 4) : tp == 2 ? LAUNCH_MERGE(float, 2) : LAUNCH_MERGE(float, 1);
  else tp == 4 ? LAUNCH_MERGE(__bf16, 4) : tp == 2 ? LAUNCH_MERGE(__bf16, 2) : LAUNCH_MERGE(__bf16, 1);
#undef LAUNCH_MERGE
  return hipGetLastError();
}

}  // namespace td
