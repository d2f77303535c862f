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
#include <algorithm>

#include "attn_prefix.h"

namespace td {

namespace {

constexpr float kMost = 8192.0f;  // a row's shift moves once 16 of its probabilities add up to more
constexpr float kSlack = 8.0f;    // ... to its largest score, if that is 2^8 above

// RW waves hold 32 rows each; KW groups of RW waves take the 32-key halves of each tile in turn.
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
  static constexpr int WAVES = D <= 128 ? 2 : 1;      // per SIMD: as many as the LDS allows
  static constexpr int VROT = 8 % NBLK == 0 ? 1 : 4;  // rotations of V rows 8 apart
};

template <int D, int RW, int KW>
__global__ __launch_bounds__(64 * RW * KW, (PrefixCfg<D, RW, KW>::WAVES)) void k_attn_prefix(DevState s, PrefixArgs a) {
  using C = PrefixCfg<D, RW, KW>;
  static_assert(KW == 1 || (KW == 2 && RW <= 2), "the second group's O fits the K buffers");
  constexpr int NH = 2 / KW;  // 32-key halves of a tile per wave
  // (four arrays, each used for one buffer only: the compiler can tell an operand read of one buffer
  // from the direct loads under way into the other)
  __shared__ __attribute__((aligned(16))) unsigned char kbuf0[2 * C::HALF], vbuf0[2 * C::HALF];
  __shared__ __attribute__((aligned(16))) unsigned char kbuf1[2 * C::HALF], vbuf1[2 * C::HALF];
  __shared__ int wred[2][RW];
  const PrefixUnit u = prefix_unit(s, a);
  const PrefixHdr p = *s.prefix;
  const int lab = a.layer_begin + u.li;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rw = wave % RW, kw = wave / RW;
  const int col = lane & 31, hh = lane >> 5;

  const PrefixRow q = prefix_row(s, a, p, u.li, (u.rb * RW + rw) * 32 + col);
  const PrefixSpan span = prefix_span(q);
  if (lane == 0 && kw == 0) {
    wred[0][rw] = span.lo;
    wred[1][rw] = span.hi;
  }
  __syncthreads();
  int lo = INT_MAX, hi = 0;
  for (int w = 0; w < RW; ++w) {
    lo = min(lo, wred[0][w]);
    hi = max(hi, wred[1][w]);
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  hi = __builtin_amdgcn_readfirstlane(hi);
  // tiles of 64 keys, at multiples of 64: this split's share
  const int first = hi > 0 ? lo / 64 : 0, tiles = hi > 0 ? (hi + 63) / 64 - first : 0;
  const int per = (tiles + a.splits - 1) / a.splits;
  const int t0 = first + u.split * per, t1 = min(first + tiles, t0 + per);

  const size_t head = ((size_t)lab * s.Hkv + u.g) << p.shift;  // rows before this (layer, KV head) in a page
  const size_t page_rows = ((size_t)s.L * s.Hkv) << p.shift;
  const __bf16* kpages = static_cast<const __bf16*>(p.k);
  const __bf16* vpages = static_cast<const __bf16*>(p.v);

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

  // the lane's query row as B operands of S^T: half hh of its d range
  bf16x8 qv[C::KSTEPS];
  {
    const bool some = q.lo < q.hi;
    const uint4* qp = reinterpret_cast<const uint4*>(static_cast<const __bf16*>(a.q) +
                                                     ((some ? q.at : 0) * s.Hq + u.g * (s.Hq / s.Hkv) + q.head) * D + hh * (D / 2));
#pragma unroll
    for (int k = 0; k < C::KSTEPS; ++k) qv[k] = __builtin_bit_cast(bf16x8, some ? qp[k] : make_uint4(0, 0, 0, 0));
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

  TilePages next;
  auto step = [&](int tile, const unsigned char* kb, const unsigned char* vb, unsigned char* knext,
                  unsigned char* vnext) __attribute__((always_inline)) {
    __builtin_amdgcn_s_waitcnt(kWaitVmAll);  // this thread's loads of the tile have landed
    __syncthreads();                         // every thread's have; the other buffer is free
    if (tile + 1 < t1) {
      issue(tile + 1, next, knext, vnext);
      if (tile + 2 < t1) next = tile_pages(p, tile + 2);
    }
    const int tb = tile * 64;
    if (tb >= span.hi || tb + 64 <= span.lo) return;  // (wave-uniform) no row sees the tile
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
    // a row's interval cuts the tile: hidden scores become -inf
    const bool cut = tb < span.all_lo || tb + 64 > span.all_hi;
    if (cut) {
#pragma unroll
      for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int n = tb + 32 * (KW == 2 ? kw : h) + 8 * (v >> 2) + 4 * hh + (v & 3);
          acc[h][v] = (n >= q.lo) & (n < q.hi) ? acc[h][v] : -INFINITY;
        }
    }
    const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
    for (int h = 0; h < NH; ++h) {
      const int half = KW == 2 ? kw : h;
      // Probabilities relative to the row's shift m, rounded to bf16 (the operand type of the second
      // product; the sum takes the rounded ones, so the rounding errors of numerator and denominator
      // go together), and their sum over this lane's 16 keys.  Softmax does not depend on the shift:
      // it moves only when the probabilities leave their range, which their sum tells.
      bf16x8 pb[2];
      float ps = 0.0f;
      auto weights = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int v = 0; v < 16; ++v)
          pb[v >> 3][v & 7] = (__bf16)__builtin_amdgcn_exp2f(__builtin_fmaf(acc[h][v], scale, -m));
        ps = 0.0f;
#pragma unroll
        for (int v = 0; v < 16; v += 2) {
          const bf16x2 pair = {pb[v >> 3][v & 7], pb[v >> 3][(v & 7) + 1]};
          ps = __builtin_amdgcn_fdot2_f32_bf16(pair, ones, ps, false);
        }
      };
      weights();
      if (__any(ps > kMost)) {
        float tmax = acc[h][0];
#pragma unroll
        for (int v = 1; v < 16; ++v) tmax = fmaxf(tmax, acc[h][v]);
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
      const unsigned char* vh = vb + half * C::HALF;
      if (cut) {
        // A hidden key weighs 0, but 0 times an infinite or NaN V is NaN: a tile that is cut and
        // holds such a V adds its products key by key, to the rows that see the key.
        bool odd = false;
#pragma unroll
        for (int uu = 0; uu < 2; ++uu)
#pragma unroll
          for (int dt = 0; dt < C::DT; ++dt) {
            const i16x8 x = vop(vh, uu, dt);
#pragma unroll
            for (int e = 0; e < 8; ++e) odd |= (x[e] & 0x7f80) == 0x7f80;
          }
        if (__any(odd)) {
#pragma unroll 1
          for (int i = 0; i < 32; ++i) {  // key tb + 32 half + i, held by half-wave (i / 4) % 2
            const int n = tb + 32 * half + i, vi = (i >> 3) * 4 + (i & 3);
            float w = 0.0f;
#pragma unroll
            for (int v = 0; v < 16; ++v) w = v == vi ? (float)pb[v >> 3][v & 7] : w;
            w = __shfl(w, col + 32 * ((i >> 2) & 1));
            const bool own = n >= q.lo && n < q.hi;
#pragma unroll
            for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
              for (int q4 = 0; q4 < 4; ++q4) {
                // elements 32 dt + 8 q4 + 4 hh .. + 3 of the key's V row
                const bf16x4 x = *reinterpret_cast<const bf16x4*>(
                    vh + i * (2 * D) + phys_chunk<C::CPR, C::NBLK>(i, 4 * dt + q4) * 16 + 8 * hh);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[dt][4 * q4 + e] += own ? w * (float)x[e] : 0.0f;
              }
          }
          continue;
        }
      }
#pragma unroll
      for (int uu = 0; uu < 2; ++uu)
#pragma unroll
        for (int dt = 0; dt < C::DT; ++dt)
          o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vop(vh, uu, dt)), pb[uu], o[dt], 0, 0, 0);
    }
  };
  if (t0 < t1) {
    issue(t0, tile_pages(p, t0), kbuf0, vbuf0);
    if (t0 + 1 < t1) next = tile_pages(p, t0 + 1);
  }
  for (int t = t0; t < t1; t += 2) {
    step(t, kbuf0, vbuf0, kbuf1, vbuf1);
    if (t + 1 < t1) step(t + 1, kbuf1, vbuf1, kbuf0, vbuf0);
  }

  if constexpr (KW == 2) {
    // the second group hands its state over through LDS, lane by lane
    __syncthreads();  // every wave has read its last tile
    float* const o0 = reinterpret_cast<float*>(kbuf0);
    float* const o1 = reinterpret_cast<float*>(kbuf1);
    float* const ml = reinterpret_cast<float*>(vbuf0);
    if (kw == 1) {
#pragma unroll
      for (int x = 0; x < D / 4; ++x) {
        const int at = (rw * (D / 4) + x) * 64 + lane, y = x + D / 4;
        o0[at] = o[x / 16][x % 16];
        o1[at] = o[y / 16][y % 16];
      }
      ml[rw * 128 + lane] = m;
      ml[rw * 128 + 64 + lane] = lsum;
    }
    __syncthreads();
    if (kw == 1) return;
    const float m1 = ml[rw * 128 + lane], l1 = ml[rw * 128 + 64 + lane];
    const float mn = fmaxf(m, m1);
    const float f0 = __builtin_amdgcn_exp2f(m - mn), f1 = __builtin_amdgcn_exp2f(m1 - mn);
    m = mn;
    lsum = lsum * f0 + l1 * f1;
#pragma unroll
    for (int x = 0; x < D / 4; ++x) {
      const int at = (rw * (D / 4) + x) * 64 + lane, y = x + D / 4;
      o[x / 16][x % 16] = o[x / 16][x % 16] * f0 + o0[at] * f1;
      o[y / 16][y % 16] = o[y / 16][y % 16] * f0 + o1[at] * f1;
    }
  }

  lsum += __shfl_xor(lsum, 32);
  if (!q.in) return;
  const bool some = q.lo < q.hi && lsum != 0.0f;  // (a NaN sum is a NaN row)
  if (a.part != nullptr) {
    float* rec = prefix_record(s, a, u, q);
#pragma unroll
    for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        float2* r2 = reinterpret_cast<float2*>(rec + 32 * dt + 8 * q4 + 4 * hh);
        r2[0] = make_float2(o[dt][4 * q4], o[dt][4 * q4 + 1]);
        r2[1] = make_float2(o[dt][4 * q4 + 2], o[dt][4 * q4 + 3]);
      }
    if (hh == 0) *reinterpret_cast<float2*>(rec + D) = make_float2(some ? m : kPrefixNegBig, some ? lsum : 0.0f);
  } else {
    const float inv = some ? 1.0f / lsum : 0.0f;
    __bf16* orow = static_cast<__bf16*>(a.out) + (q.at * s.Hq + u.g * (s.Hq / s.Hkv) + q.head) * D;
#pragma unroll
    for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        bf16x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = (__bf16)(some ? o[dt][4 * q4 + e] * inv : 0.0f);
        *reinterpret_cast<bf16x4*>(orow + 32 * dt + 8 * q4 + 4 * hh) = y;
      }
  }
}

template <int D>
void launch_d(const DevState& s, const PrefixArgs& a, int rpb, hipStream_t st, hipEvent_t ev0, hipEvent_t ev1) {
  const dim3 grid(a.n_layers * s.Hkv * a.splits * a.row_blocks);
  if (rpb == 32) hipExtLaunchKernelGGL((k_attn_prefix<D, 1, 2>), grid, dim3(128), 0, st, ev0, ev1, 0, s, a);
  else if (rpb == 64) hipExtLaunchKernelGGL((k_attn_prefix<D, 2, 2>), grid, dim3(256), 0, st, ev0, ev1, 0, s, a);
  else hipExtLaunchKernelGGL((k_attn_prefix<D, 4, 1>), grid, dim3(256), 0, st, ev0, ev1, 0, s, a);
}

// One wave per (row, merge): lanes hold the row's d in 8-byte pieces.  Every record's shift and sum
// first, then the weighted O of all of them.
constexpr int kMergeThreads = 256;

template <typename T>
__global__ __launch_bounds__(kMergeThreads) void k_prefix_merge(DevState s, PrefixMergeArgs a) {
  const int D = s.D, G = s.Hq / s.Hkv;
  const int lane = threadIdx.x & 63;
  const long rows = (long)a.n_layers * a.tries * a.per_trie * s.Hq;
  const long row = (long)blockIdx.x * (kMergeThreads / 64) + (threadIdx.x >> 6);
  if (row >= rows) return;
  const int head = row % s.Hq;
  const long o = row / s.Hq;  // (li tries + t) per_trie + j
  const int j = o % a.per_trie;
  const int t = (o / a.per_trie) % a.tries, li = (int)(o / a.per_trie / a.tries);
  const float* prec = a.prefix + row * a.prefix_splits * (D + 2);
  const float* trec = nullptr;
  size_t tstep = 0;
  if (a.trie != nullptr) {
    const int r = j * G + head % G;
    const size_t unit = (((size_t)t * a.n_layers + li) * s.Hkv + head / G) * a.row_blocks + r / a.block_rows;
    trec = a.trie + (unit * a.trie_splits * a.block_rows + r % a.block_rows) * (D + 2);
    tstep = (size_t)a.block_rows * (D + 2);
  }
  const bool live = a.rows != PrefixRows::kLeaves || j < s.hdr[t].n_live;
  const int n = (a.trie != nullptr ? a.trie_splits : 0) + a.prefix_splits;
  auto record = [&](int i) {
    return trec != nullptr && i < a.trie_splits ? trec + i * tstep
                                                 : prec + (size_t)(i - (trec != nullptr ? a.trie_splits : 0)) * (D + 2);
  };
  // lane i: record i, i + 64, ...
  float m = kPrefixNegBig, l = 0.0f;
  for (int i = lane; i < n; i += 64) {
    const float2 ml = *reinterpret_cast<const float2*>(record(i) + D);
    if (ml.y == 0.0f) continue;
    const float mn = fmaxf(m, ml.x);
    l = l * exp2f(m - mn) + ml.y * exp2f(ml.x - mn);
    m = mn;
  }
  float M = m;
  for (int x = 32; x > 0; x >>= 1) M = fmaxf(M, __shfl_xor(M, x));
  float L = l * exp2f(m - M);
  for (int x = 32; x > 0; x >>= 1) L += __shfl_xor(L, x);
  T* out = static_cast<T*>(a.out) + ((((size_t)li * a.tries + t) * a.q_stride + a.q0 + j) * s.Hq + head) * D;
  const bool some = live && L != 0.0f;
  for (int c = 2 * lane; c < D; c += 128) {
    float x = 0.0f, y = 0.0f;
    if (some) {
      for (int i = 0; i < n; ++i) {
        const float* rec = record(i);
        const float2 ml = *reinterpret_cast<const float2*>(rec + D);
        if (ml.y == 0.0f) continue;
        const float f = exp2f(ml.x - M);
        const float2 v = *reinterpret_cast<const float2*>(rec + c);
        x += v.x * f;
        y += v.y * f;
      }
      x /= L;
      y /= L;
    }
    typedef T t2 __attribute__((ext_vector_type(2)));
    t2 w = {(T)x, (T)y};
    *reinterpret_cast<t2*>(out + c) = w;
  }
}

}  // namespace

int prefix_rows_per_block(const DevState& s, long rows) {
  if (s.dtype == TD_F32) return rows <= 32 ? 32 : rows <= 64 ? 64 : 128;
  return rows <= 32 ? 32 : rows <= 64 ? 64 : 128;
}

int prefix_splits(const DevState& s, long rows, long units, long keys, long most) {
  (void)s;
  (void)rows;
  const long tiles = (keys + 63) / 64;
  const long n = std::min({(512 + units - 1) / units, (tiles + 3) / 4, most, 64l});
  return (int)std::max(1l, n);
}

hipError_t launch_prefix(const DevState& s, const PrefixArgs& a, hipStream_t st, hipEvent_t ev0, hipEvent_t ev1) {
  const int rpb = prefix_rows_per_block(s, (long)a.tries * a.per_trie * (s.Hq / s.Hkv));
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

hipError_t launch_prefix_merge(const DevState& s, const PrefixMergeArgs& a, hipStream_t st, hipEvent_t ev0, hipEvent_t ev1) {
  const long rows = (long)a.n_layers * a.tries * a.per_trie * s.Hq;
  const dim3 grid((rows + kMergeThreads / 64 - 1) / (kMergeThreads / 64));
  if (s.dtype == TD_F32) hipExtLaunchKernelGGL(k_prefix_merge<float>, grid, dim3(kMergeThreads), 0, st, ev0, ev1, 0, s, a);
  else hipExtLaunchKernelGGL(k_prefix_merge<__bf16>, grid, dim3(kMergeThreads), 0, st, ev0, ev1, 0, s, a);
  return hipGetLastError();
}

}  // namespace td
