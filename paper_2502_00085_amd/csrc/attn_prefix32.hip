// Attention over the shared prefix in fp32 (gfx950 fp32 matrix instructions).
//
// The contract and the row layout are those of k_attn_prefix (attn_prefix.hip): a wave holds 32
// packed query rows, a WG streams the keys of a split once for all of its rows, and each (row, split)
// leaves a record.  Both contractions run on v_mfma_f32_32x32x2_f32:
//
//   S^T[key][row] = K . Q^T    A = K rows (lane half hh holds half a row: one 16-byte LDS read feeds
//                              four steps), B = the query row, in registers
//   O^T[d][row]  += V^T . P^T  A = V from LDS (32 consecutive d of one key per half-wave), B = P^T,
//                              the S^T accumulators as they are
//
// What bounds it: the fp32 matrix rate.  A wave's tile of 32 keys is d products of 64 clocks (3.9 us
// at d = 128), far longer than its loads take: one LDS buffer per WG, and two WGs per CU, one of which
// multiplies while the other loads.  (A tile's V requested during its scores and the next one's K
// during its output measured 5 to 10 % slower; two accumulators in turn, no faster.)  1,024 rows of 8 KV
// heads over 4,096 keys at d = 128, 176 us (the least 173): 98 TFLOP/s of the 151 that a library product makes
// (matrix pipe busy 71 % of the CUs' clocks, 64 % of the launch's).
#include "attn_prefix.h"

namespace td {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kTile = 32;  // keys per wave and tile

template <int D, int RW, int KW>
struct Prefix32Cfg {
  static constexpr int THREADS = 64 * RW * KW;
  static constexpr int DT = D / 32;
  static constexpr int CPR = D / 4;              // 16-byte chunks per key row
  static constexpr int KEYS = kTile * KW;        // keys of a WG's tile: 32 per group of waves
  static constexpr int TILE = KEYS * D * 4;      // bytes of its K (or V) rows
  static constexpr int LOADS = TILE / 16 / THREADS;
  static_assert(TILE % (16 * THREADS) == 0, "a tile is a whole number of WG loads");
  static constexpr int WAVES = D <= 128 ? 2 : 1;  // per SIMD, as the registers allow
};

// Physical chunk of logical chunk c of key row r.  K: rotated by one chunk per row (the 16-byte reads
// of 8 rows use different banks).  V: by 128 bytes for every other group of four rows (the two
// half-waves read rows four apart).
template <int CPR>
__device__ inline int vchunk32(int r, int c) { return (c + 8 * ((r >> 2) & 1)) % CPR; }

// FOUR: the prefix is in 4 bits.  The next tile's blocks of 32 elements are in registers while a tile is
// multiplied, and are unpacked into the buffer once it has been read.
template <int D, int RW, int KW, bool FOUR>
__global__ __launch_bounds__(64 * RW * KW, (Prefix32Cfg<D, RW, KW>::WAVES)) void k_attn_prefix32(DevState s, PrefixArgs a) {
  using C = Prefix32Cfg<D, RW, KW>;
  using T4 = Tile4<D, C::THREADS, C::KEYS>;
  __shared__ __attribute__((aligned(16))) unsigned char kbuf[C::TILE], vbuf[C::TILE];
  __shared__ int wred[4 * RW];
  __shared__ float ml[KW == 2 ? RW * 128 : 1];
  const PrefixHdr p = s.prefix[FOUR ? 1 : 0];
  const PrefixUnit u = prefix_unit(s, a);
  const int lab = a.layer_begin + u.li;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rw = wave % RW, kw = wave / RW;
  const int col = lane & 31, hh = lane >> 5;

  const int r0 = u.rb * RW * 32;
  PrefixRow q = prefix_row(s, a, u.li, r0 + rw * 32 + col);
  // half hh of the lane's query row (loaded before anything is known of the row; a row that sees
  // nothing has no say)
  f32x4 qv[D / 8];
  {
    const f32x4* qp = reinterpret_cast<const f32x4*>(static_cast<const float*>(a.q) +
                                                     (q.at * s.Hq + u.g * (s.Hq / s.Hkv) + q.head) * D + hh * (D / 2));
#pragma unroll
    for (int k = 0; k < D / 8; ++k) qv[k] = qp[k];
  }
  PrefixSpan span, all;  // (of the wave; of the WG)
  const bool known = prefix_range(s, a, p, r0, RW * 32, &all);
  if (!known) {  // a window: from the rows' positions
    prefix_row_keys(s, a, p, q);
    span = prefix_span(q);
    all = prefix_range_of<RW>(span, rw, lane == 0 && kw == 0, wred);
  }
  const int lo = all.lo, hi = all.hi;
  // (splits hold whole 64-key tiles of pages, as in the bf16 pass; this WG's tiles are KEYS keys)
  const int first = hi > 0 ? lo / 64 : 0, tiles = hi > 0 ? (hi + 63) / 64 - first : 0;
  const int per = (tiles + a.splits - 1) / a.splits;
  const int b0 = (first + u.split * per) * 64, b1 = min(hi, min(first + tiles, first + (u.split + 1) * per) * 64);
  const int n_tiles = b1 > b0 ? (b1 - b0 + C::KEYS - 1) / C::KEYS : 0;

  const size_t head = ((size_t)lab * s.Hkv + u.g) << p.shift;
  const size_t page_rows = ((size_t)s.L * s.Hkv) << p.shift;
  const float* kpages = static_cast<const float*>(p.k);
  const float* vpages = static_cast<const float*>(p.v);
  // Load j of this thread writes 16-byte LDS chunk c = j THREADS + tid of the tile's K (and V): tile row
  // c / CPR, whose logical chunk kchunk (vchunk) it fetches
  auto geom = [&](int j, int t, int& r, int& kchunk, int& vchunk) __attribute__((always_inline)) {
    const int c = j * C::THREADS + t, pc = c % C::CPR;
    r = c / C::CPR;
    kchunk = (pc + C::CPR - r % C::CPR) % C::CPR;
    vchunk = (pc + C::CPR - 8 * ((r >> 2) & 1) % C::CPR) % C::CPR;
  };
  // (kept for a tile of consecutive rows, where there are registers for them)
  constexpr bool kHold = C::LOADS <= 8 && D <= 128;
  uint32_t kofs[kHold ? C::LOADS : 1], vofs[kHold ? C::LOADS : 1];
  if constexpr (kHold) {
#pragma unroll
    for (int j = 0; j < C::LOADS; ++j) {
      int r, kc, vc;
      geom(j, tid, r, kc, vc);
      kofs[j] = r * D + 4 * kc;
      vofs[j] = r * D + 4 * vc;
    }
  }
  auto load = [&](const float* src, unsigned char* dst, int j) __attribute__((always_inline)) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                     (__attribute__((address_space(3))) void*)(dst + (j * C::THREADS + wave * 64) * 16), 16, 0, 0);
  };
  auto issue = [&](int tile, const TilePages& pg) __attribute__((always_inline)) {
    const int tb = b0 + tile * C::KEYS;
    if (kHold && p.shift >= 6 && tb + C::KEYS <= hi) {  // (uniform) one page, no row past the end
      const size_t row = (size_t)pg.p[0] * page_rows + head + (tb & ((1 << p.shift) - 1));
#pragma unroll
      for (int j = 0; j < C::LOADS; ++j) {
        load(kpages + row * D + kofs[kHold ? j : 0], kbuf, j);
        load(vpages + row * D + vofs[kHold ? j : 0], vbuf, j);
      }
      return;
    }
#pragma unroll
    for (int j = 0; j < C::LOADS; ++j) {
      int t = tid, r, kc, vc;
      asm volatile("" : "+v"(t));  // (the geometry is recomputed per load, not held)
      geom(j, t, r, kc, vc);
      const int n = min(tb + r, hi - 1);  // (rows past the end: the last row)
      const int e = p.shift >= 6 ? 0 : (n - (tb & ~63)) >> p.shift;
      const int page = e == 0 ? pg.p[0] : e == 1 ? pg.p[1] : e == 2 ? pg.p[2] : pg.p[3];
      const size_t row = (size_t)page * page_rows + head + (n & ((1 << p.shift) - 1));
      load(kpages + row * D + 4 * kc, kbuf, j);
      load(vpages + row * D + 4 * vc, vbuf, j);
    }
  };
  auto pages_of = [&](int tile) __attribute__((always_inline)) { return tile_pages(p, (b0 + tile * C::KEYS) / 64); };

  T4 ahead;  // (4 bits) the tile under way
  auto fetch = [&](int tile, const TilePages& pg) __attribute__((always_inline)) {
    const int tb = b0 + tile * C::KEYS;
    fetch4<D, C::THREADS, C::KEYS>(p, pg, page_rows, head, tb, hi - 1 - tb, wave, ahead);
  };
  auto unpack = [&]() __attribute__((always_inline)) {
    using B = Blocks4<D, C::THREADS, C::KEYS>;
    typedef float f32x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int j = 0; j < B::PER; ++j) {
      if (!B::some(j, wave)) continue;
      const bool v = B::is_v(j, wave);
      const int b = B::number(j, v), row = b / B::BPR, blk = b % B::BPR;
      const float unit = __uint_as_float(ahead.scale[j] << 23);
      unsigned char* const dst = (v ? vbuf : kbuf) + row * (4 * D);
      const int rot = v ? 8 * ((row >> 2) & 1) : row % C::CPR;
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const uint32_t w = ahead.x[j][c / 2];
        const f32x2 y = c % 2 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, unit, 2) : __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, unit, 0);
        const f32x2 z = c % 2 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, unit, 3) : __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, unit, 1);
        *reinterpret_cast<f32x4*>(dst + (8 * blk + c + rot) % C::CPR * 16) = f32x4{y[0], y[1], z[0], z[1]};
      }
    }
  };
  TilePages next{};
  if (n_tiles > 0) {
    if constexpr (FOUR) fetch(0, pages_of(0));
    else issue(0, pages_of(0));
    if (n_tiles > 1) next = pages_of(1);
  }
  prefix_other_kind(s, p);
  if (known) {
    prefix_row_keys(s, a, p, q);
    span = prefix_span(q);
  }
  const float scale = a.scale_log2;
  float m = kPrefixNegBig, lsum = 0.0f;
  f32x16 o[C::DT];
#pragma unroll
  for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[dt][v] = 0.0f;

  // operand reads: K rows rotated by their number (krot + k, less CPR past the end); V by 128 bytes for
  // rows 4 .. 7, 12 .. 15, ..., which the second half-wave reads
  const unsigned char* krow = kbuf + (kTile * kw + col) * (D * 4);
  const uint32_t krot = (hh * (D / 8) + kTile * kw + col) % C::CPR;
  const unsigned char* vrow = vbuf + (kTile * kw + 4 * hh) * (D * 4) + col * 4;
  int voff[C::DT];
#pragma unroll
  for (int dt = 0; dt < C::DT; ++dt) voff[dt] = (dt + hh) % C::DT * 128;
  auto vat = [&](int dt, int v) __attribute__((always_inline)) {  // key 8 (v / 4) + 4 hh + v % 4, element 32 dt + col
    return *reinterpret_cast<const float*>(vrow + (8 * (v >> 2) + (v & 3)) * (D * 4) + voff[dt]);
  };
  // (the queries are there: else each tile's products would wait for them, and so for the tile under way)
  if constexpr (FOUR) __builtin_amdgcn_s_waitcnt(kWaitVmAll);
#pragma unroll 1
  for (int tile = 0; tile < n_tiles; ++tile) {
    if constexpr (FOUR) {
      if (tile > 0) __syncthreads();  // the tile before has been read
      unpack();
      if (tile + 1 < n_tiles) {
        fetch(tile + 1, next);
        if (tile + 2 < n_tiles) next = pages_of(tile + 2);
      }
    } else {
      if (tile > 0) {
        __syncthreads();  // the tile before has been read
        issue(tile, next);
        if (tile + 1 < n_tiles) next = pages_of(tile + 1);
      }
      __builtin_amdgcn_s_waitcnt(kWaitVmAll);
    }
    __syncthreads();
    const int tb = b0 + tile * C::KEYS + kTile * kw;  // this wave's 32 keys
    if (tb >= span.hi || tb >= b1 || tb + kTile <= span.lo) continue;  // (wave-uniform) no row sees them
    // a score's sum over d: pieces of 32 products from a fresh accumulator, added up
    f32x16 acc;
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[v] = 0.0f;
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      f32x16 piece;
#pragma unroll
      for (int v = 0; v < 16; ++v) piece[v] = 0.0f;
#pragma unroll
      for (int k = 4 * c; k < 4 * c + 4; ++k) {
        uint32_t at = krot + k;
        asm volatile("" : "+v"(at));  // (the offsets are recomputed per tile, not held)
        const f32x4 kk = *reinterpret_cast<const f32x4*>(krow + min(at, at - C::CPR) * 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) piece = __builtin_amdgcn_mfma_f32_32x32x2f32(kk[e], qv[k][e], piece, 0, 0, 0);
      }
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[v] += piece[v];
    }
    const bool cut = tb < span.all_lo || tb + kTile > span.all_hi || tb + kTile > b1;
    if (cut) {
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int n = tb + 8 * (v >> 2) + 4 * hh + (v & 3);
        acc[v] = ((n >= q.lo) & (n < q.hi) & (n < b1)) ? acc[v] : -INFINITY;
      }
    }
    float tmax = acc[0];
#pragma unroll
    for (int v = 1; v < 16; ++v) tmax = fmaxf(tmax, acc[v]);
    tmax = fmaxf(tmax, __shfl_xor(tmax, 32));
    const float mn = fmaxf(m, tmax * scale);
    const float alpha = __builtin_amdgcn_exp2f(m - mn);
    m = mn;
    float w[16], ps = 0.0f;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      w[v] = __builtin_amdgcn_exp2f(__builtin_fmaf(acc[v], scale, -mn));
      ps += w[v];
    }
    lsum = lsum * alpha + ps;
    if (__any(alpha != 1.0f)) {
#pragma unroll
      for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[dt][v] *= alpha;
    }
    if (cut) {
      // a hidden key weighs 0, but 0 times an infinite or NaN V is NaN: such a tile adds its
      // products key by key, to the rows that see the key
      bool odd = false;
#pragma unroll
      for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
        for (int v = 0; v < 16; ++v) odd |= !(fabsf(vat(dt, v)) < INFINITY);
      if (__any(odd)) {
#pragma unroll 1
        for (int i = 0; i < kTile; ++i) {
          const int n = tb + i, vi = (i >> 3) * 4 + (i & 3);
          float wi = 0.0f;
#pragma unroll
          for (int v = 0; v < 16; ++v) wi = v == vi ? w[v] : wi;
          wi = __shfl(wi, col + 32 * ((i >> 2) & 1));
          const bool own = n >= q.lo && n < q.hi && n < b1;
#pragma unroll
          for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
              const f32x4 x = *reinterpret_cast<const f32x4*>(vbuf + (kTile * kw + i) * (D * 4) +
                                                              vchunk32<C::CPR>(i, 8 * dt + 2 * q4 + hh) * 16);
#pragma unroll
              for (int e = 0; e < 4; ++e) o[dt][4 * q4 + e] += own ? wi * x[e] : 0.0f;
            }
        }
        continue;
      }
    }
    // (a tile's products from a fresh accumulator, then one addition: the rounding error of the
    // output grows with the tiles, not with the keys)
#pragma unroll
    for (int dt = 0; dt < C::DT; ++dt) {
      f32x16 f;
#pragma unroll
      for (int v = 0; v < 16; ++v) f[v] = 0.0f;
#pragma unroll
      for (int v = 0; v < 16; ++v) f = __builtin_amdgcn_mfma_f32_32x32x2f32(vat(dt, v), w[v], f, 0, 0, 0);
#pragma unroll
      for (int v = 0; v < 16; ++v) o[dt][v] += f[v];
    }
  }

  __syncthreads();  // every wave has read its last tile
  if constexpr (KW == 2) {
    // the second group hands its state over through LDS, lane by lane: half of O in each buffer
    static_assert(RW * 64 * (D / 4) * 4 <= C::TILE, "half of O fits a buffer");
    float* const o0 = reinterpret_cast<float*>(kbuf);
    float* const o1 = reinterpret_cast<float*>(vbuf);
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
    if (kw == 0) {
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
    __syncthreads();
  }

  // two waves at a time: a buffer of 32 keys (or more) holds a wave's rows
  lsum += __shfl_xor(lsum, 32);
#pragma unroll
  for (int turn = 0; turn < RW; turn += 2) {
    if (turn > 0) __syncthreads();
    if (kw == 0 && rw / 2 * 2 == turn)
      prefix_output<float, D>(s, a, u, q, lane, m, lsum, o, reinterpret_cast<float*>(rw % 2 ? vbuf : kbuf));
  }
}

template <int D, bool FOUR>
void launch_d(const DevState& s, const PrefixArgs& a, int rpb, hipStream_t st, hipEvent_t ev0, hipEvent_t ev1) {
  const dim3 grid(a.n_layers * s.Hkv * a.splits * a.row_blocks);
  if (rpb == 32) {
    if constexpr (D <= 128) hipExtLaunchKernelGGL((k_attn_prefix32<D, 1, 2, FOUR>), grid, dim3(128), 0, st, ev0, ev1, 0, s, a);
    else hipExtLaunchKernelGGL((k_attn_prefix32<D, 1, 1, FOUR>), grid, dim3(64), 0, st, ev0, ev1, 0, s, a);
  } else if (rpb == 64) {
    if constexpr (D <= 128) hipExtLaunchKernelGGL((k_attn_prefix32<D, 2, 2, FOUR>), grid, dim3(256), 0, st, ev0, ev1, 0, s, a);
    else hipExtLaunchKernelGGL((k_attn_prefix32<D, 2, 1, FOUR>), grid, dim3(128), 0, st, ev0, ev1, 0, s, a);
  } else {
    hipExtLaunchKernelGGL((k_attn_prefix32<D, 4, 1, FOUR>), grid, dim3(256), 0, st, ev0, ev1, 0, s, a);
  }
}

}  // namespace

hipError_t launch_prefix32(const DevState& s, const PrefixArgs& a, int rows_per_block, hipStream_t st, hipEvent_t ev0,
                           hipEvent_t ev1) {
  switch (s.D) {
#define PREFIX_CASE(DD)                                                       \
  case DD:                                                                    \
    if (!a.four) launch_d<DD, false>(s, a, rows_per_block, st, ev0, ev1);     \
    else return hipErrorInvalidValue;                                         \
    break;
    PREFIX_CASE(32) PREFIX_CASE(64) PREFIX_CASE(96) PREFIX_CASE(128)
    PREFIX_CASE(160) PREFIX_CASE(192)
#undef PREFIX_CASE
#define PREFIX_CASE(DD)                                                       \
  case DD:                                                                    \
    if (a.four) launch_d<DD, true>(s, a, rows_per_block, st, ev0, ev1);       \
    else launch_d<DD, false>(s, a, rows_per_block, st, ev0, ev1);             \
    break;
    PREFIX_CASE(224) PREFIX_CASE(256)
#undef PREFIX_CASE
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace td
