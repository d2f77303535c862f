// Attention over a shared prefix in 4 bits (gfx950 matrix cores, fp32 accumulate).
//
// The contract, the products and the softmax are those of k_attn_prefix (attn_prefix.hip); a key's values are its
// 4-bit sizes times the block's unit, exact in bf16, so that nothing is rounded on the way to the matrix cores.  A
// conversion makes two of them from a byte (v_cvt_scalef32_pk_bf16_fp4): 32 per lane for 32 keys of K or V at d = 128.
//
//   * More than 512 rows per KV head (a prefill): k_attn_prefix4, in blocks of up to 128 rows.  A tile is converted once
//     for all of them, on its way into LDS, and multiplied as a bf16 one.  Bound by the clock under matrix load, as
//     in bf16: 2,048 tokens from position 6,144 (8 KV heads, 32 query heads, d = 128) 237 us a layer, 1,012 TFLOP/s
//     (without a trace 232, 1,036; the bf16 prefix 241, a library product 1,252).
//   * Fewer (a decode step): k_attn_prefix4_few, in blocks of 32 rows.  HBM where the prefix is long: 8 rows of 32
//     KV heads, d = 96, over 50,001 positions 36.4 us, 4.5 TB/s (a copy's 4.9), 43.5 with the tries' nodes in the launch
//     (the bf16 pass 108 to 112).  Below some 4,000 keys per KV head a chain of latencies, as in bf16: 128 rows of 8 KV
//     heads over 4,096 keys, with the tries' nodes, 16.1 us (its 4.5 MB take 0.9, its records 2 to 3).
//   * fp32: the same kernel, the queries and the weights as three bf16 parts each (24 bits: all of them), three products
//     for one.  These run at 5 times the rate of the fp32 matrix instructions or more: 700 tokens from position
//     3,000 (32 heads, d = 128) 130 us against 520; 128 rows of 8 KV heads over 8,000 keys 23.6 against 80.
// Tried and not kept: eight waves per WG (the same to 1 %; more than 256 registers a wave past d = 128); one tile's loads
// under way instead of two, which the compiler made of them while the queries' loads were not waited for ahead of the
// loop (48.9 us for the 36.4 above).
#include <algorithm>
#include <type_traits>

#include "attn_prefix_wg.h"

namespace td {

namespace {

template <int D, int RW, int KW, bool TRIES>
__global__ __launch_bounds__(64 * RW * KW, (PrefixCfg<D, RW, KW>::WAVES)) void k_attn_prefix4(DevState s, PrefixArgs a) {
  constexpr int BUF = PrefixCfg<D, RW, KW>::BUF;
  __shared__ __attribute__((aligned(16))) unsigned char kbuf0[BUF], vbuf0[BUF];
  __shared__ __attribute__((aligned(16))) unsigned char kbuf1[BUF], vbuf1[BUF];
  __shared__ int wred[4 * RW];
  __shared__ float ml[KW == 2 ? RW * 128 : 1];
  if (TRIES && blockIdx.x >= a.prefix_wgs)
    prefix_wg<D, RW, KW, Wgs::kTries, false>(s, a, kbuf0, vbuf0, kbuf1, vbuf1, wred, ml);
  else prefix_wg<D, RW, KW, Wgs::kPrefix, true>(s, a, kbuf0, vbuf0, kbuf1, vbuf1, wred, ml);
}

// Blocks of 32 rows: no other wave of the WG needs a wave's keys.  (The row blocks of a KV head read and convert the same
// keys each for itself, from one XCD's L2 where they lie there: PrefixArgs::xcd_group.)  Each of the four waves of a
// WG streams tiles of 32 keys of its own, without a barrier until the end: K goes from memory to the first product's operand
// through registers alone (lane: half a row, as S^T = K Q^T takes it), V through 32 rows of LDS that the wave has
// for itself (written row by row, read transposed).  Two tiles are under way per wave.
constexpr int kFewWaves = 4;

template <int D>
struct FewCfg {
  static constexpr int KSTEPS = D / 16;  // 32x32x16 steps of S^T: 8 elements of a lane's half row
  static constexpr int DT = D / 32;
  static constexpr int CPR = D / 8;
  static constexpr int NBLK = D / 32;      // blocks (of 32 elements) per row
  static constexpr int NS = (NBLK + 1) / 2;  // blocks that half a row has a part of
  static constexpr int VBUF = 32 * D * 2;  // bytes of a wave's V rows
  static constexpr int WAVES = D <= 128 ? 2 : 1;  // per SIMD, as the registers allow
};

// Physical 16-byte chunk of logical chunk c of V row r: 16 rows written at one c, and the 4 rows that 16 lanes
// read transposed, lie in different banks (rows are 2 D bytes apart).
template <int D>
__device__ inline int few_chunk(int r, int c) {
  const int blk = c >> 2;
  const int b = D % 128 == 0 ? blk ^ (r & 3) : D % 64 == 0 ? blk ^ ((r >> 1) & 1) : blk;
  return 4 * b + ((c + (r >> 2)) & 3);
}

// Half a row of K or V, as loaded: nothing is taken apart before it is used (that would wait for the load).
template <int D>
struct HalfRow {
  static constexpr int NS = FewCfg<D>::NS;
  uint32_t x[D / 16];
  using Raw = std::conditional_t<NS == 1, uint8_t, std::conditional_t<NS == 4, uint32_t, uint16_t>>;
  Raw raw[NS == 3 ? 2 : 1];  // its scale bytes: four, two or one to a word
  __device__ uint32_t unit(int i) const {  // bits of 2^(byte i - 127)
    const uint32_t w = NS == 3 ? raw[i / 2] : raw[0];
    const int at = NS == 3 ? 8 * (i % 2) : 8 * i;
    return (at < 24 ? w << (23 - at) : w >> 1) & 0x7f800000u;
  }
};
typedef const TD_GLOBAL uint16_t __attribute__((aligned(1))) * global_u16;
typedef const TD_GLOBAL uint32_t __attribute__((aligned(1))) * global_u32;

template <int D>
__device__ inline void load_half(global_bytes rows, global_bytes scales, uint32_t row, int hh, HalfRow<D>& h) {
  const global_bytes x = rows + (row * (D / 2) + hh * (D / 4)), sc = scales + (row * (D / 32) + hh * (D / 64));
  if constexpr (D % 64 == 0) {
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      const u32x4 w = *(global_u32x4)(x + 16 * i);
#pragma unroll
      for (int e = 0; e < 4; ++e) h.x[4 * i + e] = w[e];
    }
  } else {
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      const u32x2 w = *(global_u32x2)(x + 8 * i);
      h.x[2 * i] = w[0];
      h.x[2 * i + 1] = w[1];
    }
  }
  constexpr int NS = FewCfg<D>::NS;
  if constexpr (NS == 1) {
    h.raw[0] = *sc;
  } else if constexpr (NS == 4) {
    h.raw[0] = *(global_u32)sc;
  } else {
    h.raw[0] = *(global_u16)sc;
    if constexpr (NS == 3) h.raw[1] = sc[2];
  }
}

// Elements 8 k .. 8 k + 7 of the half.
template <int D>
__device__ inline bf16x8 half_values(const HalfRow<D>& h, int hh, int k) {
  // (an odd number of blocks: the second half begins within one)
  const float unit = __uint_as_float(FewCfg<D>::NBLK % 2 == 0 ? h.unit(k / 4) : hh ? h.unit((k + 2) / 4) : h.unit(k / 4));
  const bf16x2 y0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(h.x[k], unit, 0), y1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(h.x[k], unit, 1);
  const bf16x2 y2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(h.x[k], unit, 2), y3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(h.x[k], unit, 3);
  return bf16x8{y0[0], y0[1], y1[0], y1[1], y2[0], y2[1], y3[0], y3[1]};
}

// The next 8 bits of x, in bf16; x keeps the rest.  Three in a row hold all of an fp32 number.
__device__ inline __bf16 take8(float& x) {
  const uint32_t u = __float_as_uint(x);
  x -= __uint_as_float(u & 0xffff0000u);
  return __builtin_bit_cast(__bf16, (uint16_t)(u >> 16));
}

// A lane's part of a query row as bf16 operands: in bf16 itself, in fp32 three parts of it (take8).
template <typename T, int D>
struct FewQuery {
  static constexpr int PARTS = sizeof(T) == 4 ? 3 : 1;
  bf16x8 x[PARTS][D / 16];
  __device__ void load(const T* row) {
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      if constexpr (PARTS == 1) {
        x[0][k] = reinterpret_cast<const bf16x8*>(row)[k];
      } else {
        typedef float f32x4 __attribute__((ext_vector_type(4)));
        const f32x4 a = reinterpret_cast<const f32x4*>(row)[2 * k], b = reinterpret_cast<const f32x4*>(row)[2 * k + 1];
        float rest[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
#pragma unroll
        for (int i = 0; i < PARTS; ++i)
#pragma unroll
          for (int e = 0; e < 8; ++e) x[i][k][e] = take8(rest[e]);
      }
    }
  }
};

template <typename T, int D>
__device__ __attribute__((always_inline)) inline void few_wg(const DevState& s, const PrefixArgs& a, unsigned char* vbuf, float* ml) {
  using C = FewCfg<D>;
  const PrefixHdr p = s.prefix[1];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, hh = lane >> 5;
  const PrefixUnit u = prefix_unit(s, a);
  const int lab = a.layer_begin + u.li;
  PrefixRow q = prefix_row(s, a, u.li, u.rb * 32 + col);  // (the same 32 rows in every wave)
  constexpr int PARTS = FewQuery<T, D>::PARTS;
  FewQuery<T, D> qv;
  qv.load(static_cast<const T*>(a.q) + (q.at * s.Hq + u.g * (s.Hq / s.Hkv) + q.head) * D + hh * (D / 2));
  PrefixSpan span, all;
  const bool known = prefix_range(s, a, p, u.rb * 32, 32, &all);
  if (!known) {
    prefix_row_keys(s, a, p, q);
    span = prefix_span(q);
    all = span;
  }
  // Tiles of 32 keys: of this split's share [t0, t1) the waves take [m0, m1), which every row sees whole, two
  // rounds at a time, and then the others, whose hidden keys need a mask.
  const int hi = all.hi, first = hi > 0 ? all.lo / 32 : 0, tiles = hi > 0 ? (hi + 31) / 32 - first : 0;
  const int per = (tiles + a.splits - 1) / a.splits;
  const int t0 = first + u.split * per, t1 = max(t0, min(first + tiles, t0 + per));
  const int m0 = min(max(t0, (all.all_lo + 31) / 32), t1);
  const int pairs = max(0, min(t1, all.all_hi / 32) - m0) / (2 * kFewWaves), m1 = m0 + pairs * 2 * kFewWaves;
  const int before = m0 - t0, cut = before + t1 - m1;
  const int mine = 2 * pairs + max(0, (cut - wave + kFewWaves - 1) / kFewWaves);  // tiles of this wave
  auto tile_of = [&](int i) __attribute__((always_inline)) {  // (past the last: the last)
    i = min(i, mine - 1);
    if (i < 2 * pairs) return m0 + i * kFewWaves + wave;
    i = (i - 2 * pairs) * kFewWaves + wave;
    return i < before ? t0 + i : m1 + i - before;
  };

  const size_t head = ((size_t)lab * s.Hkv + u.g) << p.shift;
  const size_t page_rows = ((size_t)s.L * s.Hkv) << p.shift;
  const global_bytes kx = to_global(p.k), vx = to_global(p.v), ksc = to_global(p.k_scale), vsc = to_global(p.v_scale);
  struct Pages {
    int p0, p1;
  };
  auto pages_of = [&](int tile) __attribute__((always_inline)) {
    typedef const __attribute__((address_space(4))) int32_t* cptr;
    const cptr e = (cptr)(uintptr_t)(p.table + (p.shift >= 5 ? tile >> (p.shift - 5) : 2 * tile));
    return Pages{e[0], e[1]};  // (past the end: padding)
  };
  auto fetch = [&](int tile, const Pages& pg, HalfRow<D>& k, HalfRow<D>& v) __attribute__((always_inline)) {
    const int tb = tile * 32;
    size_t row0 = (size_t)pg.p0 * page_rows + head;
    uint32_t row = min(col, hi - 1 - tb);  // (rows past the end: the last)
    if (p.shift >= 5) {  // (uniform)
      row0 += tb & ((1 << p.shift) - 1);
      load_half<D>(kx + row0 * (D / 2), ksc + row0 * (D / 32), row, hh, k);
      load_half<D>(vx + row0 * (D / 2), vsc + row0 * (D / 32), row, hh, v);
    } else {
      if (row >= 16) row0 = (size_t)pg.p1 * page_rows + head;
      row &= 15;
      load_half<D>(kx + row0 * (D / 2), ksc + row0 * (D / 32), row, hh, k);
      load_half<D>(vx + row0 * (D / 2), vsc + row0 * (D / 32), row, hh, v);
    }
  };
  HalfRow<D> k0, v0, k1, v1;
  Pages next{};
  if (mine > 0) {
    const Pages pg0 = pages_of(tile_of(0)), pg1 = pages_of(tile_of(1));
    fetch(tile_of(0), pg0, k0, v0);
    fetch(tile_of(1), pg1, k1, v1);
    next = pages_of(tile_of(2));
  }
  prefix_other_kind(s, p);
  if (known) {
    prefix_row_keys(s, a, p, q);
    span = prefix_span(q);
  }
  unsigned char* const vmine = vbuf + wave * C::VBUF;
  uint32_t vwrite[C::KSTEPS];
#pragma unroll
  for (int k = 0; k < C::KSTEPS; ++k) vwrite[k] = col * (2 * D) + few_chunk<D>(col, hh * (C::CPR / 2) + k) * 16;
  const int grp = lane >> 4, tm = (lane & 15) >> 2, tq = lane & 3;
  uint32_t vread[2][C::DT];  // rows 4 hh + tm and 8 more: every 16 rows alike
#pragma unroll
  for (int x = 0; x < 2; ++x)
#pragma unroll
    for (int dt = 0; dt < C::DT; ++dt) {
      const int n = 8 * x + 4 * hh + tm, c = 4 * dt + 2 * (grp & 1) + (tq >> 1);
      vread[x][dt] = n * (2 * D) + few_chunk<D>(n, c) * 16 + 8 * (tq & 1);
    }

  const float scale = a.scale_log2;
  float m = kPrefixNegBig, lsum = 0.0f;
  f32x16 o[C::DT];
#pragma unroll
  for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[dt][v] = 0.0f;
  const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};

  // tile i of the wave's
  auto step = [&](auto masked, int i, HalfRow<D>& k, HalfRow<D>& v) __attribute__((always_inline)) {
    constexpr bool CUT = decltype(masked)::value;
    const int tb = tile_of(i) * 32;
    bool odd = false;  // (a unit that is NaN, or makes a size infinite)
#pragma unroll
    for (int x = 0; x < C::NS; ++x) odd |= v.unit(x) >= 253u << 23;
#pragma unroll
    for (int x = 0; x < C::KSTEPS; ++x) *reinterpret_cast<bf16x8*>(vmine + vwrite[x]) = half_values<D>(v, hh, x);
    f32x16 acc;
#pragma unroll
    for (int x = 0; x < 16; ++x) acc[x] = 0.0f;
#pragma unroll
    for (int x = 0; x < C::KSTEPS; ++x) {
      const bf16x8 kk = half_values<D>(k, hh, x);
#pragma unroll
      for (int i = PARTS - 1; i >= 0; --i) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kk, qv.x[i][x], acc, 0, 0, 0);
    }
    // (unconditional where it matters: the wait for one tile's loads counts the other's)
    if (!CUT || i + 2 < mine) {
      fetch(tile_of(i + 2), next, k, v);
      next = pages_of(tile_of(i + 3));
    }
    const bool whole = !CUT || (tb >= span.all_lo && tb + 32 <= span.all_hi);  // (wave-uniform)
    if (!whole) {  // hidden scores become -inf
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        const int n = tb + 8 * (x >> 2) + 4 * hh + (x & 3);
        acc[x] = (n >= q.lo) & (n < q.hi) ? acc[x] : -INFINITY;
      }
    }
    // Probabilities of the lane's 16 keys, as in prefix_wg: in bf16 rounded, and summed as rounded; in fp32 in
    // three parts, like the queries.  The shift moves when they leave their range.
    float w[16];
    bf16x8 pb[PARTS][2];
    float ps = 0.0f;
    auto weights = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int x = 0; x < 16; ++x) w[x] = __builtin_amdgcn_exp2f(__builtin_fmaf(acc[x], scale, -m));
      ps = 0.0f;
      if constexpr (PARTS == 1) {
#pragma unroll
        for (int x = 0; x < 16; ++x) pb[0][x >> 3][x & 7] = (__bf16)w[x];
#pragma unroll
        for (int x = 0; x < 16; x += 2)
          ps = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{pb[0][x >> 3][x & 7], pb[0][x >> 3][(x & 7) + 1]}, ones, ps, false);
      } else {
#pragma unroll
        for (int x = 0; x < 16; ++x) ps += w[x];
      }
    };
    weights();
    if (__any(ps > kMost)) {
      float tmax = acc[0];
#pragma unroll
      for (int x = 1; x < 16; ++x) tmax = fmaxf(tmax, acc[x]);
      tmax = fmaxf(tmax, __shfl_xor(tmax, 32)) * scale;
      const float mn = tmax > m + kSlack ? tmax : m;
      const float alpha = __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      lsum *= alpha;
#pragma unroll
      for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
        for (int x = 0; x < 16; ++x) o[dt][x] *= alpha;
      weights();
    }
    lsum += ps;
    // 0 times an infinite or NaN V is NaN: a cut tile that holds such a V adds its products key by key, to
    // the rows that see the key
    if (!whole && __any(odd)) {
#pragma unroll 1
      for (int n = 0; n < 32; ++n) {
        const int vi = (n >> 3) * 4 + (n & 3);
        float wn = 0.0f;
#pragma unroll
        for (int x = 0; x < 16; ++x) wn = x == vi ? (PARTS == 1 ? (float)pb[0][x >> 3][x & 7] : w[x]) : wn;
        wn = __shfl(wn, col + 32 * ((n >> 2) & 1));
        const bool own = tb + n >= q.lo && tb + n < q.hi;
#pragma unroll
        for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            const bf16x4 x = *reinterpret_cast<const bf16x4*>(vmine + n * (2 * D) + few_chunk<D>(n, 4 * dt + q4) * 16 + 8 * hh);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[dt][4 * q4 + e] += own ? wn * (float)x[e] : 0.0f;
          }
      }
      return;
    }
    if constexpr (PARTS > 1) {
#pragma unroll
      for (int i = 0; i < PARTS; ++i)
#pragma unroll
        for (int x = 0; x < 16; ++x) pb[i][x >> 3][x & 7] = take8(w[x]);
    }
#pragma unroll
    for (int uu = 0; uu < 2; ++uu)
#pragma unroll
      for (int dt = 0; dt < C::DT; ++dt) {
        const unsigned char* vp = vmine + 16 * uu * (2 * D);
        const i16x4 p0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(vp + vread[0][dt]));
        const i16x4 p1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(vp + vread[1][dt]));
        const i16x8 x = __builtin_shufflevector(p0, p1, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
        for (int i = PARTS - 1; i >= 0; --i)
          o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), pb[i][uu], o[dt], 0, 0, 0);
      }
  };
  // (the queries and the first tiles are there: else the loop would wait for the queries, and with them for
  // every load, each time it multiplies)
  __builtin_amdgcn_s_waitcnt(kWaitVmAll);
  const bool empty = span.hi == 0;  // (no row is a query's, or sees a key)
  for (int i = empty ? 2 * pairs : 0; i < 2 * pairs; i += 2) {
    step(std::false_type{}, i, k0, v0);
    step(std::false_type{}, i + 1, k1, v1);
  }
  for (int i = empty ? mine : 2 * pairs; i < mine; i += 2) {
    step(std::true_type{}, i, k0, v0);
    if (i + 1 < mine) step(std::true_type{}, i + 1, k1, v1);
  }

  // the waves' states become one, two and two: O goes through LDS lane by lane
  static_assert(64 * (D / 2) * 4 == 2 * C::VBUF, "a wave's O takes two waves' V rows");
#pragma unroll
  for (int half = kFewWaves / 2; half >= 1; half >>= 1) {
    __syncthreads();  // (the buffers have been read)
    float* const part = reinterpret_cast<float*>(vbuf + (wave % half) * (2 * C::VBUF));
    if (wave >= half && wave < 2 * half) {
#pragma unroll
      for (int x = 0; x < D / 2; ++x) part[x * 64 + lane] = o[x / 16][x % 16];
      ml[(wave % half) * 128 + lane] = m;
      ml[(wave % half) * 128 + 64 + lane] = lsum;
    }
    __syncthreads();
    if (wave < half) {
      const float m1 = ml[wave * 128 + lane], l1 = ml[wave * 128 + 64 + lane];
      const float mn = fmaxf(m, m1);
      const float f0 = __builtin_amdgcn_exp2f(m - mn), f1 = __builtin_amdgcn_exp2f(m1 - mn);
      m = mn;
      lsum = lsum * f0 + l1 * f1;
#pragma unroll
      for (int x = 0; x < D / 2; ++x) o[x / 16][x % 16] = o[x / 16][x % 16] * f0 + part[x * 64 + lane] * f1;
    }
  }
  if (wave > 0) return;
  lsum += __shfl_xor(lsum, 32);
  prefix_output<T, D>(s, a, u, q, lane, m, lsum, o, reinterpret_cast<float*>(vbuf));
}

template <typename T, int D>
__global__ __launch_bounds__(64 * kFewWaves, (sizeof(T) == 4 && D == 128 ? 1 : FewCfg<D>::WAVES)) void k_attn_prefix4_few(DevState s, PrefixArgs a) {
  __shared__ __attribute__((aligned(16))) unsigned char vbuf[kFewWaves * FewCfg<D>::VBUF];
  __shared__ float ml[kFewWaves / 2 * 128];
  few_wg<T, D>(s, a, vbuf, ml);
}

// The same, and after prefix_wgs WGs those of the tries' own nodes, kFewTrieRows rows of a trie each.
template <int D>
__global__ __launch_bounds__(64 * kFewWaves, FewCfg<D>::WAVES) void k_attn_prefix4_few_tries(DevState s, PrefixArgs a) {
  using C = PrefixCfg<D, 2, 2>;
  static_assert(kFewTrieRows == 64, "two waves of 32 rows");
  static_assert(C::THREADS == 64 * kFewWaves && 2 * C::BUF == kFewWaves * FewCfg<D>::VBUF, "the same WG");
  __shared__ __attribute__((aligned(16))) unsigned char buf[2][C::BUF];
  __shared__ __attribute__((aligned(16))) unsigned char kbuf1[C::BUF], vbuf1[C::BUF];
  __shared__ int wred[8];
  __shared__ float ml[256];
  if (blockIdx.x >= a.prefix_wgs) prefix_wg<D, 2, 2, Wgs::kTries, false>(s, a, buf[0], buf[1], kbuf1, vbuf1, wred, ml);
  else few_wg<__bf16, D>(s, a, buf[0], ml);
}

template <int D>
void launch_d(const DevState& s, const PrefixArgs& a, int rpb, hipStream_t st, hipEvent_t ev0, hipEvent_t ev1) {
  const dim3 grid(a.n_layers * s.Hkv * (a.splits * a.row_blocks + a.tries * a.trie_blocks * a.trie_splits));
#define LAUNCH_PREFIX(RW, KW, TRIES) \
  hipExtLaunchKernelGGL((k_attn_prefix4<D, RW, KW, TRIES>), grid, dim3(64 * RW * KW), 0, st, ev0, ev1, 0, s, a)
  if constexpr (D == 64 || D == 96 || D == 128) {
    if (a.trie_splits > 0) {
      if (rpb == 32) hipExtLaunchKernelGGL(k_attn_prefix4_few_tries<D>, grid, dim3(64 * kFewWaves), 0, st, ev0, ev1, 0, s, a);
      else LAUNCH_PREFIX(4, 1, true);
      return;
    }
  }
  if (rpb == 32) {
    hipExtLaunchKernelGGL((k_attn_prefix4_few<__bf16, D>), grid, dim3(64 * kFewWaves), 0, st, ev0, ev1, 0, s, a);
    return;
  }
  if constexpr (D > 128) {  // (up to d = 128 more than 32 rows to a block are more than 512)
    if (rpb == 64) {
      LAUNCH_PREFIX(2, 2, false);
      return;
    }
  }
  LAUNCH_PREFIX(4, 1, false);
#undef LAUNCH_PREFIX
}

}  // namespace

hipError_t launch_prefix4(const DevState& s, const PrefixArgs& a, int rows_per_block, hipStream_t st, hipEvent_t ev0, hipEvent_t ev1) {
  if (s.dtype == TD_F32) {
    const dim3 grid(a.n_layers * s.Hkv * a.splits * a.row_blocks);
    switch (s.D) {
#define PREFIX_CASE(DD) \
  case DD: hipExtLaunchKernelGGL((k_attn_prefix4_few<float, DD>), grid, dim3(64 * kFewWaves), 0, st, ev0, ev1, 0, s, a); break;
      PREFIX_CASE(32) PREFIX_CASE(64) PREFIX_CASE(96) PREFIX_CASE(128)
      PREFIX_CASE(160) PREFIX_CASE(192)
#undef PREFIX_CASE
      default: return launch_prefix32(s, a, rows_per_block, st, ev0, ev1);
    }
    return hipGetLastError();
  }
  switch (s.D) {
#define PREFIX_CASE(DD) case DD: launch_d<DD>(s, a, rows_per_block, st, ev0, ev1); break;
    PREFIX_CASE(32) PREFIX_CASE(64) PREFIX_CASE(96) PREFIX_CASE(128)
    PREFIX_CASE(160) PREFIX_CASE(192) PREFIX_CASE(224) PREFIX_CASE(256)
#undef PREFIX_CASE
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace td
