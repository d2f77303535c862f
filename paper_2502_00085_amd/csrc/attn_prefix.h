// What the passes over the shared prefix have in common (attn_prefix.hip, attn_prefix32.hip): the
// placement of the row blocks, a row's query and key range, the addresses of a tile's rows.
#pragma once

#include "mfma_tile.h"
#include "prefix.h"

namespace td {

constexpr float kPrefixNegBig = -1.0e30f;

// (layer of the pass, KV head), row block and split of a WG.  The row blocks that read the same keys
// lie 8 apart in the grid when xcd_group is set: on one XCD, whose L2 serves all but the first.  The
// last block first: in a causal pass it has the longest range.  With pair_blocks an XCD takes the longer half
// of its WGs longest first, then the shorter half shortest first, so that the two WGs of a CU make up
// about the same length together.
struct PrefixUnit {
  int li, g, rb, split;
};
__device__ inline PrefixUnit prefix_unit(const DevState& s, const PrefixArgs& a) {
  int x = blockIdx.x, rb;
  if (a.xcd_group && a.pair_blocks) {
    const int n = gridDim.x / 8, units = n / a.row_blocks, xcd = x % 8;
    int k = x / 8;
    if (k >= n / 2) k = n - 1 - (k - n / 2);
    rb = k / units;
    x = k % units * 8 + xcd;
  } else if (a.xcd_group) {
    const int xcd = x % 8, k = x / 8;
    rb = k % a.row_blocks;
    x = (k / a.row_blocks) * 8 + xcd;
  } else {
    rb = x % a.row_blocks;
    x /= a.row_blocks;
  }
  PrefixUnit u;
  u.rb = a.row_blocks - 1 - rb;
  u.split = x % a.splits;
  x /= a.splits;
  u.g = x % s.Hkv;
  u.li = x / s.Hkv;
  return u;
}

// Row r of a KV head: its owner, its query's place in q and out (in rows of Hq D elements; a row past
// the end: the first's), and the keys [lo, hi) it sees (none: a row past the end, an empty query, or
// a window past the prefix).
struct PrefixRow {
  uint32_t owner;
  int head, t, j;
  size_t at;
  bool in;  // r is a row of the pass
  int lo, hi;
};
__device__ inline PrefixRow prefix_row(const DevState& s, const PrefixArgs& a, int li, uint32_t r) {
  const uint32_t G = s.Hq / s.Hkv;
  PrefixRow q;
  q.owner = r / G;
  q.head = r - q.owner * G;
  q.in = q.owner < (uint32_t)(a.tries * a.per_trie);
  const uint32_t o = q.in ? q.owner : 0;
  q.t = a.tries == 1 ? 0 : o / (uint32_t)a.per_trie;
  q.j = a.q0 + o - q.t * a.per_trie;
  q.at = ((size_t)li * a.tries + q.t) * a.q_stride + q.j;
  q.lo = q.hi = 0;
  return q;
}
__device__ inline void prefix_row_keys(const DevState& s, const PrefixArgs& a, const PrefixHdr& p, PrefixRow& q) {
  if (!q.in) return;
  int pos, hi = p.length;
  if (a.rows == PrefixRows::kChunk) {
    pos = a.pos0 + q.j;
    hi = min(pos + 1, p.room);
  } else {
    const TrieHdr& h = s.hdr[q.t];
    if (a.rows == PrefixRows::kLeaves) {
      if (q.j >= h.n_live) return;
      pos = p.length + h.leaf_depth;
    } else {
      const int slot = a.qslots[(size_t)q.t * a.q_stride + q.j];
      if (slot < 0 || slot >= h.n_nodes) return;
      const size_t n = (size_t)q.t * s.cap + h.base + slot;
      if (s.mask[n] == 0ull) return;
      pos = p.length + s.depth[n];
    }
  }
  const int lo = s.W > 0 ? max(0, pos - s.W + 1) : 0;
  if (lo >= hi) return;
  q.lo = lo;
  q.hi = hi;
}

// Over the 32 rows of a wave that see keys: the first and last key any sees, the range all see.
struct PrefixSpan {
  int lo, hi, all_lo, all_hi;
};
__device__ inline PrefixSpan prefix_span(const PrefixRow& q) {
  const bool some = q.lo < q.hi;
  PrefixSpan w = {some ? q.lo : INT_MAX, some ? q.hi : 0, some ? q.lo : 0, some ? q.hi : INT_MAX};
  for (int o = 16; o > 0; o >>= 1) {
    w.lo = min(w.lo, __shfl_xor(w.lo, o));
    w.hi = max(w.hi, __shfl_xor(w.hi, o));
    w.all_lo = max(w.all_lo, __shfl_xor(w.all_lo, o));
    w.all_hi = min(w.all_hi, __shfl_xor(w.all_hi, o));
  }
  w.lo = __builtin_amdgcn_readfirstlane(w.lo);
  w.hi = __builtin_amdgcn_readfirstlane(w.hi);
  w.all_lo = __builtin_amdgcn_readfirstlane(w.all_lo);
  w.all_hi = __builtin_amdgcn_readfirstlane(w.all_hi);
  return w;
}

// The pages of a tile of 64 keys that starts at a multiple of 64: one of 64 keys or more, or up to
// four smaller ones, by scalar loads (the entries past the table's end are padding).
struct TilePages {
  int p[4];
};
__device__ inline TilePages tile_pages(const PrefixHdr& h, int tile) {
  typedef const __attribute__((address_space(4))) int32_t* cptr;
  const int first = h.shift >= 6 ? tile >> (h.shift - 6) : tile << (6 - h.shift);
  cptr e = (cptr)(uintptr_t)(h.table + first);
  TilePages t;
#pragma unroll
  for (int i = 0; i < 4; ++i) t.p[i] = e[i];
  return t;
}

// The keys [lo, hi) that some row of rows [r0, r0 + n) of a KV head sees, and [all_lo, all_hi) that all
// of them see (those that see any), where they are known without asking every row: causal rows
// follow one another, without a window every other row sees the whole prefix, and the leaves of a trie
// are of one depth (up to 8 tries in a block, whose headers come by scalar loads).
__device__ inline bool prefix_range(const DevState& s, const PrefixArgs& a, const PrefixHdr& p, int r0, int n, PrefixSpan* w) {
  *w = {0, p.length, 0, p.length};
  if (a.rows != PrefixRows::kChunk && s.W <= 0) return true;
  if (a.rows == PrefixRows::kNodes) return false;
  if (a.rows == PrefixRows::kLeaves) {
    const int per = a.per_trie * (s.Hq / s.Hkv), t0 = r0 / per, t1 = min((r0 + n - 1) / per, a.tries - 1);
    if (t1 - t0 >= 8) return false;
    int least = INT_MAX, most = INT_MIN;  // depths
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      typedef const __attribute__((address_space(4))) int32_t* cptr;
      const int depth = *(cptr)(uintptr_t)&s.hdr[min(t0 + i, t1)].leaf_depth;
      least = min(least, depth);
      most = max(most, depth);
    }
    w->lo = max(0, p.length + least - s.W + 1);
    w->all_lo = max(0, p.length + most - s.W + 1);
    if (w->lo >= w->hi) *w = {0, 0, 0, 0};
    return true;
  }
  const int G = s.Hq / s.Hkv, first = a.pos0 + a.q0 + r0 / G, last = a.pos0 + a.q0 + min((r0 + n - 1) / G, a.per_trie - 1);
  w->hi = min(last + 1, p.room);
  w->all_hi = min(first + 1, p.room);
  if (s.W > 0) {
    w->lo = max(0, first - s.W + 1);
    w->all_lo = max(0, last - s.W + 1);
  }
  if (w->lo >= w->hi) *w = {0, 0, 0, 0};
  return true;
}

// The same from the rows of RW waves (rw < RW; every thread calls it; red: 4 RW words).
template <int RW>
__device__ inline PrefixSpan prefix_range_of(const PrefixSpan& w, int rw, bool writes, int* red) {
  if (writes) {
    red[rw] = w.lo;
    red[RW + rw] = w.hi;
    red[2 * RW + rw] = w.all_lo;
    red[3 * RW + rw] = w.all_hi;
  }
  __syncthreads();
  PrefixSpan r = {INT_MAX, 0, 0, INT_MAX};
  for (int i = 0; i < RW; ++i) {
    r.lo = min(r.lo, red[i]);
    r.hi = max(r.hi, red[RW + i]);
    r.all_lo = max(r.all_lo, red[2 * RW + i]);
    r.all_hi = min(r.all_hi, red[3 * RW + i]);
  }
  r.lo = __builtin_amdgcn_readfirstlane(r.lo);
  r.hi = __builtin_amdgcn_readfirstlane(r.hi);
  r.all_lo = __builtin_amdgcn_readfirstlane(r.all_lo);
  r.all_hi = __builtin_amdgcn_readfirstlane(r.all_hi);
  return r;
}

// A wave's rows go out: 32 rows of O (lane: row col, elements 32 dt + 8 q4 + 4 hh .. + 3), transposed
// through `buf` (32 D floats of LDS that no other wave uses) so that a row is written in one piece.
// Rows of the pass only; a record without a key has no O.  T: the type of `out`.
template <typename T, int D>
__device__ inline void prefix_output(const DevState& s, const PrefixArgs& a, const PrefixUnit& u, const PrefixRow& q, int lane,
                                     float m, float lsum, const f32x16 (&o)[D / 32], float* buf) {
  constexpr int CH = D / 4;  // 16-byte chunks of a row, rotated by the row's number
  const int col = lane & 31, hh = lane >> 5, G = s.Hq / s.Hkv;
  const bool some = q.in && q.lo < q.hi && lsum != 0.0f;  // (a NaN sum is a NaN row)
  const bool record = a.part_o != nullptr;
  const float f = record ? 1.0f : some ? 1.0f / lsum : 0.0f;
  typedef float f32x4 __attribute__((ext_vector_type(4)));
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) {
      f32x4 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = record || some ? o[dt][4 * q4 + e] * f : 0.0f;
      *reinterpret_cast<f32x4*>(buf + col * D + (8 * dt + 2 * q4 + hh + col) % CH * 4) = x;
    }
  // where the row goes: its record, or its row of out (-1: nowhere)
  int64_t at = -1;
  if (record) {
    at = (((int64_t)u.li * a.tries * a.per_trie + q.owner) * s.Hq + u.g * G + q.head) * a.records + u.split;
    if (q.in && hh == 0) a.part_ml[at] = make_float2(some ? m : kPrefixNegBig, some ? lsum : 0.0f);
    if (!some) at = -1;
  } else if (q.in) {
    at = (int64_t)q.at * s.Hq + u.g * G + q.head;
  }
  const int alo = (int)at, ahi = (int)(at >> 32);
  if (record || sizeof(T) == 4) {
    float* const dst = record ? a.part_o : reinterpret_cast<float*>(a.out);
#pragma unroll 4
    for (int k = 0; k < 32 * CH / 64; ++k) {
      const int i = 64 * k + lane, row = i / CH, c = i % CH;
      const int64_t to = ((int64_t)__shfl(ahi, row) << 32) | (uint32_t)__shfl(alo, row);
      const f32x4 x = *reinterpret_cast<const f32x4*>(buf + row * D + (c + row) % CH * 4);
      if (to >= 0) *reinterpret_cast<f32x4*>(dst + to * D + 4 * c) = x;
    }
  } else {
    typedef T t8 __attribute__((ext_vector_type(8)));
#pragma unroll 2
    for (int k = 0; k < 32 * CH / 128; ++k) {
      const int i = 64 * k + lane, row = i / (CH / 2), c = i % (CH / 2);
      const int64_t to = ((int64_t)__shfl(ahi, row) << 32) | (uint32_t)__shfl(alo, row);
      const f32x4 x = *reinterpret_cast<const f32x4*>(buf + row * D + (2 * c + row) % CH * 4);
      const f32x4 y = *reinterpret_cast<const f32x4*>(buf + row * D + (2 * c + 1 + row) % CH * 4);
      t8 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        w[e] = (T)x[e];
        w[4 + e] = (T)y[e];
      }
      if (to >= 0) *reinterpret_cast<t8*>(static_cast<T*>(a.out) + to * D + 8 * c) = w;
    }
  }
}

}  // namespace td
