// What the passes over the shared prefix have in common (attn_prefix.hip, attn_prefix32.hip): the
// placement of the row blocks, a row's query and key range, the addresses of a tile's rows.
#pragma once

#include "mfma_tile.h"
#include "prefix.h"

namespace td {

constexpr float kPrefixNegBig = -1.0e30f;

// (layer of the pass, KV head), row block and split of a WG.  The row blocks that read the same keys
// lie 8 apart in the grid when xcd_group is set: on one XCD, whose L2 serves all but the first.  The
// last block first: in a causal pass it has the longest range.
struct PrefixUnit {
  int li, g, rb, split;
};
__device__ inline PrefixUnit prefix_unit(const DevState& s, const PrefixArgs& a) {
  int x = blockIdx.x, rb;
  if (a.xcd_group) {
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

// Row r of a KV head: its owner, its query's place in q and out (in rows of Hq D elements), and the
// keys [lo, hi) it sees (none: a row past the end, an empty query, or a window past the prefix).
struct PrefixRow {
  int owner, head;
  size_t at;
  bool in;  // r is a row of the pass
  int lo, hi;
};
__device__ inline PrefixRow prefix_row(const DevState& s, const PrefixArgs& a, const PrefixHdr& p, int li, int r) {
  const int G = s.Hq / s.Hkv;
  PrefixRow q;
  q.owner = r / G;
  q.head = r % G;
  q.in = q.owner < a.tries * a.per_trie;
  q.lo = q.hi = 0;
  const int t = q.in ? q.owner / a.per_trie : 0, j = a.q0 + (q.in ? q.owner % a.per_trie : 0);
  q.at = ((size_t)li * a.tries + t) * a.q_stride + j;
  if (!q.in) return q;
  int pos;
  if (a.rows == PrefixRows::kChunk) {
    pos = a.pos0 + j;
    q.hi = min(pos + 1, p.room);
  } else if (a.rows == PrefixRows::kLeaves) {
    const TrieHdr& h = s.hdr[t];
    if (j >= h.n_live) return q;
    pos = p.length + h.leaf_depth;
    q.hi = p.length;
  } else {
    const TrieHdr& h = s.hdr[t];
    const int slot = a.qslots[(size_t)t * a.q_stride + j];
    if (slot < 0 || slot >= h.n_nodes) return q;
    const size_t n = (size_t)t * s.cap + h.base + slot;
    if (s.mask[n] == 0ull) return q;
    pos = p.length + s.depth[n];
    q.hi = p.length;
  }
  q.lo = s.W > 0 ? max(0, pos - s.W + 1) : 0;
  if (q.lo >= q.hi) q.lo = q.hi = 0;
  return q;
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

// The record of a row (PrefixArgs::part).
__device__ inline float* prefix_record(const DevState& s, const PrefixArgs& a, const PrefixUnit& u, const PrefixRow& q) {
  const size_t row = ((size_t)u.li * a.tries * a.per_trie + q.owner) * s.Hq + u.g * (s.Hq / s.Hkv) + q.head;
  return a.part + (row * a.splits + u.split) * (s.D + 2);
}

}  // namespace td
