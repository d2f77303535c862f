// What the stores of K/V rows have in common (kv_store.hip, kv_store4.hip): where the rows of a workgroup
// go, the position of each of their pairs, and the rotation of one unit of a head.
#pragma once

#include "attn_common.h"
#include "prefix.h"

namespace td {

constexpr int kStoreThreads = 256;
constexpr int kStoreRows = 8;    // rows of a WG at most
constexpr long kStoreMany = 1 << 22;  // rows of a layer from which on a WG has that many
constexpr int kStorePairs = 128;  // of a head

template <typename T>
struct StoreCfg {
  static constexpr int E = 16 / (int)sizeof(T);  // elements per 16-byte chunk
  typedef T vec __attribute__((ext_vector_type(16 / (int)sizeof(T))));
};

// Row r (trie, j) of a store: its own position (-1: no row) and its K/V row of KV head 0 (-1: none).
struct StoreRow {
  int position;
  int64_t dst;
};
__device__ inline StoreRow store_row(const DevState& s, const StoreArgs& a, const PrefixHdr& p, int lab, int r) {
  const int t = r / a.n, j = r % a.n;
  StoreRow w = {-1, -1};
  if (a.rows == PrefixRows::kChunk) {
    // (a captured call may find a shorter table than the one it was checked against, or pages of the
    // other kind)
    if (a.pos0 + j < p.room) {
      w.position = a.pos0 + j;
      const int64_t page = ((const TD_GLOBAL int32_t*)(uintptr_t)p.table)[w.position >> p.shift];
      w.dst = (((page * s.L + lab) * s.Hkv) << p.shift) + (w.position & ((1 << p.shift) - 1));
    } else {
      set_status(s.status, kDevEinval);
    }
    return w;
  }
  const TrieHdr h = s.hdr[t];
  int slot;
  if (a.rows == PrefixRows::kLeaves) slot = j < h.n_live ? h.n_nodes - h.n_live + j : -1;
  else slot = a.qslots[(size_t)t * a.n + j];
  if (slot >= 0 && slot < h.n_nodes) {
    const int at = h.base + slot;
    w.position = p.offset + (a.rows == PrefixRows::kLeaves ? h.leaf_depth : s.depth[(size_t)t * s.cap + at]);
    w.dst = (((int64_t)t * s.L + lab) * s.Hkv) * s.cap + at;
  }
  return w;
}

// The position that turns a pair of row r, whose own is `own`.
template <bool AXES>
__device__ inline double pair_position(const StoreArgs& a, int r, int own, int pair) {
  if constexpr (!AXES) return (double)own;
  const uint64_t w = pair < 64 ? (pair < 32 ? a.axis[0] : a.axis[1]) : (pair < 96 ? a.axis[2] : a.axis[3]);
  const int ax = (int)(w >> (2 * (pair & 31))) & 3;
  if (a.positions != nullptr) return (double)a.positions[(int64_t)r * a.n_axes + ax];
  return (double)own + (a.shift != nullptr ? (double)a.shift[(int64_t)(r / a.n) * a.n_axes + ax] : 0.0);
}

// Unit w of a head: E pairs of its first `rotary` elements, or 2 E copied ones, from src to out, which may
// be the same.  turn(pair): cosine and sine.  (Global accesses: a flat store, of an address chosen among pools,
// pages and q_out, also counts as one to LDS.)
template <typename T, typename Turn>
__device__ inline void store_unit(const T* src, T* out, int w, int turned, bool rotate, bool interleaved, Turn&& turn) {
  using C = StoreCfg<T>;
  using V = typename C::vec;
  constexpr int E = C::E;
  const bool split = rotate && !interleaved;
  const int c0 = split ? w : 2 * w, c1 = split ? w + turned : 2 * w + 1;
  const TD_GLOBAL V* const from = (const TD_GLOBAL V*)(uintptr_t)src;
  TD_GLOBAL V* const to = (TD_GLOBAL V*)(uintptr_t)out;
  const V x = from[c0], y = from[c1];
  V x1 = x, y1 = y;
  if (rotate) {
    if (split) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float2 f = turn(w * E + e);
        const float xe = (float)x[e], ye = (float)y[e];
        x1[e] = (T)(xe * f.x - ye * f.y);
        y1[e] = (T)(ye * f.x + xe * f.y);
      }
    } else {
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        const float2 f = turn(w * E + e / 2), g = turn(w * E + E / 2 + e / 2);
        const float xa = (float)x[e], xb = (float)x[e + 1], ya = (float)y[e], yb = (float)y[e + 1];
        x1[e] = (T)(xa * f.x - xb * f.y);
        x1[e + 1] = (T)(xb * f.x + xa * f.y);
        y1[e] = (T)(ya * g.x - yb * g.y);
        y1[e + 1] = (T)(yb * g.x + ya * g.y);
      }
    }
  }
  to[c0] = x1;
  to[c1] = y1;
}

}  // namespace td
