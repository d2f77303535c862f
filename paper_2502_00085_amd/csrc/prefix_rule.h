// The launch shape of a pass over the shared prefix, from what the host knows: rows per workgroup, splits of the
// keys, and whether the tries' own nodes go with the pass.  (The kernels take any shape; plain C++, so that the rules
// can be tested by themselves.)
#pragma once

#include <algorithm>

namespace td {

// A context's tries and heads, as far as the rules go.
struct PrefixHeads {
  int tries, q_heads, kv_heads, dim;
  bool f32;
};

constexpr long kOneRound = 512;   // WGs of a pass that run at once (two per CU)
constexpr long kTrieTiles = 8;
constexpr long kMostTrieTiles = 6;  // of a trie's WG beside a short 4-bit pass
constexpr long kShortPass = 16;   // tiles of the prefix per WG
constexpr int kFewTrieRows = 64;  // rows of a trie's WG beside a 4-bit pass in blocks of 32 rows

// A 4-bit pass takes its rows 32 at a time (k_attn_prefix4_few) in bf16 up to 512 of them and d = 128.  Measured
// against blocks of up to 128, us, with the splits below, 8 KV heads at d = 128 unless stated: 64 rows over 4,096
// keys 17.1 and 18.7, over 30,000 29.6 and 35; 128 rows 19.7 and 22.5, 40.3 and 42.6; 512 rows 30.7 and 33.1, over
// 20,000 77.9 and 75.3; 1,024 rows 43.4 and 43.2, 125 and 119; 32 KV heads, 128 rows over 20,000 73.4 and 87; at d = 256
// 256 rows over 20,000 99 and 69.  In fp32 any number up to d = 192, against the fp32 matrix instructions
// (k_attn_prefix32): d = 128, 128 rows over 8,000 45.6 and 104; d = 192, 4 KV heads, 57 and 84; d = 256, 116 and 102.
inline bool few_rows(const PrefixHeads& s, bool four, long rows) {
  return four && (s.f32 ? s.dim <= 192 : s.dim <= 128 && rows <= 512);
}
// Query rows of a workgroup for a pass of this many rows per KV head (four: over 4-bit pages).
inline int prefix_rows_per_block(const PrefixHeads& s, bool four, long rows) {
  if (few_rows(s, four, rows)) return 32;
  return rows <= 32 ? 32 : rows <= 64 ? 64 : 128;
}

// Splits of `keys` keys for `units` (layer, KV head, row block) units, at most `most` (four: over 4-bit pages, in blocks
// of 32 rows).
//
// A WG per CU, of at least 4 tiles of 64 keys; two per CU where each still has 16.  More splits make
// shorter chains of tiles and more records to merge.  Measured, 8 KV heads at d = 128, the pass and
// its merge, us: 128 rows over 4,096 keys, 8 / 16 / 32 splits: 22.6 / 20.9 / 24.6; over 16,384 keys, 16 /
// 32 / 64: 35.1 / 30.5 / 34.1; 1,024 rows (8 blocks) over 1,024 keys, 4 / 8: 25.5 / 27.7; over 8,192 keys,
// 4 / 8 / 16: 63 / 57 / 72; 32 rows over 4,096 keys, 16 / 32 / 64: 17.4 / 17.9 / 20.1.  In fp32 a tile takes
// ten times as long: one tile, and two per CU where each still has 2.
//
// In 4 bits (blocks of 32 rows, d <= 128) a record costs as much as before and a tile a quarter of the memory's
// time: of at least 6 tiles where 16 units or more write records, and two per CU where each still has 64.  us:
// 32 rows over 4,096 keys, 4 / 8 / 16 / 32 splits: 21.3 / 16.4 / 16.6 / 21.3; 64 rows, 4 / 8 / 12 / 16: 19.3 /
// 17.1 / 17.5 / 21.2; 128 rows, 4 / 6 / 8 / 12: 19.7 / 19.9 / 21.5 / 22.6, over 30,000, 4 / 8 / 16: 59 / 40.3 / 45.3; 32
// KV heads, 8 rows over 30,000, 4 / 8 / 16: 60.5 / 39.3 / 42.8; 128 rows over 20,000 (313 tiles), 2 / 4: 85 / 73.4.
inline int prefix_splits(const PrefixHeads& s, bool four, long units, long keys, long most) {
  const long tiles = (keys + 63) / 64;
  if (few_rows(s, four, 0)) {
    const long least = units < 16 ? 4 : 6;
    const long one = std::min(256 / units, (tiles + least - 1) / least);
    const long two = s.f32 && s.dim >= 128 ? 0 : std::min(512 / units, tiles / 64);  // (fp32: one fits a CU)
    return (int)std::max(1l, std::min(std::max(one, two), most));
  }
  const long few = s.f32 ? 1 : 4, many = s.f32 ? 2 : 16;
  const long one = std::min((256 + units - 1) / units, tiles / few), two = std::min((512 + units - 1) / units, tiles / many);
  return (int)std::max(1l, std::min(std::max(one, two), most));
}

// Whether (layer, KV head, split) triples come in eights, one to an XCD: what PrefixArgs::xcd_group needs.
inline bool prefix_xcd_eights(int n_layers, int kv_heads, int splits) { return (long)n_layers * kv_heads * splits % 8 == 0; }

// In 4 bits, row blocks that read the same keys belong on one XCD, if that costs less than a fifth of the splits (us, over
// 30,000 positions: 16 beams, 4 KV heads, d = 64, 30 splits 20.1, 31 21.5; 8 x 16 beams, 28 heads and 4 KV heads, d = 128,
// 97.5 and 124.6; 8 x 16 beams of 6 heads, d = 96, 8 splits 38.7, 10 36.3).
inline int prefix_grouped_splits(bool four, int n_layers, int kv_heads, int row_blocks, int splits) {
  for (int i = splits; four && row_blocks > 1 && 5 * i > 4 * splits; --i)
    if (prefix_xcd_eights(n_layers, kv_heads, i)) return i;
  return splits;
}

struct PassShape {
  int row_blocks = 1, splits = 1;
  int xcd_group = 0;
  int trie_splits = 0, trie_blocks = 0;  // of the tries' own nodes in the same launch (0: not in it)
  long prefix_wgs = 0;                   // (with them) WGs of the pass
};
// A pass of per_trie queries of every trie over `keys` keys, in at most `most` splits; a row has room for `fit`
// records.  trie_nodes > 0: the tries' own nodes, at most as many in each, may go with it.
inline PassShape prefix_pass_shape(const PrefixHeads& s, bool four, int n_layers, int per_trie, long keys, long fit, int most,
                                   long trie_nodes) {
  PassShape a;
  const int G = s.q_heads / s.kv_heads;
  const long rows = (long)s.tries * per_trie * G;
  const int rpb = prefix_rows_per_block(s, four, rows);
  const bool few = four && rpb == 32;
  a.row_blocks = (int)((rows + rpb - 1) / rpb);
  const long unit = (long)n_layers * s.kv_heads * a.row_blocks;
  auto grouped = [&](int splits) { return prefix_grouped_splits(four, n_layers, s.kv_heads, a.row_blocks, splits); };
  a.splits = grouped(prefix_splits(s, few, unit, keys, std::min<long>(fit, most)));
  if (trie_nodes > 0) {
    // the tries' own nodes in the same launch, where all of its WGs run at once, none has more than
    // kTrieTiles tiles of a trie, and the pass itself is short.  Measured over 210 shapes (1 to 16 tries of 2 to
    // 32 beams and 40 to 5,000 nodes, 64 to 50,000 positions, d = 64 to 128; graphs of one-layer calls): within
    // these limits 21 % less time than with launches of their own (4 x 8 beams of 266 nodes over 4,096
    // positions 22.1 us a layer against 30.3), at worst 4 % more (2 x 32 of 229 over 64: 21.9, 21.1).  Past
    // kTrieTiles, 11 % less to 12 % more.  The other two limits keep away from what was not measured, calls of
    // many layers, and cost one-layer calls past them 7 % (2 x 4 beams of 404 nodes over 50,000 positions, 32 KV
    // heads, 49 tiles of the prefix per WG: 117.8, 127.2).  In 4 bits the pass may be long: 8 rows of 32 KV heads
    // over 30,000 positions 38.9 us in one launch of 8 or 12 splits, 42.7 in two of 16.
    // A trie's WG has 3 of its tiles, which take about as long as the 4 that a WG of the prefix has at least:
    // over 160 of these shapes 1 or 2 took 1.4 % less in the mean, 4 took 4 % more, 6 8 %, 8 13 %.
    const long tiles = (trie_nodes + 63) / 64, prefix_tiles = (keys + 63) / 64;
    const int tr = few ? kFewTrieRows : rpb;  // a trie's rows of a WG
    const long blocks = ((long)per_trie * G + tr - 1) / tr, units = (long)n_layers * s.tries * s.kv_heads * blocks;
    long ts = std::max(1l, std::min({(tiles + 2) / 3, 256 / units, fit - a.splits}));
    // In 4 bits and blocks of 32 rows a short pass leaves CUs to the tries (128 rows over 4,096 keys, 6 splits 19.9 us, 8
    // 21.5; 64 rows over 8,000, 14 22.8, 16 25.1; 8 rows of 32 KV heads, d = 96, over 8,000, 21 tiles per WG, 6 23.8, 8
    // 22.5).  Where that would leave it too few to be short, a trie's WGs have up to 6 tiles instead (4 x 8 beams over
    // 4,096 keys, 4 layers, 14 tiles of a trie: 8 splits beside 5 88.9 us, 4 beside 4 83.5, 4 beside 5 88.6; 64 rows
    // of 8 KV heads over 2,500 23.0 and 20.0; 287 captured one-layer calls of 1 to 8 tries over 1,000 to 16,000 keys: 15 %
    // less to 3 % more; with up to 9 tiles up to 42 % more, with up to 4 a quarter of the gain), and past that it keeps
    // its splits.
    int splits = a.splits;  // (of a pass that the tries join; alone it keeps its own)
    const long least = (prefix_tiles + kShortPass - 1) / kShortPass;  // splits of a short pass
    long left = std::max(0l, 256 - units * ts) / unit;
    if (few && left < least && least < splits) {
      const long fewer = (256 - unit * least) / units;
      if (fewer >= 1 && tiles <= kMostTrieTiles * fewer) {
        ts = fewer;
        left = (256 - units * ts) / unit;
      }
    }
    if (few && least <= left && left < splits) splits = grouped((int)left);
    const long wgs = unit * splits;
    if (wgs + units * ts <= kOneRound && (four || prefix_tiles <= kShortPass * splits) && (tiles + ts - 1) / ts <= kTrieTiles &&
        splits + ts <= fit) {
      a.splits = splits;
      a.trie_splits = (int)ts;
      a.trie_blocks = (int)blocks;
      a.prefix_wgs = wgs;
    }
  }
  a.xcd_group = a.row_blocks > 1 && prefix_xcd_eights(n_layers, s.kv_heads, a.splits);
  return a;
}

}  // namespace td
