// The shared prefix: arguments of its attention pass and of the K/V stores, and the launchers.
#pragma once

#include "td_internal.h"

namespace td {

// Whose rows a prefix pass takes: the live leaves of every trie, stored nodes of every trie, or
// consecutive positions of the prefix itself (causal).
enum class PrefixRows { kLeaves, kNodes, kChunk };

// One pass over the prefix.  Row owner o in [0, tries * per_trie) is query q0 + o % per_trie of trie
// o / per_trie (kChunk: one "trie", whose query j sits at position pos0 + j); a row is a (owner,
// query head of one KV head) pair.  Each (row, split) leaves a record, number ((li * owners + o) * Hq +
// head) * records + split: D floats O at part_o, the shift m (log2 domain) and the sum l at part_ml.  A
// record with l = 0 (no key of the split) has no O.
struct PrefixArgs {
  const void* q;                    // [n_layers][tries][q_stride][Hq][D]
  float* part_o;                    // records, or null: out gets O / l (splits == 1)
  float2* part_ml;
  void* out;                        // as q
  const int32_t* qslots = nullptr;  // (kNodes) [tries][q_stride]
  PrefixRows rows;
  int layer_begin, n_layers;
  int tries, per_trie, q0, q_stride;
  int pos0 = 0;                     // (kChunk)
  float scale_log2;
  int row_blocks = 1, splits = 1;
  int records = 1;                  // per row: splits, and after them trie_splits
  int xcd_group = 0;                // row blocks of one (layer, KV head, split) on one XCD
  int pair_blocks = 0;              // (with it, kChunk) an XCD's WGs in an order that evens out its CUs
  // (kLeaves, bf16) the same launch takes the tries' own nodes too, all of which are stored: after
  // prefix_wgs WGs come those of (layer, trie, KV head, block of a trie's rows, split of its nodes)
  int trie_splits = 0, trie_blocks = 0;
  uint32_t prefix_wgs = 0;
};

// Query rows of a workgroup for a pass of this many rows per KV head.
int prefix_rows_per_block(long rows);
// Splits of `keys` keys for `units` (layer, KV head, row block) units, at most `most`.
int prefix_splits(const DevState& s, long units, long keys, long most);
hipError_t launch_prefix(const DevState& s, const PrefixArgs& a, hipStream_t st, hipEvent_t ev0, hipEvent_t ev1);
hipError_t launch_prefix32(const DevState& s, const PrefixArgs& a, int rows_per_block, hipStream_t st, hipEvent_t ev0,
                           hipEvent_t ev1);

// Merges a pass's records with those of the tries (attention partials of `splits` splits in blocks of
// block_rows rows, null: none) into out [n_layers][tries][per_trie][Hq][D].
struct PrefixMergeArgs {
  const float* prefix_o;
  const float2* prefix_ml;
  int prefix_splits;
  const float* trie;
  int trie_splits, block_rows, row_blocks;
  void* out;
  PrefixRows rows;
  int n_layers, tries, per_trie;
};
hipError_t launch_prefix_merge(const DevState& s, const PrefixMergeArgs& a, hipStream_t st, hipEvent_t ev1);

// Rotated K/V (and queries) into the pools of the tries or the pages of the prefix.
struct StoreArgs {
  const void *q, *k, *v;    // rows [n_layers][tries][n], k / v null: only the queries
  void* q_out;              // null: no queries
  const float* freq;        // [rotary / 2], null: no rotation
  const int32_t* qslots;    // (kNodes) [tries][n]
  PrefixRows rows;
  int layer_begin, n_layers, tries, n;
  int pos0;                 // (kChunk)
  int rotary, interleaved;
  int64_t q_stride, k_stride, v_stride;  // elements from one row to the next
};
hipError_t launch_store(const DevState& s, const StoreArgs& a, hipStream_t st);

}  // namespace td
