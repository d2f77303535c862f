// The context behind the C ABI (ctx.cpp, prefix.cpp), host side only.
#pragma once

#include <cstdint>
#include <string>
#include <vector>

#include "node_bound.h"
#include "td_internal.h"

struct td_ctx {
  td_desc desc;
  td::DevState dev;
  int device = 0;
  std::vector<uint8_t> inited;         // per trie: initialised by init_prompt / load_state
  bool pending = false;                // leaves' K/V rows not yet stored in the pools
  std::vector<uint8_t> layer_written;  // per layer, while pending: LayerRows
  bool moves_pending = false;          // rows moved by the last compaction not yet copied
                                       //   (for the layers not yet written)
  std::vector<int32_t> leaf_depth;     // per trie: depth of its live leaves (mirrors the
                                       //   device header; tells which appends collect)
  std::vector<td::NodeBound> start;    // per trie: its size when it was initialised or loaded
  int splits_override = 0;             // TD_ATTN_SPLITS (tuning): WGs per attention unit
  // the shared prefix (td_set_prefix): as the device header has it, and the workspaces of its passes
  bool prefix = false;                 // attached
  int32_t prefix_length = 0, prefix_room = 0;
  int32_t* prefix_table = nullptr;     // device, room for prefix_table_cap entries and the padding
  size_t prefix_table_cap = 0;
  float* prefix_o = nullptr;           // records of a pass (PrefixArgs), and the tries' partials beside it
  float2* prefix_ml = nullptr;
  float* prefix_trie_part = nullptr;
  size_t prefix_records = 0, prefix_trie_floats = 0;
  hipEvent_t ev[4][2] = {};             // td_set_kernel_events: per td_phase, the
                                       //   kernel-timestamp events of its next run
  std::vector<void*> allocs;
  std::string err;
};

namespace td {

// Sets the context's message (that of td_error_string(NULL) without one) and returns st.
td_status fail(td_ctx* c, td_status st, const char* fmt, ...) __attribute__((format(printf, 3, 4)));
td_status hip_fail(td_ctx* c, hipError_t e, const char* what);
// Device memory of the context, freed by td_destroy.
template <typename T>
hipError_t reserve(td_ctx* c, T** p, size_t n) {
  void* q = nullptr;
  const hipError_t e = hipMalloc(&q, n * sizeof(T));
  if (e != hipSuccess) return e;
  c->allocs.push_back(q);
  *p = static_cast<T*>(q);
  return e;
}
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
// TD_ESTATE unless every trie is initialised.
td_status check_ready(td_ctx* c);
// Whether a layer's leaf rows are in the pools, and from which call: the attention's k_new / v_new, which
// may come again with the next call, or trie_store_kv, whose rotated rows they must not replace.
enum class LayerRows : uint8_t { kDue = 0, kAttended = 1, kStored = 2 };
// Marks the leaves' rows of layers [layer_begin, +n_layers) as stored.
void note_written(td_ctx* c, int layer_begin, int n_layers, LayerRows by);
// Copies the rows the last collection moved, for the layers of the range that are still due (ev0, ev1:
// the copy's events, both or neither).
hipError_t copy_due_rows(td_ctx* c, int layer_begin, int n_layers, hipStream_t st, hipEvent_t ev0, hipEvent_t ev1);

// The pass over the shared prefix for the tries' rows (prefix.cpp): leaves (q_max = b, no qslots) or
// stored nodes (queries q0 .. q0 + qn - 1 of each trie), at most max_splits splits.  trie_nodes > 0, a
// bound on the nodes of any trie whose rows are all stored: it may take the tries' own nodes too
// (*tries).  *splits: its records per row.
hipError_t prefix_pass(td_ctx* c, bool nodes, int layer_begin, int n_layers, int q0, int qn, int q_max,
                       const int32_t* d_qslots, const void* d_q, float scale_log2, int max_splits, long trie_nodes,
                       hipStream_t st, hipEvent_t ev0, int* splits, bool* tries);
// Whether an unsplit attention launch merges that many splits of records into its output itself (a:
// gets the records), which saves its partials and a launch.
bool prefix_fold(const td_ctx* c, AttnArgs& a, int splits);
// Else merges them with the tries' partials (a: of the attention launch, block_rows rows per block).
hipError_t prefix_merge(td_ctx* c, bool nodes, const AttnArgs& a, int splits, int block_rows, int q_max, hipStream_t st,
                        hipEvent_t ev1);

}  // namespace td
