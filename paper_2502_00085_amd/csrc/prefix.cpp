// Host side of the shared prefix: attaching it, the K/V stores, its passes.
#include "prefix.h"

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "ctx.h"

using td::aligned16;
using td::fail;
using td::hip_fail;
using td::reserve;

namespace {

// Records an attention launch merges by itself, one after the other: more are merged by a launch of
// their own, eight at a time.
constexpr int kFoldSplits = 4;
constexpr long kOneRound = 512;  // WGs of a pass that run at once (two per CU)
constexpr long kTrieTiles = 8;
constexpr long kShortPass = 16;  // tiles of the prefix per WG
constexpr int kStoreRows = 1 << 26;  // rows per layer of a store (what a launch's grid holds)
constexpr size_t kWorkFloats = 16u << 20;  // of either workspace, unless one layer needs more

td_status bad_layers(td_ctx* c, int layer_begin, int n_layers) {
  if (n_layers < 1 || layer_begin < 0 || n_layers > c->dev.L || layer_begin > c->dev.L - n_layers)
    return fail(c, TD_EINVAL, "layer range [%d, +%d) outside [0, %d)", layer_begin, n_layers, c->dev.L);
  return TD_OK;
}

// The context's device is the current one (its memory is there, and so are the kernels).
td_status other_device(td_ctx* c) {
  int d = 0;
  const hipError_t e = hipGetDevice(&d);
  if (e != hipSuccess) return hip_fail(c, e, "hipGetDevice");
  if (d != c->device) return fail(c, TD_EINVAL, "the context lives on device %d, the current one is %d", c->device, d);
  return TD_OK;
}

// The arguments that the two stores share.
td_status store_args(td_ctx* c, const td_rope* rope, const void* q, int64_t qs, const void* k, int64_t ks, const void* v,
                     int64_t vs, void* q_out, td::StoreArgs* a) {
  const td::DevState& s = c->dev;
  if ((q == nullptr) != (q_out == nullptr) || (k == nullptr) != (v == nullptr) || (!q && !k))
    return fail(c, TD_EINVAL, "pass q with q_out, k with v, and at least one of the pairs");
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_out))
    return fail(c, TD_EINVAL, "q, k, v and q_out must be 16-byte aligned");
  const int64_t qr = (int64_t)s.Hq * s.D, kr = (int64_t)s.Hkv * s.D;
  a->q_stride = qs ? qs : qr;
  a->k_stride = ks ? ks : kr;
  a->v_stride = vs ? vs : kr;
  if (a->q_stride < qr || a->k_stride < kr || a->v_stride < kr || a->q_stride % 8 || a->k_stride % 8 || a->v_stride % 8)
    return fail(c, TD_EINVAL, "row strides must be at least heads * head_dim and multiples of 8");
  if (q && q == q_out && a->q_stride != qr) return fail(c, TD_EINVAL, "q_out may be q only where q is contiguous");
  if (rope) {
    if (!rope->d_freq || rope->dim < 16 || rope->dim > s.D || rope->dim % 16)
      return fail(c, TD_EINVAL, "rope: d_freq must be non-null and dim a multiple of 16 in [16, head_dim]");
    if (rope->interleaved != 0 && rope->interleaved != 1) return fail(c, TD_EINVAL, "rope: interleaved must be 0 or 1");
    a->freq = rope->d_freq;
    a->rotary = rope->dim;
    a->interleaved = rope->interleaved;
  }
  a->q = q;
  a->k = k;
  a->v = v;
  a->q_out = q_out;
  return TD_OK;
}

}  // namespace

namespace td {

hipError_t prefix_pass(td_ctx* c, bool nodes, int layer_begin, int n_layers, int q0, int qn, int q_max,
                       const int32_t* d_qslots, const void* d_q, float scale_log2, int max_splits, long trie_nodes,
                       hipStream_t st, hipEvent_t ev0, int* splits, bool* tries) {
  const DevState& s = c->dev;
  PrefixArgs a{};
  a.q = d_q;
  a.part_o = c->prefix_o;
  a.part_ml = c->prefix_ml;
  a.qslots = d_qslots;
  a.rows = nodes ? PrefixRows::kNodes : PrefixRows::kLeaves;
  a.layer_begin = layer_begin;
  a.n_layers = n_layers;
  a.tries = s.T;
  a.per_trie = qn;
  a.q0 = q0;
  a.q_stride = q_max;
  a.scale_log2 = scale_log2;
  const long rows = (long)s.T * qn * (s.Hq / s.Hkv);
  const int rpb = prefix_rows_per_block(rows);
  a.row_blocks = (int)((rows + rpb - 1) / rpb);
  const long keys = s.W > 0 ? std::min(c->prefix_length, s.W) : c->prefix_length;
  const long fit = (long)(c->prefix_records / ((size_t)n_layers * s.T * qn * s.Hq));
  a.splits = prefix_splits(s, (long)n_layers * s.Hkv * a.row_blocks, keys, std::min<long>(fit, max_splits));
  a.xcd_group = a.row_blocks > 1 && ((long)n_layers * s.Hkv * a.splits) % 8 == 0;
  a.records = a.splits;
  *tries = false;
  if (trie_nodes > 0) {
    // the tries' own nodes in the same launch, where all of its WGs run at once, none has more than
    // kTrieTiles tiles of a trie, and the pass itself is short.  Measured over 210 shapes (1 to 16 tries of 2 to
    // 32 beams and 40 to 5,000 nodes, 64 to 50,000 positions, d = 64 to 128; graphs of one-layer calls): within
    // these limits 21 % less time than with launches of their own (4 x 8 beams of 266 nodes over 4,096
    // positions 22.1 us a layer against 30.3), at worst 4 % more (2 x 32 of 229 over 64: 21.9, 21.1).  Past
    // kTrieTiles, 11 % less to 12 % more.  The other two limits keep away from what was not measured, calls of
    // many layers, and cost one-layer calls past them 7 % (2 x 4 beams of 404 nodes over 50,000 positions, 32 KV
    // heads, 49 tiles of the prefix per WG: 117.8, 127.2).
    // A trie's WG has 3 of its tiles, which take about as long as the 4 that a WG of the prefix has at least:
    // over 160 of these shapes 1 or 2 took 1.4 % less in the mean, 4 took 4 % more, 6 8 %, 8 13 %.
    const long wgs = (long)n_layers * s.Hkv * a.row_blocks * a.splits, tiles = (trie_nodes + 63) / 64;
    const long blocks = (qn * (s.Hq / s.Hkv) + rpb - 1) / rpb, units = (long)n_layers * s.T * s.Hkv * blocks;
    const long ts = std::max(1l, std::min({(tiles + 2) / 3, 256 / units, fit - a.splits}));
    if (wgs + units * ts <= kOneRound && (keys + 63) / 64 <= (long)kShortPass * a.splits && (tiles + ts - 1) / ts <= kTrieTiles && a.splits + ts <= fit) {
      a.trie_splits = (int)ts;
      a.trie_blocks = (int)blocks;
      a.prefix_wgs = (uint32_t)wgs;
      a.records = a.splits + a.trie_splits;
      *tries = true;
    }
  }
  *splits = a.records;
  return launch_prefix(s, a, st, ev0, nullptr);
}

bool prefix_fold(const td_ctx* c, AttnArgs& a, int splits) {
  a.prefix_o = nullptr;
  if (a.splits > 1 || splits > kFoldSplits) return false;
  a.prefix_o = c->prefix_o;
  a.prefix_ml = c->prefix_ml;
  a.prefix_splits = splits;
  return true;
}

hipError_t prefix_merge(td_ctx* c, bool nodes, const AttnArgs& a, int splits, int block_rows, int q_max, hipStream_t st,
                        hipEvent_t ev1) {
  PrefixMergeArgs m{};
  m.prefix_o = c->prefix_o;
  m.prefix_ml = c->prefix_ml;
  m.prefix_splits = splits;
  m.trie = a.prefix_tries ? nullptr : c->prefix_trie_part;
  m.trie_splits = a.splits;
  m.block_rows = block_rows;
  m.row_blocks = a.row_blocks32;
  m.out = a.out;
  m.rows = nodes ? PrefixRows::kNodes : PrefixRows::kLeaves;
  m.n_layers = a.n_layers;
  m.tries = c->dev.T;
  m.per_trie = q_max;
  return launch_prefix_merge(c->dev, m, st, ev1);
}

}  // namespace td

extern "C" {

static td_status set_prefix(td_ctx* c, const td_prefix* d) {
  const td::DevState& s = c->dev;
  td::PrefixHdr h;
  std::vector<int32_t> table;
  if (d) {
    if (!d->k_pages || !d->v_pages || !aligned16(d->k_pages) || !aligned16(d->v_pages))
      return fail(c, TD_EINVAL, "k_pages / v_pages must be non-null and 16-byte aligned");
    if (d->n_pages < 1 || !d->h_page_table || d->n_table < 1 || d->n_table > d->n_pages)
      return fail(c, TD_EINVAL, "need n_pages >= 1 and a page table of 1 .. n_pages entries");
    if (d->page_size < 16 || d->page_size > 65536 || (d->page_size & (d->page_size - 1)))
      return fail(c, TD_EINVAL, "page_size must be a power of two in [16, 65536]");
    const int64_t room = (int64_t)d->n_table * d->page_size;
    if (room > (1 << 30)) return fail(c, TD_EINVAL, "the page table holds more than 2^30 positions");
    if (d->length < 0 || d->length > room) return fail(c, TD_EINVAL, "prefix length must be in [0, n_table * page_size]");
    table.assign(d->h_page_table, d->h_page_table + d->n_table);
    for (int32_t i = 0; i < d->n_table; ++i)
      if (table[i] < 0 || table[i] >= d->n_pages)
        return fail(c, TD_EINVAL, "page table entry %d: page %d outside [0, %d)", i, table[i], d->n_pages);
    std::vector<int32_t> sorted(table);
    std::sort(sorted.begin(), sorted.end());
    const auto twice = std::adjacent_find(sorted.begin(), sorted.end());
    if (twice != sorted.end()) return fail(c, TD_EINVAL, "page table: page %d is listed twice", *twice);
    table.insert(table.end(), td::kPrefixTablePad, table[0]);
    h.k = d->k_pages;
    h.v = d->v_pages;
    h.length = d->length;
    h.room = (int32_t)room;
    while ((1 << h.shift) < d->page_size) ++h.shift;
  }
  if (td_status r = other_device(c)) return r;
  hipError_t e = hipDeviceSynchronize();
  if (d) {
    if (e == hipSuccess && table.size() > c->prefix_table_cap) {
      // (room to grow; what a captured call may still read is kept until td_destroy)
      e = reserve(c, &c->prefix_table, 2 * table.size());
      if (e == hipSuccess) c->prefix_table_cap = 2 * table.size();
    }
    if (e == hipSuccess && c->prefix_records == 0) {
      const size_t G = s.Hq / s.Hkv, rows = std::max<size_t>(s.b * G, 128), heads = (size_t)s.T * s.Hkv;
      const size_t records = std::max(kWorkFloats / s.D, heads * rows);
      const size_t trie_floats = std::max(kWorkFloats, heads * ((rows + 31) / 32 * 32) * (s.D + 2));
      e = reserve(c, &c->prefix_o, records * s.D);
      if (e == hipSuccess) e = reserve(c, &c->prefix_ml, records);
      if (e == hipSuccess) e = reserve(c, &c->prefix_trie_part, trie_floats);
      if (e == hipSuccess) {
        c->prefix_records = records;
        c->prefix_trie_floats = trie_floats;
      }
    }
    if (e == hipSuccess) e = hipMemcpy(c->prefix_table, table.data(), table.size() * 4, hipMemcpyHostToDevice);
    h.table = c->prefix_table;
  }
  if (e == hipSuccess) e = hipMemcpy(s.prefix, &h, sizeof h, hipMemcpyHostToDevice);
  if (e != hipSuccess) return hip_fail(c, e, "td_set_prefix");
  c->prefix = d != nullptr;
  c->prefix_length = h.length;
  c->prefix_room = h.room;
  return TD_OK;
}

td_status td_set_prefix(td_ctx* c, const td_prefix* d) {
  if (!c) return TD_EINVAL;
  c->err.clear();
  try {
    return set_prefix(c, d);
  } catch (const std::bad_alloc&) {  // (the table's copy)
    return fail(c, TD_EINVAL, "out of host memory for the page table");
  }
}

td_status trie_prefix_store(td_ctx* c, int32_t layer_begin, int32_t n_layers, int32_t pos, int32_t n, const td_rope* rope,
                            const void* d_q, int64_t q_stride, const void* d_k, int64_t k_stride, const void* d_v,
                            int64_t v_stride, void* d_q_out, hipStream_t st) {
  if (!c) return TD_EINVAL;
  c->err.clear();
  if (td_status r = bad_layers(c, layer_begin, n_layers)) return r;
  td::StoreArgs a{};
  if (td_status r = store_args(c, rope, d_q, q_stride, d_k, k_stride, d_v, v_stride, d_q_out, &a)) return r;
  if (!c->prefix) return fail(c, TD_ESTATE, "no prefix is attached (td_set_prefix)");
  if (n < 1 || pos < 0 || n > c->prefix_room || pos > c->prefix_room - n)
    return fail(c, TD_EINVAL, "positions [%d, +%d) outside the prefix's %d", pos, n, c->prefix_room);
  if (n > kStoreRows) return fail(c, TD_EINVAL, "n must be at most 2^26");
  if (td_status r = other_device(c)) return r;
  a.rows = td::PrefixRows::kChunk;
  a.layer_begin = layer_begin;
  a.n_layers = n_layers;
  a.tries = 1;
  a.n = n;
  a.pos0 = pos;
  const hipError_t e = td::launch_store(c->dev, a, st);
  if (e != hipSuccess) return hip_fail(c, e, "trie_prefix_store launch");
  return TD_OK;
}

td_status trie_store_kv(td_ctx* c, int32_t layer_begin, int32_t n_layers, int32_t q_max, const int32_t* d_qslots,
                        const td_rope* rope, const void* d_q, int64_t q_stride, const void* d_k, int64_t k_stride,
                        const void* d_v, int64_t v_stride, void* d_q_out, hipStream_t st) {
  td_status r = td::check_ready(c);
  if (r != TD_OK) return r;
  const td::DevState& s = c->dev;
  if ((r = bad_layers(c, layer_begin, n_layers)) != TD_OK) return r;
  if (d_qslots ? q_max < 1 : q_max != s.b) return fail(c, TD_EINVAL, "q_max must be >= 1, or the beam width for the leaves");
  if ((int64_t)s.T * q_max > kStoreRows) return fail(c, TD_EINVAL, "n_tries * q_max must be at most 2^26");
  td::StoreArgs a{};
  if ((r = store_args(c, rope, d_q, q_stride, d_k, k_stride, d_v, v_stride, d_q_out, &a)) != TD_OK) return r;
  if (d_qslots && c->pending) return fail(c, TD_ESTATE, "the leaves' K/V are pending: store them first");
  if ((r = other_device(c)) != TD_OK) return r;
  a.rows = d_qslots ? td::PrefixRows::kNodes : td::PrefixRows::kLeaves;
  a.qslots = d_qslots;
  a.layer_begin = layer_begin;
  a.n_layers = n_layers;
  a.tries = s.T;
  a.n = q_max;
  // (the leaves' rows may be sources of rows that the last collection moved)
  hipError_t e = a.k ? td::copy_due_rows(c, layer_begin, n_layers, st, nullptr, nullptr) : hipSuccess;
  if (e == hipSuccess) e = td::launch_store(s, a, st);
  if (e != hipSuccess) return hip_fail(c, e, "trie_store_kv launch");
  if (a.k) td::note_written(c, layer_begin, n_layers, td::LayerRows::kStored);
  return TD_OK;
}

td_status trie_prefix_attn(td_ctx* c, int32_t layer_begin, int32_t n_layers, int32_t pos, int32_t n, const void* d_q,
                           void* d_out, float scale, hipStream_t st) {
  if (!c) return TD_EINVAL;
  c->err.clear();
  const td::DevState& s = c->dev;
  if (td_status r = bad_layers(c, layer_begin, n_layers)) return r;
  if (!d_q || !d_out || !aligned16(d_q) || !aligned16(d_out))
    return fail(c, TD_EINVAL, "q / out must be non-null and 16-byte aligned");
  if (!(scale > 0.0f) || !std::isfinite(scale)) return fail(c, TD_EINVAL, "scale must be finite and > 0");
  if (!c->prefix) return fail(c, TD_ESTATE, "no prefix is attached (td_set_prefix)");
  if (n < 1 || pos < 0 || n > c->prefix_room || pos > c->prefix_room - n)
    return fail(c, TD_EINVAL, "positions [%d, +%d) outside the prefix's %d", pos, n, c->prefix_room);
  const int G = s.Hq / s.Hkv;
  if ((int64_t)n * G > (1 << 24)) return fail(c, TD_EINVAL, "n must be at most 2^24 / (Hq / Hkv)");
  if (td_status r = other_device(c)) return r;
  const long rows = (long)n * G;
  const int rpb = td::prefix_rows_per_block(rows), blocks = (int)((rows + rpb - 1) / rpb);
  // (as many layers per launch as its grid holds)
  const int lc = (int)std::max(1l, std::min<long>(n_layers, (1l << 22) / ((long)s.Hkv * blocks)));
  const size_t layer = (size_t)n * s.Hq * s.D * (s.dtype == TD_F32 ? 4 : 2);
  hipEvent_t ev0 = c->ev[TD_PHASE_ATTN][0], ev1 = c->ev[TD_PHASE_ATTN][1];
  c->ev[TD_PHASE_ATTN][0] = c->ev[TD_PHASE_ATTN][1] = nullptr;
  hipError_t e = hipSuccess;
  for (int l = 0; l < n_layers && e == hipSuccess; l += lc) {
    td::PrefixArgs a{};
    a.q = static_cast<const char*>(d_q) + l * layer;
    a.out = static_cast<char*>(d_out) + l * layer;
    a.rows = td::PrefixRows::kChunk;
    a.layer_begin = layer_begin + l;
    a.n_layers = std::min(lc, n_layers - l);
    a.tries = 1;
    a.per_trie = a.q_stride = n;
    a.pos0 = pos;
    a.scale_log2 = scale * 1.4426950408889634f;
    a.row_blocks = blocks;
    const long keys = s.W > 0 ? std::min(pos + n, s.W) : pos + n, units = (long)a.n_layers * s.Hkv * blocks;
    const long fit = (long)(c->prefix_records / ((size_t)a.n_layers * n * s.Hq));
    a.records = a.splits = td::prefix_splits(s, units, keys, std::max(1l, fit));
    a.xcd_group = blocks > 1 && ((long)a.n_layers * s.Hkv * a.splits) % 8 == 0;
    // Two WGs per CU at once, and no third: a long block beside a short one.  2,048 tokens of 32 heads (8
    // KV heads, d = 128) from position 0: 57.5 -> 53.7 us a layer, from 6,144: 254 -> 247.5 (graphs in turn);
    // where fewer CUs have two (1,500 tokens) 42.4 -> 41.4 from 0, 210.4 and 210.7 from 6,144.  With more WGs the
    // longest first fill the CUs evenly by themselves.
    a.pair_blocks = s.D <= 128 && units * a.splits > kOneRound / 2 && units * a.splits <= kOneRound;
    a.part_o = a.splits > 1 ? c->prefix_o : nullptr;
    a.part_ml = c->prefix_ml;
    hipEvent_t last = l + lc >= n_layers ? ev1 : nullptr;
    e = td::launch_prefix(s, a, st, l == 0 ? ev0 : nullptr, a.part_o ? nullptr : last);
    if (e == hipSuccess && a.part_o) {
      td::PrefixMergeArgs m{};
      m.prefix_o = c->prefix_o;
      m.prefix_ml = c->prefix_ml;
      m.prefix_splits = a.splits;
      m.out = a.out;
      m.rows = td::PrefixRows::kChunk;
      m.n_layers = a.n_layers;
      m.tries = 1;
      m.per_trie = n;
      e = td::launch_prefix_merge(s, m, st, last);
    }
  }
  if (e != hipSuccess) return hip_fail(c, e, "trie_prefix_attn launch");
  return TD_OK;
}

}  // extern "C"
