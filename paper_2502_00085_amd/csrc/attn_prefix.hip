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
//
// What bounds it, by the rows that share a key (one MI355X, d = 128 unless stated; kernel trace, mean of
// passes once the clocks have settled, in brackets the least):
//   * few rows: HBM.  8 rows per KV head (32 KV heads, d = 96) over 50,001 keys: 112 (108) us, 5.5 (5.7)
//     TB/s of reads.  Below some 4,000 keys per KV head a launch is a chain of latencies: 128 rows over 4,096
//     keys of 8 KV heads, with the tries' own nodes, 16.5 (14.6) us (its 17 MB take 3.4).
//   * many rows: the clock under matrix load.  1,024 rows of 8 KV heads over 8,192 keys of 4 layers: 160 (154)
//     us, 859 (892) TFLOP/s; the causal pass of 2,048 tokens from position 6,144: 249 (246) us, 966 (976)
//     TFLOP/s, and 244 us, 984, without the trace (a library product of 8,192^3 makes 1,121 here).  There the
//     card runs at 2.0 to 2.1 of its 2.4 GHz, the matrix pipe busy for half of the CUs' clocks, the vector ALU
//     (the exponentials) as long, LDS a quarter.  Each of the two waves of a SIMD fills the other's gaps: a
//     loop that interleaves one half's weights with its neighbours' products by hand took the same time to 0.3 %.
// Tried and not kept: four tile buffers (16,384 keys in 8 splits: 60 us against 48); 8 waves, of two
// groups of keys, per 128 rows (8,192 keys, 1,024 rows: 55 us against 50); a fixed order of products and
// LDS reads (1.5 % slower); 64 rows per wave, one wave per SIMD (568 us against 480 for two causal layers).
#include <algorithm>

#include "attn_prefix_wg.h"

namespace td {

namespace {

// NODES: the launch's last WGs take the tries' own nodes.
template <int D, int RW, int KW, bool NODES>
__global__ __launch_bounds__(64 * RW * KW, (PrefixCfg<D, RW, KW>::WAVES)) void k_attn_prefix(DevState s, PrefixArgs a) {
  // (an array per buffer: the compiler can tell an operand read of one buffer from the direct loads
  // under way into the others)
  constexpr int BUF = PrefixCfg<D, RW, KW>::BUF;
  __shared__ __attribute__((aligned(16))) unsigned char kbuf0[BUF], vbuf0[BUF];
  __shared__ __attribute__((aligned(16))) unsigned char kbuf1[BUF], vbuf1[BUF];
  __shared__ int wred[4 * RW];
  __shared__ float ml[KW == 2 ? RW * 128 : 1];
  if constexpr (NODES) {
    prefix_wg<D, RW, KW, Wgs::kBoth, false>(s, a, kbuf0, vbuf0, kbuf1, vbuf1, wred, ml);
  } else {
    constexpr Wgs WGS = Wgs::kPrefix;
    constexpr bool FOUR = false;
#include "attn_prefix_body.h"
  }
}

template <int D>
void launch_d(const DevState& s, const PrefixArgs& a, int rpb, hipStream_t st, hipEvent_t ev0, hipEvent_t ev1) {
  const dim3 grid(a.n_layers * s.Hkv * (a.splits * a.row_blocks + a.tries * a.trie_blocks * a.trie_splits));
#define LAUNCH_PREFIX(RW, KW, TRIES) \
  hipExtLaunchKernelGGL((k_attn_prefix<D, RW, KW, TRIES>), grid, dim3(64 * RW * KW), 0, st, ev0, ev1, 0, s, a)
  if constexpr (D == 64 || D == 96 || D == 128) {
    if (a.trie_splits > 0) {
      if (rpb == 32) LAUNCH_PREFIX(1, 2, true);
      else if (rpb == 64) LAUNCH_PREFIX(2, 2, true);
      else LAUNCH_PREFIX(4, 1, true);
      return;
    }
  }
  if (rpb == 32) LAUNCH_PREFIX(1, 2, false);
  else if (rpb == 64) LAUNCH_PREFIX(2, 2, false);
  else LAUNCH_PREFIX(4, 1, false);
#undef LAUNCH_PREFIX
}

// Each (row, 8-element chunk of d) is merged by TP adjacent lanes, lane j taking the groups of 8
// records j, j + TP, ...: every load of a group goes out before any is used; groups are merged with
// a running shift, the lanes' states pairwise, in one order.  A record with sum 0 weighs nothing
// (whatever its O); a NaN sum makes the row NaN.  Bound by the latency of its one or two loads in a
// row: 18 records each of 1,024 output rows, 4.7 to 5.1 us.
constexpr int kMergeThreads = 64;

template <typename T, int TP>
__global__ __launch_bounds__(kMergeThreads) void k_prefix_merge(DevState s, PrefixMergeArgs a, uint32_t items) {
  constexpr int GS = 8;
  const int D = s.D, G = s.Hq / s.Hkv, CH = D / 8;
  // (the host keeps items * TP below 2^31)
  const uint32_t item = (blockIdx.x * kMergeThreads + threadIdx.x) / TP;
  const int sub = threadIdx.x % TP;
  if (item >= items) return;  // (the lanes of an item leave together)
  const uint32_t row = item / CH;
  const int c = (int)(item % CH) * 8;
  const int head = row % s.Hq;
  const uint32_t o = row / s.Hq;  // (li tries + t) per_trie + j
  const int j = o % a.per_trie;
  const uint32_t tl = o / a.per_trie;
  const int t = tl % a.tries, li = tl / a.tries;
  const size_t prec = (size_t)row * a.prefix_splits;
  const int ts = a.trie != nullptr ? a.trie_splits : 0, n = ts + a.prefix_splits;
  const float* trec = nullptr;
  size_t tstep = 0;
  if (ts > 0) {
    const int r = j * G + head % G;
    const size_t unit = (((size_t)t * a.n_layers + li) * s.Hkv + head / G) * a.row_blocks + r / a.block_rows;
    trec = a.trie + (unit * ts * a.block_rows + r % a.block_rows) * (D + 2);
    tstep = (size_t)a.block_rows * (D + 2);
  }
  const bool live = a.rows != PrefixRows::kLeaves || j < s.hdr[t].n_live;
  float M = kPrefixNegBig, L = 0.0f, O[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) O[e] = 0.0f;
  for (int i0 = sub * GS; i0 < n; i0 += TP * GS) {
    float2 ml[GS];
    float2 ov[GS][4];
#pragma unroll
    for (int k = 0; k < GS; ++k) {
      const int i = i0 + k < n ? i0 + k : i0;  // (past the last: the group's first again, unused)
      // (the tries' records are D + 2 floats, 8-byte aligned)
      const float* rec = i < ts ? trec + i * tstep : a.prefix_o + (prec + i - ts) * D;
      ml[k] = i < ts ? *reinterpret_cast<const float2*>(rec + D) : a.prefix_ml[prec + i - ts];
#pragma unroll
      for (int e = 0; e < 4; ++e) ov[k][e] = *reinterpret_cast<const float2*>(rec + c + 2 * e);
    }
    float Mg = M;
#pragma unroll
    for (int k = 0; k < GS; ++k) Mg = i0 + k < n && ml[k].y != 0.0f ? fmaxf(Mg, ml[k].x) : Mg;
    const float fo = __builtin_amdgcn_exp2f(M - Mg);
    L *= fo;
#pragma unroll
    for (int e = 0; e < 8; ++e) O[e] *= fo;
#pragma unroll
    for (int k = 0; k < GS; ++k) {
      const bool use = i0 + k < n && ml[k].y != 0.0f;
      const float f = __builtin_amdgcn_exp2f(ml[k].x - Mg);
      L += use ? ml[k].y * f : 0.0f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        O[2 * e] += use ? ov[k][e].x * f : 0.0f;
        O[2 * e + 1] += use ? ov[k][e].y * f : 0.0f;
      }
    }
    M = Mg;
  }
#pragma unroll
  for (int w = 1; w < TP; w <<= 1) {
    const float M2 = __shfl_xor(M, w), L2 = __shfl_xor(L, w);
    float O2[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) O2[e] = __shfl_xor(O[e], w);
    const bool low = (sub & w) == 0;
    const float Mn = fmaxf(M, M2);
    const float f0 = __builtin_amdgcn_exp2f((low ? M : M2) - Mn), f1 = __builtin_amdgcn_exp2f((low ? M2 : M) - Mn);
    L = (low ? L : L2) * f0 + (low ? L2 : L) * f1;
#pragma unroll
    for (int e = 0; e < 8; ++e) O[e] = (low ? O[e] : O2[e]) * f0 + (low ? O2[e] : O[e]) * f1;
    M = Mn;
  }
  if (sub != 0) return;
  const float inv = live && L != 0.0f ? 1.0f / L : 0.0f;
  typedef T t8 __attribute__((ext_vector_type(8)));
  t8 y;
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = (T)(live && L != 0.0f ? O[e] * inv : 0.0f);
  *reinterpret_cast<t8*>(static_cast<T*>(a.out) + (size_t)row * D + c) = y;
}

}  // namespace

// What the kernels take for granted of a launch: a WG takes its number apart (prefix_unit) into a layer, a KV head, a
// row block and a split, which address the pages, the pools and the records.
static bool launch_fits(const DevState& s, const PrefixArgs& a) {
  return a.splits >= 1 && a.row_blocks >= 1 && a.n_layers >= 1 && a.layer_begin >= 0 && a.layer_begin + a.n_layers <= s.L &&
         a.records >= a.splits + a.trie_splits && (!a.xcd_group || prefix_xcd_eights(a.n_layers, s.Hkv, a.splits)) &&
         (a.trie_splits == 0 || a.prefix_wgs == (uint64_t)a.n_layers * s.Hkv * a.row_blocks * a.splits);
}

hipError_t launch_prefix(const DevState& s, const PrefixArgs& a, hipStream_t st, hipEvent_t ev0, hipEvent_t ev1) {
  if (!launch_fits(s, a)) return hipErrorInvalidValue;
  const int rpb = prefix_rows_per_block(prefix_heads(s), a.four, (long)a.tries * a.per_trie * (s.Hq / s.Hkv));
  if (a.trie_splits > 0 && (a.rows != PrefixRows::kLeaves || s.dtype != TD_BF16 || !mfma_head_dim(s.D))) return hipErrorInvalidValue;
  if (a.four) return launch_prefix4(s, a, rpb, st, ev0, ev1);
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

hipError_t launch_prefix_merge(const DevState& s, const PrefixMergeArgs& a, hipStream_t st, hipEvent_t ev1) {
  const long items = (long)a.n_layers * a.tries * a.per_trie * s.Hq * (s.D / 8);
  const int n = (a.trie ? a.trie_splits : 0) + a.prefix_splits;
  const int tp = n > 16 ? 4 : n > 8 ? 2 : 1;  // lanes per output chunk: 8 records each
  if (items * tp >= (1l << 31)) return hipErrorInvalidValue;  // (a workspace of records is far smaller)
  const dim3 grid((items * tp + kMergeThreads - 1) / kMergeThreads), block(kMergeThreads);
#define LAUNCH_MERGE(T, TP) \
  hipExtLaunchKernelGGL((k_prefix_merge<T, TP>), grid, block, 0, st, nullptr, ev1, 0, s, a, (uint32_t)items)
  if (s.dtype == TD_F32) tp == 4 ? LAUNCH_MERGE(float, 4) : tp == 2 ? LAUNCH_MERGE(float, 2) : LAUNCH_MERGE(float, 1);
  else tp == 4 ? LAUNCH_MERGE(__bf16, 4) : tp == 2 ? LAUNCH_MERGE(__bf16, 2) : LAUNCH_MERGE(__bf16, 1);
#undef LAUNCH_MERGE
  return hipGetLastError();
}

}  // namespace td
