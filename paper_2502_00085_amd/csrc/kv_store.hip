// Rotated K/V rows into the tries' pools or the pages of the shared prefix, and rotated queries
// (gfx950).
//
// Pair i of a head's first `rotary` elements, at position p, turns by the angle p f_i:
//   (x, y) -> (x cos - y sin, y cos + x sin),   (x, y) = elements (i, i + rotary / 2), or (2i, 2i + 1);
// the other elements, and V, are copied.  A node's position is the prefix's length plus its depth,
// both read here, on the device: the caller need not know where a trie has got to.  With positions of
// several axes (images, video) p is that of the pair's axis: given for each row, or the row's own plus a
// shift of its trie.
//
// The angle of a far position needs more than fp32: p f_i in turns, in 64 bits, less whole turns;
// the sine and cosine of the rest in fp32, once per (row, pair), in LDS for all of the row's heads.
//
// What bounds it: HBM.  8,192 tokens of a layer at the Llama-8B shape (201 MB in and out) in 40.0 us, 5.0 TB/s
// (a copy's 4.9); with few rows one launch's latency (the leaves of 16 tries of 16 beams, 6.3 MB, 4.3 us, the
// least 4.1; with several axes 5.0 and 4.7).  Rows are read and written once.  A WG has as many as give each of its
// threads a unit of two 16-byte chunks, one of 32 to 48 heads: the angles are computed once for them, and with more rows the CUs end one after another.  2
// layers of 20,000 tokens in bf16, 1 / 2 / 4 / 8 rows per WG, us: 28 q and 4 KV heads of 128 138 / 143 / 150 / 159; 8 and 8 of 128
// 100 / 98 / 109 / 113; 16 and 4 of 64 53 / 43 / 42 / 43; 8 and 2 of 64 43 / 33 / 26 / 25; 8 ragged prompts of 32 and 8 of 128 64.3 /
// 64.1 / 71.5 / 76.7.  With several axes the same: 6,001 tokens of a layer, 147 MB, 30.6 us, 4.8 TB/s.
#include <algorithm>

#include "kv_rows.h"

namespace td {

namespace {

// Grid (row groups, layers); a WG takes `group` consecutive rows (trie, j) of one layer.  (`group` ahead of the
// arguments of several axes: a line less to fetch before the first address, 0.05 us of the leaves' 3.7.)
template <typename T, bool AXES>
__global__ __launch_bounds__(kStoreThreads) void k_store(DevState s, int group, StoreArgs a) {
  using C = StoreCfg<T>;
  using V = typename C::vec;
  constexpr int E = C::E;
  __shared__ float2 turn[kStoreRows * kStorePairs];  // (cos, sin) of row, pair
  __shared__ int64_t dst[kStoreRows];                // K/V row of KV head 0, -1: none
  __shared__ int position[kStoreRows];               // -1: no row
  const int tid = threadIdx.x, li = blockIdx.y;
  // (readfirstlane keeps it here, with the other arguments: loaded where it is used, the compiler's wait for it
  // is one for the prefix's header too, before the trie's header is asked for)
  const int lab = __builtin_amdgcn_readfirstlane(a.layer_begin + li);
  const int rows = a.tries * a.n, r0 = blockIdx.x * group, count = min(group, rows - r0);
  const int pairs = a.rotary / 2;
  const bool chunk = a.rows == PrefixRows::kChunk;
  const PrefixHdr p = s.prefix[0];
  if (tid < count) {
    const StoreRow w = store_row(s, a, p, lab, r0 + tid);
    position[tid] = w.position;
    dst[tid] = w.dst;
  }
  __syncthreads();
  for (int i = tid; i < count * pairs; i += kStoreThreads) {
    const int row = i / pairs, pair = i % pairs;
    double x = pair_position<AXES>(a, r0 + row, position[row], pair) * (double)a.freq[pair] * 0.15915494309189535;  // turns
    x -= rint(x);
    float sn, cs;
    sincospif((float)(2.0 * x), &sn, &cs);
    turn[row * kStorePairs + pair] = make_float2(cs, sn);
  }
  __syncthreads();

  // units of two 16-byte chunks of one head of one row: E pairs, or 2 E copied elements
  const int D = s.D, upl = D / (2 * E), turned = a.rotary / (2 * E);
  const int heads = (a.q_out != nullptr ? s.Hq : 0) + (a.k != nullptr ? 2 * s.Hkv : 0);
  const int64_t head_step = chunk ? (int64_t)1 << p.shift : s.cap;
  T* kout = static_cast<T*>(chunk ? const_cast<void*>(p.k) : s.k_pool);
  T* vout = static_cast<T*>(chunk ? const_cast<void*>(p.v) : s.v_pool);
  for (int i = tid; i < count * heads * upl; i += kStoreThreads) {
    const int w = i % upl, row = i / upl / heads;
    int head = i / upl % heads;
    const int64_t in_row = (int64_t)li * rows + r0 + row;
    const bool some = position[row] >= 0;
    const T* src;
    T* out;
    bool rotate = w < turned;
    if (head >= 2 * s.Hkv || a.k == nullptr) {
      head -= a.k != nullptr ? 2 * s.Hkv : 0;
      src = static_cast<const T*>(a.q) + in_row * a.q_stride + (int64_t)head * D;
      out = static_cast<T*>(a.q_out) + (in_row * s.Hq + head) * D;
      if (!some) {
        const V zero = {};
        reinterpret_cast<V*>(out)[2 * w] = zero;
        reinterpret_cast<V*>(out)[2 * w + 1] = zero;
      }
    } else {
      const bool is_v = head >= s.Hkv;
      head -= is_v ? s.Hkv : 0;
      src = is_v ? static_cast<const T*>(a.v) + in_row * a.v_stride + (int64_t)head * D
                 : static_cast<const T*>(a.k) + in_row * a.k_stride + (int64_t)head * D;
      out = (is_v ? vout : kout) + (dst[row] + head * head_step) * D;
      rotate = rotate && !is_v;
    }
    if (!some) continue;
    store_unit(src, out, w, turned, rotate, a.interleaved, [&](int pair) { return turn[row * kStorePairs + pair]; });
  }
}

}  // namespace

int store_group(long rows, int n_layers, int most) {
  // (as many rows per WG as leave a few WGs per CU, at most `most`; a grid of hundreds of millions of threads is long enough)
  if (rows > kStoreMany) return kStoreRows;
  return (int)std::max(1l, std::min<long>(std::min(most, kStoreRows), rows * n_layers / 1024));
}

hipError_t launch_store(const DevState& s, const StoreArgs& a, hipStream_t st) {
  const long rows = (long)a.tries * a.n;
  const int units = ((a.q ? s.Hq : 0) + (a.k ? 2 * s.Hkv : 0)) * (s.D * (s.dtype == TD_F32 ? 4 : 2) / 32);
  const int group = store_group(rows, a.n_layers, (kStoreThreads + units - 1) / units);
  const dim3 grid((rows + group - 1) / group, a.n_layers);
#define LAUNCH_STORE(T, AXES) hipLaunchKernelGGL((k_store<T, AXES>), grid, dim3(kStoreThreads), 0, st, s, group, a)
  const bool f32 = s.dtype == TD_F32;
  if (a.n_axes > 0 && f32) LAUNCH_STORE(float, true);
  else if (a.n_axes > 0) LAUNCH_STORE(__bf16, true);
  else if (f32) LAUNCH_STORE(float, false);
  else LAUNCH_STORE(__bf16, false);
#undef LAUNCH_STORE
  return hipGetLastError();
}

}  // namespace td
