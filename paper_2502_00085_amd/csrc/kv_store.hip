// Rotated K/V rows into the tries' pools or the pages of the shared prefix, and rotated queries
// (gfx950).
//
// Pair i of a head's first `rotary` elements, at position p, turns by the angle p f_i:
//   (x, y) -> (x cos - y sin, y cos + x sin),   (x, y) = elements (i, i + rotary / 2), or (2i, 2i + 1);
// the other elements, and V, are copied.  A node's position is the prefix's length plus its depth,
// both read here, on the device: the caller need not know where a trie has got to.
//
// The angle of a far position needs more than fp32: p f_i in turns, in 64 bits, less whole turns;
// the sine and cosine of the rest in fp32, once per (row, pair), in LDS for all of the row's heads.
//
// What bounds it: HBM.  8,192 tokens of a layer at the Llama-8B shape (201 MB in and out) in 43.4 us (the
// least 38.1), 4.6 TB/s (5.3; a copy's 5.0); with few rows one launch's latency (the leaves of 16 tries of 16
// beams, 6.3 MB, 4.3 us; the least 4.1).  Rows are read and written once; up to 8 of one layer share a WG, so that the
// angles are computed once for the 32 to 48 heads of a row.
#include <algorithm>

#include "attn_common.h"
#include "prefix.h"

namespace td {

namespace {

constexpr int kStoreThreads = 256;
constexpr int kStoreRows = 8;  // rows of a WG at most

template <typename T>
struct StoreCfg {
  static constexpr int E = 16 / (int)sizeof(T);  // elements per 16-byte chunk
  typedef T vec __attribute__((ext_vector_type(16 / (int)sizeof(T))));
};

// Grid (row groups, layers); a WG takes `group` consecutive rows (trie, j) of one layer.
template <typename T>
__global__ __launch_bounds__(kStoreThreads) void k_store(DevState s, StoreArgs a, int group) {
  using C = StoreCfg<T>;
  using V = typename C::vec;
  constexpr int E = C::E;
  __shared__ float2 turn[kStoreRows * 128];  // (cos, sin) of row, pair
  __shared__ int64_t dst[kStoreRows];        // K/V row of KV head 0, -1: none
  __shared__ int position[kStoreRows];       // -1: no row
  const int tid = threadIdx.x, li = blockIdx.y, lab = a.layer_begin + li;
  const int rows = a.tries * a.n, r0 = blockIdx.x * group, count = min(group, rows - r0);
  const int pairs = a.rotary / 2;
  const bool chunk = a.rows == PrefixRows::kChunk;
  const PrefixHdr p = *s.prefix;
  if (tid < count) {
    const int t = (r0 + tid) / a.n, j = (r0 + tid) % a.n;
    int pos = -1;
    int64_t to = -1;
    if (chunk) {
      // (a captured call may find a shorter table than the one it was checked against)
      if (a.pos0 + j < p.room) {
        pos = a.pos0 + j;
        const int64_t page = p.table[pos >> p.shift];
        to = (((page * s.L + lab) * s.Hkv) << p.shift) + (pos & ((1 << p.shift) - 1));
      } else {
        set_status(s.status, kDevEinval);
      }
    } else {
      const TrieHdr h = s.hdr[t];
      int slot;
      if (a.rows == PrefixRows::kLeaves) slot = j < h.n_live ? h.n_nodes - h.n_live + j : -1;
      else slot = a.qslots[(size_t)t * a.n + j];
      if (slot >= 0 && slot < h.n_nodes) {
        const int at = h.base + slot;
        pos = p.length + (a.rows == PrefixRows::kLeaves ? h.leaf_depth : s.depth[(size_t)t * s.cap + at]);
        to = (((int64_t)t * s.L + lab) * s.Hkv) * s.cap + at;
      }
    }
    position[tid] = pos;
    dst[tid] = to;
  }
  __syncthreads();
  for (int i = tid; i < count * pairs; i += kStoreThreads) {
    const int row = i / pairs, pair = i % pairs, pos = position[row];
    double x = (double)pos * (double)a.freq[pair] * 0.15915494309189535;  // turns
    x -= rint(x);
    float sn, cs;
    sincospif((float)(2.0 * x), &sn, &cs);
    turn[row * 128 + pair] = make_float2(cs, sn);
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
    const bool split = rotate && !a.interleaved;
    const int c0 = split ? w : 2 * w, c1 = split ? w + turned : 2 * w + 1;
    const V x = reinterpret_cast<const V*>(src)[c0], y = reinterpret_cast<const V*>(src)[c1];
    V x1 = x, y1 = y;
    if (rotate) {
      const float2* cs = turn + row * 128 + w * E;
      if (split) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float2 f = cs[e];
          const float xe = (float)x[e], ye = (float)y[e];
          x1[e] = (T)(xe * f.x - ye * f.y);
          y1[e] = (T)(ye * f.x + xe * f.y);
        }
      } else {
#pragma unroll
        for (int e = 0; e < E; e += 2) {
          const float2 f = cs[e / 2], g = cs[E / 2 + e / 2];
          const float xa = (float)x[e], xb = (float)x[e + 1], ya = (float)y[e], yb = (float)y[e + 1];
          x1[e] = (T)(xa * f.x - xb * f.y);
          x1[e + 1] = (T)(xb * f.x + xa * f.y);
          y1[e] = (T)(ya * g.x - yb * g.y);
          y1[e + 1] = (T)(yb * g.x + ya * g.y);
        }
      }
    }
    reinterpret_cast<V*>(out)[c0] = x1;
    reinterpret_cast<V*>(out)[c1] = y1;
  }
}

}  // namespace

hipError_t launch_store(const DevState& s, const StoreArgs& a, hipStream_t st) {
  const long rows = (long)a.tries * a.n;
  // (as many rows per WG as leave a few WGs per CU)
  int group = (int)std::max(1l, std::min<long>(kStoreRows, rows * a.n_layers / 1024));
  const dim3 grid((rows + group - 1) / group, a.n_layers);
  if (s.dtype == TD_F32) hipLaunchKernelGGL(k_store<float>, grid, dim3(kStoreThreads), 0, st, s, a, group);
  else hipLaunchKernelGGL(k_store<__bf16>, grid, dim3(kStoreThreads), 0, st, s, a, group);
  return hipGetLastError();
}

}  // namespace td
