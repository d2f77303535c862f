// Rows into the 4-bit pages of the shared prefix, and rows of the prefix back (gfx950).
//
// A row's blocks of 32 elements share a power of two.  With m the largest size of a block, m = 2^k f, 1 <= f
// < 2: the block's unit is 2^e, e = k - 2, or k - 1 where f >= 1.75 (there m would round past 6, the largest
// size), within [-125, 125]; an element x is kept as its sign and the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 to
// |x| / 2^e, ties to the even code, past 6 as 6.  The scale byte is e + 127; a block with an infinity or a NaN
// has 255, which makes all of it NaN.
//
// K is rotated in 64 bits, sine and cosine too, and rounded once, to 4 bits: next to a border between two
// of the eight sizes an error of 2^-24 would move the element by up to half its size.  On its way a value
// passes through fp32, rounded to odd in 20 bits (the low bit stands for all that was cut off): no border
// and no tie lies between it and the exact one.
//
// What bounds it: HBM.  8,192 tokens of a layer at the Llama-8B shape, queries too (100 MB in, 76 out), 37.3 to 41 us, 4.3
// to 4.7 TB/s (a copy's 4.9), with two rows to a WG; eight of them 40.8 to 44.5.  A WG has as many rows as give each of its
// threads at most 4 units (of 8 elements of K or V, or two 16-byte chunks of q).  2 layers stored and loaded in bf16, 1 / 2 / 4 / 8
// rows, us: 8,192 tokens of 32 q and 8 KV heads of 128 104 / 101 / 106 / 106; 20,000 of 28 and 4 175 / 161 / - / 178; of 8 and 8
// 166 / 147 / 138 / 143; of 8 and 2 of 64 - / 49 / 43 / 43.  The 64-bit sines are computed once for the heads of a row; V's loads
// under way meanwhile changed nothing.
#include <algorithm>

#include "kv_rows.h"

namespace td {

namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));

__device__ inline float to_odd(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t hi = (uint32_t)(u >> 32) | ((uint32_t)u != 0u ? 1u : 0u);
  return (float)__builtin_bit_cast(double, (uint64_t)hi << 32);
}

// The largest of the four lanes of a quad.
__device__ inline uint32_t quad_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xF, 0xF, true));  // quad_perm 1, 0, 3, 2
  return max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xF, 0xF, true));  // quad_perm 2, 3, 0, 1
}

template <typename T>
struct Row8 {  // 8 elements of a row
  typedef T vec __attribute__((ext_vector_type(8)));
};

// Grid (row groups, layers), as k_store.  K and V go in units of 8 elements, four lanes to a block; the pair of
// an element that lies in another unit is read there too (from the cache).
template <typename T, bool AXES>
__global__ __launch_bounds__(kStoreThreads) void k_store4(DevState s, StoreArgs a, int group) {
  using V8 = typename Row8<T>::vec;
  constexpr int E = StoreCfg<T>::E;
  __shared__ double2 turn[kStoreRows * kStorePairs];  // (cos, sin) of row, pair
  __shared__ int64_t dst[kStoreRows];
  __shared__ int position[kStoreRows];
  const int tid = threadIdx.x, li = blockIdx.y, lab = a.layer_begin + li;
  const int rows = a.n, r0 = blockIdx.x * group, count = min(group, rows - r0);
  const int pairs = a.rotary / 2, D = s.D;
  const PrefixHdr p = s.prefix[1];
  if (tid < count) {
    const StoreRow w = store_row(s, a, p, lab, r0 + tid);
    position[tid] = w.position;
    dst[tid] = w.dst;
  }
  __syncthreads();
  for (int i = tid; i < count * pairs; i += kStoreThreads) {
    const int row = i / pairs, pair = i % pairs;
    double sn, cs;
    sincos(pair_position<AXES>(a, r0 + row, position[row], pair) * (double)a.freq[pair], &sn, &cs);
    turn[row * kStorePairs + pair] = make_double2(cs, sn);
  }
  __syncthreads();

  if (a.k != nullptr) {
    const int upl = D / 8, half = a.rotary / 16;  // units of a head, of half of its rotated part
    const global_bytes kout = to_global(p.k), vout = to_global(p.v), ksc = to_global(p.k_scale), vsc = to_global(p.v_scale);
    // (a whole number of blocks: the lanes of a quad leave together)
    for (int i = tid; i < count * 2 * s.Hkv * upl; i += kStoreThreads) {
      const int w = i % upl, row = i / upl / (2 * s.Hkv);
      int head = i / upl % (2 * s.Hkv);
      if (position[row] < 0) continue;
      const bool is_v = head >= s.Hkv;
      head -= is_v ? s.Hkv : 0;
      const int64_t in_row = (int64_t)li * rows + r0 + row;
      const T* src = is_v ? static_cast<const T*>(a.v) + in_row * a.v_stride + (int64_t)head * D
                          : static_cast<const T*>(a.k) + in_row * a.k_stride + (int64_t)head * D;
      const V8 x = reinterpret_cast<const V8*>(src)[w];
      float y[8];
      if (is_v || w >= 2 * half) {
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = (float)x[e];
      } else if (a.interleaved) {
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const double2 f = turn[row * kStorePairs + w * 4 + e / 2];
          y[e] = to_odd((double)x[e] * f.x - (double)x[e + 1] * f.y);
          y[e + 1] = to_odd((double)x[e + 1] * f.x + (double)x[e] * f.y);
        }
      } else {
        const bool second = w >= half;
        const V8 z = reinterpret_cast<const V8*>(src)[second ? w - half : w + half];
        const double2* f = turn + row * kStorePairs + (second ? w - half : w) * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = to_odd((double)x[e] * f[e].x + (second ? (double)z[e] : -(double)z[e]) * f[e].y);
      }
      uint32_t m = 0;  // (sizes compare as integers, a NaN above all)
#pragma unroll
      for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(y[e]) & 0x7fffffffu);
      m = quad_max(m);
      const bool fine = m < 0x7f800000u;
      // (+ 0.25 in units of f: carries into the exponent where f >= 1.75)
      const uint32_t byte = fine ? (uint32_t)min(max((int)((m + 0x200000u) >> 23) - 2, 2), 252) : 255u;
      const float unit = __uint_as_float(byte << 23);
      uint32_t word = 0;
      word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, y[0], y[1], unit, 0);
      word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, y[2], y[3], unit, 1);
      word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, y[4], y[5], unit, 2);
      word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, y[6], y[7], unit, 3);
      const int64_t to = dst[row] + ((int64_t)head << p.shift);
      ((TD_GLOBAL uint32_t*)(is_v ? vout : kout))[to * upl + w] = fine ? word : 0u;
      if (w % 4 == 0) ((TD_GLOBAL uint8_t*)(is_v ? vsc : ksc))[to * (D / 32) + w / 4] = (uint8_t)byte;
    }
  }
  if (a.q_out != nullptr) {
    const int upl = D / (2 * E), turned = a.rotary / (2 * E);
    for (int i = tid; i < count * s.Hq * upl; i += kStoreThreads) {
      const int w = i % upl, row = i / upl / s.Hq, head = i / upl % s.Hq;
      const int64_t in_row = (int64_t)li * rows + r0 + row;
      const T* src = static_cast<const T*>(a.q) + in_row * a.q_stride + (int64_t)head * D;
      T* out = static_cast<T*>(a.q_out) + (in_row * s.Hq + head) * D;
      if (position[row] < 0) {
        const typename StoreCfg<T>::vec zero = {};
        reinterpret_cast<typename StoreCfg<T>::vec*>(out)[2 * w] = zero;
        reinterpret_cast<typename StoreCfg<T>::vec*>(out)[2 * w + 1] = zero;
        continue;
      }
      store_unit(src, out, w, turned, w < turned, a.interleaved, [&](int pair) {
        const double2 f = turn[row * kStorePairs + pair];
        return make_float2((float)f.x, (float)f.y);
      });
    }
  }
}

// Grid (row groups, layers); units of 8 elements of a row, K's and then V's, four under way per thread.  Bound by
// HBM: 8,192 tokens of 8 heads at d = 128, 42 MB in and out, 11.1 us (3.8 TB/s) with 8 rows to a
// WG, two 17.5; K and V in one loop, of batches of 4 or 8, 12.1.
template <typename T, bool FOUR>
__global__ __launch_bounds__(kStoreThreads) void k_prefix_load(DevState s, LoadArgs a, int group) {
  using V8 = typename Row8<T>::vec;
  constexpr int kBatch = 4;
  __shared__ int64_t from[kStoreRows];  // row of KV head 0, -1: none
  const int tid = threadIdx.x, li = blockIdx.y, D = s.D, upl = D / 8;
  const int r0 = blockIdx.x * group, count = min(group, a.n - r0);
  const PrefixHdr p = s.prefix[FOUR ? 1 : 0];
  if (tid < count) {
    const int pos = a.pos0 + r0 + tid;
    int64_t at = -1;
    // (as in the stores: a captured call may find less room than it was checked against)
    if (pos < p.room) at = ((((int64_t)p.table[pos >> p.shift] * s.L + a.layer_begin + li) * s.Hkv) << p.shift) + (pos & ((1 << p.shift) - 1));
    else set_status(s.status, kDevEinval);
    from[tid] = at;
  }
  __syncthreads();
  const int units = count * s.Hkv * upl;  // of K, and as many of V
  for (int kv = 0; kv < 2; ++kv) {
    T* const out = static_cast<T*>(kv ? a.v : a.k);
    if (out == nullptr) continue;
    const global_bytes in = to_global(kv ? p.v : p.k), scales = to_global(kv ? p.v_scale : p.k_scale);
    V8* const to = reinterpret_cast<V8*>(out + ((int64_t)li * a.n + r0) * s.Hkv * D);
    for (int i0 = tid; i0 < units; i0 += kBatch * kStoreThreads) {
      uint32_t word[kBatch], byte[kBatch];
      V8 x[kBatch];
      int64_t at[kBatch];
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        const int i = i0 + b * kStoreThreads, w = i % upl, row = i / upl / s.Hkv, head = i / upl % s.Hkv;
        at[b] = i < units ? from[row] : -1;
        if (at[b] < 0) continue;
        at[b] += (int64_t)head << p.shift;
        if constexpr (FOUR) {
          word[b] = ((const TD_GLOBAL uint32_t*)in)[at[b] * upl + w];
          byte[b] = scales[at[b] * (D / 32) + w / 4];
        } else {
          x[b] = ((const TD_GLOBAL V8*)in)[at[b] * upl + w];
        }
      }
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        if (at[b] < 0) continue;
        if constexpr (FOUR) {
          const float unit = __uint_as_float(byte[b] << 23);
          f32x2 y[4];
          y[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word[b], unit, 0);
          y[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word[b], unit, 1);
          y[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word[b], unit, 2);
          y[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word[b], unit, 3);
#pragma unroll
          for (int e = 0; e < 8; ++e) x[b][e] = (T)y[e / 2][e % 2];
        }
        to[i0 + b * kStoreThreads] = x[b];
      }
    }
  }
}

}  // namespace

hipError_t launch_store4(const DevState& s, const StoreArgs& a, hipStream_t st) {
  const int units = (a.k ? 2 * s.Hkv * (s.D / 8) : 0) + (a.q ? s.Hq * (s.D * (s.dtype == TD_F32 ? 4 : 2) / 32) : 0);
  const int group = store_group(a.n, a.n_layers, 4 * kStoreThreads / units);
  const dim3 grid((a.n + group - 1) / group, a.n_layers);
#define LAUNCH_STORE(T, AXES) hipLaunchKernelGGL((k_store4<T, AXES>), grid, dim3(kStoreThreads), 0, st, s, a, group)
  const bool f32 = s.dtype == TD_F32;
  if (a.n_axes > 0 && f32) LAUNCH_STORE(float, true);
  else if (a.n_axes > 0) LAUNCH_STORE(__bf16, true);
  else if (f32) LAUNCH_STORE(float, false);
  else LAUNCH_STORE(__bf16, false);
#undef LAUNCH_STORE
  return hipGetLastError();
}

hipError_t launch_prefix_load(const DevState& s, const LoadArgs& a, hipStream_t st) {
  const int group = store_group(a.n, a.n_layers, kStoreRows);
  const dim3 grid((a.n + group - 1) / group, a.n_layers);
#define LAUNCH_LOAD(T, FOUR) hipLaunchKernelGGL((k_prefix_load<T, FOUR>), grid, dim3(kStoreThreads), 0, st, s, a, group)
  const bool f32 = s.dtype == TD_F32;
  if (a.four && f32) LAUNCH_LOAD(float, true);
  else if (a.four) LAUNCH_LOAD(__bf16, true);
  else if (f32) LAUNCH_LOAD(float, false);
  else LAUNCH_LOAD(__bf16, false);
#undef LAUNCH_LOAD
  return hipGetLastError();
}

}  // namespace td
