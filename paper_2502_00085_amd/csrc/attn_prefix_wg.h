// A workgroup of the bf16 pass over the shared prefix (attn_prefix.hip, attn_prefix4.hip): it streams the keys
// of its split, in tiles of 64, once for its 32, 64 or 128 rows.
#pragma once

#include "attn_common.h"
#include "attn_prefix.h"

namespace td {

constexpr float kMost = 8192.0f;  // a row's shift moves once 16 of its probabilities add up to more
constexpr float kSlack = 8.0f;    // ... to its largest score, if that is 2^8 above

// RW waves hold 32 rows each; KW groups of RW waves take the 32-key halves of each tile.
template <int D, int RW, int KW>
struct PrefixCfg {
  static constexpr int THREADS = 64 * RW * KW;
  static constexpr int KSTEPS = D / 16;    // 32x32x16 steps of S^T
  static constexpr int DT = D / 32;        // 32-wide d tiles of O^T
  static constexpr int CPR = D / 8;        // 16-byte chunks per key row
  static constexpr int NBLK = CPR / 4;     // 64-byte blocks per row
  static constexpr int HALF = 32 * D * 2;  // bytes of 32 K (or V) rows
  static constexpr int BUF = 2 * HALF;     // of a tile's
  static constexpr int LOADS = 2 * HALF / 16 / THREADS;  // 16-byte loads per thread: K (or V) of a tile
  static_assert(2 * HALF % (16 * THREADS) == 0, "a tile is a whole number of WG loads");
  static constexpr bool ONE_OFS = THREADS % CPR == 0 && (THREADS / CPR) % CPR == 0;
  static constexpr int OFS = ONE_OFS ? 1 : LOADS;
  static constexpr int WAVES = 8 * HALF <= 80 * 1024 ? 2 : 1;  // per SIMD, as the LDS allows
  static constexpr int VROT = 8 % NBLK == 0 ? 1 : 4;  // rotations of V rows 8 apart
};

// Physical chunk of logical chunk c of V row r.  A tile that is unpacked from 4 bits also rotates the chunks
// within a 64-byte block (which one thread writes, chunk after chunk): the threads of four rows then write to
// different banks.
template <int CPR, int NBLK, bool FOUR>
__device__ inline int v_chunk(int r, int c) {
  return FOUR ? (c / 4 + r % NBLK) % NBLK * 4 + ((c + r) & 3) : phys_chunk<CPR, NBLK>(r, c);
}
template <int CPR, int NBLK, bool FOUR>
__device__ inline int v_logical(int r, int pc) {
  return FOUR ? (pc / 4 + NBLK - r % NBLK) % NBLK * 4 + ((pc - r) & 3) : (pc + CPR - 4 * (r % NBLK)) % CPR;
}

// TRIES: the launch's last WGs take the tries' own nodes (PrefixArgs::trie_splits), for calls so small
// that a launch of their own would run after this one instead of beside it.  A trie's rows in its
// pool are one page of nodes; every live row sees its shared prefix, and of the nodes after it those
// whose ancestor mask holds the row's beam.
//
// FOUR: the prefix is in 4 bits.  Its tiles pass through registers: a thread loads blocks of 32 elements (16
// bytes and a scale) two tiles ahead and unpacks them, 16 conversions a block, into the tile buffer that the
// next step reads.  Every value is exact in bf16, and a tile's are converted once for all of its rows.
//
// WGS: which WGs' code this is, of the prefix or of the tries (kBoth: decided at run time).
enum class Wgs { kBoth, kPrefix, kTries };
template <int D, int RW, int KW, Wgs WGS, bool FOUR>
__device__ __attribute__((always_inline)) inline void prefix_wg(
    const DevState& s, const PrefixArgs& a, unsigned char (&kbuf0)[PrefixCfg<D, RW, KW>::BUF],
    unsigned char (&vbuf0)[PrefixCfg<D, RW, KW>::BUF], unsigned char (&kbuf1)[PrefixCfg<D, RW, KW>::BUF],
    unsigned char (&vbuf1)[PrefixCfg<D, RW, KW>::BUF], int (&wred)[4 * RW], float (&ml)[KW == 2 ? RW * 128 : 1]) {
#include "attn_prefix_body.h"
}

}  // namespace td
