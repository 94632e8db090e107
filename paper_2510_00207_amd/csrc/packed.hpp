// The arguments of the attention kernels, and how their blocks find their rows in a packed
// batch: sequences of any lengths side by side, whose starts are device data.
#pragma once

#include <math.h>

#include "attn_tiles.hpp"
#include "common.hpp"

namespace flowmoe {
namespace {

struct AttnArgs {
  const bf16_t* qkv;  // T x 3M = [Q | K | V]; head h at columns h * D of each
  const bf16_t* o;    // T x M: the heads' outputs (backward)
  const bf16_t* d_o;  // T x M: their gradient (backward)
  bf16_t* out;        // forward: T x M
  bf16_t* d_qkv;      // backward: T x 3M
  float* lse;         // heads x T: natural log-sum-exp of each row's scores
  float* delta;       // heads x T: rowsum(dO * O) over the head's columns
  int T, M, N, heads, nseq;
  int shared;  // query tiles of a head side by side on one XCD (decode)
  int pair;  // causal grid of one round of resident blocks: pair long and short tiles (decode)
  float c2;  // log2(e) / sqrt(D): a score times c2 is its base-2 exponent
  float rs;  // 1 / sqrt(D)
  // packed sequences (locate): nseq of them from rows starts[i] on, query heads in groups
  // that share kv key/value heads
  const int32_t* starts;
  int kv;
  // backward: a key tile of more steps than a share of the launch (unit_steps) is cut into at
  // most `units` units, whose sums go to part
  float* part;
  int units;
  int rows32;  // 32-row tiles of all sequences (tile32)
};

// A block's rows: tokens tok0 .. tok0 + N - 1 are the sequence, `tile` of it the block's;
// qkv rows are ld apart, head hd's K and V columns k and v past its Q columns.
struct Span {
  long tok0, ld, k, v;
  int N, tile, hd;
  int seq;    // packed: the sequence's index
  bool none;  // packed: no sequence's rows, whose outputs are zeros
};

// Packed sequences, sequence i from row packed_start(i) on; the rows behind the last are a
// sequence of their own. Whatever `starts` holds, rows stay in 0 .. T.
__device__ __forceinline__ int packed_start(const AttnArgs& a, int i) {
  return i == 0 ? 0 : i > a.nseq ? a.T : min(max(a.starts[i], 0), a.T);
}

// The tile of `slot` (false: none), by a wave, without sums over the lengths stored anywhere:
// tile t of sequence i has slot packed_start(i) / rows + i + t. Sequence i has at most as many
// tiles as there are slots before sequence i + 1's, so a search for the slot finds the
// sequence, 64 starts at a time, and a launch has T / rows + nseq + 1 slots whatever the
// lengths are; those behind a sequence's last tile stay empty. (A scan of all tiles, with the
// longest sequences first or without, took 2 us more of a small call.)
__device__ __forceinline__ bool locate(const AttnArgs& a, int slot, int rows, bool rev, int lane,
                                       Span& s) {
  int lo = 0, hi = a.nseq + 1;  // one of lo .. hi - 1 has the slot; lo's begin at or before it
  while (hi - lo > 1) {
    const int step = (hi - lo + 63) / 64, i = lo + lane * step;
    const bool before = i < hi && packed_start(a, i) / rows + i <= slot;
    const int n = max(1, (int)__popcll(__ballot(before)));
    lo += (n - 1) * step;
    hi = min(hi, lo + step);
  }
  // (its rows by loads of their own: from the lanes that read them last, the forward of heads
  // of 128 spilled 64 bytes a lane)
  const int i = __builtin_amdgcn_readfirstlane(lo);
  const int r0 = __builtin_amdgcn_readfirstlane(packed_start(a, i));
  s.tok0 = r0;
  s.N = __builtin_amdgcn_readfirstlane(packed_start(a, i + 1)) - r0;
  s.seq = i;
  s.none = i == a.nseq;
  const int t = slot - r0 / rows - i, nt = s.N > 0 ? (s.N + rows - 1) / rows : 0;
  s.tile = rev ? nt - 1 - t : t;
  return t >= 0 && t < nt;
}

// Block `block` of the `blocks` of a packed grid: a slot's `per` heads side by side (where per is
// a multiple of 8, those of a group on one XCD, through whose L2 they read their keys), first
// units first; the tiles of a sequence in descending order (`rev`).
__device__ __forceinline__ bool packed_span(const AttnArgs& a, int per, bool rev, int rows,
                                            int units, int lane, unsigned block, unsigned blocks,
                                            Span& s, int& unit) {
  const int j = (int)(block % per), u = (int)(block / per);
  s.hd = per % 8 == 0 ? (j & 7) * (per >> 3) + (j >> 3) : j;
  const int slots = (int)(blocks / per) / units;
  unit = u / slots;
  return locate(a, u - unit * slots, rows, rev, lane, s);
}

// zeros in `cols` columns of rows r0 .. r0 + n - 1 (16-byte vectors)
__device__ __forceinline__ void zero_rows(bf16_t* dst, long ld, long r0, int n, int cols, int tid,
                                          int threads) {
  const int c = cols / 8;
  for (int i = tid; i < n * c; i += threads)
    *reinterpret_cast<u32x4*>(dst + (r0 + i / c) * ld + 8 * (i % c)) = u32x4{0, 0, 0, 0};
}

inline AttnArgs packed_args(const PackedShape& m, int T, const void* qkv, const int32_t* starts) {
  AttnArgs a = {};
  a.T = T;
  a.M = m.heads * m.D;
  a.heads = m.heads;
  a.kv = m.kv;
  a.nseq = m.nseq;
  a.starts = starts;
  a.c2 = kLog2e / sqrtf((float)m.D);
  a.rs = 1.0f / sqrtf((float)m.D);
  a.qkv = static_cast<const bf16_t*>(qkv);
  return a;
}

}  // namespace
}  // namespace flowmoe
