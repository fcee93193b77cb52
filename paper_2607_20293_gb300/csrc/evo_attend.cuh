// What the attention kernels over a paged memory share: which keys a row sees,
// the pieces that a memory is split into, and the partial results of a piece.
//
// The rows of a (sequence, key/value head) are its chunk's tokens times the
// `group` query heads that share the head, token-major: row i is token i / group,
// query head i % group of the group.  A block takes a tile of such rows and one
// piece of the keys that any of them sees.
#pragma once

#include "evo_memory.h"

namespace evo {

struct Tile {
  int n, kv_head, tile, split;
  int first, count;             // the sequence's rows of the call
  int len;                      // tokens in its memory
};

__device__ __forceinline__ Tile tile_of_block(const AttendArgs& a) {
  Tile t;
  int b = blockIdx.x;
  t.split = b % a.splits;
  b /= a.splits;
  t.tile = b % a.tiles;
  b /= a.tiles;
  t.kv_head = b % a.m.n_kv_head;
  t.n = b / a.m.n_kv_head;
  const SeqRows s = seq_rows(a.m, t.n, a.rows, a.max_new);
  t.first = s.first;
  t.count = s.count;
  t.len = seq_len(a.m, t.n, a.max_len);
  return t;
}

// keys [lo, hi) that token j of the chunk sees
struct Range { int lo, hi; };
__device__ __forceinline__ Range seen_by(const AttendArgs& a, const Tile& t, int j) {
  Range r;
  r.hi = a.causal ? min(t.len, t.len - t.count + j + 1) : t.len;
  r.hi = max(r.hi, 0);
  r.lo = a.window ? max(0, r.hi - a.window) : 0;
  return r;
}

// keys that some row of tokens j0 .. j1 sees
__device__ __forceinline__ Range seen_by_tile(const AttendArgs& a, const Tile& t, int j0, int j1) {
  return {seen_by(a, t, j0).lo, seen_by(a, t, j1).hi};
}

// this block's piece of the range, cut at multiples of `step` keys
__device__ __forceinline__ Range piece_of(const AttendArgs& a, const Tile& t, Range r, int step) {
  const int lo = r.lo / step, hi = (r.hi + step - 1) / step;
  const int each = (max(hi - lo, 0) + a.splits - 1) / a.splits;
  return {max(r.lo, (lo + t.split * each) * step), min(r.hi, (lo + (t.split + 1) * each) * step)};
}

// index of (row of the call, query head) in the partial results of a piece
__device__ __forceinline__ long long part_index(const AttendArgs& a, int split, int row, int head) {
  return ((long long)split * a.rows + row) * a.m.n_head + head;
}

}  // namespace evo
