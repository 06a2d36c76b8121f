// Packed sequences, for the kernels that walk them.
//
// Sequence i owns rows offs[i] .. offs[i+1]-1 of every activation. Work along
// the rows is cut into tiles of R rows that never straddle two sequences:
// sequence i's tiles start at index key(i) = offs[i] / R + i, which leaves
// room for ceil(len / R) of them (and at least one, so an empty sequence has
// a tile that passes its state on), rises strictly with i, and is found from a
// tile index by bisection, without a table. rows / R + n_seq bounds the
// count on the host, which does not know the offsets.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace tcl {

struct Tile {
  int seq;   // -1: no sequence has this tile
  int j;     // its index in the sequence
  int base;  // the sequence's first row
  int len;
};

// Tile w of R rows. Offsets are read as lying in [0, rows], so a wrong one
// cannot lead outside the activations.
__device__ __forceinline__ Tile find_tile(const int* __restrict__ offs, int n_seq, int rows, int R, int w) {
  Tile t = {-1, 0, 0, 0};
  if (!offs) {
    if (w < n_seq) t = {w, 0, w, 1};
    return t;
  }
  int lo = 0, hi = n_seq;  // key(lo) <= w < key(hi), once the ends are taken
  if (R > rows) {          // one tile per sequence
    if (w >= n_seq) return t;
    lo = w;
    hi = w + 1;
  }
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (offs[mid] / R + mid <= w) lo = mid;
    else hi = mid;
  }
  const int o0 = min(max(offs[lo], 0), rows), o1 = min(max(offs[lo + 1], o0), rows);
  t.j = w - (o0 / R + lo);
  t.base = o0;
  t.len = o1 - o0;
  t.seq = t.j >= 0 && (t.j == 0 || (int64_t)t.j * R < t.len) ? lo : -1;
  return t;
}

// The state of sequence `seq` in the pool, -1 for none.
__device__ __forceinline__ int slot_of(const int* __restrict__ slots, int n_slots, int seq) {
  const int j = slots ? slots[seq] : seq;
  return j >= 0 && j < n_slots ? j : -1;
}

}  // namespace tcl
