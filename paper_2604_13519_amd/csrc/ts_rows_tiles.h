// Which rows a workgroup of the attention of chunks works on (ts_paged_rows.hip): integers, and exchanges between the 64 lanes of a wave that
// tests/native/rows_tiles.cpp stands in for, so that this file also runs on the CPU.  Offsets and lengths are what the device holds, and may
// be anything: whatever they are, a tile's rows lie in [0, n_rows).
#pragma once
#include <stdint.h>

#include "../../include/toolspec_ops.h"

// the last i in [0, n) with f(i) <= key, -1 if none, where f does not decrease (elsewhere some i).  64 at a time, one per lane.
template <typename F>
__device__ __forceinline__ int last_at_most(int n, int64_t key, F f) {
  const int lane = threadIdx.x % 64;
  int lo = 0, left = n;
  for (;;) {
    const int step = (left + 63) / 64, i = lane * step;
    const int c = __popcll(__ballot(i < left && f(lo + (i < left ? i : 0)) <= key));
    if (c == 0) return lo - 1;
    if (step == 1) return lo + c - 1;
    lo += (c - 1) * step + 1;
    left = min(step - 1, left - (c - 1) * step - 1);
    if (left <= 0) return lo - 1;
  }
}

// a sequence's rows and where they are
struct RowSeq {
  int first, end;                        // rows, within [0, n_rows)
  int64_t zero;                          // the position of row r is zero + r
  int start;                             // position of the chunk's row 0, cut to +-2^30
  int cap;                               // positions at or above are not seen
};
__device__ __forceinline__ RowSeq row_seq(const ts_kv_attend_rows_args& a, int off, int end, int64_t len) {
  RowSeq s;
  s.end = max(min(end, a.n_rows), 0);
  s.first = min(max(off, 0), a.n_rows);                      // both cut, so that their difference fits whatever the offsets are
  s.zero = len - off;
  s.start = (int)max((int64_t)-(1 << 30), min((int64_t)1 << 30, len));
  s.cap = (int)min((int64_t)a.max_len, (int64_t)a.table_width * 16);
  return s;
}
__device__ __forceinline__ RowSeq row_seq(const ts_kv_attend_rows_args& a, int seq) {
  return a.row_offsets ? row_seq(a, a.row_offsets[seq], a.row_offsets[seq + 1], a.lengths[seq]) : row_seq(a, seq, seq + 1, a.lengths[seq]);
}
// The sequence of the t-th tile of at most TM columns, its first column and their number; -1 if there is none.  A sequence's columns go
// to as many tiles as they need, evenly in units of UNIT, its last rows first, and the sequences with the highest positions
// come first (up to 16 of them): what takes longest starts first.  (rows x heads of a call are below 2^24.)
template <int TM, int UNIT>
__device__ __forceinline__ int tile_of(const ts_kv_attend_rows_args& a, int G, int seq_tiles, int t, int& m0, int& cols, RowSeq& rs) {
  int seq, tile;                                             // the tile of the sequence
  if (!a.row_offsets) {
    seq = t / seq_tiles;
    tile = t - seq * seq_tiles;
    rs = row_seq(a, seq);
  } else if (a.n_seqs < 64) {                                // offsets and lengths in one trip to memory
    const int lane = threadIdx.x % 64, off = a.row_offsets[min(lane, a.n_seqs)], len = a.lengths[min(lane, a.n_seqs - 1)];
    const int end = __shfl_down(off, 1, 64);
    const int rows = lane < a.n_seqs ? max(0, max(min(end, a.n_rows), 0) - min(max(off, 0), a.n_rows)) : 0, tiles = (rows * G + TM - 1) / TM;
    int before = 0;                                          // tiles of the sequences that come first
    if (a.n_seqs <= 16) {
      const int64_t top = (int64_t)len + rows;
      const int key = (int)max((int64_t)0, min(top, (int64_t)1 << 30));
      for (int i = 0; i < a.n_seqs; ++i) {
        const int k = __builtin_amdgcn_readlane(key, i), n = __builtin_amdgcn_readlane(tiles, i);
        before += k > key || (k == key && i < lane) ? n : 0;
      }
    } else {
      before = tiles;
#pragma unroll
      for (int o = 1; o < 64; o *= 2) {
        const int x = __shfl_up(before, o, 64);
        before += lane >= o ? x : 0;
      }
      before -= tiles;
    }
    const uint64_t in = __ballot(t >= before && t - before < tiles);
    if (!in) return -1;
    seq = __builtin_ctzll(in);
    tile = t - __builtin_amdgcn_readlane(before, seq);
    rs = row_seq(a, __builtin_amdgcn_readlane(off, seq), __builtin_amdgcn_readlane(end, seq), __builtin_amdgcn_readlane(len, seq));
  } else {
    // sequence s has places [off group / TM + s, ...): as many as its tiles or one more, without a sum over the others.  Where offsets
    // decrease the search may end at a sequence whose place lies behind t, or at an empty one: no tile of theirs, see below.
    auto place = [&](int s) { return min(max(a.row_offsets[s], 0), a.n_rows) * G / TM + s; };
    seq = __builtin_amdgcn_readfirstlane(last_at_most(a.n_seqs, t, place));
    if (seq < 0) return -1;
    tile = t - place(seq);
    rs = row_seq(a, seq);
  }
  const int M = (rs.end - rs.first) * G, tiles = (M + TM - 1) / TM;
  if (tile < 0 || tile >= tiles) return -1;                  // past this line there is a tile, and so a column
  const int step = (M + tiles * UNIT - 1) / (tiles * UNIT) * UNIT;
  m0 = (tiles - 1 - tile) * step;
  cols = min(step, M - m0);
  return seq;
}
