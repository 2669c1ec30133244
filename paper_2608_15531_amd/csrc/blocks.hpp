// Which tiles of keys the blocks of rows of fq_paged_attention see, and how blocks and ranges
// are numbered: plain arithmetic, for the kernels, the launch plan and host tests alike.
#pragma once

#include <stdint.h>

#include "host_device.hpp"

namespace fqi {

// Blocks of `rows` rows are numbered by the rows before them: a sequence whose rows are
// r .. s - 1 has at most as many as s / rows - r / rows + 1, so the numbers of sequences
// that follow one another differ and stay below dense_blocks.
FQ_HOST_DEVICE int64_t dense_number(int64_t t0, int group, int rows, int seq, int rb) {
  return t0 * group / rows + seq + rb;
}
FQ_HOST_DEVICE int64_t dense_blocks(int64_t total_q, int64_t group, int rows, int64_t n_seqs) {
  return total_q * group / rows + n_seqs;
}

// Which tiles a block of rows at positions [p_lo, p_hi] sees: with a window, the tiles of
// the first keys and those of the window, numbered one after the other.
struct TileRange {
  int first;   // tiles of the first keys
  int skip;    // tiles between those and the window
  int n;
  FQ_HOST_DEVICE int tile(int i) const { return i < first ? i : i + skip; }
};

template <int TILE>
FQ_HOST_DEVICE TileRange tile_range(int p_lo, int p_hi, int window, int sinks) {
  TileRange r;
  const int end = p_hi < 0 ? 0 : p_hi / TILE + 1;   // p_hi is the last key seen
  r.first = 0;
  r.skip = 0;
  if (window > 0 && p_lo >= window) {
    const int lo = (p_lo - window + 1) / TILE;
    const int last = sinks < p_lo + 1 ? sinks : p_lo + 1, sink_tiles = (last + TILE - 1) / TILE;
    r.first = lo < sink_tiles ? lo : sink_tiles;
    r.skip = lo - r.first;
  }
  r.n = end - r.skip;
  if (r.n < 0) r.n = 0;
  return r;
}

// How many ranges of split_tiles tiles n tiles fall into, of at most `split`.
FQ_HOST_DEVICE int range_count(int n, int split_tiles, int split) {
  const int want = (n + split_tiles - 1) / split_tiles, some = want > 1 ? want : 1;
  return some < split ? some : split;
}

}  // namespace fqi
