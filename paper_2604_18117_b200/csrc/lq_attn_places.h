// How the attention's form for few rows shares out its records over the blocks of its grid.  Apart from the kernel so that a test can compile
// it by itself.  Internal: not part of the C ABI.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define LQ_HD __host__ __device__ __forceinline__
#else
#define LQ_HD inline
#endif

// (most numbers here are below 2^32, where a division is a few instructions)
LQ_HD long long lq_quotient(long long a, long long b) {
  return ((a | b) >> 32) == 0 ? (long long)((uint32_t)a / (uint32_t)b) : a / b;
}

// A place in the launch's row of records: sequence by sequence, head by head, tile of rows by tile of rows.  SEQ: what is known of a sequence.
template <typename SEQ>
struct LqAttnPlace {
  SEQ q;
  int s, tiles, each;                    // tiles: of rows of the sequence (0: not the launch's); each: records of a tile
  int head, tile, i;                     // i: record of the tile
};
// records of a place's sequence
template <typename SEQ>
LQ_HD long long lq_attn_records(const LqAttnPlace<SEQ>& at, int heads) { return (long long)at.tiles * at.each * heads; }

// n records on; false: behind the last.  measure(s): a place at the beginning of sequence s.
template <typename SEQ, typename Measure>
LQ_HD bool lq_attn_walk(LqAttnPlace<SEQ>& at, int n, int heads, int sequences, const Measure& measure) {
  at.i += n;
  while (at.i >= at.each) {
    const int left = at.i - at.each;
    at.i = left;
    if (++at.tile < at.tiles) continue;
    at.tile = 0;
    if (++at.head < heads && at.tiles > 0) continue;
    do {
      if (at.s + 1 >= sequences) return false;
      at = measure(at.s + 1);
    } while (at.tiles == 0);
    at.i = left;
  }
  return true;
}

// Where a block's records begin that would begin with the edge-th: there, or, within a tile of at most `small` records, behind that tile.  The edge
// lies among the records of the sequences from `at` on, of which the first is the from-th.  Returns the record, `at` becomes its place within
// the tile that has the edge (i = each: behind it).
template <typename SEQ, typename Measure>
LQ_HD long long lq_attn_edge(LqAttnPlace<SEQ>& at, long long from, long long edge, int heads, int small, const Measure& measure) {
  while (edge - from >= lq_attn_records(at, heads)) {
    from += lq_attn_records(at, heads);
    at = measure(at.s + 1);
  }
  const long long tile = lq_quotient(edge - from, at.each);
  at.i = (int)(edge - from - tile * at.each);
  at.head = (int)lq_quotient(tile, at.tiles);
  at.tile = (int)(tile - (long long)at.head * at.tiles);
  if (at.i > 0 && at.each <= small) {
    edge += at.each - at.i;
    at.i = at.each;
  }
  return edge;
}

// How records are shared out over `grid` blocks.  With few tiles (at most half the blocks) every tile that is not small is cut in equal parts for
// blocks of their own: a block that has the end of one tile and the beginning of another joins twice, which took a fifth of a long sequence's time.  With
// more of them blocks have neighbouring records, as even as can be.
struct LqAttnCut {
  bool parted;
  long long share;                       // records of a block: the most, or exactly
};
LQ_HD LqAttnCut lq_attn_cut(long long records, long long tiles, int grid, int least) {
  const bool parted = 2 * tiles <= grid;
  const long long blocks = parted ? grid - tiles : grid, share = lq_quotient(records + blocks - 1, blocks);
  return {parted, share < least ? least : share};
}
// parts of a tile (parted): together no more than there are blocks
LQ_HD int lq_attn_parts(int each, const LqAttnCut& cut, int small) {
  return each <= small ? 1 : (int)lq_quotient(each + cut.share - 1, cut.share);
}
// what is counted along the sequences: blocks, or records
template <typename SEQ>
LQ_HD long long lq_attn_count(const LqAttnPlace<SEQ>& at, int heads, const LqAttnCut& cut, int small) {
  return cut.parted ? (long long)at.tiles * heads * (at.tiles > 0 ? lq_attn_parts(at.each, cut, small) : 0) : lq_attn_records(at, heads);
}
// Parted: the place where block `block` begins; the sequences from `at` on have the blocks from the from-th on.  Returns how many records it has; part:
// which of its tile's parts it is.
template <typename SEQ, typename Measure>
LQ_HD int lq_attn_part(LqAttnPlace<SEQ>& at, long long from, long long block, int heads, int small, const LqAttnCut& cut, int& part, int& parts,
                       const Measure& measure) {
  while (block - from >= lq_attn_count(at, heads, cut, small)) {
    from += lq_attn_count(at, heads, cut, small);
    at = measure(at.s + 1);
  }
  parts = lq_attn_parts(at.each, cut, small);
  const long long tile = lq_quotient(block - from, parts);
  part = (int)(block - from - tile * parts);
  at.head = (int)lq_quotient(tile, at.tiles);
  at.tile = (int)(tile - (long long)at.head * at.tiles);
  at.i = (int)lq_quotient((long long)at.each * part, parts);
  return (int)lq_quotient((long long)at.each * (part + 1), parts) - at.i;
}
