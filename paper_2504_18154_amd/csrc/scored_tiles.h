// How attention of prompts with formed scores (attn_scored_prefill.hip) numbers its tiles, and which keys and blocks a tile has to do with.  Plain arithmetic, for the kernel, its launch and for a host program alike.
#pragma once

#include <stdint.h>

#if defined(__HIPCC__)
#define ECO_TILES_HD __host__ __device__ __forceinline__
#else
#define ECO_TILES_HD inline
#endif

namespace eco {

// Tiles of `rows` rows ((position, query head) pairs of a K/V head) of a batch, and the number of sequence b's first one, `cu` tokens in front of it.  Sequences without new
// tokens have none: no more than min(b, cu) of the sequences in front of b have tokens, each of which takes one tile more than its rows fill at most.  Numbers never
// fall from sequence to sequence; a tile is the last sequence's whose first number is not above the tile's.
ECO_TILES_HD int64_t prefill_scored_tiles(int32_t rows, int32_t B, int32_t T, int32_t G) { return (int64_t)T * G / rows + (B < T ? B : T); }
ECO_TILES_HD int64_t prefill_scored_first_tile(int32_t rows, int32_t G, int32_t cu, int32_t b) { return (int64_t)cu * G / rows + (b < cu ? b : cu); }

// Keys k0 .. k0 + 63 that a row of the range [lo, hi) sees, a bit each.
ECO_TILES_HD uint64_t keys_seen(int32_t lo, int32_t hi, int32_t k0) {
  const int32_t from = lo - k0 < 0 ? 0 : lo - k0, to = hi - k0 > 64 ? 64 : hi - k0;
  return from < to ? ~(uint64_t)0 >> (64 - (to - from)) << from : 0;
}
// Whether the ranges of neighbouring rows leave keys between them, or one of the rows has none (a range of no keys: lo 2^31 - 1, hi 0).  A tile whose rows all touch their
// neighbours sees every key from its first to its last.
ECO_TILES_HD bool ranges_apart(int32_t lo, int32_t hi, int32_t next_lo, int32_t next_hi) { return next_lo > hi || lo > next_hi; }
// The entry of the block table that stands for block `blk` of a tile that sees keys of the blocks first .. last: the block's own, if the tile sees a key of it.  `gaps`: the tile
// may see none between others; `seen`: the keys of the four blocks of this one's step that it sees.
ECO_TILES_HD int32_t entry_of_block(int32_t blk, int32_t first, int32_t last, bool gaps, uint64_t seen) {
  if (gaps) return (seen >> (16 * (blk & 3)) & 0xffff) != 0 ? blk : first;
  return blk < first ? first : blk > last ? last : blk;
}

}  // namespace eco
