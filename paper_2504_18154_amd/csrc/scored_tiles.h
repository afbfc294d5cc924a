// How attention of prompts with formed scores (attn_scored_prefill.hip) numbers its tiles.  Plain arithmetic, for the kernel, its launch and for a host program alike.
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

}  // namespace eco
