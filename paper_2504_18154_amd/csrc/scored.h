// Argument blocks, partitions and workspaces of attention over the caches of ecoserve_cache.  Plain arithmetic, for the launches, the entry points and a
// host program alike.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#include "common.h"
#include "scored_tiles.h"

namespace eco {

struct ScoredArgs {
  const void* q;
  int32_t q_row_stride;
  const void *k_cache, *v_cache;
  const uint8_t* scales;
  const int32_t *cu_q, *ctx_before;  // prompts; decode: ctx_before is ctx_len and cu_q NULL
  const int32_t* block_table;
  int32_t bt_stride;
  void* out;
  float* lse;
  const float* slopes;
  const int32_t *key_begin, *key_end;
  int32_t B, T, Hq, Hkv, D, format, num_cu;
  float scale_log2e;  // scores live in the exp2 domain
  float softcap;      // 0: none
  float* states;
  uint32_t* counters;  // zero between launches
  int32_t max_ctx_len = 0;  // decode: a bound on the lengths, for the choice of a launch alone
};

constexpr int32_t scored_chunks(int32_t D) { return D <= 64 ? 2 : D <= 128 ? 4 : 8; }  // of 32 channels, that a kernel's instance holds
// Floats of a slice's state of one query head: the unnormalised head vector, its maximum and its sum, and two that keep 16 bytes aligned.
constexpr int32_t scored_state_words(int32_t D) { return D + 4; }

// Decode: the steps of 64 tokens of every (sequence, K/V head) are one numbering, cut into equal shares, one per workgroup.
constexpr int32_t kScoredMostPieces = 256;  // of a (sequence, K/V head)
constexpr int32_t kLeastSteps = 8;          // of a share
constexpr int32_t kShortShare = 16;         // (see the kernel)
constexpr int32_t kPieceCost = 4;           // units in front of a (sequence, K/V head)'s steps
// Workgroups of four wavefronts that a CU holds, by the registers of the kernel's instances (chunks: of 32 channels; wide: groups of more than eight heads, whose weights' second parts are products of their
// own.  Over codes of 128 channels these spill with two: 64 x 100 ... 4000 tokens, 40 heads on 8, as wide ones, 74 us for 57 with weights in one part; with one, 64 heads on 4, 48 for 44).
constexpr int32_t decode_scored_waves(bool narrow, int32_t chunks, bool wide) { return chunks == 8 || (chunks == 4 && (!narrow || wide)) ? 1 : 2; }
// Short batches over coded caches, a CU's share of which one workgroup takes: it has eight wavefronts, and twice as many bytes on their way.  One sequence of
// 20 000 tokens: 22.3 us with four, 20.7 with eight.  (Long ones leave no difference between two workgroups of four and one of eight but their barriers.)
inline bool decode_scored_short(int64_t steps, bool narrow, int32_t chunks, int32_t num_cu) { return narrow && chunks <= 4 && steps <= (int64_t)kShortShare * num_cu; }
// A workgroup cuts two (sequence, K/V head)s at most.
constexpr int64_t decode_scored_states(int32_t chunks, int32_t num_cu) { return 2 * (int64_t)decode_scored_waves(true, chunks, false) * num_cu; }
inline size_t decode_scored_workspace(const ecoserve_layout& L, int32_t num_cu) {
  return (size_t)decode_scored_states(scored_chunks(L.head_dim), num_cu) * (L.num_q_heads / L.num_kv_heads) * scored_state_words(L.head_dim) * 4;
}

// Prompts: tiles of 128 or 256 rows ((position, query head) pairs of a K/V head), their 64-key steps cut among `prefill_scored_splits` workgroups where tiles are few.
constexpr int32_t kTileRows = 128, kMostTileRows = 256;
// Rows of a tile, 32 to a wavefront: the more of them there are, the fewer turn a step's codes into operands for themselves.  (Heads of up to 64 channels have no 16
// bytes of a step for each of eight wavefronts, those of more than 128 no registers for two on a SIMD.)  64 heads on 8 of 128, in tiles of 128 and 256 rows: two
// prompts of 8192 tokens over e4m3 2200 and 2140 us, 2048 tokens of three over bf16 131 and 128.  Short prompts would leave the larger ones half empty.
inline int32_t prefill_scored_rows(const ecoserve_layout& L, int32_t B, int32_t T, int32_t num_cu) {
  const int32_t G = L.num_q_heads / L.num_kv_heads;
  return scored_chunks(L.head_dim) == 4 && (int64_t)T * G >= 4 * (int64_t)kMostTileRows * B && prefill_scored_tiles(kMostTileRows, B, T, G) * L.num_kv_heads >= 2 * num_cu ? kMostTileRows : kTileRows;
}
inline int32_t prefill_scored_splits(const ecoserve_layout& L, int32_t rows, int32_t B, int32_t T, int32_t num_cu) {
  const int64_t items = prefill_scored_tiles(rows, B, T, L.num_q_heads / L.num_kv_heads) * L.num_kv_heads, room = 2 * (int64_t)num_cu / std::max<int64_t>(items, 1);
  return room < 2 ? 1 : (int32_t)std::min<int64_t>(room, 32);
}
constexpr int64_t prefill_scored_state_floats(int32_t rows, int32_t D) { return rows * (32 * (int64_t)scored_chunks(D) + 2); }
inline size_t prefill_scored_workspace(const ecoserve_layout& L, int32_t B, int32_t T, int32_t num_cu) {
  const int32_t rows = prefill_scored_rows(L, B, T, num_cu), splits = prefill_scored_splits(L, rows, B, T, num_cu);
  if (splits == 1) return 0;
  return (size_t)splits * prefill_scored_tiles(rows, B, T, L.num_q_heads / L.num_kv_heads) * L.num_kv_heads * prefill_scored_state_floats(rows, L.head_dim) * 4;
}
// The largest that is: parts are two workgroups per CU at most, and tiles of 256 rows are never cut.
inline size_t prefill_scored_workspace_most(const ecoserve_layout& L, int32_t num_cu) { return 2 * (size_t)num_cu * prefill_scored_state_floats(kTileRows, L.head_dim) * 4; }

// decode of a few tokens and prompts (attn_scored_decode.hip, attn_scored_prefill.hip)
hipError_t launch_decode_scored(const ScoredArgs& a, hipStream_t s);
hipError_t launch_prefill_scored(const ScoredArgs& a, int32_t rows, int32_t splits, hipStream_t s);

// The append with norms, rotation and coding on the way, and reading back (kv_norm.hip)
struct NormAppend {
  const void* q;  // NULL: K and V alone
  int32_t q_row_stride;
  void* q_out;
  int32_t q_out_row_stride;
  void *k_cache, *v_cache;
  uint8_t* scales;
  const void *k_new, *v_new;
  int32_t new_row_stride;
  const int32_t *cu_q, *ctx_before, *block_table;
  int32_t bt_stride, B, T, max_new_len, Hq, Hkv, D, format, num_cu;
  bool norm;
  float eps;
  const float *q_weight, *k_weight;  // or NULL
  int32_t weight_stride;             // 0: one for all heads
};
hipError_t launch_kv_append_norm(const NormAppend& a, const ecoserve_rope* rope, const double* inv_freq, const int32_t* positions, hipStream_t s);
struct ReadBack {
  const void *k_cache, *v_cache;
  const uint8_t* scales;
  void *k_rows, *v_rows;
  int32_t row_stride;
  const int32_t *cu, *first, *block_table;
  int32_t bt_stride, B, T, Hkv, D, format, num_cu;
};
hipError_t launch_kv_read(const ReadBack& a, hipStream_t s);

}  // namespace eco
