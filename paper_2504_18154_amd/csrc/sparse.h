// Workspaces and argument blocks of block selection and of attention over listed blocks.  The sizes are plain arithmetic, for the
// launches, the entry points and a host program alike.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#include "summary.h"

namespace eco {

// Selection: one fp32 score per (token, K/V head, block), rows of whole tiles of 16 blocks.
inline int64_t select_row_words(int32_t max_ctx_len) { return ((int64_t)max_ctx_len + 255) / 256 * 16; }
constexpr int32_t kFusedBlocks = 2048;  // rows of a step up to which the launch that scores them also chooses
// Rows of the products that a token takes per K/V head: 1 << this, its heads padded to a power of two.
inline int32_t select_log_rows(const ecoserve_layout& L) {
  int32_t log = 0;
  while (L.num_kv_heads << log < L.num_q_heads) ++log;
  return log;
}
// Bytes of a token: its scores, and its query heads as whole numbers with a scale each.
inline int64_t select_score_bytes(const ecoserve_layout& L, int32_t max_ctx_len) { return 4 * select_row_words(max_ctx_len) * L.num_kv_heads; }
inline int64_t select_coded_bytes(const ecoserve_layout& L) { return ((int64_t)L.num_kv_heads << select_log_rows(L)) * (2 * summary_channels(L.head_dim)); }
inline int64_t select_scale_bytes(const ecoserve_layout& L) { return ((int64_t)L.num_kv_heads << select_log_rows(L)) * 4; }
inline int64_t select_token_bytes(const ecoserve_layout& L, int32_t max_ctx_len) {
  return select_score_bytes(L, max_ctx_len) + select_coded_bytes(L) + select_scale_bytes(L);
}
// Tokens that are taken at a time: as many as 192 MiB of scores, and 256 MiB in all, take, which stay in the last-level cache (256 MiB) between the launches.
// (8 prompts of 4096 tokens, 64 heads on 8 of 128: 256 MiB 577 us, with the scores bounded alone 610 MB 562; behind longer contexts the scores are what counts.)
inline int32_t select_tokens_at_a_time(const ecoserve_layout& L, int32_t T, int32_t max_ctx_len) {
  return (int32_t)std::max<int64_t>(1, std::min<int64_t>({(int64_t)T, ((int64_t)192 << 20) / select_score_bytes(L, max_ctx_len),
                                                          ((int64_t)256 << 20) / select_token_bytes(L, max_ctx_len), 32768}));
}
inline size_t select_workspace_bytes(const ecoserve_layout& L, int32_t T, int32_t max_ctx_len) {
  return ((size_t)select_tokens_at_a_time(L, T, max_ctx_len) * select_token_bytes(L, max_ctx_len) + 15) / 16 * 16;
}
// What a call is content with: 96 MiB or a token's bytes, if it could use more.  That many any call of more tokens or longer contexts has been given: whole tokens
// of at most 192 MiB of scores take more than half of those, and of at most 256 MiB in all more than half of these.
inline size_t select_workspace_least(const ecoserve_layout& L, int32_t T, int32_t max_ctx_len) {
  return std::min(select_workspace_bytes(L, T, max_ctx_len), std::max((size_t)96 << 20, select_workspace_bytes(L, 1, max_ctx_len)));
}

struct SelectArgs {
  const void* q;
  int32_t q_row_stride;
  const int32_t *cu_q, *ctx_before, *block_table;
  int32_t bt_stride;
  int32_t* blocks;
  int32_t num_selected, keep_first, keep_last, B, T, Hq, Hkv, D, num_cu;
  // the workspace: scores, rows of whole numbers (16-byte aligned: scores are whole tiles), their scales
  float* scores;
  int8_t* coded;
  float* scales;
  uint32_t* counters;  // one per (token, K/V head) where there is one token per sequence, zero between launches
  int32_t at_a_time;   // tokens that the workspace has room for, or all that are taken at a time
};

// Attention over listed blocks: a list is cut into parts, one workgroup each, where there are few (token, K/V head)s and the list is longer than a merge (2.5 us and 0.1 more
// per part) is worth: up to a workgroup per CU in all, for lists of up to 128 half of that; K entries are ceil(K / 8) parts at most, of about two blocks per wavefront (the shortest that
// are cut: 33 in 4 of 7 and one of 5; fp32: 17 in 2 of 6 and one of 5), no more than the root of K, so that a part has as many entries as there are parts, and 64.  (us, 40 heads on 8 of 128, bf16.  One token: 32 blocks whole 8.7, in 4 parts 9.6; 64 whole 11.9, in 4, 8, 16 parts 10.7, 9.9, 11.9; 1024 in 16, 32, 64 parts 20.6, 21.0, 25.7.
// 16 tokens: 64 whole 16.0, in 2, 4 parts 18.8, 20.2; 1024 whole 217, in 2, 4 parts 191, 192.  fp32, a block at a time, 8 heads on 2 of 64: 16 blocks whole 7.2, in 2 parts 8.2; 32 whole
// 10.0, in 4 8.2.)
inline int32_t sparse_parts(int32_t Hkv, int32_t T, int32_t num_selected, int32_t num_cu, int32_t dtype) {
  const int64_t rows = (int64_t)T * Hkv, room = (num_selected > 128 ? num_cu : num_cu / 2) / rows;
  if (room < 2 || num_selected <= (dtype == ECOSERVE_BF16 ? 32 : 16)) return 1;
  int32_t root = 1;
  while (root < 64 && (root + 1) * (root + 1) <= num_selected) ++root;
  return (int32_t)std::min<int64_t>({room, (num_selected + 7) / 8, root});
}
// Floats of a part's state of one query head: the unnormalised head vector, its maximum and its sum, and two that keep 16 bytes aligned.
constexpr int32_t sparse_state_words(int32_t D) { return D + 4; }
inline size_t sparse_workspace_bytes(const ecoserve_layout& L, int32_t T, int32_t num_selected, int32_t num_cu) {
  const int32_t parts = sparse_parts(L.num_kv_heads, T, num_selected, num_cu, L.dtype);
  return parts == 1 ? 0 : (size_t)parts * T * L.num_q_heads * sparse_state_words(L.head_dim) * 4;
}
// The largest that takes: parts of all lists are a workgroup per CU at most.
inline size_t sparse_workspace_most(const ecoserve_layout& L, int32_t num_cu) {
  return (size_t)num_cu * (L.num_q_heads / L.num_kv_heads) * sparse_state_words(L.head_dim) * 4;
}

struct SparseArgs {
  const void* q;
  int32_t q_row_stride;
  const void *k_cache, *v_cache;
  const int32_t *cu_q, *ctx_before, *block_table;
  int32_t bt_stride;
  const int32_t* blocks;
  int32_t num_selected;
  void* out;
  float* lse;
  int32_t B, T, Hq, Hkv, D, num_cu, dtype;
  float scale_log2e;
  float* states;
  uint32_t* counters;  // one per (token, K/V head) of lists in parts (at most one per CU), zero between launches
};

}  // namespace eco
