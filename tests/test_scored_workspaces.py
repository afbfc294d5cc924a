"""Workspaces of attention of prompts with formed scores, and the largest calls on such caches: one of the most that any call takes serves every call, whose own need rises and falls with its tokens.  Without a GPU: a
program brings its own device and counts launches; then, on one, small calls in the room of a large one leave the same results."""
import numpy as np
import pytest
import torch

from tests.test_sparse_workspaces import _run

PROGRAM = r"""
static int launches = 0;
extern "C" {
hipError_t __hipPushCallConfiguration(dim3, dim3, size_t, hipStream_t) { return hipSuccess; }
hipError_t __hipPopCallConfiguration(dim3* g, dim3* b, size_t* n, hipStream_t* s) { return *g = *b = dim3(1), *n = 0, *s = nullptr, hipSuccess; }
hipError_t hipLaunchKernel(const void*, dim3, dim3, void**, size_t, hipStream_t) { return ++launches, hipSuccess; }
}
alignas(16) static char mem[64];
int main() {
  room = (size_t)16 << 30;
  int bad = 0;
  void* const p = mem;
  int32_t* const i = (int32_t*)mem;
  const ecoserve_cache cache = {ECOSERVE_CACHE_E4M3, p, p, (uint8_t*)p};
  const struct { int Hq, Hkv, D; } lays[] = {{64, 8, 128}, {8, 1, 256}, {52, 52, 128}, {32, 8, 64}, {5, 1, 128}, {16, 1, 128}, {1, 1, 16}, {512, 512, 16}};
  for (const auto& l : lays) {
    ecoserve_layout lay = {};
    lay.num_q_heads = l.Hq, lay.num_kv_heads = l.Hkv, lay.head_dim = l.D, lay.block_size = 16, lay.num_blocks = 4, lay.dtype = ECOSERVE_BF16;
    ecoserve_ctx* c = nullptr;
    if (ecoserve_create(&c, 0, &lay, 512, 4096)) return std::printf("not created\n"), 1;
    const size_t most = ecoserve_prefill_scored_workspace_most(c);
    size_t seen = 0;
    for (int B : {1, 2, 3, 7, 24, 64, 65, 200, 512})
      for (int T = 1; T <= 70000; T += 1 + T / 9) {
        const size_t bytes = ecoserve_prefill_scored_workspace_bytes(c, B, T);
        if (bytes > seen) seen = bytes;
        const int was = launches, st = ecoserve_attn_prefill_scored(c, &cache, nullptr, p, (int64_t)l.Hq * l.D, i, i, i, 4096, p, nullptr, B, T, p, most, nullptr);
        if (bytes > most || st || launches == was) ++bad, std::printf("%d heads on %d, %d sequences, %d tokens: %zu of %zu bytes, status %d\n", l.Hq, l.Hkv, B, T, bytes, most, st);
      }
    if (2 * seen < most && l.Hkv <= 128) ++bad, std::printf("%d heads on %d: %zu bytes at most, not %zu\n", l.Hq, l.Hkv, seen, most);
    ecoserve_destroy(c);
  }
  if (ecoserve_prefill_scored_workspace_most(nullptr) != 0) ++bad;
  std::printf("%d\n", bad);
  return bad != 0;
}
"""


def test_a_workspace_for_any_call_serves_every_call(tmp_path):
    assert _run(tmp_path, PROGRAM) == "0\n"


THREADS = r"""
static int launches = 0;
static dim3 grid, block;
extern "C" {
hipError_t __hipPushCallConfiguration(dim3 g, dim3 b, size_t, hipStream_t) { return grid = g, block = b, hipSuccess; }
hipError_t __hipPopCallConfiguration(dim3* g, dim3* b, size_t* n, hipStream_t* s) { return *g = grid, *b = block, *n = 0, *s = nullptr, hipSuccess; }
hipError_t hipLaunchKernel(const void*, dim3 g, dim3 b, void**, size_t, hipStream_t) {
  ++launches;
  return (uint64_t)g.x * b.x >> 32 || (uint64_t)g.y * b.y >> 32 ? hipErrorInvalidConfiguration : hipSuccess;
}
}
alignas(16) static char mem[64];
int main() {
  room = (size_t)64 << 30;
  int bad = 0;
  void* const p = mem;
  int32_t* const i = (int32_t*)mem;
  const ecoserve_cache cache = {ECOSERVE_CACHE_INT8, p, p, (uint8_t*)p};
  const struct { int Hq, Hkv, D; } lays[] = {{1, 1, 16}, {16, 1, 16}, {512, 512, 16}, {64, 8, 128}};
  for (const auto& l : lays) {
    ecoserve_layout lay = {};
    lay.num_q_heads = l.Hq, lay.num_kv_heads = l.Hkv, lay.head_dim = l.D, lay.block_size = 16, lay.num_blocks = 4, lay.dtype = ECOSERVE_BF16;
    ecoserve_ctx* c = nullptr;
    if (ecoserve_create(&c, 0, &lay, 4096, 4096)) return std::printf("not created\n"), 1;
    const int64_t row = (int64_t)l.Hq * l.D, kv_row = (int64_t)l.Hkv * l.D;
    const size_t most = ecoserve_prefill_scored_workspace_most(c);
    auto expect = [&](const char* what, int B, int64_t T, bool ok, auto call) {
      const int was = launches, st = call(B, (int32_t)T);
      if (st != (ok ? ECOSERVE_OK : ECOSERVE_EINVAL) || (launches != was) != ok) ++bad, std::printf("%s: %d heads on %d, %d sequences, %lld tokens: status %d\n", what, l.Hq, l.Hkv, B, (long long)T, st);
    };
    for (int B : {1, 64, 4096}) {
      auto prefill = [&](int b, int32_t t) { return ecoserve_attn_prefill_scored(c, &cache, nullptr, p, row, i, i, i, 4096, p, nullptr, b, t, p, most, nullptr); };
      const int64_t threads = (0x7fffffffLL - 256LL * B * l.Hkv) / l.Hq, rows = (0x7fffffffLL - 256) / (l.Hq / l.Hkv), last = threads < rows ? threads : rows;
      expect("prompts", B, last, true, prefill), expect("prompts", B, last + 1, false, prefill);
      auto append = [&](int b, int32_t t) { return ecoserve_kv_append_norm(c, &cache, nullptr, nullptr, nullptr, nullptr, nullptr, 0, nullptr, 0, p, p, kv_row, i, i, i, 4096, b, t, t, nullptr); };
      auto read = [&](int b, int32_t t) { return ecoserve_kv_read(c, &cache, p, p, kv_row, i, i, i, 4096, b, t, nullptr); };
      const int64_t edge = (1LL << 28) - 32 * B - 1;
      expect("append", B, edge, true, append), expect("append", B, edge + 1, false, append);
      expect("read", B, edge, true, read), expect("read", B, edge + 1, false, read);
    }
    ecoserve_destroy(c);
  }
  std::printf("%d\n", bad);
  return bad != 0;
}
"""


def test_calls_of_more_threads_than_a_launch_takes_are_refused(tmp_path):
    assert _run(tmp_path, THREADS) == "0\n"


@pytest.mark.gpu
def test_small_calls_in_the_room_of_a_large_one():
    from tests.scored_util import Pools, packed
    from tests.test_gpu_scored import _prefill, _q
    total = np.array([3000, 40])
    p = Pools("int8", 128, 8, 2, total, seed=1)
    p.fill(total, 2)
    n = p.ctx.prefill_scored_workspace_most()
    room = torch.full((n + 4096,), 77, dtype=torch.uint8, device="cuda")
    for new in ([1, 0], [3, 40], [100, 7], [3000, 40]):
        new = np.array(new)
        assert p.ctx.prefill_scored_workspace_bytes(2, int(new.sum())) <= n
        q = _q(int(new.sum()), p, 3)
        want = _prefill(p, total - new, new, q)
        got = _prefill(p, total - new, new, q, workspace=room[:n])
        assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1]) and (room[n:] == 77).all()
    p.ctx.close()
