"""Workspaces of block selection and of attention over listed blocks: one that is sized for the longest contexts and the most tokens serves every smaller call.  Without a GPU: a
program brings its own device and counts launches; then, on one, calls in less room leave the same lists and touch nothing behind it."""
import os
import subprocess

import numpy as np
import pytest
import torch

from paper_2504_18154_amd import build
from paper_2504_18154_amd import workloads as wl
from tests.test_workspace import ALLOCATOR

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
  const int Ts[] = {1, 2, 3, 7, 8, 9, 64, 512, 700, 4096, 20000, 32768, 40000, 1000000}, ctxs[] = {1, 256, 2000, 32768, 50000, 131072, 1000000, 3000000, 16000000};
  const struct { int Hq, Hkv, D, dtype; } lays[] = {{64, 8, 128, ECOSERVE_BF16}, {8, 1, 256, ECOSERVE_BF16}, {52, 52, 128, ECOSERVE_BF16}, {4, 2, 64, ECOSERVE_F32}, {512, 512, 8, ECOSERVE_BF16}};
  for (const auto& l : lays) {
    ecoserve_layout lay = {};
    lay.num_q_heads = l.Hq, lay.num_kv_heads = l.Hkv, lay.head_dim = l.D, lay.block_size = 16, lay.num_blocks = 4, lay.dtype = l.dtype;
    ecoserve_ctx* c = nullptr;
    if (ecoserve_create(&c, 0, &lay, 8, 1000000)) return std::printf("not created\n"), 1;
    const int64_t row = (int64_t)l.Hq * l.D;
    for (int T : Ts)
      for (int ctx : ctxs) {
        const size_t bytes = ecoserve_select_workspace_bytes(&lay, T, ctx);
        for (int t : Ts)
          for (int n : ctxs)
            if (t <= T && n <= ctx) {
              const int was = launches;
              const int st = ecoserve_block_select(c, p, row, p, i, i, i, 1000000, i, 4, 1, 1, 8, t, n, p, bytes, nullptr);
              if (st || launches == was) ++bad, std::printf("%d heads, workspace of %d tokens, %d: %d tokens, %d: status %d\n", l.Hq, T, ctx, t, n, st);
            }
        // (less than a call is content with is refused)
        const size_t small = ecoserve_select_workspace_bytes(&lay, 1, ctx), least = bytes < small ? bytes : small;
        if (ecoserve_block_select(c, p, row, p, i, i, i, 1000000, i, 4, 1, 1, 8, T, ctx, p, least - 1, nullptr) != ECOSERVE_EINVAL) ++bad, std::printf("%d, %d: not refused\n", T, ctx);
      }
    const size_t most = ecoserve_sparse_workspace_most(c);
    size_t seen = 0;
    for (int T = 1; T <= 300; ++T)
      for (int K = 1; K <= 6000; K += K < 200 ? 1 : 97) {
        const size_t bytes = ecoserve_sparse_workspace_bytes(c, T, K);
        if (bytes > seen) seen = bytes;
        if (bytes > most) ++bad, std::printf("%d tokens, %d entries: %zu, at most %zu\n", T, K, bytes, most);
      }
    if (seen == 0 && l.Hkv * 2 < 256) ++bad, std::printf("no parts\n");
    ecoserve_destroy(c);
  }
  if (ecoserve_sparse_workspace_most(nullptr) != 0) ++bad;
  std::printf("%d\n", bad);
  return bad != 0;
}
"""


def _run(tmp_path, program):
    if not os.path.exists(build.LIB):
        pytest.skip("the library is not built")
    src, exe = tmp_path / "sizes.cpp", tmp_path / "sizes"
    src.write_text(ALLOCATOR + program)
    rocm = os.path.dirname(os.path.dirname(os.path.realpath(build._hipcc())))
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", build.INCLUDE, "-I", os.path.join(rocm, "include"), str(src), "-o", str(exe), "-rdynamic", build.LIB,
                    f"-Wl,-rpath,{os.path.dirname(build.LIB)}:{os.path.join(rocm, 'lib')}", f"-Wl,-rpath-link,{os.path.join(rocm, 'lib')}"], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.stderr == ""
    return r.stdout


def test_a_workspace_for_the_largest_call_serves_the_smaller_ones(tmp_path):
    assert _run(tmp_path, PROGRAM) == "0\n"


PARTS = r"""
int main() {
  room = (size_t)1 << 30;
  int bad = 0;
  for (int dtype : {ECOSERVE_BF16, ECOSERVE_F32}) {
    ecoserve_layout lay = {};
    lay.num_q_heads = 6, lay.num_kv_heads = 2, lay.head_dim = 64, lay.block_size = 16, lay.num_blocks = 4, lay.dtype = dtype;
    ecoserve_ctx* c = nullptr;
    if (ecoserve_create(&c, 0, &lay, 8, 1000)) return std::printf("not created\n"), 1;
    const int bf[][3] = {{1, 1, 1}, {1, 32, 1}, {1, 33, 5}, {1, 41, 6}, {1, 49, 7}, {1, 64, 8}, {1, 65, 8}, {1, 128, 11}, {1, 4095, 63}, {1, 4096, 64}, {1, 65536, 64}, {8, 64, 8},
                         {9, 64, 7}, {32, 64, 2}, {33, 64, 1}, {64, 129, 2}, {65, 129, 1}};
    const int f32[][3] = {{1, 1, 1}, {1, 16, 1}, {1, 17, 3}, {1, 25, 4}, {1, 32, 4}, {1, 33, 5}, {1, 64, 8}, {64, 17, 1}, {32, 17, 2}};
    auto check = [&](const int (&x)[3]) {
      const size_t want = x[2] == 1 ? 0 : (size_t)x[2] * x[0] * 6 * 68 * 4, got = ecoserve_sparse_workspace_bytes(c, x[0], x[1]);
      if (got != want) ++bad, std::printf("%d tokens, %d entries: %zu, not %zu (%d parts)\n", x[0], x[1], got, want, x[2]);
    };
    if (dtype == ECOSERVE_BF16) for (const auto& x : bf) check(x);
    else for (const auto& x : f32) check(x);
    ecoserve_destroy(c);
  }
  std::printf("%d\n", bad);
  return bad != 0;
}
"""


def test_parts_of_lists(tmp_path):
    """How many a list is cut into, 256 CUs (the workspace holds a state of each)."""
    assert _run(tmp_path, PARTS) == "0\n"


def test_what_is_held_at_a_time_stays_in_the_last_level_cache():
    from paper_2504_18154_amd import binding as b
    for lay in (b.make_layout(64, 8, 128, 10, "bf16"), b.make_layout(16, 1, 256, 10, "bf16"), b.make_layout(4, 2, 64, 10, "f32")):
        for ctx in (256, 5000, 131072, 1 << 20):
            assert b.select_workspace_bytes(lay, 1 << 20, ctx) <= 256 << 20, ctx


@pytest.mark.gpu
@pytest.mark.parametrize("one", [False, True], ids=["prompts", "step"])
def test_calls_in_less_room(one):
    """As many tokens at a time as the workspace holds: the same lists, whatever it holds, and nothing written behind it."""
    from paper_2504_18154_amd import binding
    from tests.parity_util import dev_i32
    blocks, T = 30000, 130
    rng = np.random.default_rng(5)
    ctx = binding.Context(16, 16, 32, 500, "bf16", T, blocks)
    summary = torch.randint(-100, 100, ctx.new_summary().shape, dtype=torch.int8, device="cuda")
    new = np.ones(T, dtype=np.int64) if one else np.array([60, 0, 70])
    before = rng.integers(0, blocks * 16, T) if one else np.array([blocks * 16 - 60, 5, 4000])
    table = dev_i32(rng.integers(0, 500, size=(len(new), blocks)))
    q = torch.randn(T, 16, 32, device="cuda").to(torch.bfloat16)
    want = None
    full = binding.select_workspace_bytes(ctx.layout, T, blocks * 16)
    assert full > 150 << 20
    for room in (full, 150 << 20, 96 << 20):
        ws = torch.full((full,), 0x5a, dtype=torch.uint8, device="cuda")
        lists = torch.full((T, 16, 20), -7, dtype=torch.int32, device="cuda")
        ctx.block_select(q, summary, dev_i32(before), table, lists, blocks * 16, keep_last=2, cu_q=None if one else dev_i32(wl.cu_from_lengths(new)), workspace=ws[:room])
        want = lists if want is None else want
        assert torch.equal(lists, want) and (ws[room:] == 0x5a).all()
    with pytest.raises(binding.EcoserveError):
        ctx.block_select(q, summary, dev_i32(before), table, lists, blocks * 16, keep_last=2, cu_q=None if one else dev_i32(wl.cu_from_lengths(new)), workspace=ws[:(96 << 20) - 16])
    ctx.close()
