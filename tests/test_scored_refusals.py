"""What the entry points for formed scores refuse at the ends of their ranges, without a GPU, and what the compiler reports of their kernels."""
import os
import re
import subprocess

import pytest

from paper_2504_18154_amd import build
from tests.test_kernel_registers import _assert_none, _scratch_and_spills
from tests.test_workspace import ALLOCATOR

LIMITS = r"""
extern "C" hipError_t hipLaunchKernel(const void*, dim3, dim3, void**, size_t, hipStream_t) { std::printf("launched\n"); std::fflush(stdout); std::_Exit(9); }
alignas(16) static char mem[4096];
static int bad = 0;
#define EXPECT(call, want) do { const int st = (call); if (st != (want)) std::printf("line %d: %d, not %d: %s\n", __LINE__, st, (int)(want), #call), ++bad; } while (0)
int main() {
  room = (size_t)1 << 34;  // (address space: nothing is touched)
  ecoserve_layout lay = {};
  lay.num_q_heads = 1, lay.num_kv_heads = 1, lay.head_dim = 16, lay.block_size = 16, lay.num_blocks = 64, lay.dtype = ECOSERVE_BF16;
  ecoserve_ctx* c = nullptr;
  if (ecoserve_create(&c, 0, &lay, 64, 1 << 26)) return std::printf("not created\n"), 1;
  const int EI = ECOSERVE_EINVAL;
  int32_t* const i = (int32_t*)mem;
  float* const w = (float*)mem;
  void* const p = mem;
  const ecoserve_cache e = {ECOSERVE_CACHE_E4M3, p, p, (uint8_t*)p};
  const size_t big = (size_t)1 << 30;
  // 64 sequences of 2^30 tokens: 2^31 half steps and more
  EXPECT(ecoserve_attn_decode_scored(c, &e, nullptr, p, 16, i, 1 << 26, i, p, w, 64, 1 << 30, p, big, nullptr), EI);
  for (const float cap : {1e-39f, 1e-45f, -0x1p-126f}) {
    const ecoserve_scores s = {cap, nullptr, nullptr, nullptr};
    EXPECT(ecoserve_attn_decode_scored(c, &e, &s, p, 16, i, 8, i, p, w, 2, 100, p, big, nullptr), EI);
    EXPECT(ecoserve_attn_prefill_scored(c, &e, &s, p, 16, i, i, i, 8, p, w, 2, 9, p, big, nullptr), EI);
  }
  // (a cap of -0 is none, and the least that there may be is one)
  for (const float cap : {-0.f, 0x1p-126f}) {
    const ecoserve_scores s = {cap, nullptr, nullptr, nullptr};
    EXPECT(ecoserve_attn_prefill_scored(c, &e, &s, p, 16, i, i, i, 8, p, w, 2, 0, p, big, nullptr), ECOSERVE_OK);
  }
  ecoserve_destroy(c);
  std::printf("%d\n", bad);
  return bad != 0;
}
"""


def test_limits_are_refused_before_any_launch(tmp_path):
    if not os.path.exists(build.LIB):
        pytest.skip("the library is not built")
    src, exe = tmp_path / "limits.cpp", tmp_path / "limits"
    src.write_text(ALLOCATOR + LIMITS)
    rocm = os.path.dirname(os.path.dirname(os.path.realpath(build._hipcc())))
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", build.INCLUDE, "-I", os.path.join(rocm, "include"), str(src), "-o", str(exe), "-rdynamic", build.LIB,
                    f"-Wl,-rpath,{os.path.dirname(build.LIB)}:{os.path.join(rocm, 'lib')}", f"-Wl,-rpath-link,{os.path.join(rocm, 'lib')}"], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and r.stdout == "0\n", r.stdout + r.stderr[-500:]


def test_append_and_read_do_not_spill(tmp_path):
    of = _scratch_and_spills(tmp_path, "kv_norm.hip")
    _assert_none(of, "kv_append_norm_kernel", 36)
    _assert_none(of, "kv_append_norm_one_kernel", 18)
    _assert_none(of, "kv_read_kernel", 3)
