"""Rotated append, block summaries, selection and attention over listed blocks, without a GPU: the oracle's definitions against one
another, sizes of buffers and workspaces, and what the entry points refuse before they launch anything (a program that brings its
own device stands in for one; a launch there would end it)."""
import os
import subprocess

import numpy as np
import pytest
import torch

from oracle import sparse_oracle as so
from paper_2504_18154_amd import build
from tests.test_workspace import ALLOCATOR


# ---- the oracle -----------------------------------------------------------------------------------


def test_a_rotation_keeps_lengths_and_the_angle_between_positions():
    """|x| stays, and q.k after both are turned depends on the distance alone, whichever way pairs lie."""
    rng = np.random.default_rng(1)
    freq = 10000.0 ** (-np.arange(8) / 8)
    for adjacent in (False, True):
        q, k = rng.normal(size=16), rng.normal(size=16)
        at = lambda x, p: so.rotate(x, np.full(8, p), freq, adjacent)[0]
        assert np.isclose(np.linalg.norm(at(q, 37)), np.linalg.norm(q), rtol=1e-12)
        assert np.isclose(at(q, 105) @ at(k, 100), at(q, 5) @ at(k, 0), rtol=0, atol=1e-12)
        assert np.allclose(at(q, 0), q, atol=0)
    # a quarter turn of one pair by hand
    one = so.rotate(np.array([2.0, 3.0]), np.array([1]), np.array([np.pi / 2]), False)[0]
    assert np.allclose(one, [-3, 2], atol=1e-15)


def test_codes_bound_the_keys_and_the_score_bounds_the_products():
    rng = np.random.default_rng(2)
    for scale in (1e-6, 1.0, 300.0):
        keys = (rng.normal(size=(16, 24)) * scale).astype(np.float32)
        codes, e = so.summarise(keys)
        assert np.abs(codes).max() <= 127 and np.abs(codes).max() >= 63
        assert (codes[0] * 2.0 ** e >= keys.max(0)).all() and (codes[1] * 2.0 ** e <= keys.min(0)).all()
        q = rng.normal(size=24)
        qc, eq = so.query_codes(q)
        coded = qc * 2.0 ** eq
        assert np.abs(coded - q).max() <= 2.0 ** eq / 2
        assert so.scores(q[None], codes[None], np.array([e]))[0] >= (keys.astype(np.float64) @ coded).max()
    assert so.summarise(np.full((16, 4), np.inf))[1] == 127 and so.summarise(np.full((16, 4), np.nan))[1] == 127
    assert so.summarise(np.zeros((16, 4)))[1] == -126
    # 127 units are the most; a hair more takes the next exponent
    assert so.code_exponent(127.0) == 0 and so.code_exponent(127.5) == 1 and so.code_exponent(63.5) == -1


def test_choosing_by_hand():
    s = np.array([5.0, 1, 7, 7, 2, 7, 0, 3])
    assert so.choose(s, 8, 4, 0, 1) == [2, 3, 5, 7]
    assert so.choose(s, 8, 3, 0, 1) == [2, 3, 7]
    assert so.choose(s, 8, 3, 1, 2) == [0, 6, 7]
    assert so.choose(s, 3, 5, 1, 2) == [0, 1, 2]


def test_attention_over_all_blocks_is_attention():
    rng = np.random.default_rng(3)
    q, k, v = rng.normal(size=(2, 8)), rng.normal(size=(5, 8)), rng.normal(size=(5, 8))
    out, lse, _, _ = so.attend(q, k, v, 0.5)
    w = np.exp(q @ k.T * 0.5)
    assert np.allclose(out, w / w.sum(1, keepdims=True) @ v, atol=1e-14) and np.allclose(lse, np.log(w.sum(1)), atol=1e-14)


# ---- sizes ----------------------------------------------------------------------------------------


def test_sizes():
    from paper_2504_18154_amd import binding as b
    assert b.summary_bytes(b.make_layout(40, 8, 128, 1000, "bf16")) == 1000 * 8 * 257
    assert b.summary_bytes(b.make_layout(4, 2, 72, 10, "bf16")) == (10 * 2 * (2 * 96 + 1) + 15) // 16 * 16
    assert b.summary_bytes(b.make_layout(5, 2, 64, 16, "f32")) == 0
    lay = b.make_layout(40, 8, 128, 1000, "bf16")
    coded = 8 * 8 * (256 + 4)            # per token: its heads, eight places per K/V head, as whole numbers with a scale
    assert b.select_workspace_bytes(lay, 1, 20000) == 8 * 1264 * 4 + coded      # 1250 blocks, in whole tiles of 16
    assert b.select_workspace_bytes(lay, 0, 20000) == 0
    assert b.select_workspace_bytes(lay, 100000, 131072) == 768 * (262144 + coded)     # 192 MiB of scores
    assert b.select_workspace_bytes(lay, 3, (1 << 31) - 1) == 8 * (1 << 27) * 4 + coded   # (one token at a time, however long)


def test_rotations_that_cannot_be():
    from paper_2504_18154_amd import binding as b
    f = torch.ones(32, dtype=torch.float64)
    with pytest.raises(ValueError):
        b.Rope(f.float())
    with pytest.raises(ValueError):
        b.Rope(f, axis=[0] * 31)
    with pytest.raises(ValueError):
        b.Rope(f, axis=[4] * 32)
    with pytest.raises(ValueError):
        b.Rope(torch.ones(129, dtype=torch.float64))
    with pytest.raises(KeyError):
        b.Rope(f, pairing="thirds")
    r = b.Rope(f, axis=[0] * 16 + [2] * 16)
    assert (r.struct.rotary_dim, r.struct.pairing, r.struct.num_axes, list(r.struct.axis)[15:17]) == (64, b.ROPE_HALVES, 3, [0, 2])


# ---- refusals -------------------------------------------------------------------------------------

# every launch goes through hipLaunchKernel: none may happen
REFUSALS = r"""
extern "C" hipError_t hipLaunchKernel(const void*, dim3, dim3, void**, size_t, hipStream_t) { std::printf("launched\n"); std::fflush(stdout); std::_Exit(9); }
alignas(16) static char mem[4096];
static int bad = 0;
#define EXPECT(call, want) do { const int st = (call); if (st != (want)) std::printf("line %d: %d, not %d: %s\n", __LINE__, st, (int)(want), #call), ++bad; } while (0)
int main() {
  room = (size_t)1 << 30;
  ecoserve_layout lay = {};
  lay.num_q_heads = 8, lay.num_kv_heads = 2, lay.head_dim = 64, lay.block_size = 16, lay.num_blocks = 64, lay.dtype = ECOSERVE_BF16;
  ecoserve_ctx* c = nullptr;
  if (ecoserve_create(&c, 0, &lay, 4, 32)) return std::printf("not created\n"), 1;
  const int EI = ECOSERVE_EINVAL;
  int32_t* const i = (int32_t*)mem;
  double* const f = (double*)mem;
  void* const p = mem;
  void* const odd = mem + 4;
  ecoserve_rope r = {};
  r.rotary_dim = 64, r.num_axes = 1;
  // (ctx, rope, freq, positions, q, stride, q_out, stride, k, v, kn, vn, stride, cu, before, table, width, B, T, most)
#define ROPE(...) ecoserve_kv_append_rope(__VA_ARGS__, nullptr)
  EXPECT(ROPE(c, &r, f, nullptr, p, 512, p, 512, p, p, p, p, 128, i, i, i, 8, 0, 9, 9), ECOSERVE_OK);
  EXPECT(ROPE(c, &r, f, nullptr, p, 512, p, 512, p, p, p, p, 128, i, i, i, 8, 2, 0, 0), ECOSERVE_OK);
  EXPECT(ROPE(nullptr, &r, f, nullptr, p, 512, p, 512, p, p, p, p, 128, i, i, i, 8, 2, 9, 9), EI);
  EXPECT(ROPE(c, nullptr, f, nullptr, p, 512, p, 512, p, p, p, p, 128, i, i, i, 8, 2, 9, 9), EI);
  EXPECT(ROPE(c, &r, nullptr, nullptr, p, 512, p, 512, p, p, p, p, 128, i, i, i, 8, 2, 9, 9), EI);
  EXPECT(ROPE(c, &r, f, nullptr, p, 512, nullptr, 512, p, p, p, p, 128, i, i, i, 8, 2, 9, 9), EI);
  EXPECT(ROPE(c, &r, f, nullptr, nullptr, 512, p, 512, p, p, p, p, 128, i, i, i, 8, 2, 9, 9), EI);
  EXPECT(ROPE(c, &r, f, nullptr, p, 504, p, 512, p, p, p, p, 128, i, i, i, 8, 2, 9, 9), EI);
  EXPECT(ROPE(c, &r, f, nullptr, p, 512, p, 516, p, p, p, p, 128, i, i, i, 8, 2, 9, 9), EI);
  EXPECT(ROPE(c, &r, f, nullptr, p, 512, p, 512, p, p, p, p, 120, i, i, i, 8, 2, 9, 9), EI);
  EXPECT(ROPE(c, &r, f, nullptr, odd, 512, p, 512, p, p, p, p, 128, i, i, i, 8, 2, 9, 9), EI);
  EXPECT(ROPE(c, &r, f, nullptr, p, 512, odd, 512, p, p, p, p, 128, i, i, i, 8, 2, 9, 9), EI);
  EXPECT(ROPE(c, &r, f, nullptr, p, 512, p, 512, odd, p, p, p, 128, i, i, i, 8, 2, 9, 9), EI);
  EXPECT(ROPE(c, &r, f, nullptr, p, 512, p, 512, p, p, p, odd, 128, i, i, i, 8, 2, 9, 9), EI);
  EXPECT(ROPE(c, &r, (double*)odd, nullptr, p, 512, p, 512, p, p, p, p, 128, i, i, i, 8, 2, 9, 9), EI);
  EXPECT(ROPE(c, &r, f, (int32_t*)(mem + 2), p, 512, p, 512, p, p, p, p, 128, i, i, i, 8, 2, 9, 9), EI);
  EXPECT(ROPE(c, &r, f, nullptr, p, 512, p, 512, p, p, p, p, 128, i, i, i, 8, 5, 9, 9), EI);    // more than max_batch
  EXPECT(ROPE(c, &r, f, nullptr, p, 512, p, 512, p, p, p, p, 128, i, i, i, 8, 2, 9, 0), EI);
  EXPECT(ROPE(c, &r, f, nullptr, p, 512, p, 512, p, p, p, p, 128, i, i, i, 8, 2, 9, 10), EI);
  EXPECT(ROPE(c, &r, f, nullptr, p, 512, p, 512, p, p, p, p, 128, i, i, i, 0, 2, 9, 9), EI);
  EXPECT(ROPE(c, &r, f, nullptr, p, 512, p, 512, p, p, p, p, 128, nullptr, i, i, 8, 2, 9, 9), EI);
  EXPECT(ROPE(c, &r, f, nullptr, p, 512, p, 512, p, p, p, p, 128, i, i, i, 8, -1, 9, 9), EI);
  for (int dim : {0, -8, 4, 12, 72}) {
    ecoserve_rope x = r;
    x.rotary_dim = dim;
    EXPECT(ROPE(c, &x, f, nullptr, p, 512, p, 512, p, p, p, p, 128, i, i, i, 8, 2, 9, 9), EI);
  }
  {
    ecoserve_rope x = r;
    x.pairing = 2;
    EXPECT(ROPE(c, &x, f, nullptr, p, 512, p, 512, p, p, p, p, 128, i, i, i, 8, 2, 9, 9), EI);
    x = r, x.num_axes = 0;
    EXPECT(ROPE(c, &x, f, i, p, 512, p, 512, p, p, p, p, 128, i, i, i, 8, 2, 9, 9), EI);
    x = r, x.num_axes = 5;
    EXPECT(ROPE(c, &x, f, i, p, 512, p, 512, p, p, p, p, 128, i, i, i, 8, 2, 9, 9), EI);
    x = r, x.num_axes = 2;  // several coordinates have to be given
    EXPECT(ROPE(c, &x, f, nullptr, p, 512, p, 512, p, p, p, p, 128, i, i, i, 8, 2, 9, 9), EI);
    x = r, x.axis[31] = 1;  // a coordinate that there is not
    EXPECT(ROPE(c, &x, f, i, p, 512, p, 512, p, p, p, p, 128, i, i, i, 8, 2, 9, 9), EI);
  }
#define SUMMARY(...) ecoserve_kv_summary(__VA_ARGS__, nullptr)
  EXPECT(SUMMARY(c, p, p, i, i, i, 8, 0, 9, 9), ECOSERVE_OK);
  EXPECT(SUMMARY(c, p, p, i, i, i, 8, 2, 0, 0), ECOSERVE_OK);
  EXPECT(SUMMARY(nullptr, p, p, i, i, i, 8, 2, 9, 9), EI);
  EXPECT(SUMMARY(c, nullptr, p, i, i, i, 8, 2, 9, 9), EI);
  EXPECT(SUMMARY(c, p, nullptr, i, i, i, 8, 2, 9, 9), EI);
  EXPECT(SUMMARY(c, odd, p, i, i, i, 8, 2, 9, 9), EI);
  EXPECT(SUMMARY(c, p, odd, i, i, i, 8, 2, 9, 9), EI);
  EXPECT(SUMMARY(c, p, p, nullptr, i, i, 8, 2, 9, 9), EI);
  EXPECT(SUMMARY(c, p, p, i, i, nullptr, 8, 2, 9, 9), EI);
  EXPECT(SUMMARY(c, p, p, i, i, i, 8, 5, 9, 9), EI);
  EXPECT(SUMMARY(c, p, p, i, i, i, 8, 2, 9, 10), EI);
  EXPECT(SUMMARY(c, p, p, i, i, i, 8, 2, 9, 0), EI);
  const size_t big = (size_t)1 << 20;
  // (ctx, q, stride, summary, cu, before, table, width, blocks, K, first, last, B, T, max_ctx, workspace, bytes)
#define SELECT(...) ecoserve_block_select(__VA_ARGS__, nullptr)
  EXPECT(SELECT(c, p, 512, p, i, i, i, 8, i, 4, 1, 1, 0, 9, 100, p, big), ECOSERVE_OK);
  EXPECT(SELECT(c, p, 512, p, i, i, i, 8, i, 4, 1, 1, 2, 0, 100, p, big), ECOSERVE_OK);
  EXPECT(SELECT(nullptr, p, 512, p, i, i, i, 8, i, 4, 1, 1, 2, 9, 100, p, big), EI);
  EXPECT(SELECT(c, nullptr, 512, p, i, i, i, 8, i, 4, 1, 1, 2, 9, 100, p, big), EI);
  EXPECT(SELECT(c, p, 500, p, i, i, i, 8, i, 4, 1, 1, 2, 9, 100, p, big), EI);
  EXPECT(SELECT(c, p, 512, nullptr, i, i, i, 8, i, 4, 1, 1, 2, 9, 100, p, big), EI);
  EXPECT(SELECT(c, p, 512, p, nullptr, i, i, 8, i, 4, 1, 1, 2, 9, 100, p, big), EI);      // one token per sequence, but 9 of 2
  EXPECT(SELECT(c, p, 512, p, i, i, i, 8, nullptr, 4, 1, 1, 2, 9, 100, p, big), EI);
  EXPECT(SELECT(c, p, 512, p, i, i, i, 8, i, 0, 0, 1, 2, 9, 100, p, big), EI);
  EXPECT(SELECT(c, p, 512, p, i, i, i, 8, i, 65537, 1, 1, 2, 9, 100, p, big), EI);
  EXPECT(SELECT(c, p, 512, p, i, i, i, 8, i, 4, 1, 0, 2, 9, 100, p, big), EI);
  EXPECT(SELECT(c, p, 512, p, i, i, i, 8, i, 4, -1, 1, 2, 9, 100, p, big), EI);
  EXPECT(SELECT(c, p, 512, p, i, i, i, 8, i, 4, 3, 2, 2, 9, 100, p, big), EI);
  EXPECT(SELECT(c, p, 512, p, i, i, i, 8, i, 4, 0x7fffffff, 0x7fffffff, 2, 9, 100, p, big), EI);
  EXPECT(SELECT(c, p, 512, p, i, i, i, 8, i, 4, 1, 1, 2, 9, 0, p, big), EI);
  EXPECT(SELECT(c, p, 512, p, i, i, i, 8, i, 4, 1, 1, 2, 9, 129, p, big), EI);             // more than the table holds
  EXPECT(SELECT(c, p, 512, p, i, i, i, 80, i, 4, 1, 1, 2, 9, 513, p, big), EI);            // more than the context's limit
  EXPECT(SELECT(c, p, 512, p, i, i, i, 8, i, 4, 1, 1, 2, 9, 100, nullptr, big), EI);
  EXPECT(SELECT(c, p, 512, p, i, i, i, 8, i, 4, 1, 1, 2, 9, 100, odd, big), EI);
  EXPECT(SELECT(c, p, 512, p, i, i, i, 8, i, 4, 1, 1, 2, 9, 100, p, ecoserve_select_workspace_bytes(&lay, 9, 100) - 1), EI);
  EXPECT(SELECT(c, p, 512, p, i, i, i, 8, i, 4, 1, 1, 5, 9, 100, p, big), EI);
  // (ctx, q, stride, k, v, cu, before, table, width, blocks, K, out, lse, B, T, workspace, bytes)
#define SPARSE(...) ecoserve_attn_sparse(__VA_ARGS__, nullptr)
  float* const w = (float*)mem;
  EXPECT(SPARSE(c, p, 512, p, p, i, i, i, 8, i, 64, p, w, 0, 9, p, big), ECOSERVE_OK);
  EXPECT(SPARSE(c, p, 512, p, p, i, i, i, 8, i, 64, p, w, 2, 0, p, big), ECOSERVE_OK);
  EXPECT(SPARSE(nullptr, p, 512, p, p, i, i, i, 8, i, 64, p, w, 2, 9, p, big), EI);
  EXPECT(SPARSE(c, p, 512, nullptr, p, i, i, i, 8, i, 64, p, w, 2, 9, p, big), EI);
  EXPECT(SPARSE(c, p, 512, p, odd, i, i, i, 8, i, 64, p, w, 2, 9, p, big), EI);
  EXPECT(SPARSE(c, p, 512, p, p, i, i, i, 8, i, 64, odd, w, 2, 9, p, big), EI);
  EXPECT(SPARSE(c, p, 512, p, p, i, i, i, 8, i, 64, p, (float*)(mem + 2), 2, 9, p, big), EI);
  EXPECT(SPARSE(c, p, 512, p, p, nullptr, i, i, 8, i, 64, p, w, 2, 9, p, big), EI);
  EXPECT(SPARSE(c, p, 512, p, p, i, i, i, 8, i, 0, p, w, 2, 9, p, big), EI);
  EXPECT(SPARSE(c, p, 512, p, p, i, i, i, 8, (int32_t*)(mem + 2), 64, p, w, 2, 9, p, big), EI);
  EXPECT(SPARSE(c, p, 512, p, p, i, i, i, 8, i, 64, p, w, 5, 9, p, big), EI);
  const size_t need = ecoserve_sparse_workspace_bytes(c, 9, 64);
  if (need == 0 || ecoserve_sparse_workspace_bytes(c, 100000, 64) != 0) std::printf("workspace: %zu\n", need), ++bad;
  EXPECT(SPARSE(c, p, 512, p, p, i, i, i, 8, i, 64, p, w, 2, 9, p, need - 1), EI);
  EXPECT(SPARSE(c, p, 512, p, p, i, i, i, 8, i, 64, p, w, 2, 9, nullptr, big), EI);
  EXPECT(SPARSE(c, p, 512, p, p, i, i, i, 8, i, 64, p, w, 2, 9, odd, big), EI);
  ecoserve_destroy(c);
  std::printf("%d\n", bad);
  return bad != 0;
}
"""


def test_what_is_refused_is_refused_before_any_launch(tmp_path):
    if not os.path.exists(build.LIB):
        pytest.skip("the library is not built")
    src, exe = tmp_path / "refusals.cpp", tmp_path / "refusals"
    src.write_text(ALLOCATOR + REFUSALS)
    rocm = os.path.dirname(os.path.dirname(os.path.realpath(build._hipcc())))
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", build.INCLUDE, "-I", os.path.join(rocm, "include"), str(src), "-o", str(exe), "-rdynamic", build.LIB,
                    f"-Wl,-rpath,{os.path.dirname(build.LIB)}:{os.path.join(rocm, 'lib')}", f"-Wl,-rpath-link,{os.path.join(rocm, 'lib')}"], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and r.stdout == "0\n", r.stdout + r.stderr[-500:]
