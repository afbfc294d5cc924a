"""Norms and codes on the way into the cache, reading back, and attention with formed scores, without a GPU: the oracle's definitions against one another and against
torch's types, sizes of buffers and workspaces, and what the entry points refuse before they launch anything."""
import os
import subprocess

import numpy as np
import pytest
import torch

from oracle import scored_oracle as so
from paper_2504_18154_amd import build
from tests.test_workspace import ALLOCATOR


def test_e4m3_is_the_type_that_torch_has():
    bits = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    assert np.array_equal(bits.view(torch.float8_e4m3fn).double().numpy(), so.E4M3, equal_nan=True)
    rng = np.random.default_rng(1)
    x = np.concatenate([rng.normal(size=500) * 100, rng.normal(size=500), rng.normal(size=300) * 0.01, so.E4M3[:127], (so.E4M3[:126] + so.E4M3[1:127]) / 2, [448.0, -448.0, 0.0]])
    x = np.clip(x, -448, 448).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(np.array([so.to_e4m3(float(v)) for v in x]), want)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_codes_are_within_half_a_step(fmt):
    rng = np.random.default_rng(2)
    for scale in (1e-30, 1e-3, 1.0, 5000.0, 1e30):
        x = rng.normal(size=64) * scale
        c, b = so.code(x, fmt)
        y = so.value(c[None], np.array([b]), fmt)[0]
        step = 2.0 ** (b - 127)
        half = np.full(64, 0.5) if fmt == "int8" else 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(np.abs(x / step), 1e-300))), -6) - 4)
        assert (np.abs(y - x) <= half * step * (1 + 1e-12)).all()
        assert np.abs(x).max() <= so.MOST[fmt] * step and np.abs(x).max() > so.MOST[fmt] * step / 2
    assert so.code(np.array([1.0, np.inf]), fmt)[1] == so.BAD and so.code(np.array([np.nan, 1.0]), fmt)[1] == so.BAD
    assert so.code(np.zeros(4), fmt) [1] == 1
    assert so.scale_byte(so.MOST[fmt], fmt) == 127 and so.scale_byte(so.MOST[fmt] * 1.0001, fmt) == 128


def test_forms_by_hand():
    q, k, v = np.array([[2.0, 0.0]]), np.array([[1.0, 5.0], [3.0, 1.0], [0.5, 0.0]]), np.array([[1.0, 0.0], [0.0, 1.0], [2.0, 2.0]])
    s = np.array([2.0, 6.0, 1.0])
    for cap, slope in ((0.0, 0.0), (4.0, 0.0), (0.0, 0.5), (4.0, 0.5)):
        t = (4 * np.tanh(s / 4) if cap else s) + slope * (np.arange(3) - 2)
        w = np.exp(t)
        out, lse, _, _ = so.attend(q, k, v, np.arange(3), 2, 1.0, cap, np.array([slope]))
        assert np.allclose(out[0], w @ v / w.sum(), atol=1e-14) and np.isclose(lse[0], np.log(w.sum()), atol=1e-14)


def test_norm_by_hand():
    x = np.array([3.0, -4.0, 0.0, 0.0])
    assert np.allclose(so.norm(x, 0.0, None), x / 2.5) and np.allclose(so.norm(x, 0.0, np.array([1.0, 2.0, 3.0, 4.0])), [1.2, -3.2, 0, 0])
    assert np.allclose(so.norm(np.zeros(4), 1e-6, None), 0)


def test_sizes():
    from paper_2504_18154_amd import binding as b
    assert b.cache_scale_bytes(b.make_layout(40, 8, 128, 1000, "bf16")) == 1000 * 8 * 32
    assert b.cache_scale_bytes(b.make_layout(5, 2, 64, 16, "bf16")) == 0


def test_structs_that_cannot_be():
    from paper_2504_18154_amd import binding as b
    z = torch.zeros
    with pytest.raises(ValueError):
        b.PagedCache(z(32, dtype=torch.uint8), z(32, dtype=torch.uint8), format="e4m3")
    with pytest.raises(ValueError):
        b.PagedCache(z(32, dtype=torch.bfloat16), z(32, dtype=torch.bfloat16), z(32, dtype=torch.uint8), format="bf16")
    with pytest.raises(ValueError):
        b.PagedCache(z(32), z(32), z(32, dtype=torch.uint8), format="int8")
    with pytest.raises(KeyError):
        b.PagedCache(z(32), z(32), format="int4")
    with pytest.raises(ValueError):
        b.HeadNorm(1e-6, z(64, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        b.HeadNorm(1e-6, z(64), z(2, 64))
    with pytest.raises(ValueError):
        b.Scores(slopes=z(8, dtype=torch.float64))
    with pytest.raises(ValueError):
        b.Scores(key_begin=z(8, dtype=torch.int64))
    n = b.HeadNorm(1e-6, None, z(2, 64))
    assert n.struct.per_head == 1 and n.struct.q_weight is None


REFUSALS = r"""
extern "C" hipError_t hipLaunchKernel(const void*, dim3, dim3, void**, size_t, hipStream_t) { std::printf("launched\n"); std::fflush(stdout); std::_Exit(9); }
alignas(16) static char mem[4096];
static int bad = 0;
#define EXPECT(call, want) do { const int st = (call); if (st != (want)) std::printf("line %d: %d, not %d: %s\n", __LINE__, st, (int)(want), #call), ++bad; } while (0)
int main() {
  room = (size_t)1 << 30;
  ecoserve_layout lay = {};
  lay.num_q_heads = 8, lay.num_kv_heads = 2, lay.head_dim = 64, lay.block_size = 16, lay.num_blocks = 64, lay.dtype = ECOSERVE_BF16;
  ecoserve_ctx *c = nullptr, *c32 = nullptr, *c72 = nullptr;
  if (ecoserve_create(&c, 0, &lay, 4, 32)) return std::printf("not created\n"), 1;
  lay.dtype = ECOSERVE_F32;
  if (ecoserve_create(&c32, 0, &lay, 4, 32)) return std::printf("not created\n"), 1;
  lay.dtype = ECOSERVE_BF16, lay.head_dim = 72;
  if (ecoserve_create(&c72, 0, &lay, 4, 32)) return std::printf("not created\n"), 1;
  const int EI = ECOSERVE_EINVAL, EU = ECOSERVE_EUNSUPPORTED;
  int32_t* const i = (int32_t*)mem;
  double* const f = (double*)mem;
  float* const w = (float*)mem;
  void* const p = mem;
  void* const odd = mem + 4;
  const ecoserve_cache e = {ECOSERVE_CACHE_E4M3, p, p, (uint8_t*)p}, native = {ECOSERVE_CACHE_LAYOUT, p, p, nullptr};
  const ecoserve_cache wrong[] = {{3, p, p, (uint8_t*)p}, {-1, p, p, (uint8_t*)p}, {1, nullptr, p, (uint8_t*)p}, {1, p, nullptr, (uint8_t*)p}, {1, p, p, nullptr}, {2, p, p, nullptr},
                                  {1, odd, p, (uint8_t*)p}, {1, p, odd, (uint8_t*)p}, {2, p, p, (uint8_t*)odd}, {0, p, odd, nullptr}};
  ecoserve_rope r = {};
  r.rotary_dim = 64, r.num_axes = 1;
  ecoserve_norm m = {1e-6f, 0, w, w};
  // (ctx, cache, norm, rope, freq, positions, q, stride, q_out, stride, kn, vn, stride, cu, before, table, width, B, T, most)
#define NORM(...) ecoserve_kv_append_norm(__VA_ARGS__, nullptr)
  EXPECT(NORM(c, &e, &m, &r, f, nullptr, p, 512, p, 512, p, p, 128, i, i, i, 8, 0, 9, 9), ECOSERVE_OK);
  EXPECT(NORM(c, &native, nullptr, nullptr, nullptr, nullptr, nullptr, 0, nullptr, 0, p, p, 128, i, i, i, 8, 2, 0, 0), ECOSERVE_OK);
  EXPECT(NORM(nullptr, &e, &m, &r, f, nullptr, p, 512, p, 512, p, p, 128, i, i, i, 8, 2, 9, 9), EI);
  EXPECT(NORM(c, nullptr, &m, &r, f, nullptr, p, 512, p, 512, p, p, 128, i, i, i, 8, 2, 9, 9), EI);
  for (const auto& x : wrong) EXPECT(NORM(c, &x, &m, &r, f, nullptr, p, 512, p, 512, p, p, 128, i, i, i, 8, 2, 9, 9), EI);
  EXPECT(NORM(c32, &e, &m, &r, f, nullptr, p, 512, p, 512, p, p, 128, i, i, i, 8, 2, 9, 9), EU);
  EXPECT(NORM(c72, &e, &m, &r, f, nullptr, p, 576, p, 576, p, p, 144, i, i, i, 8, 2, 9, 9), EU);
  EXPECT(NORM(c, &e, &m, &r, nullptr, nullptr, p, 512, p, 512, p, p, 128, i, i, i, 8, 2, 9, 9), EI);
  EXPECT(NORM(c, &e, &m, &r, (double*)odd, nullptr, p, 512, p, 512, p, p, 128, i, i, i, 8, 2, 9, 9), EI);
  EXPECT(NORM(c, &e, &m, &r, f, (int32_t*)(mem + 2), p, 512, p, 512, p, p, 128, i, i, i, 8, 2, 9, 9), EI);
  EXPECT(NORM(c, &e, &m, &r, f, nullptr, p, 512, nullptr, 512, p, p, 128, i, i, i, 8, 2, 9, 9), EI);
  EXPECT(NORM(c, &e, &m, &r, f, nullptr, nullptr, 512, p, 512, p, p, 128, i, i, i, 8, 2, 9, 9), EI);
  EXPECT(NORM(c, &e, &m, &r, f, nullptr, p, 504, p, 512, p, p, 128, i, i, i, 8, 2, 9, 9), EI);
  EXPECT(NORM(c, &e, &m, &r, f, nullptr, p, 512, p, 516, p, p, 128, i, i, i, 8, 2, 9, 9), EI);
  EXPECT(NORM(c, &e, &m, &r, f, nullptr, p, 512, p, 512, p, p, 120, i, i, i, 8, 2, 9, 9), EI);
  EXPECT(NORM(c, &e, &m, &r, f, nullptr, p, 512, p, 512, nullptr, p, 128, i, i, i, 8, 2, 9, 9), EI);
  EXPECT(NORM(c, &e, &m, &r, f, nullptr, p, 512, p, 512, p, odd, 128, i, i, i, 8, 2, 9, 9), EI);
  EXPECT(NORM(c, &e, &m, &r, f, nullptr, odd, 512, p, 512, p, p, 128, i, i, i, 8, 2, 9, 9), EI);
  EXPECT(NORM(c, &e, &m, &r, f, nullptr, p, 512, p, 512, p, p, 128, i, i, i, 8, 5, 9, 9), EI);
  EXPECT(NORM(c, &e, &m, &r, f, nullptr, p, 512, p, 512, p, p, 128, i, i, i, 8, 2, 9, 0), EI);
  EXPECT(NORM(c, &e, &m, &r, f, nullptr, p, 512, p, 512, p, p, 128, i, i, i, 8, 2, 9, 10), EI);
  EXPECT(NORM(c, &e, &m, &r, f, nullptr, p, 512, p, 512, p, p, 128, nullptr, i, i, 8, 2, 9, 9), EI);
  EXPECT(NORM(c, &e, &m, &r, f, nullptr, p, 512, p, 512, p, p, 128, i, i, i, 0, 2, 9, 9), EI);
  EXPECT(NORM(c, &e, &m, &r, f, nullptr, p, 512, p, 512, p, p, 128, i, i, i, 8, -1, 9, 9), EI);
  for (const auto& x : {ecoserve_norm{-1.f, 0, w, w}, ecoserve_norm{__builtin_nanf(""), 0, w, w}, ecoserve_norm{__builtin_inff(), 0, w, w}, ecoserve_norm{0.f, 2, w, w},
                        ecoserve_norm{0.f, 0, (float*)odd, w}, ecoserve_norm{0.f, 0, w, (float*)odd}})
    EXPECT(NORM(c, &e, &x, &r, f, nullptr, p, 512, p, 512, p, p, 128, i, i, i, 8, 2, 9, 9), EI);
  {
    ecoserve_rope x = r;
    x.rotary_dim = 72;
    EXPECT(NORM(c, &e, &m, &x, f, nullptr, p, 512, p, 512, p, p, 128, i, i, i, 8, 2, 9, 9), EI);
    x = r, x.num_axes = 2;
    EXPECT(NORM(c, &e, &m, &x, f, nullptr, p, 512, p, 512, p, p, 128, i, i, i, 8, 2, 9, 9), EI);
  }
  // (ctx, cache, k, v, stride, cu, first, table, width, B, T)
#define READ(...) ecoserve_kv_read(__VA_ARGS__, nullptr)
  EXPECT(READ(c, &e, p, p, 128, i, i, i, 8, 0, 9), ECOSERVE_OK);
  EXPECT(READ(c, &e, p, p, 128, i, i, i, 8, 2, 0), ECOSERVE_OK);
  EXPECT(READ(nullptr, &e, p, p, 128, i, i, i, 8, 2, 9), EI);
  EXPECT(READ(c, nullptr, p, p, 128, i, i, i, 8, 2, 9), EI);
  for (const auto& x : wrong) EXPECT(READ(c, &x, p, p, 128, i, i, i, 8, 2, 9), EI);
  EXPECT(READ(c32, &e, p, p, 128, i, i, i, 8, 2, 9), EU);
  EXPECT(READ(c72, &native, p, p, 144, i, i, i, 8, 2, 9), EU);
  EXPECT(READ(c, &e, nullptr, nullptr, 128, i, i, i, 8, 2, 9), EI);
  EXPECT(READ(c, &e, odd, p, 128, i, i, i, 8, 2, 9), EI);
  EXPECT(READ(c, &e, p, p, 124, i, i, i, 8, 2, 9), EI);
  EXPECT(READ(c, &e, p, p, 132, i, i, i, 8, 2, 9), EI);
  EXPECT(READ(c, &e, p, p, 128, nullptr, i, i, 8, 2, 9), EI);
  EXPECT(READ(c, &e, p, p, 128, i, nullptr, i, 8, 2, 9), EI);
  EXPECT(READ(c, &e, p, p, 128, i, i, i, 0, 2, 9), EI);
  EXPECT(READ(c, &e, p, p, 128, i, i, i, 8, 5, 9), EI);
  const ecoserve_scores none = {0.f, nullptr, nullptr, nullptr};
  const ecoserve_scores no_form[] = {{-1.f, nullptr, nullptr, nullptr}, {__builtin_nanf(""), nullptr, nullptr, nullptr}, {__builtin_inff(), nullptr, nullptr, nullptr},
                                     {0.f, (float*)(mem + 2), nullptr, nullptr}, {0.f, nullptr, (int32_t*)(mem + 2), nullptr}, {0.f, nullptr, nullptr, (int32_t*)(mem + 1)}};
  const size_t big = (size_t)1 << 30;
  // (ctx, cache, scores, q, stride, cu, before, table, width, out, lse, B, T, workspace, bytes)
#define PREFILL(...) ecoserve_attn_prefill_scored(__VA_ARGS__, nullptr)
  EXPECT(PREFILL(c, &e, &none, p, 512, i, i, i, 8, p, w, 0, 9, p, big), ECOSERVE_OK);
  EXPECT(PREFILL(c, &e, nullptr, p, 512, i, i, i, 8, p, w, 2, 0, p, big), ECOSERVE_OK);
  EXPECT(PREFILL(nullptr, &e, &none, p, 512, i, i, i, 8, p, w, 2, 9, p, big), EI);
  EXPECT(PREFILL(c, nullptr, &none, p, 512, i, i, i, 8, p, w, 2, 9, p, big), EI);
  for (const auto& x : wrong) EXPECT(PREFILL(c, &x, &none, p, 512, i, i, i, 8, p, w, 2, 9, p, big), EI);
  for (const auto& x : no_form) EXPECT(PREFILL(c, &e, &x, p, 512, i, i, i, 8, p, w, 2, 9, p, big), EI);
  EXPECT(PREFILL(c32, &e, &none, p, 512, i, i, i, 8, p, w, 2, 9, p, big), EU);
  EXPECT(PREFILL(c72, &native, &none, p, 576, i, i, i, 8, p, w, 2, 9, p, big), EU);
  EXPECT(PREFILL(c, &e, &none, nullptr, 512, i, i, i, 8, p, w, 2, 9, p, big), EI);
  EXPECT(PREFILL(c, &e, &none, odd, 512, i, i, i, 8, p, w, 2, 9, p, big), EI);
  EXPECT(PREFILL(c, &e, &none, p, 508, i, i, i, 8, p, w, 2, 9, p, big), EI);
  EXPECT(PREFILL(c, &e, &none, p, 512, nullptr, i, i, 8, p, w, 2, 9, p, big), EI);
  EXPECT(PREFILL(c, &e, &none, p, 512, i, nullptr, i, 8, p, w, 2, 9, p, big), EI);
  EXPECT(PREFILL(c, &e, &none, p, 512, i, i, nullptr, 8, p, w, 2, 9, p, big), EI);
  EXPECT(PREFILL(c, &e, &none, p, 512, i, i, i, 0, p, w, 2, 9, p, big), EI);
  EXPECT(PREFILL(c, &e, &none, p, 512, i, i, i, 8, odd, w, 2, 9, p, big), EI);
  EXPECT(PREFILL(c, &e, &none, p, 512, i, i, i, 8, p, (float*)(mem + 2), 2, 9, p, big), EI);
  EXPECT(PREFILL(c, &e, &none, p, 512, i, i, i, 8, p, w, 5, 9, p, big), EI);
  EXPECT(PREFILL(c, &e, &none, p, 512, i, i, i, 8, p, w, 2, 0x7fffffff, p, big), EI);   // more rows than 32 bits count
  const size_t need = ecoserve_prefill_scored_workspace_bytes(c, 2, 9);
  if (need == 0 || ecoserve_prefill_scored_workspace_bytes(c, 2, 1000000) != 0 || ecoserve_prefill_scored_workspace_bytes(nullptr, 2, 9) != 0) std::printf("workspace: %zu\n", need), ++bad;
  EXPECT(PREFILL(c, &e, &none, p, 512, i, i, i, 8, p, w, 2, 9, p, need - 1), EI);
  EXPECT(PREFILL(c, &e, &none, p, 512, i, i, i, 8, p, w, 2, 9, nullptr, big), EI);
  EXPECT(PREFILL(c, &e, &none, p, 512, i, i, i, 8, p, w, 2, 9, odd, big), EI);
  // (ctx, cache, scores, q, stride, table, width, len, out, lse, B, max_ctx, workspace, bytes)
#define DECODE(...) ecoserve_attn_decode_scored(__VA_ARGS__, nullptr)
  EXPECT(DECODE(c, &e, &none, p, 512, i, 8, i, p, w, 0, 100, p, big), ECOSERVE_OK);
  EXPECT(DECODE(nullptr, &e, &none, p, 512, i, 8, i, p, w, 2, 100, p, big), EI);
  EXPECT(DECODE(c, nullptr, &none, p, 512, i, 8, i, p, w, 2, 100, p, big), EI);
  for (const auto& x : wrong) EXPECT(DECODE(c, &x, &none, p, 512, i, 8, i, p, w, 2, 100, p, big), EI);
  for (const auto& x : no_form) EXPECT(DECODE(c, &e, &x, p, 512, i, 8, i, p, w, 2, 100, p, big), EI);
  EXPECT(DECODE(c32, &e, &none, p, 512, i, 8, i, p, w, 2, 100, p, big), EU);
  EXPECT(DECODE(c, &e, &none, nullptr, 512, i, 8, i, p, w, 2, 100, p, big), EI);
  EXPECT(DECODE(c, &e, &none, p, 500, i, 8, i, p, w, 2, 100, p, big), EI);
  EXPECT(DECODE(c, &e, &none, p, 512, nullptr, 8, i, p, w, 2, 100, p, big), EI);
  EXPECT(DECODE(c, &e, &none, p, 512, i, 8, nullptr, p, w, 2, 100, p, big), EI);
  EXPECT(DECODE(c, &e, &none, p, 512, i, 8, i, odd, w, 2, 100, p, big), EI);
  EXPECT(DECODE(c, &e, &none, p, 512, i, 8, i, p, w, 5, 100, p, big), EI);
  EXPECT(DECODE(c, &e, &none, p, 512, i, 8, i, p, w, 2, 0, p, big), EI);
  EXPECT(DECODE(c, &e, &none, p, 512, i, 8, i, p, w, 2, 129, p, big), EI);
  EXPECT(DECODE(c, &e, &none, p, 512, i, 80, i, p, w, 2, 513, p, big), EI);
  EXPECT(DECODE(c, &e, &none, p, 512, i, 8, i, p, w, 2, 100, p, ecoserve_decode_scored_workspace_bytes(c) - 1), EI);
  EXPECT(DECODE(c, &e, &none, p, 512, i, 8, i, p, w, 2, 100, nullptr, big), EI);
  EXPECT(DECODE(c, &e, &none, p, 512, i, 8, i, p, w, 2, 100, odd, big), EI);
  if (ecoserve_decode_scored_workspace_bytes(nullptr) != 0) ++bad;
  ecoserve_destroy(c), ecoserve_destroy(c32), ecoserve_destroy(c72);
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
