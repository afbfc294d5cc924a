"""Attention with formed scores and the normed append where a launch takes another way: long bounds of short batches, ragged batches of few and of many sequences,
scales at the ends of their range, rows beyond what squares hold, many tokens at a time, another stream than the current one."""
import numpy as np
import pytest
import torch

from oracle import scored_oracle as so
from tests.parity_util import dev_i32
from tests.scored_util import BF, Pools, check_rows, cu_of, packed
from tests.test_gpu_scored import FORMATS, _decode, _form, _prefill, _q, _scores

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D,Hq,Hkv", [(128, 40, 8), (128, 16, 1), (64, 32, 8), (48, 6, 2), (80, 8, 8)], ids=str)
def test_decode_whatever_the_bound_of_the_lengths(fmt, D, Hq, Hkv):
    """The bound chooses between workgroups of eight wavefronts and of four, and nothing else."""
    lens = np.array([1, 17, 64, 65, 300, 0, 1027, 2400, 2399], dtype=np.int32)
    p = Pools(fmt, D, Hq, Hkv, np.append(lens, 9000), seed=D + Hq)
    p.fill(lens, 51)
    q = _q(len(lens), p, 52, 1.5)
    held = p.held()
    for kind in ("plain", "both"):
        cap, slopes = _form(p, kind)
        scores = _scores(p, cap, slopes)
        for most in (2400, 9000):
            out, lse = torch.full_like(q, float("nan")), torch.full(q.shape[:2], float("nan"), device="cuda")
            p.ctx.attn_decode_scored(q, p.cache, p.dev_table[:len(lens)], dev_i32(lens), out, most, lse=lse, scores=scores)
            check_rows(p, q, out, lse, np.arange(len(lens)), lens - 1, np.zeros(len(lens)), lens, cap, slopes, held=held, label=f"bound {most}, {kind}:")
    p.ctx.close()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("B", [1, 2, 3, 7, 63, 64, 65, 130])
def test_ragged_prompts_in_any_number(fmt, B):
    """Every tile of every sequence, in whatever order they are taken: lengths of none, one and many, prefixes, places of the padding in front."""
    rng = np.random.default_rng(B)
    new = np.where(rng.random(B) < 0.15, 0, np.exp(rng.uniform(0, np.log(170 if B < 60 else 60), size=B)).astype(int))
    new[B // 2] = 200 if B < 60 else 90
    before = np.where(rng.random(B) < 0.5, 0, rng.integers(0, 300, size=B))
    if B > 2:
        before[0], new[0] = -9, 30          # nine of the padding in front
        before[1], new[1] = -40, 25         # nothing else than that
    p = Pools(fmt, 64, 6, 2, np.maximum(before + new, 0), seed=B + 1)
    p.fill(np.maximum(before + new, 0), 53)
    seq, pos = packed(before, new)
    q = _q(len(seq), p, 54)
    cap, slopes = _form(p, "slopes")
    out, lse = _prefill(p, before, new, q, _scores(p, cap, slopes))
    assert not out.isnan().any()
    check_rows(p, q, out, lse, seq, pos, np.zeros(len(seq)), np.maximum(pos + 1, 0), cap, slopes, tokens=range(0, len(seq), 1 if B < 60 else 5))
    p.ctx.close()


def test_one_long_prompt_among_short_ones():
    """Lengths in classes of more than a step, tiles of one class in several sequences."""
    before, new = np.array([0, 5000, 0, 0, 2500]), np.array([3, 40, 1100, 1, 17])
    p = Pools("e4m3", 128, 8, 1, before + new, seed=55)
    p.fill(before + new, 56)
    seq, pos = packed(before, new)
    q = _q(len(seq), p, 57, 2.0)
    out, lse = _prefill(p, before, new, q)
    assert not out.isnan().any()
    check_rows(p, q, out, lse, seq, pos, np.zeros(len(seq)), pos + 1, tokens=list(range(0, 60)) + list(range(60, len(seq), 29)))
    p.ctx.close()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("few", [False, True])
def test_scales_at_the_ends_of_their_range(fmt, few):
    """Rows of values of 2^-100 beside ordinary ones, and rows of up to 2^119; codes of zero of either sign.  Wide rows alone, tiny rows alone, and both in a tile."""
    n = 200
    p = Pools(fmt, 64, 4, 2, [n, n, n], seed=58)
    p.fill([n, n, n], 59)
    (k, v), s = p.logical(), p.scales().copy()
    rng = np.random.default_rng(60)
    zero = torch.tensor([0, 0x80 if fmt == "e4m3" else 0], dtype=torch.uint8)
    one = 0x38 if fmt == "e4m3" else 1                      # the code of 1
    for b, bytes_ in enumerate(([127 - 100, 60, 66, 67, 68], [127 + 119, 127, 127 + 60], [127 - 100, 1, 127, 0])):
        for j in range(n):
            blk, slot = p.table[b, j // 16], j % 16
            row = v[blk, :, slot]
            row[:, ::7] = zero[rng.integers(0, 2, size=row[:, ::7].shape)]
            if j % 3 == 0:
                s[blk, :, 1, slot] = bytes_[j // 3 % len(bytes_)]
            if s[blk, 0, 1, slot] > 200:
                row[:] = one                                # (sums of these stay inside fp32)
    p.put(k, v, s[:, :, 0], s[:, :, 1])
    before = np.array([n - 3] * 3) if few else np.array([n - 70] * 3)
    new = n - before
    seq, pos = packed(before, new)
    q = _q(len(seq), p, 61)
    out, lse = _prefill(p, before, new, q)
    assert out.isfinite().all()
    check_rows(p, q, out, lse, seq, pos, np.zeros(len(seq)), pos + 1)
    last = np.cumsum(new) - 1
    out, lse = _decode(p, np.full(3, n), q[torch.from_numpy(last).cuda()].contiguous())
    check_rows(p, q[torch.from_numpy(last).cuda()], out, lse, np.arange(3), np.full(3, n - 1), np.zeros(3), np.full(3, n))
    p.ctx.close()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("step", [False, True])
def test_norm_of_rows_beyond_what_squares_hold(fmt, step):
    """Squares that fp32 does not hold make a row 0, whatever its weights and angles; 2^59 is still normed."""
    new = np.array([1, 1, 1]) if step else np.array([1, 1, 20])
    before = np.array([3, 40, 7])
    p = Pools(fmt, 64, 2, 2, before + new, seed=62)
    b = p.binding
    T = int(new.sum())
    rows = torch.randn(T, 2, 64, generator=torch.Generator().manual_seed(63)).to(BF)
    rows[0] = 3.0e38
    rows[0, :, ::2] = -3.0e38
    rows[1] = rows[1] * 2.0 ** 59 / rows[1].abs().amax()
    rows = rows.cuda()
    w = torch.full((64,), 8.0, device="cuda")
    freq = torch.from_numpy(10000.0 ** (-np.arange(32) / 32.0)).cuda()
    q_out = torch.full((T, 2, 64), 55.0, dtype=BF, device="cuda")
    p.ctx.kv_append_norm(p.cache, rows, rows.clamp(-1e30, 1e30), cu_of(new), dev_i32(before), p.dev_table, norm=b.HeadNorm(1e-6, w, w), rope=b.Rope(freq), q=rows, q_out=q_out,
                         max_new_len=1 if step else None)
    held = p.held()[0]
    assert (q_out[0] == 0).all() and (held[p.table[0, 0], :, 3] == 0).all()
    got = q_out[1].double().cpu().numpy()
    x = rows[1].double().cpu().numpy()
    assert np.allclose((got ** 2).sum(-1), 64 * 64 * (x ** 2).sum(-1) / ((x ** 2).sum(-1)), rtol=2.0 ** -7)
    assert q_out.isfinite().all() and np.isfinite(held[p.table[1, 40 // 16], :, 40 % 16]).all()
    p.ctx.close()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D,Hq,Hkv,adjacent", [(64, 14, 2, False), (16, 28, 4, True), (256, 16, 1, False)], ids=str)
def test_append_of_many_tokens_is_that_of_few(fmt, D, Hq, Hkv, adjacent):
    """Tens of thousands of tokens in one call take two heads at a time: the bits are those of calls of a few hundred."""
    T, per = 33000, 330
    p, one = Pools(fmt, D, Hq, Hkv, [T], seed=64), Pools(fmt, D, Hq, Hkv, [T], seed=64)
    b = p.binding
    g = torch.Generator(device="cuda").manual_seed(65)
    q, k, v = (torch.randn(T, h, D, generator=g, device="cuda").to(BF) for h in (Hq, Hkv, Hkv))
    w = torch.rand(D, generator=g, device="cuda") + 0.5
    freq = torch.from_numpy(10000.0 ** (-np.arange(D // 2) * 2.0 / D)).cuda()
    kw = dict(norm=b.HeadNorm(1e-6, w, w.flip(0).contiguous()), rope=b.Rope(freq, pairing="adjacent" if adjacent else "halves"))
    qa, qb = torch.empty_like(q), torch.empty_like(q)
    p.ctx.kv_append_norm(p.cache, k, v, cu_of([T]), dev_i32([0]), p.dev_table, q=q, q_out=qa, **kw)
    for t in range(0, T, per):
        at = slice(t, t + per)
        one.ctx.kv_append_norm(one.cache, k[at], v[at], cu_of([per]), dev_i32([t]), one.dev_table, q=q[at], q_out=qb[at], **kw)
    assert torch.equal(qa, qb)
    same = torch.int16 if fmt == "bf16" else torch.uint8
    assert torch.equal(p.cache.k.view(same), one.cache.k.view(same)) and torch.equal(p.cache.v.view(same), one.cache.v.view(same))
    if fmt != "bf16":
        assert torch.equal(p.cache.scales, one.cache.scales)
    p.ctx.close()
    one.ctx.close()


def test_another_stream_than_the_current_one():
    """Append, prompt and step on a stream of their own, ordered by it alone."""
    before, new = np.array([0, 0]), np.array([90, 33])
    p = Pools("int8", 128, 8, 2, before + new, seed=66)
    seq, pos = packed(before, new)
    side = torch.cuda.Stream()
    rows = torch.randn(len(seq), 12, 128, generator=torch.Generator().manual_seed(67)).to(BF).cuda()
    out, lse = torch.empty(len(seq), 8, 128, dtype=BF, device="cuda"), torch.empty(len(seq), 8, device="cuda")
    cu, at = cu_of(new), dev_i32(before)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        q, k, v = rows[:, :8], rows[:, 8:10], rows[:, 10:]
        p.ctx.kv_append_norm(p.cache, k, v, cu, at, p.dev_table)
        p.ctx.attn_prefill_scored(q, p.cache, cu, at, p.dev_table, out, lse=lse)
    side.synchronize()
    check_rows(p, q, out, lse, seq, pos, np.zeros(len(seq)), pos + 1)
    p.ctx.close()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D,Hq,Hkv", [(128, 64, 8), (96, 16, 16), (128, 20, 10)], ids=str)
def test_prompts_of_many_rows(fmt, D, Hq, Hkv):
    """Enough rows for the large tiles: tokens of every place in one, at both ends of both prompts; plain, capped in a window, biased."""
    G = Hq // Hkv
    new = np.array([256 * 512 // Hq + 33, 1100 // G + 5 * 256 // G])
    before = np.array([0, 77])
    p = Pools(fmt, D, Hq, Hkv, before + new, seed=70)
    p.fill(before + new, 71)
    held = p.held()
    seq, pos = packed(before, new)
    T = len(seq)
    assert T * G >= 4 * 256 * 2 and (T * G // 256 + 2) * Hkv >= 512
    q = _q(T, p, 72, 1.5)
    some = sorted({0, 1, 31, 63, 64, 127, 128, int(new[0]) - 1, int(new[0]), int(new[0]) + 33, T - 1} | set(range(7, T, max(1, T // 25))))
    for kind, begin in (("plain", None), ("cap", np.maximum(pos - 150, 0)), ("slopes", None)):
        cap, slopes = _form(p, kind)
        out, lse = _prefill(p, before, new, q, _scores(p, cap, slopes, begin))
        assert not out.isnan().any()
        check_rows(p, q, out, lse, seq, pos, np.zeros(T) if begin is None else begin, pos + 1, cap, slopes, tokens=some, held=held, label=kind)
    p.ctx.close()


def test_a_value_that_all_rows_see_and_is_not_finite():
    """An infinity at the first position of one prompt, a NaN behind every row of the other's first tiles: the first is in every row's result, and no row is at a loss for it."""
    before, new = np.array([0, 0]), np.array([700, 700])
    p = Pools("bf16", 128, 4, 2, before + new, seed=73)
    p.fill(before + new, 74)
    k, v = p.logical()
    v[p.table[0, 0], 0, 0, 9] = float("inf")
    v[p.table[1, 650 // 16], 1, 650 % 16, 100] = float("nan")
    p.put(k, v)
    seq, pos = packed(before, new)
    q = _q(len(seq), p, 75)
    out, lse = _prefill(p, before, new, q)
    check_rows(p, q, out, lse, seq, pos, np.zeros(len(seq)), pos + 1, tokens=range(0, len(seq), 9))
    o = out.cpu()
    assert (~o[:700, :2, 9].isfinite()).all() and o[:700, :2, :9].isfinite().all() and o[:700, 2:].isfinite().all() and lse.isfinite().all()
    assert o[700:700 + 650].isfinite().all() and o[700 + 650:, 2:, 100].isnan().all()
    p.ctx.close()
