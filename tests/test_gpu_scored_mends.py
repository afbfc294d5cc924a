"""Attention with formed scores where it answered wrongly once: batches of fewer tokens than sequences, ranges that leave keys between them, caps far above the scores, keys that are
not finite in a step, values near the top of fp32's range, weights of fewer bits than those of
the calls without forms."""
import numpy as np
import pytest
import torch

from oracle import scored_oracle as so
from tests.parity_util import dev_i32
from tests.scored_util import HALF, Pools, check_rows, packed
from tests.test_gpu_scored import FORMATS, _decode, _prefill, _q, _scores

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("ranges", [False, True])
@pytest.mark.parametrize("new", [[0, 1], [0, 0, 5, 0, 0, 0, 1], [0] * 60 + [1] + [0] * 10 + [4], [0] * 90 + [70]], ids=["2", "7", "72", "91"])
def test_fewer_tokens_than_sequences(fmt, ranges, new):
    """Sequences without new tokens in front of those that have some, which are computed all the same."""
    new = np.array(new)
    before = np.arange(len(new)) * 37 % 200
    p = Pools(fmt, 64, 8, 1, before + new, seed=90)
    p.fill(before + new, 91)
    seq, pos = packed(before, new)
    begin = np.maximum(pos - 40, 0) if ranges else np.zeros(len(seq), dtype=np.int64)
    q = _q(len(seq), p, 92)
    out, lse = _prefill(p, before, new, q, _scores(p, 0.0, None, begin, pos + 1) if ranges else None)
    assert not out.isnan().any() and not lse.isnan().any()
    check_rows(p, q, out, lse, seq, pos, begin, pos + 1)
    p.ctx.close()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D,Hq,Hkv", [(64, 4, 2), (128, 64, 8), (80, 8, 8), (256, 8, 1)], ids=str)
@pytest.mark.parametrize("kind", ["ends", "begins", "both"])
def test_keys_that_no_row_sees(fmt, D, Hq, Hkv, kind):
    """Tiles whose rows' ranges leave keys between them, whole blocks and parts of blocks: what stands there (codes that are NaN, beside scales that are not, and bf16 NaN) reaches nobody, and the
    block table names a block of nothing else in their place."""
    before, new = np.array([700, 0]), np.array([520 if Hq == 64 else 60, 40])
    total = before + new
    p = Pools(fmt, D, Hq, Hkv, total, seed=93)
    p.fill(total, 94)
    seq, pos = packed(before, new)
    rng = np.random.default_rng(95)
    begin, end = np.zeros(len(seq), dtype=np.int64), pos + 1
    if kind == "begins":     # every row its own key, or none: runs of none of more than a block
        begin = np.where(np.arange(len(seq)) // 20 % 2 == 0, pos, pos + 1)
    else:                    # one segment of the past to a row: some are neighbours, most are not
        at = rng.integers(0, 12, len(seq)) * 50
        if kind == "both":
            begin = np.where(seq == 0, at + 3, pos // 9 * 9)
        end = np.where(seq == 0, at + 3 + rng.integers(0, 30, len(seq)), pos // 9 * 9 + rng.integers(0, 5, len(seq)))
        if kind == "ends":   # (begins below 0; every range from the first key on, and one that is long)
            end = np.where(seq == 0, np.minimum(end, 40), end)
            end[10] = 600
    seen = [np.zeros(t, dtype=bool) for t in total]
    for t in range(len(seq)):
        seen[seq[t]][max(int(begin[t]), 0):max(int(min(end[t], total[seq[t]])), 0)] = True
    (k, v), s = p.logical(), p.scales()
    s = None if s is None else s.copy()
    named = {int(p.table[b, j]) for b in range(2) for j in range((total[b] + 15) // 16)}
    spare = next(i for i in range(p.blocks) if i not in named)
    bad = float("nan") if fmt == "bf16" else 0x7f
    k[spare], v[spare] = bad, bad
    if s is not None:
        s[spare] = 127
    for b in range(2):
        for j in range((total[b] + 15) // 16):
            here = seen[b][16 * j:16 * j + 16]
            blk = p.table[b, j]
            for i in np.flatnonzero(~here):
                k[blk, :, i], v[blk, :, i] = bad, bad
                if s is not None:
                    s[blk, :, :, i] = 127 if i % 2 else 254
            if not here.any():
                p.table[b, j] = spare
    p.put(k, v, *((s[:, :, 0], s[:, :, 1]) if s is not None else ()))
    p.dev_table = torch.from_numpy(p.table).cuda()
    q = _q(len(seq), p, 96)
    for form in ((0.0, None), (20.0, None)):
        out, lse = _prefill(p, before, new, q, _scores(p, *form, begin if kind != "ends" else None, end if kind != "begins" else None))
        assert out.isfinite().all()
        check_rows(p, q, out, lse, seq, pos, begin, np.minimum(end, total[seq]), *form, tokens=range(0, len(seq), 1 if len(seq) < 200 else 7))
    p.ctx.close()


CAPS = [2.0 ** -126, 1.0, 64.0, 64.5, 100.0, 1e3, 1e4, 1e6, 1e30, 3.4e38]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D,Hq,Hkv,size", [(64, 4, 2, 1.5), (128, 8, 1, 40.0), (80, 6, 6, 1.5), (256, 4, 1, 12.0)], ids=str)
@pytest.mark.parametrize("biased", [False, True])
def test_caps_of_all_sizes(fmt, D, Hq, Hkv, size, biased):
    """What is small beside a cap stays as it is; scores on both sides of half a cap; caps that fp32 cannot multiply."""
    before, new = np.array([200, 0, 9]), np.array([20, 70, 1])
    total = before + new
    p = Pools(fmt, D, Hq, Hkv, total, seed=97)
    p.fill(total, 98)
    held = p.held()
    seq, pos = packed(before, new)
    q = _q(len(seq), p, 99, size)
    q[5] = 0
    slopes = (2.0 ** (-8.0 * np.arange(1, Hq + 1) / Hq)).astype(np.float32) if biased else None
    last = np.cumsum(new) - 1
    ql = q[torch.from_numpy(last).cuda()].contiguous()
    for cap in CAPS:
        out, lse = _prefill(p, before, new, q, _scores(p, cap, slopes))
        check_rows(p, q, out, lse, seq, pos, np.zeros(len(seq)), pos + 1, cap, slopes, held=held, tokens=range(0, len(seq), 3), label=f"cap {cap:g}, prompts:")
        out, lse = _decode(p, total, ql, _scores(p, cap, slopes))
        check_rows(p, ql, out, lse, np.arange(3), total - 1, np.zeros(3), total, cap, slopes, held=held, label=f"cap {cap:g}, a step:")
    p.ctx.close()


def test_a_small_cap_of_large_scales():
    """Twice the scale by the cap is beyond fp32: scores of zero stay zero, others saturate."""
    total = np.array([50])
    p = Pools("bf16", 64, 4, 2, total, seed=100, scale=1000.0)
    p.fill(total, 101)
    q = _q(50, p, 102)
    q[::3] = 0
    for cap in (2.0 ** -126, 2.0 ** -120, 5.0):
        out, lse = _prefill(p, np.array([0]), total, q, _scores(p, cap, None))
        check_rows(p, q, out, lse, np.zeros(50, dtype=int), np.arange(50), np.zeros(50), np.arange(50) + 1, cap)
        out, lse = _decode(p, total, q[48:49], _scores(p, cap, None))
        check_rows(p, q[48:49], out, lse, [0], [49], [0], [50], cap)
    p.ctx.close()


@pytest.mark.parametrize("D,Hq,Hkv", [(16, 4, 2), (48, 6, 2), (80, 8, 8), (112, 4, 1), (144, 2, 1), (208, 4, 4), (64, 8, 1), (128, 8, 1), (256, 4, 1)], ids=str)
def test_keys_that_are_not_finite_in_a_step(D, Hq, Hkv):
    """A key with an infinite channel scores plus or minus infinity: minus has no weight, whatever the head's size; NaN, and plus infinity, make the row NaN; and all of that where prompts have it too."""
    total = np.array([70, 70, 300, 33, 40, 20])
    p = Pools("bf16", D, Hq, Hkv, total, seed=103)
    p.fill(total, 104)
    k, v = p.logical()
    q = _q(len(total), p, 105)
    q[:, :, 3] = 1.0                                  # (the sign of the infinite products)
    inf = float("inf")

    def put(b, j, channel, x, pool=k):
        pool[p.table[b, j // 16], :, j % 16, channel] = x

    put(0, 20, 3, -inf)
    put(1, 69, 3, -inf)
    put(1, 0, 3, -inf)
    put(2, 130, 3, inf)
    put(3, 5, 3, float("nan"))
    for j in range(40):
        put(4, j, 3, -inf)                            # (all of them)
    put(5, 7, D - 1, inf, v)
    p.put(k, v)
    pos = total - 1
    for form in ((0.0, None), (20.0, None), (200.0, None)):
        out, lse = _decode(p, total, q, _scores(p, *form))
        if form[0] == 0:
            assert out[:2].isfinite().all() and out[2:5].isnan().all() and (lse[4] == -inf).all()
        check_rows(p, q, out, lse, np.arange(6), pos, np.zeros(6), total, *form, tokens=[0, 1, 3, 4, 5], label=f"a step, {form[0]}:")
        assert (out[5, :, D - 1] == inf).all() and out[5, :, :D - 1].isfinite().all()
        prompt, prompt_lse = _prefill(p, pos, np.ones(6, dtype=int), q, _scores(p, *form))
        assert torch.equal(prompt.isnan(), out.isnan())
        check_rows(p, q, prompt, prompt_lse, np.arange(6), pos, np.zeros(6), total, *form, tokens=[0, 1, 3, 4, 5], label=f"prompts, {form[0]}:")
    p.ctx.close()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D,Hq,Hkv", [(64, 8, 4), (128, 8, 4), (80, 8, 8), (256, 4, 4)], ids=str)
def test_values_near_the_top_of_the_range(fmt, D, Hq, Hkv):
    """Values of 2^126 at keys whose scores rise, by less than a factor of 2^8 of their weights, from step to step: the weighted means are inside fp32, and so are the sums.
    (So many sequences that no wavefront has a single step of one, and no prompt's steps are cut.)"""
    total = 1500 + np.arange(70)
    p = Pools(fmt, D, Hq, Hkv, total, seed=106, scale=1.0)
    (k, v), s = p.logical(), p.scales()
    k, v = torch.zeros_like(k), torch.zeros_like(v)
    one, big, up = {"bf16": (1.0, 2.0 ** 126, 0), "int8": (64, 64, 120), "e4m3": (0x38, 0x78, 118)}[fmt]   # (the code of 1 or 64, of 64 or 256, and the exponent of the large values' scale)
    if s is not None:
        s = np.full_like(s, 127)
        s[:, :, 0] = 127 - (6 if fmt == "int8" else 0)
    for b in range(len(total)):
        for j in (0, 600, total[b] - 1):              # the first key's score is 0, as all others' but the last one's, which is q[0]
            blk, at = p.table[b, j // 16], j % 16
            v[blk, :, at, ::2] = big
            if s is not None:
                s[blk, :, 1, at] = 127 + up
        k[blk, :, at, 0] = one
    p.put(k, v, *((s[:, :, 0], s[:, :, 1]) if s is not None else ()))
    q = _q(len(total), p, 108)
    q[:, :, 0] = 5.0                                  # 7.2 in the exponent
    held = p.held()
    for what, (out, lse) in (("a step:", _decode(p, total, q)), ("prompts:", _prefill(p, total - 1, np.ones(len(total), dtype=int), q))):
        assert out.isfinite().all(), what
        check_rows(p, q, out, lse, np.arange(len(total)), total - 1, np.zeros(len(total)), total, held=held, tokens=range(0, len(total), 9), label=what)
    p.ctx.close()


def _check_bits(p, q, out, seq, pos, cap, slopes, tokens, label):
    """Within weights of 16 bits (a part that is cut or rounded leaves less than 2^-7 of a weight, half a step of which is 2^-9), the result's rounding, and what fp32 leaves."""
    keys, vals = p.held()
    got, qh = out.double().cpu().numpy(), q.double().cpu().numpy()
    for t in tokens:
        for g in range(p.Hkv):
            heads, n = slice(g * p.G, g * p.G + p.G), int(pos[t]) + 1
            want, _, size, off = so.attend(qh[t, heads], p.rows(keys, seq[t], g, n), p.rows(vals, seq[t], g, n), np.arange(n), int(pos[t]), p.scale, cap, None if slopes is None else slopes[heads])
            tol = size * (2.0 ** -16 + 2 * off[:, None] + (n + 64) * 2.0 ** -24) + np.abs(want) * HALF
            err = np.abs(got[t, heads] - want)
            assert (err <= tol).all(), f"{label}: token {t}, K/V head {g}: {np.max(err / tol):.2f} of the bound"


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D,Hq,Hkv", [(64, 8, 2), (128, 5, 1), (128, 16, 2), (80, 3, 3), (48, 16, 1), (112, 9, 1), (128, 12, 1), (256, 4, 2), (256, 16, 1), (144, 7, 1)], ids=str)
def test_weights_keep_sixteen_bits_in_a_step(fmt, D, Hq, Hkv):
    """Groups of one head to sixteen, contexts of a few tokens to ones that are cut."""
    total = np.array([3, 10, 40, 64, 200, 1000, 3000])
    p = Pools(fmt, D, Hq, Hkv, total, seed=109)
    p.fill(total, 110)
    q = _q(len(total), p, 111, 0.4)
    slopes = (0.1 * 2.0 ** (-8.0 * np.arange(1, Hq + 1) / Hq)).astype(np.float32)
    for cap, sl in ((0.0, None), (5.0, None), (0.0, slopes), (200.0, slopes)):
        out, lse = _decode(p, total, q, _scores(p, cap, sl))
        check_rows(p, q, out, lse, np.arange(len(total)), total - 1, np.zeros(len(total)), total, cap, sl)
        _check_bits(p, q, out, np.arange(len(total)), total - 1, cap, sl, range(len(total)), f"cap {cap}, slopes {sl is not None}")
    p.ctx.close()


@pytest.mark.parametrize("D,Hq,Hkv", [(64, 8, 2), (16, 3, 1), (80, 3, 3), (48, 16, 1), (112, 9, 1), (256, 4, 2), (144, 7, 1)], ids=str)
@pytest.mark.parametrize("few", [False, True])
def test_weights_keep_sixteen_bits_in_prompts(D, Hq, Hkv, few):
    """Over bf16 caches of heads other than 128; behind contexts that are cut too; an infinite value is one in the rows that see it."""
    before, new = (np.array([1000, 0]), np.array([7, 3])) if few else (np.array([30, 0, 100]), np.array([60, 90, 1]))
    total = before + new
    p = Pools("bf16", D, Hq, Hkv, total, seed=112)
    p.fill(total, 113)
    seq, pos = packed(before, new)
    q = _q(len(seq), p, 114, 0.4)
    slopes = (0.1 * 2.0 ** (-8.0 * np.arange(1, Hq + 1) / Hq)).astype(np.float32)
    for cap, sl in ((0.0, None), (5.0, None), (0.0, slopes), (200.0, slopes)):
        out, lse = _prefill(p, before, new, q, _scores(p, cap, sl))
        check_rows(p, q, out, lse, seq, pos, np.zeros(len(seq)), pos + 1, cap, sl)
        _check_bits(p, q, out, seq, pos, cap, sl, range(0, len(seq), 3), f"cap {cap}, slopes {sl is not None}")
    k, v = p.logical()
    v[p.table[0, 0], :, 9, 5] = float("inf")
    p.put(k, v)
    out, lse = _prefill(p, before, new, q)
    row = torch.from_numpy((seq == 0) & (pos >= 9)).cuda()
    assert (out[row][..., 5] == float("inf")).all() and out[~row].isfinite().all() and lse.isfinite().all()
    out[..., 5] = 0
    assert out.isfinite().all()
    p.ctx.close()


def test_structs_whose_tensors_are_gone():
    """What a struct names and its holder no longer holds is refused, and not read."""
    total = np.array([20])
    p = Pools("e4m3", 64, 4, 2, total, seed=115)
    p.fill(total, 116)
    b = p.binding
    q = _q(1, p, 117)
    seen = torch.zeros(1, dtype=torch.int32, device="cuda")
    make = lambda: b.Scores(slopes=torch.zeros(4, device="cuda"), key_begin=seen, key_end=seen + 20)
    assert _decode(p, total, q, make())[0].isfinite().all() and _prefill(p, total - 1, np.ones(1, dtype=int), q, make())[0].isfinite().all()
    for name in ("slopes", "key_begin", "key_end"):
        scores = make()
        setattr(scores, name, None)
        with pytest.raises(ValueError):
            _decode(p, total, q, scores)
        with pytest.raises(ValueError):
            _prefill(p, total - 1, np.ones(1, dtype=int), q, scores)
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    p.ctx.attn_prefill_scored(q[:0], p.cache, dev_i32([0, 0]), dev_i32([3]), p.dev_table, q[:0].clone(), scores=b.Scores(key_begin=none))   # (no tokens, no ranges)
    rows = torch.randn(1, 2, 64, device="cuda").to(torch.bfloat16)
    w = torch.ones(64, device="cuda")
    cu, at = dev_i32([0, 1]), dev_i32([3])
    for name in ("q_weight", "k_weight"):
        norm = b.HeadNorm(1e-6, w, w)
        p.ctx.kv_append_norm(p.cache, rows, rows, cu, at, p.dev_table, norm=norm)
        setattr(norm, name, None)
        with pytest.raises(ValueError):
            p.ctx.kv_append_norm(p.cache, rows, rows, cu, at, p.dev_table, norm=norm)
    p.ctx.kv_append_norm(p.cache, rows, rows, cu, at, p.dev_table, norm=b.HeadNorm(1e-6, None, w))
    bare = b.PagedCache(p.cache.k, p.cache.v, p.cache.scales, format="e4m3")
    bare.scales = None
    with pytest.raises(ValueError):
        p.ctx.kv_append_norm(bare, rows, rows, cu, at, p.dev_table)
    p.ctx.close()
