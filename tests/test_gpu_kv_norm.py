"""Norms, rotation and codes on the way into the cache, and reading back, against the definition in 64 bits; then a model's layer as it is used: prompts and steps."""
import math

import numpy as np
import pytest
import torch

from oracle import scored_oracle as so
from oracle import sparse_oracle as ro
from tests.parity_util import dev_i32, say
from tests.scored_util import BF, HALF, Pools, check_rows, cu_of, packed

pytestmark = pytest.mark.gpu

LAYOUTS = [(128, 40, 8), (128, 5, 1), (128, 3, 3), (64, 32, 8), (16, 4, 2), (48, 6, 2), (80, 8, 8), (144, 2, 1), (256, 8, 1), (208, 4, 4)]
FORMATS = ["e4m3", "int8", "bf16"]


def _formed(x, eps, weight, where, freq, adjacent):
    """(row in 64 bits, how far fp32 may be off it, per element)"""
    y = so.norm(x, eps, weight) if eps is not None else x.astype(np.float64)
    if len(freq):
        z, size = ro.rotate(y, where, freq, adjacent)
        size = np.where(size == 0, np.abs(y), size)
    else:
        z, size = y, np.abs(y)
    # the norm: D squares summed, a division, a root, two products; the rotation: sine and cosine, two products and a sum
    return z, size * (len(x) / 2 + 16) * 2.0 ** -24 + 1e-37


def _check_cached(p, z, off, blk, g, slot, held, i):
    got = held[i][blk, g, slot]
    if not np.isfinite(z).all():
        assert np.isnan(got).all() if p.fmt != "bf16" else np.array_equal(np.isfinite(got), np.isfinite(z)), (blk, g, slot)
        return
    if p.fmt == "bf16":
        assert (np.abs(got - z) <= off + np.abs(z) * HALF).all(), (blk, g, slot, np.abs(got - z).max())
        return
    b = int(p.now[blk, g, i, slot])
    size, room = float(np.abs(z).max()), float(off.max())
    assert b in (so.scale_byte(max(size - room, 0.0), p.fmt), so.scale_byte(size + room, p.fmt)), (blk, g, slot, b)
    step = 2.0 ** (b - 127)
    half = 0.5 if p.fmt == "int8" else 2.0 ** (np.maximum(np.floor(np.log2(np.maximum((np.abs(z) + off) / step, 1e-300))), -6) - 4)
    assert (np.abs(got - z) <= off + half * step).all(), (blk, g, slot, np.max(np.abs(got - z) / (off + half * step)))


def _run(p, before, new, rng, norm=True, per_head=False, rotary=None, adjacent=False, axes=1, fused=False, with_q=True, in_place=False, most=None, extra=0):
    """One call on random rows, checked whole."""
    D, Hq, Hkv = p.D, p.Hq, p.Hkv
    seq, pos = packed(before, new)
    T = len(seq) + extra
    rows = torch.from_numpy(rng.normal(size=(T, Hq + 2 * Hkv, D)) * np.exp(rng.normal(size=(T, Hq + 2 * Hkv, 1)))).to(BF).cuda()
    q, k, v = rows[:, :Hq], rows[:, Hq:Hq + Hkv], rows[:, Hq + Hkv:]
    if not fused:
        q, k, v = (t.contiguous() for t in (q, k, v))
    qh, kh, vh = (t.double().cpu().numpy() for t in (q, k, v))
    eps = 1e-5 if norm else None
    qw, kw = (((0.5 + rng.random((h, D))) if per_head else (0.5 + rng.random(D))).astype(np.float32) if norm else None for h in (Hq, Hkv))
    R = D if rotary is None else rotary
    freq = 10000.0 ** (-np.arange(R // 2) * 2.0 / max(R, 1))
    axis = [min(i * axes // max(R // 2, 1), axes - 1) for i in range(R // 2)]
    coords = None
    if axes > 1:
        coords = np.concatenate([np.concatenate([pos, np.zeros(extra, dtype=int)])[None], rng.integers(0, 3000, size=(axes - 1, T))]).astype(np.int32)
    b = p.binding
    q_out = q if in_place else torch.full((T, Hq, D), 55.0, dtype=BF, device="cuda")
    was = [t.clone() for t in (p.cache.k, p.cache.v)] + ([p.cache.scales.clone()] if p.fmt != "bf16" else [])
    p.ctx.kv_append_norm(p.cache, k, v, cu_of(new), dev_i32(before), p.dev_table,
                         norm=b.HeadNorm(eps, torch.from_numpy(qw).cuda(), torch.from_numpy(kw).cuda()) if norm else None,
                         rope=b.Rope(torch.from_numpy(freq).cuda(), pairing="adjacent" if adjacent else "halves", axis=axis if axes > 1 else None) if R else None,
                         positions=dev_i32(coords) if coords is not None else None, q=q if with_q else None, q_out=q_out if with_q else None, max_new_len=most)
    p.now = p.scales()
    held = p.held()
    got_q = q_out.double().cpu().numpy()
    for t in range(len(seq)):
        where = np.array([coords[axis[i], t] for i in range(R // 2)]) if coords is not None else np.full(R // 2, pos[t])
        for h in range(Hq if with_q else 0):
            if pos[t] < 0:
                assert (got_q[t, h] == (qh[t, h] if in_place else 55.0)).all()
                continue
            z, off = _formed(qh[t, h], eps, None if qw is None else qw[h] if per_head else qw, where, freq, adjacent)
            assert (np.abs(got_q[t, h] - z) <= off + np.abs(z) * HALF).all(), (t, h, np.abs(got_q[t, h] - z).max())
        if pos[t] < 0:
            continue
        blk, slot = p.table[seq[t], pos[t] // 16], pos[t] % 16
        for g in range(Hkv):
            z, off = _formed(kh[t, g], eps, None if kw is None else kw[g] if per_head else kw, where, freq, adjacent)
            _check_cached(p, z, off, blk, g, slot, held, 0)
            _check_cached(p, vh[t, g], np.zeros(D), blk, g, slot, held, 1)
    if extra:
        assert (got_q[len(seq):] == 55.0).all()
    # nothing else has changed
    live = np.zeros((p.blocks, 16), dtype=bool)
    ok = pos >= 0
    live[p.table[seq[ok], pos[ok] // 16], pos[ok] % 16] = True
    x = 8 if p.fmt == "bf16" else 16
    gone = torch.from_numpy(~live).cuda()
    bits = torch.int16 if p.fmt == "bf16" else torch.uint8
    same = lambda a, o: a.view(bits) == o.view(bits)
    assert same(p.cache.k, was[0]).view(p.blocks, Hkv, D // x, 16, x).permute(0, 3, 1, 2, 4)[gone].all()
    assert same(p.cache.v, was[1]).view(p.blocks, Hkv, D, 16).permute(0, 3, 1, 2)[gone].all()
    if p.fmt != "bf16":
        assert (p.cache.scales == was[2]).permute(0, 3, 1, 2)[gone].all()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D,Hq,Hkv", LAYOUTS, ids=str)
def test_append(fmt, D, Hq, Hkv):
    before, new = np.array([0, 5, 16, 30, 0, 7]), np.array([1, 27, 16, 3, 0, 9])
    rng = np.random.default_rng(D + Hq)
    p = Pools(fmt, D, Hq, Hkv, before + new, seed=D)
    R = D // 2 // 8 * 8
    for kw in (dict(), dict(adjacent=True), dict(rotary=R, per_head=True, fused=True), dict(rotary=0), dict(norm=False), dict(norm=False, rotary=0, with_q=False), dict(rotary=8, in_place=True),
               dict(axes=3, adjacent=True, fused=True), dict(extra=3)):
        say(f"append {fmt}, D {D}, heads {Hq}/{Hkv}: {kw}")
        _run(p, before, new, rng, **kw)
    p.ctx.close()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D,Hq,Hkv", LAYOUTS, ids=str)
def test_append_of_a_step(fmt, D, Hq, Hkv):
    before = np.array([0, 15, 16, 17, 31, 100, 5])
    new = np.array([1, 1, 1, 1, 1, 1, 0])
    rng = np.random.default_rng(D + Hq)
    p = Pools(fmt, D, Hq, Hkv, before + new, seed=D)
    R = D // 2 // 8 * 8
    for kw in (dict(), dict(adjacent=True, per_head=True), dict(rotary=R, fused=True), dict(norm=False, rotary=0, with_q=False), dict(axes=2), dict(in_place=True)):
        say(f"append of a step {fmt}, D {D}, heads {Hq}/{Hkv}: {kw}")
        _run(p, before, new, rng, most=1, **kw)
    p.ctx.close()


@pytest.mark.parametrize("fmt", FORMATS)
def test_places_of_padding_store_nothing(fmt):
    rng = np.random.default_rng(5)
    p = Pools(fmt, 64, 4, 2, [13, 60, 5], seed=6)
    _run(p, np.array([-20, -16, 0]), np.array([33, 76, 5]), rng)
    _run(p, np.array([-3, 4, -1]), np.array([1, 1, 1]), rng, most=1)
    p.ctx.close()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("step", [False, True])
def test_rows_of_all_sizes(fmt, step):
    """Zeros, tiny and huge rows, the borders of a scale, NaN and infinities, as they are (no norm)."""
    p = Pools(fmt, 64, 2, 1, [40], seed=7)
    n = 20
    rng = np.random.default_rng(8)
    x = torch.from_numpy(rng.normal(size=(n, 1, 64))).to(BF)
    x[0] = 0
    x[1] *= 1e-38
    x[2] *= 1e37
    x[3] = 127.0
    x[4, 0, 3] = 448.0
    x[5, 0, 3] = 449.0
    x[6, 0, 63] = float("nan")
    x[7, 0, 0] = float("inf")
    x[8, 0, 9] = -float("inf")
    x[9, 0, 1] = 127.5
    x[10] = torch.linspace(-8, 8, 64).to(BF)
    x[11] *= 1e-41
    k, v = x.cuda(), x.flip(0).contiguous().cuda()
    if step:
        for i in range(n):
            p.ctx.kv_append_norm(p.cache, k[i:i + 1], v[i:i + 1], cu_of([1]), dev_i32([11 + i]), p.dev_table, max_new_len=1)
    else:
        p.ctx.kv_append_norm(p.cache, k, v, cu_of([n]), dev_i32([11]), p.dev_table)
    kl, vl = p.logical()
    s = p.scales()
    for i in range(n):
        blk, slot = p.table[0, (11 + i) // 16], (11 + i) % 16
        for j, (pool, row) in enumerate(((kl, x[i, 0]), (vl, x[n - 1 - i, 0]))):
            if fmt == "bf16":
                assert torch.equal(pool[blk, 0, slot].view(torch.int16), row.view(torch.int16)) or row.isnan().any()
                continue
            want, b = so.code(row.double().numpy(), fmt)
            assert s[blk, 0, j, slot] == b and np.array_equal(so.number(pool[blk, 0, slot].numpy(), fmt), so.number(want, fmt)), (i, j)
    p.ctx.close()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D,Hkv", [(128, 8), (64, 1), (16, 3), (80, 5), (256, 2), (144, 1)])
def test_read_back(fmt, D, Hkv):
    """Any run of tokens of any sequence, both or one of keys and values, rows in wider ones; NaN rows; exact."""
    total = np.array([70, 1, 40, 200, 0])
    p = Pools(fmt, D, Hkv, Hkv, total, seed=D)
    p.fill(total, 9, wide=3.0)
    if fmt != "bf16":
        p.cache.scales[p.table[0, 1], 0, :, 3] = 255
    held = p.held()
    first, count = np.array([3, 0, 16, 37, 0]), np.array([60, 1, 24, 150, 0])
    seq, pos = packed(first, count)
    want = [np.stack([[h[p.table[b, j // 16], g, j % 16] for g in range(Hkv)] for b, j in zip(seq, pos)]) for h in held]
    T = len(seq)
    for wide in (False, True):
        rows = torch.full((T + 2, 2 * Hkv + 1, D), 77.0, dtype=BF, device="cuda")
        k, v = rows[:, :Hkv], rows[:, Hkv:2 * Hkv]
        if not wide:
            k, v = k.contiguous(), v.contiguous()
        for pick in ((k, v), (k, None), (None, v)):
            for t in (k, v):
                t.fill_(77.0)
            p.ctx.kv_read(p.cache, *pick, cu_of(count), dev_i32(first), p.dev_table)
            for t, w in zip((k, v), want):
                given = any(t is x for x in pick)
                got = t.double().cpu().numpy()
                assert np.array_equal(got[:T], w, equal_nan=True) if given else (got == 77.0).all()
                assert (got[T:] == 77.0).all()
        if wide:
            assert (rows[:, -1] == 77.0).all()
    p.ctx.kv_read(p.cache, k, v, cu_of(np.array([10, 0, 0, 0, 0])), dev_i32([-4, 0, 0, 0, 0]), p.dev_table)
    assert torch.equal(k[4:10].nan_to_num(), torch.from_numpy(np.stack([[held[0][p.table[0, 0], g, j] for g in range(Hkv)] for j in range(6)])).to(BF).cuda().nan_to_num())
    p.ctx.close()


@pytest.mark.parametrize("fmt", FORMATS)
def test_a_layer_as_it_is_used(fmt):
    """Prompts, then steps, of a layer with norms, rotation, capped scores and a window: what each call leaves is what the next reads; the caches read back at the end."""
    D, Hq, Hkv, window, cap = 128, 8, 2, 100, 25.0
    lens = np.array([37, 150, 1])
    steps = 20
    p = Pools(fmt, D, Hq, Hkv, lens + steps, seed=11)
    b = p.binding
    g = torch.Generator().manual_seed(12)
    qw, kw = (0.5 + torch.rand(D, generator=g) for _ in range(2))
    norm, rope = b.HeadNorm(1e-6, qw.cuda(), kw.cuda()), b.Rope(torch.from_numpy(10000.0 ** (-np.arange(D // 2) * 2.0 / D)).cuda())

    def pass_(before, new, most):
        seq, pos = packed(before, new)
        rows = torch.randn(len(seq), Hq + 2 * Hkv, D, generator=g).to(BF).cuda()
        q = torch.empty(len(seq), Hq, D, dtype=BF, device="cuda")
        p.ctx.kv_append_norm(p.cache, rows[:, Hq:Hq + Hkv], rows[:, Hq + Hkv:], cu_of(new), dev_i32(before), p.dev_table, norm=norm, rope=rope, q=rows[:, :Hq], q_out=q, max_new_len=most)
        begin = np.maximum(pos + 1 - window, 0)
        scores = b.Scores(softcap=cap, key_begin=dev_i32(begin))
        out, lse = torch.empty_like(q), torch.empty(len(seq), Hq, device="cuda")
        if most == 1:
            p.ctx.attn_decode_scored(q, p.cache, p.dev_table, dev_i32(before + 1), out, int(before.max()) + 1, lse=lse, scores=scores)
        else:
            p.ctx.attn_prefill_scored(q, p.cache, cu_of(new), dev_i32(before), p.dev_table, out, lse=lse, scores=scores)
        check_rows(p, q, out, lse, seq, pos, begin, pos + 1, cap, tokens=range(0, len(seq), 3 if most != 1 else 1))

    pass_(np.zeros(3, dtype=int), lens, None)
    for i in range(steps):
        pass_(lens + i, np.ones(3, dtype=int), 1)
    total = lens + steps
    k, v = (torch.empty(int(total.sum()), Hkv, D, dtype=BF, device="cuda") for _ in range(2))
    p.ctx.kv_read(p.cache, k, v, cu_of(total), dev_i32(np.zeros(3)), p.dev_table)
    held = p.held()
    for t, (s, j) in enumerate(zip(*packed(np.zeros(3, dtype=int), total))):
        for i, x in enumerate((k, v)):
            assert np.array_equal(x[t].double().cpu().numpy(), held[i][p.table[s, j // 16], :, j % 16])
    # a moved sequence: its rows, appended as they are elsewhere, are the same bytes
    other = Pools(fmt, D, Hq, Hkv, total, seed=13)
    other.ctx.kv_append_norm(other.cache, k, v, cu_of(total), dev_i32(np.zeros(3)), other.dev_table)
    k2, v2 = torch.empty_like(k), torch.empty_like(v)
    other.ctx.kv_read(other.cache, k2, v2, cu_of(total), dev_i32(np.zeros(3)), other.dev_table)
    assert torch.equal(k, k2) and torch.equal(v, v2)
    p.ctx.close()
    other.ctx.close()
