"""Rotated append against the definition in 64 bits: K in the cache and Q in q_out within the roundings of the type, V bit for bit,
everything that a call does not address as it was."""
import numpy as np
import pytest
import torch

from oracle import sparse_oracle as so
from paper_2504_18154_amd import workloads as wl
from tests.parity_util import dev_i32, say

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def _within(name, got, exact, size, angle, dtype):
    """One rounding to the type; three fp32 roundings of the products and their sum and as many ulps of sine and cosine (4 + 4 times 2^-24 of
    |a| + |b|); and, of the angle itself, the three 64-bit roundings on either side (position * frequency / 2 pi here, position *
    frequency there)."""
    half = torch.finfo(dtype).eps / 2
    bound = half * np.abs(exact) + size * (2.0 ** -21 + angle * 2.0 ** -50) * (1 + half)
    err = np.abs(got - exact)
    worst = float((err / np.maximum(bound, 1e-300)).max()) if err.size else 0.0
    say(f"  {name}: worst err/bound {worst:.3f}")
    assert (err <= bound).all(), name


def _check(dtype, D, Hq, Hkv, before, new, rotary=None, adjacent=False, axes=1, fused=False, with_q=True, in_place=False, most=None, far=0, seed=0, pad=0):
    from paper_2504_18154_amd import binding
    before, new = np.asarray(before, dtype=np.int32), np.asarray(new, dtype=np.int32)
    B, T, R = len(new), int(new.sum()), rotary or D
    say(f"{dtype}, D {D}, heads {Hq}/{Hkv}, rotary {R}, adjacent {adjacent}, axes {axes}, new {new.tolist()} behind {before.tolist()}")
    model = wl.ModelShape("rope", Hq, Hkv, D, 1, dtype)
    pb = wl.prefill_batch(model, before + new, 5 + seed)
    ctx = binding.Context(Hq, Hkv, D, pb.num_blocks, dtype, B, pb.block_table.shape[1])
    dt = model.torch_dtype
    rows = wl.randn((T + pad, Hq + 2 * Hkv, D), dtype, 40 + seed).cuda()
    q, k, v = rows[:, :Hq], rows[:, Hq:Hq + Hkv], rows[:, Hq + Hkv:]
    if not fused:
        q, k, v = (t.contiguous() for t in (q, k, v))
    exact_q, exact_k, exact_v = (t.float().cpu().numpy() for t in (q, k, v))
    kc, vc = ctx.new_cache()
    ref_v = ctx.v_logical(vc).clone()
    freq = 10000.0 ** (-np.arange(R // 2) * 2.0 / R)
    axis = [(i * axes) // (R // 2) for i in range(R // 2)]
    coords = None
    place = np.concatenate([b + np.arange(n) for b, n in zip(before, new)]) if T else np.zeros(0, dtype=np.int64)
    if axes > 1 or far:
        rng = np.random.default_rng(seed)
        coords = rng.integers(-far - 3, far + 200, size=(axes, T + pad))
        if far:
            coords[0, :2] = (2 ** 31 - 1, -2 ** 31)
    q_out = None
    if with_q:
        q_out = q if in_place else torch.full((T + pad, Hq, D), float("nan"), dtype=dt, device="cuda")
    rope = binding.Rope(torch.as_tensor(freq, device="cuda"), "adjacent" if adjacent else "halves", axis if axes > 1 else None)
    ctx.kv_append_rope(kc, vc, k, v, dev_i32(wl.cu_from_lengths(new)), dev_i32(before), dev_i32(pb.block_table), rope,
                       positions=None if coords is None else dev_i32(coords), q=q if with_q else None, q_out=q_out, max_new_len=most)
    torch.cuda.synchronize()
    gk, gq = ctx.k_logical(kc).float().cpu().numpy().astype(np.float64), None
    seq = np.repeat(np.arange(B), new)
    want_k, size_k, ang_k = np.full(gk.shape, np.nan), np.zeros(gk.shape), np.zeros(gk.shape)
    want_q, size_q, ang_q = np.full((T, Hq, D), np.nan), np.zeros((T, Hq, D)), np.zeros((T, Hq, D))
    blk, slot = pb.block_table[seq, place // 16], place % 16
    for t in range(T):
        where = np.array([place[t] if coords is None else coords[axis[i], t] for i in range(R // 2)])
        angle = np.zeros(D)
        pair = np.abs(where * freq)
        angle[:R] = np.repeat(pair, 2) if adjacent else np.concatenate([pair, pair])
        want_k[blk[t], :, slot[t]], size_k[blk[t], :, slot[t]] = so.rotate(exact_k[t], where, freq, adjacent)
        ang_k[blk[t], :, slot[t]] = angle
        want_q[t], size_q[t] = so.rotate(exact_q[t], where, freq, adjacent)
        ang_q[t] = angle
    touched = ~np.isnan(want_k)
    assert np.isnan(gk[~touched]).all()                      # (the sentinel of new_cache)
    _within("K", gk[touched], want_k[touched], size_k[touched], ang_k[touched], dt)
    bits = lambda t: t.contiguous().view(torch.int16 if dt == BF else torch.int32)
    if T:
        ref_v[torch.as_tensor(blk.astype(np.int64)), :, torch.as_tensor(slot)] = v[:T].to(ref_v.device)
    assert torch.equal(bits(ctx.v_logical(vc)), bits(ref_v))
    if with_q:
        gq = q_out.float().cpu().numpy().astype(np.float64)
        _within("Q", gq[:T], want_q, size_q, ang_q, dt)
        if pad:
            assert np.array_equal(gq[T:], exact_q[T:]) if in_place else np.isnan(gq[T:]).all()
        if fused and in_place:                               # K and V of the row stay
            assert torch.equal(bits(rows[:, Hq:].float().cpu().to(dt)), bits(torch.cat([torch.as_tensor(exact_k), torch.as_tensor(exact_v)], 1).to(dt)))
    if R < D and T:                                          # what is not turned is copied
        assert np.array_equal(gk[blk, :, slot][..., R:], exact_k[:T, :, R:])
    ctx.close()


LAYOUTS = [("bf16", 128, 40, 8, None, False), ("bf16", 128, 5, 1, 64, True), ("bf16", 8, 2, 2, None, False), ("bf16", 64, 32, 8, 32, False),
           ("bf16", 72, 7, 1, None, False), ("bf16", 80, 8, 8, 48, False), ("bf16", 256, 9, 3, None, False), ("bf16", 256, 2, 1, None, True),
           ("bf16", 136, 3, 3, 8, True), ("f32", 4, 2, 1, None, False), ("f32", 64, 4, 2, 32, True), ("f32", 100, 3, 3, None, False),
           ("f32", 128, 6, 3, 44, False), ("f32", 256, 5, 5, None, False), ("f32", 256, 2, 2, None, True)]


@pytest.mark.parametrize("dtype,D,Hq,Hkv,rotary,adjacent", LAYOUTS, ids=[f"{a[0]}-d{a[1]}-{a[2]}x{a[3]}-r{a[4]}-{'adj' if a[5] else 'halves'}" for a in LAYOUTS])
def test_layouts(dtype, D, Hq, Hkv, rotary, adjacent):
    """Prompts of no, one and many tokens around block edges, then one token each."""
    _check(dtype, D, Hq, Hkv, [0, 5, 0, 16, 31, 3], [17, 0, 1, 15, 33, 40], rotary, adjacent)
    _check(dtype, D, Hq, Hkv, [0, 15, 16, 100, 7], [1, 1, 1, 1, 0], rotary, adjacent, most=1, seed=1)


@pytest.mark.parametrize("new,most", [([40, 7, 20], None), ([1, 1, 1], 1)], ids=["prompts", "step"])
def test_axes_rows_and_places(new, most):
    """Several coordinates, far and negative ones; rows of a fused projection; Q turned where it lies; K and V alone; rows behind the batch."""
    before = [9, 16, 300]
    for axes in (2, 3, 4):
        _check("bf16", 128, 8, 2, before, new, axes=axes, fused=True, most=most, seed=axes)
    _check("f32", 64, 4, 2, before, new, axes=3, far=1 << 20, most=most)
    _check("bf16", 64, 4, 2, before, new, axes=1, far=1 << 24, adjacent=True, most=most)
    _check("bf16", 64, 4, 2, before, new, fused=True, in_place=True, most=most, pad=3)
    _check("f32", 64, 4, 2, before, new, in_place=True, most=most, pad=2)
    _check("bf16", 64, 4, 2, before, new, with_q=False, most=most)
    _check("bf16", 64, 4, 2, before, new, fused=True, most=most, pad=5)


def test_many_sequences_and_a_long_prompt():
    rng = np.random.default_rng(4)
    _check("bf16", 64, 4, 1, rng.integers(0, 60, 300), rng.integers(0, 4, 300))
    _check("bf16", 64, 4, 1, rng.integers(0, 60, 300), np.ones(300), most=1)
    _check("bf16", 16, 2, 1, [37], [2500])


def test_position_zero_is_the_plain_append():
    """Turned by nothing: the same bits as kv_append leaves."""
    from paper_2504_18154_amd import binding
    model = wl.ModelShape("rope0", 4, 2, 64, 1, "bf16")
    pb = wl.prefill_batch(model, [33, 2], 3)
    ctx = binding.Context(4, 2, 64, pb.num_blocks, "bf16", 2, pb.block_table.shape[1])
    k, v = (wl.randn((35, 2, 64), "bf16", s).cuda() for s in (1, 2))
    a, b = ctx.new_cache(), ctx.new_cache()
    args = dev_i32(pb.cu_q), dev_i32(pb.ctx_before), dev_i32(pb.block_table)
    ctx.kv_append(*a, k, v, *args)
    rope = binding.Rope(torch.ones(32, dtype=torch.float64, device="cuda"))
    ctx.kv_append_rope(*b, k, v, *args, rope, positions=torch.zeros(1, 35, dtype=torch.int32, device="cuda"))
    for x, y in zip(a, b):
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))
    ctx.close()


def test_what_the_binding_refuses():
    from paper_2504_18154_amd import binding
    ctx = binding.Context(4, 2, 64, 8, "bf16", 2, 4)
    kc, vc = ctx.new_cache()
    k = torch.zeros(3, 2, 64, dtype=BF, device="cuda")
    q = torch.zeros(3, 4, 64, dtype=BF, device="cuda")
    cu, before, bt = dev_i32([0, 2, 3]), dev_i32([0, 0]), dev_i32([[0, 1], [2, 3]])
    rope = binding.Rope(torch.ones(32, dtype=torch.float64, device="cuda"), axis=[0] * 16 + [1] * 16)
    good = dict(positions=torch.zeros(2, 3, dtype=torch.int32, device="cuda"), q=q, q_out=q)
    for change in ({"positions": good["positions"][:1]}, {"positions": good["positions"].long()}, {"positions": good["positions"][:, :2]}, {"q_out": None},
                   {"q": q[:2]}, {"q_out": q[:, :2]}):
        with pytest.raises(ValueError):
            ctx.kv_append_rope(kc, vc, k, k, cu, before, bt, rope, **{**good, **change})
    with pytest.raises(binding.EcoserveError):
        ctx.kv_append_rope(kc, vc, k, k, cu, before, bt, rope)          # two coordinates and no positions
    ctx.kv_append_rope(kc, vc, k, k, cu, before, bt, rope, **good)
    ctx.close()


@pytest.mark.parametrize("dtype,D,Hq,Hkv,rotary", [("bf16", 128, 8, 2, 32), ("bf16", 256, 6, 1, 64), ("bf16", 64, 4, 4, 8), ("bf16", 80, 4, 2, 32), ("f32", 128, 4, 2, 44),
                                                   ("f32", 256, 2, 1, 32), ("f32", 8, 3, 3, 4)])
def test_parts_of_heads_in_place(dtype, D, Hq, Hkv, rotary):
    """Halves of a part of the head, each turned where it lies; slices of a projection's rows."""
    for new, before in (([40, 1, 700], [9, 16, 3]), ([2000], [5])):
        _check(dtype, D, Hq, Hkv, before, new, rotary=rotary, in_place=True, pad=2)
        _check(dtype, D, Hq, Hkv, before, new, rotary=rotary, in_place=True, fused=True)
        _check(dtype, D, Hq, Hkv, before, new, rotary=rotary, axes=2, seed=3)
