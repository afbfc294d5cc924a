"""Block selection and attention over listed blocks where a call takes another way: a few tokens a sequence, tables too wide for the groups of prompts' tokens, calls of more
threads than one launch has, calls of nothing, a context shared by calls on two streams one after the other."""
import math

import numpy as np
import pytest
import torch

from paper_2504_18154_amd import workloads as wl
from tests.parity_util import dev_i32, say
from tests.test_gpu_sparse import Batch, _all_summarised, _attend, _compare, _expected_lists, _of_prompts, _random_lists, _select

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,D,Hq,Hkv", [("bf16", 128, 40, 8), ("bf16", 64, 16, 1), ("bf16", 96, 6, 6), ("bf16", 128, 12, 2), ("bf16", 32, 6, 3), ("f32", 64, 8, 4)])
def test_a_few_tokens_a_sequence(dtype, D, Hq, Hkv):
    """Up to two tokens a sequence on average (a step that checks drafted tokens): K/V heads alone, by two and by four in a workgroup, tokens side by side in a product."""
    for new in ([2] * 7, [0, 4, 1, 0, 5, 1, 0], [1, 0, 0, 13, 0, 0, 0]):
        b = Batch(dtype, D, Hq, Hkv, [1400, 15, 700, 255, -2, 90, 1055], new, seed=D + len(set(new)))
        say(f"{dtype}, D {D}, heads {Hq}/{Hkv}: {new}")
        summary, codes, exps = _all_summarised(b)
        for K, first, last in ((3, 1, 1), (17, 0, 4)):
            assert np.array_equal(_select(b, summary, K, first, last), _expected_lists(b, codes, exps, K, first, last)), (K, first, last)
        lists = _random_lists(b, 9, np.random.default_rng(D))
        out, lse = _attend(b, lists)
        _compare(b, lists, out, lse, name="attention", tokens=np.flatnonzero(b.pos >= 0))
        nothing = torch.as_tensor(b.pos < 0)
        assert (out.cpu()[nothing] == 0).all() and torch.isneginf(lse.cpu()[nothing]).all()
        b.ctx.close()


def test_prompts_in_wide_tables():
    """Tables wider than the union of a group's lists has room for: the same call token by token; results within both ways' roundings."""
    rng = np.random.default_rng(2)
    b = Batch("bf16", 128, 16, 2, [500, 30], [1300, 900], seed=3)
    lists = _random_lists(b, 6, rng)
    some = _of_prompts(b)
    grouped, grouped_lse = _attend(b, lists)
    _compare(b, lists, grouped, grouped_lse, name="in groups", tokens=some, rounded_weights=True)
    for width in (5120, 5121):
        wide = np.full((2, width), -1, dtype=np.int32)
        wide[:, :b.table.shape[1]] = b.table
        b.dev["block_table"] = dev_i32(wide)
        out, lse = _attend(b, lists)
        if width == 5120:
            assert torch.equal(out, grouped) and torch.equal(lse, grouped_lse)
        else:
            _compare(b, lists, out, lse, name="token by token", tokens=some)
    b.ctx.close()


@pytest.mark.parametrize("Hkv,T,B", [(16, 600_000, 1), (112, 655_360, 8)], ids=["token-by-token", "groups"])
def test_more_threads_than_one_launch_has(Hkv, T, B):
    """2^31 threads and more: several launches.  Every token has the same queries and attends to the first block; the blocks of all tables are the same one."""
    from paper_2504_18154_amd import binding
    D, per = 8, T // B
    ctx = binding.Context(Hkv, Hkv, D, 4, "bf16", B, per // 16)
    say(f"{T} tokens of {B} sequences, {Hkv} heads of {D}")
    g = torch.Generator(device="cuda").manual_seed(1)
    kc, vc = (torch.randn(4 * Hkv * 16 * D, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    q1 = torch.randn(Hkv, D, generator=g, device="cuda").to(torch.bfloat16)
    q = q1.expand(T, -1, -1).contiguous()
    lists = torch.zeros(T, Hkv, 1, dtype=torch.int32, device="cuda")
    out = torch.full_like(q, float("nan"))
    table = torch.full((B, per // 16), 2, dtype=torch.int32, device="cuda")
    ctx.attn_sparse(q, kc, vc, torch.zeros(B, dtype=torch.int32, device="cuda"), table, lists, out, cu_q=dev_i32(np.arange(B + 1) * per))
    keys, vals = ctx.k_logical(kc)[2].double(), ctx.v_logical(vc)[2].double()      # [Hkv, 16, D]
    s = (keys.to(q1.device) @ q1.double()[:, :, None])[..., 0] / math.sqrt(D)
    for n in range(1, 17):
        w = torch.softmax(s[:, :n], 1)
        want, size = (w[:, :, None] * vals.to(w.device)[:, :n]).sum(1), (w[:, :, None] * vals.to(w.device)[:, :n].abs()).sum(1)
        bound = want.abs() * 2.0 ** -8 + size * 2.0 ** -7                          # (half a step of bf16 for the result, and one for the weights; all else is below 2^-15)
        for part in out.view(B, per, Hkv, D)[:, n - 1::1 if n == 16 else per].split(1 << 16, 1):
            assert ((part.double() - want).abs() <= bound).all(), n
    ctx.close()


def test_calls_of_nothing():
    from paper_2504_18154_amd import binding
    ctx = binding.Context(4, 2, 64, 8, "bf16", 2, 4)
    kc, vc = ctx.new_cache()
    summary, was = ctx.new_summary(), (kc.clone(), vc.clone())
    none = dict(dtype=torch.bfloat16, device="cuda")
    k, q, bt = torch.zeros(0, 2, 64, **none), torch.zeros(0, 4, 64, **none), dev_i32([[0, 1], [2, 3]])
    lists = torch.zeros(0, 2, 3, dtype=torch.int32, device="cuda")
    rope = binding.Rope(torch.ones(32, dtype=torch.float64, device="cuda"))
    for cu, before in ((dev_i32([0, 0, 0]), dev_i32([5, 0])), (dev_i32([0]), dev_i32([]))):
        ctx.kv_append_rope(kc, vc, k, k, cu, before, bt, rope, q=q, q_out=torch.empty_like(q))
        ctx.kv_summary(kc, summary, cu, before, bt, 0)
        ctx.block_select(q, summary, before, bt, lists, 32, cu_q=cu)
        ctx.attn_sparse(q, kc, vc, before, bt, lists, torch.empty_like(q), cu_q=cu)
    assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip((kc, vc), was)) and not summary.any()
    ctx.close()


def test_two_streams_in_turn():
    """One context's calls, a step each, on two streams that wait for one another: fused selection and lists in parts count in the context's counters."""
    b = Batch("bf16", 64, 8, 2, [9000, 3000], [1, 1], seed=6)
    summary, codes, exps = _all_summarised(b)
    want = _expected_lists(b, codes, exps, 70, 1, 2)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    first = None
    for i in range(8):
        with torch.cuda.stream(streams[i % 2]):
            streams[i % 2].wait_stream(streams[1 - i % 2])
            got = _select(b, summary, 70, 1, 2, ragged=False)
            out, _ = _attend(b, got, ragged=False)
        assert np.array_equal(got, want)
        first = out if first is None else first
        assert torch.equal(out, first)
    assert b.ctx.sparse_workspace_bytes(2, 70) > 0
    b.ctx.close()


def test_a_rotated_append_is_profiled_as_one():
    from paper_2504_18154_amd import binding
    ctx = binding.Context(4, 2, 64, 8, "bf16", 1, 4)
    kc, vc = ctx.new_cache()
    k = wl.randn((3, 2, 64), "bf16", 1).cuda()
    rope = binding.Rope(torch.ones(32, dtype=torch.float64, device="cuda"))
    ctx.set_option(binding.OPT_PROFILE, 1)
    for _ in range(2):
        ctx.kv_append_rope(kc, vc, k, k, dev_i32([0, 3]), dev_i32([0]), dev_i32([[0]]), rope)
    assert ctx.profile_read(binding.KERNEL_APPEND)[1] == 2
    ctx.close()


@pytest.mark.parametrize("D,Hq,Hkv,new", [(192, 6, 2, [1400]), (32, 16, 8, [1100, 1000]), (24, 12, 12, [1900])], ids=["d192", "d32", "d24"])
def test_groups_of_other_head_sizes(D, Hq, Hkv, new):
    rng = np.random.default_rng(D)
    b = Batch("bf16", D, Hq, Hkv, [90] * len(new), new, seed=D)
    assert b.T * Hkv * D >= 2048 * 256
    lists = _random_lists(b, 6, rng)
    out, lse = _attend(b, lists)
    _compare(b, lists, out, lse, name=f"head size {D}", tokens=_of_prompts(b), rounded_weights=True)
    b.ctx.close()


@pytest.mark.parametrize("growing", [False, True])
def test_groups_and_large_scores(growing):
    """Scores of hundreds of either sign; keys that grow along the sequence, so that the offset of the exponents is raised block by block (a list in order, and backwards)."""
    rng = np.random.default_rng(11)
    b = Batch("bf16", 128, 8, 2, [200], [2100], seed=7)
    if growing:
        for j in range(b.table.shape[1]):
            b.keys[b.table[0, j]] *= 2.0 ** (j // 12)
    else:
        b.q *= 16
        b.keys *= 16
    b.upload()
    some = _of_prompts(b)
    lists = _random_lists(b, 8, rng)
    lists.sort(2)
    for order in (1, -1):
        mine = np.ascontiguousarray(lists[:, :, ::order])
        out, lse = _attend(b, mine)
        assert torch.isfinite(out[16:].float()).all()
        _compare(b, mine, out, lse, name=f"order {order}", tokens=some, rounded_weights=True)
    b.ctx.close()


@pytest.mark.parametrize("dtype,D,Hq,Hkv", [("bf16", 64, 5, 1), ("bf16", 128, 4, 2), ("f32", 160, 3, 1)])
def test_as_many_parts_as_there_are(dtype, D, Hq, Hkv):
    """Lists of 4096 entries and more are cut into 64; most entries hold no keys, and some parts none at all."""
    rng = np.random.default_rng(D)
    b = Batch(dtype, D, Hq, Hkv, [9000, 40], [1, 1], seed=D)
    for K in (4096, 4500):
        assert b.ctx.sparse_workspace_bytes(2, K) == 64 * 2 * Hq * (D + 4) * 4 if Hkv == 1 else b.ctx.sparse_workspace_bytes(2, K) > 0
        lists = _random_lists(b, K, rng, order=False)
        lists[:, :, 700:] = -1
        lists[0, 0, -1] = 3 if 3 not in lists[0, 0] else -1
        out, lse = _attend(b, lists, ragged=False)
        _compare(b, lists, out, lse, name=f"{K} entries")
        assert torch.equal(out, _attend(b, lists, ragged=False)[0])
    b.ctx.close()


@pytest.mark.parametrize("blocks", [300, 2040, 2100, 8190])
def test_few_and_many_rows_choose_alike(blocks):
    """Prompts of as many tokens as each way of choosing takes: the lists of a step of the token alone."""
    from paper_2504_18154_amd import binding
    rng = np.random.default_rng(blocks)
    Hq, Hkv, D, pool = 8, 4, 32, 400
    ctx = binding.Context(Hq, Hkv, D, pool, "bf16", 2, blocks)
    summary = torch.randint(-100, 100, ctx.new_summary().shape, dtype=torch.int8, device="cuda")
    table = rng.integers(0, pool, size=(2, blocks)).astype(np.int32)
    for T in (20, 250, 700):
        new = np.array([T // 3, T - T // 3])
        before = np.array([blocks * 16 - T, blocks * 16 - T - 500], dtype=np.int32)
        q = torch.randn(T, Hq, D, device="cuda").to(torch.bfloat16)
        lists = torch.full((T, Hkv, 12), -7, dtype=torch.int32, device="cuda")
        ctx.block_select(q, summary, dev_i32(before), dev_i32(table), lists, blocks * 16, keep_first=1, keep_last=2, cu_q=dev_i32(wl.cu_from_lengths(new)))
        seq, pos = np.repeat(np.arange(2), new), np.concatenate([b + np.arange(n) for b, n in zip(before, new)])
        one = torch.full((1, Hkv, 12), -7, dtype=torch.int32, device="cuda")
        for t in range(0, T, max(1, T // 40)):
            ctx.block_select(q[t:t + 1], summary, dev_i32(pos[t:t + 1]), dev_i32(table[seq[t]:seq[t] + 1]), one, blocks * 16, keep_first=1, keep_last=2)
            assert torch.equal(one[0], lists[t]), (T, t)
    ctx.close()
