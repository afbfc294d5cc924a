"""Attention over listed blocks, block summaries and selection at the ends of their ranges: scores of minus infinity, sizes of keys far apart, scores beyond what fp32 holds."""
import math

import numpy as np
import pytest
import torch

from oracle import sparse_oracle as so
from tests.parity_util import dev_i32, say
from tests.test_gpu_sparse import Batch, _all_summarised, _attend, _compare, _of_prompts, _random_lists, _select, _summary_host

pytestmark = pytest.mark.gpu


# ---- scores of minus infinity ---------------------------------------------------------------------
# A key of -inf in a channel in which the queries are positive scores -inf: its weight is 0, and a row whose keys all score so is 0 / 0.


def _with_a_block_of_minus_infinity(dtype, D, Hq, Hkv, before, new, block, seed):
    b = Batch(dtype, D, Hq, Hkv, before, new, seed=seed)
    b.q[:, :, 0] = b.q[:, :, 0].abs() + 0.5
    b.keys[b.table[:, block], 0, :, 0] = -float("inf")
    b.upload()
    return b


def _check_minus_infinity(b, lists, out, lse, block, tokens, name, **kw):
    """Rows of K/V head 0 that list `block` and others: as if they did not list it; that list it alone: NaN.  Rows without keys: 0 and -inf."""
    o, l = out.float().cpu().numpy(), lse.cpu().numpy()
    others = lists.copy()
    others[:, 0][others[:, 0] == block] = -1
    keys = lambda j, t: any(0 <= x <= b.pos[t] // 16 for x in j)
    undefined = [t for t in range(b.T) if keys(lists[t, 0], t) and not keys(others[t, 0], t)]
    assert undefined and np.isnan(o[undefined][:, :b.G]).all() and np.isnan(l[undefined][:, :b.G]).all()
    assert np.isfinite(np.delete(o[:, :b.G], undefined, 0)).all()
    empty = [t for t in range(b.T) if not keys(lists[t, 0], t)]
    assert empty and (o[empty][:, :b.G] == 0).all() and np.isneginf(l[empty][:, :b.G]).all()
    _compare(b, others, out, lse, name=name, tokens=[t for t in tokens if t not in set(undefined)], **kw)


@pytest.mark.parametrize("dtype,D,Hq,Hkv", [("bf16", 128, 16, 2), ("bf16", 64, 4, 2), ("f32", 64, 4, 2), ("f32", 256, 3, 1)])
def test_scores_of_minus_infinity_in_a_step(dtype, D, Hq, Hkv):
    b = _with_a_block_of_minus_infinity(dtype, D, Hq, Hkv, [3000] * 6, [1] * 6, 1, D)
    rng = np.random.default_rng(D)
    for K in (6, 200):                                           # whole lists, and parts
        lists = np.full((6, Hkv, K), -1, dtype=np.int32)
        for t in range(6):
            for g in range(Hkv):
                lists[t, g, K // 2:] = rng.choice(np.arange(2, 188), K - K // 2)
        lists[0, 0, 0] = 1
        lists[1, 0, :K // 2] = 1                                 # (parts that have nothing else)
        lists[2, 0] = lists[2, 0, ::-1]
        lists[2, 0, -1] = 1
        lists[3, 0] = np.where(np.arange(K) < K // 2, 1, -1)     # alone
        lists[4, 0] = -1
        out, lse = _attend(b, lists, ragged=False)
        _check_minus_infinity(b, lists, out, lse, 1, range(6), f"{K} entries")
    b.ctx.close()


def test_scores_of_minus_infinity_among_prompts():
    b = _with_a_block_of_minus_infinity("bf16", 128, 16, 2, [100], [2100], 1, 1)
    lists = _random_lists(b, 5, np.random.default_rng(1))
    for t in range(b.T):
        n = b.pos[t] // 16 + 1
        lists[t, 0] = [[1, 3, n - 1, -1, -1], [1, -1, -1, -1, -1], [3, 5, -1, -1, -1], [-1] * 5, [n - 1, 2, 0, 1, -1]][t % 5]
    out, lse = _attend(b, lists)
    _check_minus_infinity(b, lists, out, lse, 1, _of_prompts(b), "prompts", rounded_weights=True)
    lists[1000, 0, 3:] = 3                                       # (a block twice: the tokens around it are taken one by one)
    out, lse = _attend(b, lists)
    _check_minus_infinity(b, lists, out, lse, 1, range(960, 1040), "prompts, one by one", rounded_weights=True)
    b.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("key", [-float("inf"), -1e4], ids=["minus-infinity", "far-below"])
def test_an_infinite_value_under_the_smallest_weights(dtype, key):
    """It reaches the row whichever part of a list, wavefront or group the block is in, also where fp32 holds no weight so small (zero times infinity)."""
    b = _with_a_block_of_minus_infinity(dtype, 64, 4, 2, [3000] * 2, [1] * 2, 1, 3)
    b.keys[b.table[:, 1], 0, :, 0] = key
    b.vals[b.table[:, 1], 0, :, 9] = float("inf")
    b.upload()
    for K in (6, 200):
        for n in range(1, min(K, 33)):                           # (as many entries as the first part has, among others)
            lists = np.tile(2 + np.arange(K, dtype=np.int32) % 184, (2, 2, 1))
            lists[0, 0, :n] = 1
            out, _ = _attend(b, lists, ragged=False)
            o = out.float().cpu().numpy()
            assert not np.isfinite(o[0, :2, 9]).any() and np.isfinite(np.delete(o[0, :2], 9, 1)).all() and np.isfinite(o[0, 2:]).all() and np.isfinite(o[1]).all(), (K, n)
    b.ctx.close()


# ---- keys of sizes far apart ----------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_codes_bound_keys_far_below_the_largest(dtype):
    """Rounded outward however small a key is beside the block's largest: below a unit of the code by more than fp32 can say, it still takes one."""
    b = Batch(dtype, 32, 4, 2, [0], [64], seed=2)
    b.keys[:, :, :, 0] = 1e30
    for j, small in enumerate((1e-30, -1e-30, 1e-38, 3.0)):
        b.keys[b.table[0, j], :, :, 1:] = small
    b.keys[b.table[0, 3], :, :, 2] = 0
    b.upload()
    codes, exps = _summary_host(b.ctx.layout, b.summarise())
    for j in range(4):
        for g in range(2):
            want, e = so.summarise(b.keys[b.table[0, j], g].float().numpy())
            assert exps[b.table[0, j], g] == e and np.array_equal(codes[b.table[0, j], g], want), (j, g)
    b.ctx.close()


# ---- scores beyond the numbers of fp32 ------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("keys,queries", [(1e20, 1e20), (1e30, 1e10), (1e-20, 1e-20), (1e-30, 1e-12), (1e25, 1e-25)])
def test_scores_at_the_ends_of_the_range(dtype, keys, queries):
    """Scores are fp32 numbers: beyond the largest they are infinite, below the smallest zero, and equal ones go by index; in between (the last pair) the order is exact."""
    b = Batch(dtype, 32, 4, 2, [1500, 700], [1, 1], seed=3)
    b.keys *= keys
    b.q *= queries
    b.upload()
    summary, codes, exps = _all_summarised(b)
    ragged = Batch(dtype, 32, 4, 2, [1000], [500], seed=4)
    ragged.keys *= keys
    ragged.q *= queries
    ragged.upload()
    for x, one in ((b, True), (ragged, False)):
        summary, codes, exps = _all_summarised(x)
        got = _select(x, summary, 9, 1, 2, ragged=not one)
        q, ties = x.q.float().numpy(), 0
        for t in range(0, x.T, 1 if one else 31):
            n = x.pos[t] // 16 + 1
            ids = x.table[x.seq[t], :n - 1]
            for g in range(x.Hkv):
                s = so.scores(q[t, g * x.G:(g + 1) * x.G], codes[ids, g, :, :x.D], exps[ids, g])
                with np.errstate(over="ignore", under="ignore"):
                    held = s.astype(np.float32)
                ties += len(held) - len(np.unique(held))
                assert got[t, g].tolist() == so.choose(held, n, 9, 1, 2), (t, g)
                if keys == 1e25:
                    assert got[t, g].tolist() == so.choose(s, n, 9, 1, 2)
        assert ties > 0 or keys == 1e25
    b.ctx.close()
    ragged.ctx.close()


# ---- bits of the weights --------------------------------------------------------------------------


@pytest.mark.parametrize("D,Hq,Hkv,new", [(128, 16, 2, [100, 0, 2600]), (72, 14, 2, [3700]), (256, 8, 1, [2100])], ids=["d128", "d72", "d256"])
def test_prompts_keep_the_bits_of_a_step(D, Hq, Hkv, new):
    """16 bits of a weight, whether a token is alone or one of many that share blocks; an infinite value meets no weight of zero."""
    b = Batch("bf16", D, Hq, Hkv, [17 + 100 * i for i in range(len(new))], new, seed=D)
    assert b.T * Hkv * D >= 2048 * 256
    lists = _random_lists(b, 7, np.random.default_rng(D + 1))
    out, lse = _attend(b, lists)
    _compare(b, lists, out, lse, name="16 bits", tokens=_of_prompts(b))
    b.vals[b.table[len(new) - 1, 2], 0, 5, 3] = float("inf")
    b.upload()
    out, _ = _attend(b, lists)
    o = out.float().cpu().numpy()[:, :b.G]
    hit = (lists[:, 0] == 2).any(1) & (b.seq == len(new) - 1) & (b.pos >= 2 * 16 + 5)
    assert hit.any() and np.isposinf(o[hit][:, :, 3]).all() and np.isfinite(np.delete(o[hit], 3, 2)).all() and np.isfinite(o[~hit]).all()
    b.ctx.close()
