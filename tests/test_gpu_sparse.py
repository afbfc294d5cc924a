"""Block summaries, selection and attention over listed blocks against the definitions in 64 bits: whole numbers equal, results within
the roundings that the kernels make.  Then all of them together, as a decode loop uses them."""
import math

import numpy as np
import pytest
import torch

from oracle import sparse_oracle as so
from paper_2504_18154_amd import workloads as wl
from tests.parity_util import dev_i32, say

pytestmark = pytest.mark.gpu

LAYOUTS = [("bf16", 128, 40, 8), ("bf16", 128, 16, 1), ("bf16", 128, 3, 3), ("bf16", 8, 4, 2), ("bf16", 64, 32, 8), ("bf16", 72, 7, 1), ("bf16", 96, 8, 2),
           ("bf16", 136, 4, 2), ("bf16", 192, 9, 1), ("bf16", 216, 2, 1), ("bf16", 256, 16, 1), ("f32", 4, 2, 1), ("f32", 64, 4, 2), ("f32", 100, 3, 3), ("f32", 128, 6, 3),
           ("f32", 160, 16, 1), ("f32", 196, 2, 2), ("f32", 256, 5, 1), ("f32", 256, 16, 1)]
IDS = [f"{a[0]}-d{a[1]}-{a[2]}x{a[3]}" for a in LAYOUTS]


def _summary_host(lay, buf):
    """(codes int64 [blocks, Hkv, 2, Dp], exponents int64 [blocks, Hkv])"""
    Dp = (lay.head_dim + 31) // 32 * 32
    n = lay.num_blocks * lay.num_kv_heads * 2 * Dp
    a = buf.cpu().numpy().astype(np.int64)
    return a[:n].reshape(lay.num_blocks, lay.num_kv_heads, 2, Dp), a[n:n + lay.num_blocks * lay.num_kv_heads].reshape(lay.num_blocks, lay.num_kv_heads)


class Batch:
    """Sequences with `before` cached tokens that bring `new`: a context, a random cache (all of the pool, or NaN where no token is), a block table."""

    def __init__(self, dtype, D, Hq, Hkv, before, new, seed=0, spare=3, scale=0.0):
        from paper_2504_18154_amd import binding
        self.dtype, self.D, self.Hq, self.Hkv, self.G = dtype, D, Hq, Hkv, Hq // Hkv
        self.before, self.new = np.asarray(before, dtype=np.int32), np.asarray(new, dtype=np.int32)
        self.total = np.maximum(self.before + self.new, 0)
        self.B, self.T = len(self.new), int(self.new.sum())
        rng = np.random.default_rng(seed)
        per = (self.total + 15) // 16
        ids = rng.permutation(int(per.sum()) + spare)
        self.table = np.full((self.B, max(1, int(per.max()))), -1, dtype=np.int32)
        at = 0
        for b in range(self.B):
            self.table[b, :per[b]] = ids[at:at + per[b]]
            at += per[b]
        self.ctx = binding.Context(Hq, Hkv, D, len(ids), dtype, self.B, self.table.shape[1], softmax_scale=scale)
        self.scale = scale or 1 / math.sqrt(D)
        g = torch.Generator().manual_seed(seed)
        dt = self.dt = self.ctx.torch_dtype
        keys, vals = (torch.randn(len(ids), Hkv, 16, D, generator=g).to(dt) for _ in range(2))
        lay = self.ctx.layout
        live = torch.zeros(len(ids), 16, dtype=torch.bool)
        for b in range(self.B):
            for p in range(self.total[b]):
                live[self.table[b, p // 16], p % 16] = True
        keys[~live[:, None].expand(-1, Hkv, -1)] = float("nan")
        vals[~live[:, None].expand(-1, Hkv, -1)] = float("nan")
        self.keys, self.vals = keys, vals                          # logical [blocks, Hkv, 16, D]
        self.upload()
        self.q = torch.randn(self.T, Hq, D, generator=g).to(dt)
        self.cu = wl.cu_from_lengths(self.new)
        self.seq = np.repeat(np.arange(self.B), self.new)
        self.pos = np.concatenate([b + np.arange(n) for b, n in zip(self.before, self.new)]) if self.T else np.zeros(0, int)
        self.dev = dict(cu_q=dev_i32(self.cu), ctx_before=dev_i32(self.before), block_table=dev_i32(self.table))

    def upload(self):
        x = 16 // self.keys.element_size()
        nb = self.keys.shape[0]
        self.kc = self.keys.view(nb, self.Hkv, 16, self.D // x, x).permute(0, 1, 3, 2, 4).contiguous().flatten().cuda()
        self.vc = self.vals.permute(0, 1, 3, 2).contiguous().flatten().cuda()

    def summarise(self, summary=None, cu=None, before=None):
        summary = self.ctx.new_summary() if summary is None else summary
        self.ctx.kv_summary(self.kc, summary, self.dev["cu_q"] if cu is None else dev_i32(cu), self.dev["ctx_before"] if before is None else dev_i32(before),
                            self.dev["block_table"], self.T if cu is None else int(cu[-1]))
        return summary

    def sequence(self, b, of, g, upto):
        """Rows [upto, D] of K/V head g of sequence b in fp64."""
        return torch.cat([of[i, g] for i in self.table[b, :(upto + 15) // 16].tolist()])[:upto].double().numpy() if upto else np.zeros((0, self.D))


def _all_summarised(bt: Batch):
    """Summaries of every full block of the batch, on the device and from the definition."""
    summary = bt.summarise(cu=wl.cu_from_lengths(bt.total), before=np.zeros(bt.B))
    codes, exps = _summary_host(bt.ctx.layout, summary)
    return summary, codes, exps


# ---- summaries ------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype,D,Hq,Hkv", LAYOUTS, ids=IDS)
def test_summaries(dtype, D, Hq, Hkv):
    """Blocks that the call fills, and no others; keys from tiny to huge, zeros, a NaN, infinities of either sign."""
    b = Batch(dtype, D, Hq, Hkv, [0, 5, 15, 16, 0, 100, 31, 3, 0], [16, 10, 1, 15, 0, 44, 33, 61, 200], seed=D)
    say(f"{dtype}, D {D}, heads {Hq}/{Hkv}")
    k = b.keys
    k[b.table[8, 0]] *= 1e-20
    k[b.table[8, 1]] *= 1e30
    k[b.table[8, 2]] = 0
    k[b.table[8, 3], 0, 3, D - 1] = float("nan")
    k[b.table[8, 4], Hkv - 1, 15, 0] = float("inf")
    k[b.table[8, 5], 0, 0, D // 2] = -float("inf")
    k[b.table[8, 6]] *= 1e-41 / 4      # (below the normal numbers)
    k[b.table[8, 7], :, :, 0] = 127.0  # (the most that an exponent of 0 holds, and a step of the type beyond)
    k[b.table[8, 8], :, :, 0] = 127.5
    b.upload()
    summary = torch.full_like(b.ctx.new_summary(), 85)
    b.summarise(summary)
    codes, exps = _summary_host(b.ctx.layout, summary)
    filled = {int(b.table[s, j]) for s in range(b.B) for j in range(b.before[s] // 16, (b.before[s] + b.new[s]) // 16)}
    for blk in range(codes.shape[0]):
        for g in range(Hkv):
            if blk not in filled:
                assert (codes[blk, g] == 85).all() and exps[blk, g] == 85, blk
                continue
            want, e = so.summarise(b.keys[blk, g].float().numpy())
            assert exps[blk, g] == e and np.array_equal(codes[blk, g, :, :D], want) and not codes[blk, g, :, D:].any(), (blk, g, e, exps[blk, g])
    b.ctx.close()


def test_summaries_of_a_step_at_a_time():
    """One token a call: a block's summary appears with its sixteenth token; many sequences, some without a token."""
    b = Batch("bf16", 64, 4, 2, np.arange(70) % 33, np.arange(70) % 7 > 0, seed=1)
    summary = b.summarise(torch.full_like(b.ctx.new_summary(), 85))
    codes, exps = _summary_host(b.ctx.layout, summary)
    for s in range(b.B):
        for j in range((b.total[s] + 15) // 16):
            fresh = b.new[s] and b.before[s] % 16 == 15 and j == b.before[s] // 16
            assert (exps[b.table[s, j]] != 85).all() == bool(fresh)
    b.ctx.close()


# ---- selection ------------------------------------------------------------------------------------


def _expected_lists(b: Batch, codes, exps, K, first, last, q=None):
    q = (b.q if q is None else q).float().numpy()
    want = np.full((b.T, b.Hkv, K), -1, dtype=np.int32)
    for t in range(b.T):
        n = b.pos[t] // 16 + 1 if b.pos[t] >= 0 else 0
        ids = b.table[b.seq[t], :max(n - 1, 0)]
        for g in range(b.Hkv):
            s = so.scores(q[t, g * b.G:(g + 1) * b.G], codes[ids, g, :, :b.D], exps[ids, g]) if n > K else np.zeros(0)
            lst = so.choose(s, n, K, first, last)
            want[t, g, :len(lst)] = lst
    return want


def _select(b: Batch, summary, K, first, last, ragged=True, q=None, max_ctx=None, **kw):
    lists = torch.full((b.T, b.Hkv, K), -7, dtype=torch.int32, device="cuda")
    b.ctx.block_select((b.q if q is None else q).cuda(), summary, b.dev["ctx_before"], b.dev["block_table"], lists, max_ctx or max(1, int(b.total.max())),
                       keep_first=first, keep_last=last, cu_q=b.dev["cu_q"] if ragged else None, **kw)
    return lists.cpu().numpy()


@pytest.mark.parametrize("dtype,D,Hq,Hkv", LAYOUTS, ids=IDS)
def test_selection(dtype, D, Hq, Hkv):
    say(f"{dtype}, D {D}, heads {Hq}/{Hkv}: prompts")
    b = Batch(dtype, D, Hq, Hkv, [0, 300, 17, 0, 150], [1, 9, 40, 0, 130], seed=D)
    summary, codes, exps = _all_summarised(b)
    for K, first, last in ((1, 0, 1), (4, 1, 1), (7, 0, 3), (12, 2, 10)):
        assert np.array_equal(_select(b, summary, K, first, last), _expected_lists(b, codes, exps, K, first, last)), (K, first, last)
    b.ctx.close()
    say(f"{dtype}, D {D}, heads {Hq}/{Hkv}: a step, with places of the batch that are empty")
    b = Batch(dtype, D, Hq, Hkv, [0, 15, 16, 500, -1, 333, 63, -1], [1] * 8, seed=D + 1)
    summary, codes, exps = _all_summarised(b)
    for K, first, last in ((2, 0, 1), (9, 1, 2)):
        want = _expected_lists(b, codes, exps, K, first, last)
        assert np.array_equal(_select(b, summary, K, first, last, ragged=False), want)
        assert np.array_equal(_select(b, summary, K, first, last, ragged=True, max_ctx=b.table.shape[1] * 16), want)
    b.ctx.close()


def test_equal_scores_and_blocks_that_are_not_finite():
    b = Batch("bf16", 32, 4, 2, [1000, 640], [1, 1], seed=9)
    b.keys[:] = b.keys[b.table[0, 0], :, :1]                      # the same key everywhere: all scores are equal
    b.upload()
    summary, codes, exps = _all_summarised(b)
    got = _select(b, summary, 10, 2, 3, ragged=False)
    assert got[0, 0].tolist() == [0, 1, 2, 3, 4, 5, 6, 60, 61, 62] and got[1, 1].tolist() == [0, 1, 2, 3, 4, 5, 6, 38, 39, 40]
    for j, x in ((30, float("nan")), (33, float("inf")), (7, -float("inf"))):
        b.keys[b.table[0, j], 1, 4, 3] = x
    b.upload()
    summary, codes, exps = _all_summarised(b)
    got = _select(b, summary, 6, 0, 1, ragged=False)
    assert got[0, 0].tolist() == [0, 1, 2, 3, 4, 62] and got[0, 1].tolist() == [0, 1, 7, 30, 33, 62]
    assert _select(b, summary, 3, 0, 1, ragged=False)[0, 1].tolist() == [7, 30, 62]
    # queries: zeros, a NaN in one head, an infinity in all of them
    b.keys = torch.randn(b.keys.shape).to(b.dt)
    b.upload()
    summary, codes, exps = _all_summarised(b)
    q = b.q.clone()
    q[0, :2] = 0
    q[0, 2, 5] = float("nan")
    q[1, 0, 0] = float("inf")
    q[1, 1, 0] = -float("inf")
    want = _expected_lists(b, codes, exps, 8, 1, 1, q=q)
    assert np.array_equal(_select(b, summary, 8, 1, 1, ragged=False, q=q), want)
    assert want[0, 0].tolist() == [0, 1, 2, 3, 4, 5, 6, 62]
    b.ctx.close()


@pytest.mark.parametrize("blocks", [2047, 2048, 2050, 8190, 8193, 20011, 33333])
def test_long_contexts(blocks):
    """Around the numbers of blocks that the ways through the histogram change at; scores in narrow and wide ranges, many of them equal."""
    from paper_2504_18154_amd import binding
    rng = np.random.default_rng(blocks)
    Hq, Hkv, D = 4, 2, 32
    ctx = binding.Context(Hq, Hkv, D, blocks, "bf16", 2, blocks)
    lay = ctx.layout
    table = np.stack([rng.permutation(blocks), rng.permutation(blocks)]).astype(np.int32)
    for spread, units in ((1, 2), (100, 1), (127, 30)):
        codes = rng.integers(-spread, spread + 1, size=(blocks, Hkv, 2, 32)).astype(np.int8)
        codes.sort(2)
        codes = codes[:, :, ::-1]
        exps = rng.integers(-units, 1, size=(blocks, Hkv)).astype(np.int8)
        summary = torch.zeros_like(ctx.new_summary())
        flat = np.concatenate([np.ascontiguousarray(codes).ravel(), exps.ravel()])
        summary[:len(flat)] = torch.as_tensor(flat).cuda()
        q = torch.randn(2, Hq, D).to(torch.bfloat16)
        before = np.array([blocks * 16 - 1, blocks * 16 - 40], dtype=np.int32)
        for K, first, last in ((2, 0, 1), (130, 1, 4), (1500, 3, 1)):
            lists = torch.full((2, Hkv, K), -7, dtype=torch.int32, device="cuda")
            ctx.block_select(q.cuda(), summary, dev_i32(before), dev_i32(table), lists, blocks * 16, keep_first=first, keep_last=last)
            got = lists.cpu().numpy()
            lists.fill_(-7)                                   # (the same as a batch of prompts of one token)
            ctx.block_select(q.cuda(), summary, dev_i32(before), dev_i32(table), lists, blocks * 16, keep_first=first, keep_last=last, cu_q=dev_i32([0, 1, 2]))
            assert np.array_equal(lists.cpu().numpy(), got)
            for t in range(2):
                n = before[t] // 16 + 1
                ids = table[t, :n - 1]
                for g in range(Hkv):
                    s = so.scores(q[t, g * 2:g * 2 + 2].float().numpy(), codes[ids, g].astype(np.int64), exps[ids, g].astype(np.int64))
                    order = np.lexsort((np.arange(first, n - last), -s[first:n - last]))[:K - first - last] + first
                    want = np.sort(np.concatenate([np.arange(first), order, np.arange(n - last, n)]))
                    assert np.array_equal(got[t, g], want), (blocks, spread, K, t, g)
    ctx.close()


def test_tokens_in_several_passes(monkeypatch):
    """More tokens than the workspace holds scores of: the same lists as token by token."""
    from paper_2504_18154_amd import binding
    blocks, T = 30000, 130
    rng = np.random.default_rng(3)
    ctx = binding.Context(16, 16, 32, 500, "bf16", 3, blocks)
    assert binding.select_workspace_bytes(ctx.layout, 1 << 20, blocks * 16) < binding.select_workspace_bytes(ctx.layout, 1, blocks * 16) * T   # (192 MiB of scores, 1.9 MB each)
    summary = torch.randint(-100, 100, ctx.new_summary().shape, dtype=torch.int8, device="cuda")
    table = rng.integers(0, 500, size=(3, blocks)).astype(np.int32)
    new = np.array([60, 0, 70])
    before = np.array([blocks * 16 - 60, 5, 4000], dtype=np.int32)
    q = torch.randn(T, 16, 32, device="cuda").to(torch.bfloat16)
    lists = torch.full((T, 16, 20), -7, dtype=torch.int32, device="cuda")
    ctx.block_select(q, summary, dev_i32(before), dev_i32(table), lists, blocks * 16, keep_last=2, cu_q=dev_i32(wl.cu_from_lengths(new)))
    seq, pos = np.repeat(np.arange(3), new), np.concatenate([b + np.arange(n) for b, n in zip(before, new)])
    one = torch.full((1, 16, 20), -7, dtype=torch.int32, device="cuda")
    for t in range(0, T, 7):
        ctx.block_select(q[t:t + 1], summary, dev_i32(pos[t:t + 1]), dev_i32(table[seq[t]:seq[t] + 1]), one, blocks * 16, keep_last=2)
        assert torch.equal(one[0], lists[t]), t
    ctx.close()


# ---- attention ------------------------------------------------------------------------------------


def _attend(b: Batch, lists, ragged=True, with_lse=True, q=None, pad=0, **kw):
    dt = b.dt
    q = (b.q if q is None else q).cuda() if not (q is not None and q.is_cuda) else q
    out = torch.full((b.T + pad, b.Hq, b.D), float("nan"), dtype=dt, device="cuda")
    lse = torch.full((b.T + pad, b.Hq), float("nan"), device="cuda") if with_lse else None
    b.ctx.attn_sparse(q, b.kc, b.vc, b.dev["ctx_before"], b.dev["block_table"], dev_i32(lists), out, lse=lse, cu_q=b.dev["cu_q"] if ragged else None, **kw)
    torch.cuda.synchronize()
    return out, lse


def _compare(b: Batch, lists, out, lse, q=None, name="", tokens=None, rounded_weights=False):
    """Errors that the kernel makes.  A score: the fp32 sum of D products (bounded by D + 2 roundings of the sum of |q k|) and its scaling.
    A weight: twice that, the exponential (2^-21 in all), for bf16 its two parts (2^-15).  The sums over n keys: n + 8 roundings.
    A relative error d of all weights moves the result by at most 2 d sum w |v|.  Then one rounding to the type.
    rounded_weights: the weights of the values (not those of the sum) were rounded to bf16, 2^-8 each."""
    q = (b.q if q is None else q).float().cpu().numpy()
    o = out.float().cpu().numpy().astype(np.float64)
    worst = 0.0
    for t in range(b.T) if tokens is None else tokens:
        s, p = b.seq[t], b.pos[t]
        for g in range(b.Hkv):
            keys, vals = b.sequence(s, b.keys, g, p + 1), b.sequence(s, b.vals, g, p + 1)
            at = np.concatenate([np.arange(j * 16, min(j * 16 + 16, p + 1)) for j in lists[t, g] if 0 <= j <= p // 16] or [np.zeros(0, int)])
            rows = slice(g * b.G, (g + 1) * b.G)
            ref, ref_lse, size, product = so.attend(q[t, rows], keys[at], vals[at], b.scale)
            es = (b.D + 4) * 2.0 ** -24 * product
            d = 2 * es + 2.0 ** -21 + (2.0 ** -15 if b.dtype == "bf16" else 0) + (len(at) + 8) * 2.0 ** -24
            half = torch.finfo(b.dt).eps / 2
            bound = half * np.abs(ref) + (1 + half) * (2 * d[:, None] + (2.0 ** -8 if rounded_weights else 0)) * size
            err = np.abs(o[t, rows] - ref)
            assert (err <= bound).all(), (name, t, g, float(err.max()), float((err / np.maximum(bound, 1e-300)).max()))
            worst = max(worst, float((err / np.maximum(bound, 1e-300)).max()))
            if lse is not None:
                got = lse[t, rows].double().cpu().numpy()
                if len(at) == 0:
                    assert np.isneginf(got).all()
                else:
                    assert (np.abs(got - ref_lse) <= es + d + 2.0 ** -22 * (1 + np.abs(ref_lse))).all(), (name, t, g)
    say(f"  {name}: worst err/bound {worst:.3f}")


def _random_lists(b: Batch, K, rng, order=True):
    """Distinct blocks in any order, among them entries that hold no keys: -1, behind the token, far behind the table, negative."""
    lists = np.full((b.T, b.Hkv, K), -1, dtype=np.int32)
    for t in range(b.T):
        n = max(b.pos[t], -1) // 16 + 1
        for g in range(b.Hkv):
            mine = rng.permutation(n)[:rng.integers(0, K + 1)]
            row = np.concatenate([mine, rng.choice([-1, n, n + 5, 2 ** 31 - 1, -2 ** 31], size=K - len(mine))])
            lists[t, g] = rng.permutation(row) if order else row
    return lists


@pytest.mark.parametrize("dtype,D,Hq,Hkv", LAYOUTS, ids=IDS)
def test_attention(dtype, D, Hq, Hkv):
    rng = np.random.default_rng(D)
    say(f"{dtype}, D {D}, heads {Hq}/{Hkv}")
    b = Batch(dtype, D, Hq, Hkv, [0, 300, 17, 0, 31], [1, 4, 19, 0, 3], seed=D)
    for K in (1, 6, 40):
        lists = _random_lists(b, K, rng)
        out, lse = _attend(b, lists)
        _compare(b, lists, out, lse, name=f"prompts, lists of {K}")
    b.ctx.close()
    b = Batch(dtype, D, Hq, Hkv, [0, 15, 16, 2000, -1, 333], [1] * 6, seed=D + 1)
    for K in (3, 130):
        lists = _random_lists(b, K, rng)
        lists[3, 0, :min(K, 126)] = np.arange(126)[::-1][:K]
        out, lse = _attend(b, lists, ragged=False)
        _compare(b, lists, out, lse, name=f"a step, lists of {K}")
    assert b.ctx.sparse_workspace_bytes(6, 130) > 0           # (parts of lists that are added up)
    b.ctx.close()


@pytest.mark.parametrize("B,K", [(1, 700), (3, 300), (40, 300), (700, 9)])
def test_lists_of_many_lengths_and_parts(B, K):
    """One part and up to 64, rounds of more than 64 entries per wavefront, tokens by the hundred."""
    rng = np.random.default_rng(B)
    b = Batch("bf16", 128, 8, 1, rng.integers(0, 12000 if B < 10 else 600, B), np.ones(B), seed=B)
    say(f"{B} tokens, lists of {K}")
    lists = _random_lists(b, K, rng, order=B > 3)
    out, lse = _attend(b, lists, ragged=False)
    _compare(b, lists, out, lse, name="decode")
    assert torch.equal(out, _attend(b, lists, ragged=False)[0])
    b.ctx.close()


def _of_prompts(b: Batch):
    """Tokens at the edges of sequences and groups, and every 37th."""
    ends = np.cumsum(b.new)
    edges = {t for e in ends for t in (e - 1, e, e + 1, e - 31, e + 16, e + 31, e + 32)} | set(range(0, b.T, 37)) | {0, 1, 15, 16, 31, 32, 33}
    return sorted(t for t in edges if 0 <= t < b.T)


GROUPS = [(128, 16, 2, [100, 0, 2600]), (128, 5, 1, [2100, 2050]), (128, 3, 3, [1400]), (128, 16, 1, [4200]), (128, 12, 4, [1030]), (72, 14, 2, [3700]), (64, 8, 8, [40, 1200]),
          (96, 6, 2, [2800]), (160, 9, 1, [3400]), (216, 4, 2, [1300]), (256, 8, 1, [2100])]


@pytest.mark.parametrize("D,Hq,Hkv,new", GROUPS, ids=[f"d{a[0]}-{a[1]}x{a[2]}" for a in GROUPS])
def test_many_tokens_of_prompts(D, Hq, Hkv, new):
    """The kernel that shares the blocks of neighbouring tokens (524288 channels of K/V rows on 256 CUs): lists in any order with entries that hold no keys; lists that agree, as
    those of real prompts do; tails that nobody has written."""
    rng = np.random.default_rng(D)
    say(f"D {D}, heads {Hq}/{Hkv}: {new} tokens")
    b = Batch("bf16", D, Hq, Hkv, [17 + 100 * i for i in range(len(new))], new, seed=D)
    assert b.T * Hkv * D >= 2048 * 256
    some = _of_prompts(b)
    lists = _random_lists(b, 7, rng)
    out, lse = _attend(b, lists)
    _compare(b, lists, out, lse, name="lists in any order", tokens=some, rounded_weights=True)
    assert torch.equal(out, _attend(b, lists)[0])
    lists[:] = -1
    for t in range(b.T):                                                    # the first block, the last two, and four that 64 tokens agree on but for one
        n = b.pos[t] // 16 + 1
        for g in range(Hkv):
            r = np.random.default_rng((t // 64, g))
            mine = sorted({0, n - 1, max(n - 2, 0)} | set(r.choice(max(n, 4), 3).tolist()) | {int(rng.integers(n))})
            lists[t, g, :len(mine)] = mine
    out, lse = _attend(b, lists)
    _compare(b, lists, out, lse, name="lists that agree", tokens=some, rounded_weights=True)
    b.ctx.close()


def test_many_tokens_of_prompts_and_values_that_are_not_finite():
    """In the blocks that tokens side by side do not share: an infinite value and an undefined key reach the rows that list them alone; blocks that are listed twice; rows behind the
    last sequence; queries as slices of wider rows; a scale of its own."""
    rng = np.random.default_rng(1)
    b = Batch("bf16", 128, 16, 2, [64, 640], [900, 1200], seed=5, scale=0.2)
    lists = _random_lists(b, 5, rng, order=False)
    lists[1000, 0] = [3, 5, 3, 0, -1]                                       # (twice: its group goes the long way)
    some = sorted(set(_of_prompts(b)) | set(range(990, 1030)))
    wide = torch.full((b.T + 5, 24, 128), float("nan"), dtype=b.dt, device="cuda")
    wide[:b.T, 4:20] = b.q.cuda()
    padded = np.concatenate([lists, np.zeros((5, 2, 5), np.int32)])
    out, lse = _attend(b, padded, q=wide[:, 4:20], pad=5)
    _compare(b, lists, out, lse, name="a block twice", tokens=some, rounded_weights=True)
    assert out[b.T:].isnan().all() and lse[b.T:].isnan().all()
    again, _ = _attend(b, padded, q=wide[:, 4:20], pad=5, with_lse=False)
    assert torch.equal(again[:b.T], out[:b.T])
    lists[1000, 0, 2] = 9
    inf_block, nan_block = int(b.table[1, 4]), int(b.table[1, 11])
    b.vals[inf_block, 0, 3, 7] = float("inf")
    b.keys[nan_block, 1, 5, 2] = float("nan")
    b.upload()
    got, got_lse = _attend(b, lists)
    second = b.seq == 1
    has_inf, has_nan = (lists[:, 0] == 4).any(1) & second, (lists[:, 1] == 11).any(1) & second
    assert has_inf.any() and (~has_inf & second).any() and has_nan.any()
    o = got.float().cpu().numpy()
    assert np.isposinf(o[has_inf][:, :8, 7]).all() and np.isfinite(np.delete(o[has_inf][:, :8], 7, 2)).all()
    assert np.isnan(o[has_nan][:, 8:]).all()
    assert np.isfinite(o[~has_inf][:, :8]).all() and np.isfinite(o[~has_nan][:, 8:]).all()
    clean = [t for t in some if not has_inf[t] and not has_nan[t]]
    _compare(b, lists, got, got_lse, name="beside values that are not finite", tokens=clean, rounded_weights=True)
    b.ctx.close()


def test_rows_that_are_left_alone_strides_and_scales():
    """Rows behind the last sequence; queries as slices of wider rows; no log-sum-exp; a scale of its own; a workspace of the caller's."""
    rng = np.random.default_rng(8)
    b = Batch("bf16", 64, 8, 2, [40, 0], [3, 18], seed=8, scale=0.3)
    lists = _random_lists(b, 5, rng)
    padded = np.concatenate([lists, np.zeros((4, 2, 5), np.int32)])
    wide = torch.full((b.T + 4, 12, 64), float("nan"), dtype=b.dt, device="cuda")
    wide[:b.T, :8] = b.q.cuda()
    ws = torch.full((b.ctx.sparse_workspace_bytes(b.T + 4, 5) + 64,), 255, dtype=torch.uint8, device="cuda")
    out, lse = _attend(b, padded, q=wide[:, :8], pad=4, workspace=ws)
    _compare(b, lists, out, lse, name="strided")
    assert out[b.T:].isnan().all() and lse[b.T:].isnan().all()
    again, _ = _attend(b, padded, q=wide[:, :8], pad=4, with_lse=False)
    assert torch.equal(again[:b.T], out[:b.T])
    summary, codes, exps = _all_summarised(b)
    got = torch.full((b.T + 4, 2, 2), -7, dtype=torch.int32, device="cuda")
    b.ctx.block_select(wide[:, :8], summary, b.dev["ctx_before"], b.dev["block_table"], got, int(b.total.max()), keep_first=0, cu_q=b.dev["cu_q"])
    assert (got[b.T:] == -7).all() and np.array_equal(got[:b.T].cpu().numpy(), _expected_lists(b, codes, exps, 2, 0, 1))
    # (parts of lists: one token of two)
    b2 = Batch("f32", 64, 4, 2, [4000], [1], seed=1)
    lists = np.concatenate([_random_lists(b2, 200, rng), np.zeros((1, 2, 200), np.int32)])
    out, lse = _attend(b2, lists, q=torch.cat([b2.q, b2.q]), pad=1)
    _compare(b2, lists, out, lse, name="parts behind the last sequence")
    assert out[1:].isnan().all() and lse[1:].isnan().all()
    b.ctx.close()
    b2.ctx.close()


def test_values_that_are_not_finite():
    """An infinite or undefined value or key reaches the rows whose lists hold it and no other; large scores of either sign; a block that is listed twice."""
    for dtype in ("bf16", "f32"):
        b = Batch(dtype, 64, 4, 2, [100, 100, 100], [1, 1, 1], seed=2)
        b.vals[b.table[0, 2], 0, 7, 9] = float("inf")
        b.vals[b.table[1, 6], 1, 4, 3] = float("nan")           # slot 4 of the last block: the newest token
        b.keys[b.table[2, 1], 0, 0, 0] = float("nan")
        b.upload()
        lists = np.tile(np.array([0, 2, 4, 6], np.int32), (3, 2, 1))
        out, lse = _attend(b, lists, ragged=False)
        o = out.float().cpu().numpy()
        assert np.isposinf(o[0, :2, 9]).all() and np.isfinite(np.delete(o[0, :2], 9, 1)).all() and np.isfinite(o[0, 2:]).all()
        assert np.isnan(o[1, 2:, 3]).all() and np.isfinite(np.delete(o[1, 2:], 3, 1)).all() and np.isfinite(o[1, :2]).all()
        assert np.isfinite(o[2]).all() and torch.isfinite(lse).all()
        lists[:] = [1, 3, 5, -1]
        out, lse = _attend(b, lists, ragged=False)
        o = out.float().cpu().numpy()
        assert np.isfinite(o[:2]).all() and np.isnan(o[2, :2]).all() and np.isfinite(o[2, 2:]).all()
        b.ctx.close()
        b = Batch(dtype, 64, 4, 2, [200], [1], seed=3)
        b.q *= 30
        b.keys *= 30
        b.upload()
        lists = np.tile(np.array([7, 0, 3, 12, 5], np.int32), (1, 2, 1))
        _compare(b, lists, *_attend(b, lists, ragged=False), name="large scores")
        twice = np.tile(np.array([7, 0, 7, 12, 5], np.int32), (1, 2, 1))
        _compare(b, twice, *_attend(b, twice, ragged=False), name="a block twice")
        b.ctx.close()


# ---- together -------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype,D,Hq,Hkv", [("bf16", 128, 16, 2), ("f32", 64, 4, 2)])
def test_a_prompt_and_a_decode_loop(dtype, D, Hq, Hkv):
    """Rotate and append, summarise, select, attend: a prompt in two chunks, then steps that fill blocks.  While there are no more blocks than entries the result is
    dense attention's; afterwards the definition's on the cache as it is."""
    from paper_2504_18154_amd import binding
    rng = np.random.default_rng(6)
    model = wl.ModelShape("loop", Hq, Hkv, D, 1, dtype)
    lens = np.array([70, 33, 150])
    cap = lens + 24
    table, nb = wl.make_block_table(rng, cap.astype(np.int64))
    ctx = binding.Context(Hq, Hkv, D, nb, dtype, 3, table.shape[1])
    kc, vc = ctx.new_cache()
    summary = ctx.new_summary()
    rope = binding.Rope(10000.0 ** (-torch.arange(D // 2, dtype=torch.float64, device="cuda") * 2 / D))
    bt, K = dev_i32(table), 6
    before = np.zeros(3, dtype=np.int64)
    steps = [lens // 2, lens - lens // 2] + [np.ones(3, dtype=np.int64)] * 20

    class View(Batch):
        def __init__(self):
            pass

    for i, new in enumerate(steps):
        T, cu = int(new.sum()), wl.cu_from_lengths(new)
        q, k, v = (wl.randn((T, h, D), dtype, 100 + 3 * i + n).cuda() for n, h in enumerate((Hq, Hkv, Hkv)))
        one = i >= 2
        cu_d, before_d = dev_i32(cu), dev_i32(before)
        ctx.kv_append_rope(kc, vc, k, v, cu_d, before_d, bt, rope, q=q, q_out=q, max_new_len=1 if one else None)
        ctx.kv_summary(kc, summary, cu_d, before_d, bt, T, max_new_len=1 if one else None)
        lists = torch.full((T, Hkv, K), -7, dtype=torch.int32, device="cuda")
        out, lse = torch.empty_like(q), torch.empty(T, Hq, device="cuda")
        cu_or = None if one else cu_d
        ctx.block_select(q, summary, before_d, bt, lists, int((before + new).max()), keep_first=1, keep_last=2, cu_q=cu_or)
        ctx.attn_sparse(q, kc, vc, before_d, bt, lists, out, lse=lse, cu_q=cu_or)
        b = View()
        b.dtype, b.D, b.Hq, b.Hkv, b.G, b.dt, b.scale = dtype, D, Hq, Hkv, Hq // Hkv, ctx.torch_dtype, 1 / math.sqrt(D)
        b.q, b.T, b.table = q.cpu(), T, table
        b.keys, b.vals = ctx.k_logical(kc).cpu(), ctx.v_logical(vc).cpu()
        b.seq, b.pos = np.repeat(np.arange(3), new), np.concatenate([x + np.arange(n) for x, n in zip(before, new)])
        codes, exps = _summary_host(ctx.layout, summary)
        want = np.full((T, Hkv, K), -1)
        for t in range(T):
            n = b.pos[t] // 16 + 1
            for g in range(Hkv):
                pairs = [so.summarise(b.keys[table[b.seq[t], j], g].float().numpy()) for j in range(n - 1)] if n > K else []
                s = so.scores(b.q[t, g * b.G:(g + 1) * b.G].float().numpy(), np.stack([c for c, _ in pairs]), np.array([e for _, e in pairs])) if pairs else np.zeros(0)
                lst = so.choose(s, n, K, 1, 2)
                want[t, g, :len(lst)] = lst
        assert np.array_equal(lists.cpu().numpy(), want), i
        _compare(b, want, out, lse, name=f"step {i}")
        before = before + new
        if one:
            dense, dense_lse = torch.empty_like(q), torch.empty_like(lse)
            ctx.attn_decode(q, kc, vc, bt, dev_i32(before), dense, int(before.max()), dense_lse)
            few = np.flatnonzero(before <= 16 * K)
            assert len(few) and (dense[few].float() - out[few].float()).abs().max() <= (2e-2 if dtype == "bf16" else 1e-5)
    ctx.close()


def test_recorded_into_a_graph_on_another_stream():
    """The four calls as one graph, replayed with new inputs between eager work of the same shape: every replay the same bits as the eager calls."""
    from paper_2504_18154_amd import binding
    Hq, Hkv, D, B, K = 8, 2, 128, 4, 5
    lens = np.array([200, 15, 1000, 79])
    table, nb = wl.make_block_table(np.random.default_rng(1), (lens + 8).astype(np.int64))
    ctx = binding.Context(Hq, Hkv, D, nb, "bf16", B, table.shape[1])
    g = torch.Generator(device="cuda").manual_seed(5)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)
    pools = [rand(nb * Hkv * 16 * D) for _ in range(2)]
    rope = binding.Rope(10000.0 ** (-torch.arange(64, dtype=torch.float64, device="cuda") / 64))
    bt, cu, before = dev_i32(table), dev_i32(np.arange(B + 1)), dev_i32(lens)
    summary = ctx.new_summary()
    ctx.kv_summary(pools[0], summary, dev_i32(wl.cu_from_lengths(lens)), dev_i32(np.zeros(B)), bt, int(lens.sum()))
    q, k, v = rand(B, Hq, D), rand(B, Hkv, D), rand(B, Hkv, D)

    def step(kc, vc, summ, lists, q_out, out, lse, ws1=None, ws2=None):
        ctx.kv_append_rope(kc, vc, k, v, cu, before, bt, rope, q=q, q_out=q_out, max_new_len=1)
        ctx.kv_summary(kc, summ, cu, before, bt, B, max_new_len=1)
        ctx.block_select(q_out, summ, before, bt, lists, 1008, keep_last=2, workspace=ws1)
        ctx.attn_sparse(q_out, kc, vc, before, bt, lists, out, lse=lse, workspace=ws2)

    def buffers():
        return (pools[0].clone(), pools[1].clone(), summary.clone(), torch.zeros(B, Hkv, K, dtype=torch.int32, device="cuda"), torch.zeros_like(q), torch.zeros_like(q),
                torch.zeros(B, Hq, device="cuda"))

    side, mine, eager = torch.cuda.Stream(), buffers(), buffers()
    ws = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in (binding.select_workspace_bytes(ctx.layout, B, 1008), ctx.sparse_workspace_bytes(B, K))]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(*mine, *ws)
    for i in range(4):
        for t in (q, k, v):
            t.copy_(rand(*t.shape))
        step(*eager)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(mine, eager):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), i
        before += 1
    ctx.close()


def test_what_the_binding_takes_and_what_it_refuses():
    """Bounds of any integer type go the longer way with the same result; tensors of another type, size, device or layout are refused by name."""
    b = Batch("bf16", 64, 4, 2, [300, 77], [1, 1], seed=4)
    summary, _, _ = _all_summarised(b)
    q, lists, K = b.q.cuda(), torch.zeros(2, 2, 4, dtype=torch.int32, device="cuda"), 4
    d, out, lse = b.dev, torch.zeros(2, 4, 64, dtype=b.dt, device="cuda"), torch.zeros(2, 4, device="cuda")
    sel = dict(q=q, summary=summary, ctx_before=d["ctx_before"], block_table=d["block_table"], blocks=lists, max_ctx_len=301, cu_q=None, workspace=None)
    b.ctx.block_select(**sel)
    want = lists.clone()
    for bound in (np.int32(301), np.int64(301), torch.tensor(301)):
        lists.zero_()
        b.ctx.block_select(**{**sel, "max_ctx_len": bound, "keep_first": np.int64(1)})
        assert torch.equal(lists, want)
    att = dict(q=q, k_cache=b.kc, v_cache=b.vc, ctx_before=d["ctx_before"], block_table=d["block_table"], blocks=lists, out=out, lse=lse, cu_q=None, workspace=None)
    b.ctx.attn_sparse(**att)
    summ = dict(k_cache=b.kc, summary=summary, cu_q=d["cu_q"], ctx_before=d["ctx_before"], block_table=d["block_table"], T=2)
    before = summary.clone()
    b.ctx.kv_summary(**{**summ, "T": np.int32(2), "max_new_len": np.int64(1)})
    assert torch.equal(summary, before)
    small = torch.zeros(8, dtype=torch.uint8, device="cuda")
    wrong = [(b.ctx.block_select, sel, {"q": [q.float(), q.cpu(), q[:, :2], q[..., :32], q[:1]], "summary": [summary[:-99], summary.to(torch.uint8), summary.cpu()],
                                        "ctx_before": [d["ctx_before"].long(), d["ctx_before"].cpu(), torch.stack([d["ctx_before"]] * 2, 1)[:, 0]],
                                        "block_table": [d["block_table"][0], d["block_table"][:1], d["block_table"].long(), d["block_table"][:, 1:]],
                                        "blocks": [lists[:1], lists[:, :1], lists.long(), lists[..., ::2]], "cu_q": [d["cu_q"][:2], d["cu_q"].long()], "workspace": [small.cpu()]}),
             (b.ctx.attn_sparse, att, {"q": [q.float()], "k_cache": [b.kc[:-1], b.kc.float(), b.kc.cpu()], "v_cache": [b.vc[:-1]], "blocks": [lists[0], lists.cpu()],
                                       "out": [out[:1], out.float(), out.transpose(0, 1)], "lse": [lse[:1], lse.double(), lse.cpu()], "cu_q": [d["cu_q"].cpu()]}),
             (b.ctx.kv_summary, summ, {"k_cache": [b.kc[:-1], b.kc.float()], "summary": [summary[:-99]], "cu_q": [d["cu_q"][:2]], "block_table": [d["block_table"].cpu()]})]
    for call, good, changes in wrong:
        for name, values in changes.items():
            for value in values:
                with pytest.raises(ValueError):
                    call(**{**good, name: value})
    from paper_2504_18154_amd import binding
    for call, change in ((b.ctx.block_select, {**sel, "workspace": small}), (b.ctx.block_select, {**sel, "keep_last": 0}), (b.ctx.block_select, {**sel, "max_ctx_len": 0}),
                         (b.ctx.block_select, {**sel, "max_ctx_len": 1 << 20})):
        with pytest.raises(binding.EcoserveError):
            call(**change)
    b.ctx.close()
