"""Rotated append, block summaries, block selection and sparse attention over the paged cache, as measurable cases.

Four operators of one path.  A serving program rotates Q and K by their positions while K and V join the paged cache,
summarises the cache blocks that became full, lets every query choose the blocks it will read by a cheap score over the
summaries, and attends to the chosen blocks alone.  A case is one call of one of them on one layer.

Cache layout (bs = 16 tokens a block, x = 16 / sizeof(E) elements a unit):
  K [blocks][Hkv][D / x][bs][x]    V [blocks][Hkv][D][bs]
Summaries, one flat int8 buffer: codes [blocks][Hkv][2][Dp] (largest, smallest key per channel; Dp = D rounded up to 32,
zeros behind D), then exponents [blocks][Hkv]; a code c stands for c 2^e.  Lengths follow from the case (`len_seed`),
everything else from prepare()'s seed.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

BS = 16
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
ES = {"bf16": 2, "f32": 4}
NOT_FINITE = 127  # the exponent of a block that holds a NaN or an infinity


# ---- cases --------------------------------------------------------------------------------------


def _case(name, op, heads, B, pre, new, **kw):
    """B sequences with pre[0]..pre[1] cached tokens that bring new[0]..new[1] new ones; new = (1, 1): a decode step."""
    c = {"name": name, "op": op, "Hq": heads[0], "Hkv": heads[1], "D": 128, "dtype": "bf16", "B": B, "pre_lo": pre[0], "pre_hi": pre[1],
         "lo": new[0], "hi": new[1], "len_seed": 1}
    if op == "rope":
        c.update(rotary=0, adjacent=False, axes=1, fused_rows=False)
    if op in ("select", "sparse"):
        c.update(K=64, keep_first=1, keep_last=4)
    c.update(kw)
    return c


def listed():
    return [
        # a decode step of 64 conversations: one token each is rotated and appended; launch latency
        _case("rope_step", "rope", (40, 8), 64, (100, 2000), (1, 1)),
        # prompts with an image between text: three position coordinates per token, rows of a fused projection
        _case("rope_image_chunk", "rope", (64, 8), 3, (0, 500), (200, 1500), axes=3, fused_rows=True, len_seed=2),
        # a small fp32 model that rotates half of each head, neighbouring elements paired
        _case("rope_f32_partial", "rope", (4, 2), 16, (0, 90), (1, 700), D=64, dtype="f32", rotary=32, adjacent=True, len_seed=3),
        # the benchmark's prefill burst: 8 prompts of 8192 tokens; memory
        _case("rope_burst", "rope", (64, 8), 8, (0, 0), (8192, 8192)),
        # a decode step: about a sixteenth of the sequences fill a block
        _case("summary_step", "summary", (64, 8), 256, (1024, 4096), (1, 1), len_seed=4),
        # behind the prefill burst: every block of 8 prompts
        _case("summary_burst", "summary", (64, 8), 8, (0, 0), (8192, 8192)),
        # one long document, one token: latency
        _case("select_one", "select", (40, 8), 1, (20000, 20000), (1, 1)),
        # 32 long contexts in a decode step: reading the summaries
        _case("select_long", "select", (64, 8), 32, (16384, 131000), (1, 1), K=128, len_seed=5),
        # chunks of two long prompts: every token chooses for itself; products
        _case("select_chunk", "select", (64, 8), 2, (16000, 32000), (300, 600), len_seed=6),
        # one long document, one token: latency
        _case("sparse_one", "sparse", (40, 8), 1, (20000, 20000), (1, 1)),
        # 32 long contexts in a decode step: reading 128 blocks of each, K/V head by K/V head
        _case("sparse_long", "sparse", (64, 8), 32, (16384, 131000), (1, 1), K=128, len_seed=5),
        # chunks of two long prompts, 64 blocks per token
        _case("sparse_chunk", "sparse", (64, 8), 2, (16000, 32000), (300, 600), len_seed=6),
    ]


_LAYOUTS = (((40, 8), 128, "bf16"), ((64, 8), 128, "bf16"), ((52, 52), 128, "bf16"), ((8, 1), 128, "bf16"), ((5, 1), 128, "bf16"),
            ((32, 8), 64, "bf16"), ((8, 8), 80, "bf16"), ((8, 1), 256, "bf16"), ((4, 2), 64, "f32"), ((6, 3), 128, "f32"))


def _log(rng: random.Random, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng: random.Random):
    op = rng.choice(("rope", "summary", "select", "sparse"))
    heads, D, dtype = rng.choice(_LAYOUTS)
    step = rng.random() < 0.5
    kw = {"D": D, "dtype": dtype, "len_seed": rng.randrange(1, 1 << 30)}
    row = heads[1] * D * ES[dtype]                        # bytes of a token's K row
    if op in ("rope", "summary"):
        B = _log(rng, 1, 512 if step else 64)
        # at most 1.3 GB of new rows (Q, K, V), as in the largest listed case
        most = max(2, int(1.3e9 / (row * (2 + heads[0] / heads[1]) * B)))
        hi = 1 if step else _log(rng, 2, min(16384, most))
        lo = hi if step else max(1, hi // rng.choice((1, 2, 8, 64)))
        pre = _log(rng, 1, max(2, min(8192, int(2e8 / (row * B))))) if step or rng.random() < 0.5 else 0
        if op == "rope":
            kw.update(rotary=rng.choice((0, 0, 32)), adjacent=rng.random() < 0.3, axes=rng.choice((1, 1, 2, 3)), fused_rows=rng.random() < 0.4)
        c = _case("", op, heads, B, (rng.choice((0, pre // 2, pre)), pre), (lo, hi), **kw)
        while op == "summary" and len(_filled(*_lengths(c))[0]) == 0:      # (calls that fill no block have nothing to do)
            c.update(pre_lo=0, pre_hi=max(c["pre_hi"], 31), len_seed=c["len_seed"] + 1)
    else:
        B = _log(rng, 1, 128 if step else 4)
        # at most 2.4 million tokens of the largest listed layout in the cache
        pre = _log(rng, 512, min(131000, int(4.8e9 / (row * B))))
        hi = 1 if step else _log(rng, 2, 500)
        # (fewer blocks than there are: with all of them chosen there is nothing to select)
        K = _log(rng, 2, max(4, min(200 if step else 64, pre // 96)))
        # chunks: the rows times what they score, and what they read, kept to the listed cases' products
        while not step and B * hi * heads[0] * (pre + hi) / BS * D > 6e9:
            hi = max(2, hi * 2 // 3)
        while not step and B * hi * heads[1] * K * D * ES[dtype] > 1e8:
            K = max(2, K * 2 // 3)
            hi = max(2, hi * 2 // 3)
        keep = rng.choice([k for k in ((0, 1), (1, 2), (1, 4), (2, 6)) if sum(k) < K])
        kw.update(K=K, keep_first=keep[0], keep_last=keep[1])
        c = _case("", op, heads, B, (rng.choice((pre // 4, pre // 2, pre)), pre), (hi if step else max(1, hi // rng.choice((1, 2, 8))), hi), **kw)
    del c["name"]
    return c


def _lengths(c):
    """Per sequence: (tokens cached before the call, new tokens)."""
    rng = np.random.Generator(np.random.Philox(c["len_seed"]))
    before = rng.integers(c["pre_lo"], c["pre_hi"] + 1, size=c["B"])
    return before.astype(np.int64), rng.integers(c["lo"], c["hi"] + 1, size=c["B"]).astype(np.int64)


def _positions_of(c):
    """Per new token: (its sequence, its position)."""
    before, new = _lengths(c)
    seq = np.repeat(np.arange(c["B"]), new)
    first = np.concatenate([[0], np.cumsum(new)])[:-1]
    return seq, before[seq] + np.arange(len(seq)) - first[seq]


def _filled(before, new):
    """(sequence, logical block) of every block that the new tokens fill."""
    seq, blk = [], []
    for b, (s, n) in enumerate(zip(before, new)):
        j = np.arange(s // BS, (s + n) // BS)
        seq.append(np.full(len(j), b))
        blk.append(j)
    return np.concatenate(seq), np.concatenate(blk)


def _padded(D):
    return (D + 31) // 32 * 32


def work(c):
    before, new = _lengths(c)
    es, T, D, Hq, Hkv = ES[c["dtype"]], int(new.sum()), c["D"], c["Hq"], c["Hkv"]
    record = 2 * _padded(D) + 1
    blocks = (before + new + BS - 1) // BS
    if c["op"] == "rope":
        R = c["rotary"] or D
        return {"bytes": 2 * T * (Hq + 2 * Hkv) * D * es + 8 * T, "flops": 3 * T * (Hq + Hkv) * R}
    if c["op"] == "summary":
        n = len(_filled(before, new)[0]) * Hkv
        return {"bytes": n * (BS * D * es + record), "flops": 2 * n * BS * D}
    _, pos = _positions_of(c)
    if c["op"] == "select":
        return {"bytes": T * Hq * D * es + int(blocks.sum()) * (Hkv * record + 4) + T * Hkv * c["K"] * 4,
                "flops": int((pos // BS + 1).sum()) * Hq * 4 * D}
    chosen = np.minimum(pos // BS + 1, c["K"])
    read = int(np.minimum(blocks, new * c["K"]).sum()) * Hkv
    return {"bytes": read * 2 * BS * D * es + 2 * T * Hq * D * es + T * Hkv * c["K"] * 4 + T * Hq * 4,
            "flops": int(chosen.sum()) * BS * Hq * 4 * D}


# ---- inputs -------------------------------------------------------------------------------------


class _Random:
    """Tensors on the GPU from a seed."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(self, shape, dtype):
        return torch.randn(shape, generator=self.g, device="cuda", dtype=dtype)

    def uniform(self, shape):
        return torch.rand(shape, generator=self.g, device="cuda")

    def whole(self, n, shape):
        return torch.randint(n, shape, generator=self.g, device="cuda", dtype=torch.int32)


def _dev(a, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(a), device="cuda").to(dtype)


def _codes(K, D):
    """Summaries of the blocks K [..., bs, D] in fp32 or wider: (codes int8 [..., 2, Dp], exponents int8 [...])."""
    top, low = K.amax(-2), K.amin(-2)
    largest = torch.maximum(top.abs(), low.abs()).amax(-1)
    fine = torch.isfinite(largest)
    f, x = torch.frexp(torch.where(fine, largest, torch.zeros_like(largest)))
    e = torch.where(f > 127 / 128, x - 6, x - 7).clamp_min(-126)
    codes = torch.zeros(*K.shape[:-2], 2, _padded(D), dtype=torch.int8, device=K.device)
    scaled = [torch.ldexp(t, -e[..., None]) for t in (top, low)]
    codes[..., 0, :D] = torch.where(fine[..., None], torch.ceil(scaled[0]), torch.zeros_like(top)).to(torch.int8)
    codes[..., 1, :D] = torch.where(fine[..., None], torch.floor(scaled[1]), torch.zeros_like(low)).to(torch.int8)
    return codes, torch.where(fine, e, torch.full_like(e, NOT_FINITE)).to(torch.int8)


def _summary_bytes(c, blocks):
    return (blocks * c["Hkv"] * (2 * _padded(c["D"]) + 1) + 15) // 16 * 16


def _summary_views(c, summary, blocks):
    """(codes [blocks, Hkv, 2, Dp], exponents [blocks, Hkv]) of a flat summary buffer."""
    n = blocks * c["Hkv"] * 2 * _padded(c["D"])
    return summary[:n].view(blocks, c["Hkv"], 2, _padded(c["D"])), summary[n:n + blocks * c["Hkv"]].view(blocks, c["Hkv"])


class State:
    pass


def prepare(c, seed):
    """What a serving program holds before the call."""
    s, r = State(), _Random(seed)
    before, new = _lengths(c)
    B, T, D, Hq, Hkv, dt = c["B"], int(new.sum()), c["D"], c["Hq"], c["Hkv"], DT[c["dtype"]]
    x = 16 // ES[c["dtype"]]
    s.c, s.before, s.new, s.T = c, before, new, T
    s.step = c["lo"] == c["hi"] == 1
    per = (before + new + BS - 1) // BS
    need = int(per.sum())
    s.blocks = need + need // 10 + 2
    # the sequences' blocks lie anywhere in the pool
    ids = torch.randperm(s.blocks, generator=r.g, device="cuda", dtype=torch.int32)[:need].cpu().numpy()
    table = np.full((B, int(per.max())), -1, dtype=np.int32)
    at = 0
    for b in range(B):
        table[b, :per[b]] = ids[at:at + per[b]]
        at += int(per[b])
    s.table, s.ctx_before = _dev(table), _dev(before)
    s.table_host = table
    s.cu_q = _dev(np.concatenate([[0], np.cumsum(new)]))
    s.seq, s.pos = (_dev(a, torch.int64) for a in _positions_of(c))
    s.max_new, s.max_ctx = int(new.max()), int((before + new).max())
    pool = s.blocks * Hkv * BS * D
    if c["op"] == "rope":
        rows = r.normal((T, Hq + 2 * Hkv, D), dt)
        s.q, s.k, s.v = rows[:, :Hq], rows[:, Hq:Hq + Hkv], rows[:, Hq + Hkv:]
        if not c["fused_rows"]:
            s.q, s.k, s.v = (t.contiguous() for t in (s.q, s.k, s.v))
        s.q_out = torch.empty(T, Hq, D, dtype=dt, device="cuda")
        s.kc, s.vc = torch.zeros(pool, dtype=dt, device="cuda"), torch.zeros(pool, dtype=dt, device="cuda")
        R = c["rotary"] or D
        s.rotary = R
        s.freq = 10000.0 ** (-torch.arange(R // 2, device="cuda", dtype=torch.float64) * (2.0 / R))
        # several coordinates: runs of pairs, one after the other, belong to time, height, width
        s.axis = [min(i * c["axes"] // (R // 2), c["axes"] - 1) for i in range(R // 2)]
        s.coords = None
        if c["axes"] > 1:
            s.coords = torch.stack([s.pos.to(torch.int32)] + [r.whole(100, (T,)) + s.pos.to(torch.int32) // 3 for _ in range(c["axes"] - 1)])
    elif c["op"] == "summary":
        s.kc = r.normal((pool,), dt)
        s.summary = torch.zeros(_summary_bytes(c, s.blocks), dtype=torch.int8, device="cuda")
    elif c["op"] == "select":
        s.q = r.normal((T, Hq, D), dt)
        s.summary = torch.empty(_summary_bytes(c, s.blocks), dtype=torch.int8, device="cuda")
        codes, exps = _summary_views(c, s.summary, s.blocks)
        # keys have channels of their own size and offset, and drift along a sequence
        size, offset = 0.5 + r.uniform((Hkv, 1, D)) * 1.5, r.normal((Hkv, 1, D), torch.float32) * 0.5
        for b0 in range(0, s.blocks, 8192):
            b1 = min(s.blocks, b0 + 8192)
            keys = r.normal((b1 - b0, Hkv, BS, D), torch.float32) * size + offset + r.normal((b1 - b0, Hkv, 1, D), torch.float32) * 0.3
            codes[b0:b1], exps[b0:b1] = _codes(keys.to(dt).float(), D)
        s.chosen = torch.empty(T, Hkv, c["K"], dtype=torch.int32, device="cuda")
    else:
        s.q = r.normal((T, Hq, D), dt)
        s.kc, s.vc = r.normal((pool,), dt), r.normal((pool,), dt)
        s.chosen = _some_blocks(c, s, r)
        s.out = torch.empty(T, Hq, D, dtype=dt, device="cuda")
        s.lse = torch.empty(T, Hq, device="cuda")
    s.x = x
    if own:
        from paper_2504_18154_amd import binding
        s.ctx = binding.Context(Hq, Hkv, D, s.blocks, c["dtype"], B, table.shape[1])
        if c["op"] == "rope":
            s.rope = binding.Rope(s.freq, pairing="adjacent" if c["adjacent"] else "halves", axis=s.axis if c["axes"] > 1 else None)
    return s


def _some_blocks(c, s, r):
    """Lists as selection leaves them: the first and the last blocks and others, ascending, -1 behind; tokens of one prompt that
    lie close together agree on many."""
    K, Hkv = c["K"], c["Hkv"]
    chosen = torch.full((s.T, Hkv, K), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b in range(c["B"]):
        S, most = int(s.new[b]), int(s.before[b] + s.new[b] - 1) // BS + 1
        j = torch.arange(most, device="cuda")
        taste = None
        for t0 in range(0, S, 64):
            t1 = min(S, t0 + 64)
            last = (s.pos[at + t0:at + t1] // BS)[:, None, None]
            taste = r.uniform((1, Hkv, most)) if taste is None else 0.7 * taste + 0.3 * r.uniform((1, Hkv, most))
            w = taste + 0.5 * r.uniform((t1 - t0, Hkv, most))
            w = torch.where((j < c["keep_first"]) | (j > last - c["keep_last"]), w + 10, w)
            w = torch.where(j <= last, w, torch.full_like(w, -1.0))
            top = torch.topk(w, min(K, most), dim=-1)
            idx = torch.where(top.values >= 0, top.indices, most + 1).sort(-1).values
            chosen[at + t0:at + t1, :, :idx.shape[-1]] = torch.where(idx <= most, idx, -1).to(torch.int32)
        at += S
    return chosen


# ---- the operators ------------------------------------------------------------------------------


def run(s):
    return {"rope": _rope, "summary": _summary, "select": _select, "sparse": _sparse}[s.c["op"]](s)


def _destination(s):
    """(physical block, slot) of every new token."""
    return s.table[s.seq, s.pos // BS].long(), s.pos % BS


def _rope(s):
    c = s.c
    if own:
        s.ctx.kv_append_rope(s.kc, s.vc, s.k, s.v, s.cu_q, s.ctx_before, s.table, s.rope, positions=s.coords, q=s.q, q_out=s.q_out,
                             max_new_len=s.max_new)
        return {"q": s.q_out, "k_cache": s.kc, "v_cache": s.vc}
    Hkv, D, R = c["Hkv"], c["D"], s.rotary
    if s.coords is None:
        angle = s.pos.double()[:, None] * s.freq
    else:
        angle = s.coords.double()[s.axis].t() * s.freq
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

    def turned(rows):
        out = rows.clone()
        part = rows[..., :R].float()
        if c["adjacent"]:
            a, b = part[..., 0::2], part[..., 1::2]
            out[..., 0:R:2], out[..., 1:R:2] = (a * cos - b * sin).to(out.dtype), (a * sin + b * cos).to(out.dtype)
        else:
            a, b = part[..., :R // 2], part[..., R // 2:]
            out[..., :R // 2], out[..., R // 2:R] = (a * cos - b * sin).to(out.dtype), (a * sin + b * cos).to(out.dtype)
        return out

    blk, slot = _destination(s)
    s.kc.view(s.blocks, Hkv, D // s.x, BS, s.x)[blk, :, :, slot] = turned(s.k).view(s.T, Hkv, D // s.x, s.x)
    s.vc.view(s.blocks, Hkv, D, BS)[blk, :, :, slot] = s.v
    return {"q": turned(s.q), "k_cache": s.kc, "v_cache": s.vc}


def _summary(s):
    """The codes and exponents are whole numbers and part of the interface, so they are returned as they are."""
    c = s.c
    if own:
        s.ctx.kv_summary(s.kc, s.summary, s.cu_q, s.ctx_before, s.table, s.T, max_new_len=s.max_new)
        return {"summary": s.summary}
    codes, exps = _summary_views(c, s.summary, s.blocks)
    seq, blk = _filled(s.before, s.new)
    ids = _dev(s.table_host[seq, blk], torch.int64)
    pool = s.kc.view(s.blocks, c["Hkv"], c["D"] // s.x, BS, s.x)
    for i in range(0, len(seq), 4096):
        part = ids[i:i + 4096]
        keys = pool[part].permute(0, 1, 3, 2, 4).reshape(len(part), c["Hkv"], BS, c["D"]).float()
        codes[part], exps[part] = _codes(keys, c["D"])
    return {"summary": s.summary}


def _query_codes(q):
    """Whole numbers of at most 127 and exponents (q ~ code 2^e) of each row; a row with a NaN or an infinity has zeros."""
    largest = q.abs().amax(-1)
    fine = torch.isfinite(largest)
    f, x = torch.frexp(torch.where(fine, largest, torch.zeros_like(largest)))
    e = torch.where(f > 127 / 128, x - 6, x - 7).clamp_min(-126)
    codes = torch.round(torch.ldexp(q, -e[..., None]))
    return torch.where(fine[..., None], codes, torch.zeros_like(codes)), torch.where(fine, e, torch.zeros_like(e))


def _select(s):
    c = s.c
    if own:
        s.ctx.block_select(s.q, s.summary, s.ctx_before, s.table, s.chosen, s.max_ctx, keep_first=c["keep_first"], keep_last=c["keep_last"],
                           cu_q=None if s.step else s.cu_q)
        return {"blocks": s.chosen}
    Hkv, D, K = c["Hkv"], c["D"], c["K"]
    G = c["Hq"] // Hkv
    codes, exps = _summary_views(c, s.summary, s.blocks)
    s.chosen.fill_(-1)
    at = 0
    for b in range(c["B"]):
        S, full = int(s.new[b]), int(s.before[b] + s.new[b]) // BS
        most = int(s.before[b] + s.new[b] - 1) // BS + 1
        ids = s.table[b, :full].long()
        sides = codes[ids][..., :D].float().permute(1, 2, 3, 0).contiguous()            # [Hkv, 2, D, full]
        e = exps[ids].t().float()                                                       # [Hkv, full]
        step = max(1, min(S, (1 << 27) // max(1, most * c["Hq"])))
        for t0 in range(0, S, step):
            t1 = min(S, t0 + step)
            n = t1 - t0
            qc, qe = _query_codes(s.q[at + t0:at + t1].float().view(n, Hkv, G, D))
            qc = qc.permute(1, 0, 2, 3).reshape(Hkv, n * G, D)
            bound = torch.matmul(qc.clamp_min(0), sides[:, 0]) + torch.matmul(qc.clamp_max(0), sides[:, 1])
            score = torch.ldexp(bound.view(Hkv, n, G, full), qe.permute(1, 0, 2)[..., None] + e[:, None, None]).amax(2)
            score = torch.where((e == NOT_FINITE)[:, None], torch.full_like(score, math.inf), score)
            score = torch.nn.functional.pad(score, (0, most - full))
            j, last = torch.arange(most, device="cuda"), (s.pos[at + t0:at + t1] // BS)[None, :, None]
            kept = (j < c["keep_first"]) | (j > last - c["keep_last"])
            # kept blocks first, then by score; equal ones in their order; blocks behind the token never
            order = torch.sort(torch.where(j > last, torch.full_like(score, -math.inf), score), dim=-1, descending=True, stable=True).indices
            rank = torch.where(j > last, 2, torch.where(kept, 0, 1)).expand_as(score).gather(-1, order)
            order = order.gather(-1, torch.sort(rank, dim=-1, stable=True).indices)[..., :K]
            idx = torch.where(order <= last, order, most + 1).sort(-1).values
            s.chosen[at + t0:at + t1, :, :idx.shape[-1]] = torch.where(idx <= most, idx, -1).to(torch.int32).permute(1, 0, 2)
        at += S
    return {"blocks": s.chosen}


def _sparse(s):
    c = s.c
    if own:
        s.ctx.attn_sparse(s.q, s.kc, s.vc, s.ctx_before, s.table, s.chosen, s.out, lse=s.lse, cu_q=None if s.step else s.cu_q)
        return {"out": s.out, "lse": s.lse}
    Hq, Hkv, D, K = c["Hq"], c["Hkv"], c["D"], c["K"]
    G = Hq // Hkv
    kp, vp = s.kc.view(s.blocks, Hkv, D // s.x, BS, s.x), s.vc.view(s.blocks, Hkv, D, BS)
    heads = torch.arange(Hkv, device="cuda")[None, :, None]
    step = max(1, (1 << 26) // (Hkv * K * BS * D))
    for t0 in range(0, s.T, step):
        t1 = min(s.T, t0 + step)
        n = t1 - t0
        idx = s.chosen[t0:t1].long()
        ids = s.table[s.seq[t0:t1, None, None], idx.clamp_min(0)].long()
        keys = kp[ids, heads].permute(0, 1, 2, 4, 3, 5).reshape(n * Hkv, K * BS, D).float()
        vals = vp[ids, heads].permute(0, 1, 2, 4, 3).reshape(n * Hkv, K * BS, D).float()
        at = idx[..., None] * BS + torch.arange(BS, device="cuda")
        there = ((idx >= 0)[..., None] & (at <= s.pos[t0:t1, None, None, None])).view(n * Hkv, 1, K * BS)
        score = torch.matmul(s.q[t0:t1].float().view(n * Hkv, G, D), keys.transpose(1, 2).contiguous()) * D ** -0.5
        score = torch.where(there, score, torch.full_like(score, -math.inf))
        top = score.amax(-1, keepdim=True)
        w = torch.exp(score - top)
        total = w.sum(-1, keepdim=True)
        s.out[t0:t1] = (torch.matmul(w, vals) / total).to(s.out.dtype).view(n, Hq, D)
        s.lse[t0:t1] = (top + torch.log(total)).view(n, Hq)
    return {"out": s.out, "lse": s.lse}


# ---- the definitions in 64 bits -----------------------------------------------------------------


def exact(c, seed):
    """From the definitions, one sequence or token at a time, on the same inputs."""
    if own:
        raise RuntimeError("the definition needs none of the kernels")
    w = work(c)
    tokens = int(_lengths(c)[1].sum())
    if w["flops"] > 1.5e11 or (c["op"] in ("select", "sparse") and tokens * c["Hkv"] > 25000):
        return None
    s = prepare(c, seed)
    return {"rope": _exact_rope, "summary": _exact_summary, "select": _exact_select, "sparse": _exact_sparse}[c["op"]](c, s)


def _exact_rope(c, s):
    """Pairs as complex numbers, turned by multiplication with exp(i theta)."""
    D, Hkv, R = c["D"], c["Hkv"], s.rotary
    where = s.pos[None].expand(c["axes"], -1) if s.coords is None else s.coords
    theta = torch.stack([where[s.axis[i]].double() * s.freq[i] for i in range(R // 2)], dim=1)
    turn = torch.polar(torch.ones_like(theta), theta)[:, None]
    first = torch.arange(R // 2, device="cuda") * (2 if c["adjacent"] else 1)
    second = first + (1 if c["adjacent"] else R // 2)

    def turned(rows):
        out = rows.double().clone()
        z = torch.complex(out[..., first], out[..., second]) * turn
        out[..., first], out[..., second] = z.real, z.imag
        return out

    kc, vc = s.kc.double(), s.vc.double()
    blk = s.table[s.seq, torch.div(s.pos, BS, rounding_mode="floor")].long()
    slot, g, d = s.pos % BS, torch.arange(Hkv, device="cuda")[:, None], torch.arange(D, device="cuda")[None]
    piece = (blk[:, None, None] * Hkv + g) * (BS * D)
    kc[piece + (d // s.x) * (BS * s.x) + slot[:, None, None] * s.x + d % s.x] = turned(s.k)
    vc[piece + d * BS + slot[:, None, None]] = s.v.double()
    return {"q": turned(s.q), "k_cache": kc, "v_cache": vc}


def _exact_summary(c, s):
    """Block by block: the exponent by counting up, the codes by division."""
    D, Hkv, Dp = c["D"], c["Hkv"], _padded(c["D"])
    out = s.summary.cpu().numpy().copy()
    seq, blk = _filled(s.before, s.new)
    if len(seq) > 20000:
        return None
    pool = s.kc.view(s.blocks, Hkv, D // s.x, BS, s.x)
    tail = s.blocks * Hkv * 2 * Dp
    for i in range(0, len(seq), 1024):
        ids = s.table_host[seq[i:i + 1024], blk[i:i + 1024]].astype(np.int64)
        keys = pool[torch.as_tensor(ids, device="cuda")].double().cpu().numpy()          # [n, Hkv, D / x, BS, x]
        top, low = keys.max(3).reshape(len(ids), Hkv, D), keys.min(3).reshape(len(ids), Hkv, D)
        size = np.maximum(np.abs(top), np.abs(low)).max(-1)
        e = np.full(size.shape, -126)
        while (short := size > 127.0 * 2.0 ** e).any():
            e[short] += 1
        for n, p in enumerate(ids):
            for g in range(Hkv):
                at = (p * Hkv + g) * 2 * Dp
                out[at:at + D] = np.ceil(top[n, g] / 2.0 ** e[n, g])
                out[at + Dp:at + Dp + D] = np.floor(low[n, g] / 2.0 ** e[n, g])
                out[tail + p * Hkv + g] = e[n, g]
    return {"summary": torch.as_tensor(out)}


def _exact_select(c, s):
    """Token by token, in double precision, ordered by a sort over (kept, score, index)."""
    Hkv, D, K, G, Dp = c["Hkv"], c["D"], c["K"], c["Hq"] // c["Hkv"], _padded(c["D"])
    n_rec = s.blocks * Hkv * 2 * Dp
    rec = s.summary[:n_rec].view(s.blocks, Hkv, 2, Dp)
    exps = s.summary[n_rec:n_rec + s.blocks * Hkv].view(s.blocks, Hkv)
    chosen = np.full((s.T, Hkv, K), -1, dtype=np.int32)
    t = 0
    for b in range(c["B"]):
        full = int(s.before[b] + s.new[b]) // BS
        ids = torch.as_tensor(s.table_host[b, :full].astype(np.int64), device="cuda")
        unit = torch.pow(2.0, exps[ids].double()).t()                                     # [Hkv, full]
        top, low = (rec[ids][:, :, i, :D].double().permute(1, 2, 0) * unit[:, None] for i in (0, 1))
        for i in range(int(s.new[b])):
            n = int(s.before[b] + i) // BS + 1
            q = s.q[t].double().view(Hkv, G, D)
            size = q.abs().amax(-1, keepdim=True)
            e = torch.ceil(torch.log2(size.clamp_min(2.0 ** -119) / 127.0))
            e = torch.where(size > 127.0 * torch.pow(2.0, e), e + 1, torch.where(size <= 127.0 * torch.pow(2.0, e - 1), e - 1, e)).clamp_min(-126)
            q = torch.round(q / torch.pow(2.0, e)) * torch.pow(2.0, e)
            score = (q.clamp_min(0) @ top + q.clamp_max(0) @ low).amax(1).cpu().numpy()
            for g in range(Hkv):
                by = np.zeros(n)
                by[:min(n, full)] = score[g, :n]
                j = np.arange(n)
                kept = (j < c["keep_first"]) | (j >= n - c["keep_last"])
                best = np.sort(np.lexsort((j, -by, ~kept))[:K])
                chosen[t, g, :len(best)] = best
            t += 1
    return {"blocks": torch.as_tensor(chosen)}


def _exact_sparse(c, s):
    """Token by token and head by head over the listed keys."""
    Hq, Hkv, D, G = c["Hq"], c["Hkv"], c["D"], c["Hq"] // c["Hkv"]
    kp, vp = s.kc.view(s.blocks, Hkv, D // s.x, BS, s.x), s.vc.view(s.blocks, Hkv, D, BS)
    out, lse = torch.empty(s.T, Hq, D, dtype=torch.float64, device="cuda"), torch.empty(s.T, Hq, dtype=torch.float64, device="cuda")
    lists, seq, pos = s.chosen.cpu().numpy(), s.seq.cpu().numpy(), s.pos.cpu().numpy()
    for t in range(s.T):
        for g in range(Hkv):
            j = lists[t, g][lists[t, g] >= 0].astype(np.int64)
            ids = torch.as_tensor(s.table_host[seq[t], j].astype(np.int64), device="cuda")
            at = torch.as_tensor((j[:, None] * BS + np.arange(BS)).reshape(-1) <= pos[t], device="cuda")
            keys = kp[ids, g].double().transpose(1, 2).reshape(-1, D)[at]
            vals = vp[ids, g].double().transpose(1, 2).reshape(-1, D)[at]
            score = s.q[t, g * G:(g + 1) * G].double() @ keys.t() / math.sqrt(D)
            lse[t, g * G:(g + 1) * G] = torch.logsumexp(score, -1)
            out[t, g * G:(g + 1) * G] = torch.softmax(score, -1) @ vals
    return {"out": out, "lse": lse}
