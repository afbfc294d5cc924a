"""Sequences in a paged cache of any format, on the device and in 64 bits, for the tests of the normed append and of attention with formed scores."""
from __future__ import annotations

import math

import numpy as np
import torch

from oracle import scored_oracle as so
from paper_2504_18154_amd import workloads as wl
from tests.parity_util import dev_i32

BF = torch.bfloat16
HALF = torch.finfo(BF).eps / 2


class Pools:
    """A context and a cache whose slots hold garbage (bytes that stand for NaN among it) until something is stored."""

    def __init__(self, fmt, D, Hq, Hkv, total, seed=0, spare=3, scale=0.0, max_batch=None):
        from paper_2504_18154_amd import binding
        self.binding, self.fmt, self.D, self.Hq, self.Hkv, self.G = binding, fmt, D, Hq, Hkv, Hq // Hkv
        rng = np.random.default_rng(seed)
        per = (np.maximum(np.asarray(total), 0) + 15) // 16
        ids = rng.permutation(int(per.sum()) + spare)
        self.blocks = len(ids)
        self.table = np.full((len(per), max(1, int(per.max(initial=0)))), int(ids[-1]), dtype=np.int32)  # (what is not a sequence's: a block that nobody has)
        at = 0
        for b, n in enumerate(per):
            self.table[b, :n] = ids[at:at + n]
            at += n
        self.ctx = binding.Context(Hq, Hkv, D, self.blocks, "bf16", max_batch or len(per), self.table.shape[1], softmax_scale=scale)
        self.scale = scale or 1 / math.sqrt(D)
        self.cache = self.ctx.new_paged_cache(fmt)
        if fmt != "bf16":
            junk = torch.from_numpy(rng.integers(0, 256, size=self.cache.k.numel(), dtype=np.uint8))
            junk[::3] = 0x7f
            self.cache.k.copy_(junk)
            self.cache.v.copy_(junk.flip(0))
            self.cache.scales.copy_(torch.from_numpy(rng.choice(np.array([255, 255, 0, 127, 254], dtype=np.uint8), size=tuple(self.cache.scales.shape))))
        self.dev_table = dev_i32(self.table)

    # logical views of the device's bytes, on the host: [blocks, Hkv, 16, D]
    def logical(self):
        x = 8 if self.fmt == "bf16" else 16
        k = self.cache.k.cpu().view(self.blocks, self.Hkv, self.D // x, 16, x).permute(0, 1, 3, 2, 4).reshape(self.blocks, self.Hkv, 16, self.D)
        v = self.cache.v.cpu().view(self.blocks, self.Hkv, self.D, 16).permute(0, 1, 3, 2)
        return k, v

    def scales(self):
        return self.cache.scales.cpu().numpy() if self.fmt != "bf16" else None

    def put(self, k, v, ks=None, vs=None):
        """Logical pools to the device."""
        x = 8 if self.fmt == "bf16" else 16
        self.cache.k.copy_(k.view(self.blocks, self.Hkv, 16, self.D // x, x).permute(0, 1, 3, 2, 4).contiguous().flatten())
        self.cache.v.copy_(v.permute(0, 1, 3, 2).contiguous().flatten())
        if self.fmt != "bf16":
            self.cache.scales.copy_(torch.from_numpy(np.stack([ks, vs], axis=2)))

    def held(self):
        """What the bytes stand for, fp64 [blocks, Hkv, 16, D] twice."""
        k, v = self.logical()
        if self.fmt == "bf16":
            return k.double().numpy(), v.double().numpy()
        s = self.scales()
        return so.value(k.numpy(), s[:, :, 0], self.fmt), so.value(v.numpy(), s[:, :, 1], self.fmt)

    def rows(self, of, b, g, upto):
        """[upto, D] of sequence b and K/V head g."""
        return np.concatenate([of[i, g] for i in self.table[b, :(upto + 15) // 16]])[:upto] if upto > 0 else np.zeros((0, self.D))

    def fill(self, total, seed, wide=1.0):
        """Random tokens 0 .. total[b] - 1 of each sequence, coded by torch's types (fast; the oracle's coding is tested against them), the rest left as it is."""
        g = torch.Generator().manual_seed(seed)
        shape = (self.blocks, self.Hkv, 16, self.D)
        live = torch.zeros(self.blocks, 16, dtype=torch.bool)
        for b, n in enumerate(total):
            for j in range((max(n, 0) + 15) // 16):
                live[self.table[b, j], :min(16, n - 16 * j)] = True
        at = live[:, None, :, None].expand(shape)
        size = torch.exp(torch.randn(1, self.Hkv, 1, self.D, generator=g) * 0.3) * wide
        new = [torch.randn(shape, generator=g) * size, torch.randn(shape, generator=g)]
        old = self.logical()
        if self.fmt == "bf16":
            self.put(*(torch.where(at, n.to(BF), o) for n, o in zip(new, old)))
            return
        s, most = self.scales(), so.MOST[self.fmt]
        out = []
        for i, n in enumerate(new):
            top = n.abs().amax(-1).double()
            e = torch.ceil(torch.log2(top / most)).clamp_min(-126)
            y = n.double() / torch.exp2(e)[..., None]
            c = torch.round(y).to(torch.int8).view(torch.uint8) if self.fmt == "int8" else y.float().to(torch.float8_e4m3fn).view(torch.uint8)
            out.append((torch.where(at, c, old[i]), np.where(live[:, None].numpy(), (e + 127).to(torch.uint8).numpy(), s[:, :, i])))
        self.put(out[0][0], out[1][0], out[0][1], out[1][1])


def check_rows(pools: Pools, q, out, lse, seq, pos, begin, end, cap=0.0, slopes=None, tokens=None, held=None, label=""):
    """out [T, Hq, D] and lse [T, Hq] of `tokens` (all) against the definition, within the roundings that the kernels make:
    weights rounded to bf16 (half a step each), the result's rounding, and what fp32 leaves of scores and sums."""
    keys, vals = pools.held() if held is None else held
    out, lse, q = out.double().cpu().numpy(), lse.double().cpu().numpy(), q.double().cpu().numpy()
    G = pools.G
    for t in range(len(seq)) if tokens is None else tokens:
        lo, hi = int(max(begin[t], 0)), int(end[t])
        for g in range(pools.Hkv):
            heads = slice(g * G, g * G + G)
            n = max(hi, 0)
            k, v = pools.rows(keys, seq[t], g, n)[lo:], pools.rows(vals, seq[t], g, n)[lo:]
            if pos[t] < 0:
                k, v = k[:0], v[:0]
            want, want_lse, size, off = so.attend(q[t, heads], k, v, np.arange(lo, lo + len(k)), int(pos[t]), pools.scale, cap, None if slopes is None else slopes[heads])
            got, got_lse = out[t, heads], lse[t, heads]
            what = f"{label} token {t} (sequence {seq[t]}, position {pos[t]}, keys {lo}..{hi}), K/V head {g}"
            if len(k) == 0:
                assert (got == 0).all() and (got_lse == -np.inf).all(), what
                continue
            odd = ~np.isfinite(want)
            assert np.array_equal(np.isnan(got), np.isnan(want)) if np.isnan(want[odd]).all() else (~np.isfinite(got))[odd].all(), f"{what}: {got[odd]} for {want[odd]}"
            tol = size * (HALF + 2 * off[:, None] + (len(k) + 64) * 2.0 ** -24) + np.abs(want) * HALF + 1e-30
            with np.errstate(invalid="ignore"):
                err = np.abs(got - want)
            assert (err <= tol)[~odd].all(), f"{what}: off by {err[~odd].max():.3e}, {np.max((err / tol)[~odd]):.2f} of the bound"
            fine = np.isfinite(want_lse)
            assert np.array_equal(fine, np.isfinite(got_lse)), f"{what}: lse {got_lse} for {want_lse}"
            tol = off + (len(k) + 64) * 2.0 ** -24 + np.abs(want_lse) * 2.0 ** -22 + 2.0 ** -20
            assert (np.abs(got_lse - want_lse) <= tol)[fine].all(), f"{what}: lse off by {np.abs(got_lse - want_lse)[fine].max():.3e} of {tol}"


def packed(before, new):
    """(sequence, position) per new token."""
    before, new = np.asarray(before), np.asarray(new)
    seq = np.repeat(np.arange(len(new)), new)
    pos = np.concatenate([b + np.arange(n) for b, n in zip(before, new)]) if new.sum() else np.zeros(0, dtype=int)
    return seq, pos


def cu_of(new):
    return dev_i32(wl.cu_from_lengths(np.asarray(new, dtype=np.int32)))
