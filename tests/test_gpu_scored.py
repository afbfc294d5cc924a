"""Attention with formed scores over caches of 16 and 8 bits against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from tests.parity_util import dev_i32, say
from tests.scored_util import BF, Pools, check_rows, cu_of, packed

pytestmark = pytest.mark.gpu

LAYOUTS = [(128, 40, 8), (128, 8, 1), (128, 5, 1), (128, 3, 3), (128, 16, 1), (64, 32, 8), (16, 4, 2), (48, 6, 2), (80, 8, 8), (112, 4, 1), (144, 2, 1), (256, 8, 1), (256, 16, 1)]
FORMATS = ["e4m3", "int8", "bf16"]
FORMS = ["plain", "cap", "slopes", "both"]


def _form(p: Pools, kind):
    """(softcap, slopes on the host)"""
    slopes = 2.0 ** (-8.0 * np.arange(1, p.Hq + 1) / p.Hq) if kind in ("slopes", "both") else None
    return (20.0 if kind in ("cap", "both") else 0.0), None if slopes is None else slopes.astype(np.float32)


def _scores(p, cap, slopes, begin=None, end=None):
    return p.binding.Scores(softcap=cap, slopes=None if slopes is None else torch.from_numpy(slopes).cuda(), key_begin=None if begin is None else dev_i32(begin),
                            key_end=None if end is None else dev_i32(end))


def _decode(p: Pools, lens, q, scores=None, workspace=None, most=None):
    out, lse = torch.full_like(q, float("nan")), torch.full(q.shape[:2], float("nan"), device="cuda")
    p.ctx.attn_decode_scored(q, p.cache, p.dev_table, dev_i32(lens), out, most or max(1, int(np.max(lens))), lse=lse, scores=scores, workspace=workspace)
    return out, lse


def _prefill(p: Pools, before, new, q, scores=None, workspace=None):
    out, lse = torch.full_like(q, float("nan")), torch.full(q.shape[:2], float("nan"), device="cuda")
    p.ctx.attn_prefill_scored(q, p.cache, cu_of(new), dev_i32(before), p.dev_table, out, lse=lse, scores=scores, workspace=workspace)
    return out, lse


def _q(T, p, seed, size=1.0):
    return (torch.randn(T, p.Hq, p.D, generator=torch.Generator().manual_seed(seed)) * size).to(BF).cuda()


# ---- one token ------------------------------------------------------------------------------------


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D,Hq,Hkv", LAYOUTS, ids=str)
def test_decode(fmt, D, Hq, Hkv):
    """Contexts from one token over the edges of blocks and steps to ones that are cut, one of none; every form."""
    lens = np.array([1, 2, 15, 16, 17, 31, 32, 33, 47, 64, 65, 300, 0, 1027, 2400], dtype=np.int32)
    p = Pools(fmt, D, Hq, Hkv, lens, seed=D + Hq)
    p.fill(lens, 1)
    held = p.held()
    q = _q(len(lens), p, 2, 1.5)
    for kind in FORMS:
        say(f"decode {fmt}, D {D}, heads {Hq}/{Hkv}, {kind}")
        cap, slopes = _form(p, kind)
        out, lse = _decode(p, lens, q, _scores(p, cap, slopes))
        check_rows(p, q, out, lse, np.arange(len(lens)), lens - 1, np.zeros(len(lens)), lens, cap, slopes, held=held)
    p.ctx.close()


@pytest.mark.parametrize("fmt", FORMATS)
def test_decode_ranges(fmt):
    """Windows and documents that begin anywhere, ends before the token, ends behind what there is, empty ranges, begins below 0."""
    lens = np.array([1, 40, 40, 40, 40, 40, 40, 100, 700, 700, 700, 2000, 2000], dtype=np.int32)
    begin = np.array([0, 39, 40, 7, 20, -5, 30, 16, 0, 512, 699, 1000, 33], dtype=np.int32)
    end = np.array([5, 40, 50, 8, 10, 3, 33, 32, 700, 640, 10000, 1999, 34], dtype=np.int32)
    p = Pools(fmt, 128, 8, 2, lens, seed=3)
    p.fill(lens, 4)
    q = _q(len(lens), p, 5)
    for b, e in ((begin, None), (None, end), (begin, end)):
        out, lse = _decode(p, lens, q, _scores(p, 0.0, None, b, e))
        check_rows(p, q, out, lse, np.arange(len(lens)), lens - 1, np.zeros(len(lens)) if b is None else b, lens if e is None else np.minimum(e, lens))
    p.ctx.close()


@pytest.mark.parametrize("fmt", FORMATS)
def test_decode_of_one_long_context(fmt):
    """Cut into as many slices as there can be; twice the same bits; the counters are left as they were."""
    lens = np.array([40000], dtype=np.int32)
    p = Pools(fmt, 128, 8, 1, lens, seed=6)
    p.fill(lens, 7)
    q = _q(1, p, 8, 2.0)
    runs = [_decode(p, lens, q) for _ in range(4)]
    check_rows(p, q, *runs[0], [0], lens - 1, [0], lens)
    assert all(torch.equal(r[0], runs[0][0]) and torch.equal(r[1], runs[0][1]) for r in runs)
    p.ctx.close()


def test_decode_of_many_sequences():
    """More sequences than the workgroups hold ranges of, lengths all different."""
    lens = (np.arange(1500) * 7 % 130).astype(np.int32)
    p = Pools("e4m3", 64, 2, 1, lens, seed=9)
    p.fill(lens, 10)
    q = _q(len(lens), p, 11)
    begin = np.where(np.arange(1500) % 3 == 0, lens - 20, 0).astype(np.int32)
    out, lse = _decode(p, lens, q, _scores(p, 0.0, None, begin))
    check_rows(p, q, out, lse, np.arange(1500), lens - 1, begin, lens, tokens=range(0, 1500, 13))
    p.ctx.close()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_decode_with_rows_that_are_not_finite(fmt):
    """A key or a value whose scale says NaN: all of its head's results, and of no other head or sequence; out of the range: none."""
    lens = np.array([50, 50, 600, 50, 50], dtype=np.int32)
    p = Pools(fmt, 64, 4, 2, lens, seed=12)
    p.fill(lens, 13)
    (k, v), s = p.logical(), p.scales().copy()
    for b, j, g, i in ((0, 20, 0, 0), (1, 49, 1, 1), (2, 300, 0, 1), (3, 5, 0, 0), (4, 6, 1, 1)):
        blk = p.table[b, j // 16]
        s[blk, g, i, j % 16] = 255
        (k if i == 0 else v)[blk, g, j % 16] = 0
    p.put(k, v, s[:, :, 0], s[:, :, 1])
    q = _q(len(lens), p, 14)
    begin = np.array([0, 0, 0, 6, 7], dtype=np.int32)
    out, lse = _decode(p, lens, q, _scores(p, 0.0, None, begin))
    assert out[0, :2].isnan().all() and out[1, 2:].isnan().all() and out[2, :2].isnan().all() and lse[1].isfinite().all() and lse[0, :2].isnan().all()
    assert out[0, 2:].isfinite().all() and out[1, :2].isfinite().all() and out[2, 2:].isfinite().all() and out[3:].isfinite().all() and lse[3:].isfinite().all()
    check_rows(p, q, out, lse, np.arange(5), lens - 1, begin, lens, tokens=[3, 4])
    p.ctx.close()


# ---- prompts --------------------------------------------------------------------------------------


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D,Hq,Hkv", LAYOUTS, ids=str)
def test_prefill(fmt, D, Hq, Hkv):
    """Chunks of one token and of many, behind nothing and behind a cached prefix; every form."""
    before, new = np.array([0, 5, 0, 100, 16, 0, 63]), np.array([1, 1, 70, 33, 0, 140, 65])
    p = Pools(fmt, D, Hq, Hkv, before + new, seed=D + Hq)
    p.fill(before + new, 21)
    held = p.held()
    seq, pos = packed(before, new)
    q = _q(len(seq), p, 22, 1.5)
    for kind in FORMS:
        say(f"prefill {fmt}, D {D}, heads {Hq}/{Hkv}, {kind}")
        cap, slopes = _form(p, kind)
        out, lse = _prefill(p, before, new, q, _scores(p, cap, slopes))
        check_rows(p, q, out, lse, seq, pos, np.zeros(len(seq)), pos + 1, cap, slopes, held=held, tokens=None if kind == "plain" else range(0, len(seq), 5))
    p.ctx.close()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("kind", ["window", "documents", "prefix", "odd"])
def test_prefill_ranges(fmt, kind):
    before, new = np.array([0, 130, 20]), np.array([200, 90, 300])
    total = before + new
    p = Pools(fmt, 128, 8, 2, total, seed=23)
    p.fill(total, 24)
    seq, pos = packed(before, new)
    begin, end = np.zeros(len(seq), dtype=np.int64), pos + 1
    rng = np.random.default_rng(25)
    if kind == "window":
        begin = np.maximum(pos - 30, 0)
    elif kind == "documents":
        begin = np.maximum(begin, pos // 41 * 41)
    elif kind == "prefix":
        end = np.maximum(end, np.array([150, 180, 0])[seq])
    else:  # any ranges at all: empty, behind the sequence's end, one key
        begin, end = rng.integers(-20, 250, len(seq)), rng.integers(-10, 400, len(seq))
    q = _q(len(seq), p, 26)
    out, lse = _prefill(p, before, new, q, _scores(p, 0.0, None, begin, end))
    check_rows(p, q, out, lse, seq, pos, begin, np.minimum(end, total[seq]), tokens=range(0, len(seq), 2))
    p.ctx.close()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("D", [64, 128, 256])
def test_prefill_of_few_rows_behind_long_contexts(fmt, D):
    """Steps cut among workgroups: whatever comes last, the same bits."""
    before, new = np.array([3000, 7]), np.array([9, 3])
    p = Pools(fmt, D, 4, 2, before + new, seed=27)
    p.fill(before + new, 28)
    seq, pos = packed(before, new)
    q = _q(len(seq), p, 29, 2.0)
    assert p.ctx.prefill_scored_workspace_bytes(2, len(seq)) > 0
    cap, slopes = _form(p, "both")
    for form in ((0.0, None), (cap, slopes)):
        runs = [_prefill(p, before, new, q, _scores(p, *form)) for _ in range(3)]
        check_rows(p, q, *runs[0], seq, pos, np.zeros(len(seq)), pos + 1, *form)
        assert all(torch.equal(r[0], runs[0][0]) and torch.equal(r[1], runs[0][1]) for r in runs)
    p.ctx.close()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("few", [False, True])
def test_values_that_are_not_finite_reach_who_sees_them(fmt, few):
    """In the future of some rows of a tile, behind a window, and in sight."""
    before, new = (np.array([70]), np.array([90])) if not few else (np.array([1200]), np.array([20]))
    total = int(before[0] + new[0])
    p = Pools(fmt, 64, 4, 2, [total], seed=30)
    p.fill([total], 31)
    k, v = p.logical()
    s = p.scales()
    first = int(before[0])
    bad = [(first + 12, 0, 1), (first + 3, 1, 0), (first - 30, 0, 1)]   # (position, K/V head, 0: key, 1: value)
    for j, g, i in bad:
        blk = p.table[0, j // 16]
        if fmt == "bf16":
            (k if i == 0 else v)[blk, g, j % 16, 5 if i else 0] = float("inf") if i == 1 else float("nan")
        else:
            s = s.copy()
            s[blk, g, i, j % 16] = 255
            (k if i == 0 else v)[blk, g, j % 16] = 0
    p.put(k, v, *((s[:, :, 0], s[:, :, 1]) if s is not None else ()))
    seq, pos = packed(before, new)
    begin = np.maximum(pos - 25, 0)   # (the key 30 places back is out of sight of all, the others are seen by some)
    q = _q(len(seq), p, 32)
    out, lse = _prefill(p, before, new, q, _scores(p, 0.0, None, begin))
    check_rows(p, q, out, lse, seq, pos, begin, pos + 1)
    o = out.float().cpu()
    for t, at in enumerate(pos):
        sees = first + 12 <= at <= first + 12 + 25
        assert bool((~o[t, :2].isfinite()).any()) == sees, (t, at)
        assert bool((~o[t, 2:].isfinite()).any()) == (first + 3 <= at <= first + 3 + 25), (t, at)
    p.ctx.close()


def test_padded_batches():
    """Sequences that begin with places of the padding, rows behind the last sequence: the first see nothing, the others are left alone."""
    before, new = np.array([-20, 0, -70]), np.array([50, 0, 60])
    p = Pools("int8", 64, 4, 2, before + new, seed=33)
    p.fill(before + new, 34)
    seq, pos = packed(before, new)
    q = _q(len(seq) + 7, p, 35)
    out, lse = _prefill(p, before, new, q)
    check_rows(p, q, out, lse, seq, pos, np.zeros(len(seq)), np.maximum(pos + 1, 0))
    assert out[len(seq):].isnan().all() and lse[len(seq):].isnan().all()
    p.ctx.close()


def test_rows_in_wider_ones_and_no_lse():
    before, new = np.array([20, 0]), np.array([30, 41])
    p = Pools("e4m3", 128, 8, 2, before + new, seed=36)
    p.fill(before + new, 37)
    seq, pos = packed(before, new)
    wide = torch.randn(len(seq), 12, 128, generator=torch.Generator().manual_seed(38)).to(BF).cuda()
    q = wide[:, :8]
    a, b = torch.empty(len(seq), 8, 128, dtype=BF, device="cuda"), torch.empty(len(seq), 8, 128, dtype=BF, device="cuda")
    p.ctx.attn_prefill_scored(q, p.cache, cu_of(new), dev_i32(before), p.dev_table, a)
    p.ctx.attn_prefill_scored(q.contiguous(), p.cache, cu_of(new), dev_i32(before), p.dev_table, b)
    assert torch.equal(a, b)
    lens = before + new
    x, y = torch.empty(2, 8, 128, dtype=BF, device="cuda"), torch.empty(2, 8, 128, dtype=BF, device="cuda")
    p.ctx.attn_decode_scored(q[:2], p.cache, p.dev_table, dev_i32(lens), x, int(lens.max()))
    p.ctx.attn_decode_scored(q[:2].contiguous(), p.cache, p.dev_table, dev_i32(lens), y, 10 * 16 if p.table.shape[1] >= 10 else int(lens.max()))
    assert torch.equal(x, y)
    p.ctx.close()


def test_over_the_layouts_cache_both_ways_agree():
    """The calls of the layout's own cache and these, on the same bytes, within both of their roundings."""
    before, new = np.array([100, 0, 900]), np.array([60, 200, 37])
    total = before + new
    p = Pools("bf16", 128, 16, 4, total, seed=39)
    p.fill(total, 40)
    seq, pos = packed(before, new)
    q = _q(len(seq), p, 41)
    out, lse = _prefill(p, before, new, q)
    other = torch.empty_like(q)
    p.ctx.attn_prefill(q, p.cache.k, p.cache.v, cu_of(new), dev_i32(before), p.dev_table, other)
    check_rows(p, q, out, lse, seq, pos, np.zeros(len(seq)), pos + 1, tokens=range(0, len(seq), 7))
    assert (out.float() - other.float()).abs().max() < 4e-2
    d, dl = _decode(p, total, q[:3])
    want = torch.empty_like(d)
    p.ctx.attn_decode(q[:3], p.cache.k, p.cache.v, p.dev_table, dev_i32(total), want, int(total.max()))
    assert (d.float() - want.float()).abs().max() < 4e-2
    p.ctx.close()


def test_workspaces_are_not_overrun_and_calls_fit_into_graphs():
    """A workspace of the very size, guarded behind; a step and a chunk recorded, replayed on new lengths and inputs between eager calls."""
    lens = np.array([900, 33, 2000, 1], dtype=np.int32)
    p = Pools("e4m3", 128, 8, 2, lens + 64, seed=42)
    p.fill(lens + 64, 43)
    n = p.ctx.decode_scored_workspace_bytes()
    room = torch.full((n + 4096,), 77, dtype=torch.uint8, device="cuda")
    q = _q(4, p, 44)
    want = _decode(p, lens, q)
    got = _decode(p, lens, q, workspace=room[:n])
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1]) and (room[n:] == 77).all()
    before, new = lens, np.array([3, 1, 2, 4])
    qp = _q(int(new.sum()), p, 45)
    m = p.ctx.prefill_scored_workspace_bytes(4, len(qp))
    room2 = torch.full((m + 4096,), 77, dtype=torch.uint8, device="cuda")
    want2 = _prefill(p, before, new, qp)
    got2 = _prefill(p, before, new, qp, workspace=room2[:m])
    assert torch.equal(want2[0], got2[0]) and (room2[m:] == 77).all()

    length, cu, at = dev_i32(lens), cu_of(new), dev_i32(before)
    out, lse, outp = torch.empty_like(q), torch.empty(4, 8, device="cuda"), torch.empty_like(qp)
    begin = dev_i32(np.zeros(4))
    scores = p.binding.Scores(softcap=30.0, key_begin=begin)
    most = int(lens.max()) + 64

    def both():
        p.ctx.attn_decode_scored(q, p.cache, p.dev_table, length, out, most, lse=lse, scores=scores, workspace=room[:n])
        p.ctx.attn_prefill_scored(qp, p.cache, cu, at, p.dev_table, outp, workspace=room2[:m])

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        both()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        both()
    for i in range(4):
        length.copy_(dev_i32(lens + 13 * i))
        begin.copy_(dev_i32(np.maximum(lens - 300 * i, 0)))
        q.copy_(_q(4, p, 50 + i))
        qp.copy_(_q(len(qp), p, 60 + i))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        a, b, c = out.clone(), lse.clone(), outp.clone()
        both()
        torch.cuda.synchronize()
        assert torch.equal(a, out) and torch.equal(b, lse) and torch.equal(c, outp), i
        check_rows(p, q, a, b, np.arange(4), lens + 13 * i - 1, begin.cpu().numpy(), lens + 13 * i, 30.0)
    p.ctx.close()


def test_two_streams_with_a_context_each():
    lens = np.array([5000, 300], dtype=np.int32)
    pools = [Pools("int8", 128, 8, 2, lens, seed=70 + i) for i in range(2)]
    for i, p in enumerate(pools):
        p.fill(lens, 72 + i)
    qs = [_q(2, p, 74 + i) for i, p in enumerate(pools)]
    want = [_decode(p, lens, q) for p, q in zip(pools, qs)]
    streams = [torch.cuda.Stream() for _ in pools]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i, p in enumerate(pools):
            with torch.cuda.stream(streams[i]):
                got[i].append(_decode(p, lens, qs[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o, want[i][0]) and torch.equal(l, want[i][1]) for o, l in got[i])
    for p in pools:
        p.ctx.close()


def test_arguments_that_python_refuses():
    lens = np.array([20], dtype=np.int32)
    p = Pools("e4m3", 64, 4, 2, lens, seed=80)
    q = _q(1, p, 81)
    out = torch.empty_like(q)
    b = p.binding
    call = lambda **kw: p.ctx.attn_decode_scored(**{**dict(q=q, cache=p.cache, block_table=p.dev_table, ctx_len=dev_i32(lens), out=out, max_ctx_len=20), **kw})
    call()
    for kw in (dict(q=q.float()), dict(q=q[:, :2]), dict(out=out.float()), dict(out=out.cpu()), dict(ctx_len=dev_i32(lens).long()), dict(block_table=p.dev_table[0]),
               dict(lse=torch.empty(1, 2, device="cuda")), dict(scores=b.Scores(slopes=torch.zeros(2, device="cuda"))), dict(scores=b.Scores(key_begin=torch.zeros(0, dtype=torch.int32, device="cuda"))),
               dict(scores=b.Scores(slopes=torch.zeros(4)))):
        with pytest.raises(ValueError):
            call(**kw)
    small = b.PagedCache(p.cache.k[:64], p.cache.v, p.cache.scales, format="e4m3")
    with pytest.raises(ValueError):
        call(cache=small)
    with pytest.raises(b.EcoserveError):
        call(workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(b.EcoserveError):
        call(max_ctx_len=10000)
    p.ctx.close()
