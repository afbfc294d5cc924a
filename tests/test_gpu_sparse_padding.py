"""Places of a padded batch, which stand at negative positions, in the calls for long contexts: nothing is stored for them, and what the other tokens leave is what they leave
without them."""
import numpy as np
import pytest
import torch

from oracle import sparse_oracle as so
from paper_2504_18154_amd import workloads as wl
from tests.parity_util import dev_i32, say
from tests.test_gpu_sparse import Batch, _all_summarised, _attend, _compare, _expected_lists, _select, _summary_host

pytestmark = pytest.mark.gpu

STEP = [-1, 5, -20, 15, -16, -1], [1, 1, 1, 1, 1, 0]
PROMPTS = [-1, 5, -20, -3, -16, -40, 0], [1, 3, 7, 20, 49, 41, 2]


def _tables(before, new):
    """Rows of distinct blocks for what is at positions of 0 and more; in every other place one block that belongs to nobody."""
    per = (np.maximum(before + new, 0) + 15) // 16
    table = np.full((len(new), int(per.max()) + 2), int(per.sum()), dtype=np.int32)
    at = 0
    for b, n in enumerate(per):
        table[b, :n] = np.arange(at, at + n)
        at += n
    return table, at + 1


@pytest.mark.parametrize("dtype,D,Hq,Hkv,rotary,adjacent", [("bf16", 128, 8, 2, None, False), ("bf16", 128, 8, 2, 32, False), ("bf16", 72, 3, 3, 24, True), ("f32", 64, 4, 1, None, False)])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("batch,most", [(STEP, 1), (STEP, None), (PROMPTS, None)], ids=["step", "step-as-prompts", "prompts"])
def test_rotated_append(batch, most, in_place, dtype, D, Hq, Hkv, rotary, adjacent):
    from paper_2504_18154_amd import binding
    before, new = (np.array(x) for x in batch)
    table, blocks = _tables(before, new)
    B, T = len(new), int(new.sum())
    say(f"{dtype}, D {D}, heads {Hq}/{Hkv}, new {new.tolist()} behind {before.tolist()}")
    ctx = binding.Context(Hq, Hkv, D, blocks, dtype, B, table.shape[1])
    rope = binding.Rope(10000.0 ** (-torch.arange((rotary or D) // 2, dtype=torch.float64, device="cuda") / 32), "adjacent" if adjacent else "halves")
    q, k, v = (wl.randn((T, h, D), dtype, 7 + n).cuda() for n, h in enumerate((Hq, Hkv, Hkv)))

    def append(before, new, q, k, v, most):
        kc, vc = ctx.new_cache()
        out = q.clone() if in_place else torch.full_like(q, 7.0)
        ctx.kv_append_rope(kc, vc, k, v, dev_i32(wl.cu_from_lengths(new)), dev_i32(before), dev_i32(table), rope, q=out if in_place else q, q_out=out, max_new_len=most)
        return kc, vc, out

    place = np.concatenate([b + np.arange(n) for b, n in zip(before, new)])
    there = torch.as_tensor(place >= 0)
    got = append(before, new, q, k, v, most)
    skipped = np.minimum(np.maximum(-before, 0), new)
    want = append(before + skipped, new - skipped, *(t[there].contiguous() for t in (q, k, v)), most)
    bits = lambda t: t.contiguous().view(torch.uint8)
    assert torch.equal(bits(got[0]), bits(want[0])) and torch.equal(bits(got[1]), bits(want[1]))
    assert torch.equal(bits(got[2][there]), bits(want[2])) and torch.equal(bits(got[2][~there]), bits(q[~there] if in_place else torch.full_like(q[~there], 7.0)))
    assert ctx.k_logical(got[0])[blocks - 1].isnan().all() and ctx.v_logical(got[1])[blocks - 1].isnan().all()      # (the sentinel of new_cache)
    ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("batch", [([-1, 15, -20, 31, -16, -1], [1, 1, 1, 1, 1, 0]), (PROMPTS[0] + [-2, -5], PROMPTS[1] + [34, 21])], ids=["step", "prompts"])
def test_summaries(batch, dtype):
    """A sequence that begins with places of the padding has its blocks summarised all the same."""
    b = Batch(dtype, 40, 6, 2, *batch, seed=3)
    summary = torch.full_like(b.ctx.new_summary(), 85)
    codes, exps = _summary_host(b.ctx.layout, b.summarise(summary))
    filled = {int(b.table[s, j]) for s in range(b.B) for j in range(max(b.before[s], 0) // 16, b.total[s] // 16) if b.new[s]}
    assert len(filled) >= 2
    for blk in range(codes.shape[0]):
        for g in range(b.Hkv):
            if blk not in filled:
                assert (codes[blk, g] == 85).all() and exps[blk, g] == 85, blk
                continue
            want, e = so.summarise(b.keys[blk, g].float().numpy())
            assert exps[blk, g] == e and np.array_equal(codes[blk, g, :, :b.D], want), (blk, g)
    b.ctx.close()


@pytest.mark.parametrize("dtype,D,Hq,Hkv,before,new", [("bf16", 128, 8, 2, [-40, 100], [2100, 900]), ("bf16", 64, 6, 3, [-3, -100], [60, 90]), ("f32", 64, 4, 2, [-17, 20], [300, 9])])
def test_selection_and_attention(dtype, D, Hq, Hkv, before, new):
    """Prompts that begin with places of the padding, token by token and in groups."""
    b = Batch(dtype, D, Hq, Hkv, before, new, seed=5)
    summary, codes, exps = _all_summarised(b)
    want = _expected_lists(b, codes, exps, 6, 1, 2)
    assert np.array_equal(_select(b, summary, 6, 1, 2), want)
    out, lse = _attend(b, want)
    nothing = torch.as_tensor(b.pos < 0)
    assert nothing.any() and (out.cpu()[nothing] == 0).all() and torch.isneginf(lse.cpu()[nothing]).all()
    some = [t for t in range(b.T) if b.pos[t] >= 0 and (b.pos[t] < 70 or t % 41 == 0)]
    _compare(b, want, out, lse, name="attention", tokens=some)
    b.ctx.close()


def test_a_prompt_recorded_into_a_graph():
    """The four calls of a prompt's chunk whose batch has places of the padding, replayed with new inputs between eager work of the same shape: every replay the same bits as the eager calls."""
    from paper_2504_18154_amd import binding
    Hq, Hkv, D, K = 8, 2, 128, 5
    before, new = np.array([200, -30, 700]), np.array([1400, 60, 700])
    T, B = int(new.sum()), 3
    table, nb = _tables(before, new)
    ctx = binding.Context(Hq, Hkv, D, nb, "bf16", B, table.shape[1])
    g = torch.Generator(device="cuda").manual_seed(5)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)
    pools = [rand(nb * Hkv * 16 * D) for _ in range(2)]
    rope = binding.Rope(10000.0 ** (-torch.arange(64, dtype=torch.float64, device="cuda") / 64))
    bt, cu, at = dev_i32(table), dev_i32(wl.cu_from_lengths(new)), dev_i32(before)
    first = ctx.new_summary()
    ctx.kv_summary(pools[0], first, dev_i32(wl.cu_from_lengths(np.maximum(before, 0))), dev_i32(np.zeros(B)), bt, int(np.maximum(before, 0).sum()))
    q, k, v = rand(T, Hq, D), rand(T, Hkv, D), rand(T, Hkv, D)

    def chunk(kc, vc, summ, lists, q_out, out, lse):
        ctx.kv_append_rope(kc, vc, k, v, cu, at, bt, rope, q=q, q_out=q_out)
        ctx.kv_summary(kc, summ, cu, at, bt, T)
        ctx.block_select(q_out, summ, at, bt, lists, 1600, keep_last=2, cu_q=cu)
        ctx.attn_sparse(q_out, kc, vc, at, bt, lists, out, lse=lse, cu_q=cu)

    def buffers():
        return (pools[0].clone(), pools[1].clone(), first.clone(), torch.zeros(T, Hkv, K, dtype=torch.int32, device="cuda"), torch.zeros_like(q), torch.zeros_like(q),
                torch.zeros(T, Hq, device="cuda"))

    mine, eager, graph = buffers(), buffers(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        chunk(*mine)
    for i in range(4):
        for t in (q, k, v):
            t.copy_(rand(*t.shape))
        chunk(*eager)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(mine, eager):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), i
    ctx.close()
