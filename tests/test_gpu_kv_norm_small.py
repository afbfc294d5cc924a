"""Norms without an eps of rows whose squares are below fp32, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from tests.parity_util import dev_i32
from tests.scored_util import BF, HALF, Pools, cu_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("eps", [0.0, 1e-38])
@pytest.mark.parametrize("step", [False, True])
@pytest.mark.parametrize("D", [64, 128, 256, 80])
def test_norm_of_rows_whose_squares_are_below_fp32(D, step, eps):
    """Rows of 1e-30 down to numbers of few bits beside ordinary ones; a row of zeros is 0 / 0 without an eps, and 0 with one."""
    sizes = np.array([1.0, 1e-10, 1e-17, 1e-18, 1e-19, 1e-20, 1e-25, 1e-30, 1e-36, 1e-38, 1e-39, 0.0])
    T = len(sizes)
    new = np.ones(T, dtype=int) if step else np.array([T])
    p = Pools("bf16", D, 2, 1, np.ones(T, dtype=int) if step else [T], seed=1)
    b = p.binding
    x = (torch.randn(T, 3, D, generator=torch.Generator().manual_seed(2), dtype=torch.float64) * torch.from_numpy(sizes)[:, None, None]).to(BF)
    w = 0.5 + torch.rand(D, generator=torch.Generator().manual_seed(3))
    freq = 10000.0 ** (-np.arange(D // 2) * 2.0 / D)
    rows = x.cuda()
    q_out = torch.full((T, 2, D), 55.0, dtype=BF, device="cuda")
    p.ctx.kv_append_norm(p.cache, rows[:, 2:], rows[:, 2:], cu_of(new), dev_i32(np.zeros(len(new))), p.dev_table, norm=b.HeadNorm(eps, w.cuda(), w.cuda()), rope=b.Rope(torch.from_numpy(freq).cuda()),
                         q=rows[:, :2], q_out=q_out, max_new_len=1 if step else None)
    held = p.held()[0]
    for t in range(T):
        for h in range(3):
            v = x[t, h].double().numpy()
            blk, slot = (p.table[t, 0], 0) if step else (p.table[0, t // 16], t % 16)
            got = q_out[t, h].double().cpu().numpy() if h < 2 else held[blk, 0, slot]
            with np.errstate(all="ignore"):
                z = v / np.sqrt((v * v).mean() + float(np.float32(eps))) * w.double().numpy()
            a, c = z[:D // 2], z[D // 2:]
            th = (0 if step else t) * freq
            want = np.concatenate([a * np.cos(th) - c * np.sin(th), a * np.sin(th) + c * np.cos(th)])
            size = np.concatenate([np.abs(a) + np.abs(c)] * 2)
            if np.isnan(want).any():
                assert np.isnan(got).all() and sizes[t] == 0
                continue
            # half a step of bf16, and what fp32 leaves: D squares and their sum, a root, three products, sine and cosine
            assert (np.abs(got - want) <= np.abs(want) * HALF + size * (D / 2 + 16) * 2.0 ** -24 + 1e-37).all(), (t, h, np.abs(got - want).max())
    p.ctx.close()
