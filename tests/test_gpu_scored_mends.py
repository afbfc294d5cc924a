"""Attention with formed scores where it answered wrongly once: batches of fewer tokens than sequences."""
import numpy as np
import pytest
import torch

from tests.scored_util import Pools, check_rows, packed
from tests.test_gpu_scored import FORMATS, _prefill, _q, _scores

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("ranges", [False, True])
@pytest.mark.parametrize("new", [[0, 1], [0, 0, 5, 0, 0, 0, 1], [0] * 60 + [1] + [0] * 10 + [4], [0] * 90 + [70]], ids=["2", "7", "72", "91"])
def test_fewer_tokens_than_sequences(fmt, ranges, new):
    """Sequences without new tokens in front of those that have some, which are computed all the same."""
    new = np.array(new)
    before = np.arange(len(new)) * 37 % 200
    p = Pools(fmt, 64, 8, 1, before + new, seed=90)
    p.fill(before + new, 91)
    seq, pos = packed(before, new)
    begin = np.maximum(pos - 40, 0) if ranges else np.zeros(len(seq), dtype=np.int64)
    q = _q(len(seq), p, 92)
    out, lse = _prefill(p, before, new, q, _scores(p, 0.0, None, begin, pos + 1) if ranges else None)
    assert not out.isnan().any() and not lse.isnan().any()
    check_rows(p, q, out, lse, seq, pos, begin, pos + 1)
    p.ctx.close()
