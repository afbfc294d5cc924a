"""What the compiler reports of the kernels for long contexts: none goes through scratch memory but the one that takes prompts' tokens in groups, by so many registers: in front of and behind its main
loop, and in the loop that takes rows again."""
import re

import pytest

from tests.test_kernel_registers import _assert_none, _scratch_and_spills

KERNELS = {"kv_rope.hip": {"kv_append_rope": 10}, "kv_summary.hip": {"kv_summary_kernel": 2},
           "block_select.hip": {"score_step_kernel": 32, "score_prompt_kernel": 40, "code_kernel": 16, "choose_kernel": 6}, "attn_sparse.hip": {"attn_sparse_kernel": 16}}


@pytest.mark.parametrize("source", KERNELS)
def test_kernels_for_long_contexts_do_not_spill(tmp_path, source):
    of = _scratch_and_spills(tmp_path, source)
    for kernel, least in KERNELS[source].items():
        _assert_none(of, kernel, least)
    if source == "attn_sparse.hip":
        groups = {int(m.group(1)): v[1] for n, v in of.items() if (m := re.search(r"attn_sparse_prompt_kernelILi(\d)E", n))}
        most = {1: 0, 2: 12, 3: 18, 4: 52, 5: 0, 6: 0, 7: 0, 8: 4}
        assert groups.keys() == most.keys() and all(groups[k] <= most[k] for k in most), groups
