"""Where the areas of a workspace start."""
import pytest

import paper_2503_10017_amd as fnn
from test_abi import lib  # noqa: F401


def test_shares_of_split_attention_lie_on_16_byte_boundaries(lib):  # noqa: F811
    """A share's rows are stored and read in runs of 16 bytes, so what lies before them has to be whole runs: what the workspace has beside the
    rows, whose size is linear in the elements of a row."""
    seen_odd = False
    for queries, keys, batch, heads, groups in ((1, 700, 1, 1, 1), (1, 6000, 1, 1, 1), (3, 700, 1, 1, 1), (1, 100000, 1, 3, 1), (3, 3000, 3, 1, 1), (2, 5000, 1, 4, 2), (5, 2000, 1, 7, 7)):
        need = [fnn.fnn_attention_workspace_bytes(queries, keys, batch, heads, groups, d) for d in (8, 16)]
        assert need[0] > 0
        rows = need[1] - need[0]                        # 8 floats of every share
        shares = rows // 32
        before = need[0] - rows
        assert shares % (queries * heads) == 0 and before >= shares * 8
        assert before % 16 == 0, (queries, keys, heads)
        seen_odd |= shares % 2 == 1
    assert seen_odd


@pytest.mark.gpu
@pytest.mark.parametrize("case", [([1], [700], 1, 1, 64), ([3], [900], 1, 1, 40), ([1], [6000], 3, 1, 128)])
def test_odd_numbers_of_shares(case):
    from test_gpu_attention import Problem, check_forward

    prob = Problem(*case, True, "bf16")
    check_forward(prob, *prob.call())


def test_few_rows_need_no_copies(lib):  # noqa: F811
    """Up to 16 rows the product is one pass over the weights at any alignment: there is nothing to copy, however large and odd they are."""
    import torch

    for rows in (1, 16):
        for dtype in (torch.float16, torch.float32):
            assert fnn.fnn_linear_workspace_bytes(rows, 50001, 250001, dtype) == 0
    assert fnn.fnn_linear_workspace_bytes(17, 50001, 250001, torch.float16) > 2 * 50001 * 250001
