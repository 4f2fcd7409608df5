"""What is not finite in a row, a gradient or a factor goes where the formulas take it, and nowhere else."""
import pytest
import torch

import paper_2506_21263_amd as dlcx
from gpu_util import DEV
from test_gpu_adapter import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,m,n,r,count", [(40, 136, 72, 12, 8), (300, 127, 130, 33, 4), (5000, 64, 264, 20, 3),
                                              (700, 264, 520, 70, 4)])
def test_columns_beyond_a_rank_are_zeros_whatever_the_rows_hold(rows, m, n, r, count, dtype):
    c = Case(rows, m, n, r, count, dtype, ranks=True, outside=False)
    assert 1 in c.rank and (count < 4 or 0 in c.rank)
    _, h = c.forward()
    for row, what in ((0, float("nan")), (rows // 2, float("inf")), (rows - 1, float("-inf"))):
        c.x[row, row % n] = what
        c.dy[row, row % m] = what
    for a in range(count):  # one more in a row of every adapter
        at = (c.ids == a).nonzero()[:, 0]
        if len(at):
            c.x[at[-1], n - 1] = float("nan")
            c.dy[at[-1], m - 1] = float("nan")
    _, dq, dp = c.backward(h)
    for a in range(count):
        assert not dq[a, c.rank[a]:].any() and not dp[a, c.rank[a]:].any(), a
        if c.rank[a] and (c.ids == a).any():
            assert torch.isnan(dq[a, 0]).any() and torch.isnan(dp[a, 0]).any(), a
