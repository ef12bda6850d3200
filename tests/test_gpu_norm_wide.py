"""Layer norm's column sums where they take several launches."""

import pytest
import torch

import paper_2609_02846_amd as ue
from gpu_util import say

pytestmark = pytest.mark.gpu


def test_column_sums_of_more_than_2_28_columns():
    """Whole numbers under a mean of 0 and a factor of 1: every sum is exact."""
    rows, cols = 2, 2 ** 28 + 72
    say("norm wide", rows, cols)
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dy = (torch.randint(-3, 4, (rows, cols), generator=g, dtype=torch.int8, device="cuda").to(torch.bfloat16)
             for _ in range(2))
    mean, rstd = torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda")
    dx, dw, db = ue.layer_norm_grad(x, dy, None, mean, rstd, need=(False, True, True))
    assert dx is None and torch.equal(dw, x[0] * dy[0] + x[1] * dy[1]) and torch.equal(db, dy[0] + dy[1])
