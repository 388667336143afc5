"""Clipping of networks of wide strided rows, few of them and many, and of rows that lie in one another's gaps."""
import math

import pytest
import torch

from test_gpu_clip import check, clip, grads

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ebs():
    from paper_2003_07577_b200 import binding
    return binding


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows,cols,pad", [(512, 4090, 6), (64, 4090, 5), (1000, 8100, 3), (300, 1537, 1), (9, 4095, 1), (2000, 4000, 8), (8, 8192, 8)])
@pytest.mark.parametrize("ratio", [0.3, 2.0])
def test_wide_rows(ebs, dtype, rows, cols, pad, ratio):
    big = grads(1, [((rows, cols + pad), dtype)])[0]
    t, between = big[:, :cols], big[:, cols:]
    between.fill_(math.nan)
    out = torch.full((rows, cols + 8), 7.0, dtype=dtype, device="cuda")
    max_norm = ratio * 0.01 * math.sqrt(rows * cols)
    kept = t.clone()
    check([kept], [out[:, :cols]], clip(ebs, [t], max_norm, [out[:, :cols]]), max_norm)
    assert (out[:, cols:] == 7.0).all()
    check([kept], [t], clip(ebs, [t], max_norm), max_norm)
    assert between.isnan().all()


def test_rows_in_the_gaps_of_a_matrix(ebs):
    big = grads(2, [((40, 1000), torch.float32)])[0]
    parts = [big[:, :600], big[0:1, 600:], big[1, 600:999], big[39, 700:]]
    kept, rest = [p.clone() for p in parts], big[2:39, 600:].clone()
    check(kept, parts, clip(ebs, parts, 0.05), 0.05)
    assert torch.equal(big[2:39, 600:], rest)
