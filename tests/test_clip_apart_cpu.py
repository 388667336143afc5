"""Clipping of gradients: which tensors lie apart (host arithmetic: no GPU needed)."""
import ctypes

import pytest
import torch

P = [0x10000000000 + (i << 36) for i in range(4)]      # aligned, far apart, never dereferenced


@pytest.fixture(scope="module")
def ebs():
    import paper_2003_07577_b200 as pkg
    pkg.build()
    return pkg.binding


def tensor(ebs, p, rows, cols, ld=0, dtype=0, out=None):
    return ebs.ebs_clip_tensor(p, p if out is None else out, rows, cols, ld, ld, dtype)


def plan(ebs, tensors):
    arr, n = (ebs.ebs_clip_tensor * len(tensors))(*tensors), ctypes.c_longlong(0)
    return ebs.lib().ebs_clip_plan(arr, len(tensors), None, ctypes.byref(n))


def test_a_row_between_strided_rows(ebs):
    """One row has no stride: whether it shares an element with a matrix goes by the matrix's rows."""
    matrix = lambda rows=10: tensor(ebs, P[0], rows, 60, 100)  # noqa: E731
    row = lambda at, cols, ld=0: tensor(ebs, P[0] + 4 * at, 1, cols, ld)  # noqa: E731
    ok, bad = ebs.EBS_OK, ebs.EBS_ERR_INVALID_ARG
    for at, cols, want in ((60, 40, ok), (60, 41, bad), (59, 2, bad), (59, 1, bad), (60, 1, ok), (99, 1, ok), (100, 1, bad), (860, 40, ok), (860, 41, bad), (960, 500, ok), (959, 1, bad),
                           (0, 60, bad), (160, 10, ok), (170, 30, ok), (170, 31, bad)):
        assert plan(ebs, [matrix(), row(at, cols)]) == plan(ebs, [row(at, cols), matrix()]) == want, (at, cols)
        assert plan(ebs, [matrix(), row(at, cols, 300)]) == (want if cols <= 300 else bad), (at, cols)
    for before, want in ((40, ok), (41, bad)):                  # a row that ends where the matrix begins
        assert plan(ebs, [matrix(), tensor(ebs, P[0] - 160, 1, before)]) == want
    # rows of several places of one matrix, and an output between another's rows
    assert plan(ebs, [matrix(), row(60, 20), row(80, 20), row(160, 40), row(960, 7)]) == ok
    assert plan(ebs, [matrix(), row(60, 21), row(80, 20)]) == bad
    assert plan(ebs, [matrix(), tensor(ebs, P[1], 1, 40, out=P[0] + 240)]) == ok and plan(ebs, [matrix(), tensor(ebs, P[1], 1, 40, out=P[0] + 236)]) == bad
    # a view of its first row's rest, as torch has it
    big = torch.zeros(10, 100)
    records_ = [ebs._clip_record(t, t) for t in (big[:, :60], big[0:1, 60:], big[1, 60:99])]
    assert plan(ebs, records_) == ok
