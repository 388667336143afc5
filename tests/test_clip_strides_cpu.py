"""Clipping of gradients: which tensors the binding takes as rows of memory (host arithmetic: no GPU needed)."""
import pytest
import torch


@pytest.fixture(scope="module")
def ebs():
    import paper_2003_07577_b200 as pkg
    pkg.build()
    return pkg.binding


EXPANDED = [torch.zeros(1, 8).expand(4, 8), torch.zeros(8).expand(4, 8), torch.zeros(1, 1).expand(4, 1), torch.zeros(3, 1)[1:2].expand(5, 1),
            torch.zeros(32).as_strided((4, 8), (3, 1)), torch.zeros(1, 3, 8).expand(2, 3, 8), torch.zeros(1).expand(6), torch.zeros(4, 1).expand(4, 8)]


@pytest.mark.parametrize("t", EXPANDED, ids=lambda t: f"{tuple(t.shape)}-{t.stride()}")
def test_rows_that_share_memory_are_refused(ebs, t):
    """A row stride of 0 means dense to the library: the list would reach behind such a tensor's memory."""
    with pytest.raises(ValueError):
        ebs._clip_rows(t)
    with pytest.raises(ValueError):
        ebs._clip_record(t, t)
    with pytest.raises(ValueError):
        ebs._clip_record(t, torch.zeros(t.shape))
    with pytest.raises(ValueError):
        ebs._clip_record(torch.zeros(t.shape), t)


def test_one_row_may_have_any_stride(ebs):
    assert ebs._clip_rows(torch.zeros(1, 8).expand(1, 8)) == (1, 8, 8)
    assert ebs._clip_rows(torch.zeros(8).as_strided((1, 8), (0, 1))) == (1, 8, 8)


@pytest.mark.parametrize("t,o,want", [
    (torch.zeros(4, 8), torch.zeros(4, 8), (1, 32, 32, 32)),
    (torch.zeros(4, 8), torch.zeros(4, 12)[:, :8], (4, 8, 8, 12)),
    (torch.zeros(4, 12)[:, :8], torch.zeros(4, 8), (4, 8, 12, 8)),
    (torch.zeros(4, 12)[:, :8], torch.zeros(4, 9)[:, 1:], (4, 8, 12, 9)),
    (torch.zeros(4, 3)[:, :1], torch.zeros(4, 1), (4, 1, 3, 1)),
])
def test_records(ebs, t, o, want):
    r = ebs._clip_record(t, o)
    assert (r.rows, r.cols, r.ld_in, r.ld_out) == want and (r.in_dev, r.out_dev) == (t.data_ptr(), o.data_ptr()) and r.dtype == ebs.EBS_F32
