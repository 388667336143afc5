"""The work list of clipped gradients: how strided matrices are cut (host arithmetic: no GPU needed)."""
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


def records(ebs, tensors):
    """(address, rows, columns, bytes of an element) of each record."""
    n = ebs.ebs_clip_plan(tensors)
    host = torch.zeros(max(1, n) * ebs.EBS_CLIP_CHUNK_BYTES, dtype=torch.uint8)
    ebs.ebs_clip_plan(tensors, host, n)
    return [(w[0], w[4] & 0xffffffff, w[4] >> 32, 2 if w[5] & 0xffffffff else 4) for w in host.view(torch.int64).view(-1, 6)[:n].tolist()]


@pytest.mark.parametrize("rows,cols,pad,dtype,most", [(512, 4090, 6, 0, 16384), (64, 4090, 6, 0, 16384), (8, 4000, 1, 0, 16384), (512, 8100, 5, 4, 16384), (900, 2049, 3, 0, 16384), (1000, 1300, 1, 0, 48 << 10),
                                                      (900, 2100, 3, 3, 48 << 10), (900, 510, 2, 0, 16384), (700, 33, 1, 3, 4096), (3000, 4000, 8, 0, 128 << 10), (5000, 2049, 1, 4, 48 << 10)])
def test_records_of_strided_rows(ebs, rows, cols, pad, dtype, most):
    """The last two have eight rows for every SM, the others are small: wide rows one by one, so that they are work for all blocks.  Every element is in one record."""
    size = 4 if dtype == 0 else 2
    list_ = records(ebs, [tensor(ebs, P[0], rows, cols, cols + pad, dtype)])
    assert max(r * c * s for _, r, c, s in list_) <= most
    seen = set()
    for at, r, c, s in list_:
        assert s == size and (at - P[0]) % size == 0
        for i in range(r):
            row, col = divmod((at - P[0]) // size + i * (cols + pad), cols + pad)
            assert row < rows and col + c <= cols and (row, col) not in seen
            seen.add((row, col))
    assert sum(r * c for _, r, c, _ in list_) == rows * cols and len(seen) == sum(r for _, r, _, _ in list_)
