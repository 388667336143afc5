"""Clipping of gradients: the work list, its refusals and those of the call (host arithmetic: no GPU needed)."""
import ctypes
import math

import pytest
import torch

CHUNK = 16384
P = [0x10000000000 + (i << 36) for i in range(8)]      # aligned, far apart, never dereferenced


@pytest.fixture(scope="module")
def ebs():
    import paper_2003_07577_b200 as pkg
    pkg.build()
    return pkg.binding


def tensor(ebs, p=P[0], out=None, rows=1, cols=100, ld_in=0, ld_out=0, dtype=0):
    return ebs.ebs_clip_tensor(p, p if out is None else out, rows, cols, ld_in, ld_out, dtype)


def plan(ebs, tensors):
    arr = (ebs.ebs_clip_tensor * max(1, len(tensors)))(*tensors)
    n = ctypes.c_longlong(0)
    rc = ebs.lib().ebs_clip_plan(arr, len(tensors), None, ctypes.byref(n))
    return rc, n.value


def covered(ebs, tensors):
    """Every element's (input, output, type) address, from the work list."""
    n = ebs.ebs_clip_plan(tensors)
    host = torch.zeros(max(1, n) * ebs.EBS_CLIP_CHUNK_BYTES, dtype=torch.uint8)
    assert ebs.ebs_clip_plan(tensors, host, n) == n
    seen = []
    words = host.view(torch.int64).view(-1, 6)[:n]
    for w in words.tolist():
        rows, cols, dtype = w[4] & 0xffffffff, w[4] >> 32, w[5] & 0xffffffff
        size = 4 if dtype == 0 else 2
        assert rows >= 1 and 1 <= cols <= CHUNK and (rows == 1 or cols * size <= 16384)
        for r in range(rows):
            for c in range(cols):
                seen.append((w[0] + (r * w[2] + c) * size, w[1] + (r * w[3] + c) * size, dtype))
    return seen


@pytest.mark.parametrize("shapes", [
    [(1, 1, 0, 0, 0)], [(1, CHUNK, 0, 0, 0)], [(1, CHUNK + 1, 0, 0, 4)], [(3, 5, 7, 9, 3)], [(100, 300, 301, 300, 0)], [(2, CHUNK + 3, CHUNK + 8, 0, 4)],
    [(300, 1, 2, 1, 3), (0, 5, 0, 0, 0), (5, 0, 0, 0, 0), (7, 9, 9, 9, 0), (1, 3 * CHUNK - 1, 0, 0, 3)], [],
])
def test_every_element_is_in_the_list_once(ebs, shapes):
    ts, want = [], []
    for i, (rows, cols, ld_in, ld_out, dtype) in enumerate(shapes):
        p, q, size = P[i] + 4 * i, P[i] + (1 << 34), 4 if dtype == 0 else 2
        ts.append(tensor(ebs, p, q, rows, cols, ld_in, ld_out, dtype))
        want += [(p + (r * (ld_in or cols) + c) * size, q + (r * (ld_out or cols) + c) * size, dtype) for r in range(rows) for c in range(cols)]
    assert sorted(covered(ebs, ts)) == sorted(want)


def test_refused_tensors(ebs):
    bad = ebs.EBS_ERR_INVALID_ARG
    for change in (dict(rows=-1), dict(cols=-2), dict(dtype=1), dict(dtype=5), dict(rows=3, ld_in=99), dict(rows=3, ld_out=99), dict(p=P[0] + 2),
                   dict(out=P[1] + 2), dict(p=0), dict(out=0), dict(rows=2, ld_in=128), dict(dtype=3, p=P[0] + 1)):
        assert plan(ebs, [tensor(ebs, **change)])[0] == bad, change
    for change in (dict(cols=(1 << 40) + 1), dict(rows=1 << 30, cols=1 << 11), dict(rows=4, ld_in=1 << 39, ld_out=1 << 39), dict(rows=1 << 62)):
        assert plan(ebs, [tensor(ebs, **change)])[0] == ebs.EBS_ERR_OVERFLOW, change
    n = ctypes.c_longlong(0)
    assert ebs.lib().ebs_clip_plan(None, 1, None, ctypes.byref(n)) == bad
    assert ebs.lib().ebs_clip_plan(None, -1, None, ctypes.byref(n)) == bad
    assert ebs.lib().ebs_clip_plan(None, 0, None, None) == bad
    assert plan(ebs, []) == (0, 0)
    # a list that does not fit where it is to be written
    arr, n = (ebs.ebs_clip_tensor * 1)(tensor(ebs, cols=CHUNK + 1)), ctypes.c_longlong(1)
    assert ebs.lib().ebs_clip_plan(arr, 1, (ctypes.c_char * 48)(), ctypes.byref(n)) == bad


def test_overlaps(ebs):
    bad = ebs.EBS_ERR_INVALID_ARG
    a, q = P[0], P[1]
    assert plan(ebs, [tensor(ebs, a), tensor(ebs, a)])[0] == bad                               # twice in place
    assert plan(ebs, [tensor(ebs, a), tensor(ebs, a + 396)])[0] == bad                         # the last element
    assert plan(ebs, [tensor(ebs, a), tensor(ebs, a + 400)]) == (0, 2)
    assert plan(ebs, [tensor(ebs, a, a + 16)])[0] == bad                                       # shifted onto itself
    assert plan(ebs, [tensor(ebs, a, q), tensor(ebs, a, q + 400)]) == (0, 2)                   # an input twice
    assert plan(ebs, [tensor(ebs, a, q), tensor(ebs, a + 4000, q + 396)])[0] == bad            # outputs that meet
    assert plan(ebs, [tensor(ebs, a, q), tensor(ebs, q + 100, P[2])])[0] == bad                # an output that is another's input
    left = tensor(ebs, a, rows=10, cols=60, ld_in=100, ld_out=100)
    assert plan(ebs, [left, tensor(ebs, a + 240, rows=10, cols=40, ld_in=100, ld_out=100)]) == (0, 2)      # column ranges of one matrix
    assert plan(ebs, [left, tensor(ebs, a + 236, rows=10, cols=40, ld_in=100, ld_out=100)])[0] == bad
    assert plan(ebs, [left, tensor(ebs, a + 240, rows=10, cols=41, ld_in=100, ld_out=100)])[0] == bad
    assert plan(ebs, [tensor(ebs, a), tensor(ebs, 0, rows=0)]) == (0, 1)                       # an empty one is nowhere


def test_call_refusals(ebs):
    bad, call = ebs.EBS_ERR_INVALID_ARG, ebs.lib().ebs_clip_gradients
    need = ebs.ebs_clip_workspace_bytes(10)
    assert need >= 80 and ebs.ebs_clip_workspace_bytes(0) > 0 and ebs.ebs_clip_workspace_bytes(1 << 31) == ebs.ebs_clip_workspace_bytes(1184)
    assert ebs.ebs_clip_workspace_bytes(-1) == ebs.ebs_clip_workspace_bytes((1 << 31) + 1) == 0
    good = dict(plan=P[0], chunks=10, max_norm=1.0, norm=P[1], ws=P[2], bytes=need)
    for change in (dict(plan=None), dict(chunks=-1), dict(chunks=(1 << 31) + 1), dict(max_norm=-1.0), dict(max_norm=math.nan), dict(norm=None), dict(ws=None),
                   dict(bytes=need - 1), dict(plan=P[0] + 8), dict(norm=P[1] + 2), dict(ws=P[2] + 8)):
        a = {**good, **change}
        assert call(a["plan"], a["chunks"], a["max_norm"], a["norm"], a["ws"], a["bytes"], None) == bad, change


def test_binding_refusals(ebs):
    for t in (torch.zeros(4), torch.zeros(4, dtype=torch.int32), torch.zeros(4, dtype=torch.float64)):
        with pytest.raises(ValueError):
            ebs.clip_plan([t])
    with pytest.raises(ValueError):
        ebs.clip_plan([torch.zeros(4)], [])
    for t in (torch.zeros(4, 6).t(), torch.zeros(2, 3, 8)[:, :, :4], torch.zeros(8)[::2]):
        with pytest.raises(ValueError):
            ebs._clip_rows(t)
    assert ebs._clip_rows(torch.zeros(4, 8)[:, :5]) == (4, 5, 8) and ebs._clip_rows(torch.zeros(4, 8)) == (1, 32, 32) and ebs._clip_rows(torch.zeros(0, 3))[1] == 0
    assert ebs._clip_rows(torch.zeros(4, 8)[:, :1]) == (4, 1, 8)
