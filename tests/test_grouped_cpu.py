"""Layers of experts: sizes and refusals (validation on the host, no GPU needed)."""
import ctypes

import pytest

P = [ctypes.c_void_p(0x10000000000 + (i << 40)) for i in range(10)]      # aligned, far apart, never dereferenced


@pytest.fixture(scope="module")
def ebs():
    import paper_2003_07577_b200 as pkg
    pkg.build()
    return pkg.binding


def off(p, n):
    return ctypes.c_void_p(p.value + n)


def fwd(ebs, d, experts=4, x=P[0], w=P[1], bias=None, res=None, offsets=P[8], y=P[2], z=None, ws=P[7], ws_bytes=1 << 39):
    return ebs.lib().ebs_grouped_forward(x, w, bias, res, offsets, experts, None if d is None else ctypes.byref(d), y, z, ws, ws_bytes, None)


def bwd(ebs, d, experts=4, dy=P[0], x=P[1], w=P[2], z=P[3], offsets=P[8], dx=P[4], dw=P[5], db=None, ws=P[7], ws_bytes=1 << 39):
    return ebs.lib().ebs_grouped_backward(dy, x, w, z, offsets, experts, None if d is None else ctypes.byref(d), dx, dw, db, ws, ws_bytes, None)


@pytest.mark.parametrize("change", [dict(m=-1), dict(n=0), dict(k=0), dict(dtype=1), dict(dtype=2), dict(dtype=5), dict(act=5), dict(act=-1), dict(ldx=31), dict(ldw=31),
                                    dict(ldy=63), dict(ldr=63), dict(ldz=63), dict(experts=0), dict(experts=-2)])
def test_descriptors(ebs, change):
    args = dict(m=16, n=64, k=32, dtype=ebs.EBS_BF16, act=ebs.EBS_ACT_GELU)
    experts = change.get("experts", 4)
    args.update({a: b for a, b in change.items() if a != "experts"})
    d = ebs.linear_desc(**args)
    assert fwd(ebs, d, experts) == bwd(ebs, d, experts) == ebs.EBS_ERR_INVALID_ARG
    assert ebs.ebs_grouped_workspace_bytes(d, experts) == ebs.ebs_grouped_workspace_bytes(d, experts, True) == 0


def test_types_and_sizes_without_a_kernel(ebs):
    d = ebs.linear_desc(16, 64, 32, ebs.EBS_F32)
    assert fwd(ebs, d) == bwd(ebs, d) == ebs.EBS_ERR_UNSUPPORTED and ebs.ebs_grouped_workspace_bytes(d, 4) == 0
    for experts, args in ((1 << 20, dict(m=16, n=1 << 12, k=1 << 10)), (4, dict(m=16, n=64, k=32, ldw=1 << 35)), (1, dict(m=1 << 30, n=8, k=8)), (1 << 30, dict(m=1, n=8, k=8))):
        d = ebs.linear_desc(dtype=ebs.EBS_BF16, **args)
        assert fwd(ebs, d, experts) == bwd(ebs, d, experts) == ebs.EBS_ERR_OVERFLOW, args


def test_refusals(ebs):
    bad = ebs.EBS_ERR_INVALID_ARG
    d = ebs.linear_desc(16, 64, 33, ebs.EBS_F16, ebs.EBS_ACT_SILU)
    assert fwd(ebs, None) == bwd(ebs, None) == bad
    need = ebs.ebs_grouped_workspace_bytes(d, 4)
    assert need >= 2 * 40 * (16 + 4 * 64)                                # rows that start anywhere are copied
    y_bytes = 16 * 64 * 2
    for change in (dict(x=None), dict(w=None), dict(y=None), dict(offsets=None), dict(offsets=off(P[8], 2)), dict(x=off(P[0], 2)), dict(w=off(P[1], 8)), dict(y=off(P[2], 4)),
                   dict(z=off(P[3], 4)), dict(bias=off(P[3], 2)), dict(res=off(P[3], 2)), dict(ws=None), dict(ws_bytes=need - 1), dict(ws=off(P[7], 4)), dict(x=P[2]), dict(w=P[2]),
                   dict(bias=P[2]), dict(z=P[2]), dict(res=off(P[2], 16)), dict(ws=P[2]), dict(offsets=P[2]), dict(offsets=off(P[2], y_bytes - 4)), dict(offsets=off(P[2], -16)),
                   dict(offsets=P[7]), dict(w=off(P[2], -16 - 2 * 33 * 4 * 64 + 32))):
        assert fwd(ebs, d, **change) == bad, change
    need = ebs.ebs_grouped_workspace_bytes(d, 4, True)
    for change in (dict(dy=None), dict(x=None), dict(w=None), dict(z=None), dict(offsets=None), dict(dx=None, dw=None), dict(ws=None), dict(ws_bytes=need - 1), dict(dx=P[0]), dict(dw=P[2]),
                   dict(dx=P[5]), dict(db=P[4]), dict(db=P[8]), dict(dw=off(P[8], -32)), dict(db=off(P[6], 4)), dict(dy=off(P[0], 8)), dict(z=P[4])):
        assert bwd(ebs, d, **change) == bad, change
    empty = ebs.linear_desc(0, 64, 32, ebs.EBS_F16)
    assert fwd(ebs, empty, x=None, y=None, ws=None, ws_bytes=0) == ebs.EBS_OK       # no rows: nothing is launched
