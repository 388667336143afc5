"""Refusals and sizes of the real-valued operators: validation happens on the host before anything is launched (no GPU needed)."""
import ctypes
import math

import pytest
import torch


@pytest.fixture(scope="module")
def ebs():
    import paper_2003_07577_b200 as pkg
    pkg.build()
    return pkg.binding


P = [ctypes.c_void_p(0x10000000000 + (i << 36)) for i in range(8)]      # aligned, far apart, never dereferenced: validation fails first


def fwd(ebs, d, x=P[0], w=P[1], bias=None, res=None, y=P[2], z=None, ws=P[7], ws_bytes=1 << 36):
    return ebs.lib().ebs_linear_forward(x, w, bias, res, None if d is None else ctypes.byref(d), y, z, ws, ws_bytes, None)


def bwd(ebs, d, dy=P[0], x=P[1], w=P[2], z=P[3], dx=P[4], dw=P[5], db=None, ws=P[7], ws_bytes=1 << 36):
    return ebs.lib().ebs_linear_backward(dy, x, w, z, ctypes.byref(d), dx, dw, db, ws, ws_bytes, None)


def off(p, n):
    return ctypes.c_void_p(p.value + n)


@pytest.mark.parametrize("change", [dict(m=-1), dict(n=0), dict(k=0), dict(k=-5), dict(dtype=1), dict(dtype=2), dict(dtype=5), dict(dtype=-1), dict(act=5),
                                    dict(act=-1), dict(ldx=31), dict(ldw=31), dict(ldy=63), dict(ldr=63), dict(ldz=63), dict(ldx=-40)])
def test_descriptors(ebs, change):
    args = dict(m=16, n=64, k=32, dtype=ebs.EBS_BF16, act=ebs.EBS_ACT_GELU)
    args.update(change)
    d = ebs.linear_desc(**args)
    assert fwd(ebs, d) == bwd(ebs, d) == ebs.EBS_ERR_INVALID_ARG
    assert ebs.ebs_linear_workspace_bytes(d) == ebs.ebs_linear_workspace_bytes(d, True) == 0


def test_sizes_beyond_the_index_range(ebs):
    for change in (dict(ldx=1 << 40), dict(ldw=1 << 36), dict(ldy=1 << 37), dict(ldz=1 << 62), dict(ldr=(1 << 63) - 1)):
        d = ebs.linear_desc(1024, 1024, 32, ebs.EBS_BF16, **change)
        assert fwd(ebs, d) == ebs.EBS_ERR_OVERFLOW and ebs.ebs_linear_workspace_bytes(d) == 0


def test_missing_and_misaligned_buffers(ebs):
    bad = ebs.EBS_ERR_INVALID_ARG
    d = ebs.linear_desc(16, 64, 32, ebs.EBS_F32, ebs.EBS_ACT_SILU)
    assert fwd(ebs, None) == bad
    for name in ("x", "w", "y"):
        assert fwd(ebs, d, **{name: None}) == bad
    for name, p in (("x", P[0]), ("w", P[1]), ("bias", P[3]), ("res", P[4]), ("y", P[2]), ("z", P[5])):
        assert fwd(ebs, d, **{name: off(p, 4)}) == bad
    for name in ("dy", "x", "w", "z"):
        assert bwd(ebs, d, **{name: None}) == bad
    for name, p in (("dy", P[0]), ("x", P[1]), ("w", P[2]), ("z", P[3]), ("dx", P[4]), ("dw", P[5]), ("db", P[6]), ("ws", P[7])):
        assert bwd(ebs, d, **{name: off(p, 8)}) == bad
    assert bwd(ebs, d, dx=None, dw=None) == bad                          # nothing wanted
    need = ebs.ebs_linear_workspace_bytes(d, True)
    assert need > 0 and bwd(ebs, d, ws=None) == bad and bwd(ebs, d, ws_bytes=need - 1) == bad


def test_overlaps(ebs):
    bad = ebs.EBS_ERR_INVALID_ARG
    d = ebs.linear_desc(16, 64, 32, ebs.EBS_F32, ebs.EBS_ACT_NONE)
    y_bytes = 16 * 64 * 4
    for name in ("x", "w", "bias", "z"):
        assert fwd(ebs, d, **{name: P[2]}) == bad
        assert fwd(ebs, d, **{name: off(P[2], y_bytes - 16)}) == bad
    assert fwd(ebs, d, res=off(P[2], 16)) == bad                         # the residual itself is fine, a shifted one is not
    strided = ebs.linear_desc(16, 64, 32, ebs.EBS_F32, ebs.EBS_ACT_NONE, ldr=80)
    assert fwd(ebs, strided, res=P[2]) == bad                            # the same address with another stride
    g = ebs.linear_desc(16, 64, 32, ebs.EBS_F32, ebs.EBS_ACT_RELU)
    for a in ("dx", "dw", "db"):
        for q in (P[0], P[1], P[2], P[3], P[7]):
            assert bwd(ebs, g, **{a: q}) == bad
    assert bwd(ebs, g, dx=P[5]) == bad
    # columns 0..63 and 60..91 of rows of 128 share elements (64..95 would not)
    rows = ebs.linear_desc(16, 64, 32, ebs.EBS_F32, ebs.EBS_ACT_NONE, ldx=128, ldy=128)
    assert fwd(ebs, rows, x=off(P[2], 60 * 4)) == bad
    assert fwd(ebs, rows, x=off(P[2], (128 - 28) * 4)) == bad


def ortho(ebs, batch=2, rows=8, cols=12, dtype=0, steps=5, coeff=(3.0, -3.0, 1.0), eps=1e-7, scale=1.0, g=P[0], out=P[1], ws=P[7], ws_bytes=1 << 36):
    c = None if coeff is None else (ctypes.c_float * 3)(*coeff)
    return ebs.lib().ebs_orthogonalize(g, batch, rows, cols, dtype, steps, c, eps, scale, out, ws, ws_bytes, None)


def test_orthogonalize_refusals(ebs):
    bad = ebs.EBS_ERR_INVALID_ARG
    for change in (dict(batch=0), dict(rows=0), dict(cols=-1), dict(dtype=1), dict(dtype=5), dict(steps=-1), dict(steps=65), dict(coeff=None),
                   dict(coeff=(math.nan, 0, 0)), dict(coeff=(1, math.inf, 0)), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf), dict(scale=math.nan),
                   dict(scale=-math.inf), dict(g=None), dict(out=None), dict(ws=None), dict(g=off(P[0], 4)), dict(out=off(P[1], 8)), dict(ws=off(P[7], 2)),
                   dict(out=off(P[0], 16)), dict(ws=P[0]), dict(ws=P[1]), dict(ws_bytes=ebs.ebs_orthogonalize_workspace_bytes(2, 8, 12, 0, 5) - 1)):
        assert ortho(ebs, **change) == bad, change
    assert ortho(ebs, coeff=(1000.0, 0.0, 0.0), steps=9) == ebs.EBS_ERR_UNSUPPORTED
    assert ortho(ebs, coeff=(0.0, 0.0, 0.0)) == ebs.EBS_ERR_UNSUPPORTED
    assert ortho(ebs, batch=70000, rows=1 << 15, cols=1 << 15) == ebs.EBS_ERR_OVERFLOW
    assert ebs.ebs_orthogonalize_workspace_bytes(0, 8, 8, 0, 5) == ebs.ebs_orthogonalize_workspace_bytes(1, 8, 8, 1, 5) == 0
    assert ebs.ebs_orthogonalize_workspace_bytes(1, 8, 8, 0, 5) > 0


def test_fast_path_types(ebs):
    """The extension takes what the library takes, and refuses other types before it is reached."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(ebs.__file__), "_fastcall.so")
    spec = importlib.util.spec_from_file_location("_fastcall", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    L = ebs.lib()
    first = ("ebs_pack_acts", "ebs_pack_acts_s2d", "ebs_conv2d_mixed", "ebs_conv2d_mixed_variant", "ebs_dequant", "ebs_global_avgpool", "ebs_maxpool_packed",
             "ebs_resnet_cifar_forward", "ebs_search_weight_forward", "ebs_search_act_forward", "ebs_graph_launch")
    names = first + ("ebs_linear_forward", "ebs_linear_backward", "ebs_orthogonalize")
    m.bind({k: ctypes.cast(getattr(L, k), ctypes.c_void_p).value for k in names}, lambda device: 0, lambda: 0, ebs.ebs_conv_desc, ebs.ebs_epilogue,
           ebs.ebs_fused_head, ebs.ebs_linear_desc)
    try:
        d = ebs.linear_desc(4, 4, 4)
        assert m.linear_forward(None, None, None, None, d, None, None, None, None) == ebs.EBS_ERR_INVALID_ARG
        assert m.linear_backward(None, None, None, None, d, None, None, None, None, None) == ebs.EBS_ERR_INVALID_ARG
        assert m.orthogonalize(None, 1, 4, 4, 0, 5, (1, 2, 3), 0.0, 1.0, None, None, None) == ebs.EBS_ERR_INVALID_ARG
        for wrong in (None, bytes(d), ebs.conv_desc(8, 8, 1, 1, 1, 1, 0, 0, 2, 2, 0.1, 0.1)):
            with pytest.raises(TypeError):
                m.linear_forward(None, None, None, None, wrong, None, None, None, None)
        for coeff, error in ((3.0, TypeError), ((1.0, 2.0), ValueError), ((1.0, "x", 2.0), TypeError)):
            with pytest.raises(error):
                m.orthogonalize(None, 1, 4, 4, 0, 5, coeff, 0.0, 1.0, None, None, None)
        with pytest.raises(TypeError):
            m.orthogonalize(None, 1.5, 4, 4, 0, 5, (1, 2, 3), 0.0, 1.0, None, None, None)
        ws = torch.empty(64, dtype=torch.uint8)
        assert m.linear_forward(None, None, None, None, d, None, None, ws, None) == ebs.EBS_ERR_INVALID_ARG
    finally:
        ebs._fast = None


def test_orthogonalize_sides_beyond_the_index_range(ebs):
    """Tiles and stages of 32-bit counts: a side of more than 2^30 is refused, whichever it is, by the size query too."""
    for rows, cols in (((1 << 30) + 1, 1), (1, (1 << 30) + 1), ((1 << 31) - 1, 1), (1, (1 << 31) - 1), ((1 << 31) - 64, 17), (8, (1 << 31) - 200)):
        assert ortho(ebs, batch=1, rows=rows, cols=cols, ws_bytes=1 << 62) == ebs.EBS_ERR_OVERFLOW
        assert ebs.ebs_orthogonalize_workspace_bytes(1, rows, cols, 0, 5) == 0
    assert ebs.ebs_orthogonalize_workspace_bytes(1, 1 << 30, 1, 0, 5) > 0


def first_plane(t):
    """What is left of a matrix kept as its first fp16 plane alone."""
    scale = 2.0 ** 13 / 2.0 ** math.ceil(math.log2(float(t.abs().max())))
    return (t * scale).half().double() / scale


def orthogonalize_without(g, steps, coeff, matrix, step):
    """The iteration in 64 bits, but for one matrix of one step that lost its second plane."""
    a, b, c = coeff
    x = g.double() / (g.double().norm() + 1e-7)
    for i in range(steps):
        lost = lambda name, t: first_plane(t) if (name, i) == (matrix, step) else t  # noqa: E731
        s = x @ x.T
        p = lost("A", s)
        q = lost("Q", a * torch.eye(len(s), dtype=torch.float64) + b * p + c * (p @ p))
        x = q @ lost("X", x)
    return x.float()[None]


def test_orthogonalize_tolerance_notices_a_lost_plane():
    """The tolerance of the tests with a few steps (test_gpu_orthogonalize.py) passes the iteration and none that lost a plane."""
    from test_gpu_orthogonalize import FEW_STEPS, check, iterate64
    gen = torch.Generator().manual_seed(0)
    noticed = set()
    for rows, cols in ((64, 576), (128, 1152), (300, 700)):
        for rank, steps, coeff in FEW_STEPS:
            g = torch.randn((rows, cols), generator=gen) if rank is None else torch.randn((rows, rank), generator=gen) @ torch.randn((rank, cols), generator=gen)
            ref = iterate64(g[None], steps, coeff)
            check(orthogonalize_without(g, steps, coeff, None, 0), ref, steps, coeff)
            for matrix in "XAQ":
                for step in range(steps):
                    try:
                        check(orthogonalize_without(g, steps, coeff, matrix, step), ref, steps, coeff)
                    except AssertionError:
                        noticed.add((rows, matrix, rank))
    for rows in (64, 128, 300):
        assert {(rows, "X", None), (rows, "Q", None), (rows, "X", 1), (rows, "Q", 1), (rows, "A", 1)} <= noticed
