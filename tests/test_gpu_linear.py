"""GPU parity of the real-valued layers (forward and backward) against the formulas in 64 bits.

Tolerances, from the arithmetic alone.  u = eps/2 is the rounding of one output (relative to its value).  A sum of K products
in fp32 carries at most about K roundings of 2^-24 of the sum of the products' magnitudes, S; in practice the square root of that,
and sums here are taken in blocks, so 2^-24 * (8 + sqrt(K)) * 4 * S is generous; operands of fp32 are kept to 22 bits
(2^-22 of every product).  An activation passes an error on with a slope of at most 1.13, and its own evaluation in fp32 costs
a few 2^-24 of (1 + |z|).  The backward pass of a 16-bit type with an activation rounds dz first: u more of every product."""
import math
import os
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


@pytest.fixture(scope="module")
def ebs():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    import paper_2003_07577_b200 as pkg
    from paper_2003_07577_b200 import binding
    if not os.path.exists(binding.LIB_PATH):
        pkg.build()
    binding.lib()
    return binding


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def strided(rows, cols, ld, t, g, scale=1.0):
    """A [rows][cols] view with row stride ld; what lies between the rows is NaN."""
    full = torch.full((max(rows, 1), ld), math.nan, dtype=t, device="cuda")
    full[:, :cols] = (scale * torch.randn((max(rows, 1), cols), generator=g, device="cuda")).to(t)
    return full[:rows, :cols]


def act64(z, act):
    f = torch.nn.functional
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    return {"none": lambda v: v, "gelu": f.gelu, "gelu_tanh": lambda v: f.gelu(v, approximate="tanh"), "silu": f.silu}[act](z)


def bound(t, value, sums, K):
    """Allowed error of outputs `value` that are sums of K products whose magnitudes add up to `sums`."""
    u = torch.finfo(t).eps / 2
    tiny = torch.finfo(t).smallest_normal * torch.finfo(t).eps
    return u * value.abs() + sums * (4 * 2.0 ** -24 * (8 + math.sqrt(K)) + (2.0 ** -22 if t == torch.float32 else 0)) * (1 + u) + 8 * 2.0 ** -24 * (1 + value.abs()) + tiny


def codes(ebs, dtype, act):
    return ({"f32": ebs.EBS_F32, "f16": ebs.EBS_F16, "bf16": ebs.EBS_BF16}[dtype],
            {"none": ebs.EBS_ACT_NONE, "relu": ebs.EBS_ACT_RELU, "gelu": ebs.EBS_ACT_GELU, "gelu_tanh": ebs.EBS_ACT_GELU_TANH,
             "silu": ebs.EBS_ACT_SILU}[act])


def workspace(ebs, desc, backward, fill=0xFF):
    b = ebs.ebs_linear_workspace_bytes(desc, backward)
    return torch.full((b + 256,), fill, dtype=torch.uint8, device="cuda")[:b] if b else None


def run_forward(ebs, x, w, bias, residual, dtype, act, y, z=None, stream=None, ws=None):
    dt, ac = codes(ebs, dtype, act)
    ld = lambda t: 0 if t is None or t.shape[0] < 2 else t.stride(0)  # noqa: E731
    d = ebs.linear_desc(x.shape[0], w.shape[0], w.shape[1], dt, ac, ld(x), ld(w), ld(y), ld(residual), ld(z))
    ws = workspace(ebs, d, False) if ws is None else ws
    ebs.ebs_linear_forward(x, w, bias, residual, d, y, z, ws, stream)
    return ws


def check_forward(ebs, m, n, k, dtype, act, bias=True, residual=True, keep_z=True, pads=(0, 0, 0, 0, 0), seed=0, in_place=False):
    t, g = TYPES[dtype], gen(seed)
    x, w = strided(m, k, k + pads[0], t, g), strided(n, k, k + pads[1], t, g, 1 / math.sqrt(k))
    b = (0.3 * torch.randn(n, generator=g, device="cuda")).to(t) if bias else None
    r = strided(m, n, n + pads[3], t, g) if residual else None
    y = strided(m, n, n + pads[2], t, g) if not in_place else r
    z = strided(m, n, n + pads[4], t, g) if keep_z else None
    xd, wd = x.double(), w.double()
    z64 = xd @ wd.T + (b.double() if bias else 0.0)
    sums = xd.abs() @ wd.abs().T + (b.double().abs() if bias else 0.0)
    y64 = act64(z64, act) + (r.double() if residual else 0.0)
    run_forward(ebs, x, w, b, r, dtype, act, y, z)
    torch.cuda.synchronize()
    # the residual's addition: one more rounding of the terms
    extra = 2.0 ** -23 * (act64(z64, act).abs() + (r.double().abs() if residual and not in_place else y64.abs() + 4))
    assert ((y.double() - y64).abs() <= bound(t, y64, 1.13 * sums, k) + extra).all()
    if keep_z:
        assert ((z.double() - z64).abs() <= bound(t, z64, sums, k)).all()
    for v, p in ((y, pads[2]), (z, pads[4])):                # between the rows: left as it was
        if v is not None and p and m > 1 and not in_place:
            assert torch.isnan(torch.as_strided(v, (m - 1, p), (v.stride(0), 1), v.storage_offset() + n)).all()


SHAPES = [(1, 1, 1), (1, 1000, 512), (2, 7, 3), (3, 4096, 4096), (5, 33, 129), (8, 256, 64), (16, 130, 1027), (17, 64, 31), (31, 65, 512),
          (64, 1000, 512), (127, 129, 63), (128, 128, 128), (129, 257, 65), (250, 333, 1027), (256, 512, 2048), (300, 8, 4096), (1000, 1, 77),
          (777, 2048, 40), (1024, 768, 1), (2049, 320, 576)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_forward_sizes(ebs, m, n, k, dtype):
    check_forward(ebs, m, n, k, dtype, ACTS[(m + n + k) % 5], seed=m + n + k)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("parts", range(8))
@pytest.mark.parametrize("m", [3, 200])
def test_forward_parts(ebs, dtype, act, parts, m):
    check_forward(ebs, m, 136, 96, dtype, act, bool(parts & 1), bool(parts & 2), bool(parts & 4), seed=parts)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("pads", [(8, 8, 8, 8, 8), (1, 0, 0, 0, 0), (0, 3, 0, 0, 0), (0, 0, 5, 0, 0), (0, 0, 0, 7, 0), (0, 0, 0, 0, 1), (3, 1, 2, 5, 4)])
@pytest.mark.parametrize("m,n,k", [(4, 96, 200), (150, 200, 72), (40, 37, 129)])
def test_forward_strides(ebs, dtype, pads, m, n, k):
    check_forward(ebs, m, n, k, dtype, "gelu", pads=pads)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("m", [1, 6, 140, 1300])
def test_forward_in_place_residual(ebs, dtype, m):
    t, g = TYPES[dtype], gen(m)
    x, w, r = strided(m, 72, 72, t, g), strided(200, 72, 72, t, g, 0.1), strided(m, 200, 200, t, g)
    apart = torch.empty_like(r)
    run_forward(ebs, x, w, None, r, dtype, "silu", apart)
    run_forward(ebs, x, w, None, r, dtype, "silu", r)
    assert torch.equal(apart, r)


def check_backward(ebs, m, n, k, dtype, act, pads=(0, 0, 0, 0), want=(True, True, True), seed=0):
    t, g = TYPES[dtype], gen(seed)
    x, w = strided(m, k, k + pads[0], t, g), strided(n, k, k + pads[1], t, g, 1 / math.sqrt(k))
    dy = strided(m, n, n + pads[2], t, g)
    z = strided(m, n, n + pads[3], t, g, 1.5) if act != "none" else None
    dx, dw = strided(m, k, k + pads[0], t, g), strided(n, k, k + pads[1], t, g)
    db = torch.full((n,), math.nan, dtype=t, device="cuda")
    dt, ac = codes(ebs, dtype, act)
    d = ebs.linear_desc(m, n, k, dt, ac, k + pads[0], k + pads[1], n + pads[2], 0, n + pads[3])
    ebs.ebs_linear_backward(dy, x, w, z, d, dx if want[0] else None, dw if want[1] else None, db if want[2] else None, workspace(ebs, d, True))
    torch.cuda.synchronize()
    dz = dy.double()
    slack = 2.0 ** -23 * 4
    if z is not None:
        z64 = z.double().requires_grad_(True)
        if act == "relu":
            dz = dz * (z64 > 0)
        else:
            (dz,) = torch.autograd.grad(act64(z64, act), z64, dz)
        slack += torch.finfo(t).eps / 2 if t != torch.float32 else 0.0      # dz rounded to the type
    mag = dz.abs() + 2.0 ** -21 * dy.double().abs()                          # (a slope near zero is a difference: absolute error)
    if want[0]:
        dx64, s = dz @ w.double(), mag @ w.double().abs()
        assert ((dx.double() - dx64).abs() <= bound(t, dx64, s, n) + slack * s).all()
    if want[1]:
        dw64, s = dz.T @ x.double(), mag.T @ x.double().abs()
        assert ((dw.double() - dw64).abs() <= bound(t, dw64, s, m) + slack * s).all()
    if want[2]:
        db64, s = dz.sum(0), mag.sum(0)
        assert ((db.double() - db64).abs() <= bound(t, db64, s, m) + slack * s).all()
    for v, p in ((dx, pads[0]), (dw, pads[1])):
        if p and v.shape[0] > 1:
            assert torch.isnan(torch.as_strided(v, (v.shape[0] - 1, p), (v.stride(0), 1), v.storage_offset() + k)).all()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_backward_sizes(ebs, m, n, k, dtype):
    check_backward(ebs, m, n, k, dtype, ACTS[(m + n + k) % 5], seed=m + n + k)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("want", [(1, 1, 1), (1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 1, 0), (0, 1, 1)])
def test_backward_parts(ebs, dtype, act, want):
    check_backward(ebs, 200, 136, 96, dtype, act, want=want)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("act", ["none", "gelu"])
@pytest.mark.parametrize("pads", [(8, 8, 8, 8), (1, 0, 0, 0), (0, 3, 0, 0), (0, 0, 5, 0), (0, 0, 0, 7), (3, 1, 2, 5)])
@pytest.mark.parametrize("m,n,k", [(4, 96, 200), (150, 200, 72), (40, 37, 129)])
def test_backward_strides(ebs, dtype, act, pads, m, n, k):
    check_backward(ebs, m, n, k, dtype, act, pads=pads)


# sizes of the persistent pair kernel (32 tiles of 256 x 256 and more; fp32 on 128 columns too), of a reduction in parts, and of both
# gradients in one launch; the result's rows start on 16 bytes (they leave by TMA, clipped at n) or anywhere
LARGE = [(2049, 1283, 200, (0, 0, 5, 5, 5)), (2049, 1283, 200, (3, 5, 0, 2, 1)), (2304, 1152, 64, (0,) * 5), (4100, 2050, 330, (6, 6, 6, 6, 6)), (300, 260, 8200, (0, 0, 4, 4, 4)), (2304, 1160, 131, (5, 5, 0, 0, 0)),
         (257, 129, 4104, (1, 0, 0, 0, 0)), (1531, 259, 517, (3, 0, 0, 0, 0))]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("m,n,k,pads", LARGE)
def test_forward_large(ebs, dtype, m, n, k, pads):
    check_forward(ebs, m, n, k, dtype, "gelu", pads=pads)
    check_forward(ebs, m, n, k, dtype, "none", False, False, False, pads=pads)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("m,n,k,pads", LARGE)
def test_backward_large(ebs, dtype, m, n, k, pads):
    check_backward(ebs, m, n, k, dtype, "silu", pads=pads[:4])
    check_backward(ebs, n, m, k, dtype, "none", pads=pads[:4], want=(1, 1, 0))


@pytest.mark.parametrize("dtype", list(TYPES))
def test_empty_batch(ebs, dtype):
    t = TYPES[dtype]
    dt, _ = codes(ebs, dtype, "none")
    d = ebs.linear_desc(0, 9, 21, dt, ebs.EBS_ACT_GELU)
    x, dy, w = (torch.empty(s, dtype=t, device="cuda") for s in ((0, 21), (0, 9), (9, 21)))
    ebs.ebs_linear_forward(x, w, None, None, d, dy, None, workspace(ebs, d, False))
    dw, db = torch.full((9, 21), math.nan, dtype=t, device="cuda"), torch.full((9,), math.nan, dtype=t, device="cuda")
    ebs.ebs_linear_backward(dy, x, w, dy, d, torch.empty_like(x), dw, db, workspace(ebs, d, True))
    assert (dw == 0).all() and (db == 0).all()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("m,n,k", [(3, 40, 200), (7, 40, 200), (150, 200, 72), (2304, 1160, 72), (2100, 1200, 520), (300, 264, 8200)])
def test_nan_and_infinity_reach_their_outputs_only(ebs, dtype, m, n, k):
    t, g = TYPES[dtype], gen(3)
    x, w = strided(m, k, k, t, g), strided(n, k, k, t, g)
    x[1, 5], x[2, 7], w[9, 4], w[11, 6] = math.nan, math.inf, -math.inf, math.nan
    w[12, 7] = 0.0                                           # infinity times zero
    y, dx, dw = (torch.empty(s, dtype=t, device="cuda") for s in ((m, n), (m, k), (n, k)))
    run_forward(ebs, x, w, None, None, dtype, "none", y)
    want = x.double() @ w.double().T
    assert torch.equal(torch.isnan(y), torch.isnan(want)) and torch.equal(torch.isposinf(y), torch.isposinf(want))
    assert torch.equal(torch.isneginf(y), torch.isneginf(want))
    dy = strided(m, n, n, t, g)
    dy[0, 3], dy[2, 8] = math.inf, math.nan
    dt, ac = codes(ebs, dtype, "none")
    d = ebs.linear_desc(m, n, k, dt, ac)
    ebs.ebs_linear_backward(dy, x, w, None, d, dx, dw, None, workspace(ebs, d, True))
    for got, ref in ((dx, dy.double() @ w.double()), (dw, dy.double().T @ x.double())):
        assert torch.equal(torch.isnan(got), torch.isnan(ref)) and torch.equal(torch.isposinf(got), torch.isposinf(ref))
        assert torch.equal(torch.isneginf(got), torch.isneginf(ref))


@pytest.mark.parametrize("m", [4, 300, 9000])
def test_fp32_rows_of_very_different_size(ebs, m):
    """Rows (and columns) of 2^-60 beside rows of 2^60: every output keeps the accuracy of its own row and column."""
    g, n, k = gen(5), 72, 160
    x, w = strided(m, k, k, torch.float32, g), strided(n, k, k, torch.float32, g)
    x *= 2.0 ** torch.linspace(-60, 60, m, device="cuda").round()[:, None]
    w *= 2.0 ** torch.linspace(50, -50, n, device="cuda").round()[:, None]
    y = torch.empty((m, n), device="cuda")
    run_forward(ebs, x, w, None, None, "f32", "none", y)
    ref, s = x.double() @ w.double().T, x.double().abs() @ w.double().abs().T
    # (bound() without its absolute term: in that one, values of 2^-100 would vanish)
    assert ((y.double() - ref).abs() <= 2.0 ** -24 * ref.abs() + s * (4 * 2.0 ** -24 * (8 + math.sqrt(k)) + 2.0 ** -22) + 2.0 ** -147).all()
    dy = strided(m, n, n, torch.float32, g) * 2.0 ** torch.linspace(-50, 50, n, device="cuda").round()
    x2 = strided(m, k, k, torch.float32, g) * 2.0 ** torch.linspace(-40, 40, k, device="cuda").round()
    dw = torch.empty((n, k), device="cuda")
    d = ebs.linear_desc(m, n, k)
    ebs.ebs_linear_backward(dy.contiguous(), x2.contiguous(), w, None, d, None, dw, None, workspace(ebs, d, True))
    ref, s = dy.double().T @ x2.double(), dy.double().abs().T @ x2.double().abs()
    assert ((dw.double() - ref).abs() <= 2.0 ** -24 * ref.abs() + s * (4 * 2.0 ** -24 * (8 + math.sqrt(m)) + 2.0 ** -22) + 2.0 ** -147).all()


def test_f16_gradients_at_the_ends_of_the_range(ebs):
    """dz may exceed dy by the steepest slope (GELU 1.13): no overflow before the products."""
    m, n, k = 64, 16, 24
    g, t = gen(1), torch.float16
    dy = torch.full((m, n), 60000.0, dtype=t, device="cuda")
    z = torch.full((m, n), 1.4, dtype=t, device="cuda")
    x, w = strided(m, k, k, t, g, 2.0 ** -8), strided(n, k, k, t, g, 2.0 ** -8)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    d = ebs.linear_desc(m, n, k, ebs.EBS_F16, ebs.EBS_ACT_GELU)
    ebs.ebs_linear_backward(dy, x, w, z, d, dx, dw, None, workspace(ebs, d, True))
    z64 = z.double().requires_grad_(True)
    (dz,) = torch.autograd.grad(torch.nn.functional.gelu(z64), z64, dy.double())
    for got, ref, s in ((dx, dz @ w.double(), dz @ w.double().abs()), (dw, dz.T @ x.double(), dz.T @ x.double().abs())):
        assert torch.isfinite(got).all()
        assert ((got.double() - ref).abs() <= 2.0 ** -11 * ref.abs() + 2.0 ** -10 * s).all()


def test_gradients_against_differences(ebs):
    """fp32: the loss sum(c * y) changes along random directions as the gradients say."""
    m, n, k, act = 37, 29, 53, "gelu"
    g = gen(9)
    x, w, b, c = (torch.randn(s, generator=g, device="cuda") for s in ((m, k), (n, k), (n,), (m, n)))
    y, z = torch.empty((m, n), device="cuda"), torch.empty((m, n), device="cuda")
    run_forward(ebs, x, w, b, None, "f32", act, y, z)
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    d = ebs.linear_desc(m, n, k, ebs.EBS_F32, ebs.EBS_ACT_GELU)
    ebs.ebs_linear_backward(c, x, w, z, d, dx, dw, db, workspace(ebs, d, True))
    loss = lambda x, w, b: (c.double() * act64(x @ w.T + b, act)).sum()  # noqa: E731
    h = 1e-4
    for i in range(3):
        vx, vw, vb = (torch.randn(t.shape, generator=g, device="cuda", dtype=torch.float64) for t in (x, w, b))
        at = lambda s: loss(x.double() + s * vx, w.double() + s * vw, b.double() + s * vb)  # noqa: E731
        # fourth-order central difference: error h^4 times the fifth derivative along the direction, below 1e-6 relative
        slope = (8 * (at(h) - at(-h)) - (at(2 * h) - at(-2 * h))) / (12 * h)
        got = (dx.double() * vx).sum() + (dw.double() * vw).sum() + (db.double() * vb).sum()
        size = (dx.double() * vx).abs().sum() + (dw.double() * vw).abs().sum() + (db.double() * vb).abs().sum()
        assert abs(slope - got) <= 1e-5 * size


@pytest.mark.parametrize("dtype", list(TYPES))
def test_another_stream_and_replay(ebs, dtype):
    """Calls on a side stream, captured and replayed with other inputs in the same buffers; repeated calls are bit-identical."""
    t, g = TYPES[dtype], gen(4)
    m, n, k = 260, 200, 136
    x, w, dy = strided(m, k, k, t, g), strided(n, k, k, t, g), strided(m, n, n, t, g)
    y, z = torch.empty((m, n), dtype=t, device="cuda"), torch.empty((m, n), dtype=t, device="cuda")
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty(n, dtype=t, device="cuda")
    dt, ac = codes(ebs, dtype, "silu")
    d = ebs.linear_desc(m, n, k, dt, ac)
    wf, wb = workspace(ebs, d, False), workspace(ebs, d, True)

    def step(stream=None):
        ebs.ebs_linear_forward(x, w, None, None, d, y, z, wf, stream)
        ebs.ebs_linear_backward(dy, x, w, z, d, dx, dw, db, wb, stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    first = [v.clone() for v in (y, z, dx, dw, db)]
    step()
    assert all(torch.equal(a, b) for a, b in zip(first, (y, z, dx, dw, db)))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    x.copy_(strided(m, k, k, t, g))
    step()
    want = [v.clone() for v in (y, z, dx, dw, db)]
    for v in (y, z, dx, dw, db):
        v.zero_()
    for ws in (wf, wb):
        if ws is not None:
            ws.fill_(0xFF)
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(want, (y, z, dx, dw, db)))
    capture = ebs.ebs_graph_begin()
    step(capture)
    handle = ebs.ebs_graph_end(capture)
    for v in (y, z, dx, dw, db):
        v.zero_()
    assert ebs.ebs_graph_launch(handle)
    assert all(torch.equal(a, b) for a, b in zip(want, (y, z, dx, dw, db)))
    torch.cuda.synchronize()
    ebs.ebs_graph_destroy(handle)


def test_offsets_beyond_32_bits(ebs):
    """Rows 2^22 + 8 elements apart: the last ones start beyond 2^31 elements."""
    m, n, k, ld = 520, 24, 40, (1 << 22) + 8
    g, t = gen(2), torch.bfloat16
    xs = torch.empty(m * ld, dtype=t, device="cuda")
    x = torch.as_strided(xs, (m, k), (ld, 1))
    x.copy_(torch.randn((m, k), generator=g, device="cuda"))
    w = strided(n, k, k, t, g)
    y = torch.empty((m, n), dtype=t, device="cuda")
    run_forward(ebs, x, w, None, None, "bf16", "none", y)
    ref, s = x.double() @ w.double().T, x.double().abs() @ w.double().abs().T
    assert ((y.double() - ref).abs() <= bound(t, ref, s, k)).all()


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("m,n,k", [(4096, 2048, 256), (40, 200, 400), (1, 300, 264)])
def test_threads(ebs, dtype, m, n, k):
    """Calls from threads that made no CUDA call before, at the same time on streams of their own."""
    t, g = TYPES[dtype], gen(13)
    x, w = strided(m, k, k, t, g), strided(n, k, k, t, g, 1 / math.sqrt(k))
    want = torch.empty((m, n), dtype=t, device="cuda")
    run_forward(ebs, x, w, None, None, dtype, "silu", want)
    outs = [torch.zeros((m, n), dtype=t, device="cuda") for _ in range(4)]
    d = ebs.linear_desc(m, n, k, *codes(ebs, dtype, "silu"))
    spaces = [workspace(ebs, d, False) for _ in outs]
    streams = [torch.cuda.Stream() for _ in outs]
    torch.cuda.synchronize()
    errors = []

    def work(i):
        try:
            for _ in range(20):
                ebs.ebs_linear_forward(x, w, None, None, d, outs[i], None, spaces[i], streams[i])
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(outs))]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    torch.cuda.synchronize()
    assert not errors and all(torch.equal(o, want) for o in outs)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("m,n,k", [(24, 16, 24), (300, 264, 520)])
def test_f16_gradients_next_to_zero(ebs, act, m, n, k):
    """dy of a few times 2^-24.  None and ReLU: dz is dy or zero, no bit of it is lost.  The others keep half of dz (multiples of 2^-23)."""
    t = torch.float16
    dy = ((torch.arange(m * n, device="cuda").reshape(m, n) * 7 % 11 - 5).double() * 2.0 ** -24).to(t)
    z = (torch.arange(m * n, device="cuda").reshape(m, n) * 5 % 13 - 6).to(t)
    # one factor of 1024 in each sum: a result is one dz times 2^10
    x, w = torch.zeros((m, k), dtype=t, device="cuda"), torch.zeros((n, k), dtype=t, device="cuda")
    x[torch.arange(m), torch.arange(m) % k] = 1024
    w[torch.arange(n), torch.arange(n) % k] = 1024
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    dt, ac = codes(ebs, "f16", act)
    d = ebs.linear_desc(m, n, k, dt, ac)
    ebs.ebs_linear_backward(dy, x, w, z, d, dx, dw, None, workspace(ebs, d, True))
    z64 = z.double().requires_grad_(True)
    dz = dy.double() * (z > 0 if act == "relu" else 1)
    if act not in ("none", "relu"):
        (dz,) = torch.autograd.grad(act64(z64, act), z64, dy.double())
    # a kept dz is off by half a step: nothing, or 2^-24 (and by the slope's own 2^-21 of dy); terms a sum has at most: each is a kept dz times 2^10
    step = 0.0 if act in ("none", "relu") else 2.0 ** -24 * (1 + 2.0 ** -10)
    for got, ref, terms in ((dx, dz @ w.double(), (w != 0).double().sum(0).max()), (dw, dz.T @ x.double(), (x != 0).double().sum(0).max())):
        assert ((got.double() - ref).abs() <= 2.0 ** -11 * ref.abs() + terms * 1024 * step).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
def test_slopes_far_out(ebs, act, dtype):
    """|z| of 9 to the end of the type's range: the slope is 0 or 1 there to within what its exponential leaves, and no factor of it overflows."""
    t = TYPES[dtype]
    far = torch.tensor([9.0, 19.5, 20.0, 21.0, 1e3, 1e13, 2e13, 1e14, 5e18, 1e19, 2e19, 1e20, 1e30, 3e38], device="cuda")
    z = torch.cat([far, -far]).to(t)
    for rows in (1, 5):
        zs = z.repeat(rows, 1)
        n = z.numel()
        dy, x, w = torch.ones_like(zs), torch.ones((rows, 8), dtype=t, device="cuda"), torch.eye(n, device="cuda").to(t)[:, :8].contiguous()
        dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty(n, dtype=t, device="cuda")
        d = ebs.linear_desc(rows, n, 8, *codes(ebs, dtype, act))
        ebs.ebs_linear_backward(dy, x, w, zs, d, dx, dw, db, workspace(ebs, d, True))
        # at |z| = 9 SiLU's slope is 9 e^-9 = 1.1e-3 off; the others' 2e-16 at most
        off = 1.2e-3 if act == "silu" else 2.0 ** -21
        want = rows * (z > 0).double()
        assert ((db.double() - want).abs() <= rows * off).all() and ((dw.double() - want[:, None]).abs() <= rows * off).all()
        assert ((dx.double() - (z[:8] > 0).double()).abs() <= off).all()


def sprinkle(t, g, rows, one_in):
    """An infinity of either sign in one of `one_in` rows (or, rows = False, columns), at a place of its own."""
    count, other = (t.shape[0], t.shape[1]) if rows else (t.shape[1], t.shape[0])
    i = torch.arange(0, count, one_in, device="cuda")
    at = torch.randint(0, other, (i.numel(),), generator=g, device="cuda")
    v = torch.where(torch.rand(i.numel(), generator=g, device="cuda") < 0.5, math.inf, -math.inf).to(t.dtype)
    if rows:
        t[i, at] = v
    else:
        t[at, i] = v


def same_where_not_finite(got, ref):
    assert torch.equal(torch.isnan(got), torch.isnan(ref))
    assert torch.equal(torch.isposinf(got), torch.isposinf(ref)) and torch.equal(torch.isneginf(got), torch.isneginf(ref))


# few rows, one tile, clusters, parts through memory, pairs with rows on 16 bytes and anywhere
INFINITE = [(7, 40, 200), (40, 37, 129), (200, 300, 2000), (300, 264, 8200), (300, 261, 4103), (2304, 1160, 72), (2304, 1161, 72), (2100, 1200, 520)]


@pytest.mark.parametrize("one_in", [(1, 0), (0, 1), (1, 1), (5, 7), (33, 50)])
@pytest.mark.parametrize("m,n,k", INFINITE)
def test_fp32_infinities_in_many_rows(ebs, m, n, k, one_in):
    """An infinity in every row of x, column of W, in both or in some: which results are infinite or NaN, and that the others and a residual in
    place are what they are without."""
    g = gen(17)
    for act, in_place in (("none", True), ("relu", False), ("silu", True)):
        x, w, r = strided(m, k, k, torch.float32, g), strided(n, k, k, torch.float32, g, 1 / math.sqrt(k)), strided(m, n, n, torch.float32, g)
        b = torch.randn(n, generator=g, device="cuda")
        w[:, ::9] = 0.0                                       # infinity times zero
        if one_in[0]:
            sprinkle(x, g, True, one_in[0])
        if one_in[1]:
            sprinkle(w, g, True, one_in[1])
        x[1, 3] = math.nan
        r[2, 4] = -math.inf
        z64 = x.double() @ w.double().T + b.double()
        y64 = act64(z64, act) + r.double()
        y, z = r.clone(), torch.empty((m, n), device="cuda")
        run_forward(ebs, x, w, b, y if in_place else r, "f32", act, y, z)
        same_where_not_finite(z, z64)
        same_where_not_finite(y, y64)
        xs, ws = torch.where(torch.isfinite(x), x, torch.zeros_like(x)), torch.where(torch.isfinite(w), w, torch.zeros_like(w))
        sums = xs.double().abs() @ ws.double().abs().T + b.double().abs()
        ok = torch.isfinite(z64)
        assert ((z.double() - z64).abs() <= bound(torch.float32, z64, sums, k))[ok].all()
        ok = torch.isfinite(y64)
        assert ((y.double() - y64).abs() <= bound(torch.float32, y64, 1.13 * sums, k) + 2.0 ** -23 * (act64(z64, act).abs() + r.double().abs()))[ok].all()
    assert ebs.ebs_check_device_status() == ebs.EBS_OK


@pytest.mark.parametrize("one_in", [(1, 0), (0, 1), (1, 1), (5, 7)])
@pytest.mark.parametrize("m,n,k", INFINITE)
def test_fp32_infinities_in_many_gradients(ebs, m, n, k, one_in):
    g = gen(19)
    x, w, dy, z = (strided(*s, torch.float32, g) for s in ((m, k, k), (n, k, k), (m, n, n), (m, n, n)))
    w[::7] = 0.0
    x[::7] = 0.0
    if one_in[0]:
        sprinkle(dy, g, True, one_in[0])
    if one_in[1]:
        sprinkle(x, g, False, one_in[1])
        sprinkle(w, g, False, one_in[1])
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    for act in ("none", "gelu"):
        d = ebs.linear_desc(m, n, k, *codes(ebs, "f32", act))
        ebs.ebs_linear_backward(dy, x, w, z, d, dx, dw, None, workspace(ebs, d, True))
        dz = dy.double()
        if act == "gelu":
            dz = dz * slope64(z.double())
        same_where_not_finite(dx, dz @ w.double())
        same_where_not_finite(dw, dz.T @ x.double())
    assert ebs.ebs_check_device_status() == ebs.EBS_OK


def slope64(z):
    """GELU's derivative."""
    return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)


@pytest.mark.parametrize("m,n,k", [(4096, 2048, 131112), (700, 520, 262150), (144, 16, 200001)])
def test_fp32_infinities_along_long_reductions(ebs, m, n, k):
    """One in every row of x: a result is that infinity with the sign of the weight it meets.  No wait runs out meanwhile."""
    g = gen(23)
    x, w = torch.randn((m, k), generator=g, device="cuda"), torch.randn((n, k), generator=g, device="cuda")
    at = torch.randint(0, k, (m,), generator=g, device="cuda")
    sign = torch.where(torch.rand(m, generator=g, device="cuda") < 0.5, 1.0, -1.0)
    x[torch.arange(m, device="cuda"), at] = sign * math.inf
    y = torch.zeros((m, n), device="cuda")
    run_forward(ebs, x, w, None, None, "f32", "none", y)
    assert torch.equal(y, w[:, at].T * sign[:, None] * math.inf)
    assert ebs.ebs_check_device_status() == ebs.EBS_OK


def one_sign(rows, cols, t, g):
    """Values of 1/16 .. 1/4: columns of different size, so that the results' mantissas are spread."""
    return ((torch.rand((rows, cols), generator=g, device="cuda") * 0.5 + 0.5) * 2.0 ** (torch.rand(cols, generator=g, device="cuda") - 3)).to(t)


def long_bound(ref, t, terms):
    """The tensor core adds 16 products at a time and truncates: each of the 256 additions of a sum of up to 4096 terms loses at most 2^-23 of what it
    ends at, together 2^-15.  Such sums, `terms` / 4096 at most, are added in fp32 and rounded to nearest
    (2^-24 each, and a few for parts that meet); the output is rounded once."""
    return ref * (torch.finfo(t).eps / 2 + 2.0 ** -15 + (terms / 4096 + 16) * 2.0 ** -24)


# rows of dy, n, k: tiles on few blocks, a cluster's parts, pairs, parts through memory; a reduction that ends inside a stage
LONG = [(131072, 16, 144), (200711, 64, 577), (50176, 128, 1152), (200000, 300, 264), (32768, 2304, 2304), (8256, 2304, 2304), (8192, 2304, 2304), (70001, 5, 7)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("m,n,k", LONG)
def test_long_sums_of_one_sign(ebs, m, n, k, dtype):
    """Weight gradients over many rows, all terms of one sign: what the tensor core truncates does not add up along the reduction."""
    t, g = TYPES[dtype], gen(29)
    dy, x = one_sign(m, n, t, g), one_sign(m, k, t, g)
    dw, db = torch.empty((n, k), dtype=t, device="cuda"), torch.empty(n, dtype=t, device="cuda")
    d = ebs.linear_desc(m, n, k, *codes(ebs, dtype, "none"))
    ebs.ebs_linear_backward(dy, x, None, None, d, None, dw, db, workspace(ebs, d, True))
    some = torch.arange(0, n, max(1, n // 64), device="cuda")
    ref = dy[:, some].double().T @ x.double()
    assert ((dw[some].double() - ref).abs() <= long_bound(ref, t, m)).all()
    ref = dy.double().sum(0)
    assert ((db.double() - ref).abs() <= long_bound(ref, t, m)).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("m,n,k", [(3, 200, 131080), (40, 200, 131080), (200, 300, 70000), (2304, 2304, 16456)])
def test_long_products_of_one_sign(ebs, m, n, k, dtype):
    t, g = TYPES[dtype], gen(31)
    x, w = one_sign(m, k, t, g), one_sign(n, k, t, g)
    y = torch.empty((m, n), dtype=t, device="cuda")
    run_forward(ebs, x, w, None, None, dtype, "none", y)
    some = torch.arange(0, m, max(1, m // 64), device="cuda")
    ref = x[some].double() @ w.double().T
    assert ((y[some].double() - ref).abs() <= long_bound(ref, t, k)).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("m,n,k", [(2304, 2304, 4168), (2304, 2305, 5000), (40, 200, 5000), (200, 72, 4097), (1, 300, 9000)])
def test_long_products_with_every_part(ebs, m, n, k, dtype):
    """Sums that leave the tensor core in chunks, behind bias, activation, residual and kept z, into rows on 16 bytes and anywhere."""
    check_forward(ebs, m, n, k, dtype, "gelu")
    check_forward(ebs, m, n, k, dtype, "silu", pads=(3, 0, 1, 2, 5))
    check_forward(ebs, m, n, k, dtype, "none", False, True, False, in_place=True)
