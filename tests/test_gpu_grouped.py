"""Layers of experts, forward and backward, against the formulas in 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
F = torch.nn.functional
ACTS = [lambda v: v, torch.relu, F.gelu, lambda v: F.gelu(v, approximate="tanh"), F.silu]


@pytest.fixture(scope="module")
def ebs():
    from paper_2003_07577_b200 import binding
    return binding


def code(ebs, dtype):
    return {"f16": ebs.EBS_F16, "bf16": ebs.EBS_BF16}[dtype]


def truncation(terms):
    """What the tensor core cuts off a sum, relative to the sum of magnitudes: 2^-23 a step of 16 terms for up to 4096 terms, then a rounding for each
    further 4096; 2^-22 for alpha, bias and the like."""
    return min(terms, 4096) / 16 * 2.0 ** -23 + (terms // 4096) * 2.0 ** -24 + 2.0 ** -22


def within(got, ref, off):
    info = torch.finfo(got.dtype)
    off = off + (info.eps / 2) * ref.abs() + info.smallest_normal * info.eps
    bad = (got.double() - ref).abs() > off
    assert not bad.any(), (int(bad.sum()), float(((got.double() - ref).abs() / off).max()))


def strided(g, rows, cols, ld, t, scale=1.0, fill=math.nan):
    big = torch.full((rows, ld or cols), fill, dtype=t, device="cuda")
    big[:, :cols] = (torch.randn(rows, cols, generator=g, device="cuda") * scale).to(t)
    return big


def layer(ebs, seed, counts, n, k, dtype, act=0, bias=True, residual=False, keep=False, spare=0, first=0, ldx=0, ldw=0, ldy=0, in_place=False, want=("dx", "dw", "db")):
    """A forward and a backward call of random inputs, each checked.  first, spare: rows before and behind the experts'."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    t, experts, m = TYPES[dtype], len(counts), first + sum(counts) + spare
    x, w = strided(g, m, k, ldx, t), strided(g, experts * n, k, ldw, t, 1 / math.sqrt(k))
    b = torch.randn(experts, n, generator=g, device="cuda").to(t) if bias else None
    offsets = (torch.tensor([0] + list(counts)).cumsum(0) + first).to(torch.int32).cuda()
    nobody = torch.ones(m, dtype=torch.bool, device="cuda")
    nobody[first:first + sum(counts)] = False
    x[nobody] = math.nan                                                 # what is nobody's reaches nothing
    d = ebs.linear_desc(m, n, k, code(ebs, dtype), act, ldx=ldx, ldw=ldw, ldy=ldy, ldr=ldy if in_place else 0, ldz=ldy)
    y = strided(g, m, n, ldy, t, fill=3.0)
    y[nobody] = 3.0
    r = (y if in_place else torch.randn(m, n, generator=g, device="cuda").to(t)) if residual else None
    res = r[:, :n].clone() if residual else None
    z = torch.full_like(y, 5.0) if keep else None
    ws = torch.full((max(16, ebs.ebs_grouped_workspace_bytes(d, experts)),), 255, dtype=torch.uint8, device="cuda")
    ebs.ebs_grouped_forward(x, w, b, r, offsets, experts, d, y, z, ws)
    assert (y[nobody] == 3.0).all() and (not ldy or y[:, n:].eq(3.0).all())
    assert not keep or ((z[nobody] == 5.0).all() and (not ldy or (z[:, n:] == 5.0).all()))
    rows = [slice(int(a), int(c)) for a, c in zip(offsets[:-1], offsets[1:])]
    xs, wd = x[:, :k].double(), w[:, :k].double().view(experts, n, k)
    for e, s in enumerate(rows):
        ref, size = xs[s] @ wd[e].t(), xs[s].abs() @ wd[e].abs().t()
        if bias:
            ref, size = ref + b[e].double(), size + b[e].double().abs()
        off = truncation(k) * size
        if keep:
            within(z[s, :n], ref, off)
        out = ACTS[act](ref)
        off = 1.13 * off + (2.0 ** -19 * (out.abs() + ref.abs()) if act > 1 else 0.0)
        if residual:
            out = out + res[s].double()
            off = off + 2.0 ** -23 * out.abs()
        within(y[s, :n], out, off)

    dy, zs = strided(g, m, n, ldy, t, 0.1), strided(g, m, n, ldy, t)
    dy[nobody] = math.nan
    zs[nobody] = math.nan
    dx = torch.full((m, ldx or k), 7.0, dtype=t, device="cuda") if "dx" in want else None
    dw = torch.full((experts * n, ldw or k), 7.0, dtype=t, device="cuda") if "dw" in want else None
    db = torch.full((experts, n), 7.0, dtype=t, device="cuda") if "db" in want else None
    ws = torch.full((max(16, ebs.ebs_grouped_workspace_bytes(d, experts, True)),), 255, dtype=torch.uint8, device="cuda")
    ebs.ebs_grouped_backward(dy, x, w, zs if act else None, offsets, experts, d, dx, dw, db, ws)
    if dx is not None:
        assert (dx[nobody] == 7.0).all() and (not ldx or (dx[:, k:] == 7.0).all())
    assert dw is None or not ldw or (dw[:, k:] == 7.0).all()
    half = torch.finfo(t).eps / 2
    for e, s in enumerate(rows):
        dz = dy[s, :n].double()
        if act:
            v = zs[s, :n].double().requires_grad_(True)
            (dz,) = torch.autograd.grad(ACTS[act](v), v, dz)
        # dz is rounded to the type before the products (fp16 halved: steps of 2^-23 below), its slope is off by 2^-19
        err = (half + 2.0 ** -19) * dz.abs() + 2.0 ** -24 if act else torch.zeros_like(dz)
        if dx is not None:
            within(dx[s, :k], dz @ wd[e], truncation(n) * (dz.abs() @ wd[e].abs()) + err @ wd[e].abs())
        if dw is not None:
            within(dw[e * n:(e + 1) * n, :k], dz.t() @ xs[s], truncation(s.stop - s.start) * (dz.abs().t() @ xs[s].abs()) + err.t() @ xs[s].abs())
        if db is not None:
            within(db[e], dz.sum(dim=0), (2.0 ** -18 + (s.stop - s.start + 64) / 64 * 2.0 ** -24) * dz.abs().sum(dim=0))


COUNTS = [[1], [0], [0, 0, 5], [128], [129, 0, 127], [1] * 40, [64, 65, 63, 1, 0, 16, 15, 17], [300, 2, 0, 0, 777], [0] * 33 + [7] + [0] * 40 + [130, 3], [31, 33, 48, 47, 49]]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("counts", COUNTS, ids=str)
@pytest.mark.parametrize("n,k", [(64, 128), (33, 65), (264, 72)])
def test_rows(ebs, dtype, counts, n, k):
    layer(ebs, 1, counts, n, k, dtype, act=4, keep=True)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n,k", [(1, 1), (8, 8), (1, 200), (200, 1), (127, 63), (128, 64), (129, 257), (1000, 520), (512, 1031), (24, 5000), (5000, 24)])
def test_sizes(ebs, dtype, n, k):
    layer(ebs, 2, [70, 3, 140], n, k, dtype, act=1, residual=True)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("counts", [[1, 0, 2, 24, 31, 32, 33, 5, 0, 0, 1, 1], [40, 1, 0, 7, 0, 3, 1], [96, 1, 1, 1, 1, 1, 1, 1, 1, 1]], ids=str)
@pytest.mark.parametrize("n,k,ldy", [(256, 1024, 0), (100, 520, 0), (72, 8, 75), (64, 4200, 0)])
def test_few_rows(ebs, dtype, counts, n, k, ldy):
    """At most 32 rows an expert in the mean: tiles of 32 rows, experts with more of them among the others."""
    layer(ebs, 13, counts, n, k, dtype, act=4, residual=True, keep=True, spare=2, first=1, ldy=ldy)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("act", range(5))
@pytest.mark.parametrize("bias,residual,keep", [(False, False, False), (True, True, True), (False, True, False)])
def test_activations(ebs, dtype, act, bias, residual, keep):
    layer(ebs, 3, [50, 200, 1], 136, 264, dtype, act=act, bias=bias, residual=residual, keep=keep)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("k,ldx,ldw,ldy", [(64, 72, 80, 48), (64, 65, 64, 41), (61, 64, 67, 40), (61, 0, 0, 0), (64, 0, 66, 56)])
def test_strides(ebs, dtype, k, ldx, ldw, ldy):
    layer(ebs, 4, [20, 150, 9], 40, k, dtype, act=2, residual=True, keep=True, ldx=ldx, ldw=ldw, ldy=ldy, in_place=True)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("first,spare", [(0, 1), (5, 0), (130, 200), (7, 3)])
def test_rows_of_nobody(ebs, dtype, first, spare):
    """Rows before and behind the experts' hold NaN in every operand: nothing of it reaches a result, nothing is written there."""
    layer(ebs, 5, [33, 0, 65, 128], 72, 136, dtype, act=4, first=first, spare=spare, keep=True)


@pytest.mark.parametrize("want", [("dx",), ("dw",), ("db",), ("dx", "db"), ("dw", "db")])
@pytest.mark.parametrize("act", [0, 3])
def test_some_gradients(ebs, want, act):
    layer(ebs, 6, [40, 0, 200], 65, 130, "bf16", act=act, want=want)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n,k", [(2056, 512), (520, 2100), (2300, 2056)])
@pytest.mark.parametrize("counts", [[700, 1500, 0, 900, 129], [256, 512, 1024, 1280], [5, 300, 3, 17, 1, 2, 33, 64, 48, 2000, 9, 1, 1, 1, 1, 1]], ids=str)
def test_wide_tiles(ebs, dtype, n, k, counts):
    """Enough tiles of 256 columns for every pair of SMs, several a pair; experts of fewer rows than a stage one behind the other."""
    layer(ebs, 7, counts, n, k, dtype, act=4, keep=True, spare=100)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_long_sums(ebs, dtype):
    """Reductions that leave the tensor core on the way, in every product: input features, output features, rows."""
    layer(ebs, 8, [4097, 9000, 3], 72, 136, dtype, act=0)
    layer(ebs, 9, [40, 7], 4200, 4168, dtype, act=0)
    layer(ebs, 10, [5001, 4200], 1100, 2100, dtype, act=0)               # pairs of blocks: dW's sums are long
    layer(ebs, 11, [1500, 2000], 2056, 4200, dtype, act=0)               # y's
    layer(ebs, 12, [1500, 2000], 4200, 2056, dtype, act=0)               # dx's


def test_no_rows(ebs):
    d = ebs.linear_desc(0, 16, 24, ebs.EBS_BF16)
    w, dw, db = (torch.full(s, 7.0, dtype=torch.bfloat16, device="cuda") for s in ((3, 16, 24), (3, 16, 24), (3, 16)))
    offsets = torch.zeros(4, dtype=torch.int32, device="cuda")
    empty = torch.empty(0, 24, dtype=torch.bfloat16, device="cuda")
    ebs.ebs_grouped_forward(empty, w, None, None, offsets, 3, d, None)
    ebs.ebs_grouped_backward(None, None, w, None, offsets, 3, d, None, dw, db, None)
    assert not dw.any() and not db.any()


def test_offsets_that_are_not_in_order(ebs):
    """Taken as the nearest ones that are: nothing out of bounds is read or written, and every wait ends."""
    m, n, k, experts = 300, 40, 64, 3
    d = ebs.linear_desc(m, n, k, ebs.EBS_BF16)
    g = torch.Generator(device="cuda").manual_seed(1)
    x, w, dy = (torch.randn(s, generator=g, device="cuda").bfloat16() for s in ((m, k), (experts, n, k), (m, n)))
    ws = torch.empty(max(16, ebs.ebs_grouped_workspace_bytes(d, experts, True)), dtype=torch.uint8, device="cuda")
    before = ebs.ebs_device_wait_timeouts()
    for offsets in ([0, 200, 100, 1000], [-7, 2, 1 << 30, 4], [9, 8, 7, 6], [2147483647, -2147483648, 0, 10], [300, 300, 300, 300]):
        o = torch.tensor(offsets, dtype=torch.int32).cuda()
        y, dx, dw = torch.full((m + 2, n), 3.0).bfloat16().cuda(), torch.full((m + 2, k), 3.0).bfloat16().cuda(), torch.full((experts * n + 2, k), 3.0).bfloat16().cuda()
        ebs.ebs_grouped_forward(x, w, None, None, o, experts, d, y, None, ws)
        ebs.ebs_grouped_backward(dy, x, w, None, o, experts, d, dx, dw, None, ws)
        torch.cuda.synchronize()
        for out in (y, dx, dw):
            assert (out[-2:] == 3.0).all() and out.isfinite().all()
    assert ebs.ebs_device_wait_timeouts() == before


def test_not_finite(ebs):
    """An infinity or a NaN reaches exactly the outputs whose sums contain it."""
    n, k, counts = 40, 72, [100, 30, 60]
    m = sum(counts)
    g = torch.Generator(device="cuda").manual_seed(2)
    x, w, dy = (torch.randn(s, generator=g, device="cuda").bfloat16() for s in ((m, k), (3, n, k), (m, n)))
    x[5, 7], x[110, 3], w[2, 9, 11], dy[120, 20] = math.inf, math.nan, -math.inf, math.inf
    offsets = torch.tensor([0, 100, 130, 190], dtype=torch.int32).cuda()
    d = ebs.linear_desc(m, n, k, ebs.EBS_BF16)
    y, dx, dw, db = (torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in ((m, n), (m, k), (3, n, k), (3, n)))
    ws = torch.empty(max(16, ebs.ebs_grouped_workspace_bytes(d, 3, True)), dtype=torch.uint8, device="cuda")
    ebs.ebs_grouped_forward(x, w, None, None, offsets, 3, d, y, None, ws)
    ebs.ebs_grouped_backward(dy, x, w, None, offsets, 3, d, dx, dw, db, ws)
    for e, s in enumerate((slice(0, 100), slice(100, 130), slice(130, 190))):
        xs, ds, we = x[s].double(), dy[s].double(), w[e].double()
        for got, a, b in ((y[s], xs, we.t()), (dx[s], ds, we), (dw[e], ds.t(), xs)):
            ref = (a[:, :, None] * b[None]).sum(dim=1)
            assert torch.equal(got.isnan(), ref.isnan()) and torch.equal(got.isinf(), ref.isinf())
            assert torch.equal(got[got.isinf()].double(), ref[ref.isinf()])
        assert torch.equal(db[e].isinf(), ds.sum(dim=0).isinf())


def test_gradients_against_differences(ebs):
    """A directional derivative of a loss through the forward call against the backward call's gradients."""
    n, k, counts = 24, 40, [17, 0, 30]
    m, g = sum(counts), torch.Generator(device="cuda").manual_seed(3)
    x, w, b, c = (torch.randn(s, generator=g, device="cuda") for s in ((m, k), (3, n, k), (3, n), (m, n)))
    w /= math.sqrt(k)
    offsets = torch.tensor([0, 17, 17, 47], dtype=torch.int32).cuda()
    d = ebs.linear_desc(m, n, k, ebs.EBS_F16, ebs.EBS_ACT_SILU)
    ws = torch.empty(max(16, ebs.ebs_grouped_workspace_bytes(d, 3, True)), dtype=torch.uint8, device="cuda")
    half = lambda *v: [q.half() for q in v]  # noqa: E731

    def loss(x, w, b, z=None):
        y = torch.zeros(m, n, dtype=torch.float16, device="cuda")
        ebs.ebs_grouped_forward(*half(x, w, b), None, offsets, 3, d, y, z, ws)
        return float((y.double() * c.half().double()).sum())
    z = torch.zeros(m, n, dtype=torch.float16, device="cuda")
    loss(x, w, b, z)
    grads = [torch.zeros_like(q, dtype=torch.float16) for q in (x, w, b)]
    ebs.ebs_grouped_backward(c.half(), x.half(), w.half(), z, offsets, 3, d, *grads, ws)
    for i, v in enumerate((x, w, b)):
        step = torch.randn(v.shape, generator=g, device="cuda") * (1 / 16)
        up, down = [x, w, b], [x, w, b]
        up[i], down[i] = (v + step).half().float(), (v - step).half().float()
        slope, want = loss(*up) - loss(*down), float((grads[i].double() * (up[i] - down[i]).double()).sum())
        # y has m n = 1128 values of size about 1, each off by 2^-12 of itself at random and times c of size 1: 34 * 2^-12 * 2 = 0.016 a difference; third order of the
        # step: 1/16^2 of the slope of a smooth function
        assert abs(slope - want) <= 0.1 + 0.02 * abs(want), (i, slope, want)


def test_captured_and_replayed(ebs):
    """A step in a graph on a side stream: new rows, new shares of the experts."""
    n, k, experts, m = 136, 72, 4, 300
    t = torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(4)
    w = (torch.randn(experts, n, k, generator=g, device="cuda") / 8).to(t)
    x, dy, y, z, dx = (torch.zeros(m, c, dtype=t, device="cuda") for c in (k, n, n, n, k))
    dw, db = torch.zeros(experts, n, k, dtype=t, device="cuda"), torch.zeros(experts, n, dtype=t, device="cuda")
    offsets = torch.tensor([0, 1, 2, 3, 4], dtype=torch.int32).cuda()
    d = ebs.linear_desc(m, n, k, ebs.EBS_BF16, ebs.EBS_ACT_RELU)
    ws = torch.empty(max(ebs.ebs_grouped_workspace_bytes(d, experts, b) for b in (False, True)), dtype=torch.uint8, device="cuda")

    def step():
        ebs.ebs_grouped_forward(x, w, None, None, offsets, experts, d, y, z, ws)
        ebs.ebs_grouped_backward(dy, x, w, z, offsets, experts, d, dx, dw, db, ws)
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        step()
    for counts in ([100, 100, 50, 50], [0, 300, 0, 0], [1, 0, 200, 9]):
        x.copy_(torch.randn(m, k, generator=g, device="cuda"))
        dy.copy_(torch.randn(m, n, generator=g, device="cuda"))
        offsets.copy_(torch.tensor([0] + counts).cumsum(0))
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in (y[:sum(counts)], dx[:sum(counts)], dw, db)]
        step()
        for a, b in zip(got, (y[:sum(counts)], dx[:sum(counts)], dw, db)):
            assert torch.equal(a, b)
        row = 0
        for e, c in enumerate(counts):
            s = slice(row, row + c)
            dz = (dy[s].double() * (z[s] > 0))
            within(y[s], (x[s].double() @ w[e].double().t()).relu(), truncation(k) * (x[s].double().abs() @ w[e].double().abs().t()))
            within(dw[e], dz.t() @ x[s].double(), truncation(c) * (dz.abs().t() @ x[s].double().abs()))
            row += c


def test_elements_past_32_bits(ebs):
    m, n, k = 600000, 64, 4096
    x = torch.zeros(m, k, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(5)
    x[-100:] = torch.randn(100, k, generator=g, device="cuda").bfloat16()
    w = (torch.randn(2, n, k, generator=g, device="cuda") / 64).bfloat16()
    offsets = torch.tensor([0, m - 70, m], dtype=torch.int32).cuda()
    d = ebs.linear_desc(m, n, k, ebs.EBS_BF16)
    y = torch.full((m, n), 3.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(ebs.ebs_grouped_workspace_bytes(d, 2, True), dtype=torch.uint8, device="cuda")
    ebs.ebs_grouped_forward(x, w, None, None, offsets, 2, d, y, None, ws)
    for s, e in ((slice(m - 100, m - 70), 0), (slice(m - 70, m), 1)):
        a, b = x[s].double(), w[e].double()
        within(y[s], a @ b.t(), truncation(k) * (a.abs() @ b.abs().t()))
    assert not y[:m - 100].any()
    dy = torch.zeros(m, n, dtype=torch.bfloat16, device="cuda")
    dy[-100:] = torch.randn(100, n, generator=g, device="cuda").bfloat16()
    dx, dw = torch.full_like(x, 3.0), torch.zeros_like(w)
    ebs.ebs_grouped_backward(dy, x, w, None, offsets, 2, d, dx, dw, None, ws)
    for s, e in ((slice(m - 100, m - 70), 0), (slice(m - 70, m), 1)):
        a, b, c = dy[s].double(), w[e].double(), x[s].double()
        within(dx[s], a @ b, truncation(n) * (a.abs() @ b.abs()))
        within(dw[e], a.t() @ c, truncation(m) * (a.abs().t() @ c.abs()))
    assert not dx[:m - 100].any()
