"""A layer of the bitwidth search, trained: the operators run together, as `search.SearchLinear` calls them."""
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mods():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    import paper_2003_07577_b200 as pkg
    from paper_2003_07577_b200 import binding, search
    if not os.path.exists(binding.LIB_PATH):
        pkg.build()
    binding.lib()
    return binding, search


def make(mods, m, n, k, act, seed=0):
    ebs, search = mods
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    w = torch.randn((n, k), generator=g, device="cuda") / math.sqrt(k)
    bias = 0.1 * torch.randn(n, generator=g, device="cuda")
    return search.SearchLinear(w, m, [2, 3, 4], [0.2, 0.5, 0.3], [0.6, 0.3, 0.1], 2.0, bias, act), g


@pytest.mark.parametrize("m,n,k", [(3, 40, 72), (200, 64, 576), (3136, 128, 256), (12544, 256, 1152)])
def test_step_matches_the_formulas(mods, m, n, k):
    ebs, search = mods
    layer, g = make(mods, m, n, k, ebs.EBS_ACT_RELU, m)
    x, res, dy = (torch.randn(s, generator=g, device="cuda") for s in ((m, k), (m, n), (m, n)))
    y = layer.forward(x, res)
    # the blended tensors are compared with the formula elsewhere; here the chain behind them, in 64 bits from the same tensors
    xh, wh = layer.x_hat.double(), layer.w_hat.double()
    z = xh @ wh.T + layer.bias.double()
    sums = xh.abs() @ wh.abs().T + 1
    # fp32 sums from operands of 22 bits (2^-22 of every product), one rounding at the end: 2^-24 of the value; a residual: two more
    eps = lambda K: 2.0 ** -22 + 4 * 2.0 ** -24 * (8 + math.sqrt(K))  # noqa: E731
    assert ((y.double() - (z.clamp(min=0) + res.double())).abs() <= eps(k) * sums + 2.0 ** -22 * (sums + res.double().abs())).all()
    dx = layer.backward(dy)
    dz = dy.double() * (layer.z > 0)                          # (the kept pre-activations decide)
    mask = (x > 0) & (x < 2.0)
    assert ((dx.double() - (dz @ wh) * mask).abs() <= (eps(n) + 2.0 ** -24) * (dz.abs() @ wh.abs())).all()
    assert ((layer.dw.double() - dz.T @ xh).abs() <= (eps(m) + 2.0 ** -24) * (dz.abs().T @ xh.abs())).all()
    assert ((layer.dbias.double() - dz.sum(0)).abs() <= eps(m) * dz.abs().sum(0)).all()
    before, bias = layer.weight.clone(), layer.bias.clone()
    layer.step(0.02)
    u = layer.momentum.double()
    u = u / (u.norm() + 1e-7)
    a, b, c = search.COEFF
    for _ in range(5):
        s = u @ u.T
        u = a * u + (b * s + c * (s @ s)) @ u
    # as derived beside the orthogonalisation's own tests: a^5 / (a - 1) * 2^-20 of the rms, six times for the largest of many
    own = 6 * a ** 5 / (a - 1) * 2.0 ** -20 * (math.sqrt(1 / max(n, k)) + u.pow(2).mean().sqrt())
    assert ((layer.update.double() - u).abs() <= own).all()
    assert torch.equal(layer.weight, before.sub(layer.update, alpha=0.02)) and torch.equal(layer.bias, bias.sub(layer.dbias, alpha=0.02))


def test_two_layers_captured_and_replayed(mods):
    """Two layers' training step in one graph, replayed on new inputs, against the same calls made one by one."""
    ebs, search = mods
    (l1, g), (l2, _) = make(mods, 300, 96, 200, ebs.EBS_ACT_GELU, 1), make(mods, 300, 48, 96, ebs.EBS_ACT_NONE, 2)
    x, target = torch.randn((300, 200), generator=g, device="cuda"), torch.randn((300, 48), generator=g, device="cuda")

    def step():
        out = l2.forward(l1.forward(x))
        l1.backward(l2.backward((out - target) / 300))
        l2.step(0.01)
        l1.step(0.01)
        return out

    keep = [t for layer in (l1, l2) for t in (layer.weight, layer.bias, layer.momentum)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    start = [t.clone() for t in keep]
    x.copy_(torch.randn((300, 200), generator=g, device="cuda"))
    want = step().clone()
    after = [t.clone() for t in keep]
    for t, s in zip(keep, start):
        t.copy_(s)
    graph.replay()
    assert torch.equal(out, want) and all(torch.equal(a, b) for a, b in zip(keep, after))
    assert ebs.ebs_check_device_status() == ebs.EBS_OK


def test_refusals(mods):
    ebs, search = mods
    layer, g = make(mods, 8, 16, 24, ebs.EBS_ACT_NONE)
    x = torch.randn((8, 24), generator=g, device="cuda")
    with pytest.raises(RuntimeError):
        layer.backward(torch.zeros((8, 16), device="cuda"))
    for bad in (x[:4], x.half(), x.cpu(), torch.zeros((24, 8), device="cuda").T):
        with pytest.raises(ValueError):
            layer.forward(bad)
    with pytest.raises(ValueError):
        layer.forward(x, x)
    for weight, rows in ((torch.zeros((4, 8)), 2), (torch.zeros(8, device="cuda"), 2), (torch.zeros((4, 8), device="cuda"), 0)):
        with pytest.raises(ValueError):
            search.SearchLinear(weight, rows, [2], [1.0], [1.0], 1.0)
    with pytest.raises(ValueError):
        search.SearchLinear(torch.zeros((4, 8), dtype=torch.float64, device="cuda"), 2, [2], [1.0], [1.0], 1.0)
    layer.forward(x)
    with pytest.raises(ValueError):
        layer.backward(x)


def layer_of_dtype(mods, default):
    """A step of a layer made under another default type: its buffers, then what it leaves in them."""
    ebs, search = mods
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    w, b, x, dy = (torch.randn(s, generator=g, device="cuda", dtype=torch.float32) for s in ((40, 72), (40,), (20, 72), (20, 40)))
    before = torch.get_default_dtype()
    torch.set_default_dtype(default)
    try:
        layer = search.SearchLinear(w, 20, [2, 4], [0.5, 0.5], [0.3, 0.7], 2.0, b, ebs.EBS_ACT_SILU)
        own = [layer.w_hat, layer.dw, layer.momentum, layer.update, layer.dbias, layer.x_hat, layer.dx, layer.y, layer.z]
        assert all(t.dtype == torch.float32 for t in own)    # (before any kernel writes to them)
        layer.forward(x)
        dx = layer.backward(dy)
        layer.step(0.01)
    finally:
        torch.set_default_dtype(before)
    return own + [dx, layer.weight, layer.bias]


@pytest.mark.parametrize("default", [torch.float16, torch.bfloat16, torch.float64])
def test_another_default_type(mods, default):
    """The layer's buffers are fp32 whatever torch's default type is: the kernels write fp32 into them."""
    for got, want in zip(layer_of_dtype(mods, default), layer_of_dtype(mods, torch.float32)):
        assert got.dtype == torch.float32 and torch.equal(got, want)


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_clipped_activations_have_no_gradient(mods, bad):
    """Outside the clip range the gradient is zero, whatever the gradient of x_hat is there."""
    ebs, _ = mods
    layer, g = make(mods, 9, 16, 24, ebs.EBS_ACT_NONE)
    x, dy = torch.randn((9, 24), generator=g, device="cuda"), torch.randn((9, 16), generator=g, device="cuda")
    x[3, :4] = torch.tensor([-0.5, 3.0, 0.0, 2.0], device="cuda")
    dy[3, 5] = bad
    layer.forward(x)
    dx = layer.backward(dy)
    clipped = (x <= 0) | (x >= 2.0)
    assert (dx[clipped] == 0).all()
    assert not torch.isfinite(dx[3][~clipped[3]]).any() and torch.isfinite(dx[torch.arange(9, device="cuda") != 3]).all()


def test_parameters(mods):
    """Weights that are a module's parameters are trained as plain tensors are."""
    ebs, search = mods
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    w, b, x, dy = (torch.randn(s, generator=g, device="cuda") for s in ((40, 72), (40,), (20, 72), (20, 40)))
    results = []
    for kind in (lambda t: t.clone(), lambda t: torch.nn.Parameter(t.clone())):
        layer = search.SearchLinear(kind(w), 20, [2, 4], [0.5, 0.5], [0.3, 0.7], 2.0, kind(b), ebs.EBS_ACT_SILU)
        for _ in range(2):
            layer.forward(x)
            layer.backward(dy)
            layer.step(0.01)
        results.append((layer.weight.detach(), layer.bias.detach(), layer.momentum))
    assert all(torch.equal(p, q) for p, q in zip(*results))


def test_refused_when_made(mods):
    """What step() or backward() would refuse is refused before there is a state that they could leave half changed."""
    ebs, search = mods
    w = torch.zeros((8, 16), device="cuda")
    for change in (dict(steps=65), dict(steps=-1), dict(act=5), dict(act=-1)):
        with pytest.raises(ValueError):
            search.SearchLinear(w, 4, [2], [1.0], [1.0], 1.0, **change)
