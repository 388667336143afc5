"""A layer of experts trained, clipped, brought to 4 bits and answered from: the operators run together, as `experts` and `search.GradientClip` call them."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

F = torch.nn.functional


@pytest.fixture(scope="module")
def mods():
    from paper_2003_07577_b200 import binding, experts, search
    return binding, experts, search


def make(mods, counts, n, k, dtype, act, bias=True, spare=3, seed=0):
    ebs, ex, _ = mods
    g = torch.Generator(device="cuda").manual_seed(seed)
    E, m = len(counts), sum(counts) + spare
    w = torch.randn(E, n, k, generator=g, device="cuda") / math.sqrt(k)
    b = 0.1 * torch.randn(E, n, generator=g, device="cuda") if bias else None
    layer = ex.ExpertLinear(w, m, dtype, b, act)
    x, dy = (torch.randn(m, c, generator=g, device="cuda").to(dtype) for c in (k, n))
    offsets = torch.tensor([0] + counts).cumsum(0).to(torch.int32).cuda()
    return layer, x, dy, offsets, g


def near(got, ref, size, terms, dtype, more=0.0):
    """Sums of `terms` products of 16-bit operands, cut by the tensor core at 2^-23 a step of 16, and one rounding to the type."""
    info = torch.finfo(dtype)
    off = (min(terms, 4096) / 16 * 2.0 ** -23 + 2.0 ** -21) * size + (info.eps / 2) * ref.abs() + info.smallest_normal * info.eps + more
    assert ((got.double() - ref).abs() <= off).all()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("counts,n,k", [([5, 0, 20, 1], 40, 72), ([300, 130, 0, 257], 136, 264)])
def test_a_life(mods, dtype, counts, n, k):
    """A training step against the formulas, the clipped gradients and the update, then the answers of the layer in 4 bits against the weights they stand for."""
    ebs, ex, search = mods
    layer, x, dy, offsets, g = make(mods, counts, n, k, dtype, ebs.EBS_ACT_SILU)
    other, ox, ody, _ = search_layer(mods, g)
    clip = search.GradientClip([layer, other])
    y = layer.forward(x, offsets).clone()
    dx = layer.backward(dy).clone()
    other.forward(ox)
    other.backward(ody)
    half = torch.finfo(dtype).eps / 2
    for e in range(len(counts)):
        s = slice(int(offsets[e]), int(offsets[e + 1]))
        xs, w = x[s].double(), layer.w[e].double()
        z = xs @ w.t() + layer.b[e].double()
        size = xs.abs() @ w.abs().t() + layer.b[e].double().abs()
        near(layer.z[s], z, size, k, dtype)
        near(y[s], F.silu(z), 1.13 * size, k, dtype, 2.0 ** -19 * z.abs())
        v = layer.z[s].double().requires_grad_(True)
        (dz,) = torch.autograd.grad(F.silu(v), v, dy[s].double())
        err = (half + 2.0 ** -19) * dz.abs() + 2.0 ** -24          # dz is rounded before the products
        near(dx[s], dz @ w, dz.abs() @ w.abs(), n, dtype, err @ w.abs())
        near(layer.dw[e], dz.t() @ xs, dz.abs().t() @ xs.abs(), counts[e], dtype, err.t() @ xs.abs())
        near(layer.dbias[e], dz.sum(0), dz.abs().sum(0), 16, dtype, 2.0 ** -18 * dz.abs().sum(0))
    grads = [layer.dw, layer.dbias, other.dw, other.dbias]
    kept = [t.clone() for t in grads]
    norm = math.sqrt(sum(float(t.double().square().sum()) for t in kept))
    assert abs(float(clip(0.5 * norm)) - norm) <= (2.0 ** -23 + 2.0 ** -24) * norm
    for t, before in zip(grads, kept):
        info = torch.finfo(t.dtype)
        rounding = 2.0 ** -24 if t.dtype == torch.float32 else info.eps / 2 + 2.0 ** -24
        assert ((t.double() - 0.5 * before.double()).abs() <= (rounding + 2.0 ** -22) * 0.5 * before.double().abs() + info.smallest_normal * info.eps).all()
    before, bias = layer.weight.clone(), layer.bias.clone()
    layer.step(0.01)
    assert torch.equal(layer.bias, bias - 0.01 * layer.dbias.float()) or torch.allclose(layer.bias, bias - 0.01 * layer.dbias.float(), rtol=0, atol=2.0 ** -23)
    assert torch.equal(layer.weight, before.sub(layer.update, alpha=0.01)) and torch.equal(layer.w, layer.weight.to(dtype)) and torch.equal(layer.b, layer.bias.to(dtype))
    # the update: singular values of an orthogonalised matrix; an expert without rows had no gradient
    for e, c in enumerate(counts):
        if c == 0:
            assert not layer.update[e].any()
            continue
        sigma = torch.linalg.svdvals(layer.update[e].double())
        assert sigma.max() <= 1.3
    served = layer.quantized(8, group=32)
    values = torch.empty(len(counts), n, k, device="cuda")
    ebs.ebs_unpack_weights_q4(served.packed, served.q4, values, ebs.EBS_F32)
    step = layer.weight.abs().view(len(counts), n, -1)
    assert ((values - layer.weight).abs() <= step.amax(dim=2, keepdim=True) / 7 * (0.5 + 2.0 ** -6)).all()     # half a code of the largest scale a row can have
    for take in ([0, 0, 1, 0], [3, 0, 2, 3], [0, 8, 0, 0]):
        o = torch.tensor([0] + take).cumsum(0).to(torch.int32).cuda()
        t = torch.randn(sum(take), k, generator=g, device="cuda").to(dtype)
        out = served.answer(t, o)
        for e, c in enumerate(take):
            s = slice(int(o[e]), int(o[e + 1]))
            w = values[e].double()
            z = t[s].double() @ w.t() + served.bias[e].double()
            size = t[s].double().abs() @ w.abs().t() + served.bias[e].double().abs()
            near(out[s], F.silu(z), 1.13 * size, 64, dtype, 2.0 ** -19 * z.abs())


def search_layer(mods, g):
    ebs, _, search = mods
    w, b = torch.randn(24, 40, generator=g, device="cuda"), torch.randn(24, generator=g, device="cuda")
    layer = search.SearchLinear(w, 12, [2, 4], [0.5, 0.5], [0.3, 0.7], 2.0, b, ebs.EBS_ACT_RELU)
    return layer, torch.randn(12, 40, generator=g, device="cuda"), torch.randn(12, 24, generator=g, device="cuda"), g


def test_step_captured_and_replayed(mods):
    """Forward, backward, clip and update of both kinds of layers in one graph equal the calls one by one."""
    ebs, ex, search = mods
    results = []
    for captured in (False, True):
        layer, x, dy, offsets, g = make(mods, [40, 0, 7], 48, 64, torch.bfloat16, ebs.EBS_ACT_GELU, seed=4)
        other, ox, ody, _ = search_layer(mods, g)
        clip = search.GradientClip([layer, other])

        def step():
            layer.forward(x, offsets)
            layer.backward(dy)
            other.forward(ox)
            other.backward(ody)
            clip(0.25)
            layer.step(0.02)
            other.step(0.02)
        step()
        if captured:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
                step()
            for _ in range(3):
                graph.replay()
        else:
            for _ in range(3):
                step()
        torch.cuda.synchronize()
        results.append([t.clone() for t in (layer.weight, layer.bias, layer.w, other.weight, other.bias, clip.norm)])
    assert all(torch.equal(a, b) for a, b in zip(*results))


def test_on_another_stream_and_answers_captured(mods):
    ebs, ex, search = mods
    g = torch.Generator(device="cuda").manual_seed(9)
    w = torch.randn(5, 64, 128, generator=g, device="cuda")
    served = ex.QuantizedExperts(w, 4, torch.float16, None, ebs.EBS_ACT_NONE, 64)
    x, o = torch.randn(4, 128, generator=g, device="cuda").half(), torch.tensor([0, 1, 1, 3, 3, 4], dtype=torch.int32).cuda()
    want = served.answer(x, o).clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        served.y.zero_()
        assert torch.equal(served.answer(x, o), want)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        served.answer(x, o)
    served.y.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(served.y, want)


def test_refusals(mods):
    ebs, ex, search = mods
    w = torch.zeros(2, 8, 16, device="cuda")
    for bad in (dict(weight=w[0]), dict(weight=w.cpu()), dict(weight=w.half()), dict(rows=0), dict(dtype=torch.float32), dict(bias=torch.zeros(2, 9, device="cuda")), dict(act=7),
                dict(steps=65)):
        with pytest.raises(ValueError):
            ex.ExpertLinear(**{**dict(weight=w, rows=4, dtype=torch.bfloat16), **bad})
    layer = ex.ExpertLinear(w, 4, torch.bfloat16)
    x, o = torch.zeros(4, 16, device="cuda").bfloat16(), torch.zeros(3, dtype=torch.int32, device="cuda")
    with pytest.raises(RuntimeError):
        layer.backward(torch.zeros(4, 8, device="cuda").bfloat16())
    for args in ((x[:3], o), (x.float(), o), (x, o[:2]), (x, o.long()), (x, o.cpu()), (x.cpu(), o)):
        with pytest.raises(ValueError):
            layer.forward(*args)
    layer.forward(x, o)
    with pytest.raises(ValueError):
        layer.backward(x)
    for bad in (dict(group=16), dict(act=-1), dict(rows=0), dict(weight=w.half())):
        with pytest.raises(ValueError):
            ex.QuantizedExperts(**{**dict(weight=w, rows=4, dtype=torch.float16, group=32), **bad})
    served = layer.quantized(2, 32)
    for args in ((x, o), (x[:2].half(), o), (x[:2], o[:2])):
        with pytest.raises(ValueError):
            served.answer(*args)
    assert served.answer(x[:0], o).shape == (0, 8)
    with pytest.raises(ValueError):
        search.GradientClip([])
