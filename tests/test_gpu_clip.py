"""Clipping of gradients by their norm against the formula in 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]
# The sum of squares is off by 2^-22 of itself at most (four or eight squares added in fp32), the norm by half of that; the factor and its product
# with a gradient are rounded to fp32, the norm is stored as fp32.
NORM_TOLERANCE = 2.0 ** -23 + 2.0 ** -24
FACTOR_TOLERANCE = 2.0 ** -23 + 2.0 ** -24


@pytest.fixture(scope="module")
def ebs():
    from paper_2003_07577_b200 import binding
    return binding


def clip(ebs, tensors, max_norm, outs=None, stream=None):
    plan = ebs.clip_plan(tensors, outs)
    norm = torch.full((1,), -1.0, device="cuda")
    ws = torch.full((ebs.ebs_clip_workspace_bytes(plan),), 255, dtype=torch.uint8, device="cuda")     # (NaN: nothing of it may be read before it is written)
    ebs.ebs_clip_gradients(plan, max_norm, norm, ws, stream)
    return norm


def check(tensors, outs, norm, max_norm):
    """outs and norm against 64 bits; tensors: the gradients before the call."""
    want = math.sqrt(sum(float(t.double().square().sum()) for t in tensors))
    max_norm = float(torch.tensor(max_norm, dtype=torch.float32))        # (what the call gets)
    assert abs(float(norm) - want) <= NORM_TOLERANCE * want + 2.0 ** -149
    if want <= max_norm * (1 - NORM_TOLERANCE):
        for t, o in zip(tensors, outs):
            assert torch.equal(t, o)
        return
    f = min(1.0, max_norm / want) if want else 1.0
    for t, o in zip(tensors, outs):
        ref, info = t.double() * f, torch.finfo(t.dtype)
        half = 2.0 ** -24 if t.dtype == torch.float32 else info.eps / 2 + 2.0 ** -24                  # product in fp32, then rounded
        tiny = info.smallest_normal * info.eps                                                        # a step below the normal range (half of it, and fp32's own)
        assert ((o.double() - ref).abs() <= (half + FACTOR_TOLERANCE) * ref.abs() + tiny).all()


def grads(seed, shapes, scale=0.01):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [(torch.randn(shape, generator=g, device="cuda") * scale).to(t) for shape, t in shapes]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes", [[1], [7], [8], [9], [8191, 8192, 8193], [1, 2, 3, 4, 5, 6, 7, 8, 9, 0, 33], [100003], [1 << 20, 17], [3] * 2000])
@pytest.mark.parametrize("ratio", [0.3, 2.0])
def test_sizes(ebs, dtype, sizes, ratio):
    ts = grads(1, [((n,), dtype) for n in sizes])
    outs = [torch.empty_like(t) for t in ts]
    max_norm = ratio * 0.01 * math.sqrt(max(1, sum(sizes)))
    check(ts, outs, clip(ebs, ts, max_norm, outs), max_norm)
    kept = [t.clone() for t in ts]
    check(kept, ts, clip(ebs, ts, max_norm), max_norm)                  # in place


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,ld_in,ld_out", [(1, 100, 100, 100), (300, 1, 2, 1), (13, 7, 11, 7), (50, 1000, 1005, 1008), (9, 8195, 8200, 8195), (2000, 31, 31, 40), (64, 1536, 1537, 1536)])
@pytest.mark.parametrize("shift_in,shift_out", [(0, 0), (1, 0), (3, 3), (5, 2)])
def test_strides_and_alignment(ebs, dtype, rows, cols, ld_in, ld_out, shift_in, shift_out):
    """Rows that start anywhere; what lies between them stays as it is."""
    g = torch.Generator(device="cuda").manual_seed(2)
    a = (torch.randn(shift_in + rows * ld_in, generator=g, device="cuda") * 0.01).to(dtype)
    b = torch.full((shift_out + rows * ld_out,), 7.0, dtype=dtype, device="cuda")
    t, o = a.as_strided((rows, cols), (ld_in, 1), shift_in), b.as_strided((rows, cols), (ld_out, 1), shift_out)
    between = torch.ones_like(a, dtype=torch.bool)
    between.as_strided((rows, cols), (ld_in, 1), shift_in)[:] = False
    a[between] = math.nan                                               # never read
    kept = t.clone()
    check([kept], [o], clip(ebs, [t], 0.05, [o]), 0.05)
    outside = torch.ones_like(b, dtype=torch.bool)
    outside.as_strided((rows, cols), (ld_out, 1), shift_out)[:] = False
    assert (b[outside] == 7.0).all()
    check([kept], [t], clip(ebs, [t], 0.05), 0.05)
    assert a[between].isnan().all()


def test_types_together(ebs):
    ts = grads(3, [((64, 576), torch.bfloat16), ((64,), torch.float32), ((1000, 512), torch.float16), ((1000,), torch.float32), ((0,), torch.float16)])
    outs = [torch.empty_like(t) for t in ts]
    check(ts, outs, clip(ebs, ts, 1.0, outs), 1.0)


@pytest.mark.parametrize("dtype,scale", [(torch.float32, 1e-30), (torch.float32, 1e-18), (torch.float32, 1e25), (torch.float32, 1e-43), (torch.bfloat16, 1e-30), (torch.bfloat16, 1e28),
                                         (torch.float16, 1e-7), (torch.float16, 1e4)])
def test_squares_beyond_fp32(ebs, dtype, scale):
    ts = grads(4, [((5000,), dtype), ((333,), dtype)], scale)
    ts[1][::3] = 0
    outs = [torch.empty_like(t) for t in ts]
    max_norm = 0.25 * scale
    check(ts, outs, clip(ebs, ts, max_norm, outs), max_norm)


def test_norm_beyond_fp32(ebs):
    """The norm leaves the type's range, the factor does not."""
    t = torch.full((10000,), 3e38, device="cuda")
    out = torch.empty_like(t)
    norm = clip(ebs, [t], 1e38, [out])
    assert float(norm) == math.inf
    assert torch.allclose(out, torch.full_like(out, 1e38 / 100), rtol=1e-6, atol=0)


@pytest.mark.parametrize("dtype", TYPES)
def test_not_finite(ebs, dtype):
    for bad, max_norm in ((math.inf, 1.0), (-math.inf, 1.0), (math.nan, 1.0), (math.nan, math.inf)):
        t = grads(5, [((3000,), dtype)])[0]
        t[1234] = bad
        out = torch.empty_like(t)
        norm = float(clip(ebs, [t], max_norm, [out]))
        if math.isnan(bad):
            assert math.isnan(norm) and out.isnan().all()
        else:
            assert norm == math.inf and out[1234].isnan() and (out[:1234] == 0).all() and (out[1235:] == 0).all()
    t = grads(5, [((3000,), dtype)])[0]
    t[7] = math.inf
    out = torch.empty_like(t)
    assert float(clip(ebs, [t], math.inf, [out])) == math.inf and torch.equal(out, t)              # the norm alone


def test_zero_gradients_and_zero_bound(ebs):
    t = torch.zeros(5000, device="cuda")
    assert float(clip(ebs, [t], 0.0)) == 0.0 and (t == 0).all()
    t = grads(6, [((5000,), torch.float32)])[0]
    assert float(clip(ebs, [t], 0.0)) > 0 and (t == 0).all()
    assert float(clip(ebs, [], 1.0)) == 0.0
    assert float(clip(ebs, [torch.zeros(0, 4, device="cuda")], 1.0)) == 0.0


def test_repeatable_and_captured(ebs):
    """The same bits every time, from a graph on another stream too, with new gradients in the same places."""
    ts = grads(7, [((n,), torch.bfloat16) for n in (40000, 17, 300001)])
    outs = [torch.empty_like(t) for t in ts]
    plan = ebs.clip_plan(ts, outs)
    norm = torch.zeros(1, device="cuda")
    ws = torch.empty(ebs.ebs_clip_workspace_bytes(plan), dtype=torch.uint8, device="cuda")
    ebs.ebs_clip_gradients(plan, 0.5, norm, ws)
    first = [norm.clone()] + [o.clone() for o in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        ebs.ebs_clip_gradients(plan, 0.5, norm, ws)
    for _ in range(3):
        for o in [norm] + outs:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(first, [norm] + outs):
            assert torch.equal(a, b)
    for t in ts:
        t.mul_(3.0)
    kept = [t.clone() for t in ts]
    graph.replay()
    torch.cuda.synchronize()
    check(kept, outs, norm, 0.5)


def test_past_32_bits(ebs):
    """More than 2^31 elements in one tensor: the last ones count and are scaled."""
    n = (1 << 31) + 12345
    t = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    t[-1], t[0] = 4.0, 3.0
    norm = clip(ebs, [t], 2.5)
    assert float(norm) == 5.0 and float(t[-1]) == 2.0 and float(t[0]) == 1.5 and int((t != 0).sum()) == 2
