"""GPU parity of the Newton-Schulz orthogonalisation against the iteration in 64 bits.

Tolerance: a step passes an error E of X on as at most a |E| (the slope at zero, the steepest for these coefficients), and adds its
own: the operands keep 22 bits (2^-22), the sums a few 2^-24 sqrt(K).  Relative to the largest singular value reached (1.3), five
steps give an error of at most 2^-21 * (1 + a + .. + a^4) in the spectral norm of each rounding's error matrix; that matrix is random, its
spectral norm is 2 / sqrt(longer side) of its Frobenius norm, which is at most sqrt(shorter side).  So per element, against the rms of
out, sqrt(1 / longer): a^5 / (a - 1) * 2^-21 * 2 with sums and products joined, plus the output's own rounding."""
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
COEFF = (3.4445, -4.7750, 2.0315)


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


def iterate64(g, steps, coeff=COEFF, eps=1e-7, scale=1.0):
    x = g.double()
    x = x / (x.pow(2).sum(dim=(-2, -1), keepdim=True).sqrt() + eps)
    a, b, c = coeff
    for _ in range(steps):
        s = x @ x.mT if x.shape[-2] <= x.shape[-1] else x.mT @ x
        p = b * s + c * (s @ s)
        x = a * x + (p @ x if x.shape[-2] <= x.shape[-1] else x @ p)
    return scale * x


def run(ebs, g, steps=5, coeff=COEFF, eps=1e-7, scale=1.0, out=None, stream=None, ws=None):
    batch, rows, cols = g.shape
    dt = {torch.float32: ebs.EBS_F32, torch.float16: ebs.EBS_F16, torch.bfloat16: ebs.EBS_BF16}[g.dtype]
    out = torch.full_like(g, math.nan) if out is None else out
    if ws is None:
        ws = torch.full((ebs.ebs_orthogonalize_workspace_bytes(batch, rows, cols, dt, steps) + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    ebs.ebs_orthogonalize(g, batch, rows, cols, dt, steps, coeff, eps, scale, out, ws, stream)
    return out


def make(batch, rows, cols, t, seed=0, rank=None):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    if rank is None:
        return (0.01 * torch.randn((batch, rows, cols), generator=gen, device="cuda")).to(t)
    u, v = (torch.randn(s, generator=gen, device="cuda") for s in ((batch, rows, rank), (batch, rank, cols)))
    return (0.01 * u @ v).to(t)


def check(got, ref, steps, coeff=COEFF, scale=1.0):
    t, longer = got.dtype, max(got.shape[-2:])
    a = abs(coeff[0]) if abs(coeff[0]) > 1 else 1.0001
    rms = ref.pow(2).mean(dim=(-2, -1), keepdim=True).sqrt()
    own = a ** steps / (a - 1) * 2.0 ** -20 * (scale * math.sqrt(1.0 / longer) + rms)
    u = torch.finfo(t).eps / 2
    tiny = torch.finfo(t).smallest_normal * torch.finfo(t).eps
    err = (got.double() - ref).abs()
    assert (err <= u * ref.abs() + 6 * own + tiny).all(), float((err / (u * ref.abs() + 6 * own + tiny)).max())   # 6: the largest of many elements
    assert (err.pow(2).mean().sqrt() <= u * rms.max() + own.max() + tiny)


SHAPES = [(1, 1, 1), (3, 1, 7), (2, 5, 1), (1, 2, 2), (6, 64, 576), (2, 576, 64), (3, 16, 144), (32, 16, 16), (1, 63, 65), (2, 129, 130), (1, 128, 128), (1, 257, 100),
          (1, 512, 4608), (1, 1024, 777), (1, 8, 7057), (1, 3001, 5), (2, 200, 1000),
          # the largest that stay in one thread block's shared memory, and one column more
          (2, 64, 640), (1, 640, 64), (1, 64, 641), (2, 33, 768), (1, 33, 769), (1, 16, 2560), (1, 2561, 16), (2, 17, 1000), (200, 20, 30)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("batch,rows,cols", SHAPES)
def test_sizes(ebs, batch, rows, cols, dtype):
    g = make(batch, rows, cols, TYPES[dtype], rows + cols)
    check(run(ebs, g), iterate64(g, 5), 5)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rank", [1, 3, 40])
def test_low_rank(ebs, dtype, rank):
    """Directions that G does not have: what roundings put there is multiplied by a^steps."""
    g = make(2, 200, 328, TYPES[dtype], rank, rank)
    check(run(ebs, g), iterate64(g, 5), 5)


@pytest.mark.parametrize("steps", [0, 1, 2, 9])
@pytest.mark.parametrize("coeff", [(1.5, -0.5, 0.0), (1.875, -1.25, 0.375)])
def test_steps_and_coefficients(ebs, steps, coeff):
    g = make(2, 96, 160, torch.float32, 1)
    check(run(ebs, g, steps, coeff, scale=0.25), iterate64(g, steps, coeff, scale=0.25), steps, coeff, 0.25)


@pytest.mark.parametrize("dtype", list(TYPES))
def test_scales_and_zeros(ebs, dtype):
    """A zero matrix gives zero, a single tiny or huge one what its multiple gives."""
    t = TYPES[dtype]
    g = make(4, 48, 80, torch.float32, 2)
    g[1] = 0
    g[2] *= 2.0 ** (100 if dtype != "f16" else 18)
    g[3] *= 2.0 ** (-60 if dtype != "f16" else -6)
    g = g.to(t)
    out = run(ebs, g, eps=0.0 if dtype == "f32" else 1e-7)
    if dtype == "f32":
        assert torch.isnan(out[1]).all()                     # 0 / 0: eps = 0 asks for it
        keep = [0, 2, 3]
    else:
        assert (out[1] == 0).all()
        keep = [0, 2] if dtype == "bf16" else [0, 2, 3]
    check(out[keep], iterate64(g[keep], 5, eps=0.0 if dtype == "f32" else 1e-7), 5)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("rows,cols", [(40, 72), (300, 200)])
def test_nan_and_infinity_stay_in_their_matrix(ebs, dtype, bad, rows, cols):
    g = make(3, rows, cols, TYPES[dtype], 3)
    clean = run(ebs, g)
    g[1, 7, 9] = bad
    out = run(ebs, g)
    assert torch.isnan(out[1]).all()
    assert torch.equal(out[0], clean[0]) and torch.equal(out[2], clean[2])


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("shape", [(2, 64, 144), (1, 300, 700)])
def test_in_place_streams_and_replay(ebs, dtype, shape):
    g = make(*shape, TYPES[dtype], 5)
    want = run(ebs, g)
    same = g.clone()
    run(ebs, same, out=same)
    assert torch.equal(same, want)
    dt = {"f32": ebs.EBS_F32, "f16": ebs.EBS_F16, "bf16": ebs.EBS_BF16}[dtype]
    ws = torch.zeros(ebs.ebs_orthogonalize_workspace_bytes(*shape, dt, 5), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())             # (behind the buffers' making)
    run(ebs, g, out=out, ws=ws, stream=side)
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(ebs, g, out=out, ws=ws)
    g.copy_(make(*shape, TYPES[dtype], 6))
    want = run(ebs, g)
    ws.fill_(0xFF)
    graph.replay()
    assert torch.equal(out, want)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows,cols", [(2100, 2304), (2304, 2100), (512, 4608)])
def test_large(ebs, dtype, rows, cols):
    """Symmetric products on and below the diagonal with their mirror images; a reduction in parts."""
    g = make(1, rows, cols, TYPES[dtype], 1)
    check(run(ebs, g), iterate64(g, 5), 5)


# one to eight blocks of a cluster: short sides up to 64 and up to 128, fewer and more columns than they hold, more matrices than run at once
CLUSTERED = [(1, 65, 65), (1, 100, 300), (2, 128, 1152), (1, 1152, 128), (1, 127, 1537), (1, 128, 1600), (1, 2048, 80), (1, 80, 2049), (3, 96, 96), (1, 112, 129), (20, 66, 513),
             (40, 128, 640), (1, 64, 4096), (1, 4097, 64), (1, 9, 4095), (18, 64, 576), (37, 64, 576), (75, 48, 200), (150, 64, 130)]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("batch,rows,cols", CLUSTERED)
def test_clusters(ebs, batch, rows, cols, dtype):
    g = make(batch, rows, cols, TYPES[dtype], rows + cols)
    check(run(ebs, g), iterate64(g, 5), 5)


@pytest.mark.parametrize("shape", [(2, 128, 1152), (1, 300, 96), (9, 100, 640), (2, 64, 2000)])
def test_clusters_in_place_and_replay(ebs, shape):
    g = make(*shape, torch.float32, 8)
    want = run(ebs, g)
    same = g.clone()
    run(ebs, same, out=same)
    assert torch.equal(same, want)
    out, ws = torch.empty_like(g), torch.zeros(ebs.ebs_orthogonalize_workspace_bytes(*shape, ebs.EBS_F32, 5), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(ebs, g, out=out, ws=ws)
        run(ebs, out, out=out, ws=ws)
    graph.replay()
    assert torch.equal(out, run(ebs, want))


@pytest.mark.parametrize("steps", [0, 1, 9])
@pytest.mark.parametrize("shape", [(2, 90, 700), (1, 900, 128), (3, 30, 400)])
def test_clusters_steps(ebs, shape, steps):
    for coeff in ((1.5, -0.5, 0.0), COEFF):
        g = make(*shape, torch.float32, 9)
        check(run(ebs, g, steps=steps, coeff=coeff, scale=0.7), iterate64(g, steps, coeff, scale=0.7), steps, coeff, 0.7)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1921, 1950), (1, 1800, 1793), (1, 2048, 2049), (2, 1100, 1300), (1, 768, 770)])
def test_symmetric_halves(ebs, dtype, shape):
    """Symmetric products in squares of two tiles, the last square with one or two of them."""
    g = make(*shape, TYPES[dtype], 2)
    check(run(ebs, g), iterate64(g, 5), 5)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_nan_and_infinity_cross_a_cluster(ebs, bad):
    g = make(3, 100, 640, torch.float32, 3)
    clean = run(ebs, g)
    g[1, 7, 639] = bad
    out = run(ebs, g)
    assert torch.isnan(out[1]).all()
    assert torch.equal(out[0], clean[0]) and torch.equal(out[2], clean[2])


# A few steps, whose tolerance is far below what 11 bits leave: X and Q on matrices of full rank, A where one singular value is all of G
FEW_STEPS = [(None, 2, COEFF), (None, 3, (1.875, -1.25, 0.375)), (1, 1, COEFF), (2, 2, COEFF)]


@pytest.mark.parametrize("rank,steps,coeff", FEW_STEPS)
@pytest.mark.parametrize("shape", [(1, 64, 576), (9, 576, 64), (1, 128, 1152), (2, 300, 700), (1, 700, 300), (1, 512, 1024), (1, 768, 770), (1, 2100, 1900)])
def test_few_steps_keep_both_planes(ebs, shape, rank, steps, coeff):
    g = make(*shape, torch.float32, 21, rank)
    check(run(ebs, g, steps, coeff), iterate64(g, steps, coeff), steps, coeff)
