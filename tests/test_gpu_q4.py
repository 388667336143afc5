"""Layers with weights of 4 bits against the definition in 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

SEVENTH = 1.0 / torch.tensor(7.0)            # rounded to fp32, as the scale's definition has it
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
F = torch.nn.functional
ACTS = [lambda v: v, torch.relu, F.gelu, lambda v: F.gelu(v, approximate="tanh"), F.silu]


@pytest.fixture(scope="module")
def ebs():
    from paper_2003_07577_b200 import binding
    return binding


def code(ebs, name):
    return {"f32": ebs.EBS_F32, "f16": ebs.EBS_F16, "bf16": ebs.EBS_BF16}[name]


def values(w, group, dtype):
    """What the packed weights stand for, in 64 bits: scale (kept in the layer's type) times code."""
    out = torch.empty(w.shape, dtype=torch.float64, device=w.device)
    for c in range(0, w.shape[-1], group):
        part = w[..., c:c + group].double()
        s = (part.abs().amax(dim=-1, keepdim=True).float() * SEVENTH.to(w.device)).to(TYPES[dtype]).double()
        q = torch.floor(part / s + 0.5).clamp(-8, 7)
        out[..., c:c + group] = torch.where(s > 0, s * q, torch.zeros_like(q))
    return out


def make(ebs, w, group, dtype, source):
    experts, n, k = w.shape
    q = ebs.q4_desc(n, k, group, code(ebs, dtype), experts)
    packed = torch.full((ebs.ebs_q4_packed_bytes(q),), 255, dtype=torch.uint8, device="cuda")
    ebs.ebs_pack_weights_q4(w, code(ebs, source), q, packed)
    return q, packed


def weights(seed, *shape, dtype="f32"):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") / math.sqrt(shape[-1])).to(TYPES[dtype])


@pytest.mark.parametrize("source,dtype", [("f32", "f32"), ("f32", "f16"), ("f32", "bf16"), ("f16", "f16"), ("bf16", "bf16"), ("f16", "f32"), ("bf16", "f16")])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("experts,n,k", [(1, 1, 1), (1, 16, 64), (2, 17, 65), (1, 15, 31), (3, 33, 191), (1, 333, 1027), (2, 64, 4096), (1, 8, 33), (1, 16, 129)])
def test_pack_and_read_back(ebs, source, dtype, group, experts, n, k):
    w = weights(1, experts, n, k, dtype=source)
    q, packed = make(ebs, w, group, dtype, source)
    want = values(w, group, dtype)
    for to in ("f32", "f16", "bf16"):
        out = torch.full((experts, n, k), math.nan, dtype=TYPES[to], device="cuda")
        ebs.ebs_unpack_weights_q4(packed, q, out, code(ebs, to))
        assert torch.equal(out, want.float().to(TYPES[to]))              # a product of 24 and 4 bits, rounded to fp32 and to the type


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_borders_between_codes(ebs, dtype):
    """Weights on and next to the borders (j + 1/2) scale; magnitudes down to the smallest numbers."""
    rows = []
    for e in (0, -20, 20, -100, -126, -140, 100):
        s = torch.tensor(2.0 ** e, dtype=torch.float64)
        for top in (7.0, 7.25, 6.9):
            row = torch.zeros(64, dtype=torch.float64)
            row[0] = top * s
            scale = (row[0].float() * SEVENTH).to(TYPES[dtype]).double()
            borders = ((torch.arange(-8, 8, dtype=torch.float64) + 0.5) * scale).float()
            row[1:17] = borders.double()
            row[17:33] = torch.nextafter(borders, torch.tensor(math.inf)).double()
            row[33:49] = torch.nextafter(borders, torch.tensor(-math.inf)).double()
            row = row.clamp(-float(row[0].float()), float(row[0].float()))
            rows.append(row.float())
    w = torch.stack(rows)[None].cuda()
    q, packed = make(ebs, w, 64, dtype, "f32")
    out = torch.empty_like(w)
    ebs.ebs_unpack_weights_q4(packed, q, out, ebs.EBS_F32)
    assert torch.allclose(out, values(w, 64, dtype).float(), rtol=0, atol=0, equal_nan=True)         # (2^100 / 7 is beyond fp16: NaN)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_strided_weights_and_untouched_memory(ebs, dtype):
    experts, n, k, ld = 2, 37, 100, 105
    big = torch.full((experts * n, ld), math.nan, dtype=TYPES[dtype], device="cuda")
    big[:, :k] = weights(2, experts * n, k, dtype=dtype)
    q = ebs.q4_desc(n, k, 32, code(ebs, dtype), experts)
    packed = torch.full((ebs.ebs_q4_packed_bytes(q) + 256,), 77, dtype=torch.uint8, device="cuda")
    ebs.ebs_pack_weights_q4(big, code(ebs, dtype), q, packed, ldw=ld)
    assert (packed[-256:] == 77).all()
    out = torch.full((experts * n, ld), 5.0, dtype=TYPES[dtype], device="cuda")
    ebs.ebs_unpack_weights_q4(packed, q, out, code(ebs, dtype), ldw=ld)
    assert torch.equal(out[:, :k], values(big[:, :k], 32, dtype).float().to(TYPES[dtype])) and (out[:, k:] == 5.0).all()


def test_weights_not_finite(ebs):
    for bad in (math.inf, -math.inf, math.nan, 1e30):                    # the last: a scale beyond fp16
        w = weights(3, 1, 20, 200)
        w[0, 3, 70] = bad
        q, packed = make(ebs, w, 64, "f16", "f32")
        out = torch.empty_like(w)
        ebs.ebs_unpack_weights_q4(packed, q, out, ebs.EBS_F32)
        assert out[0, 3, 64:128].isnan().all() and int(out.isnan().sum()) == 64
        d = ebs.linear_desc(2, 20, 200, ebs.EBS_F16)
        x, y = torch.ones(2, 200, dtype=torch.float16, device="cuda"), torch.zeros(2, 20, dtype=torch.float16, device="cuda")
        ebs.ebs_linear_q4_forward(x, packed, None, None, None, d, q, y)
        assert y[:, 3].isnan().all() and int(y.isnan().sum()) == 2


def check(y, x, w, bias, residual, act, rows=None):
    """y against 64 bits.  Products are exact; a tile's sum takes up to twelve steps in the tensor core, each of which cuts at 2^-23 of what it holds (2^-20 for all),
    then a rounding for each 64 inputs of a warp's eighth, for each warp and for the bias; activations of 16-bit types within 2^-19; one rounding to the type."""
    z = x.double() @ w.t()
    size = x.double().abs() @ w.abs().t()
    if bias is not None:
        z = z + bias.double()
        size = size + bias.double().abs()
    ref = ACTS[act](z)
    steps = (x.shape[1] + 63) // 64 / 8 + 12
    off = (2.0 ** -20 + steps * 2.0 ** -24) * size * 1.13 + (2.0 ** -19 * (ref.abs() + z.abs()) if act > 1 else 0.0)
    if residual is not None:
        ref = ref + residual.double()
        off = off + 2.0 ** -23 * ref.abs()
    info = torch.finfo(y.dtype)
    off = off + (info.eps / 2) * ref.abs() + info.smallest_normal * info.eps
    bad = (y.double() - ref).abs() > off
    assert not bad.any(), (int(bad.sum()), float(((y.double() - ref).abs() / off).max()))


def run(ebs, seed, m, n, k, group, dtype, act=0, bias=False, residual=False, ldx=0, ldy=0, counts=None, in_place=False):
    """One call of random inputs, checked; counts: rows of each expert (the rest are nobody's)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = TYPES[dtype]
    experts = 1 if counts is None else len(counts)
    w = weights(seed + 1, experts, n, k, dtype=dtype)
    q, packed = make(ebs, w, group, dtype, dtype)
    xs = torch.full((m, ldx or k), math.nan, dtype=t, device="cuda")
    xs[:, :k] = torch.randn(m, k, generator=g, device="cuda").to(t)
    b = torch.randn(experts, n, generator=g, device="cuda").to(t) if bias else None
    ys = torch.full((m, ldy or n), 3.0, dtype=t, device="cuda")
    r = None
    if residual:
        r = ys if in_place else torch.randn(m, n, generator=g, device="cuda").to(t)
        if in_place:
            ys[:, :n] = torch.randn(m, n, generator=g, device="cuda").to(t)
    kept = ys.clone()
    res = r[:, :n].clone() if residual else None
    d = ebs.linear_desc(m, n, k, code(ebs, dtype), act, ldx=ldx, ldy=ldy, ldr=ldy if in_place else 0)
    ws = torch.full((max(16, ebs.ebs_linear_q4_workspace_bytes(d, q)),), 255, dtype=torch.uint8, device="cuda")
    offsets = None if counts is None else torch.tensor([0] + list(counts), dtype=torch.int32).cumsum(0).to(torch.int32).cuda()
    ebs.ebs_linear_q4_forward(xs, packed, b, r, offsets, d, q, ys, ws)
    real, row = values(w, group, dtype), 0
    for e, c in enumerate([m] if counts is None else counts):
        if c:
            s = slice(row, row + c)
            check(ys[s, :n], xs[s, :k], real[e], None if b is None else b[e], None if res is None else res[s], act)
        row += c
    assert torch.equal(ys[row:], kept[row:])                             # rows of no expert
    assert torch.equal(ys[:, n:], kept[:, n:])


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("m", [1, 2, 7, 8, 9, 16, 17, 31, 33, 64, 65, 130])
@pytest.mark.parametrize("n,k,group", [(1000, 512, 32), (17, 65, 64), (40, 4160, 128), (1, 1, 32)])
def test_rows(ebs, dtype, m, n, k, group):
    run(ebs, 5, m, n, k, group, dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("n,k", [(15, 63), (16, 64), (33, 129), (200, 1027), (64, 2048), (4096, 33)])
def test_groups(ebs, dtype, group, n, k):
    run(ebs, 6, 3, n, k, group, dtype, act=4, bias=True, residual=True)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("act", range(5))
def test_activations(ebs, dtype, act):
    run(ebs, 7, 5, 130, 300, 64, dtype, act=act, bias=True)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("m,k,ldx,ldy", [(1, 100, 101, 0), (6, 100, 101, 37), (6, 101, 0, 0), (20, 128, 136, 50), (3, 64, 65, 64)])
def test_strides(ebs, dtype, m, k, ldx, ldy):
    run(ebs, 8, m, 33, k, 32, dtype, ldx=ldx, ldy=ldy, residual=True, in_place=True)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("counts,spare", [([0, 0, 3], 0), ([1] * 40, 5), ([0] * 70 + [2], 1), ([24, 0, 1, 100, 0, 9], 7), ([0, 0], 4), ([7], 2), ([0] * 33 + [5] + [0] * 33 + [1], 0)])
def test_experts(ebs, dtype, counts, spare):
    run(ebs, 9, sum(counts) + spare, 50, 200, 64, dtype, act=4, bias=True, residual=True, counts=counts)


def test_offsets_that_are_not_in_order(ebs):
    """Taken as the nearest ones that are: nothing out of bounds is read or written."""
    q, packed = make(ebs, weights(10, 3, 20, 64), 64, "f32", "f32")
    d = ebs.linear_desc(10, 20, 64, ebs.EBS_F32)
    for offsets in ([0, 5, 3, 100], [-7, 2, 1 << 30, 4], [9, 8, 7, 6], [2147483647, -2147483648, 0, 10], [10, 10, 10, 10]):
        x, y = torch.randn(10, 64, device="cuda"), torch.full((12, 20), 3.0, device="cuda")
        ebs.ebs_linear_q4_forward(x, packed, None, None, torch.tensor(offsets, dtype=torch.int32).cuda(), d, q, y)
        torch.cuda.synchronize()
        assert (y[10:] == 3.0).all() and y.isfinite().all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_activations_not_finite(ebs, dtype):
    """An infinity or a NaN reaches its own row, as the products have it (a code of zero makes NaN of an infinity)."""
    w = weights(11, 1, 40, 128, dtype=dtype)
    q, packed = make(ebs, w, 64, dtype, dtype)
    real = values(w, 64, dtype)[0]
    x = weights(12, 12, 128, dtype=dtype)
    x[2, 5], x[4, 100], x[9, 64], x[9, 66] = math.inf, math.nan, math.inf, -math.inf
    if dtype == "f32":
        x[6, 3] = torch.tensor([0x7f800001], dtype=torch.int32).view(torch.float32)[0].cuda()           # a NaN of low bits alone
        x[7, 3] = 1e35
    y = torch.zeros(12, 40, dtype=TYPES[dtype], device="cuda")
    ebs.ebs_linear_q4_forward(x, packed, None, None, None, ebs.linear_desc(12, 40, 128, code(ebs, dtype)), q, y)
    ref = (x.double()[:, None, :] * real[None]).sum(dim=2)
    good = [r for r in range(12) if r not in (2, 4, 9, 6, 7)]
    check(y[good], x[good], real, None, None, 0)
    for r in (2, 9):
        assert torch.equal(y[r].isnan(), ref[r].isnan()) and torch.equal(y[r].double()[~ref[r].isnan()], ref[r][~ref[r].isnan()])
    assert y[4].isnan().all()
    if dtype == "f32":
        assert y[6].isnan().all()
        assert torch.allclose(y[7].double(), ref[7], rtol=1e-5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_captured_and_replayed(ebs, dtype):
    """A token's call in a graph on a side stream: new activations and new offsets in the same places."""
    t = TYPES[dtype]
    w = weights(13, 4, 96, 256, dtype=dtype)
    q, packed = make(ebs, w, 64, dtype, dtype)
    real = values(w, 64, dtype)
    x, y = torch.zeros(6, 257, dtype=t, device="cuda"), torch.zeros(6, 96, dtype=t, device="cuda")
    d = ebs.linear_desc(6, 96, 256, code(ebs, dtype), ldx=257)
    ws = torch.empty(ebs.ebs_linear_q4_workspace_bytes(d, q), dtype=torch.uint8, device="cuda")
    offsets = torch.tensor([0, 1, 2, 3, 4], dtype=torch.int32).cuda()
    ebs.ebs_linear_q4_forward(x, packed, None, None, offsets, d, q, y, ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        ebs.ebs_linear_q4_forward(x, packed, None, None, offsets, d, q, y, ws)
    for counts in ([1, 1, 1, 3], [0, 6, 0, 0], [2, 0, 2, 0]):
        x.copy_(torch.randn(6, 257, device="cuda"))
        offsets.copy_(torch.tensor([0] + counts).cumsum(0))
        y.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        row = 0
        for e, c in enumerate(counts):
            if c:
                check(y[row:row + c], x[row:row + c, :256], real[e], None, None, 0)
            row += c
        assert (y[row:] == 3.0).all()


def test_weights_past_32_bits(ebs):
    """Packed weights of more than 2^31 bytes, elements beyond 2^32: the last expert's rows."""
    experts, n, k = 70, 8192, 8192
    part = weights(14, 1, n, k, dtype="bf16")
    q = ebs.q4_desc(n, k, 128, ebs.EBS_BF16, experts)
    w = torch.zeros(experts, n, k, dtype=torch.bfloat16, device="cuda")
    w[-1] = part[0]
    packed = torch.empty(ebs.ebs_q4_packed_bytes(q), dtype=torch.uint8, device="cuda")
    assert packed.numel() > 1 << 31
    ebs.ebs_pack_weights_q4(w, ebs.EBS_BF16, q, packed)
    x, y = torch.randn(2, k, device="cuda").bfloat16(), torch.zeros(2, n, dtype=torch.bfloat16, device="cuda")
    offsets = torch.tensor([0] * 70 + [2], dtype=torch.int32).cuda()
    ebs.ebs_linear_q4_forward(x, packed, None, None, offsets, ebs.linear_desc(2, n, k, ebs.EBS_BF16), q, y)
    real = values(part, 128, "bf16")[0]
    check(y, x, real, None, None, 0)
    ebs.ebs_unpack_weights_q4(packed, q, w, ebs.EBS_BF16)
    assert torch.equal(w[-1], real.bfloat16()) and not w[:-1].any()
