"""Layers with weights of 4 bits: sums of one sign, where what the tensor core cuts off adds up."""
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ebs():
    from paper_2003_07577_b200 import binding
    return binding


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("m", [1, 8, 9, 16, 33])
@pytest.mark.parametrize("n,k", [(512, 128), (37, 64), (16, 200), (512, 4096), (40, 32)])
def test_sums_of_one_sign(ebs, dtype, group, m, n, k):
    """include/ebs.h: products are exact, a sum in the tensor core is off by 2^-21 at most (16-bit types with groups of 128, which are summed there as a whole: 2^-20): four
    (eight) steps over 16 inputs, each of which cuts at 2^-23 of what it holds; fp32 activations as three planes, the small ones first (2^-7 and 2^-15 of the sum: nothing beside it).
    Then a rounding for each sum of a warp's and for each warp.  What a 16-bit result rounds is found by a second call, with the negative result as the residual: z - y is
    exact in fp32 (the two are within a factor of two), half a step of z at most, and rounded by half a step of itself: (eps / 2)^2 of z."""
    t, code = TYPES[dtype], {"f32": ebs.EBS_F32, "f16": ebs.EBS_F16, "bf16": ebs.EBS_BF16}[dtype]
    g = torch.Generator(device="cuda").manual_seed(1)
    w = (torch.rand(1, n, k, generator=g, device="cuda") * 0.5 + 0.5).to(t)
    x = (torch.rand(m, k, generator=g, device="cuda") + 1).to(t)
    q, d = ebs.q4_desc(n, k, group, code), ebs.linear_desc(m, n, k, code)
    packed = torch.empty(ebs.ebs_q4_packed_bytes(q), dtype=torch.uint8, device="cuda")
    ebs.ebs_pack_weights_q4(w, code, q, packed)
    values = torch.empty(n, k, device="cuda")
    ebs.ebs_unpack_weights_q4(packed, q, values, ebs.EBS_F32)
    y, ws = torch.empty(m, n, dtype=t, device="cuda"), torch.empty(max(16, ebs.ebs_linear_q4_workspace_bytes(d, q)), dtype=torch.uint8, device="cuda")
    ebs.ebs_linear_q4_forward(x, packed, None, None, None, d, q, y, ws)
    got = y.double()
    if dtype != "f32":
        rest = torch.empty_like(y)
        ebs.ebs_linear_q4_forward(x, packed, None, -y, None, d, q, rest, ws)
        got = got + rest.double()
    # (values is rounded to fp32 from a product of 24 and 4 bits: the codes are brought back, their products with the kept scales are exact)
    real = values.double()
    if dtype == "f32":
        real = torch.empty_like(real)
        for c in range(0, k, group):
            part = w[0, :, c:c + group].double()
            scale = (part.abs().amax(dim=1, keepdim=True).float() * (1.0 / torch.tensor(7.0, device="cuda"))).double()
            real[:, c:c + group] = scale * torch.floor(part / scale + 0.5).clamp(-8, 7)
    ref = x.double() @ real.t()
    tiles = (k + 63) // 64
    warps = 2 if tiles <= 4 else 16
    roundings = -(-tiles // min(warps, 4)) + warps
    off = (2.0 ** (-20 if dtype != "f32" and group == 128 else -21) + roundings * 2.0 ** -24) * ref
    if dtype != "f32":
        off = off + (torch.finfo(t).eps / 2) ** 2 * ref
    assert ((got - ref).abs() <= off).all(), float(((got - ref).abs() / off).max())
