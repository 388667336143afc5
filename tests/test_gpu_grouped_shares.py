"""Layers of experts of very uneven shares, and sums of one sign, where what the tensor core cuts off adds up."""
import pytest
import torch

from test_gpu_grouped import code, layer, truncation

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ebs():
    from paper_2003_07577_b200 import binding
    return binding


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("counts", [[0] * 40 + [2048] + [0] * 23, [1] * 30 + [1500, 0, 0, 300] + [2] * 30, [33] + [0] * 62 + [2015], [0] * 99 + [70] + [0] * 3, [0] * 3], ids=lambda c: f"{len(c)}-{max(c)}")
@pytest.mark.parametrize("n,k,ldy", [(200, 328, 0), (72, 1031, 75), (2100, 72, 0)])
def test_most_rows_are_one_experts(ebs, dtype, counts, n, k, ldy):
    """At most 32 rows an expert in the mean: tiles of 32 rows, a column of many of them for the one that has the rows."""
    layer(ebs, 31, counts, n, k, dtype, act=4, residual=True, keep=True, spare=5, first=2, ldy=ldy)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("counts", [[7000] + [60] * 15, [0, 9000, 1, 0], [1] * 15 + [5000]], ids=lambda c: f"{len(c)}-{max(c)}")
def test_one_expert_has_most_of_many_rows(ebs, dtype, counts):
    layer(ebs, 32, counts, 520, 776, dtype, act=3, keep=True, spare=33)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("counts", [[24, 0, 3], [300, 129]], ids=str)
@pytest.mark.parametrize("n,k", [(136, 4096), (72, 8200), (2056, 4096)])
def test_sums_of_one_sign(ebs, dtype, counts, n, k):
    """What a result rounds is found by a second call, with the negative result as the residual (their difference is exact in fp32, and rounded by (eps / 2)^2 of the sum)."""
    g = torch.Generator(device="cuda").manual_seed(33)
    t, experts, m = torch.float16 if dtype == "f16" else torch.bfloat16, len(counts), sum(counts)
    x, w = ((torch.rand(s, generator=g, device="cuda") * 0.5 + 0.5).to(t) for s in ((m, k), (experts, n, k)))
    offsets = torch.tensor([0] + counts).cumsum(0).to(torch.int32).cuda()
    d = ebs.linear_desc(m, n, k, code(ebs, dtype))
    ws = torch.empty(max(16, ebs.ebs_grouped_workspace_bytes(d, experts)), dtype=torch.uint8, device="cuda")
    y, rest = (torch.zeros(m, n, dtype=t, device="cuda") for _ in range(2))
    ebs.ebs_grouped_forward(x, w, None, None, offsets, experts, d, y, None, ws)
    ebs.ebs_grouped_forward(x, w, None, -y, offsets, experts, d, rest, None, ws)
    row = 0
    for e, c in enumerate(counts):
        s = slice(row, row + c)
        ref = x[s].double() @ w[e].double().t()
        off = (truncation(k) + (torch.finfo(t).eps / 2) ** 2) * ref
        assert ((y[s].double() + rest[s].double() - ref).abs() <= off).all()
        row += c
