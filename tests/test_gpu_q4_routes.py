"""Layers with weights of 4 bits, large enough for the forms that small ones do not reach: two to sixteen warps a tile, fp32 rows brought into planes first.

The form goes by the blocks, pieces of rows x tiles of 16 outputs (32 from 17 rows on), and the 64s of the reduction: planes from 8192 of their product on; four warps from 592 blocks on (16-bit
types with up to eight rows: 1184), two for up to four 64s, sixteen below 444 blocks from 32 on.  The sizes lie well past these."""
import pytest
import torch

from test_gpu_q4 import TYPES, check, code, make, run, values, weights

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ebs():
    from paper_2003_07577_b200 import binding
    return binding


def planes(ebs, m, n, k, group, experts=1, ldx=0):
    """Whether fp32 rows are brought into planes: three of 16-bit numbers, rows padded to whole 64s."""
    size = ebs.ebs_linear_q4_workspace_bytes(ebs.linear_desc(m, n, k, ebs.EBS_F32, ldx=ldx), ebs.q4_desc(n, k, group, ebs.EBS_F32, experts))
    return size == (m * ((k + 63) // 64 * 64) * 6 + 255) // 256 * 256


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("m", [1, 8, 9, 16, 33])
@pytest.mark.parametrize("n,k,ldx", [(24003, 1027, 0), (24008, 320, 323), (24003, 576, 584)])
def test_four_warps(ebs, dtype, group, m, n, k, ldx):
    """1500 tiles; fp32: planes of ragged rows that start anywhere, and of whole ones."""
    assert dtype != "f32" or planes(ebs, m, n, k, group, ldx=ldx) == (k > 320)
    run(ebs, 21, m, n, k, group, dtype, act=4, bias=True, ldx=ldx)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("m", [1, 5, 12])
def test_four_warps_without_planes(ebs, group, m):
    assert not planes(ebs, m, 9700, 320, group) and not planes(ebs, m, 9700, 320, group, ldx=321)
    run(ebs, 22, m, 9700, 320, group, "f32")
    run(ebs, 23, m, 9700, 320, group, "f32", ldx=321)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("m,n,k", [(1, 50000, 200), (9, 50000, 193), (20, 90000, 200),       # two warps (20 rows: eight)
                                   (1, 8000, 1100), (16, 8000, 1100), (32, 16000, 1100),     # eight
                                   (1, 5000, 2100), (7, 5000, 2048)])                        # sixteen
def test_planes_by_other_numbers_of_warps(ebs, group, m, n, k):
    assert planes(ebs, m, n, k, group) and planes(ebs, m, n, k, group, ldx=k + 3)
    run(ebs, 24, m, n, k, group, "f32", residual=True, ldx=k + 3, ldy=n + 1, in_place=True)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("counts,spare", [([0, 3, 0, 0, 9, 1, 0, 8], 3), ([1] * 8, 0), ([70, 0, 1, 0, 17, 0, 0, 40], 5), ([0] * 8, 4)], ids=str)
def test_experts(ebs, dtype, group, counts, spare):
    """Eight experts of 650 tiles, some without rows, one with more than a piece, rows of nobody."""
    m = sum(counts) + spare
    assert dtype != "f32" or planes(ebs, m, 10399, 519, group, 8, ldx=521)
    run(ebs, 25, m, 10399, 519, group, dtype, act=2, bias=True, residual=True, ldx=521, counts=counts)


def test_planes_of_activations_not_finite(ebs):
    """As without planes: an infinity or a NaN reaches its own row."""
    n, k = 24003, 1027
    w = weights(26, 1, n, k)
    q, packed = make(ebs, w, 64, "f32", "f32")
    real = values(w, 64, "f32")[0]
    x = weights(27, 6, k)
    x[1, 5], x[3, 1026] = float("inf"), float("nan")
    x[4, 7] = torch.tensor([0x7f800001], dtype=torch.int32).view(torch.float32)[0].cuda()           # a NaN of low bits alone
    assert planes(ebs, 6, n, k, 64)
    d = ebs.linear_desc(6, n, k, ebs.EBS_F32)
    y, ws = torch.zeros(6, n, device="cuda"), torch.full((ebs.ebs_linear_q4_workspace_bytes(d, q),), 255, dtype=torch.uint8, device="cuda")
    ebs.ebs_linear_q4_forward(x, packed, None, None, None, d, q, y, ws)
    check(y[[0, 2, 5]], x[[0, 2, 5]], real, None, None, 0)
    assert y[3].isnan().all() and y[4].isnan().all()
    zero = real[:, 5] == 0
    assert y[1][zero].isnan().all() and torch.equal(y[1][~zero], torch.copysign(torch.full_like(y[1], float("inf")), real[:, 5].float())[~zero])


def test_small_activations_keep_their_bits(ebs):
    """fp32 activations down to 2^-110 are held in full by three 16-bit planes; below, to 2^-133."""
    n, k = 64, 64
    w = torch.full((1, n, k), 7.0 * 2.0 ** 60, device="cuda")
    q, packed = make(ebs, w, 64, "f32", "f32")
    real = values(w, 64, "f32")[0]
    d = ebs.linear_desc(1, n, k, ebs.EBS_F32)
    for e in (-100, -109, -120, -126, -130):
        x = torch.zeros(1, k, device="cuda")
        x[0, 3] = (1.0 + 2.0 ** -7 + 2.0 ** -15 + 2.0 ** -23) * 2.0 ** e
        y = torch.empty(1, n, device="cuda")
        ebs.ebs_linear_q4_forward(x, packed, None, None, None, d, q, y)
        ref = x.double() @ real.t()
        assert ((y.double() - ref).abs() <= 2.0 ** -24 * ref + (2.0 ** -133 * real.abs().amax() if e < -110 else 0.0)).all(), e
