"""Bounded waits of the real-valued kernels: nothing is issued to the tensor core (or one part of a split tile sends no sums), every wait runs out,
the call returns, the status says so once, and the next launch is right."""
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

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


def give_up_and_recover(ebs, call, out, skip):
    call()
    want = out.clone()
    assert ebs.ebs_check_device_status() == ebs.EBS_OK
    before = ebs.ebs_device_wait_timeouts()
    ebs.ebs_test_set_device_wait(64, skip)
    try:
        call()
        torch.cuda.synchronize()
    finally:
        ebs.ebs_test_set_device_wait(0, 0)
    assert ebs.ebs_device_wait_timeouts() > before
    assert ebs.ebs_check_device_status() == ebs.EBS_ERR_TIMEOUT
    assert ebs.ebs_check_device_status() == ebs.EBS_OK
    call()
    assert torch.equal(out, want)


# one tile a part, a cluster a tile, a pair of blocks, a reduction in parts
@pytest.mark.parametrize("m,n,k,skip", [(40, 200, 400, 1), (200, 300, 2000, 1), (200, 300, 2000, 2), (4096, 2048, 256, 1), (300, 264, 8200, 1)])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_linear(ebs, dtype, m, n, k, skip):
    t, code = {"f32": (torch.float32, ebs.EBS_F32), "f16": (torch.float16, ebs.EBS_F16), "bf16": (torch.bfloat16, ebs.EBS_BF16)}[dtype]
    g = torch.Generator(device="cuda")
    g.manual_seed(11)
    x, w = (torch.randn(s, generator=g, device="cuda").to(t) for s in ((m, k), (n, k)))
    w /= math.sqrt(k)
    y = torch.empty((m, n), dtype=t, device="cuda")
    d = ebs.linear_desc(m, n, k, code, ebs.EBS_ACT_NONE)
    ws = torch.empty(max(ebs.ebs_linear_workspace_bytes(d, False), 16), dtype=torch.uint8, device="cuda")
    give_up_and_recover(ebs, lambda: ebs.ebs_linear_forward(x, w, None, None, d, y, None, ws), y, skip)


# a block a matrix, clusters of four and eight (short side up to 64 and 128), tiles, symmetric products of both tile widths
@pytest.mark.parametrize("shape", [(60, 64, 576), (18, 64, 576), (3, 64, 576), (2, 16, 2000), (2, 128, 1152), (1, 300, 96), (1, 300, 500), (1, 1900, 1900), (1, 2100, 2100)])
def test_orthogonalize(ebs, shape):
    g = torch.Generator(device="cuda")
    g.manual_seed(7)
    x = torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)
    out = torch.empty_like(x)
    ws = torch.empty(ebs.ebs_orthogonalize_workspace_bytes(*shape, ebs.EBS_BF16, 5), dtype=torch.uint8, device="cuda")
    give_up_and_recover(ebs, lambda: ebs.ebs_orthogonalize(x, *shape, ebs.EBS_BF16, 5, COEFF, 1e-7, 1.0, out, ws), out, 1)


# 16-bit sums in chunks: tiles, a cluster's parts, pairs, parts through memory
@pytest.mark.parametrize("m,n,k", [(40, 20000, 4500), (40, 200, 40000), (4096, 2048, 4500), (300, 264, 200000)])
def test_long_sums(ebs, m, n, k):
    g = torch.Generator(device="cuda")
    g.manual_seed(13)
    x, w = (torch.randn(s, generator=g, device="cuda").bfloat16() for s in ((m, k), (n, k)))
    y = torch.empty((m, n), dtype=torch.bfloat16, device="cuda")
    d = ebs.linear_desc(m, n, k, ebs.EBS_BF16, ebs.EBS_ACT_NONE)
    ws = torch.empty(max(ebs.ebs_linear_workspace_bytes(d, False), 16), dtype=torch.uint8, device="cuda")
    give_up_and_recover(ebs, lambda: ebs.ebs_linear_forward(x, w, None, None, d, y, None, ws), y, 1)
