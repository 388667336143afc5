"""Bounded waits of the experts' products: nothing is issued to the tensor core, every wait runs out, the calls return, the status says so once, and the
next calls are right.  (Behind the tests that expect no wait to have run out.)"""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ebs():
    from paper_2003_07577_b200 import binding
    return binding


# tiles of 64, 128 and 256 columns, sums in chunks
@pytest.mark.parametrize("counts,n,k", [([40, 3], 64, 128), ([3000, 1000], 1000, 264), ([3001, 1000], 2500, 2100), ([4000, 4000], 1500, 128), ([6000, 7], 72, 4200), ([6000, 2001], 2500, 4200)])
def test_waits_that_give_up(ebs, counts, n, k):
    """Nothing is issued to the tensor core: every wait runs out, the calls return, the status says so once, and the next calls are right."""
    m, experts, t = sum(counts), len(counts), torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(6)
    x, w, dy = (torch.randn(s, generator=g, device="cuda").to(t) for s in ((m, k), (experts, n, k), (m, n)))
    offsets = torch.tensor([0] + counts).cumsum(0).to(torch.int32).cuda()
    d = ebs.linear_desc(m, n, k, ebs.EBS_BF16)
    y, dx, dw = torch.zeros(m, n, dtype=t, device="cuda"), torch.zeros(m, k, dtype=t, device="cuda"), torch.zeros(experts, n, k, dtype=t, device="cuda")
    ws = torch.empty(max(16, ebs.ebs_grouped_workspace_bytes(d, experts, True)), dtype=torch.uint8, device="cuda")

    def calls():
        ebs.ebs_grouped_forward(x, w, None, None, offsets, experts, d, y, None, ws)
        ebs.ebs_grouped_backward(dy, x, w, None, offsets, experts, d, dx, dw, None, ws)
    calls()
    want = [v.clone() for v in (y, dx, dw)]
    assert ebs.ebs_check_device_status() == ebs.EBS_OK
    before = ebs.ebs_device_wait_timeouts()
    ebs.ebs_test_set_device_wait(64, 1)
    try:
        calls()
        torch.cuda.synchronize()
    finally:
        ebs.ebs_test_set_device_wait(0, 0)
    assert ebs.ebs_device_wait_timeouts() > before
    assert ebs.ebs_check_device_status() == ebs.EBS_ERR_TIMEOUT
    assert ebs.ebs_check_device_status() == ebs.EBS_OK
    calls()
    for a, b in zip(want, (y, dx, dw)):
        assert torch.equal(a, b)
