"""A layer of experts over several steps whose batches have fewer and fewer rows that are an expert's: what it returns for the others."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mods():
    from paper_2003_07577_b200 import binding, experts
    return binding, experts


def make(mods, dtype, act):
    ebs, ex = mods
    g = torch.Generator(device="cuda").manual_seed(3)
    layer = ex.ExpertLinear(torch.randn(3, 24, 40, generator=g, device="cuda"), 50, dtype, None, act)
    return layer, *(torch.randn(50, c, generator=g, device="cuda").to(dtype) for c in (40, 24))


def starts(first, counts):
    return (torch.tensor([0] + counts).cumsum(0) + first).to(torch.int32).cuda()


STEPS = [(0, [20, 10, 20]), (0, [10, 0, 12]), (7, [1, 4, 0]), (50, [0, 0, 0]), (0, [0, 0, 50])]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("act", [0, 4])
@pytest.mark.parametrize("captured", [False, True])
def test_gradient_of_rows_that_are_no_experts_is_zero(mods, dtype, act, captured):
    """Also of those that were an expert's in the step before."""
    layer, x, dy = make(mods, dtype, act)
    offsets = starts(*STEPS[0])
    run = lambda: (layer.forward(x, offsets), layer.backward(dy))  # noqa: E731
    run()
    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            run()
        run = graph.replay
    for first, counts in STEPS:
        offsets.copy_(starts(first, counts))
        run()
        torch.cuda.synchronize()
        theirs = torch.zeros(50, dtype=torch.bool, device="cuda")
        theirs[first:first + sum(counts)] = True
        assert not layer.dx[~theirs].any(), (first, counts)
        assert (layer.dx[theirs] != 0).any(dim=1).all()


def test_answers_refuse_what_has_no_rows(mods):
    _, ex = mods
    served = ex.QuantizedExperts(torch.zeros(2, 8, 32, device="cuda"), 4, torch.float16, group=32)
    o = torch.zeros(3, dtype=torch.int32, device="cuda")
    for shape in ((), (32,), (1, 2, 32), (5, 32), (4, 31)):
        with pytest.raises(ValueError):
            served.answer(torch.zeros(shape, dtype=torch.float16, device="cuda"), o)
