"""A stream that is given: what goes in may be freed by its owner right after the call, and what comes
out by the caller, while the stream has still to get to the work."""
import pytest
import torch

from paper_2607_23115_gb300 import experts, fp8

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
LONG = 200_000_000  # cycles: about 0.1 s


@pytest.fixture
def side():
    # loading a kernel's code waits for the GPU: those of the tests run once before
    for dtype in (torch.float32, torch.uint8):
        torch.full((4,), 7, dtype=dtype, device=DEV) + 0
    torch.cuda._sleep(1)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    yield s
    torch.cuda.synchronize()


def _reused(size, dtype, at):
    """Whether new memory of the size is the one that was at `at`; it is overwritten if so."""
    new = [torch.full((size,), 7, dtype=dtype, device=DEV) for _ in range(4)]
    return any(t.data_ptr() == at for t in new)


@pytest.mark.parametrize("raw", [False, True])
@pytest.mark.parametrize("what", ["x", "weight"])
def test_inputs_freed_after_the_call(what, raw, side):
    torch.manual_seed(0)
    x = torch.randn(300, 2048, device=DEV)
    w = fp8.quantize_weight(0.02 * torch.randn(1024, 2048, device=DEV))
    want = fp8.linear(x, w)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(LONG)
    y = fp8.linear(x, w, stream=side.cuda_stream if raw else side)
    if what == "x":
        at, size, dtype = x.data_ptr(), x.numel(), x.dtype
        del x
    else:
        at, size, dtype = w.q.data_ptr(), w.q.numel(), w.q.dtype
        del w
    assert not _reused(size, dtype, at)
    side.synchronize()
    assert torch.equal(y, want)


def test_results_freed_while_the_caller_reads_them(side):
    x = torch.randn(300, 2048, device=DEV)
    w = fp8.quantize_weight(0.02 * torch.randn(1024, 2048, device=DEV))
    y = fp8.linear(x, w, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    want = y.clone()
    torch.cuda.synchronize()
    torch.cuda._sleep(LONG)
    got, at = y + 0, y.data_ptr()  # the caller's stream has this still to do
    del y
    with torch.cuda.stream(side):
        assert not _reused(300 * 1024, torch.float32, at)
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_experts_on_a_given_stream(side):
    torch.manual_seed(1)
    x, dy = torch.randn(500, 512, device=DEV), torch.randn(500, 256, device=DEV)
    w = fp8.quantize_weight(0.02 * torch.randn(8, 256, 512, device=DEV), grad=True)
    ids, g = torch.randint(0, 8, (500, 2), device=DEV), torch.rand(500, 2, device=DEV)

    def step(stream):
        plan = experts.sort(ids, 8, stream=stream)
        h = experts.linear(x, plan, w, stream=stream)
        xs = experts.gather(x, plan, stream=stream)
        y = experts.combine(h, plan, g, stream=stream)
        dh, dg = experts.combine_grad(dy, h, plan, g, stream=stream)
        drows, dw = experts.linear_grad(dh, x, plan, w, stream=stream)
        return y, dg, dw, xs, experts.combine(drows, plan, stream=stream)

    want = step(None)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(LONG)
    got = step(side)
    # the plan, the rows and their gradients are gone; memory of their sizes is written over
    junk = [torch.full((n,), 9, dtype=torch.uint8, device=DEV) for n in (1 << 12, 1 << 16, 1 << 20, 1 << 21, 1 << 22)]
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want)), len(junk)
