"""Gradients are calls of their own: a backward pass that would lose them says so, and calls on
tensors that require one answer as before."""
import pytest
import torch

from paper_2607_23115_gb300 import experts, fp8

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def _calls():
    torch.manual_seed(0)
    w = fp8.quantize_weight(torch.randn(130, 200, device=DEV))
    e = fp8.quantize_weight(torch.randn(4, 130, 200, device=DEV))
    plan = experts.sort(torch.randint(0, 4, (20, 2), device=DEV), 4)
    x, rows, g = torch.randn(20, 200, device=DEV), torch.randn(plan.rows, 200, device=DEV), torch.rand(20, 2, device=DEV)
    return [
        ("fp8.linear_grad", lambda x: fp8.linear(x, w), x),
        ("fp8.linear_grad", lambda x: fp8.linear(x, w), x.view(4, 5, 200)),
        ("fp8.linear_grad", lambda x: fp8.linear(x, w, stream=torch.cuda.current_stream()), x),
        ("fp8.linear_grad", lambda x: fp8.linear(x, w), x.t().contiguous().t()),
        ("experts.linear_grad", lambda x: experts.linear(x, plan, e), x),
        ("experts.combine", lambda x: experts.gather(x, plan), x),
        ("experts.combine_grad", lambda r: experts.combine(r, plan, g), rows),
        ("experts.combine_grad", lambda r: experts.combine(r, plan), rows),
        ("experts.combine_grad", lambda g: experts.combine(rows, plan, g), g),
    ]


@pytest.mark.parametrize("i", range(9))
def test_backward_says_what_gives_the_gradient(i):
    grad, call, x = _calls()[i]
    want = call(x)
    assert not want.requires_grad
    leaf = x.clone().requires_grad_()
    y = call(leaf)
    if grad != "experts.linear_grad":  # whose rows of no slot hold anything
        assert torch.equal(y.detach(), want)
    with pytest.raises(RuntimeError, match=grad):
        y.sum().backward()
    assert leaf.grad is None
    with torch.no_grad():
        assert not call(leaf).requires_grad
    with torch.inference_mode():
        call(leaf)
    assert not call(leaf.detach()).requires_grad


def test_gradient_calls_take_such_tensors():
    torch.manual_seed(1)
    w = fp8.quantize_weight(torch.randn(130, 200, device=DEV), grad=True)
    x, dy = torch.randn(20, 200, device=DEV), torch.randn(20, 130, device=DEV)
    dx, dw = fp8.linear_grad(dy, x, w)
    a, b = fp8.linear_grad(dy, x.clone().requires_grad_(), w)
    assert torch.equal(a, dx) and torch.equal(b, dw) and not a.requires_grad
