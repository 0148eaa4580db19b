"""What the device finds wrong reaches the Python layer's user."""
import pytest
import torch

from paper_2607_23115_gb300 import binding as B
from paper_2607_23115_gb300 import experts, fp8

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def _raises(status, **kw):
    with pytest.raises(B.GleamError) as e:
        fp8.check(**kw)
    assert e.value.rc == status
    fp8.check(**kw)  # told once


def _plan(counts, rows, tokens):
    t = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    return experts.Plan(2, 128, t([0, 128, 256]), t(counts), t([[0]] * tokens), t([0] * rows))


# a matrix of 256 rows (one kernel) and of 5,120
@pytest.mark.parametrize("rows", [256, 5120])
def test_a_plan_that_does_not_fit(rows):
    w = fp8.quantize_weight(torch.randn(2, 64, 128, device=DEV), grad=True)
    x = torch.randn(4, 128, device=DEV)
    fp8.check()
    bad, good = _plan([3, rows], rows, 4), _plan([3, 5], rows, 4)
    experts.linear(x, bad, w)
    _raises(B.GLEAM_ERR_INVALID_ARG)
    h = experts.linear(x, good, w)
    fp8.check()
    experts.linear_grad(h, x, bad, w)
    _raises(B.GLEAM_ERR_INVALID_ARG)
    experts.linear_grad(h, x, good, w)
    fp8.check()


@pytest.mark.parametrize("m", [3, 40, 300])
def test_a_wait_that_runs_out(m):
    w = fp8.quantize_weight(torch.randn(2000, 14336, device=DEV))
    x = torch.randn(m, 14336, device=DEV)
    want = fp8.linear(x, w)
    fp8.check()
    B.gleam_operators_debug_set(B.GLEAM_DEBUG_WAIT_LIMIT_NS, 2_000_000)
    try:
        B.gleam_operators_debug_set(B.GLEAM_DEBUG_SKIP_ARRIVE, 10 if m == 40 else 1)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        fp8.linear(x, w, stream=side)
        _raises(B.GLEAM_ERR_TIMEOUT, stream=side)
    finally:
        B.gleam_operators_debug_set(B.GLEAM_DEBUG_WAIT_LIMIT_NS, 4_000_000_000)
    assert torch.equal(fp8.linear(x, w), want)
    fp8.check()


def test_a_word_of_the_callers_own_is_the_only_one_written():
    w = fp8.quantize_weight(torch.randn(2, 64, 128, device=DEV))
    x = torch.randn(256, 128, device=DEV)
    plan = _plan([3, 999], 256, 256)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    y = torch.empty(256, 64, device=DEV)
    fp8.check()
    assert B.gleam_fp8_linear(B.gleam_fp8_linear_t(
        x.data_ptr(), B.GLEAM_FP32, 1, 256, 128, 128, 0, 64, w.q.data_ptr(), w.s.data_ptr(), y.data_ptr(), 64, 256,
        plan.at_src_of, 1, 0, 2, 0, plan.at_offsets, plan.at_counts, None, 0, status.data_ptr())) == 0
    assert status.item() == B.GLEAM_ERR_INVALID_ARG
    fp8.check()
