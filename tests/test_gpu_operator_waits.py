"""Waits of the products that run out: one of a block's copying threads stops in the middle, so that
what it would have brought never comes.  The call reports it and ends soon, and the next is right."""
import time

import pytest
import torch

from paper_2607_23115_gb300 import binding as B
from paper_2607_23115_gb300 import fp8

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
LIMIT_NS = 2_000_000


@pytest.fixture
def short_waits():
    assert B.gleam_operators_debug_set(B.GLEAM_DEBUG_WAIT_LIMIT_NS, LIMIT_NS) == 0
    yield
    B.gleam_operators_debug_set(B.GLEAM_DEBUG_WAIT_LIMIT_NS, 4_000_000_000)


def _linear(x, w, y, status):
    m, k = x.shape
    size = B.gleam_fp8_linear_work(m, k)
    work = torch.empty(size + 16, dtype=torch.uint8, device=DEV)
    assert B.gleam_fp8_linear(B.gleam_fp8_linear_t(
        x.data_ptr(), B.GLEAM_BF16, 1, m, k, k, 0, w.n, w.q.data_ptr(), w.s.data_ptr(), y.data_ptr(), w.n, m, None, 0,
        0, 0, 0, None, None, work.data_ptr(), size, status.data_ptr())) == 0


def _run_out(m, n, k, skips):
    torch.manual_seed(m)
    x = torch.randn(m, k, device=DEV).to(torch.bfloat16)
    w = fp8.quantize_weight(0.02 * torch.randn(n, k, device=DEV))
    want = fp8.linear(x, w)
    y = torch.zeros_like(want)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    for skip in skips:
        torch.cuda.synchronize()
        assert B.gleam_operators_debug_set(B.GLEAM_DEBUG_SKIP_ARRIVE, skip) == 0
        t0 = time.monotonic()
        _linear(x, w, y, status)
        torch.cuda.synchronize()
        # a few limits one after another, not the 4 s of a wait for what never comes
        assert time.monotonic() - t0 < 2.0, skip
        assert status.item() == B.GLEAM_ERR_TIMEOUT, skip
        assert not torch.equal(y, want)
        status.zero_()
        _linear(x, w, y, status)
        assert status.item() == 0 and torch.equal(y, want), skip


@pytest.mark.parametrize("m", [1, 12])
def test_few_rows(m, short_waits):
    _run_out(m, 4096, 7168, [1, 2, 3])
