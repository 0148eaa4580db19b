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


def _run_out(call, y, skips):
    """call(y, status), with a copying thread that stops after each of `skips` copies."""
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    call(y, status)
    want = y.clone()
    assert status.item() == 0
    for skip in skips:
        y.zero_()
        torch.cuda.synchronize()
        assert B.gleam_operators_debug_set(B.GLEAM_DEBUG_SKIP_ARRIVE, skip) == 0
        t0 = time.monotonic()
        call(y, status)
        torch.cuda.synchronize()
        # a few limits one after another, not the 4 s of a wait for what never comes
        assert time.monotonic() - t0 < 2.0, skip
        assert status.item() == B.GLEAM_ERR_TIMEOUT, skip
        assert not torch.equal(y, want)
        status.zero_()
        call(y, status)
        assert status.item() == 0 and torch.equal(y, want), skip


def _run_out_linear(m, n, k, skips):
    torch.manual_seed(m)
    x = torch.randn(m, k, device=DEV).to(torch.bfloat16)
    w = fp8.quantize_weight(0.02 * torch.randn(n, k, device=DEV))
    _run_out(lambda y, status: _linear(x, w, y, status), torch.empty(m, n, dtype=torch.bfloat16, device=DEV), skips)


@pytest.mark.parametrize("m", [1, 12])
def test_few_rows(m, short_waits):
    _run_out_linear(m, 4096, 7168, [1, 2, 3])


# w's rows as the lanes, the contraction shared out and not; x's: tiles of 128, of 256, of two blocks
@pytest.mark.parametrize("m,n,k,skips", [
    (40, 4096, 7168, [7, 8, 13]), (20, 2048, 14000, [10, 11]), (40, 20000, 4000, [7, 9, 31]),
    (300, 2000, 1152, [1, 2, 3, 4, 5, 8]), (380, 10000, 1152, [1, 2, 3, 4, 5, 8]),
    (2560, 2304, 1152, [1, 2, 3, 4, 5, 6, 8])])
def test_products(m, n, k, skips, short_waits):
    _run_out_linear(m, n, k, skips)


# a scale for each row of both: tiles of 128, of 256, of two blocks
@pytest.mark.parametrize("m,n", [(300, 500), (380, 10000), (2560, 2304)])
def test_products_of_groups(m, n, short_waits):
    torch.manual_seed(n)
    k = 1100
    a, b = torch.randn(m, k, device=DEV), torch.randn(n, k, device=DEV)
    with fp8._On(a, None) as raw:
        q, s, _, _ = fp8._quantize(raw, a, m, k, True, False)
        r, t, _, _ = fp8._quantize(raw, b, n, k, True, False)

    def call(y, status):
        p = B.gleam_fp8_product_t(m, n, k, q.data_ptr(), s.data_ptr(), r.data_ptr(), t.data_ptr(),
                                  B.GLEAM_FP8_GROUPS, B.GLEAM_FP32, y.data_ptr(), n)
        p.d_status = status.data_ptr()
        assert B.gleam_fp8_product(p) == 0

    _run_out(call, torch.empty(m, n, device=DEV), [1, 2, 3, 4, 5, 6, 8])
