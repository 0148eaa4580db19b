"""Every kind of tile of the products, against sums in 64 bits: which sizes take which is worked out
here by the rule that the library has, so that a changed rule cannot leave one untested."""
import numpy as np
import pytest
import torch

from paper_2607_23115_gb300 import binding as B
from paper_2607_23115_gb300 import experts, fp8
from tests import _operators as R

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def _np(t):
    return t.float().cpu().numpy()


def _up(a, b):
    return -(-a // b)


def _wide(m, n, n_experts=0, sums=False):
    """The tile of more than 128 rows: "pair" (256 x 256 by two blocks), "one" (128 x 256), "half"."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count

    def tiles(kx, kw):
        x = _up(m, kx) + (n_experts if n_experts and not sums else 0)
        return x * _up(n, kw) * (n_experts if sums else 1)

    pair, one, half = 20 * _up(tiles(256, 256), sms // 2), 22 * _up(tiles(128, 256), sms), 17 * _up(tiles(128, 128), sms)
    return "pair" if pair <= one and pair <= half else "one" if one <= half else "half"


# m, n and the tile they take
LINEAR = [(300, 2000, "half"), (380, 10000, "one"), (333, 9985, "one"), (2560, 2304, "pair"), (2700, 2177, "pair")]


@pytest.mark.parametrize("dtype", R.DTYPES)
@pytest.mark.parametrize("m,n,tile", LINEAR)
def test_a_scale_for_each_block(m, n, tile, dtype):
    assert _wide(m, n) == tile
    rng = np.random.default_rng(m)
    x = R.activations(rng, m, 300, dtype)
    w = torch.from_numpy(0.02 * rng.standard_normal((n, 300))).to(R.DTYPES[dtype])
    y = fp8.linear(x.to(DEV), fp8.quantize_weight(w.to(DEV)))
    R.close(y, *R.product(R.rows_v(_np(x)), R.blocks_v(_np(w)[None])[0]))


@pytest.mark.parametrize("dtype", R.DTYPES)
@pytest.mark.parametrize("n,k,tile", LINEAR)
def test_a_scale_for_each_row(n, k, tile, dtype):
    """The gradient of a weight [n, k]."""
    assert _wide(n, k) == tile
    rng = np.random.default_rng(n)
    m = 300
    x, dy = R.activations(rng, m, k, dtype), R.activations(rng, m, n, dtype)
    w = fp8.quantize_weight(torch.zeros(n, k, device=DEV), grad=True)
    _, dw = fp8.linear_grad(dy.to(DEV), x.to(DEV), w)
    R.close(dw, *R.product(R.columns_v(_np(dy)).T, R.columns_v(_np(x)).T))


def _routed(rng, tokens, per, n):
    ids = rng.integers(0, n, (tokens, per))
    ids[rng.random((tokens, per)) < 0.05] = -1
    return ids, [np.nonzero(ids.reshape(-1) == e)[0] for e in range(n)]


@pytest.mark.parametrize("tokens,n_experts,n,tile", [
    (900, 3, 500, "half"), (3000, 4, 2304, "one"), (3000, 4, 1024, "pair"), (2900, 4, 1000, "pair")])
def test_rows_by_expert(tokens, n_experts, n, tile):
    rng = np.random.default_rng(tokens + n)
    ids, slots = _routed(rng, tokens, 1, n_experts)
    plan = experts.sort(torch.from_numpy(ids).to(DEV), n_experts)
    assert _wide(plan.rows, n, n_experts) == tile
    x = R.activations(rng, tokens, 200, "bf16")
    w = torch.from_numpy(0.05 * rng.standard_normal((n_experts, n, 200))).to(torch.bfloat16)
    h = experts.linear(x.to(DEV), plan, fp8.quantize_weight(w.to(DEV)))
    wv, off = R.blocks_v(_np(w)), plan.offsets.cpu().numpy()
    for e, s in enumerate(slots):
        R.close(h[off[e]:off[e] + len(s)], *R.product(R.rows_v(_np(x)[s]), wv[e]))


@pytest.mark.parametrize("n_experts,n,k,tile", [
    (3, 300, 500, "half"), (2, 380, 5000, "one"), (2, 1024, 2304, "pair"), (2, 1000, 2200, "pair")])
def test_sums_by_expert(n_experts, n, k, tile):
    assert _wide(n, k, n_experts, sums=True) == tile
    rng = np.random.default_rng(n + k)
    tokens, per = 400, 1
    ids, slots = _routed(rng, tokens, per, n_experts)
    ids[ids == 1] = -1  # an expert without rows
    slots[1] = slots[1][:0]
    plan = experts.sort(torch.from_numpy(ids).to(DEV), n_experts)
    x = R.activations(rng, tokens, k, "bf16")
    w = fp8.quantize_weight(torch.zeros(n_experts, n, k, device=DEV), grad=True)
    dh = R.activations(rng, plan.rows, n, "bf16")
    _, dw = experts.linear_grad(dh.to(DEV), x.to(DEV), plan, w)
    off = plan.offsets.cpu().numpy()
    for e, s in enumerate(slots):
        if len(s) == 0:
            assert not dw[e].any()
        else:
            R.close(dw[e], *R.product(R.columns_v(_np(dh)[off[e]:off[e] + len(s)]).T, R.columns_v(_np(x)[s]).T))


# one kernel; w's rows as the lanes, 16 to 64 of x; x's rows, each tile
@pytest.mark.parametrize("m,n,k", [(12, 500, 700), (20, 500, 700), (40, 2000, 1400), (120, 300, 500)] +
                         [(m, n, 300) for m, n, _ in LINEAR])
def test_special_values_stay_where_they_are(m, n, k):
    torch.manual_seed(m + n)
    x = torch.randn(m, k, device=DEV).to(torch.bfloat16)
    w = (0.02 * torch.randn(n, k, device=DEV)).to(torch.bfloat16)
    good = fp8.linear(x, fp8.quantize_weight(w))
    bad = x.clone()
    rows = torch.zeros(m, dtype=torch.bool, device=DEV)
    for i, v in ((2, float("nan")), (m // 2, float("inf")), (m - 1, float("-inf"))):
        bad[i, (7 * i) % k] = v
        rows[i] = True
    y = fp8.linear(bad, fp8.quantize_weight(w))
    assert y[rows].isnan().all() and torch.equal(y[~rows], good[~rows])
    # in a weight, of a block's rows
    for v in (float("nan"), float("inf")):
        bad = w.clone()
        i = n - 1
        bad[i, k - 1] = v
        rows = torch.arange(n, device=DEV) // 128 == i // 128
        y = fp8.linear(x, fp8.quantize_weight(bad))
        assert y[:, rows].isnan().all() and torch.equal(y[:, ~rows], good[:, ~rows])


@pytest.mark.parametrize("n,k,tile", LINEAR)
def test_special_values_in_a_weights_gradient(n, k, tile):
    torch.manual_seed(n)
    x, dy = torch.randn(260, k, device=DEV), torch.randn(260, n, device=DEV)
    w = fp8.quantize_weight(torch.zeros(n, k, device=DEV), grad=True)
    _, good = fp8.linear_grad(dy, x, w)
    dy[3, 5], dy[200, n - 1], x[259, 17] = float("nan"), float("inf"), float("-inf")
    _, dw = fp8.linear_grad(dy, x, w)
    hit = torch.zeros(n, k, dtype=torch.bool, device=DEV)
    hit[5], hit[n - 1], hit[:, 17] = True, True, True
    assert dw[hit].isnan().all() and torch.equal(dw[~hit], good[~hit])


# x and its scales just fill what one kernel has for them, and do not
@pytest.mark.parametrize("m,k,one", [(1, 14848, True), (1, 14849, False), (8, 14800, True), (8, 14900, False),
                                     (9, 7424, True), (16, 7424, True), (16, 7425, False), (9, 7500, False)])
def test_the_longest_contractions_of_one_kernel(m, k, one):
    assert (B.gleam_fp8_linear_work(m, k) == 0) == one
    rng = np.random.default_rng(k)
    x = R.activations(rng, m, k, "bf16")
    w = torch.from_numpy(0.02 * rng.standard_normal((300, k))).to(torch.bfloat16)
    y = fp8.linear(x.to(DEV), fp8.quantize_weight(w.to(DEV)))
    R.close(y, *R.product(R.rows_v(_np(x)), R.blocks_v(_np(w)[None])[0]))


@pytest.mark.parametrize("tokens,n_experts", [(7, 64), (40, 8), (1500, 4)])
def test_a_layer_of_experts_repeats_bit_for_bit(tokens, n_experts):
    torch.manual_seed(tokens)
    w = fp8.quantize_weight(0.05 * torch.randn(n_experts, 384, 512, device=DEV), grad=True)
    x = torch.randn(tokens, 512, device=DEV).to(torch.bfloat16)
    dy = torch.randn(tokens, 384, device=DEV).to(torch.bfloat16)
    ids, g = torch.randint(-1, n_experts, (tokens, 4), device=DEV), torch.rand(tokens, 4, device=DEV)

    def step():
        plan = experts.sort(ids, n_experts)
        h = experts.linear(x, plan, w)
        dh, dg = experts.combine_grad(dy, h, plan, g)
        drows, dw = experts.linear_grad(dh, x, plan, w)
        return experts.combine(h, plan, g), dg, dw, experts.combine(drows, plan)

    want = step()
    for _ in range(20):
        assert all(torch.equal(a, b) for a, b in zip(step(), want))
