"""What the Python layer over the operators refuses or takes before any GPU work."""
import pytest
import torch

from paper_2607_23115_gb300 import experts, fp8


def _weight(count, n, k, grad=True):
    a, b = fp8.tiles(n), fp8.tiles(k)
    q, s = torch.zeros(count, a, b, 128, 128, dtype=torch.uint8), torch.zeros(count, a, b)
    qt, st = torch.zeros(count, b, a, 128, 128, dtype=torch.uint8), torch.zeros(count, b, a)
    return fp8.Weight(n, k, q, s, qt if grad else None, st if grad else None)


def _plan(n, tokens, per, rows):
    z = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    return experts.Plan(n, 128, z(n + 1), z(n), z(tokens, per), z(rows))


@pytest.mark.parametrize("dw_dtype", [torch.float64, torch.int32, torch.float8_e4m3fn])
def test_gradients_of_other_types_are_refused(dw_dtype):
    with pytest.raises(ValueError, match="dw_dtype"):
        fp8.linear_grad(torch.zeros(5, 4), torch.zeros(5, 6), _weight(1, 4, 6), dw_dtype=dw_dtype)
    with pytest.raises(ValueError, match="dw_dtype"):
        experts.linear_grad(torch.zeros(256, 4), torch.zeros(5, 6), _plan(2, 5, 2, 256), _weight(2, 4, 6),
                            dw_dtype=dw_dtype)


@pytest.mark.parametrize("dy,x", [(torch.float64, torch.float32), (torch.float32, torch.float64),
                                  (torch.int64, torch.float32)])
def test_inputs_of_other_types_are_refused(dy, x):
    with pytest.raises(ValueError, match="expected bfloat16"):
        fp8.linear_grad(torch.zeros(5, 4, dtype=dy), torch.zeros(5, 6, dtype=x), _weight(1, 4, 6))
    with pytest.raises(ValueError, match="expected bfloat16"):
        experts.linear_grad(torch.zeros(256, 4, dtype=dy), torch.zeros(5, 6, dtype=x), _plan(2, 5, 2, 256),
                            _weight(2, 4, 6))


@pytest.mark.parametrize("shape,rows", [((2, 3, 0), 6), ((0, 4, 0), 0), ((0,), 1), ((5, 0), 5), ((2, 0, 7), 0), ((7,), 1)])
def test_rows_of_any_shape(shape, rows):
    """Inputs of no columns too, whose number of rows their size does not tell."""
    assert fp8._rows_of(torch.zeros(shape)).shape == (rows, shape[-1])
