"""Rows that sorted slots may take, at and past the sizes that a sort takes."""
import pytest

from paper_2607_23115_gb300 import binding as B
from paper_2607_23115_gb300 import build


# more than gleam_expert_sort takes: the count must not wrap 64 bits
@pytest.mark.parametrize("tokens,per,experts,align", [
    (1 << 40, 2, 8, 128), (4, (1 << 20) + 1, 8, 128), (4, 2, 1025, 128), (4, 2, 8, (1 << 20) + 1),
    (0x7fffff00, 0xffffffff, 0xffffffff, 0xffffffff)])
def test_rows_of_sizes_that_are_refused(tokens, per, experts, align):
    build.build()
    assert B.gleam_expert_rows(tokens, per, experts, align) == 0


def test_rows_of_the_largest_sizes():
    build.build()
    slots, fill = 0x7fffff00 * (1 << 20), 1024 * ((1 << 20) - 1)
    assert B.gleam_expert_rows(0x7fffff00, 1 << 20, 1024, 1 << 20) == (slots + fill + (1 << 20) - 1) >> 20 << 20
