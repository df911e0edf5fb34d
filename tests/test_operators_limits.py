"""Sizes of adapters and vocabulary losses whose index arithmetic would pass 32 bits are refused on the host (no GPU)."""
import pytest

from test_operators_abi import _backward, _distill, _forward, _policy, p  # noqa: F401

MOST = (1 << 30) - 4096   # rows of a batch: the last block's first row is rowstart[0] + rows, both at most this


@pytest.mark.parametrize("rows", [MOST + 1, 1 << 30, (1 << 30) + (1 << 29), (1 << 31) - 1])
def test_rows_beyond_the_most_are_refused(p, rows):  # noqa: F811
    # arrays of so many rows would overlap at the addresses of these tests: the number is looked at before that
    assert _forward(p, rows=rows) == -8
    assert _backward(p, rows=rows) == -8
    assert _distill(p, rows=rows) == -8
    assert _policy(p, rows=rows) == -8


def test_as_many_rows_as_allowed_are_looked_at_further(p):  # noqa: F811
    for call in (_forward, _backward, _distill, _policy):
        assert call(p, rows=MOST) == -3   # the arrays overlap


@pytest.mark.parametrize("width", [(1 << 30) + 8, (1 << 31) - 8])
def test_widths_beyond_the_most_are_refused(p, width):  # noqa: F811
    for shape in ((width, 8, 1), (8, width, 1)):
        with pytest.raises(p.DbwError) as e:
            p.lowrank_layout([shape])
        assert e.value.code == -5
    assert _forward(p, desc=p.LowRank(width, 32, 8, 0, 512)) == -5
    lay = p.lowrank_layout([(1 << 30, 8, 64)])
    assert lay.d == 64 * (1 << 30) + 512
