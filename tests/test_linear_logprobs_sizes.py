"""Sizes of the head product next to 2^31, whose tiles the kernels count in 32 bits: refused on the host, before any launch.  The addresses are never touched."""
import pytest

from paper_2503_23367_b200 import binding as fv
from paper_2503_23367_b200 import build as fv_build
from test_logits_refusals import LINEAR, UNSUPPORTED, call

MOST = 2 ** 31 - 1


@pytest.fixture(scope="module")
def lib():
    fv_build.build()
    return fv.lib()


@pytest.mark.parametrize("big", [dict(rows=MOST), dict(rows=MOST - 254), dict(V=MOST - 7), dict(V=MOST - 247), dict(C=MOST - 7), dict(C=MOST - 247), dict(rows=MOST, V=MOST - 7), dict(rows=2 ** 30, V=2 ** 30)])
def test_sizes_beyond_32_bits_of_tiles(lib, big):
    assert call(lib.fv_linear_logprobs, LINEAR, **{"bytes": 2 ** 62, **big}) == UNSUPPORTED


@pytest.mark.parametrize("rows,V", [(MOST, 8), (8, MOST - 7), (MOST, MOST - 7)])
def test_no_workspace_for_refused_sizes(lib, rows, V):
    assert lib.fv_linear_logprobs_workspace_bytes(rows, V) == 0


def test_workspace_of_the_largest_sizes(lib):
    """Two parts of 16 bytes per row and column tile, 4 bytes per row."""
    rows = MOST - 255
    assert lib.fv_linear_logprobs_workspace_bytes(rows, 8) == -(-rows * 32 // 256) * 256 + -(-rows * 4 // 256) * 256
    parts = lib.fv_linear_logprobs_workspace_bytes(1, MOST - 255)
    assert parts in [-(-(2 * -(-(MOST - 255) // bn)) * 16 // 256) * 256 + 256 for bn in (128, 256)]
