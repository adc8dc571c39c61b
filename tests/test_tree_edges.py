"""CPU-only: the kernels that the calls of tests/tree_edges.py reach."""
import pytest

from tests.test_tree_host import _short, launched, names              # noqa: F401
from tests.tree_builds import FORMATS, Call
from tests.tree_edges import SHAPES


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,w,Hq,most,kernel", SHAPES)
def test_the_kernel_that_a_shape_reaches(names, B, w, Hq, most, kernel, d, fmt):      # noqa: F811
    assert kernel in [_short(n) for n in launched(names, Call(B, w, Hq, 2, d, 16, most, False, None), fmt)]
