"""Every build of tree_attn's kernels against the answer in 64 bits."""
import numpy as np
import pytest

from tests.test_gpu_tree_attn import _run
from tests.tree_builds import CALLS, FORMATS

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("c", CALLS, ids=str)
def test_build(c, fmt):
    got = _run(fmt, c.B, c.w, c.Hq, c.Hkv, c.d, c.page, c.n, kind="random" if c.B < 100 else "fewer", ragged=c.ragged, seed=60 + c.w, max_len=c.n)
    assert got["out"].shape == (c.B, c.w, c.Hq, c.d) and np.isfinite(got["out"].float().cpu().numpy()).all()
