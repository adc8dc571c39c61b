"""pc_cache_attn at the ends of its ranges: values of very different sizes beside one another."""
import numpy as np
import pytest
import torch

import paper_2502_14317_b200 as pc
from tests import cache_ref as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["int8", "e4m3", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,w", [(1, 1), (1, 6), (160, 1), (80, 6), (1, 40)])
@pytest.mark.parametrize("n,at", [(2, 1), (200, 9), (200, 120)])
def test_large_values_without_weight(fmt, d, B, w, n, at):
    """Entries of value zero have all the weight: the answer is zero, however large the value of an entry whose weight is none (its logit is 400 below)."""
    Hq, Hkv = 4, 2
    q, k, v = torch.zeros(B, w, Hq, d), torch.zeros(B, n, Hkv, d), torch.zeros(B, n, Hkv, d)
    q[..., 0], k[..., 0] = 20.0, 10.0
    k[:, at, :, 0] = -10.0
    v[:, at] = 2.0 ** 40
    own = {"format": "bf16", "k": k.transpose(1, 2).to(torch.bfloat16).cuda().contiguous(), "v": v.transpose(1, 2).to(torch.bfloat16).cuda().contiguous()}
    if fmt != "bf16":
        own = pc.kv_cache(B, Hkv, n, d, fmt)
        pc.kv_quantize(own, k.to(torch.bfloat16).cuda(), v.to(torch.bfloat16).cuda())
    got = pc.cache_attn(q.to(torch.bfloat16).cuda(), own=own, softmax_scale=1.0, want_lse=True)
    assert not ref.f64(got["out"]).any()
    # a logit of 200 and log(n - 1); the lowest entry adds e^-400
    assert np.abs(got["lse"].cpu().numpy() - (200.0 + np.log(n - 1.0))).max() <= 1e-4 + 200 * 2.0 ** -22
