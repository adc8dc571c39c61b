"""Bounded waits of pc_cache_attn's kernels: one that runs out is reported with its code, the call returns, and the next is right."""
import pytest
import torch

import paper_2502_14317_b200 as pc

pytestmark = pytest.mark.gpu


def _normal(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).cuda()


def _cache(seed, B, Hkv, n, d, fmt):
    k, v = _normal(seed, B, n, Hkv, d), _normal(seed + 1, B, n, Hkv, d)
    if fmt == "bf16":
        return {"format": "bf16", "k": k.transpose(1, 2).contiguous(), "v": v.transpose(1, 2).contiguous()}
    cache = pc.kv_cache(B, Hkv, n, d, fmt)
    pc.kv_quantize(cache, k, v)
    return cache


FEW = 412                                                           # few rows: the producer's wait for a stage
WIDE, PAIR = 101, 201                                               # many rows: the wait for a work item, single CTAs and pairs


@pytest.mark.parametrize("fmt", ["int8", "e4m3", "bf16"])
@pytest.mark.parametrize("own,B,w,Hq,Hkv,d,n,code", [
    (True, 1, 1, 8, 2, 128, 9000, FEW),                             # splits left as slots, or a cluster's
    (False, 1, 4, 8, 2, 64, 100, FEW),                              # a split, 16 rows
    (True, 4, 1, 4, 2, 64, 3000, FEW),
    (True, 160, 1, 2, 2, 128, 70, FEW),                             # short builds
    (False, 1, 30, 2, 1, 128, 40, WIDE),                            # and the new tokens as a phase for few rows: the first code stays
    (False, 64, 1, 4, 2, 128, 3000, WIDE),
    (False, 100, 1, 4, 2, 128, 3000, PAIR),
    (False, 100, 1, 4, 2, 64, 3000, WIDE),
    (False, 1, 20, 16, 2, 128, 700, PAIR),
])
def test_a_wait_that_runs_out_is_reported_with_its_code(fmt, own, B, w, Hq, Hkv, d, n, code):
    """The kernels wait for one signal that nobody gives, when nothing is in flight any more: 2e6 cycles, about a millisecond."""
    lib = pc.load_library()
    q, win = _normal(1, B, w, Hq, d), _normal(2, B, w, Hkv, d)
    cache = _cache(3, B if own else 1, Hkv, n, d, fmt)

    def run():
        r = pc.cache_attn(q, win, win, rope_theta=1e4, want_lse=True, **{"own" if own else "prefix": cache})
        return r["status"].item(), r["out"].clone(), r["lse"].clone()

    clean = run()
    assert clean[0] == 0
    assert lib.pc_debug_bounded_wait_test(2_000_000, 1) == 0
    try:
        hit = run()
    finally:
        assert lib.pc_debug_bounded_wait_test(0, 0) == 0
    assert hit[0] == code
    again = run()
    assert again[0] == 0
    for r in (hit, again):                                          # all work was done before the missing signal
        assert torch.equal(r[1], clean[1]) and torch.equal(r[2], clean[2])
