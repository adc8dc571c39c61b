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


FEW = 411                                                           # few rows: a warp's wait for a copy
WIDE, PAIR = 101, 201                                               # many rows: the wait for a work item, single CTAs and pairs


@pytest.mark.parametrize("fmt", ["int8", "e4m3", "bf16"])
@pytest.mark.parametrize("cache,B,w,Hq,Hkv,d,n,code", [
    ("own", 1, 1, 8, 2, 128, 1500, FEW),                            # splits left as slots
    ("own", 4, 1, 8, 2, 64, 2000, FEW),                             # or joined by a cluster
    ("prefix", 1, 4, 8, 2, 64, 100, FEW),                           # 16 rows
    ("own", 160, 1, 2, 2, 128, 70, FEW),                            # short builds
    ("own", 160, 4, 8, 2, 128, 30, FEW),
    ("", 2, 60, 4, 2, 128, 0, FEW),                                 # new tokens alone, causal
    ("prefix", 40, 1, 2, 1, 128, 200, WIDE),                        # one work item each: the message that is missed is the last
    ("prefix", 90, 1, 2, 1, 64, 256, WIDE),
    ("prefix", 100, 1, 2, 1, 128, 256, PAIR),
    ("prefix", 1, 20, 8, 1, 128, 7, PAIR),
    ("own", 1, 60, 1, 1, 64, 130, WIDE),                            # and the new tokens behind it: the first code stays
])
def test_a_wait_that_runs_out_is_reported_with_its_code(fmt, cache, B, w, Hq, Hkv, d, n, code):
    """The kernels wait for one arrival that nobody makes, with nothing in flight: 2e6 cycles, about a millisecond."""
    lib = pc.load_library()
    q, win = _normal(1, B, w, Hq, d), _normal(2, B, w, Hkv, d)
    kept = {cache: _cache(3, B if cache == "own" else 1, Hkv, n, d, fmt)} if cache else {}

    def run():
        r = pc.cache_attn(q, win, win, rope_theta=1e4, want_lse=True, **kept)
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
    for r in (hit, again) if code != FEW and w == 1 else (again,):  # many rows: all work was done before the missing signal
        assert torch.equal(r[1], clean[1]) and torch.equal(r[2], clean[2])
