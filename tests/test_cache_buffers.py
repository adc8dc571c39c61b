"""CPU-only: what cache_attn keeps in ``buffers`` from call to call, on host memory, with entry points that do nothing."""
import ctypes

import pytest
import torch

ALL = -2 ** 63


@pytest.fixture(scope="module")
def attn():
    from paper_2502_14317_b200 import binding, build
    build.build_library()
    size = ctypes.CFUNCTYPE(ctypes.c_size_t, ctypes.c_void_p)(lambda a: 4096)
    run = ctypes.CFUNCTYPE(ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p)(lambda a, s: 0)
    module = binding._host_module()

    def call(B, w, buffers, given=(None,) * 4, want_lse=True, Hq=4, Hkv=2, d=64):
        q, k, v = (torch.zeros(B, w, n, d, dtype=torch.bfloat16) for n in (Hq, Hkv, Hkv))
        rc, got = module.cache_attn(ctypes.cast(size, ctypes.c_void_p).value, ctypes.cast(run, ctypes.c_void_p).value, 0, False, q, k, v, None, None, None, None,
                                    given, buffers, ALL, ALL, 0, want_lse, 0.0, 0.0)
        assert rc == 0 and got["out"].shape == (B, w, Hq, d) and got["out"].is_contiguous()
        assert (got["lse"].shape == (B, Hq, w)) if want_lse else True
        return got

    return call


def test_a_smaller_call_leaves_the_larger_ones_buffers(attn):
    """Batches that shrink and grow again: the same memory every time (a captured CUDA graph goes on using it)."""
    keep = {}
    first = attn(8, 2, keep)
    places = {n: first[n].data_ptr() for n in first}
    for B, w in ((3, 2), (8, 2), (1, 1), (16, 1), (8, 2)):
        got = attn(B, w, keep)
        assert {n: got[n].data_ptr() for n in got} == places, (B, w)
    assert keep["out"].numel() == first["out"].numel() and keep["lse"].numel() == first["lse"].numel()
    assert attn(8, 2, keep)["out"] is first["out"]


def test_a_larger_call_replaces_what_is_too_small_once(attn):
    keep = {}
    small = attn(2, 1, keep)
    large = attn(9, 3, keep)
    assert large["out"].data_ptr() != small["out"].data_ptr() and keep["out"] is large["out"] and keep["lse"] is large["lse"]
    assert large["status"] is small["status"] and large["workspace"] is small["workspace"]
    assert attn(2, 1, keep)["out"].data_ptr() == large["out"].data_ptr() and keep["out"] is large["out"]


def test_what_the_caller_gives_is_used_and_kept(attn):
    keep = {}
    attn(2, 1, keep)
    out = torch.zeros(2, 1, 4, 64, dtype=torch.bfloat16)
    got = attn(2, 1, keep, given=(out, None, None, None), want_lse=False)
    assert got["out"] is out and keep["out"] is out and got["lse"] is None and keep["lse"] is not None
    assert attn(2, 1, None)["out"] is not out
