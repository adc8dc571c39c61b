"""CPU-only: the workspace of pc_cache_attn is sized by a call's sizes and the descriptors of its caches alone."""
import pytest
import torch

from ctypes import byref

from tests.test_cache_host import AT, UNSUPPORTED, WORKSPACE, args, cache, lib  # noqa: F401  (lib: a fixture)


@pytest.mark.skipif(torch.cuda.is_available(), reason="would launch")
@pytest.mark.parametrize("B,w,Hq,Hkv,d,n_prefix,n_own", [
    (2, 40, 2, 2, 64, 0, 100), (40, 32, 8, 8, 128, 0, 1000), (40, 16, 16, 8, 128, 0, 300), (1, 64, 8, 2, 64, 0, 300), (3, 25, 4, 1, 128, 500, 0),
    (1, 128, 32, 8, 128, 9000, 0), (64, 1, 32, 8, 128, 3000, 200), (16, 24, 8, 2, 64, 100, 2000), (16, 30, 8, 2, 64, 100, 2000), (5, 60, 4, 4, 128, 0, 0)])
@pytest.mark.parametrize("format", [0, 1, 2])
def test_what_a_call_comes_with_needs_no_more(lib, format, B, w, Hq, Hkv, d, n_prefix, n_own):  # noqa: F811
    """Sized before any pointer of the call is known: new tokens or none, contiguous or broadcast, lengths or none."""
    sizes = dict(B=B, w=w, Hq=Hq, Hkv=Hkv, d=d)
    kept = {}
    if n_prefix:
        kept["prefix"] = cache(format, 1, Hkv, d, n_prefix)
    if n_own:
        kept["own"] = cache(format, B, Hkv, d, n_own)
    early = args(**kept, **sizes, n_prefix=n_prefix, n_own=n_own, q=None, k_win=None, v_win=None, out=None, workspace=None, workspace_bytes=0)
    size = lib.pc_cache_attn_workspace_bytes(byref(early))
    assert size > 0
    row = w * Hkv * d
    for window in ({}, dict(k_win_stride=(row, 0, d), v_win_stride=(row, 0, d)), dict(k_win=None, v_win=None)):
        if not kept and "k_win" in window:
            continue                                              # nothing to attend to
        for own_len in (None, AT):
            call = args(**kept, **sizes, n_prefix=n_prefix, n_own=n_own, own_len=own_len, workspace_bytes=size, **window)
            assert lib.pc_cache_attn_workspace_bytes(byref(call)) == size
            assert lib.pc_cache_attn(byref(call), None) != WORKSPACE, (window, own_len)
            call.workspace_bytes = 100
            assert lib.pc_cache_attn(byref(call), None) == WORKSPACE


def test_limits_that_the_header_names(lib):  # noqa: F811
    for bad in (dict(Hq=2 ** 18 + 2, B=1), dict(B=2 ** 22 + 1, Hq=4)):
        a = args(prefix=cache(), **bad)
        assert lib.pc_cache_attn_workspace_bytes(byref(a)) == 0 and lib.pc_cache_attn(byref(a), None) == UNSUPPORTED
