"""Every build of cache_attn's kernels against 64 bits, and new tokens whose keys go through the matrix units: broadcast ones, and ones that are no number.
Which builds the calls reach is looked at in test_cache_builds.py."""
import numpy as np
import pytest
import torch

import paper_2502_14317_b200 as pc
from tests import cache_ref as ref
from tests.cache_builds import CALLS, FORMATS
from tests.test_gpu_cache import _cache, _check, _normal, _run, _values

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("call", CALLS, ids=str)
def test_every_build(call, fmt):
    """NaN behind every length and behind the last entry; lengths from zero on."""
    c = call
    _run(c.B, c.w, c.Hq, c.Hkv, c.d, c.n_prefix, fmt if c.n_prefix else "", c.n_own, fmt if c.n_own else "", ragged=c.ragged, window=c.window)


@pytest.mark.parametrize("w", [3, 24, 25, 40])
@pytest.mark.parametrize("same", ["heads", "sequences", "tokens"])
def test_new_tokens_through_strides_of_zero(w, same):
    """Keys and values that are the same for all heads, sequences or tokens, against 64 bits.  From 25 tokens on copies of them are a phase of their own; with a
    stride of 0, which TMA has not, each row takes them one by one."""
    B, Hq, Hkv, d, n = 4, 4, 2, 64, 200
    q = _normal(160, B, w, Hq, d)
    shape = {"heads": (B, w, 1, d), "sequences": (1, w, Hkv, d), "tokens": (B, 1, Hkv, d)}[same]
    kw, vw = (_normal(161 + i, *shape).expand(B, w, Hkv, d) for i in range(2))
    prefix = _cache(163, 1, Hkv, n, 5, d, "int8")
    on = lambda x: _device(x, shape, (B, w, Hkv, d))                                  # noqa: E731
    clean = tuple(np.nan_to_num(x) for x in _values(prefix))
    want, want_lse = ref.attention(ref.f64(q), None, 0, 0, clean, n, None, [0] * B, ref.f64(kw), ref.f64(vw))
    for k, v in ((on(kw), on(vw)), (on(kw).contiguous(), on(vw).contiguous())):
        got = pc.cache_attn(q.cuda(), k, v, prefix=prefix, n_prefix=n, want_lse=True)
        assert got["status"].item() == 0
        _check(ref.f64(got["out"]), want, same, got["lse"].cpu().numpy().astype(np.float64), want_lse)


def _device(x, shape, full):
    """a tensor of the host that was expanded from `shape`, on the GPU with the same strides of 0"""
    one = x[tuple(slice(0, n) for n in shape)].contiguous().cuda()
    return one.expand(*full)


@pytest.mark.parametrize("B,w,Hq,Hkv,d", [(5, 30, 8, 4, 128), (2, 37, 24, 8, 64), (1, 64, 64, 8, 64), (2, 64, 64, 8, 128), (20, 12, 4, 2, 64)])
@pytest.mark.parametrize("t", [0, 7, -1])
@pytest.mark.parametrize("key,value", [(None, NAN), (None, INF), (NAN, None), (INF, None), (-INF, -INF)])
def test_a_new_token_that_is_no_number(B, w, Hq, Hkv, d, t, key, value):
    """Token t of the last sequence: the rows before it, of other kv-heads and of other sequences are those of 64 bits, its own and later ones of its kv-head have
    what the definition has: no number in the value's column, or in all of them where it is the key."""
    t, b, h, G, n = t % w, B - 1, Hkv - 1, Hq // Hkv, 40
    q, kw, vw = _normal(150, B, w, Hq, d), _normal(151, B, w, Hkv, d), _normal(152, B, w, Hkv, d)
    prefix = _cache(153, 1, Hkv, n, 3, d, "bf16" if d == 64 else "e4m3")
    clean = tuple(np.nan_to_num(x) for x in _values(prefix))
    want, want_lse = ref.attention(ref.f64(q), None, 0, 0, clean, n, None, [0] * B, ref.f64(kw), ref.f64(vw))
    if value is not None:
        vw[b, t, h, 5] = value
    if key is not None:
        kw[b, t, h, 9] = key
    got = pc.cache_attn(q.cuda(), kw.cuda(), vw.cuda(), prefix=prefix, n_prefix=n, want_lse=True)
    assert got["status"].item() == 0
    out, lse = ref.f64(got["out"]), got["lse"].cpu().numpy().astype(np.float64)
    seen = np.zeros((B, w, Hq), bool)
    seen[b, t:, h * G:] = True
    hidden = ~seen.transpose(0, 2, 1)
    _check(out[~seen], want[~seen], "rows that do not see it", lse[hidden], want_lse[hidden])
    hit = out[seen]
    if key is None:
        assert np.isnan(hit[:, 5]).all() if np.isnan(value) else (hit[:, 5] == value).all()
        rest = np.delete(np.arange(d), 5)
        _check(hit[:, rest], want[seen][:, rest], "other columns", lse[~hidden], want_lse[~hidden])
    elif np.isnan(key):
        assert np.isnan(hit).all() and np.isnan(lse[~hidden]).all()
    else:                                                        # a logit of +inf: no number; of -inf: weight 0, and 0 times what is finite is nothing
        up = ref.f64(q)[seen][:, 9] * key > 0
        assert np.isnan(hit[up]).all()
