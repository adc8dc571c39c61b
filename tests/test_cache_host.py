"""CPU-only checks of the 8-bit caches and the attention over shared and own caches: the plain forms that the GPU tests use against
their definitions, the C boundary's and the binding's refusals, and the workspace's size."""
import ctypes
from ctypes import POINTER, Structure, byref, c_float, c_int32, c_int64, c_size_t, c_void_p

import numpy as np
import pytest
import torch

from tests import cache_ref as ref

INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -3                  # PC_ERR_... of include/pc.h


class Cache(Structure):
    _fields_ = [("format", c_int32), ("B", c_int32), ("Hkv", c_int32), ("d", c_int32), ("capacity", c_int64), ("k", c_void_p), ("v", c_void_p),
                ("k_scale", c_void_p), ("v_scale", c_void_p)]


class Args(Structure):
    _fields_ = [(n, c_int32) for n in ("B", "w", "Hq", "Hkv", "d", "n_prefix", "n_own", "q_pos0", "clear_status")] + \
               [("rope_theta", c_float), ("softmax_scale", c_float), ("q", c_void_p), ("q_stride", c_int64 * 3), ("k_win", c_void_p), ("v_win", c_void_p),
                ("k_win_stride", c_int64 * 3), ("v_win_stride", c_int64 * 3), ("q_pos", c_void_p), ("own_len", c_void_p),
                ("prefix", POINTER(Cache)), ("own", POINTER(Cache)), ("out", c_void_p), ("lse", c_void_p), ("status_word", c_void_p),
                ("workspace", c_void_p), ("workspace_bytes", c_size_t)]


AT = 1 << 20                                                     # an address that nothing reads: every call here is refused before a launch


def cache(format=1, B=1, Hkv=2, d=64, capacity=100, **kw):
    c = Cache(format, B, Hkv, d, capacity, AT, AT, AT, AT)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def args(prefix=None, own=None, **kw):
    a = Args(B=2, w=1, Hq=4, Hkv=2, d=64, n_prefix=100 if prefix else 0, n_own=100 if own else 0, q=AT, k_win=AT, v_win=AT, out=AT,
             workspace=AT, workspace_bytes=1 << 40)
    if prefix:
        a.prefix = ctypes.pointer(prefix)
    if own:
        a.own = ctypes.pointer(own)
    for k, v in kw.items():
        setattr(a, k, (c_int64 * 3)(*v) if k.endswith("stride") else v)
    return a


@pytest.fixture(scope="module")
def lib():
    from paper_2502_14317_b200 import binding, build
    build.build_library()
    lib = ctypes.CDLL(binding.lib_path())
    lib.pc_cache_attn_workspace_bytes.restype = c_size_t
    lib.pc_cache_attn_workspace_bytes.argtypes = [POINTER(Args)]
    lib.pc_cache_attn.argtypes = [POINTER(Args), c_void_p]
    lib.pc_kv_quantize.argtypes = [POINTER(Cache), c_void_p, c_void_p, c_void_p, c_void_p, c_int32, c_int32, c_void_p, c_void_p, c_void_p]
    lib.pc_gather_kv_quantize.argtypes = [c_void_p, c_void_p, POINTER(c_int64), c_void_p, c_void_p, c_int32, c_int32, POINTER(Cache), c_void_p, c_void_p]
    lib.pc_kv_dequantize.argtypes = [POINTER(Cache), c_int32, c_int32, c_void_p, c_void_p, c_void_p, c_void_p]
    return lib


BAD_CACHES = [(dict(format=3), INVALID), (dict(format=-1), INVALID), (dict(B=0), INVALID), (dict(Hkv=0), INVALID), (dict(capacity=0), INVALID),
              (dict(d=96), UNSUPPORTED), (dict(capacity=2 ** 28 + 1), UNSUPPORTED), (dict(k=None), INVALID), (dict(v=AT + 8), INVALID),
              (dict(k_scale=None), INVALID), (dict(v_scale=AT + 2), INVALID)]


@pytest.mark.parametrize("change,code", BAD_CACHES)
def test_caches_that_are_refused(lib, change, code):
    bad = cache(**change)
    assert lib.pc_kv_quantize(byref(bad), AT, None, AT, None, 1, 0, None, None, None) == code
    assert lib.pc_kv_dequantize(byref(bad), 1, 0, None, AT, AT, None) == code
    assert lib.pc_gather_kv_quantize(AT, AT, (c_int64 * 3)(64, 64, 64), AT, AT, 1, 1, byref(bad), None, None) == code
    assert lib.pc_cache_attn(byref(args(prefix=bad, n_prefix=1)), None) == code
    assert lib.pc_cache_attn_workspace_bytes(byref(args(prefix=bad, n_prefix=1))) == 0


def test_writes_and_reads_that_are_refused(lib):
    c, bf16 = cache(), cache(format=0)
    stride = lambda *s: (c_int64 * 3)(*s)                                                                      # noqa: E731
    for call in (lambda: lib.pc_kv_quantize(byref(c), None, None, AT, None, 1, 0, None, None, None),           # no source
                 lambda: lib.pc_kv_quantize(byref(c), AT + 2, None, AT, None, 1, 0, None, None, None),         # alignment
                 lambda: lib.pc_kv_quantize(byref(c), AT, stride(64, 4, 64), AT, None, 1, 0, None, None, None),
                 lambda: lib.pc_kv_quantize(byref(c), AT, None, AT, stride(-64, 64, 64), 1, 0, None, None, None),
                 lambda: lib.pc_kv_quantize(byref(c), AT, None, AT, None, 0, 0, None, None, None),             # no tokens
                 lambda: lib.pc_kv_quantize(byref(c), AT, None, AT, None, 1, 100, None, None, None),           # behind the capacity
                 lambda: lib.pc_kv_quantize(byref(c), AT, None, AT, None, 2 ** 31 - 1, 2 ** 31 - 1, None, None, None),
                 lambda: lib.pc_kv_quantize(byref(c), AT, None, AT, None, 1, -1, None, None, None),
                 lambda: lib.pc_kv_quantize(None, AT, None, AT, None, 1, 0, None, None, None),
                 lambda: lib.pc_gather_kv_quantize(AT, AT, None, AT, AT, 1, 1, byref(c), None, None),
                 lambda: lib.pc_gather_kv_quantize(AT, AT, stride(64, 64, 64), AT, AT, 2, 51, byref(c), None, None),      # more than the capacity
                 lambda: lib.pc_gather_kv_quantize(AT, AT, stride(64, 64, 64), AT, AT, 65536, 65536, byref(c), None, None),
                 lambda: lib.pc_gather_kv_quantize(AT, AT, stride(64, 64, 64), AT, AT, 1, 1, byref(cache(B=2)), None, None),
                 lambda: lib.pc_kv_dequantize(byref(c), 0, 0, None, AT, AT, None),
                 lambda: lib.pc_kv_dequantize(byref(c), 1, 0, None, None, AT, None)):
        assert call() == INVALID
    assert lib.pc_kv_quantize(byref(bf16), AT, None, AT, None, 1, 0, None, None, None) == UNSUPPORTED
    assert lib.pc_kv_dequantize(byref(bf16), 1, 0, None, AT, AT, None) == UNSUPPORTED


BAD_CALLS = [(dict(B=0), INVALID), (dict(w=0), INVALID), (dict(w=129), UNSUPPORTED), (dict(Hq=3), INVALID), (dict(d=96), UNSUPPORTED),
             (dict(n_prefix=-1), INVALID), (dict(n_prefix=101), INVALID), (dict(B=2 ** 23), UNSUPPORTED), (dict(q=None), INVALID), (dict(q=AT + 2), INVALID),
             (dict(out=None), INVALID), (dict(k_win=None), INVALID), (dict(v_win=AT + 8), INVALID), (dict(q_pos0=-1), INVALID), (dict(rope_theta=-1.0), INVALID),
             (dict(rope_theta=float("nan")), INVALID), (dict(softmax_scale=-1.0), INVALID), (dict(softmax_scale=float("nan")), INVALID),
             (dict(q_stride=(256, 3, 64)), INVALID), (dict(k_win_stride=(-8, 8, 8)), INVALID), (dict(workspace=None), WORKSPACE),
             (dict(workspace=AT + 16), INVALID), (dict(workspace_bytes=100), WORKSPACE)]


@pytest.mark.parametrize("change,code", BAD_CALLS)
def test_attention_calls_that_are_refused(lib, change, code):
    assert lib.pc_cache_attn(byref(args(prefix=cache(), **change)), None) == code


def test_attention_over_caches_that_do_not_go_with_the_call(lib):
    for a in (args(prefix=cache(B=2)), args(own=cache(B=1)), args(prefix=cache(Hkv=4)), args(own=cache(B=2, d=128)), args(own=cache(B=2), n_own=101),
              args(n_prefix=1), args(n_own=1), args(k_win=None, v_win=None)):
        assert lib.pc_cache_attn(byref(a), None) == INVALID
    assert lib.pc_cache_attn(None, None) == INVALID and lib.pc_cache_attn_workspace_bytes(None) == 0


@pytest.mark.skipif(torch.cuda.is_available(), reason="would launch")
def test_a_call_in_order_asks_for_the_gpu(lib):
    assert lib.pc_cache_attn(byref(args(prefix=cache(), own=cache(B=2))), None) == UNSUPPORTED
    assert lib.pc_kv_quantize(byref(cache()), AT, None, AT, None, 1, 0, None, None, None) == UNSUPPORTED


def test_workspace_holds_rows_and_slots(lib):
    size = lambda **kw: lib.pc_cache_attn_workspace_bytes(byref(args(**kw)))                                   # noqa: E731
    rows = 2 * 2 * 2 * 64 * 2                                     # rows x kv-heads x d in bf16
    assert size() >= rows
    assert size(own=cache(B=2)) >= rows                           # finished in the kernel: no slots
    both = size(prefix=cache(), own=cache(B=2))
    assert both >= rows + 2 * 2 * 2 * (64 + 2) * 4                # a slot for the prefix at least
    wide = size(prefix=cache(capacity=100000), n_prefix=100000, B=64)
    assert wide >= 2 * (64 * 2 * 2 * 64 * 2) + 64 * 2 * 2 * (64 + 2) * 4          # over codes: the rows as halves as well
    assert 0 < wide < 1 << 30


def test_binding_refuses_tensors_of_the_host():
    import paper_2502_14317_b200 as pc
    c = pc.kv_cache(2, 2, 16, 64, "int8", device="cpu")
    assert c["k"].shape == c["v"].shape == (2, 2, 16, 64) and c["k"].dtype is torch.int8 and c["k_scale"].shape == (2, 2, 16)
    assert pc.kv_cache(1, 1, 1, 64, "bf16", device="cpu")["k_scale"] is None
    assert pc.kv_cache(1, 1, 1, 64, "e4m3", device="cpu")["k"].dtype is torch.float8_e4m3fn
    x = torch.zeros(2, 1, 2, 64, dtype=torch.bfloat16)
    for call in (lambda: pc.kv_cache(1, 1, 1, 64, "fp4", device="cpu"), lambda: pc.kv_quantize(c, x, x), lambda: pc.kv_dequantize(c),
                 lambda: pc.cache_attn(x, x, x, own=c), lambda: pc.gather_kv_quantize(x, x, torch.zeros(1, dtype=torch.int32), torch.zeros(1, 2, 1, dtype=torch.int32))):
        with pytest.raises((pc.PcError, RuntimeError)):
            call()


# ---------------------------------------------------------------- the plain forms of the GPU tests
def test_rows_at_the_formats_edges():
    for fmt, top in ref.TOP.items():
        x = np.zeros((6, 64))
        x[0, 3] = -2.0                                           # one value: the code is the top one, whatever the scale
        x[1] = 2.0 ** -101                                       # too small to have a scale
        x[2, 5] = np.inf
        x[3, 9] = np.nan
        x[4, :2] = 1.0, 0.5
        code, scale = ref.quantise(x, fmt)
        assert code[0, 3] == -top and scale[0] == np.float32(2.0) / np.float32(top) and np.count_nonzero(code[0]) == 1
        assert not code[1].any() and scale[1] == 0 and not code[2].any() and np.isnan(scale[2]) and np.isnan(scale[3])
        assert code[4, 0] == top and code[4, 1] == {"int8": 64.0, "e4m3": 224.0}[fmt]        # 63.5 goes to the even one
        assert not code[5].any() and scale[5] == 0


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_codes_are_the_nearest(fmt):
    x = ref.f64((torch.randn(200, 64, generator=torch.Generator().manual_seed(3)) * 3).to(torch.bfloat16))
    code, scale = ref.quantise(x, fmt)
    a = np.abs(x).max(-1, keepdims=True)
    if fmt == "int8":
        assert np.array_equal(code, np.rint(code)) and np.abs(code).max() == 127
        assert (np.abs(code * scale[:, None].astype(np.float64) - x) <= a / 127 * 0.5 * (1 + 2.0 ** -14)).all()
    else:
        assert np.array_equal(code, ref.f64(torch.from_numpy(code).to(torch.float32).to(torch.float8_e4m3fn)))          # values of the format
        bound = np.maximum(np.abs(x) * 2.0 ** -4, a / 448 * 2.0 ** -10)              # half a step: 3 bits behind the point, 2^-9 the smallest
        assert (np.abs(code * scale[:, None].astype(np.float64) - x) <= bound * (1 + 2.0 ** -14)).all()


def test_rounding_to_bf16_is_torchs():
    x = torch.randn(4000, generator=torch.Generator().manual_seed(5)) * torch.logspace(-30, 30, 4000)
    assert np.array_equal(ref.to_bf16(x.double().numpy()).astype(np.float32), x.to(torch.bfloat16).float().numpy())
    half = 1 + 2.0 ** -8                                         # between two values: to the even one, unless a little is left over
    assert ref.to_bf16(half) == 1 and ref.to_bf16(half + 2.0 ** -40) == 1 + 2.0 ** -7


def test_attention_is_one_softmax_over_all_three():
    g = torch.Generator().manual_seed(7)
    q, k, v = (torch.randn(2, 3, h, 8, generator=g, dtype=torch.float64) for h in (4, 2, 2))
    pk, pv = (torch.randn(1, 2, 5, 8, generator=g, dtype=torch.float64) for _ in range(2))
    ok, ov = (torch.randn(2, 2, 4, 8, generator=g, dtype=torch.float64) for _ in range(2))
    lens = [4, 2]
    out, lse = ref.attention(q.numpy(), None, 0, 0, (pk.numpy(), pv.numpy()), 5, (ok.numpy(), ov.numpy()), lens, k.numpy(), v.numpy())
    keys = torch.cat([pk.expand(2, -1, -1, -1), ok, k.transpose(1, 2)], 2).repeat_interleave(2, 1)
    values = torch.cat([pv.expand(2, -1, -1, -1), ov, v.transpose(1, 2)], 2).repeat_interleave(2, 1)
    seen = torch.ones(2, 1, 3, 12, dtype=torch.bool)
    seen[1, :, :, 7:9] = False
    seen[..., 9:] &= torch.ones(3, 3, dtype=torch.bool).tril()
    s = (torch.einsum("bihd,bhnd->bhin", q, keys) * 8 ** -0.5).masked_fill(~seen, -torch.inf)
    assert np.abs(out - torch.einsum("bhin,bhnd->bihd", s.softmax(-1), values).numpy()).max() < 1e-12
    assert np.abs(lse - s.logsumexp(-1).numpy()).max() < 1e-12
    nothing, minus = ref.attention(q.numpy(), None, 0, 0, None, 0, (ok.numpy(), ov.numpy()), [4, 0], None, None)
    assert not nothing[1].any() and np.isneginf(minus[1]).all() and nothing[0].any()
