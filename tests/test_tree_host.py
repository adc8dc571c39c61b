"""CPU-only checks of the paged caches, the attention of drafted tokens and the log probabilities: the plain forms that the GPU tests use, the C boundary's and the
binding's refusals, workspace sizes, and the kernels that are launched."""
import ctypes
import os
import re
import subprocess
from ctypes import POINTER, Structure, byref, c_float, c_int32, c_int64, c_size_t, c_void_p

import numpy as np
import pytest
import torch

from tests import tree_ref as tree
from tests.test_cache_builds import ROOT, _objects
from tests.test_cache_host import AT, INVALID, UNSUPPORTED, WORKSPACE, Cache, cache
from tests.tree_builds import CALLS, FORMATS

INT64 = lambda *s: (c_int64 * 3)(*s)                              # noqa: E731


class Append(Structure):
    _fields_ = [(n, c_int32) for n in ("B", "n", "n_src", "at0", "pos0", "n_table")] + \
               [("rope_theta", c_float), ("pages", POINTER(Cache)), ("table", c_void_p), ("table_stride", c_int64), ("k", c_void_p), ("v", c_void_p),
                ("k_stride", c_int64 * 3), ("v_stride", c_int64 * 3), ("at", c_void_p), ("pos", c_void_p), ("count", c_void_p), ("pick", c_void_p),
                ("parents", c_void_p), ("pick_stride", c_int64), ("parents_stride", c_int64), ("status_word", c_void_p)]


class Tree(Structure):
    _fields_ = [(n, c_int32) for n in ("B", "w", "Hq", "n_table", "max_len", "pos0", "clear_status")] + \
               [("rope_theta", c_float), ("softmax_scale", c_float), ("q", c_void_p), ("q_stride", c_int64 * 3), ("pages", POINTER(Cache)), ("table", c_void_p),
                ("table_stride", c_int64), ("lens", c_void_p), ("pos", c_void_p), ("parents", c_void_p), ("parents_stride", c_int64), ("out", c_void_p),
                ("lse", c_void_p), ("status_word", c_void_p), ("workspace", c_void_p), ("workspace_bytes", c_size_t)]


class LogProbs(Structure):
    _fields_ = [(n, c_int32) for n in ("type", "N", "V", "top", "group")] + \
               [("scale", c_float), ("stride", c_int64)] + [(n, c_void_p) for n in ("logits", "tokens", "logprob", "entropy", "top_logprob", "top_id", "nll")]


def _set(a, kw):
    for k, v in kw.items():
        setattr(a, k, ctypes.pointer(v) if isinstance(v, Cache) else v)
    return a


def append(**kw):
    return _set(Append(B=2, n=4, at0=0, n_table=3, pages=ctypes.pointer(cache(B=6, capacity=16)), table=AT, table_stride=3, k=AT, v=AT), kw)


def attn(**kw):
    return _set(Tree(B=2, w=4, Hq=4, n_table=3, max_len=40, q=AT, pages=ctypes.pointer(cache(B=6, capacity=16)), table=AT, table_stride=3, lens=AT, out=AT,
                     workspace=AT, workspace_bytes=1 << 40), kw)


def logprobs(**kw):
    return _set(LogProbs(type=1, N=4, V=100, scale=1.0, stride=100, logits=AT, tokens=AT, logprob=AT), kw)


def _typed(lib):
    lib.pc_tree_attn_workspace_bytes.restype = c_size_t
    lib.pc_tree_attn_workspace_bytes.argtypes = [POINTER(Tree)]
    lib.pc_tree_attn.argtypes = [POINTER(Tree), c_void_p]
    lib.pc_page_append.argtypes = [POINTER(Append), c_void_p]
    lib.pc_token_logprobs.argtypes = [POINTER(LogProbs), c_void_p]
    return lib


@pytest.fixture(scope="module")
def lib():
    from paper_2502_14317_b200 import binding, build
    build.build_library()
    return _typed(ctypes.CDLL(binding.lib_path()))


BAD_POOLS = [(dict(pages=cache(format=3)), INVALID), (dict(pages=cache(B=0)), INVALID), (dict(pages=cache(k=None)), INVALID), (dict(pages=cache(v=AT + 8)), INVALID),
             (dict(pages=cache(k_scale=None)), INVALID), (dict(pages=cache(d=96)), UNSUPPORTED), (dict(pages=cache(B=6, capacity=24)), UNSUPPORTED),
             (dict(pages=cache(B=6, capacity=2 ** 28)), UNSUPPORTED), (dict(table=None), INVALID), (dict(table=AT + 2), INVALID), (dict(table_stride=-1), INVALID),
             (dict(n_table=0), INVALID)]


@pytest.mark.parametrize("change,code", BAD_POOLS)
def test_pools_that_are_refused(lib, change, code):
    assert lib.pc_page_append(byref(append(**change)), None) == code
    assert lib.pc_tree_attn(byref(attn(**change)), None) == code


@pytest.mark.parametrize("change,code", [
    (dict(B=0), INVALID), (dict(n=0), INVALID), (dict(n=-1), INVALID), (dict(k=None), INVALID), (dict(v=AT + 2), INVALID), (dict(rope_theta=-1.0), INVALID),
    (dict(rope_theta=float("nan")), INVALID), (dict(rope_theta=float("inf")), INVALID), (dict(at0=-1), INVALID), (dict(at0=45), INVALID),
    (dict(at0=2 ** 31 - 1), INVALID), (dict(pick=AT), INVALID), (dict(pick=AT, n_src=4, parents=AT), INVALID), (dict(pick=AT, n_src=4, pick_stride=-1), INVALID),
    (dict(parents=AT, parents_stride=-4), INVALID), (dict(parents=AT, n=65, at=AT), UNSUPPORTED), (dict(n=2 ** 28 + 1, at=AT), UNSUPPORTED),
    (dict(B=2 ** 24 + 1), UNSUPPORTED), (dict(k_stride=INT64(64, 4, 64)), INVALID), (dict(v_stride=INT64(-8, 64, 64)), INVALID)])
def test_appends_that_are_refused(lib, change, code):
    assert lib.pc_page_append(byref(append(**change)), None) == code
    assert lib.pc_page_append(None, None) == INVALID


@pytest.mark.parametrize("change,code", [
    (dict(B=0), INVALID), (dict(w=0), INVALID), (dict(w=65), UNSUPPORTED), (dict(Hq=3), INVALID), (dict(Hq=0), INVALID), (dict(max_len=-1), INVALID),
    (dict(max_len=45), INVALID), (dict(max_len=2 ** 28 + 1), UNSUPPORTED), (dict(B=2 ** 22), UNSUPPORTED), (dict(q=None), INVALID), (dict(q=AT + 2), INVALID),
    (dict(out=None), INVALID), (dict(out=AT + 8), INVALID), (dict(lens=None), INVALID), (dict(parents_stride=-1), INVALID), (dict(rope_theta=-1.0), INVALID),
    (dict(rope_theta=float("inf")), INVALID), (dict(softmax_scale=-1.0), INVALID), (dict(softmax_scale=float("nan")), INVALID),
    (dict(q_stride=INT64(256, 3, 64)), INVALID), (dict(workspace=None), WORKSPACE), (dict(workspace=AT + 16), INVALID), (dict(workspace_bytes=100), WORKSPACE)])
def test_attention_calls_that_are_refused(lib, change, code):
    assert lib.pc_tree_attn(byref(attn(**change)), None) == code
    assert lib.pc_tree_attn(None, None) == INVALID and lib.pc_tree_attn_workspace_bytes(None) == 0


@pytest.mark.parametrize("change,code", [
    (dict(type=3), INVALID), (dict(type=-1), INVALID), (dict(N=0), INVALID), (dict(V=0), INVALID), (dict(top=-1), INVALID), (dict(top=101), INVALID),
    (dict(top=33, top_id=AT, top_logprob=AT), UNSUPPORTED), (dict(top=3), INVALID), (dict(top=3, top_id=AT), INVALID), (dict(logits=None), INVALID),
    (dict(logits=AT + 1), INVALID), (dict(type=0, logits=AT + 2), INVALID), (dict(stride=-1), INVALID), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID),
    (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID), (dict(tokens=None), INVALID), (dict(logprob=None), INVALID),
    (dict(tokens=None, logprob=None), INVALID), (dict(nll=AT), INVALID), (dict(nll=AT, group=3), INVALID), (dict(group=-1), INVALID),
    (dict(V=2 ** 28 + 1), UNSUPPORTED), (dict(N=2 ** 27 + 1), UNSUPPORTED)])
def test_log_probabilities_that_are_refused(lib, change, code):
    assert lib.pc_token_logprobs(byref(logprobs(**change)), None) == code
    assert lib.pc_token_logprobs(None, None) == INVALID


@pytest.mark.parametrize("scale", [2.0 ** -101, 1e-38, 2.0 ** 100 * 1.001, 3e38])
def test_temperatures_that_are_refused(lib, scale):
    assert lib.pc_token_logprobs(byref(logprobs(scale=scale)), None) == INVALID


def test_more_heads_than_a_launch_has(lib):
    pool = cache(B=1, capacity=16)
    pool.Hkv = 2 ** 18 - 3
    assert lib.pc_page_append(byref(append(pages=pool, n_table=1)), None) == UNSUPPORTED


@pytest.mark.skipif(torch.cuda.is_available(), reason="would launch")
def test_a_call_in_order_asks_for_the_gpu(lib):
    assert lib.pc_page_append(byref(append()), None) == UNSUPPORTED
    assert lib.pc_tree_attn(byref(attn()), None) == UNSUPPORTED
    assert lib.pc_token_logprobs(byref(logprobs()), None) == UNSUPPORTED
    assert lib.pc_page_append(byref(append(pages=cache(B=6, capacity=7), n_table=1)), None) == UNSUPPORTED       # (of one page any number of entries)


def test_workspace_goes_by_sizes_alone(lib):
    size = lambda **kw: lib.pc_tree_attn_workspace_bytes(byref(attn(**kw)))                                    # noqa: E731
    rows = 2 * 4 * 2 * 2 * 64 * 2                                 # sequences, tokens, heads of a kv-head, kv-heads, d in bf16
    assert size() >= rows + 2 * 4 * 8
    assert size(table=None, lens=None, q=None, out=None, workspace=None, n_table=0, parents=AT) == size()
    long = cache(B=6, capacity=1 << 20)
    assert size(pages=long, max_len=100000, B=1, w=1) >= 2 * 2 * 64 * 2 + 2 * 2 * (64 + 2) * 4                  # results of more than one split
    assert size(pages=long, max_len=20000, w=64) >= 2 * (2 * 64 * 2 * 2 * 64 * 2)                               # over codes: the rows as halves as well
    assert size(w=65) == size(Hq=3) == size(max_len=-1) == 0


def test_binding_refuses_tensors_of_the_host():
    import paper_2502_14317_b200 as pc
    pages = pc.kv_cache(6, 2, 16, 64, "int8", device="cpu")
    x, one, table = torch.zeros(2, 1, 2, 64, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32), torch.zeros(2, 3, dtype=torch.int32)
    for call in (lambda: pc.page_append(pages, x, x, table, at=0), lambda: pc.tree_attn(x, pages, table, one), lambda: pc.token_logprobs(torch.zeros(2, 9), one)):
        with pytest.raises((pc.PcError, RuntimeError)):
            call()


# ---------------------------------------------------------------- the kernels of a call
@pytest.fixture(scope="module")
def names(tmp_path_factory):
    from paper_2502_14317_b200 import build
    tmp = tmp_path_factory.mktemp("names")
    out = str(tmp / "libpc_tree_names.so")
    subprocess.run([build._nvcc(), "-shared", "-cudart", "none", "-gencode", "arch=compute_100a,code=sm_100a", "-Xcompiler", "-fPIC", "-Xlinker", "-Bsymbolic",
                    "-Xlinker", "--no-undefined", os.path.join(ROOT, "tests", "fake_launches.cpp"), *_objects(tmp), "-o", out], check=True)
    lib = _typed(ctypes.CDLL(out))
    lib.fake_launched.restype = lib.fake_known.restype = ctypes.c_char_p
    return lib


def _short(name):
    few = re.search(r"tree_few_kernel.*3FewILi\d+ELi\dELi(\d)ELb(\d)E", name)
    if few:
        return ("short" if few.group(2) == "1" else "few") + str(8 * int(few.group(1)))
    return "wide" if "tree_wide_kernel" in name else "rows" if "tree_rows_kernel" in name else "merge" if "_merge_kernel" in name else name


def launched(lib, c, fmt):
    n_table = (c.n + c.w + c.page - 1) // c.page
    a = attn(B=c.B, w=c.w, Hq=c.Hq, n_table=n_table, max_len=c.n, pages=cache(FORMATS.index(fmt), c.B * n_table, c.Hkv, c.d, c.page), table_stride=n_table)
    a.workspace_bytes = lib.pc_tree_attn_workspace_bytes(byref(a))
    lib.fake_clear()
    assert lib.pc_tree_attn(byref(a), None) == 0
    return lib.fake_launched().decode().split("\n")[:-1]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("call", CALLS, ids=str)
def test_kernels_of_a_call(names, call, fmt):
    want = call.kernels["bf16" if fmt == "bf16" else "8 bits"] if isinstance(call.kernels, dict) else call.kernels
    assert [_short(n) for n in launched(names, call, fmt)] == want


def test_the_calls_reach_every_build(names):
    seen = {n for c in CALLS for fmt in FORMATS for n in launched(names, c, fmt)}
    every = {n for n in names.fake_known().decode().split("\n") if re.search("tree_(few|wide|rows|merge)_kernel", n)}
    assert len(every) == 36 and every == {n for n in seen if "tree_" in n}, sorted(every - seen)


# ---------------------------------------------------------------- the plain forms of the GPU tests
def test_who_sees_whom():
    assert tree.seen([-1, 0, 0, 1, -2, 4, 2, -1]) == [[0], [0, 1], [0, 2], [0, 1, 3], [], [], [0, 2, 6], [7]]
    assert tree.seen(tree.chain(3)) == [[0], [0, 1], [0, 1, 2]]


def test_attention_over_pages_is_one_softmax():
    g = torch.Generator().manual_seed(7)
    q = torch.randn(1, 3, 4, 8, generator=g, dtype=torch.float64)
    k, v = (torch.randn(4, 2, 4, 8, generator=g, dtype=torch.float64) for _ in range(2))
    table, n = [[2, 0, 3]], 6
    out, lse = tree.attention(q.numpy(), (k.numpy(), v.numpy()), table, [n], [[-1, 0, -1]], [n], 0)
    keys, values = (x[table[0]].transpose(0, 1).reshape(2, 12, 8)[:, :9].repeat_interleave(2, 0) for x in (k, v))
    hidden = torch.zeros(3, 9, dtype=torch.bool)
    hidden[0, 7:] = hidden[1, 8] = hidden[2, 6:8] = True
    s = (torch.einsum("ihd,hnd->hin", q[0], keys) * 8 ** -0.5).masked_fill(hidden, -torch.inf)
    assert np.abs(out[0] - torch.einsum("hin,hnd->ihd", s.softmax(-1), values).numpy()).max() < 1e-12
    assert np.abs(lse[0] - s.logsumexp(-1).numpy()).max() < 1e-12


def test_rotation_keeps_lengths_and_distances():
    g = np.random.default_rng(3)
    x, y = g.standard_normal((5, 2, 64)), g.standard_normal((5, 2, 64))
    a, b = tree.turned(x, np.arange(5) + 1000, 1e4), tree.turned(y, np.arange(5) + 1007, 1e4)
    c, d = tree.turned(x, np.arange(5), 1e4), tree.turned(y, np.arange(5) + 7, 1e4)
    assert np.abs((a ** 2).sum(-1) - (x ** 2).sum(-1)).max() < 1e-10 and np.abs((a * b).sum(-1) - (c * d).sum(-1)).max() < 1e-8
    assert np.array_equal(tree.turned(x, np.zeros(5), 1e4), x)


def test_log_probabilities_are_torchs():
    x = torch.randn(4, 50, generator=torch.Generator().manual_seed(5), dtype=torch.float64)
    x[1, 7] = x[1, 3] = 9.0
    x[2, 1:] = -torch.inf
    x[3] = -torch.inf
    got, entropy, ids, lp = tree.logprobs(x.numpy(), np.array([5, -1, 50, 2]), 3)
    want = torch.log_softmax(x, -1)
    assert abs(got[0] - want[0, 5]) < 1e-12 and got[1] == 0 and np.isnan(got[2]) and got[3] == -np.inf
    assert abs(entropy[0] + (want[0].exp() * want[0]).sum()) < 1e-12 and entropy[2] == entropy[3] == 0
    assert ids[1].tolist()[:2] == [3, 7] and ids[2].tolist() == [0, 1, 2] and ids[3].tolist() == [0, 1, 2]
    assert np.abs(lp[0] - want[0].topk(3).values.numpy()).max() < 1e-12 and lp[2, 0] == 0 and np.isneginf(lp[2, 1:]).all()
